"""More learned row operators whose speed counts: what stands around the experts' feed-forward block, and the block for few rows.

  residual, residual_grad   the block's result normed, dropped out, gated, scaled and added to its rows, and the norm before the
                            next block, in one pass; and the gradients
  dropout                   dropout of rows from a counter-based generator whose mask is never stored; on the gradient of the
                            result, with the same seed, it is the gradient
  layer, layer_mx4          a whole mixture-of-experts layer for a few rows: router, choice, gated feed-forward of the chosen
                            experts, weighted sum; with weights of 16 bits, or of 4 bits with a power of two per 32 (MX)
  mx4                       quantisation of weights to that form

A case is a dict:
  op         one of the above
  B, N       frames, rows per frame; ``fill``: share of each frame's rows that the experts own (residual), or of the rows that
             are in use (layer; B is 1)
  C, H       row width, hidden width (layer)
  E, k       experts, chosen experts per row (layer)
  dtype      type of the rows; ``branch``: of the block's result and of the normed rows (residual)
  act        "silu" or "gelu" (layer)
  p          share of dropped elements (residual, dropout)
  gated      a gate per row (residual)

With ``own`` false the operators are computed in their plain form (elementary torch operations in 32 bits; the router's logits
and sums over many rows in 64; rounded once); with ``own`` true by the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}
EPS = 1e-5
BLOCK = 32                                   # elements that share a power of two (mx4)
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(op, B, N, C, H=0, E=4, k=0, dtype="bfloat16", branch="bfloat16", act="silu", p=0.0, gated=True, fill=1.0):
    return {"op": op, "B": B, "N": N, "C": C, "H": H, "E": E, "k": k, "dtype": dtype, "branch": branch, "act": act, "p": p,
            "gated": gated, "fill": fill}


def listed():
    named = {
        # A couple of thousand rows of one frame: all latency.
        "residual_small": _case("residual", 1, 2001, 64, dtype="float32", p=0.0),
        # The dispatched rows of the nuScenes-shaped batch in training: fp32 rows, bf16 blocks, a tenth dropped.
        "residual_nuscenes": _case("residual", 4, 300000, 80, dtype="float32", p=0.1),
        # Training on KITTI-shaped half batches.
        "residual_grad_kitti": _case("residual_grad", 8, 60000, 64, dtype="float32", p=0.1),
        # A ragged batch with wide bf16 rows and room behind the last expert's rows, without dropout or gates.
        "residual_grad_wide": _case("residual_grad", 3, 33333, 256, E=5, gated=False, fill=0.9),
        # Rows of odd width of one frame, in fp16: latency.
        "dropout_frame": _case("dropout", 1, 30001, 36, dtype="float16", p=0.25),
        # A nuScenes-shaped batch, or its gradient.
        "dropout_nuscenes": _case("dropout", 4, 300000, 80, p=0.1),
        # One query through the layer: latency, and the weights of two experts.
        "layer_one": _case("layer", 1, 1, 256, 1024, E=16, k=2),
        # The proposals of a frame, in fp16 with GELU, room for more behind them.
        "layer_proposals": _case("layer", 1, 64, 80, 320, E=8, k=2, dtype="float16", act="gelu", fill=0.7),
        # Many wide experts: the reading of all weights.
        "layer_wide": _case("layer", 1, 128, 1024, 4096, E=32, k=4),
        # The 4-bit form of such a layer's weights: a third of them.
        "mx4_weights": _case("mx4", 1, 131072, 1024, E=1),
        # One query with 4-bit weights.
        "layer_mx4_one": _case("layer_mx4", 1, 1, 256, 1024, E=16, k=2),
        # Many wide experts in 4 bits.
        "layer_mx4_wide": _case("layer_mx4", 1, 128, 1024, 4096, E=32, k=4),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["residual", "residual", "residual_grad", "residual_grad", "dropout", "layer", "layer", "layer_mx4", "mx4"])
    if op in ("layer", "layer_mx4"):
        E = rng.choice([2, 3, 4, 8, 16, 32, 64])
        k = rng.choice([i for i in (1, 2, 2, 4, 8) if i <= E])
        n = _log(rng, 1, 128)
        C, H = 8 * _log(rng, 2, 128), 8 * _log(rng, 4, 512)
        H = max(8, int(min(H, 1.34e8 / (E * C), 2.1e9 / (n * k * C))) // 8 * 8)
        return _case(op, 1, n, C, H, E, k, dtype=rng.choice(["bfloat16", "bfloat16", "float16"]), act=rng.choice(["silu", "silu", "gelu"]),
                     fill=rng.choice([1.0, 1.0, 0.8]))
    if op == "mx4":
        C = 4 * _log(rng, 2, 1024)
        rows = int(min(_log(rng, 64, 1_000_000), 1.3e8 / C))
        return _case(op, 1, rows, C, 0, 1, dtype=rng.choice(["float32", "bfloat16", "float16"]) if rows * C < 6.0e7 else "bfloat16")
    B = _log(rng, 1, 16)
    rows = _log(rng, 64, 1_200_000)
    C = 4 * _log(rng, 2, 256)
    rows = int(min(rows, 9.0e7 / C if op != "residual_grad" else 3.0e7 / C))
    dtype = rng.choice(["float32", "float32", "bfloat16", "float16"])
    p = rng.choice([0.0, 0.1, 0.1, 0.5])
    if op == "dropout":
        return _case(op, B, max(1, rows // B), C, 0, 1, dtype=dtype, p=rng.choice([0.1, 0.2, 0.5]))
    E = rng.choice([1, 2, 3, 4, 4, 4, 8, 16])
    return _case(op, B, max(1, rows // B), C, 0, E, dtype=dtype, branch="float16" if dtype == "float16" else "bfloat16", p=p,
                 gated=rng.choice([True, True, False]), fill=rng.choice([1.0, 1.0, 0.9, 0.5]))


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _offsets(case, g):
    """Ascending offsets per frame: uneven shares, in every third frame one expert without rows."""
    B, N, E = case["B"], case["N"], case["E"]
    share = torch.rand((B, E), generator=g, device=DEV) ** 2 + 0.02
    if E > 1:
        share[::3, E // 2] = 0.0
    used = int(N * case["fill"])
    ends = torch.round(torch.cumsum(share, 1) / share.sum(1, keepdim=True) * used)
    ends[:, -1] = used
    return torch.cat([torch.zeros((B, 1), device=DEV), ends], 1).to(torch.int32).contiguous()


def _handle(case):
    """The handle of a program whose batches are of this size; small grids, because no case voxelizes."""
    import types

    import paper_2507_04123_b200 as pkg
    grid = types.SimpleNamespace(min=(0.0, 0.0, 0.0), voxel=(1.0, 1.0, 1.0), dims=(64, 64, 1), max_points=0)
    few = case["op"] in ("layer", "layer_mx4", "mx4")
    cfg = pkg.make_config(device=torch.cuda.current_device(), max_batch=1 if few else case["B"], max_points=128 if few else case["N"],
                          point_floats=4, grids=(grid, grid), num_cameras=1, img_h=8, img_w=8, feat_h=8, feat_w=8, feat_c=4, feat_stride=1,
                          min_depth=0.1, thresholds=(), num_experts=1 if few else case["E"], lut=((0,), (0,)))
    br = pkg.Bridge(cfg)
    if case["op"] != "mx4":
        br.reserve_rows(case["C"], case["H"])
    return br


def _pack(w):
    """Weights [.., C] in the 4-bit form: codes [.., 16 ceil(C / 32)], two elements a byte, the first in the low half, and
    exponents [.., ceil(C / 32)] of the powers of two, with a bias of 127."""
    C = w.shape[-1]
    blocks = -(-C // BLOCK)
    w = torch.nn.functional.pad(w, (0, blocks * BLOCK - C)).reshape(*w.shape[:-1], blocks, BLOCK)
    e = torch.frexp(w.abs().amax(-1))[1] - 3
    v = torch.ldexp(w, -e[..., None])
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    code = torch.bucketize(v.abs(), edges).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)
    packed = code[..., 0::2] | (code[..., 1::2] << 4)
    return {"codes": packed.reshape(*w.shape[:-2], blocks * BLOCK // 2).contiguous(), "scales": (e + 127).to(torch.uint8).contiguous()}


def prepare(case, seed):
    g = _generator(seed)
    B, N, C, H, E = (case[k] for k in ("B", "N", "C", "H", "E"))
    dt, db = TYPES[case["dtype"]], TYPES[case["branch"]]
    s = {"case": case}
    if own:
        s["bridge"] = _handle(case)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    op = case["op"]
    # The seed of the run and the number of the call, as a training loop keeps them on the device.
    s["seed"] = torch.tensor([int(seed) * 2654435761 + 12345, int(seed) % 1000], dtype=torch.int64, device=DEV)
    if op == "dropout":
        s["x"] = normal(B, N, C, dtype=dt)
        s["out"] = torch.zeros((B, N, C), dtype=dt, device=DEV)
        return s
    if op == "mx4":
        # Rows of weights with sizes of their own, and a few large elements, as trained weights have.
        w = normal(N, C) * torch.exp(normal(N, 1)) * C ** -0.5
        s["x"] = torch.where(torch.rand((N, C), generator=g, device=DEV) < 0.002, w * 8.0, w).to(dt)
        blocks = -(-C // BLOCK)
        s["out"] = {"codes": torch.zeros((N, blocks * BLOCK // 2), dtype=torch.uint8, device=DEV),
                    "scales": torch.zeros((N, blocks), dtype=torch.uint8, device=DEV), "values": torch.zeros((N, C), dtype=dt, device=DEV)}
        return s
    if op in ("layer", "layer_mx4"):
        s["x"] = normal(N, C, dtype=dt)
        s["count"] = torch.tensor([max(1, int(N * case["fill"]))], dtype=torch.int32, device=DEV)
        s["w_router"] = normal(E, C, scale=2.0 * C ** -0.5)
        for name, shape in (("w_gate", (E, H, C)), ("w_up", (E, H, C)), ("w_down", (E, C, H))):
            w = normal(*shape, scale=shape[2] ** -0.5)
            s[name] = w.to(dt) if op == "layer" else _pack(w)
            del w
        s["out"] = {"y": torch.zeros((N, C), dtype=dt, device=DEV), "ids": torch.zeros((N, case["k"]), dtype=torch.int32, device=DEV),
                    "weights": torch.zeros((N, case["k"]), device=DEV)}
        return s
    s["offsets"] = _offsets(case, g)
    f = normal(B, N, C) * 1.5 + 0.25
    x = normal(B, N, C) * 2.0 + 0.5
    # The block gives zeros for rows of points that no camera sees.
    s["f"] = torch.where(torch.rand((B, N, 1), generator=g, device=DEV) < 0.1, torch.zeros_like(f), f).to(db).contiguous()
    s["params"] = {"post_weight": 1.0 + 0.1 * normal(E, C), "post_bias": 0.1 * normal(E, C), "scale": 0.5 + 0.1 * normal(E, C),
                   "pre_weight": 1.0 + 0.1 * normal(E, C)}
    pre_bias = 0.1 * normal(E, C)
    gate = torch.rand((B, N), generator=g, device=DEV) if case["gated"] else None
    s["gate"] = gate
    if op == "residual":
        s["x"] = x.to(dt).contiguous()
        s["params"]["pre_bias"] = pre_bias
        s["out"] = {"out": torch.zeros((B, N, C), dtype=dt, device=DEV), "y": torch.zeros((B, N, C), dtype=db, device=DEV),
                    "stats": torch.zeros((B, N, 4), device=DEV)}
        return s
    # What the forward call left: the new rows, and mean and 1 / deviation of the block's result and of the new rows.
    s["x"] = x.to(dt).contiguous()
    parts = []
    for t in (s["f"].float(), s["x"].float()):
        m = t.mean(-1, keepdim=True)
        parts += [m, torch.rsqrt((t - m).square().mean(-1, keepdim=True) + EPS)]
    s["stats"] = torch.cat(parts, -1).contiguous()
    s["grad_out"], s["grad_y"] = normal(B, N, C, dtype=dt), normal(B, N, C, dtype=db)
    s["out"] = {"grad_x": torch.zeros((B, N, C), dtype=dt, device=DEV), "grad_f": torch.zeros((B, N, C), dtype=db, device=DEV),
                "grad_gate": torch.zeros((B, N), device=DEV) if case["gated"] else None}
    for name in ("grad_post_weight", "grad_post_bias", "grad_scale", "grad_pre_weight", "grad_pre_bias"):
        s["out"][name] = torch.zeros((E, C), device=DEV)
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _given(d):
    return {k: v for k, v in d.items() if v is not None}


def _own(s):
    case, br, op = s["case"], s["bridge"], s["case"]["op"]
    if op == "dropout":
        return br.row_dropout(s["x"], case["p"], s["seed"], out=s["out"])
    if op == "mx4":
        return br.mx4_quantise(s["x"], out=s["out"])["values"]
    if op in ("layer", "layer_mx4"):
        return br.expert_layer(s["x"], s["w_router"], s["w_gate"], s["w_up"], s["w_down"], case["k"], case["act"], count=s["count"],
                               out=s["out"])
    if op == "residual":
        return br.expert_residual(s["x"], s["f"], s["offsets"], gate=s["gate"], **s["params"], eps=EPS, p=case["p"], seed=s["seed"],
                                  out=s["out"])
    return _given(br.expert_residual_grad(s["x"], s["f"], s["offsets"], s["stats"], s["grad_out"], s["grad_y"], gate=s["gate"], **s["params"],
                                          p=case["p"], seed=s["seed"], out=s["out"]))


# ------------------------------------------------------------------ plain forms

def _threshold(p):
    """An element is kept where its 16 random bits are at least this."""
    return int(math.floor(p * 65536.0 + 0.5))


def _kept(seed, rows, C, p):
    """[rows, C]: the factor of every element, 0 where dropped: Philox4x32 with 10 rounds, eight elements per number."""
    low = 0xFFFFFFFF
    groups = -(-C // 8)
    c0 = torch.arange(rows, device=DEV)[:, None].expand(rows, groups)
    c1 = torch.arange(groups, device=DEV)[None, :].expand(rows, groups)
    c2, c3 = seed[1] & low, (seed[1] >> 32) & low
    k0, k1 = seed[0] & low, (seed[0] >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57              # of 64 bits, whatever the sign says
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c0 >> 16, c1, c1 >> 16, c2, c2 >> 16, c3, c3 >> 16], -1) & 0xFFFF
    t = _threshold(p)
    factor = 65536.0 / (65536 - t)
    return torch.where(words.reshape(rows, groups * 8)[:, :C] >= t, factor, 0.0)


def _expert_of_rows(offsets, N):
    """Expert of every row, E for the rows behind the last segment: [B, N]."""
    j = torch.arange(N, device=offsets.device)
    return (j[None, :, None] >= offsets[:, None, 1:]).sum(-1)


def _expert_sums(v, e, E):
    """Sums of v [rows, C] over the rows of every expert, in 64 bits: [E, C].  Rows with e = E count nowhere."""
    of = (e.reshape(-1, 1) == torch.arange(E, device=e.device)).double()
    return (of.t() @ v.reshape(-1, v.shape[-1]).double()).float()


def _plain(s):
    case = s["case"]
    op, C = case["op"], case["C"]
    dt, db = TYPES[case["dtype"]], TYPES[case["branch"]]
    if op == "dropout":
        m = _kept(s["seed"], case["B"] * case["N"], C, case["p"]).reshape(s["x"].shape)
        return torch.where(m > 0, s["x"].float() * m, 0.0).to(dt)
    if op == "mx4":
        return _plain_mx4(s["x"])
    if op in ("layer", "layer_mx4"):
        return _plain_layer(s, case, dt)
    at = _expert_of_rows(s["offsets"], case["N"])
    inside = (at < case["E"])[..., None]
    e = at.clamp(max=case["E"] - 1)
    p = s["params"]
    gate = s["gate"][..., None] if s["gate"] is not None else 1.0
    m = _kept(s["seed"], case["B"] * case["N"], C, case["p"]).reshape(s["f"].shape) if case["p"] else 1.0
    f, x = s["f"].float(), s["x"].float()
    if op == "residual":
        mean = f.mean(-1, keepdim=True)
        d = f - mean
        rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)
        o = x + p["scale"][e] * gate * (m * (d * rstd * p["post_weight"][e] + p["post_bias"][e]))
        mean2 = o.mean(-1, keepdim=True)
        d = o - mean2
        rstd2 = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)
        y = d * rstd2 * p["pre_weight"][e] + p["pre_bias"][e]
        return {"out": (o * inside).to(dt), "y": (y * inside).to(db), "stats": torch.cat([mean, rstd, mean2, rstd2], -1) * inside}
    mean, rstd, mean2, rstd2 = s["stats"].split(1, -1)
    dy = s["grad_y"].float()
    h2 = (x - mean2) * rstd2
    g = dy * p["pre_weight"][e]
    do = s["grad_out"].float() + rstd2 * (g - g.mean(-1, keepdim=True) - h2 * (g * h2).mean(-1, keepdim=True))
    h = (f - mean) * rstd
    d = m * (h * p["post_weight"][e] + p["post_bias"][e])
    through = do * p["scale"][e] * gate * m
    g = through * p["post_weight"][e]
    df = rstd * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    out = {"grad_x": (do * inside).to(dt), "grad_f": (df * inside).to(db)}
    if s["gate"] is not None:
        out["grad_gate"] = ((do * p["scale"][e] * d).sum(-1, keepdim=True) * inside)[..., 0]
    E = case["E"]
    return {**out, "grad_post_weight": _expert_sums(through * h, at, E), "grad_post_bias": _expert_sums(through, at, E),
            "grad_scale": _expert_sums(do * gate * d, at, E), "grad_pre_weight": _expert_sums(dy * h2, at, E),
            "grad_pre_bias": _expert_sums(dy, at, E)}


def _plain_mx4(x):
    """The values that the 4-bit form of the rows stands for."""
    rows, C = x.shape
    pad = -C % BLOCK
    w = torch.nn.functional.pad(x.float(), (0, pad)).reshape(rows, -1, BLOCK)
    e = (torch.frexp(w.abs().amax(-1, keepdim=True))[1] - 3).clamp(min=-127)
    v = torch.ldexp(w, -e)
    step = torch.where(v.abs() < 2.0, 0.5, torch.where(v.abs() < 4.0, 1.0, 2.0))
    v = (torch.round(v / step) * step).clamp(-6.0, 6.0)          # halves to even
    return torch.ldexp(v, e).reshape(rows, -1)[:, :C].to(x.dtype)


def _weights(w, C):
    """Weights in 32 bits, from either form."""
    if not isinstance(w, dict):
        return w.float()
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=DEV)
    codes = w["codes"]
    v = table[torch.stack([codes & 15, codes >> 4], -1).int()].reshape(*w["scales"].shape, BLOCK)
    power = (w["scales"].int() << 23).view(torch.float32)
    return (v * power[..., None]).reshape(*codes.shape[:-1], -1)[..., :C]


def _act(g, act):
    return g / (1.0 + torch.exp(-g)) if act == "silu" else g * 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))


def _rows_of(w, slots):
    return {k: v[slots] for k, v in w.items()} if isinstance(w, dict) else w[slots]


def _plain_layer(s, case, dt):
    n, C, H, E, k = (case[i] for i in ("N", "C", "H", "E", "k"))
    inside = torch.arange(n, device=DEV)[:, None] < s["count"]
    x = s["x"].float()
    logits = s["x"].double() @ s["w_router"].double().t()
    top, ids = torch.sort(logits, dim=-1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    p = torch.exp(top - top[:, :1])
    p = (p / p.sum(-1, keepdim=True)).float()
    if n * k <= E:
        # Few rows: the weights of the chosen experts alone.
        wg, wu, wd = (_weights(_rows_of(s[i], ids.reshape(-1)), c) for i, c in (("w_gate", C), ("w_up", C), ("w_down", H)))
        xs = x.repeat_interleave(k, 0)[:, :, None]
        h = _act(wg @ xs, case["act"]) * (wu @ xs)
        y = ((wd @ h).reshape(n, k, C) * p[..., None]).sum(1)
    else:
        wg, wu, wd = (_weights(s[i], c) for i, c in (("w_gate", C), ("w_up", C), ("w_down", H)))
        share = torch.zeros((n, E), device=DEV).scatter_(1, ids, p)
        h = _act(x @ wg.transpose(1, 2), case["act"]) * (x @ wu.transpose(1, 2))
        y = ((h @ wd.transpose(1, 2)) * share.t()[..., None]).sum(0)
    return {"y": torch.where(inside, y, 0.0).to(dt), "ids": (ids * inside).int(), "weights": p * inside}


# ------------------------------------------------------------------ what one pass cannot do without

def work(case):
    B, N, C, H, E, k = (case[i] for i in ("B", "N", "C", "H", "E", "k"))
    rows, used = B * N, B * int(N * case["fill"])
    sx, sb = SIZES[case["dtype"]], SIZES[case["branch"]]
    op = case["op"]
    per_row = 4 if case["gated"] else 0
    if op == "dropout":
        return {"bytes": 2 * rows * C * sx, "flops": rows * C}
    if op == "mx4":
        return {"bytes": rows * (2 * C * sx + -(-C // BLOCK) * 17), "flops": 4 * rows * C}
    if op == "residual":
        return {"bytes": used * (C * (2 * sx + 2 * sb) + 16 + per_row) + 20 * E * C, "flops": 20 * used * C}
    if op == "residual_grad":
        return {"bytes": used * (C * (3 * sx + 3 * sb) + 16 + 2 * per_row) + 40 * E * C, "flops": 40 * used * C}
    n = max(1, used)
    asked = E * (1.0 - (1.0 - k / E) ** n)                       # experts that some row asks for, of rows that choose at random
    element = sx if op == "layer" else 0.5 + 1.0 / BLOCK
    return {"bytes": int(asked * 3 * H * C * element + 4 * E * C + n * (2 * C * sx + 8 * k)), "flops": n * (6 * k * C * H + 2 * E * C)}


# ------------------------------------------------------------------ definitions in 64 bits

def _exact_kept(seed, rows, C, p):
    """The factors of _kept from the generator's definition, on the host."""
    groups = -(-C // 8)
    u = np.uint64
    word = [np.repeat(np.arange(rows, dtype=u), groups), np.tile(np.arange(groups, dtype=u), rows)]
    number, key = int(seed[1]) % 2 ** 64, int(seed[0]) % 2 ** 64
    word += [np.full(rows * groups, number & 0xFFFFFFFF, dtype=u), np.full(rows * groups, number >> 32, dtype=u)]
    for r in range(10):
        ka = u((key + r * 0x9E3779B9) & 0xFFFFFFFF)
        kb = u(((key >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = word[0] * u(0xD2511F53), word[2] * u(0xCD9E8D57)
        word = [(b >> u(32)) ^ word[1] ^ ka, b & u(0xFFFFFFFF), (a >> u(32)) ^ word[3] ^ kb, a & u(0xFFFFFFFF)]
    bits = np.empty((rows * groups, 8), dtype=np.uint16)
    for i, w in enumerate(word):
        bits[:, 2 * i] = w & u(0xFFFF)
        bits[:, 2 * i + 1] = w >> u(16)
    t = _threshold(p)
    kept = torch.from_numpy((bits.reshape(rows, -1)[:, :C] >= t)).to(DEV)
    return kept.double() * (65536.0 / (65536 - t))


def exact(case, seed):
    s = prepare(case, seed)
    op, B, N, C, E = (case[i] for i in ("op", "B", "N", "C", "E"))
    if op == "mx4":
        return _exact_mx4(s["x"])
    if op in ("layer", "layer_mx4"):
        return _exact_layer(s, case)
    kept = None
    if case["p"]:
        kept = _exact_kept(s["seed"].tolist(), B * N, C, case["p"]).reshape(B, N, C)
    if op == "dropout":
        return s["x"].double() * kept
    like = s["x"]
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=like.device)      # noqa: E731
    names = ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias")
    out = {"out": zeros(B, N, C), "y": zeros(B, N, C), "stats": zeros(B, N, 4)}
    if op == "residual_grad":
        out = {"grad_x": zeros(B, N, C), "grad_f": zeros(B, N, C)}
        if case["gated"]:
            out["grad_gate"] = zeros(B, N)
        out.update({"grad_" + i: zeros(E, C) for i in names})
    for b, bounds in enumerate(s["offsets"].tolist()):
        for k in range(E):
            i = slice(bounds[k], bounds[k + 1])
            if bounds[k] == bounds[k + 1]:
                continue
            v = {name: t[k].double() for name, t in s["params"].items()}
            f, x = s["f"][b, i].double(), s["x"][b, i].double()
            drop = kept[b, i] if kept is not None else torch.ones_like(f)
            gate = s["gate"][b, i].double()[:, None] if case["gated"] else torch.ones_like(f[:, :1])
            if op == "residual":
                var, mean = torch.var_mean(f, -1, correction=0, keepdim=True)
                rstd = (var + EPS) ** -0.5
                o = x + ((f - mean) * rstd * v["post_weight"] + v["post_bias"]) * drop * gate * v["scale"]
                var2, mean2 = torch.var_mean(o, -1, correction=0, keepdim=True)
                rstd2 = (var2 + EPS) ** -0.5
                out["out"][b, i] = o
                out["y"][b, i] = (o - mean2) * rstd2 * v["pre_weight"] + v["pre_bias"]
                out["stats"][b, i] = torch.cat([mean, rstd, mean2, rstd2], -1)
                continue
            mean, rstd, mean2, rstd2 = s["stats"][b, i].double().split(1, -1)
            dy = s["grad_y"][b, i].double()
            h2, h = (x - mean2) * rstd2, (f - mean) * rstd
            do = s["grad_out"][b, i].double() + _norm_back(dy * v["pre_weight"], h2, rstd2)
            back = do * v["scale"] * gate * drop
            normed = h * v["post_weight"] + v["post_bias"]
            out["grad_x"][b, i] = do
            out["grad_f"][b, i] = _norm_back(back * v["post_weight"], h, rstd)
            if case["gated"]:
                out["grad_gate"][b, i] = (do * v["scale"] * drop * normed).sum(-1)
            out["grad_post_weight"][k] += (back * h).sum(0)
            out["grad_post_bias"][k] += back.sum(0)
            out["grad_scale"][k] += (do * gate * drop * normed).sum(0)
            out["grad_pre_weight"][k] += (dy * h2).sum(0)
            out["grad_pre_bias"][k] += dy.sum(0)
    return out


def _norm_back(g, h, rstd):
    return rstd * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))


def _exact_mx4(x):
    """Every element to the nearest of the values that its block has, halves to the even code."""
    rows, C = x.shape
    out = torch.empty((rows, C), dtype=torch.float64, device=x.device)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64, device=x.device)
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    chunk = max(1, 2 ** 24 // C)
    for r in range(0, rows, chunk):
        w = x[r:r + chunk].double()
        w = torch.cat([w, torch.zeros((w.shape[0], -C % BLOCK), dtype=torch.float64, device=x.device)], 1).reshape(w.shape[0], -1, BLOCK)
        top = w.abs().amax(-1, keepdim=True)
        power = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -130))))
        power = torch.where(power > top, power / 2, torch.where(power * 2 <= top, power * 2, power)) / 4
        power = power.clamp(min=2.0 ** -127)
        v = w.abs() / power
        low, high = torch.bucketize(v, edges), torch.bucketize(v, edges, right=True)     # differ at a half
        code = torch.where(low % 2 == 0, low, high)
        out[r:r + chunk] = (torch.sign(w) * grid[code] * power).reshape(w.shape[0], -1)[:, :C]
    return out


def _exact_layer(s, case):
    n, C, H, E, k = (case[i] for i in ("N", "C", "H", "E", "k"))
    used = int(s["count"])
    x = s["x"][:used].double()
    logits = torch.nn.functional.linear(x, s["w_router"].double())
    y = torch.zeros((n, C), dtype=torch.float64, device=DEV)
    ids = torch.zeros((n, k), dtype=torch.int32, device=DEV)
    weights = torch.zeros((n, k), dtype=torch.float64, device=DEV)
    left = logits.clone()
    for j in range(k):
        at = (left == left.amax(-1, keepdim=True)).int().argmax(-1)                      # the first of the largest
        ids[:used, j] = at.int()
        left.scatter_(1, at[:, None], -torch.inf)
    chosen = ids[:used].long()
    weights[:used] = torch.softmax(logits.gather(1, chosen), -1)
    act = torch.nn.functional.silu if case["act"] == "silu" else torch.nn.functional.gelu
    for e in range(E):
        row, j = (chosen == e).nonzero(as_tuple=True)
        if not len(row):
            continue
        wg, wu, wd = (_exact_weights(s[i], e, c) for i, c in (("w_gate", C), ("w_up", C), ("w_down", H)))
        part = x[row]
        y.index_add_(0, row, (act(part @ wg.T) * (part @ wu.T)) @ wd.T * weights[row, j][:, None])
    return {"y": y, "ids": ids, "weights": weights}


def _exact_weights(w, e, C):
    if not isinstance(w, dict):
        return w[e].double()
    codes, scales = w["codes"][e], w["scales"][e]
    both = torch.empty((codes.shape[0], codes.shape[1] * 2), dtype=torch.uint8, device=codes.device)
    both[:, 0::2], both[:, 1::2] = codes & 15, codes >> 4
    size = torch.tensor(E2M1, dtype=torch.float64, device=codes.device)[(both & 7).long()]
    power = torch.pow(2.0, scales.double() - 127.0).repeat_interleave(BLOCK, 1)
    return (torch.where(both >= 8, -size, size) * power)[:, :C]
