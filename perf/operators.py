"""The learned row operators whose speed counts: what the experts do with the rows that the dispatch leaves by expert.

The bridge ends with feature rows in contiguous segments per expert, ``[B, N, C]`` with ``offsets [B, E + 1]`` on the
device, and with the voxel row of every point (-1 where it has none).  Each case is one pass through one operator on them:

  lookup, lookup_grad   rows of a table by integer id, scaled (voxel rows back to their points, learned rows by ring or
                        class), and the table's gradient
  norm, norm_grad       layer norm with a weight and a bias per expert, and its gradients
  ffn, ffn_grad         gated feed-forward block with weights per expert, and its gradients

A case is a dict:
  op         one of the above
  B, N       frames, rows per frame; ``fill``: share of each frame's rows that the experts own (rows behind stay as they are)
  C, H       row width, hidden width (ffn)
  E          experts
  dtype      type of the rows (lookup, ffn); of the input rows (norm), whose output has ``dtype_out``
  V          table rows (lookup)
  act        "silu" or "gelu" (ffn)

With ``own`` false the operators are computed in their plain form (elementary torch operations in 32 bits, sums over many
rows in 64, rounded once); with ``own`` true by the library.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}
EPS = 1e-5


def _case(op, B, N, C, H=0, E=4, dtype="bfloat16", dtype_out="bfloat16", V=0, act="silu", fill=1.0):
    return {"op": op, "B": B, "N": N, "C": C, "H": H, "E": E, "dtype": dtype, "dtype_out": dtype_out, "V": V, "act": act,
            "fill": fill}


def listed():
    named = {
        # A small learned table (a row per laser ring) read for a thousand points: all latency.
        "lookup_rings": _case("lookup", 1, 1024, 64, dtype="float32", V=64),
        # Voxel rows back to the points of an aggregated nuScenes-shaped batch.
        "lookup_voxels": _case("lookup", 4, 300000, 80, V=600000),
        # The gradient of that: every voxel's row sums its points' rows.
        "lookup_grad_voxels": _case("lookup_grad", 4, 300000, 80, dtype="float32", V=600000),
        # The gradient of a tiny table read by a whole KITTI-shaped batch: long sums into few rows.
        "lookup_grad_hot": _case("lookup_grad", 8, 120000, 64, V=16),
        # A couple of thousand rows of one frame: all latency.
        "norm_small": _case("norm", 1, 2001, 64, dtype="float32"),
        # The dispatched rows of the nuScenes-shaped batch, fp32 in, bf16 out for the experts' products.
        "norm_nuscenes": _case("norm", 4, 300000, 80, dtype="float32"),
        # Training on KITTI-shaped batches.
        "norm_grad_kitti": _case("norm_grad", 8, 120000, 64, dtype="float32"),
        # A ragged batch with wide rows and room behind the last expert's rows.
        "norm_grad_wide": _case("norm_grad", 3, 33333, 256, E=5, fill=0.9),
        # The rows of a few proposals: latency of one small block.
        "ffn_few": _case("ffn", 1, 64, 64, 256),
        # Experts over the dispatched rows of the nuScenes-shaped batch.
        "ffn_nuscenes": _case("ffn", 4, 300000, 80, 320),
        # Training on KITTI-shaped half batches, in fp16 with GELU.
        "ffn_grad_kitti": _case("ffn_grad", 8, 60000, 64, 256, dtype="float16", act="gelu"),
        # Training wide experts on a ragged batch.
        "ffn_grad_wide": _case("ffn_grad", 3, 33333, 256, 1024, E=5, fill=0.95),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "norm", "norm_grad", "ffn", "ffn", "ffn_grad", "ffn_grad"])
    B = _log(rng, 1, 16)
    E = rng.choice([1, 2, 3, 4, 4, 4, 8, 16])
    fill = rng.choice([1.0, 1.0, 1.0, 0.9, 0.5])
    rows = _log(rng, 64, 1_200_000)
    if op in ("ffn", "ffn_grad"):
        C = 8 * _log(rng, 2, 32)
        H = 8 * _log(rng, 4, 128)
        most = 1.8e11 / (6.0 * C * H) if op == "ffn" else 4.0e11 / (16.0 * C * H)
        rows = int(min(rows, most, 3.8e8 / H))
        return _case(op, B, max(1, rows // B), C, H, E, dtype=rng.choice(["bfloat16", "bfloat16", "float16"]),
                     act=rng.choice(["silu", "silu", "gelu"]), fill=fill)
    C = 4 * _log(rng, 2, 128)
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    rows = int(min(rows, 9.6e7 / C))
    if op in ("norm", "norm_grad"):
        return _case(op, B, max(1, rows // B), C, 0, E, dtype=dtype,
                     dtype_out=rng.choice(["bfloat16", dtype]), fill=fill)
    V = int(min(_log(rng, 1, 600_000), 4.8e7 / C))
    return _case(op, B, max(1, rows // B), C, 0, E, dtype=dtype, V=max(1, V))


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
    cfg = pkg.make_config(device=torch.cuda.current_device(), max_batch=case["B"], max_points=case["N"], point_floats=4,
                          grids=(grid, grid), num_cameras=1, img_h=8, img_w=8, feat_h=8, feat_w=8, feat_c=4, feat_stride=1,
                          min_depth=0.1, thresholds=(), num_experts=case["E"], lut=((0,), (0,)))
    br = pkg.Bridge(cfg)
    br.reserve_rows(case["C"], case["H"])
    return br


def prepare(case, seed):
    g = _generator(seed)
    B, N, C, H, E = (case[k] for k in ("B", "N", "C", "H", "E"))
    dt, dto = TYPES[case["dtype"]], TYPES[case["dtype_out"]]
    s = {"case": case}
    if own:
        s["bridge"] = _handle(case)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)

    op = case["op"]
    if op in ("lookup", "lookup_grad"):
        V = case["V"]
        # Denser ids at the low end, as near voxels have more points; a tenth of the points has no row.
        u = torch.rand((B, N), generator=g, device=DEV)
        ids = (u * u * V).to(torch.int32).clamp_(max=V - 1)
        s["ids"] = torch.where(torch.rand((B, N), generator=g, device=DEV) < 0.1, -1, ids).to(torch.int32).contiguous()
        s["scale"] = math.sqrt(C)
        if op == "lookup":
            s["table"] = normal(V, C, dtype=dt)
            s["out"] = torch.zeros((B, N, C), dtype=dt, device=DEV)
        else:
            s["grad_out"] = normal(B, N, C, dtype=dt)
            s["out"] = torch.zeros((V, C), dtype=dt, device=DEV)
        return s
    s["offsets"] = _offsets(case, g)
    if op in ("norm", "norm_grad"):
        x = normal(B, N, C) * 2.0 + 0.5
        # Rows of points that no camera sees are zeros.
        x = torch.where(torch.rand((B, N, 1), generator=g, device=DEV) < 0.1, torch.zeros_like(x), x)
        s["x"] = x.to(dt).contiguous()
        s["weight"] = 1.0 + 0.1 * normal(E, C)
        s["bias"] = 0.1 * normal(E, C)
        if op == "norm":
            s["out"] = {"y": torch.zeros((B, N, C), dtype=dto, device=DEV),
                        "mean": torch.zeros((B, N), device=DEV), "rstd": torch.zeros((B, N), device=DEV)}
        else:
            xf = s["x"].float()
            s["mean"] = xf.mean(-1)
            s["rstd"] = torch.rsqrt((xf - s["mean"][..., None]).square().mean(-1) + EPS)
            s["grad_y"] = normal(B, N, C, dtype=dto)
            s["out"] = {"grad_x": torch.zeros((B, N, C), dtype=dt, device=DEV),
                        "grad_weight": torch.zeros((E, C), device=DEV), "grad_bias": torch.zeros((E, C), device=DEV)}
        return s
    s["x"] = normal(B, N, C, dtype=dt)
    s["w_gate"] = normal(E, H, C, dtype=dt, scale=C ** -0.5)
    s["w_up"] = normal(E, H, C, dtype=dt, scale=C ** -0.5)
    s["w_down"] = normal(E, C, H, dtype=dt, scale=H ** -0.5)
    if op == "ffn":
        s["out"] = torch.zeros((B, N, C), dtype=dt, device=DEV)
    else:
        s["grad_y"] = normal(B, N, C, dtype=dt)
        s["out"] = {"grad_x": torch.zeros((B, N, C), dtype=dt, device=DEV), "grad_gate": torch.zeros_like(s["w_gate"]),
                    "grad_up": torch.zeros_like(s["w_up"]), "grad_down": torch.zeros_like(s["w_down"])}
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    case, br, op = s["case"], s["bridge"], s["case"]["op"]
    if op == "lookup":
        return br.row_lookup(s["ids"], s["table"], s["scale"], out=s["out"])
    if op == "lookup_grad":
        return br.row_lookup_grad(s["ids"], s["grad_out"], case["V"], s["scale"], out=s["out"])
    if op == "norm":
        return br.expert_norm(s["x"], s["offsets"], s["weight"], s["bias"], EPS, out=s["out"])
    if op == "norm_grad":
        return br.expert_norm_grad(s["x"], s["offsets"], s["weight"], s["mean"], s["rstd"], s["grad_y"], out=s["out"])
    if op == "ffn":
        return br.expert_ffn(s["x"], s["offsets"], s["w_gate"], s["w_up"], s["w_down"], case["act"], out=s["out"])
    return br.expert_ffn_grad(s["x"], s["offsets"], s["w_gate"], s["w_up"], s["w_down"], s["grad_y"], case["act"], out=s["out"])


# ------------------------------------------------------------------ plain forms

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
    dt, dto = TYPES[case["dtype"]], TYPES[case["dtype_out"]]
    op = case["op"]
    if op == "lookup":
        ids = s["ids"].long()
        rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return (rows * (ids >= 0)[..., None]).to(dt)
    if op == "lookup_grad":
        ids = s["ids"].long().reshape(-1)
        keep = ids >= 0
        rows = s["grad_out"].reshape(-1, case["C"])
        out = torch.zeros((case["V"], case["C"]), dtype=torch.float64, device=ids.device)
        out.index_add_(0, ids[keep], rows[keep].double())
        return (out * s["scale"]).to(dt)
    if op in ("norm", "norm_grad"):
        at = _expert_of_rows(s["offsets"], case["N"])
        inside = (at < case["E"])[..., None]
        e = at.clamp(max=case["E"] - 1)
        x = s["x"].float()
        if op == "norm":
            mean = x.mean(-1, keepdim=True)
            d = x - mean
            rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)
            y = d * rstd * s["weight"][e] + s["bias"][e]
            return {"y": (y * inside).to(dto), "mean": (mean * inside)[..., 0], "rstd": (rstd * inside)[..., 0]}
        dy = s["grad_y"].float()
        rstd = s["rstd"][..., None]
        xh = (x - s["mean"][..., None]) * rstd
        gw = dy * s["weight"][e]
        dx = rstd * (gw - gw.mean(-1, keepdim=True) - xh * (gw * xh).mean(-1, keepdim=True))
        return {"grad_x": (dx * inside).to(dt), "grad_weight": _expert_sums(dy * xh, at, case["E"]),
                "grad_bias": _expert_sums(dy, at, case["E"])}
    return _plain_ffn(s, case, dt)


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_ffn(s, case, dt):
    C, E = case["C"], case["E"]
    e = _expert_of_rows(s["offsets"], case["N"]).reshape(-1)
    x = s["x"].reshape(-1, C)
    out = torch.zeros(x.shape, dtype=torch.float32, device=x.device)
    gate, up, down = [], [], []
    for k in range(E):
        rows = (e == k).nonzero()[:, 0]
        xk, wg, wu, wd = x[rows].float(), s["w_gate"][k].float(), s["w_up"][k].float(), s["w_down"][k].float()
        g, u = xk @ wg.t(), xk @ wu.t()
        a, da = _act(g, case["act"])
        if case["op"] == "ffn":
            out[rows] = (a * u) @ wd.t()
            continue
        dy = s["grad_y"].reshape(-1, C)[rows].float()
        dh = dy @ wd
        dg, du = dh * u * da, dh * a
        out[rows] = dg @ wg + du @ wu
        gate.append(dg.t() @ xk)
        up.append(du.t() @ xk)
        down.append(dy.t() @ (a * u))
    out = out.reshape(s["x"].shape).to(dt)
    if case["op"] == "ffn":
        return out
    return {"grad_x": out, "grad_gate": torch.stack(gate).to(dt), "grad_up": torch.stack(up).to(dt),
            "grad_down": torch.stack(down).to(dt)}


# ------------------------------------------------------------------ what one pass cannot do without

def work(case):
    B, N, C, H, E = (case[k] for k in ("B", "N", "C", "H", "E"))
    rows, used = B * N, B * int(N * case["fill"])
    si, so = SIZES[case["dtype"]], SIZES[case["dtype_out"]]
    op = case["op"]
    if op == "lookup":
        return {"bytes": rows * (4 + C * si) + min(case["V"], rows) * C * si, "flops": rows * C}
    if op == "lookup_grad":
        return {"bytes": rows * (4 + C * si) + case["V"] * C * si, "flops": rows * C}
    if op == "norm":
        return {"bytes": used * (C * (si + so) + 8) + 8 * E * C, "flops": 8 * used * C}
    if op == "norm_grad":
        return {"bytes": used * (C * (2 * si + so) + 8) + 12 * E * C, "flops": 14 * used * C}
    if op == "ffn":
        return {"bytes": 2 * used * C * si + 3 * E * H * C * si, "flops": 6 * used * C * H}
    return {"bytes": 3 * used * C * si + 6 * E * H * C * si, "flops": 16 * used * C * H}


# ------------------------------------------------------------------ definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op, E = case["op"], case["E"]
    if op == "lookup":
        t = torch.cat([s["table"].double() * s["scale"], torch.zeros((1, case["C"]), dtype=torch.float64, device=DEV)])
        return t[s["ids"].long()]                      # id -1: the row of zeros behind the table
    if op == "lookup_grad":
        t = torch.zeros((case["V"] + 1, case["C"]), dtype=torch.float64, device=DEV)
        at = s["ids"].long().reshape(-1) % (case["V"] + 1)
        order = torch.argsort(at)
        run = torch.cumsum(s["grad_out"].double().reshape(-1, case["C"])[order], 0)
        run = torch.cat([torch.zeros_like(run[:1]), run])
        ends = torch.searchsorted(at[order], torch.arange(case["V"] + 1, device=DEV), right=True)
        t = run[ends] - run[torch.cat([torch.zeros_like(ends[:1]), ends[:-1]])]
        return t[:-1] * s["scale"]
    x = s["x"].double()
    bounds = s["offsets"].tolist()
    if op == "norm":
        y, mean, rstd = torch.zeros_like(x), torch.zeros_like(x[..., 0]), torch.zeros_like(x[..., 0])
        for b, row in enumerate(bounds):
            for k in range(E):
                part = x[b, row[k]:row[k + 1]]
                var, mu = torch.var_mean(part, -1, correction=0)
                r = (var + EPS) ** -0.5
                y[b, row[k]:row[k + 1]] = (part - mu[:, None]) * r[:, None] * s["weight"][k].double() + s["bias"][k].double()
                mean[b, row[k]:row[k + 1]], rstd[b, row[k]:row[k + 1]] = mu, r
        return {"y": y, "mean": mean, "rstd": rstd}
    grad_x = torch.zeros_like(x)
    if op == "norm_grad":
        w = torch.zeros((E, case["C"]), dtype=torch.float64, device=DEV)
        bias = torch.zeros_like(w)
        for b, row in enumerate(bounds):
            for k in range(E):
                i = slice(row[k], row[k + 1])
                dy, r = s["grad_y"][b, i].double(), s["rstd"][b, i].double()[:, None]
                xh = (x[b, i] - s["mean"][b, i].double()[:, None]) * r
                w[k] += (dy * xh).sum(0)
                bias[k] += dy.sum(0)
                g = dy * s["weight"][k].double()
                grad_x[b, i] = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
        return {"grad_x": grad_x, "grad_weight": w, "grad_bias": bias}
    f = torch.nn.functional.silu if case["act"] == "silu" else torch.nn.functional.gelu
    ws = [s[n].double().requires_grad_(op == "ffn_grad") for n in ("w_gate", "w_up", "w_down")]
    y = torch.zeros_like(x)
    for b, row in enumerate(bounds):
        for k in range(E):
            i = slice(row[k], row[k + 1])
            part = x[b, i].clone().requires_grad_(op == "ffn_grad")
            out = torch.nn.functional.linear(f(part @ ws[0][k].T) * (part @ ws[1][k].T), ws[2][k])
            if op == "ffn":
                y[b, i] = out
            else:
                out.backward(s["grad_y"][b, i].double())
                grad_x[b, i] = part.grad
    if op == "ffn":
        return y
    return {"grad_x": grad_x, "grad_gate": ws[0].grad, "grad_up": ws[1].grad, "grad_down": ws[2].grad}
