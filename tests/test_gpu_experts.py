"""The operators on dispatched rows as an expert uses them, behind the bridge and together, and the calls they refuse (needs a B200)."""
import ctypes

import pytest
import torch

import emc2_gen as gen
from parity import to_dev
from row_cases import ascending_offsets, expert_of_rows, ffn_reference, handle, norm_reference, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def test_expert_behind_the_bridge_forward_and_backward():
    """Frames through the bridge; per expert: its voxel's learned row added to each dispatched row, norm, feed-forward; and the
    gradients back to the voxels' rows."""
    import paper_2507_04123_b200 as pkg
    w = gen.KITTI.with_shape(2, 6001)
    br = pkg.Bridge(pkg.config_from_workload(w))
    d = to_dev(gen.make_batch(w))
    bufs = br.run(d["points"], d["proj"], d["feat"])
    br.status()
    C, H, E, V = w.feat_c, 96, w.num_experts, 3000
    br.reserve_rows(C, H)
    rd, vox = bufs["rd"], bufs["vox"]["point_voxel"][0]
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    ids = torch.gather(vox, 1, rd["perm"].long()).clamp(max=V - 1).contiguous()          # in dispatched order; -1: no voxel
    table = rand(g, V, C)
    weight, bias = 1 + 0.1 * rand(g, E, C), 0.1 * rand(g, E, C)
    wg, wu, wd = rand(g, E, H, C, dtype=torch.bfloat16, scale=C ** -0.5), rand(g, E, H, C, dtype=torch.bfloat16, scale=C ** -0.5), rand(g, E, C, H, dtype=torch.bfloat16, scale=H ** -0.5)
    dy = rand(g, w.B, w.N, C, dtype=torch.bfloat16)

    x = rd["feat_out"] + br.row_lookup(ids, table, 0.5)
    n = br.expert_norm(x, rd["offsets"], weight, bias, out_dtype=torch.bfloat16)
    y = br.expert_ffn(n["y"], rd["offsets"], wg, wu, wd)
    f = br.expert_ffn_grad(n["y"], rd["offsets"], wg, wu, wd, dy)
    m = br.expert_norm_grad(x, rd["offsets"], weight, n["mean"], n["rstd"], f["grad_x"])
    t = br.row_lookup_grad(ids, m["grad_x"], V, 0.5)
    br.status()

    # Each operator against its formula on what the one before it left.
    e = expert_of_rows(rd["offsets"], w.N, E)
    assert (e < E).all() and len(torch.unique(e)) > 1                                     # the dispatch leaves no row over
    rows = torch.where((ids >= 0)[..., None], table[ids.long().clamp(min=0)], 0.0)
    assert torch.equal(x, rd["feat_out"] + 0.5 * rows)                                    # a half is exact
    ref = norm_reference(x, e, E, weight, bias, 1e-5)
    # bf16: half a step; 2^-17 covers the fp32 arithmetic of 64 channels before it (see test_gpu_rows).
    assert ((n["y"].double() - ref["y"]).abs() <= (unit(torch.bfloat16) + 2 ** -17) * ref["y"].abs() + 2 ** -17).all()
    for k in range(E):
        want = ffn_reference(n["y"][e == k], wg[k], wu[k], wd[k], "silu", dy[e == k])
        for got, name in ((y[e == k], "y"), (f["grad_x"][e == k], "grad_x"), (f["grad_gate"][k], "grad_gate"), (f["grad_up"][k], "grad_up"), (f["grad_down"][k], "grad_down")):
            value, bound = want[name]
            assert ((got.double() - value).abs() <= bound).all(), (k, name)
    h, r = ref["h"], n["rstd"].double()[..., None]
    gw = f["grad_x"].double() * weight.double()[e]
    dx = r * (gw - gw.mean(-1, keepdim=True) - h * (gw * h).mean(-1, keepdim=True))
    size = r * (gw.abs() + gw.abs().mean(-1, keepdim=True) + h.abs() * (gw * h).abs().mean(-1, keepdim=True))
    # 64 channels: 70 roundings of fp32 in the means, and the statistics' own, of at most 2^-17 together.
    assert ((m["grad_x"].double() - dx).abs() <= 2 ** -16 * size + 1e-6 * size.amax(-1, keepdim=True)).all()
    want = torch.zeros((V, C), dtype=torch.float64, device=DEV)
    mass = torch.zeros_like(want)
    keep = ids.reshape(-1) >= 0
    at = ids.reshape(-1)[keep].long()
    want.index_add_(0, at, 0.5 * m["grad_x"].double().reshape(-1, C)[keep])
    mass.index_add_(0, at, 0.5 * m["grad_x"].double().reshape(-1, C)[keep].abs())
    times = torch.bincount(at, minlength=V)[:, None]
    assert ((t.double() - want).abs() <= (times + 1) * 2.0 ** -24 * mass * 1.01).all()
    br.close()


@pytest.mark.parametrize("C,H,act", [(80, 128, "silu"), (24, 72, "gelu"), (200, 64, "silu")])
def test_ffn_gradients_against_differences(C, H, act):
    """The formula's slope along a random direction, by central differences in 64 bits, against the library's gradients."""
    B, N, E = 1, 150, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(C)
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    offsets = torch.tensor([[0, 70, 150]], dtype=torch.int32, device=DEV)
    dt = torch.float16
    at = {"grad_x": rand(g, B, N, C, dtype=dt), "grad_gate": rand(g, E, H, C, dtype=dt, scale=C ** -0.5), "grad_up": rand(g, E, H, C, dtype=dt, scale=C ** -0.5),
          "grad_down": rand(g, E, C, H, dtype=dt, scale=H ** -0.5)}
    dy = rand(g, B, N, C, dtype=dt)
    got = br.expert_ffn_grad(at["grad_x"], offsets, at["grad_gate"], at["grad_up"], at["grad_down"], dy, act)
    f = torch.nn.functional.silu if act == "silu" else torch.nn.functional.gelu

    def loss(v):
        s = 0.0
        for k, (lo, hi) in enumerate(((0, 70), (70, 150))):
            x = v["grad_x"][0, lo:hi]
            s = s + (((f(x @ v["grad_gate"][k].T) * (x @ v["grad_up"][k].T)) @ v["grad_down"][k].T) * dy[0, lo:hi].double()).sum()
        return float(s)

    base = {k: v.double() for k, v in at.items()}
    for name in at:
        way = torch.randn(at[name].shape, generator=g, device=DEV, dtype=torch.float64)
        step = 1e-4
        slope = (loss({**base, name: base[name] + step * way}) - loss({**base, name: base[name] - step * way})) / (2 * step)
        mine = float((got[name].double() * way).sum())
        # The gradients' errors are roundings to fp16 of themselves and of the hidden values, 2^-11 at most each, of random sign
        # over many terms: five deviations of their sum.  The curvature costs 1e-7 of the slope's scale.
        scale = float((got[name].double() * way).square().sum().sqrt())
        assert abs(slope - mine) <= 5 * 3 * 2.0 ** -11 * scale + 1e-5 * abs(slope), name
    br.close()


def test_ffn_captured_replayed_and_on_another_stream():
    B, N, C, H, E = 2, 900, 72, 200, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    offsets = ascending_offsets(B, N, E, seed=4)
    x, dy = rand(g, B, N, C, dtype=torch.bfloat16), rand(g, B, N, C, dtype=torch.bfloat16)
    ws = [rand(g, *s, dtype=torch.bfloat16, scale=0.1) for s in ((E, H, C), (E, H, C), (E, C, H))]

    def run(o):
        o["y"] = br.expert_ffn(x, offsets, *ws, "gelu", out=o.get("y"))
        o["grad"] = br.expert_ffn_grad(x, offsets, *ws, dy, "gelu", out=o.get("grad"))
        return o

    def flat(o):
        return [o["y"], *o["grad"].values()]

    bufs = run({})
    for t in flat(bufs):
        t.zero_()
    run(bufs)
    want = [t.clone() for t in flat(bufs)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in flat(bufs):
            t.zero_()
        run(bufs)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(flat(bufs), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(bufs)
    # Replayed on other rows, from the same buffers.
    fresh = handle(B, N, E)
    fresh.reserve_rows(C, H)
    for seed in (5, 6):
        g.manual_seed(seed)
        x.copy_(rand(g, B, N, C))
        dy.copy_(rand(g, B, N, C))
        offsets.copy_(ascending_offsets(B, N, E, seed=seed))
        for t in flat(bufs):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        direct = {"y": torch.zeros_like(x), "grad": {k: torch.zeros_like(v) for k, v in bufs["grad"].items()}}
        fresh.expert_ffn(x, offsets, *ws, "gelu", out=direct["y"])
        fresh.expert_ffn_grad(x, offsets, *ws, dy, "gelu", out=direct["grad"])
        assert all(torch.equal(a, b) for a, b in zip(flat(bufs), flat(direct)))
    br.status()
    del graph
    br.close()
    fresh.close()


def test_ffn_gradients_on_two_streams_of_the_handle():
    """Enough rows and channels that the weights' gradients run beside the rows': the same bits as one after the other, with
    the inputs overwritten right behind the call, and captured."""
    B, N, C, H, E = 2, 6000, 136, 64, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    offsets = ascending_offsets(B, N, E, seed=9)
    rows = rand(g, 2, B, N, C, dtype=torch.bfloat16)
    ws = [rand(g, *s, dtype=torch.bfloat16, scale=0.1) for s in ((E, H, C), (E, H, C), (E, C, H))]
    x, dy = rows.clone()
    br.set_overlap(False)
    out = {k: torch.zeros_like(v) for k, v in br.expert_ffn_grad(x, offsets, *ws, dy).items()}
    br.expert_ffn_grad(x, offsets, *ws, dy, out=out)
    want = {k: v.clone() for k, v in out.items()}
    br.set_overlap(True)
    for _ in range(20):
        x.copy_(rows[0])
        dy.copy_(rows[1])
        for v in out.values():
            v.zero_()
        br.expert_ffn_grad(x, offsets, *ws, dy, out=out)
        x.zero_()
        dy.zero_()
        assert all(torch.equal(out[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.copy_(rows[0])
        dy.copy_(rows[1])
        br.expert_ffn_grad(x, offsets, *ws, dy, out=out)
        x.zero_()
        dy.zero_()
    for _ in range(3):
        for v in out.values():
            v.zero_()
        graph.replay()
        assert all(torch.equal(out[k], want[k]) for k in want)
    br.status()
    del graph
    br.close()


def test_one_expert_without_offsets_and_empty_batches():
    br = handle(2, 64, 4)
    br.reserve_rows(32, 64)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    ws = [rand(g, *s, dtype=torch.bfloat16, scale=0.2) for s in ((1, 64, 32), (1, 64, 32), (1, 32, 64))]
    x = rand(g, 2, 50, 32, dtype=torch.bfloat16)
    y = br.expert_ffn(x, None, *ws)
    value, bound = ffn_reference(x.reshape(-1, 32), ws[0][0], ws[1][0], ws[2][0], "silu")["y"]
    assert ((y.reshape(-1, 32).double() - value).abs() <= bound).all()
    # No rows: gradients of the weights are zeros, whatever was there.
    none = torch.empty((2, 0, 32), dtype=torch.bfloat16, device=DEV)
    out = {"grad_x": none.clone(), **{k: torch.full_like(w, 3.0) for k, w in zip(("grad_gate", "grad_up", "grad_down"), ws)}}
    br.expert_ffn_grad(none, None, *ws, none, out=out)
    assert all((out[k] == 0).all() for k in ("grad_gate", "grad_up", "grad_down"))
    assert br.expert_ffn(none, None, *ws).shape == (2, 0, 32)
    offsets = torch.zeros((2, 5), dtype=torch.int32, device=DEV)                          # rows, but none of an expert's
    w4 = [w.expand(4, -1, -1).contiguous() for w in ws]
    y = torch.full_like(x, 7.0)
    br.expert_ffn(x, offsets, *w4, out=y)
    assert (y == 7).all()
    out = {"grad_x": y, **{k: torch.full_like(w, 3.0) for k, w in zip(("grad_gate", "grad_up", "grad_down"), w4)}}
    br.expert_ffn_grad(x, offsets, *w4, x, out=out)
    assert (y == 7).all() and all((out[k] == 0).all() for k in ("grad_gate", "grad_up", "grad_down"))
    f32 = torch.ones((2, 0, 32), device=DEV)
    grads = {"grad_x": f32, "grad_weight": torch.ones((4, 32), device=DEV), "grad_bias": torch.ones((4, 32), device=DEV)}
    br.expert_norm_grad(f32, offsets, torch.ones((4, 32), device=DEV), torch.empty((2, 0), device=DEV), torch.empty((2, 0), device=DEV), f32, out=grads)
    assert (grads["grad_weight"] == 0).all() and (grads["grad_bias"] == 0).all()
    ids = torch.empty((0,), dtype=torch.int32, device=DEV)
    table = torch.ones((7, 32), device=DEV)
    assert br.row_lookup(ids, table).shape == (0, 32)
    assert (br.row_lookup_grad(ids, torch.empty((0, 32), device=DEV), 7) == 0).all()
    br.status()
    br.close()


def test_an_infinite_row_stays_with_its_own_expert_and_row():
    """Infinities and NaN in one expert's rows reach that expert's weights and those rows, no other, also within a tile."""
    B, N, C, H, E = 1, 100, 64, 64, 2
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    offsets = torch.tensor([[0, 40, 100]], dtype=torch.int32, device=DEV)
    x, dy = rand(g, B, N, C, dtype=torch.bfloat16), rand(g, B, N, C, dtype=torch.bfloat16)
    ws = [rand(g, *s, dtype=torch.bfloat16, scale=0.1) for s in ((E, H, C), (E, H, C), (E, C, H))]
    y0, g0 = br.expert_ffn(x, offsets, *ws), br.expert_ffn_grad(x, offsets, *ws, dy)
    x[0, 50], dy[0, 60] = float("inf"), float("nan")
    y1, g1 = br.expert_ffn(x, offsets, *ws), br.expert_ffn_grad(x, offsets, *ws, dy)
    other = torch.tensor([i for i in range(N) if i != 50], device=DEV)
    assert torch.equal(y1[0, other], y0[0, other]) and not torch.isfinite(y1[0, 50]).any()
    other = torch.tensor([i for i in range(N) if i not in (50, 60)], device=DEV)
    assert torch.equal(g1["grad_x"][0, other], g0["grad_x"][0, other])
    for k in ("grad_gate", "grad_up", "grad_down"):
        assert torch.equal(g1[k][0], g0[k][0]) and not torch.isfinite(g1[k][1]).all()
    br.status()
    br.close()


# ------------------------------------------------------------------ refusals
def test_calls_that_are_refused():
    import paper_2507_04123_b200 as pkg
    INVALID, LARGE = pkg.bridge.EMC2_ERR_INVALID_ARG, pkg.bridge.EMC2_ERR_TOO_LARGE
    br = handle(2, 64, 4)
    lib, h = br.lib, br._h
    buf = torch.zeros((1 << 20,), dtype=torch.uint8, device=DEV)
    other = torch.zeros((1 << 20,), dtype=torch.uint8, device=DEV)
    p, q = buf.data_ptr(), other.data_ptr()
    # gradients before the scratch is there
    assert lib.emc2_row_lookup_grad(h, 4, 4, 8, 0, p, p, 1.0, q, None) == LARGE
    assert lib.emc2_expert_norm_grad(h, 1, 4, 8, 0, 0, p, None, p, p, p, p, q, q, q, None) == LARGE
    assert lib.emc2_expert_ffn_grad(h, 1, 4, 8, 8, 1, 0, p, None, p, p, p, p, q, q, q, q, None) == LARGE
    for bad in ((3, 0), (1028, 0), (64, -1), (64, 8193)):
        assert lib.emc2_rows_reserve(h, *bad) == INVALID
    assert lib.emc2_rows_reserve(h, 64, 32) == 0
    before = br.scratch_bytes
    assert lib.emc2_rows_reserve(h, 32, 16) == 0 and br.scratch_bytes == before            # within what there is
    assert lib.emc2_expert_ffn_grad(h, 1, 4, 72, 8, 1, 0, p, None, p, p, p, p, q, q, q, q, None) == LARGE
    assert lib.emc2_expert_ffn_grad(h, 1, 4, 64, 40, 1, 0, p, None, p, p, p, p, q, q, q, q, None) == LARGE
    # lookup: n, rows, channels, type, ids, table, out
    good = (4, 4, 8, 0, p, p, 1.0, q)
    assert lib.emc2_row_lookup(h, *good, None) == 0
    for i, v in ((0, -1), (0, 129), (1, -1), (2, 6), (2, 0), (2, 1028), (3, 3), (3, -1), (4, None), (4, p + 2), (5, None), (5, p + 8), (7, None), (7, q + 8), (7, p)):
        bad = list(good)
        bad[i] = v
        assert lib.emc2_row_lookup(h, *bad, None) == INVALID, (i, v)
        assert lib.emc2_row_lookup_grad(h, *bad, None) == INVALID, (i, v)
    assert lib.emc2_row_lookup(h, 4, 2**31 - 1, 1024, 0, p, p, 1.0, q, None) == INVALID    # more vectors than 32 bits count
    # norm: B, N, channels, type_x, type_y, x, offsets, weight, bias, eps, y, mean, rstd
    good = (1, 4, 8, 0, 1, p, None, p, None, 1e-5, q, None, None)
    assert lib.emc2_expert_norm(h, *good, None) == 0
    for i, v in ((0, 3), (0, -1), (1, 65), (1, -1), (2, 10), (2, 1028), (3, 3), (4, -1), (5, None), (5, p + 4), (6, p + 2), (7, None), (7, p + 4), (8, p + 4), (9, -1.0),
                 (9, float("nan")), (10, None), (10, p), (10, q + 8), (11, q + 2), (12, q + 1)):
        bad = list(good)
        bad[i] = v
        assert lib.emc2_expert_norm(h, *bad, None) == INVALID, (i, v)
    # B, N, channels, types, x, offsets, weight, mean, rstd, grad_y, grad_x, grad_weight, grad_bias
    good = (1, 4, 8, 0, 1, p, None, p, p, p, p, q, q, None)
    assert lib.emc2_expert_norm_grad(h, *good, None) == 0
    for i, v in ((0, 3), (2, 2), (3, 7), (5, None), (7, None), (8, None), (9, None), (10, None), (10, p + 8), (11, None), (11, p), (12, None), (8, p + 2), (9, p + 1), (12, q + 2),
                 (13, q + 2)):
        bad = list(good)
        bad[i] = v
        assert lib.emc2_expert_norm_grad(h, *bad, None) == INVALID, (i, v)
    # ffn: B, N, channels, hidden, type, act, x, offsets, gate, up, down, y
    good = (1, 4, 8, 8, 1, 0, p, None, p, p, p, q)
    assert lib.emc2_expert_ffn(h, *good, None) == 0
    for i, v in ((0, 3), (1, 65), (2, 12), (2, 264), (2, 0), (3, 12), (3, 8200), (3, 0), (4, 0), (4, 3), (5, 2), (5, -1), (6, None), (6, p + 8), (7, p + 1), (8, None), (9, p + 2), (10, None),
                 (11, None), (11, p), (11, q + 4)):
        bad = list(good)
        bad[i] = v
        assert lib.emc2_expert_ffn(h, *bad, None) == INVALID, (i, v)
    good = (1, 4, 8, 8, 1, 0, p, None, p, p, p, p, q, q, q, q)
    for i, v in ((0, 3), (2, 4), (4, 0), (11, None), (12, None), (12, p), (13, None), (14, q + 2), (15, None)):
        bad = list(good)
        bad[i] = v
        assert lib.emc2_expert_ffn_grad(h, *bad, None) == INVALID, (i, v)
    torch.cuda.synchronize()
    br.status()
    br.close()


def test_tensors_that_the_binding_refuses():
    br = handle(1, 16, 2)
    br.reserve_rows(32, 32)
    x = torch.zeros((1, 16, 32), dtype=torch.bfloat16, device=DEV)
    off = torch.zeros((1, 3), dtype=torch.int32, device=DEV)
    w, wd = torch.zeros((2, 32, 32), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 32, 32), dtype=torch.bfloat16, device=DEV)
    f = torch.zeros((2, 32), device=DEV)
    ids = torch.zeros((16,), dtype=torch.int32, device=DEV)
    for call in (lambda: br.expert_ffn(x.float(), off, w, w, wd), lambda: br.expert_ffn(x, off, w, w, wd, act="relu"), lambda: br.expert_ffn(x, off.long(), w, w, wd),
                 lambda: br.expert_ffn(x, off, w[:1], w, wd), lambda: br.expert_ffn(x, off, w, w.half(), wd), lambda: br.expert_ffn(x.transpose(1, 2), off, w, w, wd),
                 lambda: br.expert_ffn(x, None, w, w, wd), lambda: br.expert_ffn_grad(x, off, w, w, wd, x[:, :8]), lambda: br.expert_norm(x, off, f[:, :16]),
                 lambda: br.expert_norm(x.double(), off, f), lambda: br.expert_norm(x, off, f.bfloat16()), lambda: br.expert_norm(x.cpu(), off, f),
                 lambda: br.row_lookup(ids.long(), f), lambda: br.row_lookup(ids[::2], f), lambda: br.row_lookup(ids, f.double()),
                 lambda: br.row_lookup_grad(ids, f, 4), lambda: br.row_lookup(ids, f, out=torch.zeros((16, 32)))):
        with pytest.raises(ValueError):
            call()
    br.close()
