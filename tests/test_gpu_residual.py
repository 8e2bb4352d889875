"""Dropout, and the residual operator with its gradients, against the formulas in 64 bits (needs a B200).

The bounds count roundings, see residual_cases.py: half a step each, C terms of a row's sums and n terms of the parameters'."""
import pytest
import torch

from residual_cases import PARAMS, factor, forward, gradients, kept, tiny
from row_cases import TYPES, ascending_offsets, expert_of_rows, handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def seeds(a, b):
    return torch.tensor([a, b], dtype=torch.int64, device=DEV)


def shifted(t, elements):
    """The same values in memory that begins `elements` behind the allocator's boundary."""
    room = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    at = room[elements:].view(t.shape)
    at.copy_(t)
    return at


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,C,p", [(1, 4, 0.5), (3, 36, 0.1), (1025, 64, 0.25), (4099, 80, 0.1), (77, 1024, 0.9), (500, 132, 1e-6), (9, 12, 1.0), (9, 12, 0.0)])
def test_dropout(n, C, p, dtype):
    g = generator(n)
    br = handle(1, max(n, 8))
    x = rand(g, n, C, dtype=dtype)
    x[0, 0], x[n - 1, C - 1] = float("nan"), float("inf")
    seed = seeds(-5 + 2 ** 40, 2 ** 33 + 1)
    want = kept(seed.tolist(), n, C, p).to(DEV)
    for v in (x, shifted(x, 16 // x.element_size())):
        out = br.row_dropout(v, p, seed)
        assert (out[~want] == 0).all()                                     # infinities and NaN among them
        k, rel = factor(p)
        ref = x.double()[want] * k
        fine = torch.isfinite(ref)
        tol = (rel * 2 + 2 * unit(dtype)) * ref.abs() + tiny(dtype)
        assert ((out.double()[want] - ref).abs() <= tol)[fine].all()
        assert torch.equal(torch.isnan(out.double()[want]), torch.isnan(ref)) and torch.equal(torch.isinf(out.double()[want]), torch.isinf(ref))
    br.status()
    br.close()


def test_dropout_of_shapes_and_of_the_gradient():
    """Leading sizes of any number; the call on the gradient drops the same elements."""
    g = generator(1)
    br = handle(3, 50)
    x, seed = rand(g, 3, 50, 20), seeds(11, 4)
    a = br.row_dropout(x, 0.3, seed)
    assert torch.equal(a.view(150, 20), br.row_dropout(x.view(150, 20), 0.3, seed))
    grad = br.row_dropout(torch.ones_like(x), 0.3, seed)
    assert torch.equal(grad == 0, a == 0) and torch.equal(a, x * grad)
    assert br.row_dropout(x[:, :0].contiguous(), 0.3, seed).shape == (3, 0, 20)
    br.close()


def test_a_captured_dropout_takes_new_seeds():
    br = handle(1, 300)
    x, seed, out = torch.ones((300, 64), device=DEV), seeds(1, 0), torch.empty((300, 64), device=DEV)
    br.row_dropout(x, 0.5, seed, out=out)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        br.row_dropout(x, 0.5, seed, out=out)
        seed[1] += 1
    for number in range(3):
        graph.replay()
        assert torch.equal(out != 0, kept((1, number), 300, 64, 0.5).to(DEV))
    del graph
    br.close()


# ------------------------------------------------------------------ residual
SHAPES = [(1, 1, 4, 1), (1, 130, 64, 4), (3, 777, 80, 4), (2, 300, 1024, 3), (5, 64, 36, 16), (32, 33, 256, 2), (2, 41, 516, 5), (2, 60, 772, 2), (1, 9000, 8, 3),
          (1, 777, 264, 4), (3, 401, 512, 2), (2, 333, 640, 3), (32, 5, 264, 16), (16, 40, 996, 16)]
KINDS = {  # tx, tf, ty, parameters, gate, p
    "all, fp32 rows": (torch.float32, torch.bfloat16, torch.bfloat16, PARAMS, True, 0.1),
    "all, bf16": (torch.bfloat16, torch.bfloat16, torch.bfloat16, PARAMS, True, 0.0),
    "all, bf16, dropped": (torch.bfloat16, torch.bfloat16, torch.bfloat16, PARAMS, True, 0.25),
    "all, fp16": (torch.float16, torch.float16, torch.float16, PARAMS, True, 0.0),
    "all, fp16, dropped": (torch.float16, torch.float16, torch.float16, PARAMS, False, 0.1),
    "all, fp16, to fp32": (torch.float16, torch.float16, torch.float32, PARAMS, False, 0.5),
    "norm behind": (torch.float32, torch.float32, torch.float32, ("post_weight", "post_bias"), False, 0.2),
    "norm before": (torch.float32, torch.float16, torch.bfloat16, ("pre_weight",), True, 0.0),
    "no norm": (torch.bfloat16, torch.float32, torch.float32, ("scale",), True, 0.3),
    "sum": (torch.float32, torch.bfloat16, torch.float32, (), False, 0.0),
    "weights": (torch.float32, torch.bfloat16, torch.float16, ("post_weight", "pre_weight", "pre_bias"), False, 0.0),
}


def inputs(g, B, N, C, E, kind):
    tx, tf, ty, names, gated, p = KINDS[kind]
    x, f = rand(g, B, N, C, scale=2.0) + 0.5, rand(g, B, N, C, scale=1.5) + 0.25
    f = torch.where(torch.rand((B, N, 1), generator=g, device=DEV) < 0.1, torch.zeros_like(f), f)     # rows of points that no camera sees
    params = {k: (1.0 if "weight" in k else 0.5 if k == "scale" else 0.0) + 0.1 * rand(g, E, C) for k in names}
    gate = torch.rand((B, N), generator=g, device=DEV) if gated else None
    return x.to(tx), f.to(tf), params, gate, p, ty


def near(got, want, bound, inside=None):
    ok = (got.double() - want).abs() <= bound
    return bool((ok if inside is None else ok[inside]).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,N,C,E", SHAPES)
def test_residual_and_its_gradients(B, N, C, E, kind):
    g = generator(B * N + C)
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = ascending_offsets(B, N, E, seed=N)
    x, f, params, gate, p, ty = inputs(g, B, N, C, E, kind)
    e = expert_of_rows(offsets, N, E)
    inside = e < E
    x[~inside], f[~inside] = float("nan"), float("nan")                     # rows of no expert reach nothing
    if gate is not None:
        gate[~inside] = float("nan")
    seed = seeds(123456789 + C, N)
    keep = kept(seed.tolist(), B * N, C, p).view(B, N, C).to(DEV) if p else None
    pre = "pre_weight" in params
    out = {"out": torch.full_like(x, 7.0), "y": torch.full((B, N, C), 7.0, dtype=ty, device=DEV) if pre else None,
           "stats": torch.full((B, N, 4), 7.0, device=DEV)}
    br.expert_residual(x, f, offsets, gate=gate, **params, eps=1e-5, p=p, seed=seed if p else None, out=out)
    ref = forward(x, f, offsets, E, gate, params, 1e-5, keep, p)
    for name, (want, bound) in ref.items():
        assert (out[name][~inside] == 7).all(), name
        if name == "y":
            bound = bound + unit(ty) * 1.02 * want.abs() + tiny(ty)
        assert near(out[name], want, bound, inside), name

    grad_out, grad_y = rand(g, B, N, C, dtype=x.dtype), rand(g, B, N, C, dtype=ty) if pre else None
    grad_out[~inside] = float("nan")
    if pre:
        grad_y[~inside] = float("nan")
        out["y"] = None
    back = {k: v for k, v in params.items() if k != "pre_bias"}
    rows, stats = out["out"], out["stats"] if pre or "post_weight" in params else None
    got = {"grad_x": torch.full_like(x, 7.0), "grad_f": torch.full_like(f, 7.0), "grad_gate": torch.full_like(gate, 7.0) if gate is not None else None}
    got.update({"grad_" + k: torch.full((E, C), float("nan"), device=DEV) for k in params})
    br.expert_residual_grad(rows, f, offsets, stats, grad_out, grad_y, gate=gate, **back, p=p, seed=seed, out=got)
    ref = gradients(rows, f, offsets, E, stats, grad_out, grad_y, gate, params, keep, p)
    for name, t in got.items():
        if t is None:
            continue
        want, bound = ref[name]
        if name in ("grad_x", "grad_f", "grad_gate"):
            assert (t[~inside] == 7).all(), name
            assert near(t, want, bound, inside), name
        else:
            assert near(t, want, bound + 1e-37), name
    if pre:                                                                 # no gradient from behind but the norm's
        none = br.expert_residual_grad(rows, f, offsets, stats, None, grad_y, gate=gate, **back, p=p, seed=seed)
        ref = gradients(rows, f, offsets, E, stats, None, grad_y, gate, params, keep, p)
        assert near(none["grad_x"], *ref["grad_x"], inside) and near(none["grad_f"], *ref["grad_f"], inside)
    again = br.expert_residual_grad(rows, f, offsets, stats, grad_out, grad_y, gate=gate, **back, p=p, seed=seed)
    for k in params:
        assert torch.equal(again["grad_" + k], got["grad_" + k]), k          # bit for bit
    br.status()
    br.close()


def test_residual_against_its_parts():
    """The same as the calls that it stands for, on shifted memory too: norm, dropout, sum, norm, within their roundings."""
    g = generator(2)
    B, N, C, E = 2, 333, 64, 4
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = torch.tensor([[0, 100, 100, 200, N]] * B, dtype=torch.int32, device=DEV)
    x, f, params, gate, p, _ = inputs(g, B, N, C, E, "all, fp32 rows")
    seed = seeds(9, 9)
    n = br.expert_norm(f, offsets, params["post_weight"], params["post_bias"], out_dtype=torch.float32)
    d = br.row_dropout(n["y"], p, seed)
    e = expert_of_rows(offsets, N, E)
    o = x + params["scale"][e] * gate[..., None] * d
    m = br.expert_norm(o, offsets, params["pre_weight"], params["pre_bias"], out_dtype=torch.bfloat16)
    for shift in (0, 4):
        got = br.expert_residual(shifted(x, shift), shifted(f, 2 * shift), offsets, gate=shifted(gate, shift), **params, p=p, seed=seed)
        assert torch.equal(got["out"][d == 0], x[d == 0])
        assert float((got["out"] - o).abs().max()) <= 8 * 2.0 ** -24 * float(o.abs().max() + d.abs().max())
        assert float((got["y"].double() - m["y"].double()).abs().max()) <= 2.0 ** -7 * float(m["y"].abs().max())
        assert torch.equal(got["stats"][..., 0], n["mean"]) or float((got["stats"][..., 0] - n["mean"]).abs().max()) < 1e-6
    br.close()


def test_residual_gradient_against_differences():
    g = generator(3)
    B, N, C, E = 1, 12, 20, 3
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = torch.tensor([[0, 5, 5, 12]], dtype=torch.int32, device=DEV)
    x, f, grad_out, grad_y = (rand(g, B, N, C) for _ in range(4))
    params = {k: (1.0 if "weight" in k else 0.5) + 0.1 * rand(g, E, C) for k in PARAMS}
    gate, seed, p = torch.rand((B, N), generator=g, device=DEV), seeds(4, 2), 0.3
    keep = kept(seed.tolist(), N, C, p).view(B, N, C).to(DEV)
    made = br.expert_residual(x, f, offsets, gate=gate, **params, p=p, seed=seed, y_dtype=torch.float32)
    got = br.expert_residual_grad(made["out"], f, offsets, made["stats"], grad_out, grad_y, gate=gate, p=p, seed=seed,
                                  **{k: v for k, v in params.items() if k != "pre_bias"})

    def loss(x, f, gate, params):
        r = forward(x, f, offsets, E, gate, params, 1e-5, keep, p)
        return float((r["out"][0] * grad_out.double()).sum() + (r["y"][0] * grad_y.double()).sum())

    step = 1e-5
    wide = {k: v.double() for k, v in params.items()}
    at = {"grad_x": (x, lambda t: (t, f, gate, wide)), "grad_f": (f, lambda t: (x, t, gate, wide)), "grad_gate": (gate, lambda t: (x, f, t, wide))}
    for k in PARAMS:
        at["grad_" + k] = (params[k], lambda t, k=k: (x, f, gate, {**wide, k: t}))
    for name, (value, args) in at.items():
        way = torch.randn(value.shape, generator=g, device=DEV, dtype=torch.float64)
        slope = (loss(*args(value.double() + step * way)) - loss(*args(value.double() - step * way))) / (2 * step)
        # Central differences in 64 bits: 1e-9 of curvature and 1e-10 of rounding beside the gradient's own fp32, whose norms have rows
        # in fp32.
        size = float((got[name].double().abs() * way.abs()).sum())
        assert abs(slope - float((got[name].double() * way).sum())) <= 1e-5 * size + 1e-6, name
    br.close()


def test_everything_dropped_and_infinities_in_dropped_places():
    g = generator(4)
    B, N, C = 1, 40, 24
    br = handle(B, N, 1)
    br.reserve_rows(C)
    x, f = rand(g, B, N, C), rand(g, B, N, C)
    seed = seeds(0, 0)
    got = br.expert_residual(x, f, None, p=1.0, seed=seed)
    assert torch.equal(got["out"], x)
    grad = br.expert_residual_grad(got["out"], f, None, None, torch.ones_like(x), None, p=1.0, seed=seed, scale=torch.ones((1, C), device=DEV))
    assert (grad["grad_f"] == 0).all() and (grad["grad_scale"] == 0).all() and (grad["grad_x"] == 1).all()
    keep = kept((0, 0), N, C, 0.5).view(B, N, C).to(DEV)
    bad = torch.where(keep, f, torch.full_like(f, float("nan")))
    dout = torch.where(keep, x, torch.full_like(x, float("-inf")))
    got = br.expert_residual(x, bad, None, p=0.5, seed=seed)
    assert torch.isfinite(got["out"]).all() and torch.equal(got["out"][~keep], x[~keep])
    grad = br.expert_residual_grad(got["out"], bad, None, None, dout, None, p=0.5, seed=seed, scale=torch.ones((1, C), device=DEV))
    assert torch.isfinite(grad["grad_f"]).all() and torch.isfinite(grad["grad_scale"]).all()
    br.close()


def test_offsets_that_do_not_ascend_are_reported():
    import paper_2507_04123_b200 as pkg
    br = handle(2, 40, 3)
    br.reserve_rows(8)
    x, w = torch.ones((2, 40, 8), device=DEV), torch.ones((3, 8), device=DEV)
    for row in ([0, 20, 10, 40], [-5, 1, 2, 3], [50, 60, 70, 80], [0, 10, 20, 41]):
        offsets = torch.tensor([row, [0, 0, 0, 0]], dtype=torch.int32, device=DEV)
        out = {"out": torch.full_like(x, 7.0), "y": torch.full_like(x, 7.0), "stats": torch.zeros((2, 40, 4), device=DEV)}
        br.expert_residual(x, x, offsets, pre_weight=w, out=out)
        assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
        assert (out["out"][1] == 7).all() and (out["y"][1] == 7).all()
        br.expert_residual_grad(x, x, offsets, out["stats"], x, x, pre_weight=w)
        assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
    br.close()


def test_a_block_of_a_training_step():
    """Norm, feed-forward block and residual behind one another, forward and backward, on another stream and captured: the gradients of the
    whole chain against the product rule by hand, and replays bit for bit with the seed of the replay."""
    g = generator(6)
    B, N, C, H, E = 2, 500, 64, 96, 4
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    offsets = torch.tensor([[0, 100, 180, 400, N], [0, 0, 250, 250, 480]], dtype=torch.int32, device=DEV)
    x = rand(g, B, N, C)
    w1, b1 = 1 + 0.1 * rand(g, E, C), 0.1 * rand(g, E, C)
    wg, wu, wd = rand(g, E, H, C, scale=C ** -0.5).bfloat16(), rand(g, E, H, C, scale=C ** -0.5).bfloat16(), rand(g, E, C, H, scale=H ** -0.5).bfloat16()
    params = {k: (1.0 if "weight" in k else 0.5 if k == "scale" else 0.0) + 0.1 * rand(g, E, C) for k in PARAMS}
    back = {k: v for k, v in params.items() if k != "pre_bias"}
    gate, grad_out, grad_y = torch.rand((B, N), generator=g, device=DEV), rand(g, B, N, C), rand(g, B, N, C, dtype=torch.bfloat16)
    seed = seeds(77, 0)

    def step(o):
        o["n"] = br.expert_norm(x, offsets, w1, b1, out_dtype=torch.bfloat16, out=o.get("n"))
        o["f"] = br.expert_ffn(o["n"]["y"], offsets, wg, wu, wd, out=o.get("f"))
        o["r"] = br.expert_residual(x, o["f"], offsets, gate=gate, **params, p=0.2, seed=seed, out=o.get("r"))
        o["gr"] = br.expert_residual_grad(o["r"]["out"], o["f"], offsets, o["r"]["stats"], grad_out, grad_y, gate=gate, **back, p=0.2, seed=seed,
                                          out=o.get("gr"))
        o["gf"] = br.expert_ffn_grad(o["n"]["y"], offsets, wg, wu, wd, o["gr"]["grad_f"], out=o.get("gf"))
        o["gn"] = br.expert_norm_grad(x, offsets, w1, o["n"]["mean"], o["n"]["rstd"], o["gf"]["grad_x"], out=o.get("gn"))
        return o

    def flat(o):
        return [o["f"], *(t for k in ("n", "r", "gr", "gf", "gn") for t in o[k].values())]

    bufs = step({})
    for t in flat(bufs):
        t.zero_()                                                           # rows of no expert
    want = []
    for number in range(2):
        seed[1] = number
        step(bufs)
        want.append([t.clone() for t in flat(bufs)])
    keep = kept((77, 1), B * N, C, 0.2).view(B, N, C).to(DEV)
    inside = expert_of_rows(offsets, N, E) < E
    ref = forward(x, bufs["f"], offsets, E, gate, params, 1e-5, keep, 0.2)
    assert near(bufs["r"]["out"], *ref["out"], inside)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in flat(bufs):
            t.zero_()
        step(bufs)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(flat(bufs), want[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(bufs)
    for number in (0, 1, 0):
        seed[1] = number
        for t in flat(bufs):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(bufs), want[number]))
    br.status()
    del graph
    br.close()


def test_calls_that_are_refused():
    import paper_2507_04123_b200 as pkg
    br = handle(2, 40, 3)
    lib, bad, large = pkg.load_library(), pkg.bridge.EMC2_ERR_INVALID_ARG, pkg.bridge.EMC2_ERR_TOO_LARGE
    x, f, o, y = (torch.ones((2, 40, 8), device=DEV) for _ in range(4))
    w, gate, st, seed = torch.ones((3, 8), device=DEV), torch.ones((2, 40), device=DEV), torch.ones((2, 40, 4), device=DEV), seeds(1, 1)
    P = lambda t, off=0: None if t is None else t.data_ptr() + off          # noqa: E731

    def drop(n=80, C=8, kind=0, x=P(x), p=0.5, seed=P(seed), y=P(y)):
        return lib.emc2_row_dropout(br._h, n, C, kind, x, p, seed, y, None)

    assert drop() == 0 and drop(n=0, x=None, y=None) == 0
    for wrong in (dict(n=-1), dict(n=81), dict(C=6), dict(C=0), dict(C=1028), dict(kind=3), dict(kind=-1), dict(x=None), dict(y=None), dict(p=-0.1), dict(p=1.5),
                  dict(p=float("nan")), dict(seed=None), dict(seed=P(seed, 4)), dict(x=P(x, 4)), dict(y=P(y, 8)), dict(y=P(x))):
        assert drop(**wrong) == bad, wrong

    def res(B=2, N=40, C=8, tx=0, x=P(x), f=P(f), offs=None, gate=P(gate), w=P(w), b=P(w), s=P(w), w2=P(w), b2=P(w), eps=1e-5, p=0.0, seed=None, o=P(o), y=P(y), st=P(st)):
        return lib.emc2_expert_residual(br._h, B, N, C, tx, 0, 0, x, f, offs, gate, w, b, s, w2, b2, eps, p, seed, o, y, st, None)

    assert res() == 0 and res(B=0, x=None, f=None, o=None, y=None) == 0 and res(gate=None, w=None, b=None, s=None, w2=None, b2=None, y=None, st=None) == 0
    for wrong in (dict(B=3), dict(B=-1), dict(N=41), dict(C=10), dict(tx=3), dict(x=None), dict(f=None), dict(o=None), dict(y=None), dict(w2=None, b2=None), dict(w=None),
                  dict(w2=None, y=None), dict(eps=-1.0), dict(eps=float("nan")), dict(p=0.5), dict(p=2.0, seed=P(seed)), dict(o=P(x)), dict(o=P(f)), dict(y=P(o)), dict(y=P(x)),
                  dict(x=P(x, 8)), dict(st=P(st, 4)), dict(w=P(w, 4)), dict(gate=P(gate, 2)), dict(seed=P(seed, 4)), dict(offs=P(gate, 2))):
        assert res(**wrong) == bad, wrong

    ga, gb, gc = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)

    def grad(B=2, C=8, o=P(o), f=P(f), st=P(st), do=P(x), dy=P(y), gate=P(gate), w=P(w), b=P(w), s=P(w), w2=P(w), p=0.0, seed=None, dx=P(ga), df=P(gb), dg=None, dw=P(gc), db=None, ds=None,
             dw2=None, db2=None):
        return lib.emc2_expert_residual_grad(br._h, B, 40, C, 0, 0, 0, o, f, None, st, do, dy, gate, w, b, s, w2, p, seed, dx, df, dg, dw, db, ds, dw2, db2, None)

    assert grad() == large                                                  # nothing reserved
    br.reserve_rows(4)
    assert grad() == large
    br.reserve_rows(8)
    assert grad() == 0 and grad(do=None) == 0 and grad(B=0) == 0
    for wrong in (dict(B=3), dict(o=None), dict(f=None), dict(st=None), dict(dy=None), dict(do=None, w2=None, dy=None), dict(dx=None), dict(df=None), dict(dx=P(gb)), dict(dx=P(x)), dict(df=P(f)),
                  dict(w=None, b=None), dict(gate=None, dg=P(gate)), dict(w2=None, dw2=P(gc)), dict(p=0.1), dict(dx=P(ga, 4)), dict(dw=P(gc, 2)), dict(st=P(st, 8)), dict(C=7)):
        assert grad(**wrong) == bad, wrong
    zero = torch.full((1, 8), 3.0, device=DEV)                              # without offsets there is one expert
    assert grad(B=0, dw=P(zero)) == 0
    assert (zero == 0).all()
    br.status()
    # The binding's own checks.
    with pytest.raises(ValueError):
        br.expert_residual(x, f, None, p=0.1)
    with pytest.raises(ValueError):
        br.expert_residual(x, f.transpose(0, 1).contiguous().transpose(0, 1), None)
    with pytest.raises(ValueError):
        br.row_dropout(x, 0.1, seed.int())
    with pytest.raises(ValueError):
        br.expert_residual_grad(x, f, None, None, x, None, post_weight=torch.ones((1, 8), device=DEV))
    with pytest.raises(ValueError):
        br.expert_residual(x.double(), f, None)
    br.close()
