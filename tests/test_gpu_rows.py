"""Row lookup and expert norm, forward and backward, against the formulas in 64 bits (needs a B200).

Tolerances count roundings: u = eps / 2 of a type is the relative error of one rounding to it.  A fp32 sum of n terms in any
tree or sequence is off by at most n u32 times the sum of the terms' sizes; results rounded to a 16-bit type add u of it."""
import numpy as np
import pytest
import torch

from row_cases import TYPES, ascending_offsets, expert_of_rows, handle, norm_reference, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ lookup
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,rows,C", [(1, 1, 4), (7, 3, 36), (1025, 64, 64), (4099, 100000, 80), (333, 5, 1024), (2050, 17, 132)])
def test_lookup(n, rows, C, dtype):
    g = generator(n)
    br = handle(1, max(n, 8))
    table = rand(g, rows, C, dtype=dtype)
    ids = torch.randint(-1, rows, (n,), generator=g, device=DEV, dtype=torch.int32)
    scale = 1.7
    out = br.row_lookup(ids, table, scale)
    # The scale reaches the library as fp32; the product is rounded in fp32 and then to the type.
    want = table.double()[ids.long().clamp(min=0)] * float(np.float32(scale)) * (ids >= 0)[:, None]
    tol = (2.0 ** -24 + unit(dtype)) * want.abs() * (1 + 2.0 ** -7)
    # Below the type's smallest normal number its steps are all of smallest_normal * eps, and a rounding is off by half of one.
    tol = tol + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    assert ((out.double() - want).abs() <= tol).all()
    assert (out[ids < 0] == 0).all()
    br.status()
    br.close()


def test_lookup_reports_ids_behind_the_table():
    import paper_2507_04123_b200 as pkg
    br = handle(1, 64)
    br.reserve_rows(8)
    table = torch.ones((5, 8), device=DEV)
    ids = torch.tensor([0, 5, 4, 2**31 - 1, -(2**31), -1], dtype=torch.int32, device=DEV)
    out = br.row_lookup(ids, table)
    assert out[:, 0].tolist() == [1, 0, 1, 0, 0, 0]
    assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
    grad = br.row_lookup_grad(ids, torch.ones((6, 8), device=DEV), 5)
    assert grad[:, 0].tolist() == [1, 0, 0, 0, 1]
    assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
    assert br.status() == 0
    none = br.row_lookup(ids, torch.empty((0, 8), device=DEV))             # a table without rows: zeros
    assert (none == 0).all()
    br.status(raise_on_error=False)
    br.close()


PATTERNS = {"spread": lambda n, V, g: torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32),
            "one": lambda n, V, g: torch.full((n,), V // 2, dtype=torch.int32, device=DEV),
            "none": lambda n, V, g: torch.full((n,), -1, dtype=torch.int32, device=DEV),
            "runs": lambda n, V, g: (torch.arange(n, device=DEV) * V // n).to(torch.int32),
            "ends": lambda n, V, g: torch.where(torch.rand(n, generator=g, device=DEV) < 0.5, 0, V - 1).to(torch.int32)}


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,V,C", [(1, 1, 4), (255, 256, 64), (5000, 70000, 80), (40000, 9, 64), (3001, 1000, 1024), (9999, 300, 36)])
def test_lookup_gradient(n, V, C, dtype, pattern):
    g = generator(n + V)
    br = handle(1, n)
    br.reserve_rows(C)
    ids = PATTERNS[pattern](n, V, g)
    dout = rand(g, n, C, dtype=dtype)
    scale = 0.37
    out = torch.full((V, C), float("nan"), dtype=dtype, device=DEV)
    br.row_lookup_grad(ids, dout, V, scale, out=out)
    keep = ids >= 0
    want, size = (torch.zeros((V, C), dtype=torch.float64, device=DEV) for _ in range(2))
    want.index_add_(0, ids[keep].long(), dout[keep].double())
    size.index_add_(0, ids[keep].long(), dout[keep].double().abs())
    times = torch.bincount(ids[keep].long(), minlength=V)[:, None]
    s = float(np.float32(scale))
    tol = s * ((times + 1) * 2.0 ** -24 * size * 1.01 + unit(dtype) * 1.01 * want.abs())
    # What a 16-bit result cannot hold at all is below its smallest number.
    tol = tol + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert ((out.double() - want * s).abs() <= tol).all()
    assert (out[times[:, 0] == 0] == 0).all()
    again = br.row_lookup_grad(ids, dout, V, scale)
    assert torch.equal(again.view(torch.uint8), out.view(torch.uint8))      # bit for bit
    br.status()
    br.close()


def test_lookup_and_gradient_of_the_largest_table():
    """2^31 - 1 rows: row numbers, their count of CTAs and the rows' addresses at the end of 32 bits."""
    n, V, C = 3000, 2 ** 31 - 1, 4
    g = generator(31)
    br = handle(1, n)
    br.reserve_rows(C)
    ids = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    ids[:3], ids[3:6] = V - 1, torch.tensor([0, -1, V - 2], dtype=torch.int32, device=DEV)
    dout = torch.randint(1, 4, (n, C), generator=g, device=DEV).to(torch.bfloat16)          # sums that bf16 holds
    table = torch.full((V, C), float("nan"), dtype=torch.bfloat16, device=DEV)
    br.row_lookup_grad(ids, dout, V, out=table)
    named, at = torch.unique(ids[ids >= 0].long(), return_inverse=True)
    want = torch.zeros((len(named), C), device=DEV).index_add_(0, at, dout[ids >= 0].float())
    assert torch.equal(table[named].float(), want)
    rows = br.row_lookup(ids, table)
    assert torch.equal(rows[ids >= 0].float(), want[at]) and (rows[ids < 0] == 0).all()
    table[named] = 0
    assert all(bool((part == 0).all()) for part in table.split(2 ** 26))
    br.status()
    br.close()


def test_lookup_gradient_against_differences():
    g = generator(5)
    n, V, C = 300, 40, 8
    br = handle(1, n)
    br.reserve_rows(C)
    ids = torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    dout = rand(g, n, C)
    grad = br.row_lookup_grad(ids, dout, V, 2.0)
    table = rand(g, V, C)
    # The lookup is linear: a step of 1 along a direction gives the product with the gradient.
    step = rand(g, V, C)
    a, b = (br.row_lookup(ids, t, 2.0).double() for t in (table, table + step))
    got, want = ((b - a) * dout.double()).sum(), (grad.double() * ((table + step).double() - table.double())).sum()
    # Every looked-up value is off by u32 of itself; the gradient by n u32 of its sum.
    size = (b.abs() + a.abs()).mul(dout.double().abs()).sum() + n * (grad.double().abs() * step.double().abs()).sum()
    assert abs(float(got - want)) <= 4 * 2.0 ** -24 * float(size)
    br.close()


# ------------------------------------------------------------------ norm
NORM = [(1, 1, 4, 1), (1, 130, 64, 4), (3, 777, 80, 4), (2, 500, 1024, 3), (5, 64, 36, 16), (32, 33, 256, 2), (2, 41, 516, 5)]


@pytest.mark.parametrize("tx,ty", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16),
                                   (torch.float16, torch.float16), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float32)], ids=str)
@pytest.mark.parametrize("B,N,C,E", NORM)
def test_norm_and_its_gradients(B, N, C, E, tx, ty):
    g = generator(B * N + C)
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = ascending_offsets(B, N, E, seed=N)
    x = rand(g, B, N, C, scale=2.0) + 0.5
    x = torch.where(torch.rand((B, N, 1), generator=g, device=DEV) < 0.1, torch.zeros_like(x), x).to(tx)
    e = expert_of_rows(offsets, N, E)
    x[e == E] = float("nan")                                                # rows of no expert reach nothing
    w, b = 1 + 0.1 * rand(g, E, C), 0.1 * rand(g, E, C)
    out = {"y": torch.full((B, N, C), 7.0, dtype=ty, device=DEV), "mean": torch.full((B, N), 7.0, device=DEV),
           "rstd": torch.full((B, N), 7.0, device=DEV)}
    br.expert_norm(x, offsets, w, b, 1e-5, out=out)
    ref = norm_reference(x, e, E, w, b, 1e-5)
    inside = e < E
    assert (out["y"][~inside] == 7).all() and (out["mean"][~inside] == 7).all() and (out["rstd"][~inside] == 7).all()
    u32 = 2.0 ** -24
    xd = x.double()
    size = xd.abs().mean(-1)
    # A mean of C values in fp32: C additions and a product.
    err_mean = (C + 2) * u32 * size
    assert ((out["mean"].double() - ref["mean"]).abs() <= err_mean)[inside].all()
    # A shift d of the mean adds d^2 to the variance, a relative 2 u32 per difference and C additions of squares; rstd
    # moves by half the relative change, at most by that of the variance alone, and takes an approximate root (2 ulp).
    d_abs = u32 * 2 * (xd - ref["mean"][..., None]).abs().amax(-1) + err_mean
    var = ref["var"]
    rel_var = ((C + 4) * u32 * var + 2 * d_abs * var.sqrt() + d_abs ** 2) / (var + 1e-5)
    err_rstd = (rel_var / 2 + 6 * u32) * ref["rstd"] * 1.05
    assert ((out["rstd"].double() - ref["rstd"]).abs() <= err_rstd)[inside].all()
    wd = w.double()[e.clamp(max=E - 1)]
    h = ref["h"]
    err_h = (d_abs * ref["rstd"])[..., None] + (err_rstd / ref["rstd"])[..., None] * h.abs() + 4 * u32 * h.abs()
    err_y = err_h * wd.abs() + 4 * u32 * ((h * wd).abs() + ref["y"].abs()) + unit(ty) * 1.02 * ref["y"].abs() + torch.finfo(ty).smallest_normal * torch.finfo(ty).eps
    assert ((out["y"].double() - ref["y"]).abs() <= err_y * 1.05)[inside].all()

    # Gradients, from the mean and the rstd that the call left.
    dy = rand(g, B, N, C, dtype=ty)
    dy[e == E] = float("nan")
    grads = {"grad_x": torch.full((B, N, C), 7.0, dtype=tx, device=DEV), "grad_weight": torch.full((E, C), float("nan"), device=DEV),
             "grad_bias": torch.full((E, C), float("nan"), device=DEV)}
    br.expert_norm_grad(x, offsets, w, out["mean"], out["rstd"], dy, out=grads)
    m, r = out["mean"].double()[..., None], out["rstd"].double()[..., None]
    h = (xd - m) * r
    gw = dy.double() * wd
    a, c = gw.mean(-1, keepdim=True), (gw * h).mean(-1, keepdim=True)
    want = r * (gw - a - h * c)
    assert (grads["grad_x"][~inside] == 7).all()
    # g is one product, h a difference and a product; the means add C terms.
    err_h = 2.1 * u32 * h.abs()
    err_a = (C + 3) * u32 * gw.abs().mean(-1, keepdim=True)
    err_c = (C + 6) * u32 * (gw * h).abs().mean(-1, keepdim=True)
    err = r * (u32 * gw.abs() + err_a + err_h * c.abs() + h.abs() * err_c + 4 * u32 * (gw.abs() + a.abs() + (h * c).abs())) * 1.05
    err = err + unit(tx) * 1.02 * want.abs() + torch.finfo(tx).smallest_normal * torch.finfo(tx).eps
    assert ((grads["grad_x"].double() - want).abs() <= err)[inside].all()
    for k in range(E):
        rows = e == k
        n = int(rows.sum())
        term = dy.double()[rows] * h[rows]
        tol = (n + 5) * u32 * term.abs().sum(0) * 1.05
        assert ((grads["grad_weight"][k].double() - term.sum(0)).abs() <= tol).all(), k
        bias = dy.double()[rows]
        assert ((grads["grad_bias"][k].double() - bias.sum(0)).abs() <= (n + 2) * u32 * bias.abs().sum(0) * 1.05).all(), k
    again = br.expert_norm_grad(x, offsets, w, out["mean"], out["rstd"], dy)
    for k in ("grad_weight", "grad_bias"):
        assert torch.equal(again[k], grads[k])
    br.status()
    br.close()


def test_norm_gradient_against_differences():
    g = generator(3)
    B, N, C, E = 1, 12, 16, 3
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = torch.tensor([[0, 5, 5, 12]], dtype=torch.int32, device=DEV)
    x, w, b, dy = rand(g, B, N, C), 1 + 0.1 * rand(g, E, C), 0.1 * rand(g, E, C), rand(g, B, N, C)
    f = br.expert_norm(x, offsets, w, b)
    got = br.expert_norm_grad(x, offsets, w, f["mean"], f["rstd"], dy)
    e = expert_of_rows(offsets, N, E)

    def loss(x, w, b):
        return float((norm_reference(x, e, E, w, b, 1e-5)["y"] * dy.double()).sum())

    step = 1e-5
    for name, at, args in (("grad_x", x, lambda t: (t, w.double(), b.double())), ("grad_weight", w, lambda t: (x.double(), t, b.double())),
                           ("grad_bias", b, lambda t: (x.double(), w.double(), t))):
        way = torch.randn(at.shape, generator=g, device=DEV, dtype=torch.float64)
        slope = (loss(*args(at.double() + step * way)) - loss(*args(at.double() - step * way))) / (2 * step)
        # Central differences in 64 bits: 1e-10 of curvature and 1e-11 of rounding beside the gradient's own fp32.
        size = float((got[name].double().abs() * way.abs()).sum())
        assert abs(slope - float((got[name].double() * way).sum())) <= 1e-5 * size + 1e-6, name
    br.close()


def test_norm_without_offsets_bias_or_statistics():
    g = generator(9)
    br = handle(2, 50, 4)
    br.reserve_rows(64)
    x, w = rand(g, 2, 50, 64), 1 + 0.1 * rand(g, 1, 64)
    out = br.expert_norm(x, None, w, out={"y": torch.empty_like(x), "mean": None, "rstd": None})
    want = torch.nn.functional.layer_norm(x.double(), (64,), w[0].double())
    assert float((out["y"].double() - want).abs().max()) < 1e-5
    f = br.expert_norm(x, None, w)
    got = br.expert_norm_grad(x, None, w, f["mean"], f["rstd"], torch.ones_like(x), out={"grad_x": torch.empty_like(x), "grad_weight": torch.empty_like(w), "grad_bias": None})
    assert float(got["grad_weight"].double().sub(((x.double() - x.double().mean(-1, keepdim=True)) * f["rstd"].double()[..., None]).sum((0, 1))).abs().max()) < 1e-4
    br.close()


def test_offsets_that_do_not_ascend_are_reported_and_stay_in_bounds():
    import paper_2507_04123_b200 as pkg
    br = handle(2, 40, 3)
    br.reserve_rows(8)
    x, w = torch.ones((2, 40, 8), device=DEV), torch.ones((3, 8), device=DEV)
    for row in ([0, 20, 10, 40], [-5, 1, 2, 3], [0, 10, 2**31 - 1, 40], [50, 60, 70, 80], [0, 10, 20, 41]):
        offsets = torch.tensor([row, [0, 0, 0, 0]], dtype=torch.int32, device=DEV)
        out = {"y": torch.full_like(x, 7.0), "mean": torch.zeros((2, 40), device=DEV), "rstd": torch.zeros((2, 40), device=DEV)}
        br.expert_norm(x, offsets, w, out=out)
        assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
        assert (out["y"][1] == 7).all()
        br.expert_norm_grad(x, offsets, w, out["mean"], out["rstd"], x)
        assert br.status(raise_on_error=False) == pkg.bridge.EMC2_ERR_INVALID_ARG
    br.close()


# ------------------------------------------------------------------ together, on other streams, captured
def test_calls_captured_replayed_and_on_another_stream():
    g = generator(21)
    B, N, C, E, V = 2, 1000, 64, 4, 500
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = ascending_offsets(B, N, E, seed=1)
    x, dy = rand(g, B, N, C), rand(g, B, N, C)
    w, b = 1 + 0.1 * rand(g, E, C), 0.1 * rand(g, E, C)
    ids = torch.randint(-1, V, (B, N), generator=g, device=DEV, dtype=torch.int32)
    table = rand(g, V, C)

    def run(o):
        o["look"] = br.row_lookup(ids, table, 2.0, out=o.get("look"))
        o["norm"] = br.expert_norm(x, offsets, w, b, out=o.get("norm"))
        o["grad"] = br.expert_norm_grad(x, offsets, w, o["norm"]["mean"], o["norm"]["rstd"], dy, out=o.get("grad"))
        o["table"] = br.row_lookup_grad(ids, dy, V, 2.0, out=o.get("table"))
        return o

    def flat(o):
        return [o["look"], o["table"], *o["norm"].values(), *o["grad"].values()]

    bufs = run({})
    for t in flat(bufs):
        t.zero_()                                            # rows of no expert
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
    for _ in range(2):
        for t in flat(bufs):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(bufs), want))
    # A larger area leaves the captured one in place.
    before = br.scratch_bytes
    br.reserve_rows(4 * C)
    assert br.scratch_bytes > before
    for t in flat(bufs):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat(bufs), want))
    br.status()
    del graph
    br.close()
