"""The layer with 4-bit weights whose powers of two rise and fall along a row, over several steps of the products (needs a B200).

The kernels take elements relative to the largest power that their row has had so far and scale their sums down when it rises.  In fp16 an
element is rounded to a multiple of 2^-24 of the row's largest power: it is exact if it is one, else off by half of that.  Where the
largest blocks meet zeros (of the rows, or of hidden units whose up projection is zero), only the small ones count.

Bounds.  Sums of n products: 2^-22 a term, as elsewhere.  act(g): 2^-20 of itself, its argument's error times its slope, and for the normal
distribution's argument g^2 2^-23.  A hidden value in two parts: unit^2 of it, or half of the type's smallest number.  A weight of a
choice: 2^-20."""
import pytest
import torch

from layer_cases import values_of
from row_cases import activation, handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
S = 2.0 ** -22

# Exponents of the powers along a row of `blocks` blocks, and whether the largest blocks meet zeros.  A step has eight blocks, of which two warps can
# have four each.
PATTERNS = {
    "23 below, the large last": (lambda i, n: 16 if i == n - 1 else -7, True),
    "23 below, the large first": (lambda i, n: 16 if i == 0 else -7, True),
    "23 below, at the borders of steps": (lambda i, n: 16 if i in (3, 8) else -7, True),
    "26 below, within a step": (lambda i, n: 19 if i in (5, 6) else -7, True),
    "up by threes": (lambda i, n: min(-7, -43 + 3 * i), False),
    "up and down by tens": (lambda i, n: -7 - 10 * ((i + 1) % 4), False),
    "up by thirty in the second step": (lambda i, n: -7 if i >= 9 else -37, False),
    "down by threes": (lambda i, n: -7 - 3 * min(i, 10), False),
}


def off_weights(w, values, dtype):
    """Largest error of an element of fp16."""
    if dtype == torch.bfloat16:
        return torch.zeros_like(values)
    step = torch.exp2(w["scales"].double().amax(-1, keepdim=True) - 127 - 24)
    return torch.where(torch.remainder(values, step) == 0, torch.zeros_like(values), (step / 2).expand_as(values))


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("dtype,act", [(torch.float16, "silu"), (torch.bfloat16, "gelu")], ids=str)
@pytest.mark.parametrize("n,E,k", [(1, 2, 1), (3, 2, 1), (40, 1, 1), (128, 32, 8)])          # the last: a tile of a warp's own, several passes
def test_powers_along_the_rows(n, E, k, dtype, act, pattern):
    C, H = 520, 776
    at, zeros = PATTERNS[pattern]
    g = torch.Generator(device=DEV)
    g.manual_seed(n + len(pattern))

    def weights(M, K):
        blocks = -(-K // 32)
        exponent = torch.tensor([at(i, blocks) for i in range(blocks)], device=DEV)
        scales = exponent + torch.randint(-1, 2, (E, M, 1), generator=g, device=DEV) + 127
        codes = torch.randint(0, 256, (E, M, 16 * blocks), generator=g, device=DEV).to(torch.uint8)
        codes[..., K // 2:] = 0                                            # behind the row
        large = torch.repeat_interleave(exponent > 0, 32)[:K] if zeros else torch.zeros(K, dtype=torch.bool, device=DEV)
        return {"codes": codes, "scales": scales.to(torch.uint8)}, large

    x = torch.randn((n, C), generator=g, device=DEV).to(dtype)
    (wg, none), (wu, _), (wd, idle) = weights(H, C), weights(H, C), weights(C, H)
    x[:, none] = 0
    wu["codes"][:, idle] = 0
    wr = torch.randn((E, C), generator=g, device=DEV)
    br = handle(1, 8)
    br.reserve_rows(C, H)
    got = br.expert_layer(x, wr, wg, wu, wd, k, act)
    top, ids = torch.sort(x.double() @ wr.double().t(), dim=-1, descending=True, stable=True)
    ids, p = ids[:, :k], torch.softmax(top[:, :k], -1)
    assert torch.equal(got["ids"].long(), ids)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    y, err = torch.zeros((n, C), dtype=torch.float64, device=DEV), torch.zeros((n, C), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(y)
    for e in range(E):
        row, j = (ids == e).nonzero(as_tuple=True)
        if not len(row):
            continue
        (vg, og), (vu, ou), (vd, od) = ((v, off_weights(w, v, dtype)) for w, v in (({i: t[e] for i, t in w.items()}, values_of({i: t[e] for i, t in w.items()}, K))
                                                                                   for w, K in ((wg, C), (wu, C), (wd, H))))
        r = x[row].double()
        gate, up = r @ vg.t(), r @ vu.t()
        err_g, err_u = ((C + 16) * S * (r.abs() @ v.abs().t()) + r.abs() @ o.t() for v, o in ((vg, og), (vu, ou)))
        a, _, slope, _ = activation(gate, act)
        err_a = slope * err_g + (2.0 ** -20 + gate * gate * 2.0 ** -23) * a.abs()
        h = a * up
        err_h = err_a * (up.abs() + err_u) + a.abs() * err_u + (2.0 ** -24 + 1.01 * unit(dtype) ** 2) * h.abs() + torch.where(up == 0, 0.0, tiny / 2)
        z = h @ vd.t()
        err_z = err_h @ (vd.abs() + od).t() + h.abs() @ od.t() + (H + 16) * S * ((h.abs() + err_h) @ vd.abs().t())
        q = p[row, j][:, None]
        y.index_add_(0, row, q * z)
        err.index_add_(0, row, q * (err_z + 2.0 ** -20 * z.abs()))
        size.index_add_(0, row, q * (z.abs() + err_z))
    bound = 1.05 * (err + (k + 12) * 2.0 ** -24 * size) + unit(dtype) * 1.02 * y.abs() + tiny
    off = (got["y"].double() - y).abs()
    assert torch.isfinite(y).all() and float(y.abs().max()) < 60000
    assert (off <= bound).all(), (float((off / bound).max()), int((off > bound).sum()))
    again = br.expert_layer(x, wr, wg, wu, wd, k, act)
    assert all(torch.equal(again[i], got[i]) for i in got)
    br.status()
    br.close()
