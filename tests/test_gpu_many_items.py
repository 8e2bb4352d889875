"""Calls so large that every CTA comes round its stages and rows several times (needs a B200).

The values are small whole numbers, so that every product and every sum is exact in fp32 whatever its order, and the results are
those of 64 bits rounded once: a tile, row or stage taken twice, left out or read too early shows in the bits."""
import pytest
import torch

from row_cases import TYPES, ascending_offsets, expert_of_rows, handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def whole(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).float()


def sparse(g, E, rows, columns, per_column):
    """[E, rows, columns] of 1 and -1 in `per_column` places of each column at most, zeros elsewhere."""
    w = torch.zeros((E, rows, columns), device=DEV)
    for _ in range(per_column):
        at = torch.randint(0, rows, (E, 1, columns), generator=g, device=DEV)
        w.scatter_(1, at, 1 - 2 * torch.randint(0, 2, at.shape, generator=g, device=DEV).float())
    return w


# Several tiles, or pairs of tiles, per CTA at every width of the products: whole tiles with ragged ends, and ragged ones.
FFN = [(2, 80000, 64, 72, 3), (2, 80000, 80, 40, 3), (1, 160000, 128, 72, 4), (2, 50000, 200, 40, 3), (2, 50000, 256, 72, 2), (4, 40000, 24, 136, 2),
       (32, 5000, 80, 40, 16), (32, 3000, 256, 24, 16), (16, 8000, 96, 136, 5), (4, 20000, 48, 136, 3), (3, 30000, 176, 72, 4), (1, 90000, 120, 16, 1)]


def block(B, N, C, H, E, dtype):
    """Rows of -1, 0 and 1, the first always 1, and weights with which every gate is 28 .. 36, where act(g) is g and its slope 1
    in fp32 and in 64 bits, u and dh are -4 .. 4, and h, dg and du are whole numbers up to 144, exact in 16 bits."""
    g = generator(B * N + C + H)
    offsets = ascending_offsets(B, N, E, seed=N + C)
    e = expert_of_rows(offsets, N, E)
    x, dy = whole(g, -1, 1, B, N, C), whole(g, -1, 1, B, N, C)
    x[..., 0] = 1.0
    x[e == E], dy[e == E] = float("nan"), float("inf")                     # rows of no expert reach nothing
    wg, wu = sparse(g, E, C, H, 4).transpose(1, 2).contiguous(), sparse(g, E, C, H, 4).transpose(1, 2).contiguous()
    wg[..., 0] = 32.0
    return [t.to(dtype) for t in (x, dy, wg, wu, sparse(g, E, C, H, 4))], offsets, e


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("B,N,C,H,E", FFN)
def test_feed_forward_block_and_its_gradients(B, N, C, H, E, dtype, act):
    (x, dy, wg, wu, wd), offsets, e = block(B, N, C, H, E, dtype)
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    y = br.expert_ffn(x, offsets, wg, wu, wd, act, out=torch.full_like(x, 7.0))
    out = {"grad_x": torch.full_like(x, 7.0), **{k: torch.full_like(w, float("nan")) for k, w in (("grad_gate", wg), ("grad_up", wu), ("grad_down", wd))}}
    br.expert_ffn_grad(x, offsets, wg, wu, wd, dy, act, out=out)
    br.status()
    assert (y[e == E] == 7).all() and (out["grad_x"][e == E] == 7).all()
    for k in range(E):
        xk, dk, g, u, d = (t.double() for t in (x[e == k], dy[e == k], wg[k], wu[k], wd[k]))
        gate, up = xk @ g.t(), xk @ u.t()
        h, dh = gate * up, dk @ d
        for name, got, want in (("y", y[e == k], h @ d.t()), ("grad_x", out["grad_x"][e == k], (dh * up) @ g + (dh * gate) @ u),
                                ("grad_gate", out["grad_gate"][k], (dh * up).t() @ xk), ("grad_up", out["grad_up"][k], (dh * gate).t() @ xk),
                                ("grad_down", out["grad_down"][k], dk.t() @ h)):
            assert float(want.abs().max() if want.numel() else 0.0) < 2 ** 24
            assert torch.equal(got, want.to(dtype)), (name, k, int((got != want.to(dtype)).sum()))
    again = br.expert_ffn_grad(x, offsets, wg, wu, wd, dy, act, out={k: torch.full_like(v, 7.0) for k, v in out.items()})
    assert all(torch.equal(again[k], out[k]) for k in out)
    assert torch.equal(br.expert_ffn(x, offsets, wg, wu, wd, act, out=torch.full_like(x, 7.0)), y)
    br.close()


NORM = [(8, 40000, 64, 4), (4, 50000, 80, 3), (32, 5000, 256, 16), (3, 40000, 512, 2), (2, 40000, 1024, 3), (1, 400000, 20, 1), (2, 60000, 132, 2)]


@pytest.mark.parametrize("tx,ty", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)], ids=str)
@pytest.mark.parametrize("B,N,C,E", NORM)
def test_norm_gradients(B, N, C, E, tx, ty):
    """Statistics of 0 and 1, so that h is the row itself; for widths that are powers of two the means are exact too."""
    g = generator(N + C)
    offsets = ascending_offsets(B, N, E, seed=C)
    e = expert_of_rows(offsets, N, E)
    x, dy = whole(g, -2, 2, B, N, C).to(tx), whole(g, -2, 2, B, N, C).to(ty)
    x[e == E], dy[e == E] = float("nan"), float("nan")
    w = whole(g, 1, 3, E, C)
    mean, rstd = torch.zeros((B, N), device=DEV), torch.ones((B, N), device=DEV)
    br = handle(B, N, E)
    br.reserve_rows(C)
    out = {"grad_x": torch.full_like(x, 7.0), "grad_weight": torch.full_like(w, float("nan")), "grad_bias": torch.full_like(w, float("nan"))}
    br.expert_norm_grad(x, offsets, w, mean, rstd, dy, out=out)
    br.status()
    assert (out["grad_x"][e == E] == 7).all()
    u = torch.finfo(tx).eps / 2
    for k in range(E):
        xk, dk = x[e == k].double(), dy[e == k].double()
        assert torch.equal(out["grad_weight"][k].double(), (dk * xk).sum(0)), k
        assert torch.equal(out["grad_bias"][k].double(), dk.sum(0)), k
        gw = dk * w[k].double()
        a, c = gw.mean(-1, keepdim=True), (gw * xk).mean(-1, keepdim=True)
        want, got = gw - a - xk * c, out["grad_x"][e == k]
        if C & (C - 1) == 0 and tx != torch.float32:
            assert torch.equal(got, want.float().to(tx)), k
        else:
            # Sums of whole numbers are exact; 1 / C and the product with it, the product with h and two differences are roundings
            # of fp32 each.
            bound = 4 * 2.0 ** -24 * (gw.abs() + a.abs() + (xk * c).abs())
            assert ((got.double() - want).abs() <= bound * (1 + u) + u * 1.001 * want.abs()).all(), k
    again = br.expert_norm_grad(x, offsets, w, mean, rstd, dy, out={k: torch.full_like(v, 7.0) for k, v in out.items()})
    assert all(torch.equal(again[k], out[k]) for k in out)
    br.close()


@pytest.mark.parametrize("tx,ty", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16)], ids=str)
@pytest.mark.parametrize("B,N,C,E", NORM)
def test_norm(B, N, C, E, tx, ty):
    """A row of the large call has the bits that it has in a call of its own part of the rows (whose values test_gpu_rows checks)."""
    g = generator(N + C + 1)
    offsets = ascending_offsets(B, N, E, seed=C)
    e = expert_of_rows(offsets, N, E)
    x = (torch.randn((B, N, C), generator=g, device=DEV) * 2 + 0.5).to(tx)
    x[e == E] = float("nan")
    w, b = (torch.randn((E, C), generator=g, device=DEV) for _ in range(2))
    br = handle(B, N, E)
    new = lambda n: {"y": torch.full((B, n, C), 7.0, dtype=ty, device=DEV), "mean": torch.full((B, n), 7.0, device=DEV), "rstd": torch.full((B, n), 7.0, device=DEV)}
    out = br.expert_norm(x, offsets, w, b, out=new(N))
    br.status()
    for at in (0, N // 3, N - 97):
        part = slice(at, at + 97)
        few = br.expert_norm(x[:, part].clone(memory_format=torch.contiguous_format), (offsets - at).clamp(0, 97).contiguous(), w, b, out=new(97))
        for k in few:
            assert torch.equal(few[k], out[k][:, part]), (k, at)
    inside = e < E
    assert all((out[k][~inside] == 7).all() for k in out)
    xd = x[inside].double()
    m = xd.mean(-1)
    r = ((xd - m[:, None]).square().mean(-1) + 1e-5) ** -0.5
    # Means and variances of C values near 1 in fp32: C roundings each.
    assert ((out["mean"][inside].double() - m).abs() <= (C + 2) * 2.0 ** -24 * xd.abs().mean(-1)).all()
    assert ((out["rstd"][inside].double() / r - 1).abs() <= (C + 16) * 2.0 ** -22).all()
    br.close()


LENGTHS = {"random": lambda n, V, g: torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32),
           "one": lambda n, V, g: torch.full((n,), V - 1, dtype=torch.int32, device=DEV),
           "runs": lambda n, V, g: (torch.arange(n, device=DEV) * V // n).to(torch.int32),
           "uneven": lambda n, V, g: (torch.rand(n, generator=g, device=DEV) ** 6 * (V + 1) - 1).to(torch.int32).clamp(max=V - 1)}


@pytest.mark.parametrize("pattern", LENGTHS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,V,C", [(400000, 9000, 64), (700001, 37, 64), (450000, 20000, 80), (100000, 1500, 1024), (160000, 12, 516), (2600000, 500, 8)])
def test_lookup_gradient(n, V, C, dtype, pattern):
    """Two places of sixteen and more per group of lanes, with runs that go on from one to the next, over groups and over CTAs."""
    g = generator(n + C)
    ids = LENGTHS[pattern](n, V, g)
    dout = torch.randint(-3, 4, (n, C), generator=g, device=DEV, dtype=torch.int8).to(dtype)
    br = handle(1, n)
    br.reserve_rows(C)
    out = br.row_lookup_grad(ids, dout, V, out=torch.full((V, C), float("nan"), dtype=dtype, device=DEV))
    br.status()
    want = torch.zeros((V, C), device=DEV)
    keep = ids >= 0
    want.index_add_(0, ids[keep].long(), dout[keep].float())               # exact: whole numbers below 2^24
    assert torch.equal(out, want.to(dtype))
    br.close()
