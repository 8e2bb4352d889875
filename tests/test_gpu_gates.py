"""The activation of the feed-forward block alone, at gates from far below zero to far above (needs a B200).

The weights pass single values on: the gate is the row's second value, u is 1, and every output is one hidden value, so that
the result is act(gate) rounded once to the type, and the gradients are act(gate) and act'(gate).

Bounds.  SiLU takes 1 / (1 + exp(-g)) from a fast power of two and a fast reciprocal: the argument is off by |g| (2^-24 + 2^-26)
(a product, and log2 e in fp32), the power by 2^-22, the reciprocal by 2^-23, five sums and products by 2^-24 each: all of itself, less
than |g| 2^-23 + 2^-20 together.  Gates below -41.5 count as -41.5, where act(g) is less than 2^-54.  GELU takes the normal
distribution from a formula that is off by 0.75e-7, which fp32 arithmetic makes 2^-22 more; the density is off by g^2 2^-23 + 2^-21 of
itself.  Beside that: half a step of the type."""
import pytest
import torch

from row_cases import handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 2.0 ** -54

SHAPES = [(64, 200), (64, 20000), (80, 30000), (128, 300), (128, 21000), (256, 500)]          # channels, rows
TYPES = [torch.bfloat16, torch.float16]


def gates(dtype):
    far = [-100.0, -3000.0, -60000.0, 60000.0] + ([-1e12, -1e20, -1e30, 1e20] if dtype == torch.bfloat16 else [])
    near = torch.linspace(-45.0, 16.0, 245, dtype=torch.float64)
    return torch.cat([near, torch.tensor(far + [0.0, -0.0, -41.5, -42.0, -1.28, -4.0, -6.0, -8.0, -10.0, -16.0], dtype=torch.float64)]).to(dtype).to(DEV)


def exact(g, act):
    """act(g), act'(g) in 64 bits and the bounds of their errors before rounding."""
    g = g.double()
    near = g.clamp(-700.0, 700.0)                                          # exp(-g) stays finite
    if act == "silu":
        s = 1 / (1 + torch.exp(-near))
        a, da = g * s, s * (1 + near * (1 - s))
        rel = near.abs().clamp(max=45.0) * 2.0 ** -23 + 2.0 ** -20
        return a, da, rel * a.abs() + FAR, 2 * rel * (s + a.abs() * (1 - s)) + FAR
    phi = 0.5 * torch.erfc(-near * 0.5 ** 0.5)
    density = torch.exp(-near * near / 2) / (2 * torch.pi) ** 0.5
    off = 0.75e-7 + 2.0 ** -22
    # Far gates come from outside the formula's reach, where the distribution is 0 or 1.
    size = torch.where(g.abs() > 40.0, 0.0, g.abs())
    return g * phi, phi + g * density, off * size + 2.0 ** -22 * (g * phi).abs(), off + (near * near * 2.0 ** -23 + 2.0 ** -21) * (g * density).abs()


def rounded(v, err, dtype):
    """Bound of the error of v, known to err, after one rounding to the type."""
    half = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    return err * (1 + unit(dtype)) + unit(dtype) * 1.001 * v.abs() + half


def check(got, want, bound, g, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), [(float(a), float(b), float(c)) for a, b, c in zip(g.expand_as(bad)[bad][:5], got[bad][:5], want.expand_as(bad)[bad][:5])])


def rows_of(g, N, C, dtype):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(N)
    x = torch.randn((1, N, C), generator=gen, device=DEV).to(dtype)       # the rest of the row meets weights of zero
    x[..., 0], x[..., 1] = 1.0, g
    return x


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("C,N", SHAPES)
def test_act_of_every_gate(C, N, dtype, act):
    H = 72
    some = gates(dtype)
    g = some[torch.arange(N, device=DEV) % len(some)]
    x = rows_of(g, N, C, dtype)
    wg, wu, wd = (torch.zeros(s, dtype=dtype, device=DEV) for s in ((1, H, C), (1, H, C), (1, C, H)))
    wg[0, :, 1], wu[0, :, 0] = 1.0, 1.0
    at = torch.arange(C, device=DEV)
    wd[0, at, at % H] = 1.0
    br = handle(1, N, 1)
    y = br.expert_ffn(x, None, wg, wu, wd, act)
    br.status()
    br.close()
    want, _, err, _ = exact(g, act)
    check(y[0], want[:, None], rounded(want, err, dtype)[:, None], g[:, None], "y")


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("C,N", SHAPES)
def test_gradients_at_every_gate(C, N, dtype, act):
    """One hidden unit at work: dx holds act'(gate) and act(gate), the weights' gradients their sums over the rows of each
    expert, whose rows have all the same gate."""
    H, E = 72, 16
    some = gates(dtype)
    some = some[some.abs() < (1e4 if dtype == torch.float16 else 1e25)]          # so that the sums below hold their squares
    turns = range(0, len(some), E) if N < 1000 else [len(some) - E]        # large calls: another form of the kernels, some gates
    for turn in turns:
        mine = some[(turn + torch.arange(E, device=DEV)) % len(some)]
        e = torch.arange(N, device=DEV) * E // N
        ends = torch.searchsorted(e, torch.arange(E + 1, device=DEV)).to(torch.int32)[None].contiguous()
        g = mine[e]
        x = rows_of(g, N, C, dtype)
        dy = torch.zeros_like(x)
        dy[..., 0] = 1.0
        wg, wu, wd = (torch.zeros(s, dtype=dtype, device=DEV) for s in ((E, H, C), (E, H, C), (E, C, H)))
        wg[:, 5, 1], wu[:, 5, 0], wd[:, 0, 5] = 1.0, 1.0, 1.0
        br = handle(1, N, E)
        br.reserve_rows(C, H)
        out = br.expert_ffn_grad(x, ends, wg, wu, wd, dy, act)
        br.status()
        br.close()
        a, da, err_a, err_da = exact(g, act)
        check(out["grad_x"][0, :, 1], da, rounded(da, err_da, dtype), g, "dx, act'")
        check(out["grad_x"][0, :, 0], a, rounded(a, err_a, dtype), g, "dx, act")
        # Sums of n equal terms, each rounded; a fp32 sum on the tensor cores is off by 4 * 2^-24 per term.
        n = torch.bincount(e, minlength=E).double()
        a, da, err_a, err_da = exact(mine, act)
        for name, one, err, times in (("grad_up", a, err_a, torch.ones_like(a)), ("grad_gate", da, err_da, mine.double())):
            total, each = n * one * times, rounded(one, err, dtype)
            bound = n * times.abs() * (each + 4 * (n + 700) * 2.0 ** -24 * (one.abs() + each))
            got = out[name][:, 5, 0 if name == "grad_up" else 1]
            check(got, total, rounded(total, bound, dtype), mine, name)
        each = rounded(a, err_a, dtype)
        check(out["grad_down"][:, 0, 5], n * a, rounded(n * a, n * (each + 4 * (n + 700) * 2.0 ** -24 * (a.abs() + each)), dtype), mine, "grad_down")


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_gate_that_is_no_number_reaches_the_result(dtype, act):
    C, H, N = 64, 72, 130
    x = rows_of(torch.ones(N, dtype=dtype, device=DEV), N, C, dtype)
    wg, wu, wd = (torch.zeros(s, dtype=dtype, device=DEV) for s in ((1, H, C), (1, H, C), (1, C, H)))
    wg[0, 3, 1], wu[0, :, 0], wd[0, :, 3] = float("nan"), 1.0, 1.0         # u of that unit is 1
    br = handle(1, N, 1)
    assert br.expert_ffn(x, None, wg, wu, wd, act).isnan().all()
    br.status()
    br.close()
