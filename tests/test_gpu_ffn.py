"""The experts' gated feed-forward block and its gradients against the formulas in 64 bits (needs a B200)."""
import pytest
import torch

from row_cases import ascending_offsets, expert_of_rows, ffn_reference, handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

SHAPES = [(1, 1, 8, 8, 1), (1, 128, 64, 64, 1), (1, 129, 64, 256, 4), (3, 300, 80, 320, 4), (2, 500, 128, 96, 3), (2, 260, 136, 40, 2),
          (1, 400, 256, 1024, 5), (32, 40, 24, 72, 16), (1, 3000, 72, 200, 2), (2, 700, 200, 136, 3), (1, 513, 192, 64, 1), (1, 37, 16, 2048, 1),
          (1, 300, 48, 128, 2), (2, 150, 40, 384, 3), (1, 200, 104, 64, 1), (1, 300, 176, 72, 2), (1, 140, 240, 96, 1), (1, 60, 112, 2048, 1)]


def inputs(B, N, C, H, E, dtype, seed=0, rows=lambda offsets, N: offsets):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + B * N + C)
    offsets = rows(ascending_offsets(B, N, E, seed=N + seed), N).to(torch.int32).contiguous()
    e = expert_of_rows(offsets, N, E)
    x, dy = (torch.randn((B, N, C), generator=g, device=DEV).to(dtype) for _ in range(2))
    x[e == E], dy[e == E] = float("nan"), float("inf")                     # rows of no expert reach nothing
    ws = [(torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)
          for shape, scale in (((E, H, C), C ** -0.5), ((E, H, C), C ** -0.5), ((E, C, H), H ** -0.5))]
    return x, dy, offsets, e, ws


def close(got, ref, where):
    want, bound = ref
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (where, int(bad.sum()), float((got.double() - want).abs().max()), float(bound.max()))


@pytest.mark.parametrize("reserved", [False, True])           # with scratch, few rows are shared out by hidden units
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("B,N,C,H,E", SHAPES + [(1, 20000, 120, 72, 2), (1, 21000, 96, 200, 3)])
def test_ffn(B, N, C, H, E, dtype, act, reserved):
    x, _, offsets, e, (wg, wu, wd) = inputs(B, N, C, H, E, dtype)
    br = handle(B, N, E)
    if reserved:
        br.reserve_rows(C, H)
    y = torch.full_like(x, 7.0)
    br.expert_ffn(x, offsets, wg, wu, wd, act, out=y)
    br.status()
    assert (y[e == E] == 7).all()
    for k in range(E):
        close(y[e == k], ffn_reference(x[e == k], wg[k], wu[k], wd[k], act)["y"], k)
    again = br.expert_ffn(x, offsets, wg, wu, wd, act)
    assert torch.equal(again[e < E], y[e < E])
    br.close()


def spread(offsets, N):
    return offsets


def few(offsets, N):
    """Almost every row belongs to no expert."""
    return torch.clamp(offsets - (N - 5), min=0) + 3 * (N > 200)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("B,N,C,H,E,rows", [(*shape, spread) for shape in SHAPES] + [(3, 5000, 64, 96, 3, few), (2, 9000, 200, 72, 2, few)])
def test_ffn_gradients(B, N, C, H, E, rows, dtype, act):
    x, dy, offsets, e, (wg, wu, wd) = inputs(B, N, C, H, E, dtype, rows=rows)
    br = handle(B, N, E)
    br.reserve_rows(C, H)
    out = {"grad_x": torch.full_like(x, 7.0), **{k: torch.full_like(w, float("nan")) for k, w in (("grad_gate", wg), ("grad_up", wu), ("grad_down", wd))}}
    br.expert_ffn_grad(x, offsets, wg, wu, wd, dy, act, out=out)
    br.status()
    assert (out["grad_x"][e == E] == 7).all()
    for k in range(E):
        ref = ffn_reference(x[e == k], wg[k], wu[k], wd[k], act, dy[e == k])
        close(out["grad_x"][e == k], ref["grad_x"], ("grad_x", k))
        for name in ("grad_gate", "grad_up", "grad_down"):
            close(out[name][k], ref[name], (name, k))
    again = br.expert_ffn_grad(x, offsets, wg, wu, wd, dy, act)
    for name in ("grad_gate", "grad_up", "grad_down"):
        assert torch.equal(again[name], out[name])
    br.close()
