"""The residual's gradients on memory that begins 16 bytes behind a boundary of 32, buffer by buffer (needs a B200)."""
import pytest
import torch

from residual_cases import PARAMS, gradients, kept
from row_cases import expert_of_rows, handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BUFFERS = ("rows", "f", "grad_out", "grad_y", "stats", "grad_x", "grad_f", "all")


def shifted(t):
    """The same values 16 bytes behind the allocator's boundary."""
    more = 16 // t.element_size()
    room = torch.empty(t.numel() + more, dtype=t.dtype, device=t.device)
    at = room[more:].view(t.shape)
    at.copy_(t)
    return at


@pytest.mark.parametrize("which", BUFFERS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("C", [8, 64, 264, 772, 1024])
def test_gradients_on_shifted_memory(C, dtype, which):
    g = torch.Generator(device=DEV)
    g.manual_seed(C)
    B, N, E, p = 2, 203, 3, 0.2
    rand = lambda *s: torch.randn(s, generator=g, device=DEV)               # noqa: E731
    br = handle(B, N, E)
    br.reserve_rows(C)
    offsets = torch.tensor([[0, 50, 50, 190], [3, 100, 150, N]], dtype=torch.int32, device=DEV)
    x, f, grad_out, grad_y = (rand(B, N, C).to(dtype) for _ in range(4))
    params = {k: 1 + 0.1 * rand(E, C) for k in PARAMS}
    gate, seed = torch.rand((B, N), generator=g, device=DEV), torch.tensor([4, 2], dtype=torch.int64, device=DEV)
    keep = kept((4, 2), B * N, C, p).view(B, N, C).to(DEV)
    made = br.expert_residual(x, f, offsets, gate=gate, **params, p=p, seed=seed)
    t = {"rows": made["out"], "f": f, "grad_out": grad_out, "grad_y": grad_y, "stats": made["stats"], "grad_x": torch.zeros_like(x), "grad_f": torch.zeros_like(f)}
    inside = expert_of_rows(offsets, N, E) < E
    t["stats"][~inside] = float("nan")
    at = {k: shifted(v) if which in (k, "all") else v for k, v in t.items()}
    out = {"grad_x": at["grad_x"], "grad_f": at["grad_f"], "grad_gate": torch.zeros_like(gate), **{"grad_" + k: torch.zeros((E, C), device=DEV) for k in PARAMS}}
    back = {k: v for k, v in params.items() if k != "pre_bias"}
    br.expert_residual_grad(at["rows"], at["f"], offsets, at["stats"], at["grad_out"], at["grad_y"], gate=gate, **back, p=p, seed=seed, out=out)
    for name, (want, bound) in gradients(t["rows"], f, offsets, E, t["stats"], grad_out, grad_y, gate, params, keep, p).items():
        rows = inside if name in ("grad_x", "grad_f", "grad_gate") else slice(None)
        assert ((out[name].double() - want).abs() <= bound + 1e-37)[rows].all(), name
    br.status()
    br.close()
