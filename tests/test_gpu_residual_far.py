"""The residual and its gradients on rows behind 4 GB and behind 2^31 elements of each buffer (needs a B200)."""
import pytest
import torch

from residual_cases import PARAMS, forward, gradients
from row_cases import handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("C", [1024, 1020])
def test_rows_behind_four_gigabytes(C):
    """Zeros but for a few rows at both ends and in the middle; two experts, the second from the middle rows on."""
    N, E = 2_200_000, 2
    rows = torch.cat([torch.arange(3), torch.arange(2_097_150, 2_097_156), torch.arange(N - 3, N)]).to(DEV)
    mid = 2_097_153
    g = torch.Generator(device=DEV)
    g.manual_seed(C)
    br = handle(1, N, E)
    br.reserve_rows(C)
    offsets = torch.tensor([[0, mid, N]], dtype=torch.int32, device=DEV)

    def few():
        t = torch.zeros((1, N, C), dtype=torch.bfloat16, device=DEV)
        t[0, rows] = torch.randn((len(rows), C), generator=g, device=DEV).bfloat16()
        return t

    x, f = few(), few()
    params = {k: 1 + 0.1 * torch.randn((E, C), generator=g, device=DEV) for k in PARAMS}
    made = br.expert_residual(x, f, offsets, **params)
    at = torch.tensor([[0, int((rows < mid).sum()), len(rows)]], dtype=torch.int32, device=DEV)
    ref = forward(x[:, rows], f[:, rows], at, E, None, params, 1e-5, None, 0.0)
    for name, (want, bound) in ref.items():
        if name == "y":
            bound = bound + unit(torch.bfloat16) * 1.02 * want.abs() + 1e-37
        assert ((made[name][:, rows].double() - want).abs() <= bound).all(), name
    grad_out, grad_y = few(), few()
    back = {k: v for k, v in params.items() if k != "pre_bias"}
    got = br.expert_residual_grad(made["out"], f, offsets, made["stats"], grad_out, grad_y, **back)
    ref = gradients(made["out"][:, rows], f[:, rows], at, E, made["stats"][:, rows], grad_out[:, rows], grad_y[:, rows], None, params, None, 0.0)
    for name, (want, bound) in ref.items():
        if name == "grad_gate":
            continue
        value = got[name][:, rows] if name in ("grad_x", "grad_f") else got[name]      # rows whose gradients from behind are zeros add nothing
        assert ((value.double() - want).abs() <= bound + 1e-37).all(), name
    assert int(got["grad_x"].count_nonzero()) == int(got["grad_x"][:, rows].count_nonzero())
    br.status()
    br.close()
