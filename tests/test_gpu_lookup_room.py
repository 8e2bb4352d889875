"""The lookup's gradient on handles with room for more ids than the call has (needs a B200)."""
import pytest
import torch

from row_cases import handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("ids,reserved,n,C", [(100000, 1024, 75776, 1024), (160000, 128, 151552, 128), (310000, 64, 303104, 64), (310000, 64, 150000, 20)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_calls_smaller_than_the_handle(ids, reserved, n, C, dtype):
    """Tables of few rows, so that every CTA's ends divide a run, at sizes whose parts are more than those of the handle's own."""
    V = 5
    br = handle(1, ids)
    br.reserve_rows(reserved)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    at = torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32)
    dout = torch.randn((n, C), generator=g, device=DEV).to(dtype)
    out = torch.full((V, C), float("nan"), dtype=dtype, device=DEV)
    br.row_lookup_grad(at, dout, V, out=out)
    br.status()
    keep = at >= 0
    want, size = (torch.zeros((V, C), dtype=torch.float64, device=DEV) for _ in range(2))
    want.index_add_(0, at[keep].long(), dout[keep].double())
    size.index_add_(0, at[keep].long(), dout[keep].double().abs())
    times = torch.bincount(at[keep].long(), minlength=V)[:, None]
    # A fp32 sum of n terms is off by n u32 of their sizes at most, its rounding by half a step.
    tol = (times + 1) * 2.0 ** -24 * size * 1.01 + unit(dtype) * 1.01 * want.abs()
    assert ((out.double() - want).abs() <= tol).all()
    br.close()
