"""How many bits the layer for few rows keeps between its products, whatever the number of rows of an expert (needs a B200).

All hidden units of the expert are alike and the gate's and the up projection's sums are whole numbers of 2^-5, exact in fp32, so that
a result is a hidden value times a whole number: its error is what the hidden value lost, and half a step of the type.

Bounds.  act(g): an exponential and a quotient, 2^-20 of itself; the normal distribution's argument is off by two roundings, which move it
by g^2 2^-23 of itself.  The product with u: 2^-24.  The hidden value as the sum of two numbers of the type: what the second rounding leaves,
unit^2 of it, or half of the type's smallest number.  A sum of H products on the tensor cores: 2^-22 a term, as elsewhere."""
import pytest
import torch

from layer_cases import SIZES
from row_cases import activation, handle, unit

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.bfloat16, "gelu"), (torch.float16, "silu")], ids=str)
@pytest.mark.parametrize("n", [1, 15, 16, 17, 24, 25, 32, 33, 128])
def test_hidden_values_between_the_products(n, dtype, act, form):
    C, H = 16, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    sizes = torch.tensor(SIZES[1:], device=DEV)

    def elements(*shape):
        """Elements of the 4-bit form, the first of a row the largest, so that the power of its blocks is 1."""
        w = sizes[torch.randint(0, 7, shape, generator=g, device=DEV)]
        w[..., 0] = 6.0
        return w

    x = torch.randint(-3, 4, (n, C), generator=g, device=DEV).to(dtype)
    sign = torch.where(torch.rand((2, C), generator=g, device=DEV) < 0.5, -1.0, 1.0)
    wg, wu = (elements(C) * s / 16.0 for s in sign)
    wd = elements(C)
    ws = [wg.expand(1, H, C), wu.expand(1, H, C), wd[None, :, None].expand(1, C, H)]
    br = handle(1, 8)
    br.reserve_rows(C, H)
    given = [w.to(dtype).contiguous() if form == "16 bits" else br.mx4_quantise(w.contiguous()) for w in ws]
    if form == "4 bits":                                                   # as they are
        for w, q in zip(ws, given):
            values = br.mx4_quantise(w.contiguous(), out={"values": torch.empty_like(w, memory_format=torch.contiguous_format)})["values"]
            assert torch.equal(values, w)
    y = br.expert_layer(x, torch.zeros((1, C), device=DEV), *given, 1, act)["y"]
    gate, up = x.double() @ wg.double(), x.double() @ wu.double()
    a = activation(gate, act)[0]
    h = a * up
    err = (2.0 ** -20 + gate * gate * 2.0 ** -23 + 2.0 ** -24 + unit(dtype) ** 2 * 1.01 + (H + 16) * 2.0 ** -22) * h.abs()
    err = err + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    want = H * h[:, None] * wd.double()
    bound = H * err[:, None] * wd.double() * (1 + unit(dtype)) + unit(dtype) * 1.001 * want.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    off = (y.double() - want).abs()
    assert (off <= bound).all(), (float((off / bound).max()), int((off > bound).sum()))
    br.status()
    br.close()
