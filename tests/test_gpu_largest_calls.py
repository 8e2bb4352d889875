"""The largest calls that the header allows: quantisation of 2^29 blocks, and a layer of 256 experts of 8,192 units (needs a B200)."""
import pytest
import torch

from layer_cases import layer, quantised
from row_cases import handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_quantisation_of_as_many_blocks_as_there_may_be():
    rows, C = 2 ** 21, 8192
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    br = handle(1, 8)
    x = torch.zeros((rows, C), dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 2 ** 18 - 1, 2 ** 19, 2 ** 20, rows - 1], device=DEV)
    x[at] = torch.randn((len(at), C), generator=g, device=DEV).bfloat16()
    got = br.mx4_quantise(x)
    codes, scales, _ = quantised(x[at])
    assert torch.equal(got["codes"][at].int(), codes.int()) and torch.equal(got["scales"][at].int(), scales.int())
    some = slice(rows - 4096, rows - 1)
    assert not got["codes"][some].any() and not got["scales"][some].any()
    with pytest.raises(Exception, match="emc2_mx4_quantise"):
        br.mx4_quantise(torch.empty((rows + 1, 8192), dtype=torch.bfloat16, device=DEV))
    br.close()


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
def test_layer_of_many_wide_experts(form):
    n, C, H, E, k = 128, 1024, 8192, 256, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x = torch.randn((n, C), generator=g, device=DEV).bfloat16()
    wr = torch.randn((E, C), generator=g, device=DEV) * 2 * C ** -0.5
    ws = []
    for shape in ((H, C), (H, C), (C, H)):
        w = torch.empty((E, *shape), dtype=torch.bfloat16, device=DEV)
        for e in range(E):
            w[e] = torch.randn(shape, generator=g, device=DEV) * shape[1] ** -0.5
        ws.append(w if form == "16 bits" else br.mx4_quantise(w))
        del w
    got = br.expert_layer(x, wr, *ws, k)
    ids, (p, err_p), (y, err) = layer(x, wr, None, *ws, k, "silu")
    assert torch.equal(got["ids"].long(), ids) and int(got["ids"].max()) > 250
    assert ((got["weights"].double() - p).abs() <= err_p).all()
    assert ((got["y"].double() - y).abs() <= err).all()
    br.status()
    br.close()
