"""The first CUDA call of a host thread can be any call of the library (needs a B200)."""
import threading

import pytest
import torch

import paper_2507_04123_b200 as pkg
from row_cases import handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("name", ["expert_ffn", "expert_ffn_grad", "expert_norm", "row_lookup", "row_lookup_grad"])
def test_on_a_thread_without_a_context(name):
    N, C, H = 200, 64, 72
    br = handle(1, N, 1)
    br.reserve_rows(C, H)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x, dy, wg, wu, wd = (torch.randn(s, generator=g, device=DEV).bfloat16() for s in ((1, N, C), (1, N, C), (1, H, C), (1, H, C), (1, C, H)))
    weight = torch.ones((1, C), device=DEV)
    ids = torch.arange(N, dtype=torch.int32, device=DEV) % 7
    out = [torch.zeros_like(t) for t in (x, wg, wu, wd)]
    p = [t.data_ptr() for t in out]
    kind, lib = pkg.bridge.ROW_TYPES[x.dtype], pkg.load_library()
    calls = {
        "expert_ffn": lambda: lib.emc2_expert_ffn(br._h, 1, N, C, H, kind, 0, x.data_ptr(), None, wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), p[0], None),
        "expert_ffn_grad": lambda: lib.emc2_expert_ffn_grad(br._h, 1, N, C, H, kind, 0, x.data_ptr(), None, wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), dy.data_ptr(), *p, None),
        "expert_norm": lambda: lib.emc2_expert_norm(br._h, 1, N, C, kind, kind, x.data_ptr(), None, weight.data_ptr(), None, 1e-5, p[0], None, None, None),
        "row_lookup": lambda: lib.emc2_row_lookup(br._h, N, N, C, kind, ids.data_ptr(), x.data_ptr(), 1.0, p[0], None),
        "row_lookup_grad": lambda: lib.emc2_row_lookup_grad(br._h, N, N, C, kind, ids.data_ptr(), dy.data_ptr(), 1.0, p[0], None)}
    torch.cuda.synchronize()
    rc = []
    thread = threading.Thread(target=lambda: rc.append(calls[name]()))
    thread.start()
    thread.join()
    assert rc == [0], lib.emc2_bridge_last_cuda_error(br._h)
    br.status()
    first = [t.clone() for t in out]
    assert calls[name]() == 0                                              # the same from this thread
    br.status()
    assert all(torch.equal(a, b) for a, b in zip(out, first)) and bool(first[0].any())
    br.close()
