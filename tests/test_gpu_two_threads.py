"""Two host threads, a handle and a stream each, in the same call with different widths: no call is refused because the other
thread set up the same kernel for its own size in between (needs a B200)."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2507_04123_b200 as pkg
from row_cases import handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TESTS = os.path.dirname(os.path.abspath(__file__))
TIMES = 20000
vp, i32 = ctypes.c_void_p, ctypes.c_int32


def fields(*groups):
    return [(n, t) for t, names in groups for n in names.split()]


class FfnCall(ctypes.Structure):
    _fields_ = fields((vp, "bridge"), (i32, "B N channels hidden type act"), (vp, "x offsets gate up down y stream"))


class NormGradCall(ctypes.Structure):
    _fields_ = fields((vp, "bridge"), (i32, "B N channels type_x type_y"), (vp, "x offsets weight mean rstd dy dx dweight dbias stream"))


class LookupGradCall(ctypes.Structure):
    _fields_ = fields((vp, "bridge"), (i32, "n rows channels type"), (vp, "ids dout"), (ctypes.c_float, "scale"), (vp, "dtable stream"))


@pytest.fixture(scope="module")
def threads(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("threads") / "libthreads.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-pthread", "-fPIC", "-shared", "-o", lib, os.path.join(TESTS, "two_threads_shim.cpp")], check=True)
    return ctypes.CDLL(lib)


@pytest.fixture
def pair():
    """Handles with scratch and their streams."""
    handles = [handle(1, 300, 1) for _ in range(2)]
    for br in handles:
        br.reserve_rows(1024, 64)
    yield list(zip(handles, [torch.cuda.Stream() for _ in handles]))
    torch.cuda.synchronize()
    for br in handles:
        br.status()
        br.close()


def run(shim, call, calls):
    torch.cuda.synchronize()
    array = (type(calls[0]) * 2)(*calls)
    rc = shim(ctypes.cast(call, vp), array, TIMES)
    assert rc == 0, [pkg.load_library().emc2_bridge_last_cuda_error(c.bridge) for c in calls]
    torch.cuda.synchronize()


def test_feed_forward_block(threads, pair):
    N, H = 130, 32
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    keep, calls = [], []
    for (br, stream), C in zip(pair, (104, 256)):
        x, wg, wu, wd = ((torch.randn(s, generator=g, device=DEV) * 0.2).bfloat16() for s in ((1, N, C), (1, H, C), (1, H, C), (1, C, H)))
        y = torch.zeros_like(x)
        keep.append((br, y, (x, None, wg, wu, wd)))
        calls.append(FfnCall(br._h, 1, N, C, H, pkg.bridge.ROW_TYPES[x.dtype], 0, x.data_ptr(), None, wg.data_ptr(), wu.data_ptr(), wd.data_ptr(), y.data_ptr(), stream.cuda_stream))
    run(threads.two_ffn, pkg.load_library().emc2_expert_ffn, calls)
    for br, y, args in keep:
        assert torch.equal(y, br.expert_ffn(*args))


def test_norm_gradients(threads, pair):
    N = 130
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    keep, calls = [], []
    for (br, stream), C in zip(pair, (904, 1024)):
        x, dy = (torch.randn((1, N, C), generator=g, device=DEV) for _ in range(2))
        w = torch.ones((1, C), device=DEV)
        f = br.expert_norm(x, None, w)
        dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)
        keep.append((br, (dx, dw, db), (x, None, w, f["mean"], f["rstd"], dy)))
        calls.append(NormGradCall(br._h, 1, N, C, 0, 0, x.data_ptr(), None, w.data_ptr(), f["mean"].data_ptr(), f["rstd"].data_ptr(), dy.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
                                  stream.cuda_stream))
    run(threads.two_norm_grad, pkg.load_library().emc2_expert_norm_grad, calls)
    for br, got, args in keep:
        want = br.expert_norm_grad(*args)
        assert all(torch.equal(a, want[k]) for a, k in zip(got, ("grad_x", "grad_weight", "grad_bias")))


def test_lookup_gradient(threads, pair):
    n, V = 300, 40
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    keep, calls = [], []
    for (br, stream), C in zip(pair, (904, 1024)):
        ids = torch.randint(-1, V, (n,), generator=g, device=DEV, dtype=torch.int32)
        dout = torch.randn((n, C), generator=g, device=DEV)
        dtable = torch.zeros((V, C), device=DEV)
        keep.append((br, dtable, (ids, dout, V)))
        calls.append(LookupGradCall(br._h, n, V, C, 0, ids.data_ptr(), dout.data_ptr(), 1.0, dtable.data_ptr(), stream.cuda_stream))
    run(threads.two_lookup_grad, pkg.load_library().emc2_row_lookup_grad, calls)
    for br, got, args in keep:
        assert torch.equal(got, br.row_lookup_grad(*args))
