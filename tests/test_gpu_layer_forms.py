"""The layer for few rows in the forms that its plan takes for wide layers, and the rows in use of calls of one and two rows (needs a B200).

A warp has a tile of weights to itself where the CTAs fill the SMs, with several steps of the products, whole and ragged; twice the CTAs where they
take a few waves; several passes where an expert has many rows; shares of the hidden units of several steps, the last without any."""
import pytest
import torch

import paper_2507_04123_b200 as pkg
from layer_cases import layer
from row_cases import handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def problem(seed, n, C, H, E, dtype, form, br):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x, wr = rand(g, n, C, dtype=dtype), rand(g, E, C, scale=2 * C ** -0.5)
    ws = [rand(g, E, H, C, scale=C ** -0.5), rand(g, E, H, C, scale=C ** -0.5), rand(g, E, C, H, scale=H ** -0.5)]
    return x, wr, [w.to(dtype) if form == "16 bits" else br.mx4_quantise(w) for w in ws]


def check(got, want, rows=slice(None)):
    ids, (p, err_p), (y, err) = want
    assert torch.equal(got["ids"][rows].long(), ids)
    assert ((got["weights"][rows].double() - p).abs() <= err_p).all()
    off = (got["y"][rows].double() - y).abs()
    assert (off <= err).all(), float((off / err).max())


# On 148 SMs.  (128, 520, 2056, 16, 4): 272 CTAs of first products, nine steps of 64 or three of 256; four shares of the last, one of them without
# units; 32 rows per expert on average.  (128 and 20, 776, 2568, 32, 4): 672 CTAs, in 16 bits taken as 1,344; (96, 328, 2568, 32, 4): not.
# (128, 1024, 1288, 40, 3): 160 CTAs of last products, all hidden units in one.  (128, 264, 8192, 2, 2): 128 rows per expert in shared passes, eight shares.
# (5, 1000, 4104, 30, 8): few rows of each expert, filled SMs.
SHAPES = [(128, 1024, 2048, 32, 4), (128, 520, 2056, 16, 4), (128, 776, 2568, 32, 4), (20, 776, 2568, 32, 4), (128, 1024, 1288, 40, 3), (128, 264, 8192, 2, 2), (5, 1000, 4104, 30, 8), (96, 328, 2568, 32, 4)]


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.float16, "gelu")], ids=str)
@pytest.mark.parametrize("n,C,H,E,k", SHAPES)
def test_wide_layers(n, C, H, E, k, dtype, act, form):
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, ws = problem(n + H, n, C, H, E, dtype, form, br)
    got = br.expert_layer(x, wr, *ws, k, act)
    check(got, layer(x, wr, None, *ws, k, act))
    again = br.expert_layer(x, wr, *ws, k, act)
    assert all(torch.equal(again[i], got[i]) for i in got)
    br.status()
    br.close()


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
@pytest.mark.parametrize("n", [1, 2])
def test_rows_in_use_of_small_calls(n, form):
    """Counts of none, of all, and counts that are none, each before a full call on the same handle."""
    C, H, E, k = 72, 136, 6, 3
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, ws = problem(n, n, C, H, E, torch.bfloat16, form, br)
    full = br.expert_layer(x, wr, *ws, k)
    check(full, layer(x, wr, None, *ws, k, "silu"))
    for used in (n, 0, -3, n + 1, 1):
        real = min(max(used, 0), n)
        v = x.clone()
        v[real:] = float("nan")
        out = {"y": torch.full_like(x, 7.0), "ids": torch.full((n, k), 77, dtype=torch.int32, device=DEV), "weights": torch.full((n, k), 7.0, device=DEV)}
        br.expert_layer(v, wr, *ws, k, count=torch.tensor([used], dtype=torch.int32, device=DEV), out=out)
        if real:
            check(out, layer(x[:real], wr, None, *ws, k, "silu"), slice(0, real))
        assert (out["y"][real:] == 7).all() and (out["ids"][real:] == 77).all() and (out["weights"][real:] == 7).all()
        assert br.status(raise_on_error=False) == (0 if used == real else pkg.bridge.EMC2_ERR_INVALID_ARG)
        again = br.expert_layer(x, wr, *ws, k)
        assert all(torch.equal(again[i], full[i]) for i in full)
    br.close()


@pytest.mark.parametrize("n", [1, 2])
def test_a_captured_call_with_another_count(n):
    C, H, E, k = 256, 1024, 16, 2
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, ws = problem(n, n, C, H, E, torch.bfloat16, "16 bits", br)
    count, out = torch.tensor([n], dtype=torch.int32, device=DEV), br.expert_layer(x, wr, *ws, k)
    want = {i: t.clone() for i, t in out.items()}
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(2):                                                  # one call behind another
            br.expert_layer(x, wr, *ws, k, count=count, out=out)
    for used in (n, 0, n, 1, 0, 0, n):
        count.fill_(used)
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for i in out:
            assert (out[i][used:] == 0).all()
            assert torch.equal(out[i][:used], want[i][:used]) if used == n else torch.isfinite(out[i]).all()
    br.status()
    del graph
    br.close()
