"""Residual, dropout, 4-bit weights and the layer: offsets behind 32 bits, many segments and passes, two handles on two host threads
(needs a B200)."""
import threading

import numpy as np
import pytest
import torch

from layer_cases import layer, quantised
from residual_cases import forward, gradients, kept, philox, threshold
from row_cases import expert_of_rows, handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def test_dropout_of_rows_behind_four_gigabytes():
    n, C, p = 5_000_000, 1024, 0.5
    br = handle(1, n)
    x = torch.ones((n, C), dtype=torch.bfloat16, device=DEV)
    seed = torch.tensor([3, 9], dtype=torch.int64, device=DEV)
    out = br.row_dropout(x, p, seed)
    for row in (0, 2 ** 21, n - 1):
        group = np.arange(C // 8)
        words = philox([np.full(C // 8, row), group, np.full(C // 8, 9), np.zeros(C // 8)], (3, 0))
        bits = np.stack([(w >> np.uint64(16 * half)) & np.uint64(0xFFFF) for w in words for half in (0, 1)], -1).reshape(C)
        want = torch.from_numpy(bits >= threshold(p)).to(DEV)
        assert torch.equal(out[row] != 0, want), row
    br.close()


def test_quantisation_of_rows_behind_four_gigabytes():
    g = generator(1)
    rows, C = 700_000, 8192
    br = handle(1, 8)
    x = torch.zeros((rows, C), dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 262144, 262145, rows - 1], device=DEV)
    x[at] = rand(g, 4, C, dtype=torch.bfloat16)
    got = br.mx4_quantise(x, out={"codes": torch.empty((rows, C // 2), dtype=torch.uint8, device=DEV), "scales": torch.empty((rows, C // 32), dtype=torch.uint8, device=DEV),
                                  "values": torch.empty_like(x)})
    codes, scales, values = quantised(x[at])
    assert torch.equal(got["codes"][at].int(), codes.int()) and torch.equal(got["scales"][at].int(), scales.int())
    assert torch.equal(got["values"][at].double(), values)
    assert int(got["codes"].count_nonzero()) == int(codes.count_nonzero())
    br.close()


@pytest.mark.parametrize("C", [8, 64, 80, 88, 136, 256, 264, 20, 132])
def test_residual_of_many_short_segments(C):
    """Frames and experts of a few rows each, so that the rows that a warp has side by side lie in several frames; several runs per CTA."""
    g = generator(C)
    B, N, E = 32, 41, 16
    br = handle(B, N, E)
    br.reserve_rows(C)
    cuts = torch.sort(torch.randint(0, N + 1, (B, E + 1), generator=torch.Generator().manual_seed(C)), 1).values
    offsets = cuts.to(torch.int32).to(DEV)
    x, f = rand(g, B, N, C), rand(g, B, N, C, dtype=torch.bfloat16)
    grad_out, grad_y = rand(g, B, N, C), rand(g, B, N, C, dtype=torch.bfloat16)
    params = {k: 1 + 0.1 * rand(g, E, C) for k in ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias")}
    gate = torch.rand((B, N), generator=g, device=DEV)
    seed = torch.tensor([5, 5], dtype=torch.int64, device=DEV)
    keep = kept((5, 5), B * N, C, 0.2).view(B, N, C).to(DEV)
    made = br.expert_residual(x, f, offsets, gate=gate, **params, p=0.2, seed=seed)
    inside = expert_of_rows(offsets, N, E) < E
    ref = forward(x, f, offsets, E, gate, params, 1e-5, keep, 0.2)
    assert ((made["out"].double() - ref["out"][0]).abs() <= ref["out"][1])[inside].all()
    back = {k: v for k, v in params.items() if k != "pre_bias"}
    made["stats"][~inside] = float("nan")
    got = br.expert_residual_grad(made["out"], f, offsets, made["stats"], grad_out, grad_y, gate=gate, **back, p=0.2, seed=seed)
    ref = gradients(made["out"], f, offsets, E, made["stats"], grad_out, grad_y, gate, params, keep, 0.2)
    for name, (want, bound) in ref.items():
        rows = inside if name in ("grad_x", "grad_f", "grad_gate") else slice(None)
        assert ((got[name].double() - want).abs() <= bound + 1e-37)[rows].all(), name
    br.status()
    br.close()


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
@pytest.mark.parametrize("n,E,k", [(128, 1, 1), (128, 2, 2), (77, 3, 2)])
def test_layer_whose_experts_have_several_passes(n, E, k, form):
    """More rows of an expert than fit a pass, whole and ragged, in the second kernel and the third."""
    g = generator(n + E)
    C, H = 200, 328
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr = rand(g, n, C, dtype=torch.float16), rand(g, E, C)
    ws = [rand(g, E, H, C, scale=C ** -0.5), rand(g, E, H, C, scale=C ** -0.5), rand(g, E, C, H, scale=H ** -0.5)]
    ws = [w.half() if form == "16 bits" else br.mx4_quantise(w) for w in ws]
    got = br.expert_layer(x, wr, *ws, k, "silu")
    ids, (p, err_p), (y, err) = layer(x, wr, None, *ws, k, "silu")
    assert torch.equal(got["ids"].long(), ids) and ((got["weights"].double() - p).abs() <= err_p).all()
    assert ((got["y"].double() - y).abs() <= err).all()
    br.status()
    br.close()


def test_two_handles_on_two_threads():
    """Calls of two handles at the same time, on streams of their own: the results of calls one after another."""
    shapes = [(60, 256, 512, 8, 2), (100, 128, 1024, 16, 4)]
    made = []
    for i, (n, C, H, E, k) in enumerate(shapes):
        g = generator(i)
        br = handle(2, 300, 2)
        br.reserve_rows(C, H)
        x, wr = rand(g, n, C, dtype=torch.bfloat16), rand(g, E, C)
        ws = [rand(g, E, H, C, scale=C ** -0.5).bfloat16(), rand(g, E, H, C, scale=C ** -0.5).bfloat16(), rand(g, E, C, H, scale=H ** -0.5).bfloat16()]
        rows, w = rand(g, 2, 300, C), torch.ones((1, C), device=DEV)
        packed = [br.mx4_quantise(m) for m in ws]

        def call(br=br, x=x, wr=wr, ws=ws, packed=packed, k=k, rows=rows, w=w):
            out = list(br.expert_layer(x, wr, *ws, k).values()) + list(br.expert_layer(x, wr, *packed, k).values())
            r = br.expert_residual(rows, rows, None, post_weight=w, pre_weight=w)
            grads = br.expert_residual_grad(r["out"], rows, None, r["stats"], rows, rows, post_weight=w, pre_weight=w)
            return out + list(r.values()) + [t for t in grads.values() if t is not None]

        made.append((br, call, call()))
    torch.cuda.synchronize()
    faults = []

    def work(i):
        br, call, want = made[i]
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                got = call()
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    faults.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert faults == []
    for br, _, _ in made:
        br.status()
        br.close()
