"""4-bit weights, and the layer for few rows with weights of 16 and of 4 bits, against the formulas in 64 bits (needs a B200).

Quantisation has to be exact; the layer's choices too (its logits are as of a sum in 48 bits); its results within the bounds of
layer_cases.py."""
import pytest
import torch

from layer_cases import layer, quantised, values_of
from row_cases import TYPES, handle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def shifted(t, elements):
    room = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    at = room[elements:].view(t.shape)
    at.copy_(t)
    return at


# ------------------------------------------------------------------ 4-bit weights
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,C", [(1, 4), (7, 36), (33, 80), (1000, 1024), (5, 8192), (3, 100), (2051, 32), (9, 72)])
def test_quantise(rows, C, dtype):
    g = generator(rows + C)
    br = handle(1, 8)
    x = rand(g, rows, C) * torch.exp2(torch.randint(-12, 12, (rows, C), generator=g, device=DEV).float() * (torch.rand((rows, 1), generator=g, device=DEV) < 0.5))
    x = x.to(dtype)
    blocks = -(-C // 32)
    for v in (x, shifted(x, 16 // x.element_size())):
        out = {"codes": torch.full((rows, 16 * blocks), 99, dtype=torch.uint8, device=DEV), "scales": torch.full((rows, blocks), 99, dtype=torch.uint8, device=DEV),
               "values": torch.full_like(x, 7.0)}
        br.mx4_quantise(v, out=out)
        codes, scales, values = quantised(x)
        assert torch.equal(out["codes"].int(), codes.int()) and torch.equal(out["scales"].int(), scales.int())
        assert torch.equal(out["values"].double(), values)
        assert torch.equal(values_of(out, C), values)
    only = br.mx4_quantise(x)
    assert set(only) == {"codes", "scales"} and torch.equal(only["codes"], out["codes"]) and torch.equal(only["scales"], out["scales"])
    values = br.mx4_quantise(x, out={"values": torch.empty_like(x)})
    assert torch.equal(values["values"], out["values"])
    br.status()
    br.close()


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_quantise_borders(dtype):
    """Halves between elements, blocks of zeros, of the smallest and largest numbers, infinities and NaN."""
    f = torch.finfo(dtype)
    steps = torch.arange(-32, 32, device=DEV, dtype=torch.float32) * 0.25          # every half between two elements, with 8 = 2^3 in the block
    blocks = [steps[:32], steps[32:], torch.zeros(32, device=DEV), torch.full((32,), -0.0, device=DEV), torch.full((32,), f.max, device=DEV, dtype=torch.float32),
              torch.full((32,), f.smallest_normal, device=DEV, dtype=torch.float32)]
    x = torch.stack(blocks).to(dtype)
    tiniest = torch.zeros(32, dtype=dtype, device=DEV)
    tiniest[3], tiniest[5] = f.smallest_normal * f.eps, -3 * f.smallest_normal * f.eps
    inf, nan = torch.ones(32, dtype=dtype, device=DEV), torch.ones(32, dtype=dtype, device=DEV)
    inf[7], nan[31] = float("-inf"), float("nan")
    x = torch.cat([x, torch.stack([tiniest, inf, nan])])
    br = handle(1, 8)
    out = br.mx4_quantise(x, out={"codes": torch.empty((9, 16), dtype=torch.uint8, device=DEV), "scales": torch.empty((9, 1), dtype=torch.uint8, device=DEV),
                                  "values": torch.empty_like(x)})
    codes, scales, values = quantised(x)
    zero = (x == 0).all(-1)                                                 # any power stands for a block of zeros: the library takes 2^-127
    assert torch.equal(out["scales"][~zero].int(), scales[~zero].int()) and (out["scales"][zero] == 0).all()
    assert torch.equal(out["codes"].int(), codes.int())
    assert torch.equal(out["values"].double().nan_to_num(-1.0), values.nan_to_num(-1.0)) and torch.equal(torch.isnan(out["values"]), torch.isnan(values))
    br.close()


# ------------------------------------------------------------------ the layer
SHAPES = [(1, 8, 8, 1, 1), (1, 256, 1024, 16, 2), (3, 80, 320, 8, 2), (128, 64, 96, 4, 2), (17, 1024, 72, 64, 8), (128, 40, 264, 256, 8), (5, 136, 8192, 2, 1), (64, 72, 1032, 3, 3),
          (33, 264, 536, 1, 1), (2, 1024, 2048, 5, 4), (128, 72, 520, 2, 2), (101, 256, 1032, 3, 1), (128, 128, 264, 8, 3)]


def problem(g, n, C, H, E, k, dtype):
    x = rand(g, n, C, dtype=dtype)
    return x, rand(g, E, C, scale=2 * C ** -0.5), rand(g, E, H, C, scale=C ** -0.5), rand(g, E, H, C, scale=C ** -0.5), rand(g, E, C, H, scale=H ** -0.5)


def check(got, want, rows=slice(None)):
    ids, (p, err_p), (y, err) = want
    assert torch.equal(got["ids"][rows].long(), ids)
    assert ((got["weights"][rows].double() - p).abs() <= err_p).all()
    off = (got["y"][rows].double() - y).abs()
    assert (off <= err).all(), float((off / err).max())


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
@pytest.mark.parametrize("dtype,act", [(torch.bfloat16, "silu"), (torch.float16, "gelu"), (torch.bfloat16, "gelu")], ids=str)
@pytest.mark.parametrize("n,C,H,E,k", SHAPES)
def test_layer(n, C, H, E, k, dtype, act, form):
    g = generator(n * C + H)
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, *ws = problem(g, n, C, H, E, k, dtype)
    ws = [w.to(dtype) if form == "16 bits" else br.mx4_quantise(w) for w in ws]
    b = rand(g, E) if n % 2 else None
    got = br.expert_layer(x, wr, *ws, k, act, b_router=b)
    check(got, layer(x, wr, b, *ws, k, act))
    again = br.expert_layer(x, wr, *ws, k, act, b_router=b)
    assert all(torch.equal(again[i], got[i]) for i in got)                  # bit for bit
    br.status()
    br.close()


@pytest.mark.parametrize("form", ["16 bits", "4 bits"])
def test_rows_in_use(form):
    """Rows behind the count are not read and left as they were; no rows at all; counts that are none are reported."""
    import paper_2507_04123_b200 as pkg
    g = generator(5)
    n, C, H, E, k = 40, 72, 136, 6, 2
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, *ws = problem(g, n, C, H, E, k, torch.bfloat16)
    ws = [w.bfloat16() if form == "16 bits" else br.mx4_quantise(w) for w in ws]
    for used in (39, 1, 0, 40, -3, 41):
        real = min(max(used, 0), n)
        v = x.clone()
        v[real:] = float("nan")
        out = {"y": torch.full_like(x, 7.0), "ids": torch.full((n, k), 77, dtype=torch.int32, device=DEV), "weights": torch.full((n, k), 7.0, device=DEV)}
        br.expert_layer(v, wr, *ws, k, count=torch.tensor([used], dtype=torch.int32, device=DEV), out=out)
        if real:
            check(out, layer(x[:real], wr, None, *ws, k, "silu"), slice(0, real))
        assert (out["y"][real:] == 7).all() and (out["ids"][real:] == 77).all() and (out["weights"][real:] == 7).all()
        assert br.status(raise_on_error=False) == (0 if used == real else pkg.bridge.EMC2_ERR_INVALID_ARG)
    br.close()


def test_choices_at_borders():
    """Equal logits: the lower expert first; differences far below fp32's steps decide; experts shut off; rows with NaN or infinities
    touch no others."""
    g = generator(6)
    n, C, H, E, k = 6, 64, 72, 8, 3
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, *ws = problem(g, n, C, H, E, k, torch.bfloat16)
    ws = [w.bfloat16() for w in ws]
    wr[5], wr[2] = wr[7], wr[7]
    x[1] = 0                                                                # all equal
    check(br.expert_layer(x, wr, *ws, k), layer(x, wr, None, *ws, k, "silu"))
    # Logits of 1 and 1 + 2^-30.
    fine = torch.zeros((E, C), device=DEV)
    fine[:, 0] = 1.0
    fine[6, 1] = 2.0 ** -30
    one = torch.ones((1, C), dtype=torch.bfloat16, device=DEV)
    assert br.expert_layer(one, fine, *ws, k)["ids"].tolist() == [[6, 0, 1]]
    shut = torch.zeros(E, device=DEV)
    shut[[0, 1, 2, 4, 5, 7]] = -torch.inf
    got = br.expert_layer(x, wr, *ws, 2, b_router=shut)
    assert (got["ids"].sort(-1)[0] == torch.tensor([3, 6], device=DEV)).all()
    check(got, layer(x, wr, shut, *ws, 2, "silu"))
    bad = x.clone()
    bad[2, 5], bad[4, 0] = float("nan"), float("inf")
    want, got = br.expert_layer(x, wr, *ws, k), br.expert_layer(bad, wr, *ws, k)
    assert torch.isnan(got["y"][2]).all() and got["ids"][2].tolist() == [0, 1, 2]
    rest = [0, 1, 3, 5]
    assert all(torch.equal(got[i][rest], want[i][rest]) for i in want)
    br.status()
    br.close()


@pytest.mark.parametrize("n", [1, 2])
def test_logits_past_fp32(n):
    """Terms, sums on the way and results beyond fp32's range, which have values in 64 bits: 2^133, 0, 2^132, 2^131, -2^120 and an
    infinity."""
    C, H, E = 64, 16, 6
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x = torch.ones((n, C), dtype=torch.bfloat16, device=DEV)
    x[:, 8:] = 2.0 ** 100
    wr = torch.zeros((E, C), device=DEV)
    wr[0, 8] = 2.0 ** 33
    wr[1, 8], wr[1, 9] = 2.0 ** 40, -2.0 ** 40                              # infinities of both signs in 32 bits
    wr[2, 8:16] = 2.0 ** 29                                                 # past the range by their sum
    wr[3, 8], wr[3, 9] = 2.0 ** 32, -2.0 ** 31
    wr[4, 8] = -2.0 ** 20
    wr[5, 8] = -torch.inf
    ws = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((E, H, C), (E, H, C), (E, C, H))]
    got = br.expert_layer(x, wr, *ws, 6)
    want = (x.double() @ wr.double().t()).sort(dim=-1, descending=True, stable=True)[1]
    assert want[0].tolist() == [0, 2, 3, 1, 4, 5]
    assert torch.equal(got["ids"].long(), want)
    assert got["weights"].tolist() == [[1.0, 0.0, 0.0, 0.0, 0.0, 0.0]] * n
    assert (got["y"] == 0).all()
    br.status()
    br.close()


def test_weights_of_far_powers():
    """Powers of two at the ends of their range, and NaN in a block of one expert that other experts' rows do not see."""
    g = generator(7)
    n, C, H, E = 9, 96, 64, 3
    br = handle(1, 8)
    br.reserve_rows(C, H)
    x, wr, *ws = problem(g, n, C, H, E, 1, torch.bfloat16)
    ws = [br.mx4_quantise(w) for w in ws]
    # Gate rows tiny and up rows large: the values between stay in range.
    ws[0]["scales"] -= 60
    ws[1]["scales"] += 62
    ws[0]["scales"][:, :, 1] = 0
    got = br.expert_layer(x, wr, *ws, 1)
    check(got, layer(x, wr, None, *ws, 1, "silu"))
    ws[2]["scales"][1, 5, 0] = 255
    spoilt = br.expert_layer(x, wr, *ws, 1)
    hit = spoilt["ids"][:, 0] == 1
    assert torch.isnan(spoilt["y"][hit][:, 5]).all()
    spoilt["y"][hit, 5] = got["y"][hit, 5]
    assert torch.equal(spoilt["y"], got["y"])
    br.close()


def test_layer_behind_other_calls_on_streams_and_captured():
    """The scratch is shared with the other operators: a block of a query's decoder, norm, layer and residual, between calls that write
    there, on another stream and in two graphs that are replayed in turn."""
    g = generator(8)
    n, C, H, E, k = 30, 128, 256, 8, 2
    br = handle(1, 400)
    br.reserve_rows(C, H)
    x = rand(g, 1, n, C)
    _, wr, *ws = problem(g, n, C, H, E, k, torch.bfloat16)
    packed = [br.mx4_quantise(w) for w in ws]
    ws = [w.bfloat16() for w in ws]
    one, half = torch.ones((1, C), device=DEV), torch.full((1, C), 0.5, device=DEV)
    big, wide = rand(g, 1, 400, C, dtype=torch.bfloat16), [w[:1].contiguous() for w in ws]
    count = torch.tensor([n], dtype=torch.int32, device=DEV)

    def step(o, weights):
        o["n"] = br.expert_norm(x, None, one, out_dtype=torch.bfloat16, out=o.get("n"))
        o["l"] = br.expert_layer(o["n"]["y"][0], wr, *weights, k, count=count, out=o.get("l"))
        o["r"] = br.expert_residual(x, o["l"]["y"][None], None, scale=half, pre_weight=one, out=o.get("r"))
        o["g"] = br.expert_ffn_grad(big, None, *wide, big, out=o.get("g"))
        return o

    def flat(o):
        return [t for part in ("n", "l", "r", "g") for t in o[part].values()]

    sets = [step({}, ws), step({}, packed)]
    want = [[t.clone() for t in flat(o)] for o in sets]
    check(sets[0]["l"], layer(sets[0]["n"]["y"][0], wr, None, *ws, k, "silu"))
    check(sets[1]["l"], layer(sets[1]["n"]["y"][0], wr, None, *packed, k, "silu"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o, weights in zip(sets, (ws, packed)):
            for t in flat(o):
                t.zero_()
            step(o, weights)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for o, w in zip(sets, want) for a, b in zip(flat(o), w))
    graphs = []
    for o, weights in zip(sets, (ws, packed)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(o, weights)
    for _ in range(3):
        for i in (0, 1, 1, 0):
            for t in flat(sets[i]):
                t.zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(sets, want) for a, b in zip(flat(o), w))
    count[0] = 7                                                            # the same graph, fewer rows
    for t in flat(sets[0]):
        t.zero_()
    graphs[0].replay()
    y = want[0][len(sets[0]["n"])]                                          # the layer's, behind those of the norm
    assert torch.equal(sets[0]["l"]["y"][:7], y[:7]) and (sets[0]["l"]["y"][7:] == 0).all()
    br.status()
    del graphs
    br.close()


def test_first_call_of_a_thread_and_profile():
    import threading
    g = generator(9)
    br = handle(1, 8)
    br.reserve_rows(64, 64)
    x, wr, *ws = problem(g, 4, 64, 64, 4, 2, torch.bfloat16)
    ws = [w.bfloat16() for w in ws]
    torch.cuda.synchronize()
    want = br.expert_layer(x, wr, *ws, 2)
    got = []
    thread = threading.Thread(target=lambda: got.append(br.expert_layer(x, wr, *ws, 2)))
    thread.start()
    thread.join()
    assert all(torch.equal(got[0][i], want[i]) for i in want)
    for rows, launches in ((1, [0, 1, 1]), (2, [1, 1, 1])):        # one row is routed by the kernel of its first products
        y = x[:1].expand(rows, -1).contiguous()
        br.profile_read()
        br.expert_layer(y, wr, *ws, 2)
        counts = br.profile_read()
        assert [counts[i][0] for i in ("layer_route", "layer_hidden", "layer_down")] == launches
    br.close()


def test_calls_that_are_refused():
    import paper_2507_04123_b200 as pkg
    br = handle(1, 8)
    lib, bad, large = pkg.load_library(), pkg.bridge.EMC2_ERR_INVALID_ARG, pkg.bridge.EMC2_ERR_TOO_LARGE
    P = lambda t, off=0: None if t is None else t.data_ptr() + off          # noqa: E731
    x, codes, scales, values = torch.ones((4, 64), device=DEV), torch.empty((4, 32), dtype=torch.uint8, device=DEV), torch.empty((4, 2), dtype=torch.uint8, device=DEV), torch.empty((4, 64), device=DEV)

    def mx(rows=4, C=64, kind=0, x=P(x), c=P(codes), s=P(scales), v=P(values)):
        return lib.emc2_mx4_quantise(br._h, rows, C, kind, x, c, s, v, None)

    assert mx() == 0 and mx(v=None) == 0 and mx(c=None, s=None) == 0 and mx(rows=0, x=None, c=None, s=None, v=None) == 0
    for wrong in (dict(rows=-1), dict(C=0), dict(C=6), dict(C=8196), dict(kind=3), dict(x=None), dict(c=None), dict(s=None), dict(c=None, s=None, v=None), dict(v=P(x)), dict(x=P(x, 8)),
                  dict(c=P(codes, 4)), dict(v=P(values, 4)), dict(rows=2 ** 30)):
        assert mx(**wrong) == bad, wrong

    n, C, H, E, k = 4, 64, 72, 3, 2
    b = torch.bfloat16
    rows, wr, wg, wd = torch.ones((n, C), dtype=b, device=DEV), torch.ones((E, C), device=DEV), torch.ones((E, H, C), dtype=b, device=DEV), torch.ones((E, C, H), dtype=b, device=DEV)
    y, ids, p = torch.empty_like(rows), torch.empty((n, k), dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
    count = torch.tensor([4], dtype=torch.int32, device=DEV)

    def run(n=n, C=C, H=H, E=E, k=k, kind=1, act=0, x=P(rows), count=P(count), r=P(wr), br_=None, g=P(wg), u=P(wg), d=P(wd), y=P(y), i=P(ids), w=P(p)):
        return lib.emc2_expert_layer(br._h, n, C, H, E, k, kind, act, x, count, r, br_, g, u, d, y, i, w, None)

    assert run() == large
    br.reserve_rows(64, 0)
    assert run() == large
    br.reserve_rows(64, 64)
    assert run() == large                                                   # 72 hidden units
    br.reserve_rows(64, 72)
    assert run() == 0 and run(count=None) == 0 and run(n=0, x=None, y=None, i=None, w=None) == 0
    for wrong in (dict(n=-1), dict(n=129), dict(C=60), dict(C=0), dict(C=1032), dict(H=70), dict(H=0), dict(H=8200), dict(E=0), dict(E=257), dict(k=0), dict(k=4), dict(E=20, k=9), dict(kind=0),
                  dict(kind=3), dict(act=2), dict(act=-1), dict(x=None), dict(r=None), dict(g=None), dict(u=None), dict(d=None), dict(y=None), dict(i=None), dict(w=None), dict(y=P(rows)),
                  dict(x=P(rows, 8)), dict(r=P(wr, 4)), dict(g=P(wg, 2)), dict(y=P(y, 8)), dict(i=P(ids, 2)), dict(w=P(p, 1)), dict(count=P(count, 1)), dict(br_=P(wr, 2))):
        assert run(**wrong) == bad, wrong
    assert lib.emc2_expert_layer_mx4(br._h, n, C, H, E, k, 1, 0, P(rows), None, P(wr), None, P(codes), None, P(codes), P(scales), P(codes), P(scales), P(y), P(ids), P(p), None) == bad
    br.status()
    # The binding's own checks.
    q = br.mx4_quantise(wg)
    for args in ((rows.float(), wr, wg, wg, wd, k), (rows, wr.bfloat16(), wg, wg, wd, k), (rows, wr, wg, q, wd, k), (rows, wr, wg, wg, wg, k), (rows, wr, wg, wg, wd.transpose(1, 2), k)):
        with pytest.raises(ValueError):
            br.expert_layer(*args)
    with pytest.raises(ValueError):
        br.expert_layer(rows, wr, wg, wg, wd, k, "relu")
    with pytest.raises(ValueError):
        br.mx4_quantise(x.double())
    br.close()
