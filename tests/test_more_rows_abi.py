"""Residual, dropout, 4-bit weights and the layer for few rows: what they refuse without a handle, sizes behind 32 bits, and what the
binding refuses before it calls (CPU: no kernel runs)."""
import pytest
import torch

import paper_2507_04123_b200 as pkg
from paper_2507_04123_b200 import build


def test_calls_without_a_handle_are_refused():
    build.build()
    lib, bad = pkg.load_library(), pkg.bridge.EMC2_ERR_INVALID_ARG
    assert lib.emc2_row_dropout(None, 1, 4, 0, None, 0.5, None, None, None) == bad
    assert lib.emc2_expert_residual(None, 1, 1, 4, 0, 0, 0, *[None] * 9, 1e-5, 0.0, *[None] * 5) == bad
    assert lib.emc2_expert_residual_grad(None, 1, 1, 4, 0, 0, 0, *[None] * 11, 0.0, *[None] * 10) == bad
    assert lib.emc2_mx4_quantise(None, 1, 4, 0, *[None] * 5) == bad
    assert lib.emc2_expert_layer(None, 1, 8, 8, 1, 1, 1, 0, *[None] * 11) == bad
    assert lib.emc2_expert_layer_mx4(None, 1, 8, 8, 1, 1, 1, 0, *[None] * 14) == bad


class Recorder:
    """Stands in for the library: every call succeeds and is noted."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def bridge():
    """A bridge without a handle, whose tensors have sizes but no memory."""
    br = pkg.Bridge.__new__(pkg.Bridge)
    br.lib, br._h, br.device = Recorder(), None, torch.device("meta")
    br._stream = lambda: None
    return br


def t(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


f32, i64, u8 = torch.float32, torch.int64, torch.uint8
MANY = 2 ** 32 + 5                                            # 5 in 32 bits


def layer(br, n=4, C=64, H=72, E=3, k=2, **kw):
    return br.expert_layer(kw.pop("x", t(n, C)), t(E, C, dtype=f32), t(E, H, C), t(E, H, C), kw.pop("w_down", t(E, C, H)), k, **kw)


REFUSED = {
    "rows of dropout": lambda br: br.row_dropout(t(MANY, 8), 0.1, t(2, dtype=i64)),
    "residual rows": lambda br: br.expert_residual(t(1, MANY, 8), t(1, MANY, 8), None),
    "residual gradients": lambda br: br.expert_residual_grad(t(1, MANY, 8), t(1, MANY, 8), None, None, t(1, MANY, 8), None),
    "rows of weights": lambda br: br.mx4_quantise(t(MANY, 32)),
    "rows of the layer": lambda br: layer(br, n=MANY),
    "experts of the layer": lambda br: layer(br, E=MANY),
    "hidden units of the layer": lambda br: layer(br, H=MANY),
    "choices": lambda br: layer(br, k=MANY),
    "a seed of one number": lambda br: br.row_dropout(t(4, 8), 0.1, t(1, dtype=i64)),
    "rows in 64 bits": lambda br: br.row_dropout(t(4, 8, dtype=torch.float64), 0.1, t(2, dtype=i64)),
    "dropout without a seed": lambda br: br.expert_residual(t(1, 4, 8), t(1, 4, 8), None, p=0.1),
    "another shape of the block's result": lambda br: br.expert_residual(t(1, 4, 8), t(1, 5, 8), None),
    "weights of two experts without offsets": lambda br: br.expert_residual(t(1, 4, 8), t(1, 4, 8), None, scale=t(2, 8, dtype=f32)),
    "16-bit weights of a norm": lambda br: br.expert_residual(t(1, 4, 8), t(1, 4, 8), None, post_weight=t(1, 8)),
    "room for y without its norm": lambda br: br.expert_residual(t(1, 4, 8), t(1, 4, 8), None, out={"out": t(1, 4, 8), "y": t(1, 4, 8), "stats": None}),
    "no room for y": lambda br: br.expert_residual(t(1, 4, 8), t(1, 4, 8), None, pre_weight=t(1, 8, dtype=f32), out={"out": t(1, 4, 8), "y": None, "stats": None}),
    "a gradient of y without its norm": lambda br: br.expert_residual_grad(t(1, 4, 8), t(1, 4, 8), None, None, t(1, 4, 8), t(1, 4, 8)),
    "no gradient from behind": lambda br: br.expert_residual_grad(t(1, 4, 8), t(1, 4, 8), None, None, None, None),
    "a norm's gradient without statistics": lambda br: br.expert_residual_grad(t(1, 4, 8), t(1, 4, 8), None, None, t(1, 4, 8), None, post_weight=t(1, 8, dtype=f32)),
    "fp32 rows of the layer": lambda br: layer(br, x=t(4, 64, dtype=f32)),
    "weights of two forms": lambda br: layer(br, w_down={"codes": t(3, 64, 48, dtype=u8), "scales": t(3, 64, 3, dtype=u8)}),
    "a count of two": lambda br: layer(br, count=t(2, dtype=torch.int32)),
    "an unknown activation": lambda br: layer(br, act="relu"),
    "room for too few codes": lambda br: br.mx4_quantise(t(4, 40), out={"codes": t(4, 16, dtype=u8), "scales": t(4, 2, dtype=u8)}),
}


@pytest.mark.parametrize("name", REFUSED)
def test_what_the_binding_refuses(bridge, name):
    with pytest.raises(ValueError):
        REFUSED[name](bridge)
    assert bridge.lib.calls == []


def test_calls_that_reach_the_library(bridge):
    w = t(1, 8, dtype=f32)
    bridge.row_dropout(t(2, 3, 8), 0.1, t(2, dtype=i64))
    out = bridge.expert_residual(t(1, 4, 8, dtype=f32), t(1, 4, 8), None, pre_weight=w, post_weight=w)
    assert out["y"].dtype == torch.bfloat16 and out["out"].dtype == f32 and out["stats"].shape == (1, 4, 4)
    grads = bridge.expert_residual_grad(out["out"], t(1, 4, 8), None, out["stats"], None, out["y"], pre_weight=w, post_weight=w)
    assert grads["grad_gate"] is None and grads["grad_scale"] is None and grads["grad_pre_bias"].shape == (1, 8)
    q = bridge.mx4_quantise(t(3, 72, 40))
    assert q["codes"].shape == (3, 72, 32) and q["scales"].shape == (3, 72, 2)
    layer(bridge, count=t(1, dtype=torch.int32))
    down = {"codes": t(3, 40, 48, dtype=u8), "scales": t(3, 40, 3, dtype=u8)}
    bridge.expert_layer(t(4, 40), t(3, 40, dtype=f32), q, q, down, 2)
    assert bridge.lib.calls == ["emc2_row_dropout", "emc2_expert_residual", "emc2_expert_residual_grad", "emc2_mx4_quantise", "emc2_expert_layer", "emc2_expert_layer_mx4"]
