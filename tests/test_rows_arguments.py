"""Sizes that do not fit the C interface's 32 bits are refused by the binding, not cut down to those that do (CPU: no kernel runs)."""
import pytest
import torch

import paper_2507_04123_b200 as pkg


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


def rows(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


MANY = 2 ** 32 + 5                                            # 5 in 32 bits
CALLS = {
    "ids": lambda br: br.row_lookup(rows(MANY, dtype=torch.int32), rows(9, 4)),
    "ids of the gradient": lambda br: br.row_lookup_grad(rows(MANY, dtype=torch.int32), rows(MANY, 4), 9),
    "table": lambda br: br.row_lookup(rows(7, dtype=torch.int32), rows(MANY, 4)),
    "table of the gradient": lambda br: br.row_lookup_grad(rows(7, dtype=torch.int32), rows(7, 4), MANY),
    "2^31 rows": lambda br: br.row_lookup(rows(7, dtype=torch.int32), rows(2 ** 31, 4)),
    "reserved channels": lambda br: br.reserve_rows(MANY),
    "reserved hidden units": lambda br: br.reserve_rows(64, MANY),
    "norm": lambda br: br.expert_norm(rows(1, MANY, 4), None, rows(1, 4, dtype=torch.float32)),
    "norm gradients": lambda br: br.expert_norm_grad(rows(1, MANY, 4), None, rows(1, 4, dtype=torch.float32), rows(1, MANY, dtype=torch.float32),
                                                     rows(1, MANY, dtype=torch.float32), rows(1, MANY, 4)),
    "feed-forward": lambda br: br.expert_ffn(rows(1, MANY, 8), None, rows(1, 8, 8), rows(1, 8, 8), rows(1, 8, 8)),
    "feed-forward gradients": lambda br: br.expert_ffn_grad(rows(1, MANY, 8), None, rows(1, 8, 8), rows(1, 8, 8), rows(1, 8, 8), rows(1, MANY, 8)),
    "hidden units": lambda br: br.expert_ffn(rows(1, 3, 8), None, rows(1, MANY, 8), rows(1, MANY, 8), rows(1, 8, MANY)),
}


@pytest.mark.parametrize("name", CALLS)
def test_sizes_behind_32_bits_are_refused(bridge, name):
    with pytest.raises(ValueError):
        CALLS[name](bridge)
    assert bridge.lib.calls == []


def test_sizes_of_31_bits_reach_the_library(bridge):
    bridge.row_lookup(rows(7, dtype=torch.int32), rows(2 ** 31 - 1, 4))
    bridge.row_lookup_grad(rows(7, dtype=torch.int32), rows(7, 4), 2 ** 31 - 1)
    bridge.expert_ffn(rows(1, 3, 8), None, rows(1, 8, 8), rows(1, 8, 8), rows(1, 8, 8))
    bridge.reserve_rows(64)
    assert bridge.lib.calls == ["emc2_row_lookup", "emc2_row_lookup_grad", "emc2_expert_ffn", "emc2_rows_reserve"]
