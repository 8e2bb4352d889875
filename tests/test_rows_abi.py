"""The operators on dispatched rows: what they refuse without a handle, and constants that the binding and the header share (CPU)."""
import os
import re

import paper_2507_04123_b200 as pkg
from paper_2507_04123_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_without_a_handle_are_refused():
    build.build()
    lib, bad = pkg.load_library(), pkg.bridge.EMC2_ERR_INVALID_ARG
    assert lib.emc2_rows_reserve(None, 64, 64) == bad
    assert lib.emc2_row_lookup(None, 1, 1, 4, 0, None, None, 1.0, None, None) == bad
    assert lib.emc2_row_lookup_grad(None, 1, 1, 4, 0, None, None, 1.0, None, None) == bad
    assert lib.emc2_expert_norm(None, 1, 1, 4, 0, 0, *[None] * 4, 1e-5, *[None] * 4) == bad
    assert lib.emc2_expert_norm_grad(None, 1, 1, 4, 0, 0, *[None] * 10) == bad
    assert lib.emc2_expert_ffn(None, 1, 1, 8, 8, 1, 0, *[None] * 7) == bad
    assert lib.emc2_expert_ffn_grad(None, 1, 1, 8, 8, 1, 0, *[None] * 11) == bad


def test_types_and_activations_are_the_header_s():
    header = open(os.path.join(ROOT, "include", "emc2_bridge.h")).read()
    values = {n: int(v) for n, v in re.findall(r"(EMC2_(?:F32|BF16|F16|ACT_\w+)) = (\d)", header)}
    import torch
    assert pkg.bridge.ROW_TYPES == {torch.float32: values["EMC2_F32"], torch.bfloat16: values["EMC2_BF16"], torch.float16: values["EMC2_F16"]}
    assert pkg.bridge.ACTIVATIONS == {"silu": values["EMC2_ACT_SILU"], "gelu": values["EMC2_ACT_GELU"]}
