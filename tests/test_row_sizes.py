"""The scratch of the lookup's gradient holds every call that the handle takes (csrc/row_sizes.cuh compiled for the host, CPU)."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SMS = 148
MOST_IDS = 1 << 24                                            # of a handle


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("row_sizes") / "librow_sizes.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-fPIC", "-shared",
                    "-I", os.path.join(ROOT, "paper_2507_04123_b200", "csrc"), "-o", lib, os.path.join(ROOT, "tests", "row_sizes_shim.cpp")], check=True)
    so = ctypes.CDLL(lib)
    i32, i64, u64 = ctypes.c_int, ctypes.c_int64, ctypes.c_uint64
    so.parts.argtypes = [i32, i64, i32, ctypes.POINTER(i32)]
    so.need.restype, so.need.argtypes = u64, [i32, i64, i32]
    so.most.restype, so.most.argtypes = u64, [i32, i64, i32]
    so.largest_need.restype, so.largest_need.argtypes = u64, [i32, i64, i64, i32]
    return so


def steps(sizes, channels, n_max):
    """Numbers of ids up to n_max at which a group's places go up."""
    step = sizes.groups(channels) * 4 * SMS * 16
    return range(step, n_max + 1, step)


@pytest.mark.parametrize("ids,reserved,call", [(75777, 1024, 75776), (80000, 1024, 75000), (100000, 1024, 75776), (80000, 512, 74000),
                                               (160000, 128, 151552), (310000, 64, 303104)])
def test_smaller_calls_than_the_handle_fit(sizes, ids, reserved, call):
    assert sizes.need(SMS, call, reserved) <= sizes.most(SMS, ids, reserved)


@pytest.mark.parametrize("channels", [4, 8, 36, 64, 80, 128, 132, 256, 388, 516, 1024])
def test_every_call_up_to_the_handle_s_fits(sizes, channels):
    """The need at both sides of every step, and of handles that end there or anywhere."""
    rng = random.Random(channels)
    handles = [1, 7, 1000, 75777, 1_200_000, MOST_IDS] + [rng.randint(2, 2_000_000) for _ in range(40)]
    handles += [n + d for n in list(steps(sizes, channels, 4_000_000))[:6] for d in (0, 1, 5000)]
    for n_max in handles:
        room = sizes.most(SMS, n_max, channels)
        calls = {1, n_max, max(1, n_max // 2)} | {m for n in steps(sizes, channels, n_max) for m in (n, n + 1) if m <= n_max}
        for n in calls:
            for c in {4, channels // 8 * 4 or 4, channels}:
                assert sizes.need(SMS, n, c) <= room, (n_max, n, c)


def test_all_numbers_of_ids_around_a_step(sizes):
    for channels in (64, 256, 1024):
        step = next(iter(steps(sizes, channels, MOST_IDS)))
        for n_max in (step - 1, step, step + 1, step + 3000):
            assert sizes.largest_need(SMS, max(1, n_max - 6000), n_max, channels) <= sizes.most(SMS, n_max, channels)


def test_parts_cover_the_list_with_four_ctas_per_sm_at_most(sizes):
    items = ctypes.c_int()
    rng = random.Random(1)
    for channels in (4, 64, 80, 512, 1024):
        for n in [1, 16, 17, MOST_IDS] + [rng.randint(1, MOST_IDS) for _ in range(200)]:
            ctas = sizes.parts(SMS, n, channels, items)
            per = items.value * sizes.groups(channels)
            assert items.value % 16 == 0 and (ctas - 1) * per < n <= ctas * per and ctas <= 4 * SMS
