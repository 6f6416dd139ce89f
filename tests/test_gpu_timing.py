"""Per-kernel timing: what the C ABI writes into arrays of the caller's, whose length it cannot see."""
import ctypes

import pytest
import torch

import paper_2409_09099_amd as sste

FIRST = 8              # entries of sste_timing_end in every version of the library


def header_value(name):
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    return int(re.search(r"\b%s = (\d+)" % name, open(os.path.join(root, "include", "sste.h")).read()).group(1))


def test_the_number_of_entries_stays():
    from paper_2409_09099_amd import binding
    assert header_value("SSTE_K_COUNT") == FIRST and header_value("SSTE_K_ALL") == len(binding.KERNEL_NAMES)
    assert header_value("SSTE_K_ADAPTER") == binding.KERNEL_NAMES.index("adapter") and header_value("SSTE_K_CHECKPOINT") == binding.KERNEL_NAMES.index("checkpoint")


def test_refusals():
    lib = sste.library()
    assert lib.sste_timing_end_all(None, None, -1) == 5 and lib.sste_timing_end_all(None, None, 4) == 5 and lib.sste_timing_end(None, None) == 5      # timing is not on


def timed():
    x = torch.ones((64, 96), dtype=torch.bfloat16, device="cuda")
    sste.timing_begin(16)
    sste.checkpoint_pack(x)
    sste.cast_fp8(x, 1.0)


@pytest.mark.gpu
def test_entries_behind_the_first_are_left_alone():
    """Arrays as long as the first header asked for, with something else behind them."""
    ms, n = (ctypes.c_double * (FIRST + 4))(*[-1.0] * (FIRST + 4)), (ctypes.c_int * (FIRST + 4))(*[-1] * (FIRST + 4))
    timed()
    assert sste.library().sste_timing_end(ms, n) == 0
    assert list(n) == [0] * 7 + [1] + [-1] * 4 and list(ms)[FIRST:] == [-1.0] * 4 and ms[7] > 0 and list(ms)[:7] == [0.0] * 7


@pytest.mark.gpu
@pytest.mark.parametrize("entries", [0, 7, 8, 9, 10, 12])
def test_entries_asked_for(entries):
    ms, n = (ctypes.c_double * 14)(*[-1.0] * 14), (ctypes.c_int * 14)(*[-1] * 14)
    timed()
    assert sste.library().sste_timing_end_all(ms, n, entries) == 0
    want = [0] * 7 + [1, 0, 1] + [0] * 4
    assert list(n) == want[:entries] + [-1] * (14 - entries)
    assert [m > 0 for m in list(ms)[:entries]] == [bool(w) for w in want[:entries]] and list(ms)[entries:] == [-1.0] * (14 - entries)


@pytest.mark.gpu
def test_binding_reports_every_kernel():
    timed()
    times = sste.timing_end()
    assert times["checkpoint"][1] == 1 and times["cast"][1] == 1 and times["checkpoint"][0] > 0 and times["adapter"] == (0.0, 0)
