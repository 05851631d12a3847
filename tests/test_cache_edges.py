"""Refusals and checks of the cache calls that need no device (see test_cache_refusals.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2609_22098_b200 import binding
from test_cache_refusals import OK, ctx, layout, lib   # noqa: F401 (fixtures)


def granted(lib, ctx, lay, B=2, layers=3, ptrs=None):
    return lib.ts_cache_commit_granted(ctx, C.byref(lay), B, layers, lib.ts_cache_bytes(C.byref(lay)), *(ptrs or [OK] * 7), None)


def test_commit_with_status_checks_what_commit_checks(lib, ctx):
    for bad in (None, OK + 2):
        for i in range(7):
            assert granted(lib, ctx, layout(), ptrs=[bad if j == i else OK for j in range(7)]) == -1, i
            assert lib.ts_last_error_string().startswith(b"ts_cache_commit_granted: ")
    assert granted(lib, None, layout()) == -1 and granted(lib, ctx, layout(), B=9) == -1 and granted(lib, ctx, layout(), layers=0) == -1
    assert granted(lib, ctx, layout(Dh=96)) == -2 and lib.ts_last_error_string().startswith(b"ts_cache_commit_granted: head size")
    assert granted(lib, ctx, layout()) == -1 and lib.ts_last_error_string() == b"ts_cache_commit_granted: the context's device is not the current one"


def test_oracle_gives_back_pages_only():
    table = np.array([[3, -1, 99, 5], [0, 1, -1, -1]])
    t, held, free, count, _, status = oc.reserve(16, 8, [-1, 20], [1, 1], [4, 2], [7, 2, 4, 6, 0, 0, 0, 0], 4, table, 1)
    assert t.tolist() == [[-1] * 4, [0, 1, -1, -1]] and held == [0, 2] and free[:count] == [7, 2, 4, 6, 3, 5] and status == [0, 0]


def test_oracle_refuses_a_request_beyond_the_table_alone():
    """Requests 0 to 4: one fits, one needs more pages than the table has columns, one fits, one finds the list too short, and so
    does the next, which needs one page of the two that are left; the last needs none."""
    table = np.full((6, 3), -1)
    table[5, 0] = 9
    t, held, free, count, slots, status = oc.reserve(16, 10, [3, 40, 20, 30, 0, 3], [4, 9, 4, 18, 2, 4], [0, 0, 0, 0, 0, 1], [0, 1, 2, 3, 4], 5, table, 18)
    assert status == [0, oc.OVERFLOW, 0, oc.OVERFLOW, oc.OVERFLOW, 0]
    assert held == [1, 0, 2, 0, 0, 1] and count == 2 and t[2].tolist() == [3, 2, -1]
    assert (slots >= 0).sum(1).tolist() == [4, 0, 4, 0, 0, 4]


@pytest.mark.parametrize("shape", [(0, 2, 64), (4, 0, 2, 64), (0, 5, 2, 64), (3, 0, 7, 2, 64)])
def test_no_rows_are_rows(shape):
    """Tensors of no rows, whatever the other dimensions are: strides say nothing there."""
    t = torch.zeros(shape, dtype=torch.bfloat16)
    assert binding._rows_of(t, 2, 64, torch.bfloat16, -1, "k") == (0, 128)
    assert binding._rows_of(torch.zeros(*shape[:-2], 6, 64, dtype=torch.bfloat16)[..., 2:4, :], 2, 64, torch.bfloat16, -1, "k") == (0, 128)
    with pytest.raises(binding.TreeSparkError):
        binding._rows_of(t, 3, 64, torch.bfloat16, -1, "k")
