"""Sizes at which the serving calls' arithmetic would pass its bits are refused on the host, before anything is launched or allocated."""
import ctypes
import os

import pytest
import torch

from paper_2603_02170_amd import binding, build, cache
from paper_2603_02170_amd.cache import CacheParams


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.HOST):
        build.build(verbose=False)
    return binding.load_library()


def _plan(lib, R=1, columns=1, rows=1):
    one = ctypes.c_void_p(256)       # (never dereferenced: the checks come first)
    return lib.sagebwd_cache_plan(one, one, one, one, one, R, columns, 32, 1, rows, one, one, one, one, one, one, ctypes.c_void_p(None))


@pytest.mark.parametrize("rows", [2 ** 30 + 1, 2 ** 31 - 1024, 2 ** 31 - 1])
def test_a_plan_of_more_rows_than_its_steps_hold_is_refused(lib, rows):
    """A row and the launch's threads, rows rounded up to 1024, are added in 32 bits: from 2^30 + 1 on the sum is negative and passes the loop's
    comparison."""
    threads = -(-rows // 1024) * 1024
    assert rows - 1 + threads >= 2 ** 31
    for R in (0, 1, 1024, 1025):
        assert _plan(lib, R=R, rows=rows) == -2


def test_a_table_of_more_entries_than_the_sums_hold_is_refused(lib):
    """Pages are counted in sums that stop at 2^31 - 1: more entries than that could be freed in part, or granted beyond the stack."""
    one, null = ctypes.c_void_p(256), ctypes.c_void_p(None)
    for R, columns in ((1 << 20, 2048), (1 << 10, 1 << 21), (129, 1 << 24)):
        assert R * columns > 2 ** 31 - 1 and R <= 1 << 20 and columns * 32 < 2 ** 30
        assert _plan(lib, R=R, columns=columns) == -2
        assert lib.sagebwd_cache_trim(one, one, one, one, one, R, columns, 32, 1, null) == -2


@pytest.mark.gpu
def test_a_plan_of_too_many_rows_allocates_nothing(lib):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    args = i32(0), i32(1), i32(0)[None], i32(0), i32(1), CacheParams(1, 64, page=32)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    with pytest.raises(binding.SageError) as e:
        cache.sagebwd_cache_plan(*args, 2 ** 30 + 1)
    assert e.value.status == -2 and torch.cuda.max_memory_allocated() == before
