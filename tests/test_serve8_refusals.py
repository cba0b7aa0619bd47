"""What the calls refuse of a cache held in 8 bits, on the host and before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest
import torch

from paper_2603_02170_amd import binding, build, cache
from paper_2603_02170_amd.cache import CacheParams
from test_serve_refusals import Call


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.HOST):
        build.build(verbose=False)
    return binding.load_library()


def test_page_bytes_and_formats_that_do_not_exist(lib):
    assert cache.cache_page_bytes(CacheParams(H=8, d=128, page=64, block=64)) == 8 * (64 * 256 + 16)
    assert cache.cache_page_bytes(CacheParams(H=3, d=64, page=32, block=32)) == 3 * (32 * 128 + 16)
    assert cache.cache_page_bytes(CacheParams(H=1, d=64, page=256, block=32)) == 256 * 128 + 64
    assert cache.cache_page_bytes(CacheParams(H=1, d=64, page=256, group=7, block=32)) == 256 * 128 + 64      # (group is not looked at)
    for bad, status in ((dict(block=16), -1), (dict(block=1), -1), (dict(block=128), -1), (dict(page=32, block=64), -2), (dict(d=96), -2), (dict(page=512), -2),
                        (dict(H=0), -1), (dict(H=2000), -2)):
        with pytest.raises(binding.SageError) as e:
            cache.cache_page_bytes(CacheParams(**{**dict(H=1, d=64, block=32), **bad}))
        assert e.value.status == status, bad


def test_the_c_calls_refuse_params_that_contradict_themselves(lib):
    P = cache._CCacheParams
    one, null, i64 = ctypes.c_void_p(256), ctypes.c_void_p(None), ctypes.c_int64       # (never dereferenced: the checks fail first)
    c = Call(1, 1, 4, 2, 1, 0, 1, 0.0, 256, 64)
    for x, status in ((P(2, 64, 64, 32, 4, 64), -1), (P(2, 64, 64, 0, 4, 48), -1), (P(2, 64, 64, 0, 4, -32), -1), (P(2, 64, 32, 0, 4, 64), -2), (P(2, 64, 64, 0, 0, 64), -1),
                      (P(2, 80, 64, 0, 4, 32), -2), (P(2, 64, 64, 0, 4, 0), -2)):
        assert lib.sagebwd_cache_append(one, one, i64(64), i64(64), i64(64), i64(64), one, 1, null, null, ctypes.byref(x), one, null) == status
        assert lib.sagebwd_cache_read(one, 1, null, null, ctypes.byref(x), one, one, one, null) == status
        assert lib.sagebwd_cache_attention(one, one, one, one, one, null, ctypes.byref(x), ctypes.byref(c), one, one, one, ctypes.c_size_t(1 << 40), null) == status
        assert lib.sagebwd_cache_workspace_bytes(ctypes.byref(x), ctypes.byref(c), ctypes.byref(ctypes.c_size_t())) == status
    p = P(2, 64, 64, 0, 4, 64)
    append = lambda k=one, ks=64, slots=one, T=1, pool=one: lib.sagebwd_cache_append(k, one, i64(ks), i64(64), i64(64), i64(64), slots, T, null, null,  # noqa: E731
                                                                                   ctypes.byref(p), pool, null)
    assert append(k=null) == -1 and append(k=ctypes.c_void_p(264)) == -1 and append(ks=63) == -1 and append(slots=null) == -1 and append(T=-1) == -1
    assert append(pool=ctypes.c_void_p(8)) == -1 and append(T=0) == 0
    most = P(1024, 128, 64, 0, 4, 64)
    assert lib.sagebwd_cache_append(one, one, i64(128), i64(128), i64(128), i64(128), one, (1 << 31) - 1, null, null, ctypes.byref(most), one, null) == -2
    assert lib.sagebwd_cache_read(one, (1 << 31) - 1, null, null, ctypes.byref(most), one, one, one, null) == -2


def test_tensors_that_do_not_fit(lib):
    p = CacheParams(H=2, d=64, page=32, block=32)
    pool = cache.alloc_cache(p, 2, device="cpu")
    assert tuple(pool.shape) == (2, 2, 32 * 128 + 16)
    K = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="cache: need contiguous cuda"):
        cache.sagebwd_cache_append(K, K, torch.zeros(3, dtype=torch.int64), pool, p)
    with pytest.raises(ValueError, match="out of range"):
        cache.cache_page_bytes(p) and cache.cache_workspace_bytes(CacheParams(H=2, d=64, block=-1), 1, 1, 2, 1, 1)
    with pytest.raises(binding.SageError):
        cache.cache_workspace_bytes(CacheParams(H=2, d=64, block=8), 1, 1, 2, 1, 1)
    assert cache.cache_workspace_bytes(p, 4, 4, 4, 10, 1) > 0


@pytest.mark.gpu
def test_a_pool_of_the_other_format_is_refused(lib):
    p8, p4 = CacheParams(H=2, d=64, page=32, block=32), CacheParams(H=2, d=64, page=32)
    K, slots = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.arange(3, device="cuda")
    for p, other in ((p8, p4), (p4, p8)):
        with pytest.raises(ValueError, match="cache"):
            cache.sagebwd_cache_append(K, K, slots, cache.alloc_cache(other, 2), p)
