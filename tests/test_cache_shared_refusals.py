"""What the calls on shared pages refuse, on the host and before anything is launched, and their kernels as they are built (no GPU needed)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2603_02170_amd import binding, build, cache
from paper_2603_02170_amd.cache import CacheParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_02170_amd", "csrc")
one, null, size_t = ctypes.c_void_p(256), ctypes.c_void_p(None), ctypes.c_size_t       # (never dereferenced: the checks fail first)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.HOST):
        build.build(verbose=False)
    return binding.load_library()


BAD_SIZES = [(dict(R=-1), -1), (dict(columns=0), -1), (dict(capacity=-1), -1), (dict(pages=0), -1), (dict(lengths=null), -1), (dict(table=null), -1), (dict(stack=null), -1),
             (dict(count=null), -1), (dict(shares=null), -1), (dict(asked=null), -1), (dict(page=48), -2), (dict(page=16), -2), (dict(columns=1 << 26), -2),
             (dict(R=1 << 21), -2), (dict(R=1 << 20, columns=1 << 12), -2), (dict(pages=(1 << 28) + 1), -2)]


def test_free_and_fork(lib):
    def free(asked=one, lengths=one, table=one, stack=one, count=one, shares=one, R=1, columns=2, page=32, capacity=3, pages=3):
        return lib.sagebwd_cache_free(asked, lengths, table, stack, count, shares, R, columns, page, capacity, pages, null)

    def fork(asked=one, lengths=one, table=one, stack=one, count=one, shares=one, R=1, columns=2, page=32, capacity=3, pages=3, ws=one, n=1 << 40):
        return lib.sagebwd_cache_fork(asked, lengths, table, stack, count, shares, R, columns, page, capacity, pages, ws, size_t(n), null)

    for bad, status in BAD_SIZES:
        assert free(**bad) == status and fork(**bad) == status, bad
    assert free(R=0) == 0 and fork(R=0, ws=null, n=0) == 0
    assert fork(ws=null) == -1 and fork(ws=ctypes.c_void_p(128)) == -1 and fork(n=511) == -3
    n = size_t()
    for R, columns, want in ((1, 2, 512), (0, 1, 0), (100, 100, 40192 + 512), (-1, 1, None), (1, 0, None), (1 << 20, 1 << 12, None)):
        rc = lib.sagebwd_cache_fork_workspace_bytes(R, columns, ctypes.byref(n))
        assert (rc == 0 and n.value == want) if want is not None else rc < 0
    assert lib.sagebwd_cache_fork_workspace_bytes(1, 1, None) == -1


def test_own_and_compact(lib):
    P = cache._CCacheParams

    def own(asked=one, lengths=one, table=one, stack=one, count=one, shares=one, R=1, columns=2, page=64, capacity=3, pages=3, p=None, pool=one, out=one, ws=one, n=1 << 40):
        p = p or P(1, 64, page, 0, pages, 32)
        return lib.sagebwd_cache_own(asked, lengths, table, stack, count, shares, R, columns, capacity, ctypes.byref(p), pool, out, ws, size_t(n), null)

    def compact(lengths=one, table=one, out=one, stack=one, count=one, shares=one, used=one, R=1, columns=2, page=64, capacity=3, pages=3, p=None, pool=one, ws=one, n=1 << 40):
        p = p or P(1, 64, page, 0, pages, 32)
        return lib.sagebwd_cache_compact(lengths, table, R, columns, ctypes.byref(p), pool, out, stack, capacity, count, shares, used, ws, size_t(n), null)

    for bad, status in BAD_SIZES:
        assert own(**bad) == status, bad
        if "asked" not in bad:
            assert compact(**bad) == status, bad
    for p, status in ((P(1, 64, 64, 32, 3, 32), -1), (P(1, 64, 32, 0, 3, 64), -2), (P(1, 72, 64, 0, 3, 32), -2), (P(0, 64, 64, 64, 3, 0), -1)):
        assert own(p=p) == status and compact(p=p) == status
    assert own(pool=null) == -1 and own(pool=ctypes.c_void_p(8)) == -1 and own(out=null) == -1 and own(ws=null) == -1 and own(n=7) == -3 and own(R=0, out=null, ws=null, n=0) == 0
    assert compact(pool=null) == -1 and compact(out=null) == -1 and compact(used=null) == -1 and compact(capacity=2) == -1 and compact(ws=null) == -1
    assert compact(ws=ctypes.c_void_p(64)) == -1 and compact(n=1) == -3
    n = size_t()
    assert lib.sagebwd_cache_compact_workspace_bytes(100, ctypes.byref(n)) == 0 and n.value >= 51 * 8
    assert lib.sagebwd_cache_compact_workspace_bytes(0, ctypes.byref(n)) == -1 and lib.sagebwd_cache_compact_workspace_bytes((1 << 28) + 1, ctypes.byref(n)) == -2


def test_tensors_of_other_types_shapes_and_places(lib):
    p = CacheParams(H=1, d=64, page=32, block=32)
    i = torch.zeros(3, dtype=torch.int32)
    shares, pool = cache.alloc_shares(4, device="cpu"), cache.alloc_cache(p, 4, device="cpu")
    assert shares.shape == (3, 4) and shares.dtype == torch.int32 and not shares.any()
    state = i, i[:, None], i, i[:1], shares
    for call, name in ((lambda: cache.sagebwd_cache_free(i, *state, p), "keep"), (lambda: cache.sagebwd_cache_fork(i, *state, p), "parents"),
                       (lambda: cache.sagebwd_cache_own(i, *state, pool, p), "cache"), (lambda: cache.sagebwd_cache_compact(i, i[:, None], pool, p), "cache")):
        with pytest.raises(ValueError, match=name + ": need contiguous cuda"):
            call()
    with pytest.raises(TypeError):
        cache.sagebwd_cache_free(None, *state, p)
    with pytest.raises(binding.SageError):
        cache.sagebwd_cache_own(i, *state, pool, CacheParams(H=1, d=64, page=33))


@pytest.mark.gpu
def test_device_tensors_that_do_not_fit(lib):
    p = CacheParams(H=1, d=64, page=32, block=32)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool, shares = cache.alloc_cache(p, 4), cache.alloc_shares(4)
    names = ("lengths", "block_table", "free_pages", "free_count", "shares")
    state = [torch.zeros(2, **i32), torch.full((2, 3), -1, **i32), torch.zeros(4, **i32), torch.zeros(1, **i32), shares]
    asked = torch.zeros(2, **i32)
    calls = (lambda s: cache.sagebwd_cache_free(asked, *s, p), lambda s: cache.sagebwd_cache_fork(asked, *s, p), lambda s: cache.sagebwd_cache_own(asked, *s, pool, p))
    for call in calls:
        call(state)
        for k, bad in ((0, torch.zeros(3, **i32)), (0, state[0].long()), (1, state[1][:1]), (1, torch.full((2, 6), -1, **i32)[:, ::2]), (2, state[2][None]), (3, torch.zeros(2, **i32)),
                       (4, shares[0]), (4, shares[:2]), (4, shares.cpu()), (1, state[1][:, :0])):
            with pytest.raises(ValueError, match=names[k]):
                call(state[:k] + [bad] + state[k + 1:])
    with pytest.raises(ValueError, match="shares"):
        calls[2](state[:4] + [cache.alloc_shares(5)])
    with pytest.raises(ValueError, match="out"):
        cache.sagebwd_cache_own(asked, *state, pool, p, out=torch.zeros(3, **i32))
    ok = cache.sagebwd_cache_compact(state[0], state[1], pool, p)
    for k, bad, match in ((0, state[1][:, :2].contiguous(), "block_table"), (1, torch.zeros(3, **i32), "free_pages"), (2, asked, "free_count"), (3, cache.alloc_shares(3), "shares"),
                          (4, asked, "used")):
        with pytest.raises(ValueError, match=match):
            cache.sagebwd_cache_compact(state[0], state[1], pool, p, out=ok[:k] + (bad,) + ok[k + 1:])
    with pytest.raises(ValueError, match="five tensors"):
        cache.sagebwd_cache_compact(state[0], state[1], pool, p, out=ok[:4])


def test_the_kernels_have_no_scratch_and_no_packed_fp32(tmp_path):
    out = str(tmp_path / "pages.s")
    cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
           os.path.join(CSRC, "pages_api.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    text = open(out).read()
    assert not re.search(r"\bv_pk_(fma|mul|add)_f32\b", text)
    blocks = text.split(".amdhsa_kernel ")[1:]
    assert len(blocks) >= 10
    for block in blocks:
        get = lambda key: int(re.search(key + r"\s+(\d+)", block).group(1))  # noqa: E731
        assert get(r"\.amdhsa_private_segment_fixed_size") == 0 and get(r"\.amdhsa_next_free_vgpr") <= 64, block.split("\n")[0]
