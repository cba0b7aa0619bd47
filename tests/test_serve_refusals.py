"""What the operators of sagebwd_serve.h refuse, on the host and before anything is launched (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2603_02170_amd import binding, build, cache
from paper_2603_02170_amd.autograd import sage_rotary
from paper_2603_02170_amd.cache import CacheParams

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.HOST):
        build.build(verbose=False)
    return binding.load_library()


class Call(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("R", "T", "Hq", "columns", "max_new", "max_length", "causal")] + [("sm_scale", ctypes.c_float)] + \
        [("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64)]


class Rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "N", "Hq", "Hk", "d", "rotary_dim", "axes")] + [("sections", ctypes.c_int32 * 4)] + \
        [(n, ctypes.c_int32) for n in ("adjacent", "inverse", "positions64")] + [(n, ctypes.c_int64 * 3) for n in ("q", "k", "qo", "ko")]


def _vp(x):
    return ctypes.c_void_p(x)


def test_the_header_and_the_library_name_the_same_calls(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sagebwd_serve.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(sagebwd_[a-z0-9_]+)\s*\(", text))) == sorted(cache.EXPORTS)
    for name in cache.EXPORTS:
        assert hasattr(lib, name)


def test_page_bytes(lib):
    assert cache.cache_page_bytes(CacheParams(H=8, d=128, page=64, group=64)) == 8 * 64 * (128 + 8)
    assert cache.cache_page_bytes(CacheParams(H=3, d=64, page=32, group=32)) == 3 * 32 * (64 + 8)
    for bad, status in ((dict(H=0), -1), (dict(d=96), -2), (dict(page=16), -2), (dict(page=48), -2), (dict(page=512), -2), (dict(group=128), -2), (dict(H=5000), -2)):
        with pytest.raises(binding.SageError) as e:
            cache.cache_page_bytes(CacheParams(**{**dict(H=1, d=64), **bad}))
        assert e.value.status == status


def test_the_c_calls_refuse_bad_arguments(lib):
    P = cache._CCacheParams
    p = P(2, 64, 64, 32, 4, 0)
    c = Call(1, 1, 4, 2, 1, 0, 1, 0.0, 256, 64)
    one, null, big = _vp(256), _vp(None), 1 << 40       # (never dereferenced: the checks fail first)
    attend = lambda p=p, c=c, q=one, pool=one, ws=one, n=big: lib.sagebwd_cache_attention(  # noqa: E731
        q, pool, one, one, one, null, ctypes.byref(p), ctypes.byref(c), one, one, ws, ctypes.c_size_t(n), null)
    assert attend(q=null) == -1 and attend(pool=null) == -1 and attend(ws=null) == -1
    assert attend(q=_vp(264)) == -1 and attend(pool=_vp(264)) == -1 and attend(ws=_vp(128)) == -1 and attend(n=16) == -3
    for k, bad, status in (("R", -1, -1), ("T", -1, -1), ("Hq", 0, -1), ("Hq", 5, -2), ("Hq", 130, -2), ("columns", 0, -1), ("columns", 1 << 30, -2), ("max_new", 0, -1),
                           ("max_length", -1, -1), ("causal", 2, -1), ("sm_scale", -1.0, -1), ("sm_scale", float("nan"), -1), ("sm_scale", float("inf"), -1),
                           ("q_token_stride", 12, -1), ("q_head_stride", -8, -1), ("R", 1 << 21, -2)):
        x = Call(1, 1, 4, 2, 1, 0, 1, 0.0, 256, 64)
        setattr(x, k, bad)
        assert attend(c=x) == status, (k, bad)
        assert lib.sagebwd_cache_workspace_bytes(ctypes.byref(p), ctypes.byref(x), ctypes.byref(ctypes.c_size_t())) == status
    for x, status in ((P(2, 64, 64, 32, 0, 0), -1), (P(2, 64, 64, 32, 4, 1), -1), (P(2, 96, 64, 32, 4, 0), -2), (P(2, 64, 16, 32, 4, 0), -2)):
        assert attend(p=x) == status
        assert lib.sagebwd_cache_append(one, one, ctypes.c_int64(64), ctypes.c_int64(64), ctypes.c_int64(64), ctypes.c_int64(64), one, 1, null, null, ctypes.byref(x), one, null) == status
        assert lib.sagebwd_cache_read(one, 1, null, null, ctypes.byref(x), one, one, one, null) == status
    i64 = ctypes.c_int64
    append = lambda k=one, ks=64, slots=one, T=1: lib.sagebwd_cache_append(k, one, i64(ks), i64(64), i64(64), i64(64), slots, T, null, null, ctypes.byref(p), one, null)  # noqa: E731
    assert append(k=null) == -1 and append(k=_vp(264)) == -1 and append(ks=63) == -1 and append(slots=null) == -1 and append(T=-1) == -1 and append(T=0) == 0
    assert lib.sagebwd_cache_read(null, 1, null, null, ctypes.byref(p), one, one, one, null) == -1
    plan = lambda held=one, R=1, columns=1, page=32, capacity=1, rows=1, stack=one, slots=one: lib.sagebwd_cache_plan(  # noqa: E731
        held, one, one, stack, one, R, columns, page, capacity, rows, slots, one, one, one, one, one, null)
    assert plan(held=null) == -1 and plan(R=-1) == -1 and plan(columns=0) == -1 and plan(page=33) == -2 and plan(stack=null) == -1
    assert plan(slots=null) == -1 and plan(columns=1 << 28) == -2 and plan(R=1 << 21) == -2 and plan(rows=-1) == -1
    trim = lambda R=1, keep=one, page=32: lib.sagebwd_cache_trim(keep, one, one, one, one, R, 1, page, 1, null)  # noqa: E731
    assert trim(R=-1) == -1 and trim(keep=null) == -1 and trim(page=31) == -2 and trim(R=0) == 0
    r = lambda **kw: Rotary(**{**dict(B=1, N=1, Hq=1, Hk=0, d=64, rotary_dim=64, axes=1, sections=(32, 0, 0, 0)), **kw})  # noqa: E731
    rotate = lambda p, q=one, f=one: lib.sagebwd_rotary(q, null, one, null, one, f, ctypes.byref(p), null)  # noqa: E731
    assert rotate(r(), q=null) == -1 and rotate(r(), f=null) == -1 and rotate(r(Hk=1)) == -1 and rotate(r(), q=_vp(8)) == -1
    assert rotate(r(sections=(31, 0, 0, 0))) == -1 and rotate(r(axes=5)) == -1 and rotate(r(axes=2, sections=(40, -8, 0, 0))) == -1
    assert rotate(r(d=72)) == -2 and rotate(r(rotary_dim=80)) == -2 and rotate(r(rotary_dim=24, sections=(12, 0, 0, 0))) == -2
    assert rotate(r(q=(0, 4, 8))) == -1 and rotate(r(N=0)) == 0 and rotate(r(inverse=2)) == -1


def test_tensors_of_other_types_shapes_and_places_are_refused(lib):
    p = CacheParams(H=2, d=64, page=32, group=32)
    i = torch.zeros(3, dtype=torch.int32)
    pool = cache.alloc_cache(p, 2, device="cpu")
    assert tuple(pool.shape) == (2, 2, 32 * 72)
    K = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="held: need contiguous cuda"):
        cache.sagebwd_cache_plan(i, i, i[None], i, i[:1], p, 3)
    with pytest.raises(ValueError, match="keep"):
        cache.sagebwd_cache_trim(i, i, i[None], i, i[:1], p)
    with pytest.raises(ValueError, match="cache: need contiguous cuda"):
        cache.sagebwd_cache_append(K, K, torch.zeros(3, dtype=torch.int64), pool, p)
    with pytest.raises(ValueError, match="cache"):
        cache.sagebwd_cache_read(torch.zeros(3, dtype=torch.int64), pool, p)
    with pytest.raises(ValueError, match="cache"):
        cache.sagebwd_cache_attention(K, pool, i[None], i[:1], i[:2], p, 1)
    with pytest.raises(TypeError):
        cache.sagebwd_cache_attention(K, None, i[None], i[:1], i[:2], p, 1)
    for bad in (CacheParams(H=2, d=80), CacheParams(H=2, d=64, page=20), CacheParams(H=0, d=64)):
        with pytest.raises(binding.SageError):
            cache.sagebwd_cache_append(K, K, i, pool, bad)
    with pytest.raises(ValueError, match="out of range"):
        cache.cache_workspace_bytes(p, -1, 1, 2, 1, 1)
    with pytest.raises(binding.SageError):
        cache.cache_workspace_bytes(p, 1, 1, 3, 1, 1)       # three query heads for two
    assert cache.cache_workspace_bytes(p, 4, 4, 4, 10, 1) > 0
    f = torch.ones(32)
    with pytest.raises(ValueError, match="Q: need cuda"):
        sage_rotary(K, None, i, f)
    with pytest.raises(TypeError):
        sage_rotary(None, K, i, f)


def test_rotary_refuses_what_it_has_no_derivative_for(lib):
    import torch.autograd.forward_ad as fwAD
    x, f, pos = torch.randn(4, 2, 64).to(torch.bfloat16), torch.ones(32), torch.arange(4)
    with fwAD.dual_level():
        with pytest.raises(NotImplementedError):
            sage_rotary(fwAD.make_dual(x, torch.ones_like(x)), None, pos, f)
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda a: sage_rotary(x, a, pos, f)[0].float().sum())(x)


@pytest.mark.gpu
def test_device_tensors_that_do_not_fit(lib):
    p = CacheParams(H=2, d=64, page=32, group=32)
    cu = dict(device="cuda")
    pool, i32 = cache.alloc_cache(p, 2), dict(dtype=torch.int32, device="cuda")
    Q, cu1 = torch.zeros(3, 4, 64, dtype=torch.bfloat16, **cu), torch.zeros(2, **i32)
    table, lengths = torch.zeros(1, 2, **i32), torch.zeros(1, **i32)
    ok = dict(Q=Q, cache=pool, block_table=table, lengths=lengths, cu=cu1, p=p, max_new=1)
    cache.sagebwd_cache_attention(**ok)
    for k, bad, match in (("Q", Q.float(), "Q"), ("Q", Q[..., :32], "Q"), ("Q", Q.transpose(1, 2).contiguous().transpose(1, 2), "adjacent"), ("Q", Q[:, 0], "Q"),
                          ("Q", torch.zeros(3, 4, 68, dtype=torch.bfloat16, **cu)[..., 4:], "16 bytes"), ("cache", pool[:, :1], "cache"),
                          ("cache", pool.view(torch.int8), "cache"), ("block_table", table.long(), "block_table"), ("block_table", torch.zeros(1, 4, **i32)[:, ::2], "block_table"),
                          ("lengths", torch.zeros(2, **i32), "block_table|cu"), ("cu", lengths, "cu"), ("cu", cu1.cpu(), "cu"), ("max_new", 0, "max_new"),
                          ("v_mean", torch.zeros(2, 32, **cu), "v_mean"), ("O", torch.zeros(3, 4, 64, **cu), "O"), ("LSE", torch.zeros(3, 4, **cu), "LSE"),
                          ("max_length", -1, "max_length")):
        with pytest.raises(ValueError, match=match):
            cache.sagebwd_cache_attention(**{**ok, k: bad})
    with pytest.raises(binding.SageError):
        cache.sagebwd_cache_attention(**{**ok, "Q": Q[:, :3].contiguous()})
    with pytest.raises(ValueError, match="slots"):
        cache.sagebwd_cache_append(Q[:, :2], Q[:, 2:], cu1, pool, p)
    with pytest.raises(ValueError, match="free_count"):
        cache.sagebwd_cache_plan(lengths, lengths, table, lengths, cu1, p, 1)
    f = torch.ones(32, **cu)
    for args, kw, match in (((Q, None, torch.zeros(2, **i32), f), {}, "positions"), ((Q, None, torch.zeros(3, **cu), f), {}, "positions"),
                            ((Q, None, torch.zeros(3, **i32), f), dict(sections=[31]), "sections"), ((Q, None, torch.zeros(3, **i32), f), dict(sections=[]), "sections"),
                            ((Q, Q[:2], torch.zeros(3, **i32), f), {}, "K"), ((Q, Q.float(), torch.zeros(3, **i32), f), {}, "K"),
                            ((Q, None, torch.zeros(3, **i32), f.double()), {}, "inv_freq"), ((Q[0], None, torch.zeros(3, **i32), f), {}, "Q")):
        with pytest.raises(ValueError, match=match):
            sage_rotary(*args, **kw)
    with pytest.raises(binding.SageError):
        sage_rotary(Q, None, torch.zeros(3, **i32), torch.ones(40, **cu))        # more frequencies than the channels have pairs


def test_calls_larger_than_a_launch_are_refused(lib):
    """A launch has at most 2^31 threads, and 65535 workgroups along y: more is an unsupported shape, not an error of the runtime."""
    i64, one, null = ctypes.c_int64, _vp(256), _vp(None)
    p = cache._CCacheParams(1024, 128, 64, 64, 4, 0)
    T = 1 << 17        # 2^17 tokens x 1024 heads x 16 threads
    assert lib.sagebwd_cache_append(one, one, i64(0), i64(128), i64(0), i64(128), one, T + 1, null, null, ctypes.byref(p), one, null) == -2
    assert lib.sagebwd_cache_read(one, T + 1, null, null, ctypes.byref(p), one, one, one, null) == -2
    # 2^22 row tiles of 512 threads each: 2^20 requests of 2 tokens x 64 heads of the group, 4 key/value heads, and one tile more
    p = cache._CCacheParams(4, 64, 32, 64, 4, 0)
    need = lambda R, T, G, new: lib.sagebwd_cache_workspace_bytes(  # noqa: E731
        ctypes.byref(p), ctypes.byref(Call(R, T, 4 * G, 1, new, 0, 1, 0.0, 256, 64)), ctypes.byref(ctypes.c_size_t()))
    assert need((1 << 20) - 512, 2048, 64, 2) == 0 and need(1 << 20, 2048, 64, 2) == -2
    assert need(1 << 20, 2048, 8, 4) == 0         # (32 rows: no request has the kernel with those tiles)
    x = Rotary(1, 1, 40000, 30000, 16, 16, 1)
    x.sections[0] = 8
    for s in (x.q, x.k, x.qo, x.ko):
        s[0] = s[1] = 0
        s[2] = 16
    assert lib.sagebwd_rotary(one, one, one, one, one, one, ctypes.byref(x), null) == -2
