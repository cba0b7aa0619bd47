"""The cache held in 8 bits where calls are at their edges: slots in any order, more new tokens than the call computes, widest groups, no LSE, several
calls in a graph."""
import ctypes

import numpy as np
import pytest
import torch

import serve8_ref as ref8
import serve_ref as ref
from paper_2603_02170_amd import binding, cache
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache8 import Filled, _attend, _check, _i32, _np, _randn, _slots
from test_serve_refusals import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,block,H,T", [(64, 32, 3, 5000), (128, 64, 2, 3000), (128, 32, 1, 40), (64, 64, 16, 700)])
def test_blocks_in_any_order_and_slots_read_in_any_order(d, block, H, T):
    """Runs of one to a whole block's tokens at the fronts of blocks that lie anywhere, then more of each behind them; every second slot read, backwards,
    some twice, some that are none."""
    g, rng = torch.Generator().manual_seed(T), np.random.default_rng(T)
    p = CacheParams(H=H, d=d, page=64, block=block)
    blocks, model = T // 10 + 5, ref8.Pages(H, d, 64, block)
    pool = torch.full(tuple(cache.alloc_cache(p, blocks * block // 64 + 1).shape), 0xFF, dtype=torch.uint8, device="cuda")
    held = {}
    for call in range(2):
        slots = []
        for b in rng.permutation(blocks):
            o = held.get(b, 0)
            n = min(int(rng.choice([1, 1, 2, 9, block])), block - o)
            if n > 0 and len(slots) + n <= T:
                slots += list(range(b * block + o, b * block + o + n))
                held[b] = o + n
        K, V = _randn((len(slots), H, d), g), _randn((len(slots), H, d), g)
        cache.sagebwd_cache_append(K.cuda(), V.cuda(), _slots(slots), pool, p)
        model.append(_np(K), _np(V), slots)
    stored = [b * block + t for b in held for t in range(held[b])]
    want = stored[::-2] + stored[:7] + stored[:7]
    none = [-1, 1 << 50, -(1 << 60)]
    Kr, Vr = cache.sagebwd_cache_read(_slots(want[:11] + none + want[11:]), pool, p)
    for got, which in ((Kr, 0), (Vr, 1)):
        got, values = _np(got), ref.bf16_round(model.gather(want, which, "read"))
        assert np.array_equal(got[:11], values[:11]) and (got[11:14] == 0).all() and np.array_equal(got[14:], values[11:])


@pytest.mark.parametrize("n,most,Hq,L,d", [(9, 4, 2, 90, 64), (9, 4, 16, 1300, 128), (40, 25, 8, 700, 128), (300, 150, 4, 500, 64), (5, 1, 4, 9000, 128)])
def test_new_tokens_beyond_the_bound_are_not_computed(n, most, Hq, L, d):
    g = torch.Generator().manual_seed(n)
    f = Filled([L, 33], CacheParams(H=2, d=d, page=32, block=32), g)
    q = _randn((n + 1, Hq, d), g)
    O, lse = torch.full((n + 1, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((Hq, n + 1), 7.0, device="cuda")
    cache.sagebwd_cache_attention(q.cuda(), f.pool, f.table, f.lengths, _i32([0, n, n + 1]), f.p, most, O=O, LSE=lse)
    assert (O[most:n] == 7).all() and (lse[:, most:n] == 7).all()
    want, wl = cache.sagebwd_cache_attention(q.cuda(), f.pool, f.table, f.lengths, _i32([0, n, n + 1]), f.p, n)
    _check(f, q, [0, n, n + 1], want, wl, True)
    keep = list(range(most)) + [n]
    assert (O[keep].float() - want[keep].float()).abs().max() <= 2.0 ** -6 * want.float().abs().max() and (lse[:, keep] - wl[:, keep]).abs().max() < 1e-4


@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("d,L", [(64, 50), (128, 900), (128, 5000)])
def test_the_widest_groups(n, d, L):
    g = torch.Generator().manual_seed(n * d)
    f = Filled([L, 1, L // 2], CacheParams(H=1, d=d, page=64, block=64), g)
    q, cu, O, lse = _attend(f, [n, 1, n], 64, g)
    _check(f, q, cu, O, lse, True)


@pytest.mark.parametrize("lens,news,Hq", [([100, 20], [1, 1], 4), ([600, 70], [2, 1], 8), ([5000, 70], [9, 1], 8), ([900], [200], 4), ([3000], [520], 8)])
def test_no_lse_is_written_where_none_is_asked_for(lens, news, Hq):
    """The C call without LSE in every form: O's bits are the same."""
    g = torch.Generator().manual_seed(sum(lens))
    p = CacheParams(H=2, d=128, page=64, block=32)
    f = Filled(lens, p, g)
    q, cu, O, lse = _attend(f, news, Hq, g)
    lib, T = binding.load_library(), sum(news)
    cp, call = cache._CCacheParams(2, 128, 64, 0, f.pool.shape[0], 32), Call(len(lens), T, Hq, f.table.shape[1], max(news), 0, 1, 0.0, Hq * 128, 128)
    ws = torch.empty(cache.cache_workspace_bytes(p, len(lens), T, Hq, f.table.shape[1], max(news)) + 256, dtype=torch.uint8, device="cuda")
    out, dq, dcu = torch.zeros_like(O), q.cuda(), _i32(cu)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    torch.cuda.synchronize()
    rc = lib.sagebwd_cache_attention(ptr(dq), ptr(f.pool), ptr(f.table), ptr(f.lengths), ptr(dcu), None, ctypes.byref(cp), ctypes.byref(call), ptr(out), None,
                                     ptr(ws), ctypes.c_size_t(ws.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert rc == 0 and torch.equal(out, O)


def test_prompts_and_decoding_in_one_captured_graph_with_other_work_between_replays():
    """Two attentions of different forms and an append in a graph, each with a workspace of its own, replayed between eager calls."""
    g = torch.Generator().manual_seed(9)
    p = CacheParams(H=2, d=128, page=64, block=64)
    f, other = Filled([2000, 700], p, g), Filled([3000], p, g)
    q1, q2 = _randn((2, 8, 128), g).cuda(), _randn((530, 8, 128), g).cuda()
    cu1, cu2 = _i32([0, 1, 2]), _i32([0, 530])
    K = _randn((2, 2, 128), g).cuda()
    ends = [f.slots[1999], f.slots[-1]]            # the two last tokens are written again
    slots = _slots(ends)

    def work():
        cache.sagebwd_cache_append(K, K, slots, f.pool, p)
        a = cache.sagebwd_cache_attention(q1, f.pool, f.table, f.lengths, cu1, p, 1)
        b = cache.sagebwd_cache_attention(q2, other.pool, other.table, other.lengths, cu2, p, 530)
        return a + b

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for i in range(5):
        q1.copy_(_randn((2, 8, 128), g))
        q2.copy_(_randn((530, 8, 128), g))
        K.copy_(_randn((2, 2, 128), g, 0.5))       # (below the block's magnitude: its other codes stay)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = work()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("R,n,G,H,d,block", [(16, 1, 4, 8, 128, 64), (9, 16, 1, 16, 64, 32), (48, 2, 3, 24, 64, 64), (5, 30, 2, 14, 128, 32), (2, 100, 1, 16, 64, 64)])
def test_many_undivided_requests(R, n, G, H, d, block):
    """Up to 1536 tokens are walked in one go where requests and heads fill half of the machine, by a workgroup an item or a wave an item; requests
    of one token, and one without new ones, in between."""
    g, rng = torch.Generator().manual_seed(R * n), np.random.default_rng(R)
    p = CacheParams(H=H, d=d, page=64, block=block)
    base = Filled([1536], p, g, spare_columns=0)       # (its pages are every request's)
    lens = [1536 - int(x) for x in rng.integers(0, 1536 - n, R)]
    news = [int(x) for x in rng.integers(1, n + 1, R)]
    lens[0], news[0], lens[-1] = 1536, n, news[-1]
    lens[R // 2] = 1 if news[R // 2] == 1 else lens[R // 2]
    if R > 8:
        news[3] = 0
    q = _randn((sum(news), H * G, d), g)
    cu = np.concatenate([[0], np.cumsum(news)]).astype(int).tolist()
    for causal in (True, False):
        O, lse = cache.sagebwd_cache_attention(q.cuda(), base.pool, base.table.expand(R, -1).contiguous(), _i32(lens), _i32(cu), p, n, causal=causal)
        again = cache.sagebwd_cache_attention(q.cuda(), base.pool, base.table.expand(R, -1).contiguous(), _i32(lens), _i32(cu), p, n, causal=causal)
        assert torch.equal(O, again[0]) and torch.equal(lse, again[1])
        for r in sorted({0, R // 2, R - 1, int(rng.integers(0, R))}):
            a, b = cu[r], cu[r + 1]
            for h in (0, H - 1):
                if a == b:
                    continue
                one = type("One", (), dict(p=p, lens=[lens[r]], k=base.k[:lens[r], h:h + 1], v=base.v[:lens[r], h:h + 1], at=[0, lens[r]]))
                heads = slice(h * G, h * G + G)
                _check(one, q[a:b, heads], [0, b - a], O[a:b, heads], lse[heads, a:b], causal)
