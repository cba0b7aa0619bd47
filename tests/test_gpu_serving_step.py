"""The operators of serving together, as a decoding loop runs them: plan, rotary positions, append, attention; eager and captured."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_02170_amd import binding, cache
from paper_2603_02170_amd.autograd import sage_rotary
from paper_2603_02170_amd.cache import CacheParams

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Loop:
    """A serving loop's state, and beside it, in float64, every request's tokens as they were handed over."""

    def __init__(self, R, p, Hq, columns, pages, k_mean=None, v_mean=None):
        self.R, self.p, self.Hq = R, p, Hq
        self.lengths, self.table = _i32([0] * R), torch.full((R, columns), -1, dtype=torch.int32, device="cuda")
        self.free_pages, self.free_count = _i32(list(range(pages))), _i32([pages])
        self.pool = torch.full(tuple(cache.alloc_cache(p, pages).shape), 0xFF, dtype=torch.uint8, device="cuda")
        self.inv_freq = (10000.0 ** (-torch.arange(p.d // 2, dtype=torch.float64) / (p.d // 2))).float().cuda()
        self.k_mean, self.v_mean = k_mean, v_mean
        self.kept = [(np.zeros((0, p.H, p.d)), np.zeros((0, p.H, p.d))) for _ in range(R)]

    def step(self, qkv, added, rows, max_new):
        p, H, Hq = self.p, self.p.H, self.Hq
        plan = cache.sagebwd_cache_plan(self.lengths, added, self.table, self.free_pages, self.free_count, p, rows)
        Q, K = sage_rotary(qkv[:, :Hq], qkv[:, Hq:Hq + H], plan.positions, self.inv_freq)
        V = qkv[:, Hq + H:]
        cache.sagebwd_cache_append(K, V, plan.slots, self.pool, p, k_mean=self.k_mean, v_mean=self.v_mean)
        O, lse = cache.sagebwd_cache_attention(Q, self.pool, self.table, plan.lengths, plan.cu_new, p, max_new, v_mean=self.v_mean)
        self.lengths.copy_(plan.lengths)
        self.free_count.copy_(plan.free_left)
        return O, lse, Q, K, V

    def check(self, added, O, lse, Q, K, V):
        """Against exact attention on the quantised keys and values.  (Tolerances as in test_gpu_cache.)"""
        at = 0
        for r, n in enumerate(added):
            k, v = _np(K[at:at + n]).astype(np.float32), _np(V[at:at + n]).astype(np.float32)
            if self.k_mean is not None:
                k, v = k - _np(self.k_mean).astype(np.float32), v - _np(self.v_mean).astype(np.float32)
            kept = self.kept[r] = (np.concatenate([self.kept[r][0], ref.quantise(k, self.p.group)[2]]),
                                   np.concatenate([self.kept[r][1], ref.quantise(v, self.p.group)[2]]))
            q, scale = _np(Q[at:at + n]), self.p.d ** -0.5
            want, wl, A = ref.attention(q, *kept, n, True, scale, None if self.v_mean is None else _np(self.v_mean))
            s = max(np.abs(kept[0]).max(), np.abs(kept[1]).max()) / 7 * 17 / 16 if kept[0].size else 0
            e = scale * 8 * 2.0 ** -24 * 32 * s * np.abs(q).sum(-1) + 2.0 ** -18
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * e[..., None]) * A + 32 * s * 2 * 2.0 ** -24 * (len(kept[0]) / 32 + 1)
            assert (np.abs(_np(O[at:at + n]) - want) <= tol).all(), r
            assert (np.abs(_np(lse[:, at:at + n]) - wl) <= e.T + 2.0 ** -22 * (1 + np.abs(wl))).all(), r
            at += n


@pytest.mark.parametrize("d,group,page,Hq,H,mean", [(128, 64, 32, 8, 2, False), (64, 32, 64, 3, 3, True)])
def test_prompts_chunks_and_decoding(d, group, page, Hq, H, mean):
    g = torch.Generator().manual_seed(d)
    R, p = 5, CacheParams(H=H, d=d, page=page, group=group)
    means = [0.5 * torch.randn((H, d), generator=g).cuda() for _ in range(2)] if mean else [None, None]
    loop = Loop(R, p, Hq, columns=12, pages=60, k_mean=means[0], v_mean=means[1])
    for added in ([40, 0, 130, 7, 0], [1, 65, 1, 1, 0], [1, 1, 1, 1, 3], [1, 4, 1, 60, 1], [1, 1, 1, 1, 1], [1, 1, 1, 1, 1]):
        rows = sum(added)
        qkv = torch.randn((rows, Hq + 2 * H, d), generator=g).to(torch.bfloat16).cuda()
        loop.check(added, *loop.step(qkv, _i32(added), rows, max(added)))
    # a request ends and another one takes its place and its pages; a drafted token is taken back
    lens = loop.lengths.tolist()
    cache.sagebwd_cache_trim(_i32([lens[0] - 1, 0, lens[2], lens[3], lens[4]]), loop.lengths, loop.table, loop.free_pages, loop.free_count, p)
    loop.kept[0] = tuple(x[:-1] for x in loop.kept[0])
    loop.kept[1] = tuple(x[:0] for x in loop.kept[1])
    for added in ([2, 33, 1, 1, 1], [1, 1, 1, 1, 1]):
        qkv = torch.randn((sum(added), Hq + 2 * H, d), generator=g).to(torch.bfloat16).cuda()
        loop.check(added, *loop.step(qkv, _i32(added), sum(added), max(added)))
    assert sorted(loop.free_pages[:loop.free_count].tolist() + [x for row in loop.table.tolist() for x in row if x >= 0]) == list(range(60))


def test_a_request_without_pages_writes_and_changes_nothing():
    g = torch.Generator().manual_seed(1)
    p = CacheParams(H=1, d=64, page=32)
    loop = Loop(3, p, 2, columns=4, pages=3)
    qkv = torch.randn((60, 4, 64), generator=g).to(torch.bfloat16).cuda()
    loop.check([20, 20, 20], *loop.step(qkv, _i32([20, 20, 20]), 60, 20))
    pool = loop.pool.clone()
    qkv = torch.randn((16 + 14 + 1, 4, 64), generator=g).to(torch.bfloat16).cuda()
    loop.step(qkv, _i32([16, 14, 1]), 31, 16)        # no page is left for the first two; the third needs none
    assert loop.lengths.tolist() == [20, 20, 21] and loop.free_count.item() == 0
    for r in range(2):
        assert torch.equal(loop.pool[loop.table[r, 0].item()], pool[loop.table[r, 0].item()])
    assert not torch.equal(loop.pool[loop.table[2, 0].item()], pool[loop.table[2, 0].item()])


def test_a_captured_step_replayed_against_the_eager_one():
    """Decoding in a graph: plan, rotary, append and attention are replayed on what the replay before left."""
    g = torch.Generator().manual_seed(5)
    R, Hq, p = 4, 8, CacheParams(H=2, d=128, page=32)
    loops = [Loop(R, p, Hq, columns=40, pages=120) for _ in range(2)]
    prompt = [100, 31, 700, 64]
    qkv = torch.randn((sum(prompt), Hq + 4, 128), generator=g).to(torch.bfloat16).cuda()
    for loop in loops:
        loop.step(qkv, _i32(prompt), sum(prompt), max(prompt))
    one = _i32([1] * R)
    new = torch.randn((R, Hq + 4, 128), generator=g).to(torch.bfloat16).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):            # (warms up; its token is taken back)
        loops[0].step(new, one, R, 1)
        cache.sagebwd_cache_trim(_i32(prompt), loops[0].lengths, loops[0].table, loops[0].free_pages, loops[0].free_count, p)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, lse, *_ = loops[0].step(new, one, R, 1)
    for step in range(40):                   # (across the ends of pages)
        new.copy_(torch.randn((R, Hq + 4, 128), generator=g).to(torch.bfloat16))
        graph.replay()
        want, wl, *_ = loops[1].step(new, one, R, 1)
        torch.cuda.synchronize()
        assert torch.equal(O, want) and torch.equal(lse, wl), step
        assert torch.equal(loops[0].lengths, loops[1].lengths) and torch.equal(loops[0].table, loops[1].table)
        assert torch.equal(loops[0].free_count, loops[1].free_count)


def test_the_prompt_through_the_int8_forward_and_the_smoothing_means():
    """The means that the INT8 forward's pre-pass smooths K by go into the cache's quantiser; decoding over it then agrees with exact attention
    on the keys themselves as far as 4 bits do, and better than without the means."""
    g = torch.Generator().manual_seed(6)
    H, d, N = 2, 128, 512
    p = CacheParams(H=H, d=d)
    Q, V = (torch.randn((1, H, N, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    K = (torch.randn((1, H, N, d), generator=g) + 6 * torch.randn((1, H, 1, d), generator=g)).to(torch.bfloat16).cuda()
    sp = binding.SageParams(1, H, N, d)
    ws = binding.alloc_workspace(sp)
    binding.sagebwd_fwd(Q, K, V, sp, ws)
    k_mean, _, _ = binding.sagebwd_export_stats(sp, ws)
    err = []
    for mean in (None, k_mean[0].contiguous()):
        pool = cache.alloc_cache(p, N // p.page)
        slots = torch.arange(N, device="cuda")
        cache.sagebwd_cache_append(K[0].transpose(0, 1), V[0].transpose(0, 1), slots, pool, p, k_mean=mean)
        q = Q[0, :, -1:].transpose(0, 1).contiguous()
        O, _ = cache.sagebwd_cache_attention(q, pool, torch.arange(N // p.page, device="cuda", dtype=torch.int32)[None], _i32([N]), _i32([0, 1]), p, 1)
        want, _, _ = ref.attention(_np(q), _np(K[0].transpose(0, 1)), _np(V[0].transpose(0, 1)), 1, True, d ** -0.5)
        err.append(np.linalg.norm(_np(O) - want) / np.linalg.norm(want))
    assert err[1] < 0.5 * err[0]
