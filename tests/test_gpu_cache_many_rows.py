"""Attention over the 4-bit cache of many query rows a request: prompts, chunks, batches that mix them with decoding.

Which kernels a call takes goes by its sizes (query rows = new tokens x query heads of a key/value head): up to 32 rows, more, or at least 2048 with the
keys and values unpacked beforehand; and by how many row tiles of 256 there are a request's keys are divided or not."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_02170_amd import cache
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache import Filled, _attend, _i32, _np, _randn

pytestmark = pytest.mark.gpu


def _check_rows(f, q, cu, O, lse, causal, rows, v_mean=None):
    """The given rows of Q against 64 bits; tolerances as in test_gpu_cache._check."""
    d, H = f.p.d, f.p.H
    G = q.shape[1] // H
    for t in rows:
        r = int(np.searchsorted(cu, t, side="right")) - 1
        n, L, i = cu[r + 1] - cu[r], f.lens[r], t - cu[r]
        sees = max(0, min(L, L - n + i + 1)) if causal else L
        k, v = f.k[f.at[r]:f.at[r] + sees], f.v[f.at[r]:f.at[r] + sees]
        want, wl, A = ref.attention(_np(q[t:t + 1]).astype(np.float64), k, v, 1, False, d ** -0.5, None if v_mean is None else _np(v_mean))
        got, gl = _np(O[t]).astype(np.float64), lse[:, t].cpu().numpy().astype(np.float64)
        if sees == 0:
            assert (got == 0).all() and np.isneginf(gl).all()
            continue
        s = max(np.abs(k).max(), np.abs(v).max()) / 7 * 17 / 16
        e = d ** -0.5 * 8 * 2.0 ** -24 * 32 * s * np.abs(_np(q[t])).sum(-1) + 2.0 ** -18
        tol = 2.0 ** -8 * np.abs(want[0]) + (2.0 ** -8 + 2 * e[:, None]) * A[0] + 32 * s * 2 * 2.0 ** -24 * (L / 32 + 1)
        assert (np.abs(got - want[0]) <= tol).all(), (t, r, float((np.abs(got - want[0]) / tol).max()))
        assert (np.abs(gl - wl[:, 0]) <= e + 2.0 ** -22 * (1 + np.abs(wl[:, 0]))).all(), (t, r)


def _some(cu, g, n=40):
    T = cu[-1]
    edges = [t + k for t in cu for k in (-1, 0, 1) if 0 <= t + k < T]
    return sorted(set(edges[:30] + torch.randint(0, T, (n,), generator=g).tolist()))


@pytest.mark.parametrize("lens,news,Hq,H,d,group,page", [
    ([1500], [700], 8, 2, 128, 64, 64),                                   # unpacked beforehand, keys divided
    ([2100, 2049], [2100, 2049], 3, 3, 64, 32, 32),
    ([900, 3000], [600, 2], 8, 2, 128, 32, 128),                          # beside a request with few rows
    ([40, 5000, 700, 1, 0, 64], [1, 800, 300, 1, 1, 40], 12, 4, 64, 64, 256),
    ([4100], [4100], 64, 2, 64, 64, 64),                                  # so many row tiles that none is divided
    ([70 + r for r in range(300)], [20] * 300, 64, 4, 64, 32, 32),        # the same, unpacked by every tile
    ([33 + 7 * r for r in range(40)], [33] * 40, 5, 5, 128, 64, 32),
    ([3000], [9], 64, 1, 128, 64, 64),                                    # 64 query heads for one
    ([600, 20], [500, 30], 7, 7, 128, 32, 64),                            # a request shorter than its new tokens
    ([45] * 600 + [300], [1] * 600 + [300], 4, 4, 64, 64, 32),            # more requests than threads
])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_against_64_bits(lens, news, Hq, H, d, group, page, causal):
    g = torch.Generator().manual_seed(sum(news) + d)
    f = Filled(lens, CacheParams(H=H, d=d, page=page, group=group), g)
    v_mean = torch.randn((H, d), generator=g).cuda() if page == 64 else None
    q, cu, O, lse = _attend(f, news, Hq, g, causal=causal, v_mean=v_mean)
    assert torch.isfinite(O).all()
    _check_rows(f, q, cu, O, lse, causal, _some(cu, g), v_mean)


@pytest.mark.parametrize("n,L,G,d,group,page", [(2100, 2300, 1, 128, 64, 32), (1100, 1100, 2, 64, 32, 64), (300, 900, 4, 128, 32, 128), (700, 700, 1, 64, 64, 256)])
def test_every_token_is_weighed_alone(n, L, G, d, group, page):
    """Every query row points at one key so sharply that its value alone comes out; the rows between them at every key."""
    g = torch.Generator().manual_seed(L)
    f = Filled([L], CacheParams(H=1, d=d, page=page, group=group), g)
    target = (torch.randperm(n * G, generator=g) % L).reshape(n, G)
    q = torch.tensor(f.k[:, 0])[target] * 8
    _, _, O, _ = _attend(f, [n], G, g, causal=False, sm_scale=1.0, q=q.to(torch.bfloat16))
    want = torch.tensor(f.v[:, 0])[target]
    assert (O.double().cpu() - want).abs().max() <= 2.0 ** -7 * want.abs().max()


@pytest.mark.parametrize("n,L", [(2200, 2400), (300, 900)])
def test_the_mask_hides_what_is_not_a_number(n, L):
    g = torch.Generator().manual_seed(n)
    f = Filled([L, 64], CacheParams(H=2, d=128, page=32), g)
    bad_k, bad_v = L - 50, L - 130
    f.K[bad_k, 0, 3], f.V[bad_v, 1, 70] = float("nan"), float("inf")
    f.store()
    q, cu, O, lse = _attend(f, [n, 1], 2, g)
    first_k, first_v = bad_k - (L - n), bad_v - (L - n)        # the first rows that see them
    O = O.float().cpu()
    assert torch.isnan(O[first_k:n, 0]).all() and torch.isfinite(O[:first_k, 0]).all()
    assert torch.isnan(O[first_v:n, 1, 64:]).all() and torch.isfinite(O[first_v:n, 1, :64]).all() and torch.isfinite(O[:first_v, 1]).all()
    assert torch.isfinite(O[n]).all()
    f.k, f.v = np.nan_to_num(f.k), np.nan_to_num(f.v)
    _check_rows(f, q, cu, O, lse, True, [0, first_v - 1, n])


@pytest.mark.parametrize("n", [2200, 200])
def test_pages_that_do_not_exist(n):
    g = torch.Generator().manual_seed(n)
    L = n + 300
    f = Filled([L], CacheParams(H=1, d=64, page=32), g)
    q = _randn((n, 1, 64), g)
    gone = [2, 3, 7, (L - 1) // 32]
    f.table[0, gone[0]], f.table[0, gone[1]], f.table[0, gone[2]], f.table[0, gone[3]] = -1, f.pool.shape[0], -(1 << 31), 1 << 30
    _, cu, O, lse = _attend(f, [n], 1, g, causal=False, q=q)
    keep = np.array([t for t in range(L) if t // 32 not in gone])
    f.k, f.v, f.lens, f.at = f.k[keep], f.v[keep], [len(keep)], [0, len(keep)]
    _check_rows(f, q, cu, O, lse, False, [0, 1, 31, 32, n // 2, n - 1])


def test_one_workspace_for_calls_of_every_kind_and_replays():
    g = torch.Generator().manual_seed(3)
    p = CacheParams(H=2, d=128)
    calls = []
    for lens, news in (([3000, 40], [1, 1]), ([2500], [600]), ([500, 900], [100, 3]), ([8000], [1]), ([2500, 2000], [520, 1])):
        f = Filled(lens, p, g)
        q, cu, O, lse = _attend(f, news, 8, g)
        calls.append((f, q.cuda(), _i32(cu), max(news), O, lse))
    size = max(cache.cache_workspace_bytes(p, len(f.lens), q.shape[0], 8, f.table.shape[1], m) for f, q, cu, m, O, lse in calls)
    ws = torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda")
    run = lambda: [cache.sagebwd_cache_attention(q, f.pool, f.table, f.lengths, cu, p, m, workspace=ws) for f, q, cu, m, _, _ in calls]  # noqa: E731
    for _ in range(2):
        for (O, lse), c in zip(run(), calls):
            assert torch.equal(O, c[4]) and torch.equal(lse, c[5])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for step in range(3):
        for c in calls:
            c[1].mul_(0.5)
        ws.fill_(0xFF if step == 1 else 0)
        graph.replay()
        torch.cuda.synchronize()
        for (O, lse), c in zip(out, calls):
            want = cache.sagebwd_cache_attention(c[1], c[0].pool, c[0].table, c[0].lengths, c[2], p, c[3])
            assert torch.equal(O, want[0]) and torch.equal(lse, want[1])


def test_offsets_that_do_not_rise_stay_within_the_tensors():
    """What `cu` says is bounded by the rows of Q: the results mean nothing then, and nothing else is touched."""
    g = torch.Generator().manual_seed(4)
    p = CacheParams(H=1, d=64, page=32)
    f = Filled([600] * 6, p, g)
    T = 640
    q = _randn((T, 4, 64), g).cuda()
    before = f.pool.clone()
    for cu in ([0, T, 0, T, 0, T, 0], [T, T, T, T, T, T, T], [0, -5, 1 << 30, 3, 2, 1, 0], [-(1 << 31), (1 << 31) - 1, 0, 0, 0, 0, 0]):
        for m in (1, 100, T):
            O, lse = cache.sagebwd_cache_attention(q, f.pool, f.table, f.lengths, _i32(cu), p, m)
            torch.cuda.synchronize()
            assert O.shape == (T, 4, 64)
    assert torch.equal(f.pool, before)
    O, lse = cache.sagebwd_cache_attention(q, f.pool, f.table, f.lengths, _i32([0, 100, 200, 201, 300, 301, T]), p, 400)
    _check_rows(f, q.cpu(), [0, 100, 200, 201, 300, 301, T], O, lse, True, [0, 99, 200, 250, 300, T - 1])


def test_rows_behind_the_last_request_stay():
    g = torch.Generator().manual_seed(5)
    p = CacheParams(H=2, d=64, page=64)
    for lens, news in (([1500], [1100]), ([400], [200])):
        f = Filled(lens, p, g)
        T = sum(news) + 70
        q = _randn((T, 4, 64), g).cuda()
        O, lse = torch.full((T, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda"), torch.full((4, T), 5.0, device="cuda")
        cache.sagebwd_cache_attention(q, f.pool, f.table, f.lengths, _i32([0, news[0]]), p, news[0], O=O, LSE=lse)
        assert (O[news[0]:] == 5).all() and (lse[:, news[0]:] == 5).all()
        _check_rows(f, q.cpu(), [0, news[0]], O, lse, True, [0, 127, 128, news[0] - 1])


# ---- 33 to 128 rows a request: groups of 32 rows by tiles of 64 tokens in one workgroup ---------------------------------------
@pytest.mark.parametrize("lens,news,Hq,H,d,group,page", [
    ([700], [33], 2, 2, 128, 64, 64),                                     # one item, its keys divided over the machine
    ([257, 64, 65, 1, 0, 1000], [40, 33, 64, 1, 1, 50], 6, 6, 64, 32, 32),
    ([320, 300, 511, 513], [16, 9, 5, 13], 12, 3, 128, 32, 256),          # 64 rows and fewer, beside requests of few
    ([300 + 3 * r for r in range(70)], [64] * 70, 8, 8, 64, 64, 64),
    ([128, 900, 640], [128, 100, 65], 3, 3, 128, 64, 32),                 # up to 128
    ([3, 600, 20], [100, 127, 31], 4, 4, 64, 32, 128),                    # a request shorter than its new tokens
    ([290] * 600, [20] * 600, 12, 2, 128, 64, 32),                        # 120 rows; none divided
    ([270] * 520, [34] * 520, 2, 1, 64, 64, 64),
])
@pytest.mark.parametrize("causal", [True, False])
def test_up_to_128_rows_against_64_bits(lens, news, Hq, H, d, group, page, causal):
    g = torch.Generator().manual_seed(sum(news) + d + 1)
    f = Filled(lens, CacheParams(H=H, d=d, page=page, group=group), g)
    v_mean = torch.randn((H, d), generator=g).cuda() if page == 64 else None
    q, cu, O, lse = _attend(f, news, Hq, g, causal=causal, v_mean=v_mean, max_length=max(max(lens), 257))
    assert torch.isfinite(O).all()
    _check_rows(f, q, cu, O, lse, causal, _some(cu, g), v_mean)


@pytest.mark.parametrize("n,G,d,group", [(50, 1, 128, 64), (16, 8, 64, 32), (30, 4, 128, 32), (31, 2, 64, 64)])
def test_up_to_128_rows_every_token_is_weighed_alone(n, G, d, group):
    g, L = torch.Generator().manual_seed(n), 1000
    f = Filled([L], CacheParams(H=1, d=d, page=32, group=group), g)
    for part in range(-(-L // (n * G))):
        target = ((torch.arange(n * G) + part * n * G) % L).reshape(n, G)
        q = torch.tensor(f.k[:, 0])[target] * 8
        _, _, O, _ = _attend(f, [n], G, g, causal=False, sm_scale=1.0, q=q.to(torch.bfloat16))
        want = torch.tensor(f.v[:, 0])[target]
        assert (O.double().cpu() - want).abs().max() <= 2.0 ** -7 * want.abs().max()


@pytest.mark.parametrize("n", [40, 100])
@pytest.mark.parametrize("d,group", [(128, 64), (64, 32)])
def test_up_to_128_rows_what_is_not_a_number_and_pages_that_do_not_exist(n, d, group):
    """A NaN in one token's V reaches the rows that see it and the group's channels alone; a missing page is left out; every replay the same."""
    g, L, page = torch.Generator().manual_seed(n + d), 900, 64
    f = Filled([L], CacheParams(H=1, d=d, page=page, group=group), g)
    at = L - n // 2                                       # (half of the rows see it)
    f.V[at, 0, 3] = float("nan")
    cache.sagebwd_cache_append(f.K.cuda(), f.V.cuda(), f.slots, f.pool, f.p)
    table = f.table.clone()
    table[0, 5] = -1
    kept = np.r_[0:5 * page, 6 * page:L]
    q = _randn((n, 1, d), g)
    cu = _i32([0, n])
    O, lse = cache.sagebwd_cache_attention(q.cuda(), f.pool, table, f.lengths, cu, f.p, n)
    sees = torch.arange(n) + L - n + 1 > at
    nan = torch.isnan(O.cpu()).squeeze(1)
    assert nan[sees][:, :group].all() and not nan[~sees].any() and not nan[:, group:].any() and torch.isfinite(lse).all()
    v = f.v.copy()
    v[np.isnan(v)] = 0
    for i in (0, n // 4, n - 1):
        keys = kept[kept < L - n + i + 1]
        want, wl, A = ref.attention(_np(q[i:i + 1]).astype(np.float64), f.k[keys], v[keys], 1, False, d ** -0.5, None)
        got, ok = _np(O[i]).astype(np.float64), ~nan[i].numpy()
        # (roundings of O and of the probabilities, 2^-8 of each; logits and sums in FP32 below 2^-14)
        assert (np.abs(got - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + (2.0 ** -8 + 2.0 ** -13) * A[0] + 1e-5)[:, ok].all(), i
        assert abs(lse[0, i].item() - wl[0, 0]) <= 2.0 ** -14
    for _ in range(3):
        again, _ = cache.sagebwd_cache_attention(q.cuda(), f.pool, table, f.lengths, cu, f.p, n)
        assert torch.equal(again.view(torch.int16), O.view(torch.int16))


# ---- unpacked beforehand, at 128 channels: 4096 rows and more --------------------------------------------------------------
@pytest.mark.parametrize("lens,news,Hq,H,group,page", [([1500], [1100], 8, 2, 64, 64), ([1300, 900, 77], [1050, 3, 1], 8, 2, 32, 32),
                                                       ([4200, 4100], [4200, 4097], 1, 1, 64, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_4096_rows_and_more_of_128_channels(lens, news, Hq, H, group, page, causal):
    test_rows_against_64_bits(lens, news, Hq, H, 128, group, page, causal)


@pytest.mark.parametrize("group", [32, 64])
def test_4096_rows_every_token_is_weighed_alone(group):
    test_every_token_is_weighed_alone(4200, 4300, 1, 128, group, 32)


def test_4096_rows_masks_and_pages():
    test_the_mask_hides_what_is_not_a_number(4200, 4400)
    test_pages_that_do_not_exist(4200)
