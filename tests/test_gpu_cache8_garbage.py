"""The cache held in 8 bits over memory that held other things: whatever words stand where no token was stored, results have the bits that
they have over zeros.  (Small integers, as tables and slots are, read as positive numbers far below any magnitude that is stored.)"""
import pytest
import torch

from paper_2603_02170_amd import cache
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache8 import Filled, _attend, _check, _i32, _randn

pytestmark = pytest.mark.gpu

# 1, 5, 63; bytes of ones; 2^-126; about 3.7e-37 and below it; just below and at the least magnitude stored, 2^-100; large and largest numbers; an infinity, a NaN
WORDS = [1, 5, 63, 0x01010101, 0x00800000, 0x02FE0000, 0x037E0000, 0x0D7FFFFF, 0x0D800000, 0x7E7E7E7E, 0x7F7FFFFF, 0x7F800000, 0x7FC00001]
# few rows; their tiles; the kernels for many rows, undivided and divided; unpacked beforehand; prompts beside decoding.  Lengths end in the first half of
# 64 tokens, the second of which is then no block's, or in the second.
FORMS = [([70, 5, 129], [1, 1, 1], 4), ([70, 65, 300], [20, 9, 40], 4), ([284, 33], [284, 33], 2), ([4100], [140], 4), ([650], [600], 8), ([1050, 650], [530, 520], 8),
         ([2060, 90, 640, 30], [150, 1, 1, 1], 4)]


def _words(like, word):
    return torch.full((like.numel() // 4,), word, dtype=torch.int64).to(torch.int32).cuda().view(torch.uint8).view(like.shape)


@pytest.mark.parametrize("word", WORDS, ids=hex)
@pytest.mark.parametrize("d,block", [(128, 32), (128, 64), (64, 32), (64, 64)])
def test_words_behind_a_length_reach_nothing(word, d, block):
    for lens, news, Hq in FORMS:
        g = torch.Generator().manual_seed(len(lens))
        f = Filled(lens, CacheParams(H=2, d=d, page=128, block=block), g)
        q = _randn((sum(news), Hq, d), g)
        for causal in (True, False):
            out = []
            for fill in (word, 0):
                f.pool = _words(f.pool, fill)
                f.store()
                out.append(_attend(f, news, Hq, g, causal=causal, q=q))
            assert torch.equal(out[0][2], out[1][2]) and torch.equal(out[0][3], out[1][3]), (lens, causal)
            if word == WORDS[0]:
                _check(f, *out[0], causal)


@pytest.mark.parametrize("word", WORDS, ids=hex)
@pytest.mark.parametrize("d,block,n,Hq", [(128, 32, 1, 4), (128, 32, 30, 4), (128, 64, 100, 4), (128, 32, 200, 2), (64, 64, 200, 4), (128, 32, 530, 8), (64, 64, 530, 8)])
def test_words_of_the_page_in_place_of_one_that_does_not_exist_reach_nothing(word, d, block, n, Hq):
    """Page 0, which is read for those, is no request's."""
    g = torch.Generator().manual_seed(9)
    f = Filled([640, 96], CacheParams(H=2, d=d, page=64, block=block), g)
    q = _randn((n + 1, Hq, d), g)
    f.table = torch.where(f.table >= 0, f.table + 1, f.table)
    f.table[0, 3], f.table[0, 7], f.table[1, :2] = -1, f.pool.shape[0] + 1, _i32([-7, 1 << 30])
    pool, out = f.pool, []
    for fill in (word, 0):
        f.pool = torch.cat([_words(pool[:1], fill), pool])
        for causal in (False, True):
            out.append(_attend(f, [n, 1], Hq, g, causal=causal, q=q)[2:])
    for a, b in zip(out[:2], out[2:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.isfinite(a[0].float()).all() and torch.isinf(a[1][:, n]).all() and torch.isfinite(a[1][:, :n]).all()


def test_a_pool_that_held_a_table_serves_as_a_new_one():
    """A step of the operators over memory that has held int32 numbers, 1 and up."""
    p = CacheParams(H=2, d=128, page=64, block=32)
    g = torch.Generator().manual_seed(4)
    prompt = [284, 33, 650]
    pool = torch.arange(1, 1 + 20 * cache.cache_page_bytes(p) // 4, dtype=torch.int32, device="cuda").view(torch.uint8).view(20, p.H, -1)
    table = torch.full((3, 16), -1, dtype=torch.int32, device="cuda")
    rows = sum(prompt)
    plan = cache.sagebwd_cache_plan(_i32([0] * 3), _i32(prompt), table, _i32(list(range(20))), _i32([20]), p, rows)
    K, V, Q = _randn((rows, 2, 128), g).cuda(), _randn((rows, 2, 128), g).cuda(), _randn((rows, 4, 128), g).cuda()
    results = []
    for _ in range(2):
        cache.sagebwd_cache_append(K, V, plan.slots, pool, p)
        results.append(cache.sagebwd_cache_attention(Q, pool, table, plan.lengths, plan.cu_new, p, max(prompt)))
        pool = torch.zeros_like(pool)
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
