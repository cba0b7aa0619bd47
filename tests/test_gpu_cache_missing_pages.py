"""Attention over requests that have let go of pages: the first ones, some, all; in every form that reads pages."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2603_02170_amd import cache
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache import Filled, _check, _i32, _randn

pytestmark = pytest.mark.gpu


def _gone(pages, kind, rng):
    """Which of a request's pages are gone."""
    gone = np.zeros(pages, bool)
    if kind == "first":
        gone[:int(rng.integers(0, pages))] = True
    elif kind == "all but the last":
        gone[:-1] = True
    elif kind == "some":
        gone = rng.random(pages) < 0.3
    elif kind == "most":
        gone = rng.random(pages) < 0.9
    elif kind == "every second":
        gone[int(rng.integers(2))::2] = True
    elif kind == "all":
        gone[:] = True
    return gone


KINDS = ["none", "first", "all but the last", "some", "most", "every second", "all"]


@pytest.mark.parametrize("L,R,n,G,H,d,group,page", [
    (9000, 520, 1, 2, 1, 64, 64, 64),       # an item's tiles are more than a wave looks up at once, and hardly an item is divided
    (9000, 14, 3, 4, 2, 128, 32, 32),       # divided
    (5000, 21, 5, 4, 1, 128, 64, 128),      # two tiles of 16 rows
    (5000, 14, 5, 4, 1, 128, 32, 256),
    (900, 7, 2, 1, 3, 64, 32, 32), (130, 7, 1, 3, 1, 128, 64, 32),
    (1500, 7, 12, 4, 2, 128, 64, 64), (1500, 7, 25, 4, 1, 64, 32, 32),       # 64 and 128 rows in a workgroup
    (700, 7, 100, 3, 1, 128, 32, 32), (300, 7, 530, 4, 1, 64, 64, 64),       # 256 rows; keys unpacked beforehand
])
def test_pages_that_are_gone_count_for_nothing(L, R, n, G, H, d, group, page):
    rng, g = np.random.default_rng(L + R + n), torch.Generator().manual_seed(L + d)
    p = CacheParams(H=H, d=d, page=page, group=group)
    f = Filled([L], p, g, spare_columns=0)          # (its pages are every request's)
    kinds = [KINDS[r % len(KINDS)] for r in range(R)]
    gone = [_gone(f.table.shape[1], k, rng) for k in kinds]
    nowhere = torch.tensor([-1, f.pool.shape[0], -(1 << 31), (1 << 31) - 1])
    table = torch.stack([torch.where(torch.from_numpy(x), nowhere[torch.randint(0, 4, x.shape, generator=g)].to(torch.int32), f.table[0].cpu()) for x in gone])
    q = _randn((R * n, H * G, d), g)
    causal = n <= L
    O, lse = cache.sagebwd_cache_attention(q.cuda(), f.pool, table.cuda(), _i32([L] * R), _i32([n * r for r in range(R + 1)]), p, n, causal=False)
    for r in sorted(set(list(range(min(R, 7))) + rng.integers(0, R, 7).tolist())):
        keep = ~np.repeat(gone[r], page)[:L]
        one = SimpleNamespace(p=p, lens=[int(keep.sum())], k=f.k[keep], v=f.v[keep], at=np.array([0, int(keep.sum())]))
        rows = slice(n * r, n * r + n)
        _check(one, q[rows], [0, n], O[rows], lse[:, rows], False)
    assert not torch.isnan(O).any()
    # under the mask a row sees what its place among all the tokens lets it
    if causal and n > 1:
        Oc, lc = cache.sagebwd_cache_attention(q.cuda(), f.pool, table.cuda(), _i32([L] * R), _i32([n * r for r in range(R + 1)]), p, n)
        for r in range(min(R, 7)):
            for i in (0, n - 1):
                keep = ~np.repeat(gone[r], page)[:L - n + 1 + i]
                keep = np.concatenate([keep, np.zeros(L - keep.size, bool)])
                one = SimpleNamespace(p=p, lens=[int(keep.sum())], k=f.k[keep], v=f.v[keep], at=np.array([0, int(keep.sum())]))
                _check(one, q[n * r + i:n * r + i + 1], [0, 1], Oc[n * r + i:n * r + i + 1], lc[:, n * r + i:n * r + i + 1], False)
