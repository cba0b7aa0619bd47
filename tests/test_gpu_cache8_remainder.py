"""Attention over the cache held in 8 bits in tiles of up to 32 query rows: the probabilities meet the values with 16 bits, the rounding to bf16 and what it
left, so that O's error is that of its own rounding."""
import math

import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache8 import Filled, _attend, _np

pytestmark = pytest.mark.gpu


# a wave an item; undivided; divided and joined, by few and by many; tiles of 32 rows; several of them
@pytest.mark.parametrize("d,block,R,L,n,Hq,H", [(64, 32, 3, 100, 1, 2, 2), (128, 64, 2, 128, 7, 4, 1), (128, 32, 2, 900, 1, 16, 2), (64, 64, 2, 900, 8, 8, 2), (128, 64, 1, 6000, 1, 16, 1),
                                                (64, 32, 1, 6000, 6, 5, 1), (128, 32, 70, 2500, 4, 8, 1), (128, 64, 2, 1500, 30, 4, 2), (64, 64, 2, 3000, 100, 2, 2), (128, 32, 1, 700, 100, 1, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_what_rounding_leaves_of_the_probabilities_reaches_the_values(d, block, R, L, n, Hq, H, causal):
    """Half of the keys have logit 0 and values of 1, the others a row's own logit near log(127 / 64) and values of -64 / 127: O is nearly nothing, A = sum p |v| is not,
    and each half's probabilities are rounded alike.

    Tolerances: O's rounding, 2^-8 of it; of A 2^-16 (2^-8 of the 2^-8 that a first rounding leaves at most), twice a logit's error and that of exp2 as in the
    other tests, a rounding of 2^-24 for each of a tile's two products and 40 more.  With one product the error is a rounding of bf16, which a plain
    computation shows to pass them."""
    g = torch.Generator().manual_seed(L + n)
    f = Filled([L], CacheParams(H=H, d=d, page=64, block=block), g)
    second = (torch.arange(L) % 2 == 1)[:, None, None]
    f.K = (second & (torch.arange(d) == 0)).expand(L, H, d).to(torch.bfloat16)
    f.V = torch.where(second, -64 / 127, 1.0).expand(L, H, d).to(torch.bfloat16)
    f.store()
    logits = math.log(127 / 64) + 0.1 * (2 * torch.rand((n, Hq), generator=g) - 1)
    q = torch.zeros((n, Hq, d))
    q[..., 0] = logits * d ** 0.5
    q = q.to(torch.bfloat16)
    f.table, f.lengths = f.table.expand(R, -1).contiguous(), f.lengths.expand(R).contiguous()
    _, _, O, _ = _attend(f, [n] * R, Hq, g, causal=causal, q=q.repeat(R, 1, 1))
    O, qs = _np(O[(R - 1) * n:]).astype(np.float64), _np(q).astype(np.float64)
    want, _, A = ref.attention(qs, f.k, f.v, n, causal, d ** -0.5, None)
    e = d ** -0.5 * (d + 6) * 2.0 ** -24 * np.abs(qs).sum(-1) + 2.0 ** -18
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2 * e[..., None] + 2.0 ** -24 * (2 * L / 32 + 40)) * A
    err = np.abs(O - want)
    assert (err <= tol).all(), float((err / tol).max())
    s = np.einsum("nhd,lhd->nhl", qs, np.repeat(f.k, Hq // H, axis=1)) * d ** -0.5
    s = np.where(np.arange(L) <= L - n + np.arange(n)[:, None, None], s, -np.inf) if causal else s
    p = np.exp(s - s.max(-1, keepdims=True))
    rounded = ref.bf16_round((p / 127).astype(np.float32)).astype(np.float64)
    alone = np.einsum("nhl,lhd->nhd", rounded, 127 * np.repeat(f.v, Hq // H, axis=1)) / p.sum(-1)[..., None]
    assert (np.abs(alone - want) > 2 * tol).any()
