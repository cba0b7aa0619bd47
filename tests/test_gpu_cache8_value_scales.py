"""Attention over the cache held in 8 bits where V's magnitudes are at the ends of what is stored: the softmax and its LSE do not depend on V."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache8 import Filled, _attend, _check, _np, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,R,n,Hq", [(64, 1, 1, 4), (128, 1, 20, 4), (128, 1, 100, 2), (64, 1, 530, 8), (128, 1, 530, 8), (64, 130, 1, 4), (128, 130, 20, 4),
                                      (64, 130, 150, 2), (128, 130, 150, 2)])
@pytest.mark.parametrize("values", ["least", "least in places", "large"])
def test_many_keys_of_small_weight_count_whatever_their_values_are(d, R, n, Hq, values):
    """One key's logit is 15 above all others', of which there are 20000: each is 2^-21.6 of the softmax's reference, together 1 %.  V's magnitudes are about 2^-100
    (less is zero), so that weight times scale is below 2^-126, or 2^97.  130 requests, of the same pages, are hardly divided.

    O as in the other tests; but weights times scale of less than 2^-126 may count as nothing, for 127 times that each (l is at least 1)."""
    L, g = 20000, torch.Generator().manual_seed(n)
    f = Filled([L], CacheParams(H=2, d=d, page=64, block=32), g)
    sign = torch.randint(0, 2, (d,), generator=g).float() * 2 - 1
    f.K = (0.01 * torch.randn((L, 2, d), generator=g)).to(torch.bfloat16)
    f.K[5] = (15 / d ** 0.5 * sign).to(torch.bfloat16)
    blocks = torch.arange(L) // 32
    exponent = torch.where((blocks % 2 == 0) | torch.tensor(values != "least in places"), -101.5 if values != "large" else 95.0, 0.0)
    f.V = (f.V.float() * torch.exp2(exponent)[:, None, None]).to(torch.bfloat16)
    f.store()
    q = (sign + 0.02 * torch.randn((n, Hq, d), generator=g)).to(torch.bfloat16)
    f.table, f.lengths = f.table.expand(R, -1).contiguous(), f.lengths.expand(R).contiguous()
    _, _, O, lse = _attend(f, [n] * R, Hq, g, causal=False, q=q.repeat(R, 1, 1))
    at = (R // 2) * n
    O, lse = O[at:at + n], lse[:, at:at + n]
    rows = sorted({0, n // 3, n - 1})
    one = type("One", (), dict(p=f.p, lens=[L], k=f.k, v=f.v, at=[0, L]))
    _check(one, q[rows], [0, len(rows)], O[rows], lse[:, rows], False)
    qs = _np(q[rows]).astype(np.float64)
    want, wlse, A = ref.attention(qs, f.k, f.v, len(rows), False, d ** -0.5, None)
    others = 1 - np.exp((np.einsum("nhd,hd->nh", qs, np.repeat(f.k[5], Hq // 2, axis=0)) * d ** -0.5).T - wlse)
    assert (others > 0.004).all() and (others < 0.02).all()
    e = d ** -0.5 * (d + 6) * 2.0 ** -24 * np.abs(f.k).max() * np.abs(qs).sum(-1) + 2.0 ** -18
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * e[..., None] + 2.0 ** -24 * (L / 32 + 40)) * A + L * 127 * 2.0 ** -126
    err = np.abs(_np(O[rows]).astype(np.float64) - want)
    assert (err <= tol).all(), float((err / tol).max())
