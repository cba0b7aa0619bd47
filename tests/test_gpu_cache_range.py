"""Attention over the cache at the ends of the range that the header gives: |Q| below 2^117, and V's largest magnitude times a request's keys
below 2^117."""
import math

import pytest
import torch

from paper_2603_02170_amd.cache import CacheParams
from test_gpu_cache import Filled, _attend, _check

pytestmark = pytest.mark.gpu

# keys, new tokens, heads of the group: one and two tiles of 16 rows, parts, each kernel for many rows, keys unpacked beforehand
FORMS = [([700, 3], [1, 1], 4), ([5000], [2], 2), ([900, 60], [5, 8], 4), ([600, 300], [20, 30], 2), ([700], [40], 3), ([500], [70], 4), ([600], [520], 4)]


@pytest.mark.parametrize("lens,news,G", FORMS)
@pytest.mark.parametrize("d,group", [(64, 32), (128, 64), (128, 32)])
def test_values_as_large_as_their_number_allows(lens, news, G, d, group):
    """The sums are formed before they are divided: of probabilities of up to 2^8 (the reference may be that far below the maximum) times V's
    scale (a seventh of a group's maximum and a 16th) times up to 31, over a request's keys: 2^8 x 31 x 17 / 112 < 2^11 times the bound stays
    below 2^128."""
    g = torch.Generator().manual_seed(sum(lens) + d)
    f = Filled(lens, CacheParams(H=2, d=d, page=64, group=group), g)
    f.V *= 2.0 ** math.floor(117 - math.log2(float(f.V.abs().max()) * max(lens)))
    assert 2.0 ** 116 <= float(f.V.abs().max()) * max(lens) < 2.0 ** 117
    f.store()
    q, cu, O, lse = _attend(f, news, 2 * G, g)
    assert torch.isfinite(O).all()
    _check(f, q, cu, O, lse, True)


@pytest.mark.parametrize("lens,news,G", FORMS)
@pytest.mark.parametrize("d,group", [(64, 64), (128, 32)])
def test_queries_as_large_as_the_header_allows(lens, news, G, d, group):
    g = torch.Generator().manual_seed(sum(lens) + d)
    f = Filled(lens, CacheParams(H=2, d=d, page=32, group=group), g, sigma=2.0 ** -98)
    q = torch.randn((sum(news), 2 * G, d), generator=g).to(torch.bfloat16)
    q *= 2.0 ** math.floor(117 - math.log2(float(q.abs().max())))
    assert 2.0 ** 115 <= float(q.abs().max()) < 2.0 ** 117
    scale = 2.0 ** (98 - math.log2(float(q.abs().max()))) * d ** -0.5
    _, cu, O, lse = _attend(f, news, 2 * G, g, q=q, sm_scale=scale)
    assert torch.isfinite(O).all() and torch.isfinite(lse).all()
    _check(f, q, cu, O, lse, True, sm_scale=scale)
