"""Eviction from one pool of pages into another."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import dev, host, make_cache

pytestmark = pytest.mark.gpu


def test_into_another_pool_with_the_same_table():
    import paper_2410_02367_amd as sage
    D, page, group, B, H = 64, 16, 32, 2, 3
    c, table = make_cache(40, B, H, D, page, group, [70, 33], 5)
    weights = dev(np.random.default_rng(40).random((B, H, 5 * page)).astype(np.float32))
    cache, pages, lengths = dev(c.data), dev(table), dev(np.int32([70, 33]))
    fresh = torch.full_like(cache, 0xff)
    kept, n, w = sage.sage_cache4_evict(cache, pages, lengths, weights, pages, 30, 4, D, page, group, out_cache=fresh)
    want, new = so.evict(weights.cpu().numpy(), [70, 33], 5 * page, 30, 4)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(n.cpu().numpy(), new)
    assert np.array_equal(cache.cpu().numpy(), c.data)
    old_k, old_v, _ = c.load(table, None, 5 * page)
    k, v = sage.sage_cache4_load(fresh, pages, None, 30, D, n, page=page, group=group)
    for b in range(B):
        for h in range(H):
            for got, old in ((k, old_k), (v, old_v)):
                assert np.array_equal(host(got[b, h]), old[b, h, want[b, h]].astype(np.float16).astype(np.float64))
