"""The weight of each key where one key head serves very many query heads."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import attention_bounds, dev, host, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq", [700, 40000])
def test_key_weights_of_very_many_heads_in_a_wide_table(Hq):
    """A table of 60K slots with a short sequence in it: the workgroups behind the sequence have no row (a slot's distance times the query heads
    per key head passes 2^31 there)."""
    import paper_2410_02367_amd as sage
    D, page, group, n, columns = 64, 256, 32, 70, 234
    c, table = make_cache(3, 1, 1, D, page, group, [n], columns)
    q = np.random.default_rng(Hq).standard_normal((1, Hq, 1, D)).astype(np.float16)
    k, v, there = c.load(table[:, :1], None, page, [n])
    want, lse, w = so.attention(q, k, v, there, [n])
    args = (dev(q), dev(c.data), dev(table), dev(np.int32([n])))
    out, got = sage.sage_cache4_attn(*args, page=page, group=group, return_lse=True)
    had = torch.rand(1, 1, columns * page, device="cuda")
    r = sage.sage_cache4_weights(*args, got, had, page=page, group=group)
    do, dl = attention_bounds(q, k, v, there, [n], None, True, 1 / np.sqrt(D), lse)
    assert np.all(np.abs(host(out) - want) <= do + 2.0 ** -11 * np.abs(want) + 2.0 ** -25) and np.all(np.abs(host(got) - lse) <= dl)
    # a weight is off by what its score and its row's lse are, the sum of Hq of them in fp32 by half a step per term
    rel = 4 * dl.max() + (Hq + 8) * 2.0 ** -24
    full = host(had)
    full[..., :page] += w
    assert np.all(np.abs(host(r) - full)[..., :page] <= rel * w + 2.0 ** -23 * full[..., :page] + 2.0 ** -40)
    assert torch.equal(r[..., n:], had[..., n:])
