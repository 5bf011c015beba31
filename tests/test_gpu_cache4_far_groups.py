"""Attention over the cache held in 4 bits where the keys that a row looks at have no values in one group of channels: what the group does
hold has weights far below the others', down to where fp32 ends."""
import numpy as np
import pytest

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, attention_bounds, dev, host, make_cache, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [20, 60, 90, 115, 140, 300])
@pytest.mark.parametrize("size", [0, -14, 6])
@pytest.mark.parametrize("Hq,Nq,room,n_splits", [(4, 1, 0, 0), (3, 1, 1280, 3), (4, 4, 0, 0), (4, 8, 0, 0), (4, 8, 1280, 3), (4, 30, 2048, 1)])
@pytest.mark.parametrize("D,group,page", [(64, 32, 16), (128, 64, 64), (128, 32, 64)])
def test_weights_far_below_the_largest(D, group, page, Hq, Nq, room, n_splits, size, bits):
    """The scores of 2 of 3 keys lie `bits` (of the exponent of 2) higher, and those have values of 2^size in all groups but the last, in
    which only the third ones have any."""
    import paper_2410_02367_amd as sage
    n = 160
    columns = -(-(n + room) // page)
    g = np.random.default_rng(bits + D)
    k = g.standard_normal((1, 1, n, D)) * 0.2
    v = g.standard_normal((1, 1, n, D)) * 2.0 ** size
    q = g.standard_normal((1, Hq, Nq, D)) * 0.2
    low = np.arange(n) % 3 == 2
    k[..., 0], q[..., 0] = 7.0, 8.0
    k[:, :, low, 0] = 7.0 - bits * np.log(2) * np.sqrt(D) / 8.0
    v[:, :, :, D - group:] *= low[:, None]
    v[:, :, low, :D - group] = 0.0
    c, table = make_cache(bits, 1, 1, D, page, group, [0], columns)
    c.append(k.astype(np.float16), v.astype(np.float16), table, [0], [n])
    q = rounded(q, "bf16")              # (its results reach far down)
    kk, vv, there = c.load(table, None, columns * page, [n])
    want, lse, _ = so.attention(q, kk, vv, there, [n], None, False)
    out = sage.sage_cache4_attn(dev(q, TORCH["bf16"]), dev(c.data), dev(table), dev(np.int32([n])), causal=False, page=page, group=group, n_splits=n_splits)
    _, ds = attention_bounds(q, kk, vv, there, [n], None, False, 1 / np.sqrt(D), lse)
    got = host(out)
    scales = np.abs(vv[0, 0]).reshape(-1, D // group, group).max(-1)
    for hq in range(Hq):
        for t in range(Nq):
            p = np.exp(kk[0, 0] @ q[0, hq, t] / np.sqrt(D) - lse[0, hq, t]) * there[0]
            largest = (p[:, None] * scales).max(0)
            bound = (p @ np.abs(vv[0, 0])) * (2.0 ** -11 + 3 * ds[0, hq, t]) + n * np.repeat(np.maximum(largest * 2.0 ** -23, largest.max() * 2.0 ** -100), group)
            assert np.all(np.abs(got[0, hq, t] - want[0, hq, t]) <= bound + HALF_STEP["bf16"] * np.abs(want[0, hq, t]) + TINY["bf16"])
