"""The logarithm of the sums: it does not depend on the values, whatever their size."""
import numpy as np
import pytest

from serving_util import dev, host, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gain", [0.0, 2.0 ** -20, 2.0 ** -8, 1.0, 2.0 ** 12])
@pytest.mark.parametrize("Hq,Nq,room,n_splits", [(4, 1, 0, 0), (4, 4, 0, 0), (4, 8, 0, 0), (4, 30, 2048, 1), (4, 1, 1280, 5), (4, 8, 512, 2)])
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 128)])
def test_values_of_any_size(D, group, Hq, Nq, room, n_splits, gain):
    """Queries of 0: every score is 0 and the logarithm that of the number of keys."""
    import paper_2410_02367_amd as sage
    page, lengths = 64, [Nq, 90, 200 + Nq]
    columns = -(-(lengths[2] + room) // page)
    g = np.random.default_rng(D + Nq)
    c, table = make_cache(2, 3, 1, D, page, group, [0] * 3, columns)
    k = g.standard_normal((3, 1, lengths[2], D)).astype(np.float16)
    c.append(k, (g.standard_normal(k.shape) * gain).astype(np.float16), table, [0] * 3, lengths)
    q = np.zeros((3, Hq, Nq, D), np.float16)
    _, lse = sage.sage_cache4_attn(dev(q), dev(c.data), dev(table), dev(np.int32(lengths)), page=page, group=group, n_splits=n_splits, return_lse=True)
    want = np.log(np.array(lengths)[:, None, None] - Nq + 1 + np.arange(Nq)) + np.zeros((1, Hq, 1))
    # the sum is a whole number times a power of two, exact; a logarithm is off by 2^-24 and its share of its size, in a chunk and in the join of
    # chunks, then the factor ln 2 and its product
    assert np.all(np.abs(host(lse) - want) <= want * 4 * 2.0 ** -24 + 2.0 ** -22), np.abs(host(lse) - want).max()
