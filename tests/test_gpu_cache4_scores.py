"""Attention over the cache held in 4 bits with scores as large as the calls take."""
import numpy as np
import pytest

from serving_util import HALF_STEP, dev, host, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exponent", [20, 24, 25])
@pytest.mark.parametrize("Hq,Nq,room", [(4, 1, 0), (4, 4, 0), (4, 8, 0), (4, 30, 2048)])
@pytest.mark.parametrize("D,group", [(64, 32), (128, 128), (128, 32)])
def test_keys_of_equal_scores(D, group, Hq, Nq, room, exponent, sign):
    """All keys are one and the same, so whatever its score is the weights are equal, up to 2^25 in the exponent of 2."""
    import paper_2410_02367_amd as sage
    page, n = 64, 150
    columns = -(-(n + room) // page)
    g = np.random.default_rng(D + Nq)
    c, table = make_cache(1, 1, 1, D, page, group, [0], columns)
    k = np.zeros((1, 1, n, D), np.float16)
    k[..., 5] = 7 * 2.0 ** 8
    v = g.standard_normal((1, 1, n, D)).astype(np.float16)
    c.append(k, v, table, [0])
    _, vv, _ = c.load(table, None, n)
    q = np.zeros((1, Hq, Nq, D), np.float16)
    q[..., 5] = sign * 2.0 ** 10
    score = 7 * 2.0 ** 18
    scale = 2.0 ** exponent / (score * np.log2(np.e))
    out, lse = sage.sage_cache4_attn(dev(q), dev(c.data), dev(table), dev(np.int32([n])), causal=False, sm_scale=scale, page=page, group=group,
                                     n_splits=1, return_lse=True)
    want = vv[0, 0].mean(0)
    # equal weights, each rounded with its key's scale to 2^-11, 150 of them added up in fp32, and the rounding of the result
    bound = np.abs(vv[0, 0]).mean(0) * (2.0 ** -11 + 150 * 2.0 ** -24) + HALF_STEP["f16"] * np.abs(want) + 2.0 ** -25
    assert np.all(np.abs(host(out) - want) <= bound)
    # the logarithm is an fp32 number, as the score that it stands for is (three roundings on either way)
    exact = sign * score * np.float64(np.float32(scale)) + np.log(n)
    assert np.all(np.abs(host(lse) - exact) <= np.abs(exact) * 6 * 2.0 ** -24)
