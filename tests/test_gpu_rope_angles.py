"""Rotary positions of fp32 tensors: sine and cosine as near as the type has them, at any position."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(128, 128), (64, 32), (72, 54)])
@pytest.mark.parametrize("far", [100, 10 ** 5, 2 ** 20])
def test_sine_and_cosine_of_fp32(far, D, R, interleaved):
    import paper_2410_02367_amd as sage
    N = 500
    x = np.zeros((1, 1, N, D), np.float32)
    a = slice(0, R, 2) if interleaved else slice(0, R // 2)
    x[..., a] = 1.0                                         # the results are the cosine and the sine themselves
    pos = np.random.default_rng(far).integers(0, far, N).astype(np.int32)
    freq = 10000.0 ** (-np.arange(R // 2) / (R // 2))
    y = sage.sage_rope(dev(x), None, dev(pos), dev(freq), interleaved)
    want = so.rope(x, pos, freq, interleaved)
    # a sine or cosine is off by a unit in the last place, 2^-24 below 1, and rounded once more, 2^-25; the angle by 2^-53 of up to 2^20 / pi turns
    assert np.abs(host(y) - want)[..., :R].max() <= 2.0 ** -24 + 2.0 ** -25 + 2 * np.pi * 2.0 ** (20 - 2 - 52) + 2.0 ** -40
    assert torch.equal(y[..., R:], dev(x)[..., R:])
