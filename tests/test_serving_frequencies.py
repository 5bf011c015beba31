"""Frequencies of scaled contexts, pair by pair from their formulas."""
import math

import numpy as np
import pytest


def ramp(rotated, base, factor, original_length, low, high):
    """The mixture of scaling="ramp", linear in the pair's index between the pair that turns `high` times in original_length (rounded
    down, from 0 on) and the one that turns `low` times (rounded up, at most rotated - 1, which lies behind the last pair)."""
    def pair(turns):
        return rotated * math.log(original_length / (2 * math.pi * turns)) / (2 * math.log(base))
    first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotated - 1)
    res = []
    for i in range(rotated // 2):
        f = base ** (-2 * i / rotated)
        part = min(max((i - first) / (last - first), 0.0), 1.0)
        res.append(f * (1 - part) + f / factor * part)
    return np.array(res)


@pytest.mark.parametrize("rotated,base,original_length", [(64, 1e4, 4096), (64, 1e4, 65536), (128, 1e4, 131072), (128, 5e5, 8192), (32, 1e4, 1 << 20)])
@pytest.mark.parametrize("factor", [4.0, 16.0])
def test_ramp_that_ends_before_and_behind_the_last_pair(rotated, base, original_length, factor):
    import paper_2410_02367_amd as sage
    f, a = sage.sage_rope_frequencies(rotated, base, "ramp", factor, original_length, 1.0, 32.0)
    assert a == 0.1 * math.log(factor) + 1.0
    # products and a sum of fp64 numbers
    np.testing.assert_allclose(f.numpy(), ramp(rotated, base, factor, original_length, 1.0, 32.0), rtol=2.0 ** -48)


@pytest.mark.parametrize("rotated,original_length", [(64, 65536), (128, 131072)])
def test_a_slowest_pair_that_turns_is_not_divided_as_one_that_does_not(rotated, original_length):
    import paper_2410_02367_amd as sage
    slowest = 1e4 ** (2 / rotated - 1)
    assert original_length * slowest / (2 * math.pi) > 1.0                       # more than `low` times
    f, _ = sage.sage_rope_frequencies(rotated, scaling="ramp", factor=4.0, original_length=original_length, low=1.0, high=32.0)
    assert f[-1] > slowest / 4.0 * 1.25


def test_the_turns_that_each_scaling_leaves_alone_by_default():
    """"parts" mixes between 1 and 4 turns, "ramp" (YaRN) between 1 and 32."""
    import paper_2410_02367_amd as sage
    for scaling, high in (("parts", 4.0), ("ramp", 32.0)):
        f, _ = sage.sage_rope_frequencies(128, scaling=scaling, factor=8.0)
        g, _ = sage.sage_rope_frequencies(128, scaling=scaling, factor=8.0, low=1.0, high=high)
        assert np.array_equal(f.numpy(), g.numpy())
    np.testing.assert_allclose(sage.sage_rope_frequencies(128, scaling="ramp", factor=8.0)[0].numpy(), ramp(128, 1e4, 8.0, 8192, 1.0, 32.0), rtol=2.0 ** -48)
    for bad in (dict(scaling="ramp", low=40.0), dict(scaling="parts", low=5.0), dict(low=2.0, high=1.0)):
        with pytest.raises(ValueError):
            sage.sage_rope_frequencies(64, **bad)
