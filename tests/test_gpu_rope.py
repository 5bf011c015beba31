"""Rotary positions and their gradient against the fp64 definition."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, dev, host, rounded

pytestmark = pytest.mark.gpu


def check(y, x, kind, positions, freq, interleaved, amplitude, backward):
    want = so.rope(x, positions, freq, interleaved, amplitude, backward)
    R = 2 * len(freq)
    pairs = np.abs(x).copy()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    pairs[..., a] = pairs[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    # the fraction of a turn in fp32 (2^-26 turns, 2^-23 of an angle), sine and cosine to 4 units of 2^-24, two products and a sum
    bound = HALF_STEP[kind] * np.abs(want) * (1 + 2.0 ** -10) + pairs * abs(amplitude) * 2.0 ** -21 + TINY[kind]
    bound[..., R:] = 0.0
    err = np.abs(host(y) - want)
    assert np.all(err <= bound), (err - bound).max()


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hk,N,D,R", [(1, 1, 0, 1, 8, 2), (2, 4, 1, 1, 128, 128), (3, 2, 2, 7, 64, 64), (1, 3, 1, 130, 96, 24),
                                            (2, 5, 3, 33, 80, 32), (1, 2, 1, 65, 128, 64), (1, 1, 1, 257, 256, 198), (65, 1, 1, 1, 64, 16)])
def test_against_the_definition(B, Hq, Hk, N, D, R, kind, interleaved, backward):
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(B * 1000 + N * 10 + R)
    x = rounded(g.standard_normal((B, Hq, N, D)), kind)
    y = rounded(g.standard_normal((B, max(Hk, 1), N, D)), kind)
    pos = g.integers(-1000, 2 ** 20, (B, N)).astype(np.int32)
    pos[0, 0] = 0
    freq = 10000.0 ** (-np.arange(R // 2) / (R // 2))
    call = sage.sage_rope_bwd if backward else sage.sage_rope
    xd, yd = dev(x, TORCH[kind]), dev(y, TORCH[kind]) if Hk else None
    r = call(xd, yd, dev(pos), dev(freq), interleaved, 1.25)
    for got, src in zip(r if Hk else (r,), (x, y)):
        check(got, src, kind, pos, freq, interleaved, 1.25, backward)
    assert np.array_equal(host(xd), x)


def test_shared_positions_strides_and_in_place():
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(5)
    B, Hq, Hk, N, D = 2, 4, 2, 19, 64
    fused = dev(g.standard_normal((B, N, Hq + 2 * Hk, D)), torch.float16)          # q, k and v of a projection in one tensor
    before = host(fused)
    q, k = fused[:, :, :Hq].transpose(1, 2), fused[:, :, Hq:Hq + Hk].transpose(1, 2)
    pos = dev(np.arange(100, 100 + N, dtype=np.int32))
    freq = dev(10000.0 ** (-np.arange(32) / 32))
    a, b = sage.sage_rope(q, k, pos, freq)
    assert a.stride() == (N * Hq * D, D, Hq * D, 1)
    check(a, before[:, :, :Hq].transpose(0, 2, 1, 3), "f16", host(pos), host(freq), False, 1.0, False)
    check(b, before[:, :, Hq:Hq + Hk].transpose(0, 2, 1, 3), "f16", host(pos), host(freq), False, 1.0, False)
    r = sage.sage_rope(q, k, pos, freq, q_out=q, k_out=k)
    assert r[0] is q and torch.equal(q, a) and torch.equal(k, b)
    assert np.array_equal(host(fused)[:, :, Hq + Hk:], before[:, :, Hq + Hk:])
    # one head for all (stride 0): read as it is, written as rows of its own
    one = dev(g.standard_normal((B, 1, N, D)), torch.float16)
    y = sage.sage_rope(one.expand(B, 3, N, D), None, pos, freq)
    assert torch.equal(y, sage.sage_rope(one, None, pos, freq).expand(B, 3, N, D))
    with pytest.raises(sage.SageError):
        sage.sage_rope(one.expand(B, 3, N, D), None, pos, freq, q_out=one.expand(B, 3, N, D))


def test_far_positions_and_back():
    """Positions up to 2^31 - 1: the angle is reduced in fp64 (2^31 turns to 2^-22 of one), and the gradient undoes the turn."""
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(6)
    x = g.standard_normal((1, 2, 4, 64)).astype(np.float32).astype(np.float64)
    pos = np.array([2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, 2 ** 24 + 1], np.int32)
    freq = 10000.0 ** (-np.arange(32) / 32)
    y = sage.sage_rope(dev(x, torch.float32), None, dev(pos), dev(freq))
    # 2^31 radians in fp64 are off by 2^-22 in either computation
    assert np.abs(host(y) - so.rope(x, pos, freq)).max() <= 8 * 2.0 ** -21
    assert np.abs(host(sage.sage_rope_bwd(y, None, dev(pos), dev(freq))) - x).max() <= 8 * 2.0 ** -21


def test_scaled_frequencies():
    import paper_2410_02367_amd as sage
    plain, a = sage.sage_rope_frequencies(64)
    assert a == 1.0 and np.allclose(plain.numpy(), 10000.0 ** (-np.arange(32) / 32))
    f, a = sage.sage_rope_frequencies(64, scaling="linear", factor=4.0, device="cuda")
    assert f.is_cuda and a == 1.0 and np.allclose(f.cpu().numpy(), plain.numpy() / 4)
