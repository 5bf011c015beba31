"""The plain definitions of the serving calls pinned against closed forms and independent statements of the same thing."""
import numpy as np
import pytest

from oracle import serving as so


def test_rope_is_a_turn_of_complex_numbers():
    g = np.random.default_rng(1)
    x = g.standard_normal((2, 3, 5, 16))
    f = 100.0 ** (-np.arange(6) / 6)
    pos = g.integers(0, 10 ** 6, (2, 5))
    y = so.rope(x, pos, f)
    z = (x[..., :6] + 1j * x[..., 6:12]) * np.exp(1j * pos[:, None, :, None] * f)
    assert np.allclose(y[..., :6], z.real) and np.allclose(y[..., 6:12], z.imag) and np.array_equal(y[..., 12:], x[..., 12:])
    y = so.rope(x, pos, f, interleaved=True, amplitude=1.5)
    z = 1.5 * (x[..., 0:12:2] + 1j * x[..., 1:12:2]) * np.exp(1j * pos[:, None, :, None] * f)
    assert np.allclose(y[..., 0:12:2], z.real) and np.allclose(y[..., 1:12:2], z.imag)


def test_rope_backward_is_the_transpose():
    g = np.random.default_rng(2)
    x, dy = g.standard_normal((2, 1, 2, 4, 8))
    f, pos = np.array([1.0, 0.1, 0.01]), np.array([3, 70, 900, 5])
    for interleaved in (False, True):
        a = (so.rope(x, pos, f, interleaved, 1.2) * dy).sum()
        b = (x * so.rope(dy, pos, f, interleaved, 1.2, backward=True)).sum()
        assert abs(a - b) < 1e-12
        # and the derivative by differences: the map is linear
        for d in range(8):
            e = np.zeros_like(x)
            e[0, 1, 2, d] = 1e-3
            slope = ((so.rope(x + e, pos, f, interleaved, 1.2) - so.rope(x - e, pos, f, interleaved, 1.2)) * dy).sum() / 2e-3
            assert abs(slope - so.rope(dy, pos, f, interleaved, 1.2, backward=True)[0, 1, 2, d]) < 1e-9


def test_psi4_by_hand():
    x = np.zeros((1, 32), np.float32)
    x[0, :8] = [7.0, -7.0, 0.5, 1.5, 2.5, -0.5, 3.49, 100.0 / 100]
    code, scale = so.psi4(x, 32)
    assert scale[0, 0] == 1.0
    # halves go to the even neighbour
    assert code[0, :8].tolist() == [7, -7, 0, 2, 2, 0, 3, 1]
    assert so.psi4(np.zeros((1, 64)), 32)[1].tolist() == [[0.0, 0.0]] and not so.psi4(np.zeros((1, 64)), 32)[0].any()


def test_psi4_round_trip_and_odd_values():
    g = np.random.default_rng(3)
    x = (g.standard_normal((100, 128)) * 10.0 ** g.uniform(-2, 3, (100, 1))).astype(np.float32)
    code, scale = so.psi4(x, 32)
    back = code * np.repeat(scale.astype(np.float64), 32, -1)
    # half a step, and what the largest value loses where the fp16 scale was rounded down: 7 * 2^-11 of a step
    assert np.all(np.abs(back - x) <= np.repeat(scale.astype(np.float64), 32, -1) * (0.5 + 7 * 2.0 ** -11))
    x = np.full((1, 32), np.nan, np.float32)
    x[0, 0], x[0, 1] = 14.0, -np.inf
    code, scale = so.psi4(x, 32)
    assert scale[0, 0] == 65504 and code[0, 0] == 0 and code[0, 1] == -7 and not code[0, 2:].any()


@pytest.mark.parametrize("D,group,page", [(64, 32, 16), (64, 64, 32), (128, 32, 16), (128, 64, 64), (128, 128, 16)])
def test_cache_places_every_nibble_once_and_reads_back(D, group, page):
    c = so.Cache(3, 2, D, page, group)
    assert sorted(c._k_nibble(d) for d in range(D)) == list(range(D))
    assert c.data.shape[2] == page * (D // 2 + D // 2 + 4 * (D // group))
    g = np.random.default_rng(4)
    k, v = g.standard_normal((2, 1, 2, page + 3, D)).astype(np.float16)
    table = np.array([[2, 0]], np.int32)
    c.append(k, v, table, [1])
    rk, rv, there = c.load(table, [1], page + 3)
    assert there.all()
    for x, r in ((k, rk), (v, rv)):
        code, scale = so.psi4(x.astype(np.float32), group)
        assert np.array_equal(r, code * np.repeat(scale.astype(np.float64), group, -1))
    assert not c.data[1].any()


def test_subtracting_a_mean_changes_no_softmax():
    g = np.random.default_rng(5)
    q, k, v = g.standard_normal((1, 2, 3, 64)), g.standard_normal((1, 1, 9, 64)), g.standard_normal((1, 1, 9, 64))
    there = np.ones((1, 9), bool)
    a = so.attention(q, k, v, there, [9])
    b = so.attention(q, k + g.standard_normal((1, 1, 1, 64)) * 5, v, there, [9])
    assert np.allclose(a[0], b[0]) and np.allclose(a[2], b[2]) and not np.allclose(a[1], b[1])


def test_attention_closed_forms():
    g = np.random.default_rng(6)
    v = g.standard_normal((1, 1, 6, 64))
    there = np.ones((1, 6), bool)
    k = np.ones((1, 1, 6, 64))
    q = g.standard_normal((1, 2, 3, 64))
    out, lse, w = so.attention(q, k, v, there, [5])
    # equal keys: the mean of the visible values; query t of 3 sees 3 + t tokens
    for t in range(3):
        assert np.allclose(out[0, :, t], v[0, 0, :3 + t].mean(0))
    assert np.allclose(w[0, 0], [2 * (1 / 3 + 1 / 4 + 1 / 5)] * 3 + [2 * (1 / 4 + 1 / 5), 2 / 5, 0])
    # more queries than tokens: the first ones see nothing
    out, lse, w = so.attention(q, k, v, there, [1])
    assert not out[0, :, :2].any() and np.isneginf(lse[0, :, :2]).all() and np.allclose(out[0, :, 2], v[0, 0, 0])
    # one weight per query and head in all
    out, lse, w = so.attention(q, g.standard_normal((1, 1, 6, 64)), v, there, [6], count=[2])
    assert np.isclose(w.sum(), 4.0) and not out[0, :, 2].any()
    there[0, 1:] = False
    assert np.allclose(so.attention(q, k, v, there, [6], causal=False)[0], v[:, :, :1])


def test_evict_by_hand():
    w = np.array([[[5, 1, 9, 5, 0, 5, 2, 8]]], np.float32)
    kept, n = so.evict(w, [8], 8, 4, 1)
    assert kept.tolist() == [[[0, 2, 3, 7]]] and n.tolist() == [4]
    assert so.evict(w, [8], 8, 3, 3)[0].tolist() == [[[5, 6, 7]]]
    assert so.evict(w, [3], 8, 4, 2)[0].tolist() == [[[0, 1, 2, -1]]]
    w[0, 0, 2] = np.nan
    assert so.evict(w, [8], 8, 4, 0)[0].tolist() == [[[0, 3, 5, 7]]]
