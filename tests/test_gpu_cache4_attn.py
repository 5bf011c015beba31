"""Attention over the cache held in 4 bits, and the weight of each key, against the fp64 definition."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, attention_bounds, dev, host, make_cache, rounded

pytestmark = pytest.mark.gpu


def case(seed, B, Hq, Hkv, Nq, D, page, group, kind, lengths, count=None, causal=True, bad=(), extra=1, q_gain=1.5, n_splits=0,
         sm_scale=None, gain=1.0, weights=True):
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(seed)
    columns = -(-max(max(lengths), 1) // page) + extra
    capacity = columns * page
    c, table = make_cache(seed, B, Hkv, D, page, group, [max(0, min(n, capacity)) for n in lengths], columns, bad, gain=gain)
    q = rounded(g.standard_normal((B, Hq, Nq, D)) * q_gain, kind)
    k, v, there = c.load(table, None, capacity, [max(0, min(n, capacity)) for n in lengths])
    scale = 1 / np.sqrt(D) if sm_scale is None else sm_scale
    want, lse, w = so.attention(q, k, v, there, lengths, count, causal, scale)
    args = (dev(q, TORCH[kind]), dev(c.data), dev(table), dev(np.int32(lengths)))
    form = dict(count=None if count is None else dev(np.int32(count)), causal=causal, sm_scale=sm_scale, page=page, group=group)
    out, got_lse = sage.sage_cache4_attn(*args, n_splits=n_splits, return_lse=True, **form)
    do, dl = attention_bounds(q, k, v, there, lengths, count, causal, scale, lse)
    err = np.abs(host(out) - want)
    bound = do + HALF_STEP[kind] * np.abs(want) + TINY[kind]
    assert np.all(err <= bound), ("out", (err / bound).max())
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(host(got_lse)), empty) and not host(out)[empty].any()
    err = np.abs(host(got_lse)[~empty] - lse[~empty])
    assert np.all(err <= dl[~empty]), ("lse", (err / dl[~empty]).max())
    assert torch.equal(out, sage.sage_cache4_attn(*args, n_splits=n_splits, **form))
    if not weights:
        return
    had = np.abs(g.standard_normal((B, Hkv, capacity + 5))).astype(np.float32)
    mine = dev(had)
    got = sage.sage_cache4_weights(*args, got_lse, mine, out=mine, **form)
    assert got is mine
    # a weight is off by what its score and its row's lse are, the sum by a rounding per term
    rel = 2 * 2 * dl.max() + (Nq * Hq // Hkv + 8) * 2.0 ** -24
    full = had.astype(np.float64)
    full[..., :capacity] += w
    err = np.abs(host(got) - full)
    assert np.all(err[..., :capacity] <= rel * w + 2.0 ** -23 * full[..., :capacity] + 2.0 ** -40), "weights"
    assert np.array_equal(host(got)[..., capacity:], had[..., capacity:])
    only = sage.sage_cache4_weights(*args, got_lse, **form)
    assert only.shape == (B, Hkv, capacity) and np.all(np.abs(host(only) - w) <= rel * w + 2.0 ** -40)


FORMS = [(64, 32, 16), (64, 64, 64), (128, 32, 16), (128, 64, 32), (128, 128, 256)]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("lengths", [[1, 0, 2], [15, 16, 17], [63, 65, 64], [130, 257, 100]])
def test_one_token(D, group, page, lengths, kind):
    case(sum(lengths), 3, 4, 2, 1, D, page, group, kind, lengths)


@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("Hq,Hkv,Nq", [(1, 1, 2), (7, 1, 3), (3, 3, 17), (8, 2, 5), (12, 1, 6), (2, 2, 70), (16, 2, 9)])
def test_heads_and_queries(Hq, Hkv, Nq, D, group, page):
    # the second sequence has fewer tokens than queries: its first ones see nothing
    case(Hq + Nq, 2, Hq, Hkv, Nq, D, page, group, "f16", [Nq + 83, max(1, Nq - 1)])


# 3 to 16 rows of queries per key head: one, two and four of them per lane
@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("Hq,Hkv,Nq", [(3, 1, 1), (5, 1, 1), (14, 2, 1), (8, 1, 1), (9, 1, 1), (6, 2, 5), (16, 1, 1)])
def test_a_few_rows(Hq, Hkv, Nq, D, group, page):
    case(100 + Hq + Nq, 3, Hq, Hkv, Nq, D, page, group, "bf16", [Nq + 83, 2, 300], count=[Nq, 1, max(1, Nq - 1)])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,group,page", FORMS[1:4])
def test_padded_batch(D, group, page, causal):
    case(5, 5, 4, 2, 9, D, page, group, "bf16", [100, 40, 9, 3, 0], count=[9, 1, 0, 9, 4], causal=causal)


@pytest.mark.parametrize("Nq", [1, 4, 33])
def test_pages_that_are_none(Nq):
    case(6, 3, 4, 2, Nq, 64, 16, 32, "f16", [150, 64, 40], bad=[(0, 0), (0, 4), (1, 3), (2, 0), (2, 1), (2, 2)])


@pytest.mark.parametrize("n_splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("Nq", [1, 40])
def test_keys_shared_by_workgroups(n_splits, Nq):
    case(7, 2, 4, 1, Nq, 128, 64, 32, "f16", [1100, 130], n_splits=n_splits)


# a table with room for 2048 tokens and more: with one chunk, the form for many rows
@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("Hq,Hkv,Nq,lengths,count", [(1, 1, 97, [97, 300], None), (8, 2, 33, [200, 20], None), (4, 1, 70, [70, 333], [70, 3]),
                                                     (6, 2, 128, [1, 129], [128, 128])])
def test_many_rows(Hq, Hkv, Nq, lengths, count, D, group, page, kind):
    case(Nq + page, 2, Hq, Hkv, Nq, D, page, group, kind, lengths, count, extra=2048 // page, n_splits=1, weights=False)


@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_pages_that_are_none_and_several_chunks(causal):
    case(21, 2, 2, 1, 60, 64, 16, 32, "f16", [150, 64], bad=[(0, 0), (0, 4), (1, 3), (1, 2)], extra=128, n_splits=1, causal=causal, weights=False)
    case(22, 1, 2, 1, 49, 128, 64, 32, "f16", [2700], extra=24, n_splits=2, causal=causal, weights=False)
    case(23, 1, 1, 1, 130, 128, 64, 64, "f16", [4200], q_gain=25.0, n_splits=2, causal=causal, weights=False)
    case(24, 2, 4, 2, 80, 64, 16, 64, "bf16", [90, 85], extra=128, n_splits=1, q_gain=25.0, causal=causal, weights=False)


# tables with room for 1K, 8K and 16K tokens: 64 keys per workgroup with 8 or 4 wavefronts, and 256 keys
@pytest.mark.parametrize("room", [1024, 8192, 16384])
@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("Hq,Hkv,Nq,lengths,count,causal", [(2, 2, 65, [65, 300], None, True), (6, 2, 41, [200, 20], [41, 30], True),
                                                           (2, 2, 150, [70, 333], [149, 3], False), (14, 2, 30, [1, 129], [30, 0], True)])
def test_weights_of_many_rows(Hq, Hkv, Nq, lengths, count, causal, D, group, page, room):
    case(Nq + page, 2, Hq, Hkv, Nq, D, page, group, "bf16", lengths, count, causal, extra=room // page)


@pytest.mark.parametrize("room", [1024, 8192, 16384])
def test_weights_of_many_rows_with_pages_that_are_none(room):
    case(31, 2, 4, 2, 60, 64, 16, 32, "f16", [150, 64], bad=[(0, 0), (0, 4), (1, 3), (1, 2)], extra=room // 16)


def test_lengths_beyond_the_table_and_below_zero():
    case(8, 3, 2, 2, 3, 64, 16, 64, "f16", [40, 7, 33], count=[5, -1, 3])
    import paper_2410_02367_amd as sage
    c, table = make_cache(8, 2, 1, 64, 16, 32, [32, 32], 2)
    q = dev(np.random.default_rng(1).standard_normal((2, 1, 1, 64)), torch.float16)
    at = [sage.sage_cache4_attn(q, dev(c.data), dev(table), dev(np.int32(n)), page=16) for n in ([32, 0], [2 ** 31 - 1, -2 ** 31])]
    assert torch.equal(at[0], at[1]) and not at[1][1].any()


@pytest.mark.parametrize("D,group,page", FORMS)
def test_peaked_rows_and_scales_far_apart(D, group, page):
    """Scores up to +-200 apart, and values whose scales span 2^20: the large values at keys of next to no weight do not cost
    the small ones their precision."""
    case(9, 2, 4, 2, 3, D, page, group, "f16", [200, 90], q_gain=25.0)
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(10)
    H, n = 1, 150
    k = rounded(g.standard_normal((1, H, n, D)), "f16")
    v = rounded(g.standard_normal((1, H, n, D)) * 2.0 ** -8, "f16")
    q = rounded(g.standard_normal((1, 2, 1, D)) * 0.1, "f16")
    # a direction that only every seventh key has: its score is 40 lower, its values 2^20 times larger
    k[..., 0], q[..., 0] = 0.0, 4.0
    k[:, :, ::7, 0] = -10.0 * np.sqrt(D)
    v[:, :, ::7] *= 2.0 ** 18
    c, table = make_cache(3, 1, H, D, page, group, [0], -(-n // page))
    c.append(k, v, table, [0])
    kk, vv, there = c.load(table, None, n)
    want, lse, w = so.attention(q, kk, vv, there, [n])
    out = sage.sage_cache4_attn(dev(q, torch.float16), dev(c.data), dev(table), dev(np.int32([n])), page=page, group=group)
    do, _ = attention_bounds(q, kk, np.where(np.arange(n)[:, None] % 7 == 0, 0.0, vv), there, [n], None, True, 1 / np.sqrt(D), lse)
    heavy = np.abs(so.attention(q, kk, np.where(np.arange(n)[:, None] % 7 == 0, np.abs(vv), 0.0), there, [n])[0])
    assert np.all(np.abs(host(out) - want) <= do + heavy * 2.0 ** -9 + 2.0 ** -11 * np.abs(want) + 2.0 ** -25)


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_values_that_are_all_zero_and_scales_at_the_edges(kind):
    import paper_2410_02367_amd as sage
    D, page, group, n = 64, 16, 32, 70
    g = np.random.default_rng(11)
    q = dev(g.standard_normal((1, 2, 1, D)), TORCH[kind])
    for gain in (0.0, 2.0 ** -20, 9000.0):
        c, table = make_cache(4, 1, 1, D, page, group, [0], 5)
        k = g.standard_normal((1, 1, n, D)).astype(np.float16)
        v = (g.standard_normal((1, 1, n, D)) * gain).astype(np.float16)
        c.append(k, v, table, [0])
        kk, vv, there = c.load(table, None, n)
        want, lse, _ = so.attention(host(q), kk, vv, there, [n])
        out, got = sage.sage_cache4_attn(q, dev(c.data), dev(table), dev(np.int32([n])), page=page, group=group, return_lse=True)
        do, dl = attention_bounds(host(q), kk, vv, there, [n], None, True, 1 / np.sqrt(D), lse)
        assert np.all(np.abs(host(out) - want) <= do + HALF_STEP[kind] * np.abs(want) + TINY[kind])
        assert np.all(np.abs(host(got) - lse) <= dl)


def test_queries_of_any_size_and_not_numbers():
    """bf16 queries far outside fp16's range, zeros, and a NaN or an infinity that stays in its row."""
    import paper_2410_02367_amd as sage
    D, page, group, n = 128, 16, 32, 90
    c, table = make_cache(5, 1, 1, D, page, group, [n], 6)
    kk, vv, there = c.load(table, None, n)
    g = np.random.default_rng(12)
    q = rounded(g.standard_normal((1, 1, 20, D)), "bf16")
    q[0, 0, 0] *= 2.0 ** 100
    q[0, 0, 1] *= 2.0 ** -100
    q[0, 0, 2] = 0.0
    q[0, 0, 3, 1:] *= 2.0 ** -30
    q[0, 0, 4] *= 2.0 ** -120
    for scale in (2.0 ** -100, 0.1):
        keep = slice(0, 5) if scale != 0.1 else slice(1, 20)
        want, lse, _ = so.attention(q[:, :, keep], kk, vv, there, [n], None, False, scale)
        args = (dev(c.data), dev(table), dev(np.int32([n])))
        out = sage.sage_cache4_attn(dev(q[:, :, keep], torch.bfloat16), *args, causal=False, sm_scale=scale, page=page, group=group)
        do, _ = attention_bounds(q[:, :, keep], kk, vv, there, [n], None, False, scale, lse)
        assert np.all(np.abs(host(out) - want) <= do + 2.0 ** -8 * np.abs(want))
    q = q[:, :, 5:]
    clean = sage.sage_cache4_attn(dev(q, torch.bfloat16), *args, causal=False, page=page, group=group)
    q[0, 0, 3, 7], q[0, 0, 9, 100] = np.nan, np.inf
    out = sage.sage_cache4_attn(dev(q, torch.bfloat16), *args, causal=False, page=page, group=group)
    rest = [t for t in range(15) if t not in (3, 9)]
    assert torch.equal(out[0, 0, rest], clean[0, 0, rest]) and torch.isnan(out[0, 0, 3]).all()


def test_strides():
    import paper_2410_02367_amd as sage
    B, Hq, Hkv, Nq, D, page, group = 2, 6, 2, 5, 64, 16, 32
    c, table = make_cache(6, B, Hkv, D, page, group, [60, 33], 4)
    g = np.random.default_rng(13)
    fused = dev(g.standard_normal((B, Nq, Hq + 4, D)), torch.bfloat16)
    q = fused[:, :, 2:2 + Hq].transpose(1, 2)
    args = (dev(c.data), dev(table), dev(np.int32([60, 33])))
    want, lse = sage.sage_cache4_attn(q.contiguous(), *args, page=page, return_lse=True)
    out = sage.sage_cache4_attn(q, *args, page=page)
    assert out.transpose(1, 2).is_contiguous() and torch.equal(out, want)
    frame = torch.full((B, Nq, Hq + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    sage.sage_cache4_attn(q, *args, page=page, out=frame[:, :, 1:].transpose(1, 2))
    assert torch.equal(frame[:, :, 1:].transpose(1, 2), want) and torch.all(frame[:, :, 0] == 7.0)
    assert torch.equal(sage.sage_cache4_weights(q, *args, lse, page=page), sage.sage_cache4_weights(q.contiguous(), *args, lse, page=page))


# at most four rows: their kernel's raised references, absent pages, cut keys, and rows that are no numbers
@pytest.mark.parametrize("D,group,page", FORMS)
@pytest.mark.parametrize("Hq,Hkv,Nq", [(1, 1, 1), (4, 2, 2), (3, 1, 1), (4, 1, 1), (2, 1, 2), (1, 1, 4)])
def test_up_to_four_rows(Hq, Hkv, Nq, D, group, page):
    case(50 + Hq + Nq, 2, Hq, Hkv, Nq, D, page, group, "f16", [1300, 333], q_gain=25.0, bad=[(0, 1), (1, 0)])
    case(60 + Hq + Nq, 3, Hq, Hkv, Nq, D, page, group, "bf16", [700, 3, 64], count=[Nq, 1, 0], n_splits=3, q_gain=10.0, causal=False)


@pytest.mark.parametrize("D,group,page", FORMS)
def test_four_rows_of_which_one_is_no_number(D, group, page):
    import paper_2410_02367_amd as sage
    n = 300
    c, table = make_cache(71, 1, 1, D, page, group, [n], -(-n // page))
    q = rounded(np.random.default_rng(71).standard_normal((1, 4, 1, D)) * 3, "f16")
    args = (dev(c.data), dev(table), dev(np.int32([n])))
    clean, lse = sage.sage_cache4_attn(dev(q, torch.float16), *args, page=page, group=group, return_lse=True)
    q[0, 2, 0, 5] = np.nan
    out, got = sage.sage_cache4_attn(dev(q, torch.float16), *args, page=page, group=group, return_lse=True)
    rest = [0, 1, 3]
    assert torch.equal(out[0, rest], clean[0, rest]) and torch.equal(got[0, rest], lse[0, rest])
    assert torch.isnan(out[0, 2]).all() and torch.isnan(got[0, 2]).all()
