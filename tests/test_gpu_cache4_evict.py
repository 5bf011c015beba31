"""Eviction by accumulated weight: the slots that stay, exactly, and their rows, byte for byte."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import dev, host, make_cache

pytestmark = pytest.mark.gpu


def case(seed, B, H, D, page, group, lengths, keep, recent, weights=None, bad=()):
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(seed)
    columns, out_columns = -(-max(max(lengths), 1) // page) + 1, -(-keep // page)
    c, table = make_cache(seed, B, H, D, page, group, lengths, columns, bad, spare=B * out_columns + 2)
    free = np.setdiff1d(np.arange(c.num_pages, dtype=np.int32), table)
    out_table = g.permutation(free)[:B * out_columns].reshape(B, out_columns).astype(np.int32)
    w = np.exp(2 * g.standard_normal((B, H, columns * page + 3))).astype(np.float32) if weights is None else weights(g, (B, H, columns * page + 3))
    cache = dev(c.data)
    kept, n, ow = sage.sage_cache4_evict(cache, dev(table), dev(np.int32(lengths)), dev(w), dev(out_table), keep, recent, D, page, group)
    want, wn = so.evict(w, lengths, columns * page, keep, recent)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(n.cpu().numpy(), wn)
    picked = np.take_along_axis(w, np.maximum(want, 0).astype(np.int64), -1)
    full = np.zeros((B, H, out_columns * page), np.float32)
    full[..., :keep] = np.where(want >= 0, picked, 0)
    assert np.array_equal(ow.cpu().numpy().view(np.uint32), full.view(np.uint32))
    # the bytes of the rows, and nothing else written
    before = so.Cache(c.num_pages, H, D, page, group, c.data)
    for b in range(B):
        for h in range(H):
            for j in range(wn[b]):
                src, dst = before._place(table[b], int(want[b, h, j])), c._place(out_table[b], j)
                for to, part in zip(c._parts(dst[0], h, dst[1]), range(4)):
                    to[:] = before._parts(src[0], h, src[1])[part] if src is not None else (0x88 if part < 2 else 0)
    assert np.array_equal(cache.cpu().numpy(), c.data)


@pytest.mark.parametrize("D,group,page", [(64, 32, 16), (64, 64, 32), (128, 32, 64), (128, 64, 16), (128, 128, 256)])
@pytest.mark.parametrize("lengths,keep,recent", [([1, 0, 5], 1, 0), ([40, 41, 39], 40, 8), ([100, 200, 33], 50, 50), ([300, 17, 64], 33, 0),
                                                  ([1100, 900, 1030], 100, 7)])
def test_kept_slots_and_rows(D, group, page, lengths, keep, recent):
    case(sum(lengths), 3, 2, D, page, group, lengths, keep, recent)


def test_ties_go_to_the_lowest_slot():
    case(1, 2, 2, 64, 16, 32, [700, 650], 300, 20, lambda g, s: g.integers(0, 3, s).astype(np.float32))
    case(2, 2, 2, 64, 16, 32, [700, 650], 300, 20, lambda g, s: np.zeros(s, np.float32))


def test_signs_zeros_infinities_and_nan():
    def odd(g, s):
        w = (g.standard_normal(s) * 10.0 ** g.integers(-42, 30, s)).astype(np.float32)
        w[g.random(s) < 0.2] = 0.0
        w[g.random(s) < 0.2] = -0.0
        w[g.random(s) < 0.05] = np.inf
        w[g.random(s) < 0.05] = -np.inf
        w[g.random(s) < 0.1] = np.nan
        return w
    for keep in (10, 200, 560, 595):
        case(keep, 2, 2, 64, 16, 32, [600, 598], keep, 4, odd)


def test_pages_that_are_none():
    case(3, 2, 1, 64, 16, 32, [60, 64], 40, 8, bad=[(0, 1), (1, 3)])


def test_into_another_pool_and_long():
    import paper_2410_02367_amd as sage
    D, page, group, n, keep, recent = 128, 64, 128, 50001, 20000, 64
    g = np.random.default_rng(4)
    nb = sage.sage_cache4_block_bytes(D, page, group)
    cache = dev(g.integers(0, 256, (800, 1, nb), dtype=np.uint8))
    table = dev(g.permutation(800)[:782].astype(np.int32)[None])
    w = np.round(g.standard_normal((1, 1, 782 * page)) * 300).astype(np.float32)
    other = torch.zeros((313, 1, nb), dtype=torch.uint8, device="cuda")
    before = cache.clone()
    kept, m, _ = sage.sage_cache4_evict(cache, table, dev(np.int32([n])), dev(w), dev(np.arange(313, dtype=np.int32)[None]), keep, recent, D, page,
                                        group, out_cache=other)
    order = np.lexsort((np.arange(n - recent), -w[0, 0, :n - recent]))[:keep - recent]
    want = np.concatenate((np.sort(order), np.arange(n - recent, n)))
    assert np.array_equal(kept.cpu().numpy()[0, 0], want) and m.tolist() == [keep] and torch.equal(cache, before)
    a = sage.sage_cache4_load(cache, table, None, n, D, page=page, group=group)
    b = sage.sage_cache4_load(other, dev(np.arange(313, dtype=np.int32)[None]), None, keep, D, page=page, group=group)
    at = dev(want)
    for x, y in zip(a, b):
        assert torch.equal(x[:, :, at].view(torch.int16), y.view(torch.int16))


def bits(low, high):
    """Weights whose bit patterns are evenly spread: as many powers of two as there are."""
    return lambda g, s: g.integers(low, high, s, dtype=np.uint32).view(np.float32)


@pytest.mark.parametrize("weights", [bits(0, 0x7f800000), bits(0x3f800000, 0x3f800800), bits(0x3f800000, 0x3f800801), bits(0x3f800000, 0x3f800002),
                                     lambda g, s: np.where(g.random(s) < 0.9, 1.0, g.random(s)).astype(np.float32),
                                     lambda g, s: np.where(g.random(s) < 0.97, 2.0 ** -100, np.repeat(g.random((*s[:2], 1)), s[2], 2)).astype(np.float32),
                                     lambda g, s: np.where(g.random(s) < 0.01, np.inf, 1.0 + g.integers(0, 90, s) * 2.0 ** -23).astype(np.float32)],
                         ids=["all", "2048", "2049", "two", "mostly one", "mostly the least", "neighbours"])
@pytest.mark.parametrize("keep", [9, 65, 700, 1090])
def test_weights_that_are_alike(weights, keep):
    case(keep, 2, 2, 64, 16, 32, [1100, 1095], keep, 8, weights)


def test_many_alike_beyond_the_registers():
    # one key in 1000 differs; 40000 of them
    case(7, 1, 1, 64, 256, 64, [40000], 39950, 3, lambda g, s: np.where(g.random(s) < 1e-3, g.random(s), 0.5).astype(np.float32))
    case(8, 1, 1, 64, 256, 64, [40000], 60, 3, bits(0x3f800000, 0x40000000))
