"""Attention over the cache held in 4 bits, cut in every way that a call can be: sequences and heads dealt out to the chip's parts,
tiles of rows, chunks of keys and what joins them."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, attention_bounds, dev, host, make_cache, rounded

pytestmark = pytest.mark.gpu


def case(seed, B, Hq, Hkv, Nq, D, page, group, lengths, columns, n_splits, chunks, kind="f16", count=None, causal=True, q_gain=1.5):
    """chunks: how many the keys are cut into (1: no scratch)"""
    import paper_2410_02367_amd as sage
    need = sage.sage_cache4_attn_workspace(B, Hq, Hkv, Nq, D, columns, page, n_splits)
    assert need == (0 if chunks == 1 else chunks * B * Hq * Nq * (D + 1) * 4)
    c, table = make_cache(seed, B, Hkv, D, page, group, lengths, columns)
    q = rounded(np.random.default_rng(seed).standard_normal((B, Hq, Nq, D)) * q_gain, kind)
    k, v, there = c.load(table, None, max(lengths), lengths)
    want, lse, _ = so.attention(q, k, v, there, lengths, count, causal)
    # what is not written shows
    out = torch.full((B, Hq, Nq, D), float("nan"), dtype=TORCH[kind], device="cuda")
    got_lse = torch.full((B, Hq, Nq), float("nan"), device="cuda")
    workspace = torch.full((max(need, 1),), 0xff, dtype=torch.uint8, device="cuda")
    sage.sage_cache4_attn(dev(q, TORCH[kind]), dev(c.data), dev(table), dev(np.int32(lengths)), None if count is None else dev(np.int32(count)), causal,
                          page=page, group=group, n_splits=n_splits, out=out, lse=got_lse, workspace=workspace)
    do, dl = attention_bounds(q, k, v, there, lengths, count, causal, 1 / np.sqrt(D), lse)
    err = np.abs(host(out) - want)
    assert np.all(err <= do + HALF_STEP[kind] * np.abs(want) + TINY[kind])
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(host(got_lse)), empty) and not host(out)[empty].any()
    assert np.all(np.abs(host(got_lse)[~empty] - lse[~empty]) <= dl[~empty])


# sequences times key heads a multiple of 8, several tiles of rows: dealt out to the XCDs
@pytest.mark.parametrize("B,Hkv", [(1, 8), (2, 8), (8, 3), (4, 12)])
@pytest.mark.parametrize("D,group,page", [(64, 32, 16), (128, 64, 64)])
@pytest.mark.parametrize("chunks", [1, 3])
def test_slabs_dealt_out_with_32_rows(B, Hkv, D, group, page, chunks):
    lengths = [720 - 40 * b for b in range(B)]
    count = [40] + [max(0, 40 - 13 * b) for b in range(1, B)]
    case(B + D, B, 2 * Hkv, Hkv, 40, D, page, group, lengths, 768 // page, chunks, chunks, "bf16", count)


@pytest.mark.parametrize("B,Hkv", [(1, 8), (2, 8)])
@pytest.mark.parametrize("D,group,page,length,room,chunks", [(64, 64, 64, 170, 2048, 1), (128, 128, 64, 170, 2048, 1), (128, 32, 128, 2300, 4096, 2)])
def test_slabs_dealt_out_with_128_rows(B, Hkv, D, group, page, length, room, chunks):
    Nq = 150
    case(B + D + chunks, B, 2 * Hkv, Hkv, Nq, D, page, group, [length - 20 * b for b in range(B)], room // page, chunks, chunks, "f16",
         [Nq - 60 * b for b in range(B)])


# chunks of 256 keys, all with keys: as many as the join takes at once, one more, more than a round of it
@pytest.mark.parametrize("q_gain", [1.5, 20.0])
@pytest.mark.parametrize("D,group,page,chunks", [(64, 32, 64, 2), (64, 32, 16, 4), (64, 64, 64, 5), (64, 32, 256, 16), (64, 32, 64, 17), (64, 64, 128, 65),
                                                 (128, 128, 64, 3), (128, 32, 64, 4), (128, 64, 32, 5), (128, 32, 256, 8), (128, 128, 64, 9),
                                                 (128, 32, 64, 33)])
@pytest.mark.parametrize("Hq,Nq", [(4, 1), (8, 3)])
def test_joins_of_chunks(D, group, page, chunks, q_gain, Hq, Nq):
    room = 256 * chunks
    case(chunks + D, 2, Hq, 2, Nq, D, page, group, [room, room // 2 + 77], room // page, chunks, chunks, "f16", q_gain=q_gain)


@pytest.mark.parametrize("D,group,chunks", [(64, 32, 4), (64, 32, 6), (128, 64, 3), (128, 64, 7)])
def test_joins_of_many_rows(D, group, chunks):
    """More than 2048 rows: each has its threads alone."""
    room = 256 * chunks
    case(chunks, 1, 8, 2, 260, D, 64, group, [room], room // 64, chunks, chunks, "bf16", q_gain=4.0)


@pytest.mark.parametrize("chunks", [5, 17])
def test_joins_of_sequences_that_end_in_an_earlier_chunk(chunks):
    room = 256 * chunks
    case(chunks, 5, 4, 4, 2, 64, 64, 32, [1, room, 256, 257, 0], room // 64, chunks, chunks, "f16", count=[2, 2, 1, 2, 2])
