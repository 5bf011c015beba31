"""Attention over the cache held in 4 bits where the groups of a token's channels differ in size: every group is held to a bound of its
own, relative to what its own values add up to."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, attention_bounds, dev, host, make_cache, rounded

pytestmark = pytest.mark.gpu

# (query heads, key heads, queries, room for tokens beyond the longest sequence, chunks): at most 4 rows, 16, 32 and 128 per workgroup
CALLS = {"four rows": (4, 1, 1, 0, 0), "four rows, three chunks": (3, 1, 1, 900, 3), "16 rows": (6, 2, 4, 0, 0), "32 rows": (8, 1, 9, 0, 0),
         "32 rows, three chunks": (8, 2, 5, 900, 3), "128 rows": (4, 1, 30, 2048, 1)}


def case(seed, D, page, group, kind, call, gains, q_gain=1.5, shape=None):
    """gains: log2 of each group's size; shape(v, q, k): changes of the inputs before they are stored"""
    import paper_2410_02367_amd as sage
    Hq, Hkv, Nq, room, n_splits = CALLS[call]
    g = np.random.default_rng(seed)
    B, lengths = 2, [230 + Nq, 77 + Nq]
    columns = -(-(max(lengths) + room) // page)
    c, table = make_cache(seed, B, Hkv, D, page, group, [0] * B, columns)
    k = g.standard_normal((B, Hkv, max(lengths), D))
    v = g.standard_normal((B, Hkv, max(lengths), D)) * np.repeat(2.0 ** np.array(gains, np.float64), group)
    q = g.standard_normal((B, Hq, Nq, D)) * q_gain
    if shape is not None:
        shape(v, q, k)
    q = rounded(q, kind)
    c.append(rounded(k, "f16"), rounded(v, "f16"), table, [0] * B, lengths)
    kk, vv, there = c.load(table, None, columns * page, lengths)
    args = (dev(q, TORCH[kind]), dev(c.data), dev(table), dev(np.int32(lengths)))
    out, lse = sage.sage_cache4_attn(*args, page=page, group=group, n_splits=n_splits, return_lse=True)
    want, wl, _ = so.attention(q, kk, vv, there, lengths)
    _, ds = attention_bounds(q, kk, vv, there, lengths, None, True, 1 / np.sqrt(D), wl)
    scales = np.abs(vv).reshape(*vv.shape[:3], -1, group).max(-1)           # 7 scales at most
    bound = np.zeros(want.shape)
    for b in range(B):
        for hq in range(Hq):
            h = hq // (Hq // Hkv)
            for t in range(Nq):
                end = lengths[b] - Nq + t + 1
                p = np.exp(kk[b, h, :end] @ q[b, hq, t] / np.sqrt(D) - wl[b, hq, t])
                # a weight times its scale is rounded to fp16: 2^-11 of itself, or half a step of the subnormal numbers, 2^-25, for a key
                # whose weight is stored at 2^-4 2^-21.  The group's largest is stored at 2^2 at least (raised to 2^9 .. 2^10, 2^-7 of that
                # where a group shares another's reference): 2^-23 of it; codes are at most 7
                largest = np.repeat((p[:, None] * scales[b, h, :end]).max(0), group)
                bound[b, hq, t] = (p @ np.abs(vv[b, h, :end])) * (2.0 ** -11 + 3 * ds[b, hq, t]) + end * 2.0 ** -23 * largest
    bound += HALF_STEP[kind] * np.abs(want) + TINY[kind]
    err = np.abs(host(out) - want)
    assert np.all(err <= bound), [(e, (err / bound)[..., e * group:(e + 1) * group].max()) for e in range(D // group)]
    assert np.all(np.abs(host(lse) - wl) <= ds)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("D,group,page,gains", [(64, 32, 16, (10, -10)), (64, 32, 64, (-8, 5)), (128, 64, 32, (-10, 10)), (128, 64, 64, (0, -14)),
                                                (128, 32, 64, (-12, 8, -4, 1)), (128, 32, 16, (9, -4, 0, -12)), (128, 32, 256, (0, -8, -8, -8))])
def test_groups_of_different_sizes(D, group, page, gains, call):
    case(D + page, D, page, group, "f16", call, gains)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("D,group", [(64, 32), (128, 64), (128, 32)])
def test_a_group_whose_large_values_have_no_weight(D, group, call):
    """Every seventh key has next to no weight, and values 2^19 times the others' in one group only."""
    for which in (0, D // group - 1):
        def shape(v, q, k):
            k[..., 0], q[..., 0] = 0.0, 4.0
            k[:, :, ::7, 0] = -10.0 * np.sqrt(D)
            v *= 2.0 ** -8
            v[:, :, ::7, which * group:(which + 1) * group] *= 2.0 ** 19
        case(D + group + which, D, 32, group, "f16", call, (0,) * (D // group), 0.1, shape)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("q_gain", [0.5, 12.0])
@pytest.mark.parametrize("late", [5, 40, 64, 200])
def test_groups_without_values_and_peaked_rows(late, q_gain, call):
    def shape(v, q, k):
        v[..., 32:64] = 0.0
        v[:, :, :late, 64:96] = 0.0             # nothing in a group until late
    case(late, 128, 16, 32, "bf16", call, (8, 0, -6, -12), q_gain, shape)

    def shape(v, q, k):
        v[:, :, :late, :32] = 0.0
    case(late + 1, 64, 64, 32, "f16", call, (-12, 8), q_gain, shape)
    case(late + 2, 128, 64, 64, "f16", call, (-10, 10), q_gain, shape)
