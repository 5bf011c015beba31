"""Helpers of the serving tests: caches with shuffled pages and rubbish in every row that holds no token, the bounds that
results are held to."""
from __future__ import annotations

import numpy as np
import torch

import oracle.serving as so

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step relative to the value
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}       # half a step of the smallest numbers


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().double().cpu().numpy() if t.dtype.is_floating_point else t.cpu().numpy()


def rounded(a, kind):
    """fp64 values that are numbers of the type"""
    return torch.from_numpy(np.ascontiguousarray(a, np.float64)).to(TORCH[kind]).double().numpy()


def make_cache(seed, B, H, D, page, group, lengths, columns, bad=(), spare=3, gain=1.0):
    """A cache of tokens ~ N(0, gain^2): (oracle's cache, table); `bad`: (sequence, column) pairs whose table entry is no page.
    Rows without a token hold 0xff bytes: codes of 7 and scales that are NaN."""
    g = np.random.default_rng(seed)
    pool = B * columns + spare
    c = so.Cache(pool, H, D, page, group)
    c.data[:] = 0xff
    table = g.permutation(pool)[:B * columns].reshape(B, columns).astype(np.int32)
    wrong = (-1, pool, 2 ** 30, -2 ** 31)
    for i, (b, col) in enumerate(bad):
        table[b, col] = wrong[i % 4]
    n = max(1, max(lengths))
    k, v = (g.standard_normal((2, B, H, n, D)) * gain).astype(np.float16)
    c.append(k, v, table, [0] * B, lengths)
    return c, table


def attention_bounds(q, k, v, there, lengths, count, causal, sm_scale, lse):
    """How far out and lse may be off, without the rounding of the result.

    A score is a sum of D products (exact in fp32: 11 bits times 4) in fp32 times scales: D additions and a few products,
    2^-24 of the sum of magnitudes each.  A weight is the exponential of that (relative error: the score's, and 2^-21 of the
    exponential and its argument's rounding), times a scale and rounded to fp16: 2^-11 of itself, or 2^-25 of the largest one."""
    q = np.asarray(q, np.float64)
    T = np.einsum("bhtd,bhsd->bht", np.abs(q).reshape(q.shape[0], k.shape[1], -1, q.shape[3]), np.abs(k).max(2, keepdims=True)).reshape(q.shape[:3]) * sm_scale
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    ds = T * (q.shape[3] + 8) * 2.0 ** -24 + (1.0 + T + finite) * 2.0 ** -21 + k.shape[2] / 16 * 2.0 ** -24
    magnitude = so.attention(q, k, np.abs(v), there, lengths, count, causal, sm_scale)[0]
    top = np.abs(v).max()
    do = magnitude * (2.0 ** -11 + 3 * ds)[..., None] + k.shape[2] * 2.0 ** -25 * top
    return do, ds
