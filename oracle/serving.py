"""Plain definitions of the serving calls in numpy, fp64 unless a step is fp32 or fp16 by definition: rotary positions, the
cache held in 4 bits, attention over it, the weight of each key, eviction.  Written from the formulas, token by token and head
by head; shares nothing with the kernels."""
from __future__ import annotations

import numpy as np


# ---- rotary positions

def rope(x, positions, inv_freq, interleaved=False, amplitude=1.0, backward=False):
    """x [B,H,N,D] (any float type) -> fp64: pair i turned by positions[b, n] * inv_freq[i]."""
    x = np.asarray(x, np.float64)
    B, H, N, D = x.shape
    half = len(inv_freq)
    positions = np.broadcast_to(np.asarray(positions, np.float64), (B, N))
    y = x.copy()
    for i, f in enumerate(np.asarray(inv_freq, np.float64)):
        first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = positions * f * (-1.0 if backward else 1.0)
        c, s = amplitude * np.cos(angle)[:, None], amplitude * np.sin(angle)[:, None]
        y[..., first] = x[..., first] * c - x[..., second] * s
        y[..., second] = x[..., second] * c + x[..., first] * s
    return y


# ---- the cache

def psi4(x, group):
    """Section 3.2's quantizer with 7 in place of 127: fp32 [..., D] -> (codes int8, scales fp16 [..., D / group])"""
    x = np.asarray(x, np.float32)
    g = x.reshape(*x.shape[:-1], -1, group)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        amax = np.where(np.isnan(g), np.float32(0), np.abs(g)).max(-1)
        scale = np.minimum(amax / np.float32(7), np.float32(65504)).astype(np.float16)
        step = scale.astype(np.float32)[..., None]
        code = np.clip(np.rint(g / step), -7, 7)
        code = np.where((step > 0) & ~np.isnan(g), code, 0)
    return code.reshape(x.shape).astype(np.int8), scale


def block_bytes(D, page, group):
    return page * (D + 4 * (D // group))


class Cache:
    """A pool of pages as bytes, written and read one token and head at a time."""

    def __init__(self, num_pages, heads, D, page, group, data=None):
        self.num_pages, self.heads, self.D, self.page, self.group = num_pages, heads, D, page, group
        self.data = np.zeros((num_pages, heads, block_bytes(D, page, group)), np.uint8) if data is None else np.array(data, np.uint8)

    def _parts(self, page, head, row):
        """the bytes of a token's K codes, V codes, K scales and V scales"""
        b, half, sc = self.data[page, head], self.D // 2, 2 * (self.D // self.group)
        at = [row * half, self.page * half + row * half, self.page * self.D + row * sc, self.page * (self.D + sc) + row * sc]
        return [b[a:a + n] for a, n in zip(at, (half, half, sc, sc))]

    def _k_nibble(self, d):
        i, h, e = d // 32, d % 32 // 8, d % 8
        return 8 * (h * self.D // 32 + i) + e // 2 + 4 * (e % 2)

    def _place(self, table_row, slot):
        """(page, row) of a slot, or None where the table has no page for it"""
        if slot < 0 or slot >= len(table_row) * self.page:
            return None
        p = int(table_row[slot // self.page])
        return (p, slot % self.page) if 0 <= p < self.num_pages else None

    def append(self, k, v, table, start, count=None, k_mean=None):
        k, v = np.asarray(k, np.float32), np.asarray(v, np.float32)
        B, H, N, D = k.shape
        if k_mean is not None:
            k = k - np.asarray(k_mean, np.float32)[:, :, None]
        kc, ks = psi4(k, self.group)
        vc, vs = psi4(v, self.group)
        for b in range(B):
            for n in range(N if count is None else min(N, int(count[b]))):
                at = self._place(table[b], int(start[b]) + n)
                if at is None:
                    continue
                for h in range(H):
                    pk, pv, psk, psv = self._parts(at[0], h, at[1])
                    for part, code, place in ((pk, kc[b, h, n], self._k_nibble), (pv, vc[b, h, n], lambda d: d)):
                        nib = np.zeros(D, np.uint8)
                        nib[[place(d) for d in range(D)]] = (code + 8).astype(np.uint8)
                        part[:] = nib[0::2] | (nib[1::2] << 4)
                    psk[:] = ks[b, h, n].view(np.uint8)
                    psv[:] = vs[b, h, n].view(np.uint8)

    def load(self, table, start, N, count=None, k_mean=None):
        """-> K, V [B,H,N,D] fp64, and there [B,N]: whether a slot holds a token"""
        B = len(table)
        k, v = np.zeros((B, self.heads, N, self.D)), np.zeros((B, self.heads, N, self.D))
        there = np.zeros((B, N), bool)
        for b in range(B):
            for n in range(N if count is None else max(0, min(N, int(count[b])))):
                at = self._place(table[b], (0 if start is None else int(start[b])) + n)
                if at is None:
                    continue
                there[b, n] = True
                for h in range(self.heads):
                    pk, pv, psk, psv = self._parts(at[0], h, at[1])
                    for to, part, scale, place in ((k, pk, psk, self._k_nibble), (v, pv, psv, lambda d: d)):
                        nib = np.stack((part & 15, part >> 4), -1).reshape(-1)
                        code = nib[[place(d) for d in range(self.D)]].astype(np.float64) - 8
                        to[b, h, n] = code * np.repeat(scale.copy().view(np.float16).astype(np.float64), self.group)
                if k_mean is not None:
                    k[b, :, n] += np.asarray(k_mean, np.float64)[b]
        return k, v, there


# ---- attention over it

def attention(q, k, v, there, lengths, count=None, causal=True, sm_scale=None):
    """q [B,Hq,Nq,D] over K, V [B,Hkv,capacity,D] -> out, lse, weights [B,Hkv,capacity] (sums of the softmax), all fp64."""
    q = np.asarray(q, np.float64)
    B, Hq, Nq, D = q.shape
    Hkv, capacity = k.shape[1], k.shape[2]
    sm_scale = 1.0 / np.sqrt(D) if sm_scale is None else sm_scale
    out, lse, weights = np.zeros(q.shape), np.full((B, Hq, Nq), -np.inf), np.zeros((B, Hkv, capacity))
    for b in range(B):
        length = min(max(int(lengths[b]), 0), capacity)
        n = Nq if count is None else min(max(int(count[b]), 0), Nq)
        for t in range(n):
            end = min(length, length - n + t + 1) if causal else length
            see = np.flatnonzero(there[b, :max(end, 0)])
            if len(see) == 0:
                continue
            for hq in range(Hq):
                h = hq // (Hq // Hkv)
                s = k[b, h, see] @ q[b, hq, t] * sm_scale
                top = s.max()
                e = np.exp(s - top)
                total = e.sum()
                lse[b, hq, t] = top + np.log(total)
                out[b, hq, t] = (e / total) @ v[b, h, see]
                weights[b, h, see] += e / total
    return out, lse, weights


# ---- eviction

def evict(weights, lengths, capacity, keep, recent):
    """-> kept [B,H,keep] (slots, then -1), new lengths"""
    B, H, _ = weights.shape
    kept = np.full((B, H, keep), -1, np.int32)
    new = np.zeros(B, np.int32)
    for b in range(B):
        n = min(max(int(lengths[b]), 0), capacity)
        new[b] = min(n, keep)
        for h in range(H):
            if n <= keep:
                stay = list(range(n))
            else:
                w = [(-np.inf, -1) if np.isnan(x) else (float(x), 0) for x in weights[b, h, :n - recent]]
                best = sorted(range(n - recent), key=lambda i: (tuple(-y for y in w[i]), i))[:keep - recent]
                stay = sorted(best) + list(range(n - recent, n))
            kept[b, h, :len(stay)] = stay
    return kept, new
