"""Binding of the serving calls of libsage.so (declared in include/sage.h): rotary positions, and the cache of K and V held
in 4 bits with what works on it.  Argument marshalling only, as in :mod:`binding`, but for sage_rope_frequencies() and the gradients of
the rotation: the extension module makes the calls that are in order, the code here the others, or their errors.  Results of the
other calls take no part in autograd.

Tensors are [B, H, N, D] with neighbouring channels and any distances between the rows (a transposed view of [B, N, H, D] as a
projection leaves it is taken as it is); all of a call's tensors are on one device, which need not be the current one."""
from __future__ import annotations

import contextlib
import ctypes
import math

import torch

from . import binding
from .binding import SageError, _answer, _fast, _handle, load

_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_HALVES = (torch.float16, torch.bfloat16)


def _tensor(t, name, dtypes, dims, device=None):
    """A device tensor of one of these types with so many dimensions, on `device` if one is named."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or t.dim() != dims:
        raise TypeError(f"{name}: expected a {dims}-dimensional tensor of {' or '.join(str(d) for d in dtypes)} in device memory")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: is on {t.device}, not on {device} as the call's other tensors are")
    return t


def _flat(t, name, dtype, shape, device):
    """A contiguous tensor of this type and shape."""
    _tensor(t, name, (dtype,), len(shape), device)
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, name):
    """Pointer and strides of a tensor whose channels are next to each other (None: contiguous)."""
    if t.stride(3) != 1 and t.shape[3] != 1:
        raise ValueError(f"{name}: the channels have to be next to each other")
    return t.data_ptr(), None if t.is_contiguous() else (ctypes.c_int64 * 3)(*t.stride()[:3])


def _maybe(t, name, dtype, shape, device):
    return None if t is None else _flat(t, name, dtype, shape, device)


def _like(x, out, name):
    """`out`, checked, or a new tensor laid out as x is where x's rows are its own."""
    if out is None:
        return torch.empty_like(x)
    _tensor(out, name, (x.dtype,), 4, x.device)
    if out.shape != x.shape:
        raise ValueError(f"{name}: expected shape {tuple(x.shape)}, got {tuple(out.shape)}")
    return out


@contextlib.contextmanager
def _placed(device, stream, caller):
    """The tensors' device and the call's stream as the current ones."""
    with torch.cuda.device(device):
        caller.append(torch.cuda.current_stream())
        if stream is None:
            yield
            return
        if not isinstance(stream, torch.cuda.Stream):
            handle = binding._stream(stream)
            stream = torch.cuda.ExternalStream(handle) if handle not in (0, 1) else torch.cuda.default_stream()
        with torch.cuda.stream(stream):
            yield


def _elsewhere(device, stream) -> bool:
    return device.index != torch._C._cuda_getDevice() or (stream is not None and binding._elsewhere(stream))


def _there(device, stream, call, *args, **kwargs):
    """call(..., stream=None) with the tensors' device and `stream` as the current ones: what the call allocates is then in
    the order of the stream that it is used on.  The caller's own stream is noted on new outputs, which it will read."""
    caller = []
    with _placed(device, stream, caller):
        r = call(*args, **kwargs)
    given = list(args) + list(kwargs.values())
    for t in r if isinstance(r, tuple) else (r,):
        if not any(t is a for a in given):
            t.record_stream(caller[0])
    return r


def _check(status, where):
    if status != 0:
        raise SageError(status, where)


# ---- rotary positions

def sage_rope_frequencies(rotated: int, base: float = 10000.0, scaling: str | None = None, factor: float = 1.0,
                          original_length: int = 8192, low: float = 1.0, high: float | None = None, device=None):
    """Radians per position of each pair of channels, fp64 [rotated / 2], and the amplitude that goes with them.
    base^(-2 i / rotated), for contexts `factor` times as long as the model's own changed by `scaling`:
      None      not
      "linear"  every frequency divided by factor (position interpolation)
      "base"    the base raised so that the slowest pair is divided by factor and the fastest stays
      "parts"   a pair that turns less than `low` times in original_length positions divided by factor, more than `high` times
                left, in between a mixture, linear in the number of turns
      "ramp"    the same with the mixture linear in the pair's index, and an amplitude of 0.1 ln(factor) + 1 (YaRN)
    high None: 32 for "ramp", 4 otherwise.
    """
    if high is None:
        high = 32.0 if scaling == "ramp" else 4.0
    if rotated < 2 or rotated % 2 != 0:
        raise ValueError("rotated: an even number of channels")
    if not (base > 0 and factor >= 1 and original_length > 0 and 0 < low < high):
        raise ValueError("base and original_length are positive, factor at least 1, 0 < low < high")
    if scaling == "ramp" and base <= 1:
        raise ValueError("base: above 1, where the pairs differ in frequency")
    index = torch.arange(0, rotated, 2, dtype=torch.float64)
    if scaling == "base":
        base = base * factor ** (rotated / (rotated - 2)) if rotated > 2 else base
    freq = base ** (-index / rotated)
    amplitude = 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling in ("parts", "ramp"):
        if scaling == "parts":
            turns = original_length * freq / (2 * math.pi)
            stay = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        else:
            def pair(turns):            # index of the pair that turns so often
                return rotated * math.log(original_length / (turns * 2 * math.pi)) / (2 * math.log(base))
            # (where all pairs turn more than `low` times the ramp ends behind the last one)
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotated - 1)
            stay = 1.0 - ((index / 2 - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
            amplitude = 0.1 * math.log(factor) + 1.0
        freq = freq * stay + freq / factor * (1.0 - stay)
    elif scaling not in (None, "base"):
        raise ValueError(f"scaling: {scaling!r} is none of 'linear', 'base', 'parts', 'ramp'")
    return freq.to(device), amplitude


def _rope(entry, x, y, positions, inv_freq, interleaved, amplitude, x_out, y_out, stream):
    _tensor(x, "q", tuple(_TYPES), 4)
    if _elsewhere(x.device, stream):
        return _there(x.device, stream, _rope, entry, x, y, positions, inv_freq, interleaved, amplitude, x_out, y_out, None)
    B, H, N, D = x.shape
    px, sx = _rows(x, "q")
    x_out = _like(x, x_out, "q_out")
    pxo, sxo = _rows(x_out, "q_out")
    Hk, py, sy, pyo, syo = 0, None, None, None, None
    if y is not None:
        _tensor(y, "k", (x.dtype,), 4, x.device)
        if y.shape[0] != B or y.shape[2] != N or y.shape[3] != D:
            raise ValueError("q and k differ in batch, tokens or head dimension")
        Hk = y.shape[1]
        py, sy = _rows(y, "k")
        y_out = _like(y, y_out, "k_out")
        pyo, syo = _rows(y_out, "k_out")
    positions_shape = (B, N) if isinstance(positions, torch.Tensor) and positions.dim() == 2 else (N,)
    pp = _flat(positions, "positions", torch.int32, positions_shape, x.device)
    _tensor(inv_freq, "inv_freq", (torch.float64,), 1, x.device)
    pf = _flat(inv_freq, "inv_freq", torch.float64, inv_freq.shape, x.device)
    _check(getattr(load(), entry)(px, sx, pxo, sxo, py, sy, pyo, syo, pp, N if len(positions_shape) == 2 else 0, pf, float(amplitude),
                                  B, H, Hk, N, D, 2 * inv_freq.shape[0], _TYPES[x.dtype], int(bool(interleaved)), binding._stream(None)), entry)
    return x_out if y is None else (x_out, y_out)


def _tracked(*tensors) -> bool:
    """Whether autograd takes note of a call (the extension module, which asks the same, leaves such calls to the code here)."""
    return any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors) and torch.is_grad_enabled()


def _whole_rows(t):
    """t, or a copy of it where its rows are not as the calls take them (a gradient may be an expanded number)."""
    if t is None or t.shape[3] < 2 or (t.stride(3) == 1 and all(x % 16 == 0 for x in (t.data_ptr(), *(s * t.element_size() for s in t.stride()[:3])))):
        return t
    return t.clone(memory_format=torch.contiguous_format)


class _Turn(torch.autograd.Function):
    """The rotation, or where `back` the turn back, each the gradient of the other."""

    @staticmethod
    def forward(ctx, q, k, positions, inv_freq, interleaved, amplitude, back):
        ctx.save_for_backward(positions, inv_freq)
        ctx.form, ctx.back = (interleaved, amplitude), back
        ctx.set_materialize_grads(False)
        r = (sage_rope_bwd if back else sage_rope)(q, k, positions, inv_freq, interleaved, amplitude)
        constant = [y for y, needed in zip((r,) if k is None else r, ctx.needs_input_grad) if not needed]
        ctx.mark_non_differentiable(*constant)
        return r

    @staticmethod
    def backward(ctx, *grads):
        positions, inv_freq = ctx.saved_tensors
        turn = sage_rope if ctx.back else sage_rope_bwd
        grads = [_whole_rows(g if needed else None) for g, needed in zip((*grads, None), ctx.needs_input_grad)][:2]
        there = [g for g in grads if g is not None]
        if len(there) == 2:
            grads = turn(*there, positions, inv_freq, *ctx.form)
        elif there:
            there = turn(there[0], None, positions, inv_freq, *ctx.form)
            grads = [None if g is None else there for g in grads]
        return (*grads, *[None] * 5)


def _turn(back, q, k, positions, inv_freq, interleaved, amplitude, q_out, k_out, stream):
    """A call that autograd takes note of."""
    _tensor(q, "q", tuple(_TYPES), 4)
    if q_out is not None or k_out is not None:
        raise ValueError("q_out, k_out: an output of the caller's has no gradient, but an input requires one")
    if _tracked(inv_freq):
        raise ValueError("inv_freq: there is no gradient of the frequencies")
    args = q, k, positions, inv_freq, interleaved, amplitude, back
    return _there(q.device, stream, _Turn.apply, *args) if _elsewhere(q.device, stream) else _Turn.apply(*args)


def sage_rope(q, k, positions, inv_freq, interleaved: bool = False, amplitude: float = 1.0, q_out=None, k_out=None, stream=None):
    """q [B,Hq,N,D] and k [B,Hk,N,D] (or None) with their pairs of channels turned by position * inv_freq -> (q', k'), or q'.
    positions int32 [N] or [B,N]; inv_freq fp64 [rotated / 2], the channels from `rotated` on pass; outputs may be the inputs.
    Differentiable in q and k, where no output is given: the gradients are sage_rope_bwd()'s."""
    r = _fast().rope(q, k, positions, inv_freq, interleaved, amplitude, q_out, k_out, _handle(stream))
    if r is not None:
        return _answer(r, "sage_rope")
    if _tracked(q, k, inv_freq):
        return _turn(False, q, k, positions, inv_freq, interleaved, amplitude, q_out, k_out, stream)
    return _rope("sage_rope", q, k, positions, inv_freq, interleaved, amplitude, q_out, k_out, stream)


def sage_rope_bwd(dq, dk, positions, inv_freq, interleaved: bool = False, amplitude: float = 1.0, dq_out=None, dk_out=None, stream=None):
    """The gradients of sage_rope()'s inputs from those of its outputs, dq [B,Hq,N,D] and dk [B,Hk,N,D] (or None).  Differentiable as
    that is."""
    r = _fast().rope_bwd(dq, dk, positions, inv_freq, interleaved, amplitude, dq_out, dk_out, _handle(stream))
    if r is not None:
        return _answer(r, "sage_rope_bwd")
    if _tracked(dq, dk, inv_freq):
        return _turn(True, dq, dk, positions, inv_freq, interleaved, amplitude, dq_out, dk_out, stream)
    return _rope("sage_rope_bwd", dq, dk, positions, inv_freq, interleaved, amplitude, dq_out, dk_out, stream)


# ---- the cache held in 4 bits

def sage_cache4_block_bytes(D: int, page: int = 64, group: int = 32) -> int:
    """Bytes of one head of one page: a cache is a uint8 tensor [num_pages, Hkv, sage_cache4_block_bytes(D, page, group)]."""
    return int(load().sage_cache4_block_bytes(int(D), int(page), int(group)))


def _cache(cache, pages, B, Hkv, D, page, group, device, name="cache", pages_name="pages"):
    """(pointer, number of pages, pointer of the table, its columns)"""
    need = sage_cache4_block_bytes(D, page, group)
    if need == 0:
        raise SageError(3, f"{name}: head dimension {D}, page {page}, group {group}")
    _tensor(cache, name, (torch.uint8,), 3, device)
    _flat(cache, name, torch.uint8, (cache.shape[0], Hkv, need), device)
    _tensor(pages, pages_name, (torch.int32,), 2, device)
    _flat(pages, pages_name, torch.int32, (B, pages.shape[1]), device)
    return cache.data_ptr(), cache.shape[0], pages.data_ptr(), pages.shape[1]


def sage_cache4_append(k, v, cache, pages, start, count=None, k_mean=None, page: int = 64, group: int = 32, stream=None):
    """New tokens k, v [B,Hkv,N,D] into slots start[b] .. of the sequences' pages, the first count[b] of each; k_mean [B,Hkv,D]
    fp32 is subtracted from the keys.  -> cache"""
    r = _fast().cache4_append(k, v, cache, pages, start, count, k_mean, page, group, _handle(stream))
    if r is not None:
        return _answer(r, "sage_cache4_append")
    _tensor(k, "k", _HALVES, 4)
    if _elsewhere(k.device, stream):
        return _there(k.device, stream, sage_cache4_append, k, v, cache, pages, start, count, k_mean, page, group)
    B, Hkv, N, D = k.shape
    dev = k.device
    _tensor(v, "v", (k.dtype,), 4, dev)
    if v.shape != k.shape:
        raise ValueError("k and v differ in shape")
    (pk, sk), (pv, sv) = _rows(k, "k"), _rows(v, "v")
    pc, P, pt, columns = _cache(cache, pages, B, Hkv, D, page, group, dev)
    _check(load().sage_cache4_append(pk, sk, pv, sv, _maybe(k_mean, "k_mean", torch.float32, (B, Hkv, D), dev), pc, pt,
                                     _flat(start, "start", torch.int32, (B,), dev), _maybe(count, "count", torch.int32, (B,), dev),
                                     B, Hkv, N, D, _TYPES[k.dtype], P, columns, page, group, binding._stream(None)), "sage_cache4_append")
    return cache


def sage_cache4_load(cache, pages, start, N: int, D: int, count=None, k_mean=None, dtype=torch.float16, page: int = 64, group: int = 32,
                     k=None, v=None, stream=None):
    """Slots start[b] .. start[b] + N - 1 (start None: from 0) as the values they stand for -> (k, v) [B,Hkv,N,D]; zeros from
    count[b] on and where no token is."""
    if dtype in _HALVES:
        r = _fast().cache4_load(cache, pages, start, N, D, count, k_mean, dtype == torch.bfloat16, page, group, k, v, _handle(stream))
        if r is not None:
            return _answer(r, "sage_cache4_load")
    _tensor(cache, "cache", (torch.uint8,), 3)
    if _elsewhere(cache.device, stream):
        return _there(cache.device, stream, sage_cache4_load, cache, pages, start, N, D, count, k_mean, dtype, page, group, k, v)
    dev, Hkv = cache.device, cache.shape[1]
    _tensor(pages, "pages", (torch.int32,), 2, dev)
    B = pages.shape[0]
    if dtype not in _HALVES:
        raise TypeError("dtype: torch.float16 or torch.bfloat16")
    pc, P, pt, columns = _cache(cache, pages, B, Hkv, D, page, group, dev)
    if k is None:
        k = torch.empty((B, Hkv, N, D), dtype=dtype, device=dev)
    if v is None:
        v = torch.empty((B, Hkv, N, D), dtype=dtype, device=dev)
    _check(load().sage_cache4_load(pc, pt, _maybe(start, "start", torch.int32, (B,), dev), _maybe(count, "count", torch.int32, (B,), dev),
                                   _maybe(k_mean, "k_mean", torch.float32, (B, Hkv, D), dev), _flat(k, "k", dtype, (B, Hkv, N, D), dev),
                                   _flat(v, "v", dtype, (B, Hkv, N, D), dev), B, Hkv, N, D, _TYPES[dtype], P, columns, page, group,
                                   binding._stream(None)), "sage_cache4_load")
    return k, v


def sage_cache4_attn_workspace(B: int, Hq: int, Hkv: int, Nq: int, D: int, columns: int, page: int = 64, n_splits: int = 0) -> int:
    return int(load().sage_cache4_attn_workspace(B, Hq, Hkv, Nq, D, columns, page, n_splits))


def _scale(sm_scale, D):
    return binding.sage_default_sm_scale(D) if sm_scale is None else float(sm_scale)


def sage_cache4_attn(q, cache, pages, lengths, count=None, causal: bool = True, sm_scale: float | None = None, page: int = 64,
                     group: int = 32, n_splits: int = 0, return_lse: bool = False, out=None, lse=None, workspace=None, stream=None):
    """Attention of the queries q [B,Hq,Nq,D] over the first lengths[b] tokens of the cache -> out [B,Hq,Nq,D], or (out, lse).
    Query head hq reads key head hq / (Hq / Hkv).  A sequence has its first count[b] queries (None: all; the rows behind them
    become zeros), query t being token lengths[b] - count[b] + t, which with the causal mask sees the tokens up to itself.
    workspace: uint8 tensor of at least sage_cache4_attn_workspace(...) bytes (allocated here if not given)."""
    r = _fast().cache4_attn(q, cache, pages, lengths, count, causal, sm_scale, page, group, n_splits, return_lse, out, lse, workspace,
                            _handle(stream))
    if r is not None:
        return _answer(r, "sage_cache4_attn")
    _tensor(q, "q", _HALVES, 4)
    if _elsewhere(q.device, stream):
        return _there(q.device, stream, sage_cache4_attn, q, cache, pages, lengths, count, causal, sm_scale, page, group, n_splits,
                      return_lse, out, lse, workspace)
    B, Hq, Nq, D = q.shape
    dev = q.device
    _tensor(cache, "cache", (torch.uint8,), 3, dev)
    Hkv = cache.shape[1]
    pq, sq = _rows(q, "q")
    pc, P, pt, columns = _cache(cache, pages, B, Hkv, D, page, group, dev)
    out = _like(q, out, "out")
    po, so = _rows(out, "out")
    if lse is None and return_lse:
        lse = torch.empty((B, Hq, Nq), dtype=torch.float32, device=dev)
    if workspace is None:
        need = sage_cache4_attn_workspace(B, Hq, Hkv, Nq, D, columns, page, n_splits)
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    pw, nw = (0, 0) if workspace is None else (_flat(workspace, "workspace", torch.uint8, workspace.shape, dev), workspace.numel())
    _check(load().sage_cache4_attn(pq, sq, pc, pt, _flat(lengths, "lengths", torch.int32, (B,), dev),
                                   _maybe(count, "count", torch.int32, (B,), dev), po, so, _maybe(lse, "lse", torch.float32, (B, Hq, Nq), dev),
                                   pw, nw, B, Hq, Hkv, Nq, D, _TYPES[q.dtype], P, columns, page, group, int(bool(causal)),
                                   _scale(sm_scale, D), int(n_splits), binding._stream(None)), "sage_cache4_attn")
    return (out, lse) if lse is not None else out


def sage_cache4_weights(q, cache, pages, lengths, lse, weights=None, count=None, causal: bool = True, sm_scale: float | None = None,
                        page: int = 64, group: int = 32, out=None, stream=None):
    """What the queries of sage_cache4_attn() gave to each slot, summed over the queries and the query heads of each key head and
    added to `weights` [B,Hkv,W] fp32 (None: zeros), W at least the tokens that the table has room for -> out, which may be
    `weights` itself.  lse is that call's."""
    r = _fast().cache4_weights(q, cache, pages, lengths, lse, weights, count, causal, sm_scale, page, group, out, _handle(stream))
    if r is not None:
        return _answer(r, "sage_cache4_weights")
    _tensor(q, "q", _HALVES, 4)
    if _elsewhere(q.device, stream):
        return _there(q.device, stream, sage_cache4_weights, q, cache, pages, lengths, lse, weights, count, causal, sm_scale, page, group, out)
    B, Hq, Nq, D = q.shape
    dev = q.device
    _tensor(cache, "cache", (torch.uint8,), 3, dev)
    Hkv = cache.shape[1]
    pq, sq = _rows(q, "q")
    pc, P, pt, columns = _cache(cache, pages, B, Hkv, D, page, group, dev)
    like = weights if weights is not None else out
    width = columns * page if like is None else _tensor(like, "weights", (torch.float32,), 3, dev).shape[2]
    if out is None:
        out = torch.empty((B, Hkv, width), dtype=torch.float32, device=dev)
    _check(load().sage_cache4_weights(pq, sq, pc, pt, _flat(lengths, "lengths", torch.int32, (B,), dev),
                                      _maybe(count, "count", torch.int32, (B,), dev), _flat(lse, "lse", torch.float32, (B, Hq, Nq), dev),
                                      _maybe(weights, "weights", torch.float32, (B, Hkv, width), dev),
                                      _flat(out, "out", torch.float32, (B, Hkv, width), dev), width, B, Hq, Hkv, Nq, D, _TYPES[q.dtype],
                                      P, columns, page, group, int(bool(causal)), _scale(sm_scale, D), binding._stream(None)), "sage_cache4_weights")
    return out


def sage_cache4_evict(cache, pages, lengths, weights, out_pages, keep: int, recent: int, D: int, page: int = 64, group: int = 32,
                      out_cache=None, out_weights=None, kept=None, out_lengths=None, stream=None):
    """Every sequence cut to `keep` tokens: each head keeps the last `recent` and, of those before, the ones with the largest
    weights (ties: the lowest slots); their rows are copied in order into the pages that out_pages [B,columns'] names (of
    out_cache; None: of cache itself), none of which may be one that `pages` names.
    -> (kept [B,Hkv,keep] int32, the slots, then -1; out_lengths [B] int32; out_weights [B,Hkv,W'] fp32, zeros behind)"""
    r = _fast().cache4_evict(cache, pages, lengths, weights, cache if out_cache is None else out_cache, out_pages, keep, recent, D, page, group,
                             out_weights, kept, out_lengths, _handle(stream))
    if r is not None:
        return _answer(r, "sage_cache4_evict")
    _tensor(cache, "cache", (torch.uint8,), 3)
    if _elsewhere(cache.device, stream):
        return _there(cache.device, stream, sage_cache4_evict, cache, pages, lengths, weights, out_pages, keep, recent, D, page, group,
                      out_cache, out_weights, kept, out_lengths)
    dev, Hkv = cache.device, cache.shape[1]
    _tensor(pages, "pages", (torch.int32,), 2, dev)
    B = pages.shape[0]
    pc, P, pt, columns = _cache(cache, pages, B, Hkv, D, page, group, dev)
    po, Po, pto, out_columns = _cache(cache if out_cache is None else out_cache, out_pages, B, Hkv, D, page, group, dev, "out_cache", "out_pages")
    _tensor(weights, "weights", (torch.float32,), 3, dev)
    width = weights.shape[2]
    if keep < 1:
        raise SageError(2, "sage_cache4_evict: keep")
    if out_weights is None:
        out_weights = torch.empty((B, Hkv, out_columns * page), dtype=torch.float32, device=dev)
    _tensor(out_weights, "out_weights", (torch.float32,), 3, dev)
    out_width = out_weights.shape[2]
    if kept is None:
        kept = torch.empty((B, Hkv, keep), dtype=torch.int32, device=dev)
    if out_lengths is None:
        out_lengths = torch.empty((B,), dtype=torch.int32, device=dev)
    _check(load().sage_cache4_evict(pc, P, pt, columns, _flat(lengths, "lengths", torch.int32, (B,), dev),
                                    _flat(weights, "weights", torch.float32, (B, Hkv, width), dev), width, po, Po, pto, out_columns,
                                    _flat(out_weights, "out_weights", torch.float32, (B, Hkv, out_width), dev), out_width,
                                    _flat(kept, "kept", torch.int32, (B, Hkv, keep), dev), _flat(out_lengths, "out_lengths", torch.int32, (B,), dev),
                                    B, Hkv, D, page, group, int(keep), int(recent), binding._stream(None)), "sage_cache4_evict")
    return kept, out_lengths, out_weights
