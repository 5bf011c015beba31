"""The serving calls on the host: every refusal before any launch (nothing here runs on a GPU), the sizes they report."""
import ctypes
import math

import numpy as np
import pytest

GOOD, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1002)       # never dereferenced: validation fails first
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    from paper_2410_02367_amd import binding
    return binding.load()


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def test_block_bytes(lib):
    assert lib.sage_cache4_block_bytes(128, 64, 32) == 64 * (64 + 64 + 8 + 8)
    assert lib.sage_cache4_block_bytes(64, 16, 64) == 16 * (32 + 32 + 2 + 2)
    for form in ((96, 64, 32), (128, 48, 32), (128, 8, 32), (128, 512, 32), (64, 64, 128), (128, 64, 16), (0, 0, 0), (-64, -64, -32)):
        assert lib.sage_cache4_block_bytes(*form) == 0


@pytest.mark.parametrize("name", ["sage_rope", "sage_rope_bwd"])
def test_rope_refusals(lib, name):
    def call(q=GOOD, qs=None, qo=GOOD, qos=None, k=None, ks=None, ko=None, kos=None, pos=GOOD, ps=0, freq=GOOD, amp=1.0, B=1, Hq=2, Hk=0, N=4,
             D=64, R=64, type=0, inter=0):
        return getattr(lib, name)(q, qs, qo, qos, k, ks, ko, kos, pos, ps, freq, F(amp), B, Hq, Hk, N, D, R, type, inter, None)
    assert call(q=None) == 1 and call(qo=None) == 1 and call(pos=None) == 1 and call(freq=None) == 1 and call(Hk=1) == 1 and call(Hk=1, k=GOOD) == 1
    assert call(B=0) == 2 and call(Hq=0) == 2 and call(N=0) == 2 and call(Hk=-1) == 2 and call(N=(1 << 23) + 1) == 2 and call(ps=-1) == 2
    assert call(B=256, Hq=256) == 2 and call(B=65535, Hq=1, Hk=1, k=GOOD, ko=GOOD) == 2 and call(D=0, R=0) == 2
    for bad in (dict(D=60), dict(D=520), dict(R=0), dict(R=63), dict(R=66), dict(type=3), dict(type=-1)):
        assert call(**bad) == 3
    assert call(amp=math.inf) == 7 and call(amp=math.nan) == 7
    assert call(q=ODD) == 5 and call(qo=ODD) == 5 and call(pos=ODD) == 5 and call(freq=ctypes.c_void_p(0x1004)) == 5
    assert call(Hk=1, k=ODD, ko=GOOD) == 5 and call(Hk=1, k=GOOD, ko=ODD) == 5
    assert call(qs=strides(512, 256, 60)) == 5 and call(qs=strides(512, 250, 64)) == 5
    # outputs that are each other's memory
    assert call(qos=strides(512, 0, 64)) == 5 and call(qos=strides(512, 256, 0)) == 5


def test_append_and_load_refusals(lib):
    def append(k=GOOD, ks=None, v=GOOD, vs=None, mean=None, cache=GOOD, pages=GOOD, start=GOOD, count=None, B=1, H=1, N=4, D=64, type=0, P=4,
               columns=2, page=16, group=32):
        return lib.sage_cache4_append(k, ks, v, vs, mean, cache, pages, start, count, B, H, N, D, type, P, columns, page, group, None)

    def load(cache=GOOD, pages=GOOD, start=None, count=None, mean=None, k=GOOD, v=GOOD, B=1, H=1, N=4, D=64, type=0, P=4, columns=2, page=16, group=32):
        return lib.sage_cache4_load(cache, pages, start, count, mean, k, v, B, H, N, D, type, P, columns, page, group, None)
    for call in (append, load):
        for name in ("k", "v", "cache", "pages"):
            assert call(**{name: None}) == 1
            assert call(**{name: ODD}) == 5
        assert call(count=ctypes.c_void_p(0x1001)) == 5 and call(start=ctypes.c_void_p(0x1001)) == 5 and call(mean=ctypes.c_void_p(0x1004)) == 5
        for bad in (dict(B=0), dict(H=0), dict(N=0), dict(P=0), dict(columns=0), dict(B=300, H=300), dict(columns=(1 << 23) // 16 + 1), dict(N=(1 << 23) + 1)):
            assert call(**bad) == 2, bad
        for bad in (dict(D=96), dict(page=8), dict(page=24), dict(group=16), dict(group=128), dict(type=2), dict(type=9)):
            assert call(**bad) == 3, bad
    assert append(start=None) == 1 and append(ks=strides(256, 256, 4)) == 5 and append(vs=strides(256, 256, 65)) == 5


def test_attention_and_weights_refusals(lib):
    def attn(q=GOOD, qs=None, cache=GOOD, pages=GOOD, lengths=GOOD, count=None, out=GOOD, os=None, lse=None, ws=GOOD, wb=1 << 40, B=1, Hq=4, Hkv=2, Nq=1,
             D=64, type=0, P=4, columns=2, page=16, group=32, causal=1, scale=0.125, splits=0):
        return lib.sage_cache4_attn(q, qs, cache, pages, lengths, count, out, os, lse, ws, wb, B, Hq, Hkv, Nq, D, type, P, columns, page, group,
                                    causal, F(scale), splits, None)

    def weights(q=GOOD, qs=None, cache=GOOD, pages=GOOD, lengths=GOOD, count=None, lse=GOOD, w=None, out=GOOD, width=32, B=1, Hq=4, Hkv=2, Nq=1, D=64,
                type=0, P=4, columns=2, page=16, group=32, causal=1, scale=0.125):
        return lib.sage_cache4_weights(q, qs, cache, pages, lengths, count, lse, w, out, width, B, Hq, Hkv, Nq, D, type, P, columns, page, group, causal,
                                       F(scale), None)
    for call in (attn, weights):
        for name in ("q", "cache", "pages", "lengths", "out"):
            assert call(**{name: None}) == 1, name
            assert call(**{name: ctypes.c_void_p(0x1001)}) == 5, name
        assert call(count=ctypes.c_void_p(0x1001)) == 5 and call(lse=ctypes.c_void_p(0x1001)) == 5 and call(qs=strides(256, 64, 4), Nq=2) == 5
        for bad in (dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Nq=0), dict(P=0), dict(columns=0), dict(B=30000, Hq=4), dict(columns=1 << 22, width=1 << 23)):
            bad.pop("width", None) if call is attn else None
            assert call(**bad) == 2, bad
        for bad in (dict(Hq=3), dict(D=32), dict(page=20), dict(group=96), dict(type=2)):
            assert call(**bad) == 3, bad
        for scale in (0.0, -1.0, math.inf, math.nan):
            assert call(scale=scale) == 7
    assert attn(splits=-1) == 7 and attn(Nq=2, os=strides(512, 0, 64)) == 5
    assert weights(lse=None) == 1 and weights(width=31) == 2 and weights(width=(1 << 23) + 1) == 2 and weights(w=ctypes.c_void_p(0x1001)) == 5
    need = lib.sage_cache4_attn_workspace(1, 4, 2, 1, 64, 512, 16, 4)
    if need:
        assert attn(columns=512, splits=4, wb=need - 1) == 4 and attn(columns=512, splits=4, ws=None) == 1 and attn(columns=512, splits=4, ws=ODD) == 5
    for bad in ((0, 4, 2, 1, 64, 2, 16, 0), (1, 3, 2, 1, 64, 2, 16, 0), (1, 4, 2, 0, 64, 2, 16, 0), (1, 4, 2, 1, 96, 2, 16, 0), (1, 4, 2, 1, 64, 0, 16, 0),
                (1, 4, 2, 1, 64, 2, 17, 0), (1, 4, 2, 1, 64, 2, 16, -1)):
        assert lib.sage_cache4_attn_workspace(*bad) == 0


def test_workgroups_beyond_what_the_kernels_count(lib):
    args = dict(B=64, Hq=1 << 10, Hkv=1, Nq=1 << 15)
    def attn(splits, columns):
        return lib.sage_cache4_attn(GOOD, None, GOOD, GOOD, GOOD, None, GOOD, None, None, GOOD, 1 << 62, args["B"], args["Hq"], args["Hkv"], args["Nq"], 64,
                                    0, 1 << 20, columns, 256, 32, 1, F(0.125), splits, None)
    assert args["B"] * args["Hq"] * args["Nq"] == 1 << 31 and attn(1, 1) == 2                # rows
    args["B"] = 32
    assert attn(1 << 15, 1 << 15) == 2                                                       # 2^26 and more tiles of rows times 2^15 chunks
    assert lib.sage_cache4_attn_workspace(64, 1 << 10, 1, 1 << 15, 64, 1, 256, 0) == 0


def test_workspace_holds_the_partial_results(lib):
    # [chunks][rows] of D fp32 numbers and a logarithm; none for one chunk
    assert lib.sage_cache4_attn_workspace(2, 8, 2, 1, 128, 64, 64, 1) == 0 and lib.sage_cache4_attn_workspace(2, 8, 2, 1, 128, 4, 64, 9) == 0
    assert lib.sage_cache4_attn_workspace(2, 8, 2, 1, 128, 64, 64, 4) == 4 * 2 * 8 * 129 * 4
    assert lib.sage_cache4_attn_workspace(1, 8, 2, 3, 64, 256, 16, 3) == 3 * 8 * 3 * 65 * 4
    for splits in range(0, 40):
        for columns, page in ((64, 64), (100, 16), (7, 256)):
            n = lib.sage_cache4_attn_workspace(1, 4, 4, 1, 64, columns, page, splits) / (4 * 65 * 4)
            assert n == int(n) and (n == 0 or 2 <= n <= max(2, columns * page // 256))


SYMBOLIC = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.fx.experimental.symbolic_shapes import ShapeEnv
from paper_2410_02367_amd import binding
binding.load()
native, env = binding._native, ShapeEnv()
with FakeTensorMode(shape_env=env):
    x = torch.empty(1, 2, env.create_unbacked_symint(), 64, dtype=torch.float16, device="cuda")
    i, f, u = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.float64, device="cuda"), torch.empty(4, 2, 1152, dtype=torch.uint8, device="cuda")
    p = torch.empty(1, env.create_unbacked_symint(), dtype=torch.int32, device="cuda")
    assert native.rope(x, None, i, f, 0, 1.0, None, None, 0) is None and native.rope_bwd(x, x, i, f, 0, 1.0, None, None, 0) is None
    assert native.cache4_append(x, x, u, p, i, None, None, 16, 32, 0) is None
    assert native.cache4_load(u, p, None, 4, 64, None, None, 0, 16, 32, None, None, 0) is None
    assert native.cache4_attn(x, u, p, i, None, 1, None, 16, 32, 0, 0, None, None, None, 0) is None
    assert native.cache4_weights(x, u, p, i, x, None, None, 1, None, 16, 32, None, 0) is None
    assert native.cache4_evict(u, p, i, x, u, p, 4, 0, 64, 16, 32, None, None, None, 0) is None
print("all left to Python")
"""


def test_tensors_without_sizes_in_numbers_are_left_to_python(lib):
    """In a process of its own, which is what an exception that passes through the interpreter would end."""
    import os
    import subprocess
    import sys
    run = subprocess.run([sys.executable, "-c", SYMBOLIC], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True,
                         timeout=300)
    assert run.returncode == 0 and "all left to Python" in run.stdout, (run.returncode, run.stderr[-500:])


def test_the_extension_module_takes_no_arguments_that_are_not_in_order(lib):
    import torch
    from paper_2410_02367_amd import binding
    n = binding._native
    x = torch.zeros(1, 2, 4, 64, dtype=torch.float16)
    for bad in ([], [x], [None] * 9, [x] * 9, [1] * 13, ["q"] * 15, [None] * 10, [x] * 13, [x] * 15, [object()] * 15, [x] * 10):
        for f in (n.rope, n.rope_bwd, n.cache4_append, n.cache4_load, n.cache4_attn, n.cache4_weights, n.cache4_evict):
            assert f(*bad) is None


def test_evict_refusals(lib):
    other, third = ctypes.c_void_p(0x2000), ctypes.c_void_p(0x3000)

    def call(cache=GOOD, P=8, pages=GOOD, columns=4, lengths=GOOD, w=GOOD, width=64, oc=GOOD, oP=8, op=other, ocols=2, ow=other, owidth=32, kept=GOOD,
             ol=other, B=1, H=1, D=64, page=16, group=32, keep=20, recent=4):
        return lib.sage_cache4_evict(cache, P, pages, columns, lengths, w, width, oc, oP, op, ocols, ow, owidth, kept, ol, B, H, D, page, group, keep,
                                     recent, None)
    for name in ("cache", "pages", "lengths", "w", "oc", "op", "ow", "kept", "ol"):
        assert call(**{name: None}) == 1, name
        assert call(**{name: ctypes.c_void_p(0x5001)}) == 5, name
    for bad in (dict(keep=0), dict(keep=33, owidth=64), dict(width=63), dict(owidth=19), dict(B=0), dict(P=0), dict(oP=0), dict(ocols=0)):
        assert call(**bad) == 2, bad
    assert call(recent=-1) == 7 and call(recent=21) == 7
    assert call(op=GOOD) == 7 and call(ow=GOOD) == 7 and call(ol=GOOD) == 7
    for bad in (dict(D=80), dict(page=10), dict(group=8)):
        assert call(**bad) == 3, bad


def test_wrappers_refuse_what_is_not_in_device_memory():
    import torch
    import paper_2410_02367_amd as sage
    x = torch.zeros(1, 2, 4, 64, dtype=torch.float16)
    i = torch.zeros(4, dtype=torch.int32)
    cache, pages = torch.zeros(4, 2, 16 * 72, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: sage.sage_rope(x, None, i, torch.ones(32, dtype=torch.float64)), lambda: sage.sage_rope_bwd(x, x, i, i),
                 lambda: sage.sage_cache4_append(x, x, cache, pages, i[:1], page=16), lambda: sage.sage_cache4_load(cache, pages, None, 4, 64, page=16),
                 lambda: sage.sage_cache4_attn(x, cache, pages, i[:1], page=16), lambda: sage.sage_cache4_weights(x, cache, pages, i[:1], x, page=16),
                 lambda: sage.sage_cache4_evict(cache, pages, i[:1], x, pages, 4, 0, 64, page=16), lambda: sage.sage_cache4_attn(None, cache, pages, i)):
        with pytest.raises(TypeError):
            call()


def test_scaled_frequencies():
    import paper_2410_02367_amd as sage
    plain = 10000.0 ** (-np.arange(32) / 32)
    f, a = sage.sage_rope_frequencies(64)
    assert a == 1.0 and np.allclose(f.numpy(), plain) and str(f.dtype) == "torch.float64"
    assert np.allclose(sage.sage_rope_frequencies(64, scaling="linear", factor=8)[0].numpy(), plain / 8)
    # the base raised: fastest as it was, slowest divided by the factor
    f = sage.sage_rope_frequencies(64, scaling="base", factor=8)[0].numpy()
    assert np.isclose(f[0], 1.0) and np.isclose(f[-1], plain[-1] / 8) and np.all((f <= plain * (1 + 1e-12)) & (f >= plain / 8 * (1 - 1e-12)))
    turns = 8192 * plain / (2 * np.pi)
    f, a = sage.sage_rope_frequencies(64, scaling="parts", factor=8)
    f = f.numpy()
    assert a == 1.0 and np.allclose(f[turns > 4], plain[turns > 4]) and np.allclose(f[turns < 1], plain[turns < 1] / 8)
    some = (turns > 1) & (turns < 4)
    mix = (turns[some] - 1) / 3
    assert some.any() and np.allclose(f[some], plain[some] * mix + plain[some] / 8 * (1 - mix))
    f, a = sage.sage_rope_frequencies(64, scaling="ramp", factor=8, low=1.0, high=32.0)
    f = f.numpy()
    assert np.isclose(a, 0.1 * math.log(8) + 1) and np.allclose(f[turns > 40], plain[turns > 40]) and np.allclose(f[turns < 0.8], plain[turns < 0.8] / 8)
    assert np.all(np.diff(f) < 0)
    for bad in (dict(rotated=3), dict(rotated=0), dict(rotated=64, scaling="other"), dict(rotated=64, factor=0.5), dict(rotated=64, base=-1.0),
                dict(rotated=64, low=4.0, high=1.0)):
        with pytest.raises(ValueError):
            sage.sage_rope_frequencies(**bad)


def test_launches_beyond_what_32_bits_count(lib):
    """A launch of 2^32 threads and more is refused before anything runs."""
    def attn(B, Hq, Nq, splits, columns):
        return lib.sage_cache4_attn(GOOD, None, GOOD, GOOD, GOOD, None, GOOD, None, None, GOOD, 1 << 62, B, Hq, 1, Nq, 64, 0, 1 << 20, columns, 256, 32, 1,
                                    F(0.125), splits, None)
    assert attn(1 << 14, 1, 1, 1 << 10, 1 << 10) == 2                   # 2^24 chunks of one row each
    assert attn(1 << 4, 1 << 10, 1 << 14, 2, 2) == 2                    # 2^28 rows of two chunks: the merge's threads
    for name in ("sage_rope", "sage_rope_bwd"):
        for rotated in (64, 2):
            assert getattr(lib, name)(GOOD, None, GOOD, None, None, None, None, None, GOOD, 0, GOOD, F(1.0), 16, 1, 0, 1 << 23, 64, rotated, 0, 0, None) == 2


def test_frequencies_that_are_refused():
    import paper_2410_02367_amd as sage
    for bad in (dict(rotated=7), dict(rotated=0), dict(base=0.0), dict(factor=0.5), dict(original_length=0), dict(low=2.0, high=1.0),
                dict(scaling="other"), dict(scaling="ramp", base=1.0)):
        with pytest.raises(ValueError):
            sage.sage_rope_frequencies(**{"rotated": 64, **bad})
