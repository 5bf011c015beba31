"""What the serving wrappers refuse with tensors on the device, their two ways into the library, streams, scratch and graphs."""
import numpy as np
import pytest
import torch

import paper_2410_02367_amd as sage
from paper_2410_02367_amd import binding
from serving_util import dev, make_cache

pytestmark = pytest.mark.gpu

B, HQ, HKV, N, D, PAGE, GROUP = 2, 4, 2, 5, 64, 16, 32


class Setup:
    def __init__(self, columns=6, lengths=(70, 33)):
        g = np.random.default_rng(1)
        c, table = make_cache(1, B, HKV, D, PAGE, GROUP, lengths, columns, spare=B * columns)
        self.cache, self.pages = dev(c.data), dev(table)
        self.out_pages = dev(np.setdiff1d(np.arange(c.num_pages, dtype=np.int32), table)[:B * columns].reshape(B, columns))
        self.lengths, self.count = dev(np.int32(lengths)), dev(np.int32([5, 3]))
        self.q = dev(g.standard_normal((B, HQ, N, D)), torch.float16)
        self.k, self.v = (dev(g.standard_normal((B, HKV, N, D)), torch.float16) for _ in range(2))
        self.mean = dev(g.standard_normal((B, HKV, D)).astype(np.float32))
        self.freq, self.positions = dev(1e4 ** (-np.arange(16) / 16)), dev(np.arange(B * N, dtype=np.int32).reshape(B, N))
        self.weights = torch.rand(B, HKV, columns * PAGE, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
        self.lse = sage.sage_cache4_attn(self.q, self.cache, self.pages, self.lengths, page=PAGE, return_lse=True)[1]

    def calls(self, **more):
        """each call with all it may be given"""
        s, form = self, dict(page=PAGE, group=GROUP, **more)
        scratch = self.cache.clone()
        return {
            "rope": lambda: sage.sage_rope(s.q, s.k, s.positions, s.freq, True, 1.5, **more),
            "rope_bwd": lambda: sage.sage_rope_bwd(s.q, None, s.positions[0].contiguous(), s.freq, **more),
            "append": lambda: sage.sage_cache4_append(s.k, s.v, scratch, s.pages, s.lengths, s.count, s.mean, **form),
            "load": lambda: sage.sage_cache4_load(s.cache, s.pages, s.count, 20, D, s.lengths, s.mean, torch.bfloat16, **form),
            "attn": lambda: sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, s.count, False, 0.2, return_lse=True, **form),
            "attn_default": lambda: sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, **form),
            "weights": lambda: sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, s.lse, s.weights, **form),
            "evict": lambda: sage.sage_cache4_evict(scratch, s.pages, s.lengths, s.weights, s.out_pages, 30, 4, D, **form),
        }


def flat(r):
    return [t.clone() for t in (r if isinstance(r, tuple) else (r,))]


def test_both_ways_into_the_library_give_the_same(monkeypatch):
    s = Setup()
    native = {name: flat(call()) for name, call in s.calls().items()}
    taken = []

    class Counting:
        def __getattr__(self, name):
            f = getattr(real, name)

            def g(*args):
                r = f(*args)
                taken.append(r is not None)
                return r
            return g
    real = binding._native
    monkeypatch.setattr(binding, "_native", Counting())
    for call in s.calls().values():
        call()
    assert taken and all(taken)               # what is in order is the extension module's
    monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    for name, call in s.calls().items():
        got = flat(call())
        assert len(got) == len(native[name])
        for x, y in zip(got, native[name]):
            assert x.dtype == y.dtype and x.shape == y.shape and x.stride() == y.stride()
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name


def test_given_outputs_are_the_results():
    s = Setup()
    out, lse, ws = torch.empty_like(s.q), torch.empty_like(s.lse), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    r = sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, page=PAGE, out=out, lse=lse, workspace=ws)
    assert r[0] is out and r[1] is lse and torch.equal(lse, s.lse)
    kept, n, w = (torch.empty(sh, dtype=t, device="cuda") for sh, t in (((B, HKV, 9), torch.int32), ((B,), torch.int32), ((B, HKV, 11), torch.float32)))
    r = sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages, 9, 2, D, PAGE, out_weights=w, kept=kept, out_lengths=n)
    assert r[0] is kept and r[1] is n and r[2] is w and not w[..., 9:].any()
    k, v = torch.empty(B, HKV, 3, D, dtype=torch.float16, device="cuda"), torch.empty(B, HKV, 3, D, dtype=torch.float16, device="cuda")
    r = sage.sage_cache4_load(s.cache, s.pages, None, 3, D, page=PAGE, k=k, v=v)
    assert r[0] is k and r[1] is v


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    s = Setup()
    if not native:
        monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    f32, i64 = s.q.float(), s.lengths.long()
    attn, form = sage.sage_cache4_attn, dict(page=PAGE)
    wrong = [
        (TypeError, lambda: attn(f32, s.cache, s.pages, s.lengths, **form)),
        (TypeError, lambda: attn(s.q, s.cache.int(), s.pages, s.lengths, **form)),
        (TypeError, lambda: attn(s.q, s.cache, s.pages.long(), s.lengths, **form)),
        (TypeError, lambda: attn(s.q, s.cache, s.pages, i64, **form)),
        (TypeError, lambda: attn(s.q, s.cache, s.pages, s.lengths.cpu(), **form)),
        (TypeError, lambda: attn(s.q[0], s.cache, s.pages, s.lengths, **form)),
        (TypeError, lambda: attn(s.q, s.cache, s.pages[0], s.lengths, **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages[:1], s.lengths, **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages, s.lengths[:1], **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages, s.lengths, page=32)),                       # the bytes of another form
        (ValueError, lambda: attn(s.q, s.cache, s.pages, s.lengths, page=PAGE, group=64)),
        (ValueError, lambda: attn(s.q, s.cache[:, :, ::2], s.pages, s.lengths, **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages.t().contiguous().t(), s.lengths, **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages, s.lengths, out=s.q[:, :, :3], **form)),
        (TypeError, lambda: attn(s.q, s.cache, s.pages, s.lengths, out=s.q.bfloat16(), **form)),
        (ValueError, lambda: attn(s.q, s.cache, s.pages, s.lengths, lse=s.lse[:, :1], **form)),
        (ValueError, lambda: attn(s.q.transpose(2, 3).contiguous().transpose(2, 3), s.cache, s.pages, s.lengths, **form)),
        (sage.SageError, lambda: attn(s.q, s.cache, s.pages, s.lengths, page=24)),
        (sage.SageError, lambda: attn(s.q[:, :3], s.cache, s.pages, s.lengths, **form)),               # 3 heads on 2
        (sage.SageError, lambda: attn(s.q, s.cache, s.pages, s.lengths, sm_scale=-1.0, **form)),
        (sage.SageError, lambda: attn(s.q, s.cache, s.pages, s.lengths, n_splits=-1, **form)),
        (sage.SageError, lambda: attn(s.q[:, :, :0], s.cache, s.pages, s.lengths, **form)),
        (TypeError, lambda: sage.sage_cache4_append(s.k, s.v.bfloat16(), s.cache, s.pages, s.lengths, **form)),
        (ValueError, lambda: sage.sage_cache4_append(s.k, s.v[:, :1], s.cache, s.pages, s.lengths, **form)),
        (ValueError, lambda: sage.sage_cache4_append(s.k[:, :1], s.v[:, :1], s.cache, s.pages, s.lengths, **form)),
        (ValueError, lambda: sage.sage_cache4_append(s.k, s.v, s.cache, s.pages, s.lengths, k_mean=s.mean[0:1], **form)),
        (TypeError, lambda: sage.sage_cache4_append(s.k, s.v, s.cache, s.pages, None, **form)),
        (TypeError, lambda: sage.sage_cache4_load(s.cache, s.pages, None, 4, D, dtype=torch.float32, **form)),
        (sage.SageError, lambda: sage.sage_cache4_load(s.cache, s.pages, None, 4, 96, **form)),
        (sage.SageError, lambda: sage.sage_cache4_load(s.cache, s.pages, None, 0, D, **form)),
        (ValueError, lambda: sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, s.lse[:, :, :2].contiguous(), **form)),
        (sage.SageError, lambda: sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, s.lse, s.weights[..., :40].contiguous(), **form)),
        (ValueError, lambda: sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, s.lse, s.weights, out=s.weights[..., :40].contiguous(), **form)),
        (sage.SageError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages, 0, 0, D, PAGE)),
        (sage.SageError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages, 5, 6, D, PAGE)),
        (sage.SageError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages, 1000, 6, D, PAGE)),
        (sage.SageError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.pages, 5, 1, D, PAGE)),
        (sage.SageError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages, 5, 1, D, PAGE, out_weights=s.weights)),
        (ValueError, lambda: sage.sage_cache4_evict(s.cache, s.pages, s.lengths, s.weights, s.out_pages[:1], 5, 1, D, PAGE)),
        (TypeError, lambda: sage.sage_rope(s.q, s.k, s.positions.long(), s.freq)),
        (TypeError, lambda: sage.sage_rope(s.q, s.k, s.positions, s.freq.float())),
        (TypeError, lambda: sage.sage_rope(s.q, s.k.bfloat16(), s.positions, s.freq)),
        (ValueError, lambda: sage.sage_rope(s.q, s.k[:, :, :2], s.positions, s.freq)),
        (ValueError, lambda: sage.sage_rope(s.q, s.k, s.positions[:, :2].contiguous(), s.freq)),
        (sage.SageError, lambda: sage.sage_rope(s.q, s.k, s.positions, torch.ones(40, dtype=torch.float64, device="cuda"))),
        (sage.SageError, lambda: sage.sage_rope(s.q[..., 4:], None, s.positions, s.freq)),             # rows that start between 16-byte boundaries
        (ValueError, lambda: sage.sage_rope(s.q, None, s.positions, s.freq, q_out=s.q[:, :, :1])),
    ]
    before = [t.clone() for t in (s.cache, s.weights)]
    for i, (error, call) in enumerate(wrong):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
    assert torch.equal(s.cache, before[0]) and torch.equal(s.weights, before[1])


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("what", ["rope", "load", "attn", "attn_split", "weights", "evict"])
def test_a_named_streams_memory_is_not_handed_out_while_it_runs(what, handle):
    """The named stream is kept busy, so the call's kernels run after later work of the current stream has taken and filled
    memory of the same sizes: scratch and outputs must not be among it."""
    s = Setup(columns=80, lengths=(1200, 700))

    def call(stream):
        if what == "attn_split":
            return sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, page=PAGE, n_splits=4, return_lse=True, stream=stream)
        return s.calls(stream=stream)[what]()
    expected = flat(call(None))
    side = torch.cuda.Stream()
    busy = torch.ones(1 << 26, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy.mul_(1.0)
    r = call(side.cuda_stream if handle else side)
    r = r if isinstance(r, tuple) else (r,)
    size = sage.sage_cache4_attn_workspace(B, HQ, HKV, N, D, 80, PAGE, 4)
    fill = [torch.full((max(n, 1),), 0x7f, dtype=torch.uint8, device="cuda") for n in [size] + [t.nbytes for t in r] for _ in range(3)]
    torch.cuda.synchronize()
    for got, want in zip(r, expected):
        assert torch.equal(got, want)
    del fill


def test_two_graphs_that_share_a_workspace():
    """Captured with one workspace and replayed in turn, with eager calls between them."""
    s, t = Setup(columns=100, lengths=(1500, 900)), Setup(columns=100, lengths=(1590, 33))
    ws = torch.empty(sage.sage_cache4_attn_workspace(B, HQ, HKV, N, D, 100, PAGE, 5), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0

    def attn(x):
        return sage.sage_cache4_attn(x.q, x.cache, x.pages, x.lengths, page=PAGE, n_splits=5, return_lse=True, workspace=ws)
    want = [flat(attn(x)) for x in (s, t)]
    graphs, outs = [], []
    for x in (s, t):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(attn(x))
        graphs.append(graph)
    for i in (0, 1, 0, 0, 1):
        for o in outs[i]:
            o.fill_(7.0)
        ws.fill_(0xff)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
        assert all(torch.equal(a, b) for a, b in zip(attn((s, t)[1 - i]), want[1 - i]))


def test_results_do_not_change_from_call_to_call():
    s = Setup(columns=300, lengths=(4700, 4000))
    for n_splits in (0, 1, 7):
        first = flat(sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, page=PAGE, n_splits=n_splits, return_lse=True))
        w = sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, first[1], page=PAGE)
        e = flat(sage.sage_cache4_evict(s.cache, s.pages, s.lengths, w, s.out_pages, 1000, 30, D, PAGE))
        for _ in range(3):
            again = sage.sage_cache4_attn(s.q, s.cache, s.pages, s.lengths, page=PAGE, n_splits=n_splits, return_lse=True)
            assert all(torch.equal(a, b) for a, b in zip(first, again))
            assert torch.equal(w, sage.sage_cache4_weights(s.q, s.cache, s.pages, s.lengths, first[1], page=PAGE))
            assert all(torch.equal(a, b) for a, b in zip(e, sage.sage_cache4_evict(s.cache, s.pages, s.lengths, w, s.out_pages, 1000, 30, D, PAGE)))
