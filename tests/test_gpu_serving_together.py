"""The serving calls as a program runs them together: a prompt in chunks, single tokens, eviction, more tokens -- eagerly, on
another stream and from a captured graph."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, attention_bounds, dev, host

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, PAGE, GROUP, COLUMNS = 2, 4, 2, 64, 16, 32, 12


class Program:
    def __init__(self, seed):
        import paper_2410_02367_amd as sage
        self.sage, self.g = sage, np.random.default_rng(seed)
        self.cache = torch.full((2 * B * COLUMNS, HKV, sage.sage_cache4_block_bytes(D, PAGE, GROUP)), 0xff, dtype=torch.uint8, device="cuda")
        self.tables = [dev(t) for t in self.g.permutation(2 * B * COLUMNS).astype(np.int32).reshape(2, B, COLUMNS)]
        self.lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.weights = torch.zeros(B, HKV, COLUMNS * PAGE, device="cuda")
        self.freq, self.amplitude = sage.sage_rope_frequencies(D, scaling="parts", factor=4.0, device="cuda")
        self.mean = dev((3 * self.g.standard_normal((B, HKV, D))).astype(np.float32))
        self.seen = torch.zeros(B, dtype=torch.int32, device="cuda")              # positions go on counting through evictions

    def inputs(self, n):
        qkv = dev(self.g.standard_normal((B, n, HQ + 2 * HKV, D)), torch.float16)
        qkv[:, :, HQ:HQ + HKV] += self.mean[:, None].half()
        return qkv

    def step(self, qkv, count):
        s, n = self.sage, qkv.shape[1]
        q, k, v = (x.transpose(1, 2) for x in qkv.split([HQ, HKV, HKV], 2))
        q, k = s.sage_rope(q, k, self.seen[:, None] + torch.arange(n, device="cuda", dtype=torch.int32), self.freq, amplitude=self.amplitude)
        s.sage_cache4_append(k, v, self.cache, self.tables[0], self.lengths, count, self.mean, PAGE, GROUP)
        self.lengths += count
        self.seen += count
        out, lse = s.sage_cache4_attn(q, self.cache, self.tables[0], self.lengths, count, page=PAGE, group=GROUP, return_lse=True)
        s.sage_cache4_weights(q, self.cache, self.tables[0], self.lengths, lse, self.weights, count, page=PAGE, group=GROUP, out=self.weights)
        return q, out

    def evict(self, keep, recent):
        kept, self.lengths, self.weights = self.sage.sage_cache4_evict(self.cache, self.tables[0], self.lengths, self.weights, self.tables[1], keep,
                                                                       recent, D, PAGE, GROUP)
        self.tables.reverse()
        return kept

    def check(self, q, out, count):
        c = so.Cache(self.cache.shape[0], HKV, D, PAGE, GROUP, self.cache.cpu().numpy())
        lengths, count = self.lengths.tolist(), count.tolist()
        k, v, there = c.load(self.tables[0].cpu().numpy(), None, COLUMNS * PAGE, lengths)
        want, lse, w = so.attention(host(q), k, v, there, lengths, count)
        do, _ = attention_bounds(host(q), k, v, there, lengths, count, True, 1 / np.sqrt(D), lse)
        assert np.all(np.abs(host(out) - want) <= do + HALF_STEP["f16"] * np.abs(want) + 2.0 ** -25)
        return w


def counts(*n):
    return dev(np.int32(n))


def test_a_run():
    p = Program(1)
    total = np.zeros((B, HKV, COLUMNS * PAGE))
    for n, count in ((37, (37, 20)), (5, (5, 5)), (1, (1, 1)), (1, (1, 0)), (60, (44, 60)), (1, (1, 1))):
        count = counts(*count)
        q, out = p.step(p.inputs(n), count)
        total += p.check(q, out, count)
    assert np.allclose(host(p.weights), total, rtol=1e-4, atol=1e-6) and np.isclose(total.sum(), HQ * (37 + 20 + 10 + 3 + 104 + 2))
    before, had = p.lengths.clone(), host(p.weights)
    kept = p.evict(48, 10).cpu().numpy()
    assert p.lengths.tolist() == [48, 48]
    want, _ = so.evict(had.astype(np.float32), before.tolist(), COLUMNS * PAGE, 48, 10)
    assert np.array_equal(kept, want)
    for n, count in ((1, (1, 1)), (9, (9, 2))):
        count = counts(*count)
        p.check(*p.step(p.inputs(n), count), count)


def test_decoding_from_a_captured_graph():
    """A step captured once and replayed, with eager steps of the same program on other memory between the replays."""
    runs = [Program(2), Program(2), Program(3)]
    prompt = runs[0].inputs(50)
    runs[1].inputs(50)
    for p in runs:
        p.step(prompt, counts(50, 31))
    one = counts(1, 1)
    token = torch.zeros_like(runs[0].inputs(1))
    runs[1].inputs(1)
    tokens = [runs[0].inputs(1) for _ in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    warm = Program(4)
    with torch.cuda.stream(side):
        warm.step(token, one)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, out = runs[0].step(token, one)
    for t in tokens:
        token.copy_(t)
        graph.replay()
        _, eager = runs[1].step(t, one)
        runs[2].step(t, one)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert torch.equal(runs[0].cache, runs[1].cache) and torch.equal(runs[0].weights, runs[1].weights)
        runs[0].check(q, out, one)


def test_on_a_stream_that_is_not_the_current_one():
    import paper_2410_02367_amd as sage
    p = Program(5)
    q, _ = p.step(p.inputs(90), counts(90, 70))
    args = (q, p.cache, p.tables[0], p.lengths)
    want, lse = sage.sage_cache4_attn(*args, page=PAGE, group=GROUP, return_lse=True)
    w = sage.sage_cache4_weights(*args, lse, page=PAGE, group=GROUP)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        out, l2 = sage.sage_cache4_attn(*args, page=PAGE, group=GROUP, return_lse=True, n_splits=3, stream=stream)
        w2 = sage.sage_cache4_weights(*args, lse, page=PAGE, group=GROUP, stream=stream)
        out2 = sage.sage_cache4_attn(*args, page=PAGE, group=GROUP, stream=stream)
        k, v = sage.sage_cache4_load(p.cache, p.tables[0], None, 90, D, p.lengths, page=PAGE, group=GROUP, stream=stream)
        r = sage.sage_rope(q, None, counts(*range(90)), p.freq, stream=stream)
        side.synchronize()
        assert torch.equal(out2, want) and torch.equal(w2, w) and torch.isfinite(k).all() and torch.isfinite(out).all()
        assert torch.equal(r, sage.sage_rope(q, None, counts(*range(90)), p.freq))
        kept = sage.sage_cache4_evict(p.cache, p.tables[0], p.lengths, w, p.tables[1], 33, 5, D, PAGE, GROUP, stream=stream)[0]
        side.synchronize()
        assert torch.equal(kept, sage.sage_cache4_evict(p.cache, p.tables[0], p.lengths, w, p.tables[1], 33, 5, D, PAGE, GROUP)[0])
