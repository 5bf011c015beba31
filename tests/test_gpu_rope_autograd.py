"""Rotary positions within autograd: the gradients of q and k, against the formula and against differences."""
import numpy as np
import pytest
import torch

import oracle.serving as so
from serving_util import HALF_STEP, TINY, TORCH, dev, host, rounded

pytestmark = pytest.mark.gpu

FREQ = 10000.0 ** (-np.arange(16) / 16)


def inputs(seed, kind, B=2, Hq=4, Hk=2, N=9, D=64):
    g = np.random.default_rng(seed)
    q, k, dq, dk = (rounded(g.standard_normal((B, H, N, D)), kind) for H in (Hq, Hk, Hq, Hk))
    return q, k, dq, dk, g.integers(0, 5000, (B, N)).astype(np.int32)


def close(got, dy, kind, pos, interleaved, amplitude):
    want = so.rope(dy, pos, FREQ, interleaved, amplitude, backward=True)
    # sums of two products of at most 4 * amplitude each and a sine or cosine to 2^-21, then the rounding of the result
    assert np.all(np.abs(host(got) - want) <= HALF_STEP[kind] * np.abs(want) * (1 + 2.0 ** -10) + 2 * np.abs(dy).max() * amplitude * 2.0 ** -21 + TINY[kind])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
def test_gradients_of_both(kind, interleaved):
    import paper_2410_02367_amd as sage
    q, k, dq, dk, pos = inputs(1, kind)
    qt, kt = (dev(x, TORCH[kind]).requires_grad_() for x in (q, k))
    p, f = dev(pos), dev(FREQ)
    a, b = sage.sage_rope(qt, kt, p, f, interleaved, 1.5)
    assert a.requires_grad and b.requires_grad
    with torch.no_grad():
        plain = sage.sage_rope(qt, kt, p, f, interleaved, 1.5)
    assert all(torch.equal(x, y) and not y.requires_grad for x, y in zip((a, b), plain))
    ga, gb = torch.autograd.grad((a, b), (qt, kt), (dev(dq, TORCH[kind]), dev(dk, TORCH[kind])))
    close(ga, dq, kind, pos, interleaved, 1.5)
    close(gb, dk, kind, pos, interleaved, 1.5)
    wa, wb = sage.sage_rope_bwd(dev(dq, TORCH[kind]), dev(dk, TORCH[kind]), p, f, interleaved, 1.5)
    assert torch.equal(ga, wa) and torch.equal(gb, wb)


def test_gradients_against_differences():
    """The rotation is linear: the difference of two results is the gradient's product with the step but for rounding."""
    import paper_2410_02367_amd as sage
    q, _, dq, step, pos = inputs(2, "f32", Hq=1, Hk=1, N=3)
    qt = dev(q, torch.float32).requires_grad_()
    y = sage.sage_rope(qt, None, dev(pos), dev(FREQ))
    (y * dev(dq, torch.float32)).sum().backward()
    with torch.no_grad():
        moved = sage.sage_rope(dev(q + step, torch.float32), None, dev(pos), dev(FREQ))
    lhs = float(np.sum((host(moved) - host(y)) * dq))
    rhs = float(np.sum(host(qt.grad) * step))
    # every element of either result is off by some 2^-21 of at most 8
    assert abs(lhs - rhs) <= 3 * q.size * 8 * 2.0 ** -21 * 4


@pytest.mark.parametrize("which", ["q", "k", "q of both", "k of both"])
def test_gradients_of_one(which):
    import paper_2410_02367_amd as sage
    q, k, dq, dk, pos = inputs(3, "f16")
    p, f = dev(pos), dev(FREQ)
    qt, kt = dev(q, torch.float16), dev(k, torch.float16)
    if which in ("q", "k"):                     # one tensor requires a gradient
        x, d = (qt, dq) if which == "q" else (kt, dk)
        x.requires_grad_()
        a, b = sage.sage_rope(qt, kt, p, f)
        assert a.requires_grad == (which == "q") and b.requires_grad == (which == "k")
        (a if which == "q" else b).backward(dev(d, torch.float16))
        close(x.grad, d, "f16", pos, False, 1.0)
    else:                                       # both do, one result is used
        qt.requires_grad_(), kt.requires_grad_()
        a, b = sage.sage_rope(qt, kt, p, f)
        used, x, other, d = (a, qt, kt, dq) if which[0] == "q" else (b, kt, qt, dk)
        used.backward(dev(d, torch.float16))
        close(x.grad, d, "f16", pos, False, 1.0)
        assert other.grad is None


def test_gradients_that_are_expanded_numbers_or_strided():
    import paper_2410_02367_amd as sage
    q, k, _, _, pos = inputs(4, "f32")
    qt, kt = (dev(x, torch.float32).requires_grad_() for x in (q, k))
    a, b = sage.sage_rope(qt, kt, dev(pos), dev(FREQ))
    (a.sum() + b[..., 1:].sum()).backward()
    close(qt.grad, np.ones_like(q), "f32", pos, False, 1.0)
    ones = np.ones_like(k)
    ones[..., 0] = 0
    close(kt.grad, ones, "f32", pos, False, 1.0)
    qt.grad = None
    sage.sage_rope(qt, None, dev(pos), dev(FREQ)).transpose(1, 3).contiguous().sum().backward()
    close(qt.grad, np.ones_like(q), "f32", pos, False, 1.0)


def test_projection_views_and_the_gradient_of_the_gradient():
    import paper_2410_02367_amd as sage
    g = np.random.default_rng(5)
    p, f = dev(np.arange(7, dtype=np.int32)), dev(FREQ)
    fused = dev(g.standard_normal((2, 7, 6, 64)), torch.float32).requires_grad_()
    q, k = fused[:, :, :4].transpose(1, 2), fused[:, :, 4:].transpose(1, 2)
    a, b = sage.sage_rope(q, k, p, f)
    da, db = torch.randn_like(a).requires_grad_(), torch.randn_like(b).requires_grad_()
    (grad,) = torch.autograd.grad((a, b), fused, (da, db), create_graph=True)
    wa, wb = sage.sage_rope_bwd(da.detach(), db.detach(), p, f)
    assert torch.equal(grad[:, :, :4].transpose(1, 2), wa) and torch.equal(grad[:, :, 4:].transpose(1, 2), wb)
    # linear in da: its gradient along fused's own values is the rotation of them
    (again,) = torch.autograd.grad(grad, da, fused.detach())
    assert torch.equal(again, a)


def test_refusals_and_calls_without_gradients():
    import paper_2410_02367_amd as sage
    q, k, _, _, pos = inputs(6, "f16")
    p, f = dev(pos), dev(FREQ)
    qt = dev(q, torch.float16).requires_grad_()
    with pytest.raises(ValueError):
        sage.sage_rope(qt, None, p, f, q_out=torch.empty_like(qt))
    with pytest.raises(ValueError):
        sage.sage_rope(qt.detach(), None, p, f.requires_grad_())
    with pytest.raises(TypeError):
        sage.sage_rope(qt, None, p.long(), f.detach())
    with torch.no_grad():
        out = torch.empty_like(qt)
        assert sage.sage_rope(qt, None, p, f, q_out=out) is out and not out.requires_grad


def test_on_a_named_stream():
    import paper_2410_02367_amd as sage
    q, k, dq, dk, pos = inputs(7, "f32")
    p, f = dev(pos), dev(FREQ)
    qt = dev(q, torch.float32).requires_grad_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = sage.sage_rope(qt, None, p, f, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    y.backward(dev(dq, torch.float32))
    torch.cuda.synchronize()
    close(qt.grad, dq, "f32", pos, False, 1.0)


def test_a_captured_training_step():
    """Forward and backward captured, replayed with new values and eager steps of other leaves between."""
    import paper_2410_02367_amd as sage
    q, k, dq, dk, pos = inputs(8, "bf16")
    p, f = dev(pos), dev(FREQ)

    def step(x, d):
        return torch.autograd.grad(sage.sage_rope(x, None, p, f, True), x, d)[0]
    x, d = dev(q, torch.bfloat16).requires_grad_(), dev(dq, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(dev(q, torch.bfloat16).requires_grad_(), d)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, d)
    for seed in (10, 11, 12):
        new = dev(inputs(seed, "bf16")[2], torch.bfloat16)
        d.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, step(dev(q, torch.bfloat16).requires_grad_(), new))
        torch.cuda.synchronize()
