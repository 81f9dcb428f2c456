"""Calls with `stream=` that autograd records: their gradients are computed on that stream, after what the forward call
left there, and whatever is allocated next on either stream leaves them alone."""

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say
from layer_helpers import BF16, F32, lengths, rand

pytestmark = pytest.mark.gpu


def _norm(type_):
    x, res, w = rand(40, 17, 96, type_=type_, seed=1), rand(40, 17, 96, seed=2), rand(96, seed=3)
    return [x, res, w], [rand(40, 17, 96, type_=type_, seed=4), rand(40, 17, 96, seed=5)], \
        lambda x, res, w, **k: rd.rdf2v_residual_norm(x, res, w, center=True, drop=0.1, seed=3, **k)[:2]


def _distill(type_):
    ids = torch.arange(600, device=device(), dtype=torch.int32).view(200, 3)
    teacher = rand(200, 3, seed=2)
    return [rand(200, 700, type_=type_, seed=1)], [rand(200, seed=3)], \
        lambda z, **k: rd.rdf2v_distill_loss(z, ids, teacher, **k)[:1]


def _conv(type_):
    lens = lengths([r % 18 for r in range(40)])
    return [rand(40, 17, 64, type_=type_, seed=1), rand(64, 4, seed=2), rand(64, seed=3)], \
        [rand(40, 17, 64, type_=type_, seed=4), rand(40, 3, 64, type_=type_, seed=5)], \
        lambda x, w, b, **k: rd.rdf2v_causal_conv(x, w, b, lens=lens, want_state=True, **k)


def _scan(type_):
    return [rand(4, 300, 30, type_=type_, seed=1), rand(4, 300, 30, type_=type_, seed=2), -rand(30, 8, seed=3).abs(),
            rand(4, 300, 1, 8, type_=type_, seed=4), rand(4, 300, 1, 8, type_=type_, seed=5)], \
        [rand(4, 300, 30, type_=type_, seed=6), rand(4, 30, 8, seed=7)], \
        lambda *a, **k: rd.rdf2v_selective_scan(*a, want_state=True, **k)


def _attention(type_):
    decay = -torch.rand(3, device=device())
    return [rand(5, 40, 3, 16, type_=type_, seed=k) for k in (1, 2, 3)], [rand(5, 40, 3, 16, type_=type_, seed=4)], \
        lambda q, k, v, **kw: rd.rdf2v_decay_attention(q, k, v, decay, **kw)[:1]


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("made", [_norm, _distill, _conv, _scan, _attention])
def test_gradients_follow_the_stream(made, type_):
    """The current stream is busy where the gradients are asked for, and both streams' memory is written anew after:
    what the forward call saved is in no other's hands before the gradients have read it."""
    say(f"[recorded streams] {made.__name__} {type_}")
    tensors, gradients, call = made(type_)
    leaves = [t.requires_grad_() for t in tensors]
    want = [g.clone() for g in torch.autograd.grad(call(*leaves), leaves, gradients)]
    side = torch.cuda.Stream()
    for again in range(3):
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        inputs = [t * 1 for t in leaves]                       # not leaves: the graph alone holds them in the end
        side.wait_stream(torch.cuda.current_stream())
        outs = call(*inputs, stream=side)
        sizes = {t.numel() * t.element_size() for t in (*inputs, *outs)} | {40 * 17 * 8, 800}
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(20_000_000)
        got = torch.autograd.grad(outs, leaves, gradients)
        del inputs, outs
        new = []
        for stream in (side, torch.cuda.current_stream()):
            with torch.cuda.stream(stream):
                new += [torch.full((size,), 0xFF, dtype=torch.uint8, device=device()) for size in sizes for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), again


@pytest.mark.parametrize("made", [_norm, _distill, _scan])
def test_a_loss_on_the_calls_stream(made):
    """Call and loss on a stream of their own, the gradients asked for on another without a word between the two."""
    say(f"[recorded streams] {made.__name__}, loss there too")
    tensors, gradients, call = made(F32)
    leaves = [t.requires_grad_() for t in tensors]
    for t in leaves:
        t.grad = None
    sum((o * g).sum() for o, g in zip(call(*leaves), gradients)).backward()
    want = [t.grad.clone() for t in leaves]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for t in leaves:
        t.grad = None
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        outs = call(*leaves, stream=side)
        loss = sum((o * g).sum() for o, g in zip(outs, gradients))
    del outs
    loss.backward()
    got = [t.grad for t in leaves]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
