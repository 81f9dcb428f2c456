"""The operators within autograd: gradients are the ones of their own backward calls, and nothing that asks
for a gradient is cut off without a word."""

import warnings

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _rand(*shape, type_=F32, seed=0):
    g = torch.Generator(device=device()).manual_seed(seed)
    return torch.randn(*shape, device=device(), generator=g).to(type_)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("length", [17, 130, 600])
def test_decay_attention(length, type_):
    say(f"[autograd] decay attention, {length} tokens {type_}")
    n, heads, kv, dk, dv = 2, 4, 2, 32, 48
    wide = _rand(n, length, heads * dk + kv * (dk + dv), type_=type_, seed=1).requires_grad_()
    q, k, v = wide.split([heads * dk, kv * dk, kv * dv], dim=-1)
    q, k, v = q.unflatten(-1, (heads, dk)), k.unflatten(-1, (kv, dk)), v.unflatten(-1, (kv, dv))
    state = _rand(n, heads, dk, dv, seed=2).requires_grad_()
    decay = torch.tensor([-0.1, -0.01, 0.0, -1.0], device=device())
    lens = torch.tensor([length, length // 2], dtype=torch.int32, device=device())
    w, u = _rand(n, length, heads, dv, type_=type_, seed=3), _rand(n, heads, dk, dv, seed=4)
    out, end = rd.rdf2v_decay_attention(q, k, v, decay, scale=0.3, lens=lens, state=state, want_state=True)
    assert out.requires_grad and end.requires_grad
    wide_grad, state_grad = torch.autograd.grad([out, end], [wide, state], [w, u])
    with torch.no_grad():
        plain = rd.rdf2v_decay_attention(q, k, v, decay, scale=0.3, lens=lens, state=state, want_state=True)
        want = rd.rdf2v_decay_attention_backward(q, k, v, decay, w, scale=0.3, lens=lens, state=state, dstate_out=u)
    assert torch.equal(out, plain[0]) and torch.equal(end, plain[1]) and not plain[0].requires_grad
    assert torch.equal(wide_grad, torch.cat([x.flatten(2) for x in want[:3]], -1)) and torch.equal(state_grad, want[3])
    # the states alone, the outputs alone through a gradient of stride 0, no states
    got = torch.autograd.grad(rd.rdf2v_decay_attention(q, k, v, decay, state=state, want_state=True)[1], wide, u)[0]
    want = rd.rdf2v_decay_attention_backward(q.detach(), k.detach(), v.detach(), decay, torch.zeros_like(w),
                                             state=state.detach(), dstate_out=u)
    assert torch.equal(got, torch.cat([x.flatten(2) for x in want[:3]], -1))
    out, none = rd.rdf2v_decay_attention(q, k, v, decay)
    assert none is None
    got = torch.autograd.grad(out.sum(), wide)[0]
    want = rd.rdf2v_decay_attention_backward(q.detach(), k.detach(), v.detach(), decay, torch.ones_like(w))
    assert torch.equal(got, torch.cat([x.flatten(2) for x in want[:3]], -1))


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [700, 100_050])
def test_distill(vocab, type_):
    say(f"[autograd] distillation, vocabulary of {vocab} {type_}")
    z = _rand(6, vocab, type_=type_, seed=5).requires_grad_()
    ids = torch.randint(-1, vocab, (6, 9), device=device(), dtype=torch.int32)
    t, w = _rand(6, 9, seed=6), _rand(6, seed=7)
    loss, lse = rd.rdf2v_distill_loss(z, ids, t, temperature=2.0)
    assert loss.requires_grad and not lse.requires_grad
    plain = rd.rdf2v_distill_loss(z.detach(), ids, t, temperature=2.0)
    assert torch.equal(loss, plain[0]) and torch.equal(lse, plain[1]) and not plain[0].requires_grad
    want = rd.rdf2v_distill_loss_backward(z.detach(), ids, t, plain[1], w, temperature=2.0)
    assert torch.equal(torch.autograd.grad(loss, z, w, retain_graph=True)[0], want)
    mean = rd.rdf2v_distill_loss_backward(z.detach(), ids, t, plain[1], torch.full((6,), 1 / 6, device=device()),
                                          temperature=2.0)
    assert torch.equal(torch.autograd.grad(loss.mean(), z)[0], mean)
    # a gradient that is asked for in the call is the call's own matter
    got = rd.rdf2v_distill_loss(z, ids, t, temperature=2.0, dloss=w)
    assert not any(x.requires_grad for x in got)


def test_nothing_is_cut_off_without_a_word():
    say("[autograd] outputs that are given, constants, calls for answering")
    q, k, v = (_rand(1, 5, 2, 8, seed=i) for i in range(3))
    decay = torch.full((2,), -0.1, device=device())
    state = _rand(1, 2, 8, 8, seed=4)
    hot = q.clone().requires_grad_()
    for name, x in (("out", torch.empty_like(v)), ("state_out", state)):
        with pytest.raises(ValueError):
            rd.rdf2v_decay_attention(hot, k, v, decay, **{name: x})
        with torch.no_grad():
            rd.rdf2v_decay_attention(hot, k, v, decay, **{name: x})
    z, ids, t = _rand(3, 40, seed=8), torch.zeros(3, 2, device=device(), dtype=torch.int32), _rand(3, 2, seed=9)
    with pytest.raises(ValueError):
        rd.rdf2v_distill_loss(z.clone().requires_grad_(), ids, t, loss=torch.empty(3, device=device()))
    scores = torch.zeros(1, 3, device=device())
    cases = (lambda g: rd.rdf2v_decay_attention(q, k, v, decay.clone().requires_grad_(g)),
             lambda g: rd.rdf2v_decay_attention_step(q[:, 0].clone().requires_grad_(g), k[:, 0], v[:, 0], decay, state),
             lambda g: rd.rdf2v_beam_select(z.view(1, 3, 40).clone().requires_grad_(g), scores, 2),
             lambda g: rd.rdf2v_distill_loss(z, ids, t.clone().requires_grad_(g)))
    for call in cases:
        with pytest.warns(UserWarning, match="no gradient"):
            call(True)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call(False)
            with torch.no_grad():
                call(True)
