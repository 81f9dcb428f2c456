"""The layer operators within autograd: gradients are the ones of their own backward calls, in the inputs' shapes and
layouts, and nothing that asks for a gradient is cut off without a word."""

import warnings

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say
from layer_helpers import BF16, F32, lengths, rand

pytestmark = pytest.mark.gpu


def _hot(**tensors):
    return {k: None if v is None else v.clone().requires_grad_() for k, v in tensors.items()}


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("length", [3, 40])
def test_conv(length, type_):
    say(f"[layer autograd] convolution, {length} tokens {type_}")
    n, d, width = 3, 20, 4
    hot = _hot(x=rand(n, length, d, type_=type_, seed=1), weight=rand(d, width, seed=2), bias=rand(d, seed=3),
               state=rand(n, width - 1, d, type_=type_, seed=4))
    lens = lengths([length, 0, 2])
    w, u = rand(n, length, d, type_=type_, seed=5), rand(n, width - 1, d, type_=type_, seed=6)
    out, end = rd.rdf2v_causal_conv(**hot, lens=lens, want_state=True)
    assert out.requires_grad and end.requires_grad
    got = torch.autograd.grad([out, end], list(hot.values()), [w, u], retain_graph=True)
    cold = {k: v.detach() for k, v in hot.items()}
    want = rd.rdf2v_causal_conv_backward(cold["x"], cold["weight"], cold["bias"], w, lens=lens, state=cold["state"],
                                         dstate_out=u)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # the states alone; the outputs alone, by a gradient of stride 0, without bias and states
    got = torch.autograd.grad(end, hot["x"], u)[0]
    want = rd.rdf2v_causal_conv_backward(cold["x"], cold["weight"], cold["bias"], torch.zeros_like(w), lens=lens,
                                         state=cold["state"], dstate_out=u)[0]
    assert torch.equal(got, want)
    out, none = rd.rdf2v_causal_conv(hot["x"], hot["weight"], silu=False)
    assert none is None
    got = torch.autograd.grad(out.sum(), [hot["x"], hot["weight"]])
    want = rd.rdf2v_causal_conv_backward(cold["x"], cold["weight"], None, torch.ones_like(w), silu=False)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("length,gated", [(3, True), (300, True), (40, False)])
def test_scan(length, gated, type_):
    say(f"[layer autograd] scan, {length} tokens {type_}, gate {gated}")
    n, d, groups, states = 2, 12, 2, 5
    hot = _hot(x=rand(n, length, d, type_=type_, seed=1), dt=rand(n, length, d, type_=type_, seed=2),
               a=-rand(d, states, seed=3).abs(), b=rand(n, length, groups, states, type_=type_, seed=4),
               c=rand(n, length, groups, states, type_=type_, seed=5), dt_bias=rand(d, seed=6) if gated else None,
               skip=rand(d, seed=7) if gated else None,
               gate=rand(n, length, d, type_=type_, seed=8) if gated else None, state=rand(n, d, states, seed=9))
    lens = lengths([length, length // 2])
    w, u = rand(n, length, d, type_=type_, seed=10), rand(n, d, states, seed=11)
    out, end = rd.rdf2v_selective_scan(**hot, lens=lens, want_state=True)
    given = {k: v for k, v in hot.items() if v is not None}
    got = torch.autograd.grad([out, end], list(given.values()), [w, u], retain_graph=True)
    cold = {k: None if v is None else v.detach() for k, v in hot.items()}
    want = rd.rdf2v_selective_scan_backward(dout=w, dstate_out=u, lens=lens, **cold)._asdict()
    for name, g in zip(given, got):
        assert torch.equal(g, want[name if name.startswith("d") and "d" + name not in want else "d" + name]), name
    got = torch.autograd.grad(end, hot["a"], u)[0]
    want = rd.rdf2v_selective_scan_backward(dout=torch.zeros_like(w), dstate_out=u, lens=lens, **cold).da
    assert torch.equal(got, want)


@pytest.mark.parametrize("type_,stream", [(F32, F32), (BF16, F32), (BF16, BF16)], ids=["f32", "bf16-f32", "bf16"])
def test_norm(type_, stream):
    say(f"[layer autograd] norm {type_} {stream}")
    n, t, d = 3, 5, 30
    hot = _hot(x=rand(n, t, d, type_=type_, seed=1), residual=rand(n, t, d, type_=stream, seed=2),
               weight=rand(d, seed=3), bias=rand(d, seed=4), scale=rand(d, seed=5))
    lens = lengths([t, 2, 0])
    w, u = rand(n, t, d, type_=type_, seed=6), rand(n, t, d, type_=stream, seed=7)
    given = dict(drop=0.25, seed=5, center=True, lens=lens)
    out, hidden, stats = rd.rdf2v_residual_norm(**hot, **given)
    assert out.requires_grad and hidden.requires_grad and not stats.requires_grad
    names = ("x", "residual", "weight", "bias", "scale")
    got = torch.autograd.grad([out, hidden], [hot[k] for k in names], [w, u], retain_graph=True)
    cold = {k: v.detach() for k, v in hot.items()}
    scale = cold.pop("scale")
    want = rd.rdf2v_residual_norm_backward(**cold, stats=stats, dout=w, dhidden=u, scale=scale, **given)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = torch.autograd.grad(hidden, hot["x"], u)[0]                       # the stream alone: dropout and scale
    kept = (rd.rdf2v_residual_norm(torch.ones_like(cold["x"]), None, cold["weight"], **given)[1] != 0)
    assert bool((got[~kept] == 0).all())
    off = (got.float() - torch.where(kept, u.float() * scale / 0.75, 0.0)).abs()
    assert float(off.max()) <= 2.0 ** -7 * float((u.float() * scale).abs().max())
    # no residual, a stream of 32 bits all the same; rows without a length
    out, hidden, _ = rd.rdf2v_residual_norm(hot["x"][:, 0], None, hot["weight"], hidden_dtype=F32)
    assert hidden.dtype == F32
    assert torch.autograd.grad(out.sum() + hidden.sum(), hot["x"])[0].shape == hot["x"].shape


def test_a_gradient_through_several_calls_adds_up():
    """Leaves that two calls share: autograd adds the calls' gradients."""
    say("[layer autograd] shared leaves")
    x, w = rand(2, 6, 8, seed=1).requires_grad_(), rand(8, 3, seed=2).requires_grad_()
    one = torch.autograd.grad(rd.rdf2v_causal_conv(x, w)[0].sum(), [x, w])
    two = torch.autograd.grad(rd.rdf2v_causal_conv(x, w)[0].sum() + rd.rdf2v_causal_conv(x, w)[0].sum(), [x, w])
    assert all(torch.equal(2 * a, b) for a, b in zip(one, two))


def test_nothing_is_cut_off_without_a_word():
    say("[layer autograd] outputs that are given, calls for answering")
    x, w, bias = rand(2, 4, 6, seed=1), rand(6, 3, seed=2), rand(6, seed=3)
    state = rand(2, 2, 6, seed=4)
    hot = x.clone().requires_grad_()
    for kw in (dict(out=torch.empty_like(x)), dict(state_out=torch.empty_like(state))):
        with pytest.raises(ValueError):
            rd.rdf2v_causal_conv(hot, w, **kw)
        with torch.no_grad():
            rd.rdf2v_causal_conv(hot, w, **kw)
    a, b = -rand(6, 4, seed=5).abs(), rand(2, 4, 1, 4, seed=6)
    with pytest.raises(ValueError):
        rd.rdf2v_selective_scan(x, x, a.clone().requires_grad_(), b, b, out=torch.empty_like(x))
    for kw in (dict(out=torch.empty_like(x)), dict(hidden=torch.empty_like(x)),
               dict(stats=torch.empty(2, 4, 2, device=device()))):
        with pytest.raises(ValueError):
            rd.rdf2v_residual_norm(hot, None, bias, **kw)
    held = rand(2, 6, 4, seed=7)
    calls = (lambda g: rd.rdf2v_causal_conv_step(x[:, 0].clone().requires_grad_(g), w, bias, state.clone()),
             lambda g: rd.rdf2v_selective_scan_step(x[:, 0], x[:, 0], a.clone().requires_grad_(g), b[:, 0], b[:, 0],
                                                    held.clone()))
    for call in calls:
        with pytest.warns(UserWarning, match="no gradient"):
            call(True)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call(False)
            with torch.no_grad():
                call(True)


def test_arguments_are_checked():
    say("[layer autograd] arguments")
    x, w = rand(2, 4, 6, seed=1), rand(6, 3, seed=2)
    a, b = -rand(6, 4, seed=5).abs(), rand(2, 4, 1, 4, seed=6)
    for error, call in (
            (TypeError, lambda: rd.rdf2v_causal_conv(x.cpu(), w)), (TypeError, lambda: rd.rdf2v_causal_conv(x.half(), w)),
            (ValueError, lambda: rd.rdf2v_causal_conv(x[0], w)), (ValueError, lambda: rd.rdf2v_causal_conv(x, w.T)),
            (TypeError, lambda: rd.rdf2v_causal_conv(x, w.bfloat16())),
            (ValueError, lambda: rd.rdf2v_causal_conv(x.transpose(1, 2), rand(4, 3))),
            (ValueError, lambda: rd.rdf2v_causal_conv(x, rand(6, 9))),
            (ValueError, lambda: rd.rdf2v_causal_conv(x, w, state=rand(2, 3, 6))),
            (TypeError, lambda: rd.rdf2v_causal_conv(x, w, state=rand(2, 2, 6).bfloat16())),
            (ValueError, lambda: rd.rdf2v_causal_conv(x, w, lens=lengths([1]))),
            (ValueError, lambda: rd.rdf2v_causal_conv_step(x[:, 0], w, None, rand(3, 2, 6))),
            (ValueError, lambda: rd.rdf2v_causal_conv_step(x[:, 0], w, None, rand(3, 2, 6), parents=lengths([1]))),
            (TypeError, lambda: rd.rdf2v_causal_conv_step(x[:, 0], w, None, None)),
            (TypeError, lambda: rd.rdf2v_selective_scan(x, x.bfloat16(), a, b, b)),
            (ValueError, lambda: rd.rdf2v_selective_scan(x, x, a, b, b[:, :, :, :3])),
            (ValueError, lambda: rd.rdf2v_selective_scan(x, x, a, b.expand(2, 4, 4, 4), b.expand(2, 4, 4, 4))),
            (ValueError, lambda: rd.rdf2v_selective_scan(x, x, a[:5], b, b)),
            (TypeError, lambda: rd.rdf2v_selective_scan(x, x, None, b, b)),
            (ValueError, lambda: rd.rdf2v_selective_scan(x, x, a, b, b, gate=x[:, :3])),
            (ValueError, lambda: rd.rdf2v_selective_scan(x, x, rand(6, 65), rand(2, 4, 1, 65), rand(2, 4, 1, 65))),
            (TypeError, lambda: rd.rdf2v_residual_norm(x, x.bfloat16(), w[:, 0].contiguous())),
            (ValueError, lambda: rd.rdf2v_residual_norm(x, x[:1], w[:, 0].contiguous())),
            (ValueError, lambda: rd.rdf2v_residual_norm(x, x, rand(5))),
            (ValueError, lambda: rd.rdf2v_residual_norm(x, x, rand(6), drop=1.0)),
            (ValueError, lambda: rd.rdf2v_residual_norm(x, x, rand(6), row_begin=-1)),
            (TypeError, lambda: rd.rdf2v_residual_norm(x, x, rand(6), seed_offset=lengths([1]))),
            (ValueError, lambda: rd.rdf2v_residual_norm(rand(1, 1, 16385), None, rand(16385))),
            (rd.Rdf2vError, lambda: rd.rdf2v_residual_norm(x, x, rand(6), eps=float("nan")))):
        with pytest.raises(error):
            call()
