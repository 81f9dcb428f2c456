"""What a call writes to a tensor that it was given counts as a change in place, as in torch: autograd does not compute
gradients from a saved tensor that has been written over, but says so."""

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say
from layer_helpers import BF16, F32, lengths, rand

pytestmark = pytest.mark.gpu

N, T, D, W, S = 3, 5, 6, 4, 2


def _calls():
    """name -> (call, names of the arguments that it writes to, the other arguments)."""
    x, dout, weight, taps = rand(N, T, D, seed=1), rand(N, T, D, seed=2), rand(D, seed=3), rand(D, W, seed=4)
    a, b, near, far = -rand(D, S, seed=5).abs(), rand(N, T, 1, S, seed=6), rand(N, W - 1, D, seed=7), rand(N, D, S, seed=8)
    e = lambda *s, dtype=F32: torch.empty(s, device=device(), dtype=dtype)                  # noqa: E731
    i32 = torch.int32
    q, decay, mem = rand(N, T, 2, 4, seed=9), -torch.rand(2, device=device()), rand(N, 2, 4, 4, seed=10)
    z, ids, teacher = rand(N, 20, seed=11), lengths([[1, 2], [3, -1], [0, 5]]), rand(N, 2, seed=12)
    stats = rd.rdf2v_residual_norm(x, x.clone(), weight)[2]
    lse = rd.rdf2v_distill_loss(z, ids, teacher)[1]
    parents = lengths([2, 0, 1])
    scan = dict(x=x, dt=x.clone(), a=a, b=b, c=b.clone())
    one = {k: v if k == "a" else v[:, 0] for k, v in scan.items()}
    sg = rd.ScanGradients(e(N, T, D), e(N, T, D), e(D, S), e(N, T, 1, S), e(N, T, 1, S), e(D), e(D), None, e(N, D, S))
    ng = rd.NormGradients(e(N, T, D), e(N, T, D), e(D), e(D), e(D))
    return {
        "conv": (rd.rdf2v_causal_conv, dict(out=e(N, T, D), state_out=e(N, W - 1, D)), dict(x=x, weight=taps)),
        "conv backward": (rd.rdf2v_causal_conv_backward,
                          dict(dx=e(N, T, D), dweight=e(D, W), dbias=e(D), dstate=e(N, W - 1, D)),
                          dict(x=x, weight=taps, bias=weight, dout=dout)),
        "conv step": (rd.rdf2v_causal_conv_step, dict(out=e(N, D), state_out=e(N, W - 1, D)),
                      dict(x=x[:, 0], weight=taps, bias=None, state=near, parents=parents)),
        "conv step in place": (rd.rdf2v_causal_conv_step, dict(state=near.clone()),
                               dict(x=x[:, 0], weight=taps, bias=None)),
        "scan": (rd.rdf2v_selective_scan, dict(out=e(N, T, D), state_out=e(N, D, S)), scan),
        "scan backward": (rd.rdf2v_selective_scan_backward, dict(out=sg), dict(scan, dout=dout, dt_bias=weight)),
        "scan step": (rd.rdf2v_selective_scan_step, dict(out=e(N, D), state_out=e(N, D, S)),
                      dict(one, state=far, parents=parents)),
        "scan step in place": (rd.rdf2v_selective_scan_step, dict(state=far.clone()), one),
        "norm": (rd.rdf2v_residual_norm, dict(out=e(N, T, D), hidden=e(N, T, D), stats=e(N, T, 2)),
                 dict(x=x, residual=x.clone(), weight=weight)),
        "norm backward": (rd.rdf2v_residual_norm_backward, dict(out=ng),
                          dict(x=x, residual=x.clone(), weight=weight, bias=weight, stats=stats, dout=dout,
                               scale=weight)),
        "attention": (rd.rdf2v_decay_attention, dict(out=e(N, T, 2, 4), state_out=e(N, 2, 4, 4)),
                      dict(q=q, k=q.clone(), v=q.clone(), log_decay=decay)),
        "attention backward": (rd.rdf2v_decay_attention_backward,
                               dict(dq=e(N, T, 2, 4), dk=e(N, T, 2, 4), dv=e(N, T, 2, 4), dstate=e(N, 2, 4, 4)),
                               dict(q=q, k=q.clone(), v=q.clone(), log_decay=decay, dout=q.clone(), state=mem)),
        "attention step in place": (rd.rdf2v_decay_attention_step, dict(state=mem.clone()),
                                    dict(q=q[:, 0], k=q[:, 0], v=q[:, 0], log_decay=decay)),
        "select": (rd.rdf2v_beam_select, dict(scores_out=e(1, 2), tokens=e(1, 2, dtype=i32),
                                              parents=e(1, 2, dtype=i32)),
                   dict(logits=z.view(1, N, 20), scores=rand(1, N, seed=13), num_out=2)),
        "reorder": (rd.rdf2v_beam_reorder, dict(out=e(N, 20)), dict(src=z, parents=parents)),
        "distill": (rd.rdf2v_distill_loss, dict(loss=e(N), lse=e(N), dlogits=e(N, 20)),
                    dict(logits=z, ids=ids, teacher=teacher, dloss=rand(N, seed=14))),
        "distill backward": (rd.rdf2v_distill_loss_backward, dict(dlogits=e(N, 20)),
                             dict(logits=z, ids=ids, teacher=teacher, lse=lse, dloss=rand(N, seed=14)))}


def _tensors(arguments):
    flat = []
    for v in arguments.values():
        flat += [t for t in (v if isinstance(v, tuple) else (v,)) if isinstance(t, torch.Tensor)]
    return flat


@pytest.mark.parametrize("name", ["conv", "conv backward", "conv step", "conv step in place", "scan", "scan backward",
                                  "scan step", "scan step in place", "norm", "norm backward", "attention",
                                  "attention backward", "attention step in place", "select", "reorder", "distill",
                                  "distill backward"])
def test_what_is_written_is_a_version_on(name):
    say(f"[versions] {name}")
    call, written, read = _calls()[name]
    before = [t._version for t in _tensors(written)], [t._version for t in _tensors(read)]
    call(**read, **written)
    assert all(t._version > v for t, v in zip(_tensors(written), before[0]))
    assert [t._version for t in _tensors(read)] == before[1]
    with torch.inference_mode():                                               # tensors that have no versions
        call, written, read = _calls()[name]
        call(**read, **written)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
def test_a_saved_state_that_a_step_has_changed(type_):
    """A row is scored from a state, which a step then takes further in place: no gradients from the wrong state."""
    say(f"[versions] saved states {type_}")
    x, taps = rand(N, T, D, type_=type_, seed=1), rand(D, W, seed=2).requires_grad_()
    a, b = (-rand(D, S, seed=3).abs()).requires_grad_(), rand(N, T, 1, S, type_=type_, seed=4)
    q, decay = rand(N, T, 2, 4, type_=type_, seed=5).requires_grad_(), -torch.rand(2, device=device())
    near, far, mem = rand(N, W - 1, D, type_=type_, seed=6), rand(N, D, S, seed=7), rand(N, 2, 4, 4, seed=8)
    outs = (rd.rdf2v_causal_conv(x, taps, state=near)[0], rd.rdf2v_selective_scan(x, x, a, b, b, state=far)[0],
            rd.rdf2v_decay_attention(q, q, q, decay, state=mem)[0])
    with torch.no_grad():
        rd.rdf2v_causal_conv_step(x[:, 0], taps, None, near)
        rd.rdf2v_selective_scan_step(x[:, 0], x[:, 0], a, b[:, 0], b[:, 0], far)
        rd.rdf2v_decay_attention_step(q[:, 0], q[:, 0], q[:, 0], decay, mem)
    for out in outs:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.float().sum().backward()


def test_a_buffer_that_a_saved_tensor_lies_in():
    """Outputs of a call that another operation has saved, and the call again with the same `out`."""
    say("[versions] a buffer used twice")
    x, taps, w = rand(N, T, D, seed=1), rand(D, W, seed=2), rand(D, seed=3).requires_grad_()
    out = torch.empty_like(x)
    y = rd.rdf2v_causal_conv(x, taps, out=out)[0] * w
    rd.rdf2v_causal_conv(x + 1, taps, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
