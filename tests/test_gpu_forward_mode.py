"""Forward-mode derivatives: there are none, and an input with a tangent is refused instead of losing it."""

import pytest
import torch
from torch.autograd import forward_ad

import paper_2508_01073_amd as rd
from gpu_helpers import device, say
from layer_helpers import lengths, rand

pytestmark = pytest.mark.gpu

N, T, D, W, S = 3, 5, 6, 4, 2


def _calls():
    x, weight, taps = rand(N, T, D, seed=1), rand(D, seed=3), rand(D, W, seed=4)
    a, b, near, far = -rand(D, S, seed=5).abs(), rand(N, T, 1, S, seed=6), rand(N, W - 1, D, seed=7), rand(N, D, S, seed=8)
    q, decay, mem = rand(N, T, 2, 4, seed=9), -torch.rand(2, device=device()), rand(N, 2, 4, 4, seed=10)
    z, ids, teacher = rand(N, 20, seed=11), lengths([[1, 2], [3, -1], [0, 5]]), rand(N, 2, seed=12)
    return {
        "conv": (rd.rdf2v_causal_conv, dict(x=x, weight=taps, bias=weight, state=near)),
        "conv step": (rd.rdf2v_causal_conv_step, dict(x=x[:, 0], weight=taps, bias=weight, state=near)),
        "scan": (rd.rdf2v_selective_scan, dict(x=x, dt=x.clone(), a=a, b=b, c=b.clone(), dt_bias=weight,
                                               skip=weight.clone(), gate=x.clone(), state=far)),
        "scan step": (rd.rdf2v_selective_scan_step, dict(x=x[:, 0], dt=x[:, 1], a=a, b=b[:, 0], c=b[:, 1], state=far,
                                                         dt_bias=weight, skip=weight.clone(), gate=x[:, 2])),
        "norm": (rd.rdf2v_residual_norm, dict(x=x, residual=x.clone(), weight=weight, bias=weight.clone(),
                                              scale=weight.clone())),
        "attention": (rd.rdf2v_decay_attention, dict(q=q, k=q.clone(), v=q.clone(), log_decay=decay, state=mem)),
        "attention step": (rd.rdf2v_decay_attention_step, dict(q=q[:, 0], k=q[:, 1], v=q[:, 2], log_decay=decay,
                                                               state=mem)),
        "distill": (lambda **k: rd.rdf2v_distill_loss(ids=ids, **k), dict(logits=z, teacher=teacher)),
        "distill, gradients too": (lambda **k: rd.rdf2v_distill_loss(ids=ids, dloss=torch.ones(N, device=device()), **k),
                                   dict(logits=z, teacher=teacher)),
        "select": (lambda **k: rd.rdf2v_beam_select(num_out=2, **k), dict(logits=z.view(1, N, 20),
                                                                          scores=rand(1, N, seed=13))),
        "reorder": (lambda **k: rd.rdf2v_beam_reorder(parents=lengths([2, 0, 1]), **k), dict(src=z))}


@pytest.mark.parametrize("name", ["conv", "conv step", "scan", "scan step", "norm", "attention", "attention step",
                                  "distill", "distill, gradients too", "select", "reorder"])
@pytest.mark.parametrize("recorded", [False, True])
def test_a_tangent_is_refused(name, recorded):
    say(f"[forward mode] {name}, recorded {recorded}")
    call, arguments = _calls()[name]
    with torch.set_grad_enabled(recorded), forward_ad.dual_level():
        for key, t in arguments.items():
            if recorded and "step" not in name and name not in ("select", "reorder"):
                t = t.clone().requires_grad_()
            with pytest.raises(NotImplementedError):
                call(**(arguments | {key: forward_ad.make_dual(t, torch.ones_like(t))}))
        call(**arguments)                                      # without one they are as ever


def test_a_reordering_says_that_it_has_no_gradient():
    say("[forward mode] reordering")
    src = rand(3, 20, seed=11).requires_grad_()
    with pytest.warns(UserWarning, match="no gradient"):
        rd.rdf2v_beam_reorder(src, lengths([2, 0, 1]))
