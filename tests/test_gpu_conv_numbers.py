"""Causal convolution: infinite taps, and NaN among them, reach the gradients of the inputs that they multiply and no
others. What lies before a row's first token and behind its last has no outputs."""

import pytest
import torch

import layer_refs as refs
import paper_2508_01073_amd as rd
from gpu_helpers import say
from layer_helpers import BF16, F32, check, conv_kinds, lengths, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("t,width", [(1, 2), (2, 8), (3, 4), (16, 4), (17, 3), (40, 8), (150, 5)])
def test_taps_that_are_no_numbers(t, width, state, type_):
    say(f"[conv numbers] {t} tokens, width {width}, state {state}, {type_}")
    d = 2 * width + 1
    lens = [t, 0, t - 1, t // 2, max(t - 3, 0), 1]
    n = len(lens)
    w = rand(d, width, seed=1)
    for j in range(width):
        w[2 * j, j], w[2 * j + 1, j] = float("inf"), float("nan")
    x, dout = rand(n, t, d, type_=type_, seed=2), rand(n, t, d, type_=type_, seed=3)
    held = rand(n, width - 1, d, type_=type_, seed=4) if state else None
    u = rand(n, width - 1, d, type_=type_, seed=5) if state else None
    dx, dw, _, ds = rd.rdf2v_causal_conv_backward(x, w, None, dout, silu=False, lens=lengths(lens), state=held,
                                                  dstate_out=u)
    given = dict(x=x, weight=w, silu=False, lens=lengths(lens), state=held, dout=dout, dstate_out=u)
    ref, size = refs.conv(**given), refs.conv(**given, absolute=True)
    for name, got in (("dx", dx), ("dweight", dw), ("dstate", ds)):
        if got is None:
            continue
        got, want = got.cpu(), ref[name]
        hit = want.isfinite()
        assert torch.equal(got.isfinite(), hit), (name, int((got.isfinite() != hit).sum()))
        exact = hit | want.isnan()
        assert torch.equal(got.double()[~exact], want[~exact]), name
        clean = lambda v: torch.where(hit, v, 0.0)                                          # noqa: E731
        check({name: clean(got.double())}, {name: clean(want)}, {name: clean(size[name])}, conv_kinds(t, width, n), type_,
              name, ("dweight",))
    if t > width:
        assert bool(ref["dx"].isfinite().any(0)[t - 1, 0]) and not bool(ref["dx"].isfinite().all())
