"""Causal convolution on the GPU against plain 64-bit loops: whole rows, gradients, single tokens."""

import pytest
import torch

import layer_refs as refs
import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from layer_helpers import BF16, F32, check, conv_kinds, junk, lengths, rand

pytestmark = pytest.mark.gpu

# rows, length, channels, width
SIZES = [(1, 1, 1, 1), (2, 1, 5, 4), (3, 17, 8, 4), (4, 33, 13, 3), (2, 40, 64, 2), (1, 70, 130, 8), (3, 2, 24, 8),
         (2, 16, 516, 5), (1, 130, 7, 6), (5, 9, 33, 7)]


def _case(n, t, d, width, type_, state, ragged, seed=0):
    wide = rand(n, t, 2 * d + 3, type_=type_, seed=seed + 1)
    x = wide[..., d:2 * d]                                                   # a slice at any alignment
    lens = lengths([(t * (3 * r + 1) // 4 if r % 3 else 0) % (t + 1) if n > 1 else t - t // 5 for r in range(n)]) \
        if ragged else None
    return dict(x=junk(x, lens) if ragged else x, weight=rand(d, width, seed=seed + 2), bias=rand(d, seed=seed + 3),
                lens=lens, state=rand(n, width - 1, d, type_=type_, seed=seed + 4) if state else None)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,t,d,width", SIZES)
@pytest.mark.parametrize("ragged,state,silu", [(False, False, True), (True, True, True), (True, False, False)])
def test_against_loops(n, t, d, width, type_, ragged, state, silu):
    say(f"[conv] {n} rows of {t}, {d} channels, width {width}, {type_}, ragged {ragged}, state {state}")
    c = _case(n, t, d, width, type_, state, ragged)
    w, u = rand(n, t, d, type_=type_, seed=8), rand(n, width - 1, d, type_=type_, seed=9)
    w = junk(w, c["lens"])
    status = new_status()
    out, end = rd.rdf2v_causal_conv(**c, silu=silu, want_state=True, status=status)
    dx, dweight, dbias, dstate = rd.rdf2v_causal_conv_backward(c["x"], c["weight"], c["bias"], w, silu=silu,
                                                               lens=c["lens"], state=c["state"], dstate_out=u,
                                                               dstate=torch.empty_like(u), status=status)
    rd.check_device_status(status)
    given = dict(c, silu=silu, dout=w, dstate_out=u)
    ref, sizes = refs.conv(**given), refs.conv(**given, absolute=True)
    check(dict(out=out, state=end, dx=dx, dweight=dweight, dbias=dbias, dstate=dstate), ref, sizes,
          conv_kinds(t, width, n), type_, (n, t, d, width), ("state", "dweight", "dbias"))
    assert torch.equal(end.double().cpu(), ref["state"])                     # inputs are handed on as they are
    for x in (out, dx):
        dead = torch.arange(t) >= (torch.full((n,), t) if c["lens"] is None else c["lens"].cpu())[:, None]
        assert bool((x.cpu()[dead] == 0).all())
    # without a bias, without states
    out, none = rd.rdf2v_causal_conv(c["x"], c["weight"], silu=silu, lens=c["lens"])
    assert none is None
    given = dict(x=c["x"], weight=c["weight"], silu=silu, lens=c["lens"])
    check(dict(out=out), refs.conv(**given), refs.conv(**given, absolute=True), conv_kinds(t, width, n), type_, "bare")


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("width", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [1, 12, 100])
def test_a_step_is_a_row_of_one_token(d, width, type_):
    say(f"[conv] step, {d} channels, width {width}, {type_}")
    states, rows = 5, 7
    x = rand(rows, 3 * d, type_=type_, seed=1)[:, d:2 * d]
    w, bias = rand(d, width, seed=2), rand(d, seed=3)
    state = rand(states, width - 1, d, type_=type_, seed=4)
    parents = lengths([4, 0, 0, 3, 1, 4, 2])
    status = new_status()
    out, new = rd.rdf2v_causal_conv_step(x, w, bias, state, parents=parents, status=status)
    whole, end = rd.rdf2v_causal_conv(x[:, None], w, bias, state=state[parents.long()], want_state=True)
    assert torch.equal(new, end)
    given = dict(x=x[:, None], weight=w, bias=bias, state=state[parents.long()])
    check(dict(out=out[:, None]), refs.conv(**given), refs.conv(**given, absolute=True), conv_kinds(1, width, rows),
          type_, "step")
    rd.check_device_status(status)
    # in place, and parents that there are not: zeros
    held = state[:3].clone()
    out, new = rd.rdf2v_causal_conv_step(x[:3], w, bias, held, silu=False)
    assert new.data_ptr() == held.data_ptr() or width == 1
    assert torch.equal(new, torch.cat((state[:3], x[:3, None]), 1)[:, 1:])
    bad = lengths([-1, 5, 2])
    out, new = rd.rdf2v_causal_conv_step(x[:3], w, bias, state, parents=bad, status=status)
    assert int(status.item()) == rd.RDF2V_STATUS_ID_OUT_OF_RANGE
    zeros = torch.zeros_like(state[:2])
    assert torch.equal(new, torch.cat((torch.cat((zeros, state[2:3])), x[:3, None]), 1)[:, 1:])


def test_parts_of_a_row_are_the_row():
    say("[conv] a row in parts")
    x, w, bias = rand(2, 61, 20, type_=BF16, seed=1), rand(20, 4, seed=2), rand(20, seed=3)
    whole, end = rd.rdf2v_causal_conv(x, w, bias, want_state=True)
    state, outs, at = None, [], 0
    for part in (1, 2, 30, 0, 28):
        out, state = rd.rdf2v_causal_conv(x[:, at:at + part], w, bias, state=state, want_state=True)
        outs.append(out)
        at += part
    assert torch.equal(torch.cat(outs, 1), whole) and torch.equal(state, end)


def test_what_is_no_number_stays_where_the_formula_has_it():
    say("[conv] NaN")
    x, w = rand(2, 40, 12, seed=1), rand(12, 4, seed=2)
    clean = rd.rdf2v_causal_conv(x, w)[0]
    x[0, 15, 5] = float("nan")
    got = rd.rdf2v_causal_conv(x, w)[0]
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[0, 15:19, 5] = True
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])


def test_lengths_out_of_range_and_no_rows():
    say("[conv] lengths out of range, no rows, no tokens")
    x, w = rand(3, 4, 6, seed=1), rand(6, 3, seed=2)
    status = new_status()
    out = rd.rdf2v_causal_conv(x, w, lens=lengths([5, -1, 4]), status=status)[0]
    assert int(status.item()) == rd.RDF2V_STATUS_BAD_LENGTH
    assert torch.equal(out[0], rd.rdf2v_causal_conv(x, w)[0][0]) and bool((out[1] == 0).all())
    for n, t in ((0, 5), (3, 0), (0, 0)):
        x, state = x.new_empty(n, t, 6), rand(n, 2, 6, seed=3)
        out, end = rd.rdf2v_causal_conv(x, w, state=state, want_state=True)
        assert out.shape == (n, t, 6) and torch.equal(end, state)
        dx, dw, db, ds = rd.rdf2v_causal_conv_backward(x, w, w[:, 0].contiguous(), x, state=state, dstate_out=state)
        assert bool((dw == 0).all()) and bool((db == 0).all()) and torch.equal(ds, state)


def test_outputs_over_inputs_are_refused():
    say("[conv] overlaps")
    x, w, state = rand(2, 8, 4, seed=1), rand(4, 3, seed=2), rand(2, 2, 4, seed=3)
    for kw in (dict(out=x), dict(state_out=state), dict(out=x.view(-1)[:64].view(2, 8, 4))):
        with pytest.raises(rd.Rdf2vError):
            rd.rdf2v_causal_conv(x, w, state=state, **kw)
    buffer = torch.empty(2, 8, 8, device=device())
    rd.rdf2v_causal_conv(buffer[..., :4].copy_(x), w, out=torch.empty_like(x))   # a slice beside others is not refused
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_causal_conv_backward(x, w, None, x.clone(), dx=x)
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_causal_conv_step(x[:, 0], w, None, state, parents=lengths([1, 0]), state_out=state)
