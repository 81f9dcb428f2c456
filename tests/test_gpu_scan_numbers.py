"""Selective scan: infinities and NaN in a row's last token and in the states' gradients, and rates of any size. The
tokens that fill a row's last chunk are not there, whatever the row leaves behind."""

import pytest
import torch

import layer_refs as refs
import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from layer_helpers import BF16, F32, check, lengths, rand, scan_kinds

pytestmark = pytest.mark.gpu

D, GROUPS, STATES = 6, 2, 5
SUMS = ("da", "db", "dc", "ddt_bias", "dskip")
F32_OUTS = ("state", "dstate", "da", "ddt_bias", "dskip")


def _case(n, t, type_, seed=0):
    """All values positive: an infinity stays one in the sums."""
    pos = lambda *s, k, t_=type_: rand(*s, seed=seed + k).abs().add(0.25).to(t_)           # noqa: E731
    return dict(x=pos(n, t, D, k=1), dt=rand(n, t, D, type_=type_, seed=seed + 2), a=-pos(D, STATES, k=3, t_=F32),
                b=pos(n, t, GROUPS, STATES, k=4), c=pos(n, t, GROUPS, STATES, k=5), dt_bias=rand(D, seed=seed + 6) - 2.0,
                skip=pos(D, k=7, t_=F32), gate=pos(n, t, D, k=8), state=pos(n, D, STATES, k=9, t_=F32))


def _rows(c, lens, dout, dstate_out, absolute):
    """The definition, each row by itself and no longer than it is; parameters' gradients added up."""
    n, t = c["x"].shape[:2]
    whole = None
    for r in range(n):
        length = int(lens[r])
        cut = {k: v[r:r + 1, :length] if k in ("x", "dt", "b", "c", "gate") else v[r:r + 1] if k == "state" else v
               for k, v in c.items()}
        got = refs.scan(**cut, dout=dout[r:r + 1, :length], dstate_out=dstate_out[r:r + 1], absolute=absolute)
        if whole is None:
            whole = {k: torch.zeros_like(v) if k in ("da", "ddt_bias", "dskip") else
                     torch.zeros(n, *(v.shape[1:] if k in ("state", "dstate") else (t, *v.shape[2:])), dtype=v.dtype)
                     for k, v in got.items()}
        for k, v in got.items():
            if k in ("da", "ddt_bias", "dskip"):
                whole[k] += v
            elif k in ("state", "dstate"):
                whole[k][r] = v[0]
            else:
                whole[k][r, :length] = v[0]
    return whole


def _held(c, lens, dout, dstate_out, type_, what):
    """Finite values within their bounds, NaN and infinities where the definition has them and nowhere else."""
    n, t = c["x"].shape[:2]
    given = dict(c, lens=lengths(lens))
    out, end = rd.rdf2v_selective_scan(**given, want_state=True)
    g = rd.rdf2v_selective_scan_backward(dout=dout, dstate_out=dstate_out, **given)
    got = dict(out=out, state=end) | g._asdict()
    ref, size = (_rows(c, lens, dout, dstate_out, absolute) for absolute in (False, True))
    for k, v in got.items():
        v, hit = v.cpu(), ref[k].isfinite()
        assert torch.equal(v.isfinite(), hit), (what, k, v[v.isfinite() != hit], ref[k][v.isfinite() != hit])
        exact = hit | ref[k].isnan()
        assert torch.equal(v.double()[~exact], ref[k][~exact]), (what, k)
        clean = lambda x: torch.where(hit, x, 0.0)                                          # noqa: E731
        check({k: clean(v.double())}, {k: clean(ref[k])}, {k: clean(size[k])}, scan_kinds(t, STATES, D, n), type_,
              (what, k), F32_OUTS)
    return ref


def _lens(t, ragged):
    return [t, 0, t - 1, max(t - 2, 0), t // 2, max(t - 3, 1)] if ragged else [t]


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("t", [1, 4, 5, 6, 7, 8, 9, 14, 19, 296, 297, 298, 299])
def test_a_last_token_that_is_no_number(t, ragged, type_):
    say(f"[scan numbers] last token, {t} tokens, ragged {ragged}, {type_}")
    lens = _lens(t, ragged)
    n = len(lens)
    c = _case(n, t, type_)
    w, u = rand(n, t, D, type_=type_, seed=20).abs(), rand(n, D, STATES, seed=21).abs()
    last = torch.tensor([max(v - 1, 0) for v in lens], device=device())
    rows = torch.arange(n, device=device())
    x = c["x"].clone()
    x[rows, last, 4] = float("inf")
    ref = _held(c | dict(x=x), lens, w, u, type_, "x")
    assert bool(ref["da"].isfinite().all()) and not bool(ref["dskip"].isfinite().all())
    b = c["b"].clone()
    b[rows, last, 1, 2] = float("nan")
    ref = _held(c | dict(b=b), lens, w, u, type_, "b")
    assert bool(ref["da"].isfinite().all()) and not bool(ref["state"].isfinite().all())


@pytest.mark.parametrize("t", [1, 6, 7, 8, 9, 297, 299])
def test_infinite_gradients_of_states(t):
    say(f"[scan numbers] infinite gradient of a state, {t} tokens")
    for lens in (_lens(t, False), _lens(t, True)):
        n = len(lens)
        c = _case(n, t, F32)
        w, u = rand(n, t, D, seed=20).abs(), rand(n, D, STATES, seed=21).abs()
        u[0, 3, 1] = float("inf")
        ref = _held(c, lens, w, u, F32, "dstate_out")
        assert float(ref["da"][3, 1]) == float("inf") and int((~ref["da"].isfinite()).sum()) == 1


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("t", [1, 4, 5, 6, 7, 18, 297, 299])
def test_rates_of_any_size(t, type_):
    """The lowest rate there is forgets everything, tokens with a step of 0 (and those that fill a chunk) nothing."""
    say(f"[scan numbers] rates, {t} tokens, {type_}")
    for ragged in (False, True):
        lens = _lens(t, ragged)
        n = len(lens)
        c = _case(n, t, type_)
        a = c["a"].clone()
        a[1, 0] = a[2, 3] = a[5, 4] = torch.finfo(F32).min
        a[0, 1], a[3, 3], a[4, 0] = -3e38, -2.0 ** 100, -1e-40
        w, u = rand(n, t, D, type_=type_, seed=20), rand(n, D, STATES, seed=21)
        ref = _held(c | dict(a=a), lens, w, u, type_, "rates")
        assert all(bool(v.isfinite().all()) for v in ref.values())
        dt = c["dt"].clone()
        dt[:, t // 2] = torch.finfo(type_).min if ragged else float("-inf")                 # steps of 0
        given = c | dict(a=a, dt=dt)
        status = new_status()
        out, end = rd.rdf2v_selective_scan(**given, lens=lengths(lens), want_state=True, status=status)
        g = rd.rdf2v_selective_scan_backward(dout=w, dstate_out=u, **given, lens=lengths(lens), status=status)
        rd.check_device_status(status)
        low = given | dict(dt=dt.float().clamp(min=-1000.0))                                # a step of 0 in 64 bits too
        ref, size = (_rows(low, lens, w, u, absolute) for absolute in (False, True))
        check(dict(out=out, state=end) | g._asdict(), ref, size, scan_kinds(t, STATES, D, n), type_, "no step", F32_OUTS)


@pytest.mark.parametrize("states", [1, 4, 7, 16])
def test_a_step_with_rates_of_any_size(states):
    say(f"[scan numbers] step, {states} states")
    n, d = 5, 9
    a = -rand(d, states, seed=1).abs()
    a[::2] = torch.finfo(F32).min
    dt = rand(n, d, seed=2)
    dt[1] = float("-inf")
    b = rand(n, 1, states, seed=3)
    state, x = rand(n, d, states, seed=4), rand(n, d, seed=5)
    status = new_status()
    out, new = rd.rdf2v_selective_scan_step(x, dt, a, b, b, state.clone(), status=status)
    rd.check_device_status(status)
    given = dict(x=x[:, None], dt=dt[:, None].clamp(min=-1000.0), a=a, b=b[:, None], c=b[:, None], state=state)
    check(dict(out=out[:, None], state=new), refs.scan(**given), refs.scan(**given, absolute=True),
          scan_kinds(1, states, d, n), F32, "step", ("state",))
    assert torch.equal(new[1], state[1])
