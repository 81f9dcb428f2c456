"""Selective scan on the GPU against plain 64-bit loops: whole rows, gradients, single tokens."""

import pytest
import torch

import layer_refs as refs
import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from layer_helpers import BF16, F32, check, junk, lengths, rand, scan_kinds

pytestmark = pytest.mark.gpu

# rows, length, channels, groups, states
SIZES = [(1, 1, 1, 1, 1), (2, 1, 6, 2, 4), (3, 17, 64, 1, 16), (4, 33, 70, 1, 11), (2, 16, 24, 4, 3), (3, 5, 130, 2, 16),
         (1, 100, 20, 1, 64), (2, 47, 129, 3, 17), (1, 300, 80, 1, 16), (1, 531, 66, 2, 5), (2, 90, 65, 1, 32),
         (1, 130, 30, 2, 23), (3, 33, 70, 1, 33)]


def case(n, t, d, groups, states, type_, state=True, ragged=True, extras=True, seed=0):
    lens = lengths([(t * (3 * r + 1) // 4 if r % 3 else 0) % (t + 1) if n > 1 else t - t // 5 for r in range(n)]) \
        if ragged else None
    bc = rand(n, t, 2, groups, states + 1, type_=type_, seed=seed + 4)
    c = dict(x=rand(n, t, d, type_=type_, seed=seed + 1), dt=rand(n, t, d, type_=type_, seed=seed + 2),
             b=bc[:, :, 0, :, :states], c=bc[:, :, 1, :, 1:], gate=None, dt_bias=None, skip=None)
    if extras:
        c["gate"] = rand(n, t, 2 * d + 1, type_=type_, seed=seed + 3)[..., d:2 * d]
        c["dt_bias"], c["skip"] = rand(d, seed=seed + 5) - 3.0, rand(d, seed=seed + 6)
    for name in ("x", "dt", "b", "c", "gate"):
        if c[name] is not None:
            c[name] = junk(c[name], lens)
    a = -torch.exp(rand(d, states, seed=seed + 7))
    a[0, 0] = 0.0                                                            # a state that does not decay
    return c | dict(a=a, lens=lens, state=rand(n, d, states, seed=seed + 8) if state else None)


def both(c, n, t, d, states, type_, what, w, u):
    status = new_status()
    out, end = rd.rdf2v_selective_scan(**c, want_state=True, status=status)
    given = dict(c, dstate_out=u)
    g = rd.rdf2v_selective_scan_backward(dout=w, **given, status=status,
                                         out=rd.ScanGradients(*[None] * 8, dstate=torch.empty_like(end)))
    rd.check_device_status(status)
    got = dict(out=out, state=end) | {k: v for k, v in g._asdict().items() if v is not None}
    ref, sizes = refs.scan(**given, dout=w), refs.scan(**given, dout=w, absolute=True)
    check(got, ref, sizes, scan_kinds(t, states, d, n), type_, what, ("state", "dstate", "da", "ddt_bias", "dskip"))
    dead = torch.arange(t) >= (torch.full((n,), t) if c["lens"] is None else c["lens"].cpu())[:, None]
    for name in ("out", "dx", "ddt", "db", "dc"):
        assert bool((got[name].cpu()[dead] == 0).all()), name


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,t,d,groups,states", SIZES)
@pytest.mark.parametrize("ragged,state,extras", [(False, False, True), (True, True, True), (True, False, False)])
def test_against_loops(n, t, d, groups, states, type_, ragged, state, extras):
    say(f"[scan] {n} rows of {t}, {d} channels in {groups}, {states} states, {type_}, {ragged} {state} {extras}")
    c = case(n, t, d, groups, states, type_, state, ragged, extras)
    w = junk(rand(n, t, d, type_=type_, seed=20), c["lens"])
    u = rand(n, d, states, seed=21) if state else None
    both(c, n, t, d, states, type_, (n, t, d, groups, states), w, u)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d,groups,states", [(1, 1, 1), (64, 1, 16), (70, 2, 11), (12, 4, 64), (9, 1, 3)])
def test_a_step_is_a_row_of_one_token(d, groups, states, type_):
    say(f"[scan] step, {d} channels in {groups}, {states} states, {type_}")
    held, rows = 5, 7
    c = case(rows, 1, d, groups, states, type_, state=False, ragged=False)
    state, parents = rand(held, d, states, seed=4), lengths([4, 0, 0, 3, 1, 4, 2])
    one = {k: c[k][:, 0] for k in ("x", "dt", "b", "c", "gate")} | {k: c[k] for k in ("a", "dt_bias", "skip")}
    status = new_status()
    out, new = rd.rdf2v_selective_scan_step(**one, state=state, parents=parents, status=status)
    given = dict(c, state=state[parents.long()])
    check(dict(out=out[:, None], state=new), refs.scan(**given), refs.scan(**given, absolute=True),
          scan_kinds(1, states, d, rows), type_, "step", ("state",))
    rd.check_device_status(status)
    # in place; parents that there are not: zeros
    given["state"] = rand(rows, d, states, seed=5)
    mine = given["state"].clone()
    out, new = rd.rdf2v_selective_scan_step(**one, state=mine)
    assert new.data_ptr() == mine.data_ptr()
    check(dict(out=out[:, None], state=new), refs.scan(**given), refs.scan(**given, absolute=True),
          scan_kinds(1, states, d, rows), type_, "step in place", ("state",))
    parents[0], parents[3] = -1, held
    out, new = rd.rdf2v_selective_scan_step(**one, state=state, parents=parents, status=status)
    assert int(status.item()) == rd.RDF2V_STATUS_ID_OUT_OF_RANGE
    given["state"] = torch.where((parents >= 0)[:, None, None] & (parents < held)[:, None, None],
                                 state[parents.long().clamp(0, held - 1)], 0.0)
    check(dict(out=out[:, None], state=new), refs.scan(**given), refs.scan(**given, absolute=True),
          scan_kinds(1, states, d, rows), type_, "step without parents", ("state",))


@pytest.mark.parametrize("t", [40, 700])
def test_parts_of_a_row_are_the_row(t):
    """A row in two calls and in one: the same sums up to roundings."""
    say(f"[scan] a row of {t} in parts")
    c = case(1, t, 30, 1, 16, F32, state=True, ragged=False)
    whole, end = rd.rdf2v_selective_scan(**c, want_state=True)
    state, outs, at = c["state"], [], 0
    for part in (1, 2, 30, 0, t - 33):
        cut = {k: c[k][:, at:at + part] for k in ("x", "dt", "b", "c", "gate")}
        out, state = rd.rdf2v_selective_scan(**(c | cut | dict(state=state)), want_state=True)
        outs.append(out)
        at += part
    sizes = refs.scan(**c, absolute=True)
    kinds = scan_kinds(t, 16, 30, 1)
    check(dict(out=torch.cat(outs, 1), state=state), dict(out=whole.double().cpu(), state=end.double().cpu()),
          sizes, {k: 2 * v for k, v in kinds.items()}, F32, "parts")


@pytest.mark.parametrize("n,t,d", [(1, 37, 70), (1, 700, 70), (40, 37, 70)])
def test_what_is_no_number_stays_where_the_formula_has_it(n, t, d):
    say(f"[scan] NaN in {n} rows of {t}")
    groups, states, at = 2, 3, t // 2
    c = case(n, t, d, groups, states, F32, state=False, ragged=False)
    w = rand(n, t, d, seed=20)
    run = lambda **kw: (rd.rdf2v_selective_scan(**(c | kw))[0],                     # noqa: E731
                        rd.rdf2v_selective_scan_backward(dout=kw.pop("dout", w), **(c | kw)))
    clean_out, clean = run()

    def same(x, y, hit):
        assert torch.equal(x[~hit], y[~hit]) and bool(x[hit].isnan().all())

    hit = lambda *shape: torch.zeros(shape, dtype=torch.bool, device=device())     # noqa: E731
    # an input: the states after it, in its channel alone
    x = c["x"].clone()
    x[0, at, 5] = float("nan")
    out, g = run(x=x)
    h = hit(n, t, d)
    h[0, at:, 5] = True
    same(out, clean_out, h)
    h = hit(n, t, groups, states)
    h[0, at:, 0] = True
    same(g.dc, clean.dc, h)
    h = hit(n, t, groups, states)
    h[0, at, 0] = True
    same(g.db, clean.db, h)
    assert torch.equal(g.dx, clean.dx)                                              # linear in x
    # an output's gradient: the states before it
    v = w.clone()
    v[0, at, 5] = float("nan")
    g = rd.rdf2v_selective_scan_backward(dout=v, **c)
    h = hit(n, t, groups, states)
    h[0, :at + 1, 0] = True
    same(g.db, clean.db, h)
    h = hit(n, t, groups, states)
    h[0, at, 0] = True
    same(g.dc, clean.dc, h)
    h = hit(n, t, d)
    h[0, :at + 1, 5] = True
    same(g.dx, clean.dx, h)
    # an infinite c: all channels of its group
    cc = c["c"].clone()
    cc[0, at, 1, 0] = float("inf")
    out, g = run(c=cc)
    assert torch.equal(out[1:], clean_out[1:]) and torch.equal(out[0, :, :d // 2], clean_out[0, :, :d // 2])
    assert torch.equal(g.dc, clean.dc) and torch.equal(g.db[0, at + 1:], clean.db[0, at + 1:])
    assert not bool(g.db[0, :at + 1, 1, 0].isfinite().any())
    assert torch.equal(g.db[0, :, 0], clean.db[0, :, 0]) and torch.equal(g.db[0, :, 1, 1:], clean.db[0, :, 1, 1:])


def test_rates_out_of_range_lengths_and_no_rows():
    say("[scan] rates, lengths, no rows, no tokens")
    c = case(3, 6, 10, 1, 4, F32, state=True, ragged=False)
    bad = c["a"].clone()
    zero = c["a"].clone()
    for i, v in enumerate((0.5, float("nan"), float("-inf"), float("inf"))):
        bad[i, i], zero[i, i] = v, 0.0
    status = new_status()
    w = rand(3, 6, 10, seed=3)
    out = rd.rdf2v_selective_scan(**(c | dict(a=bad)), status=status)[0]
    assert int(status.item()) == rd.RDF2V_STATUS_BAD_VALUE
    assert torch.equal(out, rd.rdf2v_selective_scan(**(c | dict(a=zero)))[0])
    g, h = (rd.rdf2v_selective_scan_backward(dout=w, **(c | dict(a=a))) for a in (bad, zero))
    assert all(torch.equal(x, y) for x, y in zip(g, h))
    status.zero_()
    out = rd.rdf2v_selective_scan(**(c | dict(lens=lengths([7, -2, 6]))), status=status)[0]
    assert int(status.item()) == rd.RDF2V_STATUS_BAD_LENGTH
    assert torch.equal(out[0], rd.rdf2v_selective_scan(**c)[0][0]) and bool((out[1] == 0).all())
    for n, t in ((0, 5), (3, 0), (0, 0)):
        c = case(n, t, 10, 1, 4, F32, state=True, ragged=False)
        out, end = rd.rdf2v_selective_scan(**c, want_state=True)
        assert out.shape == (n, t, 10) and torch.equal(end, c["state"])
        u = rand(n, 10, 4, seed=5)
        g = rd.rdf2v_selective_scan_backward(dout=c["x"], dstate_out=u, **c)
        assert torch.equal(g.dstate, u)
        assert all(bool((v == 0).all()) for v in (g.da, g.ddt_bias, g.dskip))


def test_steps_of_any_size():
    """delta from 1e-30 to 100: relative precision where it is small, states forgotten where it is large."""
    say("[scan] steps of any size")
    c = case(1, 34, 64, 1, 8, F32, state=True, ragged=False)
    c["dt"] = torch.linspace(-70, 100, 34, device=device())[None, :, None].expand(1, 34, 64).contiguous()
    both(c, 1, 34, 64, 8, F32, "steps", rand(1, 34, 64, seed=3), rand(1, 64, 8, seed=4))
    c["dt"][0, 3], c["dt"][0, 20] = float("-inf"), -200.0                  # steps of 0: the tokens are not there
    out, end = rd.rdf2v_selective_scan(**c, want_state=True)
    ref = refs.scan(**(c | dict(dt=c["dt"].clamp(min=-1000.0))))
    sizes = refs.scan(**(c | dict(dt=c["dt"].clamp(min=-1000.0))), absolute=True)
    check(dict(out=out, state=end), ref, sizes, scan_kinds(34, 8, 64, 1), F32, "no step")


def test_outputs_over_inputs_are_refused():
    say("[scan] overlaps")
    c = case(2, 8, 6, 1, 4, F32, state=True, ragged=False)
    for kw in (dict(out=c["x"]), dict(out=c["dt"]), dict(state_out=c["a"].new_empty(0))):
        with pytest.raises((rd.Rdf2vError, ValueError)):
            rd.rdf2v_selective_scan(**c, **kw)
    held = c["state"].clone()
    want = rd.rdf2v_selective_scan(**c, want_state=True)[1]
    got = rd.rdf2v_selective_scan(**(c | dict(state=held)), state_out=held)[1]
    assert got.data_ptr() == held.data_ptr() and torch.equal(got, want)
    g = rd.rdf2v_selective_scan_backward(dout=c["x"], **c)
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_selective_scan_backward(dout=c["x"], **c, out=g._replace(dx=c["x"]))
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_selective_scan_backward(dout=c["x"], **c, out=g._replace(ddt=g.dx))
    u = rand(2, 6, 4, seed=9)
    want = rd.rdf2v_selective_scan_backward(dout=c["x"], dstate_out=u, **c).dstate
    got = rd.rdf2v_selective_scan_backward(dout=c["x"], dstate_out=u, **c, out=g._replace(dstate=u)).dstate
    assert got.data_ptr() == u.data_ptr() and torch.equal(got, want)
    one = {k: c[k][:, 0] for k in ("x", "dt", "b", "c", "gate")}
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_selective_scan_step(**one, a=c["a"], state=held, parents=lengths([1, 0]), state_out=held)


def test_parameters_of_more_values_than_a_launch_sums():
    """2^20 + 64 channels of 64 states: gradients of 69 million parameters, equal to those of parts of the channels."""
    say("[scan] many parameters")
    d, states = (1 << 20) + 64, 64
    gen = torch.Generator(device=device()).manual_seed(3)
    x, dt, dout = (torch.randn(2, 1, d, generator=gen, device=device()) for _ in range(3))
    b, c = (torch.randn(2, 1, 1, states, generator=gen, device=device()) for _ in range(2))
    a = -torch.rand(d, states, generator=gen, device=device())
    dt_bias, skip = (torch.randn(d, generator=gen, device=device()) for _ in range(2))
    state = torch.randn(2, d, states, generator=gen, device=device())
    got = rd.rdf2v_selective_scan_backward(x, dt, a, b, c, dout, dt_bias=dt_bias, skip=skip, state=state)
    half = d // 128 * 64
    for s in (slice(0, half), slice(half, d)):
        want = rd.rdf2v_selective_scan_backward(x[..., s], dt[..., s], a[s], b, c, dout[..., s], dt_bias=dt_bias[s],
                                                skip=skip[s], state=state[:, s].contiguous())
        for name in ("da", "ddt_bias", "dskip"):
            assert torch.equal(getattr(got, name)[s], getattr(want, name)), name


@pytest.mark.parametrize("states", [1, 3, 4, 6, 33])
def test_an_infinite_input_stays_infinite_in_a_step(states):
    """Places of a vector that hold no state add nothing, whatever the token is."""
    say(f"[scan] infinite input, {states} states")
    x = torch.full((2, 5), float("inf"), device=device())
    x[1] = 1.0
    one = torch.ones(2, 1, states, device=device())
    out, state = rd.rdf2v_selective_scan_step(x, torch.zeros_like(x), -torch.ones(5, states, device=device()), one, one,
                                              torch.zeros(2, 5, states, device=device()))
    assert bool((out[0] == float("inf")).all()) and bool((state[0] == float("inf")).all())
    assert bool(torch.isfinite(out[1]).all()) and bool(torch.isfinite(state[1]).all())


def test_without_a_skip_nothing_is_added():
    """An infinite token without a skip: infinite outputs and gradients where the formula has them, not 0 times
    infinity."""
    say("[scan] infinite input without a skip")
    x = torch.ones(2, 5, 70, device=device())
    x[0, 2] = float("inf")
    one = torch.ones(2, 5, 1, 6, device=device())
    given = (x, torch.zeros_like(x), -torch.ones(70, 6, device=device()), one, one)
    out, _ = rd.rdf2v_selective_scan(*given)
    assert bool((out[0, 2:] == float("inf")).all())
    assert bool(torch.isfinite(out[0, :2]).all()) and bool(torch.isfinite(out[1]).all())
    dout = torch.ones_like(x)
    dout[1, 3] = float("inf")
    g = rd.rdf2v_selective_scan_backward(*given, dout)
    assert bool((g.dx[1, :4] == float("inf")).all())
    assert bool(torch.isfinite(g.dx[1, 4]).all()) and bool(torch.isfinite(g.dx[0]).all())
