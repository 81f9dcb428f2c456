"""Decay attention (forward, gradients, single tokens) against a plain implementation in 64 bits, at
lengths around the tiles' edges, odd head sizes, shared heads, ragged rows, strided and unaligned
inputs; gradients also against differences of the forward call."""

import math

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from model_refs import U32, UBF16, attention, attention_bounds

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _layout(x, how):
    """The same values in another layout."""
    n, t, h, d = x.shape
    if how == "heads_first":
        return x.transpose(1, 2).contiguous().transpose(1, 2)
    if how == "slice":                       # one slice of a wider projection, 16-byte aligned
        wide = torch.full((n, t, h * d + 24), math.nan, device=x.device, dtype=x.dtype)
        wide[..., 8:8 + h * d] = x.flatten(2)
        return wide[..., 8:8 + h * d].unflatten(2, (h, d))
    if how == "odd":                         # no wide read is aligned
        wide = torch.full((n, t, h * d + 3), math.nan, device=x.device, dtype=x.dtype)
        wide[..., 1:1 + h * d] = x.flatten(2)
        return wide[..., 1:1 + h * d].unflatten(2, (h, d))
    return x.contiguous()


def _inputs(n, t, heads, kv, dk, dv, type_, seed, lens=False, state=False, layout="plain"):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, device=device(), generator=g)                  # noqa: E731
    q, k, v = r(n, t, heads, dk).to(type_), r(n, t, kv, dk).to(type_), r(n, t, kv, dv).to(type_)
    do = r(n, t, heads, dv).to(type_)
    x = dict(q=q, k=k, v=v, dout=do)
    x["log_decay"] = -torch.exp(r(heads) * 1.5 - 3.0)
    x["lens"] = None
    if lens:
        x["lens"] = torch.randint(0, t + 1, (n,), device=device(), generator=g, dtype=torch.int32)
        x["lens"][0], x["lens"][-1] = t, 0
        for y in (q, k, v, do):              # what lies beyond a row's length is not used, whatever it is
            y[torch.arange(t, device=device()) >= x["lens"][:, None]] = math.nan
    for name in ("q", "k", "v", "dout"):
        x[name] = _layout(x[name], layout)
    x["state"] = r(n, heads, dk, dv) if state else None
    x["dstate_out"] = r(n, heads, dk, dv) if state else None
    return x


def _clean(x):
    return {k: (torch.nan_to_num(v.float()) if k in ("q", "k", "v", "dout") and v is not None else v) for k, v in x.items()}


def _reference(x, scale):
    x = _clean(x)
    args = lambda f: dict(lens=x["lens"], **{k: None if x[k] is None else f(x[k])  # noqa: E731
                                             for k in ("state", "dout", "dstate_out")})
    same, size = (lambda y: y), torch.abs
    ref = attention(x["q"], x["k"], x["v"], x["log_decay"], scale, **args(same))
    sizes = attention(*(x[k].abs() for k in "qkv"), x["log_decay"], abs(scale), **args(size))
    return ref, sizes


def _run(x, scale=None, want_state=True):
    st = new_status()
    out, state = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], scale=scale, lens=x["lens"],
                                          state=x["state"], want_state=want_state, status=st)
    dstate = torch.empty_like(state)
    dq, dk, dv, dstate = rd.rdf2v_decay_attention_backward(
        x["q"], x["k"], x["v"], x["log_decay"], x["dout"], scale=scale, lens=x["lens"], state=x["state"],
        dstate_out=x["dstate_out"], dstate=dstate, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return dict(out=out, state=state, dq=dq, dk=dk, dv=dv, dstate=dstate)


def _check(got, ref, bounds, what):
    for name in got:
        x = got[name].double().cpu()
        assert x.shape == ref[name].shape, (what, name)
        off = (x - ref[name]).abs() - bounds[name]
        assert bool((off <= 0).all()), f"{what}: {name} is off by {float((x - ref[name]).abs().max()):.3g} " \
                                       f"({int((off > 0).sum())} values beyond the bound)"


SIZES = [  # rows, length, heads, kv_heads, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 2, 2, 1, 7, 5), (3, 17, 4, 4, 32, 32), (5, 9, 6, 3, 48, 80), (2, 63, 2, 2, 64, 64),
    (2, 64, 3, 1, 16, 128), (1, 65, 2, 2, 128, 64), (3, 33, 2, 1, 100, 33), (2, 129, 2, 2, 128, 128),
    (1, 300, 3, 3, 40, 24), (40, 16, 2, 2, 32, 16), (1, 1100, 2, 1, 64, 96), (2, 32, 1, 1, 128, 8),
]


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("ragged,state", [(False, False), (True, True)], ids=["plain", "ragged_state"])
def test_against_64_bits(size, type_, ragged, state):
    say(f"[attention] {size} {type_} ragged {ragged} state {state}")
    x = _inputs(*size, type_, 7, ragged, state)
    ref, sizes = _reference(x, size[4] ** -0.5)
    _check(_run(x), ref, attention_bounds(ref, sizes, type_, size[2] // size[3]), f"{size}")


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["heads_first", "slice", "odd"])
def test_layouts_give_the_same_bits(layout, type_):
    say(f"[attention] layout {layout} {type_}")
    for size in ((2, 70, 4, 2, 64, 48), (9, 17, 2, 2, 32, 32)):
        x = _inputs(*size, type_, 11, True, True)
        y = dict(x, **{k: _layout(x[k], layout) for k in ("q", "k", "v", "dout")})
        a, b = _run(x), _run(y)
        for name in a:
            assert torch.equal(a[name], b[name]), (size, name)


def test_broadcast_rows_and_negative_scale():
    say("[attention] keys shared by all rows through a stride of 0, negative scale")
    x = _inputs(4, 40, 2, 2, 32, 32, F32, 3)
    x["k"] = x["k"][:1].expand(4, -1, -1, -1)
    ref, sizes = _reference(x, -0.3)
    _check(_run(x, scale=-0.3), ref, attention_bounds(ref, sizes, F32), "broadcast")


def test_decays_at_their_limits():
    say("[attention] decays of 1, of 0 and in between; bad ones are reported and taken as 1")
    for length in (5, 70, 200):
        x = _inputs(2, length, 6, 6, 16, 16, F32, 5, state=True)
        x["log_decay"] = torch.tensor([0.0, -math.inf, -30.0, -1e-6, -200.0, -0.5], device=device())
        ref, sizes = _reference(x, 0.25)
        _check(_run(x), ref, attention_bounds(ref, sizes, F32), f"decays, length {length}")
        st = new_status()
        bad = torch.tensor([math.nan, 1e-3, 0.0, math.inf, 0.0, 0.0], device=device())
        out, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], bad, status=st)
        ones, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], torch.zeros_like(bad))
        assert int(st.item()) == rd.RDF2V_STATUS_BAD_VALUE and torch.equal(out, ones)


def test_no_rows_no_tokens():
    say("[attention] no rows, rows without tokens")
    d = device()
    g = torch.full((2,), -0.1, device=d)
    z = lambda *s: torch.zeros(*s, device=d)                                      # noqa: E731
    out, s = rd.rdf2v_decay_attention(z(0, 5, 2, 8), z(0, 5, 2, 8), z(0, 5, 2, 8), g, want_state=True)
    assert out.shape == (0, 5, 2, 8) and s.shape == (0, 2, 8, 8)
    state = torch.randn(3, 2, 8, 8, device=d)
    out, s = rd.rdf2v_decay_attention(z(3, 0, 2, 8), z(3, 0, 2, 8), z(3, 0, 2, 8), g, state=state, want_state=True)
    assert out.shape == (3, 0, 2, 8) and torch.equal(s, state)
    out, s = rd.rdf2v_decay_attention(z(3, 0, 2, 8), z(3, 0, 2, 8), z(3, 0, 2, 8), g, want_state=True)
    assert bool((s == 0).all())
    got = rd.rdf2v_decay_attention_backward(z(3, 0, 2, 8), z(3, 0, 2, 8), z(3, 0, 2, 8), g, z(3, 0, 2, 8),
                                            state=state, dstate_out=state)
    assert torch.equal(got[3], state)


def test_state_in_place_and_pieces():
    """A row in two pieces, the state carried in place, gives what the whole row gives."""
    say("[attention] pieces with the state in place")
    x = _inputs(2, 150, 2, 2, 64, 64, F32, 9)
    ref, sizes = _reference(x, 0.125)
    bounds = attention_bounds(ref, sizes, F32)
    state = torch.zeros(2, 2, 64, 64, device=device())
    outs = []
    for lo, hi in ((0, 64), (64, 65), (65, 150)):
        o, s = rd.rdf2v_decay_attention(x["q"][:, lo:hi], x["k"][:, lo:hi], x["v"][:, lo:hi], x["log_decay"],
                                        state=state, state_out=state)
        assert s is state
        outs.append(o)
    _check({"out": torch.cat(outs, 1), "state": state}, ref, bounds, "pieces")


def test_lengths_out_of_range():
    say("[attention] lengths out of range are reported and clamped")
    x = _inputs(3, 20, 2, 2, 16, 16, F32, 13)
    st = new_status()
    bad = torch.tensor([-4, 20, 99], dtype=torch.int32, device=device())
    good = torch.tensor([0, 20, 20], dtype=torch.int32, device=device())
    a, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], lens=bad, status=st)
    b, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], lens=good)
    assert torch.equal(a, b) and int(st.item()) == rd.RDF2V_STATUS_BAD_LENGTH


@pytest.mark.parametrize("size", [(2, 50, 2, 1, 24, 40), (1, 130, 2, 2, 64, 64)], ids=["small", "long"])
def test_gradients_against_differences(size):
    """The loss sum(out * dout) + sum(state * dstate_out) is linear in each input alone, so a central
    difference of any step has no truncation error: with a direction d of the step, half of
    loss(x + d) - loss(x - d) is the gradient's product with d, up to the roundings of the two calls,
    which the bounds of the outputs at |x| + |d| sum to."""
    say(f"[attention] gradients against differences, {size}")
    x = _inputs(*size, F32, 17, True, True)
    got = _run(x)
    scale = size[4] ** -0.5

    def loss(y):
        out, state = rd.rdf2v_decay_attention(y["q"], y["k"], y["v"], y["log_decay"], lens=y["lens"],
                                              state=y["state"], want_state=True)
        live = torch.arange(size[1], device=device()) < y["lens"][:, None]
        do = torch.where(live[..., None, None], y["dout"].double(), 0.0)
        return float((out.double() * do).sum() + (state.double() * y["dstate_out"].double()).sum())

    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("state", "dstate")):
        d = torch.randn_like(x[name].contiguous())
        diff = (loss(dict(x, **{name: x[name] + d})) - loss(dict(x, **{name: x[name] - d}))) / 2
        live = torch.nan_to_num(got[grad].double()) * torch.where(torch.isnan(x[name]), 0.0, 1.0) * d.double()
        wide = dict(x, **{name: x[name].abs() + d.abs()})
        ref, sizes = _reference(wide, scale)
        b = attention_bounds(ref, sizes, F32, size[2] // size[3])
        clean = _clean(x)
        tol = float((b["out"] * clean["dout"].double().cpu().abs()).sum()
                    + (b["state"] * x["dstate_out"].double().cpu().abs()).sum()
                    + (b[grad] * d.double().cpu().abs()).sum())
        assert abs(diff - float(live.sum())) <= tol, (name, diff, float(live.sum()), tol)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 4, 4, 64, 64), (5, 6, 2, 33, 70), (64, 2, 2, 128, 128), (300, 1, 1, 8, 4),
                                  (3, 2, 1, 128, 1), (7, 3, 3, 1, 128)], ids=lambda s: "x".join(map(str, s)))
def test_step(size, type_):
    """One token: with and without parents, in place and out of place."""
    n, heads, kv, dk, dv = size
    say(f"[attention step] {size} {type_}")
    x = _inputs(n, 1, heads, kv, dk, dv, type_, 19, state=True)
    q, k, v = (x[y][:, 0] for y in "qkv")
    g = torch.Generator().manual_seed(1)
    parents = torch.randint(0, n, (n,), generator=g, dtype=torch.int32).to(device())
    for p in (None, parents):
        s0 = x["state"] if p is None else x["state"][p.long()]
        ref, sizes = _reference(dict(x, state=s0, dout=None), dk ** -0.5)
        b = attention_bounds(ref, sizes, type_)
        st = new_status()
        out, state = rd.rdf2v_decay_attention_step(q, k, v, x["log_decay"], x["state"], parents=p,
                                                   state_out=torch.empty_like(x["state"]), status=st)
        _check({"out": out[:, None], "state": state}, ref, b, f"step {size}")
        assert int(st.item()) == 0
        if p is None:
            mine = x["state"].clone()
            o2, s2 = rd.rdf2v_decay_attention_step(q, k, v, x["log_decay"], mine)
            assert s2 is mine and torch.equal(o2, out) and torch.equal(mine, state)


def test_step_parents_elsewhere():
    say("[attention step] more rows than states, parents out of range")
    x = _inputs(6, 1, 2, 2, 32, 32, F32, 23)
    state = torch.randn(2, 2, 32, 32, device=device())
    parents = torch.tensor([0, 1, 1, -1, 2, 0], dtype=torch.int32, device=device())
    st = new_status()
    q, k, v = (x[y][:, 0] for y in "qkv")
    out, new = rd.rdf2v_decay_attention_step(q, k, v, x["log_decay"], state, parents=parents, status=st)
    assert int(st.item()) == rd.RDF2V_STATUS_ID_OUT_OF_RANGE
    start = torch.cat([state, torch.zeros(1, 2, 32, 32, device=device())])[[0, 1, 1, 2, 2, 0]]
    ref, sizes = _reference(dict(x, state=start, dout=None), 32 ** -0.5)
    _check({"out": out[:, None], "state": new}, ref, attention_bounds(ref, sizes, F32), "parents")


def test_step_continues_rows():
    say("[attention step] tokens one by one give what the whole row gives")
    x = _inputs(3, 40, 4, 2, 64, 32, BF16, 29)
    ref, sizes = _reference(x, 0.125)
    state = torch.zeros(3, 4, 64, 32, device=device())
    outs = [rd.rdf2v_decay_attention_step(x["q"][:, i], x["k"][:, i], x["v"][:, i], x["log_decay"], state)[0]
            for i in range(40)]
    _check({"out": torch.stack(outs, 1), "state": state}, ref, attention_bounds(ref, sizes, BF16), "tokens")


def test_states_at_far_offsets():
    """A cache of states of more than 2^32 bytes and 2^31 values: the last rows are read and written."""
    say("[attention step] states beyond 2^31 values")
    n = 2 ** 31 // (8 * 128 * 128) + 3
    state = torch.zeros(n, 8, 128, 128, device=device())
    state[-2:] = torch.randn(2, 8, 128, 128, device=device())
    last = state[-2:].clone()
    x = _inputs(2, 1, 8, 8, 128, 128, F32, 31)
    parents = torch.tensor([n - 2, n - 1], dtype=torch.int32, device=device())
    q, k, v = (x[y][:, 0] for y in "qkv")
    out, new = rd.rdf2v_decay_attention_step(q, k, v, x["log_decay"], state, parents=parents)
    o2, s2 = rd.rdf2v_decay_attention_step(q, k, v, x["log_decay"], last.clone())
    assert torch.equal(out, o2) and torch.equal(new, s2)
    # and written there, in place
    big = lambda y: y.expand(n, -1, -1)                                           # noqa: E731
    rd.rdf2v_decay_attention_step(big(q[1:]), big(k[1:]), big(v[1:]), x["log_decay"], state)
    assert torch.equal(state[-1], s2[1])


def test_on_a_side_stream_and_repeated():
    """On another stream behind queued work, and twice: the same bits."""
    say("[attention] side stream, repeated calls")
    x = _inputs(2, 500, 4, 2, 64, 64, BF16, 37, True, True)
    a = _run(x)
    side = torch.cuda.Stream(device=device())
    side.wait_stream(torch.cuda.current_stream())
    out, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], lens=x["lens"], state=x["state"],
                                      stream=side)
    got = rd.rdf2v_decay_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], lens=x["lens"],
                                            state=x["state"], dstate_out=x["dstate_out"], stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, a["out"])
    for y, name in zip(got, ("dq", "dk", "dv", "dstate")):
        assert torch.equal(y, a[name]), name


def test_refusals():
    say("[attention] refusals")
    x = _inputs(2, 8, 4, 2, 16, 16, F32, 41, state=True)
    q, k, v, g = x["q"], x["k"], x["v"], x["log_decay"]
    call = rd.rdf2v_decay_attention
    for bad in (dict(q=q.cpu()), dict(q=q.half()), dict(k=k.to(BF16)), dict(lens=torch.zeros(2, device=device())),
                dict(state=x["state"].double())):
        with pytest.raises(TypeError):
            a = dict(q=q, k=k, v=v, log_decay=g, **{n: b for n, b in bad.items() if n not in "qkv"})
            a.update({n: b for n, b in bad.items() if n in "qkv"})
            call(**a)
    for bad in (dict(q=q[:, :7]), dict(k=k[..., :15]), dict(v=v.transpose(-1, -2)), dict(log_decay=g[:3]),
                dict(q=q[:, :, :3]), dict(lens=torch.zeros(3, dtype=torch.int32, device=device())),
                dict(state=x["state"][..., :8]), dict(state_out=x["state"][:1]),
                dict(out=torch.empty(2, 8, 4, 17, device=device()))):
        with pytest.raises(ValueError):
            call(**{**dict(q=q, k=k, v=v, log_decay=g), **bad})
    wide = torch.zeros(1, 2, 1, 129, device=device())
    with pytest.raises(ValueError):
        call(wide, wide, wide, g[:1])
    with pytest.raises(rd.Rdf2vError):
        call(q, k, v, g, scale=math.inf)
    state = x["state"]
    parents = torch.zeros(2, dtype=torch.int32, device=device())
    with pytest.raises(rd.Rdf2vError):       # a parent's state may be overwritten before it is read
        rd.rdf2v_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], g, state, parents=parents, state_out=state)
    with pytest.raises(ValueError):
        rd.rdf2v_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], g, state[:1])
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_decay_attention_backward(q, k, v, g, x["dout"],
                                          workspace=torch.empty(16, dtype=torch.uint8, device=device()))


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 33, 4, 2, 48, 64), (5, 48, 2, 2, 64, 33), (300, 16, 6, 2, 40, 20),
                                  (9, 47, 3, 1, 52, 36)], ids=lambda s: "x".join(map(str, s)))
def test_short_rows_with_states(size, type_):
    say(f"[attention] short rows with states {size} {type_}")
    x = _inputs(*size, type_, 17, True, True)
    ref, sizes = _reference(x, size[4] ** -0.5)
    _check(_run(x), ref, attention_bounds(ref, sizes, type_, size[2] // size[3]), f"{size}")


def test_gradients_of_shared_heads_beyond_a_row():
    """Zeros for tokens beyond a row's length, whatever the outputs and the workspace hold."""
    say("[attention] shared heads' gradients of the padding")
    for length, type_ in ((20, F32), (20, BF16), (150, F32), (150, BF16)):
        x = _inputs(7, length, 6, 2, 24, 20, type_, 23, True)
        ws = torch.full((rd.rdf2v_decay_attention_backward_workspace_size(7, length, 6, 2, 24, 20, type_),), 255,
                        dtype=torch.uint8, device=device())
        outs = dict(dq=torch.full_like(x["q"], math.nan), dk=torch.full_like(x["k"], math.nan),
                    dv=torch.full_like(x["v"], math.nan))
        args = (x["q"], x["k"], x["v"], x["log_decay"], x["dout"])
        rd.rdf2v_decay_attention_backward(*args, lens=x["lens"], workspace=ws, **outs)
        ref = rd.rdf2v_decay_attention_backward(*args, lens=x["lens"])
        beyond = torch.arange(length, device=device()) >= x["lens"][:, None]
        for name, want in zip(("dq", "dk", "dv"), ref):
            assert torch.equal(outs[name], want) and bool((outs[name][beyond] == 0).all()), (length, type_, name)


@pytest.mark.parametrize("size", [(4, 1, 2, 2, 32, 32), (2, 1, 2, 1, 64, 128), (3, 40, 2, 2, 32, 16),
                                  (2, 70, 2, 1, 64, 64), (1, 700, 2, 2, 128, 128)],
                         ids=lambda s: "x".join(map(str, s)))
def test_states_that_cancel_in_bfloat16(size):
    """States of 100 and a little, and tokens whose neighbouring values cancel: what is left of a state's
    product is the little. States, and the weights of pairs, are operands of 16 bits (2^-16 each, of terms
    that are disjoint), and a state may also be a sum of such terms: 2^-15 of the terms' absolute values,
    beside float32's roundings and the result's own to bfloat16."""
    say(f"[attention] states that cancel {size}")
    x = _inputs(*size, BF16, 67, False, True)
    for name in ("q", "k", "v", "dout"):
        y = x[name].unflatten(-1, (-1, 2))
        x[name] = torch.stack((y[..., 0], -y[..., 0]), -1).flatten(-2)
    for name in ("state", "dstate_out"):
        x[name] = x[name] + 100.0
    x["log_decay"] = x["log_decay"] * 0.01
    ref, sizes = _reference(x, size[4] ** -0.5)
    b = attention_bounds(ref, sizes, F32, size[2] // size[3])
    for name in b:
        if "state" not in name:
            b[name] = b[name] + 1.01 * 2.0 ** -15 * sizes[name] + 1.01 * UBF16 * ref[name].abs()
    _check(_run(x), ref, b, f"cancel {size}")


def test_outputs_between_an_inputs_rows():
    """An output that lies between the rows of an input shares nothing with it."""
    say("[attention] outputs between the rows of an input")
    x = _inputs(2, 20, 2, 2, 16, 16, F32, 71)
    a, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"])
    whole = torch.full((4096,), math.nan, device=device())
    q = whole.as_strided((2, 20, 2, 16), (2048, 32, 16, 1))            # 640 values at 0 and at 2048
    q.copy_(x["q"])
    out = whole[640:640 + 1280].view(2, 20, 2, 16)
    got, _ = rd.rdf2v_decay_attention(q, x["k"], x["v"], x["log_decay"], out=out)
    assert got is out and torch.equal(out, a) and torch.equal(q, x["q"])
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_decay_attention(q, x["k"], x["v"], x["log_decay"], out=whole[800:800 + 1280].view(2, 20, 2, 16))
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], out=x["v"])
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_decay_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], dk=x["k"])


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 12, 2, 1, 16, 24), (2, 31, 2, 2, 40, 33), (1, 48, 4, 2, 32, 64), (2, 70, 2, 1, 64, 20),
                                  (1, 130, 2, 2, 128, 128), (1, 200, 1, 1, 24, 64), (1, 700, 2, 1, 64, 64)],
                         ids=lambda s: "x".join(map(str, s)))
def test_no_numbers_stay_where_the_formula_has_them(size, type_):
    """A NaN or an infinity in a token: what the formula makes no number of it is none, and all the rest is
    what it is with a zero there: earlier tokens' outputs, later tokens' gradients, other columns. The same
    bits, or within the bounds where a short row's columns are done again."""
    n, t, heads, kv, dk, dv = size
    say(f"[attention] no numbers {size} {type_}")
    for state in (False, True):
        x = _inputs(*size, type_, 73, False, state)
        places = sorted({0, t // 2, t - 1, min(63, t - 1), min(64, t - 1), min(17, t - 1)})
        for i, name in enumerate(("q", "k", "v", "dout")):
            for place in places:
                for bad in (math.nan, math.inf) if place == t // 2 else ((math.nan, -math.inf)[place % 2],):
                    y, z = dict(x), dict(x)
                    y[name], z[name] = x[name].clone(), x[name].clone()
                    at = (n - 1, place, (place + i) % x[name].shape[2], (3 * place + i) % x[name].shape[3])
                    y[name][at], z[name][at] = bad, 0.0
                    a, b = _run(y), _run(z)
                    ref = attention(y["q"], y["k"], y["v"], y["log_decay"], dk ** -0.5, state=y["state"],
                                    dout=y["dout"], dstate_out=y["dstate_out"])
                    near = {out: a[out].cpu() == b[out].cpu() for out in a}
                    if t <= 48:
                        clean, sizes = _reference(z, dk ** -0.5)
                        bounds = attention_bounds(clean, sizes, type_, heads // kv)
                        near = {out: x | ((a[out].cpu() - clean[out]).abs() <= bounds[out]) for out, x in near.items()}
                    for out in a:
                        none = ~torch.isfinite(ref[out])
                        assert torch.equal(~torch.isfinite(a[out]).cpu(), none), (name, place, bad, out)
                        assert bool(near[out][~none].all()), (name, place, bad, out)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(256, 17, 4, 4, 32, 32), (350, 9, 6, 2, 20, 31), (130, 33, 8, 4, 32, 16),
                                  (270, 48, 8, 8, 64, 40), (520, 20, 4, 2, 33, 64)], ids=lambda s: "x".join(map(str, s)))
def test_many_short_rows_with_states(size, type_):
    """As many rows as a wave each is taken for with states; the states also in place; and no numbers."""
    say(f"[attention] many short rows with states {size} {type_}")
    x = _inputs(*size, type_, 79, True, True)
    ref, sizes = _reference(x, size[4] ** -0.5)
    bounds = attention_bounds(ref, sizes, type_, size[2] // size[3])
    got = _run(x)
    _check(got, ref, bounds, f"{size}")
    end, grad = x["state"].clone(), x["dstate_out"].clone()
    out, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], lens=x["lens"], state=end, state_out=end)
    grads = rd.rdf2v_decay_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], lens=x["lens"],
                                              state=x["state"], dstate_out=grad, dstate=grad)
    for y, name in zip((out, end, *grads), ("out", "state", "dq", "dk", "dv", "dstate")):
        assert torch.equal(y, got[name]), name
    place = size[1] // 2
    for name in ("q", "k", "v", "dout"):
        y = dict(x, **{name: x[name].clone()})
        y[name][0, place, -1, 3] = math.nan                # the first row has all of its tokens
        a = _run(y)
        none = attention(*(y[n][:1] for n in "qkv"), y["log_decay"], size[4] ** -0.5, state=y["state"][:1],
                         dout=y["dout"][:1], dstate_out=y["dstate_out"][:1])
        for out in a:
            assert torch.equal(a[out][1:], got[out][1:]), (name, out)
            bad = ~torch.isfinite(none[out][0])
            assert torch.equal(~torch.isfinite(a[out][0]).cpu(), bad), (name, out)
            assert bool(((a[out][0].cpu() - ref[out][0]).abs() <= bounds[out][0])[~bad].all()), (name, out)
