"""Decay attention over rows long enough to be cut into segments, and rows whose tokens lie far apart:
lengths that end before, at and behind segments, chunks and tiles, states in and out, shared heads, odd
sizes, against the plain implementation in 64 bits."""

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from model_refs import attention_bounds
from test_gpu_decay_attention import BF16, F32, _check, _inputs, _layout, _reference, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size,layout", [((5, 700, 2, 2, 64, 64), "plain"), ((4, 1029, 3, 1, 40, 24), "odd"),
                                         ((6, 576, 2, 1, 33, 100), "plain"), ((3, 900, 1, 1, 128, 128), "slice"),
                                         ((2, 2050, 2, 2, 16, 32), "heads_first")],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else s)
def test_segments(size, layout, type_):
    say(f"[attention] segments {size} {layout} {type_}")
    x = _inputs(*size, type_, 43, False, True)
    t = size[1]
    x["lens"] = torch.tensor([t, 256, 513, 0, 1, t - 1][:size[0]], dtype=torch.int32, device=device())
    for name in ("q", "k", "v", "dout"):
        x[name][torch.arange(t, device=device()) >= x["lens"][:, None]] = float("nan")
        x[name] = _layout(x[name], layout)
    ref, sizes = _reference(x, size[4] ** -0.5)
    _check(_run(x), ref, attention_bounds(ref, sizes, type_, size[2] // size[3]), f"segments {size}")


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
def test_segments_without_states(type_):
    say(f"[attention] segments, no states given or wanted {type_}")
    size = (2, 800, 2, 1, 48, 48)
    x = _inputs(*size, type_, 47)
    ref, sizes = _reference(x, size[4] ** -0.5)
    b = attention_bounds(ref, sizes, type_, 2)
    out, state = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"])
    assert state is None
    dq, dk, dv, dstate = rd.rdf2v_decay_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"])
    assert dstate is None
    _check(dict(out=out, dq=dq, dk=dk, dv=dv), ref, b, "no states")


@pytest.mark.parametrize("length", [20, 90, 600])
def test_states_in_place(length):
    """state_out over state, and dstate over dstate_out: what is read and written are one array."""
    say(f"[attention] states in place, {length} tokens")
    for d in (32, 64):
        x = _inputs(3, length, 2, 1, d, d, F32, 53, True, True)
        a = _run(x)
        end = x["state"].clone()
        out, _ = rd.rdf2v_decay_attention(x["q"], x["k"], x["v"], x["log_decay"], lens=x["lens"], state=end,
                                          state_out=end)
        grad = x["dstate_out"].clone()
        got = rd.rdf2v_decay_attention_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], lens=x["lens"],
                                                state=x["state"], dstate_out=grad, dstate=grad)
        assert got[3] is grad
        for y, name in ((out, "out"), (end, "state"), (got[0], "dq"), (got[1], "dk"), (got[2], "dv"), (grad, "dstate")):
            assert torch.equal(y, a[name]), (d, name)


@pytest.mark.parametrize("length", [20, 70])
def test_tokens_far_apart(length):
    """Tokens 2^23 values and more apart: their places in a chunk do not fit 32 bits everywhere."""
    say(f"[attention] tokens far apart, {length} tokens")
    for step in (2 ** 23 - 8, 2 ** 23 + 8):
        x = _inputs(1, length, 1, 1, 32, 32, BF16, 59)
        y = dict(x)
        for name in ("q", "k", "v", "dout"):
            far = torch.empty((length - 1) * step + 32, device=device(), dtype=BF16)
            y[name] = far.as_strided((1, length, 1, 32), (1, step, 32, 1))
            y[name].copy_(x[name])
        ref, sizes = _reference(x, 32 ** -0.5)
        _check(_run(y), ref, attention_bounds(ref, sizes, BF16), f"step {step}")


def test_rows_at_far_offsets():
    """Rows beyond 2^32 bytes of q, k, v and out are read and written where they are."""
    say("[attention] rows beyond 2^32 bytes")
    n, t, h, d = 1030, 1024, 8, 128                        # 2.2 GB an operand in bfloat16: 2^30 values and more
    g = torch.Generator(device=device())
    g.manual_seed(61)
    q, k, v = (torch.zeros(2 * n, t, h, d, device=device(), dtype=BF16) for _ in range(3))
    for x in (q, k, v):
        x[-2:] = torch.randn(2, t, h, d, device=device(), generator=g)
    decay = torch.linspace(-1.0, -0.01, h, device=device())
    st = new_status()
    out, _ = rd.rdf2v_decay_attention(q, k, v, decay, status=st)
    small, _ = rd.rdf2v_decay_attention(q[-2:].clone(), k[-2:].clone(), v[-2:].clone(), decay)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and bool((out[:4] == 0).all())
    # the few rows are cut into segments and the many are not: equal up to the roundings of bfloat16 (once
    # for the states as operands and once for the result) of sums of 1,024 products of normal values
    size = (k[-2:].float().abs().amax() * q[-2:].float().abs().amax() * v[-2:].float().abs().amax() * d ** 0.5)
    assert float((out[-2:].float() - small.float()).abs().max()) <= 2 ** -7 * float(size)
    assert float(out[-1].float().abs().max()) > 0
