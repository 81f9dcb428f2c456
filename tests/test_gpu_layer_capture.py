"""The layer operators inside a HIP graph, on other streams, and at offsets beyond 32 bits. The calls only enqueue
kernels, so with outputs and workspaces of the caller they can be captured: each of three replays, with the outputs
cleared by eager work in between and other inputs in the same buffers, equals the eager run."""

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say
from layer_helpers import BF16, F32, lengths, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,length", [(40, 17), (2, 700)], ids=["short", "long"])
def test_replays_equal_the_eager_run(n, length):
    say(f"[layer capture] {n} rows of {length}")
    dev, d, states, width = device(), 70, 16, 4
    e = lambda *s, dtype=BF16: torch.empty(s, device=dev, dtype=dtype)              # noqa: E731
    x = dict(x=e(n, length, d), dt=e(n, length, d), gate=e(n, length, d), b=e(n, length, 1, states),
             c=e(n, length, 1, states), dout=e(n, length, d), near=e(n, width - 1, d), far=e(n, d, states, dtype=F32),
             residual=e(n, length, d, dtype=F32), dhidden=e(n, length, d, dtype=F32))
    weight, bias, a, one = rand(d, width, seed=1), rand(d, seed=2), -rand(d, states, seed=3).abs(), rand(d, seed=4)
    lens = lengths([(7 * r) % (length + 1) for r in range(n)])
    parents = lengths([(3 * r + 1) % n for r in range(n)])
    offset = torch.zeros(1, dtype=torch.int64, device=dev)
    work = [torch.empty(max(b, 1), dtype=torch.uint8, device=dev) for b in (
        rd.rdf2v_causal_conv_backward_workspace_size(n, length, d, width, BF16),
        rd.rdf2v_selective_scan_workspace_size(n, length, d, 1, states, BF16),
        rd.rdf2v_selective_scan_backward_workspace_size(n, length, d, 1, states, BF16),
        rd.rdf2v_residual_norm_backward_workspace_size(n, length, d, BF16, F32))]
    o = dict(conv=e(n, length, d), near=e(n, width - 1, d), cdx=e(n, length, d), cdw=e(d, width, dtype=F32),
             cdb=e(d, dtype=F32), cds=e(n, width - 1, d), cstep=e(n, d), cnext=e(n, width - 1, d), scan=e(n, length, d),
             far=e(n, d, states, dtype=F32), sstep=e(n, d), snext=e(n, d, states, dtype=F32), norm=e(n, length, d),
             hidden=e(n, length, d, dtype=F32), stats=e(n, length, 2, dtype=F32))
    sg = rd.ScanGradients(e(n, length, d), e(n, length, d), e(d, states, dtype=F32), e(n, length, 1, states),
                          e(n, length, 1, states), e(d, dtype=F32), e(d, dtype=F32), e(n, length, d),
                          e(n, d, states, dtype=F32))
    ng = rd.NormGradients(e(n, length, d), e(n, length, d, dtype=F32), e(d, dtype=F32), e(d, dtype=F32),
                          e(d, dtype=F32))
    outs = o | {"s" + k: v for k, v in sg._asdict().items()} | {"n" + k: v for k, v in ng._asdict().items()}

    def fill(seed):
        g = torch.Generator(device=dev).manual_seed(seed)
        for t in x.values():
            t.copy_(torch.randn(t.shape, device=dev, generator=g))
        offset.fill_(seed)

    def calls():
        rd.rdf2v_causal_conv(x["x"], weight, bias, lens=lens, state=x["near"], out=o["conv"], state_out=o["near"])
        rd.rdf2v_causal_conv_backward(x["x"], weight, bias, x["dout"], lens=lens, state=x["near"], dstate_out=o["near"],
                                      dx=o["cdx"], dweight=o["cdw"], dbias=o["cdb"], dstate=o["cds"], workspace=work[0])
        rd.rdf2v_causal_conv_step(x["x"][:, 0], weight, bias, o["near"], parents=parents, out=o["cstep"],
                                  state_out=o["cnext"])
        given = dict(dt_bias=bias, skip=one, gate=x["gate"])
        first = {k: v if v.dim() == 1 else v[:, 0] for k, v in given.items()}
        rd.rdf2v_selective_scan(x["x"], x["dt"], a, x["b"], x["c"], **given, lens=lens, state=x["far"], out=o["scan"],
                                state_out=o["far"], workspace=work[1])
        rd.rdf2v_selective_scan_backward(x["x"], x["dt"], a, x["b"], x["c"], x["dout"], **given, lens=lens,
                                         state=x["far"], dstate_out=o["far"], out=sg, workspace=work[2])
        rd.rdf2v_selective_scan_step(x["x"][:, 0], x["dt"][:, 0], a, x["b"][:, 0], x["c"][:, 0], o["far"], **first,
                                     parents=parents, out=o["sstep"], state_out=o["snext"])
        given = dict(scale=one, drop=0.2, seed=3, seed_offset=offset, center=True, lens=lens)
        rd.rdf2v_residual_norm(x["x"], x["residual"], one, bias, **given, out=o["norm"], hidden=o["hidden"],
                               stats=o["stats"])
        rd.rdf2v_residual_norm_backward(x["x"], x["residual"], one, bias, o["stats"], x["dout"], dhidden=x["dhidden"],
                                        **given, out=ng, workspace=work[3])

    fill(0)
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    before = None
    for seed in (1, 2, 3):
        fill(seed)
        calls()
        torch.cuda.synchronize()
        eager = {name: t.clone() for name, t in outs.items()}
        for t in outs.values():
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in outs.items():
            assert torch.equal(t, eager[name]), (seed, name)
        mask = (ng.dx == 0).clone()
        assert before is None or not torch.equal(mask, before)                     # the offset draws another mask
        before = mask


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
def test_a_captured_training_step(type_):
    """A layer forward and backward through autograd, workspaces and all its own, in a graph that is replayed."""
    say(f"[layer capture] training step {type_}")
    n, length, d, states = 30, 17, 70, 11
    leaves = [rand(n, length, d, type_=type_, seed=1), rand(n, length, d, seed=2), rand(d, seed=3),
              rand(d, 4, seed=4), -rand(d, states, seed=5).abs(), rand(n, length, 1, states, type_=type_, seed=6),
              rand(d, seed=7)]
    for t in leaves:
        t.requires_grad_()
    x, stream, weight, taps, a, b, skip = leaves
    lens = lengths([(7 * r) % (length + 1) for r in range(n)])
    offset = torch.zeros(1, dtype=torch.int64, device=device())
    dout, dstream = rand(n, length, d, type_=type_, seed=8), rand(n, length, d, seed=9)

    def step():
        y, hidden, _ = rd.rdf2v_residual_norm(x, stream, weight, drop=0.2, seed=3, seed_offset=offset, lens=lens)
        u, _ = rd.rdf2v_causal_conv(y, taps, lens=lens)
        out, _ = rd.rdf2v_selective_scan(u, y, a, b, b, skip=skip, gate=u, lens=lens)
        return (out, hidden, *torch.autograd.grad((out, hidden), leaves, (dout, dstream)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = [t.detach() for t in step()]
    for seed in (1, 2, 3):
        gen = torch.Generator(device=device()).manual_seed(seed)
        with torch.no_grad():
            for t in (x, stream, b, dout, dstream):
                t.copy_(torch.randn(t.shape, device=device(), generator=gen))
            offset.fill_(seed)
        eager = [t.detach().clone() for t in step()]
        for t in captured:
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (got, want) in enumerate(zip(captured, eager)):
            assert torch.equal(got, want), (seed, i)


def test_another_stream():
    """Calls on a stream that is not the current one, with what they allocate."""
    say("[layer capture] another stream")
    x, w = rand(30, 17, 64, seed=1), rand(64, 4, seed=2)
    a, b = -rand(64, 16, seed=3).abs(), rand(30, 17, 1, 16, seed=4)
    one = rand(64, seed=5)
    calls = (lambda **k: rd.rdf2v_causal_conv(x, w, want_state=True, **k),
             lambda **k: rd.rdf2v_causal_conv_backward(x, w, None, x, **k)[:2],
             lambda **k: rd.rdf2v_selective_scan(x, x, a, b, b, want_state=True, **k),
             lambda **k: [g for g in rd.rdf2v_selective_scan_backward(x, x, a, b, b, x, **k) if g is not None],
             lambda **k: rd.rdf2v_residual_norm(x, x, one, **k))
    want = [[t.clone() for t in call()] for call in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [[t for t in call(stream=side)] for call in calls]
    side.synchronize()
    assert all(torch.equal(p, q) for g, w_ in zip(got, want) for p, q in zip(g, w_))


def test_rows_far_apart():
    """Inputs whose second row lies more than 2^32 bytes behind the first, and outputs that are as far apart."""
    say("[layer capture] rows far apart")
    d, t = 64, 20
    far = 2 ** 31 + 4096                                                            # values of two bytes
    base = torch.empty(far + t * d, dtype=BF16, device=device())
    x = torch.as_strided(base, (2, t, d), (far, d, 1))
    x.copy_(rand(2, t, d, type_=BF16, seed=1))
    near = x.contiguous()
    w, a, one = rand(d, 4, seed=2), -rand(d, 8, seed=3).abs(), rand(d, seed=5)
    b = rand(2, t, 1, 8, type_=BF16, seed=4)
    for call in (lambda v: rd.rdf2v_causal_conv(v, w, want_state=True), lambda v: rd.rdf2v_causal_conv_backward(v, w, one, v)[:3],
                 lambda v: rd.rdf2v_selective_scan(v, v, a, b, b, gate=v, want_state=True),
                 lambda v: rd.rdf2v_selective_scan_backward(v, v, a, b, b, v, gate=v)[:5],
                 lambda v: rd.rdf2v_residual_norm(v, v, one),
                 lambda v: rd.rdf2v_causal_conv_step(v[:, 0], w, one, rand(2, 3, d, type_=BF16, seed=6)),
                 lambda v: rd.rdf2v_selective_scan_step(v[:, 0], v[:, 0], a, b[:, 0], b[:, 0], rand(2, d, 8, seed=7))):
        assert all(torch.equal(p, q) for p, q in zip(call(x), call(near)))


def test_more_than_32_bits_of_values():
    """2^31 values and more in one call: the last rows are what they are in a call of their own."""
    say("[layer capture] more than 2^31 values")
    d, t, n = 1024, 128, 2 ** 14 + 3
    x = torch.zeros(n, t, d, dtype=BF16, device=device())
    last = rand(3, t, d, type_=BF16, seed=1)
    x[-3:] = last
    w, one = rand(d, 4, seed=2), rand(d, seed=3)
    out = rd.rdf2v_causal_conv(x, w)[0]
    assert torch.equal(out[-3:], rd.rdf2v_causal_conv(last, w)[0]) and bool((out[:-3, 0] == 0).all())
    del out
    given = dict(drop=0.5, seed=1)
    out, hidden, stats = rd.rdf2v_residual_norm(x, None, one, **given)
    want = rd.rdf2v_residual_norm(last, None, one, row_begin=n - 3, **given)
    assert torch.equal(out[-3:], want[0]) and torch.equal(hidden[-3:], want[1]) and torch.equal(stats[-3:], want[2])
    del out, hidden
    a = -rand(d, 4, seed=4).abs()
    b = torch.zeros(n, t, 1, 4, dtype=BF16, device=device())
    b[-3:] = rand(3, t, 1, 4, type_=BF16, seed=5)
    out = rd.rdf2v_selective_scan(x, x, a, b, b)[0]
    few = x[-67:].contiguous(), b[-67:].contiguous()       # rows enough that none is cut into segments, as here
    assert torch.equal(out[-67:], rd.rdf2v_selective_scan(few[0], few[0], a, few[1], few[1])[0])
