"""The plain implementations of the layer operators against autograd in 64 bits and against differences."""

import math

import pytest
import torch

import layer_refs as refs


def _rand(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


def _differences(f, x, gradient, h=1e-6):
    """Central differences of f at x along three directions against a gradient."""
    for k in range(3):
        v = _rand(*x.shape, seed=90 + k)
        slope = (f(x + h * v) - f(x - h * v)) / (2 * h)
        along = float((gradient * v).sum())
        assert abs(slope - along) < 1e-6 * (1 + abs(along)), (slope, along)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("t,width", [(1, 1), (5, 4), (2, 8)])
def test_conv(t, width, silu):
    lens = torch.tensor([t, 0, t // 2])
    given = dict(x=_rand(3, t, 2, seed=1), weight=_rand(2, width, seed=2), bias=_rand(2, seed=3),
                 state=_rand(3, width - 1, 2, seed=4))
    w, u = _rand(3, t, 2, seed=5), _rand(3, width - 1, 2, seed=6)
    got = refs.conv(**given, silu=silu, lens=lens, dout=w, dstate_out=u)

    def loss(**kw):
        r = refs.conv(**(given | kw), silu=silu, lens=lens)
        return float((r["out"] * w).sum() + (r["state"] * u).sum())

    for name in given:
        _differences(lambda v: loss(**{name: v}), given[name], got["d" + name])
    assert bool((got["out"][1] == 0).all()) and bool((got["dx"][1] == 0).all())
    if t == 5 and silu:                                                   # one value by hand
        near = [given["state"][0, 1, 0], given["state"][0, 2, 0], given["x"][0, 0, 0], given["x"][0, 1, 0]]
        v = float(given["bias"][0] + sum(given["weight"][0, j] * near[j] for j in range(4)))
        assert abs(float(got["out"][0, 1, 0]) - v / (1 + math.exp(-v))) < 1e-12


@pytest.mark.parametrize("gated", [True, False])
def test_scan(gated):
    n, t, d, groups, states = 3, 4, 6, 2, 3
    lens = torch.tensor([4, 0, 2])
    given = dict(x=_rand(n, t, d, seed=1), dt=_rand(n, t, d, seed=2), a=-_rand(d, states, seed=3).abs(),
                 b=_rand(n, t, groups, states, seed=4), c=_rand(n, t, groups, states, seed=5), dt_bias=_rand(d, seed=6),
                 skip=_rand(d, seed=7), state=_rand(n, d, states, seed=8))
    if gated:
        given["gate"] = _rand(n, t, d, seed=9)
    w, u = _rand(n, t, d, seed=10), _rand(n, d, states, seed=11)
    got = refs.scan(**given, lens=lens, dout=w, dstate_out=u)

    def loss(**kw):
        r = refs.scan(**(given | kw), lens=lens)
        return float((r["out"] * w).sum() + (r["state"] * u).sum())

    for name in given:
        _differences(lambda v: loss(**{name: v}), given[name], got["d" + name])
    assert torch.equal(got["state"][1], given["state"][1]) and torch.equal(got["dstate"][1], u[1])


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_norm(center, drop):
    n, t, d = 3, 2, 7
    lens = torch.tensor([2, 0, 1])
    mask = refs.kept(n, t, d, drop, 77, 5) if drop else None
    given = dict(x=_rand(n, t, d, seed=1), residual=_rand(n, t, d, seed=2), weight=_rand(d, seed=3),
                 bias=_rand(d, seed=4), scale=_rand(d, seed=5))
    w, u = _rand(n, t, d, seed=6), _rand(n, t, d, seed=7)
    fixed = dict(mask=mask, drop=drop, center=center, lens=lens)
    got = refs.norm(**given, **fixed, dout=w, dhidden=u)

    def loss(**kw):
        r = refs.norm(**(given | kw), **fixed)
        return float((r["out"] * w).sum() + (r["hidden"] * u).sum())

    for name in given:
        _differences(lambda v: loss(**{name: v}), given[name], got["d" + name])


def test_the_mask_is_the_generators(rocrand_ref):
    """The words against rocRAND's generator, whose stream is the row and whose block number is channel / 4 and, 2^32
    times, token + 1; and that a row's mask is its own."""
    seed, row, tokens, channels = 0x1234567890ABCDEF, (1 << 33) + 9, 4, 10
    blocks = [(seed, row, (t + 1 << 32) + k) for t in range(tokens) for k in range(3)]
    words = rocrand_ref(4, blocks).reshape(tokens, 12)[:, :channels]
    for drop in (0.1, 0.5):
        mask = refs.kept(1, tokens, channels, drop, seed, row)
        assert torch.equal(mask[0], torch.from_numpy(words.astype("int64") >= round(drop * 2 ** 32)))
    whole, again = refs.kept(1, 4, 8, 0.5, seed, row), refs.kept(3, 6, 8, 0.5, seed, row - 1)
    assert torch.equal(whole[0], again[1, :4]) and not torch.equal(again[0], again[1])
