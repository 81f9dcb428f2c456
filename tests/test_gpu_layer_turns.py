"""The layer operators where there is more work than the chip holds at once, so that threads, waves and workgroups go
round: the second tile of a thread, the second segment of a wave, the second token of a team, and what each carries on.

Bounds of the parameters' gradients count the values that one thread adds up one after the other, and no more: what a
thread leaves is added up by a workgroup in a few steps, and in 64 bits from there. A sum over all tokens that lacks a
turn is off by ten times as much and more."""

import pytest
import torch

import layer_refs as refs
import layer_wide as wide
import paper_2508_01073_amd as rd
from gpu_helpers import new_status, say
from layer_helpers import BF16, F32, check, conv_kinds, junk, lengths, norm_kinds, rand, scan_kinds

pytestmark = pytest.mark.gpu


def _ragged(n, t):
    return lengths([(7 * r) % (t + 1) for r in range(n)])


# Gradients of rows of at most 64 tokens to a tile: 2,048 workgroups over the blocks of 64 vectors (of two channels, four
# in bfloat16), each 256 threads over the vectors of a block. 408 channels: 4 blocks of 51 vectors, 5 tiles at a time to
# 512 workgroups, 2,560 in a turn (bfloat16: 2 blocks, 5,120); 130 channels: 2 of 33, 7 to 1,024.
CONV = [(4100, 17, 408, 3, F32, True), (6100, 17, 408, 4, BF16, True), (1300, 150, 408, 4, F32, False),
        (2100, 150, 408, 2, BF16, True), (8000, 20, 130, 8, F32, True), (15000, 3, 256, 5, F32, False)]


@pytest.mark.parametrize("n,t,d,width,type_,silu", CONV)
def test_conv(n, t, d, width, type_, silu):
    say(f"[turns] convolution, {n} rows of {t}, {d} channels, width {width}, {type_}")
    lens = _ragged(n, t)
    x, w, bias = junk(rand(n, t, d, type_=type_, seed=1), lens), rand(d, width, seed=2), rand(d, seed=3)
    state, u = rand(n, width - 1, d, type_=type_, seed=4), rand(n, width - 1, d, type_=type_, seed=5)
    dout = junk(rand(n, t, d, type_=type_, seed=6), lens)
    status = new_status()
    out, end = rd.rdf2v_causal_conv(x, w, bias, silu=silu, lens=lens, state=state, want_state=True, status=status)
    dx, dw, db, ds = rd.rdf2v_causal_conv_backward(x, w, bias, dout, silu=silu, lens=lens, state=state, dstate_out=u,
                                                   status=status)
    rd.check_device_status(status)
    given = dict(x=x, weight=w, bias=bias, silu=silu, lens=lens, state=state, dout=dout, dstate_out=u)
    ref, size = ({k: v.cpu() for k, v in wide.conv(**given, absolute=absolute).items()} for absolute in (False, True))
    # a thread takes 4 tiles of 64 tokens at most, a workgroup adds up 256 threads
    kinds = conv_kinds(t, width, n)
    kinds["dweight"] = kinds["dbias"] = 2 * width + 24 + 4 * 64 + 256
    check(dict(out=out, state=end, dx=dx, dweight=dw, dbias=db, dstate=ds), ref, size, kinds, type_, (n, t, d, width),
          ("state", "dweight", "dbias"))


# Gradients: 2,048 waves over the columns (64 channels of a group at most), each with rows or segments in turn.
# rows, length, channels, groups, states, segments in a turn's wave at most, its tokens
SCAN = [(2500, 19, 65, 1, 4, 3, 24),        # 2 columns, rows whole
        (300, 19, 128, 64, 3, 10, 24),      # 64 columns, rows whole: in the forward call and the states in turn, too
        (20, 256, 128, 64, 5, 2, 88),       # rows cut into 3
        (24, 300, 128, 64, 20, 3, 80),      # into 4; the kernels for 17 to 32 states
        (24, 300, 64, 64, 40, 3, 80),       # and for more
        (3, 900, 1024, 512, 2, 3, 232),     # 512 columns, 4 waves along the segments
        (17, 900, 64, 64, 3, 5, 104)]       # rows cut into 9, in turn where their states are made, too


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,t,d,groups,states,turns,tokens", SCAN)
def test_scan(n, t, d, groups, states, turns, tokens, type_):
    say(f"[turns] scan, {n} rows of {t}, {d} channels in {groups}, {states} states, {type_}")
    lens = _ragged(n, t) if n > 3 else lengths([t, t // 2, t - 5])
    r = lambda *s, k: junk(rand(*s, type_=type_, seed=k), lens)                             # noqa: E731
    c = dict(x=r(n, t, d, k=1), dt=r(n, t, d, k=2), b=r(n, t, groups, states, k=3), c=r(n, t, groups, states, k=4),
             gate=r(n, t, d, k=5), a=-rand(d, states, seed=6).abs(), dt_bias=rand(d, seed=7) - 3.0, skip=rand(d, seed=8),
             lens=lens, state=rand(n, d, states, seed=9))
    w, u = r(n, t, d, k=10), rand(n, d, states, seed=11)
    status = new_status()
    out, end = rd.rdf2v_selective_scan(**c, want_state=True, status=status)
    g = rd.rdf2v_selective_scan_backward(dout=w, dstate_out=u, **c, status=status)
    rd.check_device_status(status)
    ref, size = (refs.scan(**c, dout=w, dstate_out=u, absolute=absolute) for absolute in (False, True))
    kinds = scan_kinds(t, states, d // groups, n)
    for name in ("da", "ddt_bias", "dskip"):
        kinds[name] = kinds["out"] + turns * tokens
    check(dict(out=out, state=end) | g._asdict(), ref, size, kinds, type_, (n, t, d, groups, states),
          ("state", "dstate", "da", "ddt_bias", "dskip"))


# Teams of 16 threads to a token, 16 teams to a workgroup, 1,536 workgroups (1,024 in the gradients) at most; of 64, four
# teams; of 256 and 1,024, one team, 1,024 and 256 workgroups in the gradients.
@pytest.mark.parametrize("n,t,d,type_,stream,drop,center,affine", [
    (60, 1201, 12, F32, F32, 0.1, True, True), (60, 1201, 12, BF16, F32, 0.0, False, False),
    (7, 2500, 260, F32, F32, 0.0, True, True), (7, 2500, 257, BF16, BF16, 0.0, False, False),
    (5, 900, 1100, F32, F32, 0.0, True, True), (3, 300, 4100, BF16, F32, 0.0, True, True),
    (3, 300, 4100, F32, F32, 0.0, False, False), (2, 300, 9000, BF16, BF16, 0.0, True, True)])
def test_norm(n, t, d, type_, stream, drop, center, affine):
    say(f"[turns] norm, {n} rows of {t}, {d} channels, {type_} {stream}, drop {drop} center {center} {affine}")
    lens = lengths([max(0, t - 3 * r) for r in range(n)])
    x, res = junk(rand(n, t, d, type_=type_, seed=1), lens), junk(rand(n, t, d, type_=stream, seed=2), lens)
    weight, bias, scale = (rand(d, seed=k) for k in (3, 4, 5))
    bias, scale = (bias, scale) if affine else (None, None)
    w, u = junk(rand(n, t, d, type_=type_, seed=6), lens), junk(rand(n, t, d, type_=stream, seed=7), lens)
    given = dict(scale=scale, drop=drop, seed=77, center=center, lens=lens, hidden_dtype=stream)
    status = new_status()
    out, hidden, stats = rd.rdf2v_residual_norm(x, res, weight, bias, **given, status=status)
    g = rd.rdf2v_residual_norm_backward(x, res, weight, bias, stats, w, dhidden=u, **given, status=status)
    rd.check_device_status(status)
    mask = refs.kept(n, t, d, drop, 77) if drop else None
    plain = dict(x=x, residual=res, weight=weight, bias=bias, scale=scale, mask=mask, drop=drop, center=center, lens=lens,
                 dout=w, dhidden=u)
    ref, size = refs.norm(**plain), refs.norm(**plain, absolute=True)
    # a team takes 5 tokens at most, a workgroup adds up 16 teams
    kinds = norm_kinds(d, 5 + 16)
    got = dict(out=out, hidden=hidden, stats=stats) | {k: v for k, v in g._asdict().items() if v is not None}
    keep32 = ("stats", "dweight", "dbias", "dscale") + (("hidden", "dresidual") if stream == F32 else ())
    check(got, ref, size, kinds, type_, (n, t, d), keep32)
