"""Distillation loss and gradient against a plain implementation in 64 bits and against differences, at
vocabularies from one token up, with absent, repeated and out-of-range teacher entries, masked logits and
padding rows."""

import math

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from model_refs import U32, UBF16, distill

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _inputs(rows, vocab, top, type_, seed):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    z = (torch.randn(rows, vocab, device=device(), generator=g) * 2.0).to(type_)
    ids = torch.randint(0, vocab, (rows, top), device=device(), generator=g, dtype=torch.int32)
    ids[torch.rand(rows, top, device=device(), generator=g) < 0.2] = -1
    if rows > 2:
        ids[1] = -1                                        # a padding row
    t = torch.randn(rows, top, device=device(), generator=g) * 2.0
    d = torch.randn(rows, device=device(), generator=g)
    return z, ids, t, d


def _bounds(z, t, tau, loss, lse, grad, dloss, type_):
    """big: the largest of a row's numbers over tau, and of its lse. Exponentials are off by 4 u and by
    their argument's 3 u big; a sum over the vocabulary by up to (sqrt vocab + 64) u in the partial sums
    that any of the kernels makes of it (at most sqrt vocab / 2 + 64 in a row per thread); lse by that and
    u big, the loss by tau^2 times all of it, p's sum to 1. A gradient is off by w (q + p) times that, and
    is rounded once."""
    vocab = z.shape[1]
    fin = lambda x: torch.where(torch.isfinite(x), x, 0.0)                        # noqa: E731
    big = (fin(z.double().cpu()).abs().amax(1) + (fin(t.double().cpu()).abs().amax(1) if t.shape[1] else 0.0)) / tau
    e = (8.0 * big + 2.0 * fin(lse).abs() + 2.0 * vocab ** 0.5 + 96.0) * U32
    w = dloss.double().cpu().abs() * tau
    q_p = 2.0 * torch.ones_like(grad) * 0.0 + fin(torch.exp(z.double().cpu() / tau - lse[:, None]))
    g = (w * e)[:, None] * (2.0 * q_p + fin(grad).abs() / w.clamp(min=1e-30)[:, None]) + 1e-30
    # where q and p cancel the sizes are those of the two
    g = g + (w * e)[:, None] * 2.0 * (q_p + (q_p - fin(grad) / w.clamp(min=1e-30)[:, None]).abs())
    if type_ == BF16:
        g = g + UBF16 * fin(grad).abs()
    return tau * tau * e * (2.0 + 0.0 * fin(loss)), e, g


def _near(x, ref, tol):
    x = x.double().cpu()
    same = (x == ref) | (torch.isnan(x) & torch.isnan(ref))
    return bool((same | ((x - ref).abs() <= tol)).all())


def _check(z, ids, t, d, tau, status=0):
    st = new_status()
    loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, temperature=tau, dloss=d, status=st)
    l1, e1 = rd.rdf2v_distill_loss(z, ids, t, temperature=tau)
    g1 = rd.rdf2v_distill_loss_backward(z, ids, t, e1, d, temperature=tau)
    torch.cuda.synchronize()
    assert int(st.item()) == status
    ref = distill(z, ids, t, tau, d.cpu())
    bl, be, bg = _bounds(z, t, tau, *ref, d, z.dtype)
    for got, gl, ge in ((grad, loss, lse), (g1, l1, e1)):
        assert _near(gl, ref[0], bl), float((gl.double().cpu() - ref[0]).abs().max())
        assert _near(ge, ref[1], be)
        assert _near(got, ref[2], bg), float((got.double().cpu() - ref[2]).abs().max())
    return loss, lse, grad


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1), (3, 2, 5), (90, 1_020, 8), (7, 1_023, 64), (33, 10_100, 32),
                                  (5, 16_385, 100), (4, 40_001, 512), (3, 65_536, 16), (2, 100_050, 7),
                                  (3, 1_000_200, 64)], ids=lambda s: "x".join(map(str, s)))
def test_against_64_bits(size, type_):
    say(f"[distill] {size} {type_}")
    for tau in (1.0, 3.0):
        _check(*_inputs(*size, type_, 5), tau)


def test_no_teacher_no_rows():
    say("[distill] no entries, no rows")
    z, ids, t, d = _inputs(3, 700, 0, F32, 1)
    loss, lse, grad = _check(z, ids, t, d, 1.0)
    assert bool((loss == 0).all()) and bool((lse == 0).all()) and bool((grad == 0).all())
    z, ids, t, d = _inputs(0, 700, 4, F32, 1)
    loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, dloss=d)
    assert loss.shape == (0,) and grad.shape == (0, 700)


@pytest.mark.parametrize("vocab", [500, 9_000, 120_000])
def test_repeated_and_bad_ids(vocab):
    say(f"[distill] repeated ids, ids out of range, entries of -inf, vocabulary of {vocab}")
    z, ids, t, d = _inputs(6, vocab, 40, F32, 2)
    ids[0] = 3
    ids[2, ::2] = ids[2, 1::2]
    ids[3, :5] = vocab
    ids[3, 5:9] = 2 ** 31 - 1
    t[4, 3:] = -math.inf
    t[5] = -math.inf                                       # every entry absent: a row without entries
    loss, _, grad = _check(z, ids, t, d, 2.0, rd.RDF2V_STATUS_ID_OUT_OF_RANGE)
    assert float(loss[5]) == 0.0 and bool((grad[5] == 0).all())


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [600, 9_000, 120_000])
def test_masked_logits(vocab, type_):
    say(f"[distill] masked logits, vocabulary of {vocab} {type_}")
    z, ids, t, d = _inputs(7, vocab, 6, type_, 3)
    z[0, ::3] = -math.inf
    ids[0] = torch.arange(1, 7, device=device()).int() * 3 - 2     # none of them masked
    z[2] = -math.inf                                       # a row of nothing: loss +inf, gradient -p
    ids[2, 0] = vocab - 1
    z[3, 5] = -math.inf
    ids[3, 2] = 5                                          # a masked token the teacher wants: loss +inf
    z[4] = torch.finfo(type_).min
    z[4, 7] = 1.0
    z[5] = torch.finfo(type_).min
    z[6, 11] = 80.0                                        # nearly all of the mass
    loss, lse, grad = _check(z, ids, t, d, 1.0)
    assert float(loss[2]) == math.inf and float(lse[2]) == -math.inf and float(loss[3]) == math.inf
    assert not bool(torch.isnan(grad).any())


def test_numbers_that_are_none():
    """NaN in a row stays in that row; it is not hidden and does not spread. A padding row's logits are
    not read."""
    say("[distill] NaN and +inf")
    for vocab in (600, 120_000):
        z, ids, t, d = _inputs(5, vocab, 6, F32, 4)
        ids[2, 0] = ids[3, 0] = 1
        ref = rd.rdf2v_distill_loss(z, ids, t, dloss=d)
        z[1] = math.nan                                    # the padding row
        z[2, vocab // 2] = math.nan
        z[3, 7] = math.inf
        loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, dloss=d)
        assert bool(torch.isnan(loss[2])) and bool(torch.isnan(grad[2]).all())
        assert not bool(torch.isfinite(loss[3])) and bool(torch.isnan(grad[3, 7]))
        for i in (0, 1, 4):
            assert torch.equal(loss[i], ref[0][i]) and torch.equal(grad[i], ref[2][i])


@pytest.mark.parametrize("vocab", [1_020, 10_100, 70_000, 200_001])
def test_strides_in_place_and_streams(vocab):
    say(f"[distill] strides, unaligned rows, in place, side stream, vocabulary of {vocab}")
    for type_ in (F32, BF16):
        z, ids, t, d = _inputs(6, vocab, 9, type_, 6)
        ref = rd.rdf2v_distill_loss(z, ids, t, dloss=d)
        for pad in (1, 8, 13):
            wide = torch.full((6, vocab + pad), math.nan, device=device(), dtype=type_)
            wide[:, :vocab] = z
            rows = torch.full((6, vocab + 3), 5.0, device=device(), dtype=type_)
            got = rd.rdf2v_distill_loss(wide[:, :vocab], ids, t, dloss=d, dlogits=rows[:, :vocab])
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
            assert bool((rows[:, vocab:] == 5.0).all())
            got = rd.rdf2v_distill_loss(wide[:, :vocab], ids, t, dloss=d, dlogits=wide[:, :vocab])
            assert torch.equal(got[2], ref[2]) and bool(torch.isnan(wide[:, vocab:]).all())
        mine = z.clone()
        rd.rdf2v_distill_loss_backward(mine, ids, t, ref[1], d, dlogits=mine)
        assert torch.equal(mine, rd.rdf2v_distill_loss_backward(z, ids, t, ref[1], d))
        side = torch.cuda.Stream(device=device())
        side.wait_stream(torch.cuda.current_stream())
        got = rd.rdf2v_distill_loss(z, ids, t, dloss=d, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("vocab", [37, 1_020, 20_000])
def test_gradient_against_differences(vocab):
    """Central differences of step h along a direction of values in [-1, 1]: the third derivative of
    tau^2 lse(z / tau) along it is tau^-1 times a third central moment of a variable in [-1, 1], at most
    2, so the truncation is at most h^2 / (3 tau); two losses' roundings are at most their bounds over h."""
    say(f"[distill] gradient against differences, vocabulary of {vocab}")
    tau, h = 2.0, 0.03
    z, ids, t, d = _inputs(16, vocab, 12, F32, 7)
    ones = torch.ones_like(d)
    loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, temperature=tau, dloss=ones)
    dirs = torch.rand_like(z) * 2 - 1
    hi, lo = z + h * dirs, z - h * dirs
    step = (hi.double() - lo.double()) / (2 * h)           # the direction as float32 took it
    a = rd.rdf2v_distill_loss(hi, ids, t, temperature=tau)[0].double()
    b = rd.rdf2v_distill_loss(lo, ids, t, temperature=tau)[0].double()
    ref = distill(z, ids, t, tau, ones.cpu())
    bl, _, bg = _bounds(z, t, tau, *ref, ones, F32)
    tol = h * h / (3 * tau) * 1.1 + 1.1 * bl / h + (bg * dirs.double().cpu().abs()).sum(1)
    off = ((a - b) / (2 * h) - (grad.double() * step).sum(1)).abs().cpu()
    assert bool((off <= tol).all()), (off.max(), tol.min())


def test_far_offsets():
    say("[distill] logits beyond 2^32 bytes")
    vocab, rows = 1_000_200, 2_200
    z = torch.zeros(rows, vocab, dtype=BF16, device=device())
    ids = torch.full((rows, 2), -1, dtype=torch.int32, device=device())
    t = torch.zeros(rows, 2, device=device())
    z[-2:] = torch.randn(2, vocab, device=device())
    ids[-2:] = torch.tensor([5, vocab - 1], dtype=torch.int32, device=device())
    d = torch.ones(rows, device=device())
    loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, dloss=d)
    small = rd.rdf2v_distill_loss(z[-2:], ids[-2:], t[-2:], dloss=d[-2:])
    assert torch.equal(loss[-2:], small[0]) and torch.equal(grad[-2:], small[2])
    assert bool((grad[:8] == 0).all()) and bool((loss[:-2] == 0).all())


def test_refusals():
    say("[distill] refusals")
    z, ids, t, d = _inputs(4, 50, 3, F32, 8)
    call = rd.rdf2v_distill_loss
    for bad in (dict(logits=z.half()), dict(logits=z.cpu()), dict(ids=ids.long()), dict(teacher=t.to(BF16)),
                dict(dloss=d.double()), dict(dloss=d, dlogits=torch.empty(4, 50, device=device(), dtype=BF16))):
        with pytest.raises(TypeError):
            call(**{**dict(logits=z, ids=ids, teacher=t), **bad})
    for bad in (dict(logits=z.T), dict(ids=ids[:3]), dict(teacher=t[:, :2]), dict(dloss=d[:2]), dict(dlogits=z),
                dict(loss=torch.empty(3, device=device()))):
        with pytest.raises(ValueError):
            call(**{**dict(logits=z, ids=ids, teacher=t), **bad})
    for tau in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(rd.Rdf2vError):
            call(z, ids, t, temperature=tau)
    wide = torch.zeros(4, 513, dtype=torch.int32, device=device())
    with pytest.raises(rd.Rdf2vError):
        call(z, wide, wide.float())
    big = torch.zeros(4, 60, device=device())
    with pytest.raises(rd.Rdf2vError):                     # overlapping, and not element by element
        call(big[:, :50], ids, t, dloss=d, dlogits=big[:, 5:55])


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("vocab", [600, 9_000, 120_000])
def test_teachers_far_from_zero(vocab, tau):
    """A teacher's distribution is that of its logits' differences, wherever they lie; entries that are all of
    the type's lowest value weigh the same. The bounds are those of logits whose largest is 0, for their
    differences are exact or rounded once."""
    say(f"[distill] teachers far from zero, vocabulary of {vocab}, temperature {tau}")
    z, ids, t, d = _inputs(8, vocab, 40, F32, 9)
    low = torch.finfo(F32).min
    for i, offset in enumerate((3.0e4, -3.0e4, 1.0e6, -1.0e6, 1.0e30, low, low, 0.0)):
        t[i] += offset
    t[6] = low
    t[7, 3:] = low                                         # three entries and masked ones
    loss, lse, grad = rd.rdf2v_distill_loss(z, ids, t, temperature=tau, dloss=d)
    alone = rd.rdf2v_distill_loss_backward(z, ids, t, rd.rdf2v_distill_loss(z, ids, t, temperature=tau)[1], d,
                                           temperature=tau)
    ref = distill(z, ids, t, tau, d.cpu())
    there = torch.where(ids >= 0, t.double(), -math.inf)
    shift = (t.double() - there.amax(1, keepdim=True)).clamp(min=-1.0e3)    # beyond, an entry weighs nothing
    bl, be, bg = _bounds(z, torch.where((ids >= 0) & (shift > -1.0e3), shift, 0.0), tau, *ref, d, F32)
    assert _near(loss, ref[0], bl), (loss.double().cpu() - ref[0]).abs() / bl
    assert _near(lse, ref[1], be)
    assert _near(grad, ref[2], bg) and _near(alone, ref[2], bg)


@pytest.mark.parametrize("vocab", [600, 9_000, 120_000])
def test_entries_of_hardly_any_weight(vocab):
    """An entry whose weight is too small for float32 adds nothing, and infinity where its token's q is 0."""
    say(f"[distill] entries of hardly any weight, vocabulary of {vocab}")
    z, ids, t, d = _inputs(6, vocab, 5, F32, 10)
    ids[:] = torch.tensor([3, 5, 7, 11, vocab - 1], dtype=torch.int32)
    t[:, 1] = -130.0                                       # exp(-130) is below float32's smallest
    t[:, 2] = -500.0
    z[1, 5] = -math.inf
    z[2, 7] = -math.inf
    z[3, 3] = -math.inf
    t[4, 2], z[4, 7] = torch.finfo(F32).min, -300.0
    z[5] = -math.inf
    loss, lse, grad = _check(z, ids, t, d, 1.0)
    assert [i for i in range(6) if float(loss[i]) == math.inf] == [1, 2, 3, 5]
    assert not bool(torch.isnan(grad).any())
    z[4, 7] = -math.inf                                    # beyond what 64 bits say: the same rule
    assert float(rd.rdf2v_distill_loss(z, ids, t)[0][4]) == math.inf
