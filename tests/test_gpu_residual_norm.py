"""Residual norm on the GPU against a plain 64-bit implementation: outputs, dropout's mask, gradients."""

import pytest
import torch

import layer_refs as refs
import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from layer_helpers import BF16, F32, check, junk, lengths, norm_kinds, rand

pytestmark = pytest.mark.gpu

TYPES = [(F32, F32), (BF16, F32), (BF16, BF16)]
IDS = ["f32", "bf16-f32", "bf16"]


def _run(n, t, d, type_, stream, drop, center, affine, ragged, residual=True, seed=0):
    lens = lengths([(t * (3 * r + 1) // 4 if r % 3 else 0) % (t + 1) if n > 1 else t - t // 5 for r in range(n)]) \
        if ragged else None
    x = junk(rand(n, t, d + 3, type_=type_, seed=seed + 1)[..., 2:-1], lens)
    res = junk(rand(n, t, 2 * d, type_=stream, seed=seed + 2)[..., d:], lens) if residual else None
    weight, bias, scale = (rand(d, seed=seed + k) for k in (3, 4, 5))
    bias, scale = (bias, scale) if affine else (None, None)
    w, u = junk(rand(n, t, d, type_=type_, seed=seed + 6), lens), junk(rand(n, t, d, type_=stream, seed=seed + 7), lens)
    key, row = 0x9E3779B97F4A7C15 * (seed + 3) % 2 ** 64, 2 ** 35 + 7
    offset = torch.tensor([12345], dtype=torch.int64, device=device())
    given = dict(scale=scale, drop=drop, seed=key - 12345, seed_offset=offset, row_begin=row, center=center, eps=1e-3,
                 lens=lens, hidden_dtype=stream)
    status = new_status()
    out, hidden, stats = rd.rdf2v_residual_norm(x, res, weight, bias, **given, status=status)
    g = rd.rdf2v_residual_norm_backward(x, res, weight, bias, stats, w, dhidden=u, **given, status=status)
    rd.check_device_status(status)
    assert hidden.dtype == stream and g.dx.dtype == type_ and (g.dresidual is None) == (not residual)
    mask = refs.kept(n, t, d, drop, key, row) if drop else None
    plain = dict(x=x, residual=res, weight=weight, bias=bias, scale=scale, mask=mask, drop=drop, center=center,
                 eps=1e-3, lens=lens, dout=w, dhidden=u)
    ref, sizes = refs.norm(**plain), refs.norm(**plain, absolute=True)
    got = dict(out=out, hidden=hidden, stats=stats) | {k: v for k, v in g._asdict().items() if v is not None}
    keep32 = ("stats", "dweight", "dbias", "dscale") + (("hidden", "dresidual") if stream == F32 else ())
    check(got, ref, sizes, norm_kinds(d, n * t), type_, (n, t, d, drop, center, affine), keep32)
    dead = torch.arange(t) >= (torch.full((n,), t) if lens is None else lens.cpu())[:, None]
    for name in ("out", "hidden", "dx") + (("dresidual",) if residual else ()):
        assert bool((got[name].cpu()[dead] == 0).all()), name
    if drop:
        live = ~dead[..., None] & (ref["dx"] != 0)
        assert torch.equal((g.dx.cpu() != 0) & live, mask & live)


@pytest.mark.parametrize("type_,stream", TYPES, ids=IDS)
@pytest.mark.parametrize("n,t,d", [(1, 1, 1), (2, 3, 4), (3, 5, 63), (4, 7, 66), (2, 9, 256), (3, 4, 301), (2, 3, 1000)])
@pytest.mark.parametrize("drop,center,affine,ragged", [(0.0, False, False, False), (0.3, True, True, True),
                                                       (0.1, False, True, False), (0.0, True, False, True)])
def test_against_plain(n, t, d, type_, stream, drop, center, affine, ragged):
    say(f"[norm] {n} rows of {t}, {d} channels, {type_} {stream}, drop {drop} center {center} {affine} {ragged}")
    _run(n, t, d, type_, stream, drop, center, affine, ragged)


@pytest.mark.parametrize("type_,stream", TYPES, ids=IDS)
@pytest.mark.parametrize("d", [1025, 2048, 4095, 8000, 16384])
def test_wide_tokens(d, type_, stream):
    say(f"[norm] {d} channels, {type_} {stream}")
    _run(2, 2, d, type_, stream, 0.5, True, True, True, seed=3)
    _run(1, 3, d, type_, stream, 0.0, False, False, False, residual=False, seed=4)


def test_many_tokens():
    say("[norm] more tokens than workgroups")
    _run(5, 1201, 12, F32, F32, 0.0, True, True, True, seed=5)
    _run(2, 1100, 260, BF16, F32, 0.0, False, True, True, seed=6)


def test_a_mask_is_a_function_of_the_row():
    """Parts of a batch, other lengths and single tokens drop what the whole batch drops."""
    say("[norm] masks of parts")
    n, t, d = 5, 6, 37
    x, w = rand(n, t, d, seed=1).abs() + 1, torch.ones(d, device=device())
    run = lambda x, **kw: rd.rdf2v_residual_norm(x, None, w, drop=0.4, seed=11, **kw)[1]     # noqa: E731
    whole = run(x, row_begin=100)
    assert torch.equal(run(x[2:].contiguous(), row_begin=102), whole[2:])
    assert torch.equal(run(x[:, :3].contiguous(), row_begin=100), whole[:, :3])
    assert torch.equal(run(x[:, 0], row_begin=100), whole[:, 0])                             # [rows, channels]
    assert torch.equal(run(x, row_begin=100, seed_offset=torch.zeros(1, dtype=torch.int64, device=device())), whole)
    other = run(x, row_begin=100, seed_offset=torch.ones(1, dtype=torch.int64, device=device()))
    assert not torch.equal(other, whole)
    assert torch.equal(other, rd.rdf2v_residual_norm(x, None, w, drop=0.4, seed=12, row_begin=100)[1])
    # what is dropped counts as 0 whatever it holds
    bad = torch.where(whole == 0, float("nan"), x)
    assert torch.equal(run(bad, row_begin=100), whole)


def test_large_means_and_small_variances():
    """The mean is taken off before squares are summed."""
    say("[norm] a large mean")
    x = rand(2, 3, 512, seed=1) + 1000.0
    w = torch.ones(512, device=device())
    out = rd.rdf2v_residual_norm(x, None, w, center=True)[0]
    ref = torch.nn.functional.layer_norm(x.double(), (512,), eps=1e-5)
    # a value of 1000 is known to 2^-15, the mean to as much
    assert float((out - ref).abs().max()) < 2.0 ** -14 * 4


def test_what_is_no_number_stays_in_its_token():
    say("[norm] NaN")
    for d in (12, 100, 1500):
        x, res, w = rand(3, 4, d, seed=1), rand(3, 4, d, seed=2), rand(d, seed=3)
        clean = rd.rdf2v_residual_norm(x, res, w, center=True)
        x[1, 2, 5] = float("inf")
        got = rd.rdf2v_residual_norm(x, res, w, center=True)
        for a, b in zip(clean, got):
            hit = torch.zeros_like(a, dtype=torch.bool)
            hit[1, 2] = True
            assert torch.equal(a[~hit], b[~hit])
        assert bool(got[0][1, 2].isnan().all()) and int((~got[1].isfinite()).sum()) == 1


def test_lengths_out_of_range_no_rows_and_overlaps():
    say("[norm] lengths, no rows, no tokens, overlaps")
    x, w = rand(3, 4, 6, seed=1), rand(6, seed=2)
    status = new_status()
    out = rd.rdf2v_residual_norm(x, None, w, lens=lengths([5, -1, 4]), status=status)[0]
    assert int(status.item()) == rd.RDF2V_STATUS_BAD_LENGTH
    assert torch.equal(out[0], rd.rdf2v_residual_norm(x, None, w)[0][0]) and bool((out[1] == 0).all())
    for shape in ((0, 5, 6), (3, 0, 6), (0, 6)):
        e = x.new_empty(shape)
        out, hidden, stats = rd.rdf2v_residual_norm(e, e.clone(), w)
        assert out.shape == shape and stats.shape == (*shape[:-1], 2)
        g = rd.rdf2v_residual_norm_backward(e, e.clone(), w, w, stats, e, scale=w)
        assert all(bool((v == 0).all()) for v in (g.dweight, g.dbias, g.dscale))
    for kw in (dict(out=x), dict(hidden=x)):
        with pytest.raises(rd.Rdf2vError):
            rd.rdf2v_residual_norm(x, None, w, **kw)
    y = torch.empty_like(x)
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_residual_norm(x, None, w, out=y, hidden=y)
