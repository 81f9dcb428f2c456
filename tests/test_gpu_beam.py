"""Beam selection and reordering against plain implementations: totals in 64 bits, places by a stable
order where totals are exact, masks, ties, finished and dead beams."""

import math

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, new_status, say
from model_refs import U32, beam_select

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _inputs(groups, beams, vocab, type_, seed, spread=2.0):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    logits = (torch.randn(groups, beams, vocab, device=device(), generator=g) * spread).to(type_)
    scores = torch.rand(groups, beams, device=device(), generator=g) * -6.0
    return logits, scores


def _check(logits, scores, num_out, finished=None, status=0, vocab=None):
    """A total is a sum in float32 of three numbers no larger than `big`, one of them lse, whose sum of
    exponentials is off by up to (sqrt vocab + 64) u in the partial sums that the work is split into, and
    by 4 u for exp and u big for its argument: (8 big + sqrt vocab + 64) u together. The k-th best total
    in 64 bits is that near to the k-th written, and so is the total of the place written."""
    st = new_status()
    got, tokens, parents = rd.rdf2v_beam_select(logits, scores, num_out, finished=finished, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == status
    groups, beams, v = logits.shape
    best, total = beam_select(logits, scores, num_out, finished)
    got, tokens, parents = got.double().cpu(), tokens.cpu().long(), parents.cpu().long()
    most = lambda x: float(x[torch.isfinite(x)].abs().max()) if bool(torch.isfinite(x).any()) else 0.0  # noqa: E731
    big = most(logits.double()) * 2 + math.log(v) + most(scores)
    tol = (8 * big + v ** 0.5 + 64) * U32
    dead = best == -math.inf
    assert torch.equal(got == -math.inf, dead)
    assert bool(((got - best).abs()[~dead] <= tol).all())
    first = torch.arange(groups)[:, None] * beams
    assert torch.equal(parents[dead], first.expand_as(parents)[dead]) and bool((tokens[dead] == -1).all())
    beam = parents - first
    assert bool(((beam >= 0) & (beam < beams)).all())
    end = torch.zeros(groups, beams, dtype=torch.bool) if finished is None else finished.cpu() != 0
    is_end = end.gather(1, beam)
    assert torch.equal((tokens == -1) & ~dead, is_end & ~dead)
    place = beam * v + tokens.clamp(min=0)
    own = total.gather(1, place)                 # the chosen places' totals are the totals written
    assert bool(((own - got).abs()[~dead] <= tol).all())
    for row, no in zip(place, dead):             # and no place is chosen twice
        assert len(set(row[~no].tolist())) == int((~no).sum())
    # descending; equal totals in ascending order of place
    a, b = got[:, :-1], got[:, 1:]
    assert bool((a >= b).all())
    tie = (a == b) & ~dead[:, 1:]
    assert bool((place[:, :-1] < place[:, 1:])[tie].all())
    return got, tokens, parents


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 4, 1_020, 4), (3, 2, 5, 64), (2, 64, 333, 64), (5, 8, 4_097, 8),
                                  (2, 3, 100_050, 7), (1, 1, 250_001, 50), (33, 5, 1_023, 16), (1, 16, 16_384, 1),
                                  (2, 1, 65_537, 64), (1, 8, 1_000_200, 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_against_64_bits(size, type_):
    groups, beams, vocab, num_out = size
    say(f"[beam] {size} {type_}")
    logits, scores = _inputs(groups, beams, vocab, type_, 3)
    _check(logits, scores, num_out)
    torch.manual_seed(vocab)
    finished = (torch.rand(groups, beams, device=device()) < 0.3).int()
    scores[:, -1] = -math.inf
    logits[:, :, vocab // 2:][torch.rand(groups, beams, vocab - vocab // 2, device=device()) < 0.5] = -math.inf
    _check(logits, scores, num_out, finished)


@pytest.mark.parametrize("vocab", [7, 1_020, 40_000, 300_000])
def test_places_by_order_where_totals_are_exact(vocab):
    """One beam: totals order as the logits do, so the places are those of a stable sort, with many
    ties in between (logits of few values)."""
    say(f"[beam] ties, vocabulary of {vocab}")
    g = torch.Generator(device=device())
    g.manual_seed(vocab)
    for values in (1, 2, 40):
        logits = torch.randint(0, values, (3, 1, vocab), device=device(), generator=g).float()
        for type_ in (F32, BF16):
            for k in (1, 5, 64):
                _, tokens, _ = rd.rdf2v_beam_select(logits.to(type_), torch.zeros(3, 1, device=device()), k)
                want = logits[:, 0].cpu().sort(dim=1, descending=True, stable=True).indices[:, :k]
                n = want.shape[1]
                assert torch.equal(tokens.cpu()[:, :n].long(), want) and bool((tokens[:, n:] == -1).all())


def test_equal_beams_tie_to_the_lowest():
    say("[beam] equal beams")
    x = torch.randn(1, 1, 5_000, device=device()).repeat(1, 4, 1)
    _, tokens, parents = rd.rdf2v_beam_select(x, torch.zeros(1, 4, device=device()), 12)
    top = x[0, 0].cpu().sort(descending=True, stable=True).indices[:3]
    assert torch.equal(tokens.cpu().long()[0], top.repeat_interleave(4))
    assert parents.cpu()[0].tolist() == [0, 1, 2, 3] * 3


def test_sorted_and_adversarial_orders():
    say("[beam] ascending, descending and clustered logits")
    for vocab in (4_096, 50_001):
        x = torch.linspace(-8, 8, vocab, device=device())
        clustered = torch.full((vocab,), -5.0, device=device())
        clustered[vocab // 3: vocab // 3 + 300] = torch.linspace(1, 4, 300, device=device())
        strided = torch.full((vocab,), -5.0, device=device())
        strided[::256] = torch.linspace(1, 4, strided[::256].numel(), device=device())
        for y in (x, x.flip(0), clustered, strided):
            _check(y.repeat(2, 3, 1), torch.tensor([[0.0, -0.5, -1.0]], device=device()).repeat(2, 1), 64)


def test_masks_that_leave_nothing():
    say("[beam] nothing to choose: masked rows, dead beams, the lowest value")
    logits, scores = _inputs(4, 3, 2_000, F32, 5)
    logits[0] = -math.inf                                  # no beam has a token
    logits[1, :2] = -math.inf                              # one beam has
    logits[2] = -math.inf
    logits[2, 1, 77] = -3.4e38                             # one candidate in the group, of the lowest value
    scores[3] = -math.inf                                  # no beam is alive
    got, tokens, parents = _check(logits, scores, 3)
    assert tokens[0].tolist() == [-1] * 3 and parents[3].tolist() == [9] * 3
    assert tokens[2].tolist() == [77, -1, -1] and abs(float(got[2, 0] - scores[2, 1].double().cpu())) == 0.0
    low = torch.full((1, 2, 500), torch.finfo(BF16).min, device=device(), dtype=BF16)
    low[0, 1, 3] = 0.0
    _check(low, torch.zeros(1, 2, device=device()), 4)


def test_values_that_are_no_numbers():
    say("[beam] NaN and +inf are reported and masked")
    for vocab in (900, 60_000):
        for bad in (math.nan, math.inf):
            logits, scores = _inputs(2, 2, vocab, F32, 6)
            logits[0, 1, vocab - 5] = bad
            _check(logits, scores, 4, status=rd.RDF2V_STATUS_BAD_VALUE)
    logits, scores = _inputs(1, 2, 900, F32, 6)
    scores[0, 0] = math.nan
    _, _, parents = rd.rdf2v_beam_select(logits, scores, 4)
    assert parents.cpu()[0].tolist() == [1] * 4
    # a finished or dead beam's logits are not read
    logits[0, 1] = math.nan
    st = new_status()
    got, tokens, _ = rd.rdf2v_beam_select(logits, torch.tensor([[-math.inf, -2.5]], device=device()), 2,
                                          finished=torch.tensor([[0, 1]], dtype=torch.int32, device=device()),
                                          status=st)
    assert int(st.item()) == 0 and got[0].tolist() == [-2.5, -math.inf] and tokens[0].tolist() == [-1, -1]


def test_strides_and_in_place_scores():
    say("[beam] row strides, unaligned rows, scores in place, workspace of the caller")
    for vocab in (1_001, 40_013):
        for type_ in (F32, BF16):
            logits, scores = _inputs(3, 4, vocab, type_, 8)
            ref = rd.rdf2v_beam_select(logits, scores, 4)
            for pad in (1, 8, 7):
                wide = torch.full((3, 4, vocab + pad), math.nan, device=device(), dtype=type_)
                wide[..., :vocab] = logits
                got = rd.rdf2v_beam_select(wide[..., :vocab], scores, 4)
                assert all(torch.equal(a, b) for a, b in zip(got, ref))
            ws = torch.full((rd.rdf2v_beam_select_workspace_size(3, 4, vocab, 4),), 255, dtype=torch.uint8,
                            device=device())
            mine = scores.clone()
            got = rd.rdf2v_beam_select(logits, mine, 4, scores_out=mine, workspace=ws)
            assert got[0] is mine and all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("shape,dtype", [((5,), torch.int32), ((3, 7), torch.uint8), ((4, 16, 16), F32), ((), BF16),
                                         ((9, 1_001), torch.int16), ((2, 300, 8), torch.int64)],
                         ids=lambda s: str(s).replace(" ", ""))
def test_reorder(shape, dtype):
    say(f"[beam reorder] {shape} {dtype}")
    src = torch.randint(0, 100, (11,) + shape, device=device()).to(dtype)
    parents = torch.randint(0, 11, (4, 6), dtype=torch.int32, device=device())
    assert torch.equal(rd.rdf2v_beam_reorder(src, parents), src[parents.flatten().long()])
    st = new_status()
    bad = torch.tensor([3, -1, 11, 0], dtype=torch.int32, device=device())
    got = rd.rdf2v_beam_reorder(src, bad, status=st)
    assert int(st.item()) == rd.RDF2V_STATUS_ID_OUT_OF_RANGE
    assert torch.equal(got[0], src[3]) and torch.equal(got[3], src[0]) and bool((got[1:3] == 0).all())
    assert rd.rdf2v_beam_reorder(src, bad[:0]).shape == (0,) + shape


def test_reorder_far_offsets():
    say("[beam reorder] rows beyond 2^32 bytes")
    src = torch.zeros(5, 2 ** 30 + 4, dtype=torch.uint8, device=device())
    src[4, -3:] = 7
    got = rd.rdf2v_beam_reorder(src, torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device=device()))
    assert torch.equal(got, src)


def test_refusals():
    say("[beam] refusals")
    logits, scores = _inputs(2, 3, 50, F32, 9)
    call = rd.rdf2v_beam_select
    with pytest.raises(TypeError):
        call(logits.half(), scores, 2)
    with pytest.raises(TypeError):
        call(logits.cpu(), scores, 2)
    with pytest.raises(TypeError):
        call(logits, scores.double(), 2)
    with pytest.raises(TypeError):
        call(logits, scores, 2, finished=torch.zeros(2, 3, dtype=torch.bool, device=device()))
    for bad in (logits[0], logits.transpose(1, 2), logits.transpose(0, 1)):
        with pytest.raises(ValueError):
            call(bad, scores, 2)
    with pytest.raises(ValueError):
        call(logits, scores[:, :2], 2)
    for k in (0, 65):
        with pytest.raises(rd.Rdf2vError):
            call(logits, scores, k)
    with pytest.raises(rd.Rdf2vError):
        call(logits, scores, 2, workspace=torch.empty(8, dtype=torch.uint8, device=device()))
    flat = torch.zeros(12, device=device())
    with pytest.raises(rd.Rdf2vError):                     # written where another group's scores are read
        call(logits, flat[:6].view(2, 3), 2, scores_out=flat[2:6].view(2, 2))
    src = torch.zeros(4, 8, device=device())
    p = torch.zeros(4, dtype=torch.int32, device=device())
    with pytest.raises(rd.Rdf2vError):
        rd.rdf2v_beam_reorder(src, p, out=src)
    with pytest.raises(ValueError):
        rd.rdf2v_beam_reorder(src.T, p)
    with pytest.raises(TypeError):
        rd.rdf2v_beam_reorder(src, p.long())


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5_000, 40_000])
def test_totals_that_round_together_at_powers_of_two(vocab, type_):
    """Scores so low that many logits have the same total: the lowest tokens of it are chosen, wherever
    their logits stand. The totals here are exact to predict: scores are powers of two whose float32
    step is far above the logits' spread, or at it."""
    say(f"[beam] totals that round together, vocabulary of {vocab} {type_}")
    g = torch.Generator(device=device())
    g.manual_seed(vocab)
    for power in (10, 16, 22, 30):
        logits = torch.randn(2, 2, vocab, device=device(), generator=g).to(type_)
        scores = torch.tensor([[-2.0 ** power, -2.0 ** power], [-2.0 ** power, -2.0 ** power * 1.5]], device=device())
        got, tokens, parents = rd.rdf2v_beam_select(logits, scores, 7)
        x = logits.float().cpu()
        # the totals with the log-sum-exp as float32 has it, one unit up and down: the choice is that of one of them
        lse = torch.logsumexp(x.double(), -1, keepdim=True).float()
        ok = torch.zeros(2, dtype=torch.bool)
        steps = [lse, torch.nextafter(lse, lse + 1), torch.nextafter(lse, lse - 1)]
        for a in steps:
            for b in steps:
                both = torch.cat([a[:, :1], b[:, 1:]], 1)
                total = (scores.cpu()[..., None] + (x - both)).flatten(1)
                place = total.sort(dim=1, descending=True, stable=True).indices[:, :7]
                mine = (parents.cpu() - torch.arange(2)[:, None] * 2).long() * vocab + tokens.cpu().long()
                ok |= (place == mine).all(1)
        assert bool(ok.all()), (power, ok)


@pytest.mark.parametrize("size", [(1, 1, 900, 64), (2, 3, 100_001, 8), (1, 4, 300_007, 64), (2, 2, 16_500, 1)],
                         ids=lambda s: "x".join(map(str, s)))
def test_totals_that_round_together(size):
    """Scores near -1.5e7 leave totals whole numbers, so logits of one level tie, however a row's own
    order ranks them, and the first of them win. The levels are far from where lse makes them round the
    other way: lse is off by less than 1e-3 (its sum of exponentials, relative), the distance is 0.1."""
    groups, beams, vocab, num_out = size
    say(f"[beam] rounded totals {size}")
    for type_ in (F32, BF16):
        for seed in range(100):
            g = torch.Generator()
            g.manual_seed(seed)
            level = torch.zeros(vocab)
            level[torch.randperm(vocab, generator=g)[:vocab // (2 + seed)]] = 4.0
            level[torch.randperm(vocab, generator=g)[:5]] = 8.0
            fine = torch.rand(vocab, generator=g) if type_ == F32 else torch.randint(0, 2, (vocab,), generator=g)
            x = (level + fine * 0.0625).to(type_)
            part = (0.03 - torch.logsumexp(x.double(), 0)) % 1.0
            if abs(float(part) - 0.5) > 0.14:
                break
        else:
            raise AssertionError("no levels clear of the rounding")
        logits = x.to(device()).repeat(groups, beams, 1)
        _, tokens, parents = rd.rdf2v_beam_select(logits, torch.full((groups, beams), -1.5e7, device=device()), num_out)
        order = level.repeat(beams).sort(descending=True, stable=True).indices[:num_out]
        for i in range(groups):
            assert torch.equal(tokens[i].cpu().long(), order % vocab)
            assert torch.equal(parents[i].cpu().long(), i * beams + order // vocab)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 64, 40_000, 64), (2, 2, 700_000, 64)], ids=lambda s: "x".join(map(str, s)))
def test_more_entries_than_stay_on_the_chip(size, type_):
    groups, beams, vocab, num_out = size
    say(f"[beam] many entries {size} {type_}")
    logits, scores = _inputs(groups, beams, vocab, type_, 12)
    _check(logits, scores, num_out)
    _check(logits, scores * 0.0, num_out)


def _totals(logits, scores):
    """The totals that the definition gives in float32, on the CPU. The log-sum-exp is the kernel's own: a
    token of logit 0 has at score 0 the total 0 + (0 - lse), which is exact. Every row has one, token 2,
    among its 64 best."""
    groups, beams, vocab = logits.shape
    rows = logits.reshape(-1, 1, vocab)
    got, tokens, _ = rd.rdf2v_beam_select(rows, torch.zeros(rows.shape[0], 1, device=device()), min(64, vocab))
    lse = -got[tokens == 2].view(groups, beams, 1).cpu()
    return scores.cpu()[..., None] + (logits.float().cpu() - lse)


def _check_places(logits, scores, num_out):
    want = _totals(logits, scores)
    groups, beams, vocab = want.shape
    got, tokens, parents = rd.rdf2v_beam_select(logits, scores, num_out)
    first = torch.arange(groups)[:, None] * beams
    best = want.flatten(1).sort(dim=1, descending=True, stable=True)
    place = (parents.cpu() - first).long() * vocab + tokens.cpu()
    wrong = (place != best.indices[:, :num_out]).any(1)
    assert torch.equal(got.cpu(), best.values[:, :num_out])
    assert not bool(wrong.any()), f"{int(wrong.sum())} of {groups} groups"


def test_ties_of_neighbouring_logits():
    """Logits whose totals are equal though they differ: the lowest token is chosen, be it the one that a
    slice left out. Two examples, in which the next smaller float has a smaller total."""
    say("[beam] ties of neighbouring logits: examples")
    for score, row in ((-65.54468536376953, [-5.0, 3.113436222076416, -5.0, 3.1134371757507324]),
                       (-6.0, [1.0000001192092896, 1.000000238418579])):
        logits, scores = torch.tensor([[row]], device=device()), torch.tensor([[score]], device=device())
        at = sorted(range(len(row)), key=lambda i: -row[i])[:2]
        # the kernel's log-sum-exp, by a difference that is exact: the two are within a factor of two
        lse = logits[0, 0, at[0]] - rd.rdf2v_beam_select(logits, scores * 0.0, 1)[0][0, 0]
        total = (scores[0] + (logits[0, 0] - lse)).tolist()
        below = float(scores + (torch.nextafter(logits[0, 0, at[1]], scores[0] - 9.0) - lse))
        assert total[at[0]] == total[at[1]] > below
        _, tokens, _ = rd.rdf2v_beam_select(logits, scores, 1)
        assert tokens[0].tolist() == [min(at)]


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("num_out", [1, 2, 3, 7])
@pytest.mark.parametrize("vocab", [13, 300])
def test_ties_of_neighbouring_logits_over_many_values(vocab, num_out, type_):
    """Tokens a few units of the type apart, in random order, with scores of any size."""
    say(f"[beam] ties of neighbouring logits {vocab} {num_out} {type_}")
    g = torch.Generator().manual_seed(vocab * 8 + num_out)
    groups, unit = 4_000, 2.0 ** (-23 if type_ == F32 else -7)
    for beams in (1, 3):
        base = torch.rand(groups, 1, 1, generator=g) * 3 + 0.25
        steps = torch.randint(0, 12, (groups, beams, vocab), generator=g).float()
        logits = (base.to(type_).float() + steps * unit * 2.0 ** base.log2().floor()).to(type_)
        logits[..., 16:] -= 5.0                            # a few of them at the top
        logits[..., 2] = 0.0
        if vocab > 64:
            logits[..., 64:] -= 9.0                        # the logit of 0 is among the 64 best
        scores = torch.rand(groups, 1, generator=g) * 8.0
        scores = -torch.exp2(scores if type_ == F32 else scores + 13.0).expand(-1, beams).contiguous()
        _check_places(logits.to(device()), scores.to(device()), num_out)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9_000, 40_003, 150_001])
def test_ties_across_slices(vocab, type_):
    """The tied tokens lie all over a row of many slices, its last values among them, and there are more of
    them than are chosen."""
    say(f"[beam] ties across slices {vocab} {type_}")
    unit = 2.0 ** (-23 if type_ == F32 else -7)
    for seed in range(12):
        g = torch.Generator().manual_seed(vocab + seed)
        logits = torch.randn(4, 2, vocab, generator=g) - 8.0
        for i in range(8):
            n = (3, 20, 200, 3_000)[i % 4]
            at = torch.cat((torch.randperm(vocab, generator=g)[:n], vocab - 1 - torch.arange(seed % 3)))
            logits[i // 2, i % 2, at] = -1.0 - torch.randint(0, 16, (len(at),), generator=g) * unit
        logits[..., 2] = 0.0
        scores = -torch.exp2(torch.rand(4, 1, generator=g) * 8.0 + (0.0 if type_ == F32 else 13.0))
        for num_out in (1, 2, 8, 64):
            _check_places(logits.to(type_).to(device()), scores.expand(-1, 2).contiguous().to(device()), num_out)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", [0.0, -0.0, 1.0, -3.0e38])
def test_equal_logits_everywhere(value, type_):
    """What a model without training gives: the first tokens of the first beams, and before them a beam that
    has ended. At -3e38 the vocabulary's logarithm is lost beside the logits in float32, as the definition has
    it, and the living beam of score -6.5 stays before the ended one of -7."""
    say(f"[beam] all logits {value} {type_}")
    for vocab in (70, 20_001, 1_000_200):
        logits = torch.full((2, 3, vocab), value, device=device(), dtype=type_)
        scores = torch.tensor([[-7.0, -7.0, -7.0], [-9.0, -6.5, -7.0]], device=device())
        finished = torch.tensor([[0, 0, 0], [0, 0, 1]], dtype=torch.int32, device=device())
        for k in (1, 7, 64):
            got, tokens, parents = rd.rdf2v_beam_select(logits, scores, k, finished=finished)
            assert tokens[0].tolist() == list(range(k)) and parents[0].tolist() == [0] * k
            ended = [] if value < -1.0e38 else [-1]
            assert tokens[1].tolist() == ended + list(range(k - len(ended)))
            assert parents[1].tolist() == [5] * len(ended) + [4] * (k - len(ended))


@pytest.mark.parametrize("vocab", [50, 30_000])
def test_scores_of_infinity(vocab):
    """A beam of score +inf: all of its totals are, and its lowest tokens are chosen, but for masked ones."""
    say(f"[beam] scores of infinity, vocabulary of {vocab}")
    logits, scores = _inputs(2, 3, vocab, F32, 14)
    scores[0, 1] = math.inf
    scores[1, 0] = scores[1, 2] = math.inf
    logits[0, 1, 4] = -math.inf
    got, tokens, parents = rd.rdf2v_beam_select(logits, scores, 9)
    assert bool((got == math.inf).all())
    assert tokens[0].tolist() == [0, 1, 2, 3, 5, 6, 7, 8, 9] and parents[0].tolist() == [1] * 9
    assert tokens[1].tolist() == list(range(9)) and parents[1].tolist() == [3] * 9
