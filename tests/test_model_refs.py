"""The plain implementations that the operators are held to, against independent ones: automatic
differentiation, torch's own losses, brute force over all candidates."""

import itertools
import math

import torch

from model_refs import attention, beam_select, distill


def test_attention_against_the_sum_and_autograd():
    torch.manual_seed(0)
    n, t, heads, kv, dk, dv = 3, 9, 4, 2, 5, 3
    d = torch.float64
    q, k, v = (torch.randn(n, t, h, s, dtype=d, requires_grad=True) for h, s in ((heads, dk), (kv, dk), (kv, dv)))
    state = torch.randn(n, heads, dk, dv, dtype=d, requires_grad=True)
    g = torch.tensor([0.0, -0.1, -1.0, -math.inf], dtype=d)
    lens = torch.tensor([9, 4, 0])
    do, ds = torch.randn(n, t, heads, dv, dtype=d), torch.randn(n, heads, dk, dv, dtype=d)
    ref = attention(q.detach(), k.detach(), v.detach(), g, 0.7, lens, state.detach(), do, ds)
    total = torch.zeros((), dtype=d)
    for i, h in itertools.product(range(n), range(heads)):
        gamma, kk, vv = float(torch.exp(g[h])), k[i, :, h // 2], v[i, :, h // 2]
        length = int(lens[i])
        power = lambda m: gamma ** m if m > 0 else 1.0                            # noqa: E731
        for a in range(t):
            if a >= length:
                assert bool((ref["out"][i, a, h] == 0).all())
                continue
            o = sum(power(a - s) * (q[i, a, h] @ kk[s]) * vv[s] for s in range(a + 1))
            o = 0.7 * (o + power(a + 1) * (q[i, a, h] @ state[i, h]))
            assert torch.allclose(o, ref["out"][i, a, h], rtol=1e-12, atol=1e-12)
            total = total + (o * do[i, a, h]).sum()
        end = power(length) * state[i, h] + sum(power(length - 1 - s) * torch.outer(kk[s], vv[s]) for s in range(length))
        assert torch.allclose(end, ref["state"][i, h], rtol=1e-12, atol=1e-12)
        total = total + (end * ds[i, h]).sum()
    total.backward()
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv"), (state, "dstate")):
        assert torch.allclose(x.grad, ref[name], rtol=1e-10, atol=1e-10), name


def test_distill_against_torch():
    torch.manual_seed(1)
    rows, vocab, top, tau = 6, 11, 4, 2.5
    z = torch.randn(rows, vocab, dtype=torch.float64, requires_grad=True)
    ids = torch.stack([torch.randperm(vocab)[:top] for _ in range(rows)])
    ids[2, 1:] = -1
    ids[3] = -1
    ids[4] = 7                                             # one id four times
    t, w = torch.randn(rows, top, dtype=torch.float64), torch.randn(rows, dtype=torch.float64)
    loss, lse, grad = distill(z.detach(), ids, t, tau, w)
    for r in range(rows):
        use = ids[r] >= 0
        if not bool(use.any()):
            assert float(loss[r]) == 0 and bool((grad[r] == 0).all())
            continue
        p = torch.softmax(t[r][use] / tau, 0)
        target = torch.zeros(vocab, dtype=torch.float64).index_add_(0, ids[r][use], p)
        soft = torch.nn.functional.cross_entropy(z[r:r + 1] / tau, target[None]) + (p * p.log()).sum()
        assert abs(float(tau ** 2 * soft.detach()) - float(loss[r])) < 1e-12
        (g,) = torch.autograd.grad(w[r] * tau ** 2 * soft, z)
        assert torch.allclose(g[r], grad[r], atol=1e-12)
        assert abs(float(torch.logsumexp(z[r].detach() / tau, 0)) - float(lse[r])) < 1e-12


def test_beam_select_against_brute_force():
    torch.manual_seed(2)
    logits, scores = torch.randn(2, 3, 5, dtype=torch.float64), -torch.rand(2, 3, dtype=torch.float64)
    logits[0, 1, 2] = -math.inf
    logits[1, 0] = -math.inf
    finished = torch.tensor([[0, 0, 1], [0, 0, 0]])
    best, _ = beam_select(logits, scores, 20, finished)
    for n in range(2):
        every = []
        for b in range(3):
            if finished[n, b]:
                every.append(float(scores[n, b]))
                continue
            e = [math.exp(float(x)) for x in logits[n, b]]
            every += [float(scores[n, b]) + math.log(x / sum(e)) for x in e if x > 0]
        every = sorted(every, reverse=True)
        got = best[n].tolist()
        assert all(abs(a - b) < 1e-12 for a, b in zip(got, every)) and all(x == -math.inf for x in got[len(every):])
