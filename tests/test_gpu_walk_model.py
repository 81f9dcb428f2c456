"""The operators together, as the example uses them: a model of walks trained to the graph's own
transitions finds the graph's walks; its gradients are those of automatic differentiation."""

import importlib.util
import math
import os

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "walk_model.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("walk_model", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_training_and_search(example, capsys):
    """A hop drawn by chance is an edge in one case of 4,000 (5,000 edges, 20 x 1,000 continuations of an
    entity each with 1 / 4): more than half of them cannot be chance."""
    say("[walk model] 150 steps, then beam search")
    losses, real, every = example.main(["--steps", "150", "--beams", "3", "--hops", "3"])
    assert all(math.isfinite(x) for x in losses)
    assert losses[-1] < losses[0] / 3
    assert every > 64 and real > every / 2


def test_gradients_against_autograd(example):
    """Float32 products of at most 1,020 terms, three in a row: 3 * 1,020 * 2^-24 = 1.8e-4 of the sizes."""
    say("[walk model] gradients against automatic differentiation in 64 bits")
    dev = device()
    csr, starts = example.load_graph(dev)
    model = example.WalkModel(csr.num_entities + csr.num_predicates, dev, seed=3)
    tokens, lens = rd.rdf2v_random_walks(csr, starts[:24], 1, 4, 5)
    lens[3], lens[7] = 1, 4                                    # rows that end early
    ids, weights = example.teacher(csr, tokens, lens)
    loss = model.train_step(tokens, lens, ids, weights)
    embed, qkv, out = (p.double().cpu().requires_grad_() for p in model.params)
    at, n = tokens.cpu().clamp(min=0).long(), lens.cpu()
    x = embed[at]
    q, k, v = (x @ qkv).unflatten(-1, (3 * example.HEADS, example.SIZE)).split(example.HEADS, dim=-2)
    t = torch.arange(tokens.shape[1])
    decay = model.log_decay.double().cpu()
    weight = torch.where(t[:, None] >= t, torch.exp((t[:, None] - t).clamp(min=0) * decay[:, None, None]), 0.0)
    score = torch.einsum("nthd,nshd->nhts", q, k) * example.SIZE ** -0.5 * weight
    a = torch.einsum("nhts,nshd->nthd", score, v) * (t < n[:, None])[..., None, None]
    z = (x + a.flatten(-2) @ out) @ embed.T / example.SIZE
    logp = torch.log_softmax(z, -1)
    there = ids.cpu() >= 0
    p = there / there.sum(-1, keepdim=True).clamp(min=1)
    each = (p * (p.clamp(min=1e-30).log() - logp.gather(-1, ids.cpu().clamp(min=0).long()))).sum(-1)
    mean = each.sum() / there.any(-1).sum()
    mean.backward()
    mean = float(mean.detach())
    assert abs(float(loss) - mean) <= 1.8e-4 * max(1.0, mean)
    for mine, ref in zip(model.params, (embed, qkv, out)):
        off = float((mine.grad.double().cpu() - ref.grad).norm() / ref.grad.norm())
        assert off <= 1.8e-4, off
