"""The layer operators together, as the example uses them: a model of two layers runs, its gradients are those of
differences and of the plain forms, and one token at a time, with beams changing places, gives what whole rows give."""

import importlib.util
import math
import os

import pytest
import torch

import layer_refs as refs
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


def _plain(model, tokens, lens):
    """Logits in 64 bits on the CPU, and the parameters that they depend on."""
    f = lambda p: p.detach().double().cpu()                                        # noqa: E731
    part, hidden = f(model.embed)[tokens.cpu().clamp(min=0).long()], None
    n = lens.cpu()
    for layer in model.layers:
        w = {k: f(v) for k, v in layer.items()}
        got = refs.norm(part, hidden, w["norm"], lens=n)
        hidden = got["hidden"]
        x, gate = (got["out"] @ w["enter"]).split(model.size, dim=-1)
        x = refs.conv(x, w["taps"], w["taps_bias"], lens=n)["out"]
        dt, b, c = (x @ w["select"]).split([model.size, model.states, model.states], dim=-1)
        y = refs.scan(x, dt, -w["log_rates"].exp(), b[:, :, None], c[:, :, None], dt_bias=w["dt_bias"], skip=w["skip"],
                      gate=gate, lens=n)["out"]
        part = y @ w["leave"]
    return refs.norm(part, hidden, f(model.last), lens=n)["out"] @ f(model.embed).T


def test_training_and_search(example, capsys):
    say("[scan model] 20 steps, then beam search")
    losses, _, every = example.main(["--mixer", "scan", "--steps", "20", "--beams", "3", "--hops", "3"])
    assert len(losses) == 20 and all(math.isfinite(x) for x in losses) and every >= 0


def test_whole_rows_against_the_plain_forms_and_single_tokens(example):
    """Products of 128 terms and the operators between them, each good to about 2^-20 of its sizes; layers and norms
    leave those as they are, and the embeddings' product sums 128 of them: 2^-12 of the logits' size is far beyond."""
    say("[scan model] whole rows, plain forms, single tokens with beams changing places")
    dev = device()
    csr, starts = example.load_graph(dev)
    model = example.ScanModel(csr.num_entities + csr.num_predicates, dev, seed=2)
    tokens, lens = rd.rdf2v_random_walks(csr, starts[:12], 1, 4, 5)
    lens[3] = 1
    with torch.no_grad():
        whole = model(tokens, lens)
    ref = _plain(model, tokens, lens) / example.SIZE
    size = float(ref.abs().max())
    off = (whole.double().cpu() - ref).abs()
    assert float(off.max()) <= 2.0 ** -12 * size, (float(off.max()), size)
    states = model.begin(12)
    order = torch.arange(12, device=dev)
    parents = order.int()
    for i in range(int(lens.max())):
        z, states = model.step(tokens[order, i], states, parents)
        live = (i < lens[order])
        near = (z - whole[order, i])[live].abs().max()
        assert float(near) <= 2.0 ** -11 * size, (i, float(near))
        turn = torch.randperm(12, device=dev)                                      # rows change places
        order, parents = order[turn], turn.int()


def test_gradients_against_differences(example):
    """Along the gradient and a little of a random direction, of length about 1, of each parameter: central differences
    of the loss with a step of 2^-8. The loss, of at most 8, is good to about 2^-20 of that, so a slope to 2^-9; the
    third derivative adds 2^-16 of what is some tens of times the slope: 1 % of it holds that."""
    say("[scan model] gradients against differences")
    dev = device()
    csr, starts = example.load_graph(dev)
    model = example.ScanModel(csr.num_entities + csr.num_predicates, dev, seed=4, drop=0.2)
    tokens, lens = rd.rdf2v_random_walks(csr, starts[:64], 1, 4, 7)
    lens[5], lens[6] = 1, 4
    ids, weights = example.teacher(csr, tokens, lens)

    def loss():
        with torch.no_grad():
            z = model(tokens, lens, model.drop)
            each, _ = rd.rdf2v_distill_loss(z.flatten(0, 1), ids.flatten(0, 1), weights.flatten(0, 1))
            return float(each.double().sum() / (ids >= 0).any(-1).sum())

    model.train_step(tokens, lens, ids, weights)
    model.steps -= 1                                                               # the same masks again
    for k, p in enumerate(model.params):
        g = torch.Generator(device=dev).manual_seed(k)
        v = p.grad / p.grad.norm().clamp(min=1e-20) + 0.1 * torch.randn(p.shape, device=dev, generator=g) / p.numel() ** 0.5
        h = 2.0 ** -8
        with torch.no_grad():
            p += h * v
            up = loss()
            p -= 2 * h * v
            down = loss()
            p += h * v
        along, slope = float((p.grad * v).sum()), (up - down) / (2 * h)
        assert abs(slope - along) <= 0.01 * abs(along) + 2.0 ** -9, (k, slope, along)
