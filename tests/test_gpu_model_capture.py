"""The operators over walk tokens inside a HIP graph: the calls only enqueue kernels, so with outputs and
workspaces of the caller they can be captured. Each of three replays, with the outputs cleared by eager
work in between and other inputs in the same buffers, equals the eager run."""

import pytest
import torch

import paper_2508_01073_amd as rd
from gpu_helpers import device, say

pytestmark = pytest.mark.gpu


def _fill(x, seed):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    for name in ("q", "k", "v", "do", "state", "z", "teacher", "logits"):
        x[name].copy_(torch.randn(x[name].shape, device=device(), generator=g))
    x["scores"].copy_(-torch.rand(x["scores"].shape, device=device(), generator=g))
    x["ids"].copy_(torch.randint(-1, x["z"].shape[1], x["ids"].shape, device=device(), generator=g))


@pytest.mark.parametrize("length,vocab", [(20, 1_020), (1_400, 90_000)], ids=["short", "long"])
def test_replays_equal_the_eager_run(length, vocab):
    say(f"[model capture] rows of {length}, vocabulary of {vocab}")
    dev = device()
    n, h, d = 3, 4, 64
    e = lambda *s, dtype=torch.float32: torch.empty(s, device=dev, dtype=dtype)   # noqa: E731
    bf = torch.bfloat16
    x = dict(q=e(n, length, h, d, dtype=bf), k=e(n, length, 2, d, dtype=bf), v=e(n, length, 2, d, dtype=bf),
             do=e(n, length, h, d, dtype=bf), state=e(n, h, d, d), z=e(7, vocab), teacher=e(7, 9),
             logits=e(2, 3, vocab, dtype=bf), scores=e(2, 3), ids=e(7, 9, dtype=torch.int32))
    decay = torch.tensor([-0.01, -0.1, -0.5, -2.0], device=dev)
    lens = torch.tensor([length, length // 2, 0], dtype=torch.int32, device=dev)
    dloss = torch.ones(7, device=dev)
    sizes = (n, length, h, 2, d, d, bf)
    work = [torch.empty(max(b, 1), dtype=torch.uint8, device=dev) for b in (
        rd.rdf2v_decay_attention_workspace_size(*sizes), rd.rdf2v_decay_attention_backward_workspace_size(*sizes),
        rd.rdf2v_distill_workspace_size(7, vocab, 9), rd.rdf2v_beam_select_workspace_size(2, 3, vocab, 3))]
    out = dict(out=torch.empty_like(x["do"]), end=e(n, h, d, d), dq=torch.empty_like(x["q"]),
               dk=torch.empty_like(x["k"]), dv=torch.empty_like(x["v"]), dstate=e(n, h, d, d),
               step=e(n, h, d, dtype=bf), next=e(n, h, d, d), loss=e(7), lse=e(7), dz=e(7, vocab),
               best=e(2, 3), tokens=e(2, 3, dtype=torch.int32), parents=e(2, 3, dtype=torch.int32),
               moved=e(6, h, d, d))
    six = torch.randn(6, h, d, d, device=dev)
    moved_by = torch.tensor([2, 0, 1], dtype=torch.int32, device=dev)

    def calls():
        q, k, v = x["q"], x["k"], x["v"]
        rd.rdf2v_decay_attention(q, k, v, decay, lens=lens, state=x["state"], out=out["out"], state_out=out["end"],
                                 workspace=work[0])
        rd.rdf2v_decay_attention_backward(q, k, v, decay, x["do"], lens=lens, state=x["state"], dstate_out=out["end"],
                                          dq=out["dq"], dk=out["dk"], dv=out["dv"], dstate=out["dstate"],
                                          workspace=work[1])
        rd.rdf2v_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, out["end"], parents=moved_by,
                                      out=out["step"], state_out=out["next"])
        rd.rdf2v_distill_loss(x["z"], x["ids"], x["teacher"], temperature=2.0, dloss=dloss, loss=out["loss"],
                              lse=out["lse"], dlogits=out["dz"], workspace=work[2])
        rd.rdf2v_beam_select(x["logits"], x["scores"], 3, scores_out=out["best"], tokens=out["tokens"],
                             parents=out["parents"], workspace=work[3])
        rd.rdf2v_beam_reorder(six, out["parents"], out=out["moved"])

    _fill(x, 0)
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2, 3):
        _fill(x, seed)
        calls()
        torch.cuda.synchronize()
        eager = {name: t.clone() for name, t in out.items()}
        for t in out.values():
            t.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            assert torch.equal(t, eager[name]), (seed, name)
