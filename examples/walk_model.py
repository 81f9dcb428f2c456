"""A small sequence model of walks: trained on a graph's walks, then asked for likely walks.

The corpus pipeline gives walk rows. A model with one layer of decay attention reads them and is
trained to the graph's own transitions, a teacher whose top tokens are an entity's out-edges: at an
entity the predicates it can leave by, at a predicate the objects it can reach. Beam search then
extends start entities token by token, the attention's states following the beams.

    python examples/walk_model.py                 # 1,000 entities, 5,000 triples, a few seconds
    python examples/walk_model.py --steps 400
    python examples/walk_model.py --mixer scan    # two layers of convolution and selective scan instead
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2508_01073_amd as rd  # noqa: E402
import synth  # noqa: E402

HEADS, SIZE = 4, 32          # heads of the attention, and their keys' and values' size
TOP = 16                     # out-edges of an entity that the teacher names


def load_graph(dev):
    w = synth.WORKLOADS["tiny_uniform"]
    s, p, o = (torch.from_numpy(x).to(dev) for x in synth.triples(w))
    csr = rd.rdf2v_build_csr(s, p, o, w.num_entities, w.num_predicates)
    return csr, rd.rdf2v_nonsink_starts(csr)


def teacher(csr, tokens, lens):
    """(ids [rows, length, TOP], logits) of the tokens that may follow each token of the walk rows: equal
    logits for each out-edge, so that what several edges lead to counts several times. -1: no entry."""
    rows, length = tokens.shape
    at = torch.arange(length, device=tokens.device)
    entity = tokens[:, at - at % 2].clamp(min=0).long()        # the entity a position stands at or has left
    edge = csr.row_ptr[entity][..., None] + torch.arange(TOP, device=tokens.device)
    there = edge < csr.row_ptr[entity + 1][..., None]
    there &= (at + 1 < lens[:, None])[..., None]               # nothing follows a walk's last token
    pred, obj = csr.edges[edge.clamp(max=csr.num_edges - 1).long()].unbind(-1)
    pred = pred + csr.num_entities
    at_entity = (at % 2 == 0)[None, :, None]
    ids = torch.where(at_entity, pred, torch.where(pred == tokens[..., None], obj, -1))
    ids = torch.where(there, ids, -1).int()
    return ids, torch.zeros(ids.shape, device=tokens.device)


class WalkModel:
    """Embeddings, one residual layer of decay attention, logits by the embeddings. The gradients are
    written out: the operators compute theirs, products are torch's."""

    def __init__(self, vocab, dev, seed=0):
        g = torch.Generator(device=dev).manual_seed(seed)
        d = HEADS * SIZE
        r = lambda *s: torch.randn(*s, device=dev, generator=g)  # noqa: E731
        self.embed = r(vocab, d)
        self.qkv = r(d, 3 * d) / math.sqrt(d)
        self.out = r(d, d) / math.sqrt(d)
        self.log_decay = torch.log1p(-torch.exp2(-1.0 - torch.arange(HEADS, device=dev, dtype=torch.float32)))
        self.params = [self.embed, self.qkv, self.out]

    def split(self, x):
        return (x @ self.qkv).unflatten(-1, (3 * HEADS, SIZE)).split(HEADS, dim=-2)

    def logits(self, x, attended):
        return (x + attended.flatten(-2) @ self.out) @ self.embed.T / SIZE

    def begin(self, rows):
        """The states of `rows` walks without tokens, and as much memory for those after a token."""
        state = torch.zeros(rows, HEADS, SIZE, SIZE, device=self.embed.device)
        return state, torch.empty_like(state)

    def step(self, last, states, parents):
        """(logits, states) of one token more for each row, from the states of the parents' rows."""
        state, other = states
        x = self.embed[last.clamp(min=0).long()]
        q, k, v = self.split(x)
        attended, new = rd.rdf2v_decay_attention_step(q, k, v, self.log_decay, state, parents=parents, state_out=other)
        return self.logits(x, attended), (new, state)

    def train_step(self, tokens, lens, ids, weights):
        """Mean loss over the positions that something follows, and the gradients in .grad."""
        at = tokens.clamp(min=0).long()                        # rows are padded with -1; lens says where they end
        x = self.embed[at]
        q, k, v = self.split(x)
        attended, _ = rd.rdf2v_decay_attention(q, k, v, self.log_decay, lens=lens)
        hidden = x + attended.flatten(-2) @ self.out
        z = hidden @ self.embed.T / SIZE
        counts = (ids >= 0).any(-1).flatten()
        dloss = counts.float() / counts.sum()
        loss, _, dz = rd.rdf2v_distill_loss(z.flatten(0, 1), ids.flatten(0, 1), weights.flatten(0, 1), dloss=dloss)
        dz = dz / SIZE
        dhidden = (dz @ self.embed).view_as(hidden)
        dout = attended.flatten(-2).flatten(0, 1).T @ dhidden.flatten(0, 1)
        dattended = (dhidden @ self.out.T).unflatten(-1, (HEADS, SIZE))
        dq, dk, dv, _ = rd.rdf2v_decay_attention_backward(q, k, v, self.log_decay, dattended, lens=lens)
        dsplit = torch.cat((dq, dk, dv), dim=-2).flatten(-2)
        dx = dhidden + dsplit @ self.qkv.T
        dembed = dz.T @ hidden.flatten(0, 1)
        dembed.index_add_(0, at.flatten(), dx.flatten(0, 1))
        for p, g in zip(self.params, (dembed, x.flatten(0, 1).T @ dsplit.flatten(0, 1), dout)):
            p.grad = g
        return (loss * dloss).sum()


class ScanModel:
    """Embeddings, layers of a causal convolution and a selective scan joined by residual norms, logits by the
    embeddings. Autograd records the operators."""

    def __init__(self, vocab, dev, seed=0, layers=2, size=HEADS * SIZE, states=8, width=4, drop=0.1):
        g = torch.Generator(device=dev).manual_seed(seed)
        r = lambda *s: torch.randn(*s, device=dev, generator=g)  # noqa: E731
        self.size, self.states, self.width, self.drop, self.seed, self.steps = size, states, width, drop, seed, 0
        self.embed = r(vocab, size)
        rates = torch.arange(1.0, states + 1, device=dev).repeat(size, 1)
        self.layers = [dict(norm=torch.ones(size, device=dev), enter=r(size, 2 * size) / math.sqrt(size),
                            taps=r(size, width) / math.sqrt(width), taps_bias=torch.zeros(size, device=dev),
                            select=r(size, size + 2 * states) / math.sqrt(size), log_rates=rates.log(),
                            dt_bias=torch.full((size,), -2.0, device=dev), skip=torch.ones(size, device=dev),
                            leave=r(size, size) / math.sqrt(size)) for _ in range(layers)]
        self.last = torch.ones(size, device=dev)
        self.params = [self.embed, self.last, *(p for layer in self.layers for p in layer.values())]
        for p in self.params:
            p.requires_grad_()

    def select(self, layer, x):
        """dt, b and c of the convolution's outputs."""
        dt, b, c = (x @ layer["select"]).split([self.size, self.states, self.states], dim=-1)
        return dt, b.unsqueeze(-2), c.unsqueeze(-2)

    def __call__(self, tokens, lens, drop=0.0):
        """Logits of whole rows."""
        part, hidden = self.embed[tokens.clamp(min=0).long()], None
        for i, layer in enumerate(self.layers):
            given = dict(drop=drop if i else 0.0, seed=self.seed + 1000 * self.steps + i, lens=lens)
            normed, hidden, _ = rd.rdf2v_residual_norm(part, hidden, layer["norm"], **given)
            x, gate = (normed @ layer["enter"]).split(self.size, dim=-1)
            x, _ = rd.rdf2v_causal_conv(x, layer["taps"], layer["taps_bias"], lens=lens)
            dt, b, c = self.select(layer, x)
            y, _ = rd.rdf2v_selective_scan(x, dt, -layer["log_rates"].exp(), b, c, dt_bias=layer["dt_bias"],
                                           skip=layer["skip"], gate=gate, lens=lens)
            part = y @ layer["leave"]
        given = dict(drop=drop, seed=self.seed + 1000 * self.steps + len(self.layers), lens=lens)
        return rd.rdf2v_residual_norm(part, hidden, self.last, **given)[0] @ self.embed.T / SIZE

    def train_step(self, tokens, lens, ids, weights):
        """Mean loss over the positions that something follows, and the gradients in .grad."""
        z = self(tokens, lens, self.drop)
        self.steps += 1
        loss, _ = rd.rdf2v_distill_loss(z.flatten(0, 1), ids.flatten(0, 1), weights.flatten(0, 1))
        mean = loss.sum() / (ids >= 0).any(-1).sum()
        for p in self.params:
            p.grad = None
        mean.backward()
        return mean.detach()

    def begin(self, rows):
        """The states of `rows` walks without tokens."""
        new = lambda *s: torch.zeros(rows, *s, device=self.embed.device)  # noqa: E731
        return [(new(self.width - 1, self.size), new(self.size, self.states)) for _ in self.layers]

    @torch.no_grad()
    def step(self, last, states, parents):
        """(logits, states) of one token more for each row, from the states of the parents' rows."""
        part, hidden, after = self.embed[last.clamp(min=0).long()], None, []
        for layer, (near, far) in zip(self.layers, states):
            normed, hidden, _ = rd.rdf2v_residual_norm(part, hidden, layer["norm"])
            x, gate = (normed @ layer["enter"]).split(self.size, dim=-1)
            x, near = rd.rdf2v_causal_conv_step(x, layer["taps"], layer["taps_bias"], near, parents=parents)
            dt, b, c = self.select(layer, x)
            y, far = rd.rdf2v_selective_scan_step(x, dt, -layer["log_rates"].exp(), b, c, far,
                                                  dt_bias=layer["dt_bias"], skip=layer["skip"], gate=gate,
                                                  parents=parents)
            part = y @ layer["leave"]
            after.append((near, far))
        return rd.rdf2v_residual_norm(part, hidden, self.last)[0] @ self.embed.T / SIZE, after


def search(model, csr, starts, hops, beams):
    """Likely walks of `hops` hops from each start: (tokens [starts, beams, 2 * hops + 1], scores). A walk
    that reaches an entity without out-edges ends there and is padded with -1."""
    dev, groups = starts.device, starts.shape[0]
    vocab = csr.num_entities + csr.num_predicates
    is_pred = torch.arange(vocab, device=dev) >= csr.num_entities
    degree = csr.row_ptr[1:] - csr.row_ptr[:-1]
    rows = groups * beams
    states = model.begin(rows)
    walks = torch.full((rows, 2 * hops + 1), -1, dtype=torch.int32, device=dev)
    walks[:, 0] = starts.repeat_interleave(beams)
    scores = torch.full((groups, beams), -math.inf, device=dev)
    scores[:, 0] = 0.0                                         # one walk each to begin with
    finished = torch.zeros(groups, beams, dtype=torch.int32, device=dev)
    parents = torch.arange(rows, dtype=torch.int32, device=dev)
    for i in range(2 * hops):
        last = walks[:, i]
        if i % 2 == 0:
            finished |= ((last < 0) | (degree[last.clamp(min=0).long()] == 0)).int().view(groups, beams)
        z, states = model.step(last, states, parents)
        z = z.masked_fill_(is_pred if i % 2 else ~is_pred, -math.inf)
        scores, tokens, parents = rd.rdf2v_beam_select(z.view(groups, beams, vocab), scores, beams, finished=finished)
        parents = parents.flatten()
        walks = rd.rdf2v_beam_reorder(walks, parents)          # the states follow in the next step
        finished = rd.rdf2v_beam_reorder(finished.view(-1, 1), parents).view(groups, beams)
        walks[:, i + 1] = tokens.flatten()
    return walks.view(groups, beams, -1), scores


def real_hops(csr, walks):
    """How many of the walks' hops are edges of the graph: (real, all)."""
    keys = {(int(s), int(p) + csr.num_entities, int(o)) for s in range(csr.num_entities)
            for p, o in csr.edges_of[s]}
    hops = [tuple(w[i:i + 3]) for w in walks.flatten(0, 1).tolist() for i in range(0, len(w) - 2, 2) if w[i + 2] >= 0]
    return sum(h in keys for h in hops), len(hops)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=256, help="walks of a step")
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--hops", type=int, default=4)
    ap.add_argument("--mixer", choices=["decay", "scan"], default="decay", help="decay attention, or selective scan")
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    csr, starts = load_graph(dev)
    vocab = csr.num_entities + csr.num_predicates
    model = (WalkModel if a.mixer == "decay" else ScanModel)(vocab, dev)
    optimizer = torch.optim.Adam(model.params, lr=0.01)
    n = starts.shape[0]
    torch.manual_seed(0)
    losses = []
    for step in range(a.steps):
        pick = starts[torch.randint(0, n, (a.batch,), device=dev)]
        tokens, lens = rd.rdf2v_random_walks(csr, pick, 1, a.hops, synth.WALK_SEED + step)
        ids, weights = teacher(csr, tokens, lens)
        losses.append(model.train_step(tokens, lens, ids, weights))
        optimizer.step()
    losses = torch.stack(losses).tolist()
    print(f"loss: {losses[0]:.3f} at first, {losses[-1]:.3f} after {a.steps} steps")
    rp, edges = csr.row_ptr.tolist(), csr.edges.tolist()
    csr.edges_of = [edges[rp[e]:rp[e + 1]] for e in range(csr.num_entities)]
    walks, scores = search(model, csr, starts[:64], a.hops, a.beams)
    real, every = real_hops(csr, walks)
    print(f"{walks.shape[0]} searches of {a.beams} beams: {real} of {every} hops are edges of the graph")
    print("most likely walk of the first:", walks[0, 0].tolist(), f"log probability {float(scores[0, 0]):.2f}")
    return losses, real, every


if __name__ == "__main__":
    main()
