"""The work whose speed the operators of a walk model are measured by.

The framework's walk rows (entity / predicate tokens, ragged lengths) are what a sequence model
trains on and answers with. Each case is one pass through one operator of such a model, as a program
calls it:

  prompt   decay attention over whole rows of tokens: outputs, and the states where ``state`` says so
  train    the same forward and backward: outputs, states and every gradient
  step     decay attention of one more token per row, the states of the parents' rows taken over
  select   beam search's selection over beams and vocabulary, and the beams' histories in the new order
  distill  loss and gradient of the logits against a teacher's top logits

Sizes are those of the repository's workloads: vocabularies of entities plus predicates (1,020 up to
1,000,200 tokens), rows of 2 * depth + 1 tokens, and longer rows as walks laid end to end give them.
Values are random: logits spread as a trained model's are, some tokens masked with -inf, some rows
padding, some beams finished, decays between 1 - 1/8 and 1 - 1/256 a token.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CHUNK = 64  # positions of a chunk of the plain form


def listed():
    return [
        # One walk extended by one token: latency is all there is to it.
        dict(name="step_one", kind="step", type="bf16", groups=1, beams=1, heads=4, kv_heads=4, dk=64, dv=64),
        # 64 beam searches of 8 beams extended by a token: every beam takes its parent's states over.
        dict(name="step_beams", kind="step", type="bf16", groups=64, beams=8, heads=8, kv_heads=2, dk=128, dv=128),
        # Scoring of a batch of depth-8 walk rows: very many very short ragged rows.
        dict(name="prompt_walks", kind="prompt", type="bf16", rows=4000, length=17, ragged=True, heads=4, kv_heads=4,
             dk=32, dv=32, state=False),
        # One long row, 1,177 walks end to end: few rows, so the work lies along the length.
        dict(name="prompt_long", kind="prompt", type="bf16", rows=1, length=20_011, ragged=False, heads=8, kv_heads=8,
             dk=128, dv=128, state=True),
        # Training on depth-16 walk rows in 32 bits: ragged, shared key and value heads, odd head sizes.
        dict(name="train_walks", kind="train", type="f32", rows=1024, length=33, ragged=True, heads=6, kv_heads=3,
             dk=48, dv=80, state=False),
        # Training on long rows, states carried from the rows before (truncated backpropagation).
        dict(name="train_long", kind="train", type="bf16", rows=4, length=4096, ragged=False, heads=16, kv_heads=16,
             dk=128, dv=128, state=True),
        # A beam search over the smallest workload's vocabulary.
        dict(name="select_tiny", kind="select", type="f32", groups=1, beams=4, vocab=1_020, out=4, history=9),
        # A batch of searches over the vocabulary of the 1M-triple workload.
        dict(name="select_batch", kind="select", type="f32", groups=32, beams=8, vocab=100_050, out=8, history=17),
        # Searches over the vocabulary of the 20M-triple workload, the logits as a 16-bit product leaves them.
        dict(name="select_large", kind="select", type="bf16", groups=8, beams=8, vocab=1_000_200, out=8, history=17),
        # Ten depth-4 walks over the smallest vocabulary.
        dict(name="distill_tiny", kind="distill", type="f32", rows=90, vocab=1_020, top=8, temperature=1.0),
        # 256 depth-8 walks over the dense workload's vocabulary: a row fits on chip.
        dict(name="distill_walks", kind="distill", type="bf16", rows=4_352, vocab=10_100, top=32, temperature=2.0),
        # 30 depth-8 walks over the 20M-triple workload's vocabulary: a row is 2 MB.
        dict(name="distill_large", kind="distill", type="bf16", rows=510, vocab=1_000_200, top=64, temperature=2.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "prompt", "train", "select", "distill"])
    c = dict(kind=kind, type=rng.choice(["bf16", "f32"]))
    if kind in ("step", "prompt", "train"):
        c["kv_heads"] = rng.randint(1, 8)
        c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 3])
        if rng.random() < 0.5:
            c["dk"] = c["dv"] = rng.choice([16, 32, 64, 128])
        else:
            c["dk"], c["dv"] = _log(rng, 8, 128), _log(rng, 8, 128)
    if kind == "step":
        c["beams"] = rng.randint(1, 16)
        most = 2 ** 26 // (c["heads"] * c["dk"] * c["dv"] * c["beams"])  # states of at most 256 MB
        c["groups"] = _log(rng, 1, max(1, min(512, most)))
    elif kind in ("prompt", "train"):
        c["length"] = _log(rng, 1, 16_384)
        width = c["heads"] * (c["dk"] + c["dv"]) * 2
        most = 2 ** (26 if kind == "prompt" else 25) // (width * c["length"])
        c["rows"] = _log(rng, 1, max(1, min(4096, most)))
        c["ragged"] = rng.random() < 0.5
        c["state"] = rng.random() < 0.5 and c["rows"] * c["heads"] * c["dk"] * c["dv"] <= 2 ** 25
    elif kind == "select":
        c["vocab"] = _log(rng, 1_020, 1_000_200)
        c["beams"] = rng.randint(1, 16)
        c["out"] = rng.choice([c["beams"], rng.randint(1, 16)])
        c["groups"] = _log(rng, 1, max(1, min(32, 2 ** 25 // (c["vocab"] * c["beams"]))))
        c["history"] = 2 * rng.randint(1, 16) + 1
    else:
        c["vocab"] = _log(rng, 1_020, 1_000_200)
        c["rows"] = _log(rng, 1, max(1, min(8192, 2 ** 28 // c["vocab"])))
        c["top"] = rng.randint(1, 64)
        c["temperature"] = rng.choice([1.0, 1.0, 2.0, 4.0])
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _log_decay(heads):
    e = 3.0 + 5.0 * torch.arange(heads, device=DEV, dtype=torch.float64) / max(1, heads)
    return torch.log1p(-torch.exp2(-e)).float()


def _projections(c, lead, g):
    """q, k and v as one product gives them: slices of one buffer."""
    hq, hk, dk, dv = c["heads"], c["kv_heads"], c["dk"], c["dv"]
    x = torch.randn(*lead, hq * dk + hk * (dk + dv), device=DEV, generator=g).to(TYPES[c["type"]])
    q, k, v = x.split([hq * dk, hk * dk, hk * dv], dim=-1)
    return q.unflatten(-1, (hq, dk)), k.unflatten(-1, (hk, dk)), v.unflatten(-1, (hk, dv))


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    kind = c["kind"]
    if kind == "step":
        rows = c["groups"] * c["beams"]
        st["q"], st["k"], st["v"] = _projections(c, (rows,), g)
        st["log_decay"] = _log_decay(c["heads"])
        st["state"] = torch.randn(rows, c["heads"], c["dk"], c["dv"], device=DEV, generator=g)
        st["state_out"] = torch.empty_like(st["state"])  # the two change places from token to token
        first = torch.arange(c["groups"], device=DEV, dtype=torch.int32)[:, None] * c["beams"]
        pick = torch.randint(0, c["beams"], (c["groups"], c["beams"]), device=DEV, generator=g, dtype=torch.int32)
        st["parents"] = (first + pick).flatten()
    elif kind in ("prompt", "train"):
        n, t = c["rows"], c["length"]
        st["q"], st["k"], st["v"] = _projections(c, (n, t), g)
        st["log_decay"] = _log_decay(c["heads"])
        st["lens"] = (torch.randint(0, t + 1, (n,), device=DEV, generator=g, dtype=torch.int32) if c["ragged"] else None)
        shape = (n, c["heads"], c["dk"], c["dv"])
        st["state"] = torch.randn(shape, device=DEV, generator=g) if c["state"] else None
        if kind == "train":
            st["dout"] = torch.randn(n, t, c["heads"], c["dv"], device=DEV, generator=g).to(TYPES[c["type"]])
            st["dstate"] = torch.randn(shape, device=DEV, generator=g) if c["state"] else None
    elif kind == "select":
        n, b, v = c["groups"], c["beams"], c["vocab"]
        logits = torch.randn(n, b, v, device=DEV, generator=g).mul_(2.0)
        logits[3::4, :, v // 64:] = -math.inf  # searches that stand at a predicate: the entities are masked
        st["logits"] = logits.to(TYPES[c["type"]])
        st["scores"] = torch.rand(n, b, device=DEV, generator=g).mul_(-6.0).sort(dim=1, descending=True).values
        st["scores"][1::4, 1:] = -math.inf  # searches at their first token: one beam is alive
        st["finished"] = (torch.rand(n, b, device=DEV, generator=g) < 0.125).int()
        st["history"] = torch.randint(0, v, (n * b, c["history"]), device=DEV, generator=g, dtype=torch.int32)
    else:
        n, v, k = c["rows"], c["vocab"], c["top"]
        st["logits"] = torch.randn(n, v, device=DEV, generator=g, dtype=torch.float32).mul_(2.0).to(TYPES[c["type"]])
        at = torch.randint(0, v, (n, 1), device=DEV, generator=g)
        step = torch.randint(1, max(2, v // k), (n, 1), device=DEV, generator=g)
        ids = (at + step * torch.arange(k, device=DEV)) % v
        # as many as the graph has out-edges, none where the walk row is padding
        some = torch.randint(1, 2 * k, (n, 1), device=DEV, generator=g).clamp_(max=k)
        some *= torch.rand(n, 1, device=DEV, generator=g) >= 0.125
        st["ids"] = torch.where(torch.arange(k, device=DEV) < some, ids, -1).int()
        st["teacher"] = torch.randn(n, k, device=DEV, generator=g).mul_(2.0)
        st["dloss"] = torch.full((n,), 1.0 / n, device=DEV)  # the mean over the rows
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

def _heads_first(x, heads):
    """[n, t, h, d] -> [n, heads, t, d] in 32 bits, shared heads repeated."""
    x = x.float().transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], dim=1)


def _scan(a, b, c, decay):
    """out[t] = sum over s <= t of exp(decay (t - s)) (a[t] . b[s]) c[s], in chunks."""
    n, h, t, _ = a.shape
    m = -(-t // CHUNK)
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, m * CHUNK - t)).unflatten(2, (m, CHUNK)) for x in (a, b, c))
    i = torch.arange(CHUNK, device=a.device, dtype=torch.float32)
    j = torch.arange(m, device=a.device, dtype=torch.float32)
    g = decay[:, None, None]
    inside = torch.where(i[:, None] >= i, torch.exp((i[:, None] - i).clamp(min=0) * g), 0.0)
    out = ((a @ b.transpose(-1, -2)) * inside[:, None]) @ c
    to_end = (b * torch.exp((CHUNK - 1 - i)[:, None] * g)[:, None]).transpose(-1, -2) @ c
    before = torch.where(j[:, None] > j, torch.exp((j[:, None] - 1 - j).clamp(min=0) * (CHUNK * g)), 0.0)
    came = (before @ to_end.flatten(-2)).unflatten(-1, to_end.shape[-2:])
    out += (a * torch.exp((i + 1)[:, None] * g)[:, None]) @ came
    return out.flatten(2, 3)[:, :, :t]


def _group_sum(x, kv_heads):
    """[n, h, t, d] -> [n, t, kv_heads, d]: gradients of shared heads add up."""
    return x.unflatten(1, (kv_heads, -1)).sum(2).transpose(1, 2)


def _plain_attention(st, train):
    c = st["case"]
    heads, kv, t, kind = c["heads"], c["kv_heads"], c["length"], TYPES[c["type"]]
    scale, decay = c["dk"] ** -0.5, st["log_decay"]
    q, k, v = (_heads_first(st[x], heads) for x in "qkv")
    at = torch.arange(t, device=q.device, dtype=torch.float32)
    lens = st["lens"].float() if st["lens"] is not None else torch.full((c["rows"],), float(t), device=q.device)
    valid = (at < lens[:, None])[:, None, :, None]
    q, k, v = (torch.where(valid, x, 0.0) for x in (q, k, v))
    since = torch.exp((at + 1)[:, None] * decay[:, None, None])                       # [h, t, 1]
    left = torch.exp((lens[:, None] - 1 - at).clamp(min=0)[:, None, :, None] * decay[:, None, None])  # [n, h, t, 1]
    whole = torch.exp(lens[:, None] * decay)[:, :, None, None]
    s0 = st["state"]
    out = _scan(q, k, v, decay)
    if s0 is not None:
        out = out + (q * since) @ s0
    got = {"out": (out * scale).transpose(1, 2).to(kind)}
    if c["state"]:
        got["state"] = (k * left).transpose(-1, -2) @ v + whole * s0
    if not train:
        return got
    do = torch.where(valid, _heads_first(st["dout"], heads), 0.0) * scale
    dq = _scan(do, v, k, decay)
    dk = _scan(v.flip(2), do.flip(2), q.flip(2), decay).flip(2)
    dv = _scan(k.flip(2), q.flip(2), do.flip(2), decay).flip(2)
    if s0 is not None:
        ds = st["dstate"]
        dq = dq + (do * since) @ s0.transpose(-1, -2)
        dk = dk + (v * left) @ ds.transpose(-1, -2)
        dv = dv + (k * left) @ ds
        got["dstate"] = (q * since).transpose(-1, -2) @ do + whole * ds
    dk, dv = torch.where(valid, dk, 0.0), torch.where(valid, dv, 0.0)
    got |= {"dq": dq.transpose(1, 2).to(kind), "dk": _group_sum(dk, kv).to(kind), "dv": _group_sum(dv, kv).to(kind)}
    return got


def _plain_step(st):
    c = st["case"]
    repeat = c["heads"] // c["kv_heads"]
    q = st["q"].float()
    k, v = (st[x].float().repeat_interleave(repeat, dim=1) for x in "kv")
    s = st["state"][st["parents"].long()] * torch.exp(st["log_decay"])[:, None, None] + k[..., None] * v[..., None, :]
    out = (q[..., None] * s).sum(-2) * c["dk"] ** -0.5
    return {"out": out.to(TYPES[c["type"]]), "state": s}


def _plain_select(st):
    c = st["case"]
    n, b, v, k = c["groups"], c["beams"], c["vocab"], c["out"]
    x = st["logits"].float()
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    total = st["scores"][..., None] + (x - lse)
    ended = st["finished"][..., None] != 0
    first = torch.arange(v, device=x.device) == 0
    total = torch.where(ended, torch.where(first, st["scores"][..., None], -math.inf), total) + 0.0
    # the largest totals, ties to the lowest place: the total's order and the place as one number
    bits = total.flatten(1).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * 2 ** 32 + (2 ** 32 - 1 - torch.arange(b * v, device=x.device))
    place = 2 ** 32 - 1 - (torch.topk(order, k, dim=1).values & (2 ** 32 - 1))
    scores = total.flatten(1).gather(1, place)
    beam, token = place // v, place % v
    alive = scores > -math.inf
    token = torch.where(alive & (st["finished"].gather(1, beam) == 0), token, -1)
    beam = torch.where(alive, beam, 0)
    parents = beam + torch.arange(n, device=x.device)[:, None] * b
    return {"scores": scores, "tokens": token.int(), "parents": parents.int(), "history": st["history"][parents.flatten()]}


def _plain_distill(st):
    c = st["case"]
    tau = c["temperature"]
    there = st["ids"] >= 0
    ids = st["ids"].clamp(min=0).long()
    valid = there.any(1)
    t = torch.where(there, st["teacher"] / tau, -math.inf)
    t = torch.where(valid[:, None], t, 0.0)
    t = t - t.amax(1, keepdim=True)
    log_p = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    p = torch.where(there, torch.exp(log_p), 0.0)
    z = st["logits"].float() / tau
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    log_q = z.gather(1, ids) - lse
    loss = tau * tau * torch.where(there, p * (torch.where(there, log_p, 0.0) - log_q), 0.0).sum(1)
    weight = torch.where(valid, st["dloss"], 0.0)[:, None] * tau
    dz = torch.exp(z - lse) * weight
    dz.scatter_add_(1, ids, -p * weight)
    lse = torch.where(valid, lse[:, 0], 0.0)
    return {"loss": loss, "lse": lse, "dlogits": dz.to(TYPES[c["type"]])}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    st, c = state, state["case"]
    kind = c["kind"]
    if not own:
        if kind == "step":
            return _plain_step(st)
        if kind == "select":
            return _plain_select(st)
        if kind == "distill":
            return _plain_distill(st)
        return _plain_attention(st, kind == "train")
    import paper_2508_01073_amd as rd
    if kind == "step":
        out, new = rd.rdf2v_decay_attention_step(st["q"], st["k"], st["v"], st["log_decay"], st["state"],
                                                 parents=st["parents"], state_out=st["state_out"])
        return {"out": out, "state": new}
    if kind == "select":
        scores, tokens, parents = rd.rdf2v_beam_select(st["logits"], st["scores"], c["out"], finished=st["finished"])
        return {"scores": scores, "tokens": tokens, "parents": parents,
                "history": rd.rdf2v_beam_reorder(st["history"], parents)}
    if kind == "distill":
        loss, lse, dlogits = rd.rdf2v_distill_loss(st["logits"], st["ids"], st["teacher"],
                                                   temperature=c["temperature"], dloss=st["dloss"])
        return {"loss": loss, "lse": lse, "dlogits": dlogits}
    out, new = rd.rdf2v_decay_attention(st["q"], st["k"], st["v"], st["log_decay"], lens=st["lens"],
                                        state=st["state"], want_state=c["state"])
    got = {"out": out, "state": new} if c["state"] else {"out": out}
    if kind == "train":
        dq, dk, dv, dstate = rd.rdf2v_decay_attention_backward(st["q"], st["k"], st["v"], st["log_decay"], st["dout"],
                                                               lens=st["lens"], state=st["state"],
                                                               dstate_out=st["dstate"])
        got |= {"dq": dq, "dk": dk, "dv": dv}
        if c["state"]:
            got["dstate"] = dstate
    return got


def work(case):
    """Each input once, each output once; the operations of the recurrence."""
    c, kind = case, case["kind"]
    size = 2 if c["type"] == "bf16" else 4
    if kind in ("step", "prompt", "train"):
        hq, hk, dk, dv = c["heads"], c["kv_heads"], c["dk"], c["dv"]
        tokens = c["groups"] * c["beams"] if kind == "step" else c["rows"] * c["length"] * (0.5 if c["ragged"] else 1.0)
        padded = tokens if kind == "step" else c["rows"] * c["length"]
        ins, out = hq * dk + hk * (dk + dv), hq * dv
        held = (tokens if kind == "step" else c["rows"] if c["state"] else 0) * hq * dk * dv * 4.0
        # of a step's parents some are taken more than once, and others not at all
        read = held * (1.0 - (1.0 - 1.0 / c["beams"]) ** c["beams"] if kind == "step" else 1.0)
        nbytes, flops = (ins * tokens + out * padded) * size + read + held, 4.0 * tokens * hq * dk * dv
        if kind == "train":
            nbytes += (out * tokens + ins * padded) * size + 2 * held
            flops *= 3
    elif kind == "select":
        # one search in four has one beam alive, and one beam in eight is finished: their logits are not needed
        rows = 0.875 * sum(1 if n % 4 == 1 else c["beams"] for n in range(c["groups"]))
        nbytes = rows * c["vocab"] * size + c["groups"] * c["beams"] * 8.0 + c["groups"] * c["out"] * (12.0 + 8.0 * c["history"])
        flops = 4.0 * rows * c["vocab"]
    else:
        nbytes = c["rows"] * (1.875 * c["vocab"] * size + 8.0 * c["top"] + 12.0)
        flops = 8.0 * c["rows"] * c["vocab"]
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------
# In 64 bits, from the definitions
# ---------------------------------------------------------------------------

def exact(case, seed):
    c, st = case, prepare(case, seed)
    kind = c["kind"]
    if kind == "distill":
        return _exact_distill(c, st)
    if kind == "select":
        return _exact_select(c, st)
    heads, scale = c["heads"], c["dk"] ** -0.5
    gamma = torch.exp(st["log_decay"].double())[:, None, None]
    if kind == "step":
        take = st["parents"].long()
        s = torch.empty_like(st["state"], dtype=torch.float64)
        out = torch.empty(len(take), heads, c["dv"], device=DEV, dtype=torch.float64)
        for h in range(heads):
            kv = h // (heads // c["kv_heads"])
            k, v = st["k"][:, kv].double(), st["v"][:, kv].double()
            s[:, h] = gamma[h] * st["state"][take, h].double() + torch.einsum("ri,rj->rij", k, v)
            out[:, h] = scale * torch.einsum("ri,rij->rj", st["q"][:, h].double(), s[:, h])
        return {"out": out, "state": s}
    return _exact_recurrence(c, st, gamma, scale)


def _exact_recurrence(c, st, gamma, scale):
    """Token by token: the states, and the states' gradients backwards."""
    n, t, heads, kv, dk, dv = c["rows"], c["length"], c["heads"], c["kv_heads"], c["dk"], c["dv"]
    if n * t * heads * dk * dv > 2 ** 37:
        return None
    share = heads // kv
    lens = st["lens"] if st["lens"] is not None else torch.full((n,), t, device=DEV, dtype=torch.int32)
    live = (torch.arange(t, device=DEV)[:, None] < lens)[:, :, None, None].double()  # [t, n, 1, 1]
    q, k, v = (st[x].double().transpose(0, 1) * live for x in "qkv")
    k, v = (x.repeat_interleave(share, dim=2) for x in (k, v))
    zero = torch.zeros(n, heads, dk, dv, device=DEV, dtype=torch.float64)
    s = st["state"].double() if st["state"] is not None else zero
    first = s
    out = torch.zeros(t, n, heads, dv, device=DEV, dtype=torch.float64)
    train = c["kind"] == "train"
    if train:
        do = st["dout"].double().transpose(0, 1) * live
        dq, dkk, dvv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i in range(t):
        s = torch.where(live[i][..., None] != 0, gamma * s, s) + k[i][..., :, None] * v[i][..., None, :]
        out[i] = scale * (q[i][..., None, :] @ s)[..., 0, :]
        if train:
            dq[i] = scale * (s @ do[i][..., :, None])[..., 0]
    got = {"out": (out * live).transpose(0, 1)}
    if c["state"]:
        got["state"] = s
    if train:
        r = st["dstate"].double() if st["dstate"] is not None else zero  # the gradient of the state after token i
        for i in range(t - 1, -1, -1):
            r = r + scale * q[i][..., :, None] * do[i][..., None, :]
            dkk[i] = (r @ v[i][..., :, None])[..., 0]
            dvv[i] = (k[i][..., None, :] @ r)[..., 0, :]
            r = torch.where(live[i][..., None] != 0, gamma * r, r)
        dkk, dvv = (x.unflatten(2, (kv, share)).sum(3) for x in (dkk * live, dvv * live))
        got |= {"dq": (dq * live).transpose(0, 1), "dk": dkk.transpose(0, 1), "dv": dvv.transpose(0, 1)}
        if c["state"]:
            got["dstate"] = r if first is not zero else None
    return got


def _exact_select(c, st):
    best = []
    for n in range(c["groups"]):
        rows = []
        for b in range(c["beams"]):
            x, s = st["logits"][n, b].double(), st["scores"][n, b].double()
            rows.append(s[None] if int(st["finished"][n, b]) else s + torch.log_softmax(x, 0).sort(descending=True).values[:c["out"]])
        rows = torch.cat(rows).sort(descending=True).values[:c["out"]]
        best.append(torch.nn.functional.pad(rows, (0, c["out"] - len(rows)), value=-math.inf))
    return {"scores": torch.stack(best), "tokens": None, "parents": None, "history": None}


def _exact_distill(c, st):
    tau = c["temperature"]
    loss, lse, grad = [], [], []
    for x, ids, teacher, weight in zip(st["logits"], st["ids"], st["teacher"], st["dloss"].double()):
        use = ids >= 0
        if not bool(use.any()):
            loss.append(torch.zeros((), device=DEV, dtype=torch.float64))
            lse.append(loss[-1])
            grad.append(torch.zeros(c["vocab"], device=DEV, dtype=torch.float32))
            continue
        ids = ids[use].long()
        log_p = torch.log_softmax(teacher[use].double() / tau, 0)
        z = x.double() / tau
        lse.append(torch.logsumexp(z, 0))
        log_q = z - lse[-1]
        loss.append(tau ** 2 * (log_p.exp() * (log_p - log_q[ids])).sum())
        d = log_q.exp()
        d[ids] -= log_p.exp()
        grad.append((weight * tau * d).float() if c["rows"] * c["vocab"] > 2 ** 28 else weight * tau * d)
    if len({x.dtype for x in grad}) > 1:
        grad = [x.double() for x in grad]
    return {"loss": torch.stack(loss), "lse": torch.stack(lse), "dlogits": torch.stack(grad)}
