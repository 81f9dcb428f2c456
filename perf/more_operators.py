"""The work whose speed the operators of a walk model's layers are measured by.

A layer of such a model joins the last layer's output to the residual stream and norms it, looks at
the tokens just before with a short convolution, and mixes the row with a selective scan, whose decays
the tokens themselves give. Each case is one pass through one of these, as a program calls it:

  conv        causal convolution over whole rows of tokens: outputs, states where ``state`` says so
  conv_train  the same forward and backward: outputs, states and every gradient
  conv_step   one more token per row, the states of the parents' rows taken over
  scan, scan_train, scan_step    the selective scan, likewise
  norm        residual, scale, dropout and norm: outputs
  norm_train  the same forward and backward

Rows are the repository's walk rows (2 * depth + 1 tokens, ragged), longer rows as walks laid end to
end give them, and beams of a search; widths are generic. Values are random: steps of the scan
between 0.001 and 0.1 as models begin with, rates from -1 to -states, dropout of a tenth.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # 64 beam searches of 8 beams: the convolution's part of a step.
        dict(name="conv_step_beams", kind="conv_step", type="bf16", groups=64, beams=8, channels=2048, width=4),
        # One long row, 1,177 walks end to end, the next part of it to come.
        dict(name="conv_long", kind="conv", type="bf16", rows=1, length=20_011, ragged=False, channels=2048, width=4,
             state=True),
        # Training on depth-8 walk rows in 32 bits: ragged, an odd number of channels.
        dict(name="conv_train_walks", kind="conv_train", type="f32", rows=4096, length=17, ragged=True, channels=408,
             width=3, state=False),
        # One walk extended by one token: latency is all there is to it.
        dict(name="scan_step_one", kind="scan_step", type="bf16", groups=1, beams=1, channels=256, groups_bc=1,
             states=16),
        # 64 beam searches of 8 beams extended by a token.
        dict(name="scan_step_beams", kind="scan_step", type="bf16", groups=64, beams=8, channels=2048, groups_bc=1,
             states=16),
        # Scoring of a batch of depth-8 walk rows: very many very short ragged rows.
        dict(name="scan_walks", kind="scan", type="bf16", rows=4000, length=17, ragged=True, channels=256, groups_bc=1,
             states=16, state=False),
        # One long row: little work side by side but the channels.
        dict(name="scan_long", kind="scan", type="bf16", rows=1, length=20_011, ragged=False, channels=2048,
             groups_bc=1, states=16, state=True),
        # Training on depth-16 walk rows in 32 bits: ragged, odd numbers of channels and states, two groups.
        dict(name="scan_train_walks", kind="scan_train", type="f32", rows=1024, length=33, ragged=True, channels=410,
             groups_bc=2, states=11, state=False),
        # Training on long rows, states carried from the rows before (truncated backpropagation).
        dict(name="scan_train_long", kind="scan_train", type="bf16", rows=4, length=4096, ragged=False, channels=2048,
             groups_bc=1, states=16, state=True),
        # The norm in front of a layer for the beams of one search: latency.
        dict(name="norm_one", kind="norm", type="bf16", stream="bf16", rows=8, length=1, ragged=False, channels=512,
             drop=0.0, center=False, affine=False),
        # Training on depth-8 walk rows: everything the call has, odd channels, 32 bits.
        dict(name="norm_train_walks", kind="norm_train", type="f32", stream="f32", rows=4096, length=17, ragged=True,
             channels=301, drop=0.1, center=True, affine=True),
        # Training on long rows: activations in 16 bits beside a residual stream in 32.
        dict(name="norm_train_long", kind="norm_train", type="bf16", stream="f32", rows=4, length=4096, ragged=False,
             channels=4096, drop=0.1, center=False, affine=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["conv", "conv_train", "conv_step", "scan", "scan_train", "scan", "scan_train", "scan_step", "norm",
                       "norm_train"])
    c = dict(kind=kind, type=rng.choice(["bf16", "f32"]))
    name = kind.split("_")[0]
    c["channels"] = rng.choice([_log(rng, 16, 2048), 64 * rng.randint(1, 32)])
    if name == "scan":
        c["groups_bc"] = rng.choice([1, 1, 2, 4])
        c["channels"] = max(1, c["channels"] // c["groups_bc"]) * c["groups_bc"]
        c["states"] = rng.choice([16, 16, _log(rng, 1, 64)])
    if name == "conv":
        c["width"] = rng.choice([4, 4, rng.randint(1, 8)])
    if kind.endswith("_step"):
        c["beams"] = rng.randint(1, 16)
        most = 2 ** 24 // (c["channels"] * c["beams"] * c.get("states", 1))  # states of at most 64 MB
        c["groups"] = _log(rng, 1, max(1, min(512, most)))
        return c
    c["length"] = _log(rng, 1, 16_384)
    most = 2 ** 25 // (c["channels"] * c["length"] * max(16, c.get("states", 1)) // 16)
    c["rows"] = _log(rng, 1, max(1, min(4096, most)))
    c["ragged"] = rng.random() < 0.5
    if name == "norm":
        c["stream"] = rng.choice([c["type"], "f32"])
        c["drop"] = rng.choice([0.0, 0.1, 0.5])
        c["center"], c["affine"] = rng.random() < 0.5, rng.random() < 0.5
    else:
        c["state"] = rng.random() < 0.5 and c["rows"] * c["channels"] * c.get("states", 1) <= 2 ** 24
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, g, kind=torch.float32):
    return torch.randn(shape, device=DEV, generator=g).to(kind)


def _parents(c, g):
    first = torch.arange(c["groups"], device=DEV, dtype=torch.int32)[:, None] * c["beams"]
    pick = torch.randint(0, c["beams"], (c["groups"], c["beams"]), device=DEV, generator=g, dtype=torch.int32)
    return (first + pick).flatten()


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"case": c}
    name, kind, d = c["kind"].split("_")[0], TYPES[c["type"]], c["channels"]
    step, train = c["kind"].endswith("_step"), c["kind"].endswith("_train")
    if step:
        lead = (c["groups"] * c["beams"],)
        st["parents"] = _parents(c, g)
        st["lens"] = None
    else:
        lead = (c["rows"], c["length"])
        st["lens"] = (torch.randint(0, c["length"] + 1, (c["rows"],), device=DEV, generator=g, dtype=torch.int32)
                      if c["ragged"] else None)
        if train:
            st["dout"] = _randn((*lead, d), g, kind)
    has_state = step or c.get("state", False)
    if name == "conv":
        # the scan's input and its gate come from one product
        st["x"] = _randn((*lead, 2 * d), g, kind)[..., :d]
        st["weight"] = _randn((d, c["width"]), g) * c["width"] ** -0.5
        st["bias"] = _randn((d,), g) * 0.1
        shape = (lead[0], c["width"] - 1, d)
        st["state"] = _randn(shape, g, kind) if has_state else None
        if train:
            st["dstate"] = _randn(shape, g, kind) if has_state else None
        if step:
            st["state_out"] = torch.empty(shape, device=DEV, dtype=kind)
    elif name == "scan":
        n, k = c["states"], c["groups_bc"]
        st["x"] = _randn((*lead, d), g, kind)
        st["dt"] = _randn((*lead, d), g, kind)
        st["gate"] = _randn((*lead, 2 * d), g, kind)[..., d:]
        bc = _randn((*lead, 2 * k * n), g, kind)
        st["b"], st["c"] = (y.unflatten(-1, (k, n)) for y in bc.split(k * n, dim=-1))
        st["a"] = -torch.arange(1, n + 1, device=DEV, dtype=torch.float32).repeat(d, 1)
        first = torch.exp(torch.rand(d, device=DEV, generator=g) * math.log(100.0) + math.log(0.001))
        st["dt_bias"] = first + torch.log(-torch.expm1(-first))  # its softplus is the step to begin with
        st["skip"] = torch.ones(d, device=DEV) + 0.1 * _randn((d,), g)
        shape = (lead[0], d, n)
        st["state"] = _randn(shape, g) if has_state else None
        if train:
            st["dstate"] = _randn(shape, g) if has_state else None
        if step:
            st["state_out"] = torch.empty(shape, device=DEV)
    else:
        st["x"] = _randn((*lead, d), g, kind)
        st["residual"] = _randn((*lead, d), g, TYPES[c["stream"]])
        st["weight"] = torch.ones(d, device=DEV) + 0.1 * _randn((d,), g)
        st["bias"] = 0.1 * _randn((d,), g) if c["affine"] else None
        st["scale"] = 0.5 + 0.1 * _randn((d,), g) if c["affine"] else None
        st["seed"] = seed * 1_000_003 + 12_345
        if train:
            st["dhidden"] = _randn((*lead, d), g, TYPES[c["stream"]])
    return st


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------

EPS = 1e-5


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _live(st, n, t):
    """[n, t, 1]: the tokens that count."""
    lens = st["lens"] if st["lens"] is not None else torch.full((n,), t, device=DEV, dtype=torch.int32)
    return (torch.arange(t, device=DEV) < lens[:, None])[..., None], lens.long()


def _plain_conv_step(st):
    width = st["case"]["width"]
    x = torch.cat((st["state"][st["parents"].long()], st["x"][:, None]), dim=1)
    pre = st["bias"] + (x.float() * st["weight"].T[:width]).sum(1)
    return {"out": (pre * _sigmoid(pre)).to(x.dtype), "state": x[:, 1:].contiguous()}


def _plain_conv(st, train):
    c = st["case"]
    n, t, d, width, kind = c["rows"], c["length"], c["channels"], c["width"], TYPES[c["type"]]
    live, lens = _live(st, n, t)
    before = st["state"].float() if st["state"] is not None else torch.zeros(n, width - 1, d, device=DEV)
    x = torch.cat((before, torch.where(live, st["x"].float(), 0.0)), dim=1)  # token i at width - 1 + i
    pre = st["bias"].expand(n, t, d)
    for j in range(width):
        pre = pre + st["weight"][:, j] * x[:, j:j + t]
    sig = _sigmoid(pre)
    got = {"out": torch.where(live, pre * sig, 0.0).to(kind)}
    last = (lens[:, None] + torch.arange(width - 1, device=DEV))[..., None].expand(n, width - 1, d)
    if c["state"]:
        got["state"] = x.gather(1, last).to(kind)
    if train:
        g = torch.where(live, st["dout"].float(), 0.0) * (sig * (1.0 + pre * (1.0 - sig)))
        dx = torch.zeros_like(x)
        if c["state"]:
            dx.scatter_add_(1, last, st["dstate"].float())
        dw = []
        for j in range(width):
            dx[:, j:j + t] += st["weight"][:, j] * g
            dw.append((g * x[:, j:j + t]).sum((0, 1), dtype=torch.float64))
        got["dx"] = dx[:, width - 1:].to(kind)
        got["dweight"] = torch.stack(dw, 1).float()
        got["dbias"] = g.sum((0, 1), dtype=torch.float64).float()
        if c["state"]:
            got["dstate"] = dx[:, :width - 1].to(kind)
    return got


def _softplus(x):
    return x.clamp(min=0.0) + torch.log1p(torch.exp(-x.abs()))


def _per_group(x, groups):
    """[..., channels] -> [..., groups, channels of a group, 1]"""
    return x.unflatten(-1, (groups, -1)).unsqueeze(-1)


def _plain_scan_step(st):
    c = st["case"]
    k = c["groups_bc"]
    x = st["x"].float()
    delta = _softplus(st["dt"].float() + st["dt_bias"])
    a = st["a"].unflatten(0, (k, -1))
    h = st["state"][st["parents"].long()].unflatten(1, (k, -1))
    h = torch.exp(_per_group(delta, k) * a) * h + _per_group(delta * x, k) * st["b"].float()[:, :, None]
    y = (h * st["c"].float()[:, :, None]).sum(-1).flatten(1) + st["skip"] * x
    z = st["gate"].float()
    return {"out": (y * (z * _sigmoid(z))).to(st["x"].dtype), "state": h.flatten(1, 2)}


def _plain_scan(st, train):
    """In chunks of about the root of the length: the chunks side by side token by token, each from zeros;
    from chunk to chunk; side by side again from where the chunks before have come to."""
    c = st["case"]
    n, t, d, k, states, kind = c["rows"], c["length"], c["channels"], c["groups_bc"], c["states"], TYPES[c["type"]]
    size = max(1, math.isqrt(t))
    m = -(-t // size)
    live, _ = _live(st, n, t)

    def chunks(v):
        v = torch.where(live if v.dim() == 3 else live[..., None], v.float(), 0.0)
        return torch.nn.functional.pad(v.flatten(2), (0, 0, 0, m * size - t)).unflatten(1, (m, size)).transpose(1, 2)

    def back(v):
        return v.transpose(1, 2).flatten(1, 2)[:, :t]

    a = st["a"].unflatten(0, (k, -1))
    x, z = chunks(st["x"]), chunks(st["gate"])                                  # [n, size, m, d]
    raw = st["dt"].float() + st["dt_bias"]
    delta = chunks(_softplus(raw))
    u = _per_group(delta * x, k)                                                # [n, size, m, k, d / k, 1]
    b, cc = (chunks(st[v]).unflatten(-1, (k, 1, states)) for v in "bc")         # [n, size, m, k, 1, states]
    per = _per_group(delta, k)
    whole = torch.exp(per.sum(1) * a)                                           # decays of chunks [n, m, k, d / k, states]
    h = torch.zeros(n, m, k, d // k, states, device=DEV)
    for i in range(size):
        h = torch.exp(per[:, i] * a) * h + u[:, i] * b[:, i]
    came = torch.empty_like(h)
    s = st["state"].unflatten(1, (k, -1)) if st["state"] is not None else torch.zeros_like(h[:, 0])
    for j in range(m):
        came[:, j] = s
        s = whole[:, j] * s + h[:, j]
    y, before, h = torch.empty(n, size, m, d, device=DEV), [], came
    for i in range(size):
        if train:
            before.append(h)
        h = torch.exp(per[:, i] * a) * h + u[:, i] * b[:, i]
        y[:, i] = (h * cc[:, i]).sum(-1).flatten(2)
    y = y + st["skip"] * x
    sig = _sigmoid(z)
    got = {"out": back(y * (z * sig)).to(kind)}
    if c["state"]:
        got["state"] = s.flatten(1, 2)
    if not train:
        return got
    do = chunks(st["dout"])
    g = do * (z * sig)
    pg = _per_group(g, k)
    q = torch.zeros_like(came)
    for i in range(size - 1, -1, -1):
        q = torch.exp(per[:, i] * a) * (pg[:, i] * cc[:, i] + q)
    r = st["dstate"].unflatten(1, (k, -1)) if c["state"] else torch.zeros_like(q[:, 0])
    after = torch.empty_like(q)
    for j in range(m - 1, -1, -1):
        after[:, j] = r
        r = whole[:, j] * r + q[:, j]
    ddelta, du = torch.empty_like(delta), torch.empty_like(delta)
    db, dc = (torch.empty(n, size, m, k, states, device=DEV) for _ in range(2))
    da = torch.zeros_like(came)
    q = after
    for i in range(size - 1, -1, -1):
        decay = torch.exp(per[:, i] * a)
        q = q + pg[:, i] * cc[:, i]                                             # the gradient of this token's state
        kept = decay * before.pop()
        db[:, i] = (q * u[:, i]).sum(-2)
        dc[:, i] = (pg[:, i] * (kept + u[:, i] * b[:, i])).sum(-2)
        du[:, i] = (q * b[:, i]).sum(-1).flatten(2)
        kept = q * kept
        ddelta[:, i] = (kept * a).sum(-1).flatten(2)
        da += kept * per[:, i]
        q = decay * q
    ddelta = torch.where(live, back(ddelta + x * du) * _sigmoid(raw), 0.0)
    got["dx"] = back(delta * du + st["skip"] * g).to(kind)
    got["ddt"] = ddelta.to(kind)
    got["da"] = da.sum((0, 1), dtype=torch.float64).float().flatten(0, 1)
    got["db"] = back(db).to(kind)
    got["dc"] = back(dc).to(kind)
    got["ddt_bias"] = ddelta.sum((0, 1), dtype=torch.float64).float()
    got["dskip"] = (g * x).sum((0, 1, 2), dtype=torch.float64).float()
    got["dgate"] = back(do * y * (sig * (1.0 + z * (1.0 - sig)))).to(kind)
    if c["state"]:
        got["dstate"] = r.flatten(1, 2)
    return got


def _kept(c, seed):
    """Philox4x32-10 words of (seed; channel / 4, token + 1, row): kept where not below the threshold."""
    n, t, d = c["rows"], c["length"], c["channels"]
    mask = 2 ** 32 - 1
    x0 = torch.arange(-(-d // 4), device=DEV).expand(n, t, -1)
    x1 = torch.arange(1, t + 1, device=DEV)[None, :, None].expand_as(x0)
    x2 = torch.arange(n, device=DEV)[:, None, None].expand_as(x0)
    x3 = torch.zeros_like(x0)
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p, q = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = ((q >> 32) & mask) ^ x1 ^ k0, q & mask, ((p >> 32) & mask) ^ x3 ^ k1, p & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack((x0, x1, x2, x3), dim=-1).flatten(2)[..., :d]
    return words >= round(c["drop"] * 2 ** 32)


def _plain_norm(st, train):
    c = st["case"]
    n, t, d, kind, stream = c["rows"], c["length"], c["channels"], TYPES[c["type"]], TYPES[c["stream"]]
    live, _ = _live(st, n, t)
    part = torch.where(live, st["x"].float(), 0.0)
    if c["drop"]:
        factor = torch.where(_kept(c, st["seed"]), 1.0 / (1.0 - c["drop"]), 0.0)
        part = part * factor
    hidden = part * st["scale"] if st["scale"] is not None else part
    hidden = torch.where(live, hidden + st["residual"].float(), 0.0)
    centred = hidden - hidden.mean(-1, keepdim=True) if c["center"] else hidden
    inv = 1.0 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    normed = centred * inv
    out = normed * st["weight"]
    if st["bias"] is not None:
        out = out + st["bias"]
    got = {"out": torch.where(live, out, 0.0).to(kind), "hidden": hidden.to(stream)}
    if train:
        do = torch.where(live, st["dout"].float(), 0.0)
        got["dweight"] = (do * normed).sum((0, 1), dtype=torch.float64).float()
        if st["bias"] is not None:
            got["dbias"] = do.sum((0, 1), dtype=torch.float64).float()
        do = do * st["weight"]
        dh = do - normed * (do * normed).mean(-1, keepdim=True)
        if c["center"]:
            dh = dh - do.mean(-1, keepdim=True)
        dh = torch.where(live, dh * inv + st["dhidden"].float(), 0.0)
        got["dresidual"] = dh.to(stream)
        if st["scale"] is not None:
            got["dscale"] = (dh * part).sum((0, 1), dtype=torch.float64).float()
            dh = dh * st["scale"]
        got["dx"] = (dh * factor if c["drop"] else dh).to(kind)
    return got


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    st, c = state, state["case"]
    name, _, form = c["kind"].partition("_")
    if not own:
        if form == "step":
            return _plain_conv_step(st) if name == "conv" else _plain_scan_step(st)
        return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[name](st, form == "train")
    import paper_2508_01073_amd as rd
    if name == "conv":
        if form == "step":
            out, new = rd.rdf2v_causal_conv_step(st["x"], st["weight"], st["bias"], st["state"],
                                                 parents=st["parents"], state_out=st["state_out"])
            return {"out": out, "state": new}
        out, new = rd.rdf2v_causal_conv(st["x"], st["weight"], st["bias"], lens=st["lens"], state=st["state"],
                                        want_state=c["state"])
        got = {"out": out, "state": new} if c["state"] else {"out": out}
        if form == "train":
            dx, dweight, dbias, dstate = rd.rdf2v_causal_conv_backward(
                st["x"], st["weight"], st["bias"], st["dout"], lens=st["lens"], state=st["state"],
                dstate_out=st["dstate"])
            got |= {"dx": dx, "dweight": dweight, "dbias": dbias}
            if c["state"]:
                got["dstate"] = dstate
        return got
    if name == "scan":
        given = dict(dt_bias=st["dt_bias"], skip=st["skip"], gate=st["gate"])
        if form == "step":
            out, new = rd.rdf2v_selective_scan_step(st["x"], st["dt"], st["a"], st["b"], st["c"], st["state"],
                                                    parents=st["parents"], state_out=st["state_out"], **given)
            return {"out": out, "state": new}
        given |= dict(lens=st["lens"], state=st["state"])
        out, new = rd.rdf2v_selective_scan(st["x"], st["dt"], st["a"], st["b"], st["c"], want_state=c["state"], **given)
        got = {"out": out, "state": new} if c["state"] else {"out": out}
        if form == "train":
            grads = rd.rdf2v_selective_scan_backward(st["x"], st["dt"], st["a"], st["b"], st["c"], st["dout"],
                                                     dstate_out=st["dstate"], **given)
            got |= {k: v for k, v in grads._asdict().items() if v is not None}
        return got
    given = dict(scale=st["scale"], drop=c["drop"], seed=st["seed"], center=c["center"], eps=EPS, lens=st["lens"])
    out, hidden, stats = rd.rdf2v_residual_norm(st["x"], st["residual"], st["weight"], st["bias"], **given)
    got = {"out": out, "hidden": hidden}
    if form == "train":
        grads = rd.rdf2v_residual_norm_backward(st["x"], st["residual"], st["weight"], st["bias"], stats, st["dout"],
                                                dhidden=st["dhidden"], **given)
        got |= {k: v for k, v in grads._asdict().items() if v is not None}
    return got


def work(case):
    """Each input once, each output once; the operations of the formulas."""
    c = case
    name, _, form = c["kind"].partition("_")
    size, d = 2 if c["type"] == "bf16" else 4, c["channels"]
    if form == "step":
        tokens = padded = c["groups"] * c["beams"]
        # of a step's parents some are taken more than once, and others not at all
        taken = 1.0 - (1.0 - 1.0 / c["beams"]) ** c["beams"]
    else:
        padded = c["rows"] * c["length"]
        tokens = padded * (0.5 if c["ragged"] else 1.0)
        taken = 1.0
    train = form == "train"
    if name == "conv":
        held = c.get("state", form == "step") * (tokens if form == "step" else c["rows"]) * (c["width"] - 1) * d * size
        nbytes = (tokens + padded) * d * size + held * (1.0 + taken) + d * (c["width"] + 1) * 4.0
        flops = tokens * d * (2.0 * c["width"] + 6.0)
        if train:
            nbytes += (tokens + padded) * d * size + 2 * held + d * (c["width"] + 1) * 4.0
            flops += tokens * d * (6.0 * c["width"] + 10.0)
    elif name == "scan":
        n, k = c["states"], c["groups_bc"]
        held = c.get("state", form == "step") * (tokens if form == "step" else c["rows"]) * n * d * 4.0
        nbytes = (3 * tokens + padded) * d * size + 2 * k * n * tokens * size + held * (1.0 + taken) + d * (n + 2) * 4.0
        flops = tokens * d * (7.0 * n + 12.0)
        if train:
            nbytes += (tokens + 3 * padded) * d * size + 2 * k * n * padded * size + 2 * held + d * (n + 2) * 4.0
            flops += tokens * d * (20.0 * n + 24.0)
    else:
        wide = 2 if c["stream"] == "bf16" else 4
        nbytes = (tokens + padded) * d * (size + wide) + d * 4.0
        flops = tokens * d * 8.0
        if train:
            nbytes += (tokens + padded) * d * (size + wide) + d * 4.0
            flops += tokens * d * 16.0
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------
# In 64 bits, from the definitions
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    name, _, form = case["kind"].partition("_")
    # a step is a row of one token that goes on from its parent's state
    if form == "step":
        c = dict(case, rows=case["groups"] * case["beams"], length=1, state=True)
        st["state"] = st["state"][st["parents"].long()]
        for k in ("x", "dt", "gate", "b", "c"):
            if k in st:
                st[k] = st[k][:, None]
    else:
        c = case
    got = {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm}[name](c, st, form == "train")
    if got is not None and form == "step":
        got["out"] = got["out"][:, 0]
    return got


def _swish(v):
    s = torch.sigmoid(v)
    return v * s, s + v * s * (1.0 - s)


def _exact_conv(c, st, train):
    """Row by row with the tokens that count, several rows of one length at once."""
    n, t, d, width = c["rows"], c["length"], c["channels"], c["width"]
    w, bias = st["weight"].double(), st["bias"].double()
    lens = [t] * n if st["lens"] is None else st["lens"].tolist()
    new = lambda *s: torch.zeros(s, device=DEV, dtype=torch.float64)  # noqa: E731
    got = {"out": new(n, t, d), "state": new(n, width - 1, d)}
    if train:
        got |= {"dx": new(n, t, d), "dweight": new(d, width), "dbias": new(d), "dstate": new(n, width - 1, d)}
    for length in sorted(set(lens)):
        at = torch.tensor([i for i, v in enumerate(lens) if v == length], device=DEV)
        old = st["state"][at].double() if st["state"] is not None else new(len(at), width - 1, d)
        seq = torch.cat((old, st["x"][at, :length].double()), 1)
        got["state"][at] = seq[:, length:]
        dseq = torch.zeros_like(seq)
        if train and st["dstate"] is not None:
            dseq[:, length:] += st["dstate"][at].double()
        if length:
            near = seq.unfold(1, width, 1)                          # [rows, length, d, width]
            act, slope = _swish((near * w).sum(-1) + bias)
            got["out"][at, :length] = act
            if train:
                grad = st["dout"][at, :length].double() * slope
                got["dweight"] += (grad[..., None] * near).sum((0, 1))
                got["dbias"] += grad.sum((0, 1))
                for j in range(width):
                    dseq[:, j:j + length] += grad * w[:, j]
        if train:
            got["dx"][at, :length] = dseq[:, width - 1:]
            got["dstate"][at] = dseq[:, :width - 1]
    if not c["state"]:
        got.pop("state")
        got.pop("dstate", None)
    return got


def _exact_scan(c, st, train):
    """Token by token: the states, and the states' gradients backwards."""
    n, t, d, k, states = c["rows"], c["length"], c["channels"], c["groups_bc"], c["states"]
    if t * n * d * states * (2 if train else 1) > 2 ** 31 or t > 30_000:
        return None
    lens = st["lens"] if st["lens"] is not None else torch.full((n,), t, device=DEV)
    a, bias, skip = st["a"].double(), st["dt_bias"].double(), st["skip"].double()
    wide = lambda v: v.double().repeat_interleave(d // k, dim=1)  # noqa: E731
    h = st["state"].double() if st["state"] is not None else torch.zeros(n, d, states, device=DEV, dtype=torch.float64)
    tokens = lambda *s: torch.zeros(n, t, *s, device=DEV, dtype=torch.float64)  # noqa: E731
    got, saved, ys = {"out": tokens(d)}, [], []
    for i in range(t):
        on = (lens > i)[:, None]
        x, z = (torch.where(on, st[v][:, i].double(), 0.0) for v in ("x", "gate"))
        step = torch.where(on, torch.nn.functional.softplus(st["dt"][:, i].double() + bias, threshold=50.0), 0.0)
        b, cc = (torch.where(on[..., None], wide(st[v][:, i]), 0.0) for v in "bc")
        if train:
            saved.append(h)
        h = torch.exp(step[..., None] * a) * h + (step * x)[..., None] * b
        y = (h * cc).sum(-1) + skip * x
        ys.append(y if train else None)
        got["out"][:, i] = y * _swish(z)[0]
    if c["state"]:
        got["state"] = h
    if not train:
        return got
    r = st["dstate"].double() if c["state"] else torch.zeros_like(h)
    got |= {"dx": tokens(d), "ddt": tokens(d), "da": torch.zeros_like(a), "db": tokens(k, states),
            "dc": tokens(k, states), "ddt_bias": torch.zeros_like(bias), "dskip": torch.zeros_like(skip),
            "dgate": tokens(d)}
    for i in range(t - 1, -1, -1):
        on = (lens > i)[:, None]
        x, z, do = (torch.where(on, st[v][:, i].double(), 0.0) for v in ("x", "gate", "dout"))
        raw = st["dt"][:, i].double() + bias
        step = torch.where(on, torch.nn.functional.softplus(raw, threshold=50.0), 0.0)
        b, cc = (torch.where(on[..., None], wide(st[v][:, i]), 0.0) for v in "bc")
        act, slope = _swish(z)
        g = do * act
        got["dgate"][:, i] = do * ys.pop() * slope
        decay, old = torch.exp(step[..., None] * a), saved.pop()
        h = decay * old + (step * x)[..., None] * b
        r = r + g[..., None] * cc
        got["dc"][:, i] = (g[..., None] * h).unflatten(1, (k, -1)).sum(2)
        got["db"][:, i] = ((step * x)[..., None] * r).unflatten(1, (k, -1)).sum(2)
        got["dx"][:, i] = step * (r * b).sum(-1) + skip * g
        dstep = (r * (a * decay * old + x[..., None] * b)).sum(-1) * torch.where(on, torch.sigmoid(raw), 0.0)
        got["ddt"][:, i] = dstep
        got["ddt_bias"] += dstep.sum(0)
        got["dskip"] += (g * x).sum(0)
        got["da"] += (r * step[..., None] * decay * old).sum(0)
        r = decay * r
    if c["state"]:
        got["dstate"] = r
    return got


def _exact_mask(c, seed, rows):
    """The factors that dropout leaves, by numpy's 64-bit products."""
    import numpy as np
    t, d, m = c["length"], c["channels"], np.uint64(0xFFFFFFFF)
    shape = (len(rows), t, -(-d // 4))
    ctr = [np.broadcast_to(v, shape).astype(np.uint64) for v in
           (np.arange(shape[2])[None, None, :], np.arange(1, t + 1)[None, :, None], np.asarray(rows)[:, None, None], 0)]
    key = [np.uint64(seed % 2 ** 32), np.uint64(seed // 2 ** 32 % 2 ** 32)]
    for _ in range(10):
        one, two = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(two >> np.uint64(32)) ^ ctr[1] ^ key[0], two & m, (one >> np.uint64(32)) ^ ctr[3] ^ key[1], one & m]
        key = [(key[0] + np.uint64(0x9E3779B9)) & m, (key[1] + np.uint64(0xBB67AE85)) & m]
    below = np.stack(ctr, -1).reshape(len(rows), t, -1)[..., :d] < np.uint64(round(c["drop"] * 2 ** 32))
    return torch.from_numpy(np.where(below, 0.0, 1.0 / (1.0 - c["drop"]))).to(DEV)


def _exact_norm(c, st, train):
    n, t, d = c["rows"], c["length"], c["channels"]
    weight = st["weight"].double()
    scale = st["scale"].double() if st["scale"] is not None else torch.ones_like(weight)
    bias = st["bias"].double() if st["bias"] is not None else torch.zeros_like(weight)
    lens = st["lens"] if st["lens"] is not None else torch.full((n,), t, device=DEV)
    wide = lambda: torch.zeros(n, t, d, device=DEV, dtype=torch.float64)  # noqa: E731
    got = {"out": wide(), "hidden": wide()}
    if train:
        got |= {"dweight": torch.zeros_like(weight), "dbias": torch.zeros_like(weight), "dresidual": wide(),
                "dscale": torch.zeros_like(weight), "dx": wide()}
    per = max(1, 2 ** 23 // (t * d))
    for first in range(0, n, per):
        rows = range(first, min(n, first + per))
        at = slice(rows.start, rows.stop)
        on = (torch.arange(t, device=DEV) < lens[at, None])[..., None].double()
        kept = _exact_mask(c, st["seed"], list(rows)) if c["drop"] else torch.ones(len(rows), t, d, device=DEV, dtype=torch.float64)
        x = st["x"][at].double() * kept
        h = (st["residual"][at].double() + scale * x) * on
        mid = h - h.mean(-1, keepdim=True) * float(c["center"])
        std = torch.sqrt((mid ** 2).mean(-1, keepdim=True) + EPS)
        got["hidden"][at] = h
        got["out"][at] = (mid / std * weight + bias) * on
        if train:
            do = st["dout"][at].double() * on
            got["dweight"] += (do * mid / std).sum((0, 1))
            got["dbias"] += do.sum((0, 1))
            dn = do * weight
            dm = dn / std - mid * (dn * mid).sum(-1, keepdim=True) / (d * std ** 3)
            dm = dm - dm.mean(-1, keepdim=True) * float(c["center"])
            dh = (dm + st["dhidden"][at].double()) * on
            got["dresidual"][at] = dh
            got["dscale"] += (dh * x).sum((0, 1))
            got["dx"][at] = dh * scale * kept
    if train and st["scale"] is None:
        got.pop("dscale")
    if train and st["bias"] is None:
        got.pop("dbias")
    return got
