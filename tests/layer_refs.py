"""Plain implementations in 64 bits of the operators of a model's layers, from their definitions, on the CPU,
and the error bounds that the kernels are held to.

Bounds count roundings (see model_refs): each function also runs on absolute values (`absolute`), where every
term of its sums is taken by its size. A result is then off by at most its number of roundings, in units of
2^-24, times that size, and by half a step of its type where it is rounded to bfloat16."""

import torch

from model_refs import U32, UBF16


def _f64(*xs):
    return [None if x is None else x.detach().double().cpu() for x in xs]


def _live(lens, n, t):
    lens = torch.full((n,), t) if lens is None else lens.cpu().long()
    return torch.arange(t) < lens[:, None], lens


def conv(x, weight, bias=None, silu=True, lens=None, state=None, dout=None, dstate_out=None, absolute=False):
    """Returns a dict of out, state and, with dout, the gradients."""
    x, w, bias, state, dout, dstate_out = _f64(x, weight, bias, state, dout, dstate_out)
    n, t, d = x.shape
    width = w.shape[1]
    live, lens = _live(lens, n, t)
    bias = torch.zeros(d, dtype=torch.float64) if bias is None else bias
    state = torch.zeros(n, width - 1, d, dtype=torch.float64) if state is None else state
    if absolute:
        x, w, bias, state = x.abs(), w.abs(), bias.abs(), state.abs()
    got = {"out": torch.zeros(n, t, d, dtype=torch.float64), "state": torch.zeros_like(state)}
    grads = dout is not None
    if grads:
        got |= {"dx": torch.zeros_like(x), "dweight": torch.zeros_like(w), "dbias": torch.zeros_like(bias),
                "dstate": torch.zeros_like(state)}
    for r in range(n):
        length = int(lens[r])
        seq = torch.cat((state[r], x[r, :length]))
        got["state"][r] = seq[length:]
        dseq = torch.zeros_like(seq)
        if grads and dstate_out is not None:
            dseq[length:] += dstate_out[r].abs() if absolute else dstate_out[r]
        for i in range(length):
            near = seq[i:i + width]                                  # [width, d]
            u = bias + (w.T * near).sum(0)
            s = torch.sigmoid(u)
            slope = s * (1 + u * (1 - s)) if silu else torch.ones_like(u)
            if absolute:
                slope = 1.1 + u if silu else slope                   # and what an error of u does to it
            got["out"][r, i] = u * s if silu and not absolute else u
            if grads:
                g = (dout[r, i].abs() if absolute else dout[r, i]) * slope
                got["dweight"] += (g * near).T
                got["dbias"] += g
                dseq[i:i + width] += w.T * g
        if grads:
            got["dstate"][r] = dseq[:width - 1]
            got["dx"][r, :length] = dseq[width - 1:]
    return got


def scan(x, dt, a, b, c, dt_bias=None, skip=None, gate=None, lens=None, state=None, dout=None, dstate_out=None,
         absolute=False):
    """Token by token. Returns a dict of out, state and, with dout, the gradients."""
    x, dt, a, b, c, dt_bias, skip, gate, state, dout, dstate_out = _f64(x, dt, a, b, c, dt_bias, skip, gate, state,
                                                                         dout, dstate_out)
    n, t, d = x.shape
    groups, states = b.shape[-2:]
    live = _live(lens, n, t)[0]
    mask = lambda v: torch.where(live.reshape(n, t, *[1] * (v.dim() - 2)), v, 0.0)        # noqa: E731
    raw = mask(dt) + (0.0 if dt_bias is None else dt_bias)
    step = mask(raw.clamp(min=0) + torch.log1p(torch.exp(-raw.abs())))
    sig = mask(1 / (1 + torch.exp(-raw)))
    x, b, c = mask(x), mask(b), mask(c)
    skip = torch.zeros(d, dtype=torch.float64) if skip is None else skip
    if gate is None:
        act, slope = torch.ones_like(x), torch.zeros_like(x)
    else:
        z = mask(gate)
        s = 1 / (1 + torch.exp(-z))
        act, slope = z * s, s * (1 + z * (1 - s))
    h = torch.zeros(n, d, states, dtype=torch.float64) if state is None else state
    do = None if dout is None else mask(dout)
    size = a
    if absolute:
        x, b, c, skip, act, slope, h, size = (v.abs() for v in (x, b, c, skip, act, slope, h, a))
        slope = slope + 1.0
        do = None if do is None else do.abs()
        dstate_out = None if dstate_out is None else dstate_out.abs()
    wide = lambda v: v.repeat_interleave(d // groups, 1)                                   # noqa: E731
    out, kept, hs, ys = torch.zeros_like(x), [], [], []
    for i in range(t):
        k = torch.exp(step[:, i, :, None] * a) * h
        h = k + (step[:, i] * x[:, i])[..., None] * wide(b[:, i])
        y = (h * wide(c[:, i])).sum(-1) + skip * x[:, i]
        out[:, i] = y * act[:, i]
        kept.append(k)
        hs.append(h)
        ys.append(y)
    got = {"out": mask(out), "state": h}
    if dout is None:
        return got
    r = torch.zeros_like(h) if dstate_out is None else dstate_out
    got |= {"dx": torch.zeros_like(x), "ddt": torch.zeros_like(x), "da": torch.zeros_like(a), "db": torch.zeros_like(b),
            "dc": torch.zeros_like(c), "ddt_bias": torch.zeros(d, dtype=torch.float64),
            "dskip": torch.zeros(d, dtype=torch.float64), "dgate": torch.zeros_like(x)}
    for i in range(t - 1, -1, -1):
        g = do[:, i] * act[:, i]
        got["dgate"][:, i] = do[:, i] * ys[i] * slope[:, i]
        r = r + g[..., None] * wide(c[:, i])
        got["db"][:, i] = (r * (step[:, i] * x[:, i])[..., None]).unflatten(1, (groups, -1)).sum(2)
        got["dc"][:, i] = (g[..., None] * hs[i]).unflatten(1, (groups, -1)).sum(2)
        du = (r * wide(b[:, i])).sum(-1)
        got["dx"][:, i] = step[:, i] * du + skip * g
        ddt = ((r * kept[i] * size).sum(-1) + x[:, i] * du) * sig[:, i]
        got["ddt"][:, i] = ddt
        got["ddt_bias"] += mask(ddt[:, None].expand(n, t, d))[:, i].sum(0)
        got["dskip"] += (g * x[:, i]).sum(0)
        got["da"] += (r * kept[i] * step[:, i, :, None]).sum(0)
        r = torch.exp(step[:, i, :, None] * a) * r
    for name in ("dx", "ddt", "db", "dc", "dgate"):
        got[name] = mask(got[name])
    got["dstate"] = r
    return got


def kept(rows, length, channels, drop, seed, row_begin=0):
    """The mask of dropout, word by word, from the published generator."""
    m = 2 ** 32 - 1
    out = torch.ones(rows, length, channels, dtype=torch.bool)
    limit = round(drop * 2 ** 32)
    for r in range(rows):
        for t in range(length):
            for block in range((channels + 3) // 4):
                x = [block, t + 1, (row_begin + r) & m, (row_begin + r) >> 32]
                k = [seed & m, seed >> 32 & m]
                for _ in range(10):
                    p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
                    x = [q >> 32 ^ x[1] ^ k[0], q & m, p >> 32 ^ x[3] ^ k[1], p & m]
                    k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
                for j in range(min(4, channels - 4 * block)):
                    out[r, t, 4 * block + j] = x[j] >= limit
    return out


def norm(x, residual, weight, bias=None, scale=None, mask=None, drop=0.0, center=False, eps=1e-5, lens=None, dout=None,
         dhidden=None, absolute=False):
    """mask: kept(...), where drop is not 0. Returns a dict of out, hidden, stats and, with dout, the gradients."""
    x, residual, w, bias, scale, dout, dhidden = _f64(x, residual, weight, bias, scale, dout, dhidden)
    n, t, d = x.shape
    live = _live(lens, n, t)[0][..., None]
    clean = lambda v: torch.where(live, v, 0.0)                                            # noqa: E731
    factor = torch.ones_like(x) if mask is None else mask.double() / (1 - drop)
    part = clean(torch.where(factor == 0, 0.0, x) * factor)
    scale = torch.ones(d, dtype=torch.float64) if scale is None else scale
    bias = torch.zeros(d, dtype=torch.float64) if bias is None else bias
    residual = torch.zeros_like(x) if residual is None else clean(residual)
    hidden = residual + scale * part
    mean = hidden.mean(-1, keepdim=True) * float(center)
    inv = 1 / torch.sqrt(((hidden - mean) ** 2).mean(-1, keepdim=True) + eps)
    if absolute:
        part, scale, residual, w, bias = (v.abs() for v in (part, scale, residual, w, bias))
        hidden = residual + scale * part
        mean = -hidden.mean(-1, keepdim=True) * float(center)                              # taken off: added
    normed = (hidden - mean) * inv
    got = {"out": clean(normed * w + bias), "hidden": hidden, "stats": clean(torch.cat((mean.abs() if absolute else mean,
                                                                                        inv), -1))}
    if dout is None:
        return got
    do = clean(dout)
    dhidden = torch.zeros_like(x) if dhidden is None else clean(dhidden)
    if absolute:
        do, dhidden = do.abs(), dhidden.abs()
    sign = -1.0 if absolute else 1.0
    dn = do * w
    dh = dn - sign * normed * (dn * normed).mean(-1, keepdim=True) - sign * float(center) * dn.mean(-1, keepdim=True)
    dh = clean(dh * inv + dhidden)
    return got | {"dx": dh * scale * factor, "dresidual": dh, "dweight": (do * clean(normed)).sum((0, 1)),
                  "dbias": do.sum((0, 1)), "dscale": (dh * part).sum((0, 1))}


def conv_roundings(t, width, rows):
    """u sums width + 1 products; the sigmoid, its slope and their products take 16 more; a gradient sums width of
    them, a parameter's all tokens' (a double's at the end, at most the tokens of a row for each thread)."""
    return {"token": 2 * width + 24, "sum": 2 * width + 24 + t * rows}


def scan_roundings(t, states, channels, rows):
    """delta is good to 8 units, and a decay exp(delta a) to 3 + 9 |delta a|, so that products of decays, which fall
    faster than that grows, are off by 4 units and 3 a token; states round twice a token, outputs sum `states`
    products, gradients of b and c a group's channels, those of parameters all tokens; gates take 16."""
    base = 2 * (6 * t + states + 48)
    return {"token": base, "channels": base + channels, "sum": base + t * rows}


def norm_roundings(d, tokens):
    """Sums over d channels (twice, where the mean is taken off), each used in a factor or a difference; parameters'
    gradients sum all tokens."""
    return {"token": 4 * d + 48, "sum": 4 * d + 48 + tokens}


def bounds(ref, sizes, kinds, type_, exact_types=()):
    """kinds: name -> number of roundings. Results in `type_` are rounded to it at the end but for `exact_types`
    (float32 whatever the type)."""
    found = {}
    for name, x in ref.items():
        tol = kinds[name] * U32 * sizes[name] + 1e-30
        if type_ == torch.bfloat16 and name not in exact_types:
            tol = tol + 1.01 * UBF16 * (x.abs() + tol)
        found[name] = tol
    return found
