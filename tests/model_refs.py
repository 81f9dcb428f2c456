"""Plain implementations in 64 bits of the operators over walk tokens, from their definitions, on the
CPU, and the error bounds that the kernels are held to.

Bounds count roundings: u = 2^-24 is the relative error of one float32 operation, b = 2^-8 that of a
rounding to bfloat16. A sum of n products computed in any order in float32 is off by at most (n + 1) u
times the sum of the products' absolute values, which the same implementation gives when it is run on
absolute values."""

import math

import torch

U32 = 2.0 ** -24
UBF16 = 2.0 ** -8


def attention(q, k, v, log_decay, scale, lens=None, state=None, dout=None, dstate_out=None):
    """Decay attention token by token. Returns a dict of out, state and, with dout, the gradients."""
    q, k, v = (x.double().cpu() for x in (q, k, v))
    n, t, heads, dk = q.shape
    kv, dv = v.shape[-2:]
    share = heads // kv
    gamma = torch.exp(log_decay.double().cpu().clamp(min=-1e4))[:, None, None]
    lens = torch.full((n,), t) if lens is None else lens.cpu().long()
    live = (torch.arange(t)[:, None] < lens)                                     # [t, n]
    mask = lambda x: torch.where(live.T[:, :, None, None], x, 0.0)               # noqa: E731
    q, k, v = mask(q), mask(k), mask(v)
    k, v = (x.repeat_interleave(share, 2) for x in (k, v))
    s = torch.zeros(n, heads, dk, dv, dtype=torch.float64) if state is None else state.double().cpu()
    out = torch.zeros(n, t, heads, dv, dtype=torch.float64)
    grad = dout is not None
    if grad:
        do = mask(dout.double().cpu())
        dq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i in range(t):
        on = live[i][:, None, None, None]
        s = torch.where(on, gamma * s + k[:, i, :, :, None] * v[:, i, :, None, :], s)
        out[:, i] = torch.where(on[..., 0], scale * (q[:, i, :, :, None] * s).sum(-2), 0.0)
        if grad:
            dq[:, i] = torch.where(on[..., 0], scale * (s * do[:, i, :, None, :]).sum(-1), 0.0)
    got = {"out": out, "state": s}
    if grad:
        r = torch.zeros_like(s) if dstate_out is None else dstate_out.double().cpu()
        for i in range(t - 1, -1, -1):
            on = live[i][:, None, None, None]
            r = r + scale * q[:, i, :, :, None] * do[:, i, :, None, :]
            gk[:, i] = torch.where(on[..., 0], (r * v[:, i, :, None, :]).sum(-1), 0.0)
            gv[:, i] = torch.where(on[..., 0], (r * k[:, i, :, :, None]).sum(-2), 0.0)
            r = torch.where(on, gamma * r, r)
        got |= {"dq": dq, "dk": gk.unflatten(2, (kv, share)).sum(3), "dv": gv.unflatten(2, (kv, share)).sum(3),
                "dstate": r}
    return got


def attention_bounds(ref, sizes, type_, share=1):
    """Bounds of the errors of attention()'s results, given `sizes`, its results on absolute values.

    In float32 a result is a sum of at most t + max(dk, dv) products of up to four factors. A factor's
    decay, exp(n g), is off by at most 3 u for the function, and 3 u n |g| for its argument, where
    n |g| exp(-n |g|) is at most 1 / e; a state carried over chunks or tokens is rounded, and its decay
    multiplied, once a token at most: 3 u a token. Together (4 t + d + 32) u.
    In bfloat16 a product's weights and the states may be rounded once to be operands, b each (they weigh
    disjoint terms), and the result once, b. States are summed in float32 from operands that keep 24 bits."""
    t, d = ref["out"].shape[1], max(ref["state"].shape[-2:])
    f32 = (4 * t + d + 32 + share) * U32
    found = {}
    for name, x in ref.items():
        tol = f32 * sizes[name] + 1e-30
        if type_ == torch.bfloat16 and "state" not in name:
            tol = tol + 1.01 * UBF16 * (sizes[name] + x.abs())
        found[name] = tol
    return found


def beam_select(logits, scores, num_out, finished=None):
    """(totals [groups, num_out] float64, all totals [groups, beams * vocab] float64)."""
    x = logits.double().cpu()
    x = torch.where(x < math.inf, x, -math.inf)                                   # NaN and +inf too
    groups, beams, vocab = x.shape
    s = scores.double().cpu()
    s = torch.where(torch.isnan(s), -math.inf, s)
    lse = torch.logsumexp(x, -1, keepdim=True)
    total = s[..., None] + torch.where(x == -math.inf, -math.inf, x - lse)
    if finished is not None:
        end = torch.full_like(total, -math.inf)
        end[..., 0] = s
        total = torch.where(finished.cpu()[..., None] != 0, end, total)
    total = total.flatten(1)
    best = total.sort(dim=1, descending=True, stable=True).values[:, :num_out]
    return torch.nn.functional.pad(best, (0, num_out - best.shape[1]), value=-math.inf), total


def distill(logits, ids, teacher, tau, dloss=None):
    """(loss, lse, dlogits or None) in float64, row by row."""
    z, t = logits.double().cpu() / tau, teacher.double().cpu() / tau
    ids = ids.cpu().long()
    rows, vocab = z.shape
    loss, lse = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    grad = None if dloss is None else torch.zeros(rows, vocab, dtype=torch.float64)
    for r in range(rows):
        use = (ids[r] >= 0) & (ids[r] < vocab) & (t[r] != -math.inf)
        if not bool(use.any()):
            continue
        at, log_p = ids[r][use], torch.log_softmax(t[r][use], 0)
        p = log_p.exp()
        lse[r] = torch.logsumexp(z[r], 0)
        log_q = torch.where(z[r] == -math.inf, -math.inf, z[r] - lse[r])
        loss[r] = tau ** 2 * (p * (log_p - log_q[at])).sum()
        if dloss is not None:
            d = log_q.exp()
            d.index_add_(0, at, -p)
            grad[r] = float(dloss[r]) * tau * d
    return loss, lse, grad
