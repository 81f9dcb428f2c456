"""The causal convolution of many rows at once in 64 bits, on whatever device its inputs are: layer_refs goes through
rows and tokens one by one, which takes too long for as many as a workgroup goes round with."""

import torch


def conv(x, weight, bias, silu, lens, state, dout, dstate_out, absolute=False):
    """As layer_refs.conv with all of its arguments given."""
    x, w, bias, state, dout, dstate_out = (v.detach().double() for v in (x, weight, bias, state, dout, dstate_out))
    n, t, d = x.shape
    width = w.shape[1]
    live = (torch.arange(t, device=x.device) < lens[:, None])[..., None]
    x, dout = torch.where(live, x, 0.0), torch.where(live, dout, 0.0)
    if absolute:
        x, w, bias, state, dout, dstate_out = (v.abs() for v in (x, w, bias, state, dout, dstate_out))
    seq = torch.cat((state, x), 1)
    u = bias + sum(w[:, j] * seq[:, j:j + t] for j in range(width))
    s = torch.sigmoid(u)
    slope = s * (1 + u * (1 - s)) if silu else torch.ones_like(u)
    if absolute and silu:
        slope = 1.1 + u
    g = dout * slope
    end = lens.long()[:, None] + torch.arange(width - 1, device=x.device)                  # places in seq
    rows = torch.arange(n, device=x.device)[:, None]
    dseq = torch.zeros_like(seq)
    dseq[rows, end] += dstate_out
    for j in range(width):
        dseq[:, j:j + t] += w[:, j] * g
    return {"out": torch.where(live, u * s if silu and not absolute else u, 0.0), "state": seq[rows, end],
            "dx": torch.where(live, dseq[:, width - 1:], 0.0), "dbias": g.sum((0, 1)), "dstate": dseq[:, :width - 1],
            "dweight": torch.stack([(g * seq[:, j:j + t]).sum((0, 1)) for j in range(width)], 1)}
