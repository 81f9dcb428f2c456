"""What the GPU tests of the layer operators share."""

import torch

import layer_refs as refs
from gpu_helpers import device

F32, BF16 = torch.float32, torch.bfloat16


def rand(*shape, type_=F32, seed=0, scale=1.0):
    g = torch.Generator(device=device()).manual_seed(seed)
    return (torch.randn(*shape, device=device(), generator=g) * scale).to(type_)


def lengths(values):
    return torch.tensor(values, dtype=torch.int32, device=device())


def check(got, ref, sizes, kinds, type_, what, exact_types=()):
    """got: name -> tensor; held to refs.bounds."""
    limits = refs.bounds({k: ref[k] for k in got}, sizes, kinds, type_, exact_types)
    for name, x in got.items():
        assert x.shape == ref[name].shape, (what, name, x.shape, ref[name].shape)
        off = (x.double().cpu() - ref[name]).abs()
        bad = ~(off <= limits[name])
        assert not bool(bad.any()), (what, name, int(bad.sum()), float(off[bad].max()),
                                     float((off / limits[name])[bad].max()))


def junk(x, lens):
    """x with what is no number beyond the rows' lengths."""
    if lens is None:
        return x
    dead = torch.arange(x.shape[1], device=x.device) >= lens[:, None]
    x = x.clone()
    x[dead] = float("nan")
    return x


CONV = ("out", "state")
CONV_GRADS = ("dx", "dweight", "dbias", "dstate")


def conv_kinds(t, width, rows):
    k = refs.conv_roundings(t, width, rows)
    return dict(out=k["token"], state=0, dx=k["token"], dstate=k["token"], dweight=k["sum"], dbias=k["sum"])


def scan_kinds(t, states, channels, rows):
    k = refs.scan_roundings(t, states, channels, rows)
    return dict(out=k["token"], state=k["token"], dx=k["token"], ddt=k["token"], dgate=k["token"], dstate=k["token"],
                db=k["channels"], dc=k["channels"], da=k["sum"], ddt_bias=k["sum"], dskip=k["sum"])


def norm_kinds(d, tokens):
    k = refs.norm_roundings(d, tokens)
    return dict(out=k["token"], hidden=k["token"], stats=k["token"], dx=k["token"], dresidual=k["token"],
                dweight=k["sum"], dbias=k["sum"], dscale=k["sum"])
