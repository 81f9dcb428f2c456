"""The convolution of many rows at once against the one that goes through them."""

import pytest
import torch

import layer_refs as refs
import layer_wide as wide


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("absolute", [True, False])
@pytest.mark.parametrize("t,width", [(1, 1), (1, 4), (2, 8), (9, 4), (20, 3)])
def test_conv(t, width, absolute, silu):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=g)                       # noqa: E731
    n, d = 5, 3
    lens = torch.tensor([t, 0, t // 2, max(t - 1, 0), 1])
    given = dict(x=r(n, t, d), weight=r(d, width), bias=r(d), silu=silu, lens=lens, state=r(n, width - 1, d),
                 dout=r(n, t, d), dstate_out=r(n, width - 1, d), absolute=absolute)
    want, got = refs.conv(**given), wide.conv(**given)
    for name, v in want.items():
        assert torch.allclose(got[name], v, rtol=1e-12, atol=1e-12), name
