"""The entry points of the layer operators reject bad arguments on the host, before any HIP call: the dummy
device pointers below are never dereferenced."""

import pytest

GAP = 1 << 36                                     # between the dummy arrays: more than any of them holds


def at(i, off=0):
    return (1 << 44) + i * GAP + off


@pytest.fixture(scope="module")
def lib():
    import paper_2508_01073_amd as pkg
    return pkg._native(), pkg


def _struct(kind, base, kw):
    return kind(*[{**base, **kw}.get(n) for n, _ in kind._fields_])


def _tokens(pkg, i, row=640, token=64, off=0, data=True):
    return pkg._TokensViewStruct(at(i, off) if data else None, row, token)


def _heads(pkg, i, **kw):
    v = dict(row=640, token=64, head=16, off=0) | kw
    return pkg._HeadsViewStruct(at(i, v["off"]), v["row"], v["token"], v["head"])


# ---- causal convolution ---------------------------------------------------

def _conv(pkg, **kw):
    return _struct(pkg._ConvStruct, dict(rows=4, length=10, channels=48, width=4, dtype=0, silu=1, weight=at(0),
                                         bias=at(1), len=None), kw)


def _conv_forward(lib, x=None, state=None, out=at(4), state_out=None, **kw):
    so, pkg = lib
    return so.rdf2v_causal_conv(_conv(pkg, **kw), x or _tokens(pkg, 2), state, out, state_out, None, None)


def _conv_backward(lib, x=None, dout=None, state=None, dso=None, dx=at(4), dw=at(5), db=None, ds=None, ws=at(9),
                   wsb=GAP, **kw):
    so, pkg = lib
    return so.rdf2v_causal_conv_backward(_conv(pkg, **kw), x or _tokens(pkg, 2), dout or _tokens(pkg, 3), state, dso,
                                         dx, dw, db, ds, ws, wsb, None, None)


def _conv_step(lib, x=None, state=at(3), n=4, parents=None, out=at(4), state_out=at(5), **kw):
    so, pkg = lib
    return so.rdf2v_causal_conv_step(_conv(pkg, **kw), x or _tokens(pkg, 2), state, n, parents, out, state_out, None,
                                     None)


def test_conv_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    for call in (_conv_forward, _conv_backward, _conv_step):
        for bad in (dict(rows=-1), dict(channels=0), dict(channels=-3), dict(width=0), dict(width=9), dict(dtype=2),
                    dict(dtype=-1), dict(weight=None), dict(weight=at(0, 2)), dict(bias=at(1, 1)),
                    dict(x=_tokens(pkg, 2, data=False)), dict(x=_tokens(pkg, 2, off=2)),
                    dict(x=_tokens(pkg, 2, row=2**60))):
            assert call(lib, **bad) == inv, bad
        assert call(lib, rows=2**31) == big
        assert call(lib, rows=2**30, length=2**30, channels=2**30) == big
    for call in (_conv_forward, _conv_backward):
        assert call(lib, length=-1) == inv
        assert call(lib, length=2**31) == big
        assert call(lib, len=at(7, 2)) == inv
    assert so.rdf2v_causal_conv(None, None, None, None, None, None, None) == inv
    assert _conv_forward(lib, rows=0, out=None) == pkg.RDF2V_OK
    for bad in (dict(out=None), dict(out=at(4, 2)), dict(state=at(5, 1)), dict(state_out=at(6, 2)),
                dict(out=at(2)), dict(out=at(2, 4 * 640 - 64)), dict(state=at(4)), dict(state_out=at(4)),
                dict(out=at(0, 4)), dict(out=at(1)), dict(state=at(5), state_out=at(5))):
        assert _conv_forward(lib, **bad) == inv, bad
    for bad in (dict(dx=None), dict(dw=None), dict(dx=at(4, 3)), dict(dw=at(5, 2)), dict(db=at(6, 1)),
                dict(ds=at(6, 2)), dict(state=at(6, 2)), dict(dso=at(6, 2)), dict(dx=at(2)), dict(dx=at(3)),
                dict(dw=at(4)), dict(db=at(5)), dict(ds=at(6), state=at(6)), dict(ds=at(6), dso=at(6)),
                dict(dout=_tokens(pkg, 3, data=False))):
        assert _conv_backward(lib, **bad) == inv, bad
    need = so.rdf2v_causal_conv_backward_workspace_size(_conv(pkg))
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(wsb=need - 1), dict(ws=at(9, 64))):
        assert _conv_backward(lib, **bad) == wse, bad
    assert so.rdf2v_causal_conv_backward_workspace_size(_conv(pkg, width=9)) == 0
    size = 3 * 48 * 4
    for bad in (dict(n=-1), dict(n=5), dict(out=None), dict(state=None), dict(state_out=None), dict(parents=at(6, 2)),
                dict(state_out=at(3), parents=at(6)), dict(state_out=at(3, 4)), dict(state_out=at(3, 4 * size - 4)),
                dict(out=at(3)), dict(out=at(2))):
        assert _conv_step(lib, **bad) == inv, bad
    assert _conv_step(lib, n=2**31, parents=at(6)) == big
    assert _conv_step(lib, rows=0, n=0, state=None, out=None, state_out=None) == pkg.RDF2V_OK


# ---- selective scan -------------------------------------------------------

def _scan(pkg, **kw):
    return _struct(pkg._ScanStruct, dict(rows=4, length=10, channels=48, groups=2, states=16, dtype=0, a=at(0),
                                         dt_bias=at(1), skip=at(2), len=None), kw)


def _views(pkg, kw):
    v = dict(x=_tokens(pkg, 3), dt=_tokens(pkg, 4), b=_heads(pkg, 5), c=_heads(pkg, 6), gate=_tokens(pkg, 7))
    for name in list(kw):
        if name in v:
            v[name] = kw.pop(name)
    return [v[n] for n in ("x", "dt", "b", "c", "gate")]


def _scan_forward(lib, state=None, out=at(10), state_out=None, ws=at(20), wsb=GAP, **kw):
    so, pkg = lib
    v = _views(pkg, kw)
    return so.rdf2v_selective_scan(_scan(pkg, **kw), *v, state, out, state_out, ws, wsb, None, None)


def _grads(pkg, **kw):
    base = dict(dx=at(10), ddt=at(11), db=at(12), dc=at(13), dgate=at(14), da=at(15), ddt_bias=at(16), dskip=at(17),
                dstate=None)
    return _struct(pkg._ScanGradientsStruct, base, kw)


def _scan_backward(lib, dout=None, state=None, dso=None, grads=None, ws=at(20), wsb=GAP, **kw):
    so, pkg = lib
    v = _views(pkg, kw)
    return so.rdf2v_selective_scan_backward(_scan(pkg, **kw), *v, dout or _tokens(pkg, 8), state, dso,
                                            grads or _grads(pkg), ws, wsb, None, None)


def _scan_step(lib, state=at(9), n=4, parents=None, out=at(10), state_out=at(11), **kw):
    so, pkg = lib
    v = _views(pkg, kw)
    return so.rdf2v_selective_scan_step(_scan(pkg, **kw), *v, state, n, parents, out, state_out, None, None)


def test_scan_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    for call in (_scan_forward, _scan_backward, _scan_step):
        for bad in (dict(rows=-1), dict(channels=0), dict(groups=0), dict(groups=5), dict(groups=65536, channels=65536),
                    dict(states=0), dict(states=65), dict(dtype=2), dict(a=None), dict(a=at(0, 2)),
                    dict(dt_bias=at(1, 2)), dict(skip=at(2, 1)), dict(x=None), dict(dt=_tokens(pkg, 4, data=False)),
                    dict(b=None), dict(c=_heads(pkg, 6, off=2)), dict(gate=_tokens(pkg, 7, off=1)),
                    dict(b=_heads(pkg, 5, head=-2**57))):
            assert call(lib, **bad) == inv, bad
        assert call(lib, rows=2**31) == big
        assert call(lib, channels=2**28 + 2) == big
        assert call(lib, rows=2**30, length=2**30, channels=2**20) == big
    for call in (_scan_forward, _scan_backward):
        assert call(lib, length=-1) == inv
        assert call(lib, length=2**31) == big
        assert call(lib, len=at(18, 2)) == inv
    for bad in (dict(out=None), dict(out=at(10, 1)), dict(state=at(11, 2)), dict(state_out=at(11, 2)),
                dict(out=at(3)), dict(out=at(4)), dict(out=at(5)), dict(out=at(6)), dict(out=at(7)), dict(out=at(0)),
                dict(out=at(1)), dict(out=at(2)), dict(state_out=at(10)), dict(state=at(11), state_out=at(11, 4))):
        assert _scan_forward(lib, **bad) == inv, bad
    assert _scan_forward(lib, rows=0, out=None) == pkg.RDF2V_OK
    names = [n for n, _ in pkg._ScanGradientsStruct._fields_]
    for name in names[:6]:                                            # what there has to be
        assert _scan_backward(lib, grads=_grads(pkg, **{name: None})) == inv, name
    for i, name in enumerate(names):
        assert _scan_backward(lib, grads=_grads(pkg, **{name: at(19, 1)})) == inv, name
        for over in (3, 4, 5, 6, 7, 8, 0, 1, 2):                      # an input
            assert _scan_backward(lib, grads=_grads(pkg, **{name: at(over)})) == inv, (name, over)
        other = at(10) if name != "dx" else at(11)                    # another output
        assert _scan_backward(lib, grads=_grads(pkg, **{name: other})) == inv, name
    assert _scan_backward(lib, grads=_grads(pkg, dstate=at(18)), state=at(18)) == inv
    assert _scan_backward(lib, gate=None) == inv                      # a gradient of a gate that is not there
    need = so.rdf2v_selective_scan_backward_workspace_size(_scan(pkg))
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(wsb=need - 1), dict(ws=at(20, 128))):
        assert _scan_backward(lib, **bad) == wse, bad
    few = so.rdf2v_selective_scan_workspace_size(_scan(pkg, rows=1, length=5000))
    assert few > 0 and so.rdf2v_selective_scan_workspace_size(_scan(pkg, rows=100_000, length=17)) == 0
    assert _scan_forward(lib, rows=1, length=5000, wsb=few - 1) == wse
    for bad in (dict(states=65), dict(rows=-1), dict(channels=2**29)):
        assert so.rdf2v_selective_scan_workspace_size(_scan(pkg, **bad)) == 0
        assert so.rdf2v_selective_scan_backward_workspace_size(_scan(pkg, **bad)) == 0
    for bad in (dict(n=-1), dict(n=5), dict(out=None), dict(state=None), dict(state_out=None), dict(parents=at(12, 2)),
                dict(state_out=at(9), parents=at(12)), dict(state_out=at(9, 4)), dict(out=at(9)), dict(out=at(3)),
                dict(out=at(11))):
        assert _scan_step(lib, **bad) == inv, bad
    assert _scan_step(lib, n=2**31, parents=at(12)) == big
    assert _scan_step(lib, rows=0, n=0, state=None, out=None, state_out=None) == pkg.RDF2V_OK


# ---- residual norm --------------------------------------------------------

def _norm(pkg, **kw):
    return _struct(pkg._NormStruct, dict(rows=4, length=10, channels=48, dtype=1, residual_dtype=0, center=0, eps=1e-5,
                                         weight=at(0), bias=at(1), scale=at(2), drop=0.1, seed=7, seed_offset=None,
                                         row_begin=0, len=None), kw)


def _norm_forward(lib, x=None, residual=None, out=at(10), hidden=at(11), stats=at(12), **kw):
    so, pkg = lib
    return so.rdf2v_residual_norm(_norm(pkg, **kw), x or _tokens(pkg, 3), residual or _tokens(pkg, 4), out, hidden,
                                  stats, None, None)


def _norm_backward(lib, x=None, residual=None, stats=at(5), dout=None, dhidden=None, dx=at(10), dres=at(11), dw=at(12),
                   db=at(13), dsc=at(14), ws=at(20), wsb=GAP, **kw):
    so, pkg = lib
    return so.rdf2v_residual_norm_backward(_norm(pkg, **kw), x or _tokens(pkg, 3), residual or _tokens(pkg, 4), stats,
                                           dout or _tokens(pkg, 6), dhidden or _tokens(pkg, 7), dx, dres, dw, db, dsc,
                                           ws, wsb, None, None)


def test_norm_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    nan, inf = float("nan"), float("inf")
    for call in (_norm_forward, _norm_backward):
        for bad in (dict(rows=-1), dict(length=-1), dict(channels=0), dict(channels=16385), dict(dtype=2),
                    dict(dtype=0, residual_dtype=1), dict(residual_dtype=3), dict(eps=nan), dict(eps=-1.0),
                    dict(eps=inf), dict(drop=-0.1), dict(drop=1.0), dict(drop=nan), dict(drop=1.0 - 2.0**-32),
                    dict(row_begin=-1), dict(row_begin=2**63 - 3), dict(weight=None), dict(weight=at(0, 2)),
                    dict(bias=at(1, 2)), dict(scale=at(2, 3)), dict(seed_offset=at(8, 4)), dict(len=at(8, 2)),
                    dict(x=_tokens(pkg, 3, data=False)), dict(x=_tokens(pkg, 3, off=1)),
                    dict(residual=_tokens(pkg, 4, off=2)), dict(residual=_tokens(pkg, 4, token=2**58))):
            assert call(lib, **bad) == inv, bad
        assert call(lib, rows=2**31) == big
        assert call(lib, length=2**31) == big
        assert call(lib, rows=2**30, length=2**30) == big
    for bad in (dict(out=None), dict(out=at(10, 1)), dict(hidden=at(11, 2)), dict(stats=at(12, 2)), dict(out=at(3)),
                dict(hidden=at(4)), dict(stats=at(0)), dict(hidden=at(10)), dict(stats=at(11)), dict(out=at(1)),
                dict(seed_offset=at(10))):
        assert _norm_forward(lib, **bad) == inv, bad
    assert _norm_forward(lib, rows=0, out=None) == pkg.RDF2V_OK
    for bad in (dict(stats=None), dict(stats=at(5, 2)), dict(dx=None), dict(dw=None), dict(dx=at(10, 1)),
                dict(dres=at(11, 2)), dict(dw=at(12, 2)), dict(db=at(13, 1)), dict(dsc=at(14, 2)), dict(dx=at(3)),
                dict(dres=at(4)), dict(dx=at(5)), dict(dx=at(6)), dict(dres=at(7)), dict(dx=at(11)), dict(db=at(12)),
                dict(dsc=at(2)), dict(dout=_tokens(pkg, 6, data=False)), dict(dhidden=_tokens(pkg, 7, off=2))):
        assert _norm_backward(lib, **bad) == inv, bad
    need = so.rdf2v_residual_norm_backward_workspace_size(_norm(pkg))
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(wsb=need - 1), dict(ws=at(20, 4))):
        assert _norm_backward(lib, **bad) == wse, bad
    assert so.rdf2v_residual_norm_backward_workspace_size(_norm(pkg, channels=16385)) == 0


def test_names_are_exported():
    import paper_2508_01073_amd as pkg
    for name in ("causal_conv", "causal_conv_backward", "causal_conv_step", "selective_scan",
                 "selective_scan_backward", "selective_scan_step", "residual_norm", "residual_norm_backward"):
        assert "rdf2v_" + name in pkg.__all__ and callable(getattr(pkg, "rdf2v_" + name))
    assert pkg.rdf2v_causal_conv_backward_workspace_size(4, 10, 48, 4) > 0
    assert pkg.rdf2v_selective_scan_workspace_size(1, 5000, 48, 1, 16) > 0
    assert pkg.rdf2v_selective_scan_backward_workspace_size(4, 10, 48, 1, 16) > 0
    assert pkg.rdf2v_residual_norm_backward_workspace_size(4, 10, 48) > 0
