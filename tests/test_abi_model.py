"""The entry points of the operators over walk tokens reject bad arguments on the host, before any HIP
call: the dummy device pointers below are never dereferenced."""

import ctypes

import pytest

FAKE = 1 << 40
WS = 1 << 41


@pytest.fixture(scope="module")
def lib():
    import paper_2508_01073_amd as pkg
    return pkg._native(), pkg


def _attention(pkg, **kw):
    a = dict(rows=4, length=10, heads=4, kv_heads=2, dk=16, dv=24, dtype=0, scale=0.25, log_decay=FAKE, len=None)
    a.update(kw)
    return pkg._AttentionStruct(*[a[n] for n, _ in pkg._AttentionStruct._fields_])


def _view(pkg, data=FAKE, row=640, token=64, head=16):
    return pkg._HeadsViewStruct(data, row, token, head)


def _forward(lib, a=None, q=None, k=None, v=None, state=None, out=FAKE, state_out=None, ws=WS, wsb=1 << 40, **kw):
    so, pkg = lib
    a = _attention(pkg, **kw) if a is None else a
    q, k, v = (_view(pkg) if x is None else x for x in (q, k, v))
    return so.rdf2v_decay_attention(a, q, k, v, state, out, state_out, ws, wsb, None, None)


def _backward(lib, dout=None, dq=FAKE, dk=FAKE, dv=FAKE, ws=WS, wsb=1 << 40, dstate=None, **kw):
    so, pkg = lib
    v = _view(pkg)
    return so.rdf2v_decay_attention_backward(_attention(pkg, **kw), v, v, v, v if dout is None else dout, None, None,
                                             dq, dk, dv, dstate, ws, wsb, None, None)


def _step(lib, n=4, state=FAKE, parents=None, out=FAKE, state_out=FAKE, **kw):
    so, pkg = lib
    v = _view(pkg)
    return so.rdf2v_decay_attention_step(_attention(pkg, **kw), v, v, v, state, n, parents, out, state_out, None, None)


def test_attention_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    for call in (_forward, _backward, _step):
        for bad in (dict(rows=-1), dict(heads=0), dict(heads=65536, kv_heads=1), dict(kv_heads=0), dict(kv_heads=3),
                    dict(dk=0), dict(dk=129), dict(dv=0), dict(dv=129), dict(dtype=2), dict(dtype=-1),
                    dict(scale=float("nan")), dict(scale=float("inf")), dict(log_decay=None), dict(log_decay=FAKE + 2)):
            assert call(lib, **bad) == inv, bad
        assert call(lib, rows=2**31) == big
    for call in (_forward, _backward):
        assert call(lib, length=-1) == inv
        assert call(lib, length=2**31) == big
        assert call(lib, rows=2**30, length=2**30) == big
        assert call(lib, len=FAKE + 1) == inv
        assert call(lib, rows=0) == pkg.RDF2V_OK
    assert so.rdf2v_decay_attention(None, None, None, None, None, None, None, None, 0, None, None) == inv
    assert _forward(lib, q=_view(pkg, data=None)) == inv
    assert _forward(lib, k=_view(pkg, data=FAKE + 2)) == inv          # not aligned to a float
    assert _forward(lib, v=_view(pkg, token=2**60)) == inv
    assert _forward(lib, out=None) == inv
    assert _forward(lib, out=FAKE + 1) == inv
    assert _forward(lib, state=FAKE + 2) == inv
    assert _forward(lib, state_out=FAKE + 2) == inv
    assert _backward(lib, dq=None) == inv
    assert _backward(lib, dk=FAKE + 3) == inv
    assert _backward(lib, dv=None) == inv
    assert _backward(lib, dout=_view(pkg, data=None)) == inv
    assert _backward(lib, dstate=FAKE + 2) == inv
    need = so.rdf2v_decay_attention_backward_workspace_size(_attention(pkg))
    assert need > 0 and need % 256 == 0
    assert _backward(lib, ws=None) == wse
    assert _backward(lib, wsb=need - 1) == wse
    assert _backward(lib, ws=WS + 64) == wse


def test_step_refusals(lib):
    _, pkg = lib
    inv, big = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE
    assert _step(lib, n=-1) == inv
    assert _step(lib, n=5) == inv                                     # without parents row r continues state r
    assert _step(lib, n=2**31, parents=FAKE) == big
    assert _step(lib, state=None) == inv
    assert _step(lib, state_out=None) == inv
    assert _step(lib, state_out=FAKE + 2) == inv
    assert _step(lib, parents=FAKE + 1, n=4) == inv
    size = 4 * 16 * 24 * 4
    assert _step(lib, parents=WS, n=4) == inv                         # states and new states overlap
    assert _step(lib, state_out=FAKE + 4 * size - 4) == inv
    assert _step(lib, state_out=FAKE + 4) == inv
    assert _step(lib, rows=0, n=0, state=None, out=None, state_out=None) == pkg.RDF2V_OK


def test_beam_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    need = pkg.rdf2v_beam_select_workspace_size(2, 3, 100, 4)
    ok = dict(logits=FAKE, stride=100, dtype=0, scores=FAKE, finished=None, groups=2, beams=3, vocab=100, num_out=4,
              scores_out=WS, tokens=WS, parents=WS, ws=WS, wsb=need)

    def call(**kw):
        a = dict(ok, **kw)
        return so.rdf2v_beam_select(a["logits"], a["stride"], a["dtype"], a["scores"], a["finished"], a["groups"],
                                    a["beams"], a["vocab"], a["num_out"], a["scores_out"], a["tokens"], a["parents"],
                                    a["ws"], a["wsb"], None, None)

    for bad in (dict(groups=-1), dict(beams=0), dict(beams=65), dict(num_out=0), dict(num_out=65), dict(vocab=0),
                dict(dtype=7), dict(stride=99), dict(logits=None), dict(scores=None), dict(scores_out=None),
                dict(tokens=None), dict(parents=None), dict(logits=FAKE + 2), dict(scores=FAKE + 1),
                dict(finished=FAKE + 2), dict(scores_out=FAKE), dict(scores_out=FAKE + 8, num_out=3)):
        assert call(**bad) == inv, bad
    for bad in (dict(vocab=2**31, stride=2**31), dict(groups=2**30), dict(stride=2**60)):
        assert call(**bad) == big, bad
    if need:
        for bad in (dict(ws=None), dict(wsb=need - 1), dict(ws=WS + 8)):
            assert call(**bad) == wse, bad
    assert call(groups=0, logits=None, scores=None) == pkg.RDF2V_OK
    for sizes in ((-1, 1, 1, 1), (1, 0, 1, 1), (1, 1, 2**31, 1), (2**31, 1, 1, 1), (1, 1, 1, 65)):
        assert pkg.rdf2v_beam_select_workspace_size(*sizes) == 0


def test_reorder_refusals(lib):
    so, pkg = lib
    inv, big = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE

    def call(src=FAKE, n=4, size=64, parents=FAKE, rows=4, dst=WS):
        return so.rdf2v_beam_reorder(src, n, size, parents, rows, dst, None, None)

    for bad in (dict(n=-1), dict(size=-1), dict(rows=-1), dict(src=None), dict(parents=None), dict(dst=None),
                dict(parents=FAKE + 2), dict(dst=FAKE), dict(dst=FAKE + 255), dict(dst=FAKE - 255)):
        assert call(**bad) == inv, bad
    for bad in (dict(n=2**31), dict(rows=2**31), dict(size=2**60)):
        assert call(**bad) == big, bad
    assert call(rows=0, dst=None) == pkg.RDF2V_OK and call(size=0) == pkg.RDF2V_OK


def test_distill_refusals(lib):
    so, pkg = lib
    inv, big, wse = pkg.RDF2V_ERR_INVALID_ARGUMENT, pkg.RDF2V_ERR_TOO_LARGE, pkg.RDF2V_ERR_WORKSPACE
    ok = dict(logits=FAKE, stride=100, dtype=0, ids=FAKE, teacher=FAKE, rows=8, vocab=100, top=4, tau=1.0, loss=WS,
              lse=WS, dloss=FAKE, dlogits=WS, dstride=100, ws=WS, wsb=1 << 40)

    def both(**kw):
        a = dict(ok, **kw)
        head = [a[n] for n in ("logits", "stride", "dtype", "ids", "teacher", "rows", "vocab", "top", "tau")]
        tail = [a[n] for n in ("dloss", "dlogits", "dstride", "ws", "wsb")] + [None, None]
        return (so.rdf2v_distill_loss(*head, a["loss"], a["lse"], *tail),
                so.rdf2v_distill_loss_backward(*head, a["lse"], *tail))

    for bad in (dict(rows=-1), dict(vocab=0), dict(top=-1), dict(top=513), dict(dtype=2), dict(stride=99),
                dict(dstride=99), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")),
                dict(logits=None), dict(ids=None), dict(teacher=None), dict(lse=None), dict(dloss=None),
                dict(dlogits=None), dict(logits=FAKE + 2), dict(ids=FAKE + 2), dict(dlogits=WS + 2),
                dict(dlogits=FAKE + 4), dict(dlogits=FAKE, dstride=101)):
        assert both(**bad) == (inv, inv), bad
    for bad in (dict(rows=2**31), dict(vocab=2**31, stride=2**31, dstride=2**31), dict(stride=2**60)):
        assert both(**bad) == (big, big), bad
    need = pkg.rdf2v_distill_workspace_size(8, 100, 4)
    if need:
        assert both(ws=None) == (wse, wse) and both(wsb=need - 1) == (wse, wse)
    assert both(rows=0, logits=None, ids=None) == (pkg.RDF2V_OK, pkg.RDF2V_OK)
    for sizes in ((-1, 1, 1), (1, 0, 1), (1, 1, 513), (2**31, 1, 1), (1, 2**31, 1)):
        assert pkg.rdf2v_distill_workspace_size(*sizes) == 0


@pytest.mark.parametrize("length", [0, 1, 448, 449, 1024, 2**31 - 1])
def test_attention_of_no_rows(lib, length):
    """An empty batch of rows of any length needs nothing and does nothing."""
    so, pkg = lib
    for heads, kv, d in ((1, 1, 1), (4, 2, 32), (65535, 1, 128)):
        sizes = (0, length, heads, kv, d, d)
        assert pkg.rdf2v_decay_attention_workspace_size(*sizes) == 0
        assert pkg.rdf2v_decay_attention_backward_workspace_size(*sizes) == 0
        a = dict(rows=0, length=length, heads=heads, kv_heads=kv, dk=d, dv=d)
        assert _forward(lib, **a) == pkg.RDF2V_OK and _forward(lib, ws=None, wsb=0, **a) == pkg.RDF2V_OK
        c, v = _attention(pkg, **a), _view(pkg)
        for ws, wsb in ((WS, 1 << 40), (None, 0)):
            assert so.rdf2v_decay_attention_backward(c, v, v, v, v, None, None, FAKE, FAKE, FAKE, None, ws, wsb, None,
                                                     None) == pkg.RDF2V_OK


def test_attention_refuses_overlaps(lib):
    """Outputs over inputs or over one another, by as little as a value: rows x tokens x heads of 4 x 10 x 4
    queries of 16 values and 4 x 10 x 2 keys and values of 16 and 24, float32, at places of their own."""
    so, pkg = lib
    inv = pkg.RDF2V_ERR_INVALID_ARGUMENT
    sizes = dict(q=4 * 10 * 4 * 16 * 4, k=4 * 10 * 2 * 16 * 4, v=4 * 10 * 2 * 24 * 4, out=4 * 10 * 4 * 24 * 4,
                 state=4 * 4 * 16 * 24 * 4)
    places = {n: FAKE + (i << 24) for i, n in enumerate(
        ("q", "k", "v", "dout", "out", "state", "state_out", "dstate_out", "dq", "dk", "dv", "dstate"))}
    size = lambda n: sizes["out" if n == "dout" else "state" if "state" in n else n[-1] if n != "out" else n]  # noqa: E731

    def forward(**moved):
        at = dict(places, **moved)
        views = [_view(pkg, at[n], *s) for n, s in (("q", (640, 64, 16)), ("k", (320, 32, 16)), ("v", (480, 48, 24)))]
        return so.rdf2v_decay_attention(_attention(pkg), *views, at["state"], at["out"], at["state_out"], WS, 1 << 40,
                                        None, None)

    def backward(**moved):
        at = dict(places, **moved)
        views = [_view(pkg, at[n], *s) for n, s in (("q", (640, 64, 16)), ("k", (320, 32, 16)), ("v", (480, 48, 24)),
                                                    ("dout", (960, 96, 24)))]
        return so.rdf2v_decay_attention_backward(_attention(pkg), *views, at["state"], at["dstate_out"], at["dq"],
                                                 at["dk"], at["dv"], at["dstate"], WS, 1 << 40, None, None)

    for call, outs, ins in ((forward, ("out", "state_out"), ("q", "k", "v", "state")),
                            (backward, ("dq", "dk", "dv", "dstate"), ("q", "k", "v", "dout", "state", "dstate_out"))):
        for i, x in enumerate(outs):
            for y in outs[:i] + ins:
                for step in (4, size(y) // 8 * 4, size(y) - 4, 4 - size(x)):
                    assert call(**{x: places[y] + step}) == inv, (x, y, step)
                if (x, y) not in (("state_out", "state"), ("dstate", "dstate_out")):
                    assert call(**{x: places[y]}) == inv, (x, y)


def test_attention_refuses_overlaps_with_strided_inputs(lib):
    """An output within the values of an input of any strides is refused: heads before tokens, negative
    strides, keys shared by all rows, tokens far apart."""
    so, pkg = lib
    at = FAKE + (1 << 30)

    def call(view, out):
        far = _view(pkg, FAKE + (1 << 38))
        return so.rdf2v_decay_attention(_attention(pkg, heads=2, kv_heads=2), view, far, far, None, out, None, WS,
                                        1 << 40, None, None)

    size = 4 * 10 * 2 * 24 * 4                                        # of the output
    for row, token, head in ((2 * 10 * 16, 16, 160), (-320, 32, 16), (320, -32, -16), (0, 32, 16), (16, 64, 1 << 20),
                             (1 << 20, 1 << 22, 1 << 18), (1, 2, 3)):
        for r, t, h in ((0, 0, 0), (3, 9, 1), (1, 5, 1), (2, 0, 0)):
            value = at + 4 * (r * row + t * token + h * head)
            for out in (value, value + 60, value - size + 4):         # the first or last value of a head
                assert call(_view(pkg, at, row, token, head), out) == pkg.RDF2V_ERR_INVALID_ARGUMENT, (row, token, head)
