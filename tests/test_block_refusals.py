"""Refusals of linear maps, their gradients, dropout and cross attention through the C ABI: every bad argument returns its status
before any GPU work (no GPU is needed; the addresses are never read)."""
import ctypes as C

import pytest

BASE = 0x7000_0000_0000     # an address that is only compared
G = 1 << 30


@pytest.fixture(scope="module")
def P():
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _call(P, name, a, ws=BASE + 100 * G, ws_bytes=1 << 50):
    return getattr(P.lib(), name)(C.byref(a), ws, ws_bytes, None)


def _need(P, name, a):
    size = C.c_size_t()
    return getattr(P.lib(), name + "_workspace_size")(C.byref(a), C.byref(size)), size.value


def _set(a, kw):
    for k, v in kw.items():
        if isinstance(v, dict):
            for f, x in v.items():
                setattr(getattr(a, k), f, x)
        else:
            setattr(a, k, v)
    return a


def _linear(P, **kw):
    a = P.LinearMapArgs(rows=8, in_=4096, out=32, type=P.F32, code_type=P.CODE_NONE, y_type=P.F32, act=0, w_turned=0, x=BASE,
                        ldx=4096, w=BASE + G, ldw=32, y=BASE + 2 * G, ldy=32)
    return _set(a, kw)


CODED = dict(code_type=1, alpha=BASE + 5 * G, scale=BASE + 6 * G)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=(1 << 40) + 1), dict(in_=0), dict(out=0), dict(type=3), dict(y_type=1), dict(y_type=9), dict(act=4), dict(act=-1),
    dict(w_turned=2), dict(code_type=3), dict(x=None), dict(w=None), dict(y=None), dict(ldx=-1), dict(ldw=31), dict(w_turned=1),
    dict(ldy=31), dict(ldx=1 << 60), dict(res=BASE + 3 * G, ldres=-1), dict(z=BASE + 3 * G, ldz=31), dict(alpha=BASE + 5 * G),
    dict(scale=BASE + 5 * G), dict(**{**CODED, "alpha": None}), dict(**{**CODED, "scale": None}),
    # overlaps
    dict(y=BASE), dict(y=BASE + G + 4), dict(z=BASE + 2 * G + 64, ldz=32), dict(z=BASE, ldz=32), dict(bias=BASE + 2 * G + 4),
    dict(res=BASE + 2 * G + 4, ldres=32), dict(res=BASE + 2 * G, ldres=33), dict(z=BASE + 3 * G, ldz=32, res=BASE + 3 * G, ldres=32),
    dict(**{**CODED, "alpha": BASE + 2 * G}), dict(ws=None), dict(ws=BASE + 64), dict(ws=BASE + 2 * G),
])
def test_linear_refuses(P, kw):
    kw = dict(kw)
    ws = kw.pop("ws") if "ws" in kw else BASE + 100 * G
    assert _call(P, "aecct_linear_map", _linear(P, **kw), ws) == P.ERR_INVALID_ARG


def test_linear_sizes(P):
    name = "aecct_linear_map"
    st, need = _need(P, name, _linear(P))
    assert st == P.OK and need > 0          # few rows and long sums: split
    assert _call(P, name, _linear(P), ws_bytes=need - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert _need(P, name, _linear(P, rows=0)) == (P.OK, 0)
    assert _call(P, name, _linear(P, rows=0, x=None, w=None, y=None), None, 0) == P.OK
    assert _need(P, name, _linear(P, rows=1 << 20, out=1 << 20))[0] == P.ERR_UNSUPPORTED
    for kw in (dict(in_=(1 << 20) + 1), dict(out=(1 << 20) + 1), dict(in_=131072, ldx=131072, **CODED)):
        assert _need(P, name, _linear(P, **kw))[0] == P.ERR_UNSUPPORTED
        assert _call(P, name, _linear(P, **kw)) == P.ERR_UNSUPPORTED
    assert P.lib().aecct_linear_map(None, None, 0, None) == P.ERR_INVALID_ARG
    assert P.lib().aecct_linear_map_workspace_size(C.byref(_linear(P)), None) == P.ERR_INVALID_ARG


def _linear_grad(P, **kw):
    a = P.LinearMapGradArgs(rows=64, in_=48, out=32, type=P.F32, act=1, w_turned=0, dw_type=P.F32, x=BASE, ldx=48, w=BASE + G, ldw=32,
                            dy=BASE + 2 * G, lddy=32, z=BASE + 3 * G, ldz=32, dx=BASE + 4 * G, lddx=48, dw=BASE + 5 * G, lddw=32,
                            dbias=BASE + 6 * G)
    return _set(a, kw)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(in_=0), dict(out=-2), dict(type=5), dict(dw_type=1), dict(act=7), dict(w_turned=-1), dict(dy=None), dict(x=None),
    dict(w=None), dict(z=None), dict(act=0), dict(dx=None, dw=None, dbias=None), dict(ldx=-1), dict(ldw=31), dict(lddx=47), dict(lddw=31),
    dict(dx=BASE), dict(dx=BASE + G), dict(dx=BASE + 2 * G), dict(dw=BASE), dict(dw=BASE + 4 * G), dict(dbias=BASE + 5 * G),
    dict(dbias=BASE + 3 * G), dict(dx=BASE + 3 * G), dict(ws=None), dict(ws=BASE + 100), dict(ws=BASE + 5 * G - 8),
])
def test_linear_grad_refuses(P, kw):
    kw = dict(kw)
    ws = kw.pop("ws") if "ws" in kw else BASE + 100 * G
    assert _call(P, "aecct_linear_map_grad", _linear_grad(P, **kw), ws) == P.ERR_INVALID_ARG


def test_linear_grad_sizes(P):
    name = "aecct_linear_map_grad"
    st, need = _need(P, name, _linear_grad(P))
    assert st == P.OK and need > 0
    assert _call(P, name, _linear_grad(P), ws_bytes=need - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert _need(P, name, _linear_grad(P, rows=0))[0] == P.OK
    assert _need(P, name, _linear_grad(P, in_=1 << 20, out=1 << 20))[0] == P.ERR_UNSUPPORTED
    assert _need(P, name, _linear_grad(P, rows=1, act=0, dw=None, dbias=None)) == (P.OK, 0)


def _dropout(P, **kw):
    a = P.DropoutArgs(rows=4, d=8, type=P.F32, p=0.5, seed=1, offset=2, x=BASE, ldx=8, y=BASE + G, ldy=8)
    a = _set(a, kw)
    return P.lib().aecct_dropout(C.byref(a), None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(d=0), dict(type=3), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(x=None), dict(y=None), dict(ldx=-1),
    dict(ldy=7), dict(y=BASE + 4), dict(y=BASE, ldy=9), dict(res=BASE + G + 4, ldres=8), dict(offset_device=BASE + G + 8),
])
def test_dropout_refuses(P, kw):
    assert _dropout(P, **kw) == P.ERR_INVALID_ARG


def test_dropout_sizes(P):
    assert _dropout(P, rows=0, x=None, y=None) == P.OK
    assert _dropout(P, rows=1 << 36, ldx=0) == P.ERR_UNSUPPORTED and _dropout(P, d=1 << 39) == P.ERR_UNSUPPORTED
    assert P.lib().aecct_dropout(None, None) == P.ERR_INVALID_ARG


def _heads(P, at, n, h, d=16):
    return P.Heads(BASE + at * G, n * h * d, h * d, d)


def _attention(P, **kw):
    a = P.CrossAttentionArgs(batch=2, queries=3, keys=5, heads=4, kv_heads=2, d=16, type=P.F32, scale=0.25, q=_heads(P, 0, 3, 4),
                             k=_heads(P, 1, 5, 2), v=_heads(P, 2, 5, 2), o=_heads(P, 3, 3, 4), lse=BASE + 4 * G, mask=BASE + 5 * G,
                             ldmask=5, lengths=BASE + 6 * G)
    return _set(a, kw)


BAD_SIZES = [dict(batch=-1), dict(queries=-1), dict(keys=-1), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(kv_heads=-2), dict(d=0),
             dict(type=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=dict(data=None)),
             dict(k=dict(data=None)), dict(v=dict(data=None)), dict(q=dict(row=-1)), dict(k=dict(batch=-16)), dict(v=dict(head=-1)),
             dict(k=dict(row=1 << 60)), dict(ldmask=-1), dict(ws=None), dict(ws=BASE), dict(ws=BASE + 5 * G), dict(ws=BASE + 6 * G)]


@pytest.mark.parametrize("kw", BAD_SIZES + [
    dict(o=dict(data=None)), dict(o=dict(head=15)), dict(o=dict(row=63)), dict(o=dict(batch=100)), dict(o=dict(data=BASE)),
    dict(o=dict(data=BASE + G + 8)), dict(lse=BASE + 3 * G + 4), dict(lse=BASE + 2 * G), dict(mask=BASE + 3 * G), dict(lengths=BASE + 4 * G),
    dict(ws=BASE + 3 * G), dict(ws=BASE + 4 * G)])
def test_attention_refuses(P, kw):
    kw = dict(kw)
    ws = kw.pop("ws") if "ws" in kw else BASE + 100 * G
    assert _call(P, "aecct_cross_attention", _attention(P, **kw), ws) == P.ERR_INVALID_ARG


def test_attention_sizes(P):
    name = "aecct_cross_attention"
    st, need = _need(P, name, _attention(P))
    assert st == P.OK and need > 0 and _call(P, name, _attention(P), ws_bytes=need - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert _need(P, name, _attention(P, mask=None)) == (P.OK, 0)
    assert _need(P, name, _attention(P, mask=None, queries=1, keys=8192))[1] > 0
    for kw in (dict(batch=0), dict(queries=0)):
        assert _call(P, name, _attention(P, **kw), None, 0) == P.OK
        assert _need(P, name, _attention(P, **kw))[0] == P.OK
    for kw in (dict(d=257), dict(queries=1 << 32), dict(keys=1 << 32), dict(batch=1 << 31, queries=1 << 20)):
        assert _need(P, name, _attention(P, **kw))[0] == P.ERR_UNSUPPORTED
        assert _call(P, name, _attention(P, **kw)) == P.ERR_UNSUPPORTED
    assert P.lib().aecct_cross_attention(None, None, 0, None) == P.ERR_INVALID_ARG


def _attention_grad(P, **kw):
    a = P.CrossAttentionGradArgs(batch=2, queries=3, keys=5, heads=4, kv_heads=2, d=16, type=P.F32, scale=0.25, q=_heads(P, 0, 3, 4),
                                 k=_heads(P, 1, 5, 2), v=_heads(P, 2, 5, 2), o=_heads(P, 3, 3, 4), dout=_heads(P, 7, 3, 4),
                                 lse=BASE + 4 * G, mask=BASE + 5 * G, ldmask=5, lengths=BASE + 6 * G, dq=_heads(P, 8, 3, 4),
                                 dk=_heads(P, 9, 5, 2), dv=_heads(P, 10, 5, 2))
    return _set(a, kw)


@pytest.mark.parametrize("kw", BAD_SIZES + [
    dict(o=dict(data=None)), dict(dout=dict(data=None)), dict(lse=None), dict(dk=dict(data=None)), dict(dv=dict(data=None)),
    dict(dq=dict(data=None), dk=dict(data=None), dv=dict(data=None)), dict(dq=dict(row=0)), dict(dk=dict(head=8)), dict(dv=dict(batch=150)),
    dict(dq=dict(data=BASE)), dict(dk=dict(data=BASE + G)), dict(dv=dict(data=BASE + 7 * G)), dict(dq=dict(data=BASE + 9 * G + 4)),
    dict(dk=dict(data=BASE + 10 * G + 64)), dict(lse=BASE + 8 * G), dict(ws=BASE + 8 * G), dict(ws=BASE + 7 * G + 8)])
def test_attention_grad_refuses(P, kw):
    kw = dict(kw)
    ws = kw.pop("ws") if "ws" in kw else BASE + 100 * G
    assert _call(P, "aecct_cross_attention_grad", _attention_grad(P, **kw), ws) == P.ERR_INVALID_ARG


def test_attention_grad_sizes(P):
    name = "aecct_cross_attention_grad"
    st, need = _need(P, name, _attention_grad(P))
    assert st == P.OK and need > 0 and _call(P, name, _attention_grad(P), ws_bytes=need - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert _call(P, name, _attention_grad(P, batch=0), None, 0) == P.OK
    for kw in (dict(queries=0), dict(keys=0)):
        assert _need(P, name, _attention_grad(P, **kw))[0] == P.OK
    assert _need(P, name, _attention_grad(P, d=300))[0] == P.ERR_UNSUPPORTED


def _taken(n, strides, d, first):
    """The places (in values) of a [batch][length][heads][d] tensor."""
    b, r, h = strides
    return [first + i * b + j * r + k * h + c for i in range(n[0]) for j in range(n[1]) for k in range(n[2]) for c in range(d)]


def _grad_into(P, n, strides, d, off):
    """The status of a gradient whose dk and dv are `off` values apart, with no workspace: refused before or because of that."""
    heads = lambda at: P.Heads(at, *strides)  # noqa: E731
    a = _attention_grad(P, batch=n[0], keys=n[1], heads=n[2], kv_heads=n[2], d=d, lengths=None, mask=None)
    a.q, a.o, a.dout, a.dq = (_heads(P, i, 3, n[2]) for i in (0, 3, 7, 8))
    a.k, a.v = _heads(P, 1, n[1], n[2]), _heads(P, 2, n[1], n[2])
    a.dk, a.dv = heads(BASE + 9 * G), heads(BASE + 9 * G + 4 * off)
    return _call(P, "aecct_cross_attention_grad", a, ws_bytes=0)


@pytest.mark.parametrize("n", [(2, 2, 1), (2, 3, 2), (1, 3, 2), (3, 1, 2), (2, 1, 1), (2, 2, 2), (1, 1, 3)])
def test_dk_and_dv_that_share_values_are_refused(P, n):
    """Every small layout of dk whose values lie apart, and dv at every offset: what shares a value is refused; what lies side by side in
    rows, heads or sequences of one step is not."""
    d, seen = 2, [0, 0]
    for b in (4, 6, 8, 12, 14, 15, 16, 20, 24):
        for r in (2, 4, 5, 6, 8, 10, 12, 24):
            for h in (2, 4, 5, 8):
                dk = _taken(n, (b, r, h), d, 0)
                if len(set(dk)) < len(dk) or _grad_into(P, n, (b, r, h), d, 1 << 20) != P.ERR_WORKSPACE_TOO_SMALL:
                    continue
                for off in range(0, 60):
                    share = bool(set(dk) & set(_taken(n, (b, r, h), d, off)))
                    got = _grad_into(P, n, (b, r, h), d, off)
                    assert got == P.ERR_INVALID_ARG or (got == P.ERR_WORKSPACE_TOO_SMALL and not share), (n, (b, r, h), off)
                    seen[got == P.ERR_INVALID_ARG] += 1
    assert min(seen) > 0
    # two sequences of two keys, dv 5 values behind dk in rows 10 apart: sequences 20 apart have room for both, 14 apart do not
    assert _grad_into(P, (2, 2, 1), (20, 10, 4), 4, 5) == P.ERR_WORKSPACE_TOO_SMALL
    assert _grad_into(P, (2, 2, 1), (14, 10, 4), 4, 5) == P.ERR_INVALID_ARG
    # [keys][batch][2][heads][d] and [batch][keys][heads][2][d]
    assert _grad_into(P, (3, 5, 2), (16, 48, 4), 4, 8) == P.ERR_WORKSPACE_TOO_SMALL
    assert _grad_into(P, (3, 5, 2), (80, 16, 8), 4, 4) == P.ERR_WORKSPACE_TOO_SMALL


def test_attention_limits(P):
    """Each limit that the header names, from both sides: the last size that is taken and the first that is not."""
    def need(grad, **kw):
        a = _attention_grad(P, lengths=None, **kw) if grad else _attention(P, lengths=None, **kw)
        return _need(P, "aecct_cross_attention_grad" if grad else "aecct_cross_attention", a)[0]
    one = dict(batch=1, heads=1, kv_heads=1)
    last_mask = ((1 << 26) - 8) // 1025 * 32       # queries on 131072 keys
    for kw, taken in ((dict(one, heads=32, kv_heads=2, queries=131072, keys=131072, mask=None), True),
                      (dict(one, heads=32, kv_heads=2, queries=131072, keys=131072), True),
                      (dict(one, heads=64, kv_heads=1, queries=131072, keys=131072), True),
                      (dict(one, queries=last_mask, keys=131072), True), (dict(one, queries=last_mask + 1, keys=131072), False),
                      (dict(one, queries=last_mask + 1, keys=131072, mask=None), True),
                      (dict(one, queries=(1 << 28) - 32, keys=1, mask=None), True),
                      (dict(one, queries=(1 << 28) - 31, keys=1, mask=None), False),
                      (dict(one, batch=(1 << 24) - 2, queries=1, keys=1), True), (dict(one, batch=(1 << 24) - 1, queries=1, keys=1), False),
                      (dict(one, batch=1 << 23, queries=1, keys=129), False), (dict(one, keys=1 << 30, queries=1, mask=None), True),
                      (dict(one, keys=(1 << 30) + 1, queries=1, mask=None), False),
                      (dict(one, heads=1 << 20, queries=1, keys=1), True), (dict(one, heads=(1 << 20) + 1, queries=1, keys=1), False)):
        for grad in (False, True):
            assert need(grad, **kw) == (P.OK if taken else P.ERR_UNSUPPORTED), (grad, kw)
