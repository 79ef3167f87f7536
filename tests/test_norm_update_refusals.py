"""Refusals of the row norm, its gradient, the gradient norm, clipping and the Adam update through the C ABI: every bad
argument returns its status before any GPU work (no GPU is needed; the addresses are never read)."""
import ctypes as C

import pytest

BASE = 0x7000_0000_0000     # an address that is only compared


@pytest.fixture(scope="module")
def P():
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _norm_args(P, **kw):
    rows, d = kw.get("rows", 4), kw.get("d", 64)
    a = P.RmsNormArgs(rows=rows, d=d, type=P.F32, gain_type=P.F32, eps=1e-5, code_type=P.CODE_NONE, group=0, x=BASE, ldx=d,
                      y=BASE + (1 << 30), ldy=d)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _norm(P, **kw):
    a = _norm_args(P, **kw)
    return P.lib().aecct_rms_norm(C.byref(a), None)


Y = BASE + (1 << 30)
CODED = dict(code_type=1, codes=BASE + (2 << 30), ldcodes=64, alpha=BASE + (3 << 30))


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=(1 << 40) + 1), dict(d=0), dict(d=-5), dict(type=3), dict(type=-1), dict(gain_type=1),
    dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(code_type=3), dict(group=16), dict(group=-32),
    dict(x=None), dict(y=None), dict(ldx=-1), dict(ldy=63), dict(ldx=1 << 60),
    dict(code_type=1), dict(codes=BASE + (2 << 30), ldcodes=64), dict(**{**CODED, "alpha": None}),
    dict(**{**CODED, "ldcodes": 63}),
    dict(res=BASE + (4 << 30), ldres=-1), dict(h=BASE + (4 << 30), ldh=10),
    # overlaps
    dict(y=BASE + 4), dict(y=BASE, ldy=65), dict(y=BASE + 64 * 4 * 3), dict(h=Y, ldh=64), dict(gain=Y + 8),
    dict(**{**CODED, "codes": BASE}), dict(**{**CODED, "alpha": Y + 64}), dict(**{**CODED, "alpha": CODED["codes"] + 255}),
    dict(h=BASE + (1 << 29), ldh=64, res=BASE + (1 << 29) + 4, ldres=64),
    dict(ldx=128, y=BASE + 63 * 4, ldy=128),           # columns of one wide buffer that share a column
])
def test_norm_refuses(P, kw):
    assert _norm(P, **kw) == P.ERR_INVALID_ARG


def test_norm_refuses_wide_rows_and_takes_no_rows(P):
    assert _norm(P, d=65537, ldx=65537, ldy=65537) == P.ERR_UNSUPPORTED
    assert _norm(P, rows=0) == P.OK                      # nothing to do, no GPU work
    assert _norm(P, rows=0, x=None, y=None) == P.OK
    assert P.lib().aecct_rms_norm(None, None) == P.ERR_INVALID_ARG


def _grad(P, ws=BASE + (9 << 30), ws_bytes=1 << 40, **kw):
    rows, d = kw.get("rows", 4), kw.get("d", 64)
    a = P.RmsNormGradArgs(rows=rows, d=d, type=P.F32, gain_type=P.F32, eps=1e-5, h=BASE, ldh=d, dy=BASE + (1 << 30), lddy=d,
                          dh=BASE + (2 << 30), lddh=d, dgain=BASE + (3 << 30))
    for k, v in kw.items():
        setattr(a, k, v)
    return P.lib().aecct_rms_norm_grad(C.byref(a), ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(d=0), dict(type=7), dict(gain_type=2), dict(eps=-1.0), dict(h=None), dict(dy=None),
    dict(dh=None, dgain=None), dict(ldh=-1), dict(lddh=63), dict(dh=BASE + 4), dict(dh=BASE, lddh=65), dict(dgain=BASE + 8),
    dict(dgain=BASE + (2 << 30)), dict(gain=BASE + (3 << 30) + 252), dict(gain=BASE + (2 << 30)), dict(ws=None),
])
def test_norm_grad_refuses(P, kw):
    assert _grad(P, **kw) == P.ERR_INVALID_ARG


def test_norm_grad_workspace(P):
    size = C.c_size_t()
    f = P.lib().aecct_rms_norm_grad_workspace_size
    assert f(4, 64, C.byref(size)) == P.OK and size.value > 0
    assert _grad(P, ws_bytes=size.value - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert f(-1, 64, C.byref(size)) == P.ERR_INVALID_ARG and f(4, 0, C.byref(size)) == P.ERR_INVALID_ARG
    assert f(4, 64, None) == P.ERR_INVALID_ARG and f(4, 65537, C.byref(size)) == P.ERR_UNSUPPORTED
    assert _grad(P, d=65537, ldh=65537, lddy=65537, lddh=65537) == P.ERR_UNSUPPORTED


def _list(P, *items):
    return (P.Tensor * len(items))(*[P.Tensor(*i) for i in items])


def _bytes(P, n):
    size = C.c_size_t()
    assert P.lib().aecct_update_workspace_size(n, C.byref(size)) == P.OK
    return size.value


WS, NORM, STEP = BASE + (1 << 40), BASE + (1 << 41), BASE + (1 << 42)


@pytest.mark.parametrize("item", [(None, 1, 0), (BASE, -1, 0), (BASE, 1, 3), (BASE, 1, -1), (BASE, (1 << 40) + 1, 0)])
def test_lists_with_bad_tensors_are_refused(P, item):
    t = _list(P, (BASE + (1 << 30), 8, 0), item)
    big = 1 << 30
    assert P.lib().aecct_grad_norm(t, 2, NORM, WS, big, None) == P.ERR_INVALID_ARG
    assert P.lib().aecct_grad_clip(t, None, 2, 1.0, NORM, WS, big, None) == P.ERR_INVALID_ARG


def test_lists_hold_at_most_two_to_the_forty_values(P):
    """Tensors that are in range one by one, and lie apart, but together need more launches than the workspace holds."""
    half = 1 << 39
    lists = _list(P, *[(BASE, half, 1)] * 3), _list(P, *[(BASE + i * (1 << 41), half, 1) for i in range(3)])
    for three in lists:
        assert P.lib().aecct_grad_norm(three, 3, 16, WS, 1 << 30, None) == P.ERR_INVALID_ARG
        assert P.lib().aecct_grad_clip(three, None, 3, 1.0, 16, WS, 1 << 30, None) == P.ERR_INVALID_ARG


def test_grad_norm_refuses(P):
    t = _list(P, (BASE, 8, 0), (BASE + 64, 8, 1))
    need = _bytes(P, 2)
    norm = P.lib().aecct_grad_norm
    assert norm(None, 2, NORM, WS, need, None) == P.ERR_INVALID_ARG
    assert norm(t, -1, NORM, WS, need, None) == P.ERR_INVALID_ARG
    assert norm(t, 2, None, WS, need, None) == P.ERR_INVALID_ARG
    assert norm(t, 2, NORM, None, need, None) == P.ERR_INVALID_ARG
    assert norm(t, 2, NORM, WS, need - 1, None) == P.ERR_WORKSPACE_TOO_SMALL
    assert norm(t, 2, BASE + 28, WS, need, None) == P.ERR_INVALID_ARG        # the norm inside a gradient
    size = C.c_size_t()
    assert P.lib().aecct_update_workspace_size(-1, C.byref(size)) == P.ERR_INVALID_ARG
    assert P.lib().aecct_update_workspace_size(3, None) == P.ERR_INVALID_ARG


def test_grad_clip_refuses(P):
    g = _list(P, (BASE, 8, 0), (BASE + 64, 8, 1))
    need = _bytes(P, 2)

    def clip(grads, out, n=2, max_norm=1.0, norm=NORM, ws=WS, nbytes=need):
        return P.lib().aecct_grad_clip(grads, out, n, max_norm, norm, ws, nbytes, None)
    for bad in (float("nan"), -1.0):
        assert clip(g, None, max_norm=bad) == P.ERR_INVALID_ARG
    assert clip(g, None, norm=None) == P.ERR_INVALID_ARG
    assert clip(g, None, ws=None) == P.ERR_INVALID_ARG
    assert clip(g, None, nbytes=need - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert clip(g, None, norm=BASE + 4) == P.ERR_INVALID_ARG
    assert clip(g, _list(P, (BASE + 256, 8, 0), (BASE + 512, 7, 1))) == P.ERR_INVALID_ARG           # another count
    assert clip(g, _list(P, (BASE + 256, 8, 0), (BASE + 256 + 31, 8, 1))) == P.ERR_INVALID_ARG      # outputs overlap
    assert clip(g, _list(P, (BASE + 64, 8, 0), (BASE + 512, 8, 1))) == P.ERR_INVALID_ARG            # over another gradient
    assert clip(g, _list(P, (BASE + 4, 8, 0), (BASE + 512, 8, 1))) == P.ERR_INVALID_ARG             # shifted in itself
    assert clip(g, _list(P, (BASE, 8, 1), (BASE + 512, 8, 1))) == P.ERR_INVALID_ARG                 # in place in another type
    twice = _list(P, (BASE, 8, 0), (BASE, 8, 0))
    assert clip(twice, None) == P.ERR_INVALID_ARG                                                   # scaled twice
    inside = _list(P, (BASE, 800, 0), (BASE + 64, 1, 0), (BASE + 1600, 8, 0))                       # behind a long one
    assert P.lib().aecct_grad_clip(inside, None, 3, 1.0, NORM, WS, _bytes(P, 3), None) == P.ERR_INVALID_ARG


def _adam(P, opt=None, n=2, step=STEP, norm=NORM, ws=WS, nbytes=None, copies=None, **lists):
    base = {"params": BASE, "m": BASE + (1 << 30), "v": BASE + (2 << 30), "grads": BASE + (3 << 30)}
    t = {k: lists.get(k, _list(P, (b, 8, 0), (b + 32, 8, 0))) for k, b in base.items()}
    o = P.AdamOptions(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, None)
    for k, v in (opt or {}).items():
        setattr(o, k, v)
    return P.lib().aecct_adam_step(t["params"], t["m"], t["v"], t["grads"], copies, n, C.byref(o), step, norm, ws,
                                   _bytes(P, 2) if nbytes is None else nbytes, None)


@pytest.mark.parametrize("opt", [
    {"lr": float("nan")}, {"lr": float("inf")}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": float("nan")},
    {"eps": -1e-8}, {"eps": float("inf")}, {"weight_decay": float("nan")}, {"max_norm": -1.0}, {"max_norm": float("nan")}])
def test_adam_refuses_options(P, opt):
    assert _adam(P, opt) == P.ERR_INVALID_ARG


def test_adam_refuses_lists(P):
    assert _adam(P, step=None) == P.ERR_INVALID_ARG
    assert _adam(P, ws=None) == P.ERR_INVALID_ARG
    assert _adam(P, nbytes=_bytes(P, 2) - 1) == P.ERR_WORKSPACE_TOO_SMALL
    assert _adam(P, n=-1) == P.ERR_INVALID_ARG
    far = BASE + (5 << 30)
    for k in ("params", "m", "v"):
        assert _adam(P, **{k: _list(P, (far, 8, 0), (far + 64, 8, 1))}) == P.ERR_INVALID_ARG    # not fp32
    for k in ("params", "m", "v", "grads"):
        assert _adam(P, **{k: _list(P, (far, 8, 0), (far + 64, 9, 0))}) == P.ERR_INVALID_ARG    # another count
        assert _adam(P, **{k: None}) == P.ERR_INVALID_ARG
    assert _adam(P, m=_list(P, (BASE, 8, 0), (far, 8, 0))) == P.ERR_INVALID_ARG                 # m on the parameters
    assert _adam(P, grads=_list(P, (far, 8, 0), (BASE + 60, 8, 0))) == P.ERR_INVALID_ARG        # a gradient on them
    assert _adam(P, params=_list(P, (BASE, 8, 0), (BASE, 8, 0))) == P.ERR_INVALID_ARG           # one parameter twice
    assert _adam(P, copies=_list(P, (far, 7, 1), (far + 64, 8, 1))) == P.ERR_INVALID_ARG
    assert _adam(P, copies=_list(P, (far, 8, 5), (far + 64, 8, 1))) == P.ERR_INVALID_ARG
    assert _adam(P, copies=_list(P, (BASE + 32, 8, 1), (far + 64, 8, 1))) == P.ERR_INVALID_ARG
    assert _adam(P, step=BASE + 24) == P.ERR_INVALID_ARG and _adam(P, norm=STEP + 4) == P.ERR_INVALID_ARG


@pytest.mark.parametrize("at", [BASE, BASE + 60, BASE + (2 << 30), STEP + 4, NORM])
def test_adam_refuses_a_rate_that_it_writes(P, at):
    assert _adam(P, {"lr_device": at}) == P.ERR_INVALID_ARG


def test_train_update_refuses_null(P):
    assert P.lib().aecct_train_update(None, None, None, None, None, None, None, None, None, 0, None) == P.ERR_INVALID_ARG


def test_binding_refuses_tensors_that_are_not_on_a_gpu(P):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        P.rms_norm(x)
    with pytest.raises(ValueError):
        P.rms_norm_grad(x, x)
    with pytest.raises(ValueError):
        P.TensorList([x])
    with pytest.raises(ValueError):
        P.rms_norm(torch.zeros(4, 0))
    with pytest.raises(ValueError):
        P.rms_norm(x, code_type=torch.uint8)
    with pytest.raises(ValueError):
        P.rms_norm(x, group=32)
    with pytest.raises(ValueError):
        P.rms_norm(x, res=torch.zeros(4, 8, dtype=torch.float16))
