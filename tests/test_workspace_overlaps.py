"""A workspace that shares bytes with a tensor of its own call is refused before any GPU work: it is written while they are
read or written (no GPU is needed; the addresses are only compared)."""
import ctypes as C

import pytest

WS = 0x7000_0000_0000
FAR = WS + (1 << 40)


@pytest.fixture(scope="module")
def P():
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _inside(need, size):
    """Addresses of `size` bytes in, across and at both ends of a workspace of `need` bytes."""
    return [WS, WS + 256, WS + 260, WS + need // 8 * 4, WS + need - 4, WS - size + 4]


def _list(P, *items):
    return (P.Tensor * len(items))(*[P.Tensor(*i) for i in items])


def _need(P, n):
    size = C.c_size_t()
    assert P.lib().aecct_update_workspace_size(n, C.byref(size)) == P.OK
    return size.value


@pytest.mark.parametrize("which", ["h", "dy", "dres", "gain", "dh", "dgain"])
def test_norm_grad(P, which):
    rows, d = 4, 64
    size = C.c_size_t()
    assert P.lib().aecct_rms_norm_grad_workspace_size(rows, d, C.byref(size)) == P.OK
    bytes_of = 4 * d if which in ("gain", "dgain") else 4 * d * rows
    for at in _inside(size.value, bytes_of):
        a = P.RmsNormGradArgs(rows=rows, d=d, type=P.F32, gain_type=P.F32, eps=1e-5, h=FAR, ldh=d, dy=FAR + (1 << 30), lddy=d,
                              dres=FAR + (2 << 30), lddres=d, gain=FAR + (3 << 30), dh=FAR + (4 << 30), lddh=d,
                              dgain=FAR + (5 << 30))
        setattr(a, which, at)
        assert P.lib().aecct_rms_norm_grad(C.byref(a), WS, size.value, None) == P.ERR_INVALID_ARG, hex(at)


@pytest.mark.parametrize("which", ["grads", "norm"])
def test_grad_norm(P, which):
    need = _need(P, 2)
    for at in _inside(need, 32 if which == "grads" else 4):
        grads = _list(P, (FAR, 8, 0), (at if which == "grads" else FAR + 64, 8, 0))
        norm = at if which == "norm" else FAR + (1 << 30)
        assert P.lib().aecct_grad_norm(grads, 2, norm, WS, need, None) == P.ERR_INVALID_ARG, hex(at)


@pytest.mark.parametrize("which", ["grads", "out", "norm"])
def test_grad_clip(P, which):
    need = _need(P, 2)
    for at in _inside(need, 4 if which == "norm" else 32):
        grads = _list(P, (FAR, 8, 0), (at if which == "grads" else FAR + 64, 8, 0))
        out = _list(P, (FAR + 256, 8, 0), (at if which == "out" else FAR + 512, 8, 0))
        norm = at if which == "norm" else FAR + (1 << 30)
        assert P.lib().aecct_grad_clip(grads, out, 2, 1.0, norm, WS, need, None) == P.ERR_INVALID_ARG, hex(at)
        if which == "grads":
            assert P.lib().aecct_grad_clip(grads, None, 2, 1.0, norm, WS, need, None) == P.ERR_INVALID_ARG, hex(at)


@pytest.mark.parametrize("which", ["params", "m", "v", "grads", "copies", "step", "norm", "lr"])
def test_adam(P, which):
    need = _need(P, 2)
    for at in _inside(need, {"step": 8, "norm": 4, "lr": 4}.get(which, 32)):
        lists = {k: _list(P, (FAR + (i << 30), 8, 0), (at if which == k else FAR + (i << 30) + 64, 8, 0))
                 for i, k in enumerate(("params", "m", "v", "grads", "copies"))}
        one = {k: at if which == k else FAR + ((10 + i) << 30) for i, k in enumerate(("step", "norm", "lr"))}
        o = P.AdamOptions(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, one["lr"])
        assert P.lib().aecct_adam_step(lists["params"], lists["m"], lists["v"], lists["grads"], lists["copies"], 2, C.byref(o),
                                       one["step"], one["norm"], WS, need, None) == P.ERR_INVALID_ARG, hex(at)
