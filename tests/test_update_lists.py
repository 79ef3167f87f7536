"""Host side of the calls on lists of tensors and on a trainer's: what is refused before any GPU work.  The tensors lie in
host memory and say that they are on a GPU; every call ends before the library would read them."""
import gc
import weakref

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from workloads import random_qat_params  # noqa: E402

M, N, D, LAYERS = 15, 31, 32, 3


@pytest.fixture
def P(monkeypatch):
    import paper_2410_05911_amd as P
    P.lib()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    return P


def _on_gpu(a):
    return torch.from_numpy(np.array(a, dtype=np.float32))


def _params(n=N, m=M, d=D, layers=LAYERS):
    p = random_qat_params(n, m, d, layers, seed=1)
    return {k: {kk: _on_gpu(vv) for kk, vv in v.items()} if k in ("w", "b") else _on_gpu([v] if k == "head_b1" else v)
            for k, v in p.items() if v is not None}


def _trainer(P):
    tr = P.Trainer.__new__(P.Trainer)      # the sizes of a trainer, without the library's handle
    tr.n, tr.m, tr.L, tr.d, tr.n_layers, tr._h = N, M, N + M, D, LAYERS, None
    return tr


def _state(params):
    zeros = lambda t: {k: zeros(v) for k, v in t.items()} if isinstance(t, dict) else torch.zeros_like(t)  # noqa: E731
    return {"m": zeros(params), "v": zeros(params), "step": torch.zeros(1, dtype=torch.int64)}


def test_the_trainers_sizes(P):
    tr = _trainer(P)
    fields = [f for f, _ in P.TrainGrads._fields_]
    assert len(fields) == 22 == len(tr._counts())
    flat = tr._flat(_params())
    assert [flat[f].numel() for f in fields] == tr._counts()


@pytest.mark.parametrize("other", [dict(layers=LAYERS - 1), dict(layers=LAYERS + 1), dict(d=16), dict(n=63, m=18), dict(n=30, m=16)],
                         ids=str)
def test_trainer_update_refuses_another_models_tensors(P, other):
    """Parameters, moments and gradients that fit each other but not the trainer, whose sizes the library goes by."""
    p = _params(**other)
    with pytest.raises(ValueError, match="must be float32"):
        _trainer(P).update(p, p, _state(p), 1e-3, max_norm=1.0)


@pytest.mark.parametrize("which", ["params", "m", "v", "grads"])
@pytest.mark.parametrize("field", ["embed", "delta", "head_bo"])
def test_trainer_update_refuses_one_wrong_size(P, which, field):
    dicts = {k: _params() for k in ("params", "m", "v", "grads")}
    dicts[which][field] = dicts[which][field].reshape(-1)[1:].contiguous()
    state = {"m": dicts["m"], "v": dicts["v"], "step": torch.zeros(1, dtype=torch.int64)}
    with pytest.raises(ValueError, match=field):
        _trainer(P).update(dicts["params"], dicts["grads"], state, 1e-3)


def _backed(values):
    """A tensor and a weak reference that dies with the tensor's memory."""
    a = np.array(values, dtype=np.float32)
    return torch.from_numpy(a), weakref.ref(a)


@pytest.mark.parametrize("make", [lambda P, t: P.TensorList([t]), lambda P, t: P.Adam([t], m=[_backed([0, 0])[0]], v=[_backed([0, 0])[0]],
                                                                                      step=torch.zeros(1, dtype=torch.int64))],
                         ids=["list", "adam"])
def test_kept_lists_hold_the_memory_that_they_point_to(P, make):
    """p.data = ... puts other memory under the same tensor; what the list's addresses point to must not go back to the
    allocator, which would hand it to somebody else before the next update writes there."""
    t, memory = _backed([1, 2])
    kept = make(P, t)
    t.data = _backed([3, 4])[0]
    gc.collect()
    assert memory() is not None
    del kept
    gc.collect()
    assert memory() is None


def test_adams_lists_follow_tensors_that_move(P):
    t, _ = _backed([1, 2])
    kept = P.TensorList([t])
    kept._follow()
    was = kept.array[0].data
    assert was == t.data_ptr()
    t.data = _backed([3, 4, 5])[0]
    assert t.data_ptr() != was
    kept._follow()
    assert kept.array[0].data == t.data_ptr() and kept.array[0].count == 3
    t.data = t.data.double()
    for _ in range(2):            # refused, and again: the list is as it was
        with pytest.raises(ValueError):
            kept._follow()
        assert kept.array[0].count == 3
