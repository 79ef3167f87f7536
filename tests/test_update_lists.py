"""Host side of the calls on lists of tensors and on a trainer's: what is refused before any GPU work.  The tensors lie in
host memory and only say that they were on a GPU; every call ends before the library would read them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from workloads import random_qat_params  # noqa: E402

M, N, D, LAYERS = 15, 31, 32, 3


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


@pytest.fixture
def P(monkeypatch):
    import paper_2410_05911_amd as P
    P.lib()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return P


def _on_gpu(a):
    return torch.from_numpy(np.array(a, dtype=np.float32)).as_subclass(OnGpu)


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
    return {"m": zeros(params), "v": zeros(params), "step": torch.zeros(1, dtype=torch.int64).as_subclass(OnGpu)}


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
    dicts[which][field] = dicts[which][field].reshape(-1)[1:].contiguous().as_subclass(OnGpu)
    state = {"m": dicts["m"], "v": dicts["v"], "step": torch.zeros(1, dtype=torch.int64).as_subclass(OnGpu)}
    with pytest.raises(ValueError, match=field):
        _trainer(P).update(dicts["params"], dicts["grads"], state, 1e-3)
