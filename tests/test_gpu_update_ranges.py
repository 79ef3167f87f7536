"""The Adam update and clipping of gradients whose squares, or whose factor, leave fp32's range, against the formulas in 64
bits with the tolerances of test_gpu_update.py."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_update import HALF, TINY, TYPES, U, _adam64, _near, _norm64  # noqa: E402


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("size", [1e15, 1.8e19, 2e19, 1e20, 3e20, 5e20])
@pytest.mark.parametrize("beta2", [0.999, 0.99])
def test_second_moment_of_large_gradients(P, type, size, beta2):
    """(1 - beta2) g^2 is a number of fp32 where g^2 is not."""
    if (1 - beta2) * size * size * 1.1 > 3.4e38:
        size = math.sqrt(3e38 / (1 - beta2) / 1.2)
    g = [(torch.linspace(0.25, 1.0, 5003, device="cuda") * size * (1 - 2 * (torch.arange(5003, device="cuda") % 2))).to(TYPES[type])]
    p, m, v = ([t] for t in (torch.randn(5003, device="cuda", generator=torch.Generator("cuda").manual_seed(1)), torch.zeros(5003, device="cuda"), torch.zeros(5003, device="cuda")))
    before = [t[0].clone() for t in (p, m, v)]
    opt = P.Adam(p, 1e-3, (0.9, beta2), m=m, v=v)
    opt.step(g)
    p2, m2, v2, pb, mb, vb = _adam64(before[0], before[1], before[2], g[0], 1.0, 1, 1e-3, 0.9, beta2, 1e-8, 0.0)
    for got, want, bound, what in ((p[0], p2, pb, "param"), (m[0], m2, mb, "m"), (v[0], v2, vb, "v")):
        assert got.isfinite().all(), what
        _near(got, want, bound, what)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-10, 1e-18, 1e-21, 1e-25, 1e-33, 1e-38, 1e-42, 1e-45, 1e-60])
def test_clipping_by_factors_far_below_one(P, type, max_norm):
    """The largest gradients clipped to norms down to the smallest numbers, and small ones beside them."""
    g = [(torch.linspace(0.1, 1.0, 300, device="cuda") * 3e38).to(TYPES[type]), torch.tensor([1e30, -1e10, 1.0, 1e-30, 1e-45, 0.0], device="cuda")]
    want = _norm64(g)
    keep = [t.clone() for t in g]
    P.grad_clip(g, max_norm)
    for a, k in zip(g, keep):
        x = k.double() * (max_norm / want)
        _near(a, x, (2.1 * U + HALF[a.dtype]) * x.abs() + TINY[a.dtype], max_norm)
