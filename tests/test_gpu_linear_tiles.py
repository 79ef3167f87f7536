"""Linear maps and their gradients at the sizes that take the large tiles, the split forms and the loads past the registers, by the checks
and tolerances of test_gpu_linear.py.

By plan_gemm, in 16 and 8 bits: 64 x 64 outputs a block below 192 blocks of 128 x 128; 256 x 256 from 256 of them on with a k of 1024
bytes; k is split below 256 blocks.  fp32: 64 x 64 or 128 x 128, split or not, by the time they are estimated to take.  One stage where
k is one tile of 128 bytes.  Four rows and fewer split k from 4 MB of weights on.  Factors whose rows are whole 16-byte pieces at such
addresses go past the registers; others are copied into such where each copied value enters enough products."""
import pytest

import test_gpu_linear as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = base.P


def _aligned(t, pad):
    """The same values in NaN (127 for int8) as base._in_nan, rows at 16-byte addresses and a multiple of 16 values apart."""
    r, c = t.shape
    whole = torch.full((r + 2, -(-c // 16) * 16 + 32 + 16 * (pad % 3)), 127 if t.dtype == torch.int8 else float("nan"), device="cuda").to(t.dtype)
    view = whole[1: 1 + r, 16: 16 + c]
    view.copy_(t)
    return view


@pytest.fixture(params=["aligned", "anywhere"])
def where(request, monkeypatch):
    if request.param == "aligned":
        monkeypatch.setattr(base, "_in_nan", _aligned)
    return request.param


KINDS = ["fp32", "bf16", "fp16", "int8", "e4m3"]


@pytest.mark.parametrize("turned,pad,act,res,y", [(False, 0, "gelu", True, "bf16"), (True, 8, "none", False, "fp32")])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,inputs,outputs", [
    (2000, 208, 1712), (2001, 211, 1713),      # 224 blocks of 128 x 128, ragged at each side
    (3000, 0, 1552),                           # k of one tile
    (1900, 4208, 1696),                        # 210 blocks of 128 x 128, k split in two
    (4100, 1040, 4112), (4100, 1043, 4099),    # 289 blocks of 256 x 256
    (600, 4112, 640), (65, 9000, 129)])        # few blocks of 64 x 64, k split many times
def test_maps(P, where, rows, inputs, outputs, kind, turned, pad, act, res, y):
    inputs = inputs or {"fp32": 32, "int8": 128}.get(kind, 64)
    base.test_linear(P, rows, inputs, outputs, kind, turned, pad, act, res, y)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("inputs,outputs", [(2100, 2104), (5000, 1003), (70, 70000)])
def test_few_rows_with_k_split(P, where, rows, inputs, outputs, kind):
    """More than 4 MB of weights in every type (70 x 70000: 4.9 MB, more than 512 blocks of columns, so not split)."""
    base.test_linear(P, rows, inputs, outputs, kind, False, 0, "silu", True, "fp16")


@pytest.mark.parametrize("turned,pad,act,dw32", [(False, 0, "gelu", False), (True, 8, "none", True)])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,inputs,outputs", [
    (1700, 1712, 1720), (1701, 1711, 1723),    # both products 196 blocks of 128 x 128, k split
    (4100, 4112, 4104), (4099, 4101, 4097),    # 289 blocks of 256 x 256
    (9000, 64, 1552), (257, 1000, 777)])
def test_gradients(P, where, rows, inputs, outputs, kind, turned, pad, act, dw32):
    base.test_linear_grad(P, rows, inputs, outputs, kind, turned, pad, act, dw32)


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,outputs", [(1, 1), (5, 7), (300, 129), (5000, 1000), (40000, 33)])
def test_dbias_without_an_activation(P, rows, outputs, kind):
    """The sums of dy's columns: (rows + 8) u sum|dy|, as with an activation."""
    g = torch.Generator(device="cuda").manual_seed(12)
    t = base.TYPES[kind]
    dy = base._in_nan(base._rand(g, rows, outputs).to(t), 3)
    x, w = base._rand(g, rows, 4).to(t), base._rand(g, 4, outputs).to(t)
    for more in (dict(), dict(with_dx=False), dict(with_dx=False, with_dw=False)):
        dbias = P.linear_grad(x, w, dy, **more)[2]
        base._near(dbias, dy.double().sum(0), (rows + 8) * base.U * dy.double().abs().sum(0), "dbias")


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_captured_with_splits(P, kind):
    """Few rows and few blocks, both with their sums joined by a second launch, replayed between eager calls."""
    g = torch.Generator(device="cuda").manual_seed(13)
    t = base.TYPES[kind]
    w, b = base._rand(g, 2100, 2104).to(t), base._rand(g, 2104)
    xs = [base._rand(g, r, 2100).to(t) for r in (2, 200)]
    dys = [base._rand(g, r, 2104).to(t) for r in (2, 200)]
    call = lambda: [v for x, dy in zip(xs, dys) for v in (P.linear(x, w, b, act="relu")[0], *P.linear_grad(x, w, dy))]  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(3):
        for x in xs:
            x.copy_(base._rand(g, *x.shape))
        want = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, out)), step
