"""Several rows a block, with a remainder, in every kernel of long rows: the norm and its gradient against the formulas,
and the sum over rows exactly.

Rows of +-1 with eps 0 have rho = 1 and their gradient dy = +-1 makes dgain a sum of +-1: a row that is left out, or taken
twice, moves every column by 1.  Where d is no power of two, mean(h^2) is within 2^-23 of 1; a column's error is then below
rows 2^-22 for rho, and 2^-24 of a partial sum at each of (rows a thread) + 32 additions: below 0.1 for every case here.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_norm import TYPES, _check_grad, _check_norm, _rand  # noqa: E402

LONG = [(1537, d, t) for d in (4097, 5003, 8192, 12345, 16384) for t in ("bf16", "fp16")] + \
       [(1537, d, "fp32") for d in (2049, 4100, 8191, 16384)] + [(777, d, t) for d in (16387, 20000) for t in TYPES]


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


@pytest.mark.parametrize("rows,d,type", LONG)
def test_long_rows_several_a_block(P, rows, d, type):
    print(f"[rows] {rows} x {d} {type}", flush=True)
    t = TYPES[type]
    x, res, dy = (_rand(rows, d, t, d + k) for k in range(3))
    gain = 1 + 0.3 * torch.randn(d, device="cuda", generator=torch.Generator("cuda").manual_seed(d))
    for code, kind, group in (("int8", torch.int8, 0), ("e4m3", torch.float8_e4m3fn, 64)):
        _check_norm(P.rms_norm(x, gain, res, 1e-5, code_type=kind, group=group), x, gain, res, 1e-5, code, group)
    _check_grad(P.rms_norm_grad(x, dy, gain, res), x, dy, gain, res)


@pytest.mark.parametrize("rows,d,type", LONG + [(5888, 32, "fp32"), (1200003, 128, "fp16"), (400007, 128, "fp32"), (300001, 200, "bf16"),
                                                (50003, 4096, "bf16"), (33001, 2051, "fp32"), (9001, 16384, "fp32"), (2049, 1000, "fp16")])
def test_every_row_is_in_dgain_once(P, rows, d, type):
    print(f"[rows] {rows} x {d} {type}", flush=True)
    g = torch.Generator("cuda").manual_seed(d)
    sign = lambda: torch.randint(0, 2, (rows, d), dtype=torch.int8, device="cuda", generator=g).mul_(2).sub_(1)  # noqa: E731
    h, dy = sign(), sign()
    want = sum((a * b).sum(0, dtype=torch.int64) for a, b in zip(h.split(8192), dy.split(8192)))
    _, dgain = P.rms_norm_grad(h.to(TYPES[type]), dy.to(TYPES[type]), None, None, 0.0)
    if d & (d - 1) == 0:
        assert torch.equal(dgain.double(), want.double())
    else:
        assert (dgain.double() - want.double()).abs().max().item() <= 0.25
