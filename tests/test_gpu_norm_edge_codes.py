"""The row norm's 8-bit codes where products h gain leave fp32's normal range, and in rows with NaN, infinities and zeros,
against the formulas in 64 bits.

With u = 2^-24: alpha is off by 64 u and half of fp32's smallest number, 2^-150; a code is the nearest to the exact quotient
h gain Q / max |h gain|, or that quotient is within u of a tie.  An alpha of 0 has codes 0; where alpha is NaN, int8
codes are 0 and e4m3 codes NaN.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _check(P, x, gain, eps, code, group, what):
    kind, most = CODES[code]
    d = x.shape[1]
    _, _, codes, alpha = P.rms_norm(x, gain, None, eps, with_y=False, code_type=kind, group=group)
    size = group or d
    p = x.double() * (1 if gain is None else gain.double())
    rho = 1 / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32)))
    A = torch.stack([q.abs().amax(1) for q in p.split(size, 1)], 1)
    a64 = torch.stack([(q * rho).abs().amax(1) for q in p.split(size, 1)], 1)      # amax hands NaN on
    alpha = alpha.view(a64.shape)
    nan = a64.isnan()
    assert torch.equal(alpha.isnan(), nan), what
    off = (alpha.double() - a64).abs() > 64 * U * a64 + 2.0 ** -150
    assert not off.any(), (what, alpha[off][:4].tolist(), a64[off][:4].tolist())
    at = torch.arange(d, device="cuda") // size
    got = codes.to(torch.float32).double()
    none, dead = (alpha == 0)[:, at], nan[:, at]
    assert (got[none] == 0).all(), (what, "codes of alpha 0")
    assert ((got[dead] == 0) if code == "int8" else got[dead].isnan()).all(), (what, "codes of alpha NaN")
    live = ~(none | dead)
    q = (p * (most / A[:, at]))[live]
    got = got[live]
    step = torch.ones_like(q) if code == "int8" else torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
    bad = ~((got - q).abs() <= 0.5 * step + 1.01 * U * q.abs())
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4].tolist(), q[bad][:4].tolist())


def _gain(d, exponent, columns, seed):
    """1 + 0.3 randn, times 2^exponent in the given columns; made on the host in 64 bits, rounded once."""
    g = 1 + 0.3 * torch.randn(d, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))
    g[columns] *= 2.0 ** exponent
    return g.float().cuda()


EXPONENTS = [-55, -70, -100, -120, -126, -133, -140, -145, -149]


@pytest.mark.parametrize("code", list(CODES))
@pytest.mark.parametrize("d,group", [(100, 32), (256, 64), (300, 128), (1000, 32), (2500, 64), (6000, 128), (9001, 32), (20000, 64)])
def test_groups_of_tiny_products_beside_ordinary_ones(P, d, group, code):
    """Each other group's gains far down, to the smallest numbers, for rows of every size."""
    for type in (torch.float32, torch.bfloat16):
        for scale, eps in ((1.0, 1e-5), (1e-4, 1e-5), (1e-11, 0.0), (1e17, 1e-5), (1e-20, 0.0), (1e25, 1e-5)):
            x = (torch.randn(9, d, device="cuda", generator=torch.Generator("cuda").manual_seed(d)) * scale).to(type)
            for e in EXPONENTS:
                columns = (torch.arange(d) // group) % 2 == 1
                _check(P, x, _gain(d, e, columns, d), eps, code, group, (d, group, type, scale, e))


@pytest.mark.parametrize("code", list(CODES))
@pytest.mark.parametrize("d", [3, 20, 60, 128, 250, 900, 1500, 3000, 6000, 16384, 20000])
def test_rows_of_tiny_products(P, d, code):
    for type in (torch.float32, torch.float16):
        for scale, eps in ((1.0, 1e-5), (1e-4, 1e-5), (100.0, 0.0)):
            x = (torch.randn(9, d, device="cuda", generator=torch.Generator("cuda").manual_seed(d)) * scale).to(type)
            for e in EXPONENTS:
                _check(P, x, _gain(d, e, torch.ones(d, dtype=torch.bool), d), eps, code, 0, (d, type, scale, e))


@pytest.mark.parametrize("code", list(CODES))
def test_a_group_of_a_few_smallest_numbers(P, code):
    """h = 5 times the smallest number and gain 1.25: h gain = 6.25 of it, which fp32 has not; beside a group of ones."""
    x = torch.ones(3, 64, device="cuda")
    x[:, 32:] = 5 * 2.0 ** -149
    x[1, 40] = -5 * 2.0 ** -149
    x[2, 41] = 2.0 ** -149
    _check(P, x, torch.full((64,), 1.25, device="cuda"), 1e-5, code, 32, "smallest")
    x[:, :32] = 1e-3                      # rho of about 250: alpha is not among the smallest numbers
    _check(P, x, torch.full((64,), 1.25, device="cuda"), 1e-5, code, 32, "smallest, larger alpha")


@pytest.mark.parametrize("code", list(CODES))
@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,group", [(20, 0), (64, 32), (100, 32), (250, 64), (300, 128), (900, 0), (1000, 32), (2500, 64), (6000, 128),
                                     (9001, 64), (16384, 128), (20000, 0), (20000, 32)])
def test_rows_with_nan_infinities_and_zeros(P, d, group, type, code):
    """NaN makes every alpha of its row NaN; an infinity makes its own group's NaN and the others' 0; beside ordinary rows."""
    x = torch.randn(11, d, device="cuda", generator=torch.Generator("cuda").manual_seed(d))
    x[1, d // 3] = math.nan
    x[2, d // 3] = math.inf
    x[3, 0] = -math.inf
    x[4] = 0
    x[5, : d // 2] = 0                    # whole groups of zeros
    x[6, d - 1] = math.nan
    x[7, d - 1] = math.inf
    x[8] = -0.0
    x = x.to(type)
    gain = _gain(d, 0, torch.zeros(d, dtype=torch.bool), d)
    for eps in (1e-5, 0.0):
        for g in (gain, None):
            _check(P, x, g, eps, code, group, (d, group, type, eps))
