"""The row norm (rms_norm) and its gradient against their formulas in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and w = half a step of the stored type:
  h      one fp32 addition and the rounding to the type: (u + w) |h|
  y      at most 80 additions in a row's sum of squares (64 a thread, then a tree), halved by the square root, and 10
         more roundings: 64 u |y|, then w |y|; alpha the same without w
  codes  in code units q = y Q / alpha: int8 1/2, e4m3 |q| 2^-4 or half its smallest step 2^-10, and 132 u |q| for y and
         alpha
  dh     rho (dy g - xh c) + dres with rho and xh off by 64 u, c by 140 u mean|dy g xh|
  dgain  60 u a term, and the additions of R terms, at most 512 partial sums of R / 512 terms: u sum|dy xh| each
An output in fp16 may also round below its normal range: half of 2^-24.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _rand(rows, d, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, d + pad, device="cuda", generator=g) * scale
    x[:, :: max(1, d // 4)] *= 6
    return x.to(dtype)[:, :d] if pad else x.to(dtype)


def _near(got, want, bound, what):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(),
                           torch.as_tensor(bound, device=got.device).expand_as(got)[bad][:4].tolist())


def _formula(x, gain, res, eps):
    h = x.double() + (res.double() if res is not None else 0)
    rho = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, h * rho * (gain.double() if gain is not None else 1)


def _check_norm(out, x, gain, res, eps, code, group):
    y, h, codes, alpha = out
    t = x.dtype
    hh, yy = _formula(x, gain, res, float(np.float32(eps)))
    if h is not None:
        _near(h, hh, (U + HALF[t]) * hh.abs() + TINY[t], "h")
    if y is not None:
        _near(y, yy, (64 * U + HALF[t]) * yy.abs() + TINY[t], "y")
    if code is None:
        assert codes is None and alpha is None
        return
    kind, most = CODES[code]
    d = x.shape[-1]
    step = group if group else d
    parts = [p.abs().amax(-1) for p in yy.split(step, -1)]
    a = torch.stack(parts, -1)
    assert codes.dtype == kind and alpha.shape == (a.shape if group else a.shape[:-1])
    _near(alpha.reshape(a.shape), a, 64 * U * a + 2.0 ** -149, "alpha")
    scale = a[..., torch.arange(d, device="cuda") // step]
    q = torch.where(scale > 0, yy * most / scale.clamp_min(1e-300), 0)
    slack = 0.5 if code == "int8" else (q.abs() * 2.0 ** -4).clamp_min(2.0 ** -10)
    _near(codes.to(torch.float32), q, slack + 132 * U * q.abs(), "codes")


DS = [1, 2, 7, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049,
      4096, 4097, 5003, 8192, 8200, 12345, 16384, 16387, 32768, 40001, 65536]


@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("type", list(TYPES))
def test_norm_widths(P, d, type):
    print(f"[norm] d {d} {type}", flush=True)
    t = TYPES[type]
    for rows, pad, with_res, code, group in ((1, 0, True, "int8", 0), (5, 3, False, "e4m3", 128), (19, 0, True, None, 0),
                                             (67, 1, True, "int8", 32), (3, 0, True, "e4m3", 64)):
        if rows * d > 1 << 21:
            rows = 2
        x, res = _rand(rows, d, t, d + rows, pad), _rand(rows, d, t, 7 * d + rows, pad) if with_res else None
        gain = 1 + 0.3 * torch.randn(d, device="cuda")
        if rows % 2 == 0:
            gain = gain.to(t)
        out = P.rms_norm(x, gain, res, 1e-5, code_type=CODES[code][0] if code else None, group=group)
        _check_norm(out, x, gain, res, 1e-5, code, group)
        assert (out[1] is None) == (res is None)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 15, 255, 256, 257, 1023, 2049, 4099, 10007])
@pytest.mark.parametrize("type,d", [("fp32", 32), ("fp32", 128), ("bf16", 64), ("bf16", 1000), ("fp16", 333), ("bf16", 4096)])
def test_norm_row_counts(P, rows, type, d):
    print(f"[norm] rows {rows} d {d} {type}", flush=True)
    x, res = _rand(rows, d, TYPES[type], rows), _rand(rows, d, TYPES[type], rows + 1)
    gain = torch.randn(d, device="cuda")
    _check_norm(P.rms_norm(x, gain, res, 1e-6, code_type=torch.int8), x, gain, res, 1e-6, "int8", 0)
    _check_norm(P.rms_norm(x, None, None, 1e-6, code_type=torch.float8_e4m3fn, group=32), x, None, None, 1e-6, "e4m3", 32)


@pytest.mark.parametrize("type", list(TYPES))
def test_norm_in_place_and_beside(P, type):
    """h and y over x and res, columns of one wider buffer, and nothing written outside the rows."""
    t = TYPES[type]
    for rows, d in ((9, 96), (130, 1111), (3, 9000)):
        x, res = _rand(rows, d, t, 3), _rand(rows, d, t, 4)
        gain = torch.randn(d, device="cuda")
        want = P.rms_norm(x, gain, res, code_type=torch.int8)
        x1, r1 = x.clone(), res.clone()
        y, h, codes, alpha = P.rms_norm(x1, gain, r1, y=x1, h=r1, code_type=torch.int8)
        assert y is x1 and h is r1
        for a, b in zip((y, h, codes, alpha), want):
            assert torch.equal(a, b)
        x2 = x.clone()
        y2, h2, _, _ = P.rms_norm(x2, gain, res, h=x2)
        assert torch.equal(h2, want[1]) and torch.equal(y2, want[0])
        wide = torch.full((rows, 4 * d + 7), 77.0, device="cuda", dtype=t)
        wide[:, 1:d + 1] = x
        wide[:, d + 2:2 * d + 2] = res
        P.rms_norm(wide[:, 1:d + 1], gain, wide[:, d + 2:2 * d + 2], y=wide[:, 2 * d + 3:3 * d + 3], h=wide[:, 3 * d + 4:4 * d + 4])
        assert torch.equal(wide[:, 2 * d + 3:3 * d + 3], want[0]) and torch.equal(wide[:, 3 * d + 4:4 * d + 4], want[1])
        assert torch.equal(wide[:, 1:d + 1], x) and torch.equal(wide[:, d + 2:2 * d + 2], res)
        rest = torch.cat([wide[:, c:c + 1] for c in (0, d + 1, 2 * d + 2, 3 * d + 3, 4 * d + 4, 4 * d + 6)], 1)
        assert (rest == 77.0).all()
        guard = torch.full((rows + 2, d + 5), 9, device="cuda", dtype=torch.int8)
        _, _, c3, a3 = P.rms_norm(x, gain, res, codes=guard[1:-1, 2:d + 2], with_y=False, code_type=torch.int8)
        assert torch.equal(c3, want[2]) and torch.equal(a3, want[3])
        guard[1:-1, 2:d + 2] = 9
        assert (guard == 9).all()


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("d", [1, 3, 5, 7, 259, 770, 1541, 2051, 2561, 4097, 5635, 8197, 12289, 16385])
def test_in_place_with_short_ends(P, type, d):
    """Rows whose last few values are another lane's or wavefront's neighbours, written over every input in turn."""
    t, rows = TYPES[type], 700
    x, res, dy = (_rand(rows, d, t, k) for k in (5, 6, 7))
    gain = torch.randn(d, device="cuda")
    want = P.rms_norm(x, gain, res, code_type=torch.int8)
    for k in range(2):
        a = [x.clone(), res.clone()]
        got = P.rms_norm(a[0], gain, a[1], h=a[k], y=a[1 - k], code_type=torch.int8)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    alone = P.rms_norm(x, gain)[0]
    a = x.clone()
    assert torch.equal(P.rms_norm(a, gain, y=a)[0], alone)
    dh, dg = P.rms_norm_grad(x, dy, gain, res)
    for k in range(3):
        a = [x.clone(), dy.clone(), res.clone()]
        got, g2 = P.rms_norm_grad(a[0], a[1], gain, a[2], dh=a[k])
        assert torch.equal(got, dh) and torch.equal(g2, dg)


def test_norm_shapes_and_broadcast_rows(P):
    x = _rand(24, 40, torch.bfloat16, 1).view(2, 3, 4, 40)
    y, h, codes, alpha = P.rms_norm(x, code_type=torch.int8, group=32)
    assert y.shape == x.shape and codes.shape == x.shape and alpha.shape == (2, 3, 4, 2) and h is None
    one = P.rms_norm(x.view(24, 40), code_type=torch.int8, group=32)
    assert torch.equal(y.view(24, 40), one[0]) and torch.equal(alpha.view(24, 2), one[3])
    v = P.rms_norm(x[0, 0, 0], code_type=torch.int8)
    assert v[0].shape == (40,) and v[3].shape == () and torch.equal(v[0], y[0, 0, 0])
    row = _rand(1, 200, torch.float32, 2)
    res = _rand(31, 200, torch.float32, 3)
    a = P.rms_norm(row.expand(31, 200), None, res)
    b = P.rms_norm(row.expand(31, 200).contiguous(), None, res)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    e = torch.empty(0, 64, device="cuda")
    y, h, codes, alpha = P.rms_norm(e, torch.ones(64, device="cuda"), e, code_type=torch.int8, group=32)
    assert y.shape == (0, 64) and alpha.shape == (0, 2)


@pytest.mark.parametrize("d", [5, 32, 50, 100, 250, 300, 2000, 3000, 9000, 20000])
def test_norm_of_extreme_rows(P, d):
    """Zeros, one outlier, squares past fp32's range at both ends, NaN and infinities, beside ordinary rows."""
    x = torch.randn(10, d, device="cuda")
    x[0] = 0
    x[1] *= 1e25
    x[2] *= 1e-25
    x[3] = 0
    x[3, d // 2] = 3e38
    x[4, d // 3] = math.nan
    x[5, d // 3] = math.inf
    x[6] = 1e-42
    x[7] = -0.0
    gain = 1 + torch.rand(d, device="cuda")
    for eps in (1e-5, 0.0):
        y, _, codes, alpha = P.rms_norm(x, gain, None, eps, code_type=torch.int8)
        _, _, fcodes, falpha = P.rms_norm(x, gain, None, eps, with_y=False, code_type=torch.float8_e4m3fn)
        good = [1, 2, 3, 8, 9] + ([0, 6, 7] if eps else [6])
        _check_norm((y[good], None, codes[good], alpha[good]), x[good], gain, None, eps, "int8", 0)
        _check_norm((y[good], None, fcodes[good], falpha[good]), x[good], gain, None, eps, "e4m3", 0)
        assert y[4].isnan().all() and alpha[4].isnan() and (codes[4] == 0).all() and fcodes[4].float().isnan().all()
        assert y[5, d // 3].isnan() and (torch.cat([y[5, :d // 3], y[5, d // 3 + 1:]]) == 0).all()
        assert alpha[5].isnan() and (codes[5] == 0).all()
    assert (codes[0] == 0).all()                     # eps 0, a row of zeros: 0 / 0 is NaN
    assert y[0].isnan().all()
    group = P.rms_norm(x[5:6], gain, None, code_type=torch.int8, group=32)[3] if d > 32 else None
    if group is not None:                            # only the group that holds the infinity has no scale
        k = (d // 3) // 32
        assert group[0, k].isnan() and (torch.cat([group[0, :k], group[0, k + 1:]]) == 0).all()


@pytest.mark.parametrize("d", [20, 60, 100, 200, 250, 900, 1500, 3000, 6000, 10000])
@pytest.mark.parametrize("type", ["fp32", "bf16"])
def test_norm_grad_of_extreme_rows(P, d, type):
    """Rows whose squares leave fp32's range beside ordinary ones, which keep their values bit for bit."""
    h, dy = _rand(37, d, TYPES[type], 1), _rand(37, d, TYPES[type], 2)
    plain, _ = P.rms_norm_grad(h, dy)
    odd = torch.arange(0, 37, 5, device="cuda")
    far = h.clone()
    for i, r in enumerate(odd.tolist()):
        far[r] *= (1e25, 1e-25, 0.0, 1e30)[i % 4]
    dh, dgain = P.rms_norm_grad(far, dy)
    keep = torch.ones(37, dtype=torch.bool, device="cuda")
    keep[odd] = False
    assert torch.equal(dh[keep], plain[keep])
    _check_grad((dh, dgain), far, dy, None, None)


def test_norm_codes_of_tiny_values(P):
    """alphas down to the smallest fp32 numbers: the quotient Q / alpha alone would overflow."""
    x = torch.randn(40, 256, device="cuda")
    gain = torch.ones(256, device="cuda")
    for scale in (1e-30, 1e-37, 1e-38):
        for code in ("int8", "e4m3"):
            g = gain * scale
            y, _, codes, alpha = P.rms_norm(x, g, code_type=CODES[code][0])
            most = CODES[code][1]
            yd, a = y.double(), y.abs().amax(1).double()
            assert torch.equal(alpha.double(), a)
            q = yd * most / a[:, None]
            slack = 0.5 if code == "int8" else (q.abs() * 2.0 ** -4).clamp_min(2.0 ** -10)
            _near(codes.to(torch.float32), q, slack + 8 * U * q.abs(), (scale, code))


def test_norm_past_32_bit_offsets(P):
    """Rows of a buffer of 4.6e9 values."""
    wide = torch.empty(70001, 65536, device="cuda", dtype=torch.bfloat16)
    x = wide[:, 100:133]
    x.copy_(_rand(70001, 33, torch.bfloat16, 5))
    y, h, codes, alpha = P.rms_norm(x, None, x, y=wide[:, 1000:1033], code_type=torch.int8)
    _check_norm((y, h, codes, alpha), x, None, x, 1e-5, "int8", 0)
    dh, dg = P.rms_norm_grad(x, y, None, None, dh=wide[:, 2000:2033])
    ref, rg = P.rms_norm_grad(x.contiguous(), y.contiguous())
    assert torch.equal(dh, ref) and torch.equal(dg, rg)


def _grad_formula(h, dy, gain, dres, eps):
    hd, g = h.double(), dy.double() * (gain.double() if gain is not None else 1)
    rho = 1 / torch.sqrt((hd * hd).mean(-1, keepdim=True) + eps)
    xh = hd * rho
    c = (g * xh).mean(-1, keepdim=True)
    m = (g * xh).abs().mean(-1, keepdim=True)
    dh = rho * (g - xh * c)
    bound = U * (64 * rho * (g.abs() + (xh * c).abs()) + 140 * rho * xh.abs() * m)
    if dres is not None:
        dh = dh + dres.double()
        bound = bound + 2 * U * (dh.abs() + dres.double().abs())
    terms = dy.double() * xh
    rows = h.shape[0]
    return dh, bound + HALF[h.dtype] * dh.abs() + TINY[h.dtype], terms.sum(0), \
        U * (60 + min(rows, 600 + rows / 256)) * terms.abs().sum(0) + 2.0 ** -149


def _check_grad(out, h, dy, gain, dres, eps=1e-5):
    want, bound, dgain, gbound = _grad_formula(h, dy, gain, dres, float(np.float32(eps)))
    _near(out[0], want, bound, "dh")
    _near(out[1], dgain, gbound, "dgain")


@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("type", list(TYPES))
def test_norm_grad_widths(P, d, type):
    print(f"[norm grad] d {d} {type}", flush=True)
    t = TYPES[type]
    for rows, pad, with_res, with_gain in ((1, 0, True, True), (6, 3, False, True), (37, 1, True, False)):
        if rows * d > 1 << 21:
            rows = 2
        h, dy = _rand(rows, d, t, d + rows, pad), _rand(rows, d, t, 3 * d + rows, pad, 0.1)
        dres = _rand(rows, d, t, 5 * d + rows, 2 * pad, 0.1) if with_res else None
        gain = 1 + 0.3 * torch.randn(d, device="cuda") if with_gain else None
        if with_gain and rows % 2 == 0:
            gain = gain.to(t)
        _check_grad(P.rms_norm_grad(h, dy, gain, dres), h, dy, gain, dres)


@pytest.mark.parametrize("rows", [1, 2, 3, 8, 15, 511, 512, 513, 1025, 4099, 20011])
@pytest.mark.parametrize("type,d", [("fp32", 32), ("fp32", 128), ("bf16", 64), ("bf16", 1000), ("fp16", 333), ("fp32", 2500)])
def test_norm_grad_row_counts(P, rows, type, d):
    print(f"[norm grad] rows {rows} d {d} {type}", flush=True)
    t = TYPES[type]
    h, dy, dres = _rand(rows, d, t, rows), _rand(rows, d, t, rows + 1, 0, 0.1), _rand(rows, d, t, rows + 2, 0, 0.1)
    gain = torch.randn(d, device="cuda")
    out = P.rms_norm_grad(h, dy, gain, dres)
    _check_grad(out, h, dy, gain, dres)
    again = P.rms_norm_grad(h, dy, gain, dres)
    assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1])


def test_norm_grad_outputs(P):
    """Without dgain, in place, no rows, extreme rows."""
    h, dy, dres = (_rand(70, 500, torch.bfloat16, k) for k in (1, 2, 3))
    gain = torch.randn(500, device="cuda")
    dh, dg = P.rms_norm_grad(h, dy, gain, dres)
    only, none = P.rms_norm_grad(h, dy, gain, dres, with_dgain=False)
    assert none is None and torch.equal(only, dh)
    for k in range(3):
        a = [h.clone(), dy.clone(), dres.clone()]
        got, g2 = P.rms_norm_grad(a[0], a[1], gain, a[2], dh=a[k])
        assert got is a[k] and torch.equal(got, dh) and torch.equal(g2, dg)
    e = torch.empty(0, 500, device="cuda")
    z, zg = P.rms_norm_grad(e, e)
    assert z.shape == (0, 500) and (zg == 0).all()
    x = torch.randn(6, 300, device="cuda")
    x[0] = 0
    x[1] *= 1e25
    x[2] *= 1e-25
    g = torch.randn(6, 300, device="cuda")
    _check_grad(P.rms_norm_grad(x, g), x, g, None, None)
    x[3, 7] = math.nan
    x[4, 8] = math.inf
    dh, dg = P.rms_norm_grad(x, g)
    assert dh[3].isnan().all() and dh[[0, 1, 2, 5]].isfinite().all()
    wrt = P.rms_norm_grad(x[[0, 1, 2, 5]], g[[0, 1, 2, 5]])[0]
    assert torch.equal(dh[[0, 1, 2, 5]], wrt)


@pytest.mark.parametrize("d", [17, 128, 700])
def test_norm_grad_against_differences(P, d):
    """The library's own forward, in central differences along random directions: the loss sum(dy y) + sum(dres h) summed
    in 64 bits.  With a step of 2^-8 the truncation is of third order, about (2^-8)^2 of the value; the forward's fp32
    rounding, 64 u |y dy| summed in quadrature over n values, is divided by the step."""
    h, dy, dres = (_rand(4, d, torch.float32, k + d) for k in (1, 2, 3))
    gain = 1 + 0.2 * torch.randn(d, device="cuda")
    dh, dg = P.rms_norm_grad(h, dy, gain, dres)
    step = 2.0 ** -8

    def loss(hh, gg):
        y = P.rms_norm(hh, gg)[0].double()
        return (dy.double() * y).sum() + (dres.double() * hh.double()).sum()
    for seed in range(3):
        vh, vg = torch.randn(4, d, device="cuda"), torch.randn(d, device="cuda")
        y = P.rms_norm(h, gain)[0].double()
        noise = 64 * U * (dy.double() * y).norm().item() / step
        up, down = h + step * vh, h - step * vh
        want = (loss(up, gain) - loss(down, gain)).item() / (2 * step)
        got = (dh.double() * ((up - down) / (2 * step)).double()).sum().item()
        size = (dh.double().abs() * vh.double().abs()).sum().item()
        assert abs(got - want) <= 16 * step ** 2 * size + noise, (got, want)
        want = (loss(h, gain + step * vg) - loss(h, gain - step * vg)).item() / (2 * step)
        got = (dg.double() * vg.double()).sum().item()
        assert abs(got - want) <= 2 * noise + 1e-5 * (dg.double().abs() * vg.double().abs()).sum().item()


def test_norm_on_other_streams_and_in_graphs(P):
    x, res, dy = (_rand(300, 768, torch.bfloat16, k) for k in (1, 2, 3))
    gain = torch.randn(768, device="cuda")
    want = P.rms_norm(x, gain, res, code_type=torch.int8, group=64)
    wdh, wdg = P.rms_norm_grad(want[1], dy, gain, dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = P.rms_norm(x, gain, res, code_type=torch.int8, group=64, stream=s)
    gdh, gdg = P.rms_norm_grad(got[1], dy, gain, dy, stream=s)
    s.synchronize()
    for a, b in zip(want + (wdh, wdg), got + (gdh, gdg)):
        assert torch.equal(a, b)
    xs, rs, ds = x.clone(), res.clone(), dy.clone()
    graphs = []
    for _ in range(2):      # two graphs of the same calls, replayed in turn with eager work between
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, h, codes, alpha = P.rms_norm(xs, gain, rs, code_type=torch.int8, group=64)
            dh, dg = P.rms_norm_grad(h, ds, gain, ds)
        graphs.append((graph, (y, h, codes, alpha, dh, dg)))
    for k in range(4):
        new = [_rand(300, 768, torch.bfloat16, 10 + 3 * k + j) for j in range(3)]
        for a, b in zip((xs, rs, ds), new):
            a.copy_(b)
        eager = P.rms_norm(new[0], gain, new[1], code_type=torch.int8, group=64)
        eager += P.rms_norm_grad(eager[1], new[2], gain, new[2])
        for graph, outs in graphs:
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, eager):
                assert torch.equal(a, b)


def test_norm_binding_refuses(P):
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(ValueError):
        P.rms_norm(x.t())
    with pytest.raises(ValueError):
        P.rms_norm(x, res=torch.zeros(4, 9, device="cuda"))
    with pytest.raises(ValueError):
        P.rms_norm(x, gain=torch.ones(9, device="cuda"))
    with pytest.raises(ValueError):
        P.rms_norm(x.double())
    with pytest.raises(ValueError):
        P.rms_norm(x, code_type=torch.int8, alpha=torch.empty(4, 1, device="cuda"))
    with pytest.raises(ValueError):
        P.rms_norm(x, code_type=torch.int8, codes=torch.empty(4, 8, device="cuda"))
    with pytest.raises(ValueError):
        P.rms_norm_grad(x, x, dgain=torch.empty(7, device="cuda"))
    with pytest.raises(P.AecctError) as e:
        P.rms_norm(x, gain=torch.ones(8, device="cuda", dtype=torch.float16))
    assert e.value.status == P.ERR_INVALID_ARG
    with pytest.raises(P.AecctError) as e:
        P.rms_norm(x, y=x[:, :], h=x)
    assert e.value.status == P.ERR_INVALID_ARG
    with pytest.raises(P.AecctError) as e:
        P.rms_norm(torch.zeros(1, 65537, device="cuda"))
    assert e.value.status == P.ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,d,type", [(50003, 4096, "bf16"), (33001, 2051, "fp32"), (9001, 16384, "fp32"), (1200003, 128, "fp16")])
def test_norm_of_large_batches(P, rows, d, type):
    """Inputs and outputs larger than the caches (read and written past them), many rows a block; compared on a spread of
    rows, and dgain in whole."""
    print(f"[norm] {rows} x {d} {type}", flush=True)
    t = TYPES[type]
    x, res = _rand(rows, d, t, 1), _rand(rows, d, t, 2)
    gain = 1 + 0.3 * torch.randn(d, device="cuda")
    y, h, codes, alpha = P.rms_norm(x, gain, res, code_type=torch.int8, group=64)
    at = torch.cat([torch.arange(0, rows, 97, device="cuda"), torch.arange(rows - 40, rows, device="cuda")])
    _check_norm((y[at], h[at], codes[at], alpha[at]), x[at], gain, res[at], 1e-5, "int8", 64)
    dh, dgain = P.rms_norm_grad(h, x, gain, res)
    want, bound, _, _ = _grad_formula(h[at], x[at], gain, res[at], float(np.float32(1e-5)))
    _near(dh[at], want, bound, "dh")
    total, size = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    for hp, xp in zip(h.split(4096), x.split(4096)):
        hd = hp.double()
        terms = xp.double() * hd / torch.sqrt((hd * hd).mean(1, keepdim=True) + float(np.float32(1e-5)))
        total += terms.sum(0)
        size += terms.abs().sum(0)
    _near(dgain, total, U * (60 + 600 + rows / 256) * size, "dgain")


def test_norm_of_more_rows_than_32_bits_count(P):
    """2^31 + 70 rows of one value, all of them one row of memory."""
    rows = 2 ** 31 + 70
    x = torch.tensor([[-3.0]], device="cuda", dtype=torch.bfloat16)
    y = torch.zeros(rows, 1, device="cuda", dtype=torch.bfloat16)
    P.rms_norm(x.expand(rows, 1), None, None, 0.0, y=y)
    assert (y[:100] == -1).all() and (y[-100:] == -1).all() and y.min().item() == -1 and y.max().item() == -1


@pytest.mark.parametrize("rows,d,type", [(60011, 1203, "bf16"), (40009, 512, "fp32")])
def test_large_inputs_beside_one_broadcast_row(P, rows, d, type):
    """x, res, dy and dres in turn one row for all, beside more than the caches hold: as with the row written out."""
    x, row = _rand(rows, d, TYPES[type], 1), _rand(1, d, TYPES[type], 2).expand(rows, d)
    full = row.contiguous()
    for a, b in (((x, row), (x, full)), ((row, x), (full, x))):
        got, want = P.rms_norm(a[0], None, a[1], code_type=torch.int8), P.rms_norm(b[0], None, b[1], code_type=torch.int8)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    for k in range(3):
        a, b = [x, x, x], [x, x, x]
        a[k], b[k] = row, full
        got, want = (P.rms_norm_grad(s[0], s[1], None, s[2]) for s in (a, b))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("d", [7, 200, 3001, 20000])
def test_norm_with_single_outputs(P, d):
    """h alone, codes alone, dgain alone (through the C ABI, which takes any of them)."""
    import ctypes as C
    x, res = _rand(37, d, torch.bfloat16, 1), _rand(37, d, torch.bfloat16, 2)
    y, h, codes, alpha = P.rms_norm(x, None, res, code_type=torch.float8_e4m3fn)
    h2 = torch.empty_like(x)
    P.rms_norm(x, None, res, h=h2, with_y=False)
    assert torch.equal(h2, h)
    none, _, c2, a2 = P.rms_norm(h, None, None, with_y=False, code_type=torch.int8)
    c3 = P.rms_norm(h, None, None, code_type=torch.int8)
    assert none is None and torch.equal(c2, c3[2]) and torch.equal(a2, c3[3])
    dh, dgain = P.rms_norm_grad(h, x)
    only = torch.empty(d, device="cuda")
    size = C.c_size_t()
    assert P.lib().aecct_rms_norm_grad_workspace_size(37, d, C.byref(size)) == P.OK
    for shift in (0, 4):     # a workspace at any place
        ws = torch.full((size.value + shift,), 255, dtype=torch.uint8, device="cuda")
        a = P.RmsNormGradArgs(37, d, P.BF16, P.F32, 1e-5, h.data_ptr(), d, x.data_ptr(), d, None, 0, None, None, 0, only.data_ptr())
        assert P.lib().aecct_rms_norm_grad(C.byref(a), ws.data_ptr() + shift, size.value, None) == P.OK
        assert torch.equal(only, dgain)


@pytest.mark.parametrize("d,group", [(32, 0), (128, 0), (1000, 0), (1000, 32), (4096, 128), (9001, 0), (9001, 64), (30000, 0), (30000, 128)])
def test_norm_codes_are_the_exact_ones_but_at_ties(P, d, group):
    """Without a residual h is exact, and a code's quotient h gain Q / max|h gain| (rho drops out) is off by its own last
    rounding only, u of it: the code is the nearest to the exact quotient, or the quotient is within u of a tie."""
    rows = 400 if d < 5000 else 60
    for type in TYPES:
        x = _rand(rows, d, TYPES[type], d)
        gain = 1 + 0.3 * torch.randn(d, device="cuda")
        p = x.double() * gain.double()
        a = torch.stack([q.abs().amax(1) for q in p.split(group or d, 1)], 1)[:, torch.arange(d, device="cuda") // (group or d)]
        for code, (kind, most) in CODES.items():
            q = p * most / a
            got = P.rms_norm(x, gain, None, 1e-5, with_y=False, code_type=kind, group=group)[2].to(torch.float32).double()
            step = torch.ones_like(q) if code == "int8" else torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
            _near(got, q, 0.5 * step + 1.01 * U * q.abs(), (type, code))
