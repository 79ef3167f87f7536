"""Linear maps with an epilogue (linear) and their gradients (linear_grad) against their formulas in 64 bits.

Every input is a view whose surroundings hold NaN, so that a value read past an end shows in the result.

Tolerances, with u = 2^-24 and w = half a step of the stored type:
  sums    K products summed in fp32 in any order, each addition off by at most 2 u of its result: 2 (K + 8) u sum|x w|
  codes   int8 sums are exact below 2^24, and rounded once above: 6 u |v| for the sum, alpha / Q, and the two products
  bias    u (|v| + |bias|)
  act     slopes are at most 1.13; erf, exp and the products around them: 8 u (|z| + |y|)
  y       one more addition and the rounding to the type: u |y| + w |y|
  dz      the slope's 12 u (1 + |z|) |dy|, and w |dz| for its rounding in 16-bit types
  dbias   rows + 8 additions: (rows + 8) u sum|dz|
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}
ACTS = {"none": lambda z: z, "relu": lambda z: torch.where(z > 0, z, 0 * z), "gelu": lambda z: z * torch.special.ndtr(z),
        "silu": lambda z: z * torch.sigmoid(z)}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _in_nan(t, pad):
    """The same values as a view of a buffer of NaN (or 127 for int8): rows `pad` values wider, and some rows around."""
    r, c = t.shape
    whole = torch.full((r + 2, c + pad + 3), 127 if t.dtype == torch.int8 else float("nan"), device="cuda").to(t.dtype)
    view = whole[1: 1 + r, 1: 1 + c] if pad else whole.view(-1)[3: 3 + r * c].view(r, c)
    view.copy_(t)
    return view


def _rand(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _near(got, want, bound, what):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got.numel(), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(),
                           torch.as_tensor(bound, device=got.device).expand_as(got)[bad][:4].tolist())


def _case(rows, inputs, outputs, kind, turned, pad, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[kind]
    s = {}
    if kind == "int8":
        x = torch.randint(-127, 128, (rows, inputs), device="cuda", generator=g, dtype=torch.int8)
        w = torch.randint(-128, 128, (inputs, outputs), device="cuda", generator=g, dtype=torch.int8)
    elif kind == "e4m3":
        x, w = (_rand(g, rows, inputs) * 100).clamp(-448, 448).to(t), (_rand(g, inputs, outputs) * 100).clamp(-448, 448).to(t)
    else:
        x, w = _rand(g, rows, inputs).to(t), _rand(g, inputs, outputs).mul(inputs ** -0.5).to(t)
    if kind in ("int8", "e4m3"):
        s["alpha"] = 0.5 + torch.rand(rows, device="cuda", generator=g)
        s["scale"] = (0.5 + torch.rand(outputs, device="cuda", generator=g)) / (100 if kind == "int8" else 10000) / inputs ** 0.5
    s["x"] = _in_nan(x, pad)
    s["w"] = _in_nan(w.t().contiguous(), pad).t() if turned else _in_nan(w, pad)
    s["bias"] = 0.3 * _rand(g, outputs)
    s["g"] = g
    return s


SIZES = [(1, 1, 1), (1, 64, 64), (2, 7, 5), (1, 1000, 33), (33, 65, 31), (64, 128, 64), (65, 127, 129), (130, 257, 67), (7, 3001, 130),
         (300, 96, 513), (2049, 64, 255)]


@pytest.mark.parametrize("rows,inputs,outputs", SIZES)
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16", "int8", "e4m3"])
@pytest.mark.parametrize("turned,pad,act,res,y", [(False, 0, "none", False, "fp32"), (True, 0, "relu", True, "bf16"),
                                                   (False, 5, "gelu", True, "fp16"), (True, 8, "silu", False, "fp32")])
def test_linear(P, rows, inputs, outputs, kind, turned, pad, act, res, y):
    print(f"[linear] {rows} x {inputs} -> {outputs} {kind} turned {turned} pad {pad} {act}", flush=True)
    s = _case(rows, inputs, outputs, kind, turned, pad, 1)
    yt = TYPES[y] if kind in ("int8", "e4m3") else TYPES[kind]
    r = _in_nan(_rand(s["g"], rows, outputs).to(yt), pad) if res else None
    out = torch.full((rows, outputs + pad), 77.0, device="cuda", dtype=yt)
    got, z = P.linear(s["x"], s["w"], s["bias"], r, act, alpha=s.get("alpha"), scale=s.get("scale"), y=out[:, :outputs], y_type=yt,
                      with_z=True)
    assert got.data_ptr() == out.data_ptr() and bool((out[:, outputs:] == 77).all())
    x, w = s["x"].double(), s["w"].double()
    v, each = x @ w, x.abs() @ w.abs()
    if kind in ("int8", "e4m3"):
        most = (s["alpha"].double() / (127 if kind == "int8" else 448))[:, None] * s["scale"].double()
        v, each = v * most, each * most
    err = 2 * (inputs + 8) * U * each if kind != "int8" else 6 * U * v.abs()
    if kind == "e4m3":
        err = err + 6 * U * v.abs()
    zz = v + s["bias"].double()
    err = err + U * (v.abs() + s["bias"].double().abs())
    _near(z, zz, err + HALF[yt] * zz.abs() + TINY[yt], "z")
    a = ACTS[act](zz)
    yy = a + (r.double() if res else 0)
    _near(got, yy, 1.13 * err + 8 * U * (zz.abs() + a.abs()) + (U + HALF[yt]) * yy.abs() + TINY[yt], "y")


@pytest.mark.parametrize("rows,inputs,outputs", SIZES)
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("turned,pad,act,dw32", [(False, 0, "none", True), (True, 0, "relu", False), (False, 5, "gelu", False),
                                                  (True, 8, "silu", True)])
def test_linear_grad(P, rows, inputs, outputs, kind, turned, pad, act, dw32):
    print(f"[linear_grad] {rows} x {inputs} -> {outputs} {kind} turned {turned} pad {pad} {act}", flush=True)
    s = _case(rows, inputs, outputs, kind, turned, pad, 2)
    t, g = TYPES[kind], s["g"]
    dy = _in_nan(_rand(g, rows, outputs).to(t), pad)
    z = _in_nan(_rand(g, rows, outputs).mul(2).to(t), pad) if act != "none" else None
    dx, dw, dbias = P.linear_grad(s["x"], s["w"], dy, z, act, dw_type=torch.float32 if dw32 else None)
    assert dx.dtype == t and dw.dtype == (torch.float32 if dw32 else t) and dbias.dtype == torch.float32
    x, w, d = s["x"].double(), s["w"].double(), dy.double()
    if z is None:
        dz, err = d, torch.zeros_like(d)
    else:
        zz = z.double().requires_grad_()
        dz = d * torch.autograd.grad(ACTS[act](zz).sum(), zz)[0]
        err = 12 * U * (1 + zz.detach().abs()) * d.abs()
        _near(dbias, dz.sum(0), err.sum(0) + (rows + 8) * U * dz.abs().sum(0), "dbias")
        err = err + (HALF[t] if t != torch.float32 else 0) * dz.abs() + TINY[t]
    ex = err @ w.abs().t() + 2 * (outputs + 8) * U * (dz.abs() @ w.abs().t())
    ew = x.abs().t() @ err + 2 * (rows + 8) * U * (x.abs().t() @ dz.abs())
    xx, ww = dz @ w.t(), x.t() @ dz
    _near(dx, xx, ex + HALF[t] * xx.abs() + TINY[t], "dx")
    _near(dw, ww, ew + HALF[dw.dtype] * ww.abs() + TINY[dw.dtype], "dw")


def test_grad_against_differences(P):
    """The loss sum(y c) moved along a direction of each input, in 64 bits: step 1e-4, so off by about 1e-8 of the third
    derivative, far below the gradient's own fp32 error of 2 (K + 8) u sums, K = 96."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, b, c = _rand(g, 37, 96), _rand(g, 96, 41) / 10, _rand(g, 41), _rand(g, 37, 41)
    _, z = P.linear(x, w, b, act="gelu", with_z=True)
    grads = P.linear_grad(x, w, c, z, "gelu")
    loss = lambda x, w, b: (ACTS["gelu"](x @ w + b) * c.double()).sum()  # noqa: E731
    for i, t in enumerate((x, w, b)):
        way = torch.randn(t.shape, device="cuda", generator=g).double()
        at = [v.double() for v in (x, w, b)]
        move = lambda h: loss(*[v + h * way if k == i else v for k, v in enumerate(at)])  # noqa: E731
        slope = (move(1e-4) - move(-1e-4)) / 2e-4
        got = (grads[i].double() * way).sum()
        most = (grads[i].double().abs() * way.abs()).sum()
        assert abs(got - slope) <= (2 * 104 * U * 64 + 1e-7) * most, (i, got.item(), slope.item())


def test_empty_and_single_outputs(P):
    x, w = torch.empty(0, 16, device="cuda"), torch.ones(16, 5, device="cuda")
    y, z = P.linear(x, w, with_z=True)
    assert y.shape == z.shape == (0, 5)
    dx, dw, dbias = P.linear_grad(x, w, y)
    assert dx.shape == (0, 16) and not dw.any() and not dbias.any() and dw.shape == (16, 5)
    x = torch.ones(3, 2, 16, device="cuda")
    y, z = P.linear(x, w)
    assert z is None and y.shape == (3, 2, 5) and bool((y == 16).all())
    for flags in ((True, False, False), (False, True, False), (False, False, True)):
        got = P.linear_grad(x, w, y, with_dx=flags[0], with_dw=flags[1], with_dbias=flags[2])
        assert tuple(t is not None for t in got) == flags
    assert bool((got[2] == 96).all())


def test_residual_in_place_and_one_row_for_all(P):
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = _rand(g, 70, 40), _rand(g, 40, 90)
    r = _rand(g, 70, 90)
    want, _ = P.linear(x, w, None, r, "silu")
    y, _ = P.linear(x, w, None, r, "silu", y=r)
    assert y is r and torch.equal(r, want)
    one = x[:1].expand(70, 40)
    assert torch.equal(P.linear(one, w)[0], P.linear(one.contiguous(), w)[0])


def test_rows_do_not_mix(P):
    """A NaN or an infinity of one row stays in that row's outputs, one of the weights in its column."""
    g = torch.Generator(device="cuda").manual_seed(4)
    for kind in ("fp32", "bf16", "fp16"):
        x, w = _rand(g, 131, 77).to(TYPES[kind]), _rand(g, 77, 141).to(TYPES[kind])
        clean, _ = P.linear(x, w)
        x[5, 76], x[130, 0], w[76, 140] = float("nan"), float("inf"), float("nan")
        y, _ = P.linear(x, w)
        keep = torch.ones(131, dtype=torch.bool, device="cuda")
        keep[5] = keep[130] = False
        assert torch.equal(y[keep][:, :140], clean[keep][:, :140])
        assert bool(y[5].isnan().all()) and bool(y[:, 140].isnan().all()) and not bool(y[130, :140].isfinite().any())


@pytest.mark.parametrize("kind", ["fp32", "bf16", "e4m3"])
def test_strided_after_contiguous(P, kind):
    """The same sizes with other strides take another workspace (2048 x 1024 x 1024 products are copied into whole pieces first)."""
    s = _case(2048, 1024, 1024, kind, False, 0, 8)
    more = dict(alpha=s["alpha"], scale=s["scale"]) if kind == "e4m3" else {}
    plain = [s[k].contiguous() for k in ("x", "w")]
    want = P.linear(*plain, s["bias"], **more)[0]
    for x, w in ((_in_nan(plain[0], 3), plain[1]), (plain[0], _in_nan(plain[1], 5)), (_in_nan(plain[0], 1), _in_nan(plain[1], 2)), plain):
        got = P.linear(x, w, s["bias"], **more)[0]
        # the same products in another order at most: 2 (K + 8) u of sums of about 0.8 K / sqrt(K) terms, and the rounding of the type
        assert bool(((got - want).abs() <= 4 * 1032 * U * 64 + 2 * HALF[got.dtype] * want.abs()).all())
    if kind != "e4m3":
        dy = plain[0][:, :].clone()
        want = P.linear_grad(*plain, dy)
        for x, w, d in ((_in_nan(plain[0], 3), plain[1], dy), (plain[0], _in_nan(plain[1], 5), dy), (plain[0], plain[1], _in_nan(dy, 1))):
            for p, q in zip(P.linear_grad(x, w, d), want):
                assert bool(((p - q).abs() <= 4 * 2056 * U * q.abs().max() + 2 * HALF[p.dtype] * q.abs()).all())


def test_wide_strides(P):
    """Rows 2^21 and 2^23 values apart: past what 32-bit offsets of a tile take.  The same products in the same or another order: 2 (K + 8) u
    of sums of |x w|."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for ld in (1 << 21, 1 << 23):
        x, w, dy = (torch.empty(r, ld, dtype=torch.bfloat16, device="cuda")[:, :c] for r, c in ((70, 96), (96, 80), (70, 80)))
        for t in (x, w, dy):
            t.copy_(_rand(g, *t.shape))
        near = [t.contiguous() for t in (x, w, dy)]
        each = near[0].double().abs() @ near[1].double().abs()
        y, want = P.linear(x, w)[0].double(), near[0].double() @ near[1].double()
        _near(y, want, 208 * U * each + HALF[torch.bfloat16] * want.abs(), "y")
        assert torch.equal(P.linear(x[:2], w)[0], P.linear(near[0][:2], near[1])[0])
        for a, b in zip(P.linear_grad(x, w, dy), P.linear_grad(*near)):
            assert bool(((a.float() - b.float()).abs() <= 2 * HALF[a.dtype] * b.float().abs() + 416 * U * 96).all())


def test_activation_limits(P):
    z = torch.tensor([[-float("inf"), -200.0, -0.0, 0.0, 200.0, float("inf"), float("nan")]], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    for act, values, slopes in (("relu", [0, 0, 0, 0, 200, float("inf")], [0, 0, 0, 0, 1, 1]),
                                ("gelu", [None, 0, 0, 0, 200, float("inf")], [0, 0, .5, .5, 1, 1]),
                                ("silu", [None, 0, 0, 0, 200, float("inf")], [0, 0, .5, .5, 1, 1])):
        y, _ = P.linear(one, z, act=act)
        dx, dw, dbias = P.linear_grad(one, torch.zeros_like(z), torch.ones_like(z), z, act)
        for i in range(6):
            assert values[i] is None or y[0, i].item() == values[i], (act, i, y)
            assert dbias[i].item() == slopes[i], (act, i, dbias)
        assert y[0, 6].isnan() and dbias[6].isnan()


@pytest.mark.parametrize("rows", [3, 200])
def test_captured_on_streams_and_the_same_bits(P, rows):
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w, b = _rand(g, rows, 2000).bfloat16(), _rand(g, 2000, 300).bfloat16(), _rand(g, 300)
    dy, z = _rand(g, rows, 300).bfloat16(), _rand(g, rows, 300).bfloat16()
    want = [P.linear(x, w, b, act="gelu")[0], *P.linear_grad(x, w, dy, z, "gelu")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = [P.linear(x, w, b, act="gelu", stream=side)[0], *P.linear_grad(x, w, dy, z, "gelu", stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [P.linear(x, w, b, act="gelu")[0], *P.linear_grad(x, w, dy, z, "gelu")]
    for step in range(3):
        x.copy_(_rand(g, rows, 2000))
        want = [P.linear(x, w, b, act="gelu")[0], *P.linear_grad(x, w, dy, z, "gelu")]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, out)), step


def test_codes_of_the_row_norm(P):
    """rms_norm's codes through a ternary map, as the decoder's Eq. 3: int8 sums of these lengths are exact."""
    g = torch.Generator(device="cuda").manual_seed(7)
    x = _rand(g, 50, 128)
    _, _, codes, alpha = P.rms_norm(x, with_y=False, code_type=torch.int8)
    w = torch.randint(-1, 2, (128, 512), device="cuda", generator=g, dtype=torch.int8)
    scale = torch.full((512,), 0.03, device="cuda")
    y, _ = P.linear(codes, w, None, None, "relu", alpha=alpha, scale=scale)
    want = (codes.double() @ w.double()) * (alpha.double() / 127)[:, None] * scale.double()
    _near(y, want.clamp(min=0), 6 * U * want.abs(), "y")


def test_refusals(P):
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 6, device="cuda")
    i8x, i8w = x.to(torch.int8), w.to(torch.int8)
    one = torch.ones(4, device="cuda")
    for call in (lambda: P.linear(x, w.t()), lambda: P.linear(x, w.double()), lambda: P.linear(x.double(), w.double()),
                 lambda: P.linear(x, w, act="tanh"), lambda: P.linear(x, w, alpha=one), lambda: P.linear(i8x, i8w),
                 lambda: P.linear(x, w, y_type=torch.bfloat16), lambda: P.linear(x, w, torch.zeros(5, device="cuda")),
                 lambda: P.linear(x.cpu(), w), lambda: P.linear(x, w.cpu()), lambda: P.linear(x, w, res=x),
                 lambda: P.linear(x, torch.zeros(8, 12, device="cuda")[:, ::2]),
                 lambda: P.linear(i8x, i8w, alpha=one[:3], scale=torch.ones(6, device="cuda")),
                 lambda: P.linear_grad(x, w, x), lambda: P.linear_grad(x, w, torch.zeros(4, 6, device="cuda"), act="relu"),
                 lambda: P.linear_grad(x, w, torch.zeros(4, 6, device="cuda"), torch.zeros(4, 6, device="cuda")),
                 lambda: P.linear_grad(x, w, torch.zeros(4, 6, device="cuda"), dw_type=torch.float16),
                 lambda: P.linear_grad(x, w, torch.zeros(4, 6, device="cuda"), with_dx=False, with_dw=False, with_dbias=False)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(P.AecctError):    # y overlaps x
        P.linear(x, torch.zeros(8, 8, device="cuda"), y=x)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
def test_activation_tails(P, act, kind):
    """Activations and slopes relative to their own size, where they are small too.  z is exact: one product with 1.

    Conditions: z Phi(z) moves by a share of at most (z^2 + 2) a where z moves by a share a, z / (1 + e^-z) by (|z| + 1) a.  fp32 takes erfc
    at z / sqrt(2) (off by 2 u for the factor and its product, which moves erfc's share by z^2 + 1 times that), e^x within 2 u of
    its value, and a few products: 4 (z^2 + 8) u.  16-bit types: the same, and 2^-14 for the fitted tail.  Then the type's
    half step.  Slopes are sums Phi + z phi, or products p (1 + z q), whose parts are off by such shares."""
    t = TYPES[kind]
    z = torch.linspace(-12.5, 12.5, 40001, device="cuda").to(t).unique()
    one = torch.ones(1, 1, device="cuda", dtype=t)
    y, got = P.linear(z[:, None], one, act=act, with_z=True)
    assert torch.equal(got[:, 0], z)
    zz = z.double()
    fit = 0 if kind == "fp32" or act == "silu" else 2.0 ** -14
    share = 4 * (zz * zz + 8) * U + fit
    p = 0.5 * torch.erfc(-zz * 0.5 ** 0.5) if act == "gelu" else torch.sigmoid(zz)     # (ndtr on the GPU is 0 or 2^-54 off in the tail)
    want = zz * p
    _near(y[:, 0], want, (share + HALF[t]) * want.abs() + TINY[t], "y")
    across = torch.ones(1, z.numel(), device="cuda", dtype=t)
    _, _, dbias = P.linear_grad(one, across, across, z[None], act, with_dx=False, with_dw=False)      # of one row: the slopes, in fp32
    inner = zz * torch.exp(-0.5 * zz * zz) / (2 * torch.pi) ** 0.5 if act == "gelu" else zz * p * torch.sigmoid(-zz)
    _near(dbias, p + inner, share * (p + inner.abs()) + TINY[torch.float32], "slope")


def test_silu_far_below(P):
    """e^z is a normal number to z = -87.3; 4 (|z| + 8) u as above, the slopes' two parts each."""
    z = torch.linspace(-87, -80, 50, device="cuda")
    y, _ = P.linear(z[:, None], torch.ones(1, 1, device="cuda"), act="silu")
    zz = z.double()
    _near(y[:, 0], zz * torch.sigmoid(zz), 4 * (zz.abs() + 8) * U * (zz * torch.sigmoid(zz)).abs(), "y")
    one = torch.ones(1, 50, device="cuda")
    _, _, dbias = P.linear_grad(one[:, :1], one, one, z[None], "silu", with_dx=False, with_dw=False)
    p = torch.sigmoid(zz)
    _near(dbias, p * (1 + zz * torch.sigmoid(-zz)), 4 * (zz.abs() + 8) * U * p * (1 + zz.abs()), "slope")
