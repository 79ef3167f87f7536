"""Cross attention and its gradient against their formulas in 64 bits.

Keys and values past a sequence's length hold NaN, and so does what lies around every input.

Tolerances, with u = 2^-24 and w = half a step of the stored type:
  scores  sums of d products, each addition off by at most 2 u of its result, times scale log2(e): e = 2 (d + 12) u scale sum|q k|
  p       2^x of an argument that is off by e and by 4 u (|s| + |m|) for its roundings (natural units, m the row's maximum), and 4 u
          of its own: r = max over the row's keys of e + 4 u (|s| + |m| + 1)
  lse     r, and keys + 8 additions of the sum: r + (keys + 8) u + 4 u |lse|
  o       sum p |v| (2 r + 2 (keys + 12) u + w for p's own rounding), w |o|; in fp16 weights below 2^-24 of 2^10 lose at most 2^-35 each
  D, dp   2 (d + 12) u sum|dout o|, 2 (d + 12) u sum|dout v|
  ds      p (their errors + 4 u (|dp| + |D|)) + (r' + w) |ds|, r' as r but for the given lse in place of m, over all the row's keys
  dq      scale (errors of ds times |k| + 2 (keys + 12) u sum|ds k|) + w |dq|;  dk alike over the rows;  dv alike with p and dout
          (in fp16 ds and p are held to 2^-24 of a power of two at least a quarter of the largest: 2^-38 of the largest each)
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -120, torch.bfloat16: 2.0 ** -120, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _near(got, want, bound, what):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    bad &= ~(got.eq(want))      # infinities
    assert not bad.any(), (what, int(bad.sum()), got.numel(), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(),
                           torch.as_tensor(bound, device=got.device).expand_as(got)[bad][:4].tolist())


def _tensor(g, b, n, h, d, type, layout, scale=1.0):
    """[b][n][h][d] in NaN surroundings: "plain" contiguous, "wide" part of a wider row (as of one projection to q, k and v), "heads"
    with the heads outside the rows."""
    t = torch.randn(b, n, h, d, device="cuda", generator=g).mul(scale).to(type)
    nan = lambda *s: torch.full(s, float("nan"), dtype=type, device="cuda")  # noqa: E731
    if layout == "wide":
        view = nan(b, n + 1, h + 1, d + 3)[:, 1:, 1:, 1: d + 1]
    elif layout == "heads":
        view = nan(b, h, n + 2, d).transpose(1, 2)[:, 1: n + 1]
    else:
        view = nan(b * n * h * d + 8)[5: 5 + b * n * h * d].view(b, n, h, d)
    view.copy_(t)
    return view


def _mask(g, n, m, kind):
    if kind == "none":
        return None
    if kind == "band":
        keep = (torch.arange(m, device="cuda")[None] - (torch.arange(n, device="cuda") * m // n)[:, None]).abs() <= max(1, m // 8)
    else:
        keep = torch.rand(n, m, device="cuda", generator=g) < 0.2
    if kind == "holes" and n > 1:
        keep[::3] = False
        keep[:, : m // 2] &= torch.rand(1, m // 2, device="cuda", generator=g) < 0.5
    whole = torch.ones(n, m + 7, dtype=torch.bool, device="cuda")
    whole[:, 3: 3 + m] = keep
    return whole[:, 3: 3 + m]


def _case(b, n, m, h, kv, d, kind, layout, lengths, mask, seed=1, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[kind]
    s = {"q": _tensor(g, b, n, h, d, t, layout, scale), "k": _tensor(g, b, m, kv, d, t, layout), "v": _tensor(g, b, m, kv, d, t, layout),
         "dout": _tensor(g, b, n, h, d, t, layout), "lengths": None, "mask": _mask(g, n, m, mask)}
    if lengths:
        at = [(m, 0, 1, m // 2, m - 1, m + 5, -3)[i % 7] for i in range(b)]
        s["lengths"] = torch.tensor(at, dtype=torch.int32, device="cuda")
        for i, l in enumerate(at):
            s["k"][i, max(0, min(l, m)):] = float("nan")
            s["v"][i, max(0, min(l, m)):] = float("nan")
    return s


def _formula(s, scale):
    """In 64 bits: by head, scores, weights, and what counts."""
    group = s["q"].shape[2] // s["k"].shape[2]
    m = s["k"].shape[1]
    q = s["q"].double().transpose(1, 2)
    live = torch.ones(q.shape[0], m, dtype=torch.bool, device="cuda") if s["lengths"] is None else \
        torch.arange(m, device="cuda")[None] < s["lengths"].clamp(0, m)[:, None]
    clean = lambda t: torch.where(live[:, None, :, None], t.double().transpose(1, 2), 0.0).repeat_interleave(group, 1)  # noqa: E731
    k, v = clean(s["k"]), clean(s["v"])
    counts = live[:, None, None].expand(-1, -1, q.shape[2], -1)
    if s["mask"] is not None:
        counts = counts & s["mask"]
    score = (q @ k.transpose(2, 3).contiguous()) * scale
    size = (q.abs() @ k.abs().transpose(2, 3).contiguous()) * scale
    score = score.masked_fill(~counts, -math.inf)
    lse = torch.logsumexp(score, -1) if m else torch.full(score.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    p = torch.where(counts, torch.exp(score - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    top = torch.where(lse == -math.inf, 0.0, score.amax(-1) if m else lse)
    s0 = torch.where(counts, score, 0.0)
    r = (2 * (q.shape[3] + 12) * U * size + 4 * U * (s0.abs() + top.abs()[..., None] + 1)) * counts
    r = r.amax(-1) if m else torch.zeros_like(lse)
    return q, k, v, p, lse, r


SHAPES = [  # batch, queries, keys, heads, kv_heads, d
    (1, 1, 1, 1, 1, 1), (2, 1, 33, 4, 2, 16), (3, 5, 64, 2, 2, 17), (7, 33, 31, 6, 2, 32), (2, 65, 129, 4, 1, 33), (1, 128, 100, 2, 2, 64),
    (2, 3, 1100, 8, 2, 64), (7, 130, 200, 4, 2, 128), (3, 40, 257, 2, 1, 100), (2, 70, 90, 2, 2, 256), (1, 1, 2100, 4, 1, 129),
    (2, 45, 150, 4, 2, 192), (1, 150, 330, 2, 1, 161), (2, 2, 700, 2, 2, 193),
    (2, 500, 700, 4, 2, 177), (3, 2, 9000, 2, 1, 99),       # copied into whole pieces first
    (2, 300, 65, 3, 3, 8)]


@pytest.mark.parametrize("b,n,m,h,kv,d", SHAPES)
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout,lengths,mask", [("plain", False, "none"), ("wide", True, "none"), ("plain", True, "band"),
                                                  ("heads", False, "some"), ("wide", True, "holes")])
def test_attention_and_gradient(P, b, n, m, h, kv, d, kind, layout, lengths, mask):
    print(f"[attention] {b} x {n} on {m}, {h}/{kv} x {d} {kind} {layout} lengths {lengths} mask {mask}", flush=True)
    s = _case(b, n, m, h, kv, d, kind, layout, lengths, mask)
    t, scale = TYPES[kind], d ** -0.5
    w = HALF[t]
    pw = 0 if t == torch.float32 else w      # p and ds are rounded
    out = torch.full((b, n, h, d + 2), 77.0, dtype=t, device="cuda")
    o, lse = P.cross_attention(s["q"], s["k"], s["v"], s["lengths"], s["mask"], o=out[..., :d], with_lse=True)
    q, k, v, p, want_lse, r = _formula(s, scale)
    _near(lse, want_lse, r + (m + 8) * U + 4 * U * torch.where(want_lse == -math.inf, 0.0, want_lse.abs()), "lse")
    want = p @ v
    each = p @ v.abs()
    lost = m * 2.0 ** -35 * v.abs().amax() if t == torch.float16 else 0
    _near(o.transpose(1, 2), want, each * (2 * r[..., None] + 2 * (m + 12) * U + pw) + w * want.abs() + lost + TINY[t], "o")
    assert bool((out[..., d:] == 77).all())

    wide = [torch.full((b, x, y, d + 1), 77.0, dtype=t, device="cuda") for x, y in ((n, h), (m, kv), (m, kv))]
    got = P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"], s["lengths"], s["mask"], dq=wide[0][..., :d],
                                 dk=wide[1][..., :d], dv=wide[2][..., :d])
    assert all(bool((x[..., d:] == 77).all()) for x in wide)
    od, dout = o.double().transpose(1, 2), s["dout"].double().transpose(1, 2)
    # the weights that the given lse stands for
    given = torch.where(lse == -math.inf, math.inf, lse.double())[..., None]
    pg = torch.where(p > 0, p * torch.exp(torch.where(lse == -math.inf, 0.0, want_lse - lse.double()))[..., None], 0.0)
    rr = r + 4 * U * torch.where(given[..., 0] == math.inf, 0.0, given[..., 0].abs())
    rr = rr[..., None]
    dp, dsum = dout @ v.transpose(2, 3).contiguous(), (dout * od).sum(-1, keepdim=True)
    edp = 2 * (d + 12) * U * (dout.abs() @ v.abs().transpose(2, 3).contiguous())
    edd = 2 * (d + 12) * U * (dout * od).abs().sum(-1, keepdim=True)
    ds = pg * (dp - dsum)
    eds = pg * (edp + edd + 4 * U * (dp.abs() + dsum.abs())) + (rr + pw) * ds.abs()
    ep = (rr + pw) * pg
    if t == torch.float16:
        eds = eds + 2.0 ** -38 * ds.abs().amax()
        ep = ep + 2.0 ** -38
        eds, ep = eds * (p > 0), ep * (p > 0)
    fold = lambda x: x.view(b, kv, h // kv, m, d).sum(2)  # noqa: E731
    turn = lambda x: x.transpose(2, 3).contiguous()  # noqa: E731
    dq = scale * (ds @ k)
    _near(got[0].transpose(1, 2), dq, scale * (eds @ k.abs() + 2 * (m + 12) * U * (ds.abs() @ k.abs())) + w * dq.abs() + TINY[t], "dq")
    rows = n * h // kv
    dk = scale * fold(turn(ds) @ q)
    ek = scale * fold(turn(eds) @ q.abs() + 2 * (rows + 12) * U * (turn(ds.abs()) @ q.abs()))
    _near(got[1].transpose(1, 2), dk, ek + w * dk.abs() + TINY[t], "dk")
    dv = fold(turn(pg) @ dout)
    ev = fold(turn(ep) @ dout.abs() + 2 * (rows + 12) * U * (turn(pg) @ dout.abs()))
    _near(got[2].transpose(1, 2), dv, ev + w * dv.abs() + TINY[t], "dv")


def test_gradient_against_differences(P):
    """sum(o c) moved along a direction of each input, in 64 bits with steps of 1e-4: off by about 1e-8; the kernels' own error is that
    of fp32 sums of at most 64 products, three deep: 400 u."""
    s = _case(2, 21, 30, 4, 2, 24, "fp32", "plain", False, "some", 3)
    o, lse = P.cross_attention(s["q"], s["k"], s["v"], None, s["mask"], with_lse=True)
    grads = P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"], None, s["mask"])
    at = [s[x].double() for x in "qkv"]

    def loss(q, k, v):
        q, k, v = q.transpose(1, 2), k.transpose(1, 2).repeat_interleave(2, 1), v.transpose(1, 2).repeat_interleave(2, 1)
        score = (q @ k.transpose(2, 3).contiguous() * 24 ** -0.5).masked_fill(~s["mask"], -math.inf)
        p = torch.where(s["mask"].any(-1)[:, None], torch.softmax(score, -1).nan_to_num(0.0), 0.0)
        return ((p @ v).transpose(1, 2) * s["dout"].double()).sum()
    g = torch.Generator(device="cuda").manual_seed(9)
    for i in range(3):
        way = torch.randn(at[i].shape, device="cuda", generator=g, dtype=torch.float64)
        move = lambda x: loss(*[a + x * way if j == i else a for j, a in enumerate(at)])  # noqa: E731
        slope = (move(1e-4) - move(-1e-4)) / 2e-4
        most = (grads[i].double().abs() * way.abs()).sum()
        assert abs((grads[i].double() * way).sum() - slope) <= (400 * U + 1e-6) * most, i


@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
def test_far_scores(P, kind):
    """Scores of +-1000 and more: one key takes all the weight; o is its value, to the last bit (weights of the others are 0)."""
    t = TYPES[kind]
    q = torch.full((1, 40, 2, 16), 16.0, dtype=t, device="cuda")
    k = torch.full((1, 100, 2, 16), -16.0, dtype=t, device="cuda")
    k[0, 77] = 16.0
    v = torch.randn(1, 100, 2, 16, device="cuda").to(t)
    o, lse = P.cross_attention(q, k, v, with_lse=True)
    assert torch.equal(o, v[:, 77:78].expand_as(o)) and bool(((lse - 1024).abs() <= 1024 * 4 * U).all())
    dout = torch.randn(1, 40, 2, 16, device="cuda").to(t)
    dq, dk, dv = P.cross_attention_grad(q, k, v, o, lse, dout)
    assert not dv[:, :77].any() and not dv[:, 78:].any() and bool(dq.isfinite().all()) and bool(dk.isfinite().all())
    total = dout.double().sum(1)
    # p is 2^x of an argument that two values near 1477 leave: off by 6 2^-13 at most; in fp32 40 additions besides
    assert bool(((dv[:, 77].double() - total).abs() <= (2.0 ** -10 + HALF[t]) * dout.double().abs().sum(1)).all())


def test_small_and_large_gradients_in_fp16(P):
    """dout of 2^-12 and of 2^9: gradients are linear in dout, and fp16's range is not to show in their relative size: results scaled
    by powers of two differ only where the outputs leave fp16's normal range, so by 2^-25 at most, beside the outputs' own rounding of
    2^-11 and D's, whose products are exact under the scaling."""
    s = _case(2, 50, 300, 4, 2, 64, "fp16", "plain", False, "none", 4)
    o, lse = P.cross_attention(s["q"], s["k"], s["v"], with_lse=True)
    base = P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"])
    for power in (-8, 8):
        dout = (s["dout"].float() * 2.0 ** power).half()
        if power < 0:      # what is exact in both
            dout = torch.where((dout.float() * 2.0 ** -power).half() == s["dout"], dout, torch.zeros_like(dout))
            same = (dout.float() * 2.0 ** -power).half()
            base2 = P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, same)
        else:
            base2 = base
        got = P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, dout)
        for x, y in zip(got, base2):
            want = y.double() * 2.0 ** power
            assert bool(((x.double() - want).abs() <= 2 * 2.0 ** -11 * want.abs() + 2.0 ** -24 + 2.0 ** (power - 24)).all()), power


def test_no_keys_and_no_queries(P):
    q, none = torch.randn(2, 3, 4, 8, device="cuda"), torch.empty(2, 0, 2, 8, device="cuda")
    o, lse = P.cross_attention(q, none, none, with_lse=True)
    assert not o.any() and bool((lse == -math.inf).all())
    dq, dk, dv = P.cross_attention_grad(q, none, none, o, lse, q)
    assert not dq.any() and dk.shape == none.shape
    k = torch.randn(2, 5, 2, 8, device="cuda")
    empty = torch.empty(2, 0, 4, 8, device="cuda")
    o, lse = P.cross_attention(empty, k, k, with_lse=True)
    assert o.shape == empty.shape
    dq, dk, dv = P.cross_attention_grad(empty, k, k, o, lse, empty)
    assert dq.shape == empty.shape and not dk.any() and not dv.any()
    batch0 = torch.empty(0, 3, 4, 8, device="cuda")
    assert P.cross_attention(batch0, batch0[:, :, :2], batch0[:, :, :2])[0].shape == batch0.shape
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    o, lse = P.cross_attention(q, k, k, zero, with_lse=True)
    assert not o.any()
    dq, dk, dv = P.cross_attention_grad(q, k, k, o, lse, q, zero)
    assert not dq.any() and not dk.any() and not dv.any()


def test_nan_stays_in_its_row(P):
    q, k, v = (torch.randn(1, n, 2, 32, device="cuda") for n in (70, 90, 90))
    clean, _ = P.cross_attention(q, k, v)
    q[0, 11, 1, 5] = float("nan")
    o, lse = P.cross_attention(q, k, v, with_lse=True)
    assert bool(o[0, 11, 1].isnan().all()) and bool(lse[0, 1, 11].isnan())
    keep = torch.ones(70, 2, dtype=torch.bool, device="cuda")
    keep[11, 1] = False
    assert torch.equal(o[0][keep], clean[0][keep])


def test_one_projection_and_broadcast_keys(P):
    """q of one tensor, k and v side by side in another; one sequence's keys for all queries' batches (a stride of 0)."""
    g = torch.Generator(device="cuda").manual_seed(8)
    q = torch.randn(3, 9, 4, 16, device="cuda", generator=g)
    kv = torch.randn(3, 12, 2, 2, 16, device="cuda", generator=g)
    k, v = kv[:, :, 0], kv[:, :, 1]
    o, lse = P.cross_attention(q, k, v, with_lse=True)
    assert torch.equal(o, P.cross_attention(q, k.contiguous(), v.contiguous())[0])
    dkv = torch.zeros_like(kv)
    dq, dk, dv = P.cross_attention_grad(q, k, v, o, lse, q, dk=dkv[:, :, 0], dv=dkv[:, :, 1])
    for a, b in zip((dq, dk, dv), P.cross_attention_grad(q, k.contiguous(), v.contiguous(), o, lse, q)):
        assert torch.equal(a, b)
    one = k[:1].expand(3, 12, 2, 16)
    assert torch.equal(P.cross_attention(q, one, one)[0], P.cross_attention(q, one.contiguous(), one.contiguous())[0])
    for flags in ((True, False), (False, True)):
        a = P.cross_attention_grad(q, k, v, o, lse, q, with_dq=flags[0], with_dkv=flags[1])
        assert (a[0] is not None, a[1] is not None, a[2] is not None) == (flags[0], flags[1], flags[1])


@pytest.mark.parametrize("n,m", [(1, 3000), (200, 300)])
def test_captured_on_streams_and_the_same_bits(P, n, m):
    s = _case(2, n, m, 8, 2, 64, "bf16", "plain", False, "band", 5)
    lengths = torch.tensor([m, m // 3], dtype=torch.int32, device="cuda")

    def both(stream=None):
        o, lse = P.cross_attention(s["q"], s["k"], s["v"], lengths, s["mask"], with_lse=True, stream=stream)
        return [o, lse, *P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"], lengths, s["mask"], stream=stream)]
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for step in range(3):
        s["q"].normal_()
        lengths.copy_(torch.tensor([m - step, m // 2], device="cuda"))
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), step


def test_wide_strides(P):
    """Rows 2^21 values apart, which tiles take through registers: what contiguous rows give, to the last bit but for splits, whose number
    goes by sizes alone."""
    n, m, d = 40, 90, 32
    far = [torch.empty(1, r, 1, 1 << 21, dtype=torch.bfloat16, device="cuda")[..., :d] for r in (n, m, m, n)]
    for t in far:
        t.normal_()
    near = [t.contiguous() for t in far]
    o, lse = P.cross_attention(*far[:3], with_lse=True)
    want, want_lse = P.cross_attention(*near[:3], with_lse=True)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    for a, b in zip(P.cross_attention_grad(*far[:3], o, lse, far[3]), P.cross_attention_grad(*near[:3], o, lse, near[3])):
        assert torch.equal(a, b)


def test_offsets_past_32_bits(P):
    """A cache of more than 2^32 bytes, its last sequence read: 5 sequences 2^30 bytes apart."""
    cache = torch.empty(5, 1 << 23, 1, 64, dtype=torch.bfloat16, device="cuda")
    part = cache[:, :700]
    part.normal_()
    q = torch.randn(5, 2, 4, 64, device="cuda").bfloat16()
    o, _ = P.cross_attention(q, part, part)
    assert torch.equal(o, P.cross_attention(q, part.contiguous(), part.contiguous())[0])


def test_refusals(P):
    q, k = torch.zeros(2, 3, 4, 8, device="cuda"), torch.zeros(2, 5, 2, 8, device="cuda")
    lse = torch.zeros(2, 4, 3, device="cuda")
    ok = torch.ones(3, 5, dtype=torch.bool, device="cuda")
    for call in (lambda: P.cross_attention(q, k[:1], k[:1]), lambda: P.cross_attention(q, k, k[:, :4]), lambda: P.cross_attention(q[0], k, k),
                 lambda: P.cross_attention(q, torch.zeros(2, 5, 3, 8, device="cuda"), torch.zeros(2, 5, 3, 8, device="cuda")),
                 lambda: P.cross_attention(q, k.bfloat16(), k.bfloat16()), lambda: P.cross_attention(q.double(), k.double(), k.double()),
                 lambda: P.cross_attention(q, k, k, torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: P.cross_attention(q, k, k, torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: P.cross_attention(q, k, k, None, ok.float()), lambda: P.cross_attention(q, k, k, None, ok.t()),
                 lambda: P.cross_attention(q, k, k, None, ok.cpu()), lambda: P.cross_attention(q.cpu(), k, k),
                 lambda: P.cross_attention(q, k, k, o=q[:1]), lambda: P.cross_attention(q, k, k, lse=lse[:1]),
                 lambda: P.cross_attention(torch.zeros(2, 3, 8, 4, device="cuda").transpose(2, 3), k, k),
                 lambda: P.cross_attention_grad(q, k, k, q, lse[:1], q), lambda: P.cross_attention_grad(q, k, k, q, lse, k),
                 lambda: P.cross_attention_grad(q, k, k, q, lse, q, with_dq=False, with_dkv=False)):
        with pytest.raises(ValueError):
            call()
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(P.AecctError):
            P.cross_attention(q, k, k, scale=scale)
    with pytest.raises(P.AecctError):
        P.cross_attention(q, k, k, o=q)
    wide = torch.zeros(1, 1, 1, 257, device="cuda")
    with pytest.raises(P.AecctError) as e:
        P.cross_attention(wide, wide, wide)
    assert e.value.status == P.ERR_UNSUPPORTED


@pytest.mark.parametrize("d,few", [(16, False), (16, True), (64, False), (64, True), (100, False), (250, False)])
def test_weights_of_the_gradient_in_fp32(P, d, few):
    """Single weights, from scores that are exact in fp32 (small whole numbers, a scale of 1) up to 48 and more below and above: with dout of one
    1 and o = 0, dv of a key is its p, and with v of one key only dq is p k.  p = e^t, t = s - lse the distance from the lse that is
    given: t is rounded once, its product with log2(e) is off by 2 u more, e^x by 2 u of its value, and a product or a sum with zeros
    by u: (3 |t| + 6) u."""
    b, m = 20, 70
    g = torch.Generator(device="cuda").manual_seed(31)
    k = torch.randint(-3, 4, (b, m, 1, d), device="cuda", generator=g).float()
    q = torch.randint(-2, 3, (b, 1, 1, d), device="cuda", generator=g).float()
    q[:, :, :, 8:] = 0
    k[:, 3, :, :8] = 3 * q[:, 0, :, :8].sign()
    mask = None
    if few:
        mask = torch.zeros(1, m, dtype=torch.bool, device="cuda")
        mask[0, [3, 20, 41, 69]] = True
    o, lse = P.cross_attention(q, k, k, None, mask, 1.0, with_lse=True)
    score = (q.double() * k.double()).sum(-1)[..., 0]
    t = score - lse.double()[:, 0]
    p = torch.exp(t) if mask is None else torch.exp(t) * mask
    bound = (3 * t.abs() + 6) * U * p + TINY[torch.float32]
    dout = torch.zeros_like(q)
    dout[..., 0] = 1
    none = torch.zeros_like(q)
    for at in (3, 20, 41):
        v = torch.zeros_like(k)
        v[:, at, 0, 0] = 1
        dq, dk, dv = P.cross_attention_grad(q, k, v, none, lse, dout, None, mask, 1.0)
        _near(dv[:, :, 0, 0], p, bound, "dv")
        assert not dv[..., 1:].any()
        _near(dq[:, 0, 0], p[:, at, None] * k[:, at, 0].double(), bound[:, at, None] * k[:, at, 0].double().abs(), "dq")
        _near(dk[:, at, 0], p[:, at, None] * q[:, 0, 0].double(), bound[:, at, None] * q[:, 0, 0].double().abs(), "dk")
