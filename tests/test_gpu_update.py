"""The norm of many gradients, clipping by it and the Adam update, over lists of tensors, against their formulas in 64 bits.

Tolerances, with u = 2^-24 and w = half a step of the stored type: the norm is summed in fp64 and rounded once, u; a
clipped value has the factor's rounding, the product's and the stored type's, 2 u + w; a moment at most 6 roundings of
its two terms (v: 8, for the square); the update lr m / (sqrt(v) + eps) 20 u of its size with m's terms taken
absolutely; the parameter 3 u of the decay, and u of itself before and after the subtraction.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from workloads import random_qat_params, CONFIGS  # noqa: E402
from workloads.configs import parity_check  # noqa: E402

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}

# (name, counts): one value, odd sizes, around the unit of 4096 values, empty ones, more tensors than a launch takes
LISTS = {
    "one": [1],
    "three": [3, 5, 7],
    "units": [4095, 4096, 4097, 8192, 1, 12289],
    "empty": [0, 17, 0, 0, 4096, 0],
    "many": [1 + (37 * k * k) % 977 for k in range(405)],
    "large": [3_000_001, 2, 9_999_999],
}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _tensors(counts, types, seed, scale=1.0, flat=True):
    """Tensors of the counts, types in turn; flat: views of one buffer a type, back to back from an odd place."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if not flat:
        return [(torch.randn(c, device="cuda", generator=g) * scale).to(types[i % len(types)]) for i, c in enumerate(counts)]
    buf = {t: torch.empty(sum(counts) + 1, device="cuda", dtype=t) for t in set(types)}
    at = {t: 1 for t in buf}
    out = []
    for i, c in enumerate(counts):
        t = types[i % len(types)]
        v = buf[t][at[t]:at[t] + c]
        at[t] += c
        v.copy_(torch.randn(c, device="cuda", generator=g) * scale)
        out.append(v)
    return out


def _norm64(ts):
    return math.sqrt(sum((t.double() ** 2).sum().item() for t in ts))


def _near(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist())


ALL = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("types", [ALL[:1], ALL[1:2], ALL[2:], ALL], ids=["fp32", "bf16", "fp16", "mixed"])
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clip(P, name, types):
    print(f"[clip] {name} {types}", flush=True)
    for flat in (True, False):
        g = _tensors(LISTS[name], types, 1, 0.01, flat)
        want = _norm64(g)
        norm = P.grad_norm(g)
        assert norm.shape == (1,) and abs(norm.item() - want) <= 1.01 * U * want
        assert torch.equal(norm, P.grad_norm(P.TensorList(g)))
        keep = [t.clone() for t in g]
        for most in (0.3 * want, 2 * want, math.inf, 0.0):
            f = 1.0 if most > want else most / want
            out = _tensors(LISTS[name], types[::-1], 2, flat=flat)
            n2 = P.grad_clip(g, most, out=out)
            assert torch.equal(n2, norm)
            for a, b, k in zip(out, g, keep):
                assert torch.equal(b, k)
                x = k.double() * f
                _near(a, x, (2.1 * U + HALF[a.dtype]) * x.abs() + TINY[a.dtype], "out")
        P.grad_clip(g, 0.3 * want)                   # in place
        for b, k in zip(g, keep):
            x = k.double() * 0.3
            _near(b, x, (2.1 * U + HALF[b.dtype]) * x.abs() + TINY[b.dtype], "in place")


def test_norm_out_of_range_values(P):
    """Squares far outside fp32's range, infinities and NaN; a norm that is not finite scales nothing."""
    for scale in (1e30, 1e-30, 1e-44):
        g = [torch.full((5000,), scale, device="cuda"), torch.zeros(3, device="cuda")]
        want = _norm64(g)
        norm = P.grad_clip(g, want / 4)
        assert abs(norm.item() - want) <= U * want + 2.0 ** -149
        _near(g[0], torch.full((5000,), g[0][0].double().item(), device="cuda", dtype=torch.float64), 0, "all alike")
        assert abs(g[0][0].item() - scale / 4) <= 3 * U * scale + 2.0 ** -148
    for bad in (math.inf, -math.inf, math.nan):
        g = [torch.ones(5000, device="cuda"), torch.tensor([1.0, bad], device="cuda")]
        assert not math.isfinite(P.grad_norm(g).item())
        norm = P.grad_clip(g, 0.5)
        assert not math.isfinite(norm.item()) and (g[0] == 1).all() and g[1][0] == 1
    assert P.grad_norm([]).item() == 0 and P.grad_norm([torch.empty(0, device="cuda")]).item() == 0
    assert P.grad_clip([], 1.0).item() == 0
    same = torch.ones(100, device="cuda")
    assert abs(P.grad_norm([same, same]).item() - math.sqrt(200)) <= U * 15      # read lists may overlap
    with pytest.raises(P.AecctError):
        P.grad_clip([same, same], 1.0)


def _adam64(p, m, v, g, f, t, lr, b1, b2, eps, wd):
    g = g.double() * f
    m2 = b1 * m.double() + (1 - b1) * g
    v2 = b2 * v.double() + (1 - b2) * g * g
    den = torch.sqrt(v2 / (1 - b2 ** t)) + eps
    size = lr / (1 - b1 ** t)
    p2 = p.double() - lr * wd * p.double() - size * m2 / den
    mb = b1 * m.double().abs() + (1 - b1) * g.abs()
    vb = 8 * U * (b2 * v.double() + (1 - b2) * g * g) + 2.0 ** -148
    pb = U * (20 * size / den * mb + 3 * (lr * wd * p.double()).abs() + p.double().abs() + p2.abs() + (size * m2 / den).abs())
    return p2, m2, v2, pb + 2.0 ** -148, 6 * U * mb + 2.0 ** -148, vb


@pytest.mark.parametrize("types", [ALL[:1], ALL[1:2], ALL], ids=["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("name", list(LISTS))
def test_adam(P, name, types):
    print(f"[adam] {name} {types}", flush=True)
    counts = LISTS[name]
    for flat, clip, wd, copies in ((True, True, 0.01, True), (False, False, 0.0, False)):
        p, m = _tensors(counts, ALL[:1], 1, 0.1, flat), _tensors(counts, ALL[:1], 2, 1e-3, flat)
        v = [t.square_() for t in _tensors(counts, ALL[:1], 3, 1e-2, flat)]
        g = _tensors(counts, types, 4, 0.01, flat)
        c = [torch.full_like(t, 7, dtype=ALL[1 + i % 2]) if i % 3 else torch.empty(0, device="cuda") for i, t in enumerate(p)] if copies else None
        most = 0.5 * _norm64(g) if clip else None
        step = torch.tensor([2], dtype=torch.int64, device="cuda")
        opt = P.Adam(p, 1e-3, (0.9, 0.99), 1e-8, wd, most, m, v, step, c)
        for k in range(3):
            before = [[t.clone() for t in ts] for ts in (p, m, v)]
            norm = opt.step(g if k else P.TensorList(g))
            assert step.item() == 3 + k and (norm is None) == (not clip)
            want = _norm64(g)
            if clip:
                assert abs(norm.item() - want) <= 1.01 * U * want
            for i, gi in enumerate(g):
                p2, m2, v2, pb, mb, vb = _adam64(before[0][i], before[1][i], before[2][i], gi, min(1, most / want) if clip else 1,
                                                 3 + k, 1e-3, 0.9, 0.99, 1e-8, wd)
                _near(p[i], p2, pb, "param")
                _near(m[i], m2, mb, "m")
                _near(v[i], v2, vb, "v")
                if copies and c[i].numel():
                    assert torch.equal(c[i], p[i].to(c[i].dtype))
            for gi in g:                      # other gradients for the next update
                gi.mul_(-0.5)
            if clip:
                opt.max_norm = most = 0.5 * _norm64(g)


def test_adam_starts_skips_and_follows_lr(P):
    p = [torch.randn(1000, device="cuda"), torch.randn(70, device="cuda")]
    p0 = [t.clone() for t in p]
    opt = P.Adam(p, lr=1e-2, max_norm=1.0)
    g = [torch.randn(1000, device="cuda"), torch.randn(70, device="cuda")]
    g[1][3] = math.nan
    norm = opt.step(g)                        # not finite: nothing changes
    assert norm.isnan().item() and opt.step_count.item() == 0
    assert all(torch.equal(a, b) for a, b in zip(p, p0)) and all((t == 0).all() for t in opt.m.tensors + opt.v.tensors)
    g[1][3] = math.inf
    assert math.isinf(opt.step(g).item()) and opt.step_count.item() == 0 and torch.equal(p[0], p0[0])
    g[1][3] = 0.25
    opt.step(g)                               # the first update moves each value by about lr
    assert opt.step_count.item() == 1
    moved = (p0[0] - p[0]) / 1e-2
    assert torch.equal(moved.sign(), g[0].sign()) and ((moved.abs() - 1).abs() < 1e-2).all()
    lr = torch.zeros(1, device="cuda")
    now = [t.clone() for t in p]
    opt.step(g, lr=lr)                        # lr from the GPU: 0 moves nothing but the moments
    assert all(torch.equal(a, b) for a, b in zip(p, now)) and opt.step_count.item() == 2
    lr.fill_(1e-2)
    twin = P.Adam([t.clone() for t in p], 1.0, max_norm=1.0, m=[t.clone() for t in opt.m.tensors],
                  v=[t.clone() for t in opt.v.tensors], step=opt.step_count.clone())
    opt.step(g, lr=lr)
    twin.step(g, lr=float(lr.item()))
    assert all(torch.equal(a, b) for a, b in zip(p, twin.params.tensors))
    e = P.Adam([], max_norm=1.0)
    assert e.step([]).item() == 0 and e.step_count.item() == 1
    n = P.Adam([torch.empty(0, device="cuda")])
    assert n.step([torch.empty(0, device="cuda")]) is None and n.step_count.item() == 1


def test_update_in_graphs_and_on_streams(P):
    """Captured updates (two graphs of the same optimiser, lr from the GPU) against eager ones, replay for replay."""
    counts = [5000, 3, 70001, 128]
    p, g = _tensors(counts, ALL[:1], 1), _tensors(counts, ALL, 2, 0.1)
    lr = torch.full((1,), 1e-3, device="cuda")
    opt = P.Adam(p, lr, max_norm=1.0, weight_decay=0.1)
    twin = P.Adam([t.clone() for t in p], 1e-3, max_norm=1.0, weight_decay=0.1)
    clipped = [torch.empty_like(t) for t in g]
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = opt.step(g)
            cn = P.grad_clip(g, 0.5, out=clipped)
        graphs.append((graph, norm, cn))
    side = torch.cuda.Stream()
    for k in range(4):
        for gi in g:
            gi.copy_(torch.randn(gi.shape, device="cuda") * 0.1 * (k + 1))
        lr.fill_(float(np.float32(1e-3 * (k + 1))))
        for graph, norm, cn in graphs:
            graph.replay()
            torch.cuda.synchronize()
            if k % 2:
                side.wait_stream(torch.cuda.current_stream())
                want = twin.step(g, lr=lr.item(), stream=side)
                again = [torch.empty_like(t) for t in g]
                side.wait_stream(torch.cuda.current_stream())
                n2 = P.grad_clip(g, 0.5, out=again, stream=side)
                side.synchronize()
            else:
                want = twin.step(g, lr=lr.item())
                again = [torch.empty_like(t) for t in g]
                n2 = P.grad_clip(g, 0.5, out=again)
                torch.cuda.synchronize()
            assert torch.equal(norm, want) and torch.equal(cn, n2) and torch.equal(cn, norm)
            assert all(torch.equal(a, b) for a, b in zip(p, twin.params.tensors))
            assert all(torch.equal(a, b) for a, b in zip(clipped, again))
            assert opt.step_count.item() == twin.step_count.item()


def _to_dev(p):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()  # noqa: E731
    out = {}
    for k, v in p.items():
        out[k] = {kk: dev(vv) for kk, vv in v.items()} if k in ("w", "b") else dev(np.array([v])) if k == "head_b1" else \
            None if v is None else dev(v)
    return out


@pytest.mark.parametrize("c,d,layers", [(1, 32, 2), (2, 32, 6)])
def test_trainer_updates(P, c, d, layers):
    """Training steps on the GPU: gradients, then the update of all 22 tensors, each against the formula on the same
    gradients; a captured step replays to the same bits."""
    H = parity_check(CONFIGS[c])
    m, n = H.shape
    params = _to_dev(random_qat_params(n, m, d, layers, seed=5))
    tr = P.Trainer(H, d, layers)
    state = tr.update_state(params)
    y = 1 + 0.6 * torch.randn(32, n, device="cuda")
    for k in range(3):
        loss, grads = tr.grad(params, y)
        before = [tr._flat({a: ({b: t.clone() for b, t in x.items()} if isinstance(x, dict) else x.clone()) for a, x in s.items() if x is not None})
                  for s in (params, state["m"], state["v"])]
        flat = tr._flat(grads)
        want = _norm64(list(flat.values()))
        norm = tr.update(params, grads, state, 1e-3, max_norm=0.5 * want, weight_decay=0.01)
        assert abs(norm.item() - want) <= 1.01 * U * want and state["step"].item() == k + 1
        now = [tr._flat(s) for s in (params, state["m"], state["v"])]
        assert len(flat) == 22
        for f in flat:
            got = _adam64(before[0][f], before[1][f], before[2][f], flat[f], 0.5, k + 1, 1e-3, 0.9, 0.999, 1e-8, 0.01)
            for i in range(3):
                _near(now[i][f], got[i], got[3 + i], (f, i))
    with pytest.raises(ValueError):
        tr.update(params, {**grads, "embed": grads["embed"][:1]}, state, 1e-3)
    tr.close()


def test_norm_ternary_map_gradient_and_update_together(P):
    """A ternary map behind the norm, trained for three steps: h = x + res, codes of the norm, the map of a model's output
    projection on them, a squared loss, the gradient through the norm, the norm of all gradients and the clipped update
    of the gain and of the rows; every step against the formulas on the inputs it was given."""
    from workloads import build_workload
    _, H, _, w, _, _ = build_workload(3, batch=1)
    dec = P.Decoder(H, w)
    d, rows = dec.d, 333
    T = torch.from_numpy(np.ascontiguousarray(w.w["o"][0])).cuda().double()
    s = float(w.scale[0][P.LIN_O])
    x, res = torch.randn(rows, d, device="cuda"), torch.randn(rows, d, device="cuda")
    gain, target = torch.ones(d, device="cuda"), torch.randn(rows, d, device="cuda")
    opt = P.Adam([gain, x], lr=1e-2, max_norm=0.05)
    for k in range(3):
        _, h, codes, alpha = P.rms_norm(x, gain, res, 1e-5, with_y=False, code_type=torch.int8)
        assert torch.equal(h, x + res)
        y64 = (h.double() / torch.sqrt((h.double() ** 2).mean(1, keepdim=True) + float(np.float32(1e-5)))) * gain.double()
        a64 = y64.abs().amax(1, keepdim=True)
        _near(codes.float(), y64 * 127 / a64, 0.5 + 132 * U * 127, "codes")
        acc = dec.ternary_gemm(0, P.LIN_O, codes)
        assert torch.equal(acc.double(), codes.double() @ T)
        out = acc.float() * (s / 127) * alpha[:, None]
        dout = (out - target) / rows
        dy = s * (dout @ T.float().t().contiguous())
        dh, dgain = P.rms_norm_grad(h, dy, gain)
        rho = 1 / torch.sqrt((h.double() ** 2).mean(1, keepdim=True) + float(np.float32(1e-5)))
        xh, g = h.double() * rho, dy.double() * gain.double()
        _near(dgain, (dy.double() * xh).sum(0), U * 400 * (dy.double() * xh).abs().sum(0), "dgain")
        want = rho * (g - xh * (g * xh).mean(1, keepdim=True))
        _near(dh, want, 300 * U * rho * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)), "dh")
        before = [[t.clone() for t in ts] for ts in (opt.params.tensors, opt.m.tensors, opt.v.tensors)]
        norm = opt.step([dgain, dh])
        n64 = _norm64([dgain, dh])
        assert abs(norm.item() - n64) <= 1.01 * U * n64
        for i, gi in enumerate((dgain, dh)):
            got = _adam64(before[0][i], before[1][i], before[2][i], gi, min(1, 0.05 / n64), k + 1, 1e-2, 0.9, 0.999, 1e-8, 0.0)
            for j, ts in enumerate((opt.params, opt.m, opt.v)):
                _near(ts.tensors[i], got[j], got[3 + j], (i, j))
    dec.close()


def test_update_binding_refuses(P):
    a = torch.zeros(8, device="cuda")
    with pytest.raises(ValueError):
        P.grad_norm([a[::2]])
    with pytest.raises(ValueError):
        P.grad_norm([a.double()])
    with pytest.raises(ValueError):
        P.grad_clip([a], 1.0, out=[])
    with pytest.raises(P.AecctError):
        P.grad_clip([a], -1.0)
    with pytest.raises(P.AecctError):
        P.grad_clip([a[:4], a[3:]], 1.0)
    with pytest.raises(ValueError):
        P.Adam([a], m=[])
    with pytest.raises(ValueError):
        P.Adam([a], step=torch.zeros(1, device="cuda"))
    opt = P.Adam([a])
    with pytest.raises(ValueError):
        opt.step([])
    with pytest.raises(P.AecctError):
        opt.step([torch.zeros(9, device="cuda")])
    with pytest.raises(P.AecctError):
        opt.step([a])                                  # the parameter as its own gradient
    with pytest.raises(ValueError):
        opt.step([torch.zeros(8, device="cuda")], lr=torch.zeros(2, device="cuda"))
    with pytest.raises(P.AecctError):
        P.Adam([torch.zeros(8, device="cuda", dtype=torch.float16)], m=[torch.zeros(8, device="cuda")],
               v=[torch.zeros(8, device="cuda")]).step([a])


def test_lists_of_more_values_than_32_bits_count(P):
    n = 2 ** 31 + 4100
    g = torch.full((n,), 0.5, device="cuda", dtype=torch.bfloat16)
    g[-1] = 3.0
    want = math.sqrt(0.25 * (n - 1) + 9.0)
    assert abs(P.grad_norm([g]).item() - want) <= 1.01 * U * want
    P.grad_clip([g], want / 2)
    assert (g[:5000] == 0.25).all() and (g[-5000:-1] == 0.25).all() and g[-1] == 1.5 and (g[2 ** 30:2 ** 30 + 9] == 0.25).all()
    p, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    P.Adam([p], lr=1.0, m=[m], v=[v]).step([g])
    for part in (p[:5000], p[2 ** 31 - 5000:2 ** 31 + 4099]):
        assert ((part + 1).abs() < 1e-4).all()
    assert abs(m[-1].item() - 0.15) < 1e-6 and abs(v[-1].item() - 2.25e-3) < 1e-8


def test_norm_past_fp32_still_clips(P):
    """Finite values whose norm is past fp32: it is written as infinity, and they are scaled all the same."""
    g = [torch.full((10000,), 3e38, device="cuda"), torch.full((3,), -3e38, device="cuda")]
    assert math.isinf(P.grad_clip(g, 1.0).item())
    want = 1 / math.sqrt(10003)
    assert (g[0] - want).abs().max().item() <= 4 * U * want and (g[1] + want).abs().max().item() <= 4 * U * want
    p = [torch.zeros(5, device="cuda")]
    opt = P.Adam(p, lr=0.5, max_norm=1e-3)
    assert math.isinf(opt.step([torch.full((5,), 3e38, device="cuda")]).item()) and opt.step_count.item() == 1
    assert (p[0] + 0.5).abs().max().item() < 1e-4


def test_tensors_back_to_back_and_apart_agree(P):
    """Lists that lie back to back are taken as one range, in any cut; the values do not depend on it."""
    n = 50021
    flat = torch.randn(n, device="cuda") * 0.01
    cuts = [1, 4095, 1, 0, 9000, 4097, n - 17194]
    whole, parts, apart = [flat.clone()], list(flat.clone().split(cuts)), [t.clone() for t in flat.split(cuts)]
    norms = [P.grad_clip(ts, 0.05).item() for ts in (whole, parts, apart)]
    assert max(norms) - min(norms) <= 2 * U * norms[0]
    assert torch.equal(torch.cat(parts), whole[0])            # one range either way: the same sum
    assert (torch.cat(apart) - whole[0]).abs().max().item() <= 4 * U * whole[0].abs().max().item()
    back = list(reversed(parts))                              # the list in another order than memory
    before = [t.clone() for t in back]
    P.grad_clip(back, 0.01)
    f = 0.01 / _norm64(before)
    for t, b in zip(back, before):
        _near(t, b.double() * f, 2.1 * U * (b.double() * f).abs(), "reversed")
