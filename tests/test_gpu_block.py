"""A cross-attention block and a feed-forward block of the operators together, forward and backward, against the same block in 64
bits with its gradients by autograd; and a decode of tokens one by one through a cache of the states' keys and values.

Tolerance of the training step (fp32): every sum is of at most 160 values and each operator's error at most 2 (160 + 12) u of its
terms' size, 1.3e-5 relative to sums of like sign; ten operators follow one another, and cancellation in sums of random signs grows
it by up to sqrt(160) = 13 between two of them, but errors are random as well and shrink by as much: 2-norms within 10 x 2 x 172 u =
2.1e-4 of the gradients' norms.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from workloads.configs import CONFIGS, parity_check  # noqa: E402

U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _params(g, d, ff):
    new = lambda *s: torch.randn(*s, device="cuda", generator=g) / math.sqrt(s[0])  # noqa: E731
    p = {"q": new(d, d), "k": new(d, d), "v": new(d, d), "o": new(d, d), "w1": new(d, ff), "w2": new(ff, d)}
    p.update({"b1": 0.1 * torch.randn(ff, device="cuda", generator=g), "b2": 0.1 * torch.randn(d, device="cuda", generator=g),
              "g1": 1 + 0.1 * torch.randn(d, device="cuda", generator=g), "g2": 1 + 0.1 * torch.randn(d, device="cuda", generator=g)})
    return p


def _forward(P, p, x, states, mask, heads, drop, seed, offset):
    b, n, d = x.shape
    m = states.shape[1]
    s = {"x": x, "states": states}
    s["a"], _, _, _ = P.rms_norm(x, p["g1"])
    s["q"], _ = P.linear(s["a"], p["q"])
    s["k"], _ = P.linear(states, p["k"])
    s["v"], _ = P.linear(states, p["v"])
    split = lambda t, n: t.view(b, n, heads, d // heads)  # noqa: E731
    s["att"], s["lse"] = P.cross_attention(split(s["q"], n), split(s["k"], m), split(s["v"], m), None, mask, with_lse=True)
    y, _ = P.linear(s["att"].view(b, n, d), p["o"])
    s["h"] = P.dropout(y, drop, seed, offset, x)
    s["c"], _, _, _ = P.rms_norm(s["h"], p["g2"])
    s["f"], s["z"] = P.linear(s["c"], p["w1"], p["b1"], act="gelu", with_z=True)
    y, _ = P.linear(s["f"], p["w2"], p["b2"])
    return P.dropout(y, drop, seed, offset + 1, s["h"]), s


def _backward(P, p, s, dout, mask, heads, drop, seed, offset):
    g = {}
    b, n, d = dout.shape
    m = s["states"].shape[1]
    df, g["w2"], g["b2"] = P.linear_grad(s["f"], p["w2"], P.dropout(dout, drop, seed, offset + 1))
    dc, g["w1"], g["b1"] = P.linear_grad(s["c"], p["w1"], df, s["z"], "gelu")
    dh, g["g2"] = P.rms_norm_grad(s["h"], dc, p["g2"], dout)
    split = lambda t, n: t.view(b, n, heads, d // heads)  # noqa: E731
    datt, g["o"], _ = P.linear_grad(s["att"].view(b, n, d), p["o"], P.dropout(dh, drop, seed, offset), with_dbias=False)
    dq, dk, dv = P.cross_attention_grad(split(s["q"], n), split(s["k"], m), split(s["v"], m), s["att"], s["lse"], split(datt, n),
                                        None, mask)
    da, g["q"], _ = P.linear_grad(s["a"], p["q"], dq.view(b, n, d), with_dbias=False)
    ds, g["k"], _ = P.linear_grad(s["states"], p["k"], dk.view(b, m, d), with_dbias=False)
    ds2, g["v"], _ = P.linear_grad(s["states"], p["v"], dv.view(b, m, d), with_dbias=False)
    g["x"], g["g1"] = P.rms_norm_grad(s["x"], da, p["g1"], dh)
    g["states"] = ds + ds2
    return g


def test_training_step_of_a_block(P):
    """Variable nodes of BCH(31,16) attend its check nodes under the Tanner graph."""
    H = parity_check(CONFIGS[1])
    m, n = H.shape
    mask = torch.from_numpy(np.ascontiguousarray(H.T) != 0).cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    b, d, ff, heads, drop, seed, offset = 5, 32, 128, 8, 0.2, 99, 10
    p = _params(g, d, ff)
    x, states, dout = (torch.randn(b, k, d, device="cuda", generator=g) for k in (n, m, n))
    y, s = _forward(P, p, x, states, mask, heads, drop, seed, offset)
    got = _backward(P, p, s, dout, mask, heads, drop, seed, offset)
    kept = [(P.dropout(torch.ones_like(dout), drop, seed, offset + i) != 0).double() / (1 - drop) for i in (0, 1)]
    leaves = {k: v.double().requires_grad_() for k, v in {**p, "x": x, "states": states}.items()}
    q = leaves
    norm = lambda t, gain: t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-5) * gain  # noqa: E731
    heads_of = lambda t: t.view(b, -1, heads, d // heads).transpose(1, 2).contiguous()  # noqa: E731
    a = norm(q["x"], q["g1"])
    qq, kk, vv = heads_of(a @ q["q"]), heads_of(q["states"] @ q["k"]), heads_of(q["states"] @ q["v"])
    score = (qq[..., None, :] * kk[:, :, None]).sum(-1) / math.sqrt(d // heads)
    w = torch.softmax(score.masked_fill(~mask, -math.inf), -1)
    att = (w[..., None] * vv[:, :, None]).sum(-2).transpose(1, 2).reshape(b, n, d)
    h = (att @ q["o"]) * kept[0] + q["x"]
    z = norm(h, q["g2"]) @ q["w1"] + q["b1"]
    out = (z * torch.special.ndtr(z) @ q["w2"] + q["b2"]) * kept[1] + h
    bound = 10 * 2 * 172 * U
    assert (y.double() - out).norm() <= bound * out.norm()
    want = torch.autograd.grad((out * dout.double()).sum(), list(leaves.values()))
    for name, t in zip(leaves, want):
        assert (got[name].double() - t).norm() <= bound * t.norm(), (name, ((got[name].double() - t).norm() / t.norm()).item())
    # the same step, captured and replayed
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, s2 = _forward(P, p, x, states, mask, heads, drop, seed, offset)
        got2 = _backward(P, p, s2, dout, mask, heads, drop, seed, offset)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and all(torch.equal(got[k], got2[k]) for k in got)


def test_tokens_one_by_one_are_the_batch(P):
    """A token's attention to a cache of states does not depend on the tokens beside it: one by one and as a batch differ by fp32's
    rounding and the weights' in bf16 alone, 2 (2 r + 2 m u + w) of sums of p |v| with p summing to 1, and the outputs' rounding."""
    g = torch.Generator(device="cuda").manual_seed(2)
    b, n, m, h, kv, d = 3, 140, 900, 8, 2, 64
    q = torch.randn(b, n, h, d, device="cuda", generator=g).bfloat16()
    k, v = (torch.randn(b, 1024, kv, d, device="cuda", generator=g).bfloat16()[:, :m] for _ in range(2))
    lengths = torch.tensor([900, 17, 513], dtype=torch.int32, device="cuda")
    whole, _ = P.cross_attention(q, k, v, lengths)
    most = v.float().abs().amax()
    for i in range(0, n, 20):
        one, _ = P.cross_attention(q[:, i: i + 1], k, v, lengths)
        assert bool(((one.float() - whole[:, i: i + 1].float()).abs() <= (4 * 2.0 ** -8 + 1e-3) * most).all())


def test_calls_on_two_streams_at_once(P):
    """Calls in flight together have workspaces of their own: split products, masks, joined sums."""
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    mask = torch.rand(3, 2000, device="cuda", generator=g) < 0.3
    jobs = []
    for _ in range(2):
        x, w, dy = new(20, 4000), new(4000, 200), new(20, 200)
        q, k, v, dout = new(2, 3, 8, 64), new(2, 2000, 2, 64), new(2, 2000, 2, 64), new(2, 3, 8, 64)

        def job(x=x, w=w, dy=dy, q=q, k=k, v=v, dout=dout):
            o, lse = P.cross_attention(q, k, v, None, mask, with_lse=True)
            return [P.linear(x, w)[0], *P.linear_grad(x, w, dy), o, lse, *P.cross_attention_grad(q, k, v, o, lse, dout, None, mask)]
        jobs.append(job)
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(8):
        for i, job in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                got[i].append(job())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for run in got[i] for a, b in zip(run, want[i]))
