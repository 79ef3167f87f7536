"""Cross attention and its gradient at the sizes that take 128 rows a block, and on tensors whose tiles go past the registers to LDS, by
the checks and tolerances of test_gpu_cross_attention.py.

By plan_attention: 128 rows (queries of the heads that share a key head) a block from 256 such blocks over sequences and key heads on, the
keys split below 512 where there are 1024 and more; else 32 rows whose wavefronts share the keys.  In fp32 rows of up to 64 values under
masks of few keys go pair by pair."""
import pytest

import test_gpu_cross_attention as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
P = base.P
TENSOR, MASK = base._tensor, base._mask


def _tensor(g, b, n, h, d, type, layout, scale=1.0):
    """"tight": contiguous at a 16-byte address, NaN around."""
    if layout != "tight":
        return TENSOR(g, b, n, h, d, type, layout, scale)
    whole = torch.full((b * n * h * d + 32,), float("nan"), dtype=type, device="cuda")
    view = whole[16: 16 + b * n * h * d].view(b, n, h, d)
    view.copy_(torch.randn(b, n, h, d, device="cuda", generator=g).mul(scale))
    return view


def _mask(g, n, m, kind):
    """"graph": three keys for each query, and none for every 17th."""
    if kind != "graph":
        return MASK(g, n, m, kind)
    keep = torch.zeros(n, m, dtype=torch.bool, device="cuda")
    keep.scatter_(1, torch.rand(n, m, device="cuda", generator=g).argsort(1)[:, :3], True)
    keep[::17] = False
    return keep


@pytest.fixture(autouse=True)
def layouts(monkeypatch):
    monkeypatch.setattr(base, "_tensor", _tensor)
    monkeypatch.setattr(base, "_mask", _mask)


HOW = [("tight", False, "none"), ("tight", True, "none"), ("tight", True, "band"), ("tight", False, "graph"), ("wide", True, "holes"),
       ("heads", True, "graph")]


@pytest.mark.parametrize("b,n,m,h,kv,d", [
    (16, 520, 150, 4, 4, 16), (16, 520, 150, 4, 4, 32), (16, 520, 150, 4, 4, 40), (16, 520, 150, 4, 4, 64), (16, 520, 150, 4, 4, 77),
    (16, 520, 150, 4, 4, 128), (16, 520, 150, 4, 4, 160), (16, 520, 150, 4, 4, 192), (16, 520, 150, 4, 4, 200), (16, 520, 150, 4, 4, 256),
    (40, 130, 90, 8, 2, 64), (21, 33, 300, 40, 5, 32),       # 4 and 8 heads a key head
    (8, 520, 1100, 8, 8, 64), (8, 520, 1100, 8, 8, 16)])     # keys split
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout,lengths,mask", HOW)
def test_many_rows(P, b, n, m, h, kv, d, kind, layout, lengths, mask):
    base.test_attention_and_gradient(P, b, n, m, h, kv, d, kind, layout, lengths, mask)


@pytest.mark.parametrize("b,n,m,h,kv,d", [
    (1, 1, 3, 1, 1, 16), (2, 1, 33, 4, 2, 16), (7, 33, 31, 6, 2, 32), (2, 65, 129, 4, 1, 48), (1, 128, 100, 2, 2, 64), (7, 130, 200, 4, 2, 128),
    (2, 45, 150, 4, 2, 192), (2, 70, 90, 2, 2, 256), (2, 3, 1100, 8, 2, 64), (1, 700, 2100, 4, 2, 32)])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout,lengths,mask", HOW)
def test_few_rows(P, b, n, m, h, kv, d, kind, layout, lengths, mask):
    base.test_attention_and_gradient(P, b, n, m, h, kv, d, kind, layout, lengths, mask)


def test_captured(P):
    """Many rows with split keys under a mask, and their gradient, replayed between eager calls."""
    s = base._case(8, 520, 1100, 8, 8, 64, "fp16", "tight", False, "band", 5)
    lengths = torch.full((8,), 1100, dtype=torch.int32, device="cuda")

    def call():
        o, lse = P.cross_attention(s["q"], s["k"], s["v"], lengths, s["mask"], with_lse=True)
        return [o, lse, *P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"], lengths, s["mask"])]
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(3):
        s["q"].normal_()
        lengths.copy_(torch.arange(8) * 150 + step)
        want = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), step


def test_heads_of_no_values_are_refused(P):
    q, k = torch.zeros(2, 3, 4, 0, device="cuda"), torch.zeros(2, 5, 2, 0, device="cuda")
    lse = torch.zeros(2, 4, 3, device="cuda")
    for call in (lambda: P.cross_attention(q, k, k), lambda: P.cross_attention(q, k, k, scale=1.0), lambda: P.cross_attention_grad(q, k, k, q, lse, q)):
        with pytest.raises(ValueError):
            call()


def test_one_row_of_a_mask_for_all_queries(P):
    """A mask with a stride of 0."""
    s = base._case(3, 70, 130, 4, 2, 32, "fp32", "tight", True, "none", 6)
    row = torch.rand(1, 130, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)) < 0.3
    outs = []
    for mask in (row.expand(70, 130), row.repeat(70, 1)):
        o, lse = P.cross_attention(s["q"], s["k"], s["v"], s["lengths"], mask, with_lse=True)
        outs.append([o, lse, *P.cross_attention_grad(s["q"], s["k"], s["v"], o, lse, s["dout"], s["lengths"], mask)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_keys_and_values_in_turn(P):
    """k and v, and dk and dv, in turn by heads ([batch][keys][heads][2][d]) and by sequences ([keys][batch][2][heads][d]): the bits that
    contiguous tensors give."""
    s = base._case(3, 70, 130, 4, 2, 32, "fp32", "tight", True, "none", 8)
    k, v = s["k"].contiguous(), s["v"].contiguous()
    o, lse = P.cross_attention(s["q"], k, v, s["lengths"], with_lse=True)
    want = [o, lse, *P.cross_attention_grad(s["q"], k, v, o, lse, s["dout"], s["lengths"])]
    by_heads = lambda: torch.full((3, 130, 2, 2, 32), 77.0, device="cuda")  # noqa: E731
    by_batch = lambda: torch.full((130, 3, 2, 2, 32), 77.0, device="cuda")  # noqa: E731
    for whole, parts in ((by_heads, lambda t: (t[:, :, :, 0], t[:, :, :, 1])),
                         (by_batch, lambda t: (t[:, :, 0].transpose(0, 1), t[:, :, 1].transpose(0, 1)))):
        kv, dkv = whole(), whole()
        for part, t in zip(parts(kv), (k, v)):
            part.copy_(t)
        dk, dv = parts(dkv)
        o, lse = P.cross_attention(s["q"], *parts(kv), s["lengths"], with_lse=True)
        got = [o, lse, *P.cross_attention_grad(s["q"], *parts(kv), o, lse, s["dout"], s["lengths"], dk=dk, dv=dv)]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
