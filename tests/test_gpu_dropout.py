"""Dropout against its definition: the words of Philox4x32-7 from Python's integers, values in 64 bits.

Tolerance: 1 / (1 - p) rounded to fp32, the product and the sum: 3 u |x| / (1 - p) + u |y|, and half a step of the type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def P():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2410_05911_amd as P
    P.lib()
    return P


def _words(n, seed, offset, first=0):
    """The words of n values from block `first` on."""
    low = np.uint64(0xFFFFFFFF)
    i = np.arange(first, first + (n + 3) // 4, dtype=np.uint64)
    c = [i & low, i >> np.uint64(32), np.full_like(i, offset & 0xFFFFFFFF), np.full_like(i, offset >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).reshape(-1)[:n]


@pytest.mark.parametrize("type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,d,pad", [(1, 1, 0), (1, 7, 0), (3, 4, 0), (5, 3, 0), (5, 3, 4), (17, 33, 2), (64, 32, 8), (9, 1001, 3),
                                        (2, 4099, 0), (130, 64, 1)])
@pytest.mark.parametrize("p,res,seed,offset", [(0.1, True, 1, 0), (0.5, False, 2 ** 64 - 1, 2 ** 63 + 5), (0.0, True, 12345678901234, 7),
                                               (0.999, True, 5, 2 ** 32)])
def test_dropout(P, type, rows, d, pad, p, res, seed, offset):
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda: torch.randn(rows, d + pad, device="cuda", generator=g).to(type)[:, :d]  # noqa: E731
    x, r = new(), new() if res else None
    out = torch.full((rows, d + pad), 77.0, dtype=type, device="cuda")
    y = P.dropout(x, p, seed, offset, r, y=out[:, :d])
    kept = torch.from_numpy(_words(rows * d, seed, offset) >= np.uint64(int(p * 2 ** 32))).cuda().view(rows, d)
    scaled = torch.where(kept, x.double() / (1 - p), 0.0)
    want = scaled + (r.double() if res else 0)
    assert bool(((y.double() - want).abs() <= 3 * U * scaled.abs() + (U + HALF[type]) * want.abs() + 2.0 ** -25).all())
    assert bool((out[:, d:] == 77).all())
    if not res:
        assert torch.equal(y == 0, ~kept | (x == 0))


def test_gradient_is_the_same_call(P):
    """y is linear in x, so <dropout(x), dy> = <x, dropout(dy)>: both sums in 64 bits of values off by 2 u each."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = torch.randn(33, 65, device="cuda", generator=g), torch.randn(33, 65, device="cuda", generator=g)
    a, b = (P.dropout(x, 0.3, 9, 4).double() * dy).sum(), (P.dropout(dy, 0.3, 9, 4).double() * x).sum()
    assert abs(a - b) <= 8 * U * (x.double() * dy / 0.7).abs().sum()


def test_in_place_more_dimensions_and_empty(P):
    x = torch.randn(3, 5, 6, device="cuda")
    want = P.dropout(x, 0.4, 3, 1, x)
    keep = x.clone()
    assert P.dropout(x, 0.4, 3, 1, x, y=x) is x and torch.equal(x, want) and not torch.equal(x, keep)
    assert P.dropout(torch.empty(0, 8, device="cuda"), 0.4, 3).shape == (0, 8)
    assert torch.equal(P.dropout(keep.view(-1, 6), 0.4, 3, 1), P.dropout(keep, 0.4, 3, 1).view(-1, 6))


def test_dropped_nan_is_dropped(P):
    x = torch.full((64, 64), float("nan"), device="cuda")
    y = P.dropout(x, 0.5, 1)
    kept = torch.from_numpy(_words(4096, 1, 0) >= np.uint64(2 ** 31)).cuda().view(64, 64)
    assert torch.equal(y.isnan(), kept) and not y[~kept].any()


def test_offset_from_the_gpu_in_a_graph(P):
    x, offset = torch.randn(40, 50, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    P.dropout(x, 0.5, 1, offset)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.dropout(x, 0.5, 1, offset)
        offset.add_(1)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, P.dropout(x, 0.5, 1, step)), step


def test_high_words_of_seed_and_offset(P):
    x = torch.ones(1, 64, device="cuda")
    for seed, offset in ((2 ** 40 + 3, 1), (3, 2 ** 40 + 1)):
        kept = torch.from_numpy(_words(64, seed, offset) >= np.uint64(2 ** 31)).cuda()
        assert torch.equal(P.dropout(x, 0.5, seed, offset)[0] != 0, kept)


def test_blocks_past_32_bits(P):
    """65537 rows of 2^18 values: the last row's blocks begin at 2^32.  (One row for all as the input.)"""
    d = 1 << 18
    x = torch.ones(1, d, dtype=torch.bfloat16, device="cuda").expand(65537, d)
    y = P.dropout(x, 0.5, 11, 3)
    for row in (0, 65535, 65536):
        kept = torch.from_numpy(_words(256, 11, 3, row * d // 4) >= np.uint64(2 ** 31)).cuda()
        assert torch.equal(y[row, :256] != 0, kept), row


def test_refusals(P):
    x = torch.zeros(4, 8, device="cuda")
    for call in (lambda: P.dropout(x, 0.5, -1), lambda: P.dropout(x, 0.5, 1, 2 ** 64), lambda: P.dropout(x.double(), 0.5, 1),
                 lambda: P.dropout(x, 0.5, 1, 0, x.bfloat16()), lambda: P.dropout(x, 0.5, 1, torch.zeros(1, device="cuda")),
                 lambda: P.dropout(x.cpu(), 0.5, 1), lambda: P.dropout(x.t(), 0.5, 1)):
        with pytest.raises(ValueError):
            call()
    for p in (-0.1, 1.0, float("nan")):
        with pytest.raises(P.AecctError):
            P.dropout(x, p, 1)
