"""What a block of one's own needs beside the row norm, as cases to be measured: linear maps with bias, activation and
residual, on values or on 8-bit codes, their gradients, cross attention to states of another length with its gradient, and
dropout from a counter-based generator.

A case is one call of one of them.  `own` false computes it in elementary torch operations, `own` true by the framework's
entry points.  Shapes are those of the framework's codes (workloads/configs.py: 128 words of n variable nodes and n - k
check nodes at width d), and generic ones from a single token to large training batches.

Dropout's random words are those of Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
easy as 1, 2, 3", SC 2011): value i of a tensor takes word i % 4 of the block with the counter (i / 4, offset) and the key
`seed`, and is dropped where that word is below p 2^32.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2, "int8": 1, "e4m3": 1}
MOST = {"int8": 127.0, "e4m3": 448.0}
LOW = 0xFFFFFFFF


def _linear(name, rows, inputs, outputs, type, **options):
    return {"name": name, "do": "linear", "rows": rows, "in": inputs, "out": outputs, "type": type, "y": type, "act": "none",
            "bias": True, "residual": False, "z": False, "turned": False, "pad": 0, **options}


def _linear_grad(name, rows, inputs, outputs, type, **options):
    return {"name": name, "do": "linear_grad", "rows": rows, "in": inputs, "out": outputs, "type": type, "act": "none",
            "turned": False, "pad": 0, **options}


def _dropout(name, rows, d, type, **options):
    return {"name": name, "do": "dropout", "rows": rows, "d": d, "type": type, "p": 0.1, "residual": True, "pad": 0, **options}


def _attention(name, batch, queries, keys, heads, kv_heads, d, type, **options):
    return {"name": name, "do": "attention", "batch": batch, "queries": queries, "keys": keys, "heads": heads,
            "kv_heads": kv_heads, "d": d, "type": type, "ragged": False, "mask": "none", **options}


def _attention_grad(*args, **options):
    return {**_attention(*args, **options), "do": "attention_grad"}


def listed():
    return [
        # one token of a serving loop through a wide map back to the residual: the weights are all there is to read
        _linear("linear_token_d4096", 1, 4096, 4096, "bf16", residual=True),
        # the first feed-forward map on 128 words of LDPC(256,128), 384 tokens each: codes times ternary weights, ReLU
        _linear("linear_ldpc256_128_int8", 49152, 128, 512, "int8", y="fp32", act="relu"),
        # a large training batch through the first feed-forward map, its input to the activation kept for the gradient
        _linear("linear_bulk_d4096", 16384, 4096, 8192, "bf16", act="gelu", z=True),
        # odd widths on rows of a wider buffer
        _linear_grad("linear_grad_odd", 1001, 777, 1333, "fp16", act="silu", pad=3),
        # the gradient of a large map
        _linear_grad("linear_grad_bulk_d4096", 8192, 4096, 4096, "bf16", act="gelu"),
        # the residual's dropout on 128 words of BCH(31,16), 46 tokens each: nothing but latency
        _dropout("dropout_bch31_16", 5888, 32, "fp32"),
        # a large training batch
        _dropout("dropout_bulk_d8192", 16384, 8192, "bf16"),
        # serving: one new token a sequence against the encoder's states, lengths all different
        _attention("attention_token_8192", 16, 1, 8192, 32, 8, 128, "bf16", ragged=True),
        # variable nodes attend their check nodes, 128 words of LDPC(256,128): the Tanner graph as the mask
        _attention("attention_ldpc256_128", 128, 256, 128, 8, 8, 16, "fp32", mask="graph"),
        # a training batch against an encoder's padded states of an odd length, shared key heads
        _attention("attention_bulk_2111", 2, 4096, 2111, 32, 8, 128, "bf16", ragged=True),
        # the gradient of the code's attention
        _attention_grad("attention_grad_ldpc256_128", 128, 256, 128, 8, 8, 16, "fp32", mask="graph"),
        # the gradient at odd lengths, a band of the keys for each query
        _attention_grad("attention_grad_band", 2, 2049, 1531, 16, 4, 64, "bf16", ragged=True, mask="band"),
    ]


def _log_between(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    do = rng.choice(("linear", "linear", "linear_grad", "dropout", "attention", "attention", "attention_grad"))
    if do in ("linear", "linear_grad"):
        width = lambda: rng.choice((128, 512, 1024, 4096)) if rng.random() < 0.4 else _log_between(rng, 16, 8192)  # noqa: E731
        inputs, outputs = width(), width()
        rows = _log_between(rng, 1, max(2, min(49152, int((2e11 if do == "linear_grad" else 4e11) / (inputs * outputs)))))
        act, pad, turned = rng.choice(("none", "relu", "gelu", "silu")), rng.choice((0, 0, 0, 3, 8)), rng.random() < 0.3
        if do == "linear_grad":
            case = _linear_grad("", rows, inputs, outputs, rng.choice(("fp32", "bf16", "fp16")), act=act, pad=pad, turned=turned)
        else:
            type = rng.choice(("fp32", "bf16", "fp16", "int8", "e4m3"))
            y = rng.choice(("fp32", "bf16", "fp16")) if type in MOST else type
            case = _linear("", rows, inputs, outputs, type, y=y, act=act, pad=pad, turned=turned, bias=rng.random() < 0.8,
                           residual=rng.random() < 0.5, z=act != "none" and type not in MOST and rng.random() < 0.5)
    elif do == "dropout":
        d = rng.choice((32, 128, 512, 4096, 8192)) if rng.random() < 0.4 else _log_between(rng, 1, 16384)
        case = _dropout("", _log_between(rng, 1, max(2, min(100000, 60000000 // d))), d, rng.choice(("fp32", "bf16", "fp16")),
                        p=rng.choice((0.0, 0.05, 0.1, 0.3, 0.5)), residual=rng.random() < 0.6, pad=rng.choice((0, 0, 0, 3, 8)))
    else:
        kv_heads = rng.choice((1, 2, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 4, 8))
        d = rng.choice((16, 32, 64, 128)) if rng.random() < 0.7 else rng.randrange(1, 257)
        queries = 1 if do == "attention" and rng.random() < 0.3 else _log_between(rng, 1, 4096)
        most = 2e10 if do == "attention" else 1e10      # multiplications of one product
        keys = _log_between(rng, 1, max(2, min(32768, int(most / (heads * queries * d)))))
        batch = _log_between(rng, 1, max(2, min(128, int(most / (heads * queries * d * keys)), 50000000 // (kv_heads * keys * d))))
        case = _attention("", batch, queries, keys, heads, kv_heads, d, rng.choice(("fp32", "bf16", "fp16")),
                          ragged=rng.random() < 0.5, mask=rng.choice(("none", "none", "graph", "band")))
        case["do"] = do
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, rows, d, type, pad=0, scale=1.0):
    wide = torch.randn(rows, d + pad, device="cuda", generator=g).mul_(scale)
    return wide.to(TYPES[type])[:, :d]


def _lengths(case):
    """Keys of each sequence of a padded batch, by the sizes alone; one of them has them all."""
    rng = random.Random("%(batch)d %(queries)d %(keys)d" % case)
    return [case["keys"]] + [rng.randint(case["keys"] // 2, case["keys"]) for _ in range(case["batch"] - 1)]


def _mask(case):
    """[queries][keys], 1 where a query may attend: "graph", three keys for a query as in a regular code's Tanner graph;
    "band", a window of the keys around the query's share of the way, which leaves padded keys out for some."""
    n, m = case["queries"], case["keys"]
    if case["mask"] == "graph":
        at = torch.rand(n, m, generator=torch.Generator().manual_seed(n * m)).argsort(1)[:, :3]
        return torch.zeros(n, m, dtype=torch.bool).scatter_(1, at, True).cuda()
    middle = (torch.arange(n, device="cuda") * m // n)[:, None]
    return (torch.arange(m, device="cuda")[None] - middle).abs() <= max(1, m // 8)


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["do"] in ("linear", "linear_grad"):
        rows, inputs, outputs, type = case["rows"], case["in"], case["out"], case["type"]
        coded = type in MOST
        if coded:    # as the row norm leaves them: the largest of a row is 127 or 448
            x = torch.randn(rows, inputs + case["pad"], device="cuda", generator=g)
            s["alpha"] = x.abs().amax(1)
            x = x * (MOST[type] / s["alpha"])[:, None]
            s["x"] = (x.round() if type == "int8" else x).to(TYPES[type])[:, :inputs]
            s["scale"] = 0.02 + 0.01 * torch.rand(outputs, device="cuda", generator=g)
            shape = (outputs, inputs) if case["turned"] else (inputs, outputs)
            if type == "int8":     # ternary, half of them 0
                w = torch.randint(-1, 2, shape, device="cuda", generator=g, dtype=torch.int8)
                w *= torch.randint(0, 4, shape, device="cuda", generator=g, dtype=torch.int8).clamp_(max=1)
            else:
                w = (100 * torch.randn(shape, device="cuda", generator=g)).clamp_(-448, 448).to(TYPES[type])
                s["scale"] /= 400
        else:
            s["x"] = _rows(g, rows, inputs, type, case["pad"])
            shape = (outputs, inputs) if case["turned"] else (inputs, outputs)
            w = torch.randn(shape, device="cuda", generator=g).mul_(inputs ** -0.5).to(TYPES[type])
        s["w"] = w.t() if case["turned"] else w
        if case["do"] == "linear":
            s["bias"] = torch.randn(outputs, device="cuda", generator=g).mul_(0.1) if case["bias"] else None
            s["res"] = _rows(g, rows, outputs, case["y"], case["pad"]) if case["residual"] else None
        else:
            s["dy"] = _rows(g, rows, outputs, type, case["pad"])
            s["z"] = _rows(g, rows, outputs, type, case["pad"]) if case["act"] != "none" else None
    elif case["do"] == "dropout":
        s["x"] = _rows(g, case["rows"], case["d"], case["type"], case["pad"])
        s["res"] = _rows(g, case["rows"], case["d"], case["type"], case["pad"]) if case["residual"] else None
        s["seed"], s["offset"] = 1234567890123 + seed, 7 * seed + 5    # the run's key, and the step's and layer's number
    else:
        b, n, m, h, kv, d, type = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "d", "type"))
        new = lambda length, heads: torch.randn(b, length, heads, d, device="cuda", generator=g).to(TYPES[type])  # noqa: E731
        s["q"], s["k"], s["v"] = new(n, h), new(m, kv), new(m, kv)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        s["mask"] = _mask(case) if case["mask"] != "none" else None
        if case["do"] == "attention_grad":
            o, lse = _plain_attention(case, s)
            s["o"], s["lse"], s["dout"] = o, lse, new(n, h)
    return s


# ---------------------------------------------------------------------------------------------------------- run
def run(state):
    case = state["case"]
    if own:
        import paper_2410_05911_amd as aecct
        return {"linear": _own_linear, "linear_grad": _own_linear_grad, "dropout": _own_dropout, "attention": _own_attention,
                "attention_grad": _own_attention_grad}[case["do"]](aecct, case, state)
    if case["do"] == "attention":
        o, lse = _plain_attention(case, state)
        return {"o": o, "lse": lse}
    return {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "dropout": _plain_dropout,
            "attention_grad": _plain_attention_grad}[case["do"]](case, state)


def _own_linear(aecct, case, s):
    y, z = aecct.linear(s["x"], s["w"], s["bias"], s["res"], case["act"], alpha=s.get("alpha"), scale=s.get("scale"),
                        y_type=TYPES[case["y"]], with_z=case["z"])
    return {"y": y, "z": z} if case["z"] else {"y": y}


def _own_linear_grad(aecct, case, s):
    dx, dw, dbias = aecct.linear_grad(s["x"], s["w"], s["dy"], s["z"], case["act"])
    return {"dx": dx, "dw": dw, "dbias": dbias}


def _own_dropout(aecct, case, s):
    return {"y": aecct.dropout(s["x"], case["p"], s["seed"], s["offset"], s["res"])}


def _own_attention(aecct, case, s):
    o, lse = aecct.cross_attention(s["q"], s["k"], s["v"], s["lengths"], s["mask"], with_lse=True)
    return {"o": o, "lse": lse}


def _own_attention_grad(aecct, case, s):
    dq, dk, dv = aecct.cross_attention_grad(s["q"], s["k"], s["v"], s["o"], s["lse"], s["dout"], s["lengths"], s["mask"])
    return {"dq": dq, "dk": dk, "dv": dv}


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":     # z Phi(z)
        return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":     # z / (1 + e^-z)
        return z * torch.sigmoid(z)
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p))


def _plain_linear(case, s):
    z = s["x"].float() @ s["w"].float()
    if "alpha" in s:
        z = z * (s["alpha"] * (1 / MOST[case["type"]]))[:, None] * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z, case["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    t = TYPES[case["y"]]
    return {"y": y.to(t), "z": z.to(t)} if case["z"] else {"y": y.to(t)}


def _plain_linear_grad(case, s):
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(s["z"].float(), case["act"])
    t = TYPES[case["type"]]
    return {"dx": (dz @ s["w"].float().t()).to(t), "dw": (s["x"].float().t() @ dz).to(t), "dbias": dz.sum(0)}


def _plain_dropout(case, s):
    n = case["rows"] * case["d"]
    at = torch.arange(-(-n // 4), device="cuda")
    c0, c1 = at & LOW, at >> 32
    c2, c3 = torch.full_like(at, s["offset"] & LOW), torch.full_like(at, s["offset"] >> 32)
    k0, k1 = s["seed"] & LOW, s["seed"] >> 32
    for _ in range(7):      # Philox4x32: the high and low halves of two products change places
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & LOW) ^ c1 ^ k0, p1 & LOW, ((p0 >> 32) & LOW) ^ c3 ^ k1, p0 & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    word = torch.stack((c0, c1, c2, c3), 1).view(-1)[:n].view(case["rows"], case["d"])
    y = torch.where(word >= int(case["p"] * 2.0 ** 32), s["x"].float() * (1 / (1 - case["p"])), 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"y": y.to(TYPES[case["type"]])}


def _by_heads(t, kv):
    """[batch][length][heads][d] -> [batch][kv heads][heads of one times length][d], in 32 bits."""
    b, n, h, d = t.shape
    return t.float().view(b, n, kv, h // kv, d).permute(0, 2, 3, 1, 4).reshape(b, kv, h // kv * n, d)


def _back(t, case):
    b, n, h, kv, d = (case[k] for k in ("batch", "queries", "heads", "kv_heads", "d"))
    return t.view(b, kv, h // kv, n, d).permute(0, 3, 1, 2, 4).reshape(b, n, h, d)


def _allowed(case, s):
    """[batch or 1][1][1][queries or 1][keys], or None where every key counts."""
    allowed = None
    if s["lengths"] is not None:
        allowed = (torch.arange(case["keys"], device="cuda")[None] < s["lengths"][:, None])[:, None, None, None]
    if s["mask"] is not None:
        allowed = s["mask"] & allowed if allowed is not None else s["mask"][None, None, None]
    return allowed


def _scores(case, s, q, k):
    b, n, m, h, kv, d = (case[x] for x in ("batch", "queries", "keys", "heads", "kv_heads", "d"))
    score = torch.matmul(q * d ** -0.5, k.transpose(2, 3).contiguous()).view(b, kv, h // kv, n, m)
    allowed = _allowed(case, s)
    return score if allowed is None else score.masked_fill(~allowed, -math.inf)


def _plain_attention(case, s):
    """o and the logarithm of each row's sum [batch][heads][queries]; a row that attends nothing: 0 and -inf."""
    b, n, m, h, kv = (case[x] for x in ("batch", "queries", "keys", "heads", "kv_heads"))
    score = _scores(case, s, _by_heads(s["q"], kv), _by_heads(s["k"], kv))
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul((p / total.clamp(min=1e-30)).view(b, kv, h // kv * n, m), _by_heads(s["v"], kv))
    lse = torch.where(total > 0, top + torch.log(total), -math.inf).view(b, h, n)
    return _back(o, case).to(TYPES[case["type"]]), lse


def _plain_attention_grad(case, s):
    b, n, m, h, kv, d = (case[x] for x in ("batch", "queries", "keys", "heads", "kv_heads", "d"))
    q, k, v, dout, o = (_by_heads(s[x], kv) for x in ("q", "k", "v", "dout", "o"))
    lse = s["lse"].view(b, kv, h // kv, n, 1)
    p = torch.exp(_scores(case, s, q, k) - torch.where(lse > -math.inf, lse, 0.0)).view(b, kv, h // kv * n, m)
    dp = torch.matmul(dout, v.transpose(2, 3).contiguous())
    ds = p * (dp - (dout * o).sum(-1, keepdim=True)) * d ** -0.5
    t = TYPES[case["type"]]
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q).transpose(1, 2).to(t)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), dout).transpose(1, 2).to(t)
    return {"dq": _back(torch.matmul(ds, k), case).to(t), "dk": dk.contiguous(), "dv": dv.contiguous()}


# ---------------------------------------------------------------------------------------------------- work, exact
def _pairs(case):
    """Query and key pairs of a head over the batch."""
    n, m = case["queries"], case["keys"]
    lengths = _lengths(case) if case["ragged"] else [m] * case["batch"]
    if case["mask"] == "none":
        return n * sum(lengths)
    if case["mask"] == "graph":
        return sum(n * min(3, m) * length // m for length in lengths)
    half = max(1, m // 8)
    return sum(max(0, min(length, i * m // n + half + 1) - max(0, i * m // n - half)) for length in set(lengths) for i in range(n)) \
        * len(lengths) // len(set(lengths))


def work(case):
    if case["do"] in ("linear", "linear_grad"):
        rows, inputs, outputs, size = case["rows"], case["in"], case["out"], SIZE[case["type"]]
        if case["do"] == "linear":
            coded = 4 * (rows + outputs) if case["type"] in MOST else 0
            each = SIZE[case["y"]] * (1 + case["residual"] + case["z"])
            return {"bytes": size * (rows + outputs) * inputs + each * rows * outputs + 4 * outputs * case["bias"] + coded,
                    "flops": 2 * rows * inputs * outputs}
        each = size * (1 + (case["act"] != "none"))
        return {"bytes": 2 * size * (rows + outputs) * inputs + each * rows * outputs + 4 * outputs,
                "flops": 4 * rows * inputs * outputs}
    if case["do"] == "dropout":     # seven rounds of two products and four exclusive ors for four values, and the values' own
        n = case["rows"] * case["d"]
        return {"bytes": n * SIZE[case["type"]] * (2 + case["residual"]), "flops": n * (14 + case["residual"])}
    size = SIZE[case["type"]]
    rows, keys = case["batch"] * case["queries"], sum(_lengths(case)) if case["ragged"] else case["batch"] * case["keys"]
    q, kv = rows * case["heads"] * case["d"] * size, keys * case["kv_heads"] * case["d"] * size
    masked = case["queries"] * case["keys"] if case["mask"] != "none" else 0
    product = 2 * case["heads"] * _pairs(case) * case["d"]
    if case["do"] == "attention":
        return {"bytes": 2 * q + 2 * kv + 4 * rows * case["heads"] + masked, "flops": 2 * product}
    return {"bytes": 4 * q + 4 * kv + 4 * rows * case["heads"] + masked, "flops": 5 * product}


def _exact_slope(z, act):
    """The derivative by autograd of the activation's definition in 64 bits."""
    with torch.enable_grad():
        z = z.detach().requires_grad_()
        y = {"relu": lambda: torch.where(z > 0, z, 0 * z), "gelu": lambda: z * torch.special.ndtr(z),
             "silu": lambda: z / (1 + torch.exp(-z))}[act]()
        return torch.autograd.grad(y.sum(), z)[0]


def _exact_words(n, seed, offset):
    """Philox4x32-7's words, its 32-bit products made of products of 16 bits."""
    def halves(a, b):
        a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        middle = a1 * b0 + (a0 * b0 >> 16)
        cross = a0 * b1 + (middle & 0xFFFF)
        return a1 * b1 + (middle >> 16) + (cross >> 16), (cross << 16 | a0 * b0 & 0xFFFF) & LOW
    block = torch.arange((n + 3) // 4, device="cuda")
    c = [block % (1 << 32), block // (1 << 32), block * 0 + offset % (1 << 32), block * 0 + offset // (1 << 32)]
    for r in range(7):
        key = [(part + r * step) % (1 << 32) for part, step in ((seed % (1 << 32), 0x9E3779B9), (seed // (1 << 32), 0xBB67AE85))]
        (h0, l0), (h1, l1) = halves(c[0], 0xD2511F53), halves(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
    return torch.stack(c).t().reshape(-1)[:n]


def exact(case, seed):
    """The definitions in 64 bits on the same inputs."""
    s = prepare(case, seed)
    if case["do"] == "linear":
        x, w = s["x"].double(), s["w"].double()
        if "alpha" in s:
            x, w = x * s["alpha"].double()[:, None] / MOST[case["type"]], w * s["scale"].double()
        z = x @ w if s["bias"] is None else torch.addmm(s["bias"].double(), x, w)
        y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0 * z), "gelu": lambda: z * torch.special.ndtr(z),
             "silu": lambda: z / (1 + torch.exp(-z))}[case["act"]]()
        y = y if s["res"] is None else y + s["res"]
        return {"y": y, "z": z} if case["z"] else {"y": y}
    if case["do"] == "linear_grad":
        dz = s["dy"].double() * (1 if s["z"] is None else _exact_slope(s["z"].double(), case["act"]))
        return {"dx": dz @ s["w"].double().t(), "dw": s["x"].double().t() @ dz, "dbias": torch.ones_like(dz[:, 0]) @ dz}
    if case["do"] == "dropout":
        kept = _exact_words(case["rows"] * case["d"], s["seed"], s["offset"]).view(case["rows"], -1) >= case["p"] * 2.0 ** 32 // 1
        y = s["x"].double() / (1 - case["p"]) * kept
        return {"y": y if s["res"] is None else y + s["res"]}
    # one key head of one sequence at a time
    b, h, kv = case["batch"], case["heads"], case["kv_heads"]
    names = ("q", "k", "v") if case["do"] == "attention" else ("q", "k", "v", "o", "dout")
    t = {x: s[x].double().transpose(1, 2) for x in names}      # [batch][heads][length][d]
    lengths = s["lengths"].tolist() if s["lengths"] is not None else [case["keys"]] * b
    out = {x: torch.zeros_like(t[y]) for x, y in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    lse = torch.full((b, h, case["queries"]), -math.inf, dtype=torch.float64, device="cuda")
    many = max(1, min(b, (1 << 28) // (h // kv * case["queries"] * case["keys"])))
    groups = sorted({length for length in lengths})
    for length in groups:
        same = [i for i in range(b) if lengths[i] == length]
        for first in range(0, len(same) if length else 0, many):
            at = torch.tensor(same[first: first + many], device="cuda")
            for j in range(kv):
                heads = torch.arange(j * (h // kv), (j + 1) * (h // kv), device="cuda")
                q = t["q"][at][:, heads]
                k, v = t["k"][at, j, :length][:, None], t["v"][at, j, :length][:, None]
                score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(case["d"])
                if s["mask"] is not None:
                    score = torch.where(s["mask"][:, :length], score, -math.inf)
                total = torch.logsumexp(score, -1)
                p = torch.exp(score - torch.where(total == -math.inf, 0.0, total)[..., None])
                lse[at[:, None], heads[None]] = total
                if case["do"] == "attention":
                    out["o"][at[:, None], heads[None]] = torch.matmul(p, v)
                    continue
                dout = t["dout"][at][:, heads]
                row = (dout * t["o"][at][:, heads]).sum(-1, keepdim=True)
                ds = p * (torch.matmul(dout, v.transpose(2, 3).contiguous()) - row) / math.sqrt(case["d"])
                out["dq"][at[:, None], heads[None]] = torch.matmul(ds, k)
                out["dk"][at, j, :length] = torch.matmul(ds.transpose(2, 3).contiguous(), q).sum(1)
                out["dv"][at, j, :length] = torch.matmul(p.transpose(2, 3).contiguous(), dout).sum(1)
    if case["do"] == "attention":
        return {"o": out["o"].transpose(1, 2), "lse": lse}
    return {x: out[x].transpose(1, 2) for x in ("dq", "dk", "dv")}
