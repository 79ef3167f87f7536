"""The operators around the ternary maps of a model, as cases to be measured: the root-mean-square norm with the
residual's addition and 8-bit codes, its gradient, the norm of all gradients with clipping, and the Adam update.

A case is one call of one of them.  `own` false computes it in elementary torch operations, `own` true by the
framework's entry points.  Shapes are those of the framework's training step (workloads/configs.py: 128 words of a code
of L tokens at width d, the trainer's parameter tensors), and generic ones from a single token to the largest batches.

Gradients and parameters are views of one flat buffer each, back to back, so most tensors start at an odd place.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01


def _norm(name, rows, d, type, **options):
    return {"name": name, "do": "norm", "rows": rows, "d": d, "type": type, "pad": 0, "residual": True, "y": False,
            "codes": "none", "group": 0, "eps": 1e-5, **options}


def _norm_grad(name, rows, d, type, **options):
    return {"name": name, "do": "norm_grad", "rows": rows, "d": d, "type": type, "pad": 0, "residual": True, "eps": 1e-5,
            **options}


def _clip(name, sizes, type, **options):
    return {"name": name, "do": "clip", "sizes": sizes, "type": type, "write": True, **options}


def _adam(name, sizes, type, **options):
    return {"name": name, "do": "adam", "sizes": sizes, "type": type, "clip": True, "copy": "none", **options}


def listed():
    return [
        # one token of a serving loop: residual and norm before a map on 8-bit floats; nothing but latency
        _norm("norm_token_d4096", 1, 4096, "bf16", codes="e4m3"),
        # the training step's batch, 128 words of LDPC(256,128), 384 tokens each, in front of a ternary map
        _norm("norm_ldpc256_128_int8", 49152, 128, "fp32", codes="int8"),
        # an odd width, rows of a wider buffer, the normalised row itself in 16 bits
        _norm("norm_odd_d1111", 3001, 1111, "fp16", pad=5, residual=False, y=True),
        # a large batch of wide rows with a scale for each 128 columns
        _norm("norm_bulk_d8192", 16384, 8192, "bf16", codes="e4m3", group=128),
        # the gradient at the shape of 128 words of BCH(31,16), 46 tokens each
        _norm_grad("norm_grad_bch31_16", 5888, 32, "fp32"),
        # an odd width between a small batch's rows
        _norm_grad("norm_grad_odd_d5003", 777, 5003, "fp16", residual=False),
        # a large training batch
        _norm_grad("norm_grad_bulk_d4096", 16384, 4096, "bf16"),
        # the gradients of the short code's model: 21 tensors, 83 thousand values
        _clip("clip_bch31_16", "trainer 31 15 32 6", "fp32"),
        # several hundred tensors from one value to some ten thousand, in 16 bits
        _clip("clip_many_bf16", "many 400 6000000 3", "bf16"),
        # the norm alone of a large model's gradients
        _clip("norm_of_grads_large", "many 300 250000000 4", "fp32", write=False),
        # the update of the large code's model: 21 tensors, 2 million values
        _adam("adam_ldpc256_128", "trainer 256 128 128 10", "fp32"),
        # a large model's update from 16-bit gradients, with the 16-bit copy that its forward pass reads
        _adam("adam_large", "many 150 120000000 5", "bf16", copy="bf16"),
    ]


def _log_between(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    do = rng.choice(("norm", "norm", "norm_grad", "clip", "adam"))
    type = rng.choice(("fp32", "bf16", "fp16"))
    if do in ("norm", "norm_grad"):
        d = rng.choice((32, 64, 128, 512, 2048, 4096, 8192)) if rng.random() < 0.4 else _log_between(rng, 16, 16384)
        rows = _log_between(rng, 1, max(2, min(100000, 60000000 // d)))
        options = {"residual": rng.random() < 0.7, "pad": rng.choice((0, 0, 0, 3, 8)), "eps": rng.choice((1e-5, 1e-6))}
        if do == "norm_grad":
            case = _norm_grad("", rows, d, type, **options)
        else:
            codes = rng.choice(("none", "int8", "e4m3"))
            group = rng.choice((0, 0, 32, 64, 128)) if codes != "none" else 0
            case = _norm("", rows, d, type, codes=codes, group=group, y=codes == "none" or rng.random() < 0.2, **options)
    else:
        if rng.random() < 0.3:
            n, m, d, layers = rng.choice(((31, 15, 32, 6), (128, 64, 64, 6), (256, 128, 128, 10), (1024, 512, 128, 10)))
            sizes = "trainer %d %d %d %d" % (n, m, d, max(1, layers - rng.randrange(3)))
        else:
            count = _log_between(rng, 1, 500)
            sizes = "many %d %d %d" % (count, max(count, _log_between(rng, 1000, 60000000)), rng.randrange(1000))
        if do == "clip":
            case = _clip("", sizes, type, write=rng.random() < 0.7)
        else:
            case = _adam("", sizes, type, clip=rng.random() < 0.8, copy=rng.choice(("none", "none", "bf16", "fp16")))
    del case["name"]
    return case


def _sizes(text):
    """The tensors' numbers of values: "trainer n m d layers", the parameters of the training step in the order of the
    trainer's structs, or "many tensors total spread", sizes spread over four orders of magnitude."""
    kind, *v = text.split()
    v = [int(x) for x in v]
    if kind == "trainer":
        n, m, d, layers = v
        tokens = n + m
        return ([tokens * d] + [layers * d * d] * 4 + [layers * 4 * d * d] * 2 + [layers * 6] + [layers * d] * 4
                + [layers * 4 * d, layers * d] + [layers * d] * 4 + [d, 1, tokens * n, n])
    count, total, spread = v
    rng = random.Random(spread)
    share = [10.0 ** rng.uniform(-4, 0) for _ in range(count)]
    each = [max(1, int(s / sum(share) * total)) for s in share]
    each[0] = max(1, each[0] + total - sum(each))
    return each


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(case, g, scale=1.0):
    """A batch of rows of the case's type, `pad` columns apart, with a few outlying columns as hidden states have them."""
    wide = torch.randn(case["rows"], case["d"] + case["pad"], device="cuda", generator=g)
    wide[:, :: max(1, case["d"] // 5)] *= 8
    return wide.mul_(scale).to(TYPES[case["type"]])[:, : case["d"]]


def _views(flat, sizes):
    return list(flat.split(sizes))


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["do"] in ("norm", "norm_grad"):
        back = case["do"] == "norm_grad"
        state["x"] = _rows(case, g)
        state["res"] = _rows(case, g, 1e-3 if back else 1.0) if case["residual"] else None   # back: the residual path's gradient
        state["gain"] = 1 + 0.2 * torch.randn(case["d"], device="cuda", generator=g)
        if back:
            state["dy"] = _rows(case, g, 1e-3)
        return state
    sizes = _sizes(case["sizes"])
    n = sum(sizes)
    grad = torch.randn(n, device="cuda", generator=g).mul_(1e-2).to(TYPES[case["type"]])
    state.update(grad=grad, max_norm=0.5 * 1e-2 * math.sqrt(n))   # half of what the norm will be
    if case["do"] == "clip":
        if case["write"]:
            state["out"] = torch.empty_like(grad)
        if own:   # the lists of a model's gradients, which a program keeps as it keeps the model
            import paper_2410_05911_amd as aecct
            state["grads"] = aecct.TensorList(_views(grad, sizes))
            state["outs"] = aecct.TensorList(_views(state["out"], sizes)) if case["write"] else None
        return state
    # an update in the middle of a run
    state["param"] = torch.randn(n, device="cuda", generator=g).mul_(0.1)
    state["m"] = torch.randn(n, device="cuda", generator=g).mul_(2e-3)
    state["v"] = torch.rand(n, device="cuda", generator=g).mul_(1e-4)
    state["step"] = torch.full((1,), 1000 + seed % 100, dtype=torch.int64, device="cuda")
    state["copy"] = torch.empty(n, dtype=TYPES[case["copy"]], device="cuda") if case["copy"] != "none" else None
    if own:   # the optimiser and the list of the model's gradients
        import paper_2410_05911_amd as aecct
        state["grads"] = aecct.TensorList(_views(grad, sizes))
        state["adam"] = aecct.Adam(
            _views(state["param"], sizes), lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
            max_norm=state["max_norm"] if case["clip"] else None, m=_views(state["m"], sizes), v=_views(state["v"], sizes),
            step=state["step"], copies=None if state["copy"] is None else _views(state["copy"], sizes))
    return state


# ---------------------------------------------------------------------------------------------------------- run
def run(state):
    case = state["case"]
    if own:
        import paper_2410_05911_amd as aecct
        return {"norm": _own_norm, "norm_grad": _own_norm_grad, "clip": _own_clip, "adam": _own_adam}[case["do"]](aecct, case, state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip, "adam": _plain_adam}[case["do"]](case, state)


def _said(case, y, h, codes, alpha):
    """The outputs asked for.  int8 codes are handed on as the values they stand for; those of an 8-bit float are values,
    in units of alpha / 448."""
    out = {}
    if y is not None:
        out["y"] = y
    if h is not None:
        out["h"] = h
    if codes is not None:
        out["codes"], out["alpha"] = codes, alpha
    return out


def _own_norm(aecct, case, s):
    kind = CODES[case["codes"]][0] if case["codes"] != "none" else None
    y, h, codes, alpha = aecct.rms_norm(s["x"], s["gain"], s["res"], case["eps"], with_y=case["y"], code_type=kind,
                                        group=case["group"])
    if case["codes"] == "int8":
        value = torch.empty(codes.shape, dtype=torch.bfloat16, device="cuda")
        scale = alpha * (1 / 127.0)
        if case["group"] and case["d"] % case["group"]:
            torch.mul(codes, scale.repeat_interleave(case["group"], 1)[:, : case["d"]], out=value)
        else:
            torch.mul(codes.view(*alpha.shape, -1), scale[..., None], out=value.view(*alpha.shape, -1))
        codes = value
    return _said(case, y, h, codes, alpha)


def _own_norm_grad(aecct, case, s):
    dh, dgain = aecct.rms_norm_grad(s["x"], s["dy"], s["gain"], s["res"], case["eps"])
    return {"dh": dh, "dgain": dgain}


def _own_clip(aecct, case, s):
    if not case["write"]:
        return {"norm": aecct.grad_norm(s["grads"])}
    norm = aecct.grad_clip(s["grads"], s["max_norm"], out=s["outs"])
    return {"norm": norm, "out": s["out"]}


def _own_adam(aecct, case, s):
    norm = s["adam"].step(s["grads"])
    return {k: v for k, v in (("param", s["param"]), ("m", s["m"]), ("v", s["v"]), ("step", s["step"]), ("copy", s["copy"]),
                              ("norm", norm)) if v is not None}


def _plain_norm(case, s):
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + case["eps"]) * s["gain"]
    codes = alpha = None
    if case["codes"] != "none":
        kind, most = CODES[case["codes"]]
        group = case["group"] or case["d"]
        short = -case["d"] % group
        z = torch.nn.functional.pad(y, (0, short)).view(case["rows"], -1, group)
        alpha = z.abs().amax(-1)
        z = z * (most / alpha)[..., None]
        if case["codes"] == "int8":
            codes = (z.round() * (alpha * (1 / most))[..., None]).view(case["rows"], -1)[:, : case["d"]].to(torch.bfloat16)
        else:
            codes = z.view(case["rows"], -1)[:, : case["d"]].to(kind)
        alpha = alpha if case["group"] else alpha[:, 0]
    t = TYPES[case["type"]]
    return _said(case, y.to(t) if case["y"] else None, h.to(t) if s["res"] is not None else None, codes, alpha)


def _plain_norm_grad(case, s):
    h, dy = s["x"].float(), s["dy"].float()
    rho = torch.rsqrt(h.square().mean(-1, keepdim=True) + case["eps"])
    xh = h * rho
    dgain = (dy * xh).sum(0)
    dyg = dy * s["gain"]
    dh = rho * (dyg - xh * (dyg * xh).mean(-1, keepdim=True))
    if s["res"] is not None:
        dh = dh + s["res"].float()
    return {"dh": dh.to(TYPES[case["type"]]), "dgain": dgain}


def _plain_clip(case, s):
    g = s["grad"].float()
    norm = g.square().sum().sqrt().view(1)
    if not case["write"]:
        return {"norm": norm}
    s["out"].copy_(g * (s["max_norm"] / norm).clamp(max=1.0))
    return {"norm": norm, "out": s["out"]}


def _plain_adam(case, s):
    g = s["grad"].float()
    out = {}
    if case["clip"]:
        out["norm"] = g.square().sum().sqrt().view(1)
        g = g * (s["max_norm"] / out["norm"]).clamp(max=1.0)
    s["step"] += 1
    t = s["step"].double()
    size = (LR / (1 - BETA1 ** t)).float()
    root = (1 / (1 - BETA2 ** t).sqrt()).float()
    s["m"].mul_(BETA1).add_(g * (1 - BETA1))
    s["v"].mul_(BETA2).add_(g.square() * (1 - BETA2))
    s["param"].mul_(1 - LR * DECAY).sub_(size * s["m"] / (s["v"].sqrt() * root + ADAM_EPS))
    out.update(param=s["param"], m=s["m"], v=s["v"], step=s["step"])
    if s["copy"] is not None:
        s["copy"].copy_(s["param"])
        out["copy"] = s["copy"]
    return out


# ---------------------------------------------------------------------------------------------------- work, exact
def work(case):
    size = SIZE[case["type"]]
    if case["do"] == "norm":
        n = case["rows"] * case["d"]
        values = 1 + 2 * case["residual"] + case["y"]
        scales = case["rows"] * (-(-case["d"] // case["group"]) if case["group"] else 1)
        coded = n + 4 * scales if case["codes"] != "none" else 0
        return {"bytes": values * n * size + 4 * case["d"] + coded, "flops": n * (4 + case["residual"] + 3 * bool(coded))}
    if case["do"] == "norm_grad":
        n = case["rows"] * case["d"]
        return {"bytes": (3 + case["residual"]) * n * size + 8 * case["d"], "flops": 12 * n}
    n = sum(_sizes(case["sizes"]))
    if case["do"] == "clip":
        return {"bytes": n * size * (1 + case["write"]), "flops": n * (2 + case["write"])}
    copied = SIZE[case["copy"]] if case["copy"] != "none" else 0
    return {"bytes": n * (size + 24 + copied), "flops": n * (14 + 3 * case["clip"])}


def exact(case, seed):
    """The definitions in 64 bits on the same inputs."""
    s = prepare(case, seed)
    if case["do"] == "norm":
        h = s["x"].double()
        if s["res"] is not None:
            h += s["res"].double()
        ms = torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["d"]
        y = s["gain"].double() * h / torch.sqrt(ms + case["eps"])
        codes = alpha = None
        if case["codes"] != "none":
            kind, most = CODES[case["codes"]]
            group = case["group"] or case["d"]
            parts = y.abs().split(group, 1)
            alpha = torch.stack([p.max(1).values for p in parts], 1)
            at = torch.arange(case["d"], device="cuda") // group
            scale = alpha[:, at] / most
            codes = torch.round(y / scale) * scale if case["codes"] == "int8" else (y / scale).to(kind)
            alpha = alpha if case["group"] else alpha[:, 0]
        return _said(case, y if case["y"] else None, h if s["res"] is not None else None, codes, alpha)
    if case["do"] == "norm_grad":
        h, dy, gain = s["x"].double(), s["dy"].double(), s["gain"].double()
        ms = (h * h).sum(1, keepdim=True) / case["d"] + case["eps"]
        along = (dy * gain * h).sum(1, keepdim=True) / (case["d"] * ms)
        dh = (dy * gain - along * h) / torch.sqrt(ms)
        if s["res"] is not None:
            dh += s["res"].double()
        return {"dh": dh, "dgain": (dy * h / torch.sqrt(ms)).sum(0)}
    g = s["grad"].double()
    norm = torch.linalg.vector_norm(g).view(1)
    if case["do"] == "clip":
        return {"norm": norm, "out": g * min(1.0, s["max_norm"] / norm.item())} if case["write"] else {"norm": norm}
    if case["clip"]:
        g *= min(1.0, s["max_norm"] / norm.item())
    t = s["step"].item() + 1
    m = BETA1 * s["m"].double() + (1 - BETA1) * g
    v = BETA2 * s["v"].double() + (1 - BETA2) * g * g
    denominator = torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS
    param = s["param"].double() * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** t)) / denominator
    out = {"param": param, "m": m, "v": v, "step": s["step"] + 1}
    if s["copy"] is not None:
        out["copy"] = param
    if case["clip"]:
        out["norm"] = norm
    return out
