"""Timed cases of the operators that make residual blocks and a classifier out
of layers: linear maps with an activation and a residual, norms around a gated
residual sum, log probabilities of labels with entropy and top alternatives,
and their gradients.

A case is one call that a program makes between two layers or after the last.
``run`` evaluates it with elementary torch operations in 32 bits (64 for sums
over rows and for statistics of long rows), or, with ``own`` set, through this
package's entry points.  ``exact`` evaluates the same inputs in 64 bits.
Inputs are drawn from the seed with torch and the standard library alone.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPE = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 2), "f16": (torch.float16, 2)}
EPS = 1e-5


def listed():
    return [
        # three asked-for vertices through a perceptron's first map: the
        # smallest serving call
        dict(name="linear-serve-3", kind="linear", m=3, k=1024, n=1024, act="gelu", res=True, pre=False, dtype="bf16",
             out="bf16", pad=0),
        # hidden width to hidden width in fp32, with the block's input added
        dict(name="linear-hidden-200k", kind="linear", m=200_003, k=256, n=256, act="relu", res=True, pre=False,
             dtype="f32", out="f32", pad=0),
        # a wide perceptron's first map over many rows, kept for its gradient
        dict(name="linear-wide-16k", kind="linear", m=16_384, k=2048, n=8192, act="silu", res=False, pre=True,
             dtype="bf16", out="bf16", pad=0),
        # every gradient of a mini-batch's map, widths that fit no tile
        dict(name="linear-grad-33k", kind="linear_grad", m=33_001, k=1000, n=1536, act="gelu", dtype="bf16",
             out="bf16", pad=0),
        # the same, square and large
        dict(name="linear-grad-wide-16k", kind="linear_grad", m=16_384, k=4096, n=4096, act="silu", dtype="f16",
             out="f16", pad=0),
        # a few rows between two blocks, both norms, a gate for each channel
        dict(name="resnorm-serve-5", kind="resnorm", m=5, d=4096, post="rms", pre="rms", gate="channel", segs=0,
             dtype="bf16", stream="bf16", pad=0),
        # every vertex of a graph between two layers
        dict(name="resnorm-vertices-1m", kind="resnorm", m=1_000_000, d=256, post="none", pre="layer",
             gate="channel", segs=0, dtype="bf16", stream="bf16", pad=0),
        # gradient over a batch of ragged graphs, a gate for each of them
        dict(name="resnorm-grad-batch-300k", kind="resnorm_grad", m=300_001, d=128, post="layer", pre="layer",
             gate="segment", segs=9_000, dtype="f16", stream="f16", pad=0),
        # gradient of wide rows on a residual stream of 32 bits
        dict(name="resnorm-grad-wide-33k", kind="resnorm_grad", m=33_000, d=4096, post="rms", pre="rms",
             gate="channel", segs=0, dtype="bf16", stream="f32", pad=0),
        # the answer for a few rows out of a large vocabulary
        dict(name="labels-serve-5", kind="labels", m=5, c=128_003, top=20, dtype="bf16", masked=True, pad=0),
        # the classes of every vertex, with alternatives
        dict(name="labels-vertices-1m", kind="labels", m=1_000_000, c=172, top=5, dtype="f32", masked=False, pad=0),
        # gradient of a training batch's labels and of their entropies
        dict(name="labels-grad-8k", kind="labels_grad", m=8_192, c=32_003, dtype="bf16", masked=True, entropy=True,
             pad=0),
    ]


def _spread(rng, lo, hi):
    """A whole number, uniform in its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above that costs no more than the largest of them."""
    case = _drawn(rng)
    # fp32 products run at about an eighth of the 16-bit ones' rate
    while work(case)["bytes"] > 1.6e9 or work(case)["flops"] > (1.3e11 if case["dtype"] == "f32" else 1.0e12):
        case["m"] = case["m"] * 2 // 3
        if case.get("segs"):
            case["segs"] = min(case["segs"], case["m"])
    return case


def _drawn(rng):
    kind = rng.choice(["linear", "linear_grad", "resnorm", "resnorm_grad", "labels", "labels_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if kind in ("linear", "linear_grad"):
        k, n = (rng.choice([64, 8, 1]) for _ in range(2))
        k, n = max(1, _spread(rng, 64, 4096) // k) * k, max(1, _spread(rng, 47, 4096) // n) * n
        case = dict(kind=kind, m=_spread(rng, 1, 200_000), k=k, n=n,
                    act=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), dtype=dtype, out=dtype, pad=pad)
        if kind == "linear":
            case.update(res=rng.random() < 0.5, pre=rng.random() < 0.3, out=rng.choice([dtype, dtype, "f32"]))
        return case
    if kind in ("resnorm", "resnorm_grad"):
        m = _spread(rng, 1, 500_000)
        gate = rng.choice(["none", "channel", "segment"])
        post, pre = rng.choice(["none", "layer", "rms"]), rng.choice(["layer", "rms", "rms", "none"])
        return dict(kind=kind, m=m, d=_spread(rng, 47, 8192), post=post, pre=pre, gate=gate,
                    segs=_spread(rng, 1, max(1, m // 20)) if gate == "segment" else 0, dtype=dtype,
                    stream=rng.choice([dtype, dtype, "f32"]), pad=pad)
    case = dict(kind=kind, m=_spread(rng, 1, 500_000), c=_spread(rng, 2, 200_000), dtype=dtype,
                masked=rng.random() < 0.5, pad=pad)
    if kind == "labels":
        case["top"] = min(case["c"], rng.choice([0, 1, 5, 20, 64]))
    else:
        case["entropy"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs --

def _offsets(m, parts, seed):
    """parts + 1 offsets over m rows: uneven sizes, some of them empty."""
    rng = random.Random(seed * 7919 + parts)
    if parts == 1:
        return [0, m]
    sizes = [0.0 if parts > 2 and rng.random() < 0.05 else rng.expovariate(1.0) + 0.05 for _ in range(parts)]
    if not sum(sizes):
        sizes[0] = 1.0
    total, off, at = sum(sizes), [0], 0.0
    for s in sizes:
        at += s
        off.append(min(m, int(m * at / total)))
    off[-1] = m
    return off


def _rows(values, dtype, pad):
    """The values as rows of dtype that lie pad values further apart."""
    m, d = values.shape
    if not pad:
        return values.to(dtype)
    wide = torch.zeros(m, d + pad, dtype=dtype, device="cuda")
    wide[:, :d] = values
    return wide[:, :d]


def _normal(shape, gen, scale=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, scale, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, kind, m, pad = DTYPE[case["dtype"]][0], case["kind"], case["m"], case["pad"]
    s = dict(case, in_dtype=dtype)
    if kind in ("linear", "linear_grad"):
        k, n = case["k"], case["n"]
        s["out_dtype"] = DTYPE[case["out"]][0]
        s["x"] = _rows(_normal((m, k), gen), dtype, pad)
        s["weight"] = _normal((k, n), gen, 1.0 / math.sqrt(k)).to(dtype)
        s["bias"] = _normal((n,), gen, 0.5)
        if kind == "linear":
            s["residual"] = _rows(_normal((m, n), gen), s["out_dtype"], pad) if case["res"] else None
        else:
            s["z"] = (torch.matmul(s["x"].float(), s["weight"].float()) + s["bias"]).to(dtype)
            s["grad"] = _rows(_normal((m, n), gen), dtype, pad)
        return s
    if kind in ("resnorm", "resnorm_grad"):
        d, rows = case["d"], m
        stream = DTYPE[case["stream"]][0]
        s["x"] = _rows(_normal((m, d), gen, 2.0) + _normal((d,), gen), stream, pad)
        s["f"] = _rows(_normal((m, d), gen) + _normal((d,), gen, 0.3), dtype, pad)
        s["scale"] = 0.7
        s["off"] = s["gate_at"] = s["gate_rows"] = None
        if case["gate"] == "channel":
            s["gate_rows"] = 0.5 + _normal((d,), gen, 0.2)
        elif case["gate"] == "segment":
            host = _offsets(m, case["segs"], seed)
            s["off"] = torch.tensor(host, dtype=torch.int64, device="cuda")
            s["gate_rows"] = 0.5 + _normal((case["segs"], d), gen, 0.2)
        for name in ("post", "pre"):
            s[name + "_w"] = 1.0 + _normal((d,), gen, 0.2) if case[name] != "none" else None
            s[name + "_b"] = _normal((d,), gen, 0.2) if case[name] == "layer" else None
        if kind == "resnorm_grad":
            y, _, s["stats"] = _resnorm(s)
            s["y"] = _rows(y, stream, pad)
            s["grad_y"] = _rows(_normal((m, d), gen), stream, pad)
            s["grad_h"] = _rows(_normal((m, d), gen), dtype, pad) if case["pre"] != "none" else None
        return s
    c = case["c"]
    logits = _normal((m, c), gen, 2.0) + _normal((c,), gen)
    s["labels"] = torch.randint(0, c, (m,), device="cuda", generator=gen, dtype=torch.int32)
    if case["masked"]:  # classes that cannot be the answer; rows without any; labels that pad a batch
        off = torch.rand(c, device="cuda", generator=gen) < 0.02
        logits[:, off] = -math.inf
        if m > 1:
            logits[torch.rand(m, device="cuda", generator=gen) < 0.01] = -math.inf
        s["labels"][torch.rand(m, device="cuda", generator=gen) < 1.0 / 64] = -1
    s["x"] = _rows(logits, dtype, pad)
    s["scale"] = 0.8
    if kind == "labels_grad":
        del logits
        _, s["stats"], s["entropies"] = _log_probs(s)[:3]
        s["grad_logp"] = _normal((m,), gen) - 1.0
        s["grad_entropy"] = _normal((m,), gen) if case["entropy"] else None
    return s


# ------------------------------------------------------------- plain forms --

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return q * (1.0 + z * (1.0 - q))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2.0 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * a * (1.0 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _linear(s):
    z = torch.matmul(s["x"].float(), s["weight"].float()) + s["bias"]
    y = _act(z, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(s["out_dtype"]), z.to(s["in_dtype"])) if s["pre"] else y.to(s["out_dtype"])


def _linear_grad(s):
    dz = s["grad"].float() * _slope(s["z"].float(), s["act"])
    dx = torch.matmul(dz, s["weight"].float().t())
    dw = torch.matmul(s["x"].float().t(), dz)
    return dx.to(s["in_dtype"]), dw.to(s["out_dtype"]), dz.sum(0, dtype=torch.float64).float()


def _moments(v, kind):
    """Mean and reciprocal deviation of every row, [m][1]; an RMS norm's mean
    is 0.  Sums of 64 bits."""
    mean = v.mean(1, keepdim=True, dtype=torch.float64).float() if kind == "layer" else v.new_zeros(v.shape[0], 1)
    dev = v - mean
    var = (dev * dev).mean(1, keepdim=True, dtype=torch.float64)
    return mean, (1.0 / torch.sqrt(var + EPS)).float()


def _segment_of(s):
    count = s["off"][1:] - s["off"][:-1]
    return torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count, output_size=s["m"])


def _gate(s):
    """What each value of the block's output is multiplied by."""
    if s["gate_rows"] is None:
        return torch.full((1, 1), s["scale"], device="cuda")
    if s["off"] is None:
        return (s["scale"] * s["gate_rows"]).unsqueeze(0)
    return s["scale"] * s["gate_rows"][_segment_of(s)]


def _affine(hat, w, b):
    hat = hat * w
    return hat if b is None else hat + b


def _resnorm(s):
    """The residual stream, its norm and the statistics, unrounded."""
    m = s["m"]
    p, y = s["f"].float(), s["x"].float()
    stats = torch.zeros(m, 4, device="cuda")
    if s["post_w"] is not None:
        mean, rstd = _moments(p, s["post"])
        stats[:, 0:1], stats[:, 1:2] = mean, rstd
        p = _affine((p - mean) * rstd, s["post_w"], s["post_b"])
    y = y + _gate(s) * p
    h = None
    if s["pre_w"] is not None:
        mean, rstd = _moments(y, s["pre"])
        stats[:, 2:3], stats[:, 3:4] = mean, rstd
        h = _affine((y - mean) * rstd, s["pre_w"], s["pre_b"])
    return y, h, stats


def _norm_back(g, hat, rstd, kind):
    """Gradient of a row's norm from g = d(loss)/d(hat)."""
    back = g - hat * (g * hat).mean(1, keepdim=True)
    if kind == "layer":
        back = back - g.mean(1, keepdim=True)
    return back * rstd


def _column_sums(v):
    return v.sum(0, dtype=torch.float64).float()


def _resnorm_grad(s):
    dw = dict.fromkeys(("gate", "post_w", "post_b", "pre_w", "pre_b"))
    dy = s["grad_y"].float()
    if s["pre_w"] is not None:
        rstd = s["stats"][:, 3:4]
        hat = (s["y"].float() - s["stats"][:, 2:3]) * rstd
        g = s["grad_h"].float()
        dw["pre_w"] = _column_sums(g * hat)
        if s["pre_b"] is not None:
            dw["pre_b"] = _column_sums(g)
        dy = dy + _norm_back(g * s["pre_w"], hat, rstd, s["pre"])
    p = s["f"].float()
    if s["post_w"] is not None:
        rstd = s["stats"][:, 1:2]
        hat = (p - s["stats"][:, 0:1]) * rstd
        p = _affine(hat, s["post_w"], s["post_b"])
    dp = _gate(s) * dy
    if s["gate_rows"] is not None:
        each = s["scale"] * p * dy
        if s["off"] is None:
            dw["gate"] = _column_sums(each)
        else:
            total = torch.zeros(s["gate_rows"].shape, dtype=torch.float64, device="cuda")
            dw["gate"] = total.index_add_(0, _segment_of(s), each.double()).float()
    df = dp
    if s["post_w"] is not None:
        dw["post_w"] = _column_sums(dp * hat)
        if s["post_b"] is not None:
            dw["post_b"] = _column_sums(dp)
        df = _norm_back(dp * s["post_w"], hat, rstd, s["post"])
    return (dy.to(s["grad_y"].dtype), df.to(s["in_dtype"]), *(v for v in dw.values() if v is not None))


def _log_probs(s):
    """Log probabilities of the labels, (largest, log of the sum) of every
    row, entropies, and all classes' log probabilities."""
    l = s["x"].float() * s["scale"]
    m, c = l.shape
    most = l.max(1, keepdim=True).values
    none = most == -math.inf
    d = torch.where(none, torch.full_like(l, -math.inf), l - most)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_sum = torch.where(none, 0.0, torch.log(total))
    spread = torch.where(e > 0, -d, 0.0).mul_(e).sum(1, keepdim=True)
    entropy = torch.where(none, 0.0, log_sum + spread / total)
    logp = d - log_sum
    at = s["labels"].long().unsqueeze(1)
    of_label = torch.where(at >= 0, logp.gather(1, at.clamp(min=0)), 0.0)
    return of_label.squeeze(1), torch.cat([most, log_sum], 1), entropy.squeeze(1), logp


def _top(s, logp):
    """The classes of the largest logits and their log probabilities, one at
    a time; the lowest of equal ones first, -1 where only masked ones are
    left."""
    left = s["x"].float()
    m, c = left.shape
    index = torch.arange(c, device="cuda", dtype=torch.int32).unsqueeze(0)
    ids, values = [], []
    for _ in range(s["top"]):
        best = left.max(1, keepdim=True).values
        at = torch.where(left == best, index, c).min(1, keepdim=True).values
        some = best > -math.inf
        values.append(torch.where(some, logp.gather(1, at.long()), -math.inf))
        ids.append(torch.where(some, at, -1))
        left = left.masked_fill(index == at, -math.inf)
    return torch.cat(values, 1), torch.cat(ids, 1)


def _labels_grad(s):
    l = s["x"].float() * s["scale"]
    most, log_sum = s["stats"][:, 0:1], s["stats"][:, 1:2]
    known = s["labels"] >= 0
    g = torch.where(known, s["grad_logp"], 0.0).unsqueeze(1)
    logp = (l - most) - log_sum
    p = torch.exp(logp)
    dl = -g * p
    dl.scatter_add_(1, s["labels"].long().clamp(min=0).unsqueeze(1), g)
    if s["grad_entropy"] is not None:
        spread = torch.where(p > 0, logp + s["entropies"].unsqueeze(1), 0.0)
        dl = dl - s["grad_entropy"].unsqueeze(1) * p * spread
    return torch.where(most == -math.inf, 0.0, dl * s["scale"]).to(s["in_dtype"])


def _plain(s):
    kind = s["kind"]
    if kind == "linear":
        return _linear(s)
    if kind == "linear_grad":
        return _linear_grad(s)
    if kind == "resnorm":
        y, h, _ = _resnorm(s)
        y = y.to(s["x"].dtype)
        return y if h is None else (y, h.to(s["in_dtype"]))
    if kind == "resnorm_grad":
        return _resnorm_grad(s)
    if kind == "labels":
        of_label, _, entropy, logp = _log_probs(s)
        return (of_label, entropy, *_top(s, logp)) if s["top"] else (of_label, entropy)
    return _labels_grad(s)


def _norm_args(s, name):
    if s[name + "_w"] is None:
        return None
    return dict(kind=s[name], weight=s[name + "_w"], bias=s[name + "_b"], eps=EPS)


def run(s):
    if not own:
        return _plain(s)
    import paper_2607_17374_amd as T
    kind = s["kind"]
    if kind == "linear":
        return T.linear(s["x"], s["weight"], s["bias"], s["residual"], act=s["act"], out_dtype=s["out_dtype"],
                        pre=s["pre"])
    if kind == "linear_grad":
        return T.linear_grad(s["grad"], s["x"], s["weight"], s["z"], act=s["act"], weight_dtype=s["out_dtype"])
    if kind == "resnorm":
        y, h = T.residual_norm(s["x"], s["f"], scale=s["scale"], gate=s["gate_rows"], off=s["off"],
                               post=_norm_args(s, "post"), pre=_norm_args(s, "pre"))
        return y if h is None else (y, h)
    if kind == "resnorm_grad":
        d = T.residual_norm_grad(s["grad_y"], s["grad_h"], s["y"], s["f"], s["stats"], scale=s["scale"],
                                 gate=s["gate_rows"], off=s["off"], post=_norm_args(s, "post"),
                                 pre=_norm_args(s, "pre"))
        return tuple(v for v in d if v is not None)
    if kind == "labels":
        r = T.label_log_probs(s["x"], s["labels"], s["scale"], top=s["top"], entropy=True)
        return (r.logp, r.entropy, r.top_logp, r.top_ids) if s["top"] else (r.logp, r.entropy)
    return T.label_log_probs_grad(s["x"], s["labels"], s["stats"], s["grad_logp"], s["scale"],
                                  entropy=s["entropies"] if s["entropy"] else None, grad_entropy=s["grad_entropy"])


# ----------------------------------------------------------- cost and truth --

def work(case):
    kind, m, si = case["kind"], float(case["m"]), DTYPE[case["dtype"]][1]
    if kind in ("linear", "linear_grad"):
        k, n, so = case["k"], case["n"], DTYPE[case["out"]][1]
        if kind == "linear":
            return {"bytes": m * k * si + k * n * si + 4.0 * n + m * n * so * (2 if case["res"] else 1)
                    + (m * n * si if case["pre"] else 0.0), "flops": 2.0 * m * k * n}
        return {"bytes": 2 * m * k * si + m * n * si * (1 if case["act"] == "none" else 2) + k * n * (si + so) + 4.0 * n,
                "flops": 4.0 * m * k * n}
    if kind in ("resnorm", "resnorm_grad"):
        d, ss = float(case["d"]), DTYPE[case["stream"]][1]
        post, pre = (case[v] != "none" for v in ("post", "pre"))
        rows = {"none": 0, "channel": 1, "segment": case["segs"]}[case["gate"]]
        sets = (rows + post + pre + (case["post"] == "layer") + (case["pre"] == "layer")) * 4.0 * d
        if kind == "resnorm":
            return {"bytes": m * d * (2 * ss + si * (2 if pre else 1)) + sets, "flops": m * d * (4 + 8 * (post + pre))}
        return {"bytes": m * d * (2 * ss + 2 * si + (ss + si if pre else 0)) + 16.0 * m + 2 * sets,
                "flops": m * d * (6 + 14 * (post + pre))}
    c = float(case["c"])
    if kind == "labels":
        return {"bytes": m * c * si + m * (12.0 + 8.0 * case["top"]), "flops": 6.0 * m * c}
    return {"bytes": 2 * m * c * si + m * (12.0 + (8.0 if case["entropy"] else 4.0)), "flops": 8.0 * m * c}


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "linear_grad": _exact_linear_grad, "resnorm": _exact_resnorm,
            "resnorm_grad": _exact_resnorm_grad, "labels": _exact_labels, "labels_grad": _exact_labels_grad}[
                case["kind"]](s)


def _phi(z):
    """The normal distribution function."""
    return 0.5 * torch.erfc(-z / math.sqrt(2.0))


def _exact_linear(s):
    z = s["x"].double() @ s["weight"].double()
    z += s["bias"].double()
    a = s["act"]
    if a == "relu":
        y = z.clamp(min=0)
    elif a == "silu":
        y = z * torch.sigmoid(z)
    elif a == "gelu":
        y = z * _phi(z)
    elif a == "gelu_tanh":
        y = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    else:
        y = z
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return (y, z) if s["pre"] else y


def _exact_linear_grad(s):
    z, g, a = s["z"].double(), s["grad"].double(), s["act"]
    if a == "relu":
        g = g * (z > 0)
    elif a == "silu":
        q = torch.sigmoid(z)
        g = g * (q + z * q * (1 - q))
    elif a == "gelu":
        g = g * (_phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    elif a == "gelu_tanh":
        b = 2 * math.sqrt(2 / math.pi)
        q = torch.sigmoid(b * (z + 0.044715 * z ** 3))
        g = g * (q + z * q * (1 - q) * b * (1 + 3 * 0.044715 * z ** 2))
    del z
    return g @ s["weight"].double().t().contiguous(), s["x"].double().t().contiguous() @ g, g.sum(0)


def _exact_norm(v, kind, w, b):
    mu = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    out = (v - mu) * (((v - mu) ** 2).mean(1, keepdim=True) + EPS) ** -0.5 * w.double()
    return out if b is None else out + b.double()


def _exact_gate(s):
    if s["gate_rows"] is None:
        return s["scale"]
    rows = s["gate_rows"].double() * s["scale"]
    if s["off"] is None:
        return rows
    return torch.repeat_interleave(rows, s["off"].diff(), dim=0)


def _exact_resnorm(s):
    p = s["f"].double()
    if s["post_w"] is not None:
        p = _exact_norm(p, s["post"], s["post_w"], s["post_b"])
    y = s["x"].double() + _exact_gate(s) * p
    if s["pre_w"] is None:
        return y
    return y, _exact_norm(y, s["pre"], s["pre_w"], s["pre_b"])


def _exact_resnorm_grad(s):
    """At the statistics the call is given; blocks of rows at a time, which
    keeps the memory of 64-bit intermediates small."""
    m, d = s["m"], s["d"]
    have = {v: s[v] is not None for v in ("gate_rows", "post_w", "post_b", "pre_w", "pre_b")}
    sums = {v: torch.zeros(s[v].shape, dtype=torch.float64, device="cuda") for v in have if have[v]}
    dx = torch.empty(m, d, dtype=torch.float64, device="cuda")
    df = torch.empty_like(dx)
    segment = None
    if s["off"] is not None:
        segment = torch.bucketize(torch.arange(m, device="cuda"), s["off"][1:], right=True)
    step = max(1, (1 << 25) // d)
    for b in range(0, m, step):
        e = slice(b, min(m, b + step))
        st = s["stats"][e].double()
        dy = s["grad_y"][e].double()
        if have["pre_w"]:
            hat = (s["y"][e].double() - st[:, 2:3]) * st[:, 3:4]
            g = s["grad_h"][e].double()
            sums["pre_w"] += (g * hat).sum(0)
            if have["pre_b"]:
                sums["pre_b"] += g.sum(0)
            g = g * s["pre_w"].double()
            centre = g.mean(1, keepdim=True) if s["pre"] == "layer" else 0.0
            dy = dy + st[:, 3:4] * (g - centre - hat * (g * hat).mean(1, keepdim=True))
        p = hat = s["f"][e].double()
        if have["post_w"]:
            hat = (p - st[:, 0:1]) * st[:, 1:2]
            p = hat * s["post_w"].double()
            if have["post_b"]:
                p = p + s["post_b"].double()
        g = dy * s["scale"]
        if have["gate_rows"]:
            if segment is None:
                sums["gate_rows"] += (g * p).sum(0)
                g = g * s["gate_rows"].double()
            else:
                sums["gate_rows"].index_add_(0, segment[e], g * p)
                g = g * s["gate_rows"].double()[segment[e]]
        if have["post_w"]:
            sums["post_w"] += (g * hat).sum(0)
            if have["post_b"]:
                sums["post_b"] += g.sum(0)
            g = g * s["post_w"].double()
            centre = g.mean(1, keepdim=True) if s["post"] == "layer" else 0.0
            g = st[:, 1:2] * (g - centre - hat * (g * hat).mean(1, keepdim=True))
        dx[e], df[e] = dy, g
    return (dx, df, *sums.values())


def _exact_labels(s):
    l = s["x"].double() * s["scale"]
    lse = torch.logsumexp(l, 1, keepdim=True)
    logp = torch.where(lse > -math.inf, l - lse, -math.inf)
    entropy = -torch.where(logp > -math.inf, logp, 0.0).mul_(torch.exp(logp)).sum(1)
    rows = torch.arange(s["m"], device="cuda")
    of_label = torch.where(s["labels"] < 0, 0.0, logp[rows, s["labels"].long().clamp(min=0)])
    if not s["top"]:
        return of_label, entropy
    return of_label, entropy, torch.topk(logp, s["top"], dim=1).values, None


def _exact_labels_grad(s):
    l = s["x"].double() * s["scale"]
    st = s["stats"].double()
    none = st[:, 0:1] == -math.inf
    logp = l.sub_(torch.where(none, 0.0, st[:, 0:1] + st[:, 1:2]))
    p = torch.exp(logp)
    known = s["labels"] >= 0
    g = torch.where(known, s["grad_logp"].double(), 0.0)
    d = p * -g.unsqueeze(1)
    if s["grad_entropy"] is not None:
        h = s["entropies"].double().unsqueeze(1)
        d -= s["grad_entropy"].double().unsqueeze(1) * p * torch.where(logp > -math.inf, logp + h, 0.0)
    rows = torch.arange(s["m"], device="cuda")
    d[rows, s["labels"].long().clamp(min=0)] += g
    return torch.where(none, 0.0, d * s["scale"])
