"""Performance cases of the operators beside the cached table: token embedding, root-mean-square norm, gradient clipping.

One case is one call of one operator, on inputs made from a seed on the GPU.  Where `own` is false `run` computes the
operator in its plain form (elementary torch operations in 32 bits, rounded once at the end), otherwise it makes the call
that a program makes of `DenseOps`.

Token ids are bounded-Zipf(`alpha`) over `rows` ids in a seeded order, as the click logs' are; with `pad` they come as
sequences of up to 128 tokens whose tails hold the padding id.  `types` of a case: the type of the rows, of the weights or
gradients, of the result.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn, "i8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "f8": 1, "i8": 1}
QMAX = {"f8": 448.0, "i8": 127.0}
EPS = 1e-6
MAX_NORM = 1.0
SEQ = 128
BYTES_MOST = 1_400_000_000       # of a drawn case


# ---- cases -----------------------------------------------------------------------------------------------------------
def _embed(name, kind, rows, dim, tokens, src, dst, ids="i64", alpha=1.05, scale=1.0, pad=False):
    c = dict(kind=kind, rows=rows, dim=dim, tokens=tokens, src=src, dst=dst, ids=ids, alpha=alpha, scale=scale, pad=pad)
    return {"name": name, **c} if name else c


def _norm(name, kind, tokens, dim, src, weight, dst, residual, group=0):
    c = dict(kind=kind, tokens=tokens, dim=dim, src=src, weight=weight, dst=dst, residual=residual, group=group)
    return {"name": name, **c} if name else c


def _clip(name, layers, width, inner, src, vector, factor):
    c = dict(kind="clip", layers=layers, width=width, inner=inner, src=src, vector=vector, factor=factor)
    return {"name": name, **c} if name else c


def listed():
    return [
        # serving, one new token of one sequence: latency
        _embed("embed_token", "embed_fwd", 100_000, 1024, 1, "bf16", "bf16", scale=32.0),
        # a prompt batch of 64 sequences of 128 tokens, wide rows
        _embed("embed_prompt", "embed_fwd", 131_072, 4096, 8192, "bf16", "bf16", scale=64.0, pad=True),
        # items of a click batch (16,384 samples, 26 columns) out of an f32 master table, in the model's type
        _embed("embed_items", "embed_fwd", 1_000_000, 64, 425_984, "f32", "bf16", ids="i32", scale=8.0),
        # the smallest training step: 1024 ids, 16 columns
        _embed("embed_grad_small", "embed_bwd", 100_000, 16, 1024, "f32", "f32", alpha=1.1),
        # the word table of a language model: the gradient is the size of the table, most rows zero
        _embed("embed_grad_words", "embed_bwd", 131_072, 2048, 16_384, "bf16", "f32", scale=45.25, pad=True),
        # a micro-batch added to the gradient of a large item table: popular rows have thousands of tokens
        _embed("embed_grad_add", "embed_add", 1_000_000, 128, 425_984, "bf16", "f32", alpha=1.2),
        # decoding, one token: residual added, 8-bit input of the next product with one scale
        _norm("norm_token", "norm_fwd", 1, 4096, "bf16", "bf16", "f8", True),
        # odd sizes: a head's norm, no residual, nothing in 8 bits
        _norm("norm_odd", "norm_fwd", 777, 1111, "f16", "f32", "f16", False),
        # a prompt batch, scales for groups of 128 columns
        _norm("norm_prompt", "norm_fwd", 8192, 8192, "bf16", "bf16", "f8", True, group=128),
        # the backward pass of a training step, with the gradient that comes along the residual path
        _norm("norm_grad", "norm_bwd", 16_384, 4096, "bf16", "f32", "f32", True),
        # a click model's small dense tower
        _clip("clip_tower", 4, 512, 256, "f32", "f32", 3.0),
        # a model of 48 layers (a few hundred tensors, matrices in 16 bits, vectors in 32)
        _clip("clip_model", 48, 1024, 4096, "bf16", "f32", 3.0),
    ]


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("embed_fwd", "embed_bwd", "embed_bwd", "embed_add", "norm_fwd", "norm_fwd", "norm_bwd", "clip"))
    half = rng.choice(("bf16", "f16"))
    if kind == "clip":
        width, layers = logu(16, 2048), logu(1, 64)
        inner = rng.choice((width, 4 * width, logu(16, 8192)))
        src = rng.choice(("f32", "bf16", "bf16", "f16"))
        layers = max(1, min(layers, BYTES_MOST // (2 * SIZE[src] * width * (width + 2 * inner))))
        return _clip(None, layers, width, inner, src, rng.choice(("f32", "same")), rng.choice((0.5, 3.0, 20.0)))
    if kind.startswith("embed"):
        dim = rng.choice((16, 64, 128, 256, 1024, 2048, 4096, logu(8, 8192), logu(8, 8192)))
        rows = max(64, min(logu(500, 4_000_000), BYTES_MOST // 5 // dim))
        src = rng.choice(("f32", "bf16", "bf16", half))
        dst = rng.choice((src, "f32", half)) if kind == "embed_fwd" else rng.choice(("f32", "f32", src))
        tokens = min(logu(1, 1_700_000), BYTES_MOST // 10 // dim)
        return _embed(None, kind, rows, dim, tokens, src, dst, rng.choice(("i64", "i64", "i32")), rng.choice((1.05, 1.1, 1.2)),
                      rng.choice((1.0, math.sqrt(dim))), rng.random() < 0.5)
    dim = rng.choice((64, 128, 256, 1024, 2048, 4096, 8192, logu(16, 16_384), logu(16, 16_384)))
    tokens = min(logu(1, 400_000), BYTES_MOST // 20 // dim)
    src = rng.choice(("f32", "bf16", "bf16", half))
    weight = rng.choice((src, "f32"))
    if kind == "norm_bwd":
        return _norm(None, kind, tokens, dim, src, weight, rng.choice((weight, "f32")), rng.random() < 0.7)
    dst = rng.choice((src, "f8", "f8", "i8"))
    return _norm(None, kind, tokens, dim, src, weight, dst, rng.random() < 0.7,
                 rng.choice((0, 64, 128)) if dst in QMAX else 0)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + part)
    return g


def _randn(shape, kind, g, spread=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * spread).to(TYPES[kind])


def _ids(case, g):
    n, rows, e = case["tokens"], case["rows"], 1.0 - case["alpha"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    k = ((1.0 + u * ((rows + 1.0) ** e - 1.0)) ** (1.0 / e)).floor().long().clamp_(1, rows) - 1
    order = torch.randperm(rows, generator=g, device="cuda")
    ids = order[k]
    if case["pad"]:
        most = torch.randint(SEQ // 2, SEQ + 1, (-(-n // SEQ),), generator=g, device="cuda")
        at = torch.arange(n, device="cuda")
        ids = torch.where(at % SEQ < most[at // SEQ], ids, 0)
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _shapes(case):
    w, f = case["width"], case["inner"]
    return [s for _ in range(case["layers"]) for s in ((w,), (w, w), (w, f), (f,), (f, w))]


def prepare(case, seed):
    g = _gen(seed, 1)
    kind, s = case["kind"], {"case": case}
    if kind == "clip":
        shapes, vec = _shapes(case), case["src"] if case["vector"] == "same" else case["vector"]
        n = sum(math.prod(x) for x in shapes)
        spread = case["factor"] * MAX_NORM / math.sqrt(n)        # the norm is about `factor` times the most it may be
        s["grads"] = [_randn(x, vec if len(x) == 1 else case["src"], g, spread) for x in shapes]
        # the clipped gradients go into one flat buffer of each type, which the optimizer reads
        s["flat"] = {t: torch.empty(sum(x.numel() for x in s["grads"] if x.dtype == t), dtype=t, device="cuda")
                     for t in dict.fromkeys(x.dtype for x in s["grads"])}
        at = {t: 0 for t in s["flat"]}
        s["out"] = []
        for x in s["grads"]:
            s["out"].append(s["flat"][x.dtype][at[x.dtype]:at[x.dtype] + x.numel()].view(x.shape))
            at[x.dtype] += x.numel()
        return s
    if kind.startswith("embed"):
        s["ids"] = _ids(case, g)
        if kind == "embed_fwd":
            s["table"] = _randn((case["rows"], case["dim"]), case["src"], g, 0.02)
        else:
            s["dout"] = _randn((case["tokens"], case["dim"]), case["src"], g)
        if kind == "embed_add":                                  # the gradient of the micro-batches before this one
            s["grad"] = _randn((case["rows"], case["dim"]), case["dst"], g)
        return s
    n, d = case["tokens"], case["dim"]
    wide = torch.ones(d, device="cuda")
    wide[::max(1, d // 8)] = 10.0                                # a few columns much larger than the rest
    s["weight"] = (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(TYPES[case["weight"]])
    x = (torch.randn((n, d), generator=g, device="cuda") * wide).to(TYPES[case["src"]])
    s["h" if kind == "norm_bwd" else "x"] = x
    s["residual"] = _randn((n, d), case["src"], g) if case["residual"] else None
    if kind == "norm_bwd":
        s["dy"] = _randn((n, d), case["src"], g)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
_handle = None


def _ops():
    """The handle that a program makes once and keeps."""
    global _handle
    if _handle is None:
        from paper_2208_05321_amd import DenseOps
        _handle = DenseOps()
    return _handle


def _pad(case):
    return 0 if case["pad"] else -1


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    c, ops = s["case"], _ops()
    kind = c["kind"]
    if kind == "embed_fwd":
        return ops.token_embed_fwd(s["table"], s["ids"], scale=c["scale"], out_dtype=TYPES[c["dst"]])
    if kind == "embed_bwd":
        return ops.token_embed_bwd(s["dout"], s["ids"], c["rows"], scale=c["scale"], padding_id=_pad(c), grad_dtype=TYPES[c["dst"]])
    if kind == "embed_add":
        return ops.token_embed_bwd(s["dout"], s["ids"], c["rows"], scale=c["scale"], padding_id=_pad(c), grad=s["grad"], accumulate=True)
    if kind == "norm_fwd":
        y, h, scales = ops.rms_norm_fwd(s["x"], s["weight"], residual=s["residual"], eps=EPS, out_dtype=TYPES[c["dst"]], group=c["group"])
        return _norm_outputs(c, y, h, scales)
    if kind == "norm_bwd":
        return ops.rms_norm_bwd(s["dy"], s["h"], s["weight"], grad_h=s["residual"], eps=EPS, grad_weight_dtype=TYPES[c["dst"]])
    norm = ops.grad_norm_clip(s["grads"], MAX_NORM, out=s["out"])
    return [norm, *s["flat"].values()]


def _groups(case, y):
    """y [n, dim] in groups of columns [n, groups, width], the last one filled up with zeros."""
    width = case["group"] or case["dim"]
    return torch.nn.functional.pad(y, (0, -y.shape[1] % width)).view(y.shape[0], -1, width)


def _norm_outputs(case, y, h, scales):
    out = {"y": y}
    if case["dst"] == "i8":      # as the values that the integers stand for
        out["y"] = (_groups(case, y.float()) * scales[:, :, None]).flatten(1)[:, :case["dim"]].to(torch.bfloat16)
    if case["residual"]:
        out["h"] = h
    if scales is not None:
        out["scales"] = scales
    return out


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "embed_fwd":
        return (s["table"][s["ids"]].float() * c["scale"]).to(TYPES[c["dst"]])
    if kind in ("embed_bwd", "embed_add"):
        ids, d = s["ids"], s["dout"].float() * c["scale"]
        if c["pad"]:
            d = d * (ids != 0)[:, None]
        g = torch.zeros((c["rows"], c["dim"]), device="cuda").index_add_(0, ids, d)
        return g.to(TYPES[c["dst"]]) if kind == "embed_bwd" else s["grad"].copy_(s["grad"].float() + g)
    if kind == "norm_fwd":
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
        f = h.float()
        y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["weight"].float()
        if c["dst"] not in QMAX:
            return _norm_outputs(c, y.to(TYPES[c["dst"]]), h, None)
        most = QMAX[c["dst"]]
        y = _groups(c, y)
        scales = y.abs().amax(2) / most
        q = (y / torch.where(scales > 0, scales, 1.0)[:, :, None]).clamp(-most, most).flatten(1)[:, :c["dim"]]
        return _norm_outputs(c, q.to(TYPES["f8"]) if c["dst"] == "f8" else q.round().to(torch.int8), h, scales)
    if kind == "norm_bwd":
        h, dy, w = s["h"].float(), s["dy"].float(), s["weight"].float()
        rho = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        g = dy * w
        dh = rho * g - h * (rho * rho * rho * (g * h).mean(1, keepdim=True))
        if s["residual"] is not None:
            dh = dh + s["residual"].float()
        return dh.to(s["h"].dtype), (dy * h * rho).sum(0).to(TYPES[c["dst"]])
    parts = {t: torch.cat([g.reshape(-1) for g in s["grads"] if g.dtype == t]).float() for t in s["flat"]}
    norm = torch.sqrt(sum((p * p).sum() for p in parts.values()))
    factor = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    return [norm.reshape(1), *(s["flat"][t].copy_(p * factor) for t, p in parts.items())]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def _share_padded(case):
    return 0.25 if case["pad"] and case["tokens"] >= SEQ else 0.0


def _distinct(case):
    """Distinct ids of the tokens, expected."""
    n, rows, e = case["tokens"] * (1.0 - _share_padded(case)), float(case["rows"]), 1.0 - case["alpha"]
    total, a, steps = 0.0, 1.0, 400
    for k in range(1, steps + 1):
        b = max(a + 1.0, math.floor((rows + 1.0) ** (k / steps)))
        if b > rows + 1.0:
            break
        p = (a ** e - b ** e) / (1.0 - (rows + 1.0) ** e) / (b - a)
        total += (b - a) * -math.expm1(n * math.log1p(-min(p, 1 - 1e-12)))
        a = b
    return min(n, total) + (1.0 if case["pad"] else 0.0)


def work(case):
    kind = case["kind"]
    if kind == "clip":
        size = [math.prod(x) * SIZE[case["src"] if len(x) == 2 or case["vector"] == "same" else case["vector"]] for x in _shapes(case)]
        return {"bytes": 2.0 * sum(size), "flops": 3.0 * sum(math.prod(x) for x in _shapes(case))}
    n, d = case["tokens"], case["dim"]
    src, dst = SIZE[case["src"]], SIZE[case["dst"]]
    if kind.startswith("embed"):
        ids = n * (4 if case["ids"] == "i32" else 8)
        if kind == "embed_fwd":
            return {"bytes": ids + _distinct(case) * d * src + n * d * dst, "flops": n * d}
        kept = n * (1.0 - _share_padded(case))
        rows = case["rows"] if kind == "embed_bwd" else 2 * _distinct(case)
        return {"bytes": ids + kept * d * src + rows * d * dst, "flops": kept * d}
    more = 1 if case["residual"] else 0
    if kind == "norm_bwd":
        return {"bytes": n * d * src * (3 + more) + d * (SIZE[case["weight"]] + dst), "flops": 12.0 * n * d}
    scales = n * -(-d // (case["group"] or d)) * 4 if case["dst"] in QMAX else 0
    return {"bytes": n * d * (src * (1 + 2 * more) + dst) + d * SIZE[case["weight"]] + scales, "flops": 5.0 * n * d}


# ---- the definition, in 64 bits ----------------------------------------------------------------------------------------
def _sum_by_id(ids, rows_of, count):
    """Sums of the rows of each id: tokens put in order by id, running sums, differences at the ends of each id's run."""
    order = torch.argsort(ids.long(), stable=True)
    ends = torch.bincount(ids.long(), minlength=count).cumsum(0)
    out = torch.empty((count, rows_of.shape[1]), dtype=torch.float64, device="cuda")
    step = max(1, 200_000_000 // max(1, rows_of.shape[0] + count))
    for a in range(0, rows_of.shape[1], step):
        run = torch.zeros((rows_of.shape[0] + 1, min(step, rows_of.shape[1] - a)), dtype=torch.float64, device="cuda")
        run[1:] = rows_of[order, a:a + step].double().cumsum(0)
        at = run[ends]
        out[:, a:a + step] = torch.diff(at, dim=0, prepend=torch.zeros_like(at[:1]))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed_fwd":
        return s["table"][s["ids"].long()].double() * case["scale"]
    if kind in ("embed_bwd", "embed_add"):
        keep = s["ids"] != 0 if case["pad"] else torch.ones_like(s["ids"], dtype=torch.bool)
        g = _sum_by_id(s["ids"][keep], s["dout"][keep], case["rows"]) * case["scale"]
        return g if kind == "embed_bwd" else g + s["grad"].double()
    if kind == "norm_fwd":
        h = s["x"].double()
        if case["residual"]:
            h = h + s["residual"].double()
        kept = h.to(s["x"].dtype).double()           # the norm is that of the stored sum
        root = (kept.square().sum(1) / case["dim"] + EPS).sqrt()
        y = kept / root[:, None] * s["weight"].double()
        if case["dst"] not in QMAX:
            return {"y": y, "h": h} if case["residual"] else {"y": y}
        width = case["group"] or case["dim"]
        most = torch.stack([p.abs().amax(1) for p in y.split(width, 1)], 1) / QMAX[case["dst"]]
        if case["dst"] == "f8":
            y = torch.cat([p / m[:, None] for p, m in zip(y.split(width, 1), most.unbind(1))], 1)
        out = {"y": y, "scales": most}
        return {**out, "h": h} if case["residual"] else out
    if kind == "norm_bwd":
        h, c = s["h"].double(), s["dy"].double() * s["weight"].double()
        mean2 = h.square().sum(1, keepdim=True) / case["dim"] + EPS
        dh = (c - h * ((c * h).sum(1, keepdim=True) / (case["dim"] * mean2))) / mean2.sqrt()
        if s["residual"] is not None:
            dh = dh + s["residual"].double()
        return dh, (s["dy"].double() * (h / mean2.sqrt())).sum(0)
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in s["grads"]))
    factor = min(1.0, MAX_NORM / (norm + 1e-6))
    flat = {t: [] for t in s["flat"]}
    for g in s["grads"]:
        flat[g.dtype].append(g.reshape(-1).double() * factor)
    return [torch.tensor([norm], dtype=torch.float64), *(torch.cat(v) for v in flat.values())]
