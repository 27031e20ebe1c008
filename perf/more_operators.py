"""Performance cases of the operators on rows of logits: distillation from a teacher's top logits, beam search's selection and the reordering of states.

One case is one call of one operator (`distill_pair`: the forward and the backward call of a training step), on inputs made from a seed on the GPU.  Where
`own` is false `run` computes the operator in its plain form (elementary torch operations in 32 bits, scores that are put in order in 64), otherwise it makes
the calls that a program makes of `DenseOps`.

A distillation case has `rows` rows of logits over `vocab` ids in type `src`, `top` entries of the teacher a row, `rest` (the teacher's
log-sum over all ids is known, so what its entries leave over counts), `alpha` (the share of distillation; the rest is cross entropy with a target),
`ragged` (lists end early, some are empty, some rows are left out) and `banned` (some ids' logits are -inf).  A beam case has `batch` sequences of `beams` beams, of
which `keep` go on; `first`: only one beam of a sequence is alive; `done`: some beams have ended.  A reorder case has a keys' and a values' state for each of `layers` layers,
[batch, beams, heads, length, dim] in place (`keep` 0) or into others of `keep` beams, out of buffers of `room` positions, and the beams' tokens so far.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EOS = 2
SPREAD = 3.0                     # of logits
LOSS_SCALE = 4096.0
CELLS_MOST = 500_000_000         # logits of a drawn case
STATE_MOST = 1_200_000_000       # bytes of a drawn case's states
NO_SCORE = float("-inf")


# ---- cases -----------------------------------------------------------------------------------------------------------
def _distill(name, kind, rows, vocab, src, top, teacher="f32", ids="i64", temperature=1.0, alpha=1.0, rest=False, ragged=False, banned=False):
    c = dict(kind=kind, rows=rows, vocab=vocab, src=src, top=top, teacher=teacher, ids=ids, temperature=temperature, alpha=alpha, rest=rest, ragged=ragged,
             banned=banned)
    return {"name": name, **c} if name else c


def _beam(name, batch, beams, vocab, src, keep, first=False, done=False):
    c = dict(kind="beam", batch=batch, beams=beams, vocab=vocab, src=src, keep=keep, first=first, done=done)
    return {"name": name, **c} if name else c


def _reorder(name, batch, beams, layers, heads, length, dim, src, room=0, keep=0):
    c = dict(kind="reorder", batch=batch, beams=beams, layers=layers, heads=heads, length=length, dim=dim, src=src, room=room, keep=keep)
    return {"name": name, **c} if name else c


def listed():
    return [
        # one row's loss and gradient: latency
        _distill("distill_one", "distill_grad", 1, 100_000, "bf16", 8, alpha=0.5),
        # evaluation of a next-item model: 256 samples over 5000 items
        _distill("distill_eval_items", "distill_fwd", 256, 5000, "f32", 16, alpha=0.5),
        # evaluation over the word table of a language model, the teacher's probabilities with what they leave over
        _distill("distill_eval_words", "distill_fwd", 8192, 131_072, "bf16", 64, temperature=2.0, rest=True),
        # odd sizes, lists of unequal length, rows left out: forward pass, then backward pass
        _distill("distill_pair_odd", "distill_pair", 777, 50_021, "f16", 20, teacher="f16", ids="i32", temperature=1.5, alpha=0.9, rest=True, ragged=True),
        # a training step's forward and backward pass over the word table, cross entropy beside the teacher at another temperature
        _distill("distill_pair_words", "distill_pair", 4096, 131_072, "bf16", 64, teacher="bf16", temperature=2.0, alpha=0.5),
        # loss and gradient in one call: a long batch over a table of middle size
        _distill("distill_grad_items", "distill_grad", 16_384, 32_768, "bf16", 32, alpha=0.5, rest=True),
        # serving one sequence, four beams: latency
        _beam("beam_one", 1, 4, 131_072, "bf16", 4),
        # odd sizes, some beams have ended, twice as many go on (for those that end now)
        _beam("beam_odd", 33, 5, 50_021, "f32", 10, done=True),
        # a batch of sequences
        _beam("beam_batch", 64, 8, 131_072, "bf16", 16),
        # the states of one sequence's four beams, 8 layers, after 60 tokens: latency
        _reorder("reorder_one", 1, 4, 8, 4, 60, 64, "bf16", room=128),
        # odd rows into other buffers, more beams than before
        _reorder("reorder_odd", 7, 5, 3, 3, 77, 33, "f32", keep=10),
        # the states of a batch, in place, in buffers with room for more tokens
        _reorder("reorder_batch", 16, 8, 12, 4, 500, 128, "bf16", room=512),
    ]


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("distill_fwd", "distill_pair", "distill_grad", "distill_grad", "beam", "beam", "beam", "reorder", "reorder"))
    src = rng.choice(("f32", "bf16", "bf16", "f16"))
    if kind == "reorder":
        batch, beams = logu(1, 128), rng.choice((1, 2, 3, 4, 5, 8, 10, 16, 32, 64))
        heads, length, dim = rng.choice((1, 2, 4, 8)), logu(1, 2000), rng.choice((1, 16, 64, 128, logu(8, 512)))
        layers, row = logu(1, 28), heads * length * dim * SIZE[src]
        batch = max(1, min(batch, STATE_MOST // (2 * beams * row)))
        layers = max(1, min(layers, STATE_MOST // (2 * batch * beams * row)))
        return _reorder(None, batch, beams, layers, heads, length, dim, src, rng.choice((0, length + logu(1, 64))), rng.choice((0, 0, beams, logu(1, 64))))
    vocab = rng.choice((500, 5000, 32_768, 100_000, 131_072, logu(300, 262_144), logu(300, 262_144), logu(300, 262_144)))
    if kind == "beam":
        beams = rng.choice((1, 2, 3, 4, 5, 8, 10, 16, 32))
        batch = max(1, min(logu(1, 256), CELLS_MOST // 8 // (beams * vocab)))
        return _beam(None, batch, beams, vocab, src, rng.choice((beams, beams, 2 * beams, logu(1, 64))), rng.random() < 0.2, rng.random() < 0.4)
    rows = max(1, min(logu(1, 16_384), CELLS_MOST // vocab))
    top = rng.choice((1, 8, 16, 64, logu(1, 256)))
    alpha = rng.choice((1.0, 0.5, 0.9))
    return _distill(None, kind, rows, vocab, src, top, rng.choice(("f32", src)), rng.choice(("i64", "i32")), rng.choice((1.0, 2.0, 4.0, 0.75)), alpha,
                    rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.3)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + part)
    return g


def _rand(shape, g):
    return torch.rand(shape, generator=g, device="cuda")


def _randn(shape, kind, g, spread=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(spread).to(TYPES[kind])


def _int(ids, kind):
    return ids.to(torch.int32 if kind == "i32" else torch.int64)


def _prepare_distill(case, g):
    n, v, k, t = case["rows"], case["vocab"], case["top"], case["temperature"]
    # the teacher's entries: distinct ids, one out of each of k ranges in a row's own order, values in descending order
    lot = v // k
    ids = torch.argsort(_rand((n, k), g), dim=1) * lot + (_rand((n, k), g) * lot).long().clamp_(max=lot - 1)
    z = torch.sort(torch.randn((n, k), generator=g, device="cuda") * 1.5 + 10.0, dim=1, descending=True).values
    x = torch.randn((n, v), generator=g, device="cuda").mul_(SPREAD)
    # a student that has learnt some of it
    x.scatter_(1, ids, z - 1.0 + 1.5 * torch.randn((n, k), generator=g, device="cuda"))
    target = ids[torch.arange(n, device="cuda"), (_rand(n, g) ** 2 * k).long().clamp_(max=k - 1)]
    s = {"case": case, "teacher": z.to(TYPES[case["teacher"]])}
    if case["banned"]:
        ban = _rand(v, g) < 0.05
        ban = ban.expand(n, v).clone().scatter_(1, ids, False)
        x.masked_fill_(ban, NO_SCORE)
    s["logits"] = x.to(TYPES[case["src"]])
    if case["ragged"]:
        there = (_rand(n, g) * (k + 1)).long()                            # 0 .. k entries
        ids = torch.where(torch.arange(k, device="cuda") < there[:, None], ids, -1)
        target = torch.where(_rand(n, g) < 0.1, -1, target)
    s["ids"] = _int(ids, case["ids"])
    s["target"] = _int(target, case["ids"]) if case["alpha"] < 1.0 or case["ragged"] else None
    s["lse"] = None
    if case["rest"]:
        # the entries hold a share of the teacher's probability
        zt = torch.where(ids >= 0, s["teacher"].double() / t, NO_SCORE)
        top = torch.where(ids[:, 0] >= 0, torch.logsumexp(zt, 1), 0.0)
        s["lse"] = (top - torch.log(0.5 + 0.45 * _rand(n, g).double())).float()
    # the gradient that arrives at each row's loss; in f16 with a loss scale
    s["weight"] = (0.5 + _rand(n, g)) / n * (LOSS_SCALE if case["src"] == "f16" else 1.0)
    return s


def _prepare_beam(case, g):
    b, w, v = case["batch"], case["beams"], case["vocab"]
    x = _randn((b, w, v), case["src"], g, SPREAD)
    scores = torch.sort(-8.0 * _rand((b, w), g), dim=1, descending=True).values
    s = {"case": case, "logits": x, "finished": None}
    if case["first"]:
        scores[:, 1:] = NO_SCORE
    if case["done"]:
        s["finished"] = _rand((b, w), g) < 0.3
    s["scores"] = scores
    return s


def _prepare_reorder(case, g):
    b, w, keep = case["batch"], case["beams"], case["keep"]
    parts = (b, w, case["heads"], max(case["room"], case["length"]), case["dim"])
    s = {"case": case, "states": [_randn(parts, case["src"], g)[:, :, :, :case["length"]] for _ in range(2 * case["layers"])]}
    s["states"].append((_rand((b, w, case["length"]), g) * 50_000).long())
    s["parents"] = (_rand((b, keep or w), g) * w).to(torch.int32).clamp_(max=w - 1)
    s["out"] = [torch.empty((b, keep, *t.shape[2:]), dtype=t.dtype, device="cuda") for t in s["states"]] if keep else None
    return s


def prepare(case, seed):
    g = _gen(seed, 1)
    if case["kind"] == "beam":
        return _prepare_beam(case, g)
    return (_prepare_reorder if case["kind"] == "reorder" else _prepare_distill)(case, g)


# ---- one pass --------------------------------------------------------------------------------------------------------
_handle = None


def _ops():
    """The handle that a program makes once and keeps."""
    global _handle
    if _handle is None:
        from paper_2208_05321_amd import DenseOps
        _handle = DenseOps()
    return _handle


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    c, ops = s["case"], _ops()
    kind = c["kind"]
    if kind == "beam":
        scores, parents, tokens, finished = ops.beam_select(s["logits"], s["scores"], c["keep"], finished=s["finished"], eos_id=EOS)
        return {"scores": scores, "parents": parents, "tokens": tokens, "finished": finished}
    if kind == "reorder":
        return ops.beam_reorder(s["states"], s["parents"], out=s["out"])
    how = dict(targets=s["target"], temperature=c["temperature"], alpha=c["alpha"])
    if kind == "distill_grad":
        loss, grad = ops.distill_grad(s["weight"], s["logits"], s["ids"], s["teacher"], teacher_lse=s["lse"], **how)
        return {"loss": loss, "grad": grad}
    loss, stats = ops.distill_fwd(s["logits"], s["ids"], s["teacher"], teacher_lse=s["lse"], **how)
    if kind == "distill_fwd":
        return {"loss": loss}
    return {"loss": loss, "grad": ops.distill_bwd(s["weight"], s["logits"], s["ids"], s["teacher"], stats, **how)}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "beam":
        return _plain_beam(s)
    if kind == "reorder":
        rows = torch.arange(s["parents"].shape[0], device="cuda")[:, None]
        return [o.copy_(t[rows, s["parents"].long()]) for t, o in zip(s["states"], s["out"] or s["states"])]
    return _plain_distill(s)


def _plain_beam(s):
    c, keep = s["case"], s["case"]["keep"]
    b, w, v = s["logits"].shape
    alive = torch.isfinite(s["scores"])
    x = s["logits"].double()
    m = x.amax(2, keepdim=True)
    x = x - (m + torch.exp(x - m).sum(2, keepdim=True).log()) + s["scores"].double()[:, :, None]
    if s["finished"] is not None:
        at_end = torch.arange(v, device="cuda") == EOS
        x = torch.where(s["finished"][:, :, None], torch.where(at_end, s["scores"].double()[:, :, None], NO_SCORE), x)
    x = torch.where(alive[:, :, None], x, NO_SCORE).view(b, w * v)
    least = x.topk(keep, 1).values[:, -1:]
    more, same = x > least, x == least
    taken = more | (same & (same.cumsum(1) <= keep - more.sum(1, keepdim=True)))       # of equal ones those with the lower index
    at = taken.nonzero()[:, 1].view(b, keep)
    scores, order = torch.sort(x.gather(1, at), dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    none = scores == NO_SCORE
    tokens = torch.where(none, EOS, at % v)
    return {"scores": scores.float(), "parents": torch.where(none, 0, at // v).to(torch.int32), "tokens": tokens, "finished": tokens == EOS}


def _plain_distill(s):
    c = s["case"]
    t, alpha = c["temperature"], c["alpha"]
    x, ids = s["logits"].float(), s["ids"].long()
    there = ids >= 0
    at = torch.where(there, ids, 0)
    z = torch.where(there, s["teacher"].float() / t, NO_SCORE)
    some = there.any(1)
    if s["lse"] is None:
        zm = torch.where(some, z.amax(1), 0.0)
        of = zm + torch.log(torch.exp(z - zm[:, None]).sum(1).clamp(min=1e-30))
    else:
        of = s["lse"]
    logp = z - of[:, None]
    p = torch.exp(logp)
    m = x.amax(1, keepdim=True)
    e = torch.exp((x - m) / t)
    total = e.sum(1, keepdim=True)
    logq = (x.gather(1, at) - m) / t - total.log()
    kl = torch.where(there, p * (logp - logq), 0.0).sum(1)
    p0 = q0 = None
    if s["lse"] is not None:
        named = torch.zeros(x.shape, dtype=torch.int32, device="cuda").scatter_add_(1, at, there.int()) > 0
        p0 = (1.0 - p.double().sum(1, keepdim=True)).clamp(min=0.0).float()
        q0 = torch.where(named, 0.0, e).sum(1, keepdim=True) / total
        kl = kl + (p0 * (p0.log() - q0.log()))[:, 0]
    kl = torch.where(some, kl, 0.0)
    kept = torch.ones_like(some) if s["target"] is None else s["target"] >= 0
    loss = alpha * t * t * kl
    if alpha < 1.0:
        e1 = torch.exp(x - m)
        total1 = e1.sum(1, keepdim=True)
        target = torch.where(kept, s["target"].long(), 0)[:, None]
        loss = loss + (1.0 - alpha) * (m + total1.log() - x.gather(1, target))[:, 0]
    out = {"loss": torch.where(kept, loss, 0.0)}
    if c["kind"] == "distill_fwd":
        return out
    grad = e / total
    if p0 is not None:
        grad = torch.where(named, grad, grad * (1.0 - p0 / q0))
    grad = grad.scatter_add_(1, at, torch.where(there, -p, 0.0)) * torch.where(some, alpha * t, 0.0)[:, None]
    if alpha < 1.0:
        grad = grad + (1.0 - alpha) * (e1 / total1).scatter_add_(1, target, torch.full_like(m, -1.0))
    out["grad"] = (grad * torch.where(kept, s["weight"], 0.0)[:, None]).to(s["logits"].dtype)
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "reorder":
        w, keep = case["beams"], case["keep"]
        row = case["heads"] * case["length"] * case["dim"] * SIZE[case["src"]] * 2 * case["layers"] + case["length"] * 8
        # rows read: those that are the parent of a row that changes; rows written: those that change
        read, written = (w * (1 - (1 - 1 / w) ** keep), keep) if keep else (w * (1 - (1 - 1 / w) ** (w - 1)), w - 1)
        return {"bytes": case["batch"] * (row * max(read + written, 1e-3) + 4 * (keep or w)), "flops": 0.0}
    if kind == "beam":
        read = case["batch"] * case["vocab"] * (1 if case["first"] else case["beams"]) * (0.7 if case["done"] else 1.0)
        return {"bytes": read * SIZE[case["src"]] + case["batch"] * (case["beams"] * 4 + case["keep"] * 17), "flops": 4.0 * read}
    rows = case["rows"] * (0.9 if case["ragged"] else 1.0)
    cells = rows * case["vocab"]
    entries = case["rows"] * case["top"] * (SIZE[case["teacher"]] + (4 if case["ids"] == "i32" else 8))
    exps = 2 if case["alpha"] < 1.0 and case["temperature"] != 1.0 else 1
    if kind == "distill_fwd":
        return {"bytes": cells * SIZE[case["src"]] + entries, "flops": (2 + 3 * exps) * cells}
    return {"bytes": (cells + case["rows"] * case["vocab"]) * SIZE[case["src"]] + entries, "flops": (4 + 6 * exps) * cells}


# ---- the definition, in 64 bits ----------------------------------------------------------------------------------------
def _exact_beam(case, s):
    b, w, v = s["logits"].shape
    out = {"scores": [], "parents": [], "tokens": []}
    for i in range(b):
        of = torch.log_softmax(s["logits"][i].double(), 1) + s["scores"][i].double()[:, None]
        for j in range(w):
            if s["scores"][i, j] == NO_SCORE:
                of[j] = NO_SCORE
            elif s["finished"] is not None and bool(s["finished"][i, j]):
                of[j] = NO_SCORE
                of[j, EOS] = s["scores"][i, j].double()
        best, at = torch.sort(of.reshape(-1), descending=True, stable=True)
        best, at = best[:case["keep"]], at[:case["keep"]]
        gone = torch.isinf(best)
        out["scores"].append(best)
        out["parents"].append((at // v).masked_fill(gone, 0).to(torch.int32))
        out["tokens"].append((at % v).masked_fill(gone, EOS))
    out = {k: torch.stack(x) for k, x in out.items()}
    return {**out, "finished": out["tokens"] == EOS}


def _exact_rows(case, s, a, b):
    """Loss, and gradient for a weight of one, of the rows a .. b-1."""
    t, alpha = case["temperature"], case["alpha"]
    x, ids = s["logits"][a:b].double(), s["ids"][a:b].long()
    listed_ = (ids >= 0).double()
    at = ids.clamp(min=0)
    z = s["teacher"][a:b].double() / t
    # weights of the entries, with zero in the place of those that are not there
    if s["lse"] is None:
        p = torch.softmax(z.masked_fill(ids < 0, -1e300), 1) * listed_
        over = torch.zeros(b - a, dtype=torch.float64, device="cuda")
    else:
        p = torch.exp(z - s["lse"][a:b].double()[:, None]) * listed_
        over = (1.0 - p.sum(1)).clamp(min=0.0)
    log_q = torch.log_softmax(x / t, 1)
    spot = torch.zeros_like(x).scatter_add_(1, at, listed_) > 0
    others = torch.logsumexp(log_q.masked_fill(spot, NO_SCORE), 1)
    kl = torch.special.xlogy(p, p).sum(1) - (p * torch.where(p > 0, log_q.gather(1, at), 0.0)).sum(1)
    kl = kl + torch.special.xlogy(over, over) - torch.where(over > 0, over * others, 0.0)
    has = (ids >= 0).any(1)
    share = torch.where(has, alpha * t, 0.0)[:, None]
    pulled = p.sum(1, keepdim=True) + over[:, None] - torch.where(spot, 0.0, (over / others.exp())[:, None])
    grad = share * (log_q.exp() * pulled - torch.zeros_like(x).scatter_add_(1, at, p))
    loss = torch.where(has, alpha * t * t * kl, 0.0)
    if alpha < 1.0:
        log_r = torch.log_softmax(x, 1)
        hard = s["target"][a:b].long().clamp(min=0)[:, None]
        loss = loss - (1.0 - alpha) * log_r.gather(1, hard)[:, 0]
        grad = grad + (1.0 - alpha) * (log_r.exp() - torch.zeros_like(x).scatter_(1, hard, 1.0))
    if s["target"] is not None:
        gone = s["target"][a:b] < 0
        loss, grad = loss.masked_fill(gone, 0.0), grad.masked_fill(gone[:, None], 0.0)
    return loss, grad


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "beam":
        return _exact_beam(case, s)
    if case["kind"] == "reorder":
        w = case["beams"]
        parents = (s["parents"].long() + w * torch.arange(case["batch"], device="cuda")[:, None]).view(-1)
        return [torch.index_select(t.reshape(-1, *t.shape[2:]), 0, parents).view(case["batch"], -1, *t.shape[2:]) for t in s["states"]]
    n, step = case["rows"], max(1, 60_000_000 // case["vocab"])
    loss = torch.empty(n, dtype=torch.float64, device="cuda")
    grad = None if case["kind"] == "distill_fwd" else torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda")
    for a in range(0, n, step):
        b = min(n, a + step)
        loss[a:b], of = _exact_rows(case, s, a, b)
        if grad is not None:
            grad[a:b] = of * s["weight"][a:b].double()[:, None]
    return {"loss": loss} if grad is None else {"loss": loss, "grad": grad}
