"""Plain 64-bit forms of the operators on rows of logits, and the errors that 32-bit arithmetic and one final rounding allow them."""
import math

import torch

from tests.dense_reference import U32, rounded

NONE = float("-inf")
# A sum of exponentials: a lane adds 64 or fewer of them one after the other, lanes, wavefronts and slices are joined in 12 + 3 + 14 steps, each with one more exponential
# and product; an exponential is off by a unit, and its argument by half a unit of itself, which is at most 0.4 of the largest term's (y exp(-y) <= 0.37).
SUM_STEPS = 64 + 3 * 29 + 4


def distill(logits, ids, z, lse, targets, temperature, alpha):
    """(loss, gradient for a weight of 1, bound of the loss's error, bound of the gradient's) of rows [n, V], in 64 bits."""
    x, t = logits.double(), float(temperature)
    n, v = x.shape
    ids = ids.long()
    there = (ids >= 0) & (ids < v)
    at = torch.where(there, ids, 0)
    zt = torch.where(there, z.double() / t, NONE)
    some = there.any(1) if lse is not None else (zt > NONE).any(1)
    zmax = torch.where((zt > NONE).any(1), zt.amax(1) if zt.shape[1] else torch.zeros(n, dtype=torch.float64, device=x.device), 0.0) if zt.shape[1] else torch.zeros_like(x[:, 0])
    of = lse.double() if lse is not None else zmax + torch.exp(zt - zmax[:, None]).sum(1).log()
    logp = zt - torch.where(some, of, 0.0)[:, None]
    p = torch.where(there & some[:, None], torch.exp(logp), 0.0)
    named = torch.zeros_like(x).scatter_add_(1, at, there.double()) > 0
    logq = torch.log_softmax(x / t, 1)
    lq = logq.gather(1, at)
    logr = torch.logsumexp(torch.where(named, NONE, logq), 1)
    p0 = (1.0 - p.sum(1)).clamp(min=0.0) if lse is not None else torch.zeros_like(logr)
    p0 = torch.where(some, p0, 0.0)
    term = lambda w, a, b: torch.where(w > 0, w * (a - b), 0.0)  # noqa: E731
    kl = term(p, logp, lq).sum(1) + term(p0, p0.log(), logr)
    # relative error of a probability of the teacher: its exponent's rounding (differences from the largest entry, and the log-sum), two exponentials, a sum, a quotient
    steps = ids.shape[1] / 64 + 6
    rel_p = (torch.where(p > 0, (zt - zmax[:, None]).abs(), 0.0) + (zmax - of).abs().nan_to_num(0, 0, 0)[:, None] + steps + 8) * U32
    off_p0 = (p * rel_p).sum(1) + (steps + 2) * U32 if lse is not None else torch.zeros_like(p0)
    # absolute error of log Q: the sum, its logarithm, half a unit of the exponent's scale in differences from the largest logit
    reach = torch.where(torch.isfinite(lq), lq.abs(), 0.0)
    off_q = (SUM_STEPS + 2 * math.log2(v) + 4 + reach) * U32
    off_r = (2 * SUM_STEPS + 2 * math.log2(v) + 8 + logr.abs().nan_to_num(0, 0, 0)) * U32
    dist = lambda w, a, b: torch.where(w > 0, (a - b).abs(), 0.0).nan_to_num(0, 0, 0)  # noqa: E731
    # log P: the logarithm of the sum of exponentials, or of P_0, and the rounding of the difference
    off_kl = (p * (rel_p * (dist(p, logp, lq) + 1) + off_q + (steps + 8) * U32 + 3 * U32 * (dist(p, logp, lq) + reach))).sum(1)
    off_kl = off_kl + off_p0 * (dist(p0, p0.log(), logr) + 1) + p0 * (off_r + 8 * U32 * (1 + dist(p0, p0.log(), logr) + logr.abs().nan_to_num(0, 0, 0)))
    off_kl = off_kl + (steps + 4) * U32 * (p * dist(p, logp, lq)).sum(1)
    if alpha == 0.0:                                 # (no term, also where it would be infinite)
        kl, off_kl = torch.zeros_like(kl), torch.zeros_like(kl)
    loss, off = alpha * t * t * kl, alpha * t * t * off_kl
    c = (p.sum(1) + p0)[:, None]
    q, r = logq.exp(), torch.where(named, 0.0, (logq - logr[:, None]).exp()).nan_to_num(0, 0, 0)
    psum = torch.zeros_like(x).scatter_add_(1, at, p)
    grad = alpha * t * (c * q - psum - p0[:, None] * r)
    spread = torch.where(torch.isfinite(logq), logq.abs(), 0.0)
    rel_q = (SUM_STEPS + 16 + 2 * spread) * U32
    # (of the others: a difference of c Q_0 and P_0, whose errors stay)
    q0 = logr.exp()[:, None]
    # (P_0 is what P leaves over, whatever its error: c is its error's too, and an entry that is named K times adds K of them)
    off_grad = alpha * t * (c * q * rel_q + torch.zeros_like(x).scatter_add_(1, at, p * (rel_p + (ids.shape[1] + 2) * U32)) + off_p0[:, None] * (q + r)
                            + r * (q0 * rel_q.new_tensor((2 * SUM_STEPS + 24) * U32) + p0[:, None] * (SUM_STEPS + 24 + spread) * U32 + (q0 * (1 + q0.log().abs())).nan_to_num(0, 0, 0) * 4 * U32))
    grad = torch.where(some[:, None], grad, 0.0)
    off_grad = torch.where(some[:, None], off_grad, 0.0)
    loss, off = torch.where(some, loss, 0.0), torch.where(some, off, 0.0)
    if alpha < 1.0:
        log1 = torch.log_softmax(x, 1)
        y = torch.where((targets >= 0) & (targets < v), targets.long(), 0)[:, None]
        hit = log1.gather(1, y)[:, 0]
        loss = loss - (1.0 - alpha) * hit
        off = off + (1.0 - alpha) * (SUM_STEPS + 2 * math.log2(v) + 4 + 2 * hit.abs().nan_to_num(0, 0, 0)) * U32
        one = torch.zeros_like(x).scatter_(1, y, 1.0)
        grad = grad + (1.0 - alpha) * (log1.exp() - one)
        spread1 = torch.where(torch.isfinite(log1), log1.abs(), 0.0)
        off_grad = off_grad + (1.0 - alpha) * (log1.exp() * (SUM_STEPS + 16 + 2 * spread1) * U32 + 3 * U32 * one)
    if targets is not None:
        gone = (targets < 0) | (targets >= v)
        loss, off = torch.where(gone, 0.0, loss), torch.where(gone, 0.0, off)
        grad, off_grad = torch.where(gone[:, None], 0.0, grad), torch.where(gone[:, None], 0.0, off_grad)
    return loss, grad, 1.01 * off + rounded(loss.nan_to_num(0, 0, 0), torch.float32) * 4, 1.01 * off_grad + 4 * U32 * grad.abs().nan_to_num(0, 0, 0)


def select(logits, scores, keep, finished=None, eos=-1):
    """(scores in 64 bits, parents, tokens) of each sequence, by a stable sort."""
    b, w, v = logits.shape
    x = logits.double()
    c = x - torch.logsumexp(x, 2, keepdim=True) + scores.double()[:, :, None]
    good = torch.isfinite(torch.logsumexp(x, 2)) & torch.isfinite(scores)
    c = torch.where(good[:, :, None], c, NONE)
    if finished is not None:
        end = torch.where(torch.arange(v, device=x.device) == eos, scores.double()[:, :, None], NONE)
        c = torch.where((finished & torch.isfinite(scores))[:, :, None], end, torch.where(finished[:, :, None], NONE, c))
    best, at = torch.sort(c.reshape(b, w * v), dim=1, descending=True, stable=True)
    if best.shape[1] < keep:
        best, at = (torch.nn.functional.pad(t, (0, keep - t.shape[1]), value=f) for t, f in ((best, NONE), (at, 0)))
    best, at = best[:, :keep], at[:, :keep]
    none = best == NONE
    return best, torch.where(none, 0, at // v).int(), torch.where(none, max(eos, 0), at % v)


def reordered(t, parents):
    return torch.stack([t[b, parents[b].long()] for b in range(t.shape[0])])
