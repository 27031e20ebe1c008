"""`-m gpu`: teachers whose entries hold all of the probability, with their log-sum given: where the student gives the others nothing, what roundings leave over is nothing, and does not make a
loss infinite."""
import pytest

from tests.dense_reference import U32, inside, rounded
from tests.logits_reference import NONE, SUM_STEPS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _want(x, at, z, lse, t):
    """(loss, bound, gradient, bound) for alpha 1, with nothing left over.  P's relative error: its exponent's rounding, two exponentials, products; log Q's: a sum of SUM_STEPS roundings, its logarithm, the
    scale of the exponents; the entries' sum over 64 lanes."""
    import math
    import torch
    t = float(torch.tensor(t, dtype=torch.float32))  # as the call takes it: 0.7 is off by 1.7e-8 of itself in 32 bits, and exponents of 86, in proportion to its reciprocal, by 1.5e-6: 24 units of 2^-24
    top, v = at.shape[1], x.shape[1]
    zt = z.double() / t
    p = torch.exp(zt - lse.double()[:, None])
    logq = torch.log_softmax(x.double() / t, 1)
    lq = logq.gather(1, at.long())
    d = torch.where(p > 0, (zt - lse.double()[:, None] - lq).abs(), 0.0)
    steps = top / 64 + 6
    rel = ((zt - zt.amax(1, keepdim=True)).abs() + (zt.amax(1) - lse.double()).abs()[:, None] + steps + 8) * U32
    loss = t * t * (p * (zt - lse.double()[:, None] - lq)).sum(1)
    off = t * t * (p * (rel * (d + 1) + (SUM_STEPS + 2 * math.log2(v) + 4 + 3 * (d + lq.abs()) + (steps + 4) * d) * U32)).sum(1) + 4 * U32 * loss.abs()
    q = logq.exp()
    psum = torch.zeros_like(q).scatter_add_(1, at.long(), p)
    grad = t * (p.sum(1, keepdim=True) * q - psum)
    small = (q * logq.abs()).nan_to_num(0, 0, 0)
    off_grad = t * (p.sum(1, keepdim=True) * (q * (2 * SUM_STEPS + 40 + steps) + 4 * small) * U32 + q * (p * rel).sum(1, keepdim=True)
                    + torch.zeros_like(q).scatter_add_(1, at.long(), p * (rel + 4 * U32)))
    return loss, 1.01 * off, grad, 1.01 * off_grad


def _check(ops, x, at, z, lse, t, what):
    import torch
    loss, off, grad, off_grad = _want(x, at, z, lse, t)
    w = torch.rand(len(x), device="cuda") + 0.5
    got, stats = ops.distill_fwd(x, at, z, teacher_lse=lse, temperature=t)
    inside(got, loss, off, (*what, "loss"))
    wd = w.double()[:, None]
    bound = off_grad * wd + rounded((grad * wd).abs() + off_grad * wd, x.dtype) + 2 * U32 * (grad * wd).abs()
    inside(ops.distill_bwd(w, x, at, z, stats, temperature=t), grad * wd, bound, (*what, "grad"))
    both, back = ops.distill_grad(w, x, at, z, teacher_lse=lse, temperature=t)
    inside(both, loss, off, (*what, "loss of one call"))
    inside(back, grad * wd, bound, (*what, "grad of one call"))


def _inputs(n, v, top, kind, seed, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    at = torch.argsort(torch.rand((n, v), generator=g, device="cuda"), 1)[:, :top].contiguous()
    z = 2 * torch.randn((n, top), generator=g, device="cuda") + torch.linspace(-60, 60, n, device="cuda")[:, None]
    x = (3 * torch.randn((n, v), generator=g, device="cuda")).to(kind)
    return x, at, z, torch.logsumexp(z.double() / t, 1).float()


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("v", [1, 5, 64, 200, 1024])
def test_every_id_is_named(ops, v, kind):
    import torch
    for t in (1.0, 2.0, 0.7):
        x, at, z, lse = _inputs(300, v, v, getattr(torch, kind), v, t)
        _check(ops, x, at, z, lse, t, (v, kind, t))
    ops.check()


@pytest.mark.parametrize("kind,mask", [(k, m) for k in ("float32", "bfloat16") for m in (NONE, -1e4, -1e9, -1e30, "lowest")] + [("float16", NONE), ("float16", -1e4), ("float16", "lowest")])
@pytest.mark.parametrize("v,top", [(300, 7), (9000, 64), (40_000, 300)])
def test_the_others_are_masked(ops, v, top, kind, mask):
    import torch
    k = getattr(torch, kind)
    for t in (1.0, 2.0, 0.7):
        x, at, z, lse = _inputs(100, v, top, k, v, t)
        named = torch.zeros(x.shape, dtype=torch.bool, device="cuda").scatter_(1, at, True)
        x[~named] = float(torch.finfo(k).min) if mask == "lowest" else mask
        _check(ops, x, at, z, lse, t, (v, kind, mask, t))
        # a log-sum that was worked out in 32 bits from the logits in 32 bits
        _check(ops, x, at, z, torch.logsumexp(z / t, 1), t, (v, kind, mask, t, "32 bits"))
    ops.check()


def test_what_is_left_over_in_earnest_counts(ops):
    """The same rows with a thousandth, or a hundred-thousandth, left over: infinitely much where the others have nothing, and in proportion to the mask where it is finite."""
    import torch
    for share in (1e-3, 1e-5):
        x, at, z, lse = _inputs(100, 300, 7, torch.float32, 1, 1.0)
        z = z - z.amax(1, keepdim=True)              # (about zero: differences of 1e-5 are far above the roundings of log-sums of 2)
        lse = (torch.logsumexp(z.double(), 1) - torch.log1p(torch.tensor(-share, dtype=torch.float64, device="cuda"))).float()
        named = torch.zeros(x.shape, dtype=torch.bool, device="cuda").scatter_(1, at, True)
        x[~named] = NONE
        loss, _ = ops.distill_fwd(x, at, z, teacher_lse=lse)
        assert bool((loss == float("inf")).all())
        x[~named] = -1e6
        loss, _ = ops.distill_fwd(x, at, z, teacher_lse=lse)
        left = (1 - torch.exp(z.double() - lse.double()[:, None]).sum(1)) * 1e6
        # the roundings of 7 probabilities and their sum, of 1 in all; the terms beside are below 100
        assert bool(((loss.double() - left).abs() <= 40 * U32 * 1e6 + 100).all())
    ops.check()
