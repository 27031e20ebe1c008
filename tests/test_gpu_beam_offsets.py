"""`-m gpu`: beam search's selection of logits that have an offset in common, or one for each beam: a log-softmax does not depend on it."""
import math

import pytest

from tests.dense_reference import U32
from tests.logits_reference import NONE

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _select(x, scores, keep):
    """In 64 bits; the largest logit is taken off before anything is added to it, so that offsets leave nothing behind."""
    import torch
    b, w, v = x.shape
    c = torch.log_softmax(x.double(), 2) + scores.double()[:, :, None]
    c = torch.where(torch.isfinite(x) & torch.isfinite(scores)[:, :, None], c, NONE)
    best, at = torch.sort(c.view(b, w * v), dim=1, descending=True, stable=True)
    return best[:, :keep], (at[:, :keep] // v).int(), at[:, :keep] % v


# The log-sum's error, relative to the sum, in units of 2^-24.  A slice's 64 elements of a lane: 64 additions, an exponential and its argument (1 and 0.4 of the largest term's: y 2^-y
# <= 0.54, times ln 2); a factor that refers them to the largest element: 2.  Slices of a lane, seven more: an exponential with its argument of two roundings, a product and an addition, 1 + 0.8 +
# 0.5 + 0.5 < 3 each.  Lanes, wavefronts and slices, joined in 64 bits: an exponential and its argument, and a product for the lanes: 2.3 each.  Last, that the scale of exponents is log2(e) rounded
# (half a unit): half a unit of the mean of the distances from the largest and of the log-sum over it, log(ids) each at most.
STEPS = 64 + 2 + 2 + 7 * 3 + 3 * 2.3


def _check(ops, x, scores, keep, what):
    import torch
    got, parents, tokens, _ = ops.beam_select(x, scores, keep)
    best, p, t = _select(x, scores, keep)
    assert torch.equal(tokens, t) and torch.equal(parents, p), what
    none = best == NONE
    assert torch.equal(none, got == NONE), what
    # the score's own rounding, half a unit of it
    off = (STEPS + math.log(x.shape[2]) + best.abs()) * U32
    assert bool(((got.double() - best).abs() <= off)[~none].all()), (what, float((got.double() - best).abs()[~none].max()))


def _inputs(b, w, v, seed, spread=3.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((b, w, v), generator=g, device="cuda") * spread, torch.sort(-6 * torch.rand((b, w), generator=g, device="cuda"), 1, descending=True).values


@pytest.mark.parametrize("kind,offset", [("float32", 1000.0), ("float32", -1000.0), ("float32", 30_000.0), ("float32", -1e6), ("bfloat16", 1000.0), ("bfloat16", -30_000.0),
                                         ("float16", 1000.0), ("float16", -30_000.0)])
@pytest.mark.parametrize("b,w,v,keep", [(1, 4, 131_072, 4), (3, 5, 9001, 10), (2, 3, 300, 6), (40, 8, 17_000, 16)])
def test_a_common_offset(ops, b, w, v, keep, kind, offset):
    import torch
    x, scores = _inputs(b, w, v, b + v)
    _check(ops, (x + offset).to(getattr(torch, kind)), scores, keep, (b, w, v, keep, kind, offset))
    ops.check()


@pytest.mark.parametrize("kind,grain,step", [("float32", 64, 512.0), ("float32", 64, 8192.0), ("bfloat16", 1, 40.0), ("float16", 1, 64.0)])
@pytest.mark.parametrize("v", [700, 40_000])
def test_an_offset_of_each_beam(ops, v, kind, grain, step):
    """Each beam's logits are those of the first, moved (exactly: whole numbers of grains, below the type's 24, 8 or 11 bits), so that the order of their candidates is that of the
    scores, which lie 4e-5 apart: more than twice the error of a log-sum (110 units of 2^-24 = 6.6e-6)."""
    import torch
    x = (_inputs(1, 1, v, v)[0] * grain).round() / grain
    y32 = x.expand(2, 6, v) + torch.arange(6, device="cuda").view(1, 6, 1) * step
    y = y32.to(getattr(torch, kind)).contiguous()
    assert torch.equal(y.float(), y32)
    scores = (-4e-5 * torch.arange(6, device="cuda")).expand(2, 6).contiguous()
    _check(ops, y, scores, 12, (v, kind, step))
    _check(ops, y, scores.flip(1).contiguous(), 12, (v, kind, step, "the last beam first"))
    ops.check()
