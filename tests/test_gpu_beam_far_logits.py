"""`-m gpu`: beam search's selection where finite logits are far from zero: ids masked by -1e10 or by the type's lowest value, beams of which nothing else is left, single huge logits."""
import math

import pytest

from tests.dense_reference import U32
from tests.logits_reference import NONE
from tests.test_gpu_beam_offsets import STEPS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _check(ops, x, scores, keep, what):
    """In 64 bits; equal candidates: lower beam, larger logit, lower id (beside a logit of 1e30 those of all others are equal)."""
    import torch
    b, w, v = x.shape
    order = torch.sort(x.double(), dim=2, descending=True, stable=True).indices
    c = (torch.log_softmax(x.double(), 2) + scores.double()[:, :, None]).gather(2, order).view(b, w * v)
    c = torch.where(torch.isfinite(scores)[:, :, None].expand(b, w, v).reshape(b, w * v), c, NONE)
    best, at = torch.sort(c, dim=1, descending=True, stable=True)
    best, at = best[:, :keep], at[:, :keep]
    none = best == NONE
    got, parents, tokens, _ = ops.beam_select(x, scores, keep)
    assert torch.equal(parents, torch.where(none, 0, at // v).int()), what
    assert torch.equal(tokens, torch.where(none, 0, order.view(b, w * v).gather(1, at))), what
    known = best.float() > NONE                      # (below the lowest number of 32 bits a score is stored as -infinity)
    assert torch.equal(known, got > NONE), what
    off = (STEPS + math.log(v) + best.abs()) * U32   # (derived beside STEPS)
    assert bool(((got.double() - best).abs() <= off)[known].all()), (what, float((got.double() - best).abs()[known].max()))


@pytest.mark.parametrize("kind,mask", [(k, m) for k in ("float32", "bfloat16") for m in (-1e4, -1e9, -3e9, -1e10, -1e20, -1e30, -2.4e38, "lowest")] +
                         [("float16", -1e4), ("float16", "lowest")])
@pytest.mark.parametrize("v,keep", [(6, 6), (700, 16), (40_000, 16)])
def test_finite_masks(ops, v, keep, kind, mask):
    import torch
    k = getattr(torch, kind)
    m = float(torch.finfo(k).min) if mask == "lowest" else mask
    g = torch.Generator(device="cuda").manual_seed(v)
    x = (torch.randn((5, 4, v), generator=g, device="cuda") * 3).to(k)
    scores = torch.sort(-6 * torch.rand((5, 4), generator=g, device="cuda"), 1, descending=True).values
    few = torch.zeros(v, dtype=torch.bool, device="cuda")
    few[torch.randint(0, v, (3,), generator=g, device="cuda")] = True
    x[0, 1] = m                                      # nothing is allowed here
    x[1] = m                                         # nor anywhere in this sequence
    x[2] = torch.where(few, x[2], m)                 # three ids, or fewer
    x[3, :, :v // 2] = m                             # whole lanes, wavefronts and slices
    x[4, :, v // 3:] = m
    _check(ops, x, scores, keep, (v, kind, m))
    one = scores.clone()
    one[:, 0], one[:, 2:] = NONE, NONE
    _check(ops, x, one, keep, (v, kind, m, "one beam"))
    ops.check()


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("v", [6, 700, 40_000])
def test_huge_logits(ops, v, kind):
    import torch
    k = getattr(torch, kind)
    g = torch.Generator(device="cuda").manual_seed(v)
    for far in (1e5, 3e7, 1e9, 3e9, 1e10, 1e30, 3.3e38):
        x = (torch.randn((6, 3, v), generator=g, device="cuda") * 3).to(k)
        scores = torch.sort(-6 * torch.rand((6, 3), generator=g, device="cuda"), 1, descending=True).values
        x[0, 1, v // 2] = far                        # one logit above all
        x[1, 0] = far                                # all of them
        x[2, 2, v // 3:] = far
        x[3] = (far * (1 - 0.5 * torch.rand((3, v), generator=g, device="cuda"))).to(k)      # far apart from one another
        x[4] = (-far * (1 - 0.5 * torch.rand((3, v), generator=g, device="cuda"))).to(k)
        x[5, :, 0], x[5, :, 1:] = far, -far
        _check(ops, x, scores, 6, (v, kind, far))
    ops.check()


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_what_is_no_number_stays_so(ops, kind):
    """Beside far logits too: a beam with +infinity or NaN has no candidates, one of -infinity only neither."""
    import torch
    k = getattr(torch, kind)
    low = float(torch.finfo(k).min)
    for v in (700, 40_000):
        x = torch.full((1, 4, v), low, dtype=k, device="cuda")
        x[0, 0, v // 2], x[0, 1, v - 1], x[0, 2] = float("inf"), float("nan"), NONE
        scores = torch.zeros((1, 4), device="cuda")
        got, parents, tokens, _ = ops.beam_select(x, scores, 5)
        assert parents.tolist() == [[3] * 5] and tokens.tolist() == [list(range(5))]
        assert bool(((got.double() + math.log(v)).abs() <= (STEPS + 2 * math.log(v)) * U32).all())
    ops.check()
