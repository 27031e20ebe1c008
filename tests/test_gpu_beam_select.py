"""`-m gpu`: beam search's selection against a stable sort in 64 bits: sizes, ties, masks, beams that are dead or have ended."""
import pytest

from tests.dense_reference import U32
from tests.logits_reference import NONE, SUM_STEPS, select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _check(ops, x, scores, keep, finished=None, eos=-1, what=None):
    import torch
    got, parents, tokens, ended = ops.beam_select(x, scores, keep, finished=finished, eos_id=eos)
    best, p, t = select(x, scores, keep, finished, eos)
    assert torch.equal(tokens, t), what
    assert torch.equal(parents, p), what
    none = best == NONE
    assert torch.equal(none, got == NONE), what
    # the log-sum's error, the score's own rounding
    off = (SUM_STEPS + 8 + best.abs()) * U32
    assert bool(((got.double() - best).abs() <= off)[~none].all()), what
    assert (ended is None) if eos < 0 else torch.equal(ended, tokens == eos), what
    got32 = ops.beam_select(x, scores, keep, finished=finished, eos_id=eos, token_dtype=torch.int32)
    assert got32[2].dtype == torch.int32 and torch.equal(got32[2].long(), tokens) and torch.equal(got32[0], got) and torch.equal(got32[1], parents), what


def _inputs(b, w, v, kind, seed, spread=3.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((b, w, v), generator=g, device="cuda") * spread).to(kind)
    return x, torch.sort(-6 * torch.rand((b, w), generator=g, device="cuda"), 1, descending=True).values, g


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("b,w,v,keep", [(1, 1, 1, 1), (2, 1, 3, 3), (3, 2, 7, 9), (2, 4, 8, 4), (3, 5, 9, 10), (1, 4, 64, 4), (5, 3, 600, 6), (2, 8, 4097, 16),
                                        (1, 4, 131_072, 4), (3, 5, 50_021, 10), (1, 1, 300_001, 64), (70, 8, 17_000, 16), (2, 64, 2050, 64), (9, 32, 33_000, 64),
                                        (1, 3, 1 << 20, 7)])
def test_sizes(ops, b, w, v, keep, kind):
    import torch
    x, scores, _ = _inputs(b, w, v, getattr(torch, kind), b + v)
    _check(ops, x, scores, keep, what=(b, w, v, keep, kind))
    _check(ops, x, scores, 1, eos=v - 1, what=(b, w, v, kind))
    ops.check()


@pytest.mark.parametrize("v", [5, 300, 5000, 70_000])
def test_equal_candidates(ops, v):
    """Equal logits within a beam, equal beams, few distinct values, zeros of both signs: lower beam, then lower id."""
    import torch
    for keep in (1, 4, 64):
        flat = torch.zeros((2, 4, v), device="cuda")
        _check(ops, flat, torch.zeros((2, 4), device="cuda"), keep, what=("flat", v, keep))
        _check(ops, flat.half(), torch.tensor([[-1.0, -1.0, -2.0, 0.0]] * 2, device="cuda"), keep, what=("flat, scores", v, keep))
        flat[:, :, ::3] = -0.0
        _check(ops, flat, torch.zeros((2, 4), device="cuda"), keep, what=("zeros", v, keep))
        x, _, g = _inputs(1, 1, v, torch.bfloat16, v)
        x = x.expand(3, 6, v).contiguous()
        _check(ops, x, torch.full((3, 6), -2.5, device="cuda"), keep, what=("equal beams", v, keep))
        few = torch.randint(0, 3, (3, 3, v), generator=g, device="cuda").bfloat16()
        few = few[:, :1].expand(3, 3, v).contiguous()
        _check(ops, few, torch.tensor([[0.0, -1.0, -1.0]] * 3, device="cuda"), keep, what=("few values", v, keep))
        up = torch.arange(v, device="cuda", dtype=torch.float32).expand(2, 2, v).contiguous() * 1e-3
        _check(ops, up, torch.tensor([[0.0, -0.3]] * 2, device="cuda"), keep, what=("ascending", v, keep))
        _check(ops, up.flip(2).contiguous(), torch.tensor([[0.0, -0.3]] * 2, device="cuda"), keep, what=("descending", v, keep))


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_masked_ids_and_beams(ops, kind):
    import torch
    k = getattr(torch, kind)
    for v in (9, 1000, 20_000):
        x, scores, g = _inputs(6, 5, v, k, v)
        first = scores.clone()
        first[:, 1:] = NONE
        x[0, 1] = float("nan")                       # beams that are not read: their score is -inf
        _check(ops, x, first, 8, what=("first step", v))
        x[0, 1] = NONE                               # nothing is allowed here
        x[1, :, 3:] = NONE                           # fewer candidates than places, on the whole sequence
        x[2, 2] = float("inf")
        x[3, 0, v // 2] = float("nan")               # a beam that is no distribution
        x[4, :, ::2] = torch.finfo(k).min            # masked by the lowest value: candidates, far down
        scores[5, 2], scores[5, 3], scores[5, 4] = float("inf"), float("nan"), NONE
        _check(ops, x, scores, 20, what=("masked", v))
        _check(ops, x, torch.full_like(scores, NONE), 4, what=("all dead", v))
        _check(ops, x, torch.full_like(scores, NONE), 4, eos=2, what=("all dead", v))
    ops.check()


def test_beams_that_have_ended(ops):
    import torch
    for v, eos in ((4, 0), (3000, 7), (40_000, 39_999)):
        x, scores, g = _inputs(8, 6, v, torch.float32, v)
        done = torch.rand((8, 6), generator=g, device="cuda") < 0.4
        done[0], done[1] = True, False
        scores[2, 3] = NONE
        done[2, 3] = True                            # dead and ended: nothing
        x[3][done[3]] = float("nan")                 # not read
        for keep in (1, 6, 12):
            _check(ops, x, scores, keep, done, eos, (v, keep))
    ops.check()


def test_strides(ops):
    import torch
    x, scores, _ = _inputs(3, 4, 1001, torch.bfloat16, 5)
    wide = torch.full((3, 4, 1040), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, :, 3:1004] = x
    for a, b in zip(ops.beam_select(wide[:, :, 3:1004], scores, 8), ops.beam_select(x, scores, 8)):
        assert a is b or torch.equal(a, b)


def test_no_sequences(ops):
    import torch
    out = ops.beam_select(torch.empty((0, 4, 100), device="cuda"), torch.empty((0, 4), device="cuda"), 8, eos_id=3)
    assert [tuple(t.shape) for t in out] == [(0, 8)] * 4


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_many_candidates_above_the_first_bound(ops, kind):
    """Beams far apart, logits that are nearly alike, few beams alive, scores near the lowest number: thousands of candidates lie close together."""
    import torch
    k = getattr(torch, kind)
    for b, w, v, keep, spread in ((2, 32, 40_000, 64, 3.0), (1, 64, 20_011, 64, 1e-3), (3, 10, 131_072, 37, 0.05), (2, 4, 300_001, 64, 30.0)):
        x, scores, g = _inputs(b, w, v, k, keep, spread)
        what = (b, w, v, keep, kind)
        _check(ops, x, scores, keep, what=what)
        _check(ops, x, scores.flip(1).contiguous() * 20, keep, what=(*what, "the last beam"))
        _check(ops, x, scores * 1e-4, keep, what=(*what, "close"))
        one = torch.full_like(scores, NONE)
        one[:, w // 2] = -1.0
        _check(ops, x, one, keep, what=(*what, "one alive"))
        done = torch.rand((b, w), generator=g, device="cuda") < 0.5
        _check(ops, x, scores * 1e-4, keep, done, 1, what=(*what, "ended"))
    ops.check()
