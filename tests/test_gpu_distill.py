"""`-m gpu`: distillation's loss and gradient against their 64-bit form, over types, lengths, lists, masks and strides."""
import pytest

from tests.dense_reference import inside, rounded
from tests.logits_reference import NONE, distill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _inputs(n, v, top, kind, seed, teacher=None, rest=False, ids="int64", spread=3.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = rnd(n, v) * spread
    at = torch.argsort(torch.rand((n, v), generator=g, device="cuda"), 1)[:, :top] if v < 4096 else \
        torch.randint(0, v // max(top, 1), (n, top), generator=g, device="cuda") + torch.arange(top, device="cuda") * (v // max(top, 1))
    z = torch.sort(rnd(n, top) * 1.5 + 8, 1, descending=True).values.to(teacher or torch.float32)
    x.scatter_(1, at, z.float() - 1 + rnd(n, top))
    lse = None
    lse_of = lambda t: (torch.logsumexp(z.double() / t, 1) - torch.log(torch.rand(n, generator=g, device="cuda").double() * 0.5 + 0.45)).float()  # noqa: E731
    y = torch.randint(0, v, (n,), generator=g, device="cuda")
    if top:
        y[::2] = at[::2, top // 2]
    w = torch.rand(n, generator=g, device="cuda") + 0.5
    lse = lse_of if rest else lambda t: None
    return x.to(kind), at.to(getattr(torch, ids)).contiguous(), z, lse, y.to(getattr(torch, ids)), w


def _losses(got, want, bound, what):
    """A share of the teacher's that is left over where every id is named costs infinitely much, in both."""
    import torch
    known = torch.isfinite(want)
    assert torch.equal(got[~known].double(), want[~known]), what
    inside(got[known], want[known], bound[known], what)


def _check(ops, x, at, z, lse, y, w, t, alpha, what):
    import torch
    loss, grad, off, off_grad = distill(x, at, z, lse, y, t, alpha)
    got, stats = ops.distill_fwd(x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    _losses(got, loss, off, (what, "loss"))
    back = ops.distill_bwd(w, x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    both, grad2 = ops.distill_grad(w, x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    want = grad * w.double()[:, None]
    bound = off_grad * w.double()[:, None]
    inside(back, want, bound + rounded(want.abs() + bound, x.dtype), (what, "grad"))
    inside(grad2, want, bound + rounded(want.abs() + bound, x.dtype), (what, "grad of one call"))
    _losses(both, loss, off, (what, "loss of one call"))
    own = x.clone()
    ops.distill_bwd(w, own, at, z, stats, targets=y, temperature=t, alpha=alpha, out=own)
    assert torch.equal(own, back), what
    own = x.clone()
    l2, _ = ops.distill_grad(w, own, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha, out=own)
    assert torch.equal(own, grad2) and torch.equal(l2, both), what


KINDS = ["float32", "bfloat16", "float16"]
# vocabularies: below a vector, around vectors, wavefronts' and workgroups' shares, slices (2048 vectors of 8 or 4), odd
SIZES = [(5, 1, 1), (3, 2, 2), (7, 7, 3), (9, 8, 8), (6, 9, 4), (4, 64, 5), (5, 511, 16), (3, 1023, 64), (3, 1025, 1), (2, 4096, 100), (3, 4099, 33), (2, 8193, 70),
         (3, 16_385, 64), (1, 50_021, 20), (2, 131_073, 257), (1, 1, 0), (3, 700, 0), (1, 300_007, 1024),
         (2, 7001, 8), (2, 14_003, 5), (3, 28_003, 9)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,v,top", SIZES)
@pytest.mark.parametrize("rest", [False, True])
def test_sizes(ops, n, v, top, kind, rest):
    import torch
    k = getattr(torch, kind)
    x, at, z, lse, y, w = _inputs(n, v, top, k, v + top, rest=rest)
    for t, alpha in ((1.0, 1.0), (2.0, 0.5), (0.7, 0.9), (1.0, 0.25), (3.0, 0.0)):
        _check(ops, x, at, z, lse(t), y, w, t, alpha, (n, v, top, kind, rest, t, alpha))
    ops.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rest", [False, True])
def test_many_rows(ops, kind, rest):
    """Enough rows for the widest slices, and rows that end inside a slice and inside a vector."""
    import torch
    k = getattr(torch, kind)
    for n, v, top in ((600, 16_500, 32), (1030, 2100, 8), (4097, 70, 5)):
        x, at, z, lse, y, w = _inputs(n, v, top, k, n, teacher=k, rest=rest, ids="int32")
        _check(ops, x, at, z, lse(1.5), y, w, 1.5, 0.6, (n, v, kind, rest))
    ops.check()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("v", [90, 3000, 40_000])
def test_lists_with_gaps_repeats_and_rows_left_out(ops, v, rest):
    import torch
    n, top = 40, 24
    x, at, z, lse, y, w = _inputs(n, v, top, torch.bfloat16, v, rest=rest)
    lse = lse(2.0)
    at[0] = -1                                       # no entry
    at[1, 5:] = -1
    at[2, ::2] = -1
    at[3, :] = at[3, :1]                             # one id in every place
    at[4, 10:20] = at[4, :10]
    if rest:
        lse[3:5] = torch.logsumexp(z[3:5].double() / 2, 1).float() + 1
    y[5] = -1
    y[6], y[7] = 0, v - 1
    y[8] = at[8, 3]
    y[3] = at[3, 0]
    x[5] = float("nan")                              # the row is left out
    at[9, 0], at[9, 1] = 0, v - 1
    at[9, 2:][(at[9, 2:] == 0) | (at[9, 2:] == v - 1)] = -1
    for alpha in (1.0, 0.5):
        _check(ops, x, at, z, lse, y, w, 2.0, alpha, (v, rest, alpha))
    loss, grad = ops.distill_grad(w, x, at, z, teacher_lse=lse, targets=y, temperature=2.0, alpha=0.5)
    assert float(loss[5]) == 0 and not bool(grad[5].any())
    only, _ = ops.distill_fwd(x, at, z, teacher_lse=lse, targets=y, temperature=2.0)
    assert float(only[0]) == 0
    ops.check()


def test_ids_outside_the_vocabulary(ops):
    import torch
    from paper_2208_05321_amd import FreqCacheError
    v = 3000
    x, at, z, lse, y, w = _inputs(6, v, 8, torch.float32, 1, rest=True)
    for what in ("entry", "target"):
        a, t = at.clone(), y.clone()
        if what == "entry":
            a[1, 2], a[2, 3] = v, -2
        else:
            t[1], t[4] = v + 7, -5
        _check(ops, x, a, z, lse(1.0), t, w, 1.0, 0.5, what)
        with pytest.raises(FreqCacheError) as e:
            ops.check()
        assert e.value.name == "ID_OUT_OF_RANGE"
    ops.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rest", [False, True])
def test_masked_logits_and_extremes(ops, kind, rest):
    """Ids of probability 0 (masked by -inf, or by the type's lowest value), a named id far above and far below the others."""
    import torch
    k = getattr(torch, kind)
    for v, top in ((200, 8), (9000, 16), (40_000, 16)):
        x, at, z, lse, y, w = _inputs(12, v, top, k, v, rest=rest)
        lse = lse(2.0)
        keep = torch.zeros_like(x, dtype=torch.bool).scatter_(1, at, True)
        keep[torch.arange(12), y] = True
        x[0][~keep[0]] = NONE                        # nothing but what is named (and the target)
        x[1, ::2] = torch.where(keep[1, ::2], x[1, ::2], NONE)
        x[2, 1::2] = torch.where(keep[2, 1::2], x[2, 1::2], torch.finfo(k).min)
        x[3, at[3, 0]] = 250.0                       # the others are far below 32 bits' range of it
        x[4, at[4, 1]] = -300.0
        x[5] = 1000.0
        x[6, :v // 2] = NONE
        x[6, at[6]] = 1.0
        x[6, y[6]] = 0.5
        want = distill(x, at, z, lse, y, 2.0, 0.5)
        ok = torch.isfinite(want[0])
        loss, stats = ops.distill_fwd(x, at, z, teacher_lse=lse, targets=y, temperature=2.0, alpha=0.5)
        grad = ops.distill_bwd(w, x, at, z, stats, targets=y, temperature=2.0, alpha=0.5)
        inside(loss[ok], want[0][ok], want[2][ok], (v, kind, rest, "loss"))
        assert torch.equal(torch.isinf(loss), torch.isinf(want[0]))       # a share left over where nothing is: infinite
        ok = torch.isfinite(want[1]).all(1)
        assert int(ok.sum()) >= 11
        wd = w.double()[:, None]
        bound = (want[3] * wd)[ok]
        inside(grad[ok], (want[1] * wd)[ok], bound + rounded((want[1] * wd)[ok].abs() + bound, k), (v, kind, rest, "grad"))
    ops.check()


def test_rows_that_are_no_distribution(ops):
    import torch
    x, at, z, _, y, w = _inputs(8, 5000, 4, torch.float32, 3)
    x[0, 7] = float("nan")
    x[1, 4999] = float("inf")
    x[2] = NONE
    x[3] = float("nan")
    w[4] = 0.0
    x[4] = float("nan")
    loss, grad = ops.distill_grad(w, x, at, z, targets=y, alpha=0.5)
    assert bool(torch.isnan(loss[:5]).all()) and bool(torch.isfinite(loss[5:]).all())
    assert bool(torch.isnan(grad[:4]).all()) and bool((grad[4] == 0).all()) and bool(torch.isfinite(grad[5:]).all())
    z[5] = NONE                                      # entries of no probability: none
    x[6] = float("nan")
    at[6] = -1
    loss, grad = ops.distill_grad(w, x, at, z)
    assert float(loss[5]) == 0 and float(loss[6]) == 0 and not bool(grad[5:7].any())
    ops.check()


@pytest.mark.parametrize("kind", KINDS)
def test_strides_and_shapes(ops, kind):
    """Rows out of a wider buffer, at an odd element, results into another; leading dimensions; one weight for all rows."""
    import torch
    k = getattr(torch, kind)
    n, v, top, t, alpha = 12, 1003, 6, 2.0, 0.5
    x, at, z, lse, y, w = _inputs(n, v, top, k, 9, rest=True)
    lse = lse(t)
    wide = torch.full((n, v + 40), 77.0, dtype=k, device="cuda")
    wide[:, 5:5 + v] = x
    view = wide[:, 5:5 + v]
    out = torch.full((n, v + 3), 5.0, dtype=k, device="cuda")
    loss, stats = ops.distill_fwd(x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    grad = ops.distill_bwd(w, x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    l2, s2 = ops.distill_fwd(view, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    assert torch.equal(loss, l2) and torch.equal(stats, s2)
    ops.distill_bwd(w, view, at, z, s2, targets=y, temperature=t, alpha=alpha, out=out[:, 1:1 + v])
    assert torch.equal(out[:, 1:1 + v], grad) and bool((out[:, 0] == 5).all()) and bool((out[:, 1 + v:] == 5).all())
    l3, g3 = ops.distill_grad(w, view, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha, out=view)
    assert torch.equal(l3, loss) and torch.equal(view, grad) and bool((wide[:, :5] == 77).all()) and bool((wide[:, 5 + v:] == 77).all())
    shape = lambda q: q.view(3, 4, *q.shape[1:])  # noqa: E731
    l4, g4 = ops.distill_grad(shape(w), shape(x), shape(at), shape(z), teacher_lse=shape(lse), targets=shape(y), temperature=t, alpha=alpha)
    assert l4.shape == (3, 4) and torch.equal(l4.view(-1), loss) and torch.equal(g4.view(n, v), grad)
    one = torch.full((1,), 0.25, device="cuda")
    a = ops.distill_bwd(one.expand(n), x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    b = ops.distill_bwd(one, x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    c = ops.distill_bwd(one.expand(n).contiguous(), x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    assert torch.equal(a, b) and torch.equal(a, c)
    l5, g5 = ops.distill_grad(w[0], x[0], at[0], z[0], teacher_lse=lse[0], targets=y[0], temperature=t, alpha=alpha)
    assert l5.shape == () and torch.equal(l5, loss[0]) and torch.equal(g5, grad[0])
    ops.check()


def test_no_rows(ops):
    import torch
    x, at, z, _, y, w = _inputs(1, 100, 4, torch.float32, 3)
    loss, grad = ops.distill_grad(w[:0], x[:0], at[:0], z[:0], targets=y[:0], alpha=0.5)
    assert loss.shape == (0,) and grad.shape == (0, 100)


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(ops, rest):
    """The loss itself, at logits moved by a step; f32 losses of about 3 with errors of 1e-6 over steps of 0.02 and third derivatives below 1."""
    import torch
    v, t, alpha = 300, 1.5, 0.6
    x, at, z, lse, y, _ = _inputs(1, v, 12, torch.float32, 4, rest=rest)
    lse = lse(t)
    w = torch.ones(1, device="cuda")
    _, grad = ops.distill_grad(w, x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    h = 0.02
    moved = torch.cat([x + h * torch.eye(v, device="cuda"), x - h * torch.eye(v, device="cuda")])
    many = lambda q: None if q is None else q.expand(2 * v, *q.shape[1:]).contiguous()  # noqa: E731
    loss, _ = ops.distill_fwd(moved, many(at), many(z), teacher_lse=many(lse), targets=many(y), temperature=t, alpha=alpha)
    diff = (loss[:v] - loss[v:]).double() / (2 * h)
    _, _, off, _ = distill(moved, many(at), many(z), many(lse), many(y), t, alpha)
    bound = off.view(2, v).sum(0) / (2 * h) + h * h / 6
    inside(grad[0], diff, bound, "differences")
