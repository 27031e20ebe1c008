"""`-m gpu`: distillation where finite logits are far from zero: ids masked by -1e10 or by the type's lowest value, all of the others among them, single huge logits."""
import pytest

from tests.dense_reference import U32, inside, rounded
from tests.logits_reference import SUM_STEPS, distill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _gradient(x, at, z, lse, y, t, alpha):
    """The gradient for a weight of 1, and its bound.  (The shares of the ids that are not named come of their own log-softmax: 64 bits do not hold the logarithm of their number beside 1e20.)  With q = Q_v, r the share of v among the ids that are not named: c q and c q_0 r by sums of SUM_STEPS roundings and exponents whose error is a unit of their distance
    from the largest element, in q's case (q |log q| is small where q is), or from the largest of the others, in r's; P by exponents in 64 bits, its sum and quotient in 32."""
    import torch
    xd, top = x.double() / t, at.shape[1]
    logq = torch.log_softmax(xd, 1)
    named = torch.zeros_like(xd).scatter_(1, at.long(), 1.0) > 0
    of = lse.double() if lse is not None else torch.logsumexp(z.double() / t, 1)
    p = torch.exp(z.double() / t - of[:, None])
    p0 = (1 - p.sum(1)).clamp(min=0) if lse is not None else torch.zeros_like(of)
    rel_p = (10 + (z.double() / t).amax(1).sub(of).abs() + top / 64 + 8) * U32 + (z.double() / t).sub((z.double() / t).amax(1)[:, None]).abs().amax(1) * U32
    logr = torch.log_softmax(xd.masked_fill(named, float("-inf")), 1)
    r = logr.exp().nan_to_num(0, 0, 0)
    small = lambda e: (e.exp() * e.abs()).nan_to_num(0, 0, 0)  # noqa: E731 (q |log q|)
    off_p0 = p.sum(1) * rel_p + (top / 64 + 8) * U32 if lse is not None else torch.zeros_like(p0)
    q = logq.exp()
    c = (p.sum(1) + p0)[:, None]
    grad = alpha * t * (c * q - torch.zeros_like(xd).scatter_add_(1, at.long(), p) - p0[:, None] * r)
    off = alpha * t * (c * (q * (2 * SUM_STEPS + 40) + 4 * small(logq)) * U32 + torch.zeros_like(xd).scatter_add_(1, at.long(), p * (rel_p[:, None] + 4 * U32))
                       + off_p0[:, None] * (q + r) + p0[:, None] * (r * (SUM_STEPS + 24) + 2 * small(logr)) * U32)
    # An exponential below 2^-126 is 0; they are taken from the rounded product of the largest, off by up to 32 in the exponent before it counts as far: 2^-94 of the probability's factor.  From a product of 2^30 on only what
    # is equal to the largest counts: f32's neighbours of it are 2^-24 of it, or 64 in the exponent, away: 2^-64.
    off = off + (alpha * t * c + 1 - alpha) * 2.0 ** -64
    if alpha < 1:
        log1 = torch.log_softmax(x.double(), 1)
        hit = torch.zeros_like(xd).scatter_(1, y.long()[:, None], 1.0)
        grad = grad + (1 - alpha) * (log1.exp() - hit)
        off = off + (1 - alpha) * ((log1.exp() * (SUM_STEPS + 24) + 4 * small(log1)) + 3 * hit) * U32
    return grad, off


def _losses(got, want, bound, what):
    """Terms of 1e38 may exceed 32 bits."""
    import torch
    known = want.abs() < 1e36
    inside(got[known], want[known], bound[known], what)
    assert bool((got[~known] > 1e35).all()), what


def _check(ops, x, at, z, lse, y, w, t, alpha, what):
    import torch
    loss, _, off, _ = distill(x, at, z, lse, y, t, alpha)
    want, bound = (q * w.double()[:, None] for q in _gradient(x, at, z, lse, y, t, alpha))
    bound = 1.01 * bound + 4 * U32 * want.abs()
    bound = bound + rounded(want.abs() + bound, x.dtype)
    got, stats = ops.distill_fwd(x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    _losses(got, loss, off, (*what, "loss"))
    back = ops.distill_bwd(w, x, at, z, stats, targets=y, temperature=t, alpha=alpha)
    inside(back, want, bound, (*what, "grad"))
    both, back = ops.distill_grad(w, x, at, z, teacher_lse=lse, targets=y, temperature=t, alpha=alpha)
    _losses(both, loss, off, (*what, "loss of one call"))
    inside(back, want, bound, (*what, "grad of one call"))


def _inputs(n, v, top, kind, seed, rest, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = (3 * rnd(n, v)).to(kind)
    at = torch.randint(0, v // top, (n, top), generator=g, device="cuda") + torch.arange(top, device="cuda") * (v // top)
    z = torch.sort(1.5 * rnd(n, top) + 8, 1, descending=True).values
    lse = (torch.logsumexp(z.double() / t, 1) + 0.3).float() if rest else None
    y = torch.randint(0, v, (n,), generator=g, device="cuda")
    y[::2] = at[::2, 1]
    return x, at, z, lse, y, torch.rand(n, generator=g, device="cuda") + 0.5


@pytest.mark.parametrize("kind,far", [(k, m) for k in ("float32", "bfloat16") for m in (1e4, 1e9, 3e9, 1e10, 1e20, 1e30, 2.4e38, "most")] + [("float16", 1e4), ("float16", "most")])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("n,v,top", [(12, 200, 8), (12, 9000, 16), (12, 40_000, 16), (80, 130_500, 8)])
def test_finite_masks_and_huge_logits(ops, n, v, top, kind, far, rest):
    import torch
    k = getattr(torch, kind)
    far = float(torch.finfo(k).max) if far == "most" else far
    for t, alpha in ((1.0, 1.0), (1.0, 0.5), (2.0, 0.5), (0.7, 1.0)):
        x, at, z, lse, y, w = _inputs(n, v, top, k, v, rest, t)
        keep = torch.zeros_like(x, dtype=torch.bool).scatter_(1, at, True)
        keep[torch.arange(n), y] = True
        x[0][~keep[0]] = -far                        # all that is neither named nor the target
        x[1, :v // 2] = torch.where(keep[1, :v // 2], x[1, :v // 2], -far)        # whole lanes, wavefronts and slices
        x[2, v // 3:] = torch.where(keep[2, v // 3:], x[2, v // 3:], -far)
        x[3] = -far                                  # everything
        x[4] = far
        x[5, (at[5, 0] + 1) % v] = far               # one id
        x[6, at[6, 0]] = far                         # one that is named
        x[7, y[7]] = -far                            # the target
        x[8, at[8]] = -far                           # what is named
        x[9, at[9, 1:]] = -far
        named = torch.zeros(v, dtype=torch.bool, device="cuda").scatter_(0, at[10], True)
        x[10][~named] = -far                         # the target, unless it is named, among the others
        _check(ops, x, at, z, lse, y, w, t, alpha, (n, v, kind, far, rest, t, alpha))
    ops.check()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
def test_a_common_offset(ops, kind, rest):
    import torch
    k = getattr(torch, kind)
    for offset in (1000.0, -30_000.0) + ((1e6, -1e7) if kind != "float16" else ()):
        for n, v, top in ((6, 300, 8), (6, 50_021, 16)):
            for t, alpha in ((1.0, 0.5), (2.0, 0.5), (0.7, 1.0)):
                x, at, z, lse, y, w = _inputs(n, v, top, torch.float32, v, rest, t)
                _check(ops, (x + offset).to(k), at, z, lse, y, w, t, alpha, (kind, offset, v, rest, t, alpha))
    ops.check()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("t", [2.0 ** -10, 2.0 ** 10])
def test_the_temperatures_limits(ops, t, kind, rest):
    """Scales from a thousandth to a thousand times: where logits count as far from zero moves with them."""
    import torch
    k = getattr(torch, kind)
    for far in (30.0, 6e4) + ((1e6, 3e7, 1e12, 3e12, 1e30) if kind != "float16" else ()):
        for n, v, top in ((12, 300, 8), (12, 40_000, 16)):
            for alpha in (1.0, 0.5):
                x, at, z, lse, y, w = _inputs(n, v, top, k, v, rest, t)
                x, z = (x.float() * min(t, 1.0)).to(k), z * t        # (distances that make sense over this temperature; those of cross entropy, beside, do not matter)
                lse = (torch.logsumexp(z.double() / t, 1) + 0.3).float() if rest else None
                keep = torch.zeros_like(x, dtype=torch.bool).scatter_(1, at, True)
                keep[torch.arange(n), y] = True
                x[0][~keep[0]] = -far
                x[1, v // 3:] = torch.where(keep[1, v // 3:], x[1, v // 3:], -far)
                x[2], x[3] = -far, far
                x[4, (at[4, 0] + 1) % v] = far
                x[5, at[5, 0]] = far
                x[6] = (far * (1 + 0.01 * torch.rand(v, device="cuda"))).to(k)
                _check(ops, x, at, z, lse, y, w, t, alpha, (n, v, kind, far, rest, t, alpha))
    ops.check()
