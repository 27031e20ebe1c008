"""`-m gpu`: root-mean-square norm, forward and backward, against plain 64-bit forms.

Bounds: a row's sum of squares has positive terms, each added norm_steps(dim) times at most, so it is off by that many u, u = 2^-24; the root's
reciprocal by half of it and 4 u (mean, eps, two for the reciprocal root); y by two products more.  In 8 bits the quotient t = y / s is rounded by 2^-4 |t|
(3 bits of mantissa) or 2^-10 (half the smallest step), or by half a unit.  The backward sums have terms of either sign: their error counts by the sum of absolute values."""
import itertools

import pytest

from tests.dense_reference import U, U32, inside, norm_parts, norm_steps, rounded

pytestmark = pytest.mark.gpu
FLOATS = ("float32", "bfloat16", "float16")
# every number of lanes and vectors a lane, whole vectors and not, few rows and many, rows too wide for registers
SHAPES = [(1, 1), (3, 8), (2, 17), (700, 40), (5, 64), (9, 128), (100, 333), (10, 512), (600, 1024), (7, 1111), (513, 2048), (3, 2048), (2, 4096), (515, 4096), (3, 5001), (4, 8192), (520, 8192),
          (2, 16_384), (2, 20_000), (3, 32_776), (2, 40_001)]


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _inputs(torch, n, d, kind, wkind, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * d + n + seed)
    x = torch.randn((n, d), generator=g, device="cuda")
    x[:, ::max(1, d // 4)] *= 20.0
    r = torch.randn((n, d), generator=g, device="cuda")
    w = 1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")
    return x.to(kind), r.to(kind), w.to(wkind), g


def _kinds(torch, kind, wide):
    kind = getattr(torch, kind)
    return kind, torch.float32 if wide else kind


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("kind,wide", [("float32", True), ("bfloat16", True), ("bfloat16", False), ("float16", False)])
@pytest.mark.parametrize("add", [False, True])
def test_forward(ops, n, d, kind, wide, add):
    import torch
    kind, wkind = _kinds(torch, kind, wide)
    x, r, w, _ = _inputs(torch, n, d, kind, wkind)
    h, _, _, want = norm_parts(x, r if add else None, w, 1e-5)
    y, got_h, scales = ops.rms_norm_fwd(x, w, residual=r if add else None, eps=1e-5)
    assert scales is None and torch.equal(got_h, h) and (got_h is x) == (not add)
    rel = (norm_steps(d) / 2 + 6) * U32 * 1.01
    inside(y, want, rel * want.abs() + 1.01 * rounded(want, kind), "y")


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("kind", FLOATS)
@pytest.mark.parametrize("q,group", itertools.product(("float8_e4m3fn", "int8"), (0, 32, 64, 128, 256)))
def test_forward_in_8_bits(ops, n, d, kind, q, group):
    import torch
    kind, q = getattr(torch, kind), getattr(torch, q)
    x, r, w, _ = _inputs(torch, n, d, kind, torch.float32)
    h, _, _, want = norm_parts(x, r, w, 1e-5)
    y, got_h, scales = ops.rms_norm_fwd(x, w, residual=r, eps=1e-5, out_dtype=q, group=group)
    assert torch.equal(got_h, h) and y.dtype == q
    width, most = group or d, 448.0 if q == torch.float8_e4m3fn else 127.0
    rel = (norm_steps(d) / 2 + 10) * U32 * 1.01
    s = torch.stack([p.abs().amax(1) for p in want.split(width, 1)], 1) / most
    inside(scales, s, rel * s, "scales")
    each = scales.double().repeat_interleave(width, 1)[:, :d]
    step = each * torch.maximum((want / each).abs() * 2.0 ** -4, torch.full_like(want, 2.0 ** -10)) if most == 448.0 else each * 0.5
    inside(y.float().double() * each, want, 1.001 * step + rel * want.abs(), "values")
    assert float(y.float().abs().amax()) == most


@pytest.mark.parametrize("kind", FLOATS)
@pytest.mark.parametrize("q", ["float8_e4m3fn", "int8"])
def test_8_bits_of_zeros_and_of_what_is_no_number(ops, kind, q):
    import torch
    kind, q = getattr(torch, kind), getattr(torch, q)
    x = torch.randn(6, 96, device="cuda").to(kind)
    w = torch.ones(96, device="cuda")
    x[1] = 0.0
    x[2, :32] = 0.0
    x[3, 40] = float("nan")
    x[4, 0] = float("inf")
    w[64:] = 0.0
    y, _, s = ops.rms_norm_fwd(x, w, out_dtype=q, group=32)
    v = y.float() * s.repeat_interleave(32, 1)
    assert bool((v[1] == 0).all()) and bool((s[1] == 0).all()) and bool((v[2, :32] == 0).all()) and float(s[2, 0]) == 0 and float(s[2, 1]) > 0
    assert bool((s[[0, 1, 2, 5], 2] == 0).all()) and bool((v[[0, 5], 64:] == 0).all())
    assert bool(v[3].isnan().all())                                   # a row with one has a norm that is none
    assert float(v[5, :64].abs().amax()) > 0
    plain, _, _ = ops.rms_norm_fwd(x, w)
    assert bool(plain[3].isnan().all()) and bool(plain[4, 0].isnan()) and bool((plain[4, 1:] == 0).all()) and bool((plain[1] == 0).all())
    y, _, s = ops.rms_norm_fwd(x, w, out_dtype=q)
    assert bool(s[3].isnan().all()) and float(s[1]) == 0 and bool((y[1].float() == 0).all())


@pytest.mark.parametrize("n,d", SHAPES + [(5000, 16), (2500, 264)])
@pytest.mark.parametrize("kind,wide,gw", [("float32", True, "float32"), ("bfloat16", True, "float32"), ("bfloat16", False, "bfloat16"), ("float16", False, "float16")])
@pytest.mark.parametrize("add", [False, True])
def test_backward(ops, n, d, kind, wide, gw, add):
    import torch
    kind, wkind = _kinds(torch, kind, wide)
    gw = getattr(torch, gw)
    h, gh, w, g = _inputs(torch, n, d, kind, wkind)
    dy = torch.randn((n, d), generator=g, device="cuda").to(kind)
    _, hd, rho, _ = norm_parts(h, None, w, 1e-5)
    c = dy.double() * w.double()
    mean, size = (c * hd).mean(1, keepdim=True), (c * hd).abs().mean(1, keepdim=True)
    want = rho * c - hd * rho ** 3 * mean + (gh.double() if add else 0.0)
    dx, dw = ops.rms_norm_bwd(dy, h, w, grad_h=gh if add else None, eps=1e-5, grad_weight_dtype=gw)
    steps = norm_steps(d)
    # products and sums of 32 bits on the way; rho is off by steps / 2 + 4, its cube by three times that, the mean by steps + 4 of `size`
    bound = U32 * ((steps / 2 + 8) * (rho * c).abs() + (steps * 2.5 + 20) * hd.abs() * rho ** 3 * size + 2 * want.abs())
    inside(dx, want, 1.01 * bound + 1.01 * rounded(want, kind), "grad_x")
    terms = dy.double() * hd * rho
    total = terms.sum(0)
    inside(dw, total, 1.01 * U32 * (min(n, 2000) + steps / 2 + 30) * terms.abs().sum(0) + 1.01 * rounded(total, gw), "grad_weight")
    again = ops.rms_norm_bwd(dy, h, w, grad_h=gh if add else None, eps=1e-5, grad_weight_dtype=gw)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


def test_backward_is_the_forwards(ops):
    """Differences of the forward pass along random directions v of length 1: sum(dy * (y(h + e v) - y(h - e v))) / 2e against sum(grad * v).

    y along v: each derivative brings a factor of at most 2 / |h| (|h| > 6 here), so what the difference leaves out is at most e^2 / 6 * (2 / 6)^2 * 3 times
    sum |dy| |w|; the rounding of two results adds 2 * (steps / 2 + 8) u sum |dy y| / 2e and that of grad (steps + 20) u of the like."""
    import torch
    n, d, e = 5, 64, 0.02
    x, _, w, g = _inputs(torch, n, d, torch.float32, torch.float32)
    dy = torch.randn((n, d), generator=g, device="cuda")
    dx, dw = ops.rms_norm_bwd(dy, x, w)
    y = ops.rms_norm_fwd(x, w)[0].double()
    assert float(x.norm(dim=1).min()) > 6
    for k in range(8):
        v = torch.randn((n, d), generator=g, device="cuda")
        v /= v.norm(dim=1, keepdim=True)
        hi, lo = (ops.rms_norm_fwd(x + s * e * v, w)[0].double() for s in (1, -1))
        diff = (dy.double() * (hi - lo)).sum(1) / (2 * e)
        size = (dy.double().abs() * w.double().abs()).sum(1)
        left = e * e / 6 * (2 / 6) ** 2 * 3 * size + (norm_steps(d) + 40) * U32 * (dy.double() * y).abs().sum(1) / e + U32 * 8 * size / e
        assert bool(((diff - (dx.double() * v).sum(1)).abs() <= left).all())
        u = torch.randn(d, generator=g, device="cuda")               # the weight enters linearly: its difference is exact
        off = (dy.double() * ops.rms_norm_fwd(x, u)[0].double()).sum() - (dw.double() * u).sum()
        assert abs(float(off)) <= float((norm_steps(d) + 40) * U32 * (dy.double() * y / w * u).abs().sum())


@pytest.mark.parametrize("kind", FLOATS)
@pytest.mark.parametrize("n,d", [(6, 48), (6, 50), (3, 4099), (2, 33_000)])
def test_strides_and_results_in_place(ops, kind, n, d):
    import torch
    kind = getattr(torch, kind)
    x, r, w, g = _inputs(torch, n, d, kind, torch.float32)
    dy = torch.randn((n, d), generator=g, device="cuda").to(kind)
    y0, h0, _ = ops.rms_norm_fwd(x, w, residual=r)
    dx0, dw0 = ops.rms_norm_bwd(dy, h0, w, grad_h=r)
    q0, _, s0 = ops.rms_norm_fwd(x, w, residual=r, out_dtype=torch.float8_e4m3fn, group=32)

    def spread(t):
        big = torch.full((n, d + 13), 5.0, device="cuda").to(t.dtype)
        big[:, 3:3 + d] = t
        return big[:, 3:3 + d]
    y, h = spread(y0 * 0), spread(h0 * 0)
    ops.rms_norm_fwd(spread(x), w, residual=spread(r), h_out=h, out=y)
    assert torch.equal(y, y0) and torch.equal(h, h0)
    q, _, s = ops.rms_norm_fwd(spread(x), w, residual=spread(r), out_dtype=torch.float8_e4m3fn, group=32)
    assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(s, s0)
    dx = spread(dx0 * 0)
    _, dw = ops.rms_norm_bwd(spread(dy), spread(h0), w, grad_h=spread(r), out=dx)
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0)
    for into in ("x", "residual"):                                   # h takes the place of what it is the sum of
        a, b = x.clone(), r.clone()
        y, h, _ = ops.rms_norm_fwd(a, w, residual=b, h_out=a if into == "x" else b)
        assert h is (a if into == "x" else b) and torch.equal(h, h0) and torch.equal(y, y0)
        a, b = x.clone(), r.clone()
        q, h, s = ops.rms_norm_fwd(a, w, residual=b, h_out=a if into == "x" else b, out_dtype=torch.float8_e4m3fn, group=32)
        assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(s, s0) and torch.equal(h, h0)
    for into in ("grad_y", "grad_h"):
        a, b = dy.clone(), r.clone()
        dx, dw = ops.rms_norm_bwd(a, h0, w, grad_h=b, out=a if into == "grad_y" else b)
        assert torch.equal(dx, dx0) and torch.equal(dw, dw0)


def test_leading_dimensions_and_no_rows(ops):
    import torch
    x, w = torch.randn(2, 3, 5, 24, device="cuda"), torch.randn(24, device="cuda")
    y, _, _ = ops.rms_norm_fwd(x, w)
    assert torch.equal(y.view(-1, 24), ops.rms_norm_fwd(x.view(-1, 24), w)[0])
    _, _, s = ops.rms_norm_fwd(x, w, out_dtype=torch.int8)
    assert s.shape == (2, 3, 5, 1)
    dx, dw = ops.rms_norm_bwd(x, x, w)
    assert dx.shape == x.shape and dw.shape == (24,)
    none = torch.empty(0, 24, device="cuda")
    assert ops.rms_norm_fwd(none, w)[0].shape == (0, 24)
    dx, dw = ops.rms_norm_bwd(none, none, w)
    assert dx.shape == (0, 24) and bool((dw == 0).all())
    assert U[torch.float32] == U32
