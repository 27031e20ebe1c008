"""`-m gpu`: the global norm of a list of tensors and clipping by it, against 64 bits.  The sum is kept in 64 bits: the norm is off by its rounding to 32, a
product by the factor's, its own and the stored type's."""
import math

import pytest

from tests.dense_reference import U32, inside, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _tensors(torch, sizes, kinds, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(len(sizes) + sum(sizes) % 1000)
    return [(torch.randn(n, generator=g, device="cuda") * spread).to(getattr(torch, kinds[k % len(kinds)])) for k, n in enumerate(sizes)]


def _exact(grads, max_norm):
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


# one element; a tile of 8192 and its neighbours; empty tensors among them; as many as a launch describes, more, and many more
SIZES = [[1], [8191, 8192, 8193], [0, 5, 0, 0, 70_001], [16_384] * 3 + [1], [3] * 119, [3] * 120, [17] * 121, [5, 0] * 120 + [9], list(range(241)), [40] * 700, [5_000_003, 12, 1_000_001]]
KINDS = [("float32",), ("bfloat16",), ("float16",), ("float32", "bfloat16", "float16")]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kinds", KINDS, ids="-".join)
@pytest.mark.parametrize("share", [0.3, 2.0])
def test_clip(ops, sizes, kinds, share):
    import torch
    grads = _tensors(torch, sizes, kinds)
    norm, _ = _exact(grads, 1.0)
    most = share * norm
    _, factor = _exact(grads, most)
    before = [g.clone() for g in grads]
    out = [torch.empty_like(g) for g in grads]
    got = ops.grad_norm_clip(grads, most, out=out)
    assert got.shape == (1,) and abs(float(got) - norm) <= 1.01 * U32 * norm
    for g, b, o in zip(grads, before, out):
        assert torch.equal(g, b)
        want = g.double() * factor
        inside(o, want, 1.01 * (2 * U32 * want.abs() + rounded(want, g.dtype)), "clipped")
        if share > 1:
            assert torch.equal(o, g)
    assert torch.equal(ops.grad_norm_clip(grads, most), got)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))                     # in place: the same values


def test_views_at_any_element(ops):
    import torch
    flat = torch.randn(200_000, device="cuda").bfloat16()
    cuts = [1, 2, 7, 8, 1003, 9000, 50_001]
    grads, at = [], 3
    for n in cuts:
        grads.append(flat[at:at + n])
        at += n + 1
    norm, factor = _exact(grads, 1.0)
    want = flat.clone()
    at = 3
    for n in cuts:
        want[at:at + n] = (flat[at:at + n].float() * torch.tensor(factor, dtype=torch.float32, device="cuda")).bfloat16()
        at += n + 1
    ops.grad_norm_clip(grads, 1.0)
    assert torch.equal(flat, want)                                                # the elements between them are left alone


def test_large_and_small_values(ops):
    import torch
    for size in (1e30, 1e-30):                                                    # squares beyond 32 bits, either way
        g = torch.full((1000,), size, device="cuda")
        got = ops.grad_norm_clip([g], 1.0)
        norm = float(torch.tensor(size).double()) * math.sqrt(1000)
        assert abs(float(got) - norm) <= 1.01 * U32 * norm
        assert float(g[0]) == pytest.approx(min(1.0, 1.0 / (norm + 1e-6)) * size, rel=4 * U32)
    g = [torch.full((100,), 2e38, device="cuda"), torch.ones(3, device="cuda")]
    assert math.isinf(float(ops.grad_norm_clip(g, 1.0)))                          # 2e39: beyond the norm's type, not beyond the factor's
    assert float(g[0][0]) == pytest.approx(0.1, rel=1e-6)


def test_values_that_are_no_numbers(ops):
    import torch
    a, b = torch.ones(9, device="cuda"), torch.ones(70_000, device="cuda")
    b[5] = float("inf")
    assert math.isinf(float(ops.grad_norm_clip([a, b], 1.0)))
    assert bool((a == 0).all()) and bool(b[5].isnan()) and float(b[6]) == 0
    a, b = torch.ones(9, device="cuda"), torch.ones(70_000, device="cuda")
    b[5] = float("nan")
    assert math.isnan(float(ops.grad_norm_clip([a, b], 1.0)))
    assert bool(a.isnan().all()) and bool(b.isnan().all())
    a = torch.ones(9, device="cuda")
    a[0] = float("inf")
    assert math.isinf(float(ops.grad_norm_clip([a], math.inf))) and float(a[1]) == 1          # only measured
    out = torch.empty_like(a)
    ops.grad_norm_clip([a], math.inf, out=[out])
    assert torch.equal(out, a)


def test_no_tensors(ops):
    import torch
    assert float(ops.grad_norm_clip([], 1.0)) == 0.0
    assert float(ops.grad_norm_clip([torch.empty(0, device="cuda")], 1.0)) == 0.0
    z = torch.zeros(100, device="cuda")
    assert float(ops.grad_norm_clip([z], 1.0)) == 0.0 and bool((z == 0).all())


def test_more_than_32_bits_of_elements(ops):
    import torch
    g = torch.full(((1 << 31) + 9000,), 0.5, dtype=torch.bfloat16, device="cuda")
    got = float(ops.grad_norm_clip([g, torch.ones(4, device="cuda")], 1000.0))
    norm = math.sqrt(0.25 * g.numel() + 4)
    assert abs(got - norm) <= 1.01 * U32 * norm
    want = float((torch.tensor(0.5) * torch.tensor(1000.0 / (norm + 1e-6), dtype=torch.float32)).bfloat16())
    assert all(float(g[i]) == want for i in (0, 1 << 30, (1 << 31) - 1, 1 << 31, g.numel() - 1))
