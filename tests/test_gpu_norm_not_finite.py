"""`-m gpu`: 8-bit results of finite rows whose products with the weight are not: the scale says so, the values are what include/freqcache.h states, and other
groups and rows are what they are without."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("q", ["float8_e4m3fn", "int8"])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("n,d", [(5, 96), (3, 333), (2, 1111), (600, 2048), (2, 4096), (2, 40_001)])
def test_scales_and_values(kind, q, group, n, d):
    import math
    import torch
    from paper_2208_05321_amd import DenseOps
    ops, f8 = DenseOps(), q == "float8_e4m3fn"
    kind, q = getattr(torch, kind), getattr(torch, q)
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(n, d, generator=g, device="cuda").to(kind)
    x[:, 40] = 2.0 * d ** 0.5                                     # its share of the norm is at least 4 of 5: more than 1.7 after it
    x[1, 40] *= -1
    w = torch.ones(d, device="cuda")
    usual, _, usual_scales = ops.rms_norm_fwd(x, w, out_dtype=q, group=group)
    width = group or d
    at, lo = 40 // width, 40 // width * width
    hi = min(d, lo + width)
    others = [c for c in range(usual_scales.shape[1]) if c != at]
    for value in (3e38, math.inf, math.nan):
        w[40] = value
        assert bool(x.isfinite().all())
        y, _, scales = ops.rms_norm_fwd(x, w, out_dtype=q, group=group)
        assert bool((scales[:, at].isnan() if value != value else scales[:, at] == math.inf).all())
        inside, there = y[:, lo:hi].float(), torch.arange(lo, hi, device="cuda") == 40
        if not f8:
            assert bool((inside == 0).all())
        elif value != value:
            assert bool(inside.isnan().all())
        else:
            assert bool(inside[:, there].isnan().all()) and bool((inside[:, ~there] == 0).all())
        assert torch.equal(scales[:, others], usual_scales[:, others])
        rest = torch.ones(d, dtype=torch.bool, device="cuda")
        rest[lo:hi] = False
        assert torch.equal(y.view(torch.uint8)[:, rest], usual.view(torch.uint8)[:, rest])
    ops.close()
