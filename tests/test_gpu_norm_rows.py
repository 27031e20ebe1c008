"""`-m gpu`: the norm's backward pass with more rows than workgroups, so that each goes through several, for every kind of row: a row's gradient is the one that it has
in a call with few rows, bit for bit, also where it takes the place of an input."""
import pytest

from tests.dense_reference import U32, inside, norm_parts, norm_steps

pytestmark = pytest.mark.gpu
# narrow rows, several to a workgroup; two vectors a lane; a workgroup a row with one, two and more; rows too wide for registers; whole vectors and not
SHAPES = [("bfloat16", 70_000, 40), ("float32", 70_001, 3), ("bfloat16", 9001, 1001), ("bfloat16", 9001, 1024), ("float32", 9001, 511), ("float32", 2100, 777), ("bfloat16", 2100, 2056), ("bfloat16", 2100, 2049),
          ("float32", 2100, 2049), ("float16", 2100, 4100), ("float16", 2100, 4101), ("bfloat16", 2100, 8200), ("bfloat16", 2100, 9001), ("float32", 1100, 8200), ("float32", 2100, 8193),
          ("float16", 1100, 16_400), ("bfloat16", 1100, 16_391)]


@pytest.mark.parametrize("kind,n,d", SHAPES)
@pytest.mark.parametrize("add", [False, True])
def test_many_rows(kind, n, d, add):
    import torch
    from paper_2208_05321_amd import DenseOps
    kind, ops = getattr(torch, kind), DenseOps()
    g = torch.Generator(device="cuda").manual_seed(n + d)
    h, dy, dh = (torch.randn((n, d), generator=g, device="cuda").to(kind) for _ in range(3))
    w = 1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")
    part = lambda t, k: t[k:k + 500] if add else None  # noqa: E731
    want = torch.cat([ops.rms_norm_bwd(dy[k:k + 500], h[k:k + 500], w, grad_h=part(dh, k), eps=1e-5)[0] for k in range(0, n, 500)])
    dx, dw = ops.rms_norm_bwd(dy, h, w, grad_h=dh if add else None, eps=1e-5)
    assert torch.equal(dx, want)
    _, hd, rho, _ = norm_parts(h, None, w, 1e-5)
    terms = dy.double() * hd * rho
    # a term is added to those of its workgroup's rows (n / 1024 at most), to the sums of up to 32 groups of lanes, 64 workgroups and 16 parts
    inside(dw, terms.sum(0), 1.01 * U32 * (-(-n // 1024) + 32 + 64 + 16 + norm_steps(d) / 2 + 8) * terms.abs().sum(0), "grad_weight")
    for into in ("grad_y", "grad_h") if add else ("grad_y",):
        a, b = dy.clone(), dh.clone()
        got = ops.rms_norm_bwd(a, h, w, grad_h=b if add else None, eps=1e-5, out=a if into == "grad_y" else b)
        assert torch.equal(got[0], want) and torch.equal(got[1], dw), into
    ops.close()
