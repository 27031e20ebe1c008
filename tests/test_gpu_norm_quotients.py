"""`-m gpu`: 8-bit results are those of a division: rows of ones and minus ones have a norm of one, so that y is the weight and its sign, bit for bit, and the weights lie
in the middle between two 8-bit values, as near as 32 bits allow."""
import pytest

pytestmark = pytest.mark.gpu


def _middles(torch, most, n, g):
    """n of the middles between neighbouring 8-bit values up to `most`."""
    if most == 127.0:
        return torch.randint(0, 127, (n,), generator=g) + 0.5
    values = torch.arange(0, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    return ((values[1:] + values[:-1]) / 2)[torch.randint(0, len(values) - 1, (n,), generator=g)]


@pytest.mark.parametrize("q,most", [("int8", 127.0), ("float8_e4m3fn", 448.0)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("n,d", [(3, 96), (2, 1111), (600, 1024), (3, 4096), (600, 4096), (2, 40_001)])
def test_middles(q, most, kind, group, n, d):
    import torch
    from paper_2208_05321_amd import DenseOps
    ops, q, kind = DenseOps(), getattr(torch, q), getattr(torch, kind)
    g = torch.Generator().manual_seed(d + group)
    x = torch.randint(0, 2, (n, d), generator=g) * 2.0 - 1.0
    x[0, ::5] *= -1
    width = group or d
    parts = []
    for at in range(0, d, width):
        top = torch.rand(1, generator=g) + 1.0                                     # the largest of the group
        w = (_middles(torch, most, min(width, d - at), g) * (top / most).double()).float()
        w[0] = top
        parts.append(w)
    w = torch.cat(parts)
    y = x * w
    scales = torch.stack([p.abs().amax(1) / most for p in y.split(width, 1)], 1)
    t = (y / scales.repeat_interleave(width, 1)[:, :d]).clamp(-most, most)
    want = t.round().to(torch.int8) if most == 127.0 else t.to(torch.float8_e4m3fn)
    dx, dw = x.to(kind).cuda(), w.cuda()
    if kind == torch.float32:
        assert torch.equal(ops.rms_norm_fwd(dx, dw, eps=0.0)[0].cpu(), y)           # what the test stands on
    got, _, got_scales = ops.rms_norm_fwd(dx, dw, eps=0.0, out_dtype=q, group=group)
    assert torch.equal(got_scales.cpu(), scales)
    assert torch.equal(got.cpu().float(), want.float())
    ops.close()


@pytest.mark.parametrize("q", ["int8", "float8_e4m3fn"])
def test_signs_of_zeros_and_the_smallest_scales(q):
    import torch
    from paper_2208_05321_amd import DenseOps
    ops, q = DenseOps(), getattr(torch, q)
    most = 127.0 if q == torch.int8 else 448.0
    x = torch.ones(1, 160, device="cuda")
    x[0, 1::2] = -1.0
    w = torch.ones(160, device="cuda")
    w[4:8] = 0.0                                       # zeros of either sign
    w[32:64] = 0.0
    w[64:96] = 1.2e-38 * most                          # a scale just above the least one
    w[96:128] = 1.1e-38 * most                         # and just below
    w[128:160] = 3e38
    y, _, s = ops.rms_norm_fwd(x, w, eps=0.0, out_dtype=q, group=32)
    y = y.float()[0]
    sign = x[0]
    assert torch.equal(y[:4], sign[:4] * most) and torch.equal(y[8:32], sign[8:32] * most) and bool((y[4:8] == 0).all()) and bool((y[32:64] == 0).all())
    assert torch.equal(y[64:96], sign[64:96] * most) and bool((y[96:128] == 0).all()) and torch.equal(y[128:], sign[128:] * most)
    if q != torch.int8:
        assert torch.equal(y[4:8].signbit(), sign[4:8] < 0) and torch.equal(y[32:64].signbit(), sign[32:64] < 0)
    assert float(s[0, 1]) == 0 and float(s[0, 0]) > 0 and bool(s.isfinite().all())
    ops.close()
