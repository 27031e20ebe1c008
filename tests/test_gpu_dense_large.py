"""`-m gpu`: calls whose rows need more threads than one launch can have."""
import pytest

pytestmark = pytest.mark.gpu
GIB = 1 << 30


@pytest.fixture(scope="module")
def ops():
    import torch

    from paper_2208_05321_amd import DenseOps
    if torch.cuda.mem_get_info()[0] < 64 * GIB:
        pytest.skip("64 GiB of device memory")
    o = DenseOps()
    yield o
    o.check()
    o.close()
    torch.cuda.empty_cache()


def test_lookup_of_many_narrow_rows(ops):
    import torch
    n = (1 << 29) + 3                                   # 4 threads a token
    table = torch.randn(10, 7, device="cuda").to(torch.bfloat16)
    ids = torch.arange(n, device="cuda", dtype=torch.int32).remainder_(10)
    out = ops.token_embed_fwd(table, ids)
    assert out.shape == (n, 7) and torch.equal(out[:10], table) and torch.equal(out[10:], out[:-10])


def test_norm_of_many_narrow_rows(ops):
    import torch
    n = (1 << 28) + 5                                   # 8 threads a row
    x = (torch.arange(n, device="cuda", dtype=torch.int32).remainder_(97) + 1).to(torch.float16).div_(16).view(n, 1)
    w = torch.full((1,), 1.5, device="cuda")
    y, _, _ = ops.rms_norm_fwd(x, w, eps=1.0)
    x64 = x[:97].double()
    want = x64 / (x64 * x64 + 1).sqrt() * 1.5
    # one rounding to 11 bits of a value that 32-bit steps worked out to within 6 of their units
    assert ((y[:97].double() - want).abs() <= want * (2.0 ** -11 + 6 * 2.0 ** -24)).all()
    assert torch.equal(y[97:], y[:-97])


def test_zeros_of_many_rows_apart(ops):
    import torch
    rows = (1 << 30) + 3                                # 2 threads a row
    flat = torch.ones(rows * 10, dtype=torch.float16, device="cuda")
    grad = flat.view(rows, 10)[:, :9]
    ids = torch.tensor([rows - 1, 0, 1 << 30, rows - 1], device="cuda")
    g = torch.tensor([1.0, 2.0, 3.0, 4.0], device="cuda", dtype=torch.float16).view(4, 1).expand(4, 9).contiguous()
    ops.token_embed_bwd(g, ids, rows, grad=grad)
    used = 0
    for at in range(0, rows, 1 << 26):
        part = flat.view(rows, 10)[at:at + (1 << 26)]
        used += int((part[:, :9] != 0).any(1).sum())
        assert bool((part[:, 9] == 1).all())
    assert used == 3
    assert bool((grad[rows - 1] == 5).all()) and bool((grad[0] == 2).all()) and bool((grad[1 << 30] == 3).all())


def test_gradient_of_too_many_elements_is_refused(ops):
    from paper_2208_05321_amd.binding import load_library
    a = 1 << 20                                         # (addresses that a refused call does not look at)
    assert load_library().token_embed_bwd(ops._h, a, 0, 64, a, 6, 1 << 30, 8, 64, 1.0, -1, a, 0, 64, 0) == -1
