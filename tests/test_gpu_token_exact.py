"""`-m gpu`: the token gradient on whole numbers.  Every partial sum is below 2^24 and the scale is a power of two, so every order of additions in 32 bits gives
the same result, and it is compared bit for bit: a token that is lost or counted twice shows in a row of 300,000 as it does in one of three.  No number
is zero."""
import itertools

import pytest

pytestmark = pytest.mark.gpu
TYPES = [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32")]


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.check()
    o.close()


def _odd(torch, n, dim, kind, g):
    """-7, -5 .. 7"""
    return (torch.randint(0, 8, (n, dim), generator=g, device="cuda") * 2 - 7).to(kind)


def _sums(torch, ids, grad_out, rows):
    """Running sums of the sorted tokens, and their differences between the runs' ends: exact in 64 bits."""
    run = torch.zeros((grad_out.shape[1], len(ids) + 1), dtype=torch.float64, device="cuda")
    torch.cumsum(grad_out[torch.argsort(ids)].double().T.contiguous(), 1, out=run[:, 1:])
    ends = torch.bincount(ids, minlength=rows).cumsum(0)
    return torch.diff(run[:, ends], dim=1, prepend=run[:, :1]).T.contiguous()


def _check(torch, ops, ids, grad_out, rows, dst, padding, what):
    keep = ids != padding
    want = _sums(torch, ids[keep], grad_out[keep], rows)
    assert float(want.abs().max()) < 2 ** 23
    got = ops.token_embed_bwd(grad_out, ids, rows, scale=0.5, padding_id=padding, grad_dtype=dst)
    assert torch.equal(got, (want * 0.5).float().to(dst)), what
    old = torch.arange(rows * grad_out.shape[1], device="cuda").remainder_(251).view(rows, -1).to(dst)
    added = ops.token_embed_bwd(grad_out, ids, rows, scale=2.0, padding_id=padding, grad=old.clone(), accumulate=True)
    assert torch.equal(added, (want * 2.0 + old.double()).float().to(dst)), (what, "added")


# rows, columns, tokens, share of them that has one id
CASES = [(1, 8, 9000, 0.0), (1, 1, 1024, 0.0), (5, 12, 4097, 1.0), (3, 24, 80_000, 0.9), (1, 16, 300_001, 0.0), (2, 3, 270_000, 0.5), (40, 64, 32_767, 0.4), (40, 64, 32_768, 0.4),
         (40, 64, 65_535, 0.4), (40, 64, 65_536, 0.4), (999, 257, 12_288, 0.7), (7, 2050, 10_241, 0.6), (2, 1030, 66_000, 0.9), (500, 7, 140_001, 0.3), (20, 4100, 1023, 0.3),
         (1000, 33, 1024, 0.5), (1000, 33, 1025, 0.5), (100_000, 16, 1000, 0.2), (60_001, 1030, 700, 0.2), (120_000, 512, 2000, 0.2), (9000, 1001, 9001, 0.05)]


@pytest.mark.parametrize("rows,dim,tokens,hot", CASES)
@pytest.mark.parametrize("src,dst", TYPES)
def test_popular_rows(ops, rows, dim, tokens, hot, src, dst):
    import torch
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(tokens + dim)
    ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    ids = torch.where(torch.rand(tokens, generator=g, device="cuda") < hot, rows // 2, ids)
    grad_out = _odd(torch, tokens, dim, src, g)
    for padding in (-1, 0):
        _check(torch, ops, ids, grad_out, rows, dst, padding, padding)


# a run of sorted tokens that begins and ends on and beside multiples of 4096 (and of 16 and 256), between short ones; fewer tokens than what is
# summed by 4096 from, as many, and more
@pytest.mark.parametrize("n", [65_535, 65_536, 70_001])
@pytest.mark.parametrize("dim,src,dst", [(3, "float32", "float32"), (7, "float32", "float32"), (24, "bfloat16", "float32"), (262, "bfloat16", "float32"), (40, "float16", "float16")])
def test_borders_of_a_long_run(ops, n, dim, src, dst):
    import torch
    src, dst = getattr(torch, src), getattr(torch, dst)
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    grad_out = _odd(torch, n, dim, src, g)
    at = torch.arange(n, device="cuda")
    for k, (before, after) in enumerate(itertools.product((-257, -17, -1, 0, 1, 16), (-256, -16, -1, 0, 1, 17))):
        begin, end = 2 * 4096 + before, (4, 11, 15)[k % 3] * 4096 + after
        keys = torch.where(at < begin, at // 3, torch.where(at < end, 3000, 3001 + (at - end) // 2))       # (8193 / 3 < 3000)
        ids = keys[torch.randperm(n, generator=g, device="cuda")]
        _check(torch, ops, ids, grad_out, int(keys[-1]) + 2, dst, 3000 if k % 7 == 3 else -1, (begin, end))
