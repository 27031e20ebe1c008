"""`-m gpu`: token embedding and its gradient against plain 64-bit forms: types, odd widths, strides and starting elements, few and many tokens (with
and without a sort, gradients written row by row and after a fill), popular rows around the borders of what is summed together, padding, no tokens."""
import itertools

import pytest

from tests.dense_reference import U32, embed_bound, embed_grad, inside, rounded

pytestmark = pytest.mark.gpu
FLOATS = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.check()
    o.close()


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _strided(torch, rows, dim, kind, g, pad, shift):
    """[rows, dim] whose rows are dim + pad elements apart and which starts `shift` elements into its memory."""
    flat = torch.randn(shift + rows * (dim + pad), generator=g, device="cuda").to(kind)
    return flat[shift:].view(rows, dim + pad)[:, :dim]


@pytest.mark.parametrize("src,dst", itertools.product(FLOATS, FLOATS))
@pytest.mark.parametrize("rows,dim,tokens,pad,shift", [(1, 1, 1, 0, 0), (50, 7, 3, 0, 0), (1000, 64, 513, 0, 0), (300, 1111, 70, 3, 1), (77, 2048, 5, 8, 0), (5, 4100, 9, 1, 3),
                                                       (9000, 16, 20_001, 0, 0)])
def test_lookup(ops, src, dst, rows, dim, tokens, pad, shift):
    import torch
    src, dst, g = getattr(torch, src), getattr(torch, dst), _gen(dim + tokens)
    table = _strided(torch, rows, dim, src, g, pad, shift)
    ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda", dtype=torch.int32 if tokens % 2 else torch.int64)
    want = table[ids.long()].double() * 2.75
    # one product in 32 bits, one rounding
    inside(ops.token_embed_fwd(table, ids, scale=2.75, out_dtype=dst), want, 1.01 * (rounded(want, dst) + U32 * want.abs()), "rows")
    out = _strided(torch, tokens, dim, dst, g, pad + 1, shift)
    around = out.clone()
    assert ops.token_embed_fwd(table, ids, out=out) is out
    assert torch.equal(out, table[ids.long()].float().to(dst)) and not torch.equal(out, around)


def test_lookup_shapes_and_strides_are_kept(ops):
    import torch
    table = torch.randn(40, 24, device="cuda")
    ids = torch.randint(0, 40, (3, 5), device="cuda")
    assert torch.equal(ops.token_embed_fwd(table, ids), table[ids])
    wide = torch.full((15, 30), 7.0, device="cuda")
    ops.token_embed_fwd(table, ids.view(-1), out=wide[:, 3:27])
    assert torch.equal(wide[:, 3:27], table[ids.view(-1)]) and bool((wide[:, :3] == 7).all()) and bool((wide[:, 27:] == 7).all())
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert ops.token_embed_fwd(table, none).shape == (0, 24)


def test_table_beyond_32_bits_of_elements(ops):
    import torch
    rows, dim = 1_050_000, 2050                        # 2.15e9 elements of 16 bits
    table = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, 1_047_999, rows - 1, 1_040_000], device="cuda")
    for k, i in enumerate(ids.tolist()):
        table[i] = float(k + 1)
    assert ops.token_embed_fwd(table, ids)[:, [0, -1]].tolist() == [[1.0, 1.0], [2.0, 2.0], [3.0, 3.0], [4.0, 4.0]]
    ops.token_embed_bwd(torch.ones((4, dim), dtype=torch.bfloat16, device="cuda"), ids, rows, grad=table, accumulate=True)
    assert table[ids][:, [0, -1]].tolist() == [[2.0, 2.0], [3.0, 3.0], [4.0, 4.0], [5.0, 5.0]] and float(table.sum(dtype=torch.float64)) == 14.0 * dim


# (rows, columns, tokens, share of them that has one id): single tokens; the limit of what goes without a sort; one workgroup's sort and the
# general one; chunks of 16, 256, 4096 tokens from where miles are summed on; widths of every kind; a gradient beyond 224 MB
CASES = [(1, 1, 1, 0.0), (50, 16, 1, 0.0), (3, 5, 1024, 0.0), (1000, 33, 1024, 0.5), (1000, 33, 1025, 0.5), (100_000, 16, 1024, 0.1), (20, 4100, 1023, 0.3), (2000, 130, 64, 0.0),
         (300, 1000, 5000, 0.0), (7, 2050, 10_241, 0.0), (1, 8, 9000, 0.0), (70_000, 520, 9000, 0.99), (5, 12, 4097, 1.0), (999, 257, 12_288, 0.7), (40, 64, 32_767, 0.4),
         (40, 64, 32_768, 0.4), (3, 24, 80_000, 0.9), (500, 7, 140_001, 0.05), (120_000, 512, 2000, 0.2), (60_001, 1030, 700, 0.2)]


def _inputs(torch, case, src, g, ids_kind):
    rows, dim, tokens, hot = case
    ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    ids = torch.where(torch.rand(tokens, generator=g, device="cuda") < hot, rows // 2, ids).to(ids_kind)
    return ids, torch.randn((tokens, dim), generator=g, device="cuda").to(src)


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("src,dst", [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")])
def test_gradient(ops, case, src, dst):
    import torch
    src, dst, g = getattr(torch, src), getattr(torch, dst), _gen(case[1] + case[2])
    rows, dim, tokens, _ = case
    ids, grad_out = _inputs(torch, case, src, g, torch.int32 if tokens % 2 else torch.int64)
    for padding in (-1, rows // 2):
        want, size, terms = embed_grad(ids, grad_out, rows, 0.625, padding)
        got = ops.token_embed_bwd(grad_out, ids, rows, scale=0.625, padding_id=padding, grad_dtype=dst)
        inside(got, want, embed_bound(terms, size, dst, want), f"padding {padding}")
        assert torch.equal(got, ops.token_embed_bwd(grad_out, ids, rows, scale=0.625, padding_id=padding, grad_dtype=dst))       # reproducible
        old = torch.randn((rows, dim), generator=g, device="cuda").to(dst)
        acc = old.clone()
        ops.token_embed_bwd(grad_out, ids, rows, scale=0.625, padding_id=padding, grad=acc, accumulate=True)
        inside(acc, old.double() + want, embed_bound(terms, size + old.double().abs(), dst, old.double() + want), f"added, padding {padding}")
        untouched = (terms == 0).flatten()
        assert torch.equal(acc[untouched], old[untouched])


@pytest.mark.parametrize("pad,shift", [(1, 1), (5, 0), (8, 3)])
@pytest.mark.parametrize("rows,dim,tokens", [(200, 40, 900), (200, 40, 9000), (200, 41, 3000), (300_000, 256, 2000)])
def test_gradient_strides(ops, rows, dim, tokens, pad, shift):
    import torch
    g = _gen(rows + tokens + pad)
    ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    grad_out = _strided(torch, tokens, dim, torch.bfloat16, g, pad, shift)
    flat = torch.full((shift + rows * (dim + pad),), 9.0, device="cuda")
    grad = flat[shift:].view(rows, dim + pad)[:, :dim]
    ops.token_embed_bwd(grad_out, ids, rows, grad=grad)
    want, size, terms = embed_grad(ids, grad_out, rows, 1.0)
    inside(grad, want, embed_bound(terms, size, torch.float32, want), "gradient")
    assert bool((flat[shift:].view(rows, dim + pad)[:, dim:] == 9).all()) and bool((flat[:shift] == 9).all())


@pytest.mark.parametrize("n,dim", [(1025, 8), (4096, 8), (4096, 96)])
def test_run_borders(ops, n, dim):
    """Runs whose ends lie on and beside the borders of chunks (16), blocks (64) and stretches (256)."""
    import torch
    for cut in (1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 511, 512, n - 256, n - 17, n - 16, n - 1):
        ids = (torch.arange(n, device="cuda") >= cut).long() * 2
        ids = ids[torch.randperm(n, device="cuda")]
        grad_out = torch.randn(n, dim, device="cuda")
        want, size, terms = embed_grad(ids, grad_out, 4, 1.0)
        inside(ops.token_embed_bwd(grad_out, ids, 4), want, embed_bound(terms, size, torch.float32, want), f"cut {cut}")
        acc = ops.token_embed_bwd(grad_out, ids, 4, padding_id=2, grad=torch.zeros(4, dim, device="cuda"), accumulate=True)
        want[2] = 0
        inside(acc, want, embed_bound(terms, size, torch.float32, want), f"cut {cut}, added, the second run is padding")


@pytest.mark.parametrize("tokens", [0, 3, 5000])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_nothing_but_padding(ops, tokens, kind):
    import torch
    kind = getattr(torch, kind)
    ids = torch.full((tokens,), 4, device="cuda")
    grad_out = torch.full((tokens, 12), float("nan"), dtype=kind, device="cuda")          # (what is not counted may hold anything)
    grad = torch.full((9, 12), 3.0, dtype=kind, device="cuda")
    ops.token_embed_bwd(grad_out, ids, 9, padding_id=4, grad=grad, accumulate=True)
    assert bool((grad == 3).all())
    ops.token_embed_bwd(grad_out, ids, 9, padding_id=4, grad=grad)
    assert bool((grad == 0).all())


@pytest.mark.parametrize("tokens", [100, 6000])
def test_ids_outside(ops, tokens):
    """Rows of zeros, no gradient, and an error that stays until it is asked for; a padding id outside is none."""
    import torch
    from paper_2208_05321_amd import FreqCacheError
    g = _gen(tokens)
    ids = torch.randint(0, 50, (tokens,), generator=g, device="cuda")
    table = torch.randn(50, 20, generator=g, device="cuda")
    grad_out = torch.randn(tokens, 20, generator=g, device="cuda")
    ids[::7] = -100
    want, size, terms = embed_grad(ids, grad_out, 50, 1.0)
    inside(ops.token_embed_bwd(grad_out, ids, 50, padding_id=-100), want, embed_bound(terms, size, torch.float32, want), "padding outside")
    ops.check()
    ids[3::11] = 50
    out = ops.token_embed_fwd(table, ids, scale=float("inf"))
    bad = (ids < 0) | (ids >= 50)
    assert bool((out[bad] == 0).all()) and bool(out[~bad].isinf().all())
    with pytest.raises(FreqCacheError) as e:
        ops.check()
    assert e.value.name == "ID_OUT_OF_RANGE"
    ops.check()
    want, size, terms = embed_grad(ids, grad_out, 50, 1.0)
    inside(ops.token_embed_bwd(grad_out, ids, 50), want, embed_bound(terms, size, torch.float32, want), "gradient")
    with pytest.raises(FreqCacheError):
        ops.check()


def test_gradient_is_the_lookups(ops):
    """sum(lookup(V) * G) = sum(V * gradient(G)) for any V: the lookup is linear, so its difference along V is the lookup of V."""
    import torch
    for tokens, dim in ((200, 24), (9000, 136)):
        g = _gen(tokens)
        ids = torch.randint(0, 400, (tokens,), generator=g, device="cuda")
        direction, grad_out = torch.randn(400, dim, generator=g, device="cuda"), torch.randn(tokens, dim, generator=g, device="cuda")
        there = (ops.token_embed_fwd(direction, ids, scale=3.0).double() * grad_out.double()).sum()
        back = (direction.double() * ops.token_embed_bwd(grad_out, ids, 400, scale=3.0).double()).sum()
        _, size, terms = embed_grad(ids, grad_out, 400, 3.0)
        assert abs(float(there - back)) <= float(((terms + 5) * U32 * size * direction.double().abs()).sum())
