"""`-m gpu`: reordering of beams' states, bit for bit: any types and sizes, in place and not, pieces, strides, wrong parents."""
import pytest

from tests.logits_reference import reordered

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _parents(b, w, keep, seed, kind="int32"):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, w, (b, keep), generator=g, device="cuda").to(getattr(torch, kind))


def _bytes(shape, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)


@pytest.mark.parametrize("w", [1, 2, 3, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("size", [1, 2, 3, 7, 15, 16, 17, 31, 100, 4096, 16_383, 16_384, 50_001])
def test_sizes_in_bytes(ops, w, size):
    import torch
    b = 3
    t = _bytes((b, w, size), w * size)
    for kind in ("int32", "int64"):
        p = _parents(b, w, w, w + size, kind)
        want = reordered(t, p)
        own = t.clone()
        assert ops.beam_reorder([own], p)[0] is own and torch.equal(own, want)
        guard = torch.full((b * w * size + 64,), 7, dtype=torch.uint8, device="cuda")
        out = guard[32:32 + b * w * size].view(b, w, size)
        ops.beam_reorder([t], p, out=[out])
        assert torch.equal(out, want) and bool((guard[:32] == 7).all()) and bool((guard[32 + b * w * size:] == 7).all())
    keep = min(64, 2 * w + 1)
    p = _parents(b, w, keep, size)
    out = torch.empty((b, keep, size), dtype=torch.uint8, device="cuda")
    ops.beam_reorder([t], p, out=[out])
    assert torch.equal(out, reordered(t, p))
    ops.check()


def test_patterns_in_place(ops):
    """Every pattern of parents for three beams, cycles and all from one among them, and turned-round rows of 64."""
    import itertools
    import torch
    p = torch.tensor(list(itertools.product(range(3), repeat=3)), dtype=torch.int32, device="cuda")
    t = _bytes((27, 3, 5000), 1)
    want = reordered(t, p)
    ops.beam_reorder([t], p)
    assert torch.equal(t, want)
    t = _bytes((2, 64, 40_000), 2)
    for p in (torch.arange(63, -1, -1), (torch.arange(64) + 1) % 64, torch.zeros(64)):
        p = p.int().cuda().expand(2, 64).contiguous()
        want = reordered(t, p)
        ops.beam_reorder([t], p)
        assert torch.equal(t, want)


@pytest.mark.parametrize("keep", [0, 5, 12])
def test_pieces_of_buffers_with_room(ops, keep):
    """The filled part of caches [batch, beams, heads, room, dim]; the room beyond is left alone."""
    import torch
    b, w = 4, 6
    p = _parents(b, w, keep or w, 3)
    states, want, whole = [], [], []
    for heads, room, length, dim, kind in ((4, 40, 33, 24, torch.bfloat16), (1, 9, 5, 3, torch.float32), (3, 8, 1, 1, torch.int8), (2, 300, 299, 64, torch.float16),
                                           (5, 7, 7, 9, torch.int64), (8, 16, 0, 4, torch.float32)):
        t = (torch.randn((b, w, heads, room, dim), device="cuda") * 50).to(kind)
        whole.append((t, t.clone(), length))
        states.append(t[:, :, :, :length])
        want.append(reordered(states[-1], p))
    if keep:
        out = [torch.full((b, keep, *t.shape[2:]), 3, dtype=t.dtype, device="cuda") for t in states]
        out[0] = torch.zeros((b, keep, 4, 50, 24), dtype=torch.bfloat16, device="cuda")[:, :, :, 10:43]
        ops.beam_reorder(states, p, out=out)
        assert all(torch.equal(a, c) for a, c in zip(out, want))
        assert all(torch.equal(t, c) for t, c, _ in whole)
        src = [c.contiguous() for c in states]
        ops.beam_reorder(src[:1], p, out=out[:1])
        assert torch.equal(out[0], want[0])
    else:
        ops.beam_reorder(states, p)
        assert all(torch.equal(a, c) for a, c in zip(states, want))
        assert all(torch.equal(t[:, :, :, n:], c[:, :, :, n:]) for t, c, n in whole)
    ops.check()


def test_many_tensors(ops):
    """More than one launch describes, of different sizes."""
    import torch
    p = _parents(5, 4, 4, 9)
    states = [_bytes((5, 4, 1 + 37 * k), k) for k in range(130)]
    want = [reordered(t, p) for t in states]
    ops.beam_reorder(states, p)
    assert all(torch.equal(a, c) for a, c in zip(states, want))


def test_wrong_parents(ops):
    import torch
    from paper_2208_05321_amd import FreqCacheError
    p = _parents(3, 5, 5, 4, "int64")
    p[0, 1], p[1, 0], p[2, 4] = 5, -1, 1 << 40
    t = _bytes((3, 5, 777), 6)
    good = p.clone()
    bad = [(0, 1), (1, 0), (2, 4)]
    for i, j in bad:
        good[i, j] = j
    want = reordered(t, good)
    out = torch.full_like(t, 9)
    ops.beam_reorder([t], p, out=[out])
    for i, j in bad:
        want[i, j] = 0
    assert torch.equal(out, want)
    with pytest.raises(FreqCacheError) as e:
        ops.check()
    assert e.value.name == "ID_OUT_OF_RANGE"
    for i, j in bad:
        want[i, j] = t[i, j]
    ops.beam_reorder([t], p)
    assert torch.equal(t, want)
    with pytest.raises(FreqCacheError):
        ops.check()


def test_no_sequences_and_rows_far_apart(ops):
    import torch
    ops.beam_reorder([torch.empty((0, 4, 10), device="cuda")], torch.empty((0, 4), dtype=torch.int32, device="cuda"))
    t = torch.zeros((2, 2, (1 << 30) + 16), dtype=torch.uint8, device="cuda")          # row offsets beyond 32 bits
    t[:, :, -50:] = _bytes((2, 2, 50), 1)
    v = t[:, :, -50:]
    p = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device="cuda")
    want = reordered(v, p)
    ops.beam_reorder([v], p)
    assert torch.equal(v, want)
    ops.check()
