"""`-m gpu`: what the dense operators' calls have in common: refusals, other streams than the current one, graphs, workspaces that grow."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _refused(call):
    from paper_2208_05321_amd import FreqCacheError
    with pytest.raises(FreqCacheError) as e:
        call()
    assert e.value.name == "INVALID_ARG"


def test_refusals_of_the_binding(ops):
    import torch
    cpu, f = torch.randn(4, 8), torch.randn(4, 8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    w = torch.ones(8, device="cuda")
    for bad in (cpu, f.double(), f.t(), f[0], f[:, :0], f.view(2, 2, 8)):
        _refused(lambda: ops.token_embed_fwd(bad, ids))
    for bad in (ids.cpu(), ids.float(), torch.zeros(8, dtype=torch.int64, device="cuda")[::2]):
        _refused(lambda: ops.token_embed_fwd(f, bad))
    _refused(lambda: ops.token_embed_fwd(f, ids, out=torch.empty(4, 9, device="cuda")))
    _refused(lambda: ops.token_embed_fwd(f, ids, out=f.bfloat16(), out_dtype=torch.float32))
    _refused(lambda: ops.token_embed_fwd(f, ids, out_dtype=torch.int8))
    _refused(lambda: ops.token_embed_fwd(f[:, :1].expand(4, 8), ids))
    _refused(lambda: ops.token_embed_bwd(f, ids[:3], 5))
    _refused(lambda: ops.token_embed_bwd(f, ids, 5, accumulate=True))
    _refused(lambda: ops.token_embed_bwd(f, ids, 5, grad=torch.empty(4, 8, device="cuda")))
    _refused(lambda: ops.token_embed_bwd(f, ids, 5, grad_dtype=torch.bfloat16))
    _refused(lambda: ops.token_embed_bwd(f, ids, 0))
    _refused(lambda: ops.rms_norm_fwd(f, w[:7]))
    _refused(lambda: ops.rms_norm_fwd(f, w.bfloat16()))
    _refused(lambda: ops.rms_norm_fwd(f, w, residual=f[:3]))
    _refused(lambda: ops.rms_norm_fwd(f, w, residual=f.half()))
    _refused(lambda: ops.rms_norm_fwd(f, w, h_out=f))
    _refused(lambda: ops.rms_norm_fwd(f, w, out_dtype=torch.bfloat16))
    _refused(lambda: ops.rms_norm_fwd(f, w, group=32))
    _refused(lambda: ops.rms_norm_fwd(f, w, out_dtype=torch.int8, group=48))
    _refused(lambda: ops.rms_norm_fwd(f, w, eps=-1.0))
    _refused(lambda: ops.rms_norm_fwd(f, w, eps=float("nan")))
    _refused(lambda: ops.rms_norm_fwd(f.view(2, 2, 8).transpose(0, 1), w))
    _refused(lambda: ops.rms_norm_bwd(f[:3], f, w))
    _refused(lambda: ops.rms_norm_bwd(f, f, w, grad_h=f.half()))
    _refused(lambda: ops.rms_norm_bwd(f, f, w, grad_weight_dtype=torch.int8))
    _refused(lambda: ops.grad_norm_clip([f, cpu], 1.0))
    _refused(lambda: ops.grad_norm_clip([f.t()], 1.0))
    _refused(lambda: ops.grad_norm_clip([f.double()], 1.0))
    _refused(lambda: ops.grad_norm_clip([f], 0.0))
    _refused(lambda: ops.grad_norm_clip([f], float("nan")))
    _refused(lambda: ops.grad_norm_clip([f], 1.0, out=[]))
    _refused(lambda: ops.grad_norm_clip([f], 1.0, out=[f.half()]))
    ops.check()


def test_refusals_of_the_library(ops):
    import torch
    L, h = ops._L, ops._h
    t = torch.zeros(64, 64, device="cuda")
    p = t.data_ptr()
    fwd = [h, p, 0, 64, 64, 64, p, 6, 4, 1.0, p, 0, 64]
    bwd = [h, p, 0, 64, p, 6, 4, 64, 64, 1.0, -1, p, 0, 64, 0]
    norm = [h, p, 0, 64, p, 64, p, 0, 4, 64, 1e-6, p, 64, p, 0, 64, None, 0]
    back = [h, p, 64, p, 0, 64, p, 0, p, 64, 4, 64, 1e-6, p, 64, p, 0]
    for call, good, bad in (
            (L.token_embed_fwd, fwd, {0: None, 1: None, 2: 3, 3: 63, 4: 0, 5: 0, 6: None, 7: 2, 8: -1, 10: None, 11: 4, 12: 63}),
            (L.token_embed_bwd, bwd, {0: None, 1: None, 2: 5, 3: 63, 4: None, 5: 0, 6: -1, 7: 0, 8: (1 << 20) + 1, 11: None, 12: 1, 13: 63}),
            (L.rms_norm_fwd, norm, {0: None, 1: None, 2: 4, 3: 63, 5: 63, 6: None, 7: 1, 8: -1, 9: 0, 10: -1.0, 12: 63, 13: None, 14: 3, 15: 63, 17: 32}),
            (L.rms_norm_bwd, back, {0: None, 1: None, 2: 63, 3: None, 4: 3, 5: 63, 6: None, 7: 2, 9: 63, 10: 1 << 31, 11: -5, 12: float("nan"), 13: None, 14: 63, 15: None, 16: 4})):
        for k, v in bad.items():
            args = list(good)
            args[k] = v
            assert call(*args) == -1, (call.__name__, k)
    ptrs, sizes, kinds = (ctypes.c_uint64 * 1)(p), (ctypes.c_int64 * 1)(64), (ctypes.c_int32 * 1)(0)
    a = lambda x: ctypes.addressof(x)  # noqa: E731
    good = [h, a(ptrs), None, a(sizes), a(kinds), 1, 1.0, p]
    bad_kind, bad_size, no_ptr = (ctypes.c_int32 * 1)(3), (ctypes.c_int64 * 1)(-1), (ctypes.c_uint64 * 1)(0)
    for k, v in {0: None, 1: None, 2: a(no_ptr), 3: None, 4: None, 5: -1, 6: 0.0, 7: None}.items():
        args = list(good)
        args[k] = v
        assert L.grad_norm_clip(*args) == -1, k
    assert L.grad_norm_clip(h, a(ptrs), None, a(sizes), a(bad_kind), 1, 1.0, p) == -1
    assert L.grad_norm_clip(h, a(ptrs), None, a(bad_size), a(kinds), 1, 1.0, p) == -1
    assert L.grad_norm_clip(h, a(no_ptr), None, a(sizes), a(kinds), 1, 1.0, p) == -1
    assert L.dense_reserve(h, -1, 0, 0, 0) == -1 and L.dense_reserve(None, 1, 1, 1, 1) == -1 and L.dense_reserve(h, 10, 10, 10, 10) == 0
    torch.cuda.synchronize()
    assert bool((t == 0).all())
    ops.check()


def _step(torch, ops, table, ids, weight, dy, grads, out):
    """All operators once; what they give."""
    x = ops.token_embed_fwd(table, ids, scale=2.0, out_dtype=torch.bfloat16)
    y, h, _ = ops.rms_norm_fwd(x, weight, residual=x)
    dx, dw = ops.rms_norm_bwd(dy, h, weight, grad_h=y)
    g = ops.token_embed_bwd(dx, ids, table.shape[0], scale=2.0, padding_id=0)
    norm = ops.grad_norm_clip([g, dw, *grads], 0.5, out=out)
    return [x, y, h, dx, dw, g, norm, *out]


def _inputs(torch, rows, dim, tokens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randn(rows, dim, generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, rows, (tokens,), generator=g, device="cuda")
    ids[::3] = 5
    weight = torch.randn(dim, generator=g, device="cuda")
    dy = torch.randn(tokens, dim, generator=g, device="cuda").bfloat16()
    grads = [torch.randn(50 + k, generator=g, device="cuda") for k in range(150)]
    return table, ids, weight, dy, grads


def _outs(torch, rows, dim, grads):
    return [torch.empty(rows, dim, device="cuda"), torch.empty(dim, device="cuda"), *(torch.empty_like(t) for t in grads)]


@pytest.mark.parametrize("own", [False, True])
def test_another_stream_is_current(own):
    """The handle's stream is the default one and a side stream is current, or the other way round; what is read has been enqueued on the current
    stream behind long work, and results are read there without a wait."""
    import torch
    from paper_2208_05321_amd import DenseOps
    side = torch.cuda.Stream()
    ops = DenseOps(side) if own else DenseOps()
    args = _inputs(torch, 300, 72, 5000, 1)
    want = [t.clone() for t in _step(torch, ops, *args, _outs(torch, 300, 72, args[-1]))]
    torch.cuda.synchronize()
    slow = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(torch.cuda.default_stream() if own else side):
        for _ in range(3):
            late = []
            for _ in range(10):
                slow = (slow @ slow).clamp_(-1, 1)
            for t in (*args[:4],):
                late.append(torch.zeros_like(t) if t.dtype != torch.int64 else torch.zeros_like(t))
                late[-1].copy_(t)
            got = _step(torch, ops, *late, args[4], _outs(torch, 300, 72, args[4]))
            same = torch.stack([(a == b).all() for a, b in zip(got, want)]).all()
            del late, got
            junk = [torch.full((5000, 72), float("nan"), device="cuda") for _ in range(4)]       # memory given back is used again at once
            assert bool(same)
            del junk
    torch.cuda.synchronize()
    ops.check()
    ops.close()


@pytest.mark.parametrize("rows,dim,tokens", [(400, 64, 900), (400, 64, 6000), (3000, 40, 80_000), (20_000, 24, 200_000)])
def test_graph_replays(rows, dim, tokens):
    """Captured once, replayed with new inputs, eager calls of the same handle (smaller and larger ones) between the replays."""
    import torch
    from paper_2208_05321_amd import DenseOps
    st = torch.cuda.Stream()
    ops = DenseOps(st)
    ops.reserve(max_tokens=tokens, max_rows=rows, max_dim=dim, max_tensors=200)
    args = _inputs(torch, rows, dim, tokens, 0)
    out = _outs(torch, rows, dim, args[-1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = _step(torch, ops, *args, out)
    other = DenseOps()
    for seed in range(1, 5):
        new = _inputs(torch, rows, dim, tokens, seed)
        want = _step(torch, other, *new, _outs(torch, rows, dim, new[-1]))
        for a, b in zip(args[:4], new[:4]):
            a.copy_(b)
        for a, b in zip(args[4], new[4]):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), seed
        size = tokens // 2 if seed % 2 else 3 * tokens                    # the latter makes the workspace grow: the graph's stays
        with torch.cuda.stream(st):
            more = _inputs(torch, rows, dim, size, 77)
            _step(torch, ops, *more, _outs(torch, rows, dim, more[-1]))
        torch.cuda.synchronize()
    ops.check()
    ops.close()
    other.close()


def test_workspace_grows_and_shrinks_in_use(ops):
    import torch
    from tests.dense_reference import embed_bound, embed_grad, inside
    for tokens, rows, dim in ((2000, 100, 8), (60_000, 5000, 40), (1500, 100_000, 16), (150_000, 300, 24), (3000, 50, 600), (70_000, 7, 4)):
        ids = torch.randint(0, rows, (tokens,), device="cuda")
        g = torch.randn(tokens, dim, device="cuda")
        want, size, terms = embed_grad(ids, g, rows, 1.0)
        inside(ops.token_embed_bwd(g, ids, rows), want, embed_bound(terms, size, torch.float32, want), (tokens, rows, dim))
