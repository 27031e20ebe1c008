"""`-m gpu`: what the calls on rows of logits have in common with the other dense operators': refusals, other streams than the current one, graphs, and a run of them together."""
import ctypes

import pytest

from tests.dense_reference import inside, rounded
from tests.logits_reference import distill, reordered, select

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def test_refusals_of_the_library(ops):
    import torch
    L, h = ops._L, ops._h
    t = torch.zeros(64, 64, device="cuda")
    p = t.data_ptr()
    inf, nan = float("inf"), float("nan")
    fwd = [h, p, 0, 64, 4, 64, p, 6, p, 0, 4, None, p, 6, 1.0, 0.5, p, p]
    bwd = [h, p, 1, p, 0, 64, 4, 64, p, 6, p, 0, 4, p, 6, 1.0, 0.5, p, p, 64]
    both = [h, p, 1, p, 0, 64, 4, 64, p, 6, p, 0, 4, None, p, 6, 1.0, 0.5, p, p, 64]
    sel = [h, p, 0, 64, 2, 2, 64, p, p, 3, 2, p, p, p, 6, p]
    for call, good, bad in (
            (L.distill_fwd, fwd, [(0, None), (1, None), (2, 3), (3, 63), (4, -1), (4, 1 << 31), (5, 0), (5, (1 << 20) + 1), (6, None), (7, 0), (8, None), (9, 4), (10, -1), (10, 1025),
                                  (12, None), (13, 2), (14, 0.0), (14, -1.0), (14, nan), (14, inf), (14, 2000.0), (15, -0.1), (15, 1.1), (15, nan), (16, None), (17, None)]),
            (L.distill_bwd, bwd, [(0, None), (1, None), (2, 2), (2, -1), (3, None), (4, 4), (5, 63), (6, -1), (7, 0), (8, None), (9, 1), (10, None), (11, 3), (12, 1025), (13, None),
                                  (14, 0), (15, 0.0), (16, 2.0), (17, None), (18, None), (19, 63), (19, 65)]),
            (L.distill_grad, both, [(0, None), (1, None), (2, 2), (3, None), (4, 4), (5, 63), (6, -1), (7, 0), (8, None), (9, 1), (10, None), (11, 3), (12, 1025), (14, None), (15, 0),
                                    (16, 0.0), (17, 2.0), (18, None), (19, None), (20, 63), (20, 65)]),
            (L.beam_select, sel, [(0, None), (1, None), (2, 3), (3, 63), (4, -1), (5, 0), (5, 65), (6, 0), (6, (1 << 20) + 1), (7, None), (9, -1), (9, -2), (9, 64), (10, 0), (10, 65),
                                  (11, None), (12, None), (13, None), (14, 0)])):
        for k, v in bad:
            args = list(good)
            args[k] = v
            assert call(*args) == -1, (call.__name__, k, v)
    state = lambda *v: ctypes.addressof((ctypes.c_int64 * 8)(*v))  # noqa: E731
    keep = []
    def one(**change):
        s = dict(src=p, dst=p + 8192, src_row=64, dst_row=64, src_piece=16, dst_piece=16, piece=16, pieces=4)
        s.update(change)
        keep.append((ctypes.c_int64 * 8)(*s.values()))
        return ctypes.addressof(keep[-1])
    re = [h, one(), 1, 2, 4, p, 5, 4]
    for k, v in [(0, None), (1, None), (2, -1), (3, -1), (4, 0), (4, 65), (5, None), (6, 0), (7, 0), (7, 65)] + [(1, one(**c)) for c in (
            {"src": 0}, {"dst": 0}, {"src_row": 63}, {"dst_row": 63}, {"src_piece": 15}, {"dst_piece": 15}, {"piece": -1}, {"pieces": -1}, {"piece": 1 << 31}, {"pieces": 1 << 31},
            {"dst": p, "dst_row": 128}, {"dst": p, "dst_piece": 17, "dst_row": 67, "src_row": 67})]:
        args = list(re)
        args[k] = v
        assert L.beam_reorder(*args) == -1, (k, v)
    args = list(re)
    args[1], args[7] = one(dst=p), 3                 # in place with another number of beams
    assert L.beam_reorder(*args) == -1
    torch.cuda.synchronize()
    assert bool((t == 0).all())
    ops.check()


def test_refusals_of_the_binding(ops):
    import torch
    from paper_2208_05321_amd import FreqCacheError
    x, ids, z = torch.zeros(4, 50, device="cuda"), torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(4, 3, device="cuda")
    y, w, stats, lse = ids[:, 0].contiguous(), torch.ones(4, device="cuda"), torch.zeros(4, 12, device="cuda"), torch.zeros(4, device="cuda")
    b, s = torch.zeros(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    done, p = torch.zeros(2, 3, dtype=torch.bool, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    e = lambda *shape: torch.zeros(2, 3, *shape, device="cuda")  # noqa: E731
    for call in (
            lambda: ops.distill_fwd(x.cpu(), ids, z), lambda: ops.distill_fwd(x.double(), ids, z), lambda: ops.distill_fwd(x.t(), ids, z), lambda: ops.distill_fwd(x, ids.cpu(), z),
            lambda: ops.distill_fwd(x, ids.float(), z), lambda: ops.distill_fwd(x, ids[:3], z[:3]), lambda: ops.distill_fwd(x, ids, z[:, :2]), lambda: ops.distill_fwd(x, ids, z.double()),
            lambda: ops.distill_fwd(x, ids.t().contiguous().t(), z), lambda: ops.distill_fwd(x, ids, z, alpha=0.5), lambda: ops.distill_fwd(x, ids, z, targets=y[:3]),
            lambda: ops.distill_fwd(x, ids, z, targets=y.float()), lambda: ops.distill_fwd(x, ids, z, temperature=0.0), lambda: ops.distill_fwd(x, ids, z, targets=y, alpha=1.5),
            lambda: ops.distill_fwd(x, ids, z, teacher_lse=lse.half()), lambda: ops.distill_fwd(x, ids, z, teacher_lse=lse[:3]), lambda: ops.distill_fwd(x, ids[0], z[0]),
            lambda: ops.distill_fwd(x, ids[:, :1].expand(4, 1025).contiguous(), z[:, :1].expand(4, 1025).contiguous()),
            lambda: ops.distill_bwd(w[:3], x, ids, z, stats), lambda: ops.distill_bwd(w.half(), x, ids, z, stats), lambda: ops.distill_bwd(w, x, ids, z, stats[:, :11]),
            lambda: ops.distill_bwd(w, x, ids, z, stats, out=x[:, :49]), lambda: ops.distill_bwd(w, x, ids, z, stats, out=x.half()),
            lambda: ops.distill_bwd(torch.ones(8, device="cuda")[::2], x, ids, z, stats), lambda: ops.distill_grad(w.cpu(), x, ids, z),
            lambda: ops.distill_grad(w, x, ids, z, out=torch.zeros(4, 100, device="cuda")[:, ::2]),
            lambda: ops.beam_select(x, s), lambda: ops.beam_select(b.double(), s), lambda: ops.beam_select(b, s[:, :2]), lambda: ops.beam_select(b, s.half()),
            lambda: ops.beam_select(b, s, 0), lambda: ops.beam_select(b, s, 65), lambda: ops.beam_select(b, s, eos_id=50), lambda: ops.beam_select(b, s, eos_id=-2),
            lambda: ops.beam_select(b, s, finished=done), lambda: ops.beam_select(b, s, finished=done.int(), eos_id=1), lambda: ops.beam_select(b, s, finished=done[:, :2], eos_id=1),
            lambda: ops.beam_select(b, s, token_dtype=torch.float32), lambda: ops.beam_select(b.transpose(0, 1), s.t()), lambda: ops.beam_select(torch.zeros(1, 65, 8, device="cuda"), s),
            lambda: ops.beam_reorder([], p), lambda: ops.beam_reorder([e(4)], p.float()), lambda: ops.beam_reorder([e(4)], p[:, :2].contiguous()), lambda: ops.beam_reorder([e(4).cpu()], p),
            lambda: ops.beam_reorder([e(4), e(4)[:1]], p), lambda: ops.beam_reorder([e(4)], p, out=[]), lambda: ops.beam_reorder([e(4)], p, out=[e(5)]),
            lambda: ops.beam_reorder([e(4)], p, out=[e(4).half()]), lambda: ops.beam_reorder([e(4, 4, 4)[:, :, ::2, :, ::2]], p), lambda: ops.beam_reorder([e(1).expand(2, 3, 4)[:, :1].expand(2, 3, 4)], p),
            lambda: ops.beam_reorder([e(4).transpose(0, 1).contiguous().transpose(0, 1)], p), lambda: ops.beam_reorder([torch.zeros(2, 1, 4, device="cuda").expand(2, 3, 4)], p),
            lambda: ops.beam_reorder([e(2, 5)[:, :, :, :3]], p, out=[e(3, 5)[:, :, :2, :3].transpose(2, 3).contiguous().transpose(2, 3)])):
        with pytest.raises(FreqCacheError) as err:
            call()
        assert err.value.name == "INVALID_ARG"
    ops.check()


def _inputs(torch, n, v, top, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ids = torch.randint(0, v // top, (n, top), generator=g, device="cuda") + torch.arange(top, device="cuda") * (v // top)
    return [(3 * rnd(n, v)).bfloat16(), ids, rnd(n, top) + 6, rnd(n) + 9, ids[:, 0].contiguous(), rnd(n), (3 * rnd(n // 4, 4, v)).bfloat16(), -rnd(n // 4, 4).abs(),
            rnd(n // 4, 4, 3, 40), rnd(n // 4, 4, 77)]


def _step(ops, x, ids, z, lse, y, w, logits, scores, a, b):
    """All of them once; what they give."""
    how = dict(targets=y, temperature=2.0, alpha=0.5)
    loss, stats = ops.distill_fwd(x, ids, z, teacher_lse=lse, **how)
    grad = ops.distill_bwd(w, x, ids, z, stats, **how)
    loss2, grad2 = ops.distill_grad(w, x, ids, z, teacher_lse=lse, **how)
    s, p, t, f = ops.beam_select(logits, scores, eos_id=1)
    states = ops.beam_reorder([a, b], p, out=[a.new_empty(a.shape), b.new_empty(b.shape)])
    return [loss, grad, loss2, grad2, s, p, t, f, *states]


@pytest.mark.parametrize("v", [700, 70_000])
@pytest.mark.parametrize("own", [False, True])
def test_another_stream_is_current(own, v):
    import torch
    from paper_2208_05321_amd import DenseOps
    side = torch.cuda.Stream()
    ops = DenseOps(side) if own else DenseOps()
    args = _inputs(torch, 64, v, 8, 1)
    want = [t.clone() for t in _step(ops, *args)]
    torch.cuda.synchronize()
    slow = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(torch.cuda.default_stream() if own else side):
        for _ in range(3):
            for _ in range(10):
                slow = (slow @ slow).clamp_(-1, 1)
            late = [torch.zeros_like(t).copy_(t) for t in args]
            got = _step(ops, *late)
            same = torch.stack([(a == b).all() for a, b in zip(got, want)]).all()
            del late, got
            junk = [torch.full((64, v), float("nan"), device="cuda") for _ in range(4)]
            assert bool(same)
            del junk
    torch.cuda.synchronize()
    ops.check()
    ops.close()


@pytest.mark.parametrize("v", [700, 9000, 70_000])
def test_graph_replays(v):
    """Captured once, replayed with new inputs, eager calls of the same handle between the replays."""
    import torch
    from paper_2208_05321_amd import DenseOps
    st = torch.cuda.Stream()
    ops = DenseOps(st)
    ops.reserve(max_dim=v)
    args = _inputs(torch, 80, v, 8, 0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = _step(ops, *args)
    other = DenseOps()
    for seed in range(1, 5):
        new = _inputs(torch, 80, v, 8, seed)
        want = _step(other, *new)
        for a, b in zip(args, new):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), seed
        with torch.cuda.stream(st):
            more = _inputs(torch, 40 if seed % 2 else 240, v, 8, 77)
            _step(ops, *more)
        torch.cuda.synchronize()
    ops.check()
    ops.close()
    other.close()


def test_nothing_can_be_allocated_in_a_capture():
    import torch
    from paper_2208_05321_amd import DenseOps, FreqCacheError
    st = torch.cuda.Stream()
    ops = DenseOps(st)
    x, s = torch.zeros(1, 2, 100_000, device="cuda"), torch.zeros(1, 2, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        with pytest.raises(FreqCacheError) as e:
            ops.beam_select(x, s)
        keep = x + 1  # noqa: F841 (a graph with something in it)
    assert e.value.name == "HIP"
    torch.cuda.synchronize()
    ops.close()


def test_what_is_written_in_place_is_known_to_autograd(ops):
    import torch
    x, ids, z = torch.randn(4, 50, device="cuda"), torch.zeros(4, 1, dtype=torch.int64, device="cuda"), torch.zeros(4, 1, device="cuda")
    w = torch.ones(4, device="cuda")
    before = x._version
    ops.distill_grad(w, x, ids, z, out=x)
    assert x._version > before
    t, p = torch.randn(2, 3, 8, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    before, o = t._version, torch.empty(2, 3, 8, device="cuda")
    ops.beam_reorder([t], p, out=[o])
    assert t._version == before and o._version > 0
    ops.beam_reorder([t], p)
    assert t._version > before


def test_together_a_step_of_training_and_of_search(ops):
    """Logits from a looked-up and normed row, distilled against a teacher's best; the gradient back through norm and table; and three steps of a search over the same table, states
    and tokens carried along, against the same steps in 64 bits on the operators' own logits."""
    import torch
    items, dim, n, top = 900, 64, 48, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    table, weight, head = rnd(items, dim) * 0.3, 1 + 0.1 * rnd(dim), rnd(dim, items) * 0.3
    ids = torch.randint(0, items, (n,), generator=g, device="cuda")
    x = ops.token_embed_fwd(table, ids)
    y, h, _ = ops.rms_norm_fwd(x, weight)
    logits = y @ head
    best = (logits + rnd(n, items)).topk(top, 1)
    z, t_ids = best.values.contiguous(), best.indices.contiguous()
    w = torch.full((1,), 1.0 / n, device="cuda")
    loss, gl = ops.distill_grad(w, logits, t_ids, z, temperature=2.0)
    want, grad, off, off_grad = distill(logits, t_ids, z, None, None, 2.0, 1.0)
    inside(loss, want, off, "loss")
    inside(gl, grad / n, off_grad / n + rounded(grad / n, torch.float32), "gradient of the logits")
    gx, gw = ops.rms_norm_bwd(gl @ head.t(), h, weight)
    gt = ops.token_embed_bwd(gx, ids, items)
    leaf = [q.double().requires_grad_() for q in (table, weight)]
    e = leaf[0][ids]
    lg = (e / (e.square().mean(1, keepdim=True) + 1e-6).sqrt() * leaf[1]) @ head.double()
    p = torch.softmax(z.double() / 2, 1)
    kl = 4 * (p * (p.log() - torch.log_softmax(lg / 2, 1).gather(1, t_ids))).sum(1).mean()
    for got, of in zip((gt, gw), torch.autograd.grad(kl, leaf)):
        # f32 products of 64 and 900 terms and the norm between: a thousandth of the largest is far beyond their roundings
        assert float((got.double() - of).abs().max()) <= 1e-3 * float(of.abs().max())
    batch, beams = 5, 4
    tokens = torch.randint(0, items, (batch, beams), generator=g, device="cuda")
    scores = torch.full((batch, beams), float("-inf"), device="cuda")
    scores[:, 0] = 0.0
    state, past, done = torch.zeros(batch, beams, dim, device="cuda"), torch.zeros(batch, beams, 4, dtype=torch.int64, device="cuda"), None
    for step in range(3):
        state += ops.token_embed_fwd(table, tokens)
        lg = ops.rms_norm_fwd(state, weight)[0] @ head
        want = select(lg, scores, beams, done, 7)
        scores, parents, tokens, done = ops.beam_select(lg, scores, finished=done, eos_id=7)
        assert torch.equal(parents, want[1]) and torch.equal(tokens, want[2])
        moved = [reordered(q, parents) for q in (state, past)]
        ops.beam_reorder([state, past], parents)
        assert torch.equal(state, moved[0]) and torch.equal(past, moved[1])
        past[:, :, step] = tokens
        if step == 1:
            done[2, 1] = True
    ops.check()


def test_a_state_given_twice(ops):
    """Refused, as it would be moved twice; the same tensor may be read for several that are written."""
    import torch
    from paper_2208_05321_amd import FreqCacheError
    a = torch.arange(30., device="cuda").view(2, 3, 5)
    b, p = a + 100, torch.tensor([[2, 0, 1], [1, 1, 0]], device="cuda")
    kept, none = a.clone(), torch.empty(2, 3, 0, device="cuda")
    for states, out in (([a, b, a], None), ([a, a[:, :, :2]], None), ([a, a], [b, b]), ([a, b], [b, a])):
        with pytest.raises(FreqCacheError) as err:
            ops.beam_reorder(states, p, out=out)
        assert err.value.name == "INVALID_ARG"
    torch.cuda.synchronize()
    assert torch.equal(a, kept)
    want = torch.stack([kept[i][p[i]] for i in range(2)])
    c = ops.beam_reorder([a, a, none, none], p, out=[torch.empty_like(a), torch.empty_like(a), torch.empty_like(none), torch.empty_like(none)])
    assert torch.equal(c[0], want) and torch.equal(c[1], want)
    ops.beam_reorder([a, none, none], p, out=[a, none, none])
    assert torch.equal(a, want)
    ops.check()
