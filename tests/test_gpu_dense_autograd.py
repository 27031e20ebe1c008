"""`-m gpu`: what the dense operators write in place is seen by autograd: a tensor that was saved for a backward pass and then written is an error there,
as it is after torch's own in-place operations."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ops():
    from paper_2208_05321_amd import DenseOps
    o = DenseOps()
    yield o
    o.close()


def _writes(torch, ops):
    """(name, tensors that are written, call) of every way to write into a tensor of the caller's."""
    f = lambda *shape: torch.randn(*shape, device="cuda")  # noqa: E731
    table, ids, w, x, r, dy = f(9, 16), torch.arange(6, device="cuda"), f(16), f(6, 16), f(6, 16), f(6, 16)
    rows, grad, y, h, dx = f(6, 16), f(9, 16), f(6, 16), f(6, 16), f(6, 16)
    a, b, oa, ob = f(5), f(7), f(5), f(7)
    q = torch.empty(6, 16, dtype=torch.int8, device="cuda")
    return [
        ("lookup", [rows], lambda: ops.token_embed_fwd(table, ids, out=rows)),
        ("gradient", [grad], lambda: ops.token_embed_bwd(dy, ids, 9, grad=grad)),
        ("gradient added", [grad], lambda: ops.token_embed_bwd(dy, ids, 9, grad=grad, accumulate=True)),
        ("norm", [y], lambda: ops.rms_norm_fwd(x, w, out=y)),
        ("norm in 8 bits", [q], lambda: ops.rms_norm_fwd(x, w, out=q)),
        ("sum", [h], lambda: ops.rms_norm_fwd(x, w, residual=r, h_out=h)),
        ("sum in place", [x], lambda: ops.rms_norm_fwd(x, w, residual=r, h_out=x)),
        ("norm and sum", [y, r], lambda: ops.rms_norm_fwd(x, w, residual=r, h_out=r, out=y)),
        ("norm backward", [dx], lambda: ops.rms_norm_bwd(dy, x, w, out=dx)),
        ("norm backward in place", [dy], lambda: ops.rms_norm_bwd(dy, x, w, out=dy)),
        ("clip", [a, b], lambda: ops.grad_norm_clip([a, b], 1.0)),
        ("clip, a generator", [a, b], lambda: ops.grad_norm_clip((t for t in (a, b)), 1.0)),
        ("norm of tensors, and of none", [], lambda: (ops.grad_norm_clip([a, b], float("inf")), ops.grad_norm_clip([], 1.0))),
        ("clip into others", [oa, ob], lambda: ops.grad_norm_clip([a, b], 1.0, out=[oa, ob])),
    ], [table, ids, w, x, r, dy, rows, grad, y, h, dx, a, b, oa, ob, q]


def test_versions(ops):
    import torch
    calls, everything = _writes(torch, ops)
    for name, written, call in calls:
        before = [t._version for t in everything]
        call()
        for t, was in zip(everything, before):
            assert (t._version > was) == any(t is o for o in written), name


def test_a_saved_tensor_that_is_written_is_an_error(ops):
    import torch
    calls, _ = _writes(torch, ops)
    for name, written, call in calls:
        if not all(t.is_floating_point() for t in written):
            continue
        p = torch.ones((), device="cuda", requires_grad=True)
        losses = [(p * t).sum() for t in written]               # the product saves t
        call()
        for loss in losses:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    torch.cuda.synchronize()


def test_tensors_of_inference(ops):
    import torch
    with torch.inference_mode():
        x, r, w = torch.randn(4, 32, device="cuda"), torch.randn(4, 32, device="cuda"), torch.ones(32, device="cuda")
        want = x + r
        ops.rms_norm_fwd(x, w, residual=r, h_out=x)
        assert torch.equal(x, want)
        assert float(ops.grad_norm_clip([x], 1e9)) > 0
    ops.rms_norm_fwd(x, w, out=r)
