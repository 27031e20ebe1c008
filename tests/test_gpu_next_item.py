"""`-m gpu`: the next-item example trains: the loss falls well below that of the start, and its step is the one that autograd gives."""
import pytest

pytestmark = pytest.mark.gpu


def test_it_learns_and_serves():
    import math
    import torch
    from examples.next_item import DIM, ITEMS, train
    losses, norms, model = train(40)
    assert losses[0] > 0.9 * math.log(ITEMS) and losses[-1] < 0.6 * losses[0]
    assert all(math.isfinite(x) and x > 0 for x in norms)
    y, scale = model.serve(torch.tensor([7], device="cuda"))
    x = model.items[7].double() * DIM ** 0.5
    want = x / (x.square().mean() + 1e-6).sqrt() * model.weight.double()
    # the row is rounded to bf16 before the norm (2^-8 of the largest), and to 8 bits after it (2^-4 of each, at least 2^-10 steps of the scale)
    assert bool(((y[0].double() * scale.double().view(()) - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -7 * want.abs().max()).all())
    model.close()


def test_its_step_is_autograds():
    """One step against the same model in torch's own operations, in 64 bits but for the roundings to bf16 of looked-up, summed and normed rows (2^-8 of a
    row each, in forward and backward pass: 2 % of the largest update is far beyond them)."""
    import torch
    from examples.next_item import DIM, LR, MAX_NORM, PAD, SAMPLES, SEQ, Model, batches
    model = Model(3)
    context, items, target = next(batches(5))
    p = [t.double().clone().requires_grad_() for t in (model.items, model.positions, model.weight, model.head)]
    slots = model.cache.prepare(context, model.offsets)
    pooled = model.cache.embedding_bag_fwd(slots, model.offsets).double().requires_grad_()
    real = (items != PAD).view(SAMPLES, SEQ, 1)
    table = torch.where((torch.arange(len(p[0]), device="cuda") == PAD)[:, None], p[0].detach(), p[0])
    h = table[items] * DIM ** 0.5 + p[1][model.at.long()]
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * p[2]
    state = (y.view(SAMPLES, SEQ, DIM) * real).sum(1) / real.sum(1)
    loss = torch.nn.functional.cross_entropy(torch.cat([state, pooled.view(SAMPLES, -1)], 1) @ p[3], target)
    grads = torch.autograd.grad(loss, (*p, pooled))
    norm = sum(float(g.square().sum()) for g in grads) ** 0.5
    factor = min(1.0, MAX_NORM / (norm + 1e-6))
    before = [t.clone() for t in (model.items, model.positions, model.weight, model.head)]
    got_loss, got_norm = model.step(context, items, target).tolist()
    assert got_loss == pytest.approx(float(loss.detach()), rel=1e-2) and got_norm == pytest.approx(norm, rel=2e-2)
    for b, t, g in zip(before, (model.items, model.positions, model.weight, model.head), grads):
        want = -LR * factor * g
        assert float((t.double() - b.double() - want).abs().max()) <= 0.02 * float(want.abs().max()) + 2.0 ** -23 * float(b.abs().max())
    model.close()
