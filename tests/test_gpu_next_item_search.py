"""`-m gpu`: the next-item example with a teacher and with a search: it runs, its gradients are autograd's, and what it finds is what its own logits say."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_distilled_step_is_autograds():
    """One step against the same model in torch's own operations, in 64 bits but for the roundings to bf16 of looked-up, summed and normed rows (2^-8 of a
    row each, in forward and backward pass: 2 % of the largest update is far beyond them)."""
    import torch
    from examples.next_item import DIM, LR, MAX_NORM, PAD, SAMPLES, SEQ, TEMPERATURE, Model, batches, teacher_of
    model = Model(3)
    context, items, target = next(batches(5))
    ids, z = teacher_of(target)
    p = [t.double().clone().requires_grad_() for t in (model.items, model.positions, model.weight, model.head)]
    slots = model.cache.prepare(context, model.offsets)
    pooled = model.cache.embedding_bag_fwd(slots, model.offsets).double().requires_grad_()
    real = (items != PAD).view(SAMPLES, SEQ, 1)
    table = torch.where((torch.arange(len(p[0]), device="cuda") == PAD)[:, None], p[0].detach(), p[0])
    h = table[items] * DIM ** 0.5 + p[1][model.at.long()]
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * p[2]
    state = (y.view(SAMPLES, SEQ, DIM) * real).sum(1) / real.sum(1)
    logits = torch.cat([state, pooled.view(SAMPLES, -1)], 1) @ p[3]
    share = torch.softmax(z.double() / TEMPERATURE, 1)
    kl = (share * (share.log() - torch.log_softmax(logits / TEMPERATURE, 1).gather(1, ids))).sum(1) * TEMPERATURE ** 2
    loss = (0.5 * kl - 0.5 * torch.log_softmax(logits, 1).gather(1, target[:, None])[:, 0]).mean()
    grads = torch.autograd.grad(loss, (*p, pooled))
    norm = sum(float(g.square().sum()) for g in grads) ** 0.5
    factor = min(1.0, MAX_NORM / (norm + 1e-6))
    mine = (model.items, model.positions, model.weight, model.head)
    before = [t.clone() for t in mine]
    got_loss, got_norm = model.step(context, items, target, (ids, z)).tolist()
    assert got_loss == pytest.approx(float(loss.detach()), rel=1e-2) and got_norm == pytest.approx(norm, rel=2e-2)
    for b, t, g in zip(before, mine, grads):
        want = -LR * factor * g
        assert float((t.double() - b.double() - want).abs().max()) <= 0.02 * float(want.abs().max()) + 2.0 ** -23 * float(b.abs().max())
    model.close()


def test_it_runs_with_a_teacher_and_searches():
    """The scores of what the search found, worked out again item by item."""
    import math
    import torch
    from examples.next_item import DIM, FEATURES, PAD, train
    losses, norms, model = train(6, distil=True)
    assert all(math.isfinite(x) for x in losses + norms)
    users, steps, beams = 3, 3, 4
    item, context = torch.tensor([7, 11, 30], device="cuda"), torch.randn(users, FEATURES * DIM, device="cuda") * 0.05
    found, scores = model.search(item, context, steps, beams)
    assert found.shape == (users, beams, steps) and bool((scores[:, 1:] <= scores[:, :-1]).all()) and not bool((found == PAD).any())
    assert all(len(set(map(tuple, f))) == beams for f in found.tolist())          # each sequence once
    for u in range(users):
        for b in range(beams):
            total, score = torch.zeros(DIM, dtype=torch.float64, device="cuda"), 0.0
            for k, prev in enumerate([int(item[u]), *found[u, b, :-1].tolist()]):
                x = (model.items[prev].float() * DIM ** 0.5).bfloat16().double()
                total = total + (x / (x.square().mean() + 1e-6).sqrt() * model.weight.double()).bfloat16().double()
                logits = torch.cat([total / (k + 1), context[u].double()]) @ model.head.double()
                logits[PAD] = float("-inf")
                score += float(torch.log_softmax(logits, 0)[found[u, b, k]])
            # f32 products of 576 terms, a bf16 rounding of each normed row that may fall the other way (2^-8 of an element of one row)
            assert float(scores[u, b]) == pytest.approx(score, abs=5e-2)
    model.close()
