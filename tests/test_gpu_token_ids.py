"""`-m gpu`: the id -1, which is what says "no padding id": as an id it is one outside the table, in the backward pass as in the forward pass."""
import pytest

from tests.dense_reference import embed_bound, embed_grad, inside

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [100, 6000])                     # without and with a sort
@pytest.mark.parametrize("kind", ["int32", "int64"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_minus_one_is_outside_unless_it_is_padding(tokens, kind, accumulate):
    import torch
    from paper_2208_05321_amd import DenseOps, FreqCacheError
    ops = DenseOps()
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    ids = torch.randint(0, 50, (tokens,), generator=gen, device="cuda").to(getattr(torch, kind))
    grad_out = torch.randn(tokens, 20, generator=gen, device="cuda")
    old = torch.randn(50, 20, generator=gen, device="cuda")

    def backward(**more):
        grad = old.clone()
        ops.token_embed_bwd(grad_out, ids, 50, grad=grad, accumulate=accumulate, **more)
        want, size, terms = embed_grad(ids, grad_out, 50, 1.0)
        if accumulate:
            want, size = want + old.double(), size + old.double().abs()
        inside(grad, want, embed_bound(terms, size, torch.float32, want), "gradient")

    backward()
    ops.check()                                                     # no id outside
    ids[5::9] = -1
    for more in ({}, {"padding_id": -1}, {"padding_id": 7_000_000}):
        if more.get("padding_id") == 7_000_000:                     # another padding id, which no token has
            assert not bool((ids == 7_000_000).any())
        backward(**more)
        with pytest.raises(FreqCacheError) as e:
            ops.check()
        assert e.value.name == "ID_OUT_OF_RANGE"
        ops.check()
    ids[ids == -1] = -2                                             # a padding id outside the table is padding
    backward(padding_id=-2)
    ops.check()
    ops.close()
