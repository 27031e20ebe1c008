"""`-m gpu`: what the norm's backward pass takes of device memory goes by its rows, and what is reserved is enough for any number of them."""
import pytest

from tests.dense_reference import U32, inside, norm_parts, norm_steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [0, 1, 3])
def test_few_rows_of_the_widest(n):
    import torch
    from paper_2208_05321_amd import DenseOps
    d = 1 << 20
    ops = DenseOps()
    g = torch.Generator(device="cuda").manual_seed(n)
    h, dy = (torch.randn(n, d, generator=g, device="cuda") for _ in range(2))
    w = torch.randn(d, generator=g, device="cuda")
    dx, dw = torch.empty_like(h), None
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    _, dw = ops.rms_norm_bwd(dy, h, w, out=dx, eps=1e-5)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] <= 256 << 20       # (a row of sums is 4 MB; an allocation of torch's may be among it)
    _, hd, rho, _ = norm_parts(h, None, w, 1e-5)
    terms = dy.double() * hd * rho
    # n terms, each a product of two roundings with a root's reciprocal of half a sum of positive terms
    inside(dw, terms.sum(0), 1.01 * U32 * (n + norm_steps(d) / 2 + 8) * terms.abs().sum(0), "grad_weight")
    ops.close()


@pytest.mark.parametrize("n,d", [(1500, 2000), (600, 20_000)])
def test_what_is_reserved_for_a_width_is_enough_for_any_rows(n, d):
    """Nothing can be allocated while a stream is captured."""
    import torch
    from paper_2208_05321_amd import DenseOps
    st = torch.cuda.Stream()
    ops = DenseOps(st)
    ops.reserve(max_dim=d)
    h, dy, w = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda"), torch.randn(d, device="cuda")
    want = ops.rms_norm_bwd(dy[:1], h[:1], w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        held = ops.rms_norm_bwd(dy, h, w)
    for seed in range(3):
        torch.cuda.synchronize()
        dy.copy_(torch.randn(n, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        want = ops.rms_norm_bwd(dy, h, w)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
    ops.close()
