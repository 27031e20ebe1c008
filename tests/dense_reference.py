"""Plain 64-bit forms of the operators beside the cached table, and the rounding errors that 32-bit sums and one final rounding allow."""
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float64: 0.0}   # half a unit in the last place, relative
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float64: 0.0}   # half the smallest step
U32 = U[torch.float32]


def rounded(want, kind):
    """What rounding `want` to `kind` may add."""
    return U[kind] * want.abs() + TINY[kind]


def inside(got, want, bound, what):
    """|got - want| <= bound everywhere; the largest share of it is returned."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off / bound).nan_to_num(0, 0, 0).max()):.3g} of the bound"


def embed_grad(ids, grad_out, rows, scale, padding_id=-1):
    """(sums by id, the same of absolute values, tokens of each row) in 64 bits."""
    keep = ((ids != padding_id) & (ids >= 0) & (ids < rows))
    at, g = ids[keep].long(), grad_out[keep].double() * scale
    z = lambda: torch.zeros((rows, grad_out.shape[1]), dtype=torch.float64, device=grad_out.device)  # noqa: E731
    return z().index_add_(0, at, g), z().index_add_(0, at, g.abs()), torch.bincount(at, minlength=rows)[:, None].double()


def embed_bound(terms, size, kind, want):
    """K terms of 32 bits in any order: K - 1 sums; the scale and its product, an addition to what was there; the result's rounding."""
    return 1.01 * (terms + 3) * U32 * size + rounded(want, kind) * 1.01


def norm_parts(x, residual, weight, eps):
    """h as it is stored, and in 64 bits: h, the root's reciprocal, y."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    d = h.double()
    rho = (d.square().mean(-1, keepdim=True) + eps).rsqrt()
    return h, d, rho, d * rho * weight.double()


def norm_steps(dim):
    """Additions that a term of a row's sum goes through: in its lane (32 at most, or dim / 1024 and a vector), over 64 lanes, over 16 wavefronts."""
    return max(32, dim // 1024 + 8) + 6 + 16
