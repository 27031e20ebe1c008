"""CPU-side checks of the binding of the dense operators, on tensors that have a shape and no memory, with a library that only notes its calls."""
import pytest


class _Noted:
    """Every entry point: its arguments are kept, the answer is 0."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture()
def ops():
    import torch
    from paper_2208_05321_amd.dense import _TYPE_NAMES, DenseOps
    o = DenseOps.__new__(DenseOps)
    o._L, o._torch, o._h = _Noted(), torch, 1
    o._type = {getattr(torch, name): k for name, k in _TYPE_NAMES.items()}
    o.device, o._index, o._raw, o._current = torch.device("meta"), -1, 0, lambda index: 0
    return o


def _calls(ops):
    return [name for name, _ in ops._L.calls if name != "dense_destroy"]


def test_columns_beyond_32_bits_are_refused(ops):
    """The C ABI takes 32 bits of them: 2^32 + 8 would be 8 there, and a call on the first 8 columns."""
    import torch
    from paper_2208_05321_amd import FreqCacheError
    empty = lambda *shape: torch.empty(*shape, dtype=torch.float16, device="meta")  # noqa: E731
    for d in ((1 << 20) + 1, (1 << 32) + 8):
        x, w, ids = empty(2, d), empty(d), torch.empty(2, dtype=torch.int64, device="meta")
        for call in (lambda: ops.token_embed_fwd(x, ids), lambda: ops.token_embed_bwd(x, ids, 4), lambda: ops.rms_norm_fwd(x, w),
                     lambda: ops.rms_norm_bwd(x, x, w)):
            with pytest.raises(FreqCacheError) as e:
                call()
            assert e.value.name == "INVALID_ARG"
    assert not _calls(ops)
    x, w = empty(2, 1 << 20), empty(1 << 20)
    ops.rms_norm_fwd(x, w)
    assert _calls(ops) == ["rms_norm_fwd"] and ops._L.calls[0][1][9] == 1 << 20


def test_reservations_beyond_32_bits_are_refused(ops):
    from paper_2208_05321_amd import FreqCacheError
    for sizes in ({"max_dim": (1 << 32) + 8}, {"max_tensors": (1 << 32) + 8}, {"max_dim": -(1 << 32) + 8}):
        with pytest.raises(FreqCacheError) as e:
            ops.reserve(**sizes)
        assert e.value.name == "INVALID_ARG"
    assert not _calls(ops)
    ops.reserve(max_tokens=1 << 31, max_dim=1 << 20, max_tensors=7)
    assert _calls(ops) == ["dense_reserve"]
