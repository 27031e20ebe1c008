"""CPU-side checks of the calls on rows of logits: arguments are refused before any device is touched, and sizes that the C ABI would cut do not reach it."""
import os

import pytest

from tests.test_dense_binding import _calls, ops  # noqa: F401 (a binding whose library only notes its calls)


@pytest.fixture(scope="module")
def lib():
    from paper_2208_05321_amd.binding import LIB_PATH, load_library
    if not os.path.exists(LIB_PATH):
        from paper_2208_05321_amd.build import build
        build()
    return load_library()


def test_no_handle(lib):
    assert lib.distill_fwd(None, 1, 0, 8, 2, 8, 1, 6, 1, 0, 1, None, None, 6, 1.0, 1.0, 1, 1) == -1
    assert lib.distill_bwd(None, 1, 1, 1, 0, 8, 2, 8, 1, 6, 1, 0, 1, None, 6, 1.0, 1.0, 1, 1, 8) == -1
    assert lib.distill_grad(None, 1, 1, 1, 0, 8, 2, 8, 1, 6, 1, 0, 1, None, None, 6, 1.0, 1.0, 1, 1, 8) == -1
    assert lib.beam_select(None, 1, 0, 8, 1, 2, 8, 1, None, -1, 2, 1, 1, 1, 6, None) == -1
    assert lib.beam_reorder(None, None, 0, 1, 2, 1, 5, 2) == -1


def _empty(*shape, dtype=None):
    import torch
    return torch.empty(*shape, dtype=dtype or torch.float32, device="meta")


def test_columns_beyond_32_bits_are_refused(ops):  # noqa: F811
    import torch
    from paper_2208_05321_amd import FreqCacheError
    for v in ((1 << 20) + 1, (1 << 32) + 8):
        x, ids, z = _empty(2, v), _empty(2, 3, dtype=torch.int64), _empty(2, 3)
        for call in (lambda: ops.distill_fwd(x, ids, z), lambda: ops.distill_bwd(_empty(2), x, ids, z, _empty(2, 12)), lambda: ops.distill_grad(_empty(2), x, ids, z),
                     lambda: ops.beam_select(_empty(1, 2, v), _empty(1, 2))):
            with pytest.raises(FreqCacheError) as e:
                call()
            assert e.value.name == "INVALID_ARG"
    assert not _calls(ops)


def test_what_reaches_the_library(ops):  # noqa: F811
    import torch
    ops.distill_grad(_empty(1), _empty(2, 5, 40)[:, :, :39], _empty(2, 5, 3, dtype=torch.int32), _empty(2, 5, 3, dtype=torch.float16), targets=_empty(2, 5, dtype=torch.int64), alpha=0.25)
    name, a = ops._L.calls[-1]
    assert name == "distill_grad" and a[2] == 0 and a[4:8] == (0, 40, 10, 39) and a[9] == 5 and a[11:13] == (2, 3) and a[15:18] == (6, 1.0, 0.25) and a[20] == 39
    ops.beam_select(_empty(3, 4, 50, dtype=torch.bfloat16), _empty(3, 4), 8, eos_id=2, token_dtype=torch.int32)
    name, a = ops._L.calls[-1]
    assert name == "beam_select" and a[2:7] == (1, 50, 3, 4, 50) and a[9:11] == (2, 8) and a[14] == 5


def test_layouts_of_states(ops):  # noqa: F811
    """Rows and pieces in bytes: of contiguous tensors, of the filled part of buffers, of single beams and of single sequences; what overlaps is refused."""
    from paper_2208_05321_amd import FreqCacheError
    f = lambda *s: _empty(*s)  # noqa: E731
    assert ops._state(f(2, 3, 5, 7), 2, "t") == (140, 140, 140, 1)
    assert ops._state(f(2, 3, 4, 9, 7)[:, :, :, :5], 2, "t") == (1008, 252, 140, 4)
    assert ops._state(f(2, 3, 9, 7)[:, :, :5], 2, "t") == (252, 140, 140, 1)
    assert ops._state(f(2, 1, 9, 7)[:, :, :5], 2, "t") == (252, 140, 140, 1)
    assert ops._state(f(1, 3, 9, 7)[:, :, :5], 1, "t") == (252, 140, 140, 1)
    assert ops._state(f(1, 1, 4, 9, 7)[:, :, :, :5], 1, "t") == (896, 252, 140, 4)
    for bad in (f(2, 3, 1).expand(2, 3, 4), f(2, 1, 4).expand(2, 3, 4), f(1, 3, 4).expand(2, 3, 4), f(4, 3, 8)[::2], f(2, 3, 4, 4, 4)[:, :, ::2, :, ::2], f(3, 2, 4).transpose(0, 1)):
        with pytest.raises(FreqCacheError) as e:
            ops._state(bad, 2, "t")
        assert e.value.name == "INVALID_ARG"


def test_a_state_given_twice(ops):  # noqa: F811
    """Rows would be moved twice, or read after others had taken their place; a tensor without elements may be there several times."""
    from paper_2208_05321_amd import FreqCacheError
    row, none = (20, 20, 20, 20, 20, 1), (0, 0, 0, 0, 0, 1)

    def table(*pairs):
        return [v for t, o in pairs for v in (t, o, *(row if t or o else none))]
    for pairs in ([(1, 1), (2, 2), (1, 1)], [(1, 3), (2, 3)], [(1, 3), (2, 1)], [(1, 2), (2, 1)], [(1, 1), (2, 1)], [(0, 0), (1, 2), (2, 4)]):
        with pytest.raises(FreqCacheError) as e:
            ops._apart(table(*pairs))
        assert e.value.name == "INVALID_ARG"
    for pairs in ([(1, 1), (2, 2), (0, 0), (0, 0)], [(1, 2), (1, 3)], [(1, 1), (2, 2)], [(1, 1), (2, 3), (0, 0)]):
        ops._apart(table(*pairs))
