"""CPU-side check of beam_reorder's arguments: parents that are one of the tensors written are refused, as workgroups would read them after others had moved them."""
import pytest

from tests.test_dense_binding import _calls, ops  # noqa: F401 (a binding whose library only notes its calls)


def test_parents_among_what_is_written(ops):  # noqa: F811
    import torch
    from paper_2208_05321_amd import FreqCacheError
    ops._written = lambda t: None
    p, a = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 5)
    for call in (lambda: ops.beam_reorder([a, p], p), lambda: ops.beam_reorder([p.view(2, 3, 1)], p), lambda: ops.beam_reorder([a, p.clone()], p, out=[a.clone(), p])):
        with pytest.raises(FreqCacheError) as e:
            call()
        assert e.value.name == "INVALID_ARG"
    assert not _calls(ops)
    ops.beam_reorder([a, p], p, out=[a.clone(), p.clone()])          # read only
    ops.beam_reorder([a, p.clone()], p)
    assert _calls(ops) == ["beam_reorder"] * 2
