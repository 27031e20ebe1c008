"""CPU-side checks of the dense operators' entry points: arguments are refused before any device is touched, and there is no CPU path."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2208_05321_amd.binding import LIB_PATH, load_library
    if not os.path.exists(LIB_PATH):
        from paper_2208_05321_amd.build import build
        build()
    return load_library()


def test_no_handle(lib):
    assert lib.dense_create(None, None) == -1
    assert lib.dense_reserve(None, 1, 1, 1, 1) == -1 and lib.dense_check(None) == -1 and lib.dense_destroy(None) == -1
    assert lib.token_embed_fwd(None, 1, 0, 8, 4, 8, 1, 6, 2, 1.0, 1, 0, 8) == -1
    assert lib.token_embed_bwd(None, 1, 0, 8, 1, 6, 2, 4, 8, 1.0, -1, 1, 0, 8, 0) == -1
    assert lib.rms_norm_fwd(None, 1, 0, 8, None, 0, 1, 0, 2, 8, 1e-6, None, 0, 1, 0, 8, None, 0) == -1
    assert lib.rms_norm_bwd(None, 1, 8, 1, 0, 8, 1, 0, None, 0, 2, 8, 1e-6, 1, 8, 1, 0) == -1
    assert lib.grad_norm_clip(None, None, None, None, None, 0, 1.0, 1) == -1


def test_no_gpu(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2208_05321_amd import DenseOps, FreqCacheError
    h = ctypes.c_void_p()
    assert lib.dense_create(None, ctypes.byref(h)) == -8 and not h.value
    with pytest.raises(FreqCacheError) as e:
        DenseOps()
    assert e.value.name == "HIP"
