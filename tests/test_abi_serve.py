"""Host-side checks of include/sift_serve.h that need no GPU: every declared
function is exported and bound with its argument types, and malformed arguments
are rejected before the device is touched."""

import ctypes

from paper_2606_09441_amd import _lib as B


def test_every_declared_function_is_exported_and_bound():
    L = B.lib()
    names = B.header_functions(B.SERVE_HEADER)
    assert set(names) == set(B._SERVE_SIGS)
    for n in names:
        assert getattr(L, n).argtypes == B._SERVE_SIGS[n][1]


def _create(*a):
    h = ctypes.c_void_p()
    return B.lib().sift_cache_create(*a, ctypes.byref(h))


def test_cache_sizes_are_checked_on_the_host():
    assert B.lib().sift_cache_create(1, 4, 2, 128, 64, 4, 1, None) == 1
    for bad in ((0, 4, 2), (1, 0, 2), (1, 4, 0), (1, 4, 3)):
        assert _create(*bad, 128, 64, 4, 1) == 2
    assert _create(1, 4, 2, 128, 64, 0, 1) == 2
    assert _create(1, 4, 2, 128, 64, 4, 0) == 2
    assert _create(1, 4, 2, 96, 64, 4, 1) == 4
    assert _create(1, 4, 2, 128, 48, 4, 1) == 4
    assert _create(1, 4, 2, 128, 128, 1 << 24, 1) == 5
    assert _create(1, 1 << 20, 1, 128, 64, 4, 1 << 20) == 5
    assert B.lib().sift_cache_destroy(None) == 0


def test_missing_handles_are_rejected():
    L = B.lib()
    t = B.SiftTensor(1, B.SIFT_BF16, 1, 4, 128)
    kv, score = B.SiftCacheKv(), B.SiftScore()
    b = ctypes.byref
    assert L.sift_plan_dense(None, b(t), b(t), b(t), 0, b(score), b(t), None, None) == 1
    assert L.sift_cache_attention(None, b(kv), None, b(t), b(t), b(t), None, 0, b(score), b(t), None,
                                  None) == 1
    assert L.sift_cache_accumulate(None, b(kv), None, b(t), None, None, b(score), None, 1.0, None,
                                   None) == 1
    assert L.sift_cache_evict(None, b(kv), None, None, 1, 0, 0, None, None, None, None) == 1
