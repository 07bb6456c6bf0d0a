"""What sift_cache_append and e4m3 pools refuse, on the host."""

import ctypes

import pytest
import torch

from paper_2606_09441_amd import CachePages, SiftError
from paper_2606_09441_amd import _lib as B


def test_no_handle():
    t = B.SiftTensor(16, B.SIFT_BF16, 1, 4, 128)
    kv = B.SiftCacheKv()
    b = ctypes.byref
    assert B.lib().sift_cache_append(None, b(kv), None, b(t), b(t), None, None, None, None, None) == 1


def _pool(*shape):
    """A host tensor that says it is on a GPU, for checks that come before the library."""
    class Fake(torch.Tensor):
        @property
        def is_cuda(self):
            return True
    return torch.zeros(*shape, dtype=torch.uint8).view(torch.float8_e4m3fn).as_subclass(Fake)


def _status(fn, *a, **kw):
    with pytest.raises(SiftError) as e:
        fn(*a, **kw)
    return e.value.status


def test_e4m3_only_where_it_is_meant():
    with pytest.raises(ValueError):
        B.tensor_desc(_pool(16, 2, 64))
    d = B._pool_desc(_pool(16, 2, 64))
    assert (d.dtype, d.tokens, d.heads, d.head_dim) == (B.SIFT_E4M3, 16, 2, 64)


def test_pages_need_their_scales(monkeypatch):
    k = _pool(16, 2, 64)
    i = torch.zeros(1, 1, dtype=torch.int32)
    want = []
    monkeypatch.setattr(B, "require", lambda fn, t, name, *a: want.append((name, t is None)))
    CachePages(k, k, i, i)
    assert ("k_scales", True) in want and ("v_scales", True) in want
    monkeypatch.undo()
    plain = torch.zeros(16, 2, 64).as_subclass(type(k))
    monkeypatch.setattr(B, "require", lambda *a: None)
    assert _status(CachePages, plain, plain, i, i, k_scales=i) == 4
