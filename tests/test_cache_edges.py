"""CPU-only checks of the entry points on a cache in use, beside test_cache_abi.py: limits that those do not reach."""
import ctypes

import pytest
import torch

from test_cache_abi import B, P, cache, i64  # noqa: F401  (B is the fixture)


def test_missed_is_checked(B):  # noqa: F811
    assert B._lib.structkv_cache_workspace_bytes(ctypes.byref(cache(B, missed=P)), 8, 2) > 0
    assert B._lib.structkv_cache_workspace_bytes(ctypes.byref(cache(B, missed=P + 2)), 8, 2) == 0
    assert "missed" in B.structkv_last_error()
    k, lens = torch.zeros(2, 100, 64), torch.zeros(1, dtype=torch.int32)
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(1), torch.zeros(2, dtype=torch.int32)[::2]):
        with pytest.raises(B.StructKVError):
            B.make_cache(k, k, [0, 100], lens, missed=bad)


def test_softcaps_whose_parts_leave_the_range(B):  # noqa: F811
    """Each number that the kernels work with has to be one, not their products alone: at 1 / softcap = infinity a score of zero would be NaN."""
    def call(scale, cap):
        return B._lib.structkv_cache_attend(ctypes.byref(cache(B)), 8, scale, cap, None, P, 64, 64, i64(0, 1, 2), None, 0.0, P, P, P, 8, None)

    def accept(scale, cap):
        return B._lib.structkv_cache_accept(ctypes.byref(cache(B)), 8, scale, cap, None, None, 64, 64, P, i64(0, 1, 2), None, None, None, 0.5, 1 << 21,
                                            None)
    for scale, cap in ((0.01, 1e-39), (1e-3, 2e-39), (0.0, 2e-39), (1.0, 3e38), (0.01, 1e37), (1e-38, 10.0), (1e38, 1.0)):
        assert call(scale, cap) == 2 and accept(scale, cap) == 2, (scale, cap)
        assert "softcap" in B.structkv_last_error()
    for scale, cap in ((0.01, 1e-30), (0.0, 1e36), (1.0, 30.0), (0.0, 1e-37)):
        assert call(scale, cap) == 3 and accept(scale, cap) == 1, (scale, cap)       # (what is wrong with the rest of these calls)
        assert "softcap" not in B.structkv_last_error()
