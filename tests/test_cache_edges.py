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
