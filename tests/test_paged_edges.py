"""CPU-only checks of what the entry points of the cache held in pages, and of rotary positions, refuse at the ends of their ranges; beside
test_paged_abi.py, in the same manner."""
import ctypes

from test_paged_abi import B, P, Q, cache, i64, rotary  # noqa: F401  (B is the fixture)


def test_scales_that_leave_fp32(B):  # noqa: F811
    def call(scale, cap=0.0, cu=i64(0, 1, 2), ws=None):
        return B._lib.structkv_paged_attend(ctypes.byref(cache(B)), 8, scale, cap, P, 64, 64, cu, 0.0, P, P, ws, 1 << 40, None)
    assert call(2.0 ** 63) == 2 and "2^62" in B.structkv_last_error()
    assert call(2.0 ** 62) == 3 and call(1e-44) == 3 and call(2.0 ** 63, 2.0 ** 20) == 3     # (taken so far: the workspace is NULL)
