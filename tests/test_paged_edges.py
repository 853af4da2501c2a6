"""CPU-only checks of what the entry points of the cache held in pages, and of rotary positions, refuse at the ends of their ranges; beside
test_paged_abi.py, in the same manner."""
import ctypes
import math

import pytest
import torch

import paged_precision as L

from test_paged_abi import B, P, Q, cache, i64, rotary  # noqa: F401  (B is the fixture)


def test_scales_that_leave_fp32(B):  # noqa: F811
    def call(scale, cap=0.0, cu=i64(0, 1, 2), ws=None):
        return B._lib.structkv_paged_attend(ctypes.byref(cache(B)), 8, scale, cap, P, 64, 64, cu, 0.0, P, P, ws, 1 << 40, None)
    assert call(2.0 ** 63) == 2 and "2^62" in B.structkv_last_error()
    assert call(2.0 ** 62) == 3 and call(1e-44) == 3 and call(2.0 ** 63, 2.0 ** 20) == 3     # (taken so far: the workspace is NULL)


def test_more_threads_than_a_launch_has(B):  # noqa: F811
    """Calls whose launches would have 2^32 threads or more are refused before anything touches a GPU."""
    def append(tokens, **changes):
        c = cache(B, page_size=16, batch=1, max_pages=1 << 26, pages_stride=1 << 26, **changes)
        return B._lib.structkv_paged_append(ctypes.byref(c), P, P, 1 << 40, 16, i64(0, tokens), None, None, 0, None, 0, 0, None, Q, None)
    like = dict(n_kv_heads=64, head_dim=16, stride_tok=16, stride_head=256, stride_page=64 * 256)
    if not hasattr(B._lib, "structkv_stub_last_attend"):                                      # (the launcher's own check)
        assert append(1 << 23, **like) == 2, B.structkv_last_error()                          # 2^19 pages, 128 workgroups of 64 threads each
    # (4096 tokens of each of 64 sequences, 4096 KV heads: 2^25 workgroups of 256 threads)
    c = cache(B, batch=64, head_dim=16, n_kv_heads=4096, stride_tok=16, stride_head=32 * 16, stride_page=4096 * 32 * 16)
    full = i64(*[4096 * b for b in range(65)])
    assert B._lib.structkv_paged_attend(ctypes.byref(c), 4096, 0.0, 0.0, P, 1 << 16, 16, full, 0.0, P, P, P, 1 << 60, None) == 2, B.structkv_last_error()


def test_most_rows_of_a_rotation(B):  # noqa: F811
    def call(tokens, d):
        return B._lib.structkv_rotate(ctypes.byref(rotary(B, rot_dim=min(d, 64))), P, d, d, tokens, 1, d, 1, P, 0, Q, d, d, None)
    assert call(1 << 35, 2) == 2 and call(1 << 35, 256) == 2


@pytest.mark.parametrize("d", [16, 64, 128, 256])
def test_precision_tells_fewer_bits_apart(d):
    """What test_gpu_paged_edges.py allows fp32 results is less than queries of two bf16 parts, or weights of one fp16 part, are off by."""
    c, H, q, cu_new, scale = L.case(d)
    ref, ref_lse, out_off, lse_off = L.attend(c, H, q, cu_new, scale)
    out, lse, _, _ = L.attend(c, H, q, cu_new, scale, query_bits=16)
    assert L.worst(out, ref, out_off) > 2 * L.MOST and L.worst(lse, ref_lse, lse_off) > 2 * L.MOST
    out, _, _, _ = L.attend(c, H, q, cu_new, scale, weight_bits=11)
    assert L.worst(out, ref, out_off) > 2 * L.MOST


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,T", [((500, 90), 3), ((1700, 90), 1)])
def test_last_bits_tell_weights_of_11_bits_apart(d, lens, T):
    c, H, q, cu_new, scale = L.case(d, lens, T)
    q = q.bfloat16()
    ref, _, off, _ = L.attend(c, H, q, cu_new, scale)
    few, _, _, _ = L.attend(c, H, q, cu_new, scale, weight_bits=11)
    spread = torch.randn(ref.shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * off[..., None] / math.sqrt(d)
    turned = lambda x: float((x.bfloat16() != ref.bfloat16()).double().mean())  # noqa: E731
    assert turned(few) > 2 * L.TURNED and turned(ref + L.MOST * spread) < 0.5 * L.TURNED
