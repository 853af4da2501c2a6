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


def test_workspace_is_no_larger_than_it_has_to_be(B):  # noqa: F811
    """64 sequences of up to 64 drafts: the chunks' partial results (34 MB of 128 rows a workgroup for 512 of them) and the scores of single tokens;
    twice the blocks of 16 rows where sequences from 4096 slots on may be cut."""
    def size(G, gs, cap, new, **changes):
        cu = i64(*[cap * b for b in range(65)])
        c = cache(B, cu_slots=cu, batch=64, n_kv_heads=G, head_dim=128, stride_slot=128, stride_head=64 * cap * 128, **changes)
        return B._lib.structkv_cache_workspace_bytes(ctypes.byref(c), G * gs, new)
    part = 4 * (128 + 2)
    for G, gs in ((8, 4), (32, 1), (4, 8), (1, 32)):
        scores = 4 * G * gs * 64 * (2112 + 32)
        lists = 4 * 64 * (1 + 2 * 2112) + 4096
        assert size(G, gs, 2112, 64 * 64) <= max(512 * 128 * part + scores + 4096, lists)
        blocks = 2 * (4096 * gs + 15 * 64) // 16 * 16 * G
        assert size(G, gs, 8192, 64 * 64) <= max(512 * 128, blocks) * part + 4 * G * gs * 64 * (8192 + 32) + 4096
        assert size(G, gs, 8192, 64 * 64, mass=None) < 180 << 20
        assert size(G, gs, 2112, 64) <= 512 * (16 if gs <= 16 else 32) * part + 16 * G * 2 * 64 * ((gs + 15) // 16) * part + scores + 512 * 128 * part


def test_largest_plans_fit_the_workspace(B):  # noqa: F811
    """Spreads that need most of it (sanitizer build only, whose launchers keep the plan): all sequences alike, one with all its drafts, single tokens;
    none needs more than the query says, and the query says at most three times what some spread needs, or what 512 workgroups do."""
    if not hasattr(B._lib, "structkv_stub_last_attend"):
        pytest.skip("needs the stub launchers")
    last = (ctypes.c_int64 * 6)()
    for G, gs, d, dtype in ((8, 4, 128, 1), (32, 1, 128, 1), (2, 20, 64, 1), (8, 1, 64, 0), (1, 8, 80, 1), (4, 8, 256, 0), (64, 2, 128, 1)):
        for cap in (100, 1024, 4095, 4096, 20000):
            for batch in (1, 7, 64):
                cu = i64(*[cap * b for b in range(batch + 1)])
                c = cache(B, cu_slots=cu, batch=batch, n_kv_heads=G, head_dim=d, stride_slot=d, stride_head=cap * batch * d, dtype=dtype)
                for each in (1, 3, 5, 64):
                    spreads = [[each] * batch, [min(64, each * batch)] + [0] * (batch - 1), [0] * (batch // 2) + [each] * (batch - batch // 2)]
                    need, size = 0, B._lib.structkv_cache_workspace_bytes(ctypes.byref(c), G * gs, each * batch)
                    for fresh in spreads:
                        new = i64(*[sum(fresh[:b]) for b in range(batch + 1)])
                        for q in (P, P + 4):                            # (not aligned for the bf16 kernels)
                            for lam in (0.0, 0.5) if max(fresh) == 1 else (0.0,):
                                assert B._lib.structkv_cache_attend(ctypes.byref(c), G * gs, 0.0, 0.0, None, q, G * gs * d, d, new, None, lam, P, P, P,
                                                                    size, None) == 0, B.structkv_last_error()
                                B._lib.structkv_stub_last_attend(last)
                                need = max(need, last[4])
                    assert need <= size
                    scores = 4 * G * gs * (cap + 32) * batch
                    evict = 4 * batch * (1 + 2 * cap) + 8192
                    assert size <= max(evict, 3 * need + scores + 512 * 128 * 4 * (max(64, d) + 2) + 4096)
