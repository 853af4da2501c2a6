"""CPU-only checks of the entry points on a cache in use: what they refuse, before anything touches a GPU, and their workspace."""
import ctypes

import pytest
import torch

import cache_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_amd import binding
    return binding


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


P = 1 << 20     # stands for a device address; calls that are refused do not look at it
Q = 1 << 21


def cache(B, **changes):
    cu = i64(0, 100, 250)
    c = B.structkv_cache(P, P, 250 * 64, 64, 2, 64, B.STRUCTKV_DTYPE_BF16, 1, P, P, P, ctypes.addressof(cu), 2)
    c.keep = cu
    for k, v in changes.items():
        setattr(c, k, ctypes.addressof(v) if k == "cu_slots" and v is not None else v)
        c.keep = (c.keep, v)
    return c


BAD_CACHES = [
    (dict(n_kv_heads=0), 1), (dict(n_kv_heads=5000), 2), (dict(head_dim=0), 1), (dict(head_dim=257, stride_slot=300), 2), (dict(dtype=2), 2),
    (dict(planes=3), 1), (dict(planes=0), 1), (dict(batch=-1), 1), (dict(batch=65), 2), (dict(cu_slots=None), 1), (dict(cu_slots=i64(1, 2, 3)), 1),
    (dict(cu_slots=i64(0, 9, 3)), 1), (dict(cu_slots=i64(0, 1 << 31, 1 << 31)), 2), (dict(stride_slot=63), 1), (dict(stride_head=63), 1),
    (dict(stride_head=64), 1), (dict(stride_head=249 * 64 + 63), 1), (dict(lens=None), 1), (dict(lens=P + 2), 1), (dict(k=None), 1),
    (dict(v=None), 1), (dict(k=P + 1), 1), (dict(mass=P + 1), 1), (dict(pos=P + 2), 1),
]


@pytest.mark.parametrize("changes,status", BAD_CACHES)
def test_bad_caches(B, changes, status):
    c, L = cache(B, **changes), B._lib
    r = ctypes.byref(c)
    cu = i64(0, 1, 2)
    assert L.structkv_cache_workspace_bytes(r, 8, 2) == 0
    assert B.structkv_last_error()
    for got in (L.structkv_cache_append(r, P, P, 64, 64, cu, P, None, 0, Q, None),
                L.structkv_cache_attend(r, 8, 0.0, 0.0, None, P, 64, 64, cu, None, 0.0, P, P, P, 1 << 40, None),
                L.structkv_cache_accept(r, 8, 0.0, 0.0, None, P, 64, 64, P, cu, None, None, None, 0.0, Q, None),
                L.structkv_cache_evict(r, None, i64(1, 1), 0, Q, P, 1 << 40, None)):
        assert got == status, B.structkv_last_error()
        assert B.structkv_last_error()
    assert L.structkv_cache_evict(None, None, i64(1, 1), 0, Q, P, 1 << 40, None) == 1


def test_layouts_that_do_not_overlap(B):
    for changes in (dict(stride_head=249 * 64 + 64), dict(stride_head=64, stride_slot=128), dict(n_kv_heads=1, stride_head=0),
                    dict(mass=None, pos=None, planes=2), dict(batch=0), dict(cu_slots=i64(0, 0, 0), k=None, v=None)):
        assert B._lib.structkv_cache_workspace_bytes(ctypes.byref(cache(B, **changes)), 8, 2) > 0, B.structkv_last_error()


def test_workspace_bytes(B):
    size = lambda c, H, new: B._lib.structkv_cache_workspace_bytes(ctypes.byref(c), H, new)  # noqa: E731
    c = cache(B)
    assert size(c, 8, 0) > 0 and size(c, 8, 0) % 256 == 0
    assert size(c, 7, 1) == 0 and size(c, 0, 1) == 0 and size(c, 8192, 1) == 0
    assert size(c, 8, -1) == 0 and size(c, 8, 64 * 64) > size(c, 8, 1) and size(c, 8, 64 * 64 + 1) == 0
    big = cache(B, cu_slots=i64(0, 1 << 20, 1 << 21), stride_head=1 << 27)
    assert size(big, 8, 1) > size(c, 8, 1)


def test_append_refusals(B):
    def call(changes=None, k=P, v=P, sh=64, st=64, cu=i64(0, 1, 2), pos=P, mass=None, sp=0, out=Q):
        return B._lib.structkv_cache_append(ctypes.byref(cache(B, **(changes or {}))), k, v, sh, st, cu, pos, mass, sp, out, None)
    for bad in (dict(k=None), dict(v=None), dict(k=P + 1), dict(sh=-1), dict(st=-1), dict(sp=-1), dict(cu=None), dict(cu=i64(1, 1, 2)),
                dict(cu=i64(0, 2, 1)), dict(pos=None), dict(pos=P + 1), dict(mass=P + 2), dict(changes=dict(pos=None)),
                dict(changes=dict(mass=None), mass=P), dict(out=None), dict(out=Q + 1), dict(out=P), dict(out=P + 4)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(cu=i64(0, 1, 1 << 31)) == 2
    assert call(cu=i64(0, 1, 1 << 25)) == 2          # 2^25 rows of 64 elements
    assert call(changes=dict(batch=0), cu=i64(0)) == 0


def test_attend_refusals(B):
    def call(changes=None, H=8, scale=0.0, cap=0.0, slopes=None, q=P, st=64, sh=64, cu=i64(0, 1, 2), tree=None, lam=0.0, out=P, lse=P, ws=P,
             size=1 << 40):
        return B._lib.structkv_cache_attend(ctypes.byref(cache(B, **(changes or {}))), H, scale, cap, slopes, q, st, sh, cu, tree, lam, out,
                                            lse, ws, size, None)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(H=7), dict(H=0), dict(scale=-1.0), dict(scale=nan), dict(cap=-1.0), dict(cap=inf), dict(lam=-0.5), dict(lam=1.5), dict(lam=nan),
                dict(slopes=P + 1), dict(slopes=P, changes=dict(pos=None)), dict(lam=0.9, changes=dict(mass=None)), dict(tree=P + 4),
                dict(q=None), dict(q=P + 1), dict(st=-1), dict(sh=-8), dict(cu=None), dict(cu=i64(0, 3, 1)), dict(cu=i64(2, 3, 4)),
                dict(lam=0.9, cu=i64(0, 2, 3)), dict(out=None), dict(out=P + 1), dict(lse=None), dict(lse=P + 2)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(H=8192) == 2 and call(cu=i64(0, 65, 66)) == 2 and call(cap=1e-41) == 2 and call(scale=1e10, cap=1e-29) == 2
    assert call(ws=None) == 3 and call(ws=P + 128) == 3 and call(size=100, lam=0.9) == 3
    assert call(cu=i64(0, 0, 0), q=None, out=None, lse=None, ws=None) == 0 and call(changes=dict(batch=0), cu=i64(0), ws=None) == 0


def test_accept_refusals(B):
    def call(changes=None, H=8, scale=0.0, cap=0.0, slopes=None, q=P, st=64, sh=64, lse=P, cu=i64(0, 1, 2), tree=None, path=P, n=P, lam=0.5, out=Q):
        return B._lib.structkv_cache_accept(ctypes.byref(cache(B, **(changes or {}))), H, scale, cap, slopes, q, st, sh, lse, cu, tree, path, n,
                                            lam, out, None)
    nan = float("nan")
    for bad in (dict(H=7), dict(scale=nan), dict(cap=-1.0), dict(lam=nan), dict(lam=2.0), dict(lam=-1.0), dict(slopes=P, changes=dict(pos=None)),
                dict(changes=dict(mass=None)), dict(q=None), dict(lse=None), dict(lse=P + 1), dict(path=P + 2), dict(n=P + 1), dict(st=-1),
                dict(cu=None), dict(cu=i64(0, 3, 1)), dict(out=None), dict(out=P), dict(out=Q + 2), dict(tree=P + 1)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(cu=i64(0, 65, 66)) == 2 and call(cap=1e-41) == 2
    assert call(changes=dict(batch=0), cu=i64(0)) == 0


def test_evict_refusals(B):
    def call(changes=None, scores=P, budget=i64(1, 1), tail=0, out=Q, ws=P, size=1 << 40):
        return B._lib.structkv_cache_evict(ctypes.byref(cache(B, **(changes or {}))), scores, budget, tail, out, ws, size, None)
    for bad in (dict(scores=None, changes=dict(mass=None)), dict(scores=P + 1), dict(budget=None), dict(budget=i64(1, -1)), dict(tail=-1),
                dict(tail=1, changes=dict(pos=None)), dict(out=None), dict(out=P), dict(out=P + 4)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(ws=None) == 3 and call(ws=P + 8) == 3 and call(size=8) == 3
    assert call(changes=dict(cu_slots=i64(0, 1 << 27, 1 << 27), stride_head=1 << 33), budget=i64(1 << 26, 0)) == 2
    assert call(changes=dict(batch=0)) == 0


def test_binding_refuses_what_does_not_fit(B):
    k = torch.zeros(2, 100, 64)
    lens = torch.zeros(1, dtype=torch.int32)
    for bad in (dict(v=k[:, :50]), dict(v=k.bfloat16()), dict(k=k.half(), v=k.half()), dict(k=k[0], v=k[0]), dict(k=k[:, :, ::2], v=k[:, :, ::2]),
                dict(cu=[0, 101]), dict(lens=lens.long()), dict(lens=torch.zeros(2, dtype=torch.int32)), dict(mass=torch.zeros(3, 100)),
                dict(mass=torch.zeros(100, dtype=torch.float64)), dict(mass=torch.zeros(2, 99)), dict(pos=torch.zeros(100)),
                dict(mass=torch.zeros(2, 100), pos=torch.zeros(1, 100, dtype=torch.int32)), dict(mass=torch.zeros(2, 200)[:, ::2]), dict()):
        with pytest.raises(B.StructKVError) as e:     # (the last: a cache in host memory)
            B.make_cache(bad.get("k", k), bad.get("v", bad.get("k", k)), bad.get("cu", [0, 100]), bad.get("lens", lens), bad.get("mass"), bad.get("pos"))
        assert e.value.status == B.STRUCTKV_ERR_INVALID_ARG


def test_reference_on_cases_worked_by_hand():
    """Two slots with scores ln 1 and ln 3 and values 1 and 5: weights 1/4 and 3/4; a fresh slot that sees only itself; evictions."""
    import math
    c = R.make_cache(1, 1, 1, [4], [3], torch.float32, 0)
    c.k[0, :3, 0], c.v[0, :3, 0] = torch.tensor([0.0, math.log(3.0), 9.0]), torch.tensor([1.0, 5.0, 7.0])
    c.mass[:], c.pos[0] = 1.0, torch.tensor([3, 1, 8, 0])
    q = torch.ones(1, 1, 1)
    out, lse, mass, _ = R.attend(c, 1, q, [0, 1], [0], lam=0.5, scale=1.0)
    assert abs(float(out) - 4.0) < 1e-6 and abs(float(lse) - math.log(4.0)) < 1e-6
    assert torch.allclose(mass[0], torch.tensor([0.75, 1.25, 0.5, 1.0], dtype=torch.float64), atol=1e-6)
    c.mass[0] = torch.tensor([2.0, 2.0, 1.0, 0.0])
    k, v, pos, mass, lens = R.evict(c, c.mass, [2], 3)      # positions above 5 stay: slot 2; then slot 0 before its equal
    assert lens == [2] and v[0, :2, 0].tolist() == [1.0, 7.0] and pos[0, :2].tolist() == [3, 8] and mass[0, :2].tolist() == [2.0, 1.0]
    k, v, pos, mass, lens = R.accept(c, 1, q.expand(2, 1, 1), torch.zeros(2, 1), [0, 2], [1, 0], [1])
    assert lens == [2] and v[0, :2, 0].tolist() == [1.0, 7.0]


def test_planning_with_stub_launchers(B):
    """Valid calls through checks, planning and workspace of the host code (sanitizer build only: the launchers are stubs there, which
    hold the plan to what the kernels assume): the workspace query covers every way the tokens may spread."""
    if not hasattr(B._lib, "structkv_stub_last_attend"):
        pytest.skip("needs the stub launchers")
    import random
    rng = random.Random(5)
    last = (ctypes.c_int64 * 6)()
    for trial in range(400):
        batch = rng.choice((1, 1, 2, 8, 9, 64))
        caps = [rng.choice((0, 1, rng.randrange(300), rng.randrange(200000))) for _ in range(batch)]
        fresh = [rng.choice((0, 1, 1, rng.randrange(65))) for _ in range(batch)]
        single = rng.random() < 0.4
        if single:
            fresh = [min(f, 1) for f in fresh]
        G, gs, d = rng.choice((1, 2, 8, 32)), rng.choice((1, 3, 4, 8, 20)), rng.choice((1, 64, 80, 128, 256))
        cu, new = i64(*R.cut(caps)), i64(*R.cut(fresh))
        slots = cu[batch]
        c = cache(B, cu_slots=cu, batch=batch, n_kv_heads=G, head_dim=d, stride_slot=d, stride_head=max(1, slots) * d, planes=rng.choice((1, G)),
                  dtype=rng.choice((0, 1)))
        r = ctypes.byref(c)
        size = B._lib.structkv_cache_workspace_bytes(r, G * gs, new[batch])
        assert size > 0
        lam = 0.9 if single else 0.0
        assert B._lib.structkv_cache_attend(r, G * gs, 0.0, 0.0, None, P, G * gs * d, d, new, None, lam, P, P, P, size, None) == 0, B.structkv_last_error()
        if new[batch]:
            B._lib.structkv_stub_last_attend(last)
            assert last[4] <= size
        budget = i64(*[rng.randrange(1 << 18) for _ in caps])
        assert B._lib.structkv_cache_evict(r, None, budget, 4, Q, P, size, None) == 0
        assert B._lib.structkv_cache_append(r, P, P, d, d, new, P, P, 0, Q, None) == 0
        assert B._lib.structkv_cache_accept(r, G * gs, 0.0, 0.0, None, P, G * gs * d, d, P, new, None, P, P, 0.5, Q, None) == 0
