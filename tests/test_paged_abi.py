"""CPU-only checks of rotary positions and of the cache held in 8 bits, in pages: what the entry points refuse, before anything touches a
GPU, the frequencies that the host works out, the workspace, and the 64-bit definitions that the GPU tests compare with."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

import paged_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_amd import binding
    return binding


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


P = 1 << 20     # stands for a device address; calls that are refused do not look at it
Q = 1 << 21
NAN, INF = float("nan"), float("inf")


def cache(B, **changes):
    c = B.structkv_paged(P, P, P, P, 2 * 32 * 64, 32 * 64, 64, 2, 64, B.STRUCTKV_DTYPE_BF16, 32, 100, 8, 2, 8, P, P, P, P)
    for k, v in changes.items():
        setattr(c, k, v)
    return c


def rotary(B, **changes):
    r = B.structkv_rotary(P, 64, 0, 1.0)
    for k, v in changes.items():
        setattr(r, k, v)
    return r


BAD_CACHES = [
    (dict(n_kv_heads=0), 1), (dict(n_kv_heads=5000), 2), (dict(head_dim=0), 1), (dict(head_dim=72), 2), (dict(head_dim=272), 2), (dict(dtype=2), 2),
    (dict(page_size=0), 2), (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=512), 2), (dict(n_pages=-1), 1), (dict(max_pages=-1), 1),
    (dict(max_pages=1 << 26, pages_stride=1 << 26), 2), (dict(batch=-1), 1), (dict(batch=65), 2), (dict(pages_stride=7), 1), (dict(k=None), 1), (dict(v=None), 1),
    (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(k=P + 8), 1), (dict(v=P + 1), 1), (dict(k_scale=P + 2), 1), (dict(stride_tok=72), 1),
    (dict(stride_tok=-64), 1), (dict(stride_tok=48), 1), (dict(stride_head=31 * 64), 1), (dict(stride_page=32 * 64), 1), (dict(stride_page=0), 1),
    (dict(stride_tok=1 << 26, stride_head=1 << 32, stride_page=1 << 34), 2), (dict(pages=None), 1), (dict(pages=P + 2), 1), (dict(lens=None), 1),
    (dict(lens=P + 1), 1), (dict(mass=P + 2), 1), (dict(missed=P + 1), 1),
]


@pytest.mark.parametrize("changes,status", BAD_CACHES)
def test_bad_caches(B, changes, status):
    r, L, cu = ctypes.byref(cache(B, **changes)), B._lib, i64(0, 1, 2)
    assert L.structkv_paged_workspace_bytes(r, 8, 2) == 0 and B.structkv_last_error()
    for got in (L.structkv_paged_append(r, P, P, 64, 64, cu, None, None, 0, None, 0, 0, None, Q, None),
                L.structkv_paged_attend(r, 8, 0.0, 0.0, P, 64, 64, cu, 0.0, P, P, P, 1 << 40, None)):
        assert got == status, B.structkv_last_error()
        assert B.structkv_last_error()
    assert L.structkv_paged_append(None, P, P, 64, 64, cu, None, None, 0, None, 0, 0, None, Q, None) == 1
    assert L.structkv_paged_attend(None, 8, 0.0, 0.0, P, 64, 64, cu, 0.0, P, P, P, 1 << 40, None) == 1


def test_layouts_that_lie_apart(B):
    for changes in (dict(stride_head=64, stride_tok=128), dict(stride_tok=80, stride_head=32 * 80, stride_page=2 * 32 * 80),
                    dict(n_kv_heads=1, stride_head=0), dict(stride_page=64, stride_tok=6400, stride_head=32 * 6400), dict(n_pages=0, k=None, v=None),
                    dict(batch=0, pages=None, lens=None), dict(max_pages=0, pages=None), dict(batch=1, pages_stride=0), dict(mass=None, missed=None)):
        assert B._lib.structkv_paged_workspace_bytes(ctypes.byref(cache(B, **changes)), 8, 2) > 0, (changes, B.structkv_last_error())


def test_workspace_bytes(B):
    size = lambda c, H, new: B._lib.structkv_paged_workspace_bytes(ctypes.byref(c), H, new)  # noqa: E731
    c = cache(B)
    assert size(c, 8, 0) > 0 and size(c, 8, 0) % 256 == 0
    assert size(c, 7, 1) == 0 and size(c, 0, 1) == 0 and size(c, 8192, 1) == 0 and size(c, 8, -1) == 0
    assert size(c, 8, 64 * 4096) > size(c, 8, 1) and size(c, 8, 64 * 4096 + 1) == 0
    assert size(cache(B, max_pages=1 << 20, pages_stride=1 << 20), 8, 1) > size(c, 8, 1)


def test_append_refusals(B):
    def call(changes=None, k=P, v=P, sh=64, st=64, cu=i64(0, 1, 2), rot=None, pos=None, H=8, q=None, qst=64, qsh=64, q_out=P, out=Q):
        return B._lib.structkv_paged_append(ctypes.byref(cache(B, **(changes or {}))), k, v, sh, st, cu, None if rot is None else ctypes.byref(rot),
                                            pos, H, q, qst, qsh, q_out, out, None)
    rot = rotary(B)
    for bad in (dict(k=None), dict(v=None), dict(k=P + 1), dict(v=P + 1), dict(sh=-1), dict(st=-1), dict(cu=None), dict(cu=i64(1, 1, 2)), dict(cu=i64(0, 2, 1)),
                dict(pos=P + 1), dict(q=P), dict(q=P, rot=rot, H=7), dict(q=P, rot=rot, H=0), dict(q=P + 1, rot=rot), dict(q=P, rot=rot, q_out=None),
                dict(q=P, rot=rot, q_out=P + 1), dict(q=P, rot=rot, qst=-1), dict(q=P, rot=rot, qsh=-1), dict(out=None), dict(out=Q + 1), dict(out=P), dict(out=P + 4),
                dict(rot=rotary(B, turns=None)), dict(rot=rotary(B, turns=P + 4)), dict(rot=rotary(B, rot_dim=0)), dict(rot=rotary(B, rot_dim=7)),
                dict(rot=rotary(B, rot_dim=66)), dict(rot=rotary(B, interleaved=2)), dict(rot=rotary(B, magnitude=NAN)), dict(rot=rotary(B, magnitude=INF))):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(cu=i64(0, 1, 1 << 31)) == 2 and call(q=P, rot=rot, H=8192) == 2
    assert call(cu=i64(0, 1, (1 << 31) - 1), changes=dict(page_size=16, n_kv_heads=64, stride_head=16 * 64, stride_page=64 * 16 * 64)) == 2
    assert call(changes=dict(batch=0), cu=i64(0), out=None) == 0


def test_attend_refusals(B):
    def call(changes=None, H=8, scale=0.0, cap=0.0, q=P, st=64, sh=64, cu=i64(0, 1, 2), lam=0.0, out=P, lse=P, ws=P, size=1 << 40):
        return B._lib.structkv_paged_attend(ctypes.byref(cache(B, **(changes or {}))), H, scale, cap, q, st, sh, cu, lam, out, lse, ws, size, None)
    for bad in (dict(H=7), dict(H=0), dict(scale=-1.0), dict(scale=NAN), dict(cap=-1.0), dict(cap=INF), dict(lam=-0.5), dict(lam=1.5), dict(lam=NAN),
                dict(lam=0.9, changes=dict(mass=None)), dict(q=None), dict(q=P + 1), dict(st=-1), dict(sh=-8), dict(cu=None), dict(cu=i64(0, 3, 1)),
                dict(cu=i64(2, 3, 4)), dict(lam=0.9, cu=i64(0, 2, 3)), dict(out=None), dict(out=P + 1), dict(lse=None), dict(lse=P + 2)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(H=8192) == 2 and call(cu=i64(0, 4097, 4098)) == 2 and call(cap=1e-41) == 2 and call(scale=1e10, cap=1e-29) == 2
    assert call(H=128, cu=i64(0, 4096, 4096)) == 2            # 2^18 query rows of a KV head
    assert call(ws=None) == 3 and call(ws=P + 128) == 3 and call(size=100, lam=0.9) == 3
    assert call(cu=i64(0, 0, 0), q=None, out=None, lse=None, ws=None) == 0 and call(changes=dict(batch=0), cu=i64(0), ws=None) == 0


def test_rotate_refusals(B):
    def call(rot=rotary(B), x=P, xt=64, xh=64, tokens=4, heads=1, d=64, dtype=1, pos=P, inverse=0, out=Q, ot=64, oh=64):
        return B._lib.structkv_rotate(None if rot is None else ctypes.byref(rot), x, xt, xh, tokens, heads, d, dtype, pos, inverse, out, ot, oh, None)
    for bad in (dict(rot=None), dict(rot=rotary(B, turns=None)), dict(rot=rotary(B, rot_dim=66)), dict(rot=rotary(B, rot_dim=3)), dict(rot=rotary(B, interleaved=-1)),
                dict(rot=rotary(B, magnitude=-INF)), dict(tokens=-1), dict(heads=0), dict(d=0), dict(xt=-1), dict(xh=-1), dict(ot=-1), dict(oh=-1), dict(x=None),
                dict(out=None), dict(pos=None), dict(x=P + 1), dict(out=Q + 1), dict(pos=P + 2), dict(inverse=2), dict(ot=63), dict(ot=0), dict(heads=2, oh=32),
                dict(out=P, xt=128), dict(heads=2, xh=128, xt=64, oh=256, out=P)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())
    assert call(dtype=2) == 2 and call(d=70000, ot=70000) == 2 and call(heads=65536, oh=64, ot=1 << 23) == 2 and call(tokens=1 << 40) == 2 and call(tokens=1 << 35) == 2
    assert call(tokens=0, x=None, out=None, pos=None) == 0


def test_turns_refusals(B):
    out, mag = (ctypes.c_uint64 * 64)(), ctypes.c_float()
    def call(rot=8, base=1e4, scaling=0, factor=1.0, original=8192.0, low=1.0, high=4.0, turns=out, m=ctypes.byref(mag)):
        return B._lib.structkv_rotary_turns(rot, base, scaling, factor, original, low, high, turns, m)
    assert call() == 0 and call(scaling=4, factor=8.0) == 0 and call(scaling=3, factor=8.0, low=32.0, high=1.0) == 0
    assert call(original=0.0, low=NAN, factor=0.0) == 0                 # (read by no plain frequencies)
    for bad in (dict(rot=0), dict(rot=3), dict(rot=65538), dict(base=1.0), dict(base=NAN), dict(base=INF), dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5),
                dict(scaling=1, factor=NAN), dict(scaling=2, rot=2, factor=2.0), dict(scaling=4, original=0.0), dict(scaling=4, low=4.0), dict(scaling=3, low=1.0, high=4.0),
                dict(scaling=3, low=INF, high=1.0), dict(scaling=2, factor=1e300), dict(turns=None), dict(m=None)):
        assert call(**bad) == 1, (bad, B.structkv_last_error())


def test_turns_of_exact_powers(B):
    """base 16 over 8 components: frequencies 1, 1/2, 1/4, 1/8 radians; 2^64 / (2 pi) to the nearest from pi's digits."""
    pi = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)
    def nearest(x):
        return math.floor(x + Fraction(1, 2))
    turns, mag = B.structkv_rotary_turns(8, 16.0)
    want = [nearest(2 ** 64 / (2 * pi) / 2 ** i) for i in range(4)]
    assert all(abs(a - b) <= 1 << (3 - i) for i, (a, b) in enumerate(zip(R.turns_of(turns), want))) and mag == 1.0   # (64 bits' own last one)
    turns, mag = B.structkv_rotary_turns(8, 16.0, "linear", 4.0)
    assert all(abs(a - b / 4) <= 2 for a, b in zip(R.turns_of(turns), want)) and mag == 1.0


def test_turns_scaled(B):
    """Against the formulas in 64 bits of floating point: 2^-52 of a frequency per operation, some ten of them."""
    rot, base, factor, original = 128, 500000.0, 8.0, 8192.0
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    def check(got, want):
        for a, w in zip(R.turns_of(got), want):
            assert abs(a - w / (2 * math.pi) * 2.0 ** 64) <= 16 * 2.0 ** -52 * a + 1
    check(B.structkv_rotary_turns(rot, base)[0], f)
    check(B.structkv_rotary_turns(rot, base, "linear", factor)[0], [x / factor for x in f])
    stretched = base * factor ** (rot / (rot - 2))
    check(B.structkv_rotary_turns(rot, base, "ntk", factor)[0], [stretched ** (-2.0 * i / rot) for i in range(rot // 2)])
    assert abs(stretched ** (-2.0 * 63 / rot) * factor - f[63]) < 1e-12    # the lowest frequency is divided by the factor
    turns, mag = B.structkv_rotary_turns(rot, base, "bands", factor, original, 1.0, 4.0)
    want = []
    for x in f:
        n = original * x / (2 * math.pi)
        want.append(x / factor if n < 1.0 else x if n > 4.0 else x / factor + (n - 1.0) / 3.0 * (x - x / factor))
    check(turns, want)
    assert mag == 1.0
    turns, mag = B.structkv_rotary_turns(rot, base, "yarn", factor, original, 32.0, 1.0)
    at = lambda n: rot * math.log(original / (n * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(0, math.floor(at(32.0))), min(rot - 1, math.ceil(at(1.0)))
    ramp = [min(1.0, max(0.0, (i - lo) / (hi - lo))) for i in range(rot // 2)]
    check(turns, [x * (1 - r) + x / factor * r for x, r in zip(f, ramp)])
    assert abs(mag - (0.1 * math.log(factor) + 1)) < 1e-7 and R.turns_of(turns)[0] == R.turns_of(B.structkv_rotary_turns(rot, base)[0])[0]
    with pytest.raises(B.StructKVError):
        B.structkv_rotary_turns(rot, base, "other", factor)


def test_binding_refuses_what_does_not_fit(B):
    k = torch.zeros(10, 2, 16, 64, dtype=torch.uint8)
    s, pages, lens = torch.ones(10, 2), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for bad in (dict(v=k[:5]), dict(k=k.float()), dict(k=k[0]), dict(k=k[..., ::2]), dict(ks=s[:5]), dict(ks=s.double()), dict(pages=pages.long()), dict(pages=pages[0]),
                dict(lens=lens.long()), dict(lens=lens.repeat(2)), dict(dtype=torch.half), dict(mass=torch.zeros(1, 3)), dict()):
        with pytest.raises(B.StructKVError) as e:     # (the last: a cache in host memory)
            x = bad.get("k", k)
            B.make_paged(x, bad.get("v", x), bad.get("ks", s), s, bad.get("pages", pages), bad.get("lens", lens), bad.get("dtype", torch.bfloat16), bad.get("mass"))
        assert e.value.status == B.STRUCTKV_ERR_INVALID_ARG
    for turns in (torch.zeros(4), torch.zeros(4, dtype=torch.int64), torch.zeros(2, 2, dtype=torch.int64)):
        with pytest.raises(B.StructKVError):
            B.make_rotary(turns)


def test_reference_on_cases_worked_by_hand():
    # codes: 1.0 is exponent 7; the least subnormal; ties to the even code; 448 the largest
    assert R.decode(torch.tensor([0x38, 0x01, 0x7E, 0xB8, 0x08], dtype=torch.uint8)).tolist() == [1.0, 2.0 ** -9, 448.0, -1.0, 2.0 ** -6]
    assert R.encode(torch.tensor([1.0, 1.0625, 1.1875, 448.0, -2.0 ** -10, 3 * 2.0 ** -10, math.nan], dtype=torch.float64)).tolist() == [
        0x38, 0x38, 0x3A, 0x7E, 0x80, 2, 127]
    every = torch.arange(255, dtype=torch.uint8)
    every = every[(every & 127) != 127]
    assert torch.equal(R.encode(R.decode(every)), every)
    assert R.scale_for(448.0) == 1.0 and R.scale_for(448.1) == 2.0 and R.scale_for(0.0) == 2.0 ** -64 and R.scale_for(7.0) == 2.0 ** -6
    # a quarter turn a position
    x = torch.tensor([[[1.0, 2.0, 5.0]]])
    assert torch.allclose(R.rotated(x, [1], [1 << 62], True), torch.tensor([[[-2.0, 1.0, 5.0]]], dtype=torch.float64))
    assert torch.allclose(R.rotated(x, [-1], [1 << 62], False), torch.tensor([[[2.0, -1.0, 5.0]]], dtype=torch.float64))
    # two slots with scores ln 1 and ln 3, values 1 and 5 times their scale
    c = R.make_pool(1, 16, 16, 2, [[1]], [2], torch.float32, 0)
    c.k[:], c.v[:], c.ks[:], c.vs[:], c.mass[:] = 0, 0, math.log(3.0), 0.5, 1.0
    c.k[1, 0, 1, 0], c.v[1, 0, 0, 0], c.v[1, 0, 1, 0] = 0x38, 0x38, 0x4A     # 1; 1; 5
    q = torch.zeros(1, 1, 16)
    q[0, 0, 0] = 1.0
    out, lse, mass, _, _ = R.attend(c, 1, q, [0, 1], scale=1.0, lam=0.5)
    assert abs(float(out[0, 0, 0]) - 2.0) < 1e-6 and abs(float(lse) - math.log(4.0)) < 1e-6 and abs(float(mass[0, 0]) - 1.5) < 1e-6


def test_planning_with_stub_launchers(B):
    """Valid calls through checks, planning and workspace of the host code (sanitizer build only: the launchers are stubs there): the
    workspace query covers every way the tokens may spread."""
    if not hasattr(B._lib, "structkv_stub_last_attend"):
        pytest.skip("needs the stub launchers")
    import random
    rng = random.Random(5)
    last = (ctypes.c_int64 * 6)()
    for trial in range(400):
        batch = rng.choice((1, 1, 2, 8, 9, 64))
        fresh = [rng.choice((0, 1, 1, rng.randrange(65), rng.randrange(4097))) for _ in range(batch)]
        single = rng.random() < 0.4
        if single:
            fresh = [min(f, 1) for f in fresh]
        G, gs, d, ps = rng.choice((1, 2, 8, 32)), rng.choice((1, 3, 4, 8, 20)), rng.choice((16, 64, 80, 128, 256)), rng.choice((16, 32, 64, 128, 256))
        most = rng.choice((0, 1, 5, rng.randrange(100), rng.randrange(1 << 22)))
        new = [0]
        for f in fresh:
            new.append(new[-1] + f)
        new = i64(*new)
        c = cache(B, batch=batch, n_kv_heads=G, head_dim=d, page_size=ps, stride_tok=d, stride_head=ps * d, stride_page=G * ps * d, dtype=rng.choice((0, 1)),
                  max_pages=most, pages_stride=most)
        r = ctypes.byref(c)
        size = B._lib.structkv_paged_workspace_bytes(r, G * gs, new[batch])
        assert size > 0
        assert B._lib.structkv_paged_attend(r, G * gs, 0.0, 0.0, P, G * gs * d, d, new, 0.9 if single else 0.0, P, P, P, size, None) == 0, B.structkv_last_error()
        if new[batch]:
            B._lib.structkv_stub_last_attend(last)
            assert last[4] <= size
        rot = rotary(B, rot_dim=d)
        assert B._lib.structkv_paged_append(r, P, P, d, d, new, ctypes.byref(rot), P, G * gs, P, G * gs * d, d, P, Q, None) == 0, B.structkv_last_error()
        assert B._lib.structkv_rotate(ctypes.byref(rot), P, G * d, d, max(1, new[batch]), G, d, 1, P, 0, Q, G * d, d, None) == 0
