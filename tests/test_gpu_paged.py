"""GPU parity of the operators on a cache held in 8 bits, in pages, with their 64-bit definitions.

Tolerances.  append: codes and scales of values are exact; a rotated key y is off by delta = (|a| + |b|) m 6 2^-24 (test_gpu_rotary.py), so its
code lies between those of y - delta and y + delta, and its scale between those of the largest magnitude less and plus the largest delta.
attend, of codes that are exact in the products: an fp32 dot product of d terms is off by at most d 2^-24 |q| |k|, its scale and cap by a few
roundings of the result, so a score by delta = (d max|q| max|k| scale + 8 max|x|) 2^-24, and a weight by 2 delta of its value, plus the sums'
roundings, (n / 16 + 64) 2^-24.  Weights enter their product in fp16, 2^-11 of each (for fp32 outputs in two parts, 2^-22), or 2^-25 where they are
subnormal, when the largest of a wave is 2^6 at least: 2^-31 of it for each slot.  The result is rounded once, 2^-8 of it in bf16, 2^-24 in fp32."""
import math

import numpy as np
import pytest
import torch

import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_amd import binding
    return binding


EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


class OnGpu:
    """A pool of the tests on the GPU: "heads" [page][G][row][d], "tokens" [page][row][G][d], "apart" (16 bytes between rows)."""

    def __init__(self, B, c, layout="heads", mass=True, missed=True):
        def place(x):
            if layout == "heads":
                return x.cuda()
            if layout == "tokens":
                return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            room = torch.full((*x.shape[:3], x.shape[3] + 16), 127, dtype=torch.uint8, device="cuda")
            room[..., 16:] = x.cuda()
            return room[..., 16:]
        self.c, self.k, self.v, self.ks, self.vs = c, place(c.k), place(c.v), c.ks.cuda(), c.vs.cuda()
        self.pages, self.lens = c.pages.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda")
        self.lens_out = torch.full((len(c.lens),), -9, dtype=torch.int32, device="cuda")
        self.mass = c.mass.cuda() if mass else None
        self.missed = torch.zeros(len(c.lens), dtype=torch.int32, device="cuda") if missed else None
        self.handle = B.make_paged(self.k, self.v, self.ks, self.vs, self.pages, self.lens, c.dtype, self.mass, self.missed)

    def workspace(self, B, H, new):
        n = B.structkv_paged_workspace_bytes(self.handle, H, new)
        assert n > 0
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN, should any of it be taken for a result)


def cut(parts):
    cu = [0]
    for n in parts:
        cu.append(cu[-1] + n)
    return cu


def table(lens, page_size, rng, spare=0, dropped=0.0, fresh=None):
    """Pages of each sequence, scattered over the pool, and the pool's size; those of the fresh tokens are not dropped."""
    need = [-(-max(n, 0) // page_size) + spare for n in lens]
    ids = rng.permutation(sum(need) + 3)
    out, at = [], 0
    for b, n in enumerate(need):
        first = (lens[b] - (fresh[b] if fresh else 0)) // page_size
        out.append([int(p) if j >= first or rng.random() >= dropped else -1 for j, p in enumerate(ids[at:at + n])])
        at += n
    return out, sum(need) + 3


def within(got, ref, tol, what):
    worst = ((got - ref).abs() / tol.clamp(min=1e-30)).max() if got.numel() else 0.0
    assert worst <= 1.0, "%s: %g of the tolerance" % (what, float(worst))     # (NaN is not)


def same(x, y, what):
    differ = ((x != y) & ~(x.isnan() & y.isnan())).nonzero()
    assert len(differ) == 0, "%s: %d values differ, at %s .. %s: %g and %g" % (
        what, len(differ), differ[0].tolist(), differ[-1].tolist(), float(x[tuple(differ[0])]), float(y[tuple(differ[0])]))


def queries(new, H, d, dtype, seed, layout="whole"):
    q = torch.randn(new, H, d, generator=torch.Generator().manual_seed(seed + 77)).to(dtype)
    if layout == "whole":
        return q, q.cuda()
    room = torch.zeros(new, H + 1, d + (16 if layout == "part" else 3), dtype=dtype, device="cuda")
    room[:, 1:, -d:] = q.cuda()
    return q, room[:, 1:, -d:]


def check_attend(B, c, H, fresh, *, softcap=0.0, lam=0.0, scale=0.0, layout="heads", q_layout="whole", seed=0, on=None):
    cu_new = cut(fresh)
    new = cu_new[-1]
    q, q_gpu = queries(new, H, c.d, c.dtype, seed, q_layout)
    on = on or OnGpu(B, c, layout)
    out = torch.full((new, H, c.d), math.nan, dtype=c.dtype, device="cuda")
    lse = torch.full((new, H), math.nan, device="cuda")
    ws = on.workspace(B, H, new)
    before = [x.clone() for x in (on.k, on.v, on.ks, on.vs, on.pages, on.lens)]
    call = lambda: B.structkv_paged_attend(on.handle, H, q_gpu, cu_new, out, lse, ws, scale=scale, softcap=softcap, lam=lam)  # noqa: E731
    call()
    ref, ref_lse, ref_mass, size, top = R.attend(c, H, q, cu_new, scale, softcap, lam)
    got, got_lse = out.cpu().double(), lse.cpu().double()
    finite = ref_lse > -math.inf
    assert torch.equal(finite, got_lse > -math.inf)
    x_max = float(ref_lse[finite].abs().max()) + 16 if finite.any() else 0.0
    longest = max([R.length(c, b) for b in range(len(c.lens))], default=0)
    factor = scale or 1 / math.sqrt(c.d)
    keys = (R.decode(c.k).nan_to_num(0.0) * c.ks[:, :, None, None]).norm(dim=3).max() if c.n_pages else 0.0
    delta = float(c.d * keys * (q.double().norm(dim=2).max() if new else 0.0) * factor + 8 * x_max) * 2.0 ** -24
    a_err = 2 * delta + (longest / 16 + 64) * 2.0 ** -24
    within(got_lse[finite], ref_lse[finite], a_err + 2.0 ** -23 * ref_lse[finite].abs(), "lse")
    p_err = 2.0 ** -11 if c.dtype == torch.bfloat16 else 2.0 ** -22
    within(got, ref, EPS[c.dtype] * ref.abs() + (2 * a_err + p_err) * size + longest * 2.0 ** -31 * top, "out")
    assert torch.all(got[~finite] == 0)
    if on.mass is not None:   # (the norm is rounded to fp32 once more)
        within(on.mass.cpu().double(), ref_mass, (2.0 ** -22 + 2 * a_err + 2.0 ** -22 * x_max) * ref_mass.abs(), "mass")
    for x, y in zip((on.k, on.v, on.ks, on.vs, on.pages, on.lens), before):
        assert torch.equal(x, y)
    # again, with the workspace as the call left it: bit for bit
    first, first_lse = out.clone(), lse.clone()
    out.fill_(math.nan)
    call()
    same(out, first, "out"), same(lse, first_lse, "lse")
    return on


DIMS = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64), (torch.bfloat16, 80), (torch.float32, 16), (torch.bfloat16, 256),
        (torch.float32, 256), (torch.bfloat16, 96)]


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("G,H", [(2, 8), (3, 3), (1, 20)])
@pytest.mark.parametrize("page_size", [16, 64])
def test_attend_single_tokens(B, dtype, d, G, H, page_size):
    lens = [1, 2, 33, 129, 700, 64, 15, 16, 17]
    pages, n = table(lens, page_size, np.random.default_rng(d), spare=1)
    check_attend(B, R.make_pool(G, d, page_size, n, pages, lens, dtype, 1), H, [1] * 9, lam=0.9, seed=1)


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("T,H", [(2, 4), (7, 8), (17, 2), (64, 8)])
def test_attend_chains(B, dtype, d, T, H):
    lens = [T, T + 37, 400]
    pages, n = table(lens, 32, np.random.default_rng(T))
    check_attend(B, R.make_pool(2, d, 32, n, pages, lens, dtype, T), H, [T, T, min(T, 400)], seed=T)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,n", [(200, 200), (130, 500), (300, 301)])
def test_attend_chunks_of_a_prompt(B, dtype, T, n):
    pages, total = table([n, 40], 128, np.random.default_rng(T))
    check_attend(B, R.make_pool(2, 128, 128, total, pages, [n, 40], dtype, T), 8, [T, 3], seed=T)


@pytest.mark.parametrize("page_size", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens", "apart"])
def test_attend_pages_and_layouts(B, page_size, layout):
    lens = [255, 256, 257, 1]
    pages, n = table(lens, page_size, np.random.default_rng(page_size), spare=2)
    c = R.make_pool(2, 64, page_size, n, pages, lens, torch.bfloat16, page_size)
    check_attend(B, c, 8, [3, 1, 2, 1], layout=layout, q_layout="part")
    check_attend(B, c, 8, [1, 1, 1, 1], layout=layout, q_layout="odd", lam=1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("softcap", [5.0, 30.0])
def test_attend_capped(B, dtype, softcap):
    lens = [300, 77]
    pages, n = table(lens, 16, np.random.default_rng(3))
    c = R.make_pool(2, 128, 16, n, pages, lens, dtype, 3)
    check_attend(B, c, 8, [4, 4], softcap=softcap)
    check_attend(B, c, 8, [1, 1], softcap=softcap, lam=0.5, scale=0.3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fresh", [[1, 1, 1], [5, 20, 3]])
def test_attend_dropped_pages(B, dtype, fresh):
    lens = [500, 700, 90]
    pages, n = table(lens, 16, np.random.default_rng(8), dropped=0.5, fresh=fresh)
    pages[0][0], pages[1][1], pages[2][0] = n, 2 ** 31 - 1, -2 ** 31     # (whatever lies outside the pool)
    check_attend(B, R.make_pool(2, 128, 16, n, pages, lens, dtype, 8), 8, fresh, lam=0.9 if max(fresh) == 1 else 0.0)


def test_attend_where_nothing_is_seen(B):
    """All pages dropped; lengths of zero; fewer tokens than fresh ones; lengths out of bounds; a sequence that missed its rows."""
    lens = [100, 0, 2, -5, 10 ** 6, 40]
    pages = [[-1] * 7, [], [7], [8], [1, 2, 3, 4, 5, 6, 9], [10, 11, 12]]
    c = R.make_pool(2, 64, 16, 20, pages, lens, torch.bfloat16, 9, capacity=7)
    c.lens[4] = 112
    on = OnGpu(B, c)
    on.lens[4] = 10 ** 6
    check_attend(B, c, 8, [1, 1, 3, 1, 2, 0], on=on)
    c = R.make_pool(2, 64, 16, 20, pages, lens, torch.bfloat16, 9, capacity=7)
    on = OnGpu(B, c)
    on.missed[5] = 1
    q, q_gpu = queries(6, 8, 64, torch.bfloat16, 1)
    out, lse, ws = torch.full((6, 8, 64), math.nan, dtype=torch.bfloat16, device="cuda"), torch.full((6, 8), math.nan, device="cuda"), on.workspace(B, 8, 6)
    B.structkv_paged_attend(on.handle, 8, q_gpu, [0, 1, 2, 3, 4, 5, 6], out, lse, ws, lam=0.5)
    for row in (0, 1, 3, 5):
        assert bool((out[row] == 0).all()) and bool((lse[row] == -math.inf).all())
    assert bool(out[[2, 4]].isfinite().all())
    mass = c.mass.clone()
    mass[0] *= 0.5                        # its pages gathered nothing, and decayed
    assert torch.equal(on.mass.cpu()[[0, 1, 3, 5]], mass[[0, 1, 3, 5]])


def test_attend_empty_calls(B):
    c = R.make_pool(2, 64, 16, 4, [[1], [2]], [3, 4], torch.bfloat16, 1)
    on = OnGpu(B, c)
    q, out, lse = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, 8, device="cuda")
    B.structkv_paged_attend(on.handle, 8, q, [0, 0, 0], out, lse, on.workspace(B, 8, 0))
    check_attend(B, c, 8, [0, 2])
    none = torch.zeros(0, 2, 16, 64, dtype=torch.uint8, device="cuda")
    empty = B.make_paged(none, none, torch.zeros(0, 2, device="cuda"), torch.zeros(0, 2, device="cuda"), on.pages, on.lens)
    q, out, lse = queries(2, 8, 64, torch.bfloat16, 1)[1], torch.ones(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 8, device="cuda")
    B.structkv_paged_attend(empty, 8, q, [0, 1, 2], out, lse, on.workspace(B, 8, 2))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_values_that_are_not_numbers(B, dtype):
    """NaN in fresh slots that some rows do not see; in keys that they see."""
    T, lens = 6, [70, 300]
    pages, n = table(lens, 16, np.random.default_rng(4))
    for name, at in (("v", 3), ("k", 2), ("v", 0), ("k", 5)):
        c = R.make_pool(2, 128, 16, n, pages, lens, dtype, 4)
        clean = R.make_pool(2, 128, 16, n, pages, lens, dtype, 4)
        s = lens[1] - T + at
        getattr(c, name)[pages[1][s // 16], 1, s % 16, 5:9] = 127
        q, q_gpu = queries(2 * T, 8, 128, dtype, 4)
        res = []
        for pool in (c, clean):
            on = OnGpu(B, pool)
            out, lse = torch.empty(2 * T, 8, 128, dtype=dtype, device="cuda"), torch.empty(2 * T, 8, device="cuda")
            B.structkv_paged_attend(on.handle, 8, q_gpu, [0, T, 2 * T], out, lse, on.workspace(B, 8, 2 * T))
            res.append((out, lse))
        (out, lse), (want, want_lse) = res
        sees = slice(T + at, 2 * T)
        assert torch.equal(out[:T + at], want[:T + at]) and torch.equal(lse[:T + at], want_lse[:T + at])
        assert torch.equal(out[:, :4], want[:, :4])                              # the other KV head's
        hit = out[sees, 4:] if name == "k" or at > 0 else out[sees, 4:, 5:9]
        assert bool(hit.isnan().all())
        if name == "k":
            assert bool(lse[sees, 4:].isnan().all())
        else:
            assert torch.equal(lse, want_lse)


def test_attend_scores_and_scales_far_apart(B):
    """Scores from -2^20 to 2^20, pages whose scales differ by 2^60, and a far larger page at the end."""
    lens = [640, 640]
    pages, n = table(lens, 16, np.random.default_rng(6))
    for kind in ("scores", "values", "tiny", "any"):
        c = R.make_pool(1, 64, 16, n, pages, lens, torch.float32, 6)
        if kind == "scores":
            c.ks[:, 0] = torch.exp2(torch.arange(n) % 20 - 6.0)
        elif kind == "values":
            c.vs[:, 0] = torch.exp2(torch.arange(n) % 3 * 30.0 - 30.0)
        elif kind == "tiny":
            c.vs[:, 0] = 2.0 ** -64
        else:   # (a pool that was filled by somebody else)
            c.ks, c.vs = torch.rand(n, 1) * 0.1 + 0.01, torch.rand(n, 1) * 3 + 0.01
        check_attend(B, c, 4, [1, 3])


def test_attend_long(B):
    """Many chunks, one long sequence among short ones, a page size for each."""
    for page_size, lens in ((16, [9000, 17, 300, 1]), (64, [20000, 64]), (256, [12345])):
        pages, n = table(lens, page_size, np.random.default_rng(page_size), spare=1, dropped=0.1, fresh=[1] * len(lens))
        check_attend(B, R.make_pool(2, 64, page_size, n, pages, lens, torch.bfloat16, 5), 8, [1] * len(lens), lam=0.9, layout="tokens")
        check_attend(B, R.make_pool(1, 128, page_size, n, pages, lens, torch.float32, 5), 1, [1] * len(lens))


def test_attend_many_sequences_and_shared_pages(B):
    lens = [20 + 3 * b for b in range(64)]
    rng = np.random.default_rng(12)
    pages, n = table(lens, 16, rng)
    for t in pages[1:]:
        t[0] = pages[0][0]                  # a common prefix
    check_attend(B, R.make_pool(2, 64, 16, n, pages, lens, torch.bfloat16, 12), 4, [1] * 64, lam=0.9)
    check_attend(B, R.make_pool(2, 64, 16, n, pages, lens, torch.bfloat16, 12), 4, [b % 4 for b in range(64)])


def rotary(B, rot, scaling=("none",), interleaved=False, magnitude=1.0):
    turns, m = B.structkv_rotary_turns(rot, 500000.0, *scaling)
    return B.make_rotary(turns.cuda(), interleaved=interleaved, magnitude=magnitude * m), R.turns_of(turns), magnitude * m


def check_append(B, c, fresh, rot=0, interleaved=False, magnitude=1.0, pos=None, layout="heads", new_layout="heads", H=0, seed=0, new=None, scaling=("none",)):
    """The call against the definition; returns the pool as the call left it, in host memory."""
    cu_new = cut(fresh)
    total = cu_new[-1]
    g = torch.Generator().manual_seed(seed + 5)
    k, v = new if new is not None else [torch.randn(c.G, total, c.d, generator=g).to(c.dtype) for _ in range(2)]
    def place(x):
        if new_layout == "heads":
            return x.cuda()
        room = torch.zeros(total, c.G + 1, c.d + (16 if new_layout == "part" else 1), dtype=x.dtype, device="cuda")
        room[:, 1:, -c.d:] = x.cuda().transpose(0, 1)
        return room[:, 1:, -c.d:].transpose(0, 1)
    plan, turns, m = rotary(B, rot, scaling, interleaved, magnitude) if rot else (None, None, 1.0)
    on = OnGpu(B, c, layout)
    q = torch.randn(total, H, c.d, generator=g).to(c.dtype) if H else None
    q_out = torch.full((total, H, c.d), math.nan, dtype=c.dtype, device="cuda") if H else None
    B.structkv_paged_append(on.handle, place(k), place(v), cu_new, on.lens_out, plan, None if pos is None else torch.tensor(pos, dtype=torch.int32).cuda(),
                            q.cuda() if H else None, q_out)
    parts, lens, missed = R.append(c, k, v, cu_new, pos, turns, interleaved, m)
    assert on.lens_out.tolist() == lens and on.missed.tolist() == missed and on.lens.tolist() == list(c.lens)
    got = dict(k=on.k.cpu().contiguous(), v=on.v.cpu().contiguous(), ks=on.ks.cpu(), vs=on.vs.cpu())
    want = dict(k=c.k.clone(), v=c.v.clone(), ks=c.ks.clone(), vs=c.vs.clone())
    k_delta = float(k.double().nan_to_num(0, 0, 0).abs().max()) * 2 * abs(m) * 6 * 2.0 ** -24 if rot and total else 0.0
    for name, page, head, row, values, top, before in parts:
        delta = k_delta if name == "k" else 0.0
        s = float(got[name + "s"][page, head])
        low, high = R.scale_for(max(0.0, top - delta)), R.scale_for(top + delta)
        if before is not None:
            low, high = max(low, before), max(high, before)
        assert low <= s <= high, (name, page, head, s, low, high)
        want[name + "s"][page, head] = s
        if before is not None:
            earlier = R.decode(c.__dict__[name][page, head, :row]) * (before / s)
            want[name][page, head, :row] = R.encode(earlier)
        rows = slice(row, row + values.shape[0])
        have = got[name][page, head, rows]
        want[name][page, head, rows] = have
        a, b, x = (R.decode(R.encode((y / s).clamp(-448, 448))) for y in (values - delta, values + delta, values))
        here = R.decode(have)
        assert torch.equal(here.isnan(), values.isnan())
        here = torch.where(values.isnan(), 0.0, here)
        assert bool(((here >= a.nan_to_num(0)) & (here <= b.nan_to_num(0))).all()), (name, page, head)
        if not delta:
            assert torch.equal(here, x.nan_to_num(0))
    for name in want:      # ... and nothing else was touched
        assert torch.equal(got[name], want[name]), name
    if H:
        at = [R.length(c, b) + t for b in range(len(fresh)) for t in range(fresh[b])] if pos is None else pos
        ref = R.rotated(q, at, turns, interleaved, m)
        size = float(q.double().abs().max()) * 2 * abs(m) * 6 * 2.0 ** -24 * (1 + EPS[c.dtype])
        within(q_out.cpu().double(), ref, EPS[c.dtype] * ref.abs() + size, "q")
    return on, got


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("rot,interleaved", [(0, False), (1.0, False), (1.0, True), (0.5, False), (10, False), (10, True)])
def test_append(B, dtype, d, rot, interleaved):
    rot = int(rot * d) if isinstance(rot, float) else rot
    lens, fresh = [0, 5, 16, 31, 40], [1, 1, 3, 50, 0]
    pages, n = table([a + b for a, b in zip(lens, fresh)], 16, np.random.default_rng(d), spare=1)
    c = R.make_pool(2, d, 16, n, pages, lens, dtype, d)
    check_append(B, c, fresh, rot, interleaved, H=4 if rot else 0)


@pytest.mark.parametrize("page_size", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["heads", "tokens", "apart"])
@pytest.mark.parametrize("new_layout", ["heads", "part", "odd"])
def test_append_pages_and_layouts(B, page_size, layout, new_layout):
    lens, fresh = [0, 100, 255], [300, 1, 2]
    pages, n = table([a + b for a, b in zip(lens, fresh)], page_size, np.random.default_rng(page_size))
    c = R.make_pool(3, 64, page_size, n, pages, lens, torch.bfloat16, page_size)
    check_append(B, c, fresh, 64, layout=layout, new_layout=new_layout, H=3, scaling=("yarn", 4.0, 8192.0, 32.0, 1.0))


def test_append_positions_that_are_given(B):
    lens, fresh = [4, 0], [5, 7]
    pages, n = table([9, 7], 16, np.random.default_rng(2))
    c = R.make_pool(2, 128, 16, n, pages, lens, torch.float32, 2)
    check_append(B, c, fresh, 128, pos=[100000 + 17 * i for i in range(10)] + [-3, (1 << 31) - 1], H=2, magnitude=1.25)


def test_append_scales_grow(B):
    """Rows a thousand times as large, and as small, as those that are there; zeros; rows that meet the border of a scale exactly."""
    lens = [5, 5, 5, 0, 0, 0]
    pages, n = table([16] * 6, 16, np.random.default_rng(7))
    c = R.make_pool(1, 64, 16, n, pages, lens, torch.float32, 7)
    k = torch.randn(1, 12, 64, generator=torch.Generator().manual_seed(1))
    k[:, 0:2] *= 1000.0
    k[:, 2:4] /= 1000.0
    k[:, 4:8] = 0.0
    k[:, 8] = k[:, 8].clamp(-1, 1) * 7.0
    k[0, 8, 3] = 7.0             # 448 2^-6
    k[:, 10] = 0.5
    k[0, 10, 0] = float(np.nextafter(np.float32(7.0), np.float32(8.0)))
    check_append(B, c, [2] * 6, new=(k, -k))


def test_append_values_that_cannot_be_stored(B):
    lens = [3, 0]
    pages, n = table([16, 16], 16, np.random.default_rng(7))
    for dtype in (torch.float32, torch.bfloat16):
        c = R.make_pool(2, 64, 16, n, pages, lens, dtype, 7)
        k = torch.randn(2, 8, 64, generator=torch.Generator().manual_seed(3)).to(dtype)
        k[0, 1, 5], k[1, 6, 0], k[0, 6, 9], k[0, 7, 1], k[1, 2, 2] = math.nan, math.inf, -math.inf, 3e38, 2.0 ** -120
        k[:, 3] = math.nan
        k[1, 4] = 448.0 * 2.0 ** 64
        check_append(B, c, [4, 4], new=(k, k.flip(1)))


def test_append_without_room(B):
    """Beyond the capacity, or into a page that was dropped: the sequence stays as it was, the others go on."""
    lens, fresh = [30, 14, 16, 3, 31], [3, 4, 1, 2, 1]
    c = R.make_pool(2, 64, 16, 12, [[1, 2], [3, -1], [4, 12], [5, -1], [6, 7]], lens, torch.bfloat16, 1)
    check_append(B, c, fresh, 64, H=2)
    c.lens[0], c.lens[1] = 99, -4
    check_append(B, c, [1, 0, 0, 0, 1])


def test_append_one_by_one_and_at_once(B):
    """A prompt stored at once, and token by token in steps: the same scales, and codes but for those that were rounded as subnormal before."""
    pages, n = table([100], 32, np.random.default_rng(3))
    k, v = (torch.randn(2, 100, 128, generator=torch.Generator().manual_seed(s)).cuda() for s in (1, 2))
    pools = []
    for step in (100, 1):
        c = R.make_pool(2, 128, 32, n, pages, [0], torch.float32, 3)
        on = OnGpu(B, c)
        lens = [on.lens, on.lens_out]
        plan = rotary(B, 128)[0]
        for i in range(0, 100, step):
            handle = B.make_paged(on.k, on.v, on.ks, on.vs, on.pages, lens[0], torch.float32)
            B.structkv_paged_append(handle, k[:, i:i + step], v[:, i:i + step], [0, step], lens[1], plan)
            lens.reverse()
        assert lens[0].tolist() == [100]
        used = torch.tensor(pages[0])
        pools.append([x[used].cpu() for x in (on.k, on.v, on.ks, on.vs)])
    (k1, v1, ks1, vs1), (k2, v2, ks2, vs2) = pools
    assert torch.equal(ks1, ks2) and torch.equal(vs1, vs2)
    for a, b in ((k1, k2), (v1, v2)):
        a, b = R.decode(a[:3]), R.decode(b[:3])
        near = a.abs() < 2.0 ** -6
        assert torch.equal(a[~near], b[~near]) and bool(((a - b).abs()[near] <= 2.0 ** -9).all())


def test_run_together(B):
    """A prompt goes in, a chunk of it attends, tokens follow one by one with their weights gathered, pages of least mass are dropped and
    generation goes on: each step against the definitions on the pool as it is."""
    G, H, d, ps, dtype = 2, 8, 64, 16, torch.bfloat16
    pages, n = table([150, 90], ps, np.random.default_rng(21), spare=2)
    c = R.make_pool(G, d, ps, n, pages, [0, 0], dtype, 21)
    plan, turns, _ = rotary(B, d)
    g = torch.Generator().manual_seed(4)
    on = OnGpu(B, c)
    lens = [on.lens, on.lens_out]
    handles = [B.make_paged(on.k, on.v, on.ks, on.vs, on.pages, x, dtype, on.mass, on.missed) for x in lens]
    on.mass.zero_()
    for step, fresh in enumerate(([140, 80], [1, 1], [1, 1], [1, 0], [3, 2], [1, 1])):
        cu = cut(fresh)
        q, (k, v) = torch.randn(cu[-1], H, d, generator=g).to(dtype).cuda(), torch.randn(2, G, cu[-1], d, generator=g).to(dtype).cuda()
        turned = torch.empty_like(q)
        B.structkv_paged_append(handles[0], k, v, cu, lens[1], plan, q=q, q_out=turned)
        lens.reverse(), handles.reverse()
        c.k, c.v, c.ks, c.vs, c.mass, c.pages, c.lens = on.k.cpu(), on.v.cpu(), on.ks.cpu(), on.vs.cpu(), on.mass.cpu(), on.pages.cpu(), lens[0].tolist()
        out, lse = torch.empty_like(q), torch.empty(cu[-1], H, device="cuda")
        lam = 0.9 if max(fresh) == 1 else 0.0
        ws = torch.empty(B.structkv_paged_workspace_bytes(handles[0], H, cu[-1]), dtype=torch.uint8, device="cuda")
        B.structkv_paged_attend(handles[0], H, turned, cu, out, lse, ws, lam=lam)
        ref, ref_lse, ref_mass, size, top = R.attend(c, H, turned.cpu(), cu, lam=lam)
        within(lse.cpu().double(), ref_lse, 1e-4 + 0 * ref_lse, "lse")
        within(out.cpu().double(), ref, 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 4e-4) * size, "out")
        within(on.mass.cpu().double(), ref_mass, 4e-4 * ref_mass + 1e-12, "mass")
        if step == 2:      # the three of least mass go, none of the last two pages
            for b in range(2):
                used = -(-c.lens[b] // ps)
                on.pages[b, on.mass[b, :used - 2].argsort()[:3]] = -1
    assert on.missed.tolist() == [0, 0] and lens[0].tolist() == [147, 85]


def test_captured_step(B):
    """A step (rows stored, attention, lengths taken over) in a graph, replayed while lengths grow past pages and a page is dropped."""
    G, H, d, ps, dtype = 2, 8, 128, 16, torch.bfloat16
    lens0 = [14, 100, 31]
    pages, n = table([v + 8 for v in lens0], ps, np.random.default_rng(31))
    make = lambda: OnGpu(B, R.make_pool(G, d, ps, n, pages, lens0, dtype, 31))  # noqa: E731
    plan = rotary(B, d)[0]
    a, b = make(), make()
    q, (k, v) = torch.randn(3, H, d, device="cuda").to(dtype), torch.randn(2, G, 3, d, device="cuda").to(dtype)
    res = []
    for on in (a, b):
        after = B.make_paged(on.k, on.v, on.ks, on.vs, on.pages, on.lens_out, dtype, on.mass, on.missed)
        turned, out, lse, ws = torch.empty_like(q), torch.empty_like(q), torch.empty(3, H, device="cuda"), on.workspace(B, H, 3)

        def step(on=on, after=after, turned=turned, out=out, lse=lse, ws=ws):
            B.structkv_paged_append(on.handle, k, v, [0, 1, 2, 3], on.lens_out, plan, q=q, q_out=turned)
            B.structkv_paged_attend(after, H, turned, [0, 1, 2, 3], out, lse, ws, lam=0.9)
            on.lens.copy_(on.lens_out)
        res.append((step, out, lse))
    (eager, out_a, lse_a), (step, out_b, lse_b) = res
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        q.normal_(), k.normal_(), v.normal_()
        if i == 3:
            a.pages[1, 2] = b.pages[1, 2] = -1
        graph.replay()
        eager()
        torch.cuda.synchronize()
        assert torch.equal(out_a, out_b) and torch.equal(lse_a, lse_b) and torch.equal(a.mass, b.mass) and torch.equal(a.lens, b.lens)
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.ks, b.ks)
    assert a.lens.tolist() == [x + 6 for x in lens0]


def test_other_streams(B):
    lens = [90, 33]
    pages, n = table(lens, 16, np.random.default_rng(2))
    c = R.make_pool(2, 64, 16, n, pages, lens, torch.bfloat16, 2)
    on = OnGpu(B, c)
    q, q_gpu = queries(2, 8, 64, torch.bfloat16, 2)
    res = []
    for stream in (None, torch.cuda.Stream()):
        out, lse, ws = torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, device="cuda"), on.workspace(B, 8, 2)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        B.structkv_paged_attend(on.handle, 8, q_gpu, [0, 1, 2], out, lse, ws, stream=stream)
        torch.cuda.synchronize()
        res.append((out, lse))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_pool_beyond_2_31(B):
    """Pages whose bytes lie beyond 2^31 and 2^32 from the pool's first."""
    G, d, ps = 8, 128, 64
    n = (5 << 30) // (G * d * ps)
    k, v = (torch.zeros(n, G, ps, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = torch.ones(n, G, device="cuda"), torch.ones(n, G, device="cuda")
    far = [n - 1, n // 2 + 1, 3, n - 7]
    lens = [200]
    c = R.make_pool(G, d, ps, 4, [[0, 1, 2, 3]], lens, torch.bfloat16, 5)
    k[far], v[far], ks[far], vs[far] = c.k.cuda(), c.v.cuda(), c.ks.cuda(), c.vs.cuda()
    pages, lens_gpu, lens_out = torch.tensor([far], dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    handle = B.make_paged(k, v, ks, vs, pages, lens_gpu)
    q, q_gpu = queries(1, 32, d, torch.bfloat16, 3)
    out, lse = torch.empty(1, 32, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 32, device="cuda")
    ws = torch.empty(B.structkv_paged_workspace_bytes(handle, 32, 1), dtype=torch.uint8, device="cuda")
    B.structkv_paged_attend(handle, 32, q_gpu, [0, 1], out, lse, ws)
    ref, ref_lse, _, size, _ = R.attend(c, 32, q, [0, 1])
    within(out.cpu().double(), ref, 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 4e-4) * size, "out")
    new = torch.randn(G, 2, d, generator=torch.Generator().manual_seed(1)).bfloat16()
    B.structkv_paged_append(handle, new.cuda(), new.cuda(), [0, 2], lens_out)
    s = ks[far[3]].cpu().double()
    assert torch.equal(R.decode(k[far[3], :, 8:10].cpu()), R.decode(R.encode(new.double() / s[:, None, None])))


@pytest.mark.parametrize("page_size,d,G,tokens,interleaved", [(64, 128, 8, 4200, False), (16, 64, 6, 1100, True), (256, 256, 2, 700, False), (128, 80, 3, 500, False)])
def test_append_large_batches_like_single_sequences(B, page_size, d, G, tokens, interleaved):
    """Calls that fill the chip, whose workgroups take several heads' keys, against one for each sequence, bit for bit: pages begun and
    ended anywhere, scales that grow, rows that cannot be stored, queries of large calls."""
    batch, H = 8, 2 * G
    lens = [0, 5, 63, 64, 130, 1, 200, 17]
    per = -(-(tokens + 200) // page_size)
    g = torch.Generator(device="cuda").manual_seed(d)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    total = batch * tokens
    k, v, q = normal(total, G, d).transpose(0, 1), normal(total, G, d).transpose(0, 1), normal(total, H, d)
    k[:, ::37] *= 300
    v[:, ::41] /= 1000
    k[1, 100, 3], k[0, tokens + 7, 0], v[1, 50, 9], v[0, 3 * tokens, 1] = math.nan, math.inf, 3e38, -math.inf
    n = batch * per
    codes = torch.randint(0, 126, (n, G, page_size, d), generator=g, device="cuda").to(torch.uint8)
    pages = torch.randperm(n, generator=g, device="cuda").int().view(batch, per)
    plan = rotary(B, d, ("bands", 8.0, 8192.0, 1.0, 4.0), interleaved)[0]
    res = []
    for single in (False, True):
        kc, vc, ks, vs = codes.clone(), codes.clone(), torch.full((n, G), 2.0 ** -7, device="cuda"), torch.full((n, G), 2.0 ** -9, device="cuda")
        lens_gpu, lens_out, missed = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, [-1] * batch, [0] * batch))
        q_out = torch.empty_like(q)
        if single:
            for b in range(batch):
                s = slice(b * tokens, (b + 1) * tokens)
                one = B.make_paged(kc, vc, ks, vs, pages[b:b + 1], lens_gpu[b:b + 1], missed=missed[b:b + 1])
                B.structkv_paged_append(one, k[:, s], v[:, s], [0, tokens], lens_out[b:b + 1], plan, q=q[s], q_out=q_out[s])
        else:
            every = B.make_paged(kc, vc, ks, vs, pages, lens_gpu, missed=missed)
            B.structkv_paged_append(every, k, v, cut([tokens] * batch), lens_out, plan, q=q, q_out=q_out)
        res.append((kc, vc, ks, vs, q_out, lens_out, missed))
    assert res[0][5].tolist() == [x + tokens for x in lens] and res[0][6].tolist() == [0] * batch
    for x, y in zip(*res):
        assert torch.equal(x.view(torch.int16) if x.dtype == torch.bfloat16 else x, y.view(torch.int16) if y.dtype == torch.bfloat16 else y)


def test_attend_mass_of_rows_that_are_not_numbers(B):
    """A key that is NaN: the mass of the pages that the sequence's token sees becomes NaN; other sequences, dropped pages and entries behind
    the last one keep theirs."""
    lens = [50, 50]
    c = R.make_pool(2, 64, 16, 12, [[1, 2, 3, 4], [5, -1, 6, 7]], lens, torch.bfloat16, 3, capacity=6)
    c.k[6, 1, 3, 7] = 127
    on = OnGpu(B, c)
    q, q_gpu = queries(2, 8, 64, torch.bfloat16, 1)
    out, lse = torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 8, device="cuda")
    B.structkv_paged_attend(on.handle, 8, q_gpu, [0, 1, 2], out, lse, on.workspace(B, 8, 2), lam=0.5)
    assert bool(out[1, 4:].isnan().all()) and bool(out[1, :4].isfinite().all()) and bool(out[0].isfinite().all())
    mass = on.mass.cpu()
    assert mass[1, [0, 2, 3]].isnan().all() and bool(mass[0].isfinite().all())
    assert float(mass[1, 1]) == float(c.mass[1, 1]) * 0.5 and torch.equal(mass[:, 4:], c.mass[:, 4:])


def test_attend_workspace_is_as_large_as_it_says(B):
    """Nothing behind the bytes that a call of so many tokens needs is written, nor behind out and lse."""
    for lens, fresh, H, d, dtype, lam in (([3000, 60], [1, 1], 8, 128, torch.bfloat16, 0.9), ([700, 300], [40, 9], 8, 64, torch.float32, 0.0),
                                          ([9000], [1], 32, 64, torch.bfloat16, 0.0)):
        pages, n = table(lens, 16, np.random.default_rng(1), spare=1)
        c = R.make_pool(2, d, 16, n, pages, lens, dtype, 1)
        on, new = OnGpu(B, c), sum(fresh)
        size = B.structkv_paged_workspace_bytes(on.handle, H, new)
        ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        room = torch.full((new * H * d + 512,), 7.0, dtype=dtype, device="cuda")
        norms = torch.full((new * H + 64,), 7.0, device="cuda")
        q, q_gpu = queries(new, H, d, dtype, 1)
        B.structkv_paged_attend(on.handle, H, q_gpu, cut(fresh), room[:new * H * d], norms[:new * H], ws[:size], lam=lam)
        assert bool((ws[size:] == 0xA5).all()) and bool((room[new * H * d:] == 7).all()) and bool((norms[new * H:] == 7).all())
        assert bool(room[:new * H * d].isfinite().all())


@pytest.mark.parametrize("G,H,n", [(128, 128, 70000), (64, 512, 36000)])
def test_attend_weights_of_long_shares(B, G, H, n):
    """Waves that see more blocks than have room for their weights at once."""
    pages, total = table([n], 64, np.random.default_rng(3), dropped=0.2, fresh=[1])
    check_attend(B, R.make_pool(G, 16, 64, total, pages, [n], torch.bfloat16, 3, capacity=len(pages[0])), H, [1], lam=0.9)
