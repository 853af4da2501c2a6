"""GPU parity of the operators on a cache in use (append, attend, accept, evict) with their 64-bit definitions.

Tolerances.  Scores: an fp32 dot product of d terms is off by at most d 2^-24 |q| |k|, its scale, cap and bias by a few roundings of the
result, so a score by delta = (d max|q| max|k| scale + 8 max|x|) 2^-24, and a weight by 2 delta of its value, plus the sums' roundings, (n / 16
+ 64) 2^-24 (a lane adds up a sixteenth of the terms at most one by one, then lanes, waves and chunks).  Values: bf16 kernels multiply
weights of 16 bits or more by exact values; the result is rounded once, 2^-8 of it in bf16 and 2^-24 in fp32."""
import math

import numpy as np
import pytest
import torch

import cache_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_amd import binding
    return binding


EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


class OnGpu:
    """A cache of the tests on the GPU: layout "heads" [G][slots][d], "slots" [slots][G][d], or "odd" (rows one element apart)."""

    def __init__(self, B, c, layout="heads", mass=True, pos=True):
        G, slots, d = c.k.shape
        self.c, self.mass, self.pos = c, c.mass.cuda() if mass else None, c.pos.cuda() if pos else None

        def place(x):
            if layout == "heads":
                return x.cuda()
            if layout == "slots":
                return x.transpose(0, 1).contiguous().cuda().transpose(0, 1)
            room = torch.full((G, slots, d + 1), math.nan, dtype=x.dtype, device="cuda")
            room[:, :, 1:] = x.cuda()
            return room[:, :, 1:]
        self.k, self.v = place(c.k), place(c.v)
        self.lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
        self.lens_out = torch.full((len(c.lens),), -9, dtype=torch.int32, device="cuda")
        self.handle = B.make_cache(self.k, self.v, c.cu, self.lens, self.mass, self.pos)

    def workspace(self, B, H, new):
        n = B.structkv_cache_workspace_bytes(self.handle, H, new)
        assert n > 0
        return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")   # (NaN, should any of it be taken for a result)

    def same(self, k, v, pos, mass, lens):
        assert self.lens_out.tolist() == lens
        for name, x, y in (("k", self.k, k), ("v", self.v, v)):
            as_int = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(x.cpu().contiguous().view(as_int), y.view(as_int)), name
        if self.pos is not None:
            assert torch.equal(self.pos.cpu(), pos)
        if self.mass is not None and mass is not None:
            assert torch.equal(self.mass.cpu(), mass.float())


def within(got, ref, tol, what):
    worst = ((got - ref).abs() / tol.clamp(min=1e-30)).max() if got.numel() else 0.0
    assert worst <= 1.0, "%s: %g of the tolerance" % (what, float(worst))     # (NaN is not)


def score_error(c, q, scale, x_max):
    longest = c.k.float().nan_to_num(0.0, 0.0, 0.0).norm(dim=2).max() * q.float().norm(dim=2).max() if q.numel() and c.k.numel() else 0.0
    return float(c.d * longest * scale + 8 * x_max) * 2.0 ** -24


def queries(new, H, d, dtype, seed, strided=False):
    g = torch.Generator().manual_seed(seed + 77)
    q = torch.randn(new, H, d, generator=g).to(dtype)
    if not strided:
        return q, q.cuda()
    room = torch.zeros(new, H + 1, d + 8, dtype=dtype, device="cuda")   # rows of 16-byte pieces still
    room[:, 1:, 8:] = q.cuda()
    return q, room[:, 1:, 8:]


def check_attend(B, c, H, fresh, *, tree=False, softcap=0.0, slopes=False, lam=0.0, scale=0.0, layout="heads", strided=False, seed=0,
                 masks=None):
    cu_new = R.cut(fresh)
    new = cu_new[-1]
    rng = np.random.default_rng(seed)
    if tree and masks is None:
        masks = [m for T in fresh for m in R.random_tree(T, rng)]
    slope = torch.exp2(-torch.arange(H) / max(H, 1) * 8.0) / 16 if slopes else None
    q, q_gpu = queries(new, H, c.d, c.dtype, seed, strided)
    on = OnGpu(B, c, layout)
    out = torch.full((new, H, c.d), math.nan, dtype=c.dtype, device="cuda")
    lse = torch.full((new, H), math.nan, device="cuda")
    ws = on.workspace(B, H, new)
    call = lambda: B.structkv_cache_attend(on.handle, H, q_gpu, cu_new, out, lse, ws, scale=scale, softcap=softcap, lam=lam,  # noqa: E731
                                           tree_mask=R.as_int64(masks).cuda() if masks is not None else None,
                                           slopes=slope.cuda() if slopes else None)
    call()
    ref, ref_lse, ref_mass, size = R.attend(c, H, q, cu_new, masks, scale, softcap, slope, lam)
    got, got_lse = out.cpu().double(), lse.cpu().double()
    finite = ref_lse > -math.inf
    assert torch.equal(finite, got_lse > -math.inf)
    x_max = float(ref_lse[finite].abs().max()) + 16 if finite.any() else 0.0
    longest = max(c.lens, default=0)
    sums = (longest / 16 + 64) * 2.0 ** -24
    a_err = 2 * score_error(c, q, scale or 1 / math.sqrt(c.d), x_max) + sums
    within(got_lse[finite], ref_lse[finite], a_err + 2.0 ** -23 * ref_lse[finite].abs(), "lse")
    p_err = 2.0 ** -16 if c.dtype == torch.bfloat16 else 0.0   # weights in two bf16 parts
    within(got, ref, EPS[c.dtype] * ref.abs() + (2 * a_err + p_err) * size, "out")
    assert torch.all(got[~finite] == 0)
    k, v, pos = c.k, c.v, c.pos
    on.lens_out.copy_(on.lens)
    on.same(k, v, pos, None, list(c.lens))
    within(on.mass.cpu().double(), ref_mass, (2.0 ** -23 + 2 * a_err) * ref_mass.abs(), "mass")
    # again, with the workspace as the call left it: bit for bit
    first, first_lse = out.clone(), lse.clone()
    out.fill_(math.nan)
    call()
    assert torch.equal(first, out) and torch.equal(first_lse, lse)
    return on


DIMS = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 80), (torch.float32, 33),
        (torch.float32, 256), (torch.bfloat16, 1)]


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("G,H", [(2, 8), (3, 3), (1, 20)])
def test_attend_single_tokens(B, dtype, d, G, H):
    lens = [1, 2, 33, 129, 700, 64]
    check_attend(B, R.make_cache(G, d, 1, [5, 2, 64, 129, 801, 64], lens, dtype, 1), H, [1] * 6, lam=0.9, seed=1)


@pytest.mark.parametrize("dtype,d", DIMS[:5])
@pytest.mark.parametrize("T,H", [(2, 4), (7, 8), (17, 2), (64, 8)])
def test_attend_trees(B, dtype, d, T, H):
    c = R.make_cache(2, d, 2, [T, T + 40, 500], [T, T + 37, 400], dtype, T)
    check_attend(B, c, H, [T, T, T], tree=True, seed=T)


@pytest.mark.parametrize("dtype,d", DIMS[:4])
@pytest.mark.parametrize("planes", [1, 2])
def test_attend_capped_and_biased(B, dtype, d, planes):
    c = R.make_cache(2, d, planes, [300, 90], [280, 90], dtype, 5)
    check_attend(B, c, 6, [5, 9], tree=True, softcap=20.0, slopes=True, seed=5)
    check_attend(B, c, 6, [1, 1], softcap=3.0, slopes=False, lam=1.0, scale=0.3, seed=6)
    check_attend(B, c, 6, [1, 1], slopes=True, lam=0.5, seed=7)


@pytest.mark.parametrize("dtype,d", DIMS[:4])
@pytest.mark.parametrize("layout", ["slots", "odd"])
def test_attend_layouts(B, dtype, d, layout):
    c = R.make_cache(2, d, 1, [77, 300], [70, 300], dtype, 8)
    check_attend(B, c, 4, [1, 1], layout=layout, strided=True, lam=0.9, seed=8)
    check_attend(B, c, 4, [13, 3], tree=True, layout=layout, strided=True, seed=9)


@pytest.mark.parametrize("dtype,d", DIMS[:3])
def test_attend_uneven_and_empty(B, dtype, d):
    """No fresh tokens, no slots, fewer slots than fresh tokens, lengths out of bounds, chains without a mask."""
    c = R.make_cache(2, d, 1, [40, 0, 9, 200, 30, 50], [40, 0, 3, 150, -4, 90], dtype, 3)
    check_attend(B, c, 4, [3, 0, 5, 0, 1, 50], seed=3)
    c = R.make_cache(2, d, 1, [40, 0, 9, 200, 30, 50], [40, 0, 3, 150, 0, 50], dtype, 4)
    check_attend(B, c, 4, [1, 0, 1, 0, 1, 1], lam=0.9, seed=4)


@pytest.mark.parametrize("dtype,d", DIMS[:3])
def test_attend_rows_that_see_nothing(B, dtype, d):
    """Masks without a bit over an empty cache, bits beyond the fresh tokens, and drafts that nobody sees and that are not numbers."""
    c = R.make_cache(2, d, 1, [8, 70, 40], [4, 68, 33], dtype, 11)
    c.k[:, c.cu[1] + 66], c.v[:, c.cu[1] + 66] = math.nan, math.inf     # the third draft of the second sequence
    c.k[:, c.cu[2] + 32], c.v[:, c.cu[2] + 32] = math.inf, math.nan     # the only one of the third
    masks = [0, 0b10, 0, 0b1111 << 4] + [0b1, 0b11, 0, 0b1011 | 1 << 63 | 1 << 40] + [0]
    check_attend(B, c, 4, [4, 4, 1], masks=masks, seed=11)


@pytest.mark.parametrize("dtype,d,G,H,T", [(torch.bfloat16, 128, 2, 4, 5), (torch.bfloat16, 64, 2, 10, 5), (torch.float32, 64, 2, 4, 5),
                                           (torch.bfloat16, 80, 2, 4, 5), (torch.bfloat16, 128, 32, 128, 20), (torch.bfloat16, 64, 2, 4, 1)])
def test_attend_values_that_are_not_numbers(B, dtype, d, G, H, T):
    """Rows that see them are not numbers either, the others are what they would be: a fresh value, a fresh key, a key among the old ones."""
    bad = min(3, T - 1)
    for caps, lens in (([3000, 40, 70], [2900, 40, 60]), ([3008, 32, 64], [3008, 32, 64])):
        c = R.make_cache(G, d, 1, caps, lens, dtype, 51)
        cu_new = R.cut([T] * 3)
        q, q_gpu = queries(3 * T, H, d, dtype, 51)
        ref, ref_lse, _, size = R.attend(c, H, q, cu_new, None, 0.0, 0.0, None, 0.0)
        c.v[:, lens[0] - T + bad, 1] = math.inf
        c.k[:, c.cu[1] + lens[1] - T + bad] = math.nan
        c.k[:, c.cu[2] + 7, 0] = math.nan
        on = OnGpu(B, c)
        out, lse = torch.empty(3 * T, H, d, dtype=dtype, device="cuda"), torch.empty(3 * T, H, device="cuda")
        B.structkv_cache_attend(on.handle, H, q_gpu, cu_new, out, lse, on.workspace(B, H, 3 * T), lam=0.9 if T == 1 else 0.0)
        got, got_lse = out.cpu().double(), lse.cpu().double()
        assert torch.isnan(got[bad:T]).all() and torch.isnan(got[T + bad:]).all()
        assert torch.isnan(got_lse[T + bad:]).all()
        a_err = 2 * score_error(c, q, 1 / math.sqrt(d), float(ref_lse.abs().max()) + 16) + (3008 / 16 + 64) * 2.0 ** -24
        fine = [r for r in range(2 * T) if r % T < bad]
        within(got_lse[fine + list(range(bad, T))], ref_lse[fine + list(range(bad, T))], a_err + 2.0 ** -22 * ref_lse[fine + list(range(bad, T))].abs(), "lse")
        within(got[fine], ref[fine], EPS[dtype] * ref[fine].abs() + (2 * a_err + 2.0 ** -16) * size[fine], "out")


def test_attend_large_scores(B):
    """Scores that grow along the cache by far more than 2^8 at a time, and ones of hundreds."""
    for dtype in (torch.bfloat16, torch.float32):
        c = R.make_cache(1, 64, 1, [900], [900], dtype, 12, hitters=False)
        c.k[0] = (c.k[0].float() * torch.linspace(0.1, 40.0, 900)[:, None]).to(dtype)
        check_attend(B, c, 4, [1], lam=0.9, seed=12)
        check_attend(B, c, 4, [9], tree=True, seed=13)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_attend_many_sequences(B, dtype, d):
    rng = np.random.default_rng(2)
    caps = [int(x) for x in rng.integers(1, 150, 64)]
    lens = [int(rng.integers(1, n + 1)) for n in caps]
    check_attend(B, R.make_cache(2, d, 2, caps, lens, dtype, 2), 4, [1] * 64, lam=0.9, seed=2)
    check_attend(B, R.make_cache(2, d, 2, caps, lens, dtype, 2), 4, [min(n, 3) for n in lens], tree=True, seed=2)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
def test_attend_long(B, dtype, d):
    c = R.make_cache(2, d, 2, [20000], [19999], dtype, 21)
    check_attend(B, c, 8, [1], lam=0.9, seed=21)
    check_attend(B, c, 8, [20], tree=True, softcap=30.0, seed=22)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("form", [dict(tree=True), dict(), dict(tree=True, softcap=30.0), dict(tree=True, slopes=True, softcap=5.0, scale=0.2)])
def test_attend_trees_of_many_rows(B, d, form):
    """More than two blocks of 32 rows and chunks enough: tiles shared by four waves, some without rows; fewer slots than drafts."""
    c = R.make_cache(16, d, 16, [1400, 70, 901, 2100, 40], [1391, 70, 17, 2099, 33], torch.bfloat16, 41)
    check_attend(B, c, 48, [64, 0, 20, 33, 33], layout="slots" if "softcap" in form else "heads", strided=True, seed=41, **form)
    c = R.make_cache(64, d, 1, [100] * 9, [100, 99, 50, 41, 40, 39, 0, 65, 97], torch.bfloat16, 42)    # a chunk each: written at once
    check_attend(B, c, 128, [34, 3, 35, 1, 33, 36, 2, 0, 1], seed=42, **form)


@pytest.mark.parametrize("d", [128, 64])
def test_attend_many_rows_that_see_nothing(B, d):
    c = R.make_cache(32, d, 1, [1300, 900], [64, 800], torch.bfloat16, 43)
    c.k[:, 20], c.v[:, 20] = math.nan, math.inf                     # drafts that nobody sees and that are not numbers
    c.k[:, c.cu[1] + 799], c.v[:, c.cu[1] + 799] = math.inf, math.nan
    masks = [0 if t % 3 else ((2 << t) - 1) & ~(1 << 20) for t in range(64)] + [(2 << t) - 1 for t in range(39)] + [0b1011 | 1 << 50]
    check_attend(B, c, 128, [64, 40], masks=masks, seed=43)


@pytest.mark.parametrize("dtype,d", DIMS[:3])
def test_attend_lengths_far_apart(B, dtype, d):
    """One long sequence among short and empty ones of the same capacity: it takes their share of the workgroups."""
    lens = [1, 2000, 2, 33, 0, 5, 64, 1, 3, 1, 130, 1]
    c = R.make_cache(8, d, 1, [2000] * 12, lens, dtype, 44)
    check_attend(B, c, 8, [1] * 12, lam=0.9, seed=44)
    check_attend(B, c, 8, [1] * 12, seed=45)
    check_attend(B, c, 16, [1, 7, 2, 7, 3, 0, 7, 1, 3, 1, 7, 0], tree=True, seed=46)
    c = R.make_cache(16, d, 1, [1100] * 40, [3] * 20 + [1100] + [0, 40] * 9 + [700], dtype, 49)    # more blocks of rows than half the workgroups
    check_attend(B, c, 16, [1] * 40, lam=0.9, seed=49)
    c = R.make_cache(2, d, 2, [9000, 400], [300, 400], dtype, 47)
    check_attend(B, c, 8, [1, 1], lam=0.5, seed=47)
    check_attend(B, c, 8, [64, 3], tree=True, seed=48)


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("planes", [1, 3])
def test_append(B, dtype, d, planes):
    fresh, lens = [1, 0, 700, 5, 4, 2], [3, 7, 11, 5, 8, -3]
    c = R.make_cache(3, d, planes, [4, 7, 711, 9, 9, 3], lens, dtype, 31)     # the fourth and fifth do not fit
    cu_new, g = R.cut(fresh), torch.Generator().manual_seed(9)
    new = cu_new[-1]
    k_new, v_new = (torch.randn(3, new, d, generator=g).to(dtype) for _ in range(2))
    pos_new, mass_new = torch.randint(0, 99, (planes, new), generator=g).int(), torch.rand(planes, new, generator=g)
    for layout in ("heads", "slots", "odd"):
        on = OnGpu(B, c, layout)
        B.structkv_cache_append(on.handle, k_new.cuda(), v_new.cuda(), cu_new, on.lens_out, pos_new=pos_new.cuda(), mass_new=mass_new.cuda())
        on.same(*R.append(c, k_new, v_new, cu_new, pos_new, mass_new))
        assert on.lens.tolist() == lens
        # shared by the planes, masses from zero, rows in another order
        on = OnGpu(B, c, layout)
        other = lambda x: x.transpose(0, 1).contiguous().cuda().transpose(0, 1)  # noqa: E731
        B.structkv_cache_append(on.handle, other(k_new), other(v_new), cu_new, on.lens_out, pos_new=pos_new[0].cuda())
        on.same(*R.append(c, k_new, v_new, cu_new, pos_new[:1].expand(planes, new)))


def test_append_nothing(B):
    c = R.make_cache(2, 64, 1, [4, 0], [3, 0], torch.bfloat16, 1)
    on = OnGpu(B, c)
    empty = torch.empty(2, 0, 64, dtype=torch.bfloat16, device="cuda")
    B.structkv_cache_append(on.handle, empty, empty, [0, 0, 0], on.lens_out, pos_new=torch.empty(0, dtype=torch.int32, device="cuda"))
    on.same(c.k, c.v, c.pos, c.mass, [3, 0])


def check_accept(B, c, H, fresh, paths, *, tree=True, softcap=0.0, slopes=False, lam=0.0, layout="heads", seed=0, n_accept=None, lse=None):
    cu_new = R.cut(fresh)
    new, rng = cu_new[-1], np.random.default_rng(seed)
    masks = [m for T in fresh for m in R.random_tree(T, rng)] if tree else None
    slope = torch.exp2(-torch.arange(H) / H * 8.0) / 16 if slopes else None
    q, q_gpu = queries(new, H, c.d, c.dtype, seed, strided=layout == "slots")
    if lse is None:
        lse = R.attend(c, H, q, cu_new, masks, 0.0, softcap, slope)[1].float()
    path = None
    if paths is not None:
        path = torch.zeros(new, dtype=torch.int32)
        for b, p in enumerate(paths):
            path[cu_new[b]:cu_new[b] + len(p)] = torch.tensor(p, dtype=torch.int32)
        n_accept = n_accept or [len(p) for p in paths]
    on = OnGpu(B, c, layout)
    cuda = lambda x: None if x is None else x.cuda()  # noqa: E731
    B.structkv_cache_accept(on.handle, H, q_gpu if lam else None, lse.cuda() if lam else None, cu_new, on.lens_out, path=cuda(path),
                            n_accept=torch.tensor(n_accept, dtype=torch.int32).cuda() if n_accept is not None else None,
                            tree_mask=R.as_int64(masks).cuda() if tree else None, softcap=softcap, slopes=cuda(slope), lam=lam)
    k, v, pos, mass, lens = R.accept(c, H, q, lse, cu_new, path, n_accept, masks, 0.0, softcap, slope, lam)
    on.same(k, v, pos, None, lens)
    finite = lse[lse > -math.inf].abs()
    x_max = float(finite.max()) + 16 if finite.numel() else 0.0
    a_err = 2 * score_error(c, q, 1 / math.sqrt(c.d), x_max) + (max(fresh) * H + 64) * 2.0 ** -24 + 4 * x_max * 2.0 ** -24
    within(on.mass.cpu().double(), mass, (2.0 ** -23 + a_err) * mass.abs() * bool(lam), "mass")


@pytest.mark.parametrize("dtype,d", DIMS)
@pytest.mark.parametrize("planes,H", [(1, 8), (2, 4), (2, 40)])
def test_accept(B, dtype, d, planes, H):
    c = R.make_cache(2, d, planes, [300, 26, 9, 140, 3], [280, 26, 4, 131, 2], dtype, 41)
    paths = [[0, 2, 3, 7], list(range(20)), [], [15], [1]]
    check_accept(B, c, H, [26, 26, 4, 64, 2], paths, lam=0.9, seed=41)
    check_accept(B, c, H, [26, 26, 4, 64, 2], paths, lam=0.0, seed=41)


@pytest.mark.parametrize("dtype,d", DIMS[:4])
def test_accept_capped_biased_strided(B, dtype, d):
    c = R.make_cache(2, d, 2, [300, 64], [280, 64], dtype, 43)
    check_accept(B, c, 6, [9, 64], [[0, 3, 8], list(range(1, 64))], softcap=20.0, slopes=True, lam=0.5, layout="slots", seed=43)
    check_accept(B, c, 6, [9, 64], [[0, 3, 8], list(range(1, 64))], slopes=True, lam=1.0, layout="odd", seed=44)


@pytest.mark.parametrize("dtype,d", DIMS[:2] + DIMS[5:6])
def test_accept_without_path(B, dtype, d):
    """All of a chain, or its first tokens; nothing fresh, nothing in use, fewer slots than fresh tokens; counts out of bounds."""
    c = R.make_cache(2, d, 1, [40, 30, 5, 8, 0], [40, 22, 3, 8, 0], dtype, 45)
    check_accept(B, c, 4, [7, 0, 5, 8, 0], None, tree=False, lam=0.9, seed=45)
    check_accept(B, c, 4, [7, 0, 5, 8, 0], None, tree=False, n_accept=[3, 0, 1, -2, 4], lam=0.9, seed=45)
    check_accept(B, c, 4, [7, 0, 5, 8, 0], None, tree=False, n_accept=[3, 0, 1, 99, 4], lam=0.0, seed=45)


def test_accept_any_path(B):
    """Paths out of order, with an entry twice and with entries out of bounds; rows without a norm add nothing."""
    c = R.make_cache(2, 64, 2, [60, 60], [50, 60], torch.bfloat16, 46)
    lse = torch.full((16, 4), 3.0)
    lse[5], lse[9, 2] = -math.inf, -math.inf
    check_accept(B, c, 4, [8, 8], [[7, 5, 3, 3, 1, 0], [1, 0, -5, 70]], lam=0.9, seed=46, lse=lse)


def check_evict(B, c, scores, budget, tail, layout="heads", own_scores=True):
    on = OnGpu(B, c, layout)
    ws = on.workspace(B, c.G, 1)
    B.structkv_cache_evict(on.handle, scores.cuda() if own_scores else None, budget, tail, on.lens_out, ws)
    on.same(*R.evict(c, scores, budget, tail))


@pytest.mark.parametrize("planes", [1, 3])
@pytest.mark.parametrize("tail", [0, 5, 64])
@pytest.mark.parametrize("dtype,d", DIMS[:4] + DIMS[5:6])
def test_evict(B, dtype, d, planes, tail):
    caps = [1, 90, 5000, 64, 2100, 200, 30]
    c = R.make_cache(3, d, planes, caps, [1, 88, 4100, 64, 2081, 200, 0], dtype, 51)
    budget = [0, 60, 1000, 64, 2080, 1, 7]
    check_evict(B, c, c.mass, budget, tail, own_scores=False)
    scores = torch.randn(c.mass.shape, generator=torch.Generator().manual_seed(3))
    check_evict(B, c, scores, budget, tail, layout="odd")
    check_evict(B, c, scores.mul(4).round(), [n // 2 for n in caps], tail, layout="slots")   # ties


@pytest.mark.parametrize("scores", ["equal", "signs", "zeros", "range", "rising", "falling", "infinite"])
def test_evict_scores(B, scores):
    c = R.make_cache(2, 64, 2, [3000], [2900], torch.bfloat16, 52)
    g = torch.Generator().manual_seed(4)
    x = {"equal": torch.ones(2, 3000), "signs": torch.randn(2, 3000, generator=g), "rising": torch.arange(6000.0).view(2, 3000),
         "zeros": torch.randint(0, 2, (2, 3000), generator=g) * -0.0, "falling": -torch.arange(6000.0).view(2, 3000),
         "range": torch.exp(torch.rand(2, 3000, generator=g) * 120 - 60),
         "infinite": torch.where(torch.rand(2, 3000, generator=g) < 0.2, math.inf, torch.randn(2, 3000, generator=g))}[scores]
    for budget in (1, 1000, 2899, 2900):
        check_evict(B, c, x, [budget], 0)
        check_evict(B, c, x, [budget], 40)


@pytest.mark.parametrize("planes", [1, 2])
@pytest.mark.parametrize("n", [8192, 16385, 32768, 32769, 70001])
def test_evict_long(B, planes, n):
    c = R.make_cache(2, 2, planes, [n, 100], [n - 1, 100], torch.bfloat16, 53)
    scores = torch.exp(0.5 * torch.randn(planes, n + 100, generator=torch.Generator().manual_seed(5)))
    for budget in ([n // 2, 50], [n - 2, 100], [33, 99]):
        check_evict(B, c, scores, budget, 64)
    check_evict(B, c, scores.mul(8).round(), [n // 3, 50], 0)


def test_evict_more_recent_than_budget(B):
    """Every slot is within the tail: the lower slots stay."""
    c = R.make_cache(2, 64, 1, [300], [300], torch.bfloat16, 54)
    c.pos[:] = 7
    check_evict(B, c, c.mass, [100], 8)


@pytest.mark.parametrize("dtype,planes", [(torch.bfloat16, 1), (torch.bfloat16, 2), (torch.float32, 1)])
def test_generation_with_a_prefills_cache(B, dtype, planes):
    """As they are used together: a layer's prefill, its compact cache with positions and in-degrees stored, then steps of drafts that
    attend, of which a path is accepted, single tokens, and evictions back to the budget; every step against the definitions."""
    from paper_2604_06746_amd.sweep import LayerSweep
    H, G, d, w, n, keep = 8, 2, 64, 8, 500, 120
    g = torch.Generator().manual_seed(61)
    q_win, k, v = torch.randn(1, H, w, d, generator=g).to(dtype), torch.randn(G, n, d, generator=g).to(dtype), torch.randn(G, n, d, generator=g).to(dtype)
    sw = LayerSweep(H, G, d, w, dtype, [n], [keep])
    sw.layer(q_win.cuda(), k.cuda(), v.cuda())
    rows, cap, budget = keep + w, keep + w + 40, keep + w
    c = R.make_cache(G, d, planes, [cap], [0], dtype, 62)
    on = OnGpu(B, c)
    lens = [on.lens, on.lens_out]
    handles = [on.handle, B.make_cache(on.k, on.v, c.cu, lens[1], on.mass, on.pos)]
    ws = on.workspace(B, H, 16)
    idx = sw.idx_kv[:rows]
    mass = sw.indeg[idx.long()].expand(planes, rows).contiguous()
    B.structkv_cache_append(handles[0], sw.k_cache[0][:, :rows], sw.v_cache[0][:, :rows], [0, rows], lens[1],
                            pos_new=idx.expand(planes, rows).contiguous(), mass_new=mass)
    now, position, rng = 1, n, np.random.default_rng(63)

    def state():
        torch.cuda.synchronize()
        c.k, c.v, c.mass, c.pos, c.lens = on.k.cpu(), on.v.cpu(), on.mass.cpu(), on.pos.cpu(), lens[now].tolist()
        return c
    assert state().lens == [rows] and torch.equal(c.pos[0, :rows], sw.idx_kv[:rows].cpu())
    assert torch.equal(c.k[:, :rows], k[:, c.pos[0, :rows].long()])
    for step in range(6):
        T = (1, 16, 1, 5, 16, 1)[step]
        masks = R.random_tree(T, rng)
        depth = torch.tensor([bin(m).count("1") - 1 for m in masks], dtype=torch.int32)
        q, k_new, v_new = (torch.randn(*s, generator=g).to(dtype) for s in ((T, H, d), (G, T, d), (G, T, d)))
        B.structkv_cache_append(handles[now], k_new.cuda(), v_new.cuda(), [0, T], lens[1 - now], pos_new=(position + depth).cuda())
        now = 1 - now
        before = state()
        out, lse = torch.empty(T, H, d, dtype=dtype, device="cuda"), torch.empty(T, H, device="cuda")
        lam = 0.9 if T == 1 else 0.0
        tree = R.as_int64(masks).cuda()
        B.structkv_cache_attend(handles[now], H, q.cuda(), [0, T], out, lse, ws, tree_mask=tree, lam=lam)
        ref, ref_lse, ref_mass, size = R.attend(before, H, q, [0, T], masks, lam=lam)
        within(out.cpu().double(), ref, EPS[dtype] * ref.abs() + 1e-4 * size, "out")
        assert torch.allclose(lse.cpu().double(), ref_lse, rtol=0, atol=1e-4)
        assert torch.allclose(on.mass.cpu().double(), ref_mass, rtol=1e-4, atol=0)
        if T > 1:
            last = masks[int(rng.integers(0, T))]
            path = [t for t in range(T) if last >> t & 1]
            padded = torch.zeros(T, dtype=torch.int32)
            padded[:len(path)] = torch.tensor(path)
            before = state()
            B.structkv_cache_accept(handles[now], H, q.cuda(), lse, [0, T], lens[1 - now], path=padded.cuda(), tree_mask=tree, lam=0.9,
                                    n_accept=torch.tensor([len(path)], dtype=torch.int32, device="cuda"))
            rk, rv, rpos, rmass, rlens = R.accept(before, H, q, lse.cpu(), [0, T], padded, [len(path)], masks, lam=0.9)
            now = 1 - now
            after = state()
            assert after.lens == rlens and torch.equal(after.pos, rpos)
            assert torch.equal(after.k[:, :rlens[0]], rk[:, :rlens[0]]) and torch.equal(after.v[:, :rlens[0]], rv[:, :rlens[0]])
            assert torch.allclose(after.mass.double(), rmass, rtol=1e-4, atol=0)
        position += 1 + int(depth.max())
        if c.lens[0] > budget + 2:
            before = state()
            B.structkv_cache_evict(handles[now], None, [budget], 4, lens[1 - now], ws)
            rk, rv, rpos, rmass, rlens = R.evict(before, before.mass, [budget], 4)
            now = 1 - now
            after = state()
            assert after.lens == rlens == [budget] and torch.equal(after.pos, rpos) and torch.equal(after.mass, rmass)
            assert torch.equal(after.k[:, :budget], rk[:, :budget]) and torch.equal(after.v[:, :budget], rv[:, :budget])


def test_captured_step(B):
    """A step captured once and replayed while lengths, positions and tokens change, beside eager work: as the eager calls, every time."""
    H, G, d, cap, budget, dtype = 8, 2, 128, 400, 300, torch.bfloat16
    c = R.make_cache(G, d, 2, [cap, cap], [300, 260], dtype, 71)
    g = torch.Generator(device="cuda").manual_seed(72)

    def fresh():
        on = OnGpu(B, c)
        lens = [on.lens, on.lens_out, torch.empty_like(on.lens)]
        handles = [B.make_cache(on.k, on.v, c.cu, x, on.mass, on.pos) for x in lens]
        ws = on.workspace(B, H, 2)
        q, k_new, v_new = (torch.zeros(*s, dtype=dtype, device="cuda") for s in ((2, H, d), (G, 2, d), (G, 2, d)))
        pos, out, lse = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty(2, H, d, dtype=dtype, device="cuda"), torch.empty(2, H, device="cuda")

        def step():
            B.structkv_cache_append(handles[0], k_new, v_new, [0, 1, 2], lens[1], pos_new=pos)
            B.structkv_cache_attend(handles[1], H, q, [0, 1, 2], out, lse, ws, lam=0.9)
            B.structkv_cache_evict(handles[1], None, [budget, budget], 16, lens[0], ws)
        return on, step, (q, k_new, v_new, pos), (out, lse, on.k, on.v, on.mass, on.pos, on.lens)

    eager, replayed = fresh(), fresh()
    start = [x.clone() for x in replayed[3]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        replayed[1]()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed[1]()
    for x, y in zip(replayed[3], start):
        x.copy_(y)
    for i in range(50):
        inputs = [torch.randn(x.shape, generator=g, device="cuda").to(dtype) for x in eager[2][:3]]
        for side_of in (eager, replayed):
            for x, y in zip(side_of[2][:3], inputs):
                x.copy_(y)
            side_of[2][3].fill_(5000 + i)
        eager[1]()
        graph.replay()
        torch.cuda.synchronize()
        for j, (x, y) in enumerate(zip(eager[3], replayed[3])):
            assert torch.equal(x.nan_to_num(), y.nan_to_num()), (i, j)
    assert eager[3][-1].tolist() == [300, 300]


@pytest.mark.parametrize("dtype,d,G,H,T", [(torch.bfloat16, 128, 32, 96, 23), (torch.bfloat16, 64, 2, 8, 7), (torch.float32, 64, 2, 8, 7)])
def test_captured_drafts(B, dtype, d, G, H, T):
    """Drafts appended, attended to and accepted in a graph, replayed while lengths, trees and paths change: as the eager calls, every time."""
    c = R.make_cache(G, d, 1, [900, 2100], [300, 1200], dtype, 73)
    g = torch.Generator(device="cuda").manual_seed(74)
    cu_new = [0, T, 2 * T]

    def fresh():
        on = OnGpu(B, c)
        lens = [on.lens, on.lens_out]
        handles = [B.make_cache(on.k, on.v, c.cu, x, on.mass, on.pos) for x in lens]
        ws = on.workspace(B, H, 2 * T)
        normal = [torch.zeros(*s, dtype=dtype, device="cuda") for s in ((2 * T, H, d), (G, 2 * T, d), (G, 2 * T, d))]
        whole = [torch.zeros(2 * T, dtype=torch.int64, device="cuda")] + [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (2 * T, 2 * T, 2)]
        out, lse = torch.empty(2 * T, H, d, dtype=dtype, device="cuda"), torch.empty(2 * T, H, device="cuda")

        def step():
            q, k_new, v_new = normal
            mask, path, pos, n_accept = whole
            B.structkv_cache_append(handles[0], k_new, v_new, cu_new, lens[1], pos_new=pos)
            B.structkv_cache_attend(handles[1], H, q, cu_new, out, lse, ws, tree_mask=mask)
            B.structkv_cache_accept(handles[1], H, q, lse, cu_new, lens[0], path, n_accept, mask, lam=0.9)
        return on, step, normal, whole, (out, lse, on.k, on.v, on.mass, on.pos, on.lens)

    eager, replayed = fresh(), fresh()
    start = [x.clone() for x in replayed[4]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        replayed[1]()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed[1]()
    for x, y in zip(replayed[4], start):
        x.copy_(y)
    rng, grown = np.random.default_rng(75), np.array([300, 1200])
    for i in range(30):
        taken = rng.integers(0, T + 1, 2)
        grown += taken
        inputs = [torch.randn(x.shape, generator=g, device="cuda").to(dtype) for x in eager[2]]
        masks = R.as_int64(R.random_tree(T, rng) + R.random_tree(T, rng))
        whole = [masks, torch.from_numpy(rng.integers(0, T, 2 * T)), torch.arange(2 * T) + 9000 + 100 * i, torch.from_numpy(taken)]
        for side_of in (eager, replayed):
            for x, y in zip(side_of[2] + side_of[3], inputs + whole):
                x.copy_(y)
        eager[1]()
        graph.replay()
        torch.cuda.synchronize()
        for j, (x, y) in enumerate(zip(eager[4], replayed[4])):
            assert torch.equal(x.nan_to_num(), y.nan_to_num()), (i, j)
        assert eager[4][-1].tolist() == grown.tolist()


def test_another_stream(B):
    """Calls on a stream of their own, two at once with workspaces of their own."""
    c = R.make_cache(2, 128, 1, [3000], [2900], torch.bfloat16, 81)
    q, q_gpu = queries(1, 8, 128, torch.bfloat16, 81)
    sides = [OnGpu(B, c) for _ in range(3)]
    outs = [(torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 8, device="cuda"), on.workspace(B, 8, 1)) for on in sides]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), None]
    for on, (out, lse, ws), st in zip(sides, outs, streams):
        B.structkv_cache_attend(on.handle, 8, q_gpu, [0, 1], out, lse, ws, lam=0.9, stream=st)
        B.structkv_cache_evict(on.handle, None, [2000], 8, on.lens_out, ws, stream=st)
    torch.cuda.synchronize()
    for i in (1, 2):
        assert torch.equal(outs[0][0], outs[i][0]) and torch.equal(outs[0][1], outs[i][1]) and torch.equal(sides[0].mass, sides[i].mass)
        assert torch.equal(sides[0].k.nan_to_num(), sides[i].k.nan_to_num())


@pytest.mark.parametrize("dtype,d,G,H,pad,T", [(torch.bfloat16, 128, 2, 8, 1 << 24, 7), (torch.bfloat16, 64, 32, 128, 1 << 20, 20),
                                              (torch.float32, 64, 2, 4, 1 << 25, 5), (torch.bfloat16, 1, 2, 4, 1 << 22, 3)])
def test_behind_a_long_cache(B, dtype, d, G, H, pad, T):
    """Slots whose elements lie beyond 2^31 (a sequence of `pad` slots before them, empty): as in a cache of their own.  The copies are exact;
    two results of the same sums differ by twice what either may be off."""
    c = R.make_cache(G, d, G, [2100], [2000], dtype, 61)
    new, cu_new, budget = T + 1, [0, 0, T], 1500
    small = OnGpu(B, c)
    big = OnGpu.__new__(OnGpu)
    big.k, big.v = (torch.full((G, pad + 2100, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    big.mass, big.pos = torch.zeros(G, pad + 2100, device="cuda"), torch.zeros(G, pad + 2100, dtype=torch.int32, device="cuda")
    for name in ("k", "v", "mass", "pos"):
        getattr(big, name)[:, pad:] = getattr(small, name)
    q, q_gpu = queries(T, H, d, dtype, 61)
    g = torch.Generator(device="cuda").manual_seed(62)
    k_new, v_new = (torch.randn(G, T, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    pos_new = torch.arange(20000, 20000 + T, device="cuda").int()
    mask = R.as_int64(R.random_tree(T, np.random.default_rng(6))).cuda()
    path = torch.arange(T - 1, -1, -1, device="cuda").int()
    got = []
    for on, cu, new_cu in ((small, [0, 2100], [0, T]), (big, [0, pad, pad + 2100], cu_new)):
        n = len(cu) - 1
        lens = [torch.tensor([0] * (n - 1) + [2000], dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")]
        a, b = (B.make_cache(on.k, on.v, cu, x, on.mass, on.pos) for x in lens)
        ws = torch.empty(B.structkv_cache_workspace_bytes(a, H, new), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty(T, H, d, dtype=dtype, device="cuda"), torch.empty(T, H, device="cuda")
        one, one_lse = torch.empty(1, H, d, dtype=dtype, device="cuda"), torch.empty(1, H, device="cuda")
        B.structkv_cache_append(a, k_new, v_new, new_cu, lens[1], pos_new=pos_new)
        B.structkv_cache_attend(b, H, q_gpu, new_cu, out, lse, ws, tree_mask=mask, softcap=30.0)
        B.structkv_cache_attend(b, H, q_gpu[:1], [0] * n + [1], one, one_lse, ws, lam=0.5)
        mass = on.mass[:, cu[-2]:].clone()
        on.mass[:, cu[-2]:] = small.c.mass.cuda()
        B.structkv_cache_accept(b, H, q_gpu, lse, new_cu, lens[0], path, torch.tensor([0] * (n - 1) + [T - 1], dtype=torch.int32, device="cuda"), mask,
                                softcap=30.0, lam=0.5)
        accepted = on.mass[:, cu[-2]:].clone()
        on.mass[:, cu[-2]:] = small.c.mass.cuda()
        B.structkv_cache_evict(a, None, [0] * (n - 1) + [budget], 50, lens[1], ws)
        assert lens[0].tolist()[-1] == 2000 + T - 1 and lens[1].tolist()[-1] == budget
        got.append((out, one, lse, one_lse, mass, accepted, on.k[:, cu[-2]:], on.v[:, cu[-2]:], on.pos[:, cu[-2]:]))
    for x, y in zip(got[0][6:], got[1][6:]):
        assert torch.equal(x[:, :budget], y[:, :budget])
    slots = slice(0, 2000)
    x_max = float(got[0][2].abs().max()) + 16
    a_err = 2 * score_error(c, q, 1 / math.sqrt(d), x_max) + (2100 / 16 + 64) * 2.0 ** -24
    v_max = float(torch.nan_to_num(c.v.float(), 0.0, 0.0, 0.0).abs().max().clamp(min=float(v_new.abs().max())))
    for x, y in zip(got[0][:2], got[1][:2]):
        x, y = x.double(), y.double()
        within(y.cpu(), x.cpu(), (2 * EPS[dtype] * x.abs() + 2 * (2 * a_err + 2.0 ** -16) * v_max).cpu(), "out")
    for x, y in zip(got[0][2:4], got[1][2:4]):
        x, y = x.double(), y.double()
        within(y.cpu(), x.cpu(), 2 * (a_err + 2.0 ** -23 * x.abs()).cpu(), "lse")
    for x, y in zip(got[0][4:6], got[1][4:6]):
        x, y = x[:, slots].double(), y[:, slots].double()
        within(y.cpu(), x.cpu(), 2 * ((2.0 ** -22 + 2 * a_err + 4 * x_max * 2.0 ** -24) * x.abs()).cpu(), "mass")


def test_layer_cache_after_a_sweep(B):
    """LayerCache behind LayerSweep: a ragged batch's compact caches, then tokens, drafts and evictions, beside the calls themselves."""
    from paper_2604_06746_amd.cache import LayerCache
    from paper_2604_06746_amd.sweep import LayerSweep
    H, G, d, w, lens, keep, dtype = 8, 2, 128, 8, [300, 450], [60, 90], torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(91)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    sw = LayerSweep(H, G, d, w, dtype, lens, keep)
    sw.layer(normal(2, H, w, d), normal(G, sum(lens), d), normal(G, sum(lens), d))
    rows = [k + w for k in keep]
    cu_rows = R.cut(rows)
    cache = LayerCache(H, G, d, dtype, [n + 30 for n in rows])
    first = torch.repeat_interleave(torch.tensor([0, lens[0]], device="cuda"), torch.tensor(rows, device="cuda"))
    idx = sw.idx_kv[:sum(rows)]
    cache.append(sw.k_cache[0][:, :sum(rows)], sw.v_cache[0][:, :sum(rows)], cu_rows, idx, sw.indeg[first + idx])
    assert cache.lens.tolist() == rows
    c = R.make_cache(G, d, 1, [n + 30 for n in rows], rows, dtype, 92)

    def state():
        torch.cuda.synchronize()
        c.k, c.v, c.mass, c.pos, c.lens = cache.k.cpu(), cache.v.cpu(), cache.mass.cpu(), cache.pos.cpu(), cache.lens.tolist()
        return c
    for step, T in enumerate((1, 7, 1)):
        rng, cu_new = np.random.default_rng(step), R.cut([T, T])
        masks = R.random_tree(T, rng) + R.random_tree(T, rng)
        tree, q = R.as_int64(masks).cuda(), normal(2 * T, H, d)
        cache.append(normal(G, 2 * T, d), normal(G, 2 * T, d), cu_new, torch.arange(2 * T, device="cuda").int() + 1000 + 10 * step)
        before = state()
        lam = 0.9 if T == 1 else 0.0
        out, lse = cache.attend(q, cu_new, tree, lam)
        ref, ref_lse, mass, size = R.attend(before, H, q.cpu(), cu_new, masks, lam=lam)
        within(out.cpu().double(), ref, EPS[dtype] * ref.abs() + 1e-4 * size, "out")
        within(lse.cpu().double(), ref_lse, torch.tensor(1e-4), "lse")
        within(cache.mass.cpu().double(), mass, 1e-4 * mass.abs(), "mass")
        if T > 1:
            n_accept = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
            path = torch.zeros(2 * T, dtype=torch.int32, device="cuda")
            path[1], path[T] = T - 1, 3
            before = state()
            cache.accept(cu_new, path, n_accept, q, lse, tree, 0.9)
            *_, mass, new_lens = R.accept(before, H, q.cpu(), lse.cpu(), cu_new, path.cpu(), [2, 1], masks, lam=0.9)
            assert cache.lens.tolist() == new_lens
            within(cache.mass.cpu().double(), mass, 1e-4 * mass.abs(), "mass")
    before = state()
    cache.evict([40, 50], w)
    k, v, pos, mass, new_lens = R.evict(before, before.mass, [40, 50], w)
    after = state()
    assert after.lens == new_lens == [40, 50] and torch.equal(after.pos, pos) and torch.equal(after.mass, mass)
    for b in range(2):
        used = slice(c.cu[b], c.cu[b] + new_lens[b])
        assert torch.equal(after.k[:, used], k[:, used]) and torch.equal(after.v[:, used], v[:, used])
    with pytest.raises(B.StructKVError):
        LayerCache(7, 2, 64, dtype, [10])
