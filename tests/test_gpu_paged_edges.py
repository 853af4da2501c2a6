"""GPU tests of attention over a cache held in pages, beside test_gpu_paged.py: scores, scales and values at their limits.

Tolerances as derived there, unless a test says otherwise."""
import math

import numpy as np
import pytest
import torch

import paged_precision as L
import paged_reference as R
from test_gpu_paged import B, EPS, OnGpu, cut, table, within  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


def run(B, c, H, q, fresh, *, scale=1.0, softcap=0.0, lam=0.0, on=None):  # noqa: F811
    """(out, lse, mass) in host memory; the call twice, from the same mass, with the workspace as it was left: the same bits."""
    on, new, res = on or OnGpu(B, c), sum(fresh), []
    ws, mass = on.workspace(B, H, new), on.mass.clone()
    for _ in range(2):
        out = torch.full((new, H, c.d), math.nan, dtype=c.dtype, device="cuda")
        lse = torch.full((new, H), math.nan, device="cuda")
        on.mass.copy_(mass)
        B.structkv_paged_attend(on.handle, H, q.cuda(), cut(fresh), out, lse, ws, scale=scale, softcap=softcap, lam=lam)
        res.append((out, lse, on.mass.clone()))
    for x, y in zip(*res):
        assert torch.equal(x.nan_to_num(7e30), y.nan_to_num(7e30))
    return out.cpu(), lse.cpu(), on.mass.cpu()


FORMS = [(torch.bfloat16, 128, 2, 8, 1), (torch.bfloat16, 64, 2, 8, 7), (torch.bfloat16, 128, 2, 8, 40), (torch.float32, 64, 2, 8, 7), (torch.float32, 128, 2, 40, 1),
         (torch.bfloat16, 80, 2, 4, 1), (torch.float32, 256, 1, 4, 3), (torch.bfloat16, 256, 1, 4, 20)]


@pytest.mark.parametrize("dtype,d,G,H,T", FORMS)
@pytest.mark.parametrize("lens", [[1300, 700], [300, 90]])
@pytest.mark.parametrize("score", [-2.0 ** 22, 2.0 ** 23, 2.0 ** 25, -2.0 ** 28, 2.0 ** 28, 2.0 ** 30, -2.0 ** 40, 2.0 ** 40, -2.0 ** 90, 2.0 ** 110, -2.0 ** 125])
def test_scores_far_from_zero(B, dtype, d, G, H, T, lens, score):  # noqa: F811
    """A row whose scores are huge attends to the highest: one slot's value as it is, lse its score (to log2 and back: a rounding each of score,
    factor and product on both ways), mass of one for each head."""
    best = [77 * lens[0] // 100, 0]
    pages, n = table(lens, 16, np.random.default_rng(5), spare=1)
    c = R.make_pool(G, d, 16, n, pages, lens, dtype, 41)
    c.k[:], c.ks[:] = 0, 1.0
    small, large = R.encode(torch.tensor([1.125, 2.0], dtype=torch.float64)) + (128 if score < 0 else 0)
    c.k[:, :, :, 0] = large if score < 0 else small
    for b in range(2):
        c.k[pages[b][best[b] // 16], :, best[b] % 16, 0] = small if score < 0 else large
    q = torch.zeros(2 * T, H, d, dtype=dtype)
    q[:, :, 0] = 1.2890625 * abs(score)
    want = 1.2890625 * abs(score) * (-1.125 if score < 0 else 2.0)
    out, lse, mass = run(B, c, H, q, [T, T], lam=0.5 if T == 1 else 0.0)
    for b in range(2):
        p, r = pages[b][best[b] // 16], best[b] % 16
        v = (R.decode(c.v[p, :, r]) * c.vs[p].double()[:, None]).repeat_interleave(H // G, 0)      # (exact in 16 bits)
        assert torch.equal(out[b * T:(b + 1) * T].double(), v.expand(T, H, d))
    assert torch.all((lse.double() / want - 1).abs() <= 6 * 2.0 ** -24)
    if T == 1:
        ref = c.mass.double()
        for b in range(2):
            ref[b, :len(pages[b]) - 1] *= 0.5
            ref[b, best[b] // 16] += H
        within(mass.double(), ref, H * 2.0 ** -19 * (ref > 0.0), "mass")     # (log2 of sums up to 2^16, to 2^-20 each)


@pytest.mark.parametrize("dtype,d,G,H,T", FORMS)
@pytest.mark.parametrize("score", [0.0, 5.0 * 2.0 ** 10, -5.0 * 2.0 ** 19, 5.0 * 2.0 ** 19, 5.0 * 2.0 ** 22, -5.0 * 2.0 ** 22, 5.0 * 2.0 ** 26, -5.0 * 2.0 ** 40, 5.0 * 2.0 ** 100])
def test_equal_scores_share(B, dtype, d, G, H, T, score):  # noqa: F811
    """Slots that share the highest score, in pages whose values have other scales, share the weight evenly whatever the score is; the others are
    too far below to count, or there are none (score 0).  A weight is rounded to 11 bits (fp32 outputs: 22), its sum to fp32."""
    lens = [1000, 333]
    pages, n = table(lens, 16, np.random.default_rng(6), spare=1)
    c = R.make_pool(G, d, 16, n, pages, lens, dtype, 42)
    c.k[:], c.ks[:] = 0, 1.0
    c.vs = torch.exp2(torch.randint(-9, 3, (n, G), generator=torch.Generator().manual_seed(1)).float())
    one, two = R.encode(torch.tensor([1.0, 2.0], dtype=torch.float64)) + (128 if score < 0 else 0)
    c.k[:, :, :, 0] = two if score < 0 else one
    tops = [[0, 5, 16, 300, 301, 640, 900], [3, 100, 200]]
    for b in range(2):
        for s in tops[b]:
            c.k[pages[b][s // 16], :, s % 16, 0] = one if score < 0 else two
    if score == 0.0:
        tops = [list(range(lens[b])) for b in range(2)]
    q = torch.zeros(2 * T, H, d, dtype=dtype)
    q[:, :, 0] = abs(score)
    best = abs(score) * (-1.0 if score < 0 else 2.0)
    out, lse, mass = run(B, c, H, q, [T, T], lam=0.5 if T == 1 else 0.0)
    p_err = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    ref_mass = c.mass.double()
    for b in range(2):
        for t in range(T):
            seen = [s for s in tops[b] if s <= lens[b] - T + t]
            p = torch.tensor([pages[b][s // 16] for s in seen])
            v = R.decode(c.v[p, :, torch.tensor([s % 16 for s in seen])]) * c.vs[p].double()[..., None]
            ref, size = (x.mean(0).repeat_interleave(H // G, 0) for x in (v, v.abs()))
            within(out[b * T + t].double(), ref, EPS[dtype] * ref.abs() + p_err * size + 2.0 ** -30 * v.abs().max(), "out of row %d" % t)
            norm = best + math.log(len(seen))
            assert torch.all((lse[b * T + t].double() - norm).abs() <= 6 * 2.0 ** -24 * abs(norm) + 2.0 ** -20), (t, lse[b * T + t], norm)
        ref_mass[b, :len(pages[b]) - 1] *= 0.5
        for s in seen:
            ref_mass[b, s // 16] += H / len(seen)
    if T == 1:
        within(mass.double(), ref_mass, 2.0 ** -18 * ref_mass.abs(), "mass")     # (the same, and its sums' roundings)


@pytest.mark.parametrize("dtype,d,G,H,T", FORMS)
def test_rows_of_all_sizes_side_by_side(B, dtype, d, G, H, T):  # noqa: F811
    """Heads whose scores are zero, some hundreds, thousands, 2^22, 2^30 and as far below zero share waves; each is what it is by itself.  Scores are exact
    products, equal or far apart."""
    lens = [700, 90]
    pages, n = table(lens, 32, np.random.default_rng(9), spare=1)
    c = R.make_pool(G, d, 32, n, pages, lens, dtype, 46)
    used = c.k[..., 0] != 127
    c.ks[:] = 1.0
    c.k[:] = 0
    c.k[..., 0] = R.encode((torch.rand(n, G, 32, generator=torch.Generator().manual_seed(1)) < 0.05).double() + 1.0)
    c.k[~used] = 127
    size = torch.tensor([0.0, 320.0, -320.0, 5120.0, -5120.0, 5.0 * 2 ** 22, -5.0 * 2 ** 22, 5.0 * 2 ** 30])
    q = torch.zeros(2 * T, H, d, dtype=dtype)
    q[:, :, 0] = (size[torch.arange(2 * T * H) % 8]).view(2 * T, H)
    if dtype == torch.bfloat16:
        assert torch.equal(q[:, :, 0].flatten()[:8].float(), size)
    lam = 0.5 if T == 1 else 0.0
    out, lse, mass = run(B, c, H, q, [T, T], lam=lam)
    ref, ref_lse, ref_mass, size, top = R.attend(c, H, q, [0, T, 2 * T], 1.0, 0.0, lam)
    p_err = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    within(out.double(), ref, EPS[dtype] * ref.abs() + p_err * size + 700 * 2.0 ** -31 * top, "out")
    within(lse.double(), ref_lse, 6 * 2.0 ** -24 * ref_lse.abs() + 2.0 ** -20, "lse")
    within(mass.double(), ref_mass, 2.0 ** -12 * ref_mass.abs(), "mass")      # (norms of up to 2^10 are taken off as one number: 2^-14 each, and log2's)


@pytest.mark.parametrize("G,H,n", [(128, 128, 70000), (64, 512, 36000)])
@pytest.mark.parametrize("score", [5.0 * 2.0 ** 11, -5.0 * 2.0 ** 26])
def test_large_scores_of_long_shares(B, G, H, n, score):  # noqa: F811
    """Waves that see more blocks than have room for their weights at once, the highest scores among the first, the last and some between."""
    d, ps = 16, 64
    per = -(-n // ps)
    pages = np.random.default_rng(3).permutation(per + 2)[:per].tolist()
    one, two = R.encode(torch.tensor([1.0, 2.0], dtype=torch.float64)) + (128 if score < 0 else 0)
    k = torch.zeros(per + 2, G, ps, d, dtype=torch.uint8)
    k[..., 0] = two if score < 0 else one
    tops = [1, 2, 5000, 5001, 17777, 30000, n - 1]
    c = R.make_pool(1, 16, 16, 1, [[0]], [0], torch.bfloat16, 1)
    c.G, c.d, c.ps, c.n_pages, c.lens, c.pages = G, d, ps, per + 2, [n], torch.tensor([pages], dtype=torch.int32)
    for s in tops:
        k[pages[s // ps], :, s % ps, 0] = one if score < 0 else two
    c.k, c.v = k, torch.full_like(k, int(one) & 127)
    c.ks, c.vs, c.mass = torch.ones(per + 2, G), torch.exp2(torch.arange(per + 2) % 7 - 3.0)[:, None].repeat(1, G), torch.zeros(1, per)
    q = torch.zeros(1, H, d, dtype=torch.bfloat16)
    q[:, :, 0] = abs(score)
    out, lse, mass = run(B, c, H, q, [1], lam=1.0)
    want = float(np.mean([float(c.vs[pages[s // ps], 0]) for s in tops]))
    assert torch.all((out.double() / want - 1).abs() <= 2.0 ** -8 + 2.0 ** -11)
    ref = torch.zeros(1, per, dtype=torch.float64)
    for s in tops:
        ref[0, s // ps] += H / len(tops)
    within(mass.double(), ref, 2.0 ** -18 * ref, "mass")


@pytest.mark.parametrize("dtype,d,G,H,T", FORMS)
@pytest.mark.parametrize("lens", [[1300, 700], [300, 90]])
@pytest.mark.parametrize("high", [11, 12, 13, 40, 64])
def test_value_scales_far_apart(B, dtype, d, G, H, T, lens, high):  # noqa: F811
    """The weight of a page whose values are zeros (scale 2^-64, as they are stored) or tiny, beside pages of 2^11 to 2^64: lse and mass do not depend on
    the values' scales at all, out is what the large ones make of their share.  Scores of a few units."""
    pages, n = table(lens, 16, np.random.default_rng(7), spare=1)
    for kind in ("zeros", "tiny", "few"):
        c = R.make_pool(G, d, 16, n, pages, lens, dtype, 43)
        g = torch.Generator().manual_seed(2)
        small = torch.rand(n, G, generator=g) < (0.03 if kind == "few" else 0.5)
        c.vs = torch.where(small, 2.0 ** -64, 2.0 ** high)
        if kind == "zeros":
            c.v[small & (c.v != 127).all(3).all(2)] = 0
        flat = OnGpu(B, c)
        flat.vs.fill_(2.0 ** -3)
        q = torch.randn(2 * T, H, d, generator=g).to(dtype)
        res = [run(B, c, H, q, [T, T], scale=0.0, lam=0.5 if T == 1 else 0.0, on=on) for on in (None, flat)]
        (out, lse, mass), (_, want_lse, want_mass) = res
        ref, _, _, size, top = R.attend(c, H, q, cut([T, T]))
        # the same sums in other units: their roundings, and a log2 to 2^-20
        within(lse.double(), want_lse.double(), 2.0 ** -18 + 2.0 ** -22 * want_lse.abs().double(), "lse")
        within(mass.double(), want_mass.double(), 2.0 ** -18 * want_mass.abs().double(), "mass")
        # scores of d terms of magnitude up to |q| |k|, as in test_gpu_paged.py; what tiny values add is below the last bits of the others'
        keys = (R.decode(c.k).nan_to_num(0.0) * c.ks[:, :, None, None]).norm(dim=3).max()
        a_err = 2 * float(d * keys * q.double().norm(dim=2).max() / math.sqrt(d) + 512) * 2.0 ** -24 + (max(lens) / 16 + 64) * 2.0 ** -24
        p_err = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
        within(out.double(), ref, EPS[dtype] * ref.abs() + (2 * a_err + p_err) * size + max(lens) * 2.0 ** -31 * top, "out")


def test_a_page_of_zeros_weighs_what_it_weighs(B):  # noqa: F811
    """Stored by append: zeros in the values of one page, 2^70 in another's, scores all equal: half the weight is each one's."""
    dtype, d = torch.float32, 64
    for order in (0, 1):
        c = R.make_pool(1, d, 16, 4, [[1, 2]], [0], dtype, 1)
        on = OnGpu(B, c)
        v = torch.zeros(1, 32, d)
        v[:, 16 * order:16 * order + 16] = 2.0 ** 70
        B.structkv_paged_append(on.handle, torch.ones(1, 32, d).cuda(), v.cuda(), [0, 32], on.lens_out)
        assert on.lens_out.tolist() == [32] and on.vs.cpu().flatten()[1 + (1 - order)] == 2.0 ** -64
        on.handle = B.make_paged(on.k, on.v, on.ks, on.vs, on.pages, on.lens_out, dtype, on.mass, on.missed)
        on.mass.zero_()
        out, lse, mass = run(B, c, 1, torch.zeros(1, 1, d), [1], lam=1.0, on=on)
        assert torch.all((out / 2.0 ** 69 - 1).abs() <= 2.0 ** -21), out       # (the mean: half of 2^70)
        assert abs(float(lse) - math.log(32.0)) <= 2.0 ** -20 and torch.all((mass[0, :2] - 0.5).abs() <= 2.0 ** -19), (lse, mass)


@pytest.mark.parametrize("dtype,d,G,H,lens,T", [(torch.bfloat16, 128, 2, 8, [70, 300], 64), (torch.bfloat16, 64, 1, 2, [100, 100], 100), (torch.float32, 128, 2, 4, [90, 700], 90),
                                                (torch.float32, 256, 1, 8, [40, 77], 33), (torch.bfloat16, 128, 1, 16, [1300, 40], 40)])
@pytest.mark.parametrize("at", [0, 1, 3, 17, 30])
def test_values_that_are_not_numbers_in_a_chunk(B, dtype, d, G, H, lens, T, at):  # noqa: F811
    """A fresh slot behind the first whose value has a NaN: every row that sees it gets NaN throughout, in whichever block of rows it is; the first
    fresh slot's NaN (at = 0), and an older one's, stay in their component.  Rows that do not see it, and other KV heads' heads, are as without it."""
    pages, n = table(lens, 16, np.random.default_rng(4), spare=1)
    for b in range(2):
        for s, fresh in ((lens[b] - T + at, at > 0), (3, False)):
            if s == 3 and lens[b] - T <= 3:      # (that would be a fresh one)
                continue
            c, clean = (R.make_pool(G, d, 16, n, pages, lens, dtype, 4) for _ in range(2))
            c.v[pages[b][s // 16], G - 1, s % 16, 5] = 127
            q = torch.randn(2 * T, H, d, generator=torch.Generator().manual_seed(9)).to(dtype)
            (out, lse, _), (want, want_lse, _) = (run(B, x, H, q, [T, T], scale=0.0) for x in (c, clean))
            assert torch.equal(lse, want_lse)
            sees = torch.zeros(2 * T, dtype=torch.bool)
            sees[b * T + max(0, s - (lens[b] - T)):(b + 1) * T] = True
            hit = torch.zeros_like(out, dtype=torch.bool)
            heads = slice(H // G * (G - 1), H)
            hit[sees, heads] = fresh
            hit[sees, heads, 5] = True
            assert torch.equal(out.isnan(), hit), (b, s)
            assert torch.equal(out[~hit], want[~hit])


def test_not_numbers_beside_dropped_pages(B):  # noqa: F811
    """Two fresh NaN slots, one of them in a dropped page: that one reaches nobody."""
    lens, T, d, H = [200], 60, 64, 4
    pages, n = table(lens, 16, np.random.default_rng(4), spare=1)
    c, clean = (R.make_pool(1, d, 16, n, pages, lens, torch.bfloat16, 4) for _ in range(2))
    for s in (150, 180):
        c.v[pages[0][s // 16], 0, s % 16, 7] = 127
    c.pages[0, 150 // 16] = clean.pages[0, 150 // 16] = -1
    q = torch.randn(T, H, d, generator=torch.Generator().manual_seed(9)).bfloat16()
    (out, lse, _), (want, want_lse, _) = (run(B, x, H, q, [T], scale=0.0) for x in (c, clean))
    assert torch.equal(lse, want_lse) and torch.equal(out[:40], want[:40]) and bool(out[40:].isnan().all())


@pytest.mark.parametrize("dtype,d,G,H,T", FORMS)
@pytest.mark.parametrize("scale,key_scale", [(1e-30, 2.0 ** -64), (1.2e-38, 1.0), (1e-44, 2.0 ** -20), (1e-18, 2.0 ** -64)])
def test_scores_next_to_nothing(B, dtype, d, G, H, T, scale, key_scale):  # noqa: F811
    """scale times a page's scale below fp32's least number: all scores are zero, so a row's result is the mean of the values that it sees."""
    lens = [300, 41]
    pages, n = table(lens, 16, np.random.default_rng(8), spare=1)
    c = R.make_pool(G, d, 16, n, pages, lens, dtype, 44)
    c.ks[:] = key_scale
    q = torch.randn(2 * T, H, d, generator=torch.Generator().manual_seed(3)).to(dtype)
    out, lse, mass = run(B, c, H, q, [min(T, 41), T], scale=scale, lam=0.5 if T == 1 else 0.0)
    ref, ref_lse, ref_mass, size, top = R.attend(c, H, q, cut([min(T, 41), T]), scale, 0.0, 0.5 if T == 1 else 0.0)
    p_err = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22
    within(lse.double(), ref_lse, 2.0 ** -20 + 0 * ref_lse, "lse")
    within(out.double(), ref, EPS[dtype] * ref.abs() + (p_err + 2.0 ** -18) * size + 300 * 2.0 ** -31 * top, "out")
    within(mass.double(), ref_mass, 2.0 ** -18 * ref_mass.abs(), "mass")


def test_scale_beyond_fp32(B):  # noqa: F811
    """A scale that leaves fp32's range where it meets a page's largest is refused; the largest that does not is taken."""
    c = R.make_pool(1, 64, 16, 4, [[1]], [5], torch.float32, 1)
    c.ks[:] = 2.0 ** 64
    q = torch.zeros(1, 1, 64)
    out, lse, _ = run(B, c, 1, q, [1], scale=2.0 ** 62)
    assert abs(float(lse) - math.log(5.0)) <= 2.0 ** -20 and bool(out.isfinite().all())
    with pytest.raises(B.StructKVError) as e:
        run(B, c, 1, q, [1], scale=2.0 ** 63)
    assert e.value.status == B.STRUCTKV_ERR_UNSUPPORTED


@pytest.mark.parametrize("value", [3.4028234e38, -3.4e38, 3.39e38, 2.0 ** 100 * 1.99999, 1.1754944e-38 * 3])
def test_queries_at_the_ends_of_fp32(B, value):  # noqa: F811
    """fp32 queries next to the largest number, which bf16 parts that are rounded to the nearest do not hold: scores of a few units."""
    dtype, d, H, lens = torch.float32, 64, 4, [100, 33]
    pages, n = table(lens, 16, np.random.default_rng(8), spare=1)
    c = R.make_pool(1, d, 16, n, pages, lens, dtype, 45)
    k = R.decode(c.k)
    c.k = R.encode(torch.where(torch.arange(d) == 0, (k / 512).clamp(-0.7, 0.7), 0.0 * k).nan_to_num(0.0))      # (products that stay in range)
    c.ks[:] = 2.0 ** -6
    q = torch.zeros(2, H, d)
    q[..., 0] = value * torch.tensor([1.0, 0.75, 0.9999999, 1.0])
    scale = float(min(2.0 ** 62, 2.0 ** 8 / abs(value)))
    out, lse, mass = run(B, c, H, q, [1, 1], scale=scale, lam=0.5)
    ref, ref_lse, ref_mass, size, top = R.attend(c, H, q, [0, 1, 2], scale, 0.0, 0.5)
    assert scale == 2.0 ** 62 or float(ref_lse.abs().max()) > 3.0
    # one product a score: roundings of it, of its scale and of the sums
    within(lse.double(), ref_lse, 2.0 ** -19 + 0 * ref_lse, "lse")
    within(out.double(), ref, 2.0 ** -24 * ref.abs() + 2.0 ** -18 * size + 2.0 ** -24 * top, "out")
    within(mass.double(), ref_mass, 2.0 ** -17 * ref_mass.abs(), "mass")


def test_rotation_of_more_than_one_launch(B):  # noqa: F811
    """2^32 units of 16 bytes (64 GiB, in place): more threads than a launch may have."""
    d, tokens, dtype = 65536, (1 << 32) // 8192 + 3, torch.bfloat16
    row = torch.randn(d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    x = torch.empty(tokens, 1, d, dtype=dtype, device="cuda")
    x.copy_(row.expand_as(x))
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    turns, _ = B.structkv_rotary_turns(64, 500000.0)
    plan = B.make_rotary(turns.cuda())
    B.structkv_rotate(plan, x, pos, x)
    for t in (0, 1, 262143, 262144, 262145, 300001, 524287, 524288, tokens - 1):
        want = torch.empty(1, 1, d, dtype=dtype, device="cuda")
        B.structkv_rotate(plan, row[None, None], pos[t:t + 1], want)
        assert torch.equal(x[t:t + 1], want), t
    del x
    torch.cuda.empty_cache()


def test_append_of_more_than_one_launch(B):  # noqa: F811
    """One long prompt among many short sequences: workgroups for as many pages of each would be more than a launch may have."""
    G, d, ps, batch, long = 8, 16, 16, 64, (1 << 20) + 5
    fresh = [3] * batch
    fresh[1], fresh[5] = long, 0
    total, cu = sum(fresh), cut(fresh)
    per = -(-(long + 7) // ps)
    g = torch.Generator(device="cuda").manual_seed(2)
    n = per + 2 * batch
    codes = torch.zeros(n, G, ps, d, dtype=torch.uint8, device="cuda")
    pages = torch.full((batch, per), -1, dtype=torch.int32, device="cuda")
    pages[1] = torch.randperm(per, generator=g, device="cuda").int()
    rest = [b for b in range(batch) if b != 1]
    pages[rest, 0], pages[rest, 1] = (per + torch.arange(i, 2 * batch - 2, 2, device="cuda").int() for i in (0, 1))
    k, v = (torch.randn(G, total, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(total, G, d, generator=g, device="cuda").bfloat16()
    turns, _ = B.structkv_rotary_turns(d, 500000.0)
    plan = B.make_rotary(turns.cuda())
    lens = torch.tensor([7 + (b % 9) for b in range(batch)], dtype=torch.int32, device="cuda")
    lens[1] = 2
    res = []
    for parts in ([list(range(batch))], [[b] for b in range(batch)]):
        kc, vc, ks, vs = codes.clone(), codes.clone(), torch.ones(n, G, device="cuda"), torch.ones(n, G, device="cuda")
        lens_out, missed, q_out = torch.full_like(lens, -1), torch.zeros_like(lens), torch.empty_like(q)
        for part in parts:
            s, b = slice(cu[part[0]], cu[part[-1] + 1]), slice(part[0], part[-1] + 1)
            handle = B.make_paged(kc, vc, ks, vs, pages[b], lens[b], missed=missed[b])
            B.structkv_paged_append(handle, k[:, s], v[:, s], [x - cu[part[0]] for x in cu[part[0]:part[-1] + 2]], lens_out[b], plan, q=q[s], q_out=q_out[s])
        res.append((kc, vc, ks, vs, lens_out, missed, q_out.view(torch.int16)))
    assert torch.equal(res[0][4], lens + torch.tensor(fresh, device="cuda").int()) and not res[0][5].any()
    for x, y in zip(*res):
        assert torch.equal(x, y)


def test_gathering_over_a_capacity_of_many_launches(B):  # noqa: F811
    """Stretches of 64 blocks of a capacity that more than 2^24 workgroups would go through: a few tokens in use, the last one's pages at the start."""
    lens, cap = [40, 3], (1 << 31) - 2048
    pages, n = table(lens, 256, np.random.default_rng(1))
    c = R.make_pool(1, 16, 256, n, pages, lens, torch.bfloat16, 3)
    batch, most = 9, cap // 256
    on = OnGpu(B, c)
    whole = torch.full((batch, most), -1, dtype=torch.int32, device="cuda")
    lens9 = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for b, to in ((0, 0), (1, 8)):
        whole[to, :len(pages[b])] = on.pages[b, :len(pages[b])]
        lens9[to] = lens[b]
    mass = torch.ones(batch, most, device="cuda")
    handle = B.make_paged(on.k, on.v, on.ks, on.vs, whole, lens9, torch.bfloat16, mass)
    q = torch.randn(2, 1, 16, generator=torch.Generator().manual_seed(3)).bfloat16()
    out, lse = torch.empty(2, 1, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 1, device="cuda")
    ws = torch.empty(B.structkv_paged_workspace_bytes(handle, 1, 2), dtype=torch.uint8, device="cuda")
    B.structkv_paged_attend(handle, 1, q.cuda(), [0, 1, 1, 1, 1, 1, 1, 1, 1, 2], out, lse, ws, lam=0.5)
    want, want_lse, _ = run(B, c, 1, q, [1, 1], scale=0.0, lam=0.5)
    within(out.cpu().double(), want.double(), 2.0 ** -7 * want.double().abs() + 2.0 ** -10, "out")
    within(lse.cpu().double(), want_lse.double(), 2.0 ** -18 + 0 * want_lse.double(), "lse")
    got = mass.cpu()
    assert abs(float(got[0, 0]) - 1.5) <= 2.0 ** -18 and abs(float(got[8, 0]) - 1.5) <= 2.0 ** -18
    got[0, 0] = got[8, 0] = 1.0
    assert torch.all(got == 1.0)


@pytest.mark.parametrize("d", [16, 64, 80, 128, 256])
@pytest.mark.parametrize("lens,T", [((500, 90), 3), ((1700, 90), 1), ((1700, 90), 20), ((60, 20), 20)])
def test_precision_of_fp32(B, d, lens, T):  # noqa: F811
    """The whole of out and lse against what roundings make of them: all of a query's 24 bits and 22 of the weights' are there."""
    c, H, q, cu_new, scale = L.case(d, lens, T)
    out, lse, mass = run(B, c, H, q, [T, T], scale=scale, lam=0.5 if T == 1 else 0.0)
    ref, ref_lse, out_off, lse_off = L.attend(c, H, q, cu_new, scale)
    assert L.worst(out, ref, out_off) <= L.MOST and L.worst(lse, ref_lse, lse_off) <= L.MOST
    if T == 1:      # (weights of all heads to 2^-20: the norm and log2 of the blocks' sums, of numbers up to 32, and back)
        _, _, ref_mass, _, _ = R.attend(c, H, q, cu_new, scale, 0.0, 0.5)
        within(mass.double(), ref_mass, 2.0 ** -18 * ref_mass.abs() + H * 2.0 ** -24, "mass")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H", [(1, 4), (1, 20), (7, 1), (9, 4)])
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_rise_and_rise(B, dtype, T, H, falling):  # noqa: F811
    """Exact scores from -2^20 to 2^20, page by page (or the other way round), so that the reference is raised again and again; the slots of the highest page
    are some units apart, and only they count.  Nothing but the weights' and the sums' roundings is left."""
    lens, ps, d = [640, 640], 16, 64
    pages, n = table(lens, ps, np.random.default_rng(2))
    c = R.make_pool(1, d, ps, n, pages, lens, dtype, 47)
    g = torch.Generator().manual_seed(5)
    c.k[:] = 0
    for b in range(2):
        for j, p in enumerate(pages[b]):
            i = 39 - j if falling else j
            c.ks[p, 0] = 2.0 ** (15 - i) if i < 20 else 2.0 ** (i - 24)
            c.k[p, 0, :, 0] = R.encode(torch.full((ps,), -8.0 if i < 20 else 8.0, dtype=torch.float64))
            c.k[p, 0, :, 1] = R.encode(torch.randint(-15, 16, (ps,), generator=g).double())
    q = torch.zeros(2 * T, H, d, dtype=dtype)
    q[..., 0], q[..., 1] = 4.0, 2.0 ** -17
    lam = 0.5 if T == 1 else 0.0
    out, lse, mass = run(B, c, H, q, [T, T], lam=lam)
    ref, ref_lse, ref_mass, size, top = R.attend(c, H, q, cut([T, T]), 1.0, 0.0, lam)
    p_err = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    within(out.double(), ref, EPS[dtype] * ref.abs() + (p_err + 2.0 ** -19) * size + 640 * 2.0 ** -31 * top, "out")
    within(lse.double(), ref_lse, 6 * 2.0 ** -24 * ref_lse.abs(), "lse")
    within(mass.double(), ref_mass, 2.0 ** -17 * ref_mass.abs(), "mass")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,T", [((500, 90), 3), ((1700, 90), 1), ((1700, 90), 8)])
def test_bf16_results_are_the_nearest(B, d, lens, T):  # noqa: F811
    """Of queries whose rows fit a workgroup: the last bit is another than the exact result's only next to a tie, one in some hundreds by the model of
    roundings (test_paged_edges.py); weights of 11 bits would make it one in 20 to 30."""
    c, H, q, cu_new, scale = L.case(d, lens, T)
    c.dtype, q = torch.bfloat16, q.bfloat16()
    out, _, _ = run(B, c, H, q, [T, T], scale=scale)
    ref, _, _, _ = L.attend(c, H, q, cu_new, scale)
    assert float((out != ref.bfloat16()).double().mean()) <= L.TURNED


@pytest.mark.parametrize("score", [1.0, 5.0 * 2.0 ** 9, 5.0 * 2.0 ** 26])
@pytest.mark.parametrize("G,H,lens", [(5, 5, [45]), (1, 1, [3]), (32, 4096, [40, 17]), (3, 51, [77])])
def test_gathering_at_odd_places(B, G, H, lens, score):  # noqa: F811
    """As many heads as there may be, and pairs of unit and weight that begin at an odd word; what lies behind the workspace stays."""
    pages, n = table(lens, 16, np.random.default_rng(G))
    c = R.make_pool(G, 16, 16, n, pages, lens, torch.bfloat16, 5)
    used = c.k[..., 0] != 127
    c.ks[:] = 1.0
    c.k[:] = 0
    c.k[..., 0] = R.encode((torch.rand(n, G, 16, generator=torch.Generator().manual_seed(2)) < 0.1).double() + 1.0)
    c.k[~used] = 127
    new = len(lens)
    q = torch.zeros(new, H, 16, dtype=torch.bfloat16)
    q[..., 0] = score
    on = OnGpu(B, c)
    size = B.structkv_paged_workspace_bytes(on.handle, H, new)
    ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty(new, H, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(new, H, device="cuda")
    B.structkv_paged_attend(on.handle, H, q.cuda(), list(range(new + 1)), out, lse, ws[:size], scale=1.0, lam=0.5)
    ref, ref_lse, ref_mass, norm, top = R.attend(c, H, q, list(range(new + 1)), 1.0, 0.0, 0.5)
    assert bool((ws[size:] == 0xA5).all())
    # (where a KV head's rows are more than the 16 of a workgroup, weights have 11 bits: 2^-12 of each; else 22)
    p_err = 2.0 ** -19 + (2.0 ** -12 if H // G > 16 else 0.0)
    within(out.cpu().double(), ref, 2.0 ** -8 * ref.abs() + p_err * norm + 77 * 2.0 ** -31 * top, "out")
    within(lse.cpu().double(), ref_lse, 6 * 2.0 ** -24 * ref_lse.abs() + 2.0 ** -20, "lse")
    within(on.mass.cpu().double(), ref_mass, 2.0 ** -17 * ref_mass.abs(), "mass")
