"""GPU tests of the operators on a cache in use, beside test_gpu_cache.py: sequences without room, and values and sizes at their limits.

Tolerances as derived there, unless a test says otherwise."""
import math

import numpy as np
import pytest
import torch

import cache_reference as R
from test_gpu_cache import B, EPS, within  # noqa: F401  (B is the fixture)

pytestmark = pytest.mark.gpu


def full_cache(dtype, d, G, H, planes, caps, lens, seed):
    """A LayerCache that holds lens[b] tokens, and what it holds."""
    from paper_2604_06746_amd.cache import LayerCache
    c = R.make_cache(G, d, planes, caps, lens, dtype, seed)
    cache = LayerCache(H, G, d, dtype, caps, planes)
    for name in ("k", "v", "mass", "pos"):
        getattr(cache, name).copy_(getattr(c, name))
    cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return cache, c


def rows(G, H, d, new, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(*s, generator=g).to(dtype) for s in ((G, new, d), (G, new, d), (new, H, d)))


def same_slots(cache, c, b, n):
    used = slice(c.cu[b], c.cu[b] + n)
    for name in ("k", "v", "mass", "pos"):
        assert torch.equal(getattr(cache, name)[:, used].cpu(), getattr(c, name)[:, used]), name


@pytest.mark.parametrize("dtype,d,G,H,T", [(torch.bfloat16, 128, 2, 8, 4), (torch.bfloat16, 128, 32, 128, 40), (torch.float32, 64, 2, 4, 4),
                                           (torch.bfloat16, 80, 2, 4, 7)])
def test_drafts_that_do_not_fit(B, dtype, d, G, H, T):  # noqa: F811
    """append, attend, accept in a row: the sequence without room loses nothing, its rows see nothing, its neighbour is what it is by itself."""
    cache, c = full_cache(dtype, d, G, H, 1, [1300, 1400], [1298, 1200], 7)
    cu_new, masks = [0, T, 2 * T], R.random_tree(T, np.random.default_rng(1)) + R.random_tree(T, np.random.default_rng(2))
    k, v, q = rows(G, H, d, 2 * T, dtype, 8)
    tree, path = R.as_int64(masks).cuda(), torch.zeros(2 * T, dtype=torch.int32, device="cuda")
    cache.append(k.cuda(), v.cuda(), cu_new, torch.arange(2 * T, device="cuda").int() + 9000)
    out, lse = cache.attend(q.cuda(), cu_new, tree)
    cache.accept(cu_new, path, torch.tensor([1, 1], dtype=torch.int32, device="cuda"), q.cuda(), lse, tree, 0.9)
    assert cache.lens.tolist() == [1298, 1201]
    same_slots(cache, c, 0, 1298)
    assert torch.all(out[:T] == 0) and torch.all(lse[:T] == -math.inf)
    assert cache.missed.tolist() == [1, 0]
    c.k[:, c.cu[1] + 1200: c.cu[1] + 1200 + T], c.v[:, c.cu[1] + 1200: c.cu[1] + 1200 + T] = k[:, T:], v[:, T:]
    c.lens = [0, 1200 + T]
    ref, ref_lse, _, size = R.attend(c, H, q, cu_new, masks)
    within(out[T:].cpu().double(), ref[T:], EPS[dtype] * ref[T:].abs() + 1e-4 * size[T:], "out")
    within(lse[T:].cpu().double(), ref_lse[T:], torch.tensor(1e-4), "lse")
    # with room made and the mark taken away, the rows come in
    cache.evict([1000, 1400], 8)
    cache.missed.zero_()
    cache.append(k[:, :T].contiguous().cuda(), v[:, :T].contiguous().cuda(), [0, T, T], torch.arange(T, device="cuda").int() + 9000)
    out, lse = cache.attend(q[:T].cuda(), [0, T, T], tree[:T])
    cache.accept([0, T, T], None, None, q[:T].cuda(), lse, tree[:T], 0.9)
    assert cache.lens.tolist() == [1000 + T, 1201] and cache.missed.tolist() == [0, 0] and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype,d,planes", [(torch.bfloat16, 128, 2), (torch.float32, 64, 1)])
def test_tokens_that_do_not_fit_in_a_replayed_step(B, dtype, d, planes):  # noqa: F811
    """Steps captured once and replayed past the capacity of one sequence: it stops as it is, the other goes on."""
    G, H = 2, 8
    cache, c = full_cache(dtype, d, G, H, planes, [300, 400], [296, 200], 9)
    k, v, q = (x.cuda() for x in rows(G, H, d, 2, dtype, 10))
    pos, results = torch.full((2,), 9000, dtype=torch.int32, device="cuda"), []

    def step():
        cache.append(k, v, [0, 1, 2], pos)
        results[:] = cache.attend(q, [0, 1, 2], lam=0.9)
        cache.append(k, v, [0, 1, 2], pos)
        results.extend(cache.attend(q, [0, 1, 2], lam=0.9))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    torch.cuda.synchronize()
    assert cache.lens.tolist() == [300, 204] and cache.missed.tolist() == [0, 0]
    before = {name: getattr(cache, name).clone() for name in ("k", "v", "mass", "pos")}
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert cache.lens.tolist() == [300, 206 + 2 * i] and cache.missed.tolist() == [1, 0]
        for name, x in before.items():
            assert torch.equal(getattr(cache, name)[:, :300], x[:, :300]), name
        for out, lse in (results[:2], results[2:]):
            assert torch.all(out[0] == 0) and torch.all(lse[0] == -math.inf) and torch.isfinite(lse[1]).all() and torch.any(out[1] != 0)
    assert not torch.equal(cache.mass[:, 300:500], before["mass"][:, 300:500])
    cache.reset()
    assert cache.lens.tolist() == [0, 0] and cache.missed.tolist() == [0, 0]


@pytest.mark.parametrize("dtype,d,H", [(torch.bfloat16, 128, 8), (torch.bfloat16, 64, 40), (torch.float32, 64, 8), (torch.bfloat16, 80, 4)])
@pytest.mark.parametrize("planes", [1, 2])
def test_accepted_rows_whose_norm_is_not_a_number(B, dtype, d, H, planes):  # noqa: F811
    """Their weights are not numbers either: so is the mass of what they see, in the planes of their heads; all else is as without them."""
    T, lens, masks = 8, [300, 9], [0b1, 0b11, 0b100, 0b1001, 0b10010, 0b100101, 0b1001011, 0b10000000]
    c = R.make_cache(2, d, planes, [310, 9], lens, dtype, 21)
    k, v, q = rows(2, H, d, 2 * T, dtype, 22)
    lse = R.attend(c, H, q, [0, T, 2 * T], masks * 2)[1].float()
    lse[1, 0], lse[T + 3, H - 1], lse[2] = math.nan, math.nan, math.nan     # (the last one's token is not accepted)
    path = torch.tensor([1, 4, 0, 0, 0, 0, 0, 0] + [0, 3, 7, 0, 0, 0, 0, 0], dtype=torch.int32)
    n_accept = [2, 3]
    cuda = {name: getattr(c, name).cuda() for name in ("k", "v", "mass", "pos")}
    lens_in, lens_out = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    handle = B.make_cache(cuda["k"], cuda["v"], c.cu, lens_in, cuda["mass"], cuda["pos"])
    B.structkv_cache_accept(handle, H, q.cuda(), lse.cuda(), [0, T, 2 * T], lens_out, path.cuda(), torch.tensor(n_accept, dtype=torch.int32).cuda(),
                            R.as_int64(masks * 2).cuda(), lam=0.9)
    norms = lse.nan_to_num(-math.inf, neginf=-math.inf)                     # (rows without a norm add nothing)
    *_, mass, new_lens = R.accept(c, H, q, norms, [0, T, 2 * T], path, n_accept, masks * 2, lam=0.9)
    odd = torch.zeros(c.mass.shape, dtype=torch.bool)
    for b, t, h in ((0, 1, 0), (1, 3, H - 1)):
        plane = h // (H // 2) if planes > 1 else 0
        odd[plane, [c.cu[b] + s for s in R.visible(lens[b], lens[b] - T, t, masks)]] = True
    for b in range(2):
        first, steps = c.cu[b] + lens[b] - T, path[T * b:T * b + n_accept[b]].long()
        odd[:, first:first + n_accept[b]] = odd[:, first + steps].clone()
    got = cuda["mass"].cpu().double()
    assert lens_out.tolist() == new_lens and odd.any() and not odd.all()
    assert torch.equal(torch.isnan(got), odd)
    within(got[~odd], mass[~odd], 1e-4 * mass[~odd].abs(), "mass")


def lone_scores(H, G, d, T, batch, dtype, softcap, seed):
    """Drafts that see themselves alone, with one component that counts: each row's score is one exact product, from far below the cap to beyond."""
    g = torch.Generator().manual_seed(seed)
    c = R.make_cache(G, d, G, [T + 3] * batch, [T] * batch, dtype, seed)
    q = torch.zeros(batch * T, H, d, dtype=dtype)
    used = torch.cat([torch.arange(T) + (T + 3) * b for b in range(batch)])
    c.k[:, used] = 0
    c.k[:, used, 0] = torch.exp2(8 * torch.rand(G, batch * T, generator=g) - 4).to(dtype)
    q[:, :, 0] = (softcap * torch.exp2(8 * torch.rand(batch * T, H, generator=g) - 7) * torch.randn(batch * T, H, generator=g).sign()).to(dtype)
    masks = [1 << t for t in range(T)] * batch
    y = q[:, :, 0].double() * c.k[:, used, 0].double().T.repeat_interleave(H // G, 1)      # [row, head]
    return c, q, masks, y, used


# (the bf16 matrix kernels of 16, 32 and 128 rows, the fp32 one)
CAPPED = [(torch.bfloat16, 128, 2, 8, 2, 3), (torch.bfloat16, 64, 2, 8, 8, 3), (torch.bfloat16, 128, 64, 128, 40, 9), (torch.float32, 64, 2, 8, 40, 2),
          (torch.bfloat16, 80, 2, 4, 40, 2)]


@pytest.mark.parametrize("dtype,d,G,H,T,batch", CAPPED)
@pytest.mark.parametrize("softcap", [5.0, 30.0, 50.0, 256.0, 1000.0])
@pytest.mark.parametrize("slopes", [False, True])
def test_capped_scores_to_their_last_bits(B, dtype, d, G, H, T, batch, softcap, slopes):  # noqa: F811
    """lse of a row that sees one slot is its score c tanh(y / c), y an exact product (fp32 keys: one rounding).  In halves of an ulp, 2^-24 of the
    result: near zero y and u = y / c have four roundings (u's count 2 w |P| < 1/4 each), the polynomial's fit 0.6 and its sum and last product 2;
    beyond, e has its argument's four roundings and the exponential's own ulp, each counting at most 2 |u| 2 e / (1 - e^2) < 0.8, 1 - e, 1 + e and the
    products 4, the reciprocal's ulp 2, the cap's constants 2; then the change to log2 and back 4 in either.  16 cover both."""
    c, q, masks, y, used = lone_scores(H, G, d, T, batch, dtype, softcap, 31)
    cu_new = [T * b for b in range(batch + 1)]
    slope = torch.zeros(H) if slopes else None          # (distances of zero: the form with a bias)
    cuda = {name: getattr(c, name).cuda() for name in ("k", "v", "mass", "pos")}
    lens, lens_out = (torch.tensor(c.lens, dtype=torch.int32, device="cuda") for _ in range(2))
    handle = B.make_cache(cuda["k"], cuda["v"], c.cu, lens, cuda["mass"], cuda["pos"])
    out, lse = torch.empty(batch * T, H, d, dtype=dtype, device="cuda"), torch.empty(batch * T, H, device="cuda")
    ws = torch.empty(B.structkv_cache_workspace_bytes(handle, H, batch * T), dtype=torch.uint8, device="cuda")
    form = dict(tree_mask=R.as_int64(masks).cuda(), scale=1.0, softcap=softcap, slopes=None if slope is None else slope.cuda())
    B.structkv_cache_attend(handle, H, q.cuda(), cu_new, out, lse, ws, **form)
    x = softcap * torch.tanh(y / softcap)
    within(lse.cpu().double(), x, 16 * 2.0 ** -24 * x.abs(), "lse")
    # the weights of accepted drafts, against norms that they nearly equal: e^(x - lse), off by what x is, by the norm's two roundings and by a few more
    norms = x.float()
    cuda["mass"].zero_()
    B.structkv_cache_accept(handle, H, q.cuda(), norms.cuda(), cu_new, lens_out, lam=1.0, **form)
    weights = torch.exp(x - norms.double()).view(batch * T, G, H // G)
    error = ((16 + 4) * 2.0 ** -24 * x.abs() + 8 * 2.0 ** -24).view(weights.shape)
    within(cuda["mass"][:, used].cpu().double(), weights.sum(2).T, (weights * error).sum(2).T + H // G * 2.0 ** -24 * weights.sum(2).T, "mass")


@pytest.mark.parametrize("softcap", [256.0, 300.0, 1000.0])
@pytest.mark.parametrize("d", [128, 64])
def test_large_caps_without_a_bias(B, softcap, d):  # noqa: F811
    """Caps from 256 on over whole caches: 16, 32 and 128 rows a workgroup, gathered weights, accepted drafts."""
    from test_gpu_cache import check_accept, check_attend
    c = R.make_cache(2, d, 2, [300, 90], [280, 90], torch.bfloat16, 33)
    c.k *= 8
    check_attend(B, c, 6, [1, 1], softcap=softcap, lam=0.9, seed=33)
    check_attend(B, c, 6, [5, 9], tree=True, softcap=softcap, seed=34)
    check_accept(B, c, 6, [9, 64], [[0, 3, 8], list(range(1, 64))], softcap=softcap, lam=0.5, seed=35)
    c = R.make_cache(16, d, 16, [1400, 70, 901, 2100, 40], [1391, 70, 17, 2099, 33], torch.bfloat16, 36)
    c.k *= 8
    check_attend(B, c, 48, [64, 0, 20, 33, 33], tree=True, softcap=softcap, seed=36)


@pytest.mark.parametrize("dtype,d,G,H,T", [(torch.bfloat16, 128, 2, 8, 1), (torch.bfloat16, 64, 2, 8, 7), (torch.bfloat16, 128, 32, 128, 40),
                                           (torch.float32, 64, 2, 8, 7), (torch.bfloat16, 80, 2, 4, 1)])
@pytest.mark.parametrize("score", [-2.0 ** 40, 2.0 ** 40, -2.0 ** 90, -2.0 ** 110, 2.0 ** 110, -2.0 ** 125])
def test_scores_far_from_zero(B, dtype, d, G, H, T, score):  # noqa: F811
    """A row whose scores are huge attends to the highest: one slot's value as it is, lse its score (to log2 and back), mass of one."""
    n, best = [1300, 700], [777, 0]
    c = R.make_cache(G, d, 1, n, n, dtype, 41)
    c.k[:] = 0
    small, large = math.copysign(1.1171875, score), math.copysign(2.0, score)       # (products that c2 does not divide evenly)
    c.k[:, :, 0] = large if score < 0 else small
    for b in range(2):
        c.k[:, c.cu[b] + best[b], 0] = small if score < 0 else large
    q = torch.zeros(2 * T, H, d, dtype=dtype)
    q[:, :, 0] = 1.2890625 * abs(score)
    score = 1.2890625 * abs(score) * (small if score < 0 else large)
    cuda = {name: getattr(c, name).cuda() for name in ("k", "v", "mass", "pos")}
    handle = B.make_cache(cuda["k"], cuda["v"], c.cu, torch.tensor(n, dtype=torch.int32, device="cuda"), cuda["mass"], cuda["pos"])
    out, lse = torch.empty(2 * T, H, d, dtype=dtype, device="cuda"), torch.empty(2 * T, H, device="cuda")
    ws = torch.empty(B.structkv_cache_workspace_bytes(handle, H, 2 * T), dtype=torch.uint8, device="cuda")
    B.structkv_cache_attend(handle, H, q.cuda(), [0, T, 2 * T], out, lse, ws, scale=1.0, lam=0.5 if T == 1 else 0.0)
    for b in range(2):
        v = c.v[:, c.cu[b] + best[b]].repeat_interleave(H // G, 0)
        assert torch.equal(out[b * T:(b + 1) * T].cpu(), v.expand(T, H, d))
    assert torch.all((lse.double() / score - 1).abs() <= 6 * 2.0 ** -24)
    if T == 1:
        mass = c.mass * 0.5
        mass[0, [c.cu[b] + best[b] for b in range(2)]] += H
        assert torch.equal(cuda["mass"].cpu(), mass)


def test_layers_that_share_a_workspace(B):  # noqa: F811
    """Two layers' caches, one behind the other on one stream, as with workspaces of their own; a workspace that is too small is refused."""
    from paper_2604_06746_amd.cache import LayerCache
    H, G, d, dtype, caps = 8, 2, 128, torch.bfloat16, [5000, 300]
    layers = [LayerCache(H, G, d, dtype, caps, max_new=8) for _ in range(2)]
    shared = [LayerCache(H, G, d, dtype, caps, max_new=8)]
    shared.append(LayerCache(H, G, d, dtype, caps, max_new=4, workspace=shared[0].workspace))
    assert shared[1].workspace is shared[0].workspace
    g = torch.Generator(device="cuda").manual_seed(51)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    k, v = normal(2, 2, G, 4800, d)
    for i in range(2):
        for cache in (layers[i], shared[i]):
            cache.append(k[i], v[i], [0, 4600, 4800], torch.arange(4800, device="cuda").int())
    for step in range(3):
        q, k1, v1 = normal(2, 2, H, d), normal(2, G, 2, d), normal(2, G, 2, d)
        for i in range(2):
            got = []
            for cache in (layers[i], shared[i]):
                cache.append(k1[i], v1[i], [0, 1, 2], torch.full((2,), 5000 + step, dtype=torch.int32, device="cuda"))
                got.append(cache.attend(q[i], [0, 1, 2], lam=0.9))
                cache.evict([4500, 200], 8)
            assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    for i in range(2):
        assert torch.equal(layers[i].mass, shared[i].mass) and layers[i].lens.tolist() == shared[i].lens.tolist() == [4500, 200]
    with pytest.raises(B.StructKVError):
        LayerCache(H, G, d, dtype, [5000] * 9, workspace=shared[0].workspace)
    with pytest.raises(B.StructKVError):
        LayerCache(H, G, d, dtype, [100], workspace=torch.empty(1 << 28, dtype=torch.uint8))


@pytest.mark.parametrize("dtype,G,H,planes,caps,lens", [(torch.bfloat16, 2, 32, 1, [70000, 70001, 40], [1999, 4097, 33]),
                                                       (torch.bfloat16, 1, 16, 1, [300000, 230000], [3001, 770]),
                                                       (torch.float32, 2, 36, 1, [140000, 64], [2050, 1]),
                                                       (torch.bfloat16, 8, 8, 8, [66000, 100], [2001, 98])])
def test_weights_gathered_four_slots_a_thread(B, dtype, G, H, planes, caps, lens):  # noqa: F811
    """Room for so many slots that the join takes four a thread, by waves that share a plane's heads and by threads that have all of them; lengths
    that are no multiple of four."""
    from test_gpu_cache import check_attend
    check_attend(B, R.make_cache(G, 64, planes, caps, lens, dtype, 61), H, [1] * len(caps), lam=0.9, seed=61)


def test_bf16_of_256_components(B):  # noqa: F811
    """Single tokens, trees, caps and biases, accepted drafts (fp32 matrix instructions on widened values)."""
    from test_gpu_cache import check_accept, check_attend
    c = R.make_cache(2, 256, 2, [300, 90, 5], [280, 90, 1], torch.bfloat16, 62)
    check_attend(B, c, 8, [1, 1, 1], lam=0.9, seed=62)
    check_attend(B, c, 8, [13, 64, 1], tree=True, softcap=30.0, slopes=True, seed=63)
    check_attend(B, c, 2, [5, 0, 1], layout="odd", softcap=50.0, seed=64)
    check_accept(B, c, 8, [13, 64, 1], [[0, 4, 7], list(range(30)), [0]], softcap=30.0, lam=0.9, seed=65)
    check_accept(B, c, 8, [13, 64, 1], [[12], [], [0]], slopes=True, lam=0.9, layout="slots", seed=66)


@pytest.mark.parametrize("dtype,d,planes", [(torch.bfloat16, 128, 2), (torch.float32, 33, 1)])
def test_copies_of_many_sequences(B, dtype, d, planes):  # noqa: F811
    """More sequences than the small table holds, each call with lengths out of bounds among them."""
    from test_gpu_cache import OnGpu, check_accept, check_evict
    rng, n = np.random.default_rng(7), 37
    caps = [int(x) for x in rng.integers(0, 90, n)]
    lens = [int(rng.integers(0, x + 1)) for x in caps]
    lens[3], lens[5], lens[9] = -7, caps[5] + 40, caps[9]
    c = R.make_cache(2, d, planes, caps, lens, dtype, 67)
    fresh = [int(x) for x in rng.integers(0, 30, n)]
    cu_new, g = R.cut(fresh), torch.Generator().manual_seed(68)
    k_new, v_new = (torch.randn(2, cu_new[-1], d, generator=g).to(dtype) for _ in range(2))
    pos_new, mass_new = torch.randint(0, 999, (planes, cu_new[-1]), generator=g).int(), torch.rand(planes, cu_new[-1], generator=g)
    on = OnGpu(B, c)
    B.structkv_cache_append(on.handle, k_new.cuda(), v_new.cuda(), cu_new, on.lens_out, pos_new=pos_new.cuda(), mass_new=mass_new.cuda())
    on.same(*R.append(c, k_new, v_new, cu_new, pos_new, mass_new))
    check_evict(B, c, c.mass, [int(x) for x in rng.integers(0, 60, n)], 9)
    paths = [rng.integers(0, max(T, 1), int(rng.integers(0, T + 1))).tolist() for T in fresh]
    check_accept(B, c, 4, fresh, paths, lam=0.9, seed=69)
