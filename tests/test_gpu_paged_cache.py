"""A layer's cache in pages behind a sweep: the prefill's selection goes in, tokens are generated, pages of least mass are dropped and given back,
a sequence ends and another takes its place.  Tolerances as in test_gpu_paged.py."""
import math

import pytest
import torch

import paged_reference as R
from test_gpu_paged import cut, within

pytestmark = pytest.mark.gpu


def as_pool(cache):
    """The cache as it is, for the definitions."""
    import types
    c = types.SimpleNamespace(G=cache.G, d=cache.d, ps=cache.page_size, n_pages=cache.n_pages, dtype=cache.dtype, lens=cache.lens.tolist())
    c.k, c.v = (x.view(torch.uint8).cpu() for x in (cache.k, cache.v))
    c.ks, c.vs, c.mass, c.pages = cache.k_scale.cpu(), cache.v_scale.cpu(), cache.mass.cpu(), cache.pages.cpu()
    return c


def check_step(cache, q, cu, lam):
    c = as_pool(cache)
    out, lse = cache.attend(q, cu, lam=lam)
    ref, ref_lse, ref_mass, size, top = R.attend(c, cache.Hq, q.cpu(), cu, lam=lam)
    keys = (R.decode(c.k).nan_to_num(0.0) * c.ks[:, :, None, None]).norm(dim=3).max()
    x_max = float(ref_lse.abs().max()) + 16
    delta = float(c.d * keys * q.double().norm(dim=2).max() / math.sqrt(c.d) + 8 * x_max) * 2.0 ** -24
    a_err = 2 * delta + (max(c.lens) / 16 + 64) * 2.0 ** -24
    within(lse.cpu().double(), ref_lse, a_err + 2.0 ** -23 * ref_lse.abs(), "lse")
    within(out.cpu().double(), ref, 2.0 ** -8 * ref.abs() + (2 * a_err + 2.0 ** -11) * size + max(c.lens) * 2.0 ** -31 * top, "out")
    within(cache.mass.cpu().double(), ref_mass, (2.0 ** -22 + 2 * a_err + 2.0 ** -22 * x_max) * ref_mass.abs(), "mass")
    return out


def test_generation_behind_a_sweep():
    from paper_2604_06746_amd import binding as B, sweep
    from paper_2604_06746_amd.paged import PagedCache
    H, G, d, w, n, keep = 8, 2, 64, 16, 700, 200
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    turns, _ = B.structkv_rotary_turns(d, 500000.0)
    plan = B.make_rotary(turns.cuda())
    # a prefill: queries and keys rotated, the layer scored, the compact cache of its selection stored in pages
    q, k, v = normal(n, H, d), normal(n, G, d), normal(G, n, d)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    B.structkv_rotate(plan, q, pos, q)
    turned = torch.empty(G, n, d, dtype=torch.bfloat16, device="cuda")
    B.structkv_rotate(plan, k, pos, turned.transpose(0, 1))
    sw = sweep.LayerSweep(H, G, d, w, torch.bfloat16, [n], [keep])
    sw.layer(q[-w:].transpose(0, 1).contiguous()[None], turned, v)
    rows = sw.rows
    cache = PagedCache(H, G, d, torch.bfloat16, n_pages=40, page_size=16, batch=2, max_pages=30)
    cache.reserve(0, rows + 40)
    cache.append(sw.k_cache[0][:, :rows], sw.v_cache[0][:, :rows], [0, rows, rows])
    assert cache.lens.tolist() == [rows, 0] and not cache.missed.any()
    c = as_pool(cache)
    for name, x, scales in (("k", sw.k_cache[0], c.ks), ("v", sw.v_cache[0], c.vs)):
        for s in (0, 17, rows - 1):
            p = int(c.pages[0, s // 16])
            got = R.decode(getattr(c, name)[p, :, s % 16]) * scales[p].double()[:, None]
            want = x[:, s].double().cpu()
            assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * scales[p].double()[:, None]).all())
    # generation; the compact cache's tokens stand at their positions of the prompt, the new ones behind it
    for step in range(6):
        q, k, v = normal(1, H, d), normal(G, 1, d), normal(G, 1, d)
        q = cache.append(k, v, [0, 1, 1], plan, pos_new=torch.tensor([n + step], dtype=torch.int32, device="cuda"), q=q)
        check_step(cache, q, [0, 1, 1], 0.9)
    # the four pages of least mass go, none of the last two; a second sequence takes two of them
    used = -(-(rows + 6) // 16)
    free = cache.free_pages
    cache.drop(0, cache.mass[0, :used - 2].argsort()[:4].tolist())
    assert cache.free_pages == free + 4 and int((cache.pages[0] >= 0).sum()) == -(-(rows + 40) // 16) - 4
    cache.reserve(1, 30)
    for step in range(3):
        fresh = [1, 20 if step == 0 else 1]
        cu = cut(fresh)
        q, k, v = normal(cu[-1], H, d), normal(G, cu[-1], d), normal(G, cu[-1], d)
        at = torch.tensor([n + 6 + step] + list(range(cache.lens.tolist()[1], cache.lens.tolist()[1] + fresh[1])), dtype=torch.int32, device="cuda")
        q = cache.append(k, v, cu, plan, pos_new=at, q=q)
        if step:
            check_step(cache, q, cu, 0.9)
    assert cache.lens.tolist() == [rows + 9, 22] and not cache.missed.any()
    # the first ends; what it had goes to the second, which grows past what it had reserved first
    cache.release(0)
    assert cache.lens.tolist() == [0, 22] and cache.free_pages == 40 - 2
    q, k, v = normal(20, H, d), normal(G, 20, d), normal(G, 20, d)
    cache.append(k, v, [0, 0, 20], plan)
    assert cache.missed.tolist() == [0, 1] and cache.lens.tolist() == [0, 22]
    cache.missed.zero_()
    cache.reserve(1, 42)
    q = cache.append(k, v, [0, 0, 20], plan, q=q)
    assert cache.lens.tolist() == [0, 42] and not cache.missed.any()


def test_pages_are_given_out_once():
    from paper_2604_06746_amd import binding as B
    from paper_2604_06746_amd.paged import PagedCache
    cache = PagedCache(4, 2, 64, torch.float32, n_pages=10, page_size=32, batch=3, max_pages=6)
    for b, tokens in ((0, 1), (1, 100), (0, 64), (2, 65), (0, 64)):
        cache.reserve(b, tokens)
    table = cache.pages.cpu()
    ids = table[table >= 0].tolist()
    assert len(ids) == len(set(ids)) == 9 and cache.free_pages == 1
    for bad in ((2, 200), (0, 1000)):
        with pytest.raises(B.StructKVError):
            cache.reserve(*bad)
    assert cache.free_pages == 1 and torch.equal(cache.pages.cpu(), table)
    cache.drop(1, [0, 2])
    cache.drop(1, [0])
    assert cache.free_pages == 3 and cache.pages[1].tolist()[0] == -1
    with pytest.raises(B.StructKVError):
        cache.drop(1, [4])
    cache.release(1)
    assert cache.free_pages == 5 and cache.pages[1].tolist() == [-1] * 6
    other = PagedCache(4, 2, 64, torch.float32, n_pages=4, page_size=32, batch=3, max_pages=6, workspace=cache.workspace)
    assert other.workspace is cache.workspace
    with pytest.raises(B.StructKVError):
        PagedCache(4, 2, 64, torch.float32, n_pages=4, page_size=32, batch=3, max_pages=1000, max_new=4000, workspace=cache.workspace)
    with pytest.raises(B.StructKVError):
        PagedCache(4, 2, 65, torch.float32, n_pages=4, page_size=32, batch=3, max_pages=6)
