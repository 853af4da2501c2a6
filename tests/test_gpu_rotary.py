"""GPU parity of rotary positions with their 64-bit definition.

Tolerance.  An angle is off by 2^-32 of a turn (the bits below are left out, and its conversion to fp32 keeps 24 of the rest), 2 pi 2^-32 <
2^-29, plus 2^-24 of pi / 4; cosine and sine by that, a few roundings of their series and their product with the magnitude: 4 2^-24 in all.
y = a cos - b sin rounds each product and the sum: (|a| + |b|) m (4 + 2) 2^-24, and the result to its type once, 2^-8 of it in bf16 and 2^-24 in
fp32."""
import math

import pytest
import torch

import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06746_amd import binding
    return binding


EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def rows(tokens, heads, d, dtype, seed, layout="tokens"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, heads, d, generator=g).to(dtype)
    return x, place(x, layout)


def place(x, layout):
    tokens, heads, d = x.shape
    if layout == "tokens":
        return x.cuda()
    if layout == "heads":
        return x.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    room = torch.zeros(tokens, heads + 2, d + (16 if layout == "part" else 3), dtype=x.dtype, device="cuda")   # part of a projection; or odd places
    room[:, 1:1 + heads, -d:] = x.cuda()
    return room[:, 1:1 + heads, -d:]


def tolerance(x, ref, half, interleaved, magnitude, dtype):
    tol = EPS[dtype] * ref.abs()
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    size = (x[..., first].double().abs() + x[..., second].double().abs()) * abs(magnitude) * 6 * 2.0 ** -24 * (1 + EPS[dtype])
    tol[..., first] += size
    tol[..., second] += size
    tol[..., 2 * half:] = 0.0
    return tol


def check(B, x, x_gpu, pos, rot, interleaved=False, magnitude=1.0, inverse=False, scaling=("none",), out=None):
    turns, m = B.structkv_rotary_turns(rot, 500000.0, *scaling)
    magnitude = magnitude * m
    plan = B.make_rotary(turns.cuda(), interleaved=interleaved, magnitude=magnitude)
    out = torch.full_like(x_gpu, math.nan) if out is None else out
    B.structkv_rotate(plan, x_gpu, torch.tensor(pos, dtype=torch.int32).cuda(), out, inverse=inverse)
    ref = R.rotated(x, pos, R.turns_of(turns), interleaved, magnitude, inverse)
    tol = tolerance(x, ref, rot // 2, interleaved, magnitude, x.dtype)
    off = (out.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp(min=1e-30)).max())
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 64), (128, 64), (80, 20), (256, 256), (33, 10), (2, 2), (96, 6), (16, 14), (128, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_and_layouts(B, dtype, d, rot, interleaved):
    for tokens, heads, layout in ((1, 1, "tokens"), (37, 5, "tokens"), (70, 3, "heads"), (9, 4, "part"), (9, 4, "odd")):
        x, x_gpu = rows(tokens, heads, d, dtype, tokens + d, layout)
        check(B, x, x_gpu, list(range(tokens)), rot, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(B, interleaved):
    pos = [0, 1, -1, 1 << 20, (1 << 20) + 1, -(1 << 24) - 3, (1 << 31) - 1, -(1 << 31), 12345678, 777777777]
    x, x_gpu = rows(len(pos), 2, 128, torch.float32, 3)
    check(B, x, x_gpu, pos, 128, interleaved)


@pytest.mark.parametrize("scaling", [("linear", 4.0), ("ntk", 8.0), ("yarn", 8.0, 8192.0, 32.0, 1.0), ("bands", 8.0, 8192.0, 1.0, 4.0)])
@pytest.mark.parametrize("inverse", [False, True])
def test_scalings_and_magnitude(B, scaling, inverse):
    pos = [0, 5, 8191, 8192, 100000, 1 << 20]
    for dtype in (torch.bfloat16, torch.float32):
        x, x_gpu = rows(len(pos), 3, 128, dtype, 4)
        check(B, x, x_gpu, pos, 128, False, 1.25, inverse, scaling)


def test_many_rows(B):
    """More rows than one pass of the workgroups, heads shared out among threads."""
    x, x_gpu = rows(5000, 8, 64, torch.bfloat16, 5, "heads")
    check(B, x, x_gpu, list(range(100000, 105000)), 64)
    x, x_gpu = rows(3, 300, 128, torch.bfloat16, 6)
    check(B, x, x_gpu, [7, 0, 131071], 128)


def test_in_place_and_back(B):
    x, x_gpu = rows(50, 6, 128, torch.float32, 7)
    pos = [(i * 7919) % 131072 for i in range(50)]
    want = check(B, x, x_gpu, pos, 96)
    check(B, x, x_gpu, pos, 96, out=x_gpu)
    assert torch.equal(want, x_gpu)
    turns, _ = B.structkv_rotary_turns(96, 500000.0)
    B.structkv_rotate(B.make_rotary(turns.cuda()), x_gpu, torch.tensor(pos, dtype=torch.int32).cuda(), x_gpu, inverse=True)
    size = x.double().abs().amax(-1, keepdim=True)
    assert bool(((x_gpu.cpu().double() - x.double()).abs() <= 32 * 2.0 ** -24 * size).all())     # two turns of (|a| + |b|) 6 2^-24 and a rounding


def test_moved_by_a_distance(B):
    """Keys that were turned by p, turned by q - p more, are those turned by q."""
    x, x_gpu = rows(40, 2, 128, torch.float32, 8)
    p, q = [100000 + 3 * i for i in range(40)], [i for i in range(40)]
    there = check(B, x, x_gpu, p, 128)
    turns, _ = B.structkv_rotary_turns(128, 500000.0)
    B.structkv_rotate(B.make_rotary(turns.cuda()), there, torch.tensor([b - a for a, b in zip(p, q)], dtype=torch.int32).cuda(), there)
    want = R.rotated(x, q, R.turns_of(turns), False)
    size = x.double().abs().amax(-1, keepdim=True)
    assert bool(((there.cpu().double() - want).abs() <= 32 * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(B, interleaved):
    """Of sum(w . y): the formula's, and differences along random directions (the map is linear, so they are exact but for roundings)."""
    turns, _ = B.structkv_rotary_turns(20, 500000.0)
    plan = B.make_rotary(turns.cuda(), interleaved=interleaved, magnitude=1.5)
    pos = torch.tensor([3, 90000, 17], dtype=torch.int32).cuda()
    x, x_gpu = rows(3, 2, 80, torch.float32, 9)
    w, w_gpu = rows(3, 2, 80, torch.float32, 10)
    grad, up, down = (torch.empty_like(x_gpu) for _ in range(3))
    B.structkv_rotate(plan, w_gpu, pos, grad, inverse=True)
    y = x.double().requires_grad_()
    (R_rotated_with_grad(y, pos.tolist(), R.turns_of(turns), interleaved, 1.5) * w.double()).sum().backward()
    size = w.double().abs().amax(-1, keepdim=True) * 2 * 1.5
    assert bool(((grad.cpu().double() - y.grad).abs() <= 8 * 2.0 ** -24 * size).all())
    for seed in range(5):
        v, v_gpu = rows(3, 2, 80, torch.float32, 20 + seed)
        B.structkv_rotate(plan, x_gpu + v_gpu, pos, up)
        B.structkv_rotate(plan, x_gpu - v_gpu, pos, down)
        got = ((up - down).cpu().double() / 2 * w.double()).sum()
        want = (grad.cpu().double() * v.double()).sum()
        terms = (w.double().abs() * (x.double().abs() + v.double().abs()).amax(-1, keepdim=True) * 3).sum()
        assert abs(got - want) <= 16 * 2.0 ** -24 * terms


def R_rotated_with_grad(y, pos, turns, interleaved, magnitude):
    """The definition written with differentiable operations."""
    half = len(turns)
    angle = torch.tensor([[(t * p) % (1 << 64) / 2.0 ** 64 for t in turns] for p in pos], dtype=torch.float64) * (2 * math.pi)
    c, s = (magnitude * angle.cos())[:, None], (magnitude * angle.sin())[:, None]
    if interleaved:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        z = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        z = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([z, y[..., 2 * half:]], dim=-1)


def test_unturned_components_keep_their_bits(B):
    """NaN, infinities and signed zeros behind the turned part, also in a unit that holds both."""
    odd = torch.tensor([math.nan, math.inf, -math.inf, -0.0, 0.0, 1.0])
    for rot, d in ((10, 16), (2, 33), (64, 128)):
        for interleaved in (False, True):
            x = torch.randn(4, 2, d, generator=torch.Generator().manual_seed(1))
            x[..., rot:] = odd.repeat(-(-(d - rot) // 6))[:d - rot]
            turns, _ = B.structkv_rotary_turns(rot, 10000.0)
            out = torch.empty(4, 2, d, device="cuda")
            B.structkv_rotate(B.make_rotary(turns.cuda(), interleaved=interleaved), x.cuda(), torch.arange(4, dtype=torch.int32).cuda(), out)
            assert torch.equal(out[..., rot:].cpu().view(torch.int32), x[..., rot:].view(torch.int32))
            assert bool(out[..., :rot].isfinite().all())


def test_streams_and_graph(B):
    turns, _ = B.structkv_rotary_turns(128, 500000.0)
    plan = B.make_rotary(turns.cuda())
    x, x_gpu = rows(64, 4, 128, torch.bfloat16, 11)
    pos, out = torch.arange(64, dtype=torch.int32).cuda(), torch.empty_like(x_gpu)
    want = torch.empty_like(out)
    B.structkv_rotate(plan, x_gpu, pos, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.structkv_rotate(plan, x_gpu, pos, out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.structkv_rotate(plan, x_gpu, pos, out)
    for step in range(4):
        pos += 1000 * step
        x_gpu.mul_(-1)
        graph.replay()
        B.structkv_rotate(plan, x_gpu, pos, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(B):
    turns, _ = B.structkv_rotary_turns(64, 500000.0)
    plan = B.make_rotary(turns.cuda())
    x = torch.zeros(4, 2, 64, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(x=x.half(), out=x.half()), dict(out=x.bfloat16()), dict(out=x[:2]), dict(pos=pos[:3]), dict(pos=pos.long()), dict(pos=pos.cpu()), dict(x=x.cpu()),
                dict(x=torch.zeros(4, 2, 128, device="cuda")[..., ::2]), dict(x=torch.zeros(4, 2, 32, device="cuda"), out=torch.zeros(4, 2, 32, device="cuda")),
                dict(out=torch.zeros(1, 2, 64, device="cuda").expand(4, 2, 64))):
        with pytest.raises(B.StructKVError) as e:
            B.structkv_rotate(plan, bad.get("x", x), bad.get("pos", pos), bad.get("out", torch.empty_like(x)))
        assert e.value.status == B.STRUCTKV_ERR_INVALID_ARG
    B.structkv_rotate(plan, x[:0], pos[:0], x[:0])
    B.structkv_rotate(plan, x[:, :0], pos, x[:, :0])


@pytest.mark.parametrize("tokens,heads,d,dtype,interleaved", [(40000, 32, 128, torch.bfloat16, False), (40000, 32, 128, torch.bfloat16, True),
                                                              (150000, 8, 128, torch.bfloat16, False), (20000, 20, 128, torch.float32, False),
                                                              (30001, 19, 80, torch.bfloat16, False)])
def test_large_calls_like_small_ones(B, tokens, heads, d, dtype, interleaved):
    """Calls past the caches, of many heads a thread, against calls of 1000 tokens, bit for bit."""
    turns, _ = B.structkv_rotary_turns(d, 500000.0)
    plan = B.make_rotary(turns.cuda(), interleaved=interleaved)
    x = torch.randn(tokens, heads, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda") * 3
    large, small = torch.empty_like(x), torch.empty_like(x)
    B.structkv_rotate(plan, x, pos, large)
    for i in range(0, tokens, 1000):
        s = slice(i, min(tokens, i + 1000))
        B.structkv_rotate(plan, x[s], pos[s], small[s])
    assert torch.equal(large, small)
    if heads == 8:     # the same by head
        by_head = x.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.empty_like(by_head)
        B.structkv_rotate(plan, by_head, pos, out)
        assert torch.equal(out, large)
