"""Plain 64-bit definitions of rotary positions and of the operators on a cache held in 8 bits, in pages (CPU only)."""
import math
import types

import numpy as np
import torch

LEAST, MOST = 2.0 ** -64, 2.0 ** 64


def rotated(x, pos, turns, interleaved, magnitude=1.0, inverse=False):
    """x [tokens, heads, d] turned by pos [tokens], in 64 bits; turns: whole numbers, 2^64 a turn."""
    half = len(turns)
    angle = np.array([[(t * int(p)) % (1 << 64) / 2.0 ** 64 for t in turns] for p in pos]).reshape(len(pos), half) * (2.0 * math.pi)
    cos, sin = (torch.from_numpy(magnitude * f(angle))[:, None] for f in (np.cos, np.sin))
    sin = -sin if inverse else sin
    y = x.double().clone()
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    a, b = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y


def turns_of(bits):
    """int64 bits as whole numbers."""
    return [int(t) % (1 << 64) for t in bits.tolist()]


def decode(codes):
    """uint8 -> 64-bit values, from the format's definition."""
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 8 * 2.0 ** -6)
    return torch.where((c & 127) == 127, math.nan, torch.where(c > 127, -v, v))


_VALUES = decode(torch.arange(127, dtype=torch.uint8))


def encode(v):
    """64-bit values of magnitude up to 448 (NaN: 127) -> uint8, to the nearest, ties to the even code."""
    a = v.abs().nan_to_num(0.0)
    up = torch.searchsorted(_VALUES, a.contiguous()).clamp(max=126)
    down = (up - 1).clamp(min=0)
    far_up, far_down = _VALUES[up] - a, a - _VALUES[down]
    code = torch.where((far_down < far_up) | ((far_down == far_up) & (down % 2 == 0)), down, up)
    code = torch.where(v.isnan(), 127, code)
    return (code + 128 * (torch.signbit(v) & ~v.isnan())).to(torch.uint8)


def scale_for(a):
    """The least power of two s in [2^-64, 2^64] with a <= 448 s."""
    s = LEAST
    while s < MOST and a > 448.0 * s:
        s *= 2.0
    return s


def make_pool(G, d, page_size, n_pages, table, lens, dtype, seed, capacity=None):
    """Codes of normal numbers in units of each page's and head's scale, a sixteenth of the keys four times as long; rows that are not in
    use hold NaN.  table: lists of pages of each sequence (-1: dropped)."""
    g = torch.Generator().manual_seed(seed)
    most = max([len(t) for t in table], default=0) if capacity is None else capacity
    c = types.SimpleNamespace(G=G, d=d, ps=page_size, n_pages=n_pages, lens=list(lens), dtype=dtype)
    c.pages = torch.full((len(table), most), -1, dtype=torch.int32)
    for b, t in enumerate(table):
        c.pages[b, :len(t)] = torch.tensor(t, dtype=torch.int32)
    c.k, c.v = (encode((torch.randn(n_pages, G, page_size, d, generator=g) * 24.0).clamp(-448, 448).double()) for _ in range(2))
    hit = torch.rand(n_pages, page_size, generator=g) < 1 / 16
    k = decode(c.k)
    c.k = encode(torch.where(hit[:, None, :, None], (4 * k).clamp(-448, 448), k))
    c.ks, c.vs = (torch.exp2(torch.randint(-6, -3, (n_pages, G), generator=g).float()) for _ in range(2))
    c.mass = torch.rand(len(table), most, generator=g)
    used = torch.zeros(n_pages, page_size, dtype=torch.bool)
    for b, t in enumerate(table):
        for j, p in enumerate(t):
            if 0 <= p < n_pages:
                used[p, :max(0, min(page_size, lens[b] - j * page_size))] = True
    for x in (c.k, c.v):
        x.transpose(1, 2)[~used] = 127
    return c


def length(c, b):
    return max(0, min(c.lens[b], c.pages.shape[1] * c.ps))


def seen_slots(c, b, upto):
    """Slots below `upto` in pages of the pool, and their pages and rows."""
    s = [s for s in range(upto) if 0 <= int(c.pages[b, s // c.ps]) < c.n_pages]
    return s, [int(c.pages[b, x // c.ps]) for x in s], [x % c.ps for x in s]


def attend(c, H, q, cu_new, scale=0.0, softcap=0.0, lam=0.0):
    """out [new, H, d], lse [new, H], mass in 64 bits, and size [new, H, d] = sum of a |v|, top = largest |v|."""
    scale = scale or 1.0 / math.sqrt(c.d)
    new = cu_new[-1]
    out, size = torch.zeros(new, H, c.d, dtype=torch.float64), torch.zeros(new, H, c.d, dtype=torch.float64)
    lse, mass, top = torch.full((new, H), -math.inf, dtype=torch.float64), c.mass.double(), 0.0
    for b in range(len(c.lens)):
        T, n = cu_new[b + 1] - cu_new[b], length(c, b)
        if T == 0 or n < T:
            continue
        slots, pages, rows = seen_slots(c, b, n)
        slots = torch.tensor(slots, dtype=torch.long)
        weights = torch.zeros(n, dtype=torch.float64)
        for g in range(c.G if len(slots) else 0):
            k = decode(c.k[pages, g, rows]) * c.ks[pages, g].double()[:, None]
            v = decode(c.v[pages, g, rows]) * c.vs[pages, g].double()[:, None]
            top = max(top, float(v.abs().nan_to_num(0.0).max()))
            for h in range(g * (H // c.G), (g + 1) * (H // c.G)):
                for t in range(T):
                    see = slots <= n - T + t
                    if not see.any():
                        continue
                    x = k[see] @ q[cu_new[b] + t, h].double() * scale
                    if softcap:
                        x = softcap * torch.tanh(x / softcap)
                    a = torch.softmax(x, 0)
                    lse[cu_new[b] + t, h] = torch.logsumexp(x, 0)
                    out[cu_new[b] + t, h], size[cu_new[b] + t, h] = a @ v[see], a @ v[see].abs()
                    weights[slots[see]] += a
        if lam:
            used = -(-n // c.ps)
            mass[b, :used] *= lam
            mass[b, :used] += torch.nn.functional.pad(weights, (0, used * c.ps - n)).view(used, c.ps).sum(1)
    return out, lse, mass, size, top


def append(c, k_new, v_new, cu_new, pos=None, turns=None, interleaved=False, magnitude=1.0):
    """What the pool holds after the call, as a list of (tensor "k" or "v", page, KV head, first new row, 64-bit values of the new rows,
    the magnitude that the scale must cover, the earlier scale or None), and lens, missed.  Values that cannot be stored are NaN."""
    parts, lens, missed = [], list(c.lens), [0] * len(c.lens)
    for b in range(len(c.lens)):
        T, n = cu_new[b + 1] - cu_new[b], length(c, b)
        lens[b] = n
        if T == 0:
            continue
        entries = range(n // c.ps, (n + T - 1) // c.ps + 1)
        if n + T > c.pages.shape[1] * c.ps or any(not 0 <= int(c.pages[b, j]) < c.n_pages for j in entries):
            missed[b] = 1
            continue
        lens[b] = n + T
        at = [n + t if pos is None else int(pos[cu_new[b] + t]) for t in range(T)]
        rows = slice(cu_new[b], cu_new[b + 1])
        k, v = k_new[:, rows].double(), v_new[:, rows].double()
        if turns is not None:
            k = rotated(k.transpose(0, 1), at, turns, interleaved, magnitude).transpose(0, 1)
        for j in entries:
            first, last = max(n, j * c.ps), min(n + T, (j + 1) * c.ps)
            for name, x, scales in (("k", k, c.ks), ("v", v, c.vs)):
                for g in range(c.G):
                    new = x[g, first - n:last - n].clone()
                    new[~(new.abs() <= 448.0 * MOST)] = math.nan
                    page, row = int(c.pages[b, j]), first - j * c.ps
                    parts.append((name, page, g, row, new, float(new.abs().nan_to_num(0.0).max()),
                                  float(scales[page, g]) if row else None))
    return parts, lens, missed
