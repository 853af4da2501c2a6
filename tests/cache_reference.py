"""Plain 64-bit definitions of the operators on a cache in use, and the caches that their tests run on (CPU only).

A cache is a dict of CPU tensors: k, v [G, slots, d] and mass, pos [P, slots] as the library gets them, lens, cu_slots.  Slots
that are not in use hold NaN, and positions and masses that would show."""
import math
import types

import numpy as np
import torch


def make_cache(G, d, P, caps, lens, dtype, seed, hitters=True):
    """Keys and values N(0, 1), a sixteenth of the keys four times as long; positions ascending with gaps."""
    g = torch.Generator().manual_seed(seed)
    cu = [0]
    for n in caps:
        cu.append(cu[-1] + n)
    c = types.SimpleNamespace(G=G, d=d, P=P, cu=cu, lens=list(lens), dtype=dtype)
    c.k, c.v = (torch.randn(G, cu[-1], d, generator=g).to(dtype) for _ in range(2))
    if hitters:
        c.k[:, torch.rand(cu[-1], generator=g) < 1 / 16] *= 4
    c.mass = torch.rand(P, cu[-1], generator=g)
    c.pos = torch.randint(1, 5, (P, cu[-1]), generator=g).cumsum(1).int()
    for b in range(len(caps)):
        unused = slice(cu[b] + max(0, min(lens[b], caps[b])), cu[b + 1])
        c.k[:, unused] = math.nan
        c.v[:, unused] = math.nan
        c.mass[:, unused] = -7.0
    return c


def cut(lens_of_parts):
    cu = [0]
    for n in lens_of_parts:
        cu.append(cu[-1] + n)
    return cu


def random_tree(T, rng):
    """Bits that each of T drafts sees (its ancestors and itself, parents before children)."""
    masks = []
    for t in range(T):
        parent = rng.integers(-1, t) if t else -1
        masks.append((masks[parent] if parent >= 0 else 0) | 1 << t)
    return masks


def as_int64(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64)


def visible(n, base, t, masks):
    """Slots that fresh token t sees."""
    return [s for s in range(n) if s < base or (masks[t] >> (s - base) & 1 if masks is not None else s - base <= t)]


def scores(c, q, b, t, new0, h, H, scale, softcap, slopes, base, n):
    g = h // (H // c.G)
    x = c.k[g, c.cu[b]:c.cu[b] + n].double() @ q[new0 + t, h].double() * scale
    if softcap:
        x = softcap * torch.tanh(x / softcap)
    if slopes is not None:
        pos = c.pos[g if c.P > 1 else 0, c.cu[b]:c.cu[b] + n].double()
        x = x - float(slopes[h]) * (pos[base + t] - pos)
    return x


def attend(c, H, q, cu_new, masks=None, scale=0.0, softcap=0.0, slopes=None, lam=0.0):
    """out [new, H, d], lse [new, H], mass [P, slots] in 64 bits, and size [new, H, d] = sum of a |v|."""
    scale = scale or 1.0 / math.sqrt(c.d)
    new = cu_new[-1]
    out, size = torch.zeros(new, H, c.d, dtype=torch.float64), torch.zeros(new, H, c.d, dtype=torch.float64)
    lse, mass = torch.full((new, H), -math.inf, dtype=torch.float64), c.mass.double()
    for b in range(len(c.lens)):
        T, n = cu_new[b + 1] - cu_new[b], max(0, min(c.lens[b], c.cu[b + 1] - c.cu[b]))
        base = n - T
        if T == 0 or base < 0:
            continue
        weights = torch.zeros(c.G, n, dtype=torch.float64)
        for t in range(T):
            see = visible(n, base, t, masks[cu_new[b]:] if masks is not None else None)
            for h in range(H if see else 0):
                g = h // (H // c.G)
                x = scores(c, q, b, t, cu_new[b], h, H, scale, softcap, slopes, base, n)[see]
                a, v = torch.softmax(x, 0), c.v[g, c.cu[b]:c.cu[b] + n].double()[see]
                lse[cu_new[b] + t, h] = torch.logsumexp(x, 0)
                out[cu_new[b] + t, h], size[cu_new[b] + t, h] = a @ v, a @ v.abs()
                weights[g, see] += a
        if lam:
            mass[:, c.cu[b]:c.cu[b] + n] = lam * mass[:, c.cu[b]:c.cu[b] + n] + (weights if c.P > 1 else weights.sum(0, keepdim=True))
    return out, lse, mass, size


def accept(c, H, q, lse, cu_new, path=None, n_accept=None, masks=None, scale=0.0, softcap=0.0, slopes=None, lam=0.0):
    """k, v, pos, mass (64 bits), lens after the call."""
    scale = scale or 1.0 / math.sqrt(c.d)
    k, v, pos, mass, lens = c.k.clone(), c.v.clone(), c.pos.clone(), c.mass.double(), list(c.lens)
    for b in range(len(c.lens)):
        T, n = cu_new[b + 1] - cu_new[b], max(0, min(c.lens[b], c.cu[b + 1] - c.cu[b]))
        base, lens[b] = n - T, n
        if base < 0 or T == 0:
            continue
        taken = T if n_accept is None else max(0, min(int(n_accept[b]), T))
        steps = [i if path is None else max(0, min(int(path[cu_new[b] + i]), T - 1)) for i in range(taken)]
        if lam:
            weights = torch.zeros(c.G, n, dtype=torch.float64)
            for t in steps:
                see = visible(n, base, t, masks[cu_new[b]:] if masks is not None else None)
                for h in range(H):
                    norm = float(lse[cu_new[b] + t, h])
                    if see and norm > -math.inf:
                        x = scores(c, q, b, t, cu_new[b], h, H, scale, softcap, slopes, base, n)
                        weights[h // (H // c.G), see] += torch.exp(x[see] - norm)
            mass[:, c.cu[b]:c.cu[b] + n] = lam * mass[:, c.cu[b]:c.cu[b] + n] + (weights if c.P > 1 else weights.sum(0, keepdim=True))
        to, came = (torch.tensor([c.cu[b] + base + i for i in at], dtype=torch.long) for at in (range(taken), steps))
        for x in (k, v, pos, mass):
            x[:, to] = x[:, came].clone()
        lens[b] = base + taken
    return k, v, pos, mass, lens


def append(c, k_new, v_new, cu_new, pos_new=None, mass_new=None):
    """k, v, pos, mass, lens after the call; pos_new, mass_new [P, new]."""
    k, v, pos, mass, lens = c.k.clone(), c.v.clone(), c.pos.clone(), c.mass.clone(), list(c.lens)
    for b in range(len(c.lens)):
        T, cap = cu_new[b + 1] - cu_new[b], c.cu[b + 1] - c.cu[b]
        n = lens[b] = max(0, min(c.lens[b], cap))
        if n + T > cap:
            continue
        at, new = slice(c.cu[b] + n, c.cu[b] + n + T), slice(cu_new[b], cu_new[b + 1])
        k[:, at], v[:, at] = k_new[:, new], v_new[:, new]
        if pos_new is not None:
            pos[:, at] = pos_new[:, new]
        mass[:, at] = mass_new[:, new] if mass_new is not None else 0.0
        lens[b] = n + T
    return k, v, pos, mass, lens


def evict(c, scores, budget, tail):
    """k, v, pos, mass, lens after the call."""
    k, v, pos, mass, lens = c.k.clone(), c.v.clone(), c.pos.clone(), c.mass.clone(), list(c.lens)
    for b in range(len(c.lens)):
        n = lens[b] = max(0, min(c.lens[b], c.cu[b + 1] - c.cu[b]))
        if n <= budget[b]:
            continue
        lens[b] = budget[b]
        for p in range(c.P):
            sc, ps = scores[p, c.cu[b]:c.cu[b] + n].numpy(), c.pos[p, c.cu[b]:c.cu[b] + n].numpy().astype(np.int64)
            recent = ps > ps.max() - tail if tail else np.zeros(n, bool)
            order = sorted(range(n), key=lambda s: (not recent[s], 0.0 if recent[s] else -float(sc[s]), s))
            stay = set(order[:budget[b]])
            holes = [s for s in range(budget[b]) if s not in stay]
            moved = sorted(s for s in stay if s >= budget[b])
            assert len(holes) == len(moved)
            to, came = (torch.tensor([c.cu[b] + s for s in slots], dtype=torch.long) for slots in (holes, moved))
            heads = slice(p, p + 1) if c.P > 1 else slice(0, c.G)
            k[heads, to], v[heads, to] = c.k[heads, came], c.v[heads, came]
            pos[p, to], mass[p, to] = c.pos[p, came], c.mass[p, came]
    return k, v, pos, mass, lens
