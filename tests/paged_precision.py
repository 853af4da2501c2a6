"""What fp32 attention over pages may be off by as a whole, for tests of its precision (64 bits, CPU): a model of its roundings, and the results of
arithmetic with fewer bits, which such tests have to tell apart from it."""
import math

import torch

import paged_reference as R

# A rounding to fp32 is off by up to half a step: evenly spread over +- 2^-24 of a value's power of two, which is 0.58 of 2^-24 on the mean square
# and, as values lie evenly between powers of two, 0.42 2^-24 of the value.
ROUND = 0.42 * 2.0 ** -24


def attend(c, H, q, cu_new, scale, query_bits=24, weight_bits=None):
    """out, lse in 64 bits, and the root of the sum of squares of what each is off by (out_off [new, H], lse_off [new, H]) where every rounding is by
    itself.  query_bits, weight_bits: queries or weights rounded to so many bits first.
      score: 3 d sums (three parts of a query), partial results on the way to |q o k| as a random walk's, so sqrt(3 d / 2) roundings of that, and four of
             the score (its factor, the product, the exponent, the power of two)
      weight a: its score's, 2^-22 where it is cut into two parts, two roundings more;  lse: the weights' mean of these
      out: sum of (a (v - out)) squared times that, since the norm follows the weights, and the sums' roundings: sqrt(2 n / 2) of sum a |v|"""
    new, d = cu_new[-1], c.d
    out, lse = torch.zeros(new, H, d, dtype=torch.float64), torch.zeros(new, H, dtype=torch.float64)
    out_off, lse_off = torch.zeros(new, H, dtype=torch.float64), torch.zeros(new, H, dtype=torch.float64)
    for b in range(len(c.lens)):
        T, n = cu_new[b + 1] - cu_new[b], R.length(c, b)
        slots, pages, rows = R.seen_slots(c, b, n)
        for g in range(c.G):
            k = R.decode(c.k[pages, g, rows]) * c.ks[pages, g].double()[:, None]
            v = R.decode(c.v[pages, g, rows]) * c.vs[pages, g].double()[:, None]
            for h in range(g * (H // c.G), (g + 1) * (H // c.G)):
                for t in range(T):
                    r, m = cu_new[b] + t, sum(s <= n - T + t for s in slots)
                    x = k[:m] @ rounded(q[r, h].double(), query_bits) * scale
                    walk = ((k[:m] * q[r, h].double()) ** 2).sum(1).sqrt() * scale
                    a = torch.softmax(x, 0)
                    lse[r, h] = torch.logsumexp(x, 0)
                    w = a if weight_bits is None else rounded(a, weight_bits)
                    out[r, h] = w @ v[:m]
                    off = (ROUND * (math.sqrt(1.5 * d) * walk + 4 * x.abs())) ** 2 + 2.0 ** -44 + 2 * ROUND ** 2
                    shared = (a ** 2 * off).sum()
                    lse_off[r, h] = (shared + (2 * ROUND * (lse[r, h].abs() + 1)) ** 2).sqrt()
                    sums = (1.0 * m + 3) * ROUND ** 2 * ((a @ v[:m].abs()) ** 2).sum()
                    out_off[r, h] = (((a[:, None] * (v[:m] - out[r, h])) ** 2).sum(1) @ off + sums).sqrt()
    return out, lse, out_off, lse_off


def rounded(x, bits):
    """To `bits` significant bits, the nearest."""
    if bits >= 24:
        return x
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(torch.ldexp(m, torch.tensor(bits))), e - bits)


def case(d, lens=(500, 90), T=3, page_size=16, H=4, G=2, seed=11):
    """A pool, queries, and a scale that brings scores to a few units: (c, H, q, cu_new, scale)."""
    import numpy as np
    from test_gpu_paged import cut, table
    lens = list(lens)
    pages, n = table(lens, page_size, np.random.default_rng(seed))
    c = R.make_pool(G, d, page_size, n, pages, lens, torch.float32, seed)
    q = torch.randn(2 * T, H, d, generator=torch.Generator().manual_seed(seed))
    keys = (R.decode(c.k).nan_to_num(0.0) * c.ks[:, :, None, None]).norm(dim=3)
    return c, H, q, cut([T, T]), 2.0 / float(keys[keys > 0].square().mean().sqrt())


def worst(got, ref, off):
    """The whole tensor's norm of what it is off by, in units of the model's."""
    return float((got.double() - ref).norm() / off.norm())


# The model's units that a right result may take: its parts are no more than estimates (a weight's share of the roundings, scores that add up
# alike), good to a factor of two.
MOST = 2.0
# The share of bf16 results whose last bit may be another than the exact one's.
TURNED = 0.01
