"""Plain 64-bit definitions of rotary positions, the paged bf16 cache and attention over it, for the tests.  Nothing here calls the
library."""
import math

import torch


def frequencies(rot, base, scaling=None):
    """Radians per position of each pair and the amplitude, from the formulas, in Python floats."""
    f = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling is None:
        return f, 1.0
    factor = scaling[1]
    if scaling[0] == "linear":
        return [v / factor for v in f], 1.0
    if scaling[0] == "bands":
        _, _, low, high, original = scaling
        keep = [min(1.0, max(0.0, (original * v / (2 * math.pi) - low) / (high - low))) for v in f]
        amplitude = 1.0
    else:
        _, _, high, low, original = scaling
        at = lambda n: rot * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))
        a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
        keep = [1 - min(1.0, max(0.0, (i - a) / max(b - a, 0.001))) for i in range(rot // 2)]
        amplitude = 0.1 * math.log(factor) + 1 if factor > 1 else 1.0
    return [v * w + v / factor * (1 - w) for v, w in zip(f, keep)], amplitude


def rotate(x, positions, f, amplitude, rot, interleaved):
    """Rows [T, heads, D] in 64 bits, turned."""
    y = x.double().clone()
    t = positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
    c, s = (amplitude * t.cos())[:, None], (amplitude * t.sin())[:, None]
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    u, v = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    return y


def rotate_bound(x, y, amplitude, rot, interleaved):
    """How far a rotated bf16 row may be off y: half a step of bf16 for the rounding; in fp32 the argument of the cosine (half a
    turn or less, in units of half a turn, rounded from 32 bits: 2^-25 pi radians), the cosine and sine (2 units, 2^-22), the amplitude
    (its own rounding and its product, 2^-23) and the two products and their sum (3 * 2^-24), all relative to A (|u| + |v|).  The 64-bit
    side's angle, position * f rounded, is off by 2^-52 of at most 2^21 radians, far below."""
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    size = torch.zeros_like(y)
    both = abs(amplitude) * (x.double()[..., a].abs() + x.double()[..., b].abs())
    size[..., a], size[..., b] = both, both
    return 2.0 ** -8 * y.abs() * 1.001 + (math.pi * 2.0 ** -25 + 2.0 ** -22 + 2.0 ** -23 + 3 * 2.0 ** -24) * size + 1e-38


def rows_of(cache, table, n):
    """Keys or values [n, Hkv, D] of a request, by the documented order.  cache [pages, Hkv, page, D]."""
    page = cache.shape[2]
    j = torch.arange(n, device=cache.device)
    return cache[table[j // page].long(), :, j % page]


def attention(Q, k, v, Hq, scale, causal=True):
    """One request in 64 bits: Q [r, Hq * D], k and v [n, Hkv, D].  Returns O, sum of p |v|, and the size of the largest score's
    terms, sum |q| |k| * scale."""
    r, n = Q.shape[0], k.shape[0]
    D, Hkv = k.shape[2], k.shape[1]
    q = Q.double().view(r, Hkv, Hq // Hkv, D)
    O = torch.zeros(r, Hkv, Hq // Hkv, D, dtype=torch.float64, device=Q.device)
    A, E = torch.zeros_like(O), torch.zeros(r, Hkv, Hq // Hkv, 1, dtype=torch.float64, device=Q.device)
    if n > 0 and r > 0:
        seen = torch.arange(n, device=Q.device)[None] <= (torch.arange(r, device=Q.device)[:, None] + (n - r if causal else n))
        k, v = k.double(), v.double()
        s = torch.einsum("rghd,ngd->rghn", q, k) * scale
        s = torch.where(seen[:, None, None], s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
        O, A = torch.einsum("rghn,ngd->rghd", p, v), torch.einsum("rghn,ngd->rghd", p, v.abs())
        E = torch.einsum("rghd,ngd->rghn", q.abs(), k.abs()).amax(-1, keepdim=True) * abs(scale)
    flat = lambda t: t.expand(r, Hkv, Hq // Hkv, D).reshape(r, Hq * D)
    return flat(O), flat(A), flat(E)


def attention_bound(O, A, E, D, n):
    """How far the kernel may be off.  The score: D products summed in fp32 in chains of 16, each addition off by at most one unit of
    2^-23 of sum |q k| (tensor cores cut, they do not round): (D / 16 + 16) 2^-23 E; its scaling and the base's subtraction
    2 * 2^-24 of the score's size, E again at most.  An error e of the exponent changes a probability by a factor of at most e^(2 e)
    (numerator and sum).  The exponential is good to 2^-13.7 (the cubic that a part of them takes, 7.5e-5) on both sides; the
    probabilities are rounded to bf16, 2^-8 of each term; the sums over n keys in chains of 16 keys add one unit of 2^-23 of A
    each, and the sum of exponentials n / 2 of them; O is rounded once, 2^-8."""
    e = (D / 16 + 18) * 2.0 ** -23 * E
    return 2.0 ** -8 * O.abs() * 1.01 + A * (2.0 ** -8 + 2 * 7.5e-5 + 2.1 * e + (n / 16 + n / 2 + 64) * 2.0 ** -23) * 1.01 + 1e-30
