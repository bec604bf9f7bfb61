"""Plain 64-bit definitions of the 4-bit operators, for the tests: quantisation, the cache's channel order, products,
attention.  Nothing here calls the library."""
import math

import torch


def quantize(x, G, zero_points=True):
    """Codes, scales (bf16) and zero points of groups of G along the last axis of x (any float type), from the definition."""
    v = x.double().unflatten(-1, (-1, G))
    bad = ~torch.isfinite(v).all(-1)
    v = torch.where(bad[..., None], torch.zeros_like(v), v)
    lo, hi = v.amin(-1).clamp(max=0), v.amax(-1).clamp(min=0)
    span = (hi.float() - lo.float()) / 15 if zero_points else torch.maximum(hi, -lo).float() / 7
    s = span.to(torch.bfloat16).double()
    bad |= ~torch.isfinite(s)
    some = (s > 0) & ~bad
    safe = torch.where(some, s, torch.ones_like(s))
    rint = lambda a: torch.round(a)                                  # half to even
    z = rint(-lo / safe).clamp(0, 15) if zero_points else torch.full_like(s, 8)
    q = (rint(v / safe[..., None]) + z[..., None]).clamp(0, 15)
    if zero_points:
        z = torch.where(some, z, torch.zeros_like(z))
    q = torch.where(some[..., None], q, z[..., None].expand_as(q))
    s = torch.where(bad, torch.full_like(s, math.nan), s)
    return q.flatten(-2).to(torch.uint8), s.to(torch.bfloat16), z


def values(q, s, z, G):
    """(q - z) * s in 64 bits, groups of G along the last axis."""
    return ((q.double().unflatten(-1, (-1, G)) - z.double()[..., None]) * s.double()[..., None]).flatten(-2)


def weights(gen, K, N, G, zero_points, device):
    """A random quantised matrix: codes [K, N], scales, zeros (or None), its 64-bit values [K, N], and the largest terms an
    evaluation may form of them, ((16 + q) + (16 + z)) * |s| (see product_bound)."""
    w = torch.randn(N, K, generator=gen, device=device) * K ** -0.5
    q, s, z = quantize(w, G, zero_points)
    c = lambda t: t.t().contiguous()
    terms = ((32 + q.double().unflatten(-1, (-1, G)) + z.double()[..., None]) * s.double().abs()[..., None]).flatten(-2)
    return c(q), c(s), c(z.to(torch.uint8)) if zero_points else None, c(values(q, s, z, G)), c(terms)


def product_bound(x, terms, G):
    """How far an fp32 evaluation of x @ w may be off, element by element, where it sums (16 + q) x over a group and takes
    (16 + z) sum(x) off afterwards.  Products of a bf16 number and a number below 32 are exact.  A group is at most G / 16
    accumulation steps of 16 products, sum(x) at most G additions, the difference one fused step, the groups are K / G fused
    multiply-adds, at most 16 more additions join the partial sums; each addition (16 per step) is off by at most one unit in
    the last place, 2^-23, of the sum of the absolute values, which is at most |x| @ terms."""
    K = x.shape[1]
    return (G + 1 + K / G + 16) * 2.0 ** -23 * (x.abs() @ terms)


def channel_places(D):
    """Nibble of each channel's code in its row: unit c % 32 has D / 32 nibbles, channel c is number c / 32 of them."""
    c = torch.arange(D)
    return (c % 32) * (D // 32) + c // 32


def pack_rows(q):
    """Codes [..., D] -> bytes [..., D / 2] of the cache."""
    D = q.shape[-1]
    nib = torch.zeros_like(q)
    nib[..., channel_places(D).to(q.device)] = q
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def unpack_rows(b):
    D = 2 * b.shape[-1]
    nib = torch.stack((b & 15, b >> 4), -1).flatten(-2)
    return nib[..., channel_places(D).to(b.device)]


def attention(Q, k, v, lengths, Hq, T, scale):
    """Q [B * T, Hq * D] in 64 bits; k, v: per request [len, Hkv, D] in 64 bits.  Returns O, sum of p |v|, and the largest
    error of a score (in nats) that an fp32 evaluation may make."""
    D = Q.shape[1] // Hq
    O, A, E = (torch.zeros_like(Q) for _ in range(3))
    for b, n in enumerate(lengths):
        Hkv = k[b].shape[1]
        for i in range(T):
            m = n - T + 1 + i
            if m <= 0:
                continue
            for h in range(Hq):
                q, g, at = Q[b * T + i, h * D:(h + 1) * D], h // (Hq // Hkv), slice(h * D, (h + 1) * D)
                s = k[b][:m, g] @ q * scale
                p = torch.softmax(s, 0)
                O[b * T + i, at] = p @ v[b][:m, g]
                A[b * T + i, at] = p @ v[b][:m, g].abs()
                # the terms are (16 + q) and (16 + z), at most 62 steps s of a quantiser together, and s <= max |k| / 7 (the 15 steps
                # of a group reach at least 7 to one side); D additions and a few scalings, one unit each
                E[b * T + i, at] = (62 / 7 * k[b][:m, g].abs().max() * q.abs().sum() * abs(scale) * (D + 8) + s.abs().max()) * 2.0 ** -23
    return O, A, E


def attention_bound(O, A, E, steps, spread):
    """P' is rounded to bf16 once (2^-8 of each term), O once (2^-8); a score off by E changes p by a factor e^(2 E) at most
    (numerator and sum); exp2 is good to 2^-21 on both sides; the fp32 sums over `steps` accumulations see (16 + q) and
    (16 + z), at most 62 steps of a quantiser together, weighted by p (`spread`: 62 / 7 of the largest |v|, as for the scores)."""
    return 2.0 ** -8 * (O.abs() + A) * 1.01 + (2 * E + 2.0 ** -20) * A * 1.01 + steps * 2.0 ** -23 * spread
