"""The 4-bit operators of the library as cases: products with 4-bit weights, the Gated MLP on such weights, a paged 4-bit
key/value cache (append and gather) and attention over it.

``own`` false: the plain forms in elementary torch operations, fp32 throughout, one rounding at the end.
``own`` true: the library's entry points, called as a user calls them.

Weights: q in 0..15 with one scale (bf16) and one zero point per group of G input rows and output column,
W[k, n] = (q[k, n] - z[k // G, n]) * s[k // G, n]; without zero points z = 8.
Cache: a group of G channels of one token and head holds q in 0..15, a scale (bf16) and a zero point (a bf16 integer).  The
codes of a head's D channels lie in 32 units of D / 32 nibbles: channel c is nibble c // 32 of unit c % 32.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one token through a projection of a small layer: launch latency counts
        {"name": "w4mm_m1_small", "op": "w4_matmul", "M": 1, "K": 2048, "N": 2048, "G": 128, "zeros": False},
        # a batch of 64, the largest the operator takes, through the output projection of an 8B layer
        {"name": "w4mm_m64_8b", "op": "w4_matmul", "M": 64, "K": 4096, "N": 4096, "G": 128, "zeros": False},
        # seven tokens, an odd number of outputs, zero points, the finer groups
        {"name": "w4mm_m7_odd", "op": "w4_matmul", "M": 7, "K": 5632, "N": 2047, "G": 64, "zeros": True},
        # one token through the widest matrix of a 70B layer, finest groups
        {"name": "w4mm_m1_70b", "op": "w4_matmul", "M": 1, "K": 8192, "N": 28672, "G": 32, "zeros": True},
        # the Gated MLP of a small layer, one token, with its norm
        {"name": "w4mlp_m1_small", "op": "w4_forward", "M": 1, "D": 2048, "F": 5632, "G": 128, "zeros": False, "norm": True,
         "act": "silu"},
        # the 8B layer's decode step at its benchmark batch
        {"name": "w4mlp_m8_8b", "op": "w4_forward", "M": 8, "D": 4096, "F": 14336, "G": 128, "zeros": False, "norm": True,
         "act": "silu"},
        # a larger, odd decode batch with zero points and the GELU gate
        {"name": "w4mlp_m33_8b", "op": "w4_forward", "M": 33, "D": 4096, "F": 14336, "G": 64, "zeros": True, "norm": False,
         "act": "gelu"},
        # one new token of each of sixteen requests goes into the cache and is read back
        {"name": "kv4_write_decode", "op": "kv4_write", "T": 16, "L": 16, "Hkv": 8, "D": 128, "G": 64, "page": 64},
        # a chunk of a prompt goes into the cache, then the sequence so far is read back for the prompt's attention
        {"name": "kv4_write_chunk", "op": "kv4_write", "T": 2000, "L": 8191, "Hkv": 8, "D": 128, "G": 128, "page": 64},
        # a few speculative positions of three requests, small heads, an empty and a one-token request among them
        {"name": "kv4_attn_spec", "op": "kv4_attention", "B": 3, "T": 4, "Hq": 8, "Hkv": 2, "D": 64, "G": 32, "page": 16,
         "lo": 0, "hi": 1000, "lens": 1},
        # a decode batch with ragged lengths, 8B heads
        {"name": "kv4_attn_batch", "op": "kv4_attention", "B": 64, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "G": 64, "page": 64,
         "lo": 1, "hi": 8192, "lens": 2},
        # one long conversation, 70B heads
        {"name": "kv4_attn_long", "op": "kv4_attention", "B": 1, "T": 1, "Hq": 64, "Hkv": 8, "D": 128, "G": 128, "page": 64,
         "lo": 131071, "hi": 131071, "lens": 3},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["w4_matmul", "w4_forward", "kv4_write", "kv4_attention"])
    G = rng.choice([32, 64, 128])
    if op == "w4_matmul":
        K = max(1, _log(rng, 256, 28672) // G) * G
        M = _log(rng, 1, 64)
        N = min(_log(rng, 100, 28672), 8192 * 28672 // K, 33 * 3 * 4096 * 14336 // (K * M))
        return {"op": op, "M": M, "K": K, "N": N, "G": G, "zeros": rng.random() < 0.5}
    if op == "w4_forward":
        D = max(1, _log(rng, 256, 4096) // 128) * 128
        F = max(1, _log(rng, 512, 14336) // 128) * 128
        return {"op": op, "M": _log(rng, 1, 33), "D": D, "F": F, "G": G, "zeros": rng.random() < 0.5,
                "norm": rng.random() < 0.5, "act": rng.choice(["silu", "gelu", "glu"])}
    D = rng.choice([64, 128])
    G, page = min(G, D), rng.choice([16, 32, 48, 64, 128])
    if op == "kv4_write":
        L = _log(rng, 8, 8191)
        return {"op": op, "T": rng.randint(1, min(L, 2000)), "L": L, "Hkv": rng.randint(1, 8), "D": D, "G": G, "page": page}
    Hkv = rng.choice([1, 2, 3, 4, 8])
    B = _log(rng, 1, 64)
    T = rng.choice([1, 1, 1, 2, 3, 5])
    hi = min(_log(rng, 20, 131071), 32 * 8192 // (B * T))
    return {"op": op, "B": B, "T": T, "Hq": Hkv * rng.choice([1, 2, 4, 7, 8]), "Hkv": Hkv, "D": D,
            "G": G, "page": page, "lo": rng.randint(0, hi), "hi": hi, "lens": rng.randrange(1 << 20)}


def _lengths(case):
    r = random.Random(case["lens"])
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    if case["lo"] == 0 and case["B"] >= 3:
        n[0], n[1] = 0, 1
    return n


def work(case):
    op = case["op"]
    if op in ("w4_matmul", "w4_forward"):
        per = 0.5 + (3 if case["zeros"] else 2) / case["G"]
        if op == "w4_matmul":
            weights, io = case["K"] * case["N"], case["M"] * (case["K"] + case["N"])
        else:
            weights, io = 3 * case["D"] * case["F"], 2 * case["M"] * case["D"]
        return {"bytes": int(weights * per + 2 * io), "flops": 2 * case["M"] * weights}
    row = 2 * case["Hkv"] * (case["D"] // 2 + 4 * case["D"] // case["G"])       # a token's codes, scales and zero points
    full = 2 * case["Hkv"] * case["D"] * 2                                      # the same token in bf16
    if op == "kv4_write":
        return {"bytes": case["T"] * (full + row) + case["L"] * (full + row) + 8 * (case["T"] + case["L"]),
                "flops": 4 * (case["T"] + case["L"]) * case["Hkv"] * case["D"]}
    n = sum(_lengths(case))
    return {"bytes": n * row + 2 * case["B"] * case["T"] * case["Hq"] * case["D"] * 2 + 4 * (n // case["page"] + 2 * case["B"]),
            "flops": 4 * n * case["T"] * case["Hq"] * case["D"]}


# ------------------------------------------------------------------------------------------------------------ inputs

def _quantize(x, G):
    """Codes (uint8), scales (bf16) and zero points (fp32 integers) of the groups of G along the last axis of x."""
    v = x.float().unflatten(-1, (-1, G))
    lo, hi = v.amin(-1).clamp(max=0), v.amax(-1).clamp(min=0)
    s = ((hi - lo) / 15).to(torch.bfloat16)
    sf = s.float()
    some = sf > 0
    safe = torch.where(some, sf, torch.ones_like(sf))
    z = torch.where(some, torch.round(-lo / safe).clamp(0, 15), torch.zeros_like(sf))
    q = (torch.round(v / safe[..., None]) + z[..., None]).clamp(0, 15)
    q = torch.where(some[..., None], q, torch.zeros_like(q))
    return q.flatten(-2).to(torch.uint8), s, z


def _weights(gen, K, N, G, zeros):
    """Normal weights in groups: codes [K, N], scales [K / G, N] and zero points [K / G, N] or None."""
    w = torch.randn(N, K, device=DEV, generator=gen).mul_(K ** -0.5)
    if zeros:
        q, s, z = _quantize(w, G)
        return {"codes": q.t().contiguous(), "scales": s.t().contiguous(), "zeros": z.to(torch.uint8).t().contiguous(), "G": G}
    v = w.unflatten(-1, (-1, G))
    s = (v.abs().amax(-1) / 7).to(torch.bfloat16)
    q = (torch.round(v / s.float()[..., None]) + 8).clamp_(0, 15).to(torch.uint8).flatten(-2)
    return {"codes": q.t().contiguous(), "scales": s.t().contiguous(), "zeros": None, "G": G}


def _pack_channels(q, D):
    """Codes [..., D] -> bytes [..., D / 2] in the cache's order."""
    n = q.unflatten(-1, (D // 32, 32)).transpose(-1, -2).flatten(-2)            # unit by unit, its nibbles in order
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _unpack_channels(b, D):
    n = torch.stack((b & 15, b >> 4), -1).flatten(-2)
    return n.unflatten(-1, (32, D // 32)).transpose(-1, -2).flatten(-2)


def _filled_cache(gen, n_pages, Hkv, page, D, G):
    """Codes and parameters of a cache that holds normal keys and values in every row."""
    parts = []
    for _ in range(2):
        codes = torch.empty(n_pages, Hkv, page, D // 2, dtype=torch.uint8, device=DEV)
        params = torch.empty(n_pages, Hkv, page, D // G, 2, dtype=torch.bfloat16, device=DEV)
        for p in range(0, n_pages, 512):
            x = torch.randn(min(512, n_pages - p), Hkv, page, D, device=DEV, generator=gen)
            q, s, z = _quantize(x, G)
            codes[p:p + 512] = _pack_channels(q, D)
            params[p:p + 512] = torch.stack((s, z.to(torch.bfloat16)), -1)
        parts += [codes, params]
    return parts


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if own:
        from paper_2606_26344_b200 import gmlp
        st["gmlp"] = gmlp

    def bf16(*shape):
        return torch.randn(*shape, device=DEV, generator=gen).to(torch.bfloat16)

    def matrix(K, N):
        w = _weights(gen, K, N, case["G"], case["zeros"])
        return st["gmlp"].w4_pack(w["codes"], w["scales"], w["zeros"]) if own else w

    if op == "w4_matmul":
        st["X"] = bf16(case["M"], case["K"])
        st["W"] = matrix(case["K"], case["N"])
    elif op == "w4_forward":
        D, F = case["D"], case["F"]
        st["X"] = bf16(case["M"], D)
        st["gamma"] = (torch.rand(D, device=DEV, generator=gen) + 0.5).to(torch.bfloat16) if case["norm"] else None
        st["Wg"], st["Wu"], st["Wd"] = matrix(D, F), matrix(D, F), matrix(F, D)
    else:
        Hkv, D, G, page = case["Hkv"], case["D"], case["G"], case["page"]
        if op == "kv4_write":
            tokens = [case["L"]]
        else:
            tokens = _lengths(case)
        need = [-(-n // page) for n in tokens]
        n_pages = sum(need) + 3
        st["cache"] = _filled_cache(gen, n_pages, Hkv, page, D, G)
        order = torch.randperm(n_pages, device=DEV, generator=gen).to(torch.int32)
        if op == "kv4_write":
            st["K"], st["V"] = bf16(case["T"], Hkv * D), bf16(case["T"], Hkv * D)
            at = torch.arange(case["L"], device=DEV)
            st["slots"] = order[at // page].long() * page + at % page
        else:
            width = max(1, max(need))
            table = torch.full((case["B"], width), -1, dtype=torch.int32, device=DEV)
            used = 0
            for b, k in enumerate(need):
                table[b, :k] = order[used:used + k]
                used += k
            st["table"], st["lengths"] = table, torch.tensor(tokens, dtype=torch.int32, device=DEV)
            st["Q"] = bf16(case["B"] * case["T"], case["Hq"] * D)
        if own:
            st["cache"] = st["gmlp"].Kv4Cache(*st["cache"])
    return st


# ------------------------------------------------------------------------------------------------------- plain forms

def _dequantize_weights(w):
    q = w["codes"].float().unflatten(0, (-1, w["G"]))
    z = 8.0 if w["zeros"] is None else w["zeros"].float()[:, None]
    return ((q - z) * w["scales"].float()[:, None]).flatten(0, 1)


def _dequantize_rows(codes, params, D, G):
    """Rows [..., D / 2] with parameters [..., D / G, 2] -> fp32 values [..., D]."""
    q = _unpack_channels(codes, D).float().unflatten(-1, (-1, G))
    p = params.float()
    return ((q - p[..., 1:]) * p[..., :1]).flatten(-2)


def _gate(g, act):
    if act == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    s = 1 / (1 + torch.exp(-g))
    return s if act == "glu" else g * s


EPS = 1e-5


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "w4_matmul":
        return (st["X"].float() @ _dequantize_weights(st["W"])).to(torch.bfloat16)
    if op == "w4_forward":
        x = st["X"].float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st["gamma"].float()
        h = _gate(x @ _dequantize_weights(st["Wg"]), case["act"]) * (x @ _dequantize_weights(st["Wu"]))
        return (h @ _dequantize_weights(st["Wd"])).to(torch.bfloat16)
    Hkv, D, G, page = case["Hkv"], case["D"], case["G"], case["page"]
    if op == "kv4_write":
        # the new rows are the sequence's last T; they are written, and then the whole sequence is read back
        slots = st["slots"]
        new = slots[case["L"] - case["T"]:]
        out = []
        for x, codes, params in ((st["K"], st["cache"][0], st["cache"][1]), (st["V"], st["cache"][2], st["cache"][3])):
            q, s, z = _quantize(x.view(-1, Hkv, D), G)
            codes[new // page, :, new % page] = _pack_channels(q, D)
            params[new // page, :, new % page] = torch.stack((s, z.to(torch.bfloat16)), -1)
            v = _dequantize_rows(codes[slots // page, :, slots % page], params[slots // page, :, slots % page], D, G)
            out.append(v.flatten(1).to(torch.bfloat16))
        return tuple(out)
    # attention, request by request over as many as are held at once in fp32
    B, T, Hq, table = case["B"], case["T"], case["Hq"], st["table"]
    q = st["Q"].float().view(B, T, Hkv, Hq // Hkv, D)
    kc, kp, vc, vp = st["cache"]
    keys = table.shape[1] * page
    step = max(1, (1 << 29) // (keys * Hkv * D))
    out = []
    for b in range(0, B, step):
        t = table[b:b + step].clamp(min=0).long()
        n = t.shape[0]

        def rows(codes, params):
            x = _dequantize_rows(codes[t], params[t], D, G)                     # [n, pages, Hkv, page, D]
            return x.transpose(1, 2).reshape(n, Hkv, keys, D)

        length = st["lengths"][b:b + step].long()
        seen = torch.arange(keys, device=DEV) < (length[:, None] - T + 1 + torch.arange(T, device=DEV)).unsqueeze(-1)
        seen = seen[:, None, :, None]                                           # [n, 1, T, 1, keys]
        k = rows(kc, kp)
        qq = q[b:b + step].permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, D) * D ** -0.5
        s = (qq @ k.transpose(-1, -2)).view(n, Hkv, T, -1, keys)
        del k
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True)
        p = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top)), torch.zeros_like(s))
        del s
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        v = rows(vc, vp)
        v = torch.where((torch.arange(keys, device=DEV) < length[:, None])[:, None, :, None], v, torch.zeros_like(v))
        o = p.view(n, Hkv, -1, keys) @ v
        out.append(o.view(n, Hkv, T, -1, D).permute(0, 2, 1, 3, 4).reshape(n * T, Hq * D).to(torch.bfloat16))
    return torch.cat(out)


# --------------------------------------------------------------------------------------------------- the library's own

def _own(st):
    case, gmlp = st["case"], st["gmlp"]
    op = case["op"]
    if op == "w4_matmul":
        return gmlp.w4_matmul(st["X"], st["W"])
    if op == "w4_forward":
        return gmlp.w4_forward(st["X"], st["Wg"], st["Wu"], st["Wd"], gamma=st["gamma"], eps=EPS, rmsnorm=case["norm"],
                               act=case["act"])
    if op == "kv4_write":
        gmlp.kv4_append(st["K"], st["V"], st["cache"], st["slots"][case["L"] - case["T"]:])
        return gmlp.kv4_gather(st["cache"], st["slots"])
    return gmlp.kv4_attention(st["Q"], st["cache"], st["table"], st["lengths"], case["Hq"], q_len=case["T"])


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The operators from their definitions in 64 bits: sums group by group, request by request, head by head."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op = case["op"]

    def product(x, w):
        y = torch.zeros(x.shape[0], w["codes"].shape[1], dtype=torch.float64, device=DEV)
        for i in range(w["scales"].shape[0]):
            rows = slice(i * w["G"], (i + 1) * w["G"])
            part = x[:, rows] @ w["codes"][rows].double()
            zero = 8.0 if w["zeros"] is None else w["zeros"][i].double()
            y += (part - x[:, rows].sum(1, keepdim=True) * zero) * w["scales"][i].double()
        return y

    if op == "w4_matmul":
        return product(st["X"].double(), st["W"])
    if op == "w4_forward":
        x = st["X"].double()
        if case["norm"]:
            x = x / (x.square().mean(1, keepdim=True) + EPS).sqrt() * st["gamma"].double()
        g, u = product(x, st["Wg"]), product(x, st["Wu"])
        if case["act"] == "gelu":
            a = g * torch.special.ndtr(g)
        elif case["act"] == "glu":
            a = torch.special.expit(g)
        else:
            a = g * torch.special.expit(g)
        return product(a * u, st["Wd"])
    D, G, page, Hkv = case["D"], case["G"], case["page"], case["Hkv"]
    chan = np.arange(D)
    nibble = torch.from_numpy((chan % 32) * (D // 32) + chan // 32).to(DEV)     # place of each channel's code in its row

    def values(codes, params):                                                  # rows [n, D / 2], [n, D / G, 2]
        byte = codes[:, nibble // 2].to(torch.int64)
        q = (byte >> (4 * (nibble % 2))) & 15
        group = torch.arange(D, device=DEV) // G
        return (q.double() - params[:, group, 1].double()) * params[:, group, 0].double()

    if op == "kv4_write":
        out = []
        first = case["L"] - case["T"]
        at = st["slots"]
        for x, codes, params in ((st["K"], st["cache"][0], st["cache"][1]), (st["V"], st["cache"][2], st["cache"][3])):
            y = torch.empty(case["L"], Hkv, D, dtype=torch.float64, device=DEV)
            for h in range(Hkv):
                y[:first, h] = values(codes[at[:first] // page, h, at[:first] % page], params[at[:first] // page, h, at[:first] % page])
                v = x[:, h * D:(h + 1) * D].double().reshape(-1, D // G, G)
                top, bottom = v.max(2).values.clamp(min=0), v.min(2).values.clamp(max=0)
                s = ((top - bottom) / 15).float().to(torch.bfloat16).double()[..., None]
                z = torch.round(-bottom[..., None] / s).clamp(0, 15)
                y[first:, h] = ((torch.round(v / s) + z).clamp(0, 15) - z).mul(s).nan_to_num(0.0).reshape(-1, D)
            out.append(y.reshape(case["L"], -1))
        return tuple(out)
    B, T, Hq = case["B"], case["T"], case["Hq"]
    out = torch.zeros(B * T, Hq * D, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        pages = st["table"][b, :-(-n // page)].long()
        for h in range(Hkv):
            k, v = (values(st["cache"][i][pages, h].reshape(-1, D // 2)[:n], st["cache"][i + 1][pages, h].reshape(-1, D // G, 2)[:n])
                    for i in (0, 2))
            for i in range(T):
                m = n - T + 1 + i
                if m <= 0:
                    continue
                for j in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                    p = torch.softmax(k[:m] @ st["Q"][b * T + i, j * D:(j + 1) * D].double() / math.sqrt(D), 0)
                    out[b * T + i, j * D:(j + 1) * D] = p @ v[:m]
    return out
