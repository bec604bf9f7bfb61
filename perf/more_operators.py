"""Rotary positions, a paged bf16 key/value cache and attention of new tokens over it, as cases.

``own`` false: the plain forms in elementary torch operations, fp32 throughout (angles in 64 bits), one rounding at the end.
``own`` true: the library's entry points, called as a user calls them.

Rotation: pair i of a head's first ``rot`` channels, (2 i, 2 i + 1) if interleaved, else (i, i + rot / 2), turns by the angle
position * f_i and is multiplied by an amplitude; the head's other channels stay.  f_i = base^(-2 i / rot), scaled for long contexts.
Cache: [pages, key/value heads, page size, head channels] for keys and for values; token in slot page * page_size + place.
Attention: request b has ``q`` new positions and n keys, the new ones' included; position i of it sees keys 0 .. n - q + i.
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
        # the queries of one token of a small model, before attention without a cache: launch latency counts
        {"name": "rope_one", "op": "rope", "T": 1, "H": 16, "D": 64, "rot": 64, "inter": False, "base": 1e4, "scaling": "none",
         "factor": 1.0, "far": 2000},
        # part of each head, interleaved pairs, an odd number of tokens, positions squeezed to a quarter
        {"name": "rope_part", "op": "rope", "T": 1777, "H": 24, "D": 128, "rot": 64, "inter": True, "base": 1e4, "scaling": "linear",
         "factor": 4.0, "far": 16000},
        # a long prompt through 70B heads, far positions, frequencies scaled band by band along a ramp
        {"name": "rope_prompt_70b", "op": "rope", "T": 8191, "H": 64, "D": 128, "rot": 128, "inter": False, "base": 5e5,
         "scaling": "ramp", "factor": 16.0, "far": 131072},
        # a decode batch's step between projection and attention: rotate queries and keys, store keys and values
        {"name": "append_decode_8b", "op": "append", "T": 64, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "rot": 128, "inter": False,
         "base": 5e5, "scaling": "bands", "factor": 8.0, "far": 60000},
        # the same for a chunk of a prompt, 70B heads
        {"name": "append_chunk_70b", "op": "append", "T": 4095, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "rot": 128, "inter": False,
         "base": 5e5, "scaling": "bands", "factor": 8.0, "far": 60000},
        # one token of one short request, small heads
        {"name": "attn_one", "op": "attention", "B": 1, "singles": 1, "qlo": 1, "qhi": 1, "lo": 136, "hi": 136, "pad": 0, "Hq": 8,
         "Hkv": 2, "D": 64, "page": 16, "lens": 1},
        # a decode batch with ragged lengths, 8B heads
        {"name": "attn_decode_batch", "op": "attention", "B": 64, "singles": 64, "qlo": 1, "qhi": 1, "lo": 0, "hi": 8191, "pad": 0,
         "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "lens": 2},
        # one long conversation, 70B heads
        {"name": "attn_decode_long", "op": "attention", "B": 1, "singles": 1, "qlo": 1, "qhi": 1, "lo": 131070, "hi": 131070, "pad": 0,
         "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "lens": 3},
        # a follow-up question after a long document, 70B heads
        {"name": "attn_question_long", "op": "attention", "B": 1, "singles": 0, "qlo": 61, "qhi": 61, "lo": 65475, "hi": 65475, "pad": 0,
         "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "lens": 4},
        # a chunk of a prompt after its first 6191 tokens, 8B heads
        {"name": "attn_chunk_8b", "op": "attention", "B": 1, "singles": 0, "qlo": 2048, "qhi": 2048, "lo": 6191, "hi": 6191, "pad": 0,
         "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "lens": 5},
        # continuous batching: 40 single tokens, three chunks of prompts and two empty places of a padded batch
        {"name": "attn_mixed", "op": "attention", "B": 43, "singles": 40, "qlo": 70, "qhi": 700, "lo": 0, "hi": 6000, "pad": 2,
         "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "lens": 6},
        # whole prompts of a small model with three query heads to a key head, pages that end inside the kernels' tiles
        {"name": "attn_prompts", "op": "attention", "B": 7, "singles": 0, "qlo": 5, "qhi": 4096, "lo": 0, "hi": 0, "pad": 0,
         "Hq": 12, "Hkv": 4, "D": 64, "page": 48, "lens": 7},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    D = rng.choice([64, 128])
    if op in ("rope", "append"):
        rot = rng.choice([D, D, D // 2, D // 4])
        case = {"op": op, "D": D, "rot": rot, "inter": rng.random() < 0.4, "base": rng.choice([1e4, 5e5, 1e6]),
                "scaling": rng.choice(["none", "linear", "bands", "ramp"]), "factor": rng.choice([2.0, 4.0, 8.0, 16.0]),
                "far": _log(rng, 100, 131072)}
        if op == "rope":
            return {**case, "T": _log(rng, 1, 8191), "H": rng.randint(1, 64)}
        Hkv = rng.randint(1, 8)
        return {**case, "T": _log(rng, 1, 4095), "Hkv": Hkv, "Hq": Hkv * rng.choice([1, 2, 3, 4, 7, 8]),
                "page": rng.choice([16, 32, 48, 64, 128])}
    Hkv = rng.choice([1, 2, 3, 4, 8])
    ratio = rng.choice([1, 2, 3, 4, 5, 8])
    case = {"op": op, "Hq": Hkv * ratio, "Hkv": Hkv, "D": D, "page": rng.choice([16, 32, 48, 64, 128]), "pad": rng.choice([0, 0, 0, 1, 3]),
            "lens": rng.randrange(1 << 20)}
    kind = rng.choice(["decode", "chunks", "mixed"])
    if kind == "decode":
        B = _log(rng, 1, 64)
        hi = min(_log(rng, 20, 131071), 64 * 8192 // B) - 1
        return _within({**case, "B": B, "singles": B, "qlo": 1, "qhi": 1, "lo": rng.randint(0, hi), "hi": hi})
    qhi = _log(rng, 2, 2048)
    chunks = _log(rng, 1, 8)
    hi = rng.choice([0, _log(rng, 20, 65536)])
    case = {**case, "B": chunks + (_log(rng, 1, 40) if kind == "mixed" else 0), "qlo": rng.randint(1, qhi), "qhi": qhi,
            "lo": rng.randint(0, hi), "hi": hi}
    case["singles"] = case["B"] - chunks
    return _within(case)


def _within(case):
    """The case with shorter requests if it would cost more than the largest listed ones."""
    while work(case)["bytes"] > 1.2e9 or work(case)["flops"] > 2.4e11:
        for name in ("qlo", "qhi", "lo", "hi"):
            case[name] = max(1 if name[0] == "q" else 0, case[name] * 3 // 4)
    return case


def _requests(case):
    """New positions and keys (the new positions' included) of each request; the padded batch's empty places come last, with one
    position and no key."""
    r = random.Random(case["lens"])
    new = [1 if b < case["singles"] else r.randint(case["qlo"], case["qhi"]) for b in range(case["B"])]
    keys = [q + r.randint(case["lo"], case["hi"]) for q in new]
    return new + [1] * case["pad"], keys + [0] * case["pad"]


def work(case):
    op = case["op"]
    if op == "rope":
        n = case["T"] * case["H"]
        return {"bytes": 4 * n * case["D"] + 8 * case["T"], "flops": 3 * n * case["rot"]}
    if op == "append":
        n = case["T"] * (case["Hq"] + 2 * case["Hkv"])
        return {"bytes": 4 * n * case["D"] + 16 * case["T"], "flops": 3 * case["T"] * (case["Hq"] + case["Hkv"]) * case["rot"]}
    new, keys = _requests(case)
    pairs = sum(q * n - q * (q - 1) // 2 for q, n in zip(new, keys) if n)
    return {"bytes": sum(keys) * case["Hkv"] * case["D"] * 4 + 4 * sum(new) * case["Hq"] * case["D"] + 4 * sum(-(-n // case["page"]) for n in keys),
            "flops": 4 * pairs * case["Hq"] * case["D"]}


# ------------------------------------------------------------------------------------------------------------ inputs

LOW, HIGH, ORIGINAL = 1.0, 4.0, 8192                 # bands: wavelengths that fit the trained context so often; its length
FAST, SLOW = 32.0, 1.0                               # ramp: turns within the trained context at its two ends


def _frequencies(case):
    """Radians per position of each pair, and the amplitude, in 64 bits."""
    rot, factor = case["rot"], case["factor"]
    f = case["base"] ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    turns = ORIGINAL * f / (2 * math.pi)             # of each pair within the trained context
    if case["scaling"] == "none":
        return f, 1.0
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "bands":
        keep = np.clip((turns - LOW) / (HIGH - LOW), 0, 1)
        return f * keep + f / factor * (1 - keep), 1.0
    at = lambda beta: rot * math.log(ORIGINAL / (beta * 2 * math.pi)) / (2 * math.log(case["base"]))
    lo, hi = max(math.floor(at(FAST)), 0), min(math.ceil(at(SLOW)), rot - 1)
    keep = 1 - np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 0.001), 0, 1)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, D = case["op"], case["D"]
    st = {"case": case}
    if own:
        from paper_2606_26344_b200 import gmlp
        st["gmlp"] = gmlp

    def bf16(*shape):
        return torch.randn(*shape, device=DEV, generator=gen).to(torch.bfloat16)

    if op in ("rope", "append"):
        T = case["T"]
        f, st["amplitude"] = _frequencies(case)
        st["f"] = torch.from_numpy(f).to(DEV)
        # a chunk is a run of positions, a decode batch one position of each request
        if op == "append" and T <= 64:
            st["at"] = torch.randint(0, case["far"], (T,), device=DEV, generator=gen)
        else:
            st["at"] = torch.arange(T, device=DEV) + torch.randint(0, case["far"], (1,), device=DEV, generator=gen)
        if own:
            scaling = {"none": None, "linear": ("linear", case["factor"]), "bands": ("bands", case["factor"], LOW, HIGH, ORIGINAL),
                       "ramp": ("ramp", case["factor"], FAST, SLOW, ORIGINAL)}[case["scaling"]]
            st["rope"] = st["gmlp"].Rope(case["rot"], base=case["base"], interleaved=case["inter"], scaling=scaling)
    if op == "rope":
        st["X"] = bf16(case["T"], case["H"] * D)
        return st
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    if op == "append":
        T = case["T"]
        st["Q"], st["K"], st["V"] = bf16(T, Hq * D), bf16(T, Hkv * D), bf16(T, Hkv * D)
        n_pages = (T if T <= 64 else -(-T // page)) + 3
        order = torch.randperm(n_pages, device=DEV, generator=gen)
        at = torch.arange(T, device=DEV)
        place = torch.randint(0, page, (T,), device=DEV, generator=gen)
        st["slots"] = order[at] * page + place if T <= 64 else order[at // page] * page + at % page
    else:
        new, keys = _requests(case)
        need = [-(-n // page) for n in keys]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, device=DEV, generator=gen).to(torch.int32).cpu()
        table = torch.full((len(need), max(1, max(need))), -1, dtype=torch.int32)
        used = 0
        for b, k in enumerate(need):
            table[b, :k] = order[used:used + k]
            used += k
        st["table"], st["lengths"] = table.to(DEV), torch.tensor(keys, dtype=torch.int32, device=DEV)
        st["start"] = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=DEV)
        st["Q"] = bf16(sum(new), Hq * D)
    st["k"], st["v"] = (torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for t in (st["k"], st["v"]):
        for p in range(0, n_pages, 512):
            t[p:p + 512] = torch.randn(t[p:p + 512].shape, device=DEV, generator=gen)
    if own:
        st["cache"] = st["gmlp"].KvCache(st["k"], st["v"])
    return st


# ------------------------------------------------------------------------------------------------------- plain forms

def _rotate(x, st):
    """fp32 rows [T, heads, D], rotated."""
    rot = st["case"]["rot"]
    angle = st["at"].double()[:, None] * st["f"]
    c, s = (st["amplitude"] * angle.cos()).float()[:, None], (st["amplitude"] * angle.sin()).float()[:, None]
    part = x[..., :rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if st["case"]["inter"] else (part[..., :rot // 2], part[..., rot // 2:])
    u, v = a * c - b * s, a * s + b * c
    turned = torch.stack((u, v), -1).flatten(-2) if st["case"]["inter"] else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _attend(q, k, v, seen):
    """q [n, T, Hkv, ratio, D], k and v [n, Hkv, keys, D], seen [n, T, keys] -> [n * T, Hq * D]."""
    n, T, Hkv, ratio, D = q.shape
    qq = q.permute(0, 2, 1, 3, 4).reshape(n, Hkv, T * ratio, D) * D ** -0.5
    seen = seen[:, None, :, None]
    s = (qq @ k.transpose(-1, -2)).view(n, Hkv, T, ratio, -1)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del s
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = p.view(n, Hkv, T * ratio, -1) @ v
    return o.view(n, Hkv, T, ratio, D).permute(0, 2, 1, 3, 4).reshape(n * T, -1).to(torch.bfloat16)


def _plain(st):
    case = st["case"]
    op, D = case["op"], case["D"]
    if op == "rope":
        return _rotate(st["X"].float().view(-1, case["H"], D), st).flatten(1).to(torch.bfloat16)
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    if op == "append":
        q = _rotate(st["Q"].float().view(-1, Hq, D), st).flatten(1).to(torch.bfloat16)
        at, place = st["slots"] // page, st["slots"] % page
        st["k"][at, :, place] = _rotate(st["K"].float().view(-1, Hkv, D), st).to(torch.bfloat16)
        st["v"][at, :, place] = st["V"].view(-1, Hkv, D)
        return q, st["k"], st["v"]
    # runs of requests with the same number of new positions go together, as many as are held at once in fp32
    new, keys = _requests(case)
    Q = st["Q"].view(-1, Hkv, Hq // Hkv, D)
    out, b, row = [], 0, 0
    while b < len(new):
        T, end = new[b], b + 1
        while end < len(new) and new[end] == T and (end + 1 - b) * max(keys[b:end + 1]) * max(Hkv * D, T * Hq) <= 1 << 30:
            end += 1
        n, pages = end - b, max(1, -(-max(keys[b:end]) // page))
        t = st["table"][b:end, :pages].clamp(min=0).long()
        k, v = (c[t].float().transpose(1, 2).reshape(n, Hkv, pages * page, D) for c in (st["k"], st["v"]))
        length = st["lengths"][b:end].long()[:, None]
        j = torch.arange(pages * page, device=DEV)
        v = torch.where((j < length)[:, None, :, None], v, torch.zeros_like(v))
        seen = j < (length - T + 1 + torch.arange(T, device=DEV))[..., None]
        out.append(_attend(Q[row:row + n * T].float().view(n, T, Hkv, -1, D), k, v, seen))
        b, row = end, row + n * T
    return torch.cat(out)


# --------------------------------------------------------------------------------------------------- the library's own

def _own(st):
    case, gmlp = st["case"], st["gmlp"]
    if case["op"] == "rope":
        return gmlp.rope_apply(st["X"], st["at"], st["rope"], case["H"])
    if case["op"] == "append":
        q = gmlp.kv_append(st["K"], st["V"], st["cache"], st["slots"], rope=st["rope"], positions=st["at"], Q=st["Q"])
        return q, st["k"], st["v"]
    return gmlp.kv_attention(st["Q"], st["cache"], st["table"], st["lengths"], case["Hq"], q_start=st["start"])


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The operators from their definitions in 64 bits: pairs as complex numbers, attention request by request and head by head."""
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op, D = case["op"], case["D"]

    def turned(x, heads):
        rot = case["rot"]
        y = x.double().reshape(-1, heads, D).clone()
        i = torch.arange(rot // 2, device=DEV)
        first, second = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
        angle = torch.outer(st["at"].double(), st["f"])
        z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(angle, st["amplitude"]), angle)[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if op == "rope":
        return turned(st["X"], case["H"]).flatten(1)
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    if op == "append":
        k, v = st["k"].double().transpose(1, 2).flatten(0, 1), st["v"].double().transpose(1, 2).flatten(0, 1)
        k[st["slots"]] = turned(st["K"], Hkv)
        v[st["slots"]] = st["V"].double().view(-1, Hkv, D)
        return (turned(st["Q"], Hq).flatten(1), *(c.unflatten(0, (-1, page)).transpose(1, 2) for c in (k, v)))
    new, keys = _requests(case)
    out = torch.zeros(sum(new), Hq * D, dtype=torch.float64, device=DEV)
    row = 0
    for b, (q, n) in enumerate(zip(new, keys)):
        pages = st["table"][b, :-(-n // page)].long()
        hidden = torch.ones(q, n, dtype=torch.bool, device=DEV).triu(n - q + 1) if n else None
        for h in range(Hq if n else 0):
            k, v = (c[pages, h // (Hq // Hkv)].reshape(-1, D)[:n].double() for c in (st["k"], st["v"]))
            at = slice(h * D, (h + 1) * D)
            s = (st["Q"][row:row + q, at].double() @ k.T / math.sqrt(D)).masked_fill_(hidden, -math.inf)
            out[row:row + q, at] = torch.softmax(s, 1) @ v
        row += q
    return out
