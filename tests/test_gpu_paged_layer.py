"""Rotary positions, the paged cache and its attention together, as a decoder layer uses them: three prompts go through the projection,
rotation and cache in chunks of different lengths, mixed with single tokens of requests that are further on, then tokens are decoded in a
captured graph.  Every stage is compared with its 64-bit definition on the stage's own inputs, and the tokens' keys with those that a dense
rotation of the whole prompt gives."""
import pytest
import torch

import _paged as P
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
D, Hq, Hkv, Dh, FF, PAGE, ROT, BASE = 512, 8, 2, 64, 1024, 16, 32, 5e5
SCALING = ("bands", 8.0, 1.0, 4.0, 512)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def bf16(seed, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen(seed), device=DEV) * scale).to(torch.bfloat16)


class Layer:
    def __init__(self, B, pages_each):
        w = lambda seed, K, N: bf16(seed, K, N, scale=K ** -0.5)
        self.q, self.k, self.v, self.o = w(1, D, Hq * Dh), w(2, D, Hkv * Dh), w(3, D, Hkv * Dh), w(4, Hq * Dh, D)
        self.gate, self.up, self.down = w(5, D, FF), w(6, D, FF), w(7, FF, D)
        self.gamma = (torch.rand(D, generator=gen(8), device=DEV) + 0.5).to(torch.bfloat16)
        self.rope = gmlp.Rope(ROT, base=BASE, scaling=SCALING)
        self.f, self.amplitude = P.frequencies(ROT, BASE, SCALING)
        self.cache = gmlp.kv_cache(B * pages_each, Hkv, Dh, PAGE)
        self.table = torch.randperm(B * pages_each, generator=gen(9), device=DEV).view(B, pages_each).to(torch.int32)

    def slots(self, request, at):
        return self.table[request, at // PAGE].long() * PAGE + at % PAGE

    def step(self, x, at, slots, lengths, q_start):
        q, k, v = gmlp.qkv_proj(x, self.q, self.k, self.v)
        qr = gmlp.kv_append(k, v, self.cache, slots, rope=self.rope, positions=at, Q=q)
        a = gmlp.kv_attention(qr, self.cache, self.table, lengths, Hq, q_start=q_start)
        s, n = gmlp.matmul_add_rmsnorm(a, self.o, x, gamma=self.gamma)
        y = gmlp.forward(n, self.gate, self.up, self.down)
        return dict(q=q, k=k, v=v, qr=qr, a=a, s=s, n=n, y=y)

    def check(self, out, x, request, at, start, lengths):
        near = lambda got, want, rel: float((got.double() - want).norm() / want.norm()) < rel
        for name in ("q", "k", "v"):
            assert near(out[name], x.double() @ getattr(self, name).double(), 2.0 ** -8)
        T = x.shape[0]
        qr = P.rotate(out["q"].view(T, Hq, Dh), at, self.f, self.amplitude, ROT, False)
        assert bool(((out["qr"].view(T, Hq, Dh).double() - qr).abs() <= P.rotate_bound(out["q"].view(T, Hq, Dh), qr, self.amplitude, ROT, False)).all())
        s = self.slots(request, at)
        kr = P.rotate(out["k"].view(T, Hkv, Dh), at, self.f, self.amplitude, ROT, False)
        got = self.cache.k[s // PAGE, :, s % PAGE]
        assert bool(((got.double() - kr).abs() <= P.rotate_bound(out["k"].view(T, Hkv, Dh), kr, self.amplitude, ROT, False)).all())
        assert torch.equal(self.cache.v[s // PAGE, :, s % PAGE].flatten(1), out["v"])
        for b, n in enumerate(lengths):
            rows = slice(start[b], start[b + 1])
            kv = [P.rows_of(c, self.table[b], n) for c in (self.cache.k, self.cache.v)]
            want, A, E = P.attention(out["qr"][rows], *kv, Hq, Dh ** -0.5)
            assert bool(((out["a"][rows].double() - want).abs() <= P.attention_bound(want, A, E, Dh, max(n, 1))).all())
        s64 = out["a"].double() @ self.o.double() + x.double()
        assert near(out["s"], s64, 2.0 ** -8)
        n64 = out["s"].double() * torch.rsqrt(out["s"].double().square().mean(1, keepdim=True) + 1e-5) * self.gamma.double()
        assert near(out["n"], n64, 2.0 ** -8)
        g = out["n"].double() @ self.gate.double()
        assert near(out["y"], (g * torch.sigmoid(g) * (out["n"].double() @ self.up.double())) @ self.down.double(), 2.0 ** -7)


def test_prompts_in_chunks_beside_single_tokens_then_decode():
    B, layer = 3, Layer(3, 20)
    prompt = [150, 90, 7]
    x = [bf16(20 + b, prompt[b] + 40, D) for b in range(B)]
    done = [0, 0, 0]
    rows = lambda new: torch.cat([torch.full((r,), b, device=DEV) for b, r in enumerate(new)]).long()
    place = lambda new: torch.cat([torch.arange(done[b], done[b] + r, device=DEV) for b, r in enumerate(new)])
    for new in ((100, 1, 7), (50, 60, 1), (1, 29, 1), (1, 1, 1)):            # chunks beside single tokens, one request a step ahead
        start = [0, new[0], new[0] + new[1], sum(new)]
        tokens = torch.cat([x[b][done[b]:done[b] + r] for b, r in enumerate(new)])
        request, at = rows(new), place(new)
        lengths = [d + r for d, r in zip(done, new)]
        out = layer.step(tokens, at, layer.slots(request, at), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                         torch.tensor(start, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        layer.check(out, tokens, request, at, start, lengths)
        done = lengths
    # the whole first prompt at once, rotated densely: the same keys, and the same attention without a cache (head dimension 128 only there)
    _, k, _ = gmlp.qkv_proj(x[0][:150].contiguous(), layer.q, layer.k, layer.v)
    kr = gmlp.rope_apply(k, torch.arange(150, device=DEV), layer.rope, Hkv, checked=True)
    s = layer.slots(torch.zeros(150, dtype=torch.int64, device=DEV), torch.arange(150, device=DEV))
    assert float((layer.cache.k[s // PAGE, :, s % PAGE].flatten(1).double() - kr.double()).norm() / kr.double().norm()) < 2.0 ** -7
    # decode: static buffers, one captured step, replayed with new tokens, places and lengths
    token, at, slots = torch.empty(B, D, dtype=torch.bfloat16, device=DEV), torch.zeros(B, dtype=torch.int64, device=DEV), torch.zeros(B, dtype=torch.int64, device=DEV)
    lengths, start = torch.zeros(B, dtype=torch.int32, device=DEV), torch.arange(B + 1, dtype=torch.int32, device=DEV)
    request = torch.arange(B, device=DEV)

    def feed():
        token.copy_(torch.stack([x[b][done[b]] for b in range(B)]))
        at.copy_(torch.tensor(done, device=DEV))
        slots.copy_(layer.slots(request, at))
        lengths.copy_(torch.tensor([d + 1 for d in done], dtype=torch.int32, device=DEV))

    feed()
    layer.step(token, at, slots, lengths, start)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.step(token, at, slots, lengths, start)
    for i in range(35):                                                      # over two page ends
        feed()
        graph.replay()
        torch.cuda.synchronize()
        if i in (0, 1, 17, 34):
            layer.check(out, token, request, at, [0, 1, 2, 3], [d + 1 for d in done])
        done = [d + 1 for d in done]
    assert gmlp.device_status() == 0
    del graph


def test_rotated_keys_in_the_four_bit_cache():
    """The rotation beside the 4-bit cache: rope_apply on keys and queries, then kv4_append and kv4_attention."""
    T, rope = 40, gmlp.Rope(64)
    k, v, q = bf16(1, T, Hkv * Dh), bf16(2, T, Hkv * Dh), bf16(3, 1, Hq * Dh)
    at = torch.arange(T, device=DEV)
    cache = gmlp.kv4_cache(4, Hkv, Dh, PAGE, 32)
    kr = gmlp.rope_apply(k, at, rope, Hkv)
    gmlp.kv4_append(kr, v, cache, at)
    qr = gmlp.rope_apply(q, at[-1:], rope, Hq)
    table, n = torch.arange(4, dtype=torch.int32, device=DEV)[None], torch.tensor([T], dtype=torch.int32, device=DEV)
    o = gmlp.kv4_attention(qr, cache, table, n, Hq, checked=True)
    ks, vs = gmlp.kv4_gather(cache, at, checked=True)
    plain = gmlp.kv_cache(4, Hkv, Dh, PAGE)
    gmlp.kv_append(ks, vs, plain, at)
    p = gmlp.kv_attention(qr, plain, table, n, Hq, checked=True)
    # the gathered rows are rounded once more: 2^-9 each in norm, of keys (through scores of some 3) and values
    assert float((o.double() - p.double()).norm() / p.double().norm()) < 2.0 ** -6
