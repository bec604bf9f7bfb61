"""The 4-bit operators together, as a decoder layer uses them: a prompt goes through the bf16 projection and attention and into the
4-bit cache, its second chunk attends to the cache's rows, then tokens are decoded one at a time (and in a captured graph) through
4-bit projections, cache and Gated MLP.  Every stage is compared with its 64-bit definition on the stage's own inputs."""
import pytest
import torch

import _four_bit as F
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
D, Hq, Hkv, Dh, FF, G, PAGE = 512, 8, 2, 128, 1024, 64, 16


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Layer:
    def __init__(self, seed):
        g = gen(seed)
        self.ref, self.terms, self.w = {}, {}, {}
        for name, K, N in (("q", D, Hq * Dh), ("k", D, Hkv * Dh), ("v", D, Hkv * Dh), ("o", Hq * Dh, D), ("gate", D, FF), ("up", D, FF),
                           ("down", FF, D)):
            q, s, z, self.ref[name], self.terms[name] = F.weights(g, K, N, G, name != "o", DEV)
            self.w[name] = gmlp.w4_pack(q, s, z)
        self.gamma = (torch.rand(D, generator=g, device=DEV) + 0.5).to(torch.bfloat16)

    def check_product(self, name, x, y):
        want = x.double() @ self.ref[name]
        bound = F.product_bound(x.double(), self.terms[name], G) + 2.0 ** -8 * want.abs()
        assert bool(((y.double() - want).abs() <= bound).all()), name

    def check_mlp(self, x, y):
        n = x.double() * torch.rsqrt(x.double().square().mean(1, keepdim=True) + 1e-5) * self.gamma.double()
        a, u = n @ self.ref["gate"], n @ self.ref["up"]
        da, du = (F.product_bound(n, self.terms[k], G) + 2.0 ** -16 * (n.abs() @ self.ref[k].abs()) for k in ("gate", "up"))
        act = a * torch.sigmoid(a)
        h = act * u
        dh = 1.2 * da * u.abs() + act.abs() * du + 1.2 * da * du + (2.0 ** -16 + 2.0 ** -19) * h.abs()
        want = h @ self.ref["down"]
        bound = dh @ self.ref["down"].abs() + F.product_bound(h, self.terms["down"], G) + 2.0 ** -8 * want.abs()
        assert bool(((y.double() - want).abs() <= bound).all())


class Cache:
    def __init__(self, B, pages_each):
        self.c = gmlp.kv4_cache(B * pages_each, Hkv, Dh, PAGE, G)
        order = torch.randperm(B * pages_each, generator=gen(5), device=DEV)
        self.table = order.view(B, pages_each).to(torch.int32)

    def slots(self, b, at):
        return self.table[b, at // PAGE].long() * PAGE + at % PAGE

    def rows(self, b, n):
        """64-bit keys and values of request b, read by the documented order."""
        s = self.slots(b, torch.arange(n, device=DEV))
        out = []
        for codes, params in ((self.c.k_codes, self.c.k_params), (self.c.v_codes, self.c.v_params)):
            p = params[s // PAGE, :, s % PAGE]
            out.append(F.values(F.unpack_rows(codes[s // PAGE, :, s % PAGE]), p[..., 0], p[..., 1], G))
        return out


def check_attention(cache, Q, O, lengths, T):
    kv = [cache.rows(b, n) for b, n in enumerate(lengths)]
    k, v = [x[0] for x in kv], [x[1] for x in kv]
    want, A, E = F.attention(Q.double(), k, v, lengths, Hq, T, Dh ** -0.5)
    spread = 62 / 7 * max(float(x.abs().max()) for x in v)
    assert bool(((O.double() - want).abs() <= F.attention_bound(want, A, E, max(lengths) / 16 + 64, spread)).all())


def test_prompt_in_two_chunks_then_decode():
    layer, B, prompt, first = Layer(1), 3, 45, 30
    cache = Cache(B, 8)
    x = torch.randn(B, prompt, D, generator=gen(2), device=DEV).to(torch.bfloat16)
    # the prompt runs on bf16 weights made from the 4-bit ones
    W = {n: gmlp.w4_dequantize(layer.w[n]) for n in ("q", "k", "v")}
    torch.cuda.synchronize()
    for b in range(B):
        for lo, hi in ((0, first), (first, prompt)):
            q, k, v = gmlp.qkv_proj(x[b, lo:hi].contiguous(), W["q"], W["k"], W["v"])
            at = torch.arange(lo, hi, device=DEV)
            gmlp.kv4_append(k, v, cache.c, cache.slots(b, at))
            ks, vs = gmlp.kv4_gather(cache.c, cache.slots(b, torch.arange(hi, device=DEV)), checked=True)
            o = gmlp.gqa_attention(q, ks, vs, Hq, Hkv, causal=True, checked=True)
            rk, rv = cache.rows(b, hi)
            assert torch.equal(ks, rk.flatten(1).to(torch.bfloat16)) and torch.equal(vs, rv.flatten(1).to(torch.bfloat16))
            # the same positions straight from the cache, sixteen at a time at most: both round their probabilities (2^-8 of the
            # sum of p |v|) and outputs, the gathered rows one more time
            T = min(16, hi - lo)
            direct = gmlp.kv4_attention(q[-T:].contiguous(), cache.c, cache.table[b:b + 1], torch.tensor([hi], dtype=torch.int32, device=DEV),
                                        Hq, q_len=T, checked=True)
            check_attention_of = F.attention(q[-T:].double(), [rk], [rv], [hi], Hq, T, Dh ** -0.5)
            slack = 2.0 ** -6 * check_attention_of[1] + 4 * check_attention_of[2] * check_attention_of[1] + 2.0 ** -7 * check_attention_of[0].abs() + 1e-3
            assert bool(((direct.double() - o[-T:].double()).abs() <= slack).all())
    # decode: static buffers, one captured step, replayed with new tokens and lengths
    lengths = torch.full((B,), prompt, dtype=torch.int32, device=DEV)
    token = torch.empty(B, D, dtype=torch.bfloat16, device=DEV)
    slots = torch.empty(B, dtype=torch.int64, device=DEV)
    out = {}

    def step():
        q, k, v = (gmlp.w4_matmul(token, layer.w[n]) for n in ("q", "k", "v"))
        gmlp.kv4_append(k, v, cache.c, slots)
        a = gmlp.kv4_attention(q, cache.c, cache.table, lengths, Hq)
        o = gmlp.w4_matmul(a, layer.w["o"])
        y = gmlp.w4_forward(o, layer.w["gate"], layer.w["up"], layer.w["down"], gamma=layer.gamma, rmsnorm=True)
        out.update(q=q, k=k, v=v, a=a, o=o, y=y)

    def feed(i):
        token.copy_(torch.randn(B, D, generator=gen(100 + i), device=DEV).to(torch.bfloat16))
        n = prompt + i
        slots.copy_(torch.stack([cache.slots(b, torch.tensor([n], device=DEV))[0] for b in range(B)]))
        lengths.fill_(n + 1)

    graph = torch.cuda.CUDAGraph()
    feed(0)
    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(40):                                  # over two page ends
        feed(i)
        if i % 2:
            graph.replay()
        else:
            step_out = dict(out)
            step()
        torch.cuda.synchronize()
        if i in (0, 1, 2, 3, 18, 19, 35, 39):
            for n in ("q", "k", "v"):
                layer.check_product(n, token, out[n])
            check_attention(cache, out["q"], out["a"], [prompt + i + 1] * B, 1)
            layer.check_product("o", out["a"], out["o"])
            layer.check_mlp(out["o"], out["y"])
        if i % 2 == 0:
            out.update(step_out)                         # the graph's own outputs again
    assert gmlp.device_status() == 0
    del graph
