"""GPU parity of the 4-bit key/value cache and of the attention over it against the 64-bit definitions."""
import math

import pytest
import torch

import _four_bit as F
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def bf16(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def rows_of(codes, params, slots, page, D, G):
    """64-bit values [T, Hkv, D] of the rows at `slots`, read from the cache's tensors by the documented order."""
    q = F.unpack_rows(codes[slots // page, :, slots % page])
    p = params[slots // page, :, slots % page]
    return F.values(q, p[..., 0], p[..., 1], G)


def garbage_cache(n_pages, Hkv, D, page, G):
    """A cache whose rows hold anything: all codes, NaN scales, infinite zero points."""
    c = gmlp.kv4_cache(n_pages, Hkv, D, page, G)
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=gen(1), device=DEV, dtype=torch.uint8))
    for t in (c.k_params, c.v_params):
        t[..., 0], t[..., 1] = float("nan"), float("inf")
    return c


SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("D,G", SHAPES)
@pytest.mark.parametrize("T,Hkv,page", [(1, 1, 16), (5, 3, 48), (300, 8, 64)])
def test_append_and_gather_are_exact_and_touch_nothing_else(T, Hkv, page, D, G):
    g = gen(T + D + G)
    n_pages = (T + page - 1) // page + 4
    c = garbage_cache(n_pages, Hkv, D, page, G)
    before = [t.clone() for t in (c.k_codes, c.k_params, c.v_codes, c.v_params)]
    K, V = bf16(g, T, Hkv * D), bf16(g, T, Hkv * D, scale=30.0)
    if T > 4:
        K[0] = 0
        K[1] = -1.5
        V[2, 7], V[3, 9] = float("inf"), float("nan")
        V[4] = 1e-40
        K[2, :G] = torch.linspace(1, 2, G, device=DEV).to(torch.bfloat16)        # a range that leaves 0 out
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:T]
    given = slots.clone()
    if T > 6:
        given[6] = -1
    gmlp.kv4_append(K, V, c, given, checked=True)
    kept = given[given >= 0]
    for x, codes, params, old_codes, old_params in ((K, c.k_codes, c.k_params, before[0], before[1]), (V, c.v_codes, c.v_params, before[2], before[3])):
        q, s, z = F.quantize(x.view(T, Hkv, D), G)
        want_codes, want_params = old_codes.clone(), old_params.clone()
        want_codes[kept // page, :, kept % page] = F.pack_rows(q)[given >= 0]
        want_params[kept // page, :, kept % page] = torch.stack((s, z.to(torch.bfloat16)), -1)[given >= 0]
        assert torch.equal(codes, want_codes)
        assert torch.equal(torch.isnan(params), torch.isnan(want_params))
        assert torch.equal(params.nan_to_num(-7.0), want_params.nan_to_num(-7.0))
    # back again, some slots twice, one padded
    ask = torch.cat((kept, kept[:1], torch.full((1,), -5, device=DEV)))
    gk, gv = gmlp.kv4_gather(c, ask, checked=True)
    for got, codes, params in ((gk, c.k_codes, c.k_params), (gv, c.v_codes, c.v_params)):
        want = rows_of(codes, params, ask.clamp(min=0), page, D, G).flatten(1)
        want[-1] = 0
        want = want.to(torch.bfloat16)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def test_slots_past_the_cache_are_skipped_and_reported():
    c = gmlp.kv4_cache(2, 2, 128, 16, 64)
    K = bf16(gen(1), 3, 256)
    slots = torch.tensor([5, 32, 1 << 40], device=DEV)
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_append(K, K, c, slots, checked=True)
    assert e.value.status == gmlp.ERR_INDEX
    assert int((c.k_codes != 0).any(-1).sum()) == 2 and bool((c.k_codes[0, :, 5] != 0).any())
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_gather(c, slots, checked=True)
    assert e.value.status == gmlp.ERR_INDEX
    gk, _ = gmlp.kv4_gather(c, slots)
    assert gmlp.device_status() != 0 and gmlp.device_status() == 0
    assert bool((gk[1:] == 0).all()) and bool((gk[0] != 0).any())


def filled(lengths, Hkv, D, page, G, seed, extra_pages=2, width=None, scale=1.0):
    """A cache with the given requests in shuffled pages, garbage everywhere else, and the requests' 64-bit rows."""
    g = gen(seed)
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + extra_pages
    c = garbage_cache(n_pages, Hkv, D, page, G)
    order = torch.randperm(n_pages, generator=g, device=DEV)
    width = width or max(1, max(need))
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    used, k, v = 0, [], []
    for b, n in enumerate(lengths):
        pages = order[used:used + need[b]]
        table[b, :need[b]] = pages.to(torch.int32)
        used += need[b]
        at = torch.arange(n, device=DEV)
        slots = pages[at // page] * page + at % page if n else at
        gmlp.kv4_append(bf16(g, n, Hkv * D, scale=scale), bf16(g, n, Hkv * D), c, slots, checked=True)
        k.append(rows_of(c.k_codes, c.k_params, slots, page, D, G) if n else torch.zeros(0, Hkv, D, dtype=torch.float64, device=DEV))
        v.append(rows_of(c.v_codes, c.v_params, slots, page, D, G) if n else torch.zeros(0, Hkv, D, dtype=torch.float64, device=DEV))
    return c, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), k, v


def check_attention(lengths, Hq, Hkv, D, G, page, T=1, seed=0, scale=None, key_scale=1.0, width=None):
    c, table, n, k, v = filled(lengths, Hkv, D, page, G, seed, width=width, scale=key_scale)
    Q = bf16(gen(seed + 99), len(lengths) * T, Hq * D)
    O = torch.full_like(Q, float("nan"))
    gmlp.kv4_attention(Q, c, table, n, Hq, q_len=T, scale=scale, O=O, checked=True)
    want, A, E = F.attention(Q.double(), k, v, lengths, Hq, T, D ** -0.5 if scale is None else scale)
    spread = max([62 * float(x.abs().max()) / 7 for x in v if x.numel()] + [0.0])
    bound = F.attention_bound(want, A, E, max(lengths + [0]) / 16 + 64, spread)
    off = (O.double() - want).abs()
    # rows that see a key (a channel of theirs whose values are all zero is no empty row: it is held to the bound, not to zero)
    seen = torch.tensor([[m - T + 1 + i > 0] for m in lengths for i in range(T)], device=DEV).expand_as(want)
    assert bool(torch.isfinite(O.float()).all())
    assert bool((O[~seen] == 0).all())
    if bool(seen.any()):
        err = (off / bound)[seen]
        assert float(err.max()) <= 1.0, f"{float(err.max()):.3f} of the bound"
    return O


@pytest.mark.parametrize("D,G", SHAPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 2), (7, 1), (16, 1), (24, 2)])
def test_attention_head_layouts(Hq, Hkv, D, G):
    check_attention([37, 1, 0, 200], Hq, Hkv, D, G, 16)


@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 1025])
def test_attention_lengths(n):
    check_attention([n, 300], 8, 2, 128, 64, 64, seed=n)


@pytest.mark.parametrize("page", [16, 32, 48, 80, 64, 128, 256])
def test_attention_page_sizes(page):
    check_attention([page - 1, page, page + 1, 3 * page + 7, 517], 4, 1, 128, 128, page, seed=page)
    check_attention([page - 1, 517], 4, 2, 64, 32, page, T=3, seed=page)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 8, 15, 16])
def test_attention_several_positions(T):
    # requests shorter than T: their first positions see nothing
    check_attention([T, T - 1, 0, 1, 40, 333], 8, 2, 128, 64, 16, T=T, seed=T)


@pytest.mark.parametrize("lengths,Hq,Hkv,D,G,page", [([5000], 64, 8, 128, 128, 64), ([20000], 4, 1, 128, 64, 64), ([3000, 40, 7000], 32, 8, 128, 64, 64),
                                                     ([40000], 8, 1, 64, 32, 256)])
def test_attention_long(lengths, Hq, Hkv, D, G, page):
    check_attention(lengths, Hq, Hkv, D, G, page, seed=5)


def test_attention_of_more_than_a_million_keys():
    # more keys per split than the sums of (16 + z) wait for
    check_attention([1200000], 4, 1, 64, 64, 256, seed=13)


def test_attention_many_requests_and_a_wide_table():
    # the table has room for far more pages than the requests use
    check_attention([(37 * i) % 200 for i in range(130)], 8, 4, 128, 64, 32, seed=6, width=700)


@pytest.mark.parametrize("scale", [0.0, -0.2, 0.7])
def test_attention_scales(scale):
    check_attention([100, 600], 4, 2, 128, 64, 16, seed=8, scale=scale)


def test_attention_peaked_scores():
    # scores of hundreds: the running maximum moves often, most probabilities vanish
    check_attention([900, 64], 8, 2, 128, 64, 64, seed=9, key_scale=12.0)


def test_attention_of_one_key_is_that_value():
    c, table, n, _, v = filled([1], 2, 128, 16, 128, 3)
    O = gmlp.kv4_attention(bf16(gen(1), 1, 8 * 128), c, table, n, 8, checked=True)
    want = v[0][0].repeat_interleave(4, 0).flatten()
    # P is 1; the scale is rounded into P' exactly, the product once
    assert bool(((O[0].double() - want).abs() <= 2.0 ** -8 * want.abs()).all())


def test_attention_masked_infinities_stay_out():
    # the last key and value of a request are not finite: only the last position sees them
    T, Hq, Hkv, D, page = 3, 4, 2, 128, 16
    c, table, n, k, v = filled([50], Hkv, D, page, 64, 4)
    clean = [k[0].clone()], [v[0].clone()]
    slot = table[0, 49 // page].long() * page + 49 % page
    bad = bf16(gen(2), 1, Hkv * D)
    bad[0, ::7] = float("inf")
    gmlp.kv4_append(bad, bad, c, slot.view(1), checked=True)
    Q = bf16(gen(5), T, Hq * D)
    O = gmlp.kv4_attention(Q, c, table, n, Hq, q_len=T, checked=True)
    want, A, E = F.attention(Q.double(), *clean, [50], Hq, T, D ** -0.5)
    bound = F.attention_bound(want, A, E, 68, 62 * float(clean[1][0].abs().max()) / 7)
    assert bool(((O.double() - want).abs()[:2] <= bound[:2]).all()) and bool(torch.isnan(O[2]).all())


def test_attention_bad_tables_are_left_out_and_reported():
    c, table, n, k, v = filled([60, 40], 2, 128, 16, 64, 11)
    Q = bf16(gen(5), 2, 4 * 128)
    good = gmlp.kv4_attention(Q, c, table, n, 4, checked=True)
    broken = table.clone()
    broken[0, 1], broken[1, 3] = c.n_pages, 1 << 30            # the second lies behind request 1's last page
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_attention(Q, c, broken, n, 4, checked=True)
    assert e.value.status == gmlp.ERR_INDEX
    O = gmlp.kv4_attention(Q, c, broken, n, 4)
    assert gmlp.device_status() != 0
    assert torch.equal(O[1], good[1])
    rest = [torch.cat((k[0][:16], k[0][32:]))], [torch.cat((v[0][:16], v[0][32:]))]
    want, A, E = F.attention(Q[:1].double(), *rest, [44], 4, 1, 128 ** -0.5)
    assert bool(((O[:1].double() - want).abs() <= F.attention_bound(want, A, E, 68, 62 * float(v[0].abs().max()) / 7)).all())
    for lengths in ([-3, 40], [60, 1 << 30]):
        with pytest.raises(gmlp.GmlpError) as e:
            gmlp.kv4_attention(Q, c, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), 4, checked=True)
        assert e.value.status == gmlp.ERR_INDEX
    assert gmlp.device_status() == 0


def test_cache_past_four_gigabytes():
    # codes of K alone are 4.6 GB; the request's pages lie at both ends
    n_pages, Hkv, D, page, G = 70000, 8, 128, 128, 128
    e = lambda d, t: torch.empty(n_pages, Hkv, page, *d, dtype=t, device=DEV)
    c = gmlp.Kv4Cache(e((64,), torch.uint8), e((1, 2), torch.bfloat16), e((64,), torch.uint8), e((1, 2), torch.bfloat16))
    pages = torch.tensor([n_pages - 1, 0, n_pages - 2, 35000], device=DEV)
    n = 3 * page + 50
    at = torch.arange(n, device=DEV)
    slots = pages[at // page] * page + at % page
    K, V = bf16(gen(1), n, Hkv * D), bf16(gen(2), n, Hkv * D)
    gmlp.kv4_append(K, V, c, slots, checked=True)
    k, v = rows_of(c.k_codes, c.k_params, slots, page, D, G), rows_of(c.v_codes, c.v_params, slots, page, D, G)
    q, s, z = F.quantize(K.view(n, Hkv, D), G)
    assert torch.equal(k, F.values(q, s, z, G))
    assert torch.equal(gmlp.kv4_gather(c, slots, checked=True)[0], k.flatten(1).to(torch.bfloat16))
    Q = bf16(gen(3), 1, 32 * D)
    O = gmlp.kv4_attention(Q, c, pages.to(torch.int32)[None], torch.tensor([n], dtype=torch.int32, device=DEV), 32, checked=True)
    want, A, E = F.attention(Q.double(), [k], [v], [n], 32, 1, D ** -0.5)
    assert bool(((O.double() - want).abs() <= F.attention_bound(want, A, E, n / 16 + 64, 62 * float(v.abs().max()) / 7)).all())


def test_attention_repeats_on_streams_and_in_graphs():
    c, table, n, _, _ = filled([700, 90, 2500], 4, 128, 64, 64, 12)
    Q = bf16(gen(5), 3, 16 * 128)
    first = gmlp.kv4_attention(Q, c, table, n, 16, checked=True)
    for _ in range(5):
        assert torch.equal(gmlp.kv4_attention(Q, c, table, n, 16), first)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [gmlp.kv4_attention(Q, c, table, n, 16, stream=side if i % 2 else None) for i in range(6)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph = torch.cuda.CUDAGraph()
    K = bf16(gen(6), 3, 4 * 128)
    slots = torch.tensor([int(table[b, (int(n[b]) - 1) // 64]) * 64 + (int(n[b]) - 1) % 64 for b in range(3)], device=DEV)
    with torch.cuda.graph(graph):
        gmlp.kv4_append(K, K, c, slots)
        o = gmlp.kv4_attention(Q, c, table, n, 16)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, gmlp.kv4_attention(Q, c, table, n, 16)) and not torch.equal(o, first)
    n.sub_(50)                                                 # the graph reads the lengths of the day
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, gmlp.kv4_attention(Q, c, table, n, 16))


def test_binding_refusals():
    c, table, n, _, _ = filled([20], 2, 128, 16, 64, 1)
    Q = bf16(gen(1), 1, 4 * 128)
    for args in ((Q.float(), c, table, n, 4), (Q, c, table.long(), n, 4), (Q, c, table, n.long(), 4), (Q.cpu(), c, table, n, 4)):
        with pytest.raises(TypeError):
            gmlp.kv4_attention(*args)
    for args in ((Q, c, table, n, 8), (Q, c, table[0], n, 4), (Q, c, table, n.repeat(2), 4)):
        with pytest.raises(ValueError):
            gmlp.kv4_attention(*args)
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_attention(bf16(gen(1), 1, 3 * 128), c, table, n, 3)
    assert e.value.status == gmlp.ERR_SHAPE
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_attention(bf16(gen(1), 17, 4 * 128), c, table, n, 4, q_len=17)
    assert e.value.status == gmlp.ERR_SHAPE
    K = bf16(gen(1), 2, 256)
    with pytest.raises(TypeError):
        gmlp.kv4_append(K, K, c, torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        gmlp.kv4_append(K, K, c, torch.zeros(3, dtype=torch.int64, device=DEV))
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv4_cache(4, 2, 96, 16, 32) and gmlp.kv4_append(bf16(gen(1), 1, 192), bf16(gen(1), 1, 192), gmlp.kv4_cache(4, 2, 96, 16, 32),
                                                             torch.zeros(1, dtype=torch.int64, device=DEV))
    assert e.value.status == gmlp.ERR_UNSUPPORTED
    gmlp.kv4_append(K[:0], K[:0], c, torch.zeros(0, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()
    assert gmlp.device_status() == 0


def test_an_unchecked_call_s_bad_slot_is_an_index_error_for_the_next_checked_call_of_any_operator():
    c = gmlp.kv4_cache(2, 2, 128, 16, 64)
    K = bf16(gen(1), 3, 256)
    slots = torch.tensor([5, 32, 7], device=DEV)
    X, W = bf16(gen(2), 4, 256), bf16(gen(3), 256, 256)
    W4 = gmlp.w4_quantize(W, 64, checked=True)
    for call in (lambda: gmlp.forward(X, W, W, W, checked=True), lambda: gmlp.w4_matmul(X, W4, checked=True)):
        want = call()
        gmlp.kv4_append(K, K, c, slots)
        with pytest.raises(gmlp.GmlpError) as e:
            call()
        assert e.value.status == gmlp.ERR_INDEX and gmlp.device_status() == 0
        assert torch.equal(call(), want)
