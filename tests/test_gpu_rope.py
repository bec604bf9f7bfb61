"""Rotary positions on the GPU: gmlp_rope_apply and the rotation of gmlp_kv_append, element by element against 64 bits."""
import pytest
import torch

import _paged as P
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def bf16(seed, *shape):
    return torch.randn(*shape, generator=gen(seed), device=DEV).to(torch.bfloat16)


def check_rows(got, x, positions, rope, base, scaling):
    f, a = P.frequencies(rope.rotary_dim, base, scaling)
    want = P.rotate(x, positions, f, rope.amplitude, rope.rotary_dim, rope.interleaved)
    bound = P.rotate_bound(x, want, rope.amplitude, rope.rotary_dim, rope.interleaved)
    worst = ((got.double() - want).abs() / bound).max()
    assert float(worst) <= 1.0, float(worst)
    assert torch.equal(got[..., rope.rotary_dim:].contiguous().view(torch.int16), x[..., rope.rotary_dim:].contiguous().view(torch.int16))


def check(T, H, D, rot, inter, base=1e4, scaling=None, far=5000, seed=1):
    rope = gmlp.Rope(rot, base=base, interleaved=inter, scaling=scaling)
    x = bf16(seed, T, H * D)
    at = torch.randint(-far, far, (T,), generator=gen(seed + 1), device=DEV)
    at[0] = 0
    y = gmlp.rope_apply(x, at, rope, H, checked=True)
    check_rows(y.view(T, H, D), x.view(T, H, D), at, rope, base, scaling)
    assert torch.equal(y[0].view(torch.int16), x[0].view(torch.int16)) or rope.amplitude != 1.0          # position 0 turns nothing


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (128, 16), (128, 8), (128, 4), (128, 12), (128, 20), (80, 20), (80, 32),
                                   (96, 96), (8, 8), (8, 4), (512, 512), (512, 500), (256, 64)])
def test_layouts(D, rot, inter):
    check(5, 3, D, rot, inter)


@pytest.mark.parametrize("T,H", [(1, 1), (1, 16), (1, 200), (2, 7), (64, 40), (147, 3), (149, 5), (2400, 2), (9600, 3), (3, 1000)])
@pytest.mark.parametrize("inter", [False, True])
def test_sizes(T, H, inter):
    check(T, H, 64, 64, inter, seed=T)


@pytest.mark.parametrize("scaling", [("linear", 4.0), ("bands", 8.0, 1.0, 4.0, 8192), ("ramp", 16.0, 32.0, 1.0, 4096)])
@pytest.mark.parametrize("far", [2, 1 << 20])
def test_scalings(scaling, far):
    check(33, 4, 128, 128, False, 5e5, scaling, far)
    check(33, 4, 128, 64, True, 1e4, scaling, far)


def test_far_positions_lose_nothing():
    """A position 2^40 away: the table's exact product; 64 bits hold the angle only as far as the table's own rounding is known."""
    steps, _ = gmlp.rope_steps(64, 1e4)
    rope, x = gmlp.Rope(64), bf16(3, 6, 2 * 64)
    at = torch.tensor([0, 1 << 20, (1 << 31) + 7, 1 << 40, -(1 << 40), (1 << 62) + 1], device=DEV)
    y = gmlp.rope_apply(x, at, rope, 2, checked=True)
    for i, p in enumerate(at.tolist()):
        turns = [(p * s % (1 << 64)) / 2.0 ** 64 for s in steps]          # exact integers, then one rounding
        z = P.rotate(x[i:i + 1].view(1, 2, 64), torch.ones(1, dtype=torch.int64, device=DEV), [6.283185307179586 * t for t in turns], 1.0, 64, False)
        bound = P.rotate_bound(x[i:i + 1].view(1, 2, 64), z, 1.0, 64, False)
        assert bool(((y[i:i + 1].view(1, 2, 64).double() - z).abs() <= bound).all())


def test_amplitude_in_place_and_transpose():
    x = bf16(4, 50, 4 * 64)
    at = torch.arange(50, device=DEV) * 17
    rope = gmlp.Rope(32, amplitude=-1.75)
    y = gmlp.rope_apply(x, at, rope, 4, checked=True)
    check_rows(y.view(50, 4, 64), x.view(50, 4, 64), at, rope, 1e4, None)
    z = x.clone()
    assert gmlp.rope_apply(z, at, rope, 4, Y=z, checked=True) is z and torch.equal(z.view(torch.int16), y.view(torch.int16))
    # <g, R x> = <R^T g, x>: the call with negated positions is the gradient
    g = bf16(5, 50, 4 * 64)
    back = gmlp.rope_apply(g, -at, rope, 4, checked=True)
    left, right = (g.double() * y.double()).sum(), (back.double() * x.double()).sum()
    size = (g.double().abs() * y.double().abs()).sum() + (back.double().abs() * x.double().abs()).sum()
    assert float((left - right).abs()) <= 2.0 ** -8 * float(size)
    # and it agrees with differences of the 64-bit form, a linear map
    f, _ = P.frequencies(32, 1e4)
    want = P.rotate(g.view(50, 4, 64), -at, f, -1.75, 32, False)
    assert bool(((back.view(50, 4, 64).double() - want).abs() <= P.rotate_bound(g.view(50, 4, 64), want, 1.75, 32, False)).all())


def test_infinities_and_nan_stay_in_their_pair():
    x = bf16(6, 3, 2 * 64)
    x[1, 5], x[1, 70] = float("inf"), float("nan")
    rope = gmlp.Rope(64)
    y = gmlp.rope_apply(x, torch.tensor([3, 4, 5], device=DEV), rope, 2, checked=True)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, [5, 37, 64 + 6, 64 + 38]] = True
    assert torch.equal(bad, want)


def test_no_rows_and_refusals_of_the_binding():
    rope = gmlp.Rope(64)
    assert gmlp.rope_apply(bf16(1, 0, 128), torch.zeros(0, dtype=torch.int64, device=DEV), rope, 2).shape == (0, 128)
    x, at = bf16(1, 4, 128), torch.zeros(4, dtype=torch.int64, device=DEV)
    for bad in (dict(positions=at.int()), dict(positions=at.cpu()), dict(X=x.float()), dict(X=bf16(1, 4, 256)[:, ::2]), dict(Y=x.float())):
        with pytest.raises(TypeError):
            gmlp.rope_apply(**{**dict(X=x, positions=at, rope=rope, n_heads=2), **bad})
    for bad in (dict(positions=at[:3]), dict(n_heads=3), dict(n_heads=0), dict(Y=bf16(1, 3, 128))):
        with pytest.raises(ValueError):
            gmlp.rope_apply(**{**dict(X=x, positions=at, rope=rope, n_heads=2), **bad})
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.rope_apply(x, at, rope, 4)                          # heads of 32 channels, 64 of them to be turned
    assert e.value.status == gmlp.ERR_SHAPE


# ------------------------------------------------------------------------------------------------------------- append

def slots_of(seed, T, n_pages, page):
    return torch.randperm(n_pages * page, generator=gen(seed), device=DEV)[:T].contiguous()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv,page,inter,rot", [(1, 8, 2, 16, False, 64), (5, 3, 3, 48, True, 64), (300, 32, 8, 64, False, 32), (2500, 7, 1, 32, False, 20),
                                                     (40, 0, 4, 16, True, 12)])
def test_append_rotates_keys_and_queries_and_touches_nothing_else(T, Hq, Hkv, page, inter, rot, D):
    n_pages = -(-T // page) + 2
    cache = gmlp.KvCache(bf16(1, n_pages, Hkv, page, D), bf16(2, n_pages, Hkv, page, D))
    k0, v0 = cache.k.clone(), cache.v.clone()
    K, V = bf16(3, T, Hkv * D), bf16(4, T, Hkv * D)
    Q = bf16(5, T, Hq * D) if Hq else None
    at = torch.randint(0, 100000, (T,), generator=gen(6), device=DEV)
    slots = slots_of(7, T, n_pages, page)
    skip = torch.rand(T, generator=gen(8), device=DEV) < (0.2 if T > 1 else 0.0)
    slots[skip] = -1 - slots[skip]
    rope = gmlp.Rope(rot, interleaved=inter)
    q = gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q, checked=True)
    if Hq:
        check_rows(q.view(T, Hq, D), Q.view(T, Hq, D), at, rope, 1e4, None)
    else:
        assert q is None
    keep = ~skip
    s = slots[keep]
    check_rows(cache.k[s // page, :, s % page], K.view(T, Hkv, D)[keep], at[keep], rope, 1e4, None)
    v0[s // page, :, s % page] = V.view(T, Hkv, D)[keep]
    assert torch.equal(cache.v, v0)
    k0[s // page, :, s % page] = cache.k[s // page, :, s % page]
    assert torch.equal(cache.k, k0)
    # without a rope the rows are stored as they are
    gmlp.kv_append(K, V, cache, slots, checked=True)
    k0[s // page, :, s % page] = K.view(T, Hkv, D)[keep]
    assert torch.equal(cache.k, k0) and torch.equal(cache.v, v0)


def test_append_slots_past_the_cache_are_skipped_and_reported():
    cache = gmlp.kv_cache(2, 2, 64, 16)
    K, V, Q = bf16(1, 4, 128), bf16(2, 4, 128), bf16(3, 4, 256)
    slots, at = torch.tensor([31, 32, 1 << 40, -(1 << 62)], device=DEV), torch.arange(4, device=DEV)
    rope = gmlp.Rope(64)
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q, checked=True)
    assert e.value.status == gmlp.ERR_INDEX and gmlp.device_status() == 0
    assert torch.equal(cache.v[1, :, 15], V[0].view(2, 64)) and int(torch.count_nonzero(cache.v)) == int(torch.count_nonzero(V[0]))
    gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q)
    assert gmlp.device_status() >> 16 == 200 and gmlp.device_status() == 0


def test_append_in_place_on_a_stream_and_in_a_graph():
    cache, T = gmlp.kv_cache(40, 4, 128, 16), 600
    K, V, Q0 = bf16(1, T, 512), bf16(2, T, 512), bf16(3, T, 1024)
    at, slots, rope = torch.arange(T, device=DEV), slots_of(4, T, 40, 16), gmlp.Rope(128, base=5e5)
    want = gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q0, checked=True)
    k, v = cache.k.clone(), cache.v.clone()
    Q, side = Q0.clone(), torch.cuda.Stream()
    torch.cuda.synchronize()
    cache.k.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q, Q_out=Q, stream=side)
    side.synchronize()
    assert got is Q and torch.equal(Q, want) and torch.equal(cache.k, k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gmlp.kv_append(K, V, cache, slots, rope=rope, positions=at, Q=Q0)
    for _ in range(3):
        cache.k.zero_()
        cache.v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache.k, k) and torch.equal(cache.v, v)
    del graph


def test_append_past_four_gigabytes():
    """A cache whose arrays pass 2^32 bytes each: rows at both ends and around the border."""
    n_pages, page, Hkv, D = 36000, 64, 8, 128
    k, v = (torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache = gmlp.KvCache(k, v)
    border = (1 << 32) // (Hkv * page * D * 2)
    slots = torch.tensor([0, border * page - 1, border * page, border * page + 5, n_pages * page - 1], device=DEV)
    K, V = bf16(1, 5, Hkv * D), bf16(2, 5, Hkv * D)
    gmlp.kv_append(K, V, cache, slots, checked=True)
    assert torch.equal(k[slots // page, :, slots % page].flatten(1), K) and torch.equal(v[slots // page, :, slots % page].flatten(1), V)


def test_append_refusals_of_the_binding():
    cache, rope = gmlp.kv_cache(2, 2, 64, 16), gmlp.Rope(64)
    K, Q, at, slots = bf16(1, 4, 128), bf16(2, 4, 256), torch.arange(4, device=DEV), torch.arange(4, device=DEV)
    ok = dict(K=K, V=K, cache=cache, slots=slots, rope=rope, positions=at, Q=Q)
    for bad in (dict(rope=None), dict(rope=None, Q=None), dict(positions=None), dict(K=bf16(1, 3, 128)), dict(Q=bf16(1, 4, 100)), dict(Q=bf16(1, 3, 256)),
                dict(slots=slots[None]), dict(Q=None, Q_out=Q), dict(positions=at[:3])):
        with pytest.raises(ValueError):
            gmlp.kv_append(**{**ok, **bad})
    for bad in (dict(slots=slots.int()), dict(K=K.float()), dict(V=K.cpu()), dict(Q_out=Q.float())):
        with pytest.raises(TypeError):
            gmlp.kv_append(**{**ok, **bad})
