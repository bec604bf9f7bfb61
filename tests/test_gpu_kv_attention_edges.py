"""gmlp_kv_attention at edges of its rows, values and lengths: rows that end inside a warp, rows without weight, values
near the largest bf16 and values that are no numbers."""
import math

import pytest
import torch

from paper_2606_26344_b200 import gmlp
from test_gpu_kv_attention import Batch, gen

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(3, 1), (5, 1), (14, 2)])
@pytest.mark.parametrize("r", [3, 11, 17, 45, 70])
def test_rows_that_end_inside_a_warp(r, Hq, Hkv, D):
    """Lanes without a row beside lanes with one, in items of each kind, whole (300 keys) and cut between CTAs (5000)."""
    Batch([(r, 300), (r, 5000), (r + 1, 70)], Hq, Hkv, D, 16, seed=r).check()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("r,B", [(1, 1), (1, 300), (10, 1), (10, 300), (150, 1), (150, 200)])
def test_rows_whose_scores_are_all_minus_infinity_are_zeros_whatever_their_values(r, B, value):
    """V of the newest keys, which some row must not see, holds numbers that are none.  Few, small and big items; among many requests some
    items are cut between CTAs and some whole."""
    batch = Batch([(r, 60 + r)] * B + [(2, 90)], 2, 1, 64, 16, behind=0)
    batch.Q[:, 0], batch.Q[:, 64] = 2.0, 2.0
    pages = batch.table[:B, :-(-(60 + r) // 16)].long()
    batch.cache.k[pages, 0, :, 0] = -math.inf
    for j in (59 + r, 58 + r):
        batch.cache.v[batch.table[:B, j // 16].long(), 0, j % 16, 3] = value
    O = batch.run()
    assert bool((O[:B * r] == 0).all())
    batch.check_rows(O, only=(B,))


# Items of each kind over keys that are one item or several parts: (requests, Hq, Hkv, D, page)
KINDS = [([(1, 400)], 8, 2, 128, 64), ([(1, 9000), (3, 70)], 8, 2, 128, 16), ([(2, 5000)] * 3, 4, 1, 64, 48), ([(10, 100)], 8, 2, 128, 64),
         ([(10, 9000)], 8, 2, 128, 64), ([(20, 4000)] * 3, 6, 2, 64, 16), ([(300, 3000), (1, 700)], 8, 2, 128, 64),
         ([(150, 150), (90, 2000), (1, 3000)] * 9, 12, 4, 64, 48), ([(500, 2500)], 16, 2, 64, 128),
         ([(1, 200), (1, 150), (2, 20)] * 90, 32, 8, 128, 64), ([(10, 100), (1, 70), (12, 300)] * 90, 32, 8, 64, 16),     # many items to a CTA
         ([(70, 100), (40, 400), (1, 90), (0, 10), (3, 0)] * 40, 32, 8, 128, 32)]


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", KINDS)
@pytest.mark.parametrize("size", [1e34, 1e36, 3.38e38])
@pytest.mark.parametrize("equal", [False, True])
def test_large_values(reqs, Hq, Hkv, D, page, size, equal):
    """Sums of p V pass the largest float where their mean does not: keys of about the same score (or the very same, values of one sign), every
    value near `size`, up to the largest bf16."""
    batch = Batch(reqs, Hq, Hkv, D, page)
    v = batch.cache.v
    if equal:
        batch.Q.zero_()
        v.copy_(torch.where(torch.isnan(v), v, size * (0.5 + 0.5 * torch.rand(v.shape, generator=gen(2), device=DEV)).to(torch.bfloat16)))
    else:
        v.copy_(torch.where(torch.isnan(v), v, size * (2 * torch.rand(v.shape, generator=gen(2), device=DEV) - 1).to(torch.bfloat16)))
    O = batch.check(only=range(0, len(reqs), max(1, len(reqs) // 20)))
    assert bool(torch.isfinite(O).all())


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", KINDS)
def test_large_values_leave_the_other_channels_and_requests_as_they_are(reqs, Hq, Hkv, D, page):
    """One channel of one head of the first request is near the largest bf16, the others are ordinary or tiny: those keep their bits."""
    batch = Batch(reqs, Hq, Hkv, D, page)
    batch.cache.v[..., 1::2] *= 2.0 ** -100
    some = range(0, len(reqs), max(1, len(reqs) // 20))
    clean = batch.check(only=some).view(-1, Hq, D)
    r, n = reqs[0]
    j = torch.arange(n, device=DEV)
    batch.cache.v[batch.table[0, j // page].long(), 0, j % page, 6] = 3e38
    O = batch.check(only=some).view(-1, Hq, D)
    other = torch.ones_like(O, dtype=torch.bool)
    other[:r, :Hq // Hkv, 6] = False
    assert torch.equal(O[other], clean[other])
    assert bool(((O[~other].double() - 3e38).abs() <= 2.0 ** -7 * 3e38).all())       # a constant: half a step of V, one of P and one of O


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", KINDS)
@pytest.mark.parametrize("values", [(math.inf,), (-math.inf,), (math.nan,), (math.inf, -math.inf), (math.inf, math.inf)])
def test_values_that_are_no_numbers_reach_the_rows_that_see_them(reqs, Hq, Hkv, D, page, values):
    """Wherever their keys sit, and beside nothing else: V of some keys of the first request's first head holds `values` in two channels."""
    batch = Batch(reqs, Hq, Hkv, D, page)
    clean = batch.run().view(-1, Hq, D).clone()
    r, n = reqs[0]
    want = sum(values)
    hidden = -(-(n - r) // 3)                                            # two keys that all rows see, one that some do not, one that only the last does
    for at in ((0, n // 2), (n // 3, 0), (hidden, n - 1), (n - 1 - r // 2, 5)):
        for j, value in zip(at, values):
            batch.cache.v[batch.table[0, j // page].long(), 0, j % page, [2, D - 3]] = value
        O = batch.run().view(-1, Hq, D)
        hit = torch.zeros_like(O, dtype=torch.bool)
        expect = torch.zeros(O.shape[0], device=DEV)
        for i in range(r):
            seen = [v for j, v in zip(at, values) if j <= n - r + i]
            if seen:
                hit[i, :Hq // Hkv, 2] = True
                hit[i, :Hq // Hkv, D - 3] = True
                expect[i] = sum(seen)
        assert torch.equal(O[~hit], clean[~hit])
        got = O[hit].float()
        assert torch.equal(got.nan_to_num(nan=7.0, posinf=1.0, neginf=-1.0),
                           expect[:, None, None].expand(-1, Hq, D)[hit].nan_to_num(nan=7.0, posinf=1.0, neginf=-1.0)), (at, want)
        for j in at[:len(values)]:
            batch.cache.v[batch.table[0, j // page].long(), 0, j % page, [2, D - 3]] = 0.5
        clean = batch.run().view(-1, Hq, D).clone()


@pytest.mark.parametrize("r,n", [(1, 300), (10, 300), (300, 700), (1, 9000), (10, 9000), (300, 9000)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_no_numbers_count_however_small_their_weight(r, n, value):
    """Scores rise by thousands of binary orders along the keys, so that the weight of key 3 is no fp32 number but 0."""
    batch = Batch([(r, n)], 8, 2, 128, 64)
    j = torch.arange(n, device=DEV)
    batch.Q[:, ::128], batch.cache.k[..., 0] = 64.0, 0.0
    batch.cache.k[batch.table[0, j // 64].long(), :, j % 64, 0] = (8.0 * j / n * 64)[:, None].to(torch.bfloat16)
    batch.cache.v[batch.table[0, 0].long(), :, 3, 7] = value
    o = batch.run()[:r].view(r, 8, 128)
    assert bool(torch.isnan(o[..., 7]).all()) if math.isnan(value) else bool((o[..., 7] == value).all())
    o[..., 7] = 0
    assert bool(torch.isfinite(o).all())


def test_a_second_pass_keeps_nothing():
    """Calls that need it and calls that do not, in one graph and one workspace, by turns."""
    batch = Batch([(1, 3000), (200, 900), (9, 400)], 8, 2, 128, 64, behind=0)
    v = batch.cache.v.clone()
    v[torch.isnan(v)] = 0.0
    want = []
    for x in (v, v * 1e37):
        batch.cache.v.copy_(x)
        want.append(batch.check().clone())
    ws = torch.empty(gmlp.kv_workspace_bytes(batch.Q.shape[0], 8, 2, 128), dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = [gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, 8, q_start=batch.start, workspace=ws) for _ in range(3)]
    for i in range(4):
        batch.cache.v.copy_((v, v * 1e37)[i % 2])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[i % 2]) for o in outs)
    del g


def long_sums(r, n, mean, rise=0.0, seed=1):
    """37 requests of r positions over the same n keys, 4 key heads: 148 items of one length, which stay whole, one on each SM.  Values of mean
    `mean`, scores that rise by `rise` along the keys.  Returns the error's norm over that of the last rounding alone, of two requests and heads."""
    Hkv, ratio, D, page, B, g = 4, 4, 128, 64, 37, gen(seed)
    k, v = (torch.empty(-(-n // page), Hkv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for c, at in ((k, 0.0), (v, mean)):
        for p in range(0, k.shape[0], 2048):
            c[p:p + 2048] = torch.randn(c[p:p + 2048].shape, generator=g, device=DEV) + at
    table = torch.arange(k.shape[0], dtype=torch.int32, device=DEV).expand(B, -1).contiguous()
    Q = torch.randn(B * r, Hkv * ratio * D, generator=g, device=DEV).to(torch.bfloat16)
    if rise:
        Q[:, ::D] = 8.0
        k[..., 0] = (rise * D ** 0.5 / 8 / n * torch.arange(k.shape[0] * page, device=DEV).view(-1, 1, page)).to(torch.bfloat16)
    lengths = torch.full((B,), n, dtype=torch.int32, device=DEV)
    O = gmlp.kv_attention(Q, gmlp.KvCache(k, v), table, lengths, Hkv * ratio, q_len=r, checked=True)
    err = own = 0.0
    for b, h in ((0, 0), (36, 3)):
        q = Q[b * r:(b + 1) * r].double().view(r, Hkv, ratio * D)[:, h].reshape(-1, D)
        seen = (n - r + 1 + torch.arange(r, device=DEV)).repeat_interleave(ratio)[:, None]
        top, total, acc = torch.full((len(q), 1), -1e300, dtype=torch.float64, device=DEV), 0.0, 0.0
        for lo in range(0, n, 1 << 16):
            kk, vv = (c[:, h].reshape(-1, D)[lo:min(n, lo + (1 << 16))].double() for c in (k, v))
            s = (q @ kk.T / D ** 0.5).masked_fill(lo + torch.arange(len(kk), device=DEV) >= seen, -math.inf)
            now = torch.maximum(top, s.amax(1, keepdim=True))
            p, f, top = torch.exp(s - now), torch.exp(top - now), now
            total, acc = total * f + p.sum(1, keepdim=True), acc * f + p @ vv
        want = acc / total
        got = O[b * r:(b + 1) * r].double().view(r, Hkv, ratio * D)[:, h].reshape(-1, D)
        err += float((got - want).square().sum())
        own += float((want.to(torch.bfloat16).double() - want).square().sum())
    return (err / own) ** 0.5


@pytest.mark.parametrize("n", [32768, 32769, 65535, 131071, 1 << 20])
@pytest.mark.parametrize("mean", [0.0, 1.0])
def test_long_sums_of_single_tokens(n, mean):
    """A CTA goes over all keys of an item.  Adding towards 0 costs at most 2^-23 of the sum so far each time, 16 times a block of 128 keys, 2^-24
    on average: 256 blocks 2^-13 of the sum at the end (half of that, as the sum grows along the keys), a sixteenth of the rounding to bf16
    (2^-9 / sqrt(3) = 2^-9.8) by norm or less: sqrt(1 + 2^-6.4) = 1.006, and the second terms of the probabilities, 2^-17: 1.02 in all."""
    assert long_sums(1, n, mean) <= 1.02


@pytest.mark.parametrize("rise", [8.0, 20.0])
@pytest.mark.parametrize("r,most", [(1, 1.02), (10, 1.02), (64, 1.05 * 2 ** 0.5)])
def test_long_sums_whose_base_moves(rise, r, most):
    """The base of the exponentials moves in sums that have been set aside before."""
    assert long_sums(r, 131071, 1.0, rise) <= most


@pytest.mark.parametrize("n", [65536, 65537, 65664, 131072, 131073, 1 << 20])
@pytest.mark.parametrize("r,mean,most", [(10, 0.0, 1.02), (10, 1.0, 1.02), (64, 0.0, 1.02 * 2 ** 0.5), (64, 1.0, 1.02)])
def test_long_sums_of_chunks(r, mean, most, n):
    """Small and big items: 4096 additions of 16 keys to a sum at most, as above.  Big items round probabilities to bf16: an error of about the
    last rounding's size with values of both signs; with values of mean 1 the roundings of so many probabilities cancel in the mean."""
    assert long_sums(r, n, mean) <= most


@pytest.mark.parametrize("r", [10, 64])
@pytest.mark.parametrize("value", [1e37, math.inf])
def test_pieces_of_long_items_in_a_second_pass(r, value):
    """148 whole items of three pieces over the same keys, with values near the largest bf16 in one channel and an infinity in another, at keys of
    the first piece, the last one, and the newest key."""
    n, B, Hkv, D, page, g = 140000, 37, 4, 64, 64, gen(3)
    k, v = (torch.randn(-(-n // page), Hkv, page, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    table = torch.arange(k.shape[0], dtype=torch.int32, device=DEV).expand(B, -1).contiguous()
    Q = torch.randn(B * r, Hkv * 4 * D, generator=g, device=DEV).to(torch.bfloat16)
    call = lambda: gmlp.kv_attention(Q, gmlp.KvCache(k, v), table, torch.full((B,), n, dtype=torch.int32, device=DEV), 16, q_len=r, checked=True)
    clean = call().view(B * r, Hkv, 4, D).clone()
    v[:, 1, :, 6] = 1e37
    for j, channel in ((77, 9), (n - 5000, 10), (n - 1, 11)):
        v[j // page, 1, j % page, channel] = value
    O = call().view(B * r, Hkv, 4, D)
    assert bool(((O[:, 1, :, 6].double() - 1e37).abs() <= 2.0 ** -7 * 1e37).all())
    last = torch.zeros(B, r, dtype=torch.bool, device=DEV)
    last[:, -1] = True
    if value == math.inf:
        assert bool((O[:, 1, :, 9:11] == value).all()) and bool((O[last.view(-1), 1, :, 11] == value).all())
        assert torch.equal(O[~last.view(-1), 1, :, 11], clean[~last.view(-1), 1, :, 11])
    else:
        assert bool((O[:, 1, :, 9:11] > 1e28).all())
    other = torch.ones_like(O, dtype=torch.bool)
    other[:, 1, :, 6], other[:, 1, :, 9:12] = False, False
    assert torch.equal(O[other], clean[other])


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [24, 27, 29, 30])
@pytest.mark.parametrize("r,n", [(1, 300), (1, 9000), (10, 100), (10, 5000), (300, 700)])
def test_scores_of_large_magnitude(r, n, power, sign):
    """Up to 2^30 binary orders, the stated range.  Keys that are all the same give the mean of the values that a row sees, although the fp32
    base is off the score by up to 32 binary orders there; one key that scores twice as much gives its value."""
    batch = Batch([(r, n)], 8, 2, 128, 64, behind=0)
    score = 0.99 * 2.0 ** power / (128 ** -0.5 * 1.4426950408889634)
    batch.Q.zero_()
    batch.Q[:, ::128] = 2.0 ** (power // 2)
    k = torch.zeros_like(batch.cache.k)
    k[..., 0] = sign * score / 2 / 2.0 ** (power // 2)
    batch.cache.k.copy_(torch.where(torch.isnan(batch.cache.k), batch.cache.k, k))
    O = batch.run().view(r, 2, 4, 128)
    _, v = batch.keys(0)
    seen = n - r + 1 + torch.arange(r, device=DEV)
    want = (v.double().cumsum(0) / torch.arange(1, n + 1, device=DEV)[:, None, None])[seen - 1][:, :, None]
    size = (v.double().abs().cumsum(0) / torch.arange(1, n + 1, device=DEV)[:, None, None])[seen - 1][:, :, None]
    # the last rounding, one of each probability (big items), and a sum of n terms
    assert bool(((O.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + n * 2.0 ** -23) * size).all())
    j = n - r                                                                # a key that every row sees
    batch.cache.k[batch.table[0, j // 64].long(), :, j % 64, 0] *= 2 if sign > 0 else 0.5
    # Its probability before the division is 2^e, e what the fp32 base is off: no power of two.  Two bf16 terms hold it to 2^-16, which the last
    # rounding removes (V is a bf16 number); one term (big items) to 2^-8 of the value, and the last rounding may take 2^-8 on top.
    one_term, value = r * 4 > 128, v[j].double()[None, :, None].expand(r, 2, 4, 128)
    assert bool(((batch.run().view(r, 2, 4, 128).double() - value).abs() <= (2.0 ** -7 * 1.01 if one_term else 0.0) * value.abs()).all())


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", [KINDS[1], KINDS[4], KINDS[6], KINDS[7], KINDS[9]])
@pytest.mark.parametrize("size", [1.0, 3.38e38])
def test_a_second_pass_without_a_mask_and_with_bad_pages(reqs, Hq, Hkv, D, page, size):
    """Without a causal mask; then with a page outside of the cache in the first request, whose keys are left out, beside an infinity in the next
    page of each key head."""
    batch = Batch(reqs, Hq, Hkv, D, page)
    v, some = batch.cache.v, range(0, len(reqs), max(1, len(reqs) // 20))
    v.copy_(torch.where(torch.isnan(v), v, size * (2 * torch.rand(v.shape, generator=gen(2), device=DEV) - 1).to(torch.bfloat16)))
    assert bool(torch.isfinite(batch.check(causal=False, only=some)).all())
    (r, n), ratio = reqs[0], Hq // Hkv
    v[batch.table[0, 2].long(), :, 1, 4] = math.inf
    batch.table[0, 1] = batch.cache.n_pages
    O = torch.full_like(batch.Q, 7.0)
    gmlp.kv_attention(batch.Q, batch.cache, batch.table, batch.lengths, Hq, q_start=batch.start, causal=False, O=O)
    assert gmlp.device_status() >> 16 == 200
    batch.check_rows(O, causal=False, only=[b for b in some if b > 0])
    got = O[:r].view(r, Hkv, ratio, D)
    assert bool((got[..., 4] == math.inf).all())
    j = torch.arange(n, device=DEV)
    j = j[j // page != 1]
    k, x = (c[batch.table[0, j // page].long(), :, j % page].double() for c in (batch.cache.k, v))
    q = batch.Q[:r].double().view(r, Hkv, ratio, D)
    p = (torch.einsum("rghd,ngd->rghn", q, k) * D ** -0.5).softmax(-1)
    x[..., 4] = 0.0
    want, A = torch.einsum("rghn,ngd->rghd", p, x), torch.einsum("rghn,ngd->rghd", p, x.abs())
    # rounding of O and of each probability, 2^-8; scores and sums as in the others' bound, far below
    ok = (got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -9) * A
    ok[..., 4] = True
    assert bool(ok.all())
