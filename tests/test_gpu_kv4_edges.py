"""Attention over the 4-bit cache where masked places and extreme numbers could leak into a result: parametrised edges that the
ordinary distributions of the other tests do not reach."""
import pytest
import torch

import _four_bit as F
import test_gpu_kv4 as K
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("D,G", K.SHAPES)
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_zero_points_that_are_no_numbers_stay_behind_the_mask(D, G, bad):
    # a foreign cache: the newest token's zero points are not finite, and only the newest position sees that token
    T, Hq, Hkv, page, n = 3, 4, 2, 16, 50
    c, table, lengths, k, v = K.filled([n], Hkv, D, page, G, 4)
    at = int(table[0, (n - 1) // page]), slice(None), (n - 1) % page, slice(None), 1
    c.k_params[at], c.v_params[at] = bad, bad
    Q = K.bf16(K.gen(5), T, Hq * D)
    O = gmlp.kv4_attention(Q, c, table, lengths, Hq, q_len=T, checked=True)
    want, A, E = F.attention(Q.double(), k, v, [n], Hq, T, D ** -0.5)
    bound = F.attention_bound(want, A, E, 68, 62 * float(v[0].abs().max()) / 7)
    assert bool(((O.double() - want).abs()[:2] <= bound[:2]).all()) and bool(torch.isnan(O[2]).all())


def check(Q, K_rows, V_rows, Hq, T=1, page=64, G=64, D=128):
    """Attention of one request with these keys and values against the 64-bit result on what the cache holds of them."""
    n, Hkv = K_rows.shape[0], K_rows.shape[1] // D
    n_pages = -(-n // page)
    c = gmlp.kv4_cache(n_pages, Hkv, D, page, G)
    slots = torch.arange(n, device=DEV)
    gmlp.kv4_append(K_rows, V_rows, c, slots, checked=True)
    k, v = (K.rows_of(codes, params, slots, page, D, G) for codes, params in ((c.k_codes, c.k_params), (c.v_codes, c.v_params)))
    table = torch.arange(n_pages, dtype=torch.int32, device=DEV)[None]
    O = gmlp.kv4_attention(Q, c, table, torch.tensor([n], dtype=torch.int32, device=DEV), Hq, q_len=T, checked=True)
    want, _, E = F.attention(Q.double(), [k], [v], [n], Hq, T, D ** -0.5)
    largest = v.abs().unflatten(-1, (-1, G)).amax(-1).repeat_interleave(G, -1)       # of its group, whose step is at most 1 / 7 of it
    return O, want, F.attention(Q.double(), [k], [largest], [n], Hq, T, D ** -0.5)[0], E


# The bound, relative to A = sum(p * largest value of the group): P' has 16 bits, 2^-17 of each term.  An accumulator holds 16 + q, at most
# 31 / 7 of the largest, of up to 8 tiles with two products each, every one of which may drop 2^-23 of it: 2^-16.8 in all.  exp2 is
# good to 2^-21, the sums of warps and splits to less; 2^-15 covers them.  Scores are off by E.
def check_close(O, want, A, E):
    assert bool(torch.isfinite(O.float()).all())
    assert bool(((O.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -15 + 2 * E) * A).all())


@pytest.mark.parametrize("n,T", [(900, 1), (70, 4)])
@pytest.mark.parametrize("exponent", [40, 59, 61, 80, 110, 122])
def test_values_of_any_size(exponent, n, T):
    # exact powers of two move every value and every result alike
    g = K.gen(exponent)
    Q, k, v = K.bf16(g, T, 8 * 128), K.bf16(g, n, 256), K.bf16(g, n, 256)
    small = check(Q, k, v, 8, T)
    large = check(Q, k, (v.float() * 2.0 ** exponent).to(torch.bfloat16), 8, T)
    check_close(*small)
    check_close(*large)
    assert torch.equal(large[1], small[1] * 2.0 ** exponent)


@pytest.mark.parametrize("at", [0, 333, 899])
@pytest.mark.parametrize("size", [2.0 ** 70, 2.0 ** 100, 2.0 ** 127])
def test_one_large_value_among_ordinary_ones(at, size):
    g = K.gen(at)
    Q, k, v = K.bf16(g, 1, 8 * 128), K.bf16(g, 900, 256), K.bf16(g, 900, 256)
    v[at, 5], v[at, 200] = size, -size
    check_close(*check(Q, k, v, 8))


def test_a_large_value_that_the_softmax_leaves_out():
    # its probability is 0: what the others say comes through
    g = K.gen(3)
    Q, k, v = torch.ones(1, 128, dtype=torch.bfloat16, device=DEV), K.bf16(g, 500, 128), K.bf16(g, 500, 128)
    k[7], v[7] = -1000.0, 1e38
    O, want, A, E = check(Q, k, v, 1)
    assert float(want.abs().max()) < 1.0
    check_close(O, want, A, E)


@pytest.mark.parametrize("D,G", K.SHAPES)
@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("exponent", [-100, -60, 60, 66, 100, 120])
def test_queries_of_any_size(exponent, T, D, G):
    # keys as much smaller: powers of two leave every score as it is, up to where a query times 31 steps of a key has no float
    g, n = K.gen(exponent), 300
    Q, k, v = K.bf16(g, T, 8 * D), K.bf16(g, n, 2 * D), K.bf16(g, n, 2 * D)
    plain = check(Q, k, v, 8, T, G=G, D=D)
    large = check((Q.float() * 2.0 ** exponent).to(torch.bfloat16), (k.float() * 2.0 ** -exponent).to(torch.bfloat16), v, 8, T, G=G, D=D)
    check_close(*plain)
    check_close(*large)
    assert torch.equal(large[1], plain[1])


def test_queries_near_the_largest_bf16_choose_one_key():
    # scores of 1e38: the softmax is 1 at one key, another for each head, and 0 elsewhere; ordinary heads beside them stay ordinary
    g, n = K.gen(9), 300
    Q, k, v = K.bf16(g, 1, 8 * 128), K.bf16(g, n, 256), K.bf16(g, n, 256)
    Q[:, :4 * 128] *= 2.0 ** 124
    O, want, A, E = check(Q, k, v, 8)
    chosen = want[:, :512].view(4, 128)
    assert len({tuple(r.tolist()) for r in chosen}) > 1
    assert bool(((O.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * A)[:, :512].all())
    check_close(O[:, 512:], want[:, 512:], A[:, 512:], E[:, 512:])


@pytest.mark.parametrize("B,width", [(520, 4096), (3000, 1024)])
def test_many_requests_over_a_table_for_very_long_ones(B, width):
    # fewer splits than one per 2048 keys, and a workspace that stays small: short requests, two long ones, pages shared among all
    Hq = Hkv = 4
    D, G, page, n = 64, 32, 64, 9000
    c, table, _, k, v = K.filled([n], Hkv, D, page, G, 6)
    wide = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    lengths = [(11 * i) % 90 for i in range(B)]
    lengths[1], lengths[B - 1] = n, n - 77
    assert gmlp.kv4_workspace_bytes(B, 1, Hq, Hkv, D, width, page) <= 256 << 20
    Q = K.bf16(K.gen(7), B, Hq * D)
    O = gmlp.kv4_attention(Q, c, wide, torch.tensor(lengths, dtype=torch.int32, device=DEV), Hq, checked=True)
    want, A, E = F.attention(Q.double(), [k[0][:m] for m in lengths], [v[0][:m] for m in lengths], lengths, Hq, 1, D ** -0.5)
    bound = F.attention_bound(want, A, E, 128, 62 * float(v[0].abs().max()) / 7)
    assert bool(((O.double() - want).abs() <= bound).all())
