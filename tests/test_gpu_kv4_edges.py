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
