"""gmlp_kv_attention at edges of its rows, values and lengths: rows that end inside a warp, rows without weight."""
import math

import pytest
import torch

from test_gpu_kv_attention import Batch

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
