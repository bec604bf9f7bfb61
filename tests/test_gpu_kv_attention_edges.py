"""gmlp_kv_attention at edges of its rows, values and lengths: rows that end inside a warp."""
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
