"""gmlp_kv_attention over many keys, cut between CTAs, row by row: limits that a lost or a doubled block of keys would pass by far."""
import pytest
import torch

import _paged as P
import _paged_rows as R
from test_gpu_kv_attention import Batch

pytestmark = pytest.mark.gpu


def check(reqs, Hq, Hkv, D, page, only):
    batch = Batch(reqs, Hq, Hkv, D, page, behind=0)
    O, at = batch.run(), 0
    for b, (r, n) in enumerate(reqs):
        if b in only:
            want, _, _ = P.attention(batch.Q[at:at + r], *batch.keys(b), Hq, D ** -0.5)
            worst = float(R.row_errors(O[at:at + r], want, D).max())
            assert worst <= R.limit(r, Hq, Hkv), (b, r, n, worst)
        at += r


@pytest.mark.parametrize("case", R.LONG, ids=str)
def test_rows_over_many_keys(case):
    check(*case, only=range(len(case[0])))


@pytest.mark.parametrize("reqs,Hq,Hkv,D,page", [([(33, 6000)] * 12, 8, 2, 128, 32), ([(20, 3000)] * 9, 16, 4, 64, 16), ([(1, 700)] * 300, 8, 2, 128, 64),
                                                ([(4, 1100)] * 90, 8, 2, 64, 16), ([(1, 1900)] * 45, 16, 2, 64, 48), ([(2, 4000)] * 40, 8, 2, 128, 16),
                                                ([(1, 1000 + 631 * (b % 11)) for b in range(70)], 32, 8, 128, 48),
                                                ([(200, 2500), (1, 5000), (3, 900)] * 4, 8, 2, 64, 48)])
def test_rows_of_items_cut_between_ctas(reqs, Hq, Hkv, D, page):
    check(reqs, Hq, Hkv, D, page, only=range(0, len(reqs), max(1, len(reqs) // 24)))


@pytest.mark.parametrize("r", [1, 20, 64])
def test_parts_of_more_than_one_piece(r):
    """24 items of 400000 to 600000 keys over the SMs: parts of some 600 blocks of 128 keys, more than are summed at a time."""
    check([(r, 400001), (r, 500000), (r, 599999)], 32, 8, 64, 64, only=(0, 2))
