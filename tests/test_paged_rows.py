"""The limits on rows of attention over many keys tell a lost or a doubled block of 128 keys from rounding (no GPU)."""
import pytest
import torch

import _paged as P
import _paged_rows as R


@pytest.mark.parametrize("case", R.LONG, ids=str)
def test_a_lost_or_doubled_block_is_told_from_rounding(case):
    reqs, Hq, Hkv, D, _ = case
    ratio = Hq // Hkv
    for b, (r, n) in enumerate(reqs):
        g = torch.Generator().manual_seed(b)
        Q, k, v = torch.randn(1, ratio * D, generator=g), torch.randn(n, 1, D, generator=g), torch.randn(n, 1, D, generator=g)
        Q, k, v = (x.to(torch.bfloat16) for x in (Q, k, v))                  # the last position, one key head
        want, _, _ = P.attention(Q, k, v, ratio, D ** -0.5)
        assert bool((R.row_errors(want.to(torch.bfloat16), want, D) <= 1.0).all())
        for block in (0, n // 256, n // 128 - 1):
            j = torch.arange(n)
            inside = (j >= 128 * block) & (j < 128 * block + 128)
            for keys in (j[~inside], torch.cat((j, j[inside]))):
                O, _, _ = P.attention(Q, k[keys], v[keys], ratio, D ** -0.5)
                # some row of the item by far (an item's rows lose the same block)
                assert float(R.row_errors(O.to(torch.bfloat16), want, D).min()) > 2 * R.limit(r, Hq, Hkv), (r, n, block)
