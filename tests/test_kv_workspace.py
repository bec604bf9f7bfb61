"""gmlp_kv_workspace_bytes on the host: its rule, both sides of its steps, and 0 for sizes that the call refuses (no GPU)."""
import pytest

from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp


@pytest.fixture(scope="module", autouse=True)
def library():
    B.build_libgmlp()


def expected(T, ratio, D, sms):
    """A descriptor of 32 bytes for each SM; base and weight (8 bytes) of each row of its two partial results; these rows in fp32; and the
    sums of its two tiles' rows between two pieces of an item.  A partial result has all rows of the call up to 128, else 256."""
    up = lambda n: -(-n // 256) * 256
    rows = T * ratio if T * ratio <= 128 else 256
    return up(32 * sms) + up(16 * sms * rows) + 8 * sms * D * (rows + min(rows, 128))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sms", [1, 100, 148])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 1, 1), (1, 8, 8), (1, 64, 8), (16, 64, 8), (17, 64, 8), (127, 4, 4), (128, 4, 4), (129, 4, 4), (42, 12, 4), (43, 12, 4),
                                      (1, 128, 1), (2, 128, 1), (25, 5, 1), (26, 5, 1), (2048, 32, 8), (1 << 24, 64, 8)])
def test_the_rule(T, Hq, Hkv, D, sms):
    assert gmlp.kv_workspace_bytes(T, Hq, Hkv, D, sms) == expected(T, Hq // Hkv, D, sms)


def test_without_a_number_of_sms():
    """The current device's, or 148 where there is none: a B200 has 148."""
    assert gmlp.kv_workspace_bytes(64, 32, 8, 128) == expected(64, 4, 128, 148) == gmlp.kv_workspace_bytes(64, 32, 8, 128, 148)


@pytest.mark.parametrize("T,Hq,Hkv,D", [(0, 8, 2, 128), (-1, 8, 2, 128), ((1 << 24) + 1, 8, 2, 128), (5, 0, 2, 128), (5, -8, 2, 128), (5, 8, 0, 128), (5, 8, -2, 128),
                                        (5, 9, 2, 128), (5, 2, 8, 128), (5, 129, 1, 128), (5, 65536, 8, 128), (5, 8, 2, 96), (5, 8, 2, 0), (5, 8, 2, 256)])
def test_sizes_that_are_refused(T, Hq, Hkv, D):
    assert gmlp.kv_workspace_bytes(T, Hq, Hkv, D, 148) == 0
