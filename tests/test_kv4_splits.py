"""The workspace of the attention over the 4-bit cache and the splits that it holds, over wide page tables: host arithmetic only."""
import pytest

from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp

MOST = 256 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build_libgmlp()
    return gmlp.lib()


def one_split(b, q_len, hq, hkv, d):
    """Bytes of the partial results of one split: per request, key/value head and 8 or 16 query rows, head_dim + 4 floats a row."""
    rows = q_len * (hq // hkv)
    pad = 8 if rows <= 8 else 16
    return b * hkv * -(-rows // pad) * pad * (d + 4) * 4


def splits(b, q_len, hq, hkv, d, keys, page=64):
    n, each = gmlp.kv4_workspace_bytes(b, q_len, hq, hkv, d, keys // page, page, 148), one_split(b, q_len, hq, hkv, d)
    assert n % each == 0
    return max(1, n // each)


@pytest.mark.parametrize("q_len,hq,hkv,d", [(1, 32, 8, 128), (4, 64, 8, 128), (16, 64, 8, 128), (1, 8, 8, 64), (1, 64, 1, 64)])
def test_the_workspace_stays_in_bounds_and_the_splits_fall_step_by_step(q_len, hq, hkv, d):
    for keys in (64, 2048, 8192, 131072, 262144, 1 << 20, 1 << 26):
        before = 256
        for b in (1, 2, 3, 5, 8, 16, 33, 64, 100, 128, 200, 256, 300, 400, 520, 700, 1000, 2000, 4000, 8000, 16000, 32000, 65535):
            n = splits(b, q_len, hq, hkv, d, keys)
            each = one_split(b, q_len, hq, hkv, d)
            assert n <= before and (n == 1 or n * each <= MOST)
            # as many as one per 2048 keys, where they have room: the next one up would be past the limit
            assert n >= min(256, -(-keys // 2048)) or (n + 1) * each > MOST
            before = n


def test_just_below_and_above_the_limit():
    # 32 / 8 heads of 128, 262144 keys: 128 splits of 8 * 4224 bytes a request
    at = MOST // (128 * one_split(1, 1, 32, 8, 128))
    assert splits(at, 1, 32, 8, 128, 262144) == 128 and splits(at + 1, 1, 32, 8, 128, 262144) == MOST // one_split(at + 1, 1, 32, 8, 128) >= 120
    assert splits(520, 1, 32, 8, 128, 262144) == MOST // one_split(520, 1, 32, 8, 128) > 10
    assert splits(64, 1, 32, 8, 128, 131072) == 64                              # 138 MB: as it was
