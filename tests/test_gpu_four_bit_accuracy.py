"""What the 4-bit operators promise about their accuracy: as far from the 64-bit result as its own rounding to bf16, and hardly more.
The element-wise bounds of the other tests allow for the worst case of every rounding and leave room for much larger errors than
that; a norm over all outputs does not."""
import pytest
import torch

import _four_bit as F
import test_gpu_kv4 as K
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")

# The error is the last rounding's r and, independent of it, e of everything before: their norms add as squares, and 1.05 leaves
# e / r = 0.32.
WORST = 1.05


def error_ratio(got, want):
    """Norm of the error over the norm of the error of the 64-bit result rounded to bf16."""
    return float((got.double() - want).norm() / (want.to(torch.bfloat16).double() - want).norm())


# r is 2^-9.2 of an output (a rounding of at most 2^-9 of a number's power of two, on average).  Probabilities of 16 bits and scores
# of 23 leave e / r below 2^-6.  What is left are the accumulators, which hold the offset 16 + q of up to `b` tiles: two products a
# tile, each of which may drop up to 2^-23 of what the accumulator holds, half of that on average, all to one side.  Per output that is
# b * 24 * s * 2^-24 for a quantiser's step s of 0.4 of a value's deviation, and the output is sqrt(e / length) of that deviation:
# e / r = 0.21 for 16384 keys and b = 8, 0.30 for 131071 and b = 4, 0.23 for 1200000 and b = 1 (1.2 for 131071 and b = 28, all of a warp's
# tiles).
@pytest.mark.parametrize("lengths,Hq,Hkv,D,G,page,T", [
    ([700, 90, 2500], 16, 4, 128, 64, 64, 1), ([8192, 8000, 5001, 8192], 32, 8, 128, 64, 64, 4), ([16384, 16000], 16, 8, 128, 32, 64, 16),
    ([40000], 8, 1, 64, 32, 256, 1), ([131071], 16, 8, 128, 128, 64, 1), ([1200000], 4, 1, 64, 64, 256, 1)])
def test_attention_is_as_accurate_as_its_last_rounding(lengths, Hq, Hkv, D, G, page, T):
    c, table, n, k, v = K.filled(lengths, Hkv, D, page, G, 21)
    Q = K.bf16(K.gen(22), len(lengths) * T, Hq * D)
    O = gmlp.kv4_attention(Q, c, table, n, Hq, q_len=T, checked=True)
    want = F.attention(Q.double(), k, v, lengths, Hq, T, D ** -0.5)[0]
    ratio = error_ratio(O, want)
    assert ratio <= WORST, f"{ratio:.3f}"
