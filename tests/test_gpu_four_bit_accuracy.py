"""What the 4-bit operators promise about their accuracy: as far from the 64-bit result as its own rounding to bf16, and hardly more.
The element-wise bounds of the other tests allow for the worst case of every rounding and leave room for much larger errors than
that; a norm over all outputs does not."""
import pytest
import torch

import _four_bit as F
import test_gpu_kv4 as K
import test_gpu_w4 as W
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


# Products of the weights: exact terms, fp32 sums of a group (24 times the largest part of which, the offset, is off by 2^-24 a step and
# comes off again), e / r below 2^-6.  The Gated MLP adds two bf16 terms for the normed input and the gated product, 2^-17 of each
# term (rounded to one, 2^-9 each, the error was about twice the last rounding's), the fast exponential 2^-19: below 2^-5.
@pytest.mark.parametrize("G", [32, 128])
@pytest.mark.parametrize("M,K,N", [(1, 8192, 4096), (8, 4096, 4096), (16, 2048, 2050), (24, 4096, 4096), (24, 14336, 4096), (64, 4096, 14336)])
def test_products_are_as_accurate_as_their_last_rounding(M, K, N, G):
    g = W.gen(K + M)
    q, s, z, w, _ = F.weights(g, K, N, G, True, DEV)
    X = W.bf16(g, M, K)
    ratio = error_ratio(gmlp.w4_matmul(X, gmlp.w4_pack(q, s, z), checked=True), X.double() @ w)
    assert ratio <= WORST, f"{ratio:.3f}"


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu", "glu"])
@pytest.mark.parametrize("M,D,Fd,G", [(1, 2048, 5632, 128), (4, 512, 1024, 32), (8, 4096, 14336, 64), (13, 1024, 4096, 128), (33, 4096, 14336, 64),
                                      (64, 2048, 4096, 32)])
def test_the_gated_mlp_is_as_accurate_as_its_last_rounding(M, D, Fd, G, act, norm):
    g = W.gen(M + D)
    mats = [F.weights(g, D, Fd, G, False, DEV), F.weights(g, D, Fd, G, False, DEV), F.weights(g, Fd, D, G, True, DEV)]
    X = W.bf16(g, M, D)
    gamma = (torch.rand(D, generator=g, device=DEV) + 0.5).to(torch.bfloat16) if norm else None
    Y = gmlp.w4_forward(X, *(gmlp.w4_pack(*m[:3]) for m in mats), gamma=gamma, rmsnorm=norm, act=act, checked=True)
    x = X.double()
    if norm:
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5) * gamma.double()
    ratio = error_ratio(Y, (W.ACT[act](x @ mats[0][3]) * (x @ mats[1][3])) @ mats[2][3])
    assert ratio <= WORST, f"{ratio:.3f}"


@pytest.mark.parametrize("M,K,N", [(1, 2048, 1024), (5, 4096, 4096), (16, 1024, 520), (3, 28672, 520), (40, 2048, 1000)])
def test_a_row_does_not_depend_on_its_neighbours(M, K, N):
    g = W.gen(K + N)
    q, s, z, _, _ = F.weights(g, K, N, 64, True, DEV)
    m = gmlp.w4_pack(q, s, z)
    assert gmlp.w4_plan(M, K, N, 64)[0] in (0, 1)    # the other forms; the tcgen05 one has its own test
    X = W.bf16(g, M, K)
    first = gmlp.w4_matmul(X, m, checked=True)
    for r in {0, M // 2, M - 1}:
        other = W.bf16(g, M, K, scale=100.0)
        other[r] = X[r]
        assert torch.equal(gmlp.w4_matmul(other, m, checked=True)[r], first[r])
