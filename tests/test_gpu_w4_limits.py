"""The 4-bit products at the ends of what they accept: the longest K and N, and matrices of more than four gigabytes."""
import pytest
import torch

import _four_bit as F
import test_gpu_w4 as W
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("M,K,N,G", [(1, 1 << 20, 16, 128), (3, 1 << 20, 17, 32), (16, (1 << 20) - 32, 40, 32), (20, 1 << 20, 130, 64), (64, 1 << 20, 16, 128),
                                     (1, 32, 1 << 20, 32), (16, 64, (1 << 20) - 1, 64), (17, 128, 1 << 20, 128), (64, 160, (1 << 20) - 5, 32)])
def test_longest_rows_and_columns(M, K, N, G):
    W.check_matmul(M, K, N, G, True, seed=3)


@pytest.mark.parametrize("M,D,Fd,G", [(1, 32, 1 << 20, 32), (20, 64, (1 << 20) - 64, 64), (2, 1 << 18, 128, 128), (40, 1 << 18, 64, 64)])
def test_layers_of_the_largest_sizes(M, D, Fd, G):
    W.check_forward(M, D, Fd, G, G, True, True, False, "silu")


def test_a_matrix_past_four_gigabytes():
    # 4.6 GB of codes; some columns of it, the first and the last among them, against the definition
    K, N, G = 65536, 140003, 64
    g = W.gen(1)
    w = torch.empty(K, N, dtype=torch.bfloat16, device=DEV)
    for k in range(0, K, 4096):
        w[k:k + 4096] = torch.randn(4096, N, generator=g, device=DEV).mul_(K ** -0.5)
    m = gmlp.w4_quantize(w, G, True, checked=True)
    assert m.codes.numel() > 1 << 32
    cols = torch.tensor([0, 1, 15, 16, 65535, 65536, 100000, 131071, 131072, N - 20, N - 17, N - 2, N - 1], device=DEV)
    picked = w[:, cols].t().contiguous()
    q, s, z = F.quantize(picked, G)
    ref = F.values(q, s, z, G).t()
    terms = ((32 + q.double().unflatten(-1, (-1, G)) + z.double()[..., None]) * s.double().abs()[..., None]).flatten(-2).t()
    back = gmlp.w4_dequantize(m, W=w, checked=True)
    assert torch.equal(back[:, cols], ref.to(torch.bfloat16))
    for M in (1, 8, 20, 64):
        X = W.bf16(g, M, K)
        Y = gmlp.w4_matmul(X, m, checked=True)
        want = X.double() @ ref
        bound = F.product_bound(X.double(), terms, G) + 2.0 ** -8 * want.abs()
        assert bool(((Y[:, cols].double() - want).abs() <= bound).all()), M
    del w, back, m
    torch.cuda.empty_cache()                         # 27 GB
