"""The tcgen05 form of the 4-bit products, instantiation by instantiation: every case asks gmlp_w4_plan first that this kernel is the one
that runs, with the rows, the cluster and the parts that the case is there for."""
import pytest
import torch

import _four_bit as F
import test_gpu_w4 as W
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
UMMA = 2


def plan(M, K, N, G, terms=1, gated=False):
    kind, rows, _, cluster, parts, _, _ = gmlp.w4_plan(M, K, N, G, terms=terms, gated=gated)
    return kind, rows, cluster, parts


# (tokens, K, N) -> rows of a CTA, CTAs per cluster, parts.  N ends inside a tile of 16, in a CTA's first tile (the other seven are the
# last tile again) or in its last; K + 32 (G = 32) leaves a k-block of which three quarters, and 4096 + 32 one more that is all zeros.
PLAIN = [(17, 14336, 4091, 32, 4, 1), (20, 14336, 4096, 32, 4, 1), (32, 8192, 5000, 32, 3, 1), (33, 14336, 4096, 64, 4, 1),
         (64, 8192, 5400, 64, 3, 1), (64, 8192, 9000, 64, 2, 1), (24, 8192, 12163, 32, 1, 1), (64, 1024, 14331, 64, 1, 1), (18, 1024, 18929, 32, 1, 1),
         (50, 4096, 20000, 64, 1, 1)]


@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("M,K,N,rows,cluster,parts", PLAIN)
def test_plain_products(M, K, N, rows, cluster, parts, G, zero_points):
    assert plan(M, K, N, G) == (UMMA, rows, cluster, parts)
    W.check_matmul(M, K, N, G, zero_points, seed=1)


@pytest.mark.parametrize("M,K,N,G,rows,cluster", [(20, 4096 + 32, 16384, 32, 32, 1), (64, 4096 + 96, 16383, 32, 64, 1), (40, 8192 + 32, 4100, 32, 64, 4),
                                                  (17, 8192 + 64, 9001, 64, 32, 2), (64, 4096 + 128, 12289, 128, 64, 1)])
def test_rows_that_leave_a_block_of_zeros(M, K, N, G, rows, cluster):
    assert plan(M, K, N, G) == (UMMA, rows, cluster, 1)
    W.check_matmul(M, K, N, G, True, seed=2)


# The two products of a layer: gated with one term (no norm) or two, and the down projection, which always has two.
LAYERS = [(9, 4096, 14336, True), (16, 4096, 14336, True), (17, 4096, 14336, True), (17, 4096, 14336, False), (32, 4096, 14336, False),
          (33, 4096, 14336, False), (64, 4096, 14336, True), (24, 2048, 6200, True), (40, 8192, 2080, False), (11, 1024, 8000, True)]


@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("M,D,Fd,norm", LAYERS)
def test_layers(M, D, Fd, norm, G):
    Fd = Fd // G * G
    D = D // G * G
    up, down = plan(M, D, Fd, G, 2 if norm else 1, True), plan(M, Fd, D, G, 2)
    assert up[0] == UMMA or down[0] == UMMA
    W.check_forward(M, D, Fd, G, G, M % 2 == 0, norm, norm, "silu")


def test_a_gated_product_with_a_block_of_zeros():
    M, D, Fd, G = 20, 4096 + 32, 6240, 32
    assert plan(M, D, Fd, G, 1, True)[:2] == (UMMA, 32)
    W.check_forward(M, D, Fd, G, G, True, False, False, "gelu")


def test_the_layers_above_reach_every_form():
    # rows 32 and 64, one and two terms, gated and not, one part and two, clusters of one to four
    seen = set()
    for G in (32, 64, 128):
        for M, K, N, *_ in PLAIN:
            seen.add(("plain", G, 1) + plan(M, K, N, G)[1:2])
        for M, D, Fd, norm in LAYERS:
            D, Fd = D // G * G, Fd // G * G
            for name, terms, p in (("gated", 2 if norm else 1, plan(M, D, Fd, G, 2 if norm else 1, True)), ("plain", 2, plan(M, Fd, D, G, 2))):
                if p[0] == UMMA:
                    seen.add((name, G, terms) + p[1:2])
    for G in (32, 64, 128):
        for rows in (32, 64):
            for name, terms in (("plain", 1), ("plain", 2), ("gated", 1), ("gated", 2)):
                assert (name, G, terms, rows) in seen, (name, G, terms, rows)


@pytest.mark.parametrize("K,N,M", [(14336, 4096, 20), (8192, 9000, 64), (4096, 16384, 33)])
def test_a_row_does_not_depend_on_its_neighbours(K, N, M):
    g = W.gen(K + N)
    q, s, z, _, _ = F.weights(g, K, N, 64, True, DEV)
    m = gmlp.w4_pack(q, s, z)
    X = W.bf16(g, M, K)
    assert plan(M, K, N, 64)[0] == UMMA
    first = gmlp.w4_matmul(X, m, checked=True)
    for r in (0, M // 2, M - 1):
        other = W.bf16(g, M, K, scale=100.0)
        other[(r + 1) % M] = float("inf")
        other[r] = X[r]
        assert torch.equal(gmlp.w4_matmul(other, m, checked=True)[r], first[r])


def test_repeats_streams_and_graphs():
    M, D, Fd, G = 24, 4096, 14336, 128
    g = W.gen(1)
    mats = [gmlp.w4_pack(*F.weights(g, K, N, G, False, DEV)[:3]) for K, N in ((D, Fd), (D, Fd), (Fd, D))]
    X = W.bf16(g, M, D)
    assert plan(M, D, Fd, G, 2, True)[0] == UMMA and plan(M, Fd, D, G, 2)[0] == UMMA
    first = gmlp.w4_forward(X, *mats, rmsnorm=True, checked=True)
    for _ in range(5):
        assert torch.equal(gmlp.w4_forward(X, *mats, rmsnorm=True), first)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [gmlp.w4_forward(X, *mats, rmsnorm=True, stream=side if i % 2 else None) for i in range(6)]       # two at once
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = gmlp.w4_forward(X, *mats, rmsnorm=True)
    for _ in range(3):
        o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, first)
    assert gmlp.device_status() == 0
