"""GPU parity of the 4-bit weight operators against the 64-bit definitions."""
import pytest
import torch

import _four_bit as F
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def bf16(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("K,N,G", [(32, 1, 32), (128, 16, 128), (160, 17, 32), (192, 130, 64), (256, 300, 128)])
def test_quantise_and_dequantise_are_exact(K, N, G, out_in, zero_points):
    g = gen(K + N)
    w = bf16(g, N, K)
    w[0, :G] = 0
    if N > 1:
        w[1, :G] = -2.5
        w[N - 1, K - 1], w[N // 2, 0] = float("inf"), float("nan")
    q, s, z = F.quantize(w, G, zero_points)
    want = F.values(q, s, z, G).to(torch.bfloat16)                       # [N, K]
    m = gmlp.w4_quantize(w if out_in else w.t().contiguous(), G, zero_points, weights_out_in=out_in, checked=True)
    got = gmlp.w4_dequantize(m, weights_out_in=True, checked=True)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
    assert torch.equal(gmlp.w4_dequantize(m).t().nan_to_num(0.0), want.nan_to_num(0.0))


@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("K,N,G", [(32, 3, 32), (320, 33, 64), (384, 48, 128), (1024, 1000, 32)])
def test_pack_round_trip(K, N, G, out_in, zero_points):
    q, s, z, w, _ = F.weights(gen(7 * K + N), K, N, G, zero_points, DEV)
    t = (lambda x: None if x is None else x.t().contiguous()) if out_in else (lambda x: x)
    m = gmlp.w4_pack(t(q), t(s), t(z), weights_out_in=out_in, checked=True)
    assert m.K == K and m.N == N and m.group == G
    assert torch.equal(gmlp.w4_dequantize(m, checked=True), w.to(torch.bfloat16))


def check_matmul(M, K, N, G, zero_points, seed=0):
    g = gen(1000 * seed + M + K + N + G)
    q, s, z, w, terms = F.weights(g, K, N, G, zero_points, DEV)
    X = bf16(g, M, K)
    Y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    gmlp.w4_matmul(X, gmlp.w4_pack(q, s, z), Y, checked=True)
    want = X.double() @ w
    bound = F.product_bound(X.double(), terms, G) + 2.0 ** -8 * want.abs()
    err = (Y.double() - want).abs() / bound
    assert bool(torch.isfinite(Y.float()).all()) and float(err.max()) <= 1.0, f"{float(err.max()):.3f} of the bound"


@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 128, 1), (1, 384, 16), (3, 640, 17), (8, 256, 33), (9, 1152, 47), (17, 384, 129), (64, 128, 31)])
def test_matmul_small_and_odd(M, K, N, G, zero_points):
    check_matmul(M, K, N, G, zero_points)


@pytest.mark.parametrize("M", list(range(1, 18)) + [23, 24, 25, 31, 32, 33, 40, 41, 47, 48, 49, 56, 57, 63, 64])
def test_matmul_every_token_count(M):
    check_matmul(M, 1024, 272, 64, M % 2 == 0)


@pytest.mark.parametrize("K,N,G", [(32, 64, 32), (96, 40, 32), (160, 100, 32), (2080, 48, 32), (4128, 20, 32), (192, 64, 64), (8256, 96, 64)])
@pytest.mark.parametrize("M", [1, 5, 16, 50])
def test_matmul_rows_that_do_not_fill_a_block_of_128(M, K, N, G):
    check_matmul(M, K, N, G, True)


@pytest.mark.parametrize("M,K,N,G", [(1, 2048, 2048, 128), (64, 4096, 4096, 128), (7, 5632, 2047, 64), (1, 8192, 28672, 32), (16, 28672, 1024, 128),
                                     (64, 28672, 64, 64), (40, 14336, 96, 32), (1, 28672, 40, 32), (2, 256, 28672, 64), (33, 4096, 6144, 64)])
def test_matmul_layer_sizes(M, K, N, G):
    check_matmul(M, K, N, G, G != 128)


def test_matmul_extreme_values_and_groups_of_zeros():
    K, N, G, M = 512, 96, 64, 6
    q, s, z, w, _ = F.weights(gen(3), K, N, G, True, DEV)
    s[:, 5] = 0
    s[3, 7] = float("nan")
    s[2, 9] = float("inf")
    X = bf16(gen(4), M, K)
    X[1, 100] = float("inf")
    X[2, 100] = float("nan")
    X[3] = 0
    Y = gmlp.w4_matmul(X, gmlp.w4_pack(q, s, z), checked=True).float()
    assert bool(torch.isnan(Y[2]).all()) and bool(torch.isnan(Y[:, 7]).all())
    assert not bool(torch.isfinite(Y[1, [c for c in range(N) if c != 5]]).any())
    rest = [c for c in range(N) if c not in (7, 9)]
    assert bool((Y[3, rest] == 0).all()) and bool((Y[[0, 3, 4, 5], 5] == 0).all())
    assert bool(torch.isfinite(Y[[0, 4, 5]][:, rest]).all())


def test_matmul_of_activations_near_the_largest_bf16():
    # (16 + q) x would overflow where (q - z) x does not: the sums of a row stay finite, and its neighbours exact
    K, N, G = 256, 64, 128
    q = torch.randint(7, 10, (K, N), generator=gen(1), device=DEV, dtype=torch.uint8)
    s = torch.full((2, N), 2.0 ** -20, dtype=torch.bfloat16, device=DEV)
    X = torch.zeros(3, K, device=DEV)
    X[0, 5], X[0, 200], X[1] = 2.5e38, -1.25e38, 1.0
    X = X.to(torch.bfloat16)
    Y = gmlp.w4_matmul(X, gmlp.w4_pack(q, s), checked=True)
    want = X.double() @ ((q.double() - 8) * 2.0 ** -20)
    assert bool(((Y.double() - want).abs() <= 2.0 ** -8 * want.abs()).all())


def test_matmul_of_every_code_and_zero_point():
    # X = identity rows pick single weights: the bf16 of (q - z) * s for all 256 pairs, exactly
    K, N, G = 64, 256, 64
    q = torch.arange(N, device=DEV).remainder(16).to(torch.uint8).expand(K, N).contiguous()
    z = (torch.arange(N, device=DEV) // 16).to(torch.uint8)[None].contiguous()
    s = torch.full((1, N), 0.171875, dtype=torch.bfloat16, device=DEV)
    X = torch.eye(K, device=DEV, dtype=torch.bfloat16)
    Y = gmlp.w4_matmul(X, gmlp.w4_pack(q, s, z), checked=True)
    want = ((q.double() - z.double()) * 0.171875).to(torch.bfloat16)
    assert torch.equal(Y, want)


ACT = {"silu": lambda g: g * torch.sigmoid(g), "swish": lambda g: g * torch.sigmoid(1.5 * g), "glu": torch.sigmoid,
       "gelu": lambda g: g * torch.special.ndtr(g)}


def check_forward(M, D, Fd, G, Gd, zero_points, norm, gain, act, eps=1e-5):
    g = gen(M + D + Fd + G)
    mats = [F.weights(g, D, Fd, G, zero_points, DEV), F.weights(g, D, Fd, G, zero_points, DEV), F.weights(g, Fd, D, Gd, not zero_points, DEV)]
    packed = [gmlp.w4_pack(*m[:3]) for m in mats]
    wg, wu, wd = (m[3] for m in mats)
    tg, tu, td = (m[4] for m in mats)
    X = bf16(g, M, D)
    gamma = (torch.rand(D, generator=g, device=DEV) + 0.5).to(torch.bfloat16) if gain else None
    Y = torch.full((M, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    gmlp.w4_forward(X, *packed, Y, gamma=gamma, eps=eps, rmsnorm=norm, act=act, beta=1.5, checked=True)
    x = X.double()
    slack = 0.0
    if norm:
        x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + eps) * (gamma.double() if gain else 1.0)
        # two bf16 terms leave 2^-17 of the value (2^-9 of 2^-8), the fp32 statistic and its products 2^-20
        slack = 2.0 ** -16
    a, u = x @ wg, x @ wu
    da, du = (F.product_bound(x, t, G) + slack * (x.abs() @ w.abs()) for w, t in ((wg, tg), (wu, tu)))
    h = ACT[act](a) * u
    # |act'| <= 1.2 for all four (GELU's largest slope is 1.13; swish with beta 1.5 stays below 1.1), fast exponential and
    # division 2^-19, two bf16 terms of h 2^-16
    dh = 1.2 * da * u.abs() + ACT[act](a).abs() * du + 1.2 * da * du + (2.0 ** -16 + 2.0 ** -19) * h.abs()
    want = h @ wd
    bound = dh @ wd.abs() + F.product_bound(h, td, Gd) + 2.0 ** -8 * want.abs()
    err = (Y.double() - want).abs() / bound
    assert float(err.max()) <= 1.0, f"{float(err.max()):.3f} of the bound"
    # the intermediate values keep their accuracy: the whole is hardly further off than its last rounding
    rel = float((Y.double() - want).norm() / want.norm())
    assert rel <= 2.0 ** -8


@pytest.mark.parametrize("act", ["silu", "swish", "glu", "gelu"])
@pytest.mark.parametrize("norm,gain", [(False, False), (True, False), (True, True)])
def test_forward_options(act, norm, gain):
    check_forward(5, 256, 512, 128, 64, False, norm, gain, act)


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 24, 33, 48, 64])
def test_forward_token_counts(M):
    check_forward(M, 384, 640, 64, 128, True, M % 2 == 1, True, "silu")


@pytest.mark.parametrize("M,D,Fd,G", [(1, 2048, 5632, 128), (8, 4096, 14336, 128), (33, 4096, 14336, 64), (1, 32, 32, 32), (3, 96, 160, 32),
                                      (64, 1024, 4096, 32)])
def test_forward_layer_sizes(M, D, Fd, G):
    check_forward(M, D, Fd, G, G, G != 128, True, True, "silu")


def test_forward_of_infinities():
    # an infinite activation gives what the formula gives, not a NaN made of the split into two terms
    D = Fd = 128
    q = torch.full((D, Fd), 9, dtype=torch.uint8, device=DEV)
    s = torch.ones(1, Fd, dtype=torch.bfloat16, device=DEV)
    m = gmlp.w4_pack(q, s)
    X = torch.zeros(2, D, dtype=torch.bfloat16, device=DEV)
    X[0, 3] = 3e38
    X[1, 3] = 1.0
    Y = gmlp.w4_forward(X, m, m, m, checked=True).float()
    assert bool((Y[0] == float("inf")).all()) and bool(torch.isfinite(Y[1]).all())


def test_results_repeat_and_empty_batches():
    q, s, z, _, _ = F.weights(gen(1), 2048, 1024, 128, False, DEV)
    m = gmlp.w4_pack(q, s, z)
    X = bf16(gen(2), 24, 2048)
    first = gmlp.w4_matmul(X, m)
    for _ in range(5):
        assert torch.equal(gmlp.w4_matmul(X, m), first)
    # a row's result does not depend on the rows beside it within one kernel
    assert gmlp.w4_matmul(X[:0], m).shape == (0, 1024)
    assert gmlp.w4_forward(X[:0], m, m, gmlp.w4_pack(*F.weights(gen(3), 1024, 2048, 128, False, DEV)[:2])).shape == (0, 2048)


def test_streams_graphs_and_weights_made_just_before():
    K, N = 1024, 768
    side = torch.cuda.Stream()
    w = bf16(gen(8), K, N, scale=K ** -0.5)
    X = bf16(gen(9), 4, K)
    q, s, z = F.quantize(w.t(), 128, False)
    want = X.double() @ F.values(q, s, z, 128).t()
    close = lambda y: bool(((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3).all())
    torch.cuda.synchronize()
    for _ in range(20):                                  # quantised on the stream right before the product, memory reused
        m = gmlp.w4_quantize(w, 128, stream=side)
        y = gmlp.w4_matmul(X, m, stream=side)
        side.synchronize()
        assert close(y)
        m.codes.fill_(0)
        torch.cuda.synchronize()
        del m
    m = gmlp.w4_quantize(w, 128)
    up = gmlp.w4_quantize(w, 128)
    down = gmlp.w4_quantize(w.t().contiguous(), 128)
    eager = gmlp.w4_forward(X, m, up, down, rmsnorm=True)
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y1 = gmlp.w4_matmul(X, m)
        y2 = gmlp.w4_forward(X, m, up, down, rmsnorm=True)
    with torch.cuda.graph(other):
        y3 = gmlp.w4_forward(X, m, up, down, rmsnorm=True)
    for _ in range(3):
        y1.fill_(7), y2.fill_(7), y3.fill_(7)
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        assert close(y1) and torch.equal(y2, eager) and torch.equal(y3, eager)
    X.mul_(-2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y2, gmlp.w4_forward(X, m, up, down, rmsnorm=True))


def test_binding_refusals():
    q, s, z, _, _ = F.weights(gen(1), 256, 64, 128, False, DEV)
    m = gmlp.w4_pack(q, s, z)
    X = bf16(gen(2), 4, 256)
    for bad in (X.float(), X.t().contiguous().t(), X.cpu()):
        with pytest.raises(TypeError):
            gmlp.w4_matmul(bad, m)
    with pytest.raises(ValueError):
        gmlp.w4_matmul(X[:, :128].contiguous(), m)
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.w4_matmul(bf16(gen(2), 65, 256), m)
    assert e.value.status == gmlp.ERR_SHAPE
    with pytest.raises(ValueError):
        gmlp.w4_matmul(X, m, Y=torch.empty(4, 63, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        gmlp.w4_pack(q, s, torch.zeros(1, 64, dtype=torch.uint8, device=DEV))
    with pytest.raises(gmlp.GmlpError):
        gmlp.w4_quantize(X, 48)
    with pytest.raises(gmlp.GmlpError) as e:
        gmlp.w4_forward(X, m, m, m)                      # the down projection has the wrong shape
    assert e.value.status == gmlp.ERR_SHAPE
    torch.cuda.synchronize()
    assert gmlp.device_status() == 0
