"""Host-side checks of the 4-bit operators that need no GPU: sizes, refusals before any device work, workspace arithmetic,
the struct layouts, and the plain definitions the GPU tests rely on."""
import ctypes
import os
import subprocess

import pytest
import torch

import _four_bit as F
from paper_2606_26344_b200 import build as B
from paper_2606_26344_b200 import gmlp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    B.build_libgmlp()
    return gmlp.lib()


def matrix(K=256, N=64, group=128, **kw):
    m = gmlp.GmlpW4Matrix(0x10000, 0x20000, None, K, N, group, 0)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


def cache(**kw):
    c = gmlp.GmlpKv4Cache(0x10000, 0x20000, 0x30000, 0x40000, 10, 2, 64, 128, 64, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def call(entry, a, **kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return entry(ctypes.byref(a))


BAD_MATRICES = [(dict(group=16), gmlp.ERR_SHAPE), (dict(group=0), gmlp.ERR_SHAPE), (dict(group=96), gmlp.ERR_SHAPE),
                (dict(K=200), gmlp.ERR_SHAPE), (dict(K=0), gmlp.ERR_SHAPE), (dict(N=0), gmlp.ERR_SHAPE), (dict(K=-128), gmlp.ERR_SHAPE),
                (dict(N=(1 << 20) + 1), gmlp.ERR_SHAPE), (dict(K=1 << 21), gmlp.ERR_SHAPE), (dict(codes=None), gmlp.ERR_NULL),
                (dict(scales=None), gmlp.ERR_NULL), (dict(codes=0x10008), gmlp.ERR_ALIGN), (dict(scales=0x20002), gmlp.ERR_ALIGN),
                (dict(zeros=0x30001), gmlp.ERR_ALIGN), (dict(reserved=1), gmlp.ERR_FLAGS)]


def test_w4_sizes(lib):
    # tiles of 16 columns by 128 rows, a kilobyte each, an even number of them along K
    assert gmlp.w4_sizes(128, 16, 128) == (2048, 32)
    assert gmlp.w4_sizes(160, 17, 32) == (2 * 2 * 1024, 2 * 2 * 16 * 4)
    assert gmlp.w4_sizes(4096, 14336, 64) == (4096 * 14336 // 2, 4096 * 14336 // 64)
    for K, N, G in ((0, 16, 128), (128, 0, 128), (100, 16, 32), (128, 16, 48), (1 << 21, 16, 128)):
        with pytest.raises(gmlp.GmlpError) as e:
            gmlp.w4_sizes(K, N, G)
        assert e.value.status == gmlp.ERR_SHAPE
    assert lib.gmlp_w4_code_bytes(-1, 5) == 0 and lib.gmlp_w4_scale_count(128, 16, 0) == 0


def matmul_args():
    return gmlp.GmlpW4MatmulArgs(ctypes.sizeof(gmlp.GmlpW4MatmulArgs), 0, 0x1000, 0x2000, 4, matrix(), None)


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=1), gmlp.ERR_FLAGS), (dict(M=-1), gmlp.ERR_SHAPE),
                                       (dict(M=65), gmlp.ERR_SHAPE), (dict(M=0, X=None, Y=None), gmlp.OK), (dict(X=None), gmlp.ERR_NULL),
                                       (dict(Y=None), gmlp.ERR_NULL), (dict(X=0x1008), gmlp.ERR_ALIGN), (dict(Y=0x2002), gmlp.ERR_ALIGN)] +
                         [(dict(W=matrix(**m)), s) for m, s in BAD_MATRICES])
def test_w4_matmul_refusals(lib, kw, status):
    assert call(lib.gmlp_w4_matmul, matmul_args(), **kw) == status


def forward_args():
    a = gmlp.GmlpW4Args()
    a.struct_bytes = ctypes.sizeof(gmlp.GmlpW4Args)
    a.X, a.Y, a.M = 0x1000, 0x2000, 4
    a.Wg, a.Wu, a.Wd = matrix(256, 512), matrix(256, 512), matrix(512, 256)
    a.rms_eps, a.act_beta = 1e-5, 1.0
    a.workspace, a.workspace_bytes = 0x100000, 1 << 20
    return a


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=gmlp.FLAG_Y_FP32), gmlp.ERR_FLAGS),
                                       (dict(flags=gmlp.FLAG_ACT_GLU | gmlp.FLAG_ACT_GELU), gmlp.ERR_FLAGS),
                                       (dict(flags=gmlp.FLAG_ACT_SWISH, act_beta=float("nan")), gmlp.ERR_FLAGS),
                                       (dict(reserved=1), gmlp.ERR_FLAGS), (dict(M=65), gmlp.ERR_SHAPE), (dict(M=-1), gmlp.ERR_SHAPE),
                                       (dict(M=0, X=None), gmlp.OK), (dict(X=None), gmlp.ERR_NULL), (dict(workspace=None), gmlp.ERR_NULL),
                                       (dict(workspace=0x100010), gmlp.ERR_ALIGN), (dict(workspace_bytes=100), gmlp.ERR_WORKSPACE),
                                       (dict(rms_gain=0x1001), gmlp.ERR_ALIGN),
                                       (dict(Wu=matrix(256, 384)), gmlp.ERR_SHAPE), (dict(Wu=matrix(256, 512, 64)), gmlp.ERR_SHAPE),
                                       (dict(Wu=matrix(256, 512, zeros=0x30000)), gmlp.ERR_SHAPE), (dict(Wd=matrix(512, 128)), gmlp.ERR_SHAPE),
                                       (dict(Wd=matrix(384, 256)), gmlp.ERR_SHAPE)] +
                         [(dict(Wg=matrix(**m)), s) for m, s in BAD_MATRICES])
def test_w4_forward_refusals(lib, kw, status):
    assert call(lib.gmlp_w4_forward, forward_args(), **kw) == status


def test_w4_layout_refusals(lib):
    make = lambda: gmlp.GmlpW4LayoutArgs(ctypes.sizeof(gmlp.GmlpW4LayoutArgs), 0, 0x1000, 0x2000, None, matrix(), None)
    for entry in (lib.gmlp_w4_quantize, lib.gmlp_w4_pack, lib.gmlp_w4_dequantize):
        assert entry(None) == gmlp.ERR_NULL
        assert call(entry, make(), struct_bytes=4) == gmlp.ERR_FLAGS
        assert call(entry, make(), flags=1) == gmlp.ERR_FLAGS
        assert call(entry, make(), W=None) == gmlp.ERR_NULL
        for m, s in BAD_MATRICES:
            assert call(entry, make(), m=matrix(**m)) == s
    assert call(lib.gmlp_w4_pack, make(), scales=None) == gmlp.ERR_NULL
    assert call(lib.gmlp_w4_pack, make(), zeros=0x3000) == gmlp.ERR_NULL                     # given, but nowhere to put them
    assert call(lib.gmlp_w4_pack, make(), m=matrix(zeros=0x30000)) == gmlp.ERR_NULL          # wanted, but not given
    assert lib.gmlp_w4_matmul(None) == gmlp.ERR_NULL and lib.gmlp_w4_forward(None) == gmlp.ERR_NULL


@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("G", [32, 64, 128])
def test_w4_plan_of_every_size(lib, terms, gated, G):
    """Every launch shape covers its rows, fits a CTA's shared memory (227 KB) and keeps its cluster's CTAs busy."""
    block = 1024 + 48 * (128 // G)                               # codes, scales, zero points of a tile's k-block
    for M in range(1, gmlp.W4_MAX_M + 1):
        for K in (128, 256, 1024, 2048 + 128, 4096, 4096 + 128, 8192, 11008, 14336, 28672, 1 << 20):
            for N in (1, 16, 20, 33, 48, 64, 100, 256, 1000, 4096, 14336, 28672, 1 << 20):
                kind, rpad, gw, c, parts, ctas, smem = gmlp.w4_plan(M, K, N, G, terms, gated, 148)
                kb, tiles, m_cta = -(-K // 256) * 2, -(-N // 16), -(-M // parts)
                rows = m_cta * terms
                assert rpad >= rows and (parts - 1) * m_cta < M and smem <= 227 * 1024 and 1 <= c <= 4
                if kind == 0:                                    # per warp: its sums and a ring of two or three; sums of X, all of X
                    assert rpad in (8, 16) and rows > rpad - 8 and parts == 1 and c == 1 and gw in (2, 4, 8, 16) and ctas == min(tiles, 148)
                    assert smem >= 16 * (512 + (3 if rpad == 8 else 2) * 2 * block) + kb * 128 // G * rpad * 4 + rows * (kb * 256 + 64)
                elif kind == 1:                                  # three stages of X and codes, then the sums of eight warps
                    wk = 8 // gw
                    assert rows <= 32 and rows > rpad - 8 and gw in (1, 2, 4, 8) and (c == 1 or kb >= 2 * wk * c) and parts <= 4
                    assert smem >= 3 * (rows * (wk * 256 + 64) + 16 * block) and smem >= 8 * 32 * 8 * (rpad // 8 | 1) * 4
                    assert ctas == c * -(-(-(-N // (16 if gated else 32))) // gw)
                else:
                    assert kind == 2 and M * terms > 16 and rpad in (32, 64) and (c == 1 or kb >= 8 * c) and 1 <= parts <= 2
                    assert ctas == c * -(-tiles // (4 if gated else 8)) and (c == 1 or ctas * parts <= 148)
                    # three buffers of A, four stages of X and codes, the sums in place of A, eighteen barriers
                    assert smem >= 1024 + 3 * 32768 + 4 * (rpad * 256 + 8 * 1024) + 19 * 8 and 3 * 32768 >= 128 * (rpad + 1) * 4
                    assert 2 * (128 // G) * rpad <= 512              # columns of TMEM
    out = (ctypes.c_int32 * 7)()
    for bad in ((65, 1, 128, 16, 0, 128), (0, 1, 128, 16, 0, 128), (1, 3, 128, 16, 0, 128), (1, 1, 0, 16, 0, 128), (1, 1, 128, 16, 0, 48)):
        assert lib.gmlp_w4_plan(*bad, 148, out) == gmlp.ERR_SHAPE
    assert lib.gmlp_w4_plan(1, 1, 128, 16, 0, 128, 148, None) == gmlp.ERR_NULL


def test_w4_workspace(lib):
    wb = gmlp.w4_workspace_bytes
    assert wb(8, 4096, 14336) >= 8 * 14336 * 4 and wb(8, 4096, 14336, True) >= 8 * (14336 + 4096) * 4
    assert wb(65, 4096, 14336) == 0 and wb(-1, 4096, 14336) == 0 and wb(8, 0, 14336) == 0
    a = forward_args()
    need = wb(4, 256, 512, True)
    assert call(lib.gmlp_w4_forward, a, flags=gmlp.FLAG_RMSNORM, workspace_bytes=need - 1) == gmlp.ERR_WORKSPACE


BAD_CACHES = [(dict(head_dim=96), gmlp.ERR_UNSUPPORTED), (dict(head_dim=256), gmlp.ERR_UNSUPPORTED), (dict(group=16), gmlp.ERR_SHAPE),
              (dict(head_dim=64, group=128), gmlp.ERR_SHAPE), (dict(page_size=24), gmlp.ERR_SHAPE), (dict(page_size=0), gmlp.ERR_SHAPE),
              (dict(page_size=8), gmlp.ERR_SHAPE), (dict(n_pages=0), gmlp.ERR_SHAPE), (dict(n_pages=1 << 26), gmlp.ERR_SHAPE),
              (dict(n_pages=1 << 60), gmlp.ERR_SHAPE), (dict(n_pages=-1), gmlp.ERR_SHAPE),
              (dict(n_kv_heads=0), gmlp.ERR_SHAPE), (dict(k_codes=None), gmlp.ERR_NULL), (dict(v_params=None), gmlp.ERR_NULL),
              (dict(v_codes=0x30008), gmlp.ERR_ALIGN), (dict(reserved=1), gmlp.ERR_FLAGS)]


def test_kv4_rows_refusals(lib):
    make = lambda: gmlp.GmlpKv4RowsArgs(ctypes.sizeof(gmlp.GmlpKv4RowsArgs), 0, 0x1000, 0x2000, 0x3000, 5, cache(), None)
    for entry in (lib.gmlp_kv4_append, lib.gmlp_kv4_gather):
        assert entry(None) == gmlp.ERR_NULL
        assert call(entry, make(), struct_bytes=4) == gmlp.ERR_FLAGS
        assert call(entry, make(), flags=1) == gmlp.ERR_FLAGS
        assert call(entry, make(), T=-1) == gmlp.ERR_SHAPE
        assert call(entry, make(), T=(1 << 24) + 1) == gmlp.ERR_SHAPE
        assert call(entry, make(), T=0, K=None, V=None, slots=None) == gmlp.OK
        assert call(entry, make(), K=None) == gmlp.ERR_NULL
        assert call(entry, make(), slots=None) == gmlp.ERR_NULL
        assert call(entry, make(), V=0x2008) == gmlp.ERR_ALIGN
        assert call(entry, make(), slots=0x3004) == gmlp.ERR_ALIGN
        for c, s in BAD_CACHES:
            assert call(entry, make(), cache=cache(**c)) == s


def attention_args():
    a = gmlp.GmlpKv4AttentionArgs()
    a.struct_bytes = ctypes.sizeof(gmlp.GmlpKv4AttentionArgs)
    a.Q, a.O, a.block_table, a.lengths = 0x1000, 0x2000, 0x3000, 0x4000
    a.cache = cache()
    a.B, a.table_width, a.n_q_heads, a.q_len, a.scale = 3, 4, 8, 1, 0.1
    return a


@pytest.mark.parametrize("kw,status", [(dict(struct_bytes=8), gmlp.ERR_FLAGS), (dict(flags=1 << 4), gmlp.ERR_FLAGS), (dict(reserved=1), gmlp.ERR_FLAGS),
                                       (dict(scale=float("inf")), gmlp.ERR_FLAGS), (dict(scale=float("nan")), gmlp.ERR_FLAGS),
                                       (dict(B=-1), gmlp.ERR_SHAPE), (dict(B=65536), gmlp.ERR_SHAPE), (dict(q_len=0), gmlp.ERR_SHAPE),
                                       (dict(q_len=17), gmlp.ERR_SHAPE), (dict(n_q_heads=7), gmlp.ERR_SHAPE), (dict(n_q_heads=0), gmlp.ERR_SHAPE),
                                       (dict(table_width=0), gmlp.ERR_SHAPE), (dict(table_width=1 << 40), gmlp.ERR_SHAPE),
                                       (dict(table_width=(1 << 24) + 1), gmlp.ERR_SHAPE),
                                       (dict(B=0, Q=None, O=None), gmlp.OK), (dict(Q=None), gmlp.ERR_NULL), (dict(lengths=None), gmlp.ERR_NULL),
                                       (dict(O=0x2008), gmlp.ERR_ALIGN), (dict(block_table=0x3002), gmlp.ERR_ALIGN),
                                       (dict(workspace=0x100), gmlp.ERR_ARCH if not torch.cuda.is_available() else gmlp.ERR_WORKSPACE),
                                       (dict(workspace=0x110), gmlp.ERR_ALIGN)] +
                         [(dict(cache=cache(**c)), s) for c, s in BAD_CACHES])
def test_kv4_attention_refusals(lib, kw, status):
    assert call(lib.gmlp_kv4_attention, attention_args(), **kw) == status
    assert lib.gmlp_kv4_attention(None) == gmlp.ERR_NULL


def test_kv4_workspace(lib):
    wb = gmlp.kv4_workspace_bytes
    # one split needs none; a long context is split, each split leaves head_dim + 4 floats per query row
    assert wb(1, 1, 8, 8, 128, 1, 64, 148) == 0
    n = wb(1, 1, 64, 8, 128, 2048, 64, 148)
    assert n > 0 and n % (8 * 8 * (128 + 4) * 4) == 0
    assert wb(1, 1, 64, 8, 128, 2048, 64, 148) <= 256 * 8 * 8 * 132 * 4
    for bad in ((0, 1, 8, 8, 128, 4, 64), (1, 17, 8, 8, 128, 4, 64), (1, 1, 7, 8, 128, 4, 64), (1, 1, 8, 8, 80, 4, 64), (1, 1, 8, 8, 128, 0, 64),
                (1, 1, 8, 8, 128, 4, 20)):
        assert wb(*bad, 148) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device behaviour")
def test_no_device_means_arch_error(lib):
    assert call(lib.gmlp_w4_matmul, matmul_args()) == gmlp.ERR_ARCH
    assert call(lib.gmlp_w4_forward, forward_args()) == gmlp.ERR_ARCH
    assert call(lib.gmlp_kv4_attention, attention_args()) == gmlp.ERR_ARCH


def test_binding_refuses_host_tensors_and_bad_shapes(lib):
    with pytest.raises(TypeError):
        gmlp.w4_quantize(torch.zeros(128, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        gmlp.w4_pack(torch.zeros(100, 16, dtype=torch.uint8), torch.zeros(3, 16, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        gmlp.w4_pack(torch.zeros(128, 16, dtype=torch.uint8), torch.zeros(1, 16, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        gmlp.kv4_cache(2, 2, device="cpu")
    with pytest.raises(ValueError):
        gmlp.Kv4Cache(torch.zeros(2, 2, 16), *[torch.zeros(1)] * 3)
    assert gmlp.status_string(gmlp.ERR_INDEX) != "unknown status"


def test_struct_layouts_match_the_header(lib, tmp_path):
    names = dict(gmlp_w4_matrix=gmlp.GmlpW4Matrix, gmlp_w4_layout_args=gmlp.GmlpW4LayoutArgs, gmlp_w4_matmul_args=gmlp.GmlpW4MatmulArgs,
                 gmlp_w4_args=gmlp.GmlpW4Args, gmlp_kv4_cache=gmlp.GmlpKv4Cache, gmlp_kv4_rows_args=gmlp.GmlpKv4RowsArgs,
                 gmlp_kv4_attention_args=gmlp.GmlpKv4AttentionArgs)
    lines = []
    for c, py in names.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{f[0]} %zu\\n", offsetof({c}, {f[0]}));' for f in py._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gmlp.h"\nint main(void) {' + "\n".join(lines) +
                   "return GMLP_W4_MAX_M - %d + GMLP_KV4_MAX_QUERIES - %d + GMLP_ERR_INDEX - (%d);}\n" %
                   (gmlp.W4_MAX_M, gmlp.KV4_MAX_QUERIES, gmlp.ERR_INDEX))
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    got = dict(line.split() for line in out.splitlines())
    for c, py in names.items():
        assert int(got[c]) == ctypes.sizeof(py)
        for f in py._fields_:
            assert int(got[f"{c}.{f[0]}"]) == getattr(py, f[0]).offset


def test_every_declared_four_bit_entry_is_exported(lib):
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gmlp.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(gmlp_(?:w4|kv4)_[a-z_0-9]+)\s*\(", text))
    assert len(names) == 13 and all(hasattr(lib, n) for n in names)


@pytest.mark.parametrize("D", [64, 128])
def test_plain_channel_order_round_trip(D):
    q = torch.randint(0, 16, (5, D), dtype=torch.uint8, generator=torch.Generator().manual_seed(D))
    b = F.pack_rows(q)
    assert torch.equal(F.unpack_rows(b), q)
    unit = b.view(torch.uint16 if D == 128 else torch.uint8).to(torch.int64)
    for c in (0, 1, 31, 32, 33, 63, D - 1):
        assert torch.equal((unit[:, c % 32] >> (4 * (c // 32))) & 15, q[:, c].to(torch.int64))


def test_plain_quantiser_properties():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 128, generator=g).to(torch.bfloat16)
    x[0] = 0
    x[1] = 3.0
    x[2, 5], x[3, 77] = float("inf"), float("nan")
    q, s, z = F.quantize(x, 64)
    v = F.values(q, s, z, 64)
    assert bool((v[0] == 0).all()) and bool(torch.isnan(v[2, :64]).all()) and bool(torch.isnan(v[3, 64:]).all())
    assert bool(torch.isfinite(v[2, 64:]).all()) and bool(((v[1] - 3).abs() <= 2.0 ** -8 * 3).all())
    # half a step inside the range; at its end, where the rounded scale may fall short, up to a step and the scale's rounding
    step = s.double().repeat_interleave(64, -1)
    ok = torch.isfinite(step)
    assert bool(((v - x.double()).abs()[ok] <= (1.0 + 15 * 2.0 ** -8) * step[ok]).all())
    q, s, z = F.quantize(x[4:], 32, zero_points=False)
    assert bool((z == 8).all()) and int(q.min()) >= 1


def test_a_scale_that_overflows_in_powers_of_two_is_refused():
    """The kernel multiplies scores by scale * log2(e): 3e38 is a float, 4.3e38 is not, and inf * 0 would be NaN."""
    a = attention_args()
    a.scale = 3e38
    assert gmlp.lib().gmlp_kv4_attention(ctypes.byref(a)) == gmlp.ERR_FLAGS
    a.scale, a.B = 2e38, 0
    assert gmlp.lib().gmlp_kv4_attention(ctypes.byref(a)) == gmlp.OK
