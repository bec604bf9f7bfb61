// Products with 4-bit weights for a few tokens:  Y[m, n] = sum_k X[m, k] * (q[k, n] - z[k / G, n]) * s[k / G, n],
// q in 0..15, one scale s (bf16) and one zero point z (0..15; 8 without stored zero points) per group of G = 32, 64 or 128
// input rows.  Bound by HBM: the codes are read once, half a byte per weight.
//
// Storage (made once by the pack kernels below): tiles of 16 output columns x 128 input rows, 1 KB each, [N / 16][K / 128],
// so that the stream of a warp is contiguous.  In a tile, lane 4 g + t of a warp finds its 16 bytes for column g at
// 16 * lane and for column g + 8 at 512 + 16 * lane: eight 16-bit units r = 8 t .. 8 t + 7, unit r holding the codes of
// k = r, r + 32, r + 64, r + 96 in its four nibbles.  One shift and one and-or turn a 32-bit word into two bf16 numbers
// 128 + q (128..255 has a step of one in bf16); subtracting 128 + z leaves q - z exactly.  Those pairs are A operands of
// mma.m16n8k16 as they are, columns of W as its 16 rows and tokens as its 8 columns; the k order they imply
// (32 j + 8 t + 0..7) makes the matching B operand 16 contiguous bytes of a row of X.  Products of a group are summed in
// fp32 by the tensor core, then scaled in fp32: no weight is ever rounded.
//
// A warp takes two tiles at a time (two neighbouring column tiles, or the gate and the up tile of the same columns), so one
// B operand serves both; the 8 warps of a CTA are WR column groups x WK ranges of K, and a cluster of C CTAs splits K
// further; both partial sums are added in a fixed order (shared memory, then distributed shared memory).
// X may come as two bf16 terms (hi + lo, 16 bits of significand): activations that are not bf16 by nature - the normed
// input, the gated product - keep the accuracy of the fp32 they were computed in; both terms go into the same accumulator.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "umma_gemm_2cta.cuh"

namespace gmlp {

constexpr int kW4Threads = 256;
constexpr int kW4MaxM = 64;

struct W4Operand {
    const uint8_t* codes;
    const bf16* scales;        // [N / 16][K / 128][16][128 / G]
    const uint8_t* zeros;      // the same shape, or nullptr
};
struct W4GemmArgs {
    W4Operand w[2];            // gated: gate and up; else w[0] only
    const bf16* X;             // [terms][M][K]
    bf16* out;                 // plain: [M][N]; gated: [2][M][N], hi and lo of the gated product
    int M, K, N, KB, n16, terms;
    int wr_log2, cluster, chunk;           // column groups per CTA; CTAs per cluster; steps (WK k-blocks each) of X per chunk
    int early;                 // the weights may be fetched before the preceding kernel of the call has ended
    GateAct act;
};

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t bf16x2_sub(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The codes of nibble `j` of both halves of a word as bf16 (128 + q), then minus `zc` (128 + z in both halves).
template <int SHIFT>
__device__ __forceinline__ uint32_t codes_to_bf16x2(uint32_t w, uint32_t zc) {
    return bf16x2_sub(((w >> SHIFT) & 0x000F000Fu) | 0x43004300u, zc);
}
__device__ __forceinline__ void cp_async_16_zfill(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Loads of codes and parameters.  Volatile, so that none moves ahead of griddepcontrol.wait; plain (not .nc) because the kernel
// before, which may have written them, can still be running when this one starts.
__device__ __forceinline__ uint4 ld_once_16B(const void* p) {                 // codes: read once, kept out of L1
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 ld_16B(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ld_8B(const void* p) {
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_4B(const void* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_2B(const void* p) {
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_1B(const void* p) {
    uint32_t v;
    asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

template <int G>
struct W4Stage {                                     // one k-block (128) of a warp's two tiles
    uint4 c[2][2];                                   // [tile][column half]
    uint32_t s[2][2][G == 32 ? 2 : 1];               // 128 / G scales of the lane's columns g and g + 8
    uint32_t z[2][2];                                // 128 / G zero points, one byte each
};

__host__ __device__ constexpr int w4_prefetch(int nt) { return nt <= 8 ? 2 : 1; }      // k-blocks in flight per warp
__host__ __device__ constexpr int w4_red_stride(int nt) { return 8 * (nt | 1); }      // floats; odd multiples of 8 spread the banks
__host__ __device__ constexpr uint32_t w4_red_bytes(int nt) { return 8u * 32u * (uint32_t)w4_red_stride(nt) * 4u; }

template <int NT, int G, bool GATED>
__global__ void __launch_bounds__(kW4Threads, NT <= 2 ? 2 : 1) w4_gemm_kernel(const W4GemmArgs p)
{
    extern __shared__ __align__(128) uint8_t w4_smem[];
    constexpr int PF = w4_prefetch(NT);
    constexpr int NG = 128 / G;
    const uint32_t smem = ptx::smem_addr(w4_smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int WR = 1 << p.wr_log2, wk_log2 = 3 - p.wr_log2, WK = 1 << wk_log2;
    const int wr = warp & (WR - 1), wk = warp >> p.wr_log2;
    const int C = p.cluster, rank = C > 1 ? (int)ptx::cluster_ctarank() : 0, group = (int)blockIdx.x / C;
    const int kb0 = (int)((int64_t)p.KB * rank / C), kb1 = (int)((int64_t)p.KB * (rank + 1) / C);
    const int steps = (kb1 - kb0 + WK - 1) >> wk_log2;                       // of the CTA (for its barriers)
    const int mine = (kb1 - kb0 - wk + WK - 1) >> wk_log2;                   // of this warp

    const uint8_t* codes[2];
    const bf16* scales[2];
    const uint8_t* zeros[2];
    bool have[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int tile = GATED ? group * WR + wr : (group * WR + wr) * 2 + j;
        const W4Operand& w = p.w[GATED ? j : 0];
        have[j] = tile < p.n16;
        const int64_t block = (int64_t)(have[j] ? tile : 0) * p.KB + kb0 + wk;
        codes[j] = w.codes + block * 1024 + lane * 16;
        scales[j] = w.scales + (block * 16 + g) * NG;
        zeros[j] = w.zeros == nullptr ? nullptr : w.zeros + (block * 16 + g) * NG;
    }
    W4Stage<G> st[PF];
    auto fetch = [&](W4Stage<G>& d, int i) {
        const int64_t b = (int64_t)i << wk_log2;                             // k-blocks from the warp's first one
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (!have[j]) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                d.c[j][h] = ld_once_16B(codes[j] + b * 1024 + h * 512);
                const bf16* s = scales[j] + (b * 16 + h * 8) * NG;
                if constexpr (G == 32) {
                    const uint2 v = ld_8B(s);
                    d.s[j][h][0] = v.x;
                    d.s[j][h][1] = v.y;
                } else if constexpr (G == 64) {
                    d.s[j][h][0] = ld_4B(s);
                } else {
                    d.s[j][h][0] = ld_2B(s);
                }
                if (zeros[j] != nullptr) {
                    const uint8_t* z = zeros[j] + (b * 16 + h * 8) * NG;
                    if constexpr (G == 32) d.z[j][h] = ld_4B(z);
                    else if constexpr (G == 64) d.z[j][h] = ld_2B(z);
                    else d.z[j][h] = ld_1B(z);
                } else {
                    d.z[j][h] = 0x08080808u;
                }
            }
        }
    };
    if (!p.early) ptx::grid_dependency_wait();
#pragma unroll
    for (int i = 0; i < PF; ++i) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {            // a tile past the last column computes on zeros, which are not stored
                st[i].c[j][h] = make_uint4(0, 0, 0, 0);
                st[i].s[j][h][0] = 0;
                if constexpr (G == 32) st[i].s[j][h][1] = 0;
                st[i].z[j][h] = 0;
            }
        if (i < mine) fetch(st[i], i);
    }
    if (p.early) ptx::grid_dependency_wait();
    ptx::launch_dependents();

    // X: chunks of `chunk` steps, double buffered when there is more than one
    const int chunk = max(p.chunk, 1), row_pieces = (chunk << wk_log2) * 16;                       // 16-byte pieces of a row
    const uint32_t x_stride = (uint32_t)row_pieces * 16u + 64u;                            // + 64: conflict-free quarter warps
    const uint32_t buf_bytes = x_stride * (uint32_t)(p.M * p.terms);
    auto load_x = [&](int step0, int buf) {
        const int kfirst = (kb0 + (step0 << wk_log2)) * 128, klast = min(kb1 * 128, p.K);
        const int pieces = p.M * p.terms * row_pieces;
        for (int i = threadIdx.x; i < pieces; i += kW4Threads) {
            const int row = i / row_pieces, col = i - row * row_pieces;
            const int k = kfirst + col * 8;
            const bool in = k < klast;
            cp_async_16_zfill(smem + buf * buf_bytes + row * x_stride + col * 16, p.X + (int64_t)row * p.K + (in ? k : 0), in ? 16u : 0u);
        }
    };
    load_x(0, 0);

    float y[2][NT][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) y[j][n][e] = 0.0f;

    auto step = [&](const W4Stage<G>& d, const uint8_t* xaddr) {            // xaddr: the lane's bytes of row g in this k-block
        float acc[2][NT][4];
        uint32_t zc[2][2];
        auto sub_block = [&](auto jc) {
            constexpr int J = decltype(jc)::value;                           // 32 of the 128 k
            if constexpr ((J * 32) % G == 0) {
                constexpr int gi = J * 32 / G;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) zc[j][h] = (((d.z[j][h] >> (8 * gi)) & 15u) * 0x00010001u) | 0x43004300u;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][n][e] = 0.0f;
                }
            }
            uint32_t a[2][8];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t lo[4] = {d.c[j][0].x, d.c[j][0].y, d.c[j][0].z, d.c[j][0].w};
                const uint32_t hi[4] = {d.c[j][1].x, d.c[j][1].y, d.c[j][1].z, d.c[j][1].w};
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int at = (u >> 1) * 4 + (u & 1) * 2;
                    a[j][at] = codes_to_bf16x2<4 * J>(lo[u], zc[j][0]);
                    a[j][at + 1] = codes_to_bf16x2<4 * J>(hi[u], zc[j][1]);
                }
            }
            for (int term = 0; term < p.terms; ++term) {
                const uint8_t* xt = xaddr + (uint32_t)(term * p.M) * x_stride + J * 64;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint4 b = make_uint4(0, 0, 0, 0);
                    if (n * 8 + g < p.M) b = *reinterpret_cast<const uint4*>(xt + (uint32_t)(n * 8) * x_stride);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        mma_bf16_16816(acc[j][n], a[j][0], a[j][1], a[j][2], a[j][3], b.x, b.y);
                        mma_bf16_16816(acc[j][n], a[j][4], a[j][5], a[j][6], a[j][7], b.z, b.w);
                    }
                }
            }
            if constexpr ((J * 32 + 32) % G == 0) {
                constexpr int gi = J * 32 / G;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t w0 = d.s[j][0][gi >> 1], w1 = d.s[j][1][gi >> 1];
                    const float s0 = (gi & 1) ? bf16_hi(w0) : bf16_lo(w0), s1 = (gi & 1) ? bf16_hi(w1) : bf16_lo(w1);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        y[j][n][0] = fmaf(s0, acc[j][n][0], y[j][n][0]);
                        y[j][n][1] = fmaf(s0, acc[j][n][1], y[j][n][1]);
                        y[j][n][2] = fmaf(s1, acc[j][n][2], y[j][n][2]);
                        y[j][n][3] = fmaf(s1, acc[j][n][3], y[j][n][3]);
                    }
                }
            }
        };
        sub_block(std::integral_constant<int, 0>{});
        sub_block(std::integral_constant<int, 1>{});
        sub_block(std::integral_constant<int, 2>{});
        sub_block(std::integral_constant<int, 3>{});
    };

    int buf = 0;
    for (int c0 = 0; c0 < steps; c0 += chunk) {
        cp_async_wait_all();
        __syncthreads();
        if (c0 + chunk < steps) load_x(c0 + chunk, buf ^ 1);
        const uint8_t* x0 = w4_smem + buf * buf_bytes + g * x_stride + t * 16 + (uint32_t)wk * 256u;
        const int end = min(chunk, mine - c0);
        for (int i = 0; i < end; i += PF) {          // chunk is a multiple of PF wherever there are several chunks
#pragma unroll
            for (int q = 0; q < PF; ++q) {
                if (i + q < end) {
                    step(st[q], x0 + ((uint32_t)(i + q) << (8 + wk_log2)));
                    if (c0 + i + q + PF < mine) fetch(st[q], c0 + i + q + PF);
                }
            }
        }
        buf ^= 1;
    }

    // partial sums of the warps that share columns, then of the CTAs of the cluster, each in a fixed order
    __syncthreads();
    constexpr int S = w4_red_stride(NT);
    float* red = reinterpret_cast<float*>(w4_smem);                          // [WK][WR * 32][S]
    {
        float* at = red + (size_t)((wk << p.wr_log2) + wr) * 32 * S;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                *reinterpret_cast<float2*>(at + (j * 16 + g) * S + n * 8 + 2 * t) = make_float2(y[j][n][0], y[j][n][1]);
                *reinterpret_cast<float2*>(at + (j * 16 + g + 8) * S + n * 8 + 2 * t) = make_float2(y[j][n][2], y[j][n][3]);
            }
    }
    __syncthreads();
    const int rows = WR * 32, total = rows * p.M, rows_log2 = p.wr_log2 + 5;
    const int part = rows * S;
    if (C > 1) {
        for (int i = threadIdx.x; i < total; i += kW4Threads) {
            float* e = red + (i & (rows - 1)) * S + (i >> rows_log2);
            float v = e[0];
            for (int w = 1; w < WK; ++w) v += e[w * part];
            e[0] = v;
        }
        __syncwarp();
        ptx::cluster_sync();
    }
    auto sum = [&](int row, int m) {
        float v;
        if (C > 1) {
            const uint32_t at = smem + (uint32_t)(row * S + m) * 4u;
            v = ld_cluster_f32(ptx::map_to_cta(at, 0));
            for (int r = 1; r < C; ++r) v += ld_cluster_f32(ptx::map_to_cta(at, (uint32_t)r));
        } else {
            const float* e = red + row * S + m;
            v = e[0];
            for (int w = 1; w < WK; ++w) v += e[w * part];
        }
        return v;
    };
    const int outputs = GATED ? total >> 1 : total, out_log2 = GATED ? rows_log2 - 1 : rows_log2;
    const int first = (int)((int64_t)outputs * rank / C), last = (int)((int64_t)outputs * (rank + 1) / C);
    for (int i = first + threadIdx.x; i < last; i += kW4Threads) {
        const int r = i & ((1 << out_log2) - 1), m = i >> out_log2;
        const int n = (group << out_log2) + r;
        if (n >= p.N) continue;
        if constexpr (GATED) {
            const int row = (r >> 4) * 32 + (r & 15);
            const float gate = sum(row, m), up = sum(row + 16, m);
            const float h = gate_act_f32(gate, p.act) * up;
            // two terms: the down projection reads 16 bits of the product's significand.  An infinite h has lo = 0 (not
            // inf - inf), a NaN stays in hi.
            const bf16 hi = __float2bfloat16_rn(h);
            const float rest = h - __bfloat162float(hi);
            const int64_t at = (int64_t)m * p.N + n;
            p.out[at] = hi;
            p.out[(int64_t)p.M * p.N + at] = __float2bfloat16_rn(fabsf(rest) < __int_as_float(0x7F800000) ? rest : 0.0f);
        } else {
            p.out[(int64_t)m * p.N + n] = __float2bfloat16_rn(sum(r, m));
        }
    }
    __syncwarp();
    if (C > 1) ptx::cluster_sync();                  // the peers may still be reading this CTA's sums
}

// Xn = X * rsqrt(mean X^2 + eps) * gain as two bf16 terms [2][M][K]; one CTA per token.
__global__ void __launch_bounds__(kRmsThreads)
w4_norm_kernel(const bf16* X, const bf16* gain, bf16* out, int M, int K, float eps)
{
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int64_t row = blockIdx.x;
    const uint4* x = reinterpret_cast<const uint4*>(X + row * K);
    const int nvec = K >> 3;
    float ss = 0.0f;
    for (int i = threadIdx.x; i < nvec; i += kRmsThreads) {
        const uint4 v = x[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) ss = fmaf(bf16_lo(w[j]), bf16_lo(w[j]), fmaf(bf16_hi(w[j]), bf16_hi(w[j]), ss));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
    __shared__ float warp_sums[kRmsThreads / 32];
    if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = ss;
    __syncthreads();
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < kRmsThreads / 32; ++w) total += warp_sums[w];
    const float r = rsqrtf(total / (float)K + eps);
    uint4* hi = reinterpret_cast<uint4*>(out + row * K);
    uint4* lo = reinterpret_cast<uint4*>(out + ((int64_t)M + row) * K);
    for (int i = threadIdx.x; i < nvec; i += kRmsThreads) {
        const uint4 v = x[i];
        uint4 gv = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);      // bf16 ones
        if (gain != nullptr) gv = reinterpret_cast<const uint4*>(gain)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w};
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = bf16_lo(w[j]) * r * bf16_lo(gw[j]), b = bf16_hi(w[j]) * r * bf16_hi(gw[j]);
            h[j] = pack_bf16x2(a, b);
            const float ra = a - bf16_lo(h[j]), rb = b - bf16_hi(h[j]);
            l[j] = pack_bf16x2(fabsf(ra) < __int_as_float(0x7F800000) ? ra : 0.0f, fabsf(rb) < __int_as_float(0x7F800000) ? rb : 0.0f);
        }
        hi[i] = make_uint4(h[0], h[1], h[2], h[3]);
        lo[i] = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// ------------------------------------------------------------------ layout: once per weight matrix
// One thread per output column and k-block of 128: it reads its 128 weights (or codes), forms 16 words and the groups'
// parameters.  Columns past N and rows past K get code 0 and scale 0.
enum { kW4FromCodes = 0, kW4FromBf16 = 1, kW4FromBf16Zeros = 2 };
template <int MODE>
__global__ void __launch_bounds__(128)
w4_pack_kernel(const void* src, int out_in, const bf16* scales_in, const uint8_t* zeros_in,
               uint8_t* codes, bf16* scales, uint8_t* zeros, int K, int N, int G)
{
    ptx::grid_dependency_wait();
    const int n = blockIdx.x * 128 + threadIdx.x, kb = blockIdx.y, KB = (K + 127) / 128, n16 = (N + 15) / 16;
    if (n >= n16 * 16) return;
    const int ng = 128 / G;
    const int64_t block = (int64_t)(n >> 4) * KB + kb;
    uint32_t word[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) word[j] = 0;
    const int64_t step = out_in ? 1 : N;             // distance of neighbouring k in the source
    const int64_t base = out_in ? (int64_t)n * K : n;
    for (int gi = 0; gi < ng; ++gi) {
        const int k0 = kb * 128 + gi * G;
        const bool in = n < N && k0 < K;             // K is a multiple of G
        float s = 0.0f, z = 8.0f;
        if (in) {
            if constexpr (MODE == kW4FromCodes) {
                const int64_t at = out_in ? (int64_t)n * (K / G) + k0 / G : (int64_t)(k0 / G) * N + n;
                s = __bfloat162float(scales_in[at]);
                if (zeros_in != nullptr) z = (float)(zeros_in[at] & 15);
            } else {
                const bf16* w = static_cast<const bf16*>(src) + base;
                float lo = 0.0f, hi = 0.0f;
                bool finite = true;
                for (int i = 0; i < G; ++i) {
                    const float v = __bfloat162float(w[(int64_t)(k0 + i) * step]);
                    lo = fminf(lo, v);
                    hi = fmaxf(hi, v);
                    finite = finite && v - v == 0.0f;
                }
                const float range = MODE == kW4FromBf16Zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f;
                s = __bfloat162float(__float2bfloat16_rn(range));
                finite = finite && s - s == 0.0f;
                if (!finite) s = __int_as_float(0x7FC00000);
                if (MODE == kW4FromBf16Zeros) z = s > 0.0f ? fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 0.0f;
            }
            for (int i = 0; i < G; ++i) {
                uint32_t q;
                if constexpr (MODE == kW4FromCodes) {
                    q = static_cast<const uint8_t*>(src)[base + (int64_t)(k0 + i) * step] & 15u;
                } else {
                    const float v = __bfloat162float(static_cast<const bf16*>(src)[base + (int64_t)(k0 + i) * step]);
                    q = s > 0.0f ? (uint32_t)fminf(fmaxf(rintf(v / s) + z, 0.0f), 15.0f) : (uint32_t)z;
                }
                const int k = gi * G + i, unit = k & 31;
                const uint32_t v = q << (4 * (k >> 5) + 16 * (unit & 1));
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (j == unit >> 1) word[j] |= v;
            }
        }
        const int64_t at = (block * 16 + (n & 15)) * ng + gi;
        scales[at] = __float2bfloat16_rn(s);
        if (zeros != nullptr) zeros[at] = (uint8_t)z;
    }
    uint8_t* out = codes + block * 1024 + ((n & 15) >> 3) * 512 + (n & 7) * 64;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        reinterpret_cast<uint4*>(out)[j] = make_uint4(word[4 * j], word[4 * j + 1], word[4 * j + 2], word[4 * j + 3]);
}

__global__ void __launch_bounds__(128)
w4_unpack_kernel(const uint8_t* codes, const bf16* scales, const uint8_t* zeros,
                 bf16* W, int out_in, int K, int N, int G)
{
    ptx::grid_dependency_wait();
    const int n = blockIdx.x * 128 + threadIdx.x, kb = blockIdx.y, KB = (K + 127) / 128, ng = 128 / G;
    if (n >= N) return;
    const int64_t block = (int64_t)(n >> 4) * KB + kb;
    const uint16_t* unit = reinterpret_cast<const uint16_t*>(codes + block * 1024 + ((n & 15) >> 3) * 512 + (n & 7) * 64);
    for (int k = 0; k < 128 && kb * 128 + k < K; ++k) {
        const int64_t at = (block * 16 + (n & 15)) * ng + k / G;
        const float q = (float)((unit[k & 31] >> (4 * (k >> 5))) & 15), z = zeros != nullptr ? (float)zeros[at] : 8.0f;
        const int64_t to = out_in ? (int64_t)n * K + kb * 128 + k : (int64_t)(kb * 128 + k) * N + n;
        W[to] = __float2bfloat16_rn((q - z) * __bfloat162float(scales[at]));
    }
}

}  // namespace gmlp
