// Products with 4-bit weights for a few tokens:  Y[m, n] = sum_k X[m, k] * (q[k, n] - z[k / G, n]) * s[k / G, n],
// q in 0..15, one scale s (bf16) and one zero point z (0..15; 8 without stored zero points) per group of G = 32, 64 or 128
// input rows.  Bound by HBM: the codes are read once, half a byte per weight.
//
// Storage (made once by the pack kernels below): tiles of 16 output columns x 128 input rows, 1 KB each, [N / 16][K / 128] with the
// second count even, so that the stream of a warp is contiguous.  In a tile, lane 4 g + t of a warp finds its 16 bytes for column g
// at 16 * lane and for column g + 8 at 512 + 16 * lane: eight 16-bit units r = 8 t .. 8 t + 7, unit r holding the codes of k = r,
// r + 32, r + 64, r + 96 in its four nibbles; every 32-bit word is rotated left by three bits.  One rotation and one and-or turn a
// word into two bf16 numbers 16 + q (the nibble lands in the upper four mantissa bits).  Those pairs are A operands of mma.m16n8k16 as
// they are, columns of W as its 16 rows and tokens as its 8 columns; the k order they imply (32 j + 8 t + 0..7) makes the matching B
// operand 16 contiguous bytes of a row of X.  Products of a group are summed in fp32 by the tensor core, then scaled in fp32: no
// weight is ever rounded.  16 + z comes off either before the product (q - z, exact in bf16: one more instruction per pair) or after
// it, as (16 + z) times the group's sum of X, which is formed once per call.
//
// K is split over the warps of a CTA and, where that helps, over the CTAs of a cluster; partial sums are added in a fixed order
// (shared memory, then distributed shared memory).
// X may come as two bf16 terms (hi + lo, 16 bits of significand): activations that are not bf16 by nature - the normed
// input, the gated product - keep the accuracy of the fp32 they were computed in.  The lo terms are further rows of X to the
// product; the epilogue adds the two sums of a token.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "ptx.cuh"
#include "umma_gemm_2cta.cuh"
#include "umma_skinny.cuh"

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
    int m_cta;                 // tile and umma kernels: tokens per CTA; blockIdx.y takes the tokens from blockIdx.y * m_cta on
    int group_warps;           // stream kernel: warps of a team, a power of two
    int wr_log2, cluster;      // tile kernel: column groups per CTA; tile and umma kernels: CTAs that share K
    int early;                 // the weights may be fetched before the preceding kernel of the call has ended
    GateAct act;
};

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                               uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same onto zeros: a group's first product.
__device__ __forceinline__ void mma_bf16_16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                     uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
// a * b + c in both halves.
__device__ __forceinline__ uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t bf16x2_add(uint32_t a, uint32_t b) { return bf16x2_fma(a, 0x3F803F80u, b); }
// (w & mask) | bits in one instruction (left to itself the compiler splits the and-or of two constants in two, on the
// half-rate integer pipe: 8192 x 28672 at M = 1 took 38.4 us so, 32.7 us as one).
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "r"(mask), "r"(bits));
    return d;
}
// Nibble J of both halves of a (rotated) word as bf16 16 + q.
template <int J>
__device__ __forceinline__ uint32_t w4_codes_plus_16(uint32_t w) {
    return and_or(J == 0 ? w : __funnelshift_r(w, w, 4 * J), 0x00780078u, 0x41804180u);
}
constexpr uint32_t kW4NoZeros = 0xC0C0C0C0u;         // zero points are stored as 0x80 | z << 3, the low byte of bf16 16 + z: here z = 8
__device__ __forceinline__ void cp_async_16_zfill(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most N of the thread's newest groups are still on their way.
template <int N>
__device__ __forceinline__ void cp_async_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Loads of parameters.  Volatile, so that none moves ahead of griddepcontrol.wait; plain (not .nc) because the kernel
// before, which may have written them, can still be running when this one starts.
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

// ------------------------------------------------------------------ one k-block of a tile
// In shared memory, for B neighbouring k-blocks: their kilobytes of codes, their 16 * NG scales each, their 16 * NG zero points each
// (NG = 128 / G groups of a column).
__host__ __device__ constexpr int w4_slot_bytes(int G, int B) { return B * (1024 + 48 * (128 / G)); }

// A lane's share of copying k-blocks of one tile: 16 bytes of either half of each kilobyte of codes, and (the first lanes) 16 bytes of
// scales or zero points.
struct W4Source {
    const uint8_t *codes, *params;       // params: nullptr for a lane that copies none
};
template <int B>
__device__ __forceinline__ W4Source w4_source(const W4Operand& w, int64_t block, int lane, int ng) {
    W4Source s = {w.codes + block * 1024 + lane * 16, nullptr};
    if (lane < 2 * B * ng) s.params = reinterpret_cast<const uint8_t*>(w.scales) + block * (32 * ng) + lane * 16;
    else if (lane < 3 * B * ng && w.zeros != nullptr) s.params = w.zeros + block * (16 * ng) + (lane - 2 * B * ng) * 16;
    return s;
}
// Bytes per k-block of the parameters that the lane copies.
template <int B>
__device__ __forceinline__ uint32_t w4_param_bytes(int lane, int ng) { return lane < 2 * B * ng ? 32 * ng : 16 * ng; }
// Copies B k-blocks to shared memory; `to` is the slot's address plus 16 * lane.
template <int B>
__device__ __forceinline__ void w4_copy_blocks(uint32_t to, const W4Source& s, bool params) {
#pragma unroll
    for (int i = 0; i < 2 * B; ++i) cp_async_16(to + 512 * i, s.codes + 512 * i);
    if (params) cp_async_16(to + 1024 * B, s.params);
}
// The lane's part of a k-block, in registers.
template <int G>
struct W4Block {
    uint32_t c[2][4];                    // columns g and g + 8
    uint32_t s[2][G == 32 ? 2 : 1];      // their 128 / G scales
    uint32_t z[2];                       // and zero points, one byte each
};
// k-block i of a slot of B.
template <int G, int B>
__device__ __forceinline__ void w4_read_block(W4Block<G>& d, const uint8_t* slot, int i, int lane, bool has_zeros) {
    constexpr int NG = 128 / G;
    const int g = lane >> 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 c = *reinterpret_cast<const uint4*>(slot + i * 1024 + h * 512 + lane * 16);
        d.c[h][0] = c.x; d.c[h][1] = c.y; d.c[h][2] = c.z; d.c[h][3] = c.w;
        const uint8_t* s = slot + B * 1024 + i * 32 * NG + (g + 8 * h) * 2 * NG;
        if constexpr (G == 32) {
            const uint2 v = *reinterpret_cast<const uint2*>(s);
            d.s[h][0] = v.x; d.s[h][1] = v.y;
        } else if constexpr (G == 64) {
            d.s[h][0] = *reinterpret_cast<const uint32_t*>(s);
        } else {
            d.s[h][0] = *reinterpret_cast<const uint16_t*>(s);
        }
        const uint8_t* z = slot + B * 1024 + B * 32 * NG + i * 16 * NG + (g + 8 * h) * NG;
        d.z[h] = kW4NoZeros;
        if (has_zeros) {
            if constexpr (G == 32) d.z[h] = *reinterpret_cast<const uint32_t*>(z);
            else if constexpr (G == 64) d.z[h] = *reinterpret_cast<const uint16_t*>(z);
            else d.z[h] = *z;
        }
    }
}
// SUMS: 16 + z comes off after the product; xsum: the sums of X over the k-block's groups, NT * 8 floats each, at the lane's columns.
template <int J, bool SUMS, int TP, int NT, int G>
__device__ __forceinline__ void w4_sub_block(float (&y)[TP][NT][4], float (&acc)[TP][NT][4], uint32_t (&zc)[TP][2],
                                             const W4Block<G> (&d)[TP], const uint8_t* x, const int (&row_at)[NT], const float* xsum) {
    constexpr int gi = J * 32 / G;                   // 32 of the 128 k, their group
    constexpr bool first = (J * 32) % G == 0;
    if constexpr (first && !SUMS) {
#pragma unroll
        for (int j = 0; j < TP; ++j)                                         // bf16 -(16 + z), twice: the bytes z, 0xC1, z, 0xC1
#pragma unroll
            for (int h = 0; h < 2; ++h) zc[j][h] = __byte_perm(d[j].z[h], 0xC1C1C1C1u, 0x4040u | gi | (gi << 8));
    }
    uint32_t a[TP][8];
#pragma unroll
    for (int j = 0; j < TP; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t v = w4_codes_plus_16<J>(d[j].c[h][u]);
                if constexpr (!SUMS) v = bf16x2_add(v, zc[j][h]);
                a[j][(u >> 1) * 4 + (u & 1) * 2 + h] = v;
            }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint4 b = *reinterpret_cast<const uint4*>(x + row_at[n] + J * 64);
#pragma unroll
        for (int j = 0; j < TP; ++j) {
            if constexpr (first) mma_bf16_16816_first(acc[j][n], a[j][0], a[j][1], a[j][2], a[j][3], b.x, b.y);
            else mma_bf16_16816(acc[j][n], a[j][0], a[j][1], a[j][2], a[j][3], b.x, b.y);
            mma_bf16_16816(acc[j][n], a[j][4], a[j][5], a[j][6], a[j][7], b.z, b.w);
        }
    }
    if constexpr ((J * 32 + 32) % G == 0) {
#pragma unroll
        for (int j = 0; j < TP; ++j) {
            const uint32_t w0 = d[j].s[0][gi >> 1], w1 = d[j].s[1][gi >> 1];
            const float s0 = (gi & 1) ? bf16_hi(w0) : bf16_lo(w0), s1 = (gi & 1) ? bf16_hi(w1) : bf16_lo(w1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (SUMS) {                                        // fp32 16 + z: the bytes 0, 0, z, 0x41
                    const float2 xs = *reinterpret_cast<const float2*>(xsum + (gi * NT + n) * 8);
                    const float z0 = __uint_as_float(__byte_perm(d[j].z[0], 0x41000000u, 0x7044u | (gi << 8)));
                    const float z1 = __uint_as_float(__byte_perm(d[j].z[1], 0x41000000u, 0x7044u | (gi << 8)));
                    acc[j][n][0] = fmaf(-z0, xs.x, acc[j][n][0]);
                    acc[j][n][1] = fmaf(-z0, xs.y, acc[j][n][1]);
                    acc[j][n][2] = fmaf(-z1, xs.x, acc[j][n][2]);
                    acc[j][n][3] = fmaf(-z1, xs.y, acc[j][n][3]);
                }
                y[j][n][0] = fmaf(s0, acc[j][n][0], y[j][n][0]);
                y[j][n][1] = fmaf(s0, acc[j][n][1], y[j][n][1]);
                y[j][n][2] = fmaf(s1, acc[j][n][2], y[j][n][2]);
                y[j][n][3] = fmaf(s1, acc[j][n][3], y[j][n][3]);
            }
        }
    }
}
// y += X * W over one k-block of TP tiles, which share the B operand.  x: the lane's 16 bytes (at 16 t) of the k-block's first row of
// X; row_at[n]: bytes from there to the row of the lane's column of the n-th eight.  Rows past the last one read the last row instead:
// columns of a product do not mix, and what such a column sums up is not stored.
template <bool SUMS, int TP, int NT, int G>
__device__ __forceinline__ void w4_step(float (&y)[TP][NT][4], const W4Block<G> (&d)[TP], const uint8_t* x, const int (&row_at)[NT],
                                        const float* xsum) {
    float acc[TP][NT][4];
    uint32_t zc[TP][2];
    w4_sub_block<0, SUMS, TP, NT, G>(y, acc, zc, d, x, row_at, xsum);
    w4_sub_block<1, SUMS, TP, NT, G>(y, acc, zc, d, x, row_at, xsum);
    w4_sub_block<2, SUMS, TP, NT, G>(y, acc, zc, d, x, row_at, xsum);
    w4_sub_block<3, SUMS, TP, NT, G>(y, acc, zc, d, x, row_at, xsum);
}
// Two terms of the gated product: the down projection reads 16 bits of its significand.  An infinite h has lo = 0 (not
// inf - inf), a NaN stays in hi.
__device__ __forceinline__ void w4_store_terms(bf16* out, int64_t at, int64_t term, float h) {
    const bf16 hi = __float2bfloat16_rn(h);
    const float rest = h - __bfloat162float(hi);
    out[at] = hi;
    out[at + term] = __float2bfloat16_rn(fabsf(rest) < __int_as_float(0x7F800000) ? rest : 0.0f);
}

// ------------------------------------------------------------------ up to 16 rows of X: a persistent stream
// One CTA of 16 warps per SM.  A team of GW warps walks over column tiles; its warps deal out the pairs of k-blocks of a tile (gated:
// half of them those of the gate tile, half those of the up tile), each with a ring of its own in shared memory that asynchronous
// copies fill, across tiles too, so that the stream of codes does not pause at a tile's end.  X stays in shared memory for the whole kernel, with its sums over the groups;
// only the sums of a tile cross the warps of a team.
// 8192 x 28672, groups of 32 with zero points, M = 1: 36 us (3.9 TB/s, 0.60 of the measured copy rate); 4096 x 14336, groups of 128,
// M = 8: 11 us.  No pipe is full (8192 x 28672, groups of 128: integer pipe 47 % busy, issue slots 56 %, HBM 3.8 TB/s; the copies alone
// take 24 us, the arithmetic alone 25.5, both together 30): four warps per scheduler wait in turn for copies, shared memory and products.
// Loads into registers instead of the rings: 46.9 against 42.0 us (8192 x 28672, groups of 128); 32 or 24 warps with
// shorter rings, 30 us like these 16; without the rotations, which is not a result, 24 us.
constexpr int kW4StreamWarps = 16;
__host__ __device__ constexpr int w4_ring_depth(int nt) { return nt == 1 ? 3 : 2; }      // slots; two columns of eight need the room for X
constexpr int kW4StreamThreads = 32 * kW4StreamWarps;
// Shared memory: sums of the tiles, rings, sums of X over its groups, X.
__host__ __device__ constexpr uint32_t w4_stream_fixed_bytes(int nt, int G) {
    return (uint32_t)kW4StreamWarps * (16u * 8u * 4u + (uint32_t)(w4_ring_depth(nt) * w4_slot_bytes(G, 2)));
}
__host__ __device__ constexpr uint64_t w4_stream_bytes(int rows, int KB, int G) {
    const int nt = rows <= 8 ? 1 : 2;
    return w4_stream_fixed_bytes(nt, G) + (uint64_t)KB * (128 / G) * nt * 32 + (uint64_t)rows * ((uint64_t)KB * 256 + 64);
}

template <int NT, int G, bool GATED>
__global__ void __launch_bounds__(kW4StreamThreads, 1) w4_stream_kernel(const W4GemmArgs p)
{
    extern __shared__ __align__(128) uint8_t w4_smem[];
    constexpr int WARPS = kW4StreamWarps, NG = 128 / G, SLOT = w4_slot_bytes(G, 2), DEPTH = w4_ring_depth(NT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // GW and KW are powers of two; a team is GW neighbouring warps, KW of them share the k-blocks of one tile
    const int GW = p.group_warps, KW = GATED ? GW >> 1 : GW, team = warp / GW, wk = warp & (KW - 1);
    const int KP = p.KB >> 1, mine = (KP - wk + KW - 1) / KW;                // this warp's pairs of k-blocks: wk, wk + KW, ...
    const int walkers = (int)gridDim.x * (WARPS / GW), R = p.M * p.terms;
    const bool has_zeros = p.w[0].zeros != nullptr;
    int tile = (int)blockIdx.x + team * (int)gridDim.x;

    const int x_stride = p.KB * 256 + 64;
    float* red = reinterpret_cast<float*>(w4_smem);                          // [WARPS][16][8]
    uint8_t* ring = w4_smem + WARPS * 512 + warp * (DEPTH * SLOT);
    float* xsums = reinterpret_cast<float*>(w4_smem + w4_stream_fixed_bytes(NT, G));       // [KB * NG][NT * 8]
    uint8_t* xs = reinterpret_cast<uint8_t*>(xsums + p.KB * NG * NT * 8);

    // the next pair of k-blocks to ask for; one commit group per call, empty at the end of the stream
    const bool up = GATED && (warp & KW);
    const W4Operand operand = {up ? p.w[1].codes : p.w[0].codes, up ? p.w[1].scales : p.w[0].scales, up ? p.w[1].zeros : p.w[0].zeros};
    W4Source from = w4_source<2>(operand, (int64_t)tile * p.KB + 2 * wk, lane, NG);
    const bool params = from.params != nullptr;
    const uint32_t param_block = w4_param_bytes<2>(lane, NG);
    const uint32_t jump = (uint32_t)(walkers * p.KB - 2 * (mine - 1) * KW);  // k-blocks from a tile's last pair to the next tile's first
    const uint32_t code_by = 2048u * KW, code_jump = 1024u * jump, param_by = 2 * param_block * KW, param_jump = param_block * jump;
    int next_i = mine, left = mine > 0 && tile < p.n16 ? mine * ((p.n16 - 1 - tile) / walkers + 1) : 0;
    uint32_t next_to = ptx::smem_addr(ring) + lane * 16;
    const uint32_t ring_end = next_to + DEPTH * SLOT;
    auto ask = [&]() {
        if (left > 0) {
            --left;
            w4_copy_blocks<2>(next_to, from, params);
            const bool wrap = --next_i == 0;
            from.codes += wrap ? code_jump : code_by;
            from.params += wrap ? param_jump : param_by;
            if (wrap) next_i = mine;
        }
        next_to += SLOT;
        if (next_to == ring_end) next_to -= DEPTH * SLOT;
        cp_async_commit();
    };
    if (!p.early) ptx::grid_dependency_wait();
    for (int i = 0; i < DEPTH - 1; ++i) ask();
    if (p.early) ptx::grid_dependency_wait();
    ptx::launch_dependents();
    {
        const uint32_t x_at = ptx::smem_addr(xs);
        for (int row = 0; row < R; ++row)
            for (int i = threadIdx.x; i < p.KB * 16; i += 32 * WARPS) {
                const bool in = i * 8 < p.K;
                cp_async_16_zfill(x_at + row * x_stride + i * 16, p.X + (int64_t)row * p.K + (in ? i * 8 : 0), in ? 16u : 0u);
            }
    }
    cp_async_wait_all();
    __syncthreads();
    // Sums of X over the groups, four lanes each; columns past the last row hold the last row's, like the operand itself.  Where X is
    // not finite or so large that (16 + z) times a sum might not be, the zero points come off before the product instead.
    bool large = false;
    const bool two = NT == 2 && p.terms == 2;
    auto row_of = [&](int n, int c) { return two ? n * p.M + min(c, p.M - 1) : min(n * 8 + c, R - 1); };
    for (int i = threadIdx.x; i < p.KB * NG * NT * 32; i += 32 * WARPS) {
        const int part = i & 3, c = (i >> 2) & 7, rest = i >> 5, n = rest % NT, group = rest / NT;
        const uint8_t* at = xs + row_of(n, c) * x_stride + group * (2 * G) + part * 16;
        float v = 0.0f, most = 0.0f;
#pragma unroll
        for (int k = 0; k < G / 32; ++k) {
            const uint4 u = *reinterpret_cast<const uint4*>(at + k * 64);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = bf16_lo(w[e]), b = bf16_hi(w[e]);
                v += a + b;
                most += fabsf(a) + fabsf(b);
            }
        }
        large = large || !(most < 1e30f);
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
        if (part == 0) xsums[rest * 8 + c] = v;
    }
    large = __syncthreads_or(large);

    // two terms in two columns of eight: the lo terms take the second, so that both sums of a token lie in one lane
    auto team_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(GW * 32) : "memory"); };
    int row_at[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) row_at[n] = row_of(n, g) * x_stride;
    const uint8_t* x0 = xs + t * 16 + wk * 512;
    const float* xsum0 = xsums + wk * (2 * NG * NT * 8) + 2 * t;
    const uint8_t *slot = ring, *slot_end = ring + DEPTH * SLOT;

    for (; tile < p.n16; tile += walkers) {
        float y[1][NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) y[0][n][e] = 0.0f;
        const uint8_t* x = x0;
        const float* xsum = xsum0;
        for (int i = 0; i < mine; ++i) {
            cp_async_wait_but<DEPTH - 2>();   // this step's copies have landed,
            __syncwarp();                            // every lane's, and the slot of the step before is free
            ask();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                W4Block<G> d[1];
                w4_read_block<G, 2>(d[0], slot, h, lane, has_zeros);
                if (!large) w4_step<true, 1, NT, G>(y, d, x + h * 256, row_at, xsum + h * (NG * NT * 8));
                else w4_step<false, 1, NT, G>(y, d, x + h * 256, row_at, nullptr);
            }
            slot += SLOT;
            if (slot == slot_end) slot = ring;
            x += KW * 512;
            xsum += KW * (2 * NG * NT * 8);
        }
        if (two) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[0][0][e] += y[0][NT - 1][e];
        }
        // sums over the warps in a fixed order, one column of eight rows at a time
        const int columns = two ? 1 : (R + 7) / 8;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (n >= columns) break;
            team_sync();                             // what lay there before has been read
            float* at = red + (warp * 16 + g) * 8 + 2 * t;
            *reinterpret_cast<float2*>(at) = make_float2(y[0][n][0], y[0][n][1]);
            *reinterpret_cast<float2*>(at + 8 * 8) = make_float2(y[0][n][2], y[0][n][3]);
            team_sync();
            const bool folded = p.terms == 2 && !two;                        // up to 4 tokens: the lo terms are columns M ..
            const int tokens = p.terms == 2 ? p.M : min(8, p.M - n * 8);
            for (int o = (warp & (GW - 1)) * 32 + lane; o < 16 * tokens; o += GW * 32) {
                const int r = o & 15, m = o >> 4, col = tile * 16 + r;
                auto sum = [&](int first_warp) {
                    const float* e = red + (first_warp * 16 + r) * 8 + m;
                    float v = 0.0f;
#pragma unroll 4
                    for (int w = 0; w < KW; ++w) v += e[w * 128];
                    if (folded) {
                        float lo = 0.0f;
#pragma unroll 4
                        for (int w = 0; w < KW; ++w) lo += e[w * 128 + p.M];
                        v += lo;
                    }
                    return v;
                };
                if (col < p.N) {
                    const int64_t to = (int64_t)(n * 8 + m) * p.N + col;
                    if constexpr (GATED) w4_store_terms(p.out, to, (int64_t)p.M * p.N, gate_act_f32(sum(team * GW), p.act) * sum(team * GW + KW));
                    else p.out[to] = __float2bfloat16_rn(sum(team * GW));
                }
            }
        }
    }
    cp_async_wait_all();
}

// ------------------------------------------------------------------ X too large to stay, or more rows of a small matrix: tiles
// The 8 warps of a CTA are WR groups of two column tiles (gated: of a gate and an up tile) x WK ranges of K; stages of WK k-blocks of
// codes and X pass through shared memory, three deep.  Up to 32 rows of X per CTA (blockIdx.y: further rows, which read the codes
// again, from L2: by then the products set the time), and K over a cluster of C CTAs that add their sums in distributed shared memory.
// One CTA of 8 warps per SM from 9 rows on (shared memory), two per scheduler; the register limit for two CTAs, which only one column
// of eight rows uses, makes three and four columns spill (up to 344 bytes a thread).  64 x 4096 x 4096, groups of 128: 17.8 us;
// 8 x 14336 x 4096: 14.0 us.
constexpr int kW4Stages = 3;
__host__ __device__ constexpr int w4_red_stride(int nt) { return 8 * (nt | 1); }      // floats; odd multiples of 8 spread the banks
__host__ __device__ constexpr uint32_t w4_tile_smem(int nt, int rows, int wk, int G) {
    const uint32_t red = 8u * 32u * (uint32_t)w4_red_stride(nt) * 4u;
    const uint32_t stages = kW4Stages * ((uint32_t)rows * (uint32_t)(wk * 256 + 64) + 16u * (uint32_t)w4_slot_bytes(G, 1));
    return stages > red ? stages : red;
}

// NT: columns of eight rows of X (tokens times terms).
template <int NT, int G, bool GATED>
__global__ void __launch_bounds__(kW4Threads, 2) w4_tile_kernel(const W4GemmArgs p)
{
    extern __shared__ __align__(128) uint8_t w4_smem[];
    constexpr int NG = 128 / G, BLOCK = w4_slot_bytes(G, 1);
    const uint32_t smem = ptx::smem_addr(w4_smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int WR = 1 << p.wr_log2, wk_log2 = 3 - p.wr_log2, WK = 1 << wk_log2;
    const int wr = warp & (WR - 1), wk = warp >> p.wr_log2;
    const int C = p.cluster, rank = C > 1 ? (int)ptx::cluster_ctarank() : 0, group = (int)blockIdx.x / C;
    const int kb0 = (int)((int64_t)p.KB * rank / C), kb1 = (int)((int64_t)p.KB * (rank + 1) / C);
    const int steps = (kb1 - kb0 + WK - 1) >> wk_log2;                       // of the CTA (for its barriers)
    const int mine = (kb1 - kb0 - wk + WK - 1) >> wk_log2;                   // of this warp
    const int m0 = (int)blockIdx.y * p.m_cta, M = min(p.m_cta, p.M - m0), R = M * p.terms;
    const bool has_zeros = p.w[0].zeros != nullptr;
    const uint32_t param_block = w4_param_bytes<1>(lane, NG);

    W4Source from[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {                    // a tile past the last column reads the last tile again; its sums are not stored
        const int tile = min(GATED ? group * WR + wr : (group * WR + wr) * 2 + j, p.n16 - 1);
        from[j] = w4_source<1>(p.w[GATED ? j : 0], (int64_t)tile * p.KB + kb0 + wk, lane, NG);
    }
    const bool params = from[0].params != nullptr;
    const int x_stride = WK * 256 + 64, x_bytes = p.m_cta * p.terms * x_stride, stage_bytes = x_bytes + 16 * BLOCK;
    auto ask_codes = [&](int s, int slot) {
        if (s >= mine) return;
        const uint32_t to = smem + slot * stage_bytes + x_bytes + warp * 2 * BLOCK + lane * 16;
#pragma unroll
        for (int j = 0; j < 2; ++j) {                // called for s = 0, 1, 2, ... in turn
            w4_copy_blocks<1>(to + j * BLOCK, from[j], params);
            from[j].codes += (int64_t)1024 << wk_log2;
            from[j].params += (int64_t)param_block << wk_log2;
        }
    };
    // 16-byte pieces of X: a thread keeps its column of a stage and takes every row_by-th row
    const int pieces_log2 = wk_log2 + 4, row_by = kW4Threads >> pieces_log2, x_row = threadIdx.x >> pieces_log2;
    const int x_col = threadIdx.x & ((1 << pieces_log2) - 1);
    const bf16* x_from = p.X + (int64_t)(m0 + x_row) * p.K + kb0 * 128 + x_col * 8;        // stages are asked for in turn
    int x_k = kb0 * 128 + x_col * 8;
    const int64_t x_by = (int64_t)row_by * p.K, lo_jump = (int64_t)(p.M - M) * p.K;
    const uint32_t x_to = smem + x_row * x_stride + x_col * 16;
    auto ask_x = [&](int s, int slot) {
        if (s >= steps) return;
        const bool in = x_k < p.K;
        const bf16* from_row = in ? x_from : p.X;
        uint32_t to = x_to + slot * stage_bytes;
        for (int row = x_row; row < R; row += row_by) {
            cp_async_16_zfill(to, in && row >= M ? from_row + lo_jump : from_row, in ? 16u : 0u);
            if (in) from_row += x_by;
            to += row_by * x_stride;
        }
        x_from += 128 << wk_log2;
        x_k += 128 << wk_log2;
    };
    if (!p.early) ptx::grid_dependency_wait();
    ask_codes(0, 0);
    if (p.early) {
        ask_codes(1, 1);
        ptx::grid_dependency_wait();
    }
    ptx::launch_dependents();
    ask_x(0, 0);
    cp_async_commit();
    if (!p.early) ask_codes(1, 1);
    ask_x(1, 1);
    cp_async_commit();

    float y[2][NT][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) y[j][n][e] = 0.0f;
    int row_at[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) row_at[n] = min(n * 8 + g, R - 1) * x_stride;

    for (int s = 0, slot = 0; s < steps; ++s) {
        cp_async_wait_but<1>();
        __syncthreads();                             // this stage has landed, the one before it has been read
        const int next = slot == 0 ? 2 : slot - 1;
        ask_codes(s + 2, next);
        ask_x(s + 2, next);
        cp_async_commit();
        if (s < mine) {
            const uint8_t* stage = w4_smem + slot * stage_bytes;
            W4Block<G> d[2];
            w4_read_block<G, 1>(d[0], stage + x_bytes + warp * 2 * BLOCK, 0, lane, has_zeros);
            w4_read_block<G, 1>(d[1], stage + x_bytes + warp * 2 * BLOCK + BLOCK, 0, lane, has_zeros);
            w4_step<false, 2, NT, G>(y, d, stage + wk * 256 + t * 16, row_at, nullptr);
        }
        if (++slot == kW4Stages) slot = 0;
    }

    // partial sums of the warps that share columns, then of the CTAs of the cluster, each in a fixed order
    cp_async_wait_all();
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
    const int rows = WR * 32, rows_log2 = p.wr_log2 + 5, part = rows * S;
    auto own = [&](int row, int m) {                                         // this CTA's sum, terms and warps
        const float* e = red + row * S + m;
        float v = e[0];
        for (int w = 1; w < WK; ++w) v += e[w * part];
        if (p.terms == 2) {
            e += M;
            float lo = e[0];
            for (int w = 1; w < WK; ++w) lo += e[w * part];
            v += lo;
        }
        return v;
    };
    if (C > 1) {
        // every element is read and replaced by one thread; a token's lo term is only read by that thread
        for (int i = threadIdx.x; i < rows * M; i += kW4Threads) {
            const int row = i & (rows - 1), m = i >> rows_log2;
            red[row * S + m] = own(row, m);
        }
        __syncwarp();
        ptx::cluster_sync();
    }
    auto sum = [&](int row, int m) {
        if (C == 1) return own(row, m);
        const uint32_t at = smem + (uint32_t)(row * S + m) * 4u;
        float v = ld_cluster_f32(ptx::map_to_cta(at, 0));
        for (int r = 1; r < C; ++r) v += ld_cluster_f32(ptx::map_to_cta(at, (uint32_t)r));
        return v;
    };
    const int out_log2 = GATED ? rows_log2 - 1 : rows_log2, outputs = M << out_log2;
    const int first = (int)((int64_t)outputs * rank / C), last = (int)((int64_t)outputs * (rank + 1) / C);
    for (int i = first + threadIdx.x; i < last; i += kW4Threads) {
        const int r = i & ((1 << out_log2) - 1), m = i >> out_log2;
        const int n = (group << out_log2) + r;
        if (n >= p.N) continue;
        const int64_t at = (int64_t)(m0 + m) * p.N + n;
        if constexpr (GATED) {
            const int row = (r >> 4) * 32 + (r & 15);
            w4_store_terms(p.out, at, (int64_t)p.M * p.N, gate_act_f32(sum(row, m), p.act) * sum(row + 16, m));
        } else {
            p.out[at] = __float2bfloat16_rn(sum(r, m));
        }
    }
    __syncwarp();
    if (C > 1) ptx::cluster_sync();                  // the peers may still be reading this CTA's sums
}

// ------------------------------------------------------------------ more than 16 rows of X: tcgen05
// One CTA per 128 columns of W (gated: 64 gate and the same 64 up columns) and up to 64 rows of X (blockIdx.y: further rows), K over a
// cluster of C CTAs that add their sums in distributed shared memory.  Four kinds of warps pass k-blocks of 128 on:
//   4 producers   bulk copies of two tiles' codes each, TMA boxes of X (the B operand: K-major, 128-byte swizzle); a bulk copy takes
//                 some 90 cycles however small it is, so the parameters are read a k-block ahead by the warps that need them;
//   8 unpackers   a tile each: codes to q - z, exact in bf16, straight into the same layout as the A operand (a lane's eight
//                 neighbouring k of a column are one 16-byte store; three buffers: with two, unpacking and products took turns);
//   1 issuer      the tcgen05.mma of each group of G rows of K, into columns of TMEM of its own (two buffers);
//   8 readers     tcgen05.ld of the sums (a lane per column of W, half of the rows of X per warp), scaled in fp32 and added in
//                 registers: no weight is rounded here either.
// (With all warps doing everything in step, one barrier per k-block, a k-block took 1750 cycles.)
// Bound by the hand-over from one kind of warps to the next, some 1000 cycles a k-block: 4096 x 14336 at M = 64 25 us (48 with tiles), 8B
// layer at M = 33 without a norm 94 us (158 with tiles).  Two CTAs per SM for 32 rows, with two buffers each and 40 registers, lost: 8B layer
// with the norm at M = 16 89 against 76 us.
constexpr int kW4Producers = 4, kW4Unpackers = 8, kW4Readers = 8;
constexpr int kW4UmmaThreads = 32 * (kW4Unpackers + kW4Readers + 1 + kW4Producers);
constexpr int kW4UmmaDepth = 4, kW4ABuffers = 3;
constexpr uint32_t kW4UmmaABytes = 128 * 256;
__host__ __device__ constexpr uint32_t w4_umma_smem(int rpad) {
    return 1024u + (uint32_t)kW4ABuffers * kW4UmmaABytes + (uint32_t)kW4UmmaDepth * ((uint32_t)rpad * 256u + 8u * 1024u) + 192u;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// RPAD: rows of X of the product, 32 or 64 (rows past the last one are zeros or another part's; their sums are not stored).
template <int RPAD, int G, bool GATED>
__global__ void __launch_bounds__(kW4UmmaThreads, 1)
w4_umma_kernel(const W4GemmArgs p, const __grid_constant__ CUtensorMap tmX)
{
    extern __shared__ __align__(128) uint8_t w4_smem[];
    constexpr int NG = 128 / G, COLS = RPAD / 2;     // COLS: rows of X per reader
    constexpr uint32_t X_BYTES = RPAD * 256, CODE_BYTES = 8 * 1024, TMEM_COLS = 2 * NG * RPAD;
    constexpr int KERNEL_ID = 20, DEPTH = kW4UmmaDepth;
    const uint32_t raw = ptx::smem_addr(w4_smem), base = (raw + 1023u) & ~1023u;           // the same in every CTA of a cluster
    uint8_t* base_ptr = w4_smem + (base - raw);
    // buffers of A, a ring of X (all on 1024-byte boundaries: the swizzle goes by address), a ring of eight tiles' codes
    const uint32_t x_ring = base + kW4ABuffers * kW4UmmaABytes, code_ring = x_ring + DEPTH * X_BYTES;
    uint8_t* code_ptr = base_ptr + kW4ABuffers * kW4UmmaABytes + DEPTH * X_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(code_ptr + DEPTH * CODE_BYTES);
    const uint32_t full0 = ptx::smem_addr(bars);                             // [DEPTH] a stage's copies have landed
    const uint32_t empty0 = full0 + 8 * DEPTH;                               // [DEPTH] its sums have been read: it is free
    const uint32_t a_full0 = empty0 + 8 * DEPTH;                             // [3] A is unpacked
    const uint32_t a_empty0 = a_full0 + 8 * kW4ABuffers;                     // [3] the products that read it have ended
    const uint32_t done0 = a_empty0 + 8 * kW4ABuffers;                       // [2] the products have ended: their sums
    const uint32_t d_empty0 = done0 + 16;                                    // [2] have been read
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * DEPTH + 2 * kW4ABuffers + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int C = p.cluster, rank = C > 1 ? (int)ptx::cluster_ctarank() : 0, group = (int)blockIdx.x / C;
    const int kb0 = (int)((int64_t)p.KB * rank / C), steps = (int)((int64_t)p.KB * (rank + 1) / C) - kb0;
    const int m0 = (int)blockIdx.y * p.m_cta, M = min(p.m_cta, p.M - m0);
    const bool has_zeros = p.w[0].zeros != nullptr;

    if (threadIdx.x == 0) {
        for (int i = 0; i < DEPTH; ++i) {
            ptx::mbar_init(full0 + 8 * i, kW4Producers);
            ptx::mbar_init(empty0 + 8 * i, kW4Readers);
        }
        for (int i = 0; i < kW4ABuffers; ++i) {
            ptx::mbar_init(a_full0 + 8 * i, kW4Unpackers);
            ptx::mbar_init(a_empty0 + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(done0 + 8 * i, 1);
            ptx::mbar_init(d_empty0 + 8 * i, kW4Readers);
        }
        *abort_flag = 0;
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
        ptx::prefetch_tensormap(&tmX);
    }
    __syncthreads();
    // TMEM is taken after the kernel before has ended and before the next one may start: neither is kept from its own by a kernel that
    // waits for it.  The codes may be on their way before that.
    const int issuer = kW4Unpackers + kW4Readers;
    const bool producer = warp > issuer;
    // producer: tiles 2 pw and 2 pw + 1 and, for pw < 2 * terms, a box of X (bit 0: half of the k-block, bit 1: lo rows).  A tile past the
    // last column reads the last tile again; its sums are not stored.  Two terms: hi rows from row 0, lo rows from row RPAD / 2.
    const int pw = warp - issuer - 1, x_rows = RPAD / p.terms;
    const uint32_t my_tx = 2048u + (pw < 2 * p.terms ? (uint32_t)x_rows * 128u : 0u);
    auto tile_of = [&](int i) { return min(GATED ? group * 4 + (i & 3) : group * 8 + i, p.n16 - 1); };
    auto ask_codes = [&](int s, int slot) {
        const uint32_t full = full0 + 8 * slot;
        ptx::mbar_arrive_expect_tx(full, my_tx);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = 2 * pw + j;
            bulk_load(code_ring + slot * CODE_BYTES + i * 1024,
                      (GATED && i >= 4 ? p.w[1].codes : p.w[0].codes) + ((int64_t)tile_of(i) * p.KB + kb0 + s) * 1024, 1024, full);
        }
    };
    auto ask_x = [&](int s, int slot) {
        if (pw < 2 * p.terms)
            ptx::tma_load_2d(x_ring + slot * X_BYTES + (pw & 1) * (RPAD * 128) + (pw >> 1) * (x_rows * 128), &tmX,
                             (kb0 + s) * 128 + 64 * (pw & 1), (pw >> 1) * p.M + m0, full0 + 8 * slot);
    };
    const int ahead = min(DEPTH, steps);
    if (!p.early) ptx::grid_dependency_wait();
    if (producer && lane == 0)
        for (int s = 0; s < ahead; ++s) ask_codes(s, s);
    __syncwarp();
    if (p.early) ptx::grid_dependency_wait();
    if (producer && lane == 0)
        for (int s = 0; s < ahead; ++s) ask_x(s, s);
    __syncwarp();
    if (warp == issuer) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), TMEM_COLS);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    ptx::launch_dependents();
    const uint32_t tmem = *tmem_slot;

    // A wait that runs out leaves its mark in abort_flag and the device status; nothing more is asked for, every loop below runs on without
    // waiting, so that all warps meet again at its end, and what is in flight gets a millisecond to land.
    float y[COLS];
    const int quarter = warp & 3, my_row = quarter * 32 + lane, my_col = (warp >= kW4Unpackers + 4 ? 1 : 0) * COLS;
    if (producer) {
        if (lane == 0)
            for (int s = DEPTH, slot = 0, phase = 0; s < steps; ++s) {
                if (!wait_bounded(empty0 + 8 * slot, (uint32_t)phase, abort_flag, KERNEL_ID, 1)) break;
                ask_codes(s, slot);
                ask_x(s, slot);
                if (++slot == DEPTH) {
                    slot = 0;
                    phase ^= 1;
                }
            }
        __syncwarp();
    } else if (warp == issuer) {
        const bool leader = ptx::elect_one();
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(RPAD >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t desc_hi = (uint32_t)(ptx::make_smem_desc_sw128(0, 0, 1024) >> 32);
        const uint32_t a_lo0 = (uint32_t)ptx::make_smem_desc_sw128(base, 16, 1024), x_lo0 = (uint32_t)ptx::make_smem_desc_sw128(x_ring, 16, 1024);
        for (int s = 0, slot = 0, ab = 0, a_phase = 0; s < steps; ++s) {
            const int b = s & 1;
            (void)__all_sync(0xFFFFFFFFu, wait_bounded(a_full0 + 8 * ab, (uint32_t)a_phase, abort_flag, KERNEL_ID, 2));
            if (s >= 2) (void)__all_sync(0xFFFFFFFFu, wait_bounded(d_empty0 + 8 * b, (uint32_t)((s >> 1) - 1) & 1u, abort_flag, KERNEL_ID, 3));
            ptx::tc_fence_after_sync();
            const uint32_t a_lo = a_lo0 + ab * (kW4UmmaABytes / 16), x_lo = x_lo0 + slot * (X_BYTES / 16), d = tmem + (uint32_t)(b * NG) * RPAD;
            if (leader) {
#pragma unroll
                for (int k = 0; k < 8; ++k)          // 16 rows of K each: 32 bytes on in a 64-wide half, halves 128 (RPAD) rows apart
                    ptx::umma_bf16_halves(d + (uint32_t)(k * 16 / G) * RPAD, a_lo + (k >> 2) * 1024 + (k & 3) * 2,
                                          x_lo + (k >> 2) * (RPAD * 8) + (k & 3) * 2, desc_hi, idesc, (k * 16) % G == 0 ? 0u : 1u);
            }
            if (leader) {
                ptx::umma_commit(done0 + 8 * b);
                ptx::umma_commit(a_empty0 + 8 * ab);
            }
            __syncwarp();
            if (++slot == DEPTH) slot = 0;
            if (++ab == kW4ABuffers) {
                ab = 0;
                a_phase ^= 1;
            }
        }
        // the last arrival that the tensor core owes this CTA's shared memory
        (void)__all_sync(0xFFFFFFFFu, wait_bounded(a_empty0 + 8 * ((steps - 1) % kW4ABuffers), (uint32_t)((steps - 1) / kW4ABuffers) & 1u,
                                                   abort_flag, KERNEL_ID, 8));
    } else if (warp < kW4Unpackers) {
        const uint32_t a_at = base + (warp * 16 + g) * 128;                  // rows g and g + 8 of the tile; row & 7 is g
        const uint8_t* zp = has_zeros ? (GATED && warp >= 4 ? p.w[1].zeros : p.w[0].zeros) + (((int64_t)tile_of(warp) * p.KB + kb0) * 16 + g) * NG : nullptr;
        auto read_zeros = [&](uint32_t (&z)[2], int s) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint8_t* from = zp + ((int64_t)s * 16 + 8 * h) * NG;
                if constexpr (G == 32) z[h] = ld_4B(from);
                else if constexpr (G == 64) z[h] = ld_2B(from);
                else z[h] = ld_1B(from);
            }
        };
        uint32_t z[2] = {kW4NoZeros, kW4NoZeros}, z_next[2] = {kW4NoZeros, kW4NoZeros};
        if (has_zeros) read_zeros(z_next, 0);
        for (int s = 0, slot = 0, phase = 0, ab = 0, a_phase = 1; s < steps; ++s) {
            (void)wait_bounded(full0 + 8 * slot, (uint32_t)phase, abort_flag, KERNEL_ID, 4);
            __syncwarp();
            const uint8_t* block = code_ptr + slot * CODE_BYTES + warp * 1024;
            uint32_t c[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 v = *reinterpret_cast<const uint4*>(block + h * 512 + lane * 16);
                c[h][0] = v.x; c[h][1] = v.y; c[h][2] = v.z; c[h][3] = v.w;
                z[h] = z_next[h];
            }
            if (has_zeros && s + 1 < steps) read_zeros(z_next, s + 1);
            if (s >= kW4ABuffers) {                  // the products that read this buffer of A have ended
                (void)wait_bounded(a_empty0 + 8 * ab, (uint32_t)a_phase, abort_flag, KERNEL_ID, 5);
                __syncwarp();
            }
            const uint32_t to = a_at + ab * kW4UmmaABytes;
            auto unpack = [&](auto jc) {             // k = 32 J + 8 t .. + 7: chunk 4 (J & 1) + t of its half of K
                constexpr int J = decltype(jc)::value;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t zc = __byte_perm(z[h], 0xC1C1C1C1u, 0x4040u | (J * 32 / G) | ((J * 32 / G) << 8));
                    uint32_t v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = bf16x2_add(w4_codes_plus_16<J>(c[h][u]), zc);
                    const uint32_t at = to + h * (8 * 128) + (J >> 1) * (128 * 128) + ((((J & 1) * 4 + t) ^ g) * 16);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                }
            };
            unpack(std::integral_constant<int, 0>{});
            unpack(std::integral_constant<int, 1>{});
            unpack(std::integral_constant<int, 2>{});
            unpack(std::integral_constant<int, 3>{});
            ptx::fence_proxy_async_smem();           // this thread's part of A, before the tensor core reads it
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(a_full0 + 8 * ab);
            if (++ab == kW4ABuffers) {
                ab = 0;
                a_phase ^= 1;
            }
            if (++slot == DEPTH) {
                slot = 0;
                phase ^= 1;
            }
        }
    } else {
        const uint32_t tmem_mine = tmem + ((uint32_t)(quarter * 32) << 16) + my_col;
#pragma unroll
        for (int c = 0; c < COLS; ++c) y[c] = 0.0f;
        const int i = my_row >> 4;
        const bf16* sp = (GATED && i >= 4 ? p.w[1].scales : p.w[0].scales) + (((int64_t)tile_of(i) * p.KB + kb0) * 16 + (my_row & 15)) * NG;
        uint32_t next[G == 32 ? 2 : 1];              // the next k-block's scales
        auto read_scales = [&](int s) {
            const bf16* from = sp + (int64_t)s * 16 * NG;
            if constexpr (G == 32) {
                const uint2 v = ld_8B(from);
                next[0] = v.x; next[1] = v.y;
            } else if constexpr (G == 64) {
                next[0] = ld_4B(from);
            } else {
                next[0] = ld_2B(from);
            }
        };
        read_scales(0);
        for (int s = 0, slot = 0; s < steps; ++s) {
            const int b = s & 1;
            float scale[NG];
#pragma unroll
            for (int gi = 0; gi < NG; ++gi) scale[gi] = (gi & 1) ? bf16_hi(next[gi >> 1]) : bf16_lo(next[gi >> 1]);
            if (s + 1 < steps) read_scales(s + 1);
            (void)wait_bounded(done0 + 8 * b, (uint32_t)(s >> 1) & 1u, abort_flag, KERNEL_ID, 7);
            ptx::tc_fence_after_sync();
            __syncwarp();
#pragma unroll
            for (int gi = 0; gi < NG; ++gi)
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 16) {
                    uint32_t v[16];
                    tmem_ld_32x16(tmem_mine + (uint32_t)((b * NG + gi) * RPAD + c0), v);
                    ptx::tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 16; ++c) y[c0 + c] = fmaf(scale[gi], __uint_as_float(v[c]), y[c0 + c]);
                }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(d_empty0 + 8 * b);
                ptx::mbar_arrive(empty0 + 8 * slot);
            }
            if (++slot == DEPTH) slot = 0;
        }
    }
    if (*abort_flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == issuer) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, TMEM_COLS);
    }

    // sums of the cluster's CTAs, in a fixed order
    constexpr int S = RPAD + 1;
    float* red = reinterpret_cast<float*>(base_ptr);                         // [128][S], in place of A
    if (warp >= kW4Unpackers && warp < issuer) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) red[my_row * S + my_col + c] = y[c];
    }
    __syncthreads();
    if (C > 1) ptx::cluster_sync();
    auto sum = [&](int row, int m) {
        if (C == 1) return p.terms == 2 ? red[row * S + m] + red[row * S + RPAD / 2 + m] : red[row * S + m];
        const uint32_t at = base + (uint32_t)(row * S + m) * 4u;
        float hi[8], lo[8], v = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < C) {
                const uint32_t peer = ptx::map_to_cta(at, (uint32_t)r);
                hi[r] = ld_cluster_f32(peer);
                lo[r] = p.terms == 2 ? ld_cluster_f32(peer + (RPAD / 2) * 4u) : 0.0f;
            }
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < C) v += hi[r] + lo[r];
        return v;
    };
    constexpr int OUT_LOG2 = GATED ? 6 : 7;
    const int outputs = M << OUT_LOG2, first = (int)((int64_t)outputs * rank / C), last = (int)((int64_t)outputs * (rank + 1) / C);
    for (int i = first + threadIdx.x; i < last; i += kW4UmmaThreads) {
        const int r = i & ((1 << OUT_LOG2) - 1), m = i >> OUT_LOG2, n = (group << OUT_LOG2) + r;
        if (n >= p.N) continue;
        const int64_t at = (int64_t)(m0 + m) * p.N + n;
        if constexpr (GATED) w4_store_terms(p.out, at, (int64_t)p.M * p.N, gate_act_f32(sum(r, m), p.act) * sum(r + 64, m));
        else p.out[at] = __float2bfloat16_rn(sum(r, m));
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
    const int n = blockIdx.x * 128 + threadIdx.x, kb = blockIdx.y, KB = gridDim.y, n16 = (N + 15) / 16;
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
        if (zeros != nullptr) zeros[at] = (uint8_t)(0x80 | ((int)z << 3));
    }
    uint8_t* out = codes + block * 1024 + ((n & 15) >> 3) * 512 + (n & 7) * 64;
#pragma unroll
    for (int j = 0; j < 16; ++j) word[j] = __funnelshift_l(word[j], word[j], 3);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        reinterpret_cast<uint4*>(out)[j] = make_uint4(word[4 * j], word[4 * j + 1], word[4 * j + 2], word[4 * j + 3]);
}

__global__ void __launch_bounds__(128)
w4_unpack_kernel(const uint8_t* codes, const bf16* scales, const uint8_t* zeros,
                 bf16* W, int out_in, int K, int N, int G)
{
    ptx::grid_dependency_wait();
    const int n = blockIdx.x * 128 + threadIdx.x, kb = blockIdx.y, KB = gridDim.y, ng = 128 / G;
    if (n >= N) return;
    const int64_t block = (int64_t)(n >> 4) * KB + kb;
    const uint32_t* word = reinterpret_cast<const uint32_t*>(codes + block * 1024 + ((n & 15) >> 3) * 512 + (n & 7) * 64);
    for (int k = 0; k < 128 && kb * 128 + k < K; ++k) {
        const int64_t at = (block * 16 + (n & 15)) * ng + k / G;
        const uint32_t w = __funnelshift_r(word[(k & 31) >> 1], word[(k & 31) >> 1], 3);
        const float q = (float)((w >> (4 * (k >> 5) + 16 * (k & 1))) & 15), z = zeros != nullptr ? (float)((zeros[at] >> 3) & 15) : 8.0f;
        const int64_t to = out_in ? (int64_t)n * K + kb * 128 + k : (int64_t)(kb * 128 + k) * N + n;
        W[to] = __float2bfloat16_rn((q - z) * __bfloat162float(scales[at]));
    }
}

}  // namespace gmlp
