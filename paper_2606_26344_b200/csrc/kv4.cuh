// A paged key/value cache held in 4 bits, and attention over it.
//
// Cache: codes [n_pages][n_kv_heads][page_size][D / 2] bytes and parameters [n_pages][n_kv_heads][page_size][D / G] pairs of
// bf16 (scale s, zero point z, an integer 0..15), one such pair of arrays for K and one for V; a value is (q - z) * s.  A token
// lives in slot page * page_size + place.  The D codes of a row lie in 32 units of D / 32 nibbles, channel c in nibble c / 32 of
// unit c % 32 (16-bit units for D = 128, bytes for D = 64): a lane that reads 8 neighbouring units of a key gets, with one shift
// and one and-or per pair, the A operands of the score product, a lane that reads 4 units of a value those of the output product,
// and each nibble position holds channels of one block of 32, so that every mma stays inside one group of G >= 32 channels.
#pragma once
#include <cfloat>

#include "common.cuh"
#include "ptx.cuh"
#include "w4_matmul.cuh"

namespace gmlp {

// The nibbles at bit `shift` (0, 4, 8, 12) of both halves of a word as bf16 16 + q (the nibble in the upper four mantissa bits).  The
// lowest one comes up by a multiplication: on another pipe than the shifts, whose pipe is the busier.
__device__ __forceinline__ uint32_t kv4_codes_plus_16(uint32_t w, int shift) {
    return and_or(shift == 0 ? w * 8u : w >> (shift - 3), 0x00780078u, 0x41804180u);
}

struct Kv4Cache {
    uint8_t* codes[2];         // K, V
    uint32_t* params[2];       // bf16 pairs: scale in the low half, zero point in the high half
    int n_pages, n_kv_heads, page_size, head_dim, group;
};

// ------------------------------------------------------------------------------------------------ append and gather
__device__ __forceinline__ float redux_min_nan(float v) {
    float r;
    asm("redux.sync.min.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float redux_max_nan(float v) {
    float r;
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// One warp per token, head and K or V.  Lane r holds unit r, channels r + 32 j; minimum and maximum of a group are warp
// reductions.  Bound by HBM (256 bytes in, 68 to 80 out per row of 128 channels) and, for a few tokens, by the launch.
template <int D, int G>
__global__ void __launch_bounds__(256)
kv4_append_kernel(const bf16* K, const bf16* V, const Kv4Cache c, const int64_t* slots, int64_t items, int64_t total_slots)
{
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    constexpr int NJ = D / 32, NG = D / G, PER = G / 32;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);       // (token * 2 + which) * heads + head
    if (item >= items) return;
    const int64_t tw = item / c.n_kv_heads;
    const int head = (int)(item - tw * c.n_kv_heads), which = (int)(tw & 1);
    const int64_t token = tw >> 1;
    const int64_t slot = slots[token];
    if (slot < 0) return;                            // padding: nothing is written
    if (slot >= total_slots) {
        if (lane == 0) report_index(1);
        return;
    }
    const bf16* x = (which ? V : K) + (token * c.n_kv_heads + head) * D;
    float v[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] = __bfloat162float(x[j * 32 + lane]);
    const uint32_t page = (uint32_t)slot / (uint32_t)c.page_size;
    const int64_t row = ((int64_t)page * c.n_kv_heads + head) * c.page_size + ((uint32_t)slot - page * (uint32_t)c.page_size);
    uint32_t unit = 0, par[NG];
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
        float lo = v[gi * PER], hi = lo;
        bool finite = lo - lo == 0.0f;
#pragma unroll
        for (int j = 1; j < PER; ++j) {
            const float a = v[gi * PER + j];
            lo = fminf(lo, a);
            hi = fmaxf(hi, a);
            finite = finite && a - a == 0.0f;
        }
        if (!finite) lo = hi = __int_as_float(0x7FC00000);
        lo = redux_min_nan(lo);
        hi = redux_max_nan(hi);
        finite = lo - lo == 0.0f;                    // a NaN of any lane is in both
        lo = fminf(lo, 0.0f);
        hi = fmaxf(hi, 0.0f);
        float s = __bfloat162float(__float2bfloat16_rn((hi - lo) / 15.0f));
        if (!finite || s - s != 0.0f) s = __int_as_float(0x7FC00000);
        const bool some = s > 0.0f;
        const float z = some ? fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 0.0f;
        par[gi] = pack_bf16x2(s, z);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const float q = some ? fminf(fmaxf(rintf(v[gi * PER + j] / s) + z, 0.0f), 15.0f) : 0.0f;
            unit |= (uint32_t)q << (4 * (gi * PER + j));
        }
    }
    uint8_t* codes = (which ? c.codes[1] : c.codes[0]) + row * (D / 2);
    if constexpr (D == 128) reinterpret_cast<uint16_t*>(codes)[lane] = (uint16_t)unit;
    else codes[lane] = (uint8_t)unit;
    if (lane < NG) {
        uint32_t mine = par[0];
#pragma unroll
        for (int gi = 1; gi < NG; ++gi)
            if (lane == gi) mine = par[gi];
        (which ? c.params[1] : c.params[0])[row * NG + lane] = mine;
    }
}

// Slots back to bf16 rows [T][n_kv_heads * D].  Four lanes per token, head and K or V: a lane reads 8 units and writes 8
// neighbouring channels of each block of 32.  Bound by the bf16 rows it writes.
template <int D, int G>
__global__ void __launch_bounds__(256)
kv4_gather_kernel(const Kv4Cache c, const int64_t* slots, bf16* K, bf16* V, int64_t items, int64_t total_slots)
{
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    constexpr int NJ = D / 32, NG = D / G;
    const int t = threadIdx.x & 3;
    const int64_t item = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2);
    if (item >= items) return;
    const int64_t tw = item / c.n_kv_heads;
    const int head = (int)(item - tw * c.n_kv_heads), which = (int)(tw & 1);
    const int64_t token = tw >> 1;
    const int64_t slot = slots[token];
    bf16* out = (which ? V : K) + (token * c.n_kv_heads + head) * D + 8 * t;
    if (slot < 0 || slot >= total_slots) {           // padding: a row of zeros; a slot past the cache is reported, too
        if (slot >= 0 && t == 0) report_index(2);
#pragma unroll
        for (int j = 0; j < NJ; ++j) *reinterpret_cast<uint4*>(out + 32 * j) = make_uint4(0, 0, 0, 0);
        return;
    }
    const uint32_t page = (uint32_t)slot / (uint32_t)c.page_size;
    const int64_t row = ((int64_t)page * c.n_kv_heads + head) * c.page_size + ((uint32_t)slot - page * (uint32_t)c.page_size);
    uint32_t w[D / 32], par[NG];
    const uint8_t* codes = (which ? c.codes[1] : c.codes[0]) + row * (D / 2) + t * (D / 8);
    if constexpr (D == 128) {
        const uint4 u = *reinterpret_cast<const uint4*>(codes);
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(codes);
        w[0] = u.x; w[1] = u.y;
    }
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) par[gi] = (which ? c.params[1] : c.params[0])[row * NG + gi];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const float s = bf16_lo(par[j * 32 / G]), z = bf16_hi(par[j * 32 / G]);
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                // units 2 i and 2 i + 1
            uint32_t a, b;
            if constexpr (D == 128) {
                a = (w[i] >> (4 * j)) & 15u;
                b = (w[i] >> (16 + 4 * j)) & 15u;
            } else {
                a = (w[i >> 1] >> (16 * (i & 1) + 4 * j)) & 15u;
                b = (w[i >> 1] >> (16 * (i & 1) + 8 + 4 * j)) & 15u;
            }
            o[i] = pack_bf16x2(((float)a - z) * s, ((float)b - z) * s);
        }
        *reinterpret_cast<uint4*>(out + 32 * j) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// ------------------------------------------------------------------------------------------------ attention
// T new positions per request (the last T of its sequence), O = softmax(scale * Q K^T) V over the keys up to each position's
// own.  A CTA takes one request, one key/value head, up to 8 NT of its T * (query heads per key/value head) query rows and a range
// of the keys; its four warps take 16-token tiles in turn.  Per tile and warp (running maximum and sum in fp32):
//   S^T = K Q^T   tokens are the 16 mma rows, query rows the 8 columns, 16 + q exact in bf16; (16 + z) times the query row's sum
//                 over the group comes off, the token's scale is a factor, and the softmax scale one of the sum, all in fp32;
//   P'  = exp2(S - m) * s_v as two bf16 terms (hi + lo: rounded to one, the output was 1.4 times as far off as its own rounding
//                 leaves it), transposed in registers (movmatrix);
//   O^T += V^T P'^T   with 16 + q again; the sum of P' (16 + z), a scalar per query row and group, is formed in fp32 from the same two
//                 terms and taken off at the end and every few tiles (kv4_tiles_between).
// 64 requests of 1..8192 keys, 32 / 8 heads of 128, groups of 64: 130 us (2.8 TB/s, 0.43 of the measured copy rate); one request of
// 131071 keys, 64 / 8 heads, groups of 128: 57 us (2.5 TB/s).  No pipe is full (32 requests of 4096 keys: integer pipe 58 % busy,
// issue slots 59 %, tensor pipe 24 %, HBM 2.5 TB/s): three warps per scheduler wait in turn for their copies, products and exchanges;
// a tile takes 468 warp instructions, 120 of them the unpacking.  With one term for P' 115 and 51 us; so, but with loads into
// registers instead of the rings 146 and 67; with the maximum followed at every tile and q - z formed before the products 126 and 53.
// Each warp has a ring of three tiles in shared memory that asynchronous copies fill, two tiles ahead; the page-table entry is read
// one tile earlier still.  Row g of a tile's products is token g ^ (g >> 1) of its eight (and so for the second eight), and for
// D = 128 the 16-byte chunks of rows 2, 3, 6, 7, ... swap places by two: so the keys' reads (a row by four lanes) and the values' (a
// row by eight) are both free of bank conflicts.
constexpr int kKv4Warps = 4;
constexpr int kKv4Threads = 32 * kKv4Warps;
constexpr int kKv4Tile = 16;
// Tiles of a warp between two returns of the offset (a power of two).  A product's additions may round toward zero, and while the
// accumulators hold the offset too, all of them, in all warps, lose to the same side; the output that is left shrinks with the root
// of the length.  Error of the output over that of its own rounding alone, and time, with 64, 8, 4 and 1 tiles in between:
//   64 requests of 1..8192 keys      1.0020, 1.0003, 1.0001, 1.0000      130.2, 131.4, 132.5, 138.6 us
//   131071 keys, 64 / 8 heads         1.175,  1.016,  1.007,  1.001       54.6,  55.0,  56.0,  57.6 us
//   1200000 keys, 4 / 1 heads of 64     4.4,   1.12,   1.06,   1.01       54.6,  55.6,  56.1,  57.8 us
__device__ __forceinline__ int kv4_tiles_between(int len) { return len <= 16384 ? 8 : (len <= 262144 ? 4 : 1); }

struct Kv4AttnArgs {
    const bf16* Q;             // [B * T][Hq * D]
    bf16* O;
    Kv4Cache c;
    const int32_t* table;      // [B][width]
    const int32_t* lengths;    // [B]
    float* part;               // [B * Hkv * col_tiles][splits][8 NT][D + 4]: O, maximum, sum, two unused; nothing for one split
    int B, T, Hq, ratio, width, splits, col_tiles;
    uint32_t q_scale;          // bf16, twice: a power of two that the queries are taken times, and what the scores are then multiplied with
    float s_scale;
};

// Keys per split of a request with `len` keys: the same formula in both kernels.
__device__ __forceinline__ int kv4_split_keys(int len, int splits) {
    const int per = (len + splits - 1) / splits;
    const int rounded = (per + kKv4Warps * kKv4Tile - 1) / (kKv4Warps * kKv4Tile) * (kKv4Warps * kKv4Tile);
    return rounded < 2 * kKv4Warps * kKv4Tile ? 2 * kKv4Warps * kKv4Tile : rounded;
}
// A request's keys: its length, or what its row of the page table can hold.
__device__ __forceinline__ int kv4_length(const Kv4AttnArgs& p, int b) {
    const int64_t most = (int64_t)p.width * p.c.page_size;
    const int len = p.lengths[b];
    return len < 0 ? 0 : ((int64_t)len > most ? (int)most : len);
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A tile in shared memory: codes of K, codes of V (16 rows of D / 2 bytes), parameters of K, of V (16 rows of 4 * D / G bytes).
constexpr int kKv4Depth = 3;
__host__ __device__ constexpr int kv4_slot_bytes(int D, int G) { return 16 * D + 128 * (D / G); }
__host__ __device__ constexpr int kv4_smem_bytes(int D, int G, int NT) {       // rings; at the end the warps' results in their place
    const int rings = kKv4Warps * kKv4Depth * kv4_slot_bytes(D, G), results = kKv4Warps * 8 * NT * (D + 4) * 4;
    return rings > results ? rings : results;
}
template <int N>
__device__ __forceinline__ void lds_words(uint32_t (&d)[N], const uint8_t* p) {
    if constexpr (N == 1) {
        d[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        d[0] = v.x; d[1] = v.y;
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
    }
}

// What a warp has of its query rows: the sums of P' V, one row per lane and block of channels, the base and the sum of P.
template <int D, int NT>
struct Kv4Sums {
    float o[D / 16][NT][4], m[NT][2], l[NT][2];
};
// The warp's tiles from the first to the last; false where a sum is no number or came near the end of float's range (2^100: the warps
// and splits are still to be added).  CAREFUL, the second try: a masked token's zero point is kept out of the sums whatever it is
// (ordinary ones cost nothing there: their probability is 0), and the base of the exponentials counts in what a value's scale has
// above 2^60, so that no sum of P' (16 + q) passes 2^96; the base is common to the sum of the probabilities, and the quotient
// stays what it is.
template <int D, int G, int NT, bool CAREFUL>
__device__ __forceinline__ bool kv4_warp_sums(const Kv4AttnArgs& p, Kv4Sums<D, NT>& sums)
{
    constexpr int NJ = D / 32, NG = D / G, PER = G / 32, MT = D / 16;        // blocks of 32, groups, output tiles
    constexpr int COLS = 8 * NT, SLOT = kv4_slot_bytes(D, G);
    extern __shared__ __align__(128) uint8_t kv4_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x, head = (int)blockIdx.y / p.col_tiles, ct = (int)blockIdx.y % p.col_tiles, b = blockIdx.z;
    const int cols_all = p.T * p.ratio, col0 = ct * COLS;
    const int len = kv4_length(p, b), keys = kv4_split_keys(len, p.splits), first = split * keys, last = min(first + keys, len);

    // query operands: column n = query row col0 + n of this head, channels 32 j + 8 t + 0..7
    uint32_t q[NT][NJ][4];
    int limit[NT][2];                                // keys that the lane's two columns of a tile may see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = col0 + n * 8 + g;
        const int i = col / p.ratio, r = col - i * p.ratio;
        const bf16* row = p.Q + ((int64_t)(b * (int64_t)p.T + i) * p.Hq + head * p.ratio + r) * D + 8 * t;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (col < cols_all) x = *reinterpret_cast<const uint4*>(row + 32 * j);
            if constexpr (D == 128) {
                q[n][j][0] = x.x; q[n][j][1] = x.y; q[n][j][2] = x.z; q[n][j][3] = x.w;
            } else {                                 // bytes come apart as units (0, 2), (1, 3), (4, 6), (5, 7)
                q[n][j][0] = __byte_perm(x.x, x.y, 0x5410);
                q[n][j][1] = __byte_perm(x.x, x.y, 0x7632);
                q[n][j][2] = __byte_perm(x.z, x.w, 0x5410);
                q[n][j][3] = __byte_perm(x.z, x.w, 0x7632);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) q[n][j][u] = bf16x2_fma(q[n][j][u], p.q_scale, 0x80008000u);       // - 0: a product, exact
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = col0 + n * 8 + 2 * t + e;
            limit[n][e] = c < cols_all ? min(last, len - p.T + 1 + c / p.ratio) : 0;
        }
    }

    // sums of the query rows over the groups, at the lane's columns (2 t and 2 t + 1): what (16 + z) is multiplied with
    float qsum[NT][NG][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
            float v = 0.0f;
#pragma unroll
            for (int jj = 0; jj < PER; ++jj)
#pragma unroll
                for (int u = 0; u < 4; ++u) v += bf16_lo(q[n][gi * PER + jj][u]) + bf16_hi(q[n][gi * PER + jj][u]);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
            qsum[n][gi][0] = __shfl_sync(0xFFFFFFFFu, v, 8 * t);             // lane 4 g holds column g
            qsum[n][gi][1] = __shfl_sync(0xFFFFFFFFu, v, 8 * t + 4);
        }
    const int full_limit = min(last, len - p.T + 1 + col0 / p.ratio);       // below it every column sees every key

    auto& o = sums.o;
    auto& m = sums.m;
    auto& l = sums.l;
    float zsum[NG][NT][2];
    auto take_off = [&]() {                          // o -= the sum of P' (16 + z), which every lane holds a part of
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int gi = 0; gi < NG; ++gi) {
                    float z = zsum[gi][n][e];
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, x);
#pragma unroll
                    for (int j = gi * PER; j < (gi + 1) * PER; ++j)
#pragma unroll
                        for (int hw = 0; hw < 2; ++hw) {
                            o[j * 2 + hw][n][e] -= z;
                            o[j * 2 + hw][n][2 + e] -= z;
                        }
                    zsum[gi][n][e] = 0.0f;
                }
    };
    const int32_t* table = p.table + (int64_t)b * p.width;
    // Places of this warp's tiles, stepped without divisions: page-table entry `entry`, token `place` of its page.
    const int stride = kKv4Warps * kKv4Tile, page_step = stride / p.c.page_size, place_step = stride % p.c.page_size;
    auto advance = [&](int& entry, int& place) {
        entry += page_step;
        place += place_step;
        if (place >= p.c.page_size) {
            place -= p.c.page_size;
            ++entry;
        }
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            m[n][e] = -INFINITY;
            l[n][e] = 0.0f;
#pragma unroll
            for (int gi = 0; gi < NG; ++gi) zsum[gi][n][e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][n][e] = 0.0f;
    }

    // Asks for the warp's next tile, one commit group per call; a page outside of the cache is not read.  Tokens past the end of a
    // request may hold anything.  Bit i of `ok`: the i-th tile from the current one lies in the cache.
    uint8_t* ring = kv4_smem + warp * (kKv4Depth * SLOT);
    const int lane_code = D == 128 ? (lane >> 2) * 64 + (((lane & 3) ^ (((lane >> 3) & 1) << 1)) * 16) : lane * 16;
    const bool lane_param = (lane & 15) < 4 * NG;
    const int lane_param_to = 16 * D + (lane >> 4) * (64 * NG) + (lane & 15) * 16;
    const uint8_t* param_base = reinterpret_cast<const uint8_t*>(lane >> 4 ? p.c.params[1] : p.c.params[0]) + (lane & 15) * 16;
    int ask_token = first + warp * kKv4Tile, entry = ask_token / p.c.page_size, place = ask_token - entry * p.c.page_size;
    int page = ask_token < last ? (int)ld_4B(table + entry) : -1;
    uint32_t ok = 0, ask_to = ptx::smem_addr(ring);
    const uint32_t ring_end = ask_to + kKv4Depth * SLOT;
    auto ask = [&](int bit) {
        if (ask_token < last) {
            if ((uint32_t)page < (uint32_t)p.c.n_pages) {
                const int64_t row = ((int64_t)page * p.c.n_kv_heads + head) * p.c.page_size + place;
                const uint8_t* k = p.c.codes[0] + row * (D / 2) + lane * 16;
                const uint8_t* v = p.c.codes[1] + row * (D / 2) + lane * 16;
                const uint32_t to = ask_to + lane_code;
                cp_async_16(to, k);
                cp_async_16(to + 8 * D, v);
                if constexpr (D == 128) {
                    cp_async_16(to + 512, k + 512);
                    cp_async_16(to + 8 * D + 512, v + 512);
                }
                if (lane_param) cp_async_16(ask_to + lane_param_to, param_base + row * (4 * NG));
                ok |= 1u << bit;
            }
            ask_token += stride;
            advance(entry, place);
            if (ask_token < last) page = (int)ld_4B(table + entry);
        }
        ask_to += SLOT;
        if (ask_to == ring_end) ask_to -= kKv4Depth * SLOT;
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kKv4Depth - 1; ++i) ask(i);

    const int gray = g ^ (g >> 1);                   // the token of row g
    const int swap = D == 128 ? ((gray >> 1) & 1) << 1 : 0;
    const uint8_t* slot = ring;
    const int between = kv4_tiles_between(len) - 1;
    int tiles = 0;
    for (int token = first + warp * kKv4Tile; token < last; token += stride) {
        if ((tiles++ & between) == between) take_off();
        cp_async_wait_but<kKv4Depth - 2>();          // this tile has landed,
        __syncwarp();                                // for every lane, and the slot of the tile before is free
        ask(kKv4Depth - 1);
        const bool page_ok = ok & 1;
        ok >>= 1;
        if (!page_ok && lane == 0) report_index(4);
        struct {
            uint32_t k[2][D / 32];                   // rows g and g + 8: units 8 t .. 8 t + 7
            uint32_t v[4][D / 64];                   // rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9: units 4 g .. 4 g + 3
            uint32_t kp[2][NG], vp[2][NG];
        } cur;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = gray + 8 * h;
            lds_words<D / 32>(cur.k[h], slot + row * (D / 2) + (t ^ swap) * (D / 8));
            lds_words<NG>(cur.kp[h], slot + 16 * D + row * (4 * NG));
            lds_words<NG>(cur.vp[h], slot + 16 * D + 64 * NG + row * (4 * NG));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 2 * t + i, tok = (r ^ (r >> 1)) + 8 * h;
                const int chunk = D == 128 ? (((g >> 1) ^ (((tok >> 1) & 1) << 1)) * 16 + (g & 1) * 8) : g * 4;
                lds_words<D / 64>(cur.v[2 * h + i], slot + 8 * D + tok * (D / 2) + chunk);
            }
        }
        slot += SLOT;
        if (slot == ring + kKv4Depth * SLOT) slot = ring;

        // scores of tokens (rows) g and g + 8, columns 2 t and 2 t + 1
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
            float acc[NT][4];
#pragma unroll
            for (int jj = 0; jj < PER; ++jj) {
                const int j = gi * PER + jj;
                uint32_t a[8];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int at = (u >> 1) * 4 + (u & 1) * 2;
#pragma unroll
                    for (int h = 0; h < 2; ++h) a[at + h] = kv4_codes_plus_16(D == 128 ? cur.k[h][u] : cur.k[h][u >> 1], D == 128 ? 4 * j : 8 * (u & 1) + 4 * j);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (jj == 0) mma_bf16_16816_first(acc[n], a[0], a[1], a[2], a[3], q[n][j][0], q[n][j][1]);
                    else mma_bf16_16816(acc[n], a[0], a[1], a[2], a[3], q[n][j][0], q[n][j][1]);
                    mma_bf16_16816(acc[n], a[4], a[5], a[6], a[7], q[n][j][2], q[n][j][3]);
                }
            }
            const float s0 = bf16_lo(cur.kp[0][gi]), s1 = bf16_lo(cur.kp[1][gi]);
            const float z0 = bf16_hi(cur.kp[0][gi]) + 16.0f, z1 = bf16_hi(cur.kp[1][gi]) + 16.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][0] = fmaf(fmaf(-z0, qsum[n][gi][0], acc[n][0]), s0, s[n][0]);
                s[n][1] = fmaf(fmaf(-z0, qsum[n][gi][1], acc[n][1]), s0, s[n][1]);
                s[n][2] = fmaf(fmaf(-z1, qsum[n][gi][0], acc[n][2]), s1, s[n][2]);
                s[n][3] = fmaf(fmaf(-z1, qsum[n][gi][1], acc[n][3]), s1, s[n][3]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] *= p.s_scale;
        // Masks, where a tile needs them: a masked score is -inf whatever its token holds.
        const bool full = page_ok && token + kKv4Tile <= full_limit;         // of the whole warp
        const int t0 = page_ok ? token + gray : INT_MAX - 16;
        if (!full) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (t0 >= limit[n][e]) s[n][e] = -INFINITY;
                    if (t0 + 8 >= limit[n][e]) s[n][2 + e] = -INFINITY;
#pragma unroll
                    for (int gi = 0; gi < NG; ++gi) {                        // past the request's end: parameters of no effect
                        if (t0 >= last) cur.vp[0][gi] = 0;
                        if (t0 + 8 >= last) cur.vp[1][gi] = 0;
                    }
                }
        }
        // The base of the exponentials follows the maximum of a column only once a score is more than 8 (in powers of two) above it:
        // sums of up to 2^8 are as good as sums of up to 1, and most tiles need no reduction over the lanes.
        bool above = CAREFUL;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) above = above || fmaxf(s[n][e], s[n][2 + e]) > m[n][e] + 8.0f;
        if (__any_sync(0xFFFFFFFFu, above)) {
            float lift[2] = {0.0f, 0.0f};        // of the lane's two tokens
            if constexpr (CAREFUL) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float step = 0.0f;
#pragma unroll
                    for (int gi = 0; gi < NG; ++gi) step = fmaxf(step, fabsf(bf16_lo(cur.vp[h][gi])));
                    lift[h] = fmaxf(log2f(fminf(step, FLT_MAX)) - 60.0f, 0.0f);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float alpha[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = CAREFUL ? fmaxf(s[n][e] + lift[0], s[n][2 + e] + lift[1]) : fmaxf(s[n][e], s[n][2 + e]);
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
                    alpha[e] = 1.0f;
                    if (top > m[n][e]) {
                        alpha[e] = fast_exp2(m[n][e] - top);                 // 0 from -inf
                        m[n][e] = top;
                    }
                    l[n][e] *= alpha[e];
#pragma unroll
                    for (int gi = 0; gi < NG; ++gi) zsum[gi][n][e] *= alpha[e];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    o[i][n][0] *= alpha[0];
                    o[i][n][1] *= alpha[1];
                    o[i][n][2] *= alpha[0];
                    o[i][n][3] *= alpha[1];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float base = m[n][e] == -INFINITY ? 0.0f : m[n][e];
                s[n][e] = fast_exp2(s[n][e] - base);
                s[n][2 + e] = fast_exp2(s[n][2 + e] - base);
                l[n][e] += s[n][e] + s[n][2 + e];
            }
        // second product, group by group
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
            uint32_t pb[NT][2], pl[NT][2];           // P' as two terms
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float sv = bf16_lo(cur.vp[h][gi]);
                    float a = s[n][2 * h] * sv, c = s[n][2 * h + 1] * sv;
                    if (!full) {                     // a masked token adds nothing, not even 0 * NaN
                        a = t0 + 8 * h < limit[n][0] ? a : 0.0f;
                        c = t0 + 8 * h < limit[n][1] ? c : 0.0f;
                    }
                    const uint32_t w = pack_bf16x2(a, c);
                    const float z = bf16_hi(cur.vp[h][gi]) + 16.0f;
                    const uint32_t r = pack_bf16x2(a - bf16_lo(w), c - bf16_hi(w));
                    float za = z, zc = z;
                    if constexpr (CAREFUL) {
                        if (t0 + 8 * h >= limit[n][0]) za = 0.0f;
                        if (t0 + 8 * h >= limit[n][1]) zc = 0.0f;
                    }
                    zsum[gi][n][0] = fmaf(bf16_lo(w) + bf16_lo(r), za, zsum[gi][n][0]);    // of what the product sees
                    zsum[gi][n][1] = fmaf(bf16_hi(w) + bf16_hi(r), zc, zsum[gi][n][1]);
                    pb[n][h] = movmatrix_trans(w);
                    pl[n][h] = movmatrix_trans(r);
                }
#pragma unroll
            for (int hw = 0; hw < 2; ++hw) {
                // the two tokens of a pair side by side: units 4 g + 2 hw and 4 g + 2 hw + 1
                uint32_t lo01, hi01, lo89, hi89;
                if constexpr (D == 128) {
                    lo01 = __byte_perm(cur.v[0][hw], cur.v[1][hw], 0x5410);
                    hi01 = __byte_perm(cur.v[0][hw], cur.v[1][hw], 0x7632);
                    lo89 = __byte_perm(cur.v[2][hw], cur.v[3][hw], 0x5410);
                    hi89 = __byte_perm(cur.v[2][hw], cur.v[3][hw], 0x7632);
                } else {
                    lo01 = __byte_perm(cur.v[0][0], cur.v[1][0], hw ? 0x7632 : 0x5410);
                    lo89 = __byte_perm(cur.v[2][0], cur.v[3][0], hw ? 0x7632 : 0x5410);
                    hi01 = lo01 >> 8;
                    hi89 = lo89 >> 8;
                }
#pragma unroll
                for (int jj = 0; jj < PER; ++jj) {
                    const int j = gi * PER + jj;
                    const uint32_t a0 = kv4_codes_plus_16(lo01, 4 * j), a2 = kv4_codes_plus_16(lo89, 4 * j);
                    const uint32_t a1 = kv4_codes_plus_16(hi01, 4 * j), a3 = kv4_codes_plus_16(hi89, 4 * j);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_bf16_16816(o[j * 2 + hw][n], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                        mma_bf16_16816(o[j * 2 + hw][n], a0, a1, a2, a3, pl[n][0], pl[n][1]);
                    }
                }
            }
        }
    }
    cp_async_wait_all();
    take_off();
    float size = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) size += fabsf(o[i][n][e]);
    return __all_sync(0xFFFFFFFFu, size < 1.2676506e30f);                    // the lanes are done with the ring, too
}
// The second try is a call of its own: inlined beside the first, 64 ragged requests took 131.2 us instead of 129.6.
template <int D, int G, int NT>
__device__ __noinline__ void kv4_warp_sums_careful(const Kv4AttnArgs& p, Kv4Sums<D, NT>& sums)
{
    Kv4Sums<D, NT> mine;
    (void)kv4_warp_sums<D, G, NT, true>(p, mine);
    sums = mine;
}

template <int D, int G, int NT>
__global__ void __launch_bounds__(kKv4Threads, NT == 1 ? 3 : 2) kv4_attention_kernel(const __grid_constant__ Kv4AttnArgs p)
{
    constexpr int NJ = D / 32, COLS = 8 * NT;
    extern __shared__ __align__(128) uint8_t kv4_smem[];
    float (*s_o)[COLS][D + 4] = reinterpret_cast<float (*)[COLS][D + 4]>(kv4_smem);        // [warp][column][channel]
    __shared__ float s_m[kKv4Warps][COLS], s_l[kKv4Warps][COLS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x, head = (int)blockIdx.y / p.col_tiles, ct = (int)blockIdx.y % p.col_tiles, b = blockIdx.z;
    const int cols_all = p.T * p.ratio, col0 = ct * COLS;

    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int len = kv4_length(p, b);
    if (split > 0 && split * kv4_split_keys(len, p.splits) >= len) return;   // the joining kernel uses the same formula and does not look here
    if (split == 0 && ct == 0 && head == 0 && threadIdx.x == 0 && (p.lengths[b] < 0 || p.lengths[b] > len)) report_index(3);

    Kv4Sums<D, NT> sums;
    if (!kv4_warp_sums<D, G, NT, false>(p, sums)) {
        Kv4Sums<D, NT> again;
        kv4_warp_sums_careful<D, G, NT>(p, again);
        sums = again;
    }
    auto& o = sums.o;
    auto& m = sums.m;
    auto& l = sums.l;
    __syncthreads();                                 // the rings are done with: the results take their place

    // sums over the lanes that share a column, then the warps' results side by side
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], x);
            const int c = n * 8 + 2 * t + e;
            if (g == 0) {
                s_m[warp][c] = m[n][e];
                s_l[warp][c] = l[n][e];
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int hw = 0; hw < 2; ++hw) {
                    float* at = &s_o[warp][c][32 * j + 4 * g + 2 * hw];
                    at[0] = o[j * 2 + hw][n][e];
                    at[1] = o[j * 2 + hw][n][2 + e];
                }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < COLS * (D / 4); i += kKv4Threads) {
        const int c = i / (D / 4), d = (i % (D / 4)) * 4, col = col0 + c;
        if (col >= cols_all) continue;
        float top = s_m[0][c];
#pragma unroll
        for (int w = 1; w < kKv4Warps; ++w) top = fmaxf(top, s_m[w][c]);
        float sum = 0.0f;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kKv4Warps; ++w) {
            const float f = s_m[w][c] == -INFINITY ? (s_l[w][c] != s_l[w][c] ? s_l[w][c] : 0.0f) : fast_exp2(s_m[w][c] - top);
            sum = fmaf(f, s_l[w][c], sum);
            const float4 x = *reinterpret_cast<const float4*>(&s_o[w][c][d]);
            v.x = fmaf(f, x.x, v.x);
            v.y = fmaf(f, x.y, v.y);
            v.z = fmaf(f, x.z, v.z);
            v.w = fmaf(f, x.w, v.w);
        }
        if (p.splits == 1) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;               // a row that sees no key is 0
            const int i_pos = col / p.ratio, r = col - i_pos * p.ratio;
            bf16* out = p.O + ((int64_t)(b * (int64_t)p.T + i_pos) * p.Hq + head * p.ratio + r) * D + d;
            *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
        } else {
            float* out = p.part + ((((int64_t)b * gridDim.y + blockIdx.y) * p.splits + split) * COLS + c) * (D + 4);
            *reinterpret_cast<float4*>(out + d) = v;
            if (d == 0) *reinterpret_cast<float2*>(out + D) = make_float2(top, sum);
        }
    }
}

// Joins the splits of one query row: their largest maximum, their weights, then the weighted sums, a share of the splits per group
// of threads; all in a fixed order.
constexpr int kKv4MaxSplits = 256;
template <int D, int NT, int THREADS>
__global__ void __launch_bounds__(THREADS) kv4_join_kernel(const Kv4AttnArgs p)
{
    constexpr int COLS = 8 * NT, V = D / 4, SHARES = THREADS / V;            // a thread takes four channels of every SHARES-th split
    __shared__ float s_w[kKv4MaxSplits], s_l[kKv4MaxSplits];
    __shared__ float4 s_o[SHARES][V];
    const int row = blockIdx.x, b = row / (p.T * p.Hq), rest = row % (p.T * p.Hq), i = rest / p.Hq, h = rest % p.Hq;
    const int head = h / p.ratio, col = i * p.ratio + h % p.ratio, ct = col / COLS, c = col % COLS;
    ptx::grid_dependency_wait();
    ptx::launch_dependents();
    const int len = kv4_length(p, b), keys = kv4_split_keys(len, p.splits);
    const int used = len == 0 ? 1 : (len + keys - 1) / keys;
    const float* base = p.part + ((((int64_t)b * p.c.n_kv_heads + head) * p.col_tiles + ct) * p.splits * COLS + c) * (D + 4);
    const int64_t step = (int64_t)COLS * (D + 4);
    for (int s = threadIdx.x; s < used; s += THREADS) {
        const float2 ml = *reinterpret_cast<const float2*>(base + s * step + D);
        s_w[s] = ml.x;
        s_l[s] = ml.y;
    }
    const int share = threadIdx.x / V, v = threadIdx.x % V;
    __syncthreads();
    float top = -INFINITY;
    for (int s = 0; s < used; ++s) top = fmaxf(top, s_w[s]);
    if (top == -INFINITY) top = 0.0f;                // nothing seen: every weight is 0
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int s = share; s < used; s += SHARES) {
        const float f = fast_exp2(s_w[s] - top);
        const float4 x = *reinterpret_cast<const float4*>(base + s * step + v * 4);
        o.x = fmaf(f, x.x, o.x);
        o.y = fmaf(f, x.y, o.y);
        o.z = fmaf(f, x.z, o.z);
        o.w = fmaf(f, x.w, o.w);
    }
    s_o[share][v] = o;
    __syncthreads();
    if (threadIdx.x < V) {
        float sum = 0.0f;                            // a split of which every score was NaN has a NaN sum and no maximum: it is kept
        for (int s = 0; s < used; ++s) sum += s_l[s] != s_l[s] ? s_l[s] : fast_exp2(s_w[s] - top) * s_l[s];
        float4 x = s_o[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < SHARES; ++w) {
            const float4 a = s_o[w][threadIdx.x];
            x.x += a.x;
            x.y += a.y;
            x.z += a.z;
            x.w += a.w;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        bf16* out = p.O + ((int64_t)(b * (int64_t)p.T + i) * p.Hq + h) * D + threadIdx.x * 4;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
    }
}

}  // namespace gmlp
