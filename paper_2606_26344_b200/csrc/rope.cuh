// Rotary positions, and rows of keys and values on their way into a paged bf16 cache.
//
// Pair i of a head's first `rot` channels turns by position * f_i and is multiplied by an amplitude A:
//     u' = A (u cos t - v sin t),   v' = A (u sin t + v cos t),   (u, v) = channels (2 i, 2 i + 1) or (i, i + rot / 2).
// The table holds f_i / (2 pi), turns per position, in units of 2^-64: position * step modulo 2^64 is the angle's place within the
// turn, exactly, however far the position; its upper 32 bits become the argument of one sincospi.  (In fp32 the angle of position
// 131072 would be off by 2^-8 radians: half a unit in the last place of its 17 bits before the point.)
//
// What bounds it: bytes, one read and one write of each row.  A pair's cosine and sine (some 40 instructions) serve all heads of a
// token, so a CTA takes whole tokens and computes them once, into shared memory; a thread then keeps those of its channels in
// registers and walks over the heads, 16 bytes (half layout: twice 16) at a time, four heads' loads in flight.
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace gmlp {

struct RotateArgs {
    const bf16 *Q, *K, *V;           // [T, Hq * D], [T, Hkv * D] twice; Hq or Hkv may be 0
    bf16* Qo;                        // may be Q
    bf16 *kc, *vc;                   // cache, [page][Hkv][page_size][D]
    const int64_t *positions, *slots;
    const uint64_t* steps;           // [rot / 2]
    float amplitude;
    int T, Hq, Hkv, D, rot;          // rot = 0: rows are moved as they are
    int page_size;
    int64_t total;                   // slots of the cache
    int tokens;                      // per CTA
};

constexpr int kRotateThreads = 256, kRotateBatch = 4, kRotateMaxTokens = 8;

template <int VEC> struct RotateVec;
template <> struct RotateVec<8> { typedef uint4 T; };
template <> struct RotateVec<2> { typedef uint32_t T; };

// VEC channels per access: 8, or 2 where the pairs' two halves do not start on 16 bytes.  blockDim.x = accesses ("units") per head;
// in the half layout a unit of rotated channels is the access at its first halves and the one at their partners.
template <int VEC, bool INTER>
__global__ void __launch_bounds__(kRotateThreads) rotate_kernel(const RotateArgs a)
{
    typedef typename RotateVec<VEC>::T Word;
    constexpr int PAIRS = INTER ? VEC / 2 : VEC, W = VEC / 2;
    extern __shared__ float2 cs[];                                   // [tokens][rot / 2]
    __shared__ int64_t s_row[kRotateMaxTokens];                      // row of head 0 in the cache, or -1

    const int half = a.rot >> 1;
    const int unit = threadIdx.x, n_rot = (INTER ? a.rot : half) / VEC;
    const bool turned = unit < n_rot, two = turned && !INTER;
    const int off = turned || INTER ? unit * VEC : a.rot + (unit - n_rot) * VEC;
    const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    const int t0 = blockIdx.x * a.tokens, nt = min(a.tokens, a.T - t0);

    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    for (int i = tid; i < nt * half; i += threads) {
        const int t = i / half, p = i - t * half;
        const uint64_t at = (uint64_t)a.positions[t0 + t] * a.steps[p];
        float s, c;
        sincospif((float)(int32_t)(at >> 32) * 0x1p-31f, &s, &c);
        cs[i] = make_float2(a.amplitude * c, a.amplitude * s);
    }
    if (a.Hkv > 0 && tid < nt) {
        const int64_t slot = a.slots[t0 + tid];
        int64_t row = -1;
        if (slot >= a.total) {
            if (blockIdx.y == 0) report_index(5);
        } else if (slot >= 0) {
            const int64_t page = slot / a.page_size;
            row = (page * a.Hkv) * a.page_size + (slot - page * a.page_size);
        }
        s_row[tid] = row;
    }
    __syncthreads();

    const int heads = a.Hq + 2 * a.Hkv, step = blockDim.y * gridDim.y;
    for (int t = 0; t < nt; ++t) {
        float c[PAIRS], s[PAIRS];
        if (turned) {
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) {
                const float2 v = cs[t * half + unit * PAIRS + p];
                c[p] = v.x;
                s[p] = v.y;
            }
        }
        const int64_t row = a.Hkv > 0 ? s_row[t] : 0, tok = t0 + t;
        for (int h0 = blockIdx.y * blockDim.y + threadIdx.y; h0 < heads; h0 += step * kRotateBatch) {
            union { Word v; uint32_t w[W]; } x[kRotateBatch], y[kRotateBatch];
            bf16* dst[kRotateBatch];
            bool turn[kRotateBatch];
#pragma unroll
            for (int i = 0; i < kRotateBatch; ++i) {
                const int h = h0 + i * step;
                const bf16* src = nullptr;
                dst[i] = nullptr;
                turn[i] = turned && h < a.Hq + a.Hkv;
                if (h < a.Hq) {
                    src = a.Q + ((int64_t)tok * a.Hq + h) * a.D + off;
                    dst[i] = a.Qo + ((int64_t)tok * a.Hq + h) * a.D + off;
                } else if (h < heads && row >= 0) {
                    const bool value = h >= a.Hq + a.Hkv;
                    const int g = h - a.Hq - (value ? a.Hkv : 0);
                    src = (value ? a.V : a.K) + ((int64_t)tok * a.Hkv + g) * a.D + off;
                    dst[i] = (value ? a.vc : a.kc) + (row + (int64_t)g * a.page_size) * a.D + off;
                }
                if (src != nullptr) {
                    x[i].v = *reinterpret_cast<const Word*>(src);
                    if (two) y[i].v = *reinterpret_cast<const Word*>(src + half);
                }
            }
#pragma unroll
            for (int i = 0; i < kRotateBatch; ++i) {
                if (dst[i] == nullptr) continue;
                if (turn[i]) {
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        if (INTER) {
                            const float u = bf16_lo(x[i].w[w]), v = bf16_hi(x[i].w[w]);
                            x[i].w[w] = pack_bf16x2(u * c[w] - v * s[w], u * s[w] + v * c[w]);
                        } else {
                            const float u0 = bf16_lo(x[i].w[w]), u1 = bf16_hi(x[i].w[w]), v0 = bf16_lo(y[i].w[w]), v1 = bf16_hi(y[i].w[w]);
                            const int p = 2 * w, q = PAIRS > 1 ? 2 * w + 1 : 0;
                            x[i].w[w] = pack_bf16x2(u0 * c[p] - v0 * s[p], u1 * c[q] - v1 * s[q]);
                            y[i].w[w] = pack_bf16x2(u0 * s[p] + v0 * c[p], u1 * s[q] + v1 * c[q]);
                        }
                    }
                }
                *reinterpret_cast<Word*>(dst[i]) = x[i].v;
                if (two) *reinterpret_cast<Word*>(dst[i] + half) = y[i].v;
            }
        }
    }
}

}  // namespace gmlp
