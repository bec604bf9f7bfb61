// Rotary positions, and rows of keys and values on their way into a paged bf16 cache.
//
// Pair i of a head's first `rot` channels turns by position * f_i and is multiplied by an amplitude A:
//     u' = A (u cos t - v sin t),   v' = A (u sin t + v cos t),   (u, v) = channels (2 i, 2 i + 1) or (i, i + rot / 2).
// The table holds f_i / (2 pi), turns per position, rounded to units of 2^-64: position * step modulo 2^64, an exact product, is the angle's
// place within the turn, off by the entry's rounding times the position (no more than fp32 takes anyway up to position 2^38); its upper 32 bits
// become the argument of one sincospi.  (In fp32 the angle of position
// 131072 would be off by 2^-8 radians: half a unit in the last place of its 17 bits before the point.)
//
// What bounds it: bytes, one read and one write of each row.  A pair's cosine and sine (some 40 instructions) serve all heads of a
// token, so a CTA takes whole tokens and computes them once, into shared memory; a thread then keeps those of its channels and goes
// over the heads, 16 bytes or twice 16 at a time, 64 bytes of loads in flight each, four CTAs per SM.
// 8191 tokens of 64 heads of 128 (268 MB both ways, floor 41.6 us): 69 us with 128 bytes in flight (two CTAs per SM), 51 with one token per
// CTA, 45 now; interleaved in units of one access 54.
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
    int turned_apart, apart;         // from the first to the second access of a unit that is turned, only moved; 0: it is one
    int page_size;
    int64_t total;                   // slots of the cache
    int tokens;                      // per CTA
    int lanes;                       // threads to a unit of a token's heads; blockDim.y is a multiple of it
};

constexpr int kRotateThreads = 256, kRotateMaxTokens = 8;

template <int VEC> struct RotateVec;
template <> struct RotateVec<8> { typedef uint4 T; };
template <> struct RotateVec<2> { typedef uint32_t T; };

// VEC channels per access: 8, or 2 where the pairs' two halves do not start on 16 bytes.  blockDim.x = units of a head, of two accesses each
// where the channels can be cut so: first halves and their partners, or (interleaved, and what is only moved) the lower and the upper half.
template <int VEC, bool INTER>
__global__ void __launch_bounds__(kRotateThreads, 4) rotate_kernel(const RotateArgs a)
{
    typedef typename RotateVec<VEC>::T Word;
    constexpr int W = VEC / 2, BATCH = 2;                            // W pairs of an interleaved access
    extern __shared__ float2 cs[];                                   // [tokens][rot / 2]
    __shared__ int64_t s_row[kRotateMaxTokens];                      // row of head 0 in the cache, or -1

    const int half = a.rot >> 1;
    const int unit = threadIdx.x, n_rot = (INTER && a.turned_apart == 0 ? a.rot : half) / VEC;
    const bool turned = unit < n_rot;
    const int off = turned ? unit * VEC : a.rot + (unit - n_rot) * VEC;
    const int apart = turned ? a.turned_apart : a.apart;             // from a unit's first access to its second, or 0
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

    const int heads = a.Hq + 2 * a.Hkv, step = a.lanes * gridDim.y;
    const int h_first = blockIdx.y * a.lanes + threadIdx.y % a.lanes;
    for (int t = threadIdx.y / a.lanes; t < nt; t += blockDim.y / a.lanes) {
        float c[VEC], s[VEC];                                        // of the pairs; interleaved: the first access's, the second's
        if (turned) {
#pragma unroll
            for (int p = 0; p < VEC; ++p) {
                if (INTER && p >= W && apart == 0) continue;
                const float2 v = cs[t * half + (!INTER ? unit * VEC + p : (p < W ? unit * W + p : apart / 2 + unit * W + p - W))];
                c[p] = v.x;
                s[p] = v.y;
            }
        }
        const int64_t row = a.Hkv > 0 ? s_row[t] : 0, tok = t0 + t;
        for (int h0 = h_first; h0 < heads; h0 += step * BATCH) {
            union { Word v; uint32_t w[W]; } x[BATCH], y[BATCH];
            bf16* dst[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int h = h0 + i * step;
                const bf16* src = nullptr;
                dst[i] = nullptr;
                if (h < a.Hq) {
                    const int64_t from = (tok * a.Hq + h) * a.D + off;
                    src = a.Q + from;
                    dst[i] = a.Qo + from;
                } else if (h < heads && row >= 0) {
                    const bool value = h >= a.Hq + a.Hkv;
                    const int g = h - a.Hq - (value ? a.Hkv : 0);
                    src = (value ? a.V : a.K) + (tok * a.Hkv + g) * a.D + off;
                    dst[i] = (value ? a.vc : a.kc) + (row + (int64_t)g * a.page_size) * a.D + off;
                }
                if (src != nullptr) {
                    x[i].v = *reinterpret_cast<const Word*>(src);
                    if (apart > 0) y[i].v = *reinterpret_cast<const Word*>(src + apart);
                }
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (dst[i] == nullptr) continue;
                if (turned && h0 + i * step < a.Hq + a.Hkv) {
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        if (INTER) {
                            const float u = bf16_lo(x[i].w[w]), v = bf16_hi(x[i].w[w]);
                            x[i].w[w] = pack_bf16x2(u * c[w] - v * s[w], u * s[w] + v * c[w]);
                            if (apart > 0) {
                                const float u1 = bf16_lo(y[i].w[w]), v1 = bf16_hi(y[i].w[w]);
                                y[i].w[w] = pack_bf16x2(u1 * c[W + w] - v1 * s[W + w], u1 * s[W + w] + v1 * c[W + w]);
                            }
                        } else {
                            const float u0 = bf16_lo(x[i].w[w]), u1 = bf16_hi(x[i].w[w]), v0 = bf16_lo(y[i].w[w]), v1 = bf16_hi(y[i].w[w]);
                            const int p = 2 * w, q = 2 * w + 1;
                            x[i].w[w] = pack_bf16x2(u0 * c[p] - v0 * s[p], u1 * c[q] - v1 * s[q]);
                            y[i].w[w] = pack_bf16x2(u0 * s[p] + v0 * c[p], u1 * s[q] + v1 * c[q]);
                        }
                    }
                }
                *reinterpret_cast<Word*>(dst[i]) = x[i].v;
                if (apart > 0) *reinterpret_cast<Word*>(dst[i] + apart) = y[i].v;
            }
        }
    }
}

}  // namespace gmlp
