// Attention of the new positions of ragged requests over a paged bf16 cache (first, plain form: one CTA per position and head).
#pragma once
#include "common.cuh"
#include "ptx.cuh"

namespace gmlp {

struct KvAttnArgs {
    const bf16* Q;                   // [T, Hq * D]
    bf16* O;
    const bf16 *k, *v;               // [page][Hkv][page_size][D]
    const int32_t *table, *lengths, *q_start;
    int B, T, Hq, Hkv, ratio, width, page_size, n_pages, q_len, causal;
    float scale_log2;
};

// Request b: its first row, its number of rows and keys; what the arrays hold outside of their ranges is reported and left out.
__device__ __forceinline__ void kv_request(const KvAttnArgs& a, int b, int& row0, int& rows, int& keys, bool report) {
    const int s = a.q_start ? a.q_start[b] : b * a.q_len, e = a.q_start ? a.q_start[b + 1] : s + a.q_len;
    const bool ok = s >= 0 && s <= e && e <= a.T;
    row0 = ok ? s : 0;
    rows = ok ? e - s : 0;
    keys = a.lengths[b];
    const bool fits = keys >= 0 && (int64_t)keys <= (int64_t)a.width * a.page_size;
    if (!fits) keys = 0;
    if (report && (!ok || !fits)) report_index(ok ? 7 : 6);
}

template <int D>
__global__ void __launch_bounds__(128) kv_attention_plain_kernel(const KvAttnArgs a)
{
    constexpr int C = D / 32;
    __shared__ float sm[4], sl[4], so[4][D];
    const int b = blockIdx.z, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    ptx::grid_dependency_wait();
    int row0, rows, keys;
    kv_request(a, b, row0, rows, keys, threadIdx.x == 0);
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t at = ((int64_t)(row0 + r) * a.Hq + h) * D;
        float q[C], o[C], m = -INFINITY, l = 0.0f;
        for (int c = 0; c < C; ++c) {
            q[c] = __bfloat162float(a.Q[at + lane * C + c]);
            o[c] = 0.0f;
        }
        const int seen = a.causal ? min(keys, keys - rows + r + 1) : keys;
        for (int j = warp; j < seen; j += 4) {
            const int page = a.table[(int64_t)b * a.width + j / a.page_size];
            if (page < 0 || page >= a.n_pages) {
                if (lane == 0) report_index(8);
                continue;
            }
            const int64_t kv = (((int64_t)page * a.Hkv + h / a.ratio) * a.page_size + j % a.page_size) * D + lane * C;
            float s = 0.0f;
            for (int c = 0; c < C; ++c) s += q[c] * __bfloat162float(a.k[kv + c]);
            for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, w);
            s *= a.scale_log2;
            const float top = fmaxf(m, s), base = top == -INFINITY ? 0.0f : top;
            const float f = exp2f(m - base), p = exp2f(s - base);
            l = l * f + p;
            for (int c = 0; c < C; ++c) o[c] = o[c] * f + p * __bfloat162float(a.v[kv + c]);
            m = top;
        }
        if (lane == 0) { sm[warp] = m; sl[warp] = l; }
        for (int c = 0; c < C; ++c) so[warp][lane * C + c] = o[c];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += 128) {
            float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), num = 0.0f, den = 0.0f;
            if (top == -INFINITY) top = 0.0f;
            for (int w = 0; w < 4; ++w) {
                const float f = exp2f(sm[w] - top);
                num += f * so[w][c];
                den += f * sl[w];
            }
            a.O[at + c] = __float2bfloat16_rn(den == 0.0f ? 0.0f : num / den);
        }
        __syncthreads();
    }
}

}  // namespace gmlp
