// Attention of the new positions of ragged requests over a paged bf16 cache:  O = softmax(scale Q K^T) V, request by request.
//
// Rows.  The query heads that share a key/value head are rows of one tile next to one another: with R heads to a key/value head a tile of
// 128 rows is P = 128 / R positions.  So K and V are read once for all R heads, one token of a request already fills R rows, and a causal
// tile of a chunk spans few positions.  A work item is up to 2 P positions of one request and key/value head:
//   big   (more than P positions): two tiles of 128 rows that take turns on the tensor pipe, both over every block of 128 keys;
//   small (up to P positions):     one tile of rows, the two "tiles" take the even and the odd blocks of keys and are joined at the
//                                  end.  Bytes bound these, so the probabilities get a second bf16 term (16 bits) for the tensor pipe's spare time;
//   few   (up to 16 rows, e.g. single tokens): the products are turned round, S^T = K Q^T and O^T += V^T P^T, so that the 128 keys
//                                  of a block, not 16 rows of 128, are the threads' lanes: a block's softmax takes some 16 exponentials a thread
//                                  instead of 128 (0.4 us instead of 1.9, two terms as well), which leaves the copies as the bound.  The
//                                  items of a CTA go to the two tiles in turn, so that one's end and the next one's start overlap.
// Order and split.  All items lie end to end on one axis, heads outermost, an item as long as the keys that its last position sees plus
// a constant; every CTA (one per SM) takes an equal stretch of the axis, computed by itself from the lengths on the device (the host knows
// none of them).  So a decode batch of ragged lengths, one long conversation and a prompt's chunk all load the GPU evenly, without a plan
// kernel.  A cut item's parts (at most two per CTA) leave unnormalised fp32 sums, base and weight in the workspace; a second, small
// kernel joins them in order, so results do not depend on timing.
//
//   warp 0      K/V producer: K(0), V(0), K(1), ... through one FIFO, a page (or its share of a block) per TMA box; rows of no page
//               are zeros in V, which a probability of 0 would not hide if they were NaN
//   warp 1      MMA issuer:   S_t = Q_t K^T (TMEM columns 128 t), O_t += P_t V (columns 256 + 128 t)
//   warp 2      walks the axis, hands items to the others through a ring, loads Q
//   warp 3      looks for pages outside of the cache, and mends V blocks that hold keys which some row must not see: rows past the
//               request's end become zeros, numbers that are none become 0 and are added by the epilogue for the rows that see them
//   warps 4..7  softmax and epilogue of tile A, warps 8..11 of tile B: thread = row.  As in gqa_attention.cuh: scores are read once, the base
//               of the exponentials moves only when a row's sum of a block passes 2^10, P goes back to TMEM over the scores.
// Every wait is bounded.
//
// Values of any size.  O is a sum of p V before it is divided by the sum of p, and p may pass 1 (the base moves late), so large values pass the
// largest float although the result does not; an infinity that a row sees in a block that is not mended may become NaN, since the second
// term of its probability may be negative or 0.  An epilogue that finds such a sum asks for a second pass over its CTA's stretch (`careful`):
// the same items one at a time, with every block of V mended and multiplied by 2^-48 (the sums of p stay below 2^40), and what is not finite
// from the first pass is written anew; the rest stays.  Parts of cut items are divided by their own sum of p, so that the join weighs means.
// Calls without a second pass pay for the test, the join's weights and the longer code: 256 requests of 200 keys 90 us, 87 before; one token over
// 2^20 keys 102 and 99; 64 of 4096 keys 179 and 178; a prompt of 8192 the same.  A second pass takes three to five times as long as a first.
// Scores: from 2^31 binary orders on, the rounding of the base alone (a product of a score and the scale) passes the exponents of fp32.
#pragma once
#include <type_traits>
#include <cuda.h>

#include "common.cuh"
#include "gqa_attention.cuh"
#include "ptx.cuh"
#include "umma_gemm.cuh"

namespace gmlp {

struct KvAttnArgs {
    bf16* O;                         // [T, Hq * D]
    const bf16* v;                   // [page][Hkv][page_size][D]
    const int32_t *table, *lengths, *q_start;
    uint8_t* workspace;
    int B, T, Hq, Hkv, ratio, width, page_size, n_pages, q_len, causal;
    int tile_pos;                    // positions per 128 rows
    int box;                         // keys per TMA box: the largest power of two that divides the page size, at most 128
    int few_pos;                     // positions per 16 rows (0: more than 16 heads share a key/value head)
    int q_bytes, q_few_bytes;        // of one tile's Q boxes
    int slot_rows;                   // rows of a partial result
    int min_stretch;                 // of a CTA, on the axis; more than a block of a big item
    float scale_log2;
};

constexpr int kKvThreads = 384, kKvBlock = 128, kKvRing = 4;
constexpr int kKvFew = 16;                       // rows of an item whose products are turned round
// Blocks that a few item's O is summed over before it is added to a second sum, 16 columns on.  The tensor pipe cuts where it adds, always
// towards 0, 16 times a block: over 8192 blocks in one sum (2^20 keys) the error's norm was 1.8 times that of the last rounding, 3.8 with values
// of one sign.
constexpr int kKvFewSum = 256;
// Big and small items have no tensor memory for a second sum.  They are handed out in pieces of this many blocks; between two of them their rows'
// sums wait in the workspace (one such item over 2^20 keys: 3.6 times the last rounding's error without pieces with values of one sign).
constexpr int kKvPiece = 512;
enum { kKvGoesOn = 1, kKvMore = 2 };             // a piece: earlier ones went before it, others come after it
constexpr int kKvMends = 8;                       // more than the FIFO holds blocks of V
// The axis: what a key of an item takes, and an item's start and end.  In a batch of both, big items are bound by the tensor pipe and the
// softmax and the others by the copies, which run the faster the fewer SMs make them (40 single tokens and three chunks: 301 us with the
// same for all, 265 with 3 : 2 : 2, 244 with 4 : 3 : 2, 267 with 5 : 3 : 2).  Starts: a prompt of 8192 641 us with 64 keys, 560 with 256, 515 now.
constexpr int kKvBigKey = 4, kKvSmallKey = 3, kKvFewKey = 2;
constexpr int kKvBigStart = 448 * kKvBigKey, kKvSmallStart = 384 * kKvSmallKey, kKvFewStart = 256 * kKvFewKey;
constexpr int kKvRegsLight = 72, kKvRegsSoftmax = 216;
constexpr int kKvKernelId = 30;
constexpr float kKvCareful = 0x1p-48f;                       // what the second pass multiplies V by
constexpr uint32_t kKvWaitLimit = 8;                         // some 20 s: some waits last as long as an item
__host__ __device__ constexpr int kv_slots(int D) { return D == 128 ? 5 : 10; }
__host__ __device__ constexpr uint32_t kv_tile_bytes(int D) { return 128u * D * 2; }
constexpr uint32_t kKvRegion = 32768;            // of a tile: Q, and in few items P^T behind it
// the tiles' regions, FIFO; base and weight of rows; what the warps of few items exchange; items and barriers
constexpr uint32_t kv_attn_smem(int D) { return 2 * kKvRegion + kv_slots(D) * kv_tile_bytes(D) + 1024 + 1024 + 1024; }

// Workspace: one descriptor per CTA - the cut item that its stretch ends in - then base and weight of the rows of each of its two partial
// results, then their rows, divided by the weight, then the sums of each tile's rows between two pieces of an item.
struct KvCut {
    int parts, first;                // parts (less than two: none), the CTA that has the first of them
    int head, row0, npos, two_tiles, pad[2];
};
__host__ __device__ inline uint64_t kv_ws_stats(int ctas) { return ((uint64_t)ctas * sizeof(KvCut) + 255) & ~(uint64_t)255; }
__host__ __device__ inline uint64_t kv_ws_sums(int ctas, int slot_rows) {
    return kv_ws_stats(ctas) + (((uint64_t)ctas * 2 * slot_rows * 8 + 255) & ~(uint64_t)255);
}
__host__ __device__ inline uint64_t kv_ws_pieces(int ctas, int slot_rows, int D) {
    return kv_ws_sums(ctas, slot_rows) + (uint64_t)ctas * 2 * slot_rows * D * 4;
}
__host__ __device__ inline int kv_tile_rows(int slot_rows) { return slot_rows < 128 ? slot_rows : 128; }
__host__ __device__ inline uint64_t kv_ws_bytes(int ctas, int slot_rows, int D) {
    return kv_ws_pieces(ctas, slot_rows, D) + (uint64_t)ctas * 2 * kv_tile_rows(slot_rows) * D * 4;
}

struct KvItem {
    int blk0, blk1;                  // blocks of keys; none: rows that see no key
    int b, head, row0;               // request, key/value head, row of Q of the first position
    int npos, keys;                  // positions, keys of the request
    int seen0;                       // keys that the first position sees (may be negative)
    int slot;                        // of the partial result, or -1: the rows' final values
    int last;                        // no more items (this one is none)
    int mode, tile;                  // kKvBigItem ..; the tile of a few item
    int careful;                     // the second pass
    int piece, part0;                // kKvGoesOn, kKvMore; the first block of the item's part in this CTA
    int pad;
};

// Request b: its first row, rows and keys; what the arrays hold outside of their ranges is left out (and reported by one CTA).
__device__ __forceinline__ void kv_request(const KvAttnArgs& a, int b, int& row0, int& rows, int& keys, bool report) {
    const int s = a.q_start ? a.q_start[b] : b * a.q_len, e = a.q_start ? a.q_start[b + 1] : s + a.q_len;
    const bool ok = s >= 0 && s <= e && e <= a.T;
    row0 = ok ? s : 0;
    rows = ok ? e - s : 0;
    keys = a.lengths[b];
    const bool fits = keys >= 0 && (int64_t)keys <= (int64_t)a.width * a.page_size;
    if (!fits) keys = 0;
    if (report && (!ok || !fits)) report_index(ok ? 6 : 7);
}
// Up to this length an item is never cut: a part costs as much as the keys that it saves.  Items of nearly the same length stay whole too
// where no CTA then has more than this on top of an equal share.  One token over this many keys, 32 query and 8 key/value heads of 128, cut
// and whole: 100 requests of 400 keys 65 and 58 us; 16 of 1500 30.4 and 26.7; 16 of 4000 57.8 and 53.7.  52 of 837 to 1402 with two heads
// and a quarter more per CTA than that were slower whole, 32 against 24.
constexpr int kKvSnap = 1536;
enum { kKvBigItem = 0, kKvSmallItem = 1, kKvFewItem = 2 };
constexpr uint32_t kKvHidden = 1, kKvSeen = 2;               // of keys that some row must not see; in the second pass, of the others
__device__ __forceinline__ int kv_mode(const KvAttnArgs& a, int npos) {
    return npos <= a.few_pos ? kKvFewItem : (npos <= a.tile_pos ? kKvSmallItem : kKvBigItem);
}
__host__ __device__ constexpr int kv_start(int mode) { return mode == kKvBigItem ? kKvBigStart : (mode == kKvSmallItem ? kKvSmallStart : kKvFewStart); }
__host__ __device__ constexpr int kv_key(int mode) { return mode == kKvBigItem ? kKvBigKey : (mode == kKvSmallItem ? kKvSmallKey : kKvFewKey); }
__device__ __forceinline__ int kv_tiles(const KvAttnArgs& a, int rows) { return (rows + 2 * a.tile_pos - 1) / (2 * a.tile_pos); }
// Length on the axis of the first n of a request's tiles; all but the last are big.
__device__ __forceinline__ int64_t kv_cost(const KvAttnArgs& a, int rows, int keys, int n) {
    if (n == 0) return 0;
    const int s = 2 * a.tile_pos;
    const bool whole = (int64_t)n * s >= rows;                      // the last tile ends with the request
    const int m = whole ? n - 1 : n;
    int64_t cost = (int64_t)m * kKvBigStart;
    if (whole) {
        const int mode = kv_mode(a, rows - m * s);
        cost += kv_start(mode) + (int64_t)kv_key(mode) * keys;
    }
    if (!a.causal) return cost + (int64_t)kKvBigKey * m * keys;
    const int first = keys - rows;                                  // tile i of the others sees first + (i + 1) s keys
    const int none = first < 0 ? min(m, -first / s) : 0;
    return cost + kKvBigKey * ((int64_t)(m - none) * first + (int64_t)s * ((int64_t)m * (m + 1) - (int64_t)none * (none + 1)) / 2);
}
// Blocks of an item that lie before place x of it.
__device__ __forceinline__ int kv_blocks_before(int64_t x, int mode, int blocks) {
    const int each = kKvBlock * kv_key(mode);
    const int64_t n = x <= kv_start(mode) ? 0 : (x - kv_start(mode) + each - 1) / each;
    return (int)min(n, (int64_t)blocks);
}

__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, float (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ float tmem_ld_32x1(uint32_t taddr) {
    float r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=f"(r) : "r"(taddr) : "memory");
    return r;
}
__device__ __forceinline__ void tmem_st_32x1(uint32_t taddr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "f"(v) : "memory");
}
// the largest of a warp's values, NaN left out
__device__ __forceinline__ float redux_max_f32(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// Three coordinates: channel, head, position.
__device__ __forceinline__ void tma_load_3d(uint32_t dst_smem, const void* tmap, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst_smem), "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ bool is_finite(float x) { return x - x == 0.0f; }
__device__ __forceinline__ uint32_t bf16_pair_times(uint32_t w, float f) {
    const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&w), __float2bfloat162_rn(f));
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ bool bf16_pair_not_finite(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// The same number, which the compiler takes for another one each time: conditions on it are not moved out of a loop by doubling the loop.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+r"(v));
    return v;
}
__device__ __forceinline__ uint32_t clock_hi() {
    uint32_t t;
    asm volatile("mov.u32 %0, %%clock_hi;" : "=r"(t));
    return t;
}
// A bounded wait of a whole warp.  Smaller than wait_bounded (limit in units of 2^32 cycles, reported at the kernel's end): it stands in some
// thirty places, and the kernel's code has to stay in the instruction cache - at 298 KB, everything inline several times over, each step of
// a short item cost microseconds.
__device__ __forceinline__ bool kv_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int site) {
    bool ok = ptx::mbar_try_wait(bar, parity);
    if (!ok) {
        const uint32_t start = clock_hi();
#pragma unroll 1
        while (!(ok = ptx::mbar_try_wait(bar, parity)) && *abort_flag == 0)
            if (clock_hi() - start > kKvWaitLimit) *abort_flag = site;
    }
    return __all_sync(0xFFFFFFFFu, ok);                              // the outcome is the warp's
}

// A place in the FIFO: slot and the parity of its use.
template <int SLOTS> struct KvCursor {
    uint32_t slot, phase;
    __device__ __forceinline__ void move(uint32_t n) {               // n < SLOTS
        slot += n;
        if (slot >= SLOTS) { slot -= SLOTS; phase ^= 1u; }
    }
    __device__ __forceinline__ void skip(uint32_t n) {
        const uint32_t at = slot + n;
        phase ^= (at / SLOTS) & 1u;
        slot = at % SLOTS;
    }
};

// FEW: with the code of few items; without it they are small ones.  LONG: an item may have more than kKvFewSum blocks; the others need no code for
// that (256 requests of 200 keys 91 us without it, 95 with it; 64 of 4096 keys 178 and 179).
template <int D, bool FEW, bool LONG>
__global__ void __launch_bounds__(kKvThreads, 1)
kv_attention_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmQfew, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const KvAttnArgs a)
{
    constexpr int SLOTS = kv_slots(D), HALVES = D / 64;
    constexpr uint32_t TILE = kv_tile_bytes(D), HALF = 16384;                // 128 rows of 64 channels
    // S = Q K^T: A and B K-major, N = 128 keys;  O += P V: B MN-major, N = D;  M = 128, bf16 in, fp32 accumulate
    constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);

    // few items: S^T = K Q^T, M = 128 keys, N = 16;  O^T += V^T P^T: A MN-major, B K-major, M = 128 channels
    constexpr uint32_t kIdescFewQK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kKvFew >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t kIdescFewPV = kIdescFewQK | (1u << 15);
    // P^T of a few item behind its Q: two buffers of two terms, each two blocks of 64 keys, 16 rows of 128 B
    constexpr uint32_t P_BUF = 16384, P_AT = 4096, P_TERM = 4096, P_HALF = 2048;

    // (no static shared memory: this starts the CTA's, whose first kilobyte is the system's)
    extern __shared__ __align__(1024) uint8_t base_ptr[];
    const uint32_t base = ptx::smem_addr(base_ptr);
    if (base & 1023u) {                                                      // the swizzled tiles count on it
        ptx::grid_dependency_wait();
        if (threadIdx.x == 0) {
            report_timeout(kKvKernelId, 0);
            reinterpret_cast<KvCut*>(a.workspace)[blockIdx.x] = KvCut{};         // nothing to join
        }
        return;
    }
    const uint32_t q_smem = base, fifo = base + 2 * kKvRegion;
    uint8_t* fifo_ptr = base_ptr + 2 * kKvRegion;
    uint8_t* tail_ptr = fifo_ptr + SLOTS * TILE;
    float2* stats = reinterpret_cast<float2*>(tail_ptr);                     // [128]: base and weight of tile B's rows
    float* exchange = reinterpret_cast<float*>(tail_ptr + 1024);             // [tile][maxima, sums][16 rows][4 warps]
    KvItem* items = reinterpret_cast<KvItem*>(tail_ptr + 2048);              // [ring]
    uint64_t* bars = reinterpret_cast<uint64_t*>(items + kKvRing);
    const uint32_t kv_full0 = ptx::smem_addr(bars);                          // [slots]
    const uint32_t kv_empty0 = kv_full0 + 8 * SLOTS;                         // [slots]
    // [tile][buffer], the second buffer in few items only:
    const uint32_t s_full0 = kv_empty0 + 8 * SLOTS;                          // scores of a step are in TMEM
    const uint32_t p_full0 = s_full0 + 32;                                   // its probabilities are in place
    const uint32_t o_full0 = p_full0 + 32;                                   // O += P V of a step is done
    const uint32_t q_full0 = o_full0 + 32, q_empty0 = q_full0 + 16;          // [tile] its region holds Q, is free
    const uint32_t mend0 = q_empty0 + 16, fixed0 = mend0 + 8 * kKvMends;     // a block of V to be mended is on its way, has been mended: in turn
    const uint32_t item_full0 = fixed0 + 8 * kKvMends, item_empty0 = item_full0 + 8 * kKvRing, item_fixed0 = item_empty0 + 8 * kKvRing;
    const uint32_t item_checked0 = item_fixed0 + 8 * kKvRing;
    const uint32_t stats_full = item_checked0 + 8 * kKvRing, stats_done = stats_full + 8;
    const uint32_t agree0 = stats_done + 8;                                  // [tile] the warps of a few item's tile
    constexpr int BARS = 2 * SLOTS + 20 + 2 * kKvMends + 4 * kKvRing;
    volatile uint32_t* hidden = reinterpret_cast<volatile uint32_t*>(bars + BARS);   // [ring] V held numbers that are none (kKvHidden, kKvSeen)
    volatile uint32_t* odd_pages = hidden + kKvRing;                         // [ring] the table has pages outside of the cache
    volatile uint32_t* votes = odd_pages + kKvRing;                          // [tile][parity][4 warps]
    uint32_t* tmem_slot = const_cast<uint32_t*>(votes) + 16;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* redo = abort_flag + 1;                                     // some O was not finite
    static_assert(sizeof(KvItem) * kKvRing + 8 * BARS + 4 * (2 * kKvRing + 19) <= 1024, "items and barriers");
    // (second pass) [channel]: the sum of the numbers that are none in V of keys that all rows of the item see.  One item at a time, so that
    // what the other kinds of items exchange is free.
    auto seen_by_all = [&](int mode) { return mode == kKvFewItem ? reinterpret_cast<float*>(stats) : exchange; };
    // for the start only, in the same place as `stats`: sums of costs, the place within the first item, its request and tile
    int64_t* s_scan = reinterpret_cast<int64_t*>(stats);
    int64_t* s_rest = s_scan + kKvThreads / 32;
    int* s_start = reinterpret_cast<int*>(s_rest + 1);
    int2* s_range = reinterpret_cast<int2*>(s_start + 2);                    // shortest and longest item

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    ptx::launch_dependents();
    if (tid == 0) {
        auto init = [](uint32_t bar, int n, int count) { for (int i = 0; i < n; ++i) ptx::mbar_init(bar + 8 * i, count); };
        init(kv_full0, 2 * SLOTS, 1);
        init(s_full0, 4, 1);
        init(p_full0, 4, 4);                                                 // one arrival per softmax warp of the tile
        init(o_full0, 4, 1);
        init(q_full0, 4, 1);
        init(mend0, 2 * kKvMends, 1);
        init(item_full0, kKvRing, 1);
        init(item_empty0, kKvRing, 11);                                      // producer, issuer, mender, eight softmax warps
        init(item_fixed0, kKvRing, 1);
        init(item_checked0, kKvRing, 1);
        init(stats_full, 4, 4);
        *abort_flag = 0;
        *redo = 0;
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
        ptx::prefetch_tensormap(&tmQ);
        ptx::prefetch_tensormap(&tmQfew);
        ptx::prefetch_tensormap(&tmK);
        ptx::prefetch_tensormap(&tmV);
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_addr(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    ptx::grid_dependency_wait();

    // ---------------- this CTA's stretch of the axis ----------------
    const int per = (a.B + kKvThreads - 1) / kKvThreads, b_lo = min(a.B, tid * per), b_hi = min(a.B, b_lo + per);
    int64_t mine = 0;
    int least = 0x7FFFFFFF, most = 0;                                        // shortest and longest item
    for (int b = b_lo; b < b_hi; ++b) {
        int row0, rows, keys;
        kv_request(a, b, row0, rows, keys, blockIdx.x == 0);
        mine += kv_cost(a, rows, keys, kv_tiles(a, rows));
        if (rows > 0) {
            const int mode = kv_mode(a, rows), c = kv_start(mode) + kv_key(mode) * min(keys, 1 << 28);
            least = min(least, rows > 2 * a.tile_pos ? 1 : c);               // several tiles: of unlike lengths
            most = max(most, c);
        }
    }
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    int64_t upto = mine;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const int64_t v = __shfl_up_sync(0xFFFFFFFFu, upto, w);
        if (lane >= w) upto += v;
    }
    if (lane == 31) {
        s_scan[warp] = upto;
        s_range[warp] = make_int2(least, most);
    }
    __syncthreads();
    int64_t per_head = 0;
#pragma unroll
    for (int w = 0; w < kKvThreads / 32; ++w) {
        if (w < warp) upto += s_scan[w];
        per_head += s_scan[w];
    }
    const int64_t total = per_head * a.Hkv;
    const int64_t stretch = max((total + gridDim.x - 1) / gridDim.x, (int64_t)a.min_stretch);
    const int64_t lo = stretch * blockIdx.x, hi = min(total, lo + stretch);
    const int head_lo = lo < hi ? (int)(lo / per_head) : 0;
    if (lo < hi) {
        const int64_t rest = lo - head_lo * per_head;
        if (rest >= upto - mine && rest < upto) {                            // one thread's requests hold the start
            int64_t at = upto - mine;
            for (int b = b_lo; b < b_hi; ++b) {
                int row0, rows, keys;
                kv_request(a, b, row0, rows, keys, false);
                const int n = kv_tiles(a, rows);
                const int64_t c = kv_cost(a, rows, keys, n);
                if (rest < at + c) {
                    int first = 0, last = n - 1;                             // the tile that holds it
                    while (first < last) {
                        const int mid = (first + last + 1) / 2;
                        if (at + kv_cost(a, rows, keys, mid) <= rest) first = mid;
                        else last = mid - 1;
                    }
                    s_start[0] = b;
                    s_start[1] = first;
                    *s_rest = rest - at - kv_cost(a, rows, keys, first);
                    break;
                }
                at += c;
            }
        }
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;                                   // S_t at + 128 t, O_t at + 256 + 128 t

    // All warps meet here at the end of a pass, at item i, which is the last, or after a wait that ran out.  True: there is a second pass, from the
    // next item on.
    auto next_pass = [&](uint32_t& i) -> bool {
        ptx::tc_fence_before_sync();
        asm volatile("bar.sync 0;" ::: "memory");
        ptx::tc_fence_after_sync();
        if (__builtin_expect(*redo == 0 || *abort_flag != 0, 1) || items[i % kKvRing].careful) return false;
        __syncwarp();
        if (lane == 0 && warp == 3) {                                        // (one phase of each of the place's barriers per use)
            ptx::mbar_arrive(item_checked0 + 8 * (i % kKvRing));
            ptx::mbar_arrive(item_fixed0 + 8 * (i % kKvRing));
        }
        if (lane == 0 && warp != 2) ptx::mbar_arrive(item_empty0 + 8 * (i % kKvRing));
        ++i;
        return true;
    };

    if (warp < 4) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kKvRegsLight));
      auto item_done = [&](uint32_t i) {
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(item_empty0 + 8 * (i % kKvRing));
      };
      // the item in ring place i; false when there is no more in this pass
      auto next_item = [&](uint32_t i, KvItem& it) -> bool {
          if (!kv_wait(item_full0 + 8 * (i % kKvRing), (i / kKvRing) & 1u, abort_flag, 1)) return false;
          it = items[i % kKvRing];
          return it.last == 0;
      };
      // the first key of the item that some row of it must not see
      auto first_hidden = [&](const KvItem& it) { return min(max(it.seen0, 0), it.keys); };

      if (warp == 0) {
        // ---------------- K/V producer ----------------
        KvCursor<SLOTS> at = {0, 0};
        uint32_t n_mends = 0;
        KvItem it;
        const int boxes = kKvBlock / a.box;
        const uint32_t box_bytes = (uint32_t)a.box * 128u;
        const int my = lane % boxes, half = lane / boxes;                    // this lane's box of a block and half of the channels
        const bool copies = lane < boxes * HALVES;
        uint32_t i = 0;
        do for (; next_item(i, it); ++i) {
            const int32_t* table = a.table + (int64_t)it.b * a.width;
            // the page of this lane's box in block j: -1 past the request's end, -2 outside of the cache
            auto page_of = [&](int j, int& place) -> int {
                const int key = j * kKvBlock + my * a.box;
                if (j >= it.blk1 || key >= it.keys) return -1;
                const int index = key / a.page_size;
                place = key - index * a.page_size;
                const int page = table[index];
                return page >= 0 && page < a.n_pages ? page : -2;
            };
            const int open = it.careful ? 0 : first_hidden(it) / kKvBlock;   // blocks before this one need no mending
            int place_next = 0, page_next = page_of(it.blk0, place_next);
            bool ok = true;
#pragma unroll 1
            for (int j = it.blk0; j < it.blk1 && ok; ++j) {
                const int page = page_next, place = place_next;
                page_next = page_of(j + 1, place_next);                      // asked for a block ahead
                if (page == -2 && half == 0 && copies) report_index(8);
                const bool there = page >= 0;
                const uint32_t bytes = __popc(__ballot_sync(0xFFFFFFFFu, there && copies)) * box_bytes;
                const int row = (page * a.Hkv + it.head) * a.page_size + place;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (!kv_wait(kv_empty0 + 8 * at.slot, at.phase ^ 1u, abort_flag, 2)) { ok = false; break; }
                    const uint32_t full = kv_full0 + 8 * at.slot, dst = fifo + at.slot * TILE + half * HALF + my * box_bytes;
                    if (kv == 1 && __any_sync(0xFFFFFFFFu, copies && page == -2)) {      // (past the end: the mender's)
                        if (copies && page == -2) {
                            uint4* z = reinterpret_cast<uint4*>(fifo_ptr + at.slot * TILE + half * HALF + my * box_bytes);
                            for (uint32_t n = 0; n < box_bytes / 16; ++n) z[n] = make_uint4(0, 0, 0, 0);
                        }
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                    }
                    if (lane == 0) ptx::mbar_arrive_expect_tx(full, bytes);
                    __syncwarp();
                    if (copies && there) ptx::tma_load_2d(dst, kv == 0 ? &tmK : &tmV, 64 * half, row, full);
                    if (kv == 1 && j >= open) {
                        if (lane == 0) ptx::mbar_arrive(mend0 + 8 * (n_mends % kKvMends));
                        ++n_mends;
                    }
                    at.move(1);
                }
            }
            if (!ok) break;
            item_done(i);
        } while (next_pass(i));
        __syncwarp();
      } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        // (as in gqa_attention.cuh: all lanes run the loop so that the operands are warp-uniform, one lane issues)
        const bool leader = ptx::elect_one();
        const uint32_t desc_hi = (uint32_t)(ptx::make_smem_desc_sw128(0, 0, 1024) >> 32);
        const uint32_t q_lo = (uint32_t)ptx::make_smem_desc_sw128(q_smem, 16, 1024);
        const uint32_t k_lo_base = (uint32_t)ptx::make_smem_desc_sw128(fifo, 16, 1024);
        const uint32_t v_lo_base = (uint32_t)ptx::make_smem_desc_sw128(fifo, HALF, 1024);
        const uint32_t p_lo = (uint32_t)ptx::make_smem_desc_sw128(q_smem + P_AT, 16, 1024);
        // V as the A operand of few items: 128 channels.  With D = 64 rows 64.. of O^T are never read: their atom may lie anywhere
        const uint32_t v_few_base = (uint32_t)ptx::make_smem_desc_sw128(fifo, D == 128 ? HALF : 1024, 1024);
        KvCursor<SLOTS> k_at = {0, 0}, v_at = {1, 0};
        uint32_t p_phase = 0, q_phase = 0, n_fixed = 0;                      // bits: [tile][buffer]; [tile]
        KvItem it;
        auto wait_all = [&](uint32_t bar, uint32_t phase, int site) -> bool {
            const bool ok = kv_wait(bar, phase, abort_flag, site);
            ptx::tc_fence_after_sync();
            return ok;
        };
        auto wait_q = [&](int t) -> bool {
            const bool ok = wait_all(q_full0 + 8 * t, (q_phase >> t) & 1u, 3);
            q_phase ^= 1u << t;
            return ok;
        };
        // the next block's keys, its values (mended where they hold keys that some row must not see)
        auto wait_k = [&](uint32_t& slot) -> bool {
            if (!wait_all(kv_full0 + 8 * k_at.slot, k_at.phase, 4)) return false;
            slot = k_at.slot;
            k_at.move(2);
            return true;
        };
        auto wait_v = [&](uint32_t& slot, bool mended) -> bool {
            if (!wait_all(kv_full0 + 8 * v_at.slot, v_at.phase, 6)) return false;
            slot = v_at.slot;
            v_at.move(2);
            if (!mended) return true;
            const bool ok = wait_all(fixed0 + 8 * (n_fixed % kKvMends), (n_fixed / kKvMends) & 1u, 7);
            ++n_fixed;
            return ok;
        };
        auto wait_p = [&](int at) -> bool {
            const bool ok = wait_all(p_full0 + 8 * at, (p_phase >> at) & 1u, 5);
            p_phase ^= 1u << at;
            return ok;
        };
        uint32_t i = 0;
        do for (; next_item(i, it); ++i) {
            const int blocks = it.blk1 - it.blk0;
            if (blocks == 0) { item_done(i); continue; }
            const bool big = it.mode == kKvBigItem;
            const int open = it.careful ? 0 : first_hidden(it) / kKvBlock - it.blk0;     // blocks of the item before this one need no mending
            uint32_t k_slot = 0, v_slot = 0;
            bool ok;
            if constexpr (FEW) if (it.mode == kKvFewItem) {
                const int t = it.tile;
                const uint32_t q0 = q_lo + (uint32_t)t * (kKvRegion >> 4), p0 = p_lo + (uint32_t)t * (kKvRegion >> 4);
                auto scores = [&](int n) -> bool {
                    if (!wait_k(k_slot)) return false;
                    const uint32_t a0 = k_lo_base + k_slot * (TILE >> 4);
                    uint32_t ad[D / 16], bd[D / 16];
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        ad[k] = a0 + (uint32_t)((k >> 2) * (HALF >> 4) + (k & 3) * 2);
                        bd[k] = q0 + (uint32_t)((k >> 2) * (HALF >> 4) + (k & 3) * 2);
                    }
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            ptx::umma_bf16_halves(tmem_base + 128u * (uint32_t)t + (uint32_t)(kKvFew * (n & 1)), ad[k], bd[k], desc_hi,
                                                  kIdescFewQK, k != 0 ? 1u : 0u);
                        ptx::umma_commit(s_full0 + 8 * (2 * t + (n & 1)));
                        ptx::umma_commit(kv_empty0 + 8 * k_slot);
                    }
                    __syncwarp();
                    return true;
                };
                // S(0), S(1), P V(0), S(2), P V(1), ... (one place in the code for each)
                ok = wait_q(t);
#pragma unroll 1
                for (int m = 0; m < blocks + 2 && ok; ++m) {
                  if (m >= 2) {
                    const int n = m - 2;
                    if (!wait_p(2 * t + (n & 1)) || !wait_v(v_slot, n >= open)) { ok = false; break; }
                    const uint32_t a0 = v_few_base + v_slot * (TILE >> 4), b0 = p0 + (uint32_t)(n & 1) * (P_BUF >> 4);
                    uint32_t ad[8], bd[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        ad[k] = a0 + (uint32_t)(k * 128);
                        bd[k] = b0 + (uint32_t)((k >> 2) * (P_HALF >> 4) + (k & 3) * 2);
                    }
                    if (leader) {
#pragma unroll
                        for (int k = 0; k < 16; ++k)                         // both terms
                            ptx::umma_bf16_halves(tmem_base + 256u + 128u * (uint32_t)t, ad[k & 7], bd[k & 7] + (k >= 8 ? P_TERM >> 4 : 0u), desc_hi,
                                                  kIdescFewPV, (LONG ? n % kKvFewSum != 0 : n != 0) || k != 0 ? 1u : 0u);
                        ptx::umma_commit(o_full0 + 8 * (2 * t + (n & 1)));
                        ptx::umma_commit(kv_empty0 + 8 * v_slot);
                        if (n == blocks - 1) ptx::umma_commit(q_empty0 + 8 * t);         // P lies in the region too
                    }
                    __syncwarp();
                  }
                  if (m < blocks) ok = scores(m);
                }
                if (!ok) break;
                item_done(i);
                continue;
            }
            // S_t = Q K^T with the block in k_slot; O_t += P_t V with that in v_slot: A = P_t from TMEM, 16 keys of a K step are 8 columns of
            // packed pairs, the second terms of small items 64 columns on
            auto scores = [&](int t, uint32_t q0, bool free_k) {
                const uint32_t b0 = k_lo_base + k_slot * (TILE >> 4);
                uint32_t ad[D / 16], bd[D / 16];
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    ad[k] = q0 + (uint32_t)((k >> 2) * (HALF >> 4) + (k & 3) * 2);
                    bd[k] = b0 + (uint32_t)((k >> 2) * (HALF >> 4) + (k & 3) * 2);
                }
                if (leader) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        ptx::umma_bf16_halves(tmem_base + 128u * (uint32_t)t, ad[k], bd[k], desc_hi, kIdescQK, k != 0 ? 1u : 0u);
                    ptx::umma_commit(s_full0 + 16 * t);
                    if (free_k) ptx::umma_commit(kv_empty0 + 8 * k_slot);
                }
                __syncwarp();
            };
            auto values = [&](int t, bool more, bool two, bool free_v) {
                const uint32_t v0 = v_lo_base + v_slot * (TILE >> 4);
                const uint32_t d_tmem = tmem_base + 256u + 128u * (uint32_t)t, p_tmem = tmem_base + 128u * (uint32_t)t;
                uint32_t bd[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) bd[k] = v0 + (uint32_t)(k * 128);
                if (leader) {
                    umma_bf16_tmem_a_halves(d_tmem, p_tmem, bd[0], desc_hi, kIdescPV, more ? 1u : 0u);
#pragma unroll
                    for (int k = 1; k < 8; ++k) umma_bf16_tmem_a_halves(d_tmem, p_tmem + 8u * (uint32_t)k, bd[k], desc_hi, kIdescPV, 1u);
                    if (two) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) umma_bf16_tmem_a_halves(d_tmem, p_tmem + 64u + 8u * (uint32_t)k, bd[k], desc_hi, kIdescPV, 1u);
                    }
                    ptx::umma_commit(o_full0 + 16 * t);
                    if (free_v) ptx::umma_commit(kv_empty0 + 8 * v_slot);
                }
                __syncwarp();
            };
            if (big) {
                // both tiles over each block: S_A(0), S_B(0), then P_A V(j), S_A(j + 1), P_B V(j), S_B(j + 1)
                ok = (LONG && (it.piece & kKvGoesOn)) || (wait_q(0) && wait_q(1));
#pragma unroll 1
                for (int j = -1; j < blocks && ok; ++j) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        if (j >= 0) {
                            if (!wait_p(2 * t) || (t == 0 && !wait_v(v_slot, j >= open))) { ok = false; break; }
                            values(t, j > 0, false, t == 1);
                        }
                        if (j + 1 < blocks) {
                            if (t == 0 && !wait_k(k_slot)) { ok = false; break; }
                            scores(t, q_lo + (uint32_t)t * (kKvRegion >> 4), t == 1);
                        }
                    }
                    if (j + 2 == blocks && !(LONG && (it.piece & kKvMore))) {        // Q has been used
                        if (leader) {
                            ptx::umma_commit(q_empty0);
                            ptx::umma_commit(q_empty0 + 8);
                        }
                        __syncwarp();
                    }
                }
            } else {
                // block n to tile n & 1: S(0), S(1), P V(0), S(2), P V(1), ...
                ok = (LONG && (it.piece & kKvGoesOn)) || wait_q(0);
#pragma unroll 1
                for (int m = 0; m < blocks + 2 && ok; ++m) {
                    const int t = m & 1;
                    if (m >= 2) {
                        if (!wait_p(2 * t) || !wait_v(v_slot, m - 2 >= open)) { ok = false; break; }
                        values(t, m >= 4, true, true);
                    }
                    if (m < blocks) {
                        if (!wait_k(k_slot)) { ok = false; break; }
                        scores(t, q_lo, true);
                        if (m == blocks - 1 && !(LONG && (it.piece & kKvMore))) {
                            if (leader) ptx::umma_commit(q_empty0);
                            __syncwarp();
                        }
                    }
                }
            }
            if (!ok) break;
            item_done(i);
        } while (next_pass(i));
        __syncwarp();
      } else if (warp == 2) {
        // ---------------- items and Q ----------------
        KvCut* cuts = reinterpret_cast<KvCut*>(a.workspace);
        KvCut cut = {};
        uint32_t i = 0, loads = 0, few_items = 0;                            // loads: bits, parity of [tile]'s
        bool ok = true, careful = false;
        const int b_first = s_start[0], tile_first = s_start[1];
        const int64_t x_first = lo - *s_rest;                                // where the first item starts
        least = __reduce_min_sync(0xFFFFFFFFu, s_range[lane % (kKvThreads / 32)].x);
        most = __reduce_max_sync(0xFFFFFFFFu, s_range[lane % (kKvThreads / 32)].y);
        do {
          if (lo < hi) {
            int head = head_lo, b = b_first, tile = tile_first, window = -1;
            // No more than stretch / least items, rounded up, start in one stretch: if they take little longer than it, none is cut.
            // (Worked out here: in every thread it cost the steady loops of long prompts 1 to 2 per cent.)
            const bool even = stretch < 0x40000000 && (int64_t)(((uint32_t)stretch + least - 1) / (uint32_t)least) * most <= stretch + kKvSnap;
            const int snap = even && most > kKvSnap ? most : kKvSnap;        // longest item that is not cut
            int w_row0 = 0, w_rows = 0, w_keys = 0;                          // this lane's request of the window
            int64_t x = x_first;
            while (ok && x < hi) {
                if (b >= a.B) { b = 0; ++head; tile = 0; continue; }
                if (window != b / 32) {
                    window = b / 32;
                    if (window * 32 + lane < a.B) kv_request(a, window * 32 + lane, w_row0, w_rows, w_keys, false);
                    else w_rows = 0;
                }
                const int rows = __shfl_sync(0xFFFFFFFFu, w_rows, b & 31), row0 = __shfl_sync(0xFFFFFFFFu, w_row0, b & 31);
                const int keys = __shfl_sync(0xFFFFFFFFu, w_keys, b & 31);
                const int pos0 = tile * 2 * a.tile_pos;
                if (pos0 >= rows) {                                          // on to the next request that has rows
                    const uint32_t some = __ballot_sync(0xFFFFFFFFu, w_rows > 0) & (0xFFFFFFFEu << (b & 31));
                    b = some ? window * 32 + __ffs((int)some) - 1 : window * 32 + 32;
                    tile = 0;
                    continue;
                }
                const int npos = min(2 * a.tile_pos, rows - pos0);
                const int seen_last = a.causal ? max(keys - rows + pos0 + npos, 0) : keys;
                const int mode = kv_mode(a, npos);
                const int64_t cost = kv_start(mode) + (int64_t)kv_key(mode) * seen_last;
                const int all = (seen_last + kKvBlock - 1) / kKvBlock;
                const int64_t from = max(lo - x, (int64_t)0);
                // a short item goes whole to the CTA in whose stretch it starts
                const bool short_item = cost <= snap;
                const int blk0 = short_item ? (from > 0 ? all : 0) : kv_blocks_before(from, mode, all);
                const int blk1 = short_item ? all : kv_blocks_before(min(hi - x, cost), mode, all);
                if (blk1 > blk0 || (all == 0 && from == 0)) {
                    const bool whole = blk0 == 0 && blk1 == all;
                    if (blk1 < all) {                                        // cut at the end of the stretch: whose are the parts
                        const int64_t block0 = x + kv_start(mode);
                        cut.first = (int)(block0 / stretch);
                        cut.parts = (int)((block0 + (int64_t)kKvBlock * kv_key(mode) * (all - 1)) / stretch) - cut.first + 1;
                        cut.head = head;
                        cut.npos = npos;
                        cut.row0 = row0 + pos0;
                        cut.two_tiles = npos > a.tile_pos;
                    }
                    const int tile_of = mode == kKvFewItem ? (int)(few_items & 1u) : 0;
                  for (int from_blk = blk0;;) {
                    const int to_blk = LONG && mode != kKvFewItem ? min(blk1, from_blk + kKvPiece) : blk1;
                    const uint32_t p = i % kKvRing;
                    // a free place; in the second pass all of them
                    for (uint32_t n = i; ok && n < i + (careful ? kKvRing : 1); ++n)
                        ok = kv_wait(item_empty0 + 8 * (n % kKvRing), ((n / kKvRing) & 1u) ^ 1u, abort_flag, 8);
                    if (!ok) break;
                    if (lane == 0) {
                        KvItem it;
                        it.blk0 = from_blk;
                        it.blk1 = to_blk;
                        it.b = b;
                        it.head = head;
                        it.row0 = row0 + pos0;
                        it.npos = npos;
                        it.keys = keys;
                        it.seen0 = a.causal ? keys - rows + pos0 + 1 : keys;
                        it.slot = whole ? -1 : 2 * (int)blockIdx.x + (blk0 == 0 ? 1 : 0);
                        it.last = 0;
                        it.mode = mode;
                        it.tile = tile_of;
                        it.careful = careful;
                        it.piece = (from_blk > blk0 ? kKvGoesOn : 0) | (to_blk < blk1 ? kKvMore : 0);
                        it.part0 = blk0;
                        items[p] = it;
                        hidden[p] = 0;
                        ptx::mbar_arrive(item_full0 + 8 * p);
                    }
                    __syncwarp();
                    ++i;
                    if (mode == kKvFewItem) ++few_items;
                    for (int t = tile_of; ok && blk1 > blk0 && from_blk == blk0 && t < (mode == kKvBigItem ? 2 : tile_of + 1); ++t) {
                        if (!kv_wait(q_empty0 + 8 * t, ((loads >> t) & 1u) ^ 1u, abort_flag, 9)) { ok = false; break; }
                        loads ^= 1u << t;
                        if (lane == 0) {
                            const bool few = mode == kKvFewItem;
                            const uint32_t full = q_full0 + 8 * t;
                            ptx::mbar_arrive_expect_tx(full, (uint32_t)(few ? a.q_few_bytes : a.q_bytes));
#pragma unroll
                            for (int h = 0; h < HALVES; ++h)
                                tma_load_3d(q_smem + t * kKvRegion + h * HALF, few ? &tmQfew : &tmQ, 64 * h, head * a.ratio,
                                            row0 + pos0 + (few ? 0 : t * a.tile_pos), full);
                        }
                        __syncwarp();
                    }
                    if (!ok || to_blk == blk1) break;
                    from_blk = to_blk;
                  }
                  if (!ok) break;
                }
                x += cost;
                ++tile;
            }
          }
          const uint32_t p = i % kKvRing;
          if (lane == 0) cuts[blockIdx.x] = cut;
          if (ok && kv_wait(item_empty0 + 8 * p, ((i / kKvRing) & 1u) ^ 1u, abort_flag, 10)) {
              if (lane == 0) {
                  items[p].last = 1;
                  items[p].careful = careful;
                  ptx::mbar_arrive(item_full0 + 8 * p);
              }
          }
          __syncwarp();
          careful = true;
        } while (next_pass(i));
        __syncwarp();
      } else {
        // ---------------- V mender ----------------
        KvCursor<SLOTS> at = {1, 0};
        uint32_t n_fixed = 0, i = 0;
        KvItem it;
        do for (; next_item(i, it); ++i) {
            bool pages = false;                                              // some outside of the cache
            if (it.blk1 > it.blk0) {
                const int32_t* table = a.table + (int64_t)it.b * a.width;
                const int p1 = (min(it.keys, it.blk1 * kKvBlock) - 1) / a.page_size;
#pragma unroll 4
                for (int p = it.blk0 * kKvBlock / a.page_size + lane; p <= p1; p += 32) pages |= (uint32_t)table[p] >= (uint32_t)a.n_pages;
                pages = __any_sync(0xFFFFFFFFu, pages);
            }
            if (lane == 0) {
                odd_pages[i % kKvRing] = pages;
                ptx::mbar_arrive(item_checked0 + 8 * (i % kKvRing));
            }
            const int first = first_hidden(it);
            const int from = it.careful ? it.blk0 : max(it.blk0, first / kKvBlock);
            float* of_all = seen_by_all(it.mode);
            if (__builtin_expect(it.careful && !(it.piece & kKvGoesOn), 0)) {
#pragma unroll 1
                for (int c = lane; c < D; c += 32) of_all[c] = 0.0f;
                __syncwarp();
            }
            at.skip(2u * (uint32_t)max(0, min(from, it.blk1) - it.blk0));
            bool ok = true, none = false, none_seen = false;
#pragma unroll 1
            for (int j = from; j < it.blk1; ++j) {
                // (the producer has filled the slot anew: before that, its barrier's parity could be that of an older use)
                if (!kv_wait(mend0 + 8 * (n_fixed % kKvMends), (n_fixed / kKvMends) & 1u, abort_flag, 18) ||
                    !kv_wait(kv_full0 + 8 * at.slot, at.phase, abort_flag, 11)) { ok = false; break; }
                const int r0 = max(0, first - j * kKvBlock), end = it.keys - j * kKvBlock;       // rows from r0 on; from `end` on none
                uint4* rows = reinterpret_cast<uint4*>(fifo_ptr + at.slot * TILE);               // [half][key][16 B]
                if (__builtin_expect(it.careful, 0)) {
#pragma unroll 1
                    for (int c = lane; c < HALVES * kKvBlock * 8; c += 32) {
                        const int key = (c >> 3) & (kKvBlock - 1);
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (key < end) {
                            v = rows[c];
                            if (bf16_pair_not_finite(v.x) || bf16_pair_not_finite(v.y) || bf16_pair_not_finite(v.z) || bf16_pair_not_finite(v.w)) {
                                volatile uint16_t* row = reinterpret_cast<volatile uint16_t*>(rows + c);
                                float* sum = of_all + (c >> 10) * 64 + ((c ^ key) & 7) * 8;      // (16 bytes of a row change places by its number)
#pragma unroll 1
                                for (int k = 0; k < 8; ++k) {
                                    const float x = __uint_as_float((uint32_t)row[k] << 16);
                                    if (is_finite(x)) continue;
                                    if (key < r0) {
                                        atomicAdd(sum + k, x);
                                        none_seen = true;
                                    } else {
                                        none = true;
                                    }
                                    row[k] = 0;
                                }
                                asm volatile("" ::: "memory");
                                v = rows[c];
                            }
                            v = make_uint4(bf16_pair_times(v.x, kKvCareful), bf16_pair_times(v.y, kKvCareful), bf16_pair_times(v.z, kKvCareful),
                                           bf16_pair_times(v.w, kKvCareful));
                        }
                        rows[c] = v;
                    }
                } else
#pragma unroll 1
                for (int c = r0 * 8 + lane; c < kKvBlock * 8; c += 32) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (c < end * 8) {
                            v = rows[h * 1024 + c];
                            if (!(bf16_pair_not_finite(v.x) || bf16_pair_not_finite(v.y) || bf16_pair_not_finite(v.z) ||
                                  bf16_pair_not_finite(v.w)))
                                continue;
                            none = true;
                            uint32_t* w = &v.x;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if ((w[k] & 0x7F80u) == 0x7F80u) w[k] &= 0xFFFF0000u;
                                if ((w[k] & 0x7F800000u) == 0x7F800000u) w[k] &= 0x0000FFFFu;
                            }
                        }
                        rows[h * 1024 + c] = v;
                    }
                }
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(fixed0 + 8 * (n_fixed % kKvMends));
                ++n_fixed;
                at.move(2);
            }
            if (!ok) break;
            none = __any_sync(0xFFFFFFFFu, none);
            none_seen = __any_sync(0xFFFFFFFFu, none_seen);
            if (lane == 0) {
                if (none || none_seen) hidden[i % kKvRing] = (none ? kKvHidden : 0u) | (none_seen ? kKvSeen : 0u);
                ptx::mbar_arrive(item_fixed0 + 8 * (i % kKvRing));
            }
            item_done(i);
        } while (next_pass(i));
        __syncwarp();
      }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kKvRegsSoftmax));
        // ---------------- softmax and epilogue: one group of four warps per tile, thread = row ----------------
        const int t = (warp - 4) >> 2;
        const int r = (warp & 3) * 32 + lane;                                // row within the tile = TMEM lane
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem_base + 128u * (uint32_t)t + lane_addr;
        const uint32_t o_addr = tmem_base + 256u + lane_addr;                // tile A's; tile B's 128 columns on
        const int my_pos = r / a.ratio;
        uint32_t s_phase = 0, o_phase = 0, joins = 0, agreed = 0;           // bits: [buffer]
        float m_use = -INFINITY, l_run = 0.0f;                               // exponent base, row sum
        float m_piece = 0.0f;                                                // the base of what waits in the workspace
        uint32_t odd = 0;                                                    // numbers that are none, taken out of V
        bool ok = true;

        // One step: as in gqa_attention.cuh.  `valid`: keys of the block that the row sees, `bits`: of the block's groups of 16 keys those whose
        // page exists; TWO: probabilities in two bf16 terms (small items).
        // (All exponentials take the special-function unit: with a quarter of them as a cubic, which pays in gqa_attention.cuh, a prompt of 8192
        // without a mask took 924 us instead of 880: here the step's length counts, not the unit.)
        auto step_pass = [&](auto two_tag, bool first, int valid, uint32_t bits, bool masked, bool mine) {
            constexpr bool TWO = decltype(two_tag)::value;
            constexpr int PART = TWO ? 8 : 32;                               // pairs stored at a time
            uint32_t v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32(s_addr + 32 * c, v[c]);
            ptx::tmem_ld_wait();
            if (masked) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (32 * c + i >= valid || !((bits >> (2 * c + i / 16)) & 1u)) v[c][i] = 0xFF800000u;    // -inf
            }
            // The base moves when a row's sum says that it is far too low, and from -infinity (no key so far, or only scores of
            // -infinity): the first keys after that may score far below 0.  A row goes by its own sum alone, so that what its neighbours
            // see (NaN, say) does not change its rounding.
            bool moved = first, again = first;
            float l_blk;
#pragma unroll 1
            for (;;) {
                if (again) {
                    float m_raw = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            m_raw = max3_f32(m_raw, __uint_as_float(v[c][2 * i]), __uint_as_float(v[c][2 * i + 1]));
                    const float m_new = moved ? fmaxf(m_use, m_raw * a.scale_log2) : m_use;      // the scale is positive
                    if (!first && __any_sync(0xFFFFFFFFu, mine && m_new != m_use)) {
                        // O of the steps so far is complete: this step's scores were issued after their matmuls
                        const float alpha = m_new == m_use ? 1.0f : ex2_approx(m_use - m_new);
                        l_run *= alpha;
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            float o[16];
                            uint32_t w[16];
                            tmem_ld_32x16(o_addr + 128u * (uint32_t)t + c, o);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * alpha);
                            tmem_st_32x16(o_addr + 128u * (uint32_t)t + c, w);
                        }
                    }
                    m_use = m_new;
                }
                const float b0 = m_use == -INFINITY ? 0.0f : m_use;
                const uint64_t scale2 = pack_f32x2(a.scale_log2, a.scale_log2), neg_base2 = pack_f32x2(-b0, -b0);
                uint64_t l_acc2 = pack_f32x2(0.0f, 0.0f);
#pragma unroll
                for (int c = 0; c < 64; c += PART) {                         // pairs of keys
                    float p[2 * PART];
                    uint32_t top[PART];
#pragma unroll
                    for (int i = 0; i < PART; ++i) {
                        float e0, e1;
                        const uint32_t* x = &v[(c + i) >> 4][2 * ((c + i) & 15)];
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), scale2, neg_base2), e0, e1);
                        p[2 * i] = ex2_approx(e0);
                        p[2 * i + 1] = ex2_approx(e1);
                        l_acc2 = add_f32x2(l_acc2, pack_f32x2(p[2 * i], p[2 * i + 1]));
                        top[i] = pack_bf16x2(p[2 * i], p[2 * i + 1]);
                    }
                    if constexpr (TWO) {
                        tmem_st_32x8(s_addr + c, top);
#pragma unroll
                        for (int i = 0; i < PART; ++i) top[i] = pack_bf16x2(p[2 * i] - bf16_lo(top[i]), p[2 * i + 1] - bf16_hi(top[i]));
                        tmem_st_32x8(s_addr + 64 + c, top);
                    } else {
                        tmem_st_32x32(s_addr + c, top);
                    }
                }
                float l0, l1;
                unpack_f32x2(l_acc2, l0, l1);
                l_blk = l0 + l1;
                if (again) break;
                moved = !(l_blk <= kGqaLazySum) || m_use == -INFINITY;
                again = __any_sync(0xFFFFFFFFu, mine && moved);
                if (!again) break;
            }
            l_run += l_blk;
            tmem_st_wait();
        };

        // A few item: lane = key in a block's scores, channel in its output; the four warps agree on the base of the exponentials.
        const int tile_no = t, row_no = r;
        auto few_item = [&](const KvItem& it, const int32_t* table, bool bad, uint32_t ring, uint32_t ring_phase) -> bool {
            // (nothing that follows from these is worked out ahead and kept in registers through the other items' loops)
            const int t = opaque(tile_no), r = opaque(row_no);
            const uint32_t s_addr = tmem_base + 128u * (uint32_t)t + ((uint32_t)(r & ~31) << 16), o_addr = s_addr + 256u;
            const int blocks = it.blk1 - it.blk0, rows = it.npos * a.ratio;
            // every row's part, row by row in registers, four rows at a time: those that the item does not have are not run
            auto each_row = [&](auto part) {
#pragma unroll
                for (int g = 0; g < kKvFew; g += 4) {
                    if (g < opaque(rows)) {
#pragma unroll
                        for (int n = g; n < g + 4; ++n) part(n);
                    }
                }
            };
            const int first = min(max(it.seen0, 0), it.keys);                // the first key that some row must not see
            float m[kKvFew], l[kKvFew];
            int seen[kKvFew];                                                // keys that row n sees
            {
                int pos = 0, next = a.ratio;
#pragma unroll
                for (int n = 0; n < kKvFew; ++n) {
                    if (n == next) { ++pos; next += a.ratio; }
                    m[n] = -INFINITY;
                    l[n] = 0.0f;
                    seen[n] = a.causal ? min(max(it.seen0 + pos, 0), it.keys) : it.keys;
                }
            }
            const uint32_t q4 = (uint32_t)r >> 5;
            float* maxima = exchange + t * 128;                              // [16][4]
            float* weights = maxima + 64;
            auto agree = [&]() -> bool {                                     // what the four warps wrote before it they read after it
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(agree0 + 8 * t);
                const bool ok = kv_wait(agree0 + 8 * t, agreed & 1u, abort_flag, 20);
                agreed ^= 1u;
                return ok;
            };
            // O's two sums added, into the columns from `to` on (once in many blocks: short code)
            auto add_sums = [&](bool both, uint32_t to) {
                ptx::tc_fence_after_sync();
#pragma unroll 1
                for (uint32_t n = 0; n < kKvFew; ++n) {
                    const float o = tmem_ld_32x1(o_addr + n);
                    float other = 0.0f;
                    if (both) other = tmem_ld_32x1(o_addr + kKvFew + n);
                    ptx::tmem_ld_wait();
                    tmem_st_32x1(o_addr + to + n, o + other);
                    tmem_st_wait();
                }
                ptx::tc_fence_before_sync();
            };
            const uint32_t p_at = q_smem + t * kKvRegion + P_AT + (uint32_t)(r >> 6) * P_HALF + (uint32_t)(r & 7) * 2u;
            const uint32_t chunk = (uint32_t)(r & 63) >> 3;
#pragma unroll 1
            for (int j = 0; j < blocks; ++j) {
                const uint32_t buf = (uint32_t)j & 1u;
                const int key = (it.blk0 + j) * kKvBlock + r;
                if (!kv_wait(s_full0 + 8 * (2 * t + buf), (s_phase >> buf) & 1u, abort_flag, 13)) return false;
                s_phase ^= 1u << buf;
                ptx::tc_fence_after_sync();
                float x[kKvFew];
                tmem_ld_32x16(s_addr + kKvFew * buf, x);
                ptx::tmem_ld_wait();
                ptx::tc_fence_before_sync();
                if (opaque(bad) || (it.blk0 + j + 1) * kKvBlock > first) {
                    const bool there = key < it.keys && (!bad || (uint32_t)table[key / a.page_size] < (uint32_t)a.n_pages);
                    each_row([&](int n) {
                        if (!there || key >= seen[n]) x[n] = -INFINITY;
                    });
                }
                if (LONG && opaque(j) % kKvFewSum == 0 && j > 0) {           // PV of this block begins a new sum
                    if (!kv_wait(o_full0 + 8 * (2 * t + (buf ^ 1u)), ((o_phase >> (buf ^ 1u)) & 1u) ^ 1u, abort_flag, 23)) return false;
                    add_sums(j > kKvFewSum, kKvFew);
                }
                // the base of a row moves when a score passes it by 8 (a factor of 256), and from -infinity
                const bool begins = opaque(j) == 0;
                bool moves = begins;
                if (!begins) {
                    bool over = false;
                    each_row([&](int n) {
                        if (n < rows) over |= fmaf(x[n], a.scale_log2, m[n] == -INFINITY ? INFINITY : -m[n]) > 8.0f;
                    });
                    over = __any_sync(0xFFFFFFFFu, over);
                    volatile uint32_t* v = votes + t * 8 + (agreed & 1u) * 4;
                    if (lane == 0) v[q4] = over;
                    if (!agree()) return false;
                    moves = (v[0] | v[1] | v[2] | v[3]) != 0;
                }
                if (moves) {
                    float mine = -INFINITY;
                    each_row([&](int n) {
                        const float top = redux_max_f32(x[n]);
                        if (lane == n) mine = top;
                    });
                    if (lane < kKvFew) maxima[lane * 4 + q4] = mine;
                    if (!agree()) return false;
                    float f[kKvFew];
                    bool any = false;
                    each_row([&](int n) {
                        const float4 w = *reinterpret_cast<const float4*>(maxima + 4 * n);
                        const float top = fmaxf(fmaxf(w.x, w.y), fmaxf(w.z, w.w)) * a.scale_log2;
                        const bool moved = top > m[n] + 8.0f || m[n] == -INFINITY;
                        f[n] = moved && top > m[n] ? ex2_approx(m[n] - top) : 1.0f;
                        any |= f[n] != 1.0f && n < rows;
                        if (moved) m[n] = fmaxf(m[n], top);
                        l[n] *= f[n];
                    });
                    if (any && !begins) {                                      // the same for all four warps
                        if (!kv_wait(o_full0 + 8 * (2 * t + (buf ^ 1u)), ((o_phase >> (buf ^ 1u)) & 1u) ^ 1u, abort_flag, 21)) return false;
                        ptx::tc_fence_after_sync();
                        uint32_t c = 0;
                        for (;;) {                                           // the sum that PV adds to, and the other one if there is one
                            float o[kKvFew];
                            tmem_ld_32x16(o_addr + c, o);
                            ptx::tmem_ld_wait();
                            uint32_t ow[kKvFew];
                            each_row([&](int n) { ow[n] = __float_as_uint(o[n] * f[n]); });
                            tmem_st_32x16(o_addr + c, ow);
                            tmem_st_wait();
                            if (!LONG || opaque(j) < kKvFewSum || c != 0) break;
                            c = kKvFew;
                        }
                        ptx::tc_fence_before_sync();
                    }
                }
                // P of two steps ago has been read
                if (j >= 2 && !kv_wait(o_full0 + 8 * (2 * t + buf), ((o_phase >> buf) & 1u) ^ 1u, abort_flag, 22)) return false;
                o_phase ^= 1u << buf;                                        // parity of this buffer's next use
                const uint32_t to = p_at + buf * P_BUF;
                each_row([&](int n) {
                    const float p = ex2_approx(fmaf(x[n], a.scale_log2, m[n] == -INFINITY ? 0.0f : -m[n]));
                    l[n] += p;
                    const bf16 top = __float2bfloat16_rn(p);
                    const bf16 low = __float2bfloat16_rn(p - __bfloat162float(top));
                    const uint32_t place = to + (uint32_t)n * 128u + ((chunk ^ (uint32_t)(n & 7)) << 4);
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(place), "h"(__bfloat16_as_ushort(top)) : "memory");
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(place + P_TERM), "h"(__bfloat16_as_ushort(low)) : "memory");
                });
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full0 + 8 * (2 * t + buf));
            }
            uint32_t odd = 0;
            if (blocks > 0) {
                // the rows' weights, summed over the warp's keys: at each exchange a lane keeps half of its rows, in the end row lane / 2
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) {
                    const bool up = lane & (2 * w);
#pragma unroll
                    for (int n = 0; n < w; ++n) {
                        const float keep = up ? l[n + w] : l[n], give = up ? l[n] : l[n + w];
                        l[n] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, 2 * w);
                    }
                }
                l[0] += __shfl_xor_sync(0xFFFFFFFFu, l[0], 1);
                if ((lane & 1) == 0) weights[(lane >> 1) * 4 + q4] = l[0];
                if (!agree()) return false;
                const uint32_t buf = (uint32_t)(blocks - 1) & 1u;
                if (!kv_wait(o_full0 + 8 * (2 * t + buf), ((o_phase >> buf) & 1u) ^ 1u, abort_flag, 14)) return false;
                ptx::tc_fence_after_sync();
                if (LONG && opaque(blocks) > kKvFewSum) add_sums(true, 0);
                if (!kv_wait(item_fixed0 + 8 * ring, ring_phase, abort_flag, 15)) return false;
                odd = hidden[ring];
            }
            const bool whole = it.slot < 0;
            const int64_t part = (int64_t)it.slot * a.slot_rows;
            float* sums = reinterpret_cast<float*>(a.workspace + kv_ws_sums(gridDim.x, a.slot_rows)) + part * D + r;
            bf16* out = a.O + ((int64_t)it.row0 * a.Hq + (int64_t)it.head * a.ratio) * D + r;
            if (!whole && q4 == 0 && lane < kKvFew) {
                float base_n = m[0];
#pragma unroll
                for (int n = 1; n < kKvFew; ++n)
                    if (lane == n) base_n = m[n];
                const float4 w = *reinterpret_cast<const float4*>(weights + 4 * lane);
                if (lane < rows)
                    (reinterpret_cast<float2*>(a.workspace + kv_ws_stats(gridDim.x)) + part)[lane] = make_float2(base_n, (w.x + w.y) + (w.z + w.w));
            }
            const bool careful = it.careful != 0;
            const float of_all = odd & kKvSeen ? seen_by_all(kKvFewItem)[r] : 0.0f;
            bool not_finite = false;
            int pos = 0, head = 0;
#pragma unroll 1
            for (int n = 0; n < rows; ++n) {
                const float o = blocks > 0 ? tmem_ld_32x1(o_addr + (uint32_t)n) : 0.0f;
                const float4 w = *reinterpret_cast<const float4*>(weights + 4 * n);
                const float sum = blocks > 0 ? (w.x + w.y) + (w.z + w.w) : 0.0f;             // 0: nothing was seen
                ptx::tmem_ld_wait();
                not_finite |= !is_finite(o) && is_finite(sum) && sum != 0.0f;
                float value = sum == 0.0f ? 0.0f : __fdividef(o, sum);
                if (__builtin_expect(careful, 0)) value = value * (1.0f / kKvCareful) + of_all;
                if ((odd & kKvHidden) && r < D) {
                    const int end = min(a.causal ? min(max(it.seen0 + pos, 0), it.keys) : it.keys, it.blk1 * kKvBlock);
#pragma unroll 1
                    for (int j = max(first, it.blk0 * kKvBlock); j < end; ++j) {
                        const int page = table[j / a.page_size];
                        if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
                        const float v = __bfloat162float(a.v[(((int64_t)page * a.Hkv + it.head) * a.page_size + j % a.page_size) * D + r]);
                        if (!is_finite(v)) value += v;
                    }
                    __syncwarp();
                }
                if (r < D) {
                    // (in the second pass only what was not finite)
                    if (whole) {
                        if (!careful || !is_finite(__bfloat162float(*out))) *out = __float2bfloat16_rn(sum == 0.0f ? 0.0f : value);
                    } else {
                        if (!careful || !is_finite(*sums)) *sums = value;
                    }
                }
                out += D;
                sums += D;
                if (++head == a.ratio) {
                    head = 0;
                    ++pos;
                    out += (int64_t)(a.Hq - a.ratio) * D;
                }
            }
            if (not_finite && r < D && !careful) *redo = 1;
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(item_empty0 + 8 * ring);
            return true;
        };

        uint32_t i = 0;
        do for (;; ++i) {
            const uint32_t ring = i % kKvRing, ring_phase = (i / kKvRing) & 1u;
            if (!kv_wait(item_full0 + 8 * ring, ring_phase, abort_flag, 12)) break;
            const KvItem& it = items[ring];                                  // stays until this warp lets it go
            if (it.last) break;
            const int blocks = it.blk1 - it.blk0;
            const bool big = it.mode == kKvBigItem;
            const int32_t* table = a.table + (int64_t)it.b * a.width;
            bool bad = false;                                                // pages that the cache does not have
            if (FEW && it.mode == kKvFewItem && it.tile != t) {
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(item_empty0 + 8 * ring);
                continue;
            }
            if (blocks > 0) {
                if (!kv_wait(item_checked0 + 8 * ring, ring_phase, abort_flag, 19)) break;
                bad = odd_pages[ring] != 0;
            }
            if constexpr (FEW) {
                if (it.mode == kKvFewItem) {
                    if (!few_item(it, table, bad, ring, ring_phase)) break;
                    continue;
                }
            }
            const int pos = my_pos + (big ? t * a.tile_pos : 0);
            const bool mine = my_pos < a.tile_pos && pos < it.npos;          // this thread's row exists
            const bool active = __any_sync(0xFFFFFFFFu, mine);
            const int seen = mine ? min(max(a.causal ? it.seen0 + pos : it.keys, 0), it.keys) : 0;
            const int n_steps = big ? blocks : (blocks + 1 - t) / 2;         // of this tile
            const int piece = LONG ? it.piece : 0;
            if (!(piece & kKvGoesOn)) {
                m_use = -INFINITY;
                l_run = 0.0f;
                odd = 0;
            }
            const int n_first = piece & kKvGoesOn ? -1 : 0;                  // the step that sets the base: not in a later piece
            // the steps of this tile's blocks, `stride` of them apart
            auto steps = [&](auto two_tag, int key0, int stride) {
#pragma unroll 1
                for (int n = 0; n < n_steps; ++n, key0 += stride) {
                    const int valid = max(0, min(kKvBlock, seen - key0));
                    uint32_t bits = 0xFFu;
                    if (opaque(bad)) {
                        const int key = key0 + 16 * lane;
                        bool there = true;
                        if (lane < 8 && key < it.keys) there = (uint32_t)table[key / a.page_size] < (uint32_t)a.n_pages;
                        bits = __ballot_sync(0xFFFFFFFFu, there) & 0xFFu;
                    }
                    const bool masked = __any_sync(0xFFFFFFFFu, mine && valid < kKvBlock) || bits != 0xFFu;
                    // the scores are complete, and with them every matmul issued before them
                    if (!kv_wait(s_full0 + 16 * t, s_phase & 1u, abort_flag, 13)) return false;
                    s_phase ^= 1u;
                    ptx::tc_fence_after_sync();
                    if (opaque(active)) step_pass(two_tag, opaque(n) == n_first, valid, bits, opaque(masked), mine);
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(p_full0 + 16 * t);
                }
                return true;
            };
            ok = big ? steps(std::false_type{}, it.blk0 * kKvBlock, kKvBlock) : steps(std::true_type{}, (it.blk0 + t) * kKvBlock, 2 * kKvBlock);
            if (!ok) break;
            o_phase ^= (uint32_t)n_steps & 1u;                               // parity of the next use: one phase per step
            if (n_steps > 0) {
                if (!kv_wait(o_full0 + 16 * t, (o_phase & 1u) ^ 1u, abort_flag, 14)) { ok = false; break; }
                ptx::tc_fence_after_sync();
            }
            if (blocks > 0) {
                if (!kv_wait(item_fixed0 + 8 * ring, ring_phase, abort_flag, 15)) { ok = false; break; }
                odd |= hidden[ring];
            }
            if (LONG && opaque(piece) != 0) {
                // the sum so far: into the workspace, from the last piece into tensor memory, where the rest expects it
                const int t = opaque(tile_no), r = opaque(row_no);
                const uint32_t o_addr = tmem_base + 256u + 128u * (uint32_t)t + ((uint32_t)(r & ~31) << 16);
                float* waits = reinterpret_cast<float*>(a.workspace + kv_ws_pieces(gridDim.x, a.slot_rows, D)) +
                               ((int64_t)(2 * (int)blockIdx.x + t) * kv_tile_rows(a.slot_rows) + r) * D;
                const float f = ex2_approx(m_piece - (m_use == -INFINITY ? 0.0f : m_use));
                if (active) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 4) {
                        float o[4];
                        float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[k] = opaque(n_steps) > 0 ? tmem_ld_32x1(o_addr + (uint32_t)(c + k)) : 0.0f;
                        if (mine && (piece & kKvGoesOn)) w = *reinterpret_cast<const float4*>(waits + c);
                        ptx::tmem_ld_wait();
                        if (piece & kKvGoesOn) {
                            o[0] += w.x * f;
                            o[1] += w.y * f;
                            o[2] += w.z * f;
                            o[3] += w.w * f;
                        }
                        __syncwarp();
                        if (piece & kKvMore) {
                            if (mine) *reinterpret_cast<float4*>(waits + c) = make_float4(o[0], o[1], o[2], o[3]);
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k) tmem_st_32x1(o_addr + (uint32_t)(c + k), o[k]);
                            tmem_st_wait();
                        }
                        __syncwarp();
                    }
                }
                m_piece = m_use;
                if (piece & kKvMore) {
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(item_empty0 + 8 * ring);
                    continue;
                }
            }

            // Small items of several blocks: both tiles hold sums of the same rows.  Tile B's warps hand base and weight over, tile A's (which may
            // read the same lanes of tile B's columns) do the rest.
            const bool both = !big && (blocks > 1 || (piece & kKvGoesOn));
            float f_mine = 1.0f, f_other = 0.0f;
            if (both) {
                if (t == 1) {
                    stats[r] = make_float2(m_use, l_run);
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(stats_full);
                    if (!kv_wait(stats_done, joins & 1u, abort_flag, 16)) { ok = false; break; }
                } else {
                    if (!kv_wait(stats_full, joins & 1u, abort_flag, 17)) { ok = false; break; }
                    ptx::tc_fence_after_sync();
                    const float2 other = stats[r];
                    const float m_both = fmaxf(m_use, other.x), b0 = m_both == -INFINITY ? 0.0f : m_both;
                    f_mine = ex2_approx(m_use - b0);
                    f_other = ex2_approx(other.x - b0);
                    l_run = l_run * f_mine + other.y * f_other;
                    m_use = m_both;
                }
                ++joins;
            }
            if (active && (big || t == 0)) {
                const int t = opaque(tile_no), r = opaque(row_no);           // (as in few_item)
                const int my_head = r % a.ratio;
                const uint32_t o_addr = tmem_base + 256u + ((uint32_t)(r & ~31) << 16);
                const int row_in_slot = (big ? 128 * t : 0) + r;
                const int64_t part = (int64_t)it.slot * a.slot_rows + row_in_slot;
                float* sums = reinterpret_cast<float*>(a.workspace + kv_ws_sums(gridDim.x, a.slot_rows)) + part * D;
                bf16* out = a.O + ((int64_t)(it.row0 + pos) * a.Hq + (int64_t)it.head * a.ratio + my_head) * D;
                const bool zero = l_run == 0.0f;                             // nothing was seen
                const float inv_l = 1.0f / l_run;
                if (it.slot >= 0 && mine) reinterpret_cast<float2*>(a.workspace + kv_ws_stats(gridDim.x))[part] = make_float2(m_use, l_run);
                if (__builtin_expect(opaque(it.careful), 0)) {
                    // what was not finite in the first pass; few calls come here: short code, a channel at a time
                    const float* of_all = seen_by_all(kKvBigItem);
#pragma unroll 1
                    for (int c = 0; c < D; ++c) {
                        float o = 0.0f, o1 = 0.0f;
                        if (opaque(n_steps) > 0) o = tmem_ld_32x1(o_addr + 128u * (uint32_t)t + c);
                        if (opaque(both)) o1 = tmem_ld_32x1(o_addr + 128u + c);
                        ptx::tmem_ld_wait();
                        if (both) o = o * f_mine + o1 * f_other;
                        float value = zero ? 0.0f : o * inv_l * (1.0f / kKvCareful);
                        if ((odd & kKvSeen) && !(zero && it.slot < 0)) value += of_all[c];
                        if (mine) {
                            if (it.slot < 0) {
                                if (!is_finite(__bfloat162float(out[c]))) out[c] = __float2bfloat16_rn(value);
                            } else if (!is_finite(sums[c])) {
                                sums[c] = value;
                            }
                        }
                        __syncwarp();
                    }
                } else {
                    uint64_t test = pack_f32x2(0.0f, 0.0f);                  // NaN once some O is not finite
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float o[16];
                        if (opaque(n_steps) > 0) tmem_ld_32x16(o_addr + 128u * (uint32_t)t + c, o);
                        if (opaque(both)) {
                            float o1[16];
                            tmem_ld_32x16(o_addr + 128u + c, o1);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = o[k] * f_mine + o1[k] * f_other;
                        } else {
                            ptx::tmem_ld_wait();
                        }
                        if (mine) {
#pragma unroll
                            for (int k = 0; k < 16; k += 2) test = fma_f32x2(pack_f32x2(o[k], o[k + 1]), pack_f32x2(0.0f, 0.0f), test);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = zero ? 0.0f : o[k] * inv_l;
                            if (opaque(it.slot) < 0) {
#pragma unroll
                                for (int w = 0; w < 2; ++w) {
                                    uint32_t pk[4];
#pragma unroll
                                    for (int k = 0; k < 4; ++k) pk[k] = pack_bf16x2(o[8 * w + 2 * k], o[8 * w + 2 * k + 1]);
                                    *reinterpret_cast<uint4*>(out + c + 8 * w) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                                }
                            } else {
#pragma unroll
                                for (int w = 0; w < 4; ++w)
                                    *reinterpret_cast<float4*>(sums + c + 4 * w) = make_float4(o[4 * w], o[4 * w + 1], o[4 * w + 2], o[4 * w + 3]);
                            }
                        }
                        __syncwarp();                                        // the next loads from TMEM are the whole warp's
                    }
                    float t0, t1;
                    unpack_f32x2(test, t0, t1);
                    if (mine && !is_finite(t0 + t1) && is_finite(l_run) && !zero) *redo = 1;
                }
                // the row that was just written gets what V held in place of numbers (not a row of zeros: the join tells for a cut item's)
                if ((odd & kKvHidden) && mine && !(zero && it.slot < 0)) {
#pragma unroll 1
                    for (int j = max(min(max(it.seen0, 0), it.keys), it.part0 * kKvBlock); j < min(seen, it.blk1 * kKvBlock); ++j) {
                        const int page = table[j / a.page_size];
                        if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
                        const bf16* vr = a.v + (((int64_t)page * a.Hkv + it.head) * a.page_size + j % a.page_size) * D;
#pragma unroll 1
                        for (int k = 0; k < D; ++k) {
                            const float x = __bfloat162float(vr[k]);
                            if (x - x == 0.0f) continue;
                            if (it.slot < 0) out[k] = __float2bfloat16_rn(__bfloat162float(out[k]) + x);
                            else sums[k] += x;
                        }
                    }
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (both && t == 0) ptx::mbar_arrive(stats_done);
                ptx::mbar_arrive(item_empty0 + 8 * ring);
            }
        } while (next_pass(i));
    }

    if (*abort_flag) {
        if (lane == 0) report_timeout(kKvKernelId, *abort_flag);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    if (warp == 1) ptx::tmem_dealloc(tmem_base, 512);
}

// The parts of cut items, added in order.  An item's rows are shared out to the CTAs (c, y) of all c whose stretch ends in it: one c for a
// prompt's item of two parts, nearly all where one long conversation is cut into as many parts as SMs.  A CTA takes a row at a time (its warps
// every eighth part each), or eight (a warp each), or 32 (eight lanes each), by how many it has.
constexpr int kKvJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kKvJoinThreads, 4)                       // (four per SM: all start at once)
kv_join_kernel(const KvAttnArgs a)
{
    constexpr int WARPS = kKvJoinThreads / 32;
    __shared__ float s_sum[WARPS][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    ptx::launch_dependents();
    ptx::grid_dependency_wait();
    const KvCut cut = reinterpret_cast<const KvCut*>(a.workspace)[blockIdx.x];
    if (cut.parts < 2) return;
    const float2* stats = reinterpret_cast<const float2*>(a.workspace + kv_ws_stats(gridDim.x));
    const float* sums = reinterpret_cast<const float*>(a.workspace + kv_ws_sums(gridDim.x, a.slot_rows));
    const int rows = cut.npos * a.ratio, shares = (cut.parts - 1) * gridDim.y, share = (blockIdx.x - cut.first) * gridDim.y + blockIdx.y;
    const int parts = cut.parts, mine = (rows - share + shares - 1) / shares;        // rows share, share + shares, ...
    int in_slot;                                                     // a row's place in each part, and where it goes
    bf16* out;
    auto find = [&](int i) {
        const int row = share + i * shares, pos = row / a.ratio, head = row - pos * a.ratio;
        const int t = cut.two_tiles && pos >= a.tile_pos ? 1 : 0;
        in_slot = 128 * t + (pos - t * a.tile_pos) * a.ratio + head;
        out = a.O + ((int64_t)(cut.row0 + pos) * a.Hq + (int64_t)cut.head * a.ratio + head) * D;
    };
    auto part = [&](int p) { return (int64_t)(p == 0 ? 2 * cut.first + 1 : 2 * (cut.first + p)) * a.slot_rows + in_slot; };
    // Part p's share of the row's weight, given the row's base and the inverse of its weight.
    auto share_of = [&](int p, float base, float inv) {
        const float2 s = stats[part(p)];
        return s.y * ex2_approx(s.x - base) * inv;
    };
    // LANES lanes work out a row's base and weight together
    auto base_of = [&](auto lanes_tag, int sub, float& base, float& weight) {
        constexpr int LANES = decltype(lanes_tag)::value;
        constexpr int AT_ONCE = 6;                                   // loads in flight: one round for a part per SM and 32 lanes
        float top = -INFINITY;                                       // of this lane's parts
        weight = 0.0f;
#pragma unroll 1
        for (int p0 = sub; p0 < parts; p0 += AT_ONCE * LANES) {
            float2 s[AT_ONCE];
            const float before = top;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) s[k] = p0 + k * LANES < parts ? stats[part(p0 + k * LANES)] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) top = fmaxf(top, s[k].x);
            const float b0 = top == -INFINITY ? 0.0f : top;
            weight *= ex2_approx(before - b0);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) weight += s[k].y * ex2_approx(s[k].x - b0);
        }
        const float own = top;
#pragma unroll
        for (int w = LANES / 2; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, w));
        base = top == -INFINITY ? 0.0f : top;
        weight *= ex2_approx(own - base);
#pragma unroll
        for (int w = LANES / 2; w > 0; w >>= 1) weight += __shfl_xor_sync(0xFFFFFFFFu, weight, w);
    };
    // Channel `at` of the row where the sum of its parts is no number: one that is none counts however small its part's share, and a weight
    // that is no number is the answer.
    auto with_care = [&](int at, float base, float weight) {
        float o = weight - weight;
#pragma unroll 1
        for (int p = 0; p < parts; ++p) {
            const float v = sums[part(p) * D + at], x = v * share_of(p, base, 1.0f / weight);
            o += x == x ? x : v;
        }
        return o;
    };
    if (mine > 1) {
        // eight lanes to a row, four channels at a time: sub, sub + 8, ...
        constexpr int LANES = 8, ROWS = 32 / LANES, N = D / LANES / 4;
        const int sub = lane % LANES;
#pragma unroll 1
        for (int i0 = warp * ROWS; i0 < mine; i0 += WARPS * ROWS) {
            const int i = i0 + lane / LANES;
            find(min(i, mine - 1));
            float base, weight;
            base_of(std::integral_constant<int, LANES>{}, sub, base, weight);
            const float inv = 1.0f / weight;
            float o[N][4] = {};
#pragma unroll 4
            for (int p = 0; p < parts; ++p) {
                const float4* x = reinterpret_cast<const float4*>(sums + part(p) * D) + sub;
                float4 v[N];
#pragma unroll
                for (int c = 0; c < N; ++c) v[c] = x[c * LANES];
                const float w = share_of(p, base, inv);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    o[c][0] += v[c].x * w;
                    o[c][1] += v[c].y * w;
                    o[c][2] += v[c].z * w;
                    o[c][3] += v[c].w * w;
                }
            }
            if (i < mine) {
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    uint2* to = reinterpret_cast<uint2*>(out) + sub + c * LANES;
                    if (weight == 0.0f) *to = make_uint2(0, 0);
                    else *to = make_uint2(pack_bf16x2(o[c][0], o[c][1]), pack_bf16x2(o[c][2], o[c][3]));
                }
                float test = 0.0f;
#pragma unroll
                for (int c = 0; c < N; ++c) test += (o[c][0] + o[c][1]) * 0.0f + (o[c][2] + o[c][3]) * 0.0f;
                if (__builtin_expect(!(test == 0.0f) && weight != 0.0f, 0)) {
#pragma unroll 1
                    for (int k = 0; k < 4 * N; ++k) {                // of this lane's channels those that are not finite; the others stay
                        const int c = (k / 4 * LANES + sub) * 4 + k % 4;
                        if (!is_finite(__bfloat162float(out[c]))) out[c] = __float2bfloat16_rn(with_care(c, base, weight));
                    }
                }
            }
            __syncwarp();
        }
        return;
    }
    if (mine < 1) return;
    constexpr int C = D / 32;
    find(0);
    float base, weight;
    base_of(std::integral_constant<int, 32>{}, lane, base, weight);
    const float inv = 1.0f / weight;
    float o[C] = {};
#pragma unroll 8
    for (int p = warp; p < parts; p += WARPS) {
        const float w = share_of(p, base, inv);
        const float* x = sums + part(p) * D + lane * C;
        float v[C];
        if constexpr (C == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(x);
        else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(x);
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] += v[c] * w;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) s_sum[warp][lane * C + c] = o[c];
    __syncthreads();
    if (tid < D) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) sum += s_sum[w][tid];
        if (__builtin_expect(!(sum == sum) && weight != 0.0f, 0)) sum = with_care(tid, base, weight);
        out[tid] = __float2bfloat16_rn(weight == 0.0f ? 0.0f : sum);
    }
}

}  // namespace gmlp
