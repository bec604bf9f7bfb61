// Host side of the 4-bit cache operators.  Included by api.cu inside its namespace.

int check_kv4_cache(const gmlp_kv4_cache& c) {
    if (c.reserved != 0) return GMLP_ERR_FLAGS;
    if (c.head_dim != 64 && c.head_dim != 128) return GMLP_ERR_UNSUPPORTED;
    if ((c.group != 32 && c.group != 64 && c.group != 128) || c.group > c.head_dim) return GMLP_ERR_SHAPE;
    if (c.n_pages <= 0 || c.n_kv_heads <= 0 || c.n_kv_heads > 4096 || c.page_size < 16 || c.page_size > 65536 || c.page_size % 16 != 0 ||
        c.n_pages > INT32_MAX / c.page_size)
        return GMLP_ERR_SHAPE;
    if (!c.k_codes || !c.k_params || !c.v_codes || !c.v_params) return GMLP_ERR_NULL;
    if (!aligned16(c.k_codes) || !aligned16(c.k_params) || !aligned16(c.v_codes) || !aligned16(c.v_params)) return GMLP_ERR_ALIGN;
    return GMLP_OK;
}
inline gmlp::Kv4Cache kv4_cache(const gmlp_kv4_cache& c) {
    return {{static_cast<uint8_t*>(c.k_codes), static_cast<uint8_t*>(c.v_codes)},
            {static_cast<uint32_t*>(c.k_params), static_cast<uint32_t*>(c.v_params)},
            (int)c.n_pages, c.n_kv_heads, c.page_size, c.head_dim, c.group};
}
// f<D, G>() of the cache's head dimension and group.
#define GMLP_KV4_DISPATCH(c, call)                                    \
    ((c).head_dim == 64 ? ((c).group == 32 ? call(64, 32) : call(64, 64)) \
                        : ((c).group == 32 ? call(128, 32) : ((c).group == 64 ? call(128, 64) : call(128, 128))))

int kv4_rows_impl(const gmlp_kv4_rows_args* a, bool append) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_kv4_rows_args) || (a->flags & ~(uint32_t)GMLP_FLAG_CHECKED)) return GMLP_ERR_FLAGS;
    int rc = check_kv4_cache(a->cache);
    if (rc != GMLP_OK) return rc;
    if (a->T < 0 || a->T > (1 << 24)) return GMLP_ERR_SHAPE;
    if (a->T == 0) return GMLP_OK;
    if (!a->K || !a->V || !a->slots) return GMLP_ERR_NULL;
    if (!aligned16(a->K) || !aligned16(a->V) || (reinterpret_cast<uintptr_t>(a->slots) & 7u)) return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    const gmlp::Kv4Cache c = kv4_cache(a->cache);
    const int64_t items = a->T * 2 * c.n_kv_heads, total = (int64_t)c.n_pages * c.page_size, per = append ? 8 : 64;
    if ((items + per - 1) / per > INT32_MAX) return GMLP_ERR_SHAPE;
    const dim3 grid((unsigned)((items + per - 1) / per));
    bf16 *K = static_cast<bf16*>(a->K), *V = static_cast<bf16*>(a->V);
    const int64_t* slots = static_cast<const int64_t*>(a->slots);
    prof_begin(st);
#define GMLP_KV4_APPEND(D, G) launch_chained(gmlp::kv4_append_kernel<D, G>, grid, 256, 0, 1, st, K, V, c, slots, items, total)
#define GMLP_KV4_GATHER(D, G) launch_chained(gmlp::kv4_gather_kernel<D, G>, grid, 256, 0, 1, st, c, slots, K, V, items, total)
    rc = append ? GMLP_KV4_DISPATCH(c, GMLP_KV4_APPEND) : GMLP_KV4_DISPATCH(c, GMLP_KV4_GATHER);
    if (rc != GMLP_OK) return rc;
    prof_mark(append ? "kv4_append" : "kv4_gather", st);
    return finish_checked(dev, a->flags, st);
}

struct Kv4Plan {
    int nt, col_tiles, splits;
    uint64_t workspace;
};
// How the keys of a request are split over CTAs.  The host knows the width of the page table, not the lengths: the kernel
// divides each request's own length by `splits`.  They are enough to fill the GPU and, for requests much longer than the others, one per
// 2048 keys that the table has room for, as far as the partial results of all of them fit kKv4PartialBytes.
constexpr uint64_t kKv4PartialBytes = (uint64_t)256 << 20;
Kv4Plan kv4_plan(int64_t B, int T, int ratio, int n_kv_heads, int head_dim, int64_t most_keys, int sms) {
    Kv4Plan p{};
    const int64_t cols = (int64_t)T * ratio;
    p.nt = cols <= 8 ? 1 : 2;
    p.col_tiles = (int)((cols + 8 * p.nt - 1) / (8 * p.nt));
    const int64_t ctas = B * n_kv_heads * p.col_tiles;
    const int64_t target = (int64_t)sms * 4, long_keys = 2048;
    int64_t splits = (target + ctas - 1) / ctas;
    int64_t by_length = (most_keys + long_keys - 1) / long_keys;
    const int64_t most = (most_keys + 127) / 128, split_bytes = ctas * 8 * p.nt * (head_dim + 4) * 4;
    if (by_length > (int64_t)kKv4PartialBytes / split_bytes) by_length = (int64_t)kKv4PartialBytes / split_bytes;
    if (splits < by_length) splits = by_length;
    if (splits > most) splits = most;
    if (splits > gmlp::kKv4MaxSplits) splits = gmlp::kKv4MaxSplits;
    if (splits < 1) splits = 1;
    p.splits = (int)splits;
    p.workspace = splits > 1 ? (uint64_t)(split_bytes * splits) : 0;
    return p;
}

constexpr int64_t kKv4MostKeys = (int64_t)1 << 30;       // of one request: positions stay well inside 31 bits
int check_kv4_attention(int64_t B, int T, int Hq, int Hkv, int64_t width, int page_size) {
    if (B < 0 || B > 65535 || T < 1 || T > GMLP_KV4_MAX_QUERIES || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Hq > 65535 || width < 1 ||
        width > kKv4MostKeys / page_size || B * T * Hq > INT32_MAX)
        return GMLP_ERR_SHAPE;
    return GMLP_OK;
}

int kv4_attention_impl(const gmlp_kv4_attention_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_kv4_attention_args) || (a->flags & ~(uint32_t)GMLP_FLAG_CHECKED) || a->reserved != 0)
        return GMLP_ERR_FLAGS;
    int rc = check_kv4_cache(a->cache);
    if (rc != GMLP_OK) return rc;
    rc = check_kv4_attention(a->B, a->q_len, a->n_q_heads, a->cache.n_kv_heads, a->table_width, a->cache.page_size);
    if (rc != GMLP_OK) return rc;
    const float scale_log2 = a->scale * 1.4426950408889634f;                 // exponentials are powers of two
    if (!(scale_log2 - scale_log2 == 0.0f)) return GMLP_ERR_FLAGS;
    if (a->B == 0) return GMLP_OK;
    if (!a->Q || !a->O || !a->block_table || !a->lengths) return GMLP_ERR_NULL;
    if (!aligned16(a->Q) || !aligned16(a->O) || (reinterpret_cast<uintptr_t>(a->block_table) & 3u) ||
        (reinterpret_cast<uintptr_t>(a->lengths) & 3u) || (reinterpret_cast<uintptr_t>(a->workspace) & 255u))
        return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    const int ratio = a->n_q_heads / a->cache.n_kv_heads;
    const Kv4Plan plan = kv4_plan(a->B, a->q_len, ratio, a->cache.n_kv_heads, a->cache.head_dim, a->table_width * a->cache.page_size, dev->sm_count);
    if (plan.workspace > 0) {
        if (a->workspace == nullptr) return GMLP_ERR_NULL;
        if (a->workspace_bytes < plan.workspace) return GMLP_ERR_WORKSPACE;
        claim_workspace(dev, static_cast<const uint8_t*>(a->workspace), plan.workspace, nullptr, 0);
    }
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    gmlp::Kv4AttnArgs k{};
    k.Q = static_cast<const bf16*>(a->Q);
    k.O = static_cast<bf16*>(a->O);
    k.c = kv4_cache(a->cache);
    k.table = static_cast<const int32_t*>(a->block_table);
    k.lengths = static_cast<const int32_t*>(a->lengths);
    k.part = static_cast<float*>(a->workspace);
    k.B = (int)a->B;
    k.T = a->q_len;
    k.Hq = a->n_q_heads;
    k.ratio = ratio;
    k.width = (int)a->table_width;
    k.splits = plan.splits;
    k.col_tiles = plan.col_tiles;
    // 31 steps of a query, summed over 128 channels, are 2^12 of it: times 2^-14 they have a float wherever the query has one
    const bool scaled = std::fabs(scale_log2) < 0x1p113f;
    k.q_scale = scaled ? 0x38803880u : 0x3F803F80u;
    k.s_scale = scaled ? scale_log2 * 0x1p14f : scale_log2;
    const dim3 grid((unsigned)plan.splits, (unsigned)(k.c.n_kv_heads * plan.col_tiles), (unsigned)a->B);
    if (grid.y > 65535u) return GMLP_ERR_SHAPE;
    prof_begin(st);
#define GMLP_KV4_ATTN1(D, G) launch_chained(gmlp::kv4_attention_kernel<D, G, 1>, grid, gmlp::kKv4Threads, (uint32_t)gmlp::kv4_smem_bytes(D, G, 1), 1, st, k)
#define GMLP_KV4_ATTN2(D, G) launch_chained(gmlp::kv4_attention_kernel<D, G, 2>, grid, gmlp::kKv4Threads, (uint32_t)gmlp::kv4_smem_bytes(D, G, 2), 1, st, k)
    rc = plan.nt == 1 ? GMLP_KV4_DISPATCH(k.c, GMLP_KV4_ATTN1) : GMLP_KV4_DISPATCH(k.c, GMLP_KV4_ATTN2);
    if (rc != GMLP_OK) return rc;
    prof_mark("kv4_attention", st);
    if (plan.splits > 1) {
        const dim3 rows((unsigned)(a->B * a->q_len * a->n_q_heads));
        // few splits of many rows: small CTAs; many splits: sixteen or more shares of them at once
#define GMLP_KV4_JOIN(D, NT)                                                                                        \
    (plan.splits <= 16 ? launch_chained(gmlp::kv4_join_kernel<D, NT, 128>, rows, 128, 0, 1, st, k)                  \
                       : launch_chained(gmlp::kv4_join_kernel<D, NT, 512>, rows, 512, 0, 1, st, k))
        if (k.c.head_dim == 128) rc = plan.nt == 1 ? GMLP_KV4_JOIN(128, 1) : GMLP_KV4_JOIN(128, 2);
        else rc = plan.nt == 1 ? GMLP_KV4_JOIN(64, 1) : GMLP_KV4_JOIN(64, 2);
        if (rc != GMLP_OK) return rc;
        prof_mark("kv4_join", st);
    }
    return finish_checked(dev, a->flags, st);
}
