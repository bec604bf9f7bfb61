// Host side of rotary positions, the paged bf16 cache and the attention over it.  Included by api.cu inside its namespace.

// Turns per position of each pair in units of 2^-64, and the amplitude; 80-bit arithmetic on the host.
int rope_steps_impl(int32_t rot, double base, const gmlp_rope_scaling* s, uint64_t* steps, float* amplitude) {
    if (steps == nullptr || amplitude == nullptr) return GMLP_ERR_NULL;
    if (rot < 4 || rot > 1024 || rot % 4 != 0 || !(base > 1.0) || !(base < 1e30)) return GMLP_ERR_SHAPE;
    const int kind = s == nullptr ? GMLP_ROPE_PLAIN : s->kind;
    if (kind < GMLP_ROPE_PLAIN || kind > GMLP_ROPE_RAMP || (s != nullptr && s->reserved != 0)) return GMLP_ERR_FLAGS;
    const long double turn = 6.283185307179586476925286766559005768L;
    long double lo = 0, hi = 0;
    *amplitude = 1.0f;
    if (kind != GMLP_ROPE_PLAIN && !(s->factor > 0.0 && s->factor < 1e30)) return GMLP_ERR_SHAPE;
    if (kind == GMLP_ROPE_BANDS && !(s->low >= 0.0 && s->high > s->low && s->high < 1e30 && s->original > 0.0 && s->original < 1e30))
        return GMLP_ERR_SHAPE;
    if (kind == GMLP_ROPE_RAMP) {
        if (!(s->high >= s->low && s->low > 0.0 && s->high < 1e30 && s->original > 0.0 && s->original < 1e30)) return GMLP_ERR_SHAPE;
        // the pairs that turn `high` and `low` times within the trained context
        const auto at = [&](double turns) { return rot * logl(s->original / (turns * turn)) / (2 * logl((long double)base)); };
        lo = fmaxl(floorl(at(s->high)), 0);
        hi = fminl(ceill(at(s->low)), rot - 1);
        *amplitude = s->factor > 1.0 ? (float)(0.1 * log(s->factor) + 1.0) : 1.0f;
    }
    for (int i = 0; i < rot / 2; ++i) {
        const long double f = powl((long double)base, -2.0L * i / rot) / turn;
        long double keep = 1;
        if (kind == GMLP_ROPE_LINEAR) keep = 0;
        if (kind == GMLP_ROPE_BANDS) keep = (s->original * f - s->low) / ((long double)s->high - s->low);
        if (kind == GMLP_ROPE_RAMP) keep = 1 - (i - lo) / fmaxl(hi - lo, 0.001L);
        keep = fminl(fmaxl(keep, 0), 1);
        long double g = kind == GMLP_ROPE_PLAIN ? f : f * keep + f / s->factor * (1 - keep);
        g -= floorl(g);
        const long double units = roundl(g * 18446744073709551616.0L);
        steps[i] = units >= 18446744073709551616.0L ? 0 : (uint64_t)units;
    }
    return GMLP_OK;
}

// `steps` may be NULL (no rotation) where `optional`.
int check_rope(const gmlp_rope& r, int head_dim, bool optional) {
    if (r.reserved != 0 || (r.interleaved != 0 && r.interleaved != 1)) return GMLP_ERR_FLAGS;
    if (r.steps == nullptr) return optional ? GMLP_OK : GMLP_ERR_NULL;
    if (r.rotary_dim < 4 || r.rotary_dim > head_dim || r.rotary_dim % 4 != 0 || !(r.amplitude - r.amplitude == 0.0f)) return GMLP_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(r.steps) & 7u) return GMLP_ERR_ALIGN;
    return GMLP_OK;
}

template <typename... P, typename... A>
int launch_block(void (*kernel)(P...), dim3 grid, dim3 block, uint32_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) return GMLP_ERR_LAUNCH;
    GMLP_CHECK_LAUNCH();
    return GMLP_OK;
}

int launch_rotate(DeviceState* dev, gmlp::RotateArgs& k, bool interleaved, cudaStream_t st) {
    const int half = k.rot / 2, rest = k.D - k.rot;
    const bool inter = interleaved;
    const int vec = (inter ? k.rot : half) % 8 == 0 ? 8 : 2;
    k.apart = rest % (2 * vec) == 0 ? rest / 2 : 0;
    k.turned_apart = !inter || k.rot % (2 * vec) == 0 ? half : 0;
    const int units = (k.turned_apart > 0 ? half : k.rot) / vec + rest / vec / (k.apart > 0 ? 2 : 1);
    // Threads: `lanes` to a unit of a token's heads, each with as many heads as the next, and as many tokens side by side as fit.  Whole tokens
    // per CTA, two or four rounds of them while there are enough CTAs (four per SM); the heads of few tokens go to several CTAs.
    const int heads = k.Hq + 2 * k.Hkv, sms = dev->sm_count;
    const int most = units >= gmlp::kRotateThreads ? 1 : gmlp::kRotateThreads / units, rounds = (heads + most - 1) / most;
    k.lanes = (heads + rounds - 1) / rounds;
    int side = most / k.lanes;
    if (side > gmlp::kRotateMaxTokens / 2) side = gmlp::kRotateMaxTokens / 2;
    if (side > k.T / sms) side = k.T / sms;
    if (side < 1) side = 1;
    k.tokens = k.T >= 16 * side * sms ? 4 * side : (k.T >= 8 * side * sms ? 2 * side : side);
    if (k.tokens > gmlp::kRotateMaxTokens) k.tokens = gmlp::kRotateMaxTokens;
    int split = k.T >= sms ? 1 : sms / k.T;
    if (split > rounds) split = rounds;
    const dim3 grid((unsigned)((k.T + k.tokens - 1) / k.tokens), (unsigned)split), block((unsigned)units, (unsigned)(side * k.lanes));
    const uint32_t smem = (uint32_t)(k.tokens * half * sizeof(float2));
    if (vec == 8) return inter ? launch_block(gmlp::rotate_kernel<8, true>, grid, block, smem, st, k)
                               : launch_block(gmlp::rotate_kernel<8, false>, grid, block, smem, st, k);
    return inter ? launch_block(gmlp::rotate_kernel<2, true>, grid, block, smem, st, k)
                 : launch_block(gmlp::rotate_kernel<2, false>, grid, block, smem, st, k);
}

constexpr int64_t kRopeMaxRows = (int64_t)1 << 24;

int rope_apply_impl(const gmlp_rope_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_rope_args) || (a->flags & ~(uint32_t)GMLP_FLAG_CHECKED)) return GMLP_ERR_FLAGS;
    if (a->T < 0 || a->T > kRopeMaxRows || a->n_heads <= 0 || a->n_heads > 65535 || a->head_dim < 8 || a->head_dim > 512 || a->head_dim % 8 != 0)
        return GMLP_ERR_SHAPE;
    int rc = check_rope(a->rope, a->head_dim, false);
    if (rc != GMLP_OK) return rc;
    if (a->T == 0) return GMLP_OK;
    if (!a->X || !a->Y || !a->positions) return GMLP_ERR_NULL;
    if (!aligned16(a->X) || !aligned16(a->Y) || (reinterpret_cast<uintptr_t>(a->positions) & 7u)) return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    gmlp::RotateArgs k{};
    k.Q = static_cast<const bf16*>(a->X);
    k.Qo = static_cast<bf16*>(a->Y);
    k.positions = static_cast<const int64_t*>(a->positions);
    k.steps = static_cast<const uint64_t*>(a->rope.steps);
    k.amplitude = a->rope.amplitude;
    k.T = (int)a->T;
    k.Hq = a->n_heads;
    k.D = a->head_dim;
    k.rot = a->rope.rotary_dim;
    prof_begin(st);
    rc = launch_rotate(dev, k, a->rope.interleaved != 0, st);
    if (rc != GMLP_OK) return rc;
    prof_mark("rope", st);
    return finish_checked(dev, a->flags, st);
}

int check_kv_cache(const gmlp_kv_cache& c) {
    if (c.reserved != 0) return GMLP_ERR_FLAGS;
    if (c.head_dim != 64 && c.head_dim != 128) return GMLP_ERR_UNSUPPORTED;
    if (c.n_pages <= 0 || c.n_kv_heads <= 0 || c.n_kv_heads > 4096 || c.page_size < 16 || c.page_size > 65536 || c.page_size % 16 != 0 ||
        c.n_pages > INT32_MAX / c.page_size / c.n_kv_heads)
        return GMLP_ERR_SHAPE;
    if (!c.k || !c.v) return GMLP_ERR_NULL;
    if (!aligned16(c.k) || !aligned16(c.v)) return GMLP_ERR_ALIGN;
    return GMLP_OK;
}

int kv_append_impl(const gmlp_kv_append_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_kv_append_args) || (a->flags & ~(uint32_t)GMLP_FLAG_CHECKED) || a->reserved != 0) return GMLP_ERR_FLAGS;
    int rc = check_kv_cache(a->cache);
    if (rc != GMLP_OK) return rc;
    rc = check_rope(a->rope, a->cache.head_dim, true);
    if (rc != GMLP_OK) return rc;
    const bool rope = a->rope.steps != nullptr, queries = a->Q != nullptr || a->Qout != nullptr;
    if (a->T < 0 || a->T > kRopeMaxRows || a->n_q_heads < 0 || a->n_q_heads > 65535 || (queries && a->n_q_heads == 0)) return GMLP_ERR_SHAPE;
    if (a->T == 0) return GMLP_OK;
    if (!a->K || !a->V || !a->slots || (rope && !a->positions) || (queries && (!a->Q || !a->Qout || !rope))) return GMLP_ERR_NULL;
    if (!aligned16(a->K) || !aligned16(a->V) || !aligned16(a->Q) || !aligned16(a->Qout) || (reinterpret_cast<uintptr_t>(a->slots) & 7u) ||
        (reinterpret_cast<uintptr_t>(a->positions) & 7u))
        return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    gmlp::RotateArgs k{};
    k.Q = static_cast<const bf16*>(a->Q);
    k.Qo = static_cast<bf16*>(a->Qout);
    k.K = static_cast<const bf16*>(a->K);
    k.V = static_cast<const bf16*>(a->V);
    k.kc = static_cast<bf16*>(a->cache.k);
    k.vc = static_cast<bf16*>(a->cache.v);
    k.positions = static_cast<const int64_t*>(a->positions);
    k.slots = static_cast<const int64_t*>(a->slots);
    k.steps = static_cast<const uint64_t*>(a->rope.steps);
    k.amplitude = a->rope.amplitude;
    k.T = (int)a->T;
    k.Hq = queries ? a->n_q_heads : 0;
    k.Hkv = a->cache.n_kv_heads;
    k.D = a->cache.head_dim;
    k.rot = rope ? a->rope.rotary_dim : 0;
    k.page_size = a->cache.page_size;
    k.total = a->cache.n_pages * a->cache.page_size;
    prof_begin(st);
    rc = launch_rotate(dev, k, a->rope.interleaved != 0, st);
    if (rc != GMLP_OK) return rc;
    prof_mark("kv_append", st);
    return finish_checked(dev, a->flags, st);
}

constexpr int64_t kKvMostKeys = (int64_t)1 << 30;        // of one request: positions stay well inside 31 bits
constexpr int kKvMaxRatio = 128;                         // query heads to a key/value head: a tile's rows
int check_kv_attention(int64_t B, int64_t T, int Hq, int Hkv, int64_t width, int page_size) {
    if (B < 0 || B > 65535 || T < 0 || T > kRopeMaxRows || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Hq > 65535 || width < 1 ||
        width > kKvMostKeys / page_size)
        return GMLP_ERR_SHAPE;
    return Hq / Hkv > kKvMaxRatio ? GMLP_ERR_UNSUPPORTED : GMLP_OK;
}

// Rows of a partial result: a big item's two tiles of 128, or what all rows of the call make.
int kv_slot_rows(int64_t T, int ratio) { return T * ratio <= 128 ? (int)(T * ratio) : 256; }
uint64_t kv_attention_workspace(int64_t T, int Hq, int Hkv, int head_dim, int sms) {
    return gmlp::kv_ws_bytes(sms, kv_slot_rows(T, Hq / Hkv), head_dim);
}

bool encode_kv_query(CUtensorMap* map, const void* ptr, int head_dim, int Hq, int64_t T, int box_heads, int box_rows) {
    const cuuint64_t gdim[3] = {(cuuint64_t)head_dim, (cuuint64_t)Hq, (cuuint64_t)T};
    const cuuint64_t gstride[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)head_dim * 2 * Hq};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    const cuuint32_t estride[3] = {1, 1, 1};
    return g_encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), gdim, gstride, box, estride,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
int launch_kv_attention(DeviceState* dev, const CUtensorMap& tmQ, const CUtensorMap& tmQfew, const CUtensorMap& tmK, const CUtensorMap& tmV,
                        const gmlp::KvAttnArgs& k, bool few, bool long_items, bool join, cudaStream_t st) {
    const auto kernel = few ? (long_items ? gmlp::kv_attention_kernel<D, true, true> : gmlp::kv_attention_kernel<D, true, false>)
                            : (long_items ? gmlp::kv_attention_kernel<D, false, true> : gmlp::kv_attention_kernel<D, false, false>);
    bool& set = dev->kv_attr_set[4 * (D == 128) + 2 * few + long_items];
    if (!set) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)gmlp::kv_attn_smem(D)) != cudaSuccess)
            return GMLP_ERR_LAUNCH;
        set = true;
    }
    const int ctas = dev->sm_count;
    int rc = launch_block(kernel, dim3((unsigned)ctas), dim3(gmlp::kKvThreads), gmlp::kv_attn_smem(D), st, tmQ, tmQfew, tmK, tmV, k);
    if (rc != GMLP_OK) return rc;
    prof_mark(few ? "kv_attention_few" : "kv_attention", st);
    if (!join) return GMLP_OK;
    rc = launch_block(gmlp::kv_join_kernel<D>, dim3((unsigned)ctas, k.slot_rows > 64 ? 8 : 4), dim3(gmlp::kKvJoinThreads), 0, st, k);
    if (rc != GMLP_OK) return rc;
    prof_mark("kv_join", st);
    return GMLP_OK;
}

int kv_attention_impl(const gmlp_kv_attention_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_kv_attention_args) || (a->flags & ~(uint32_t)(GMLP_FLAG_CHECKED | GMLP_KV_CAUSAL)) || a->reserved != 0)
        return GMLP_ERR_FLAGS;
    int rc = check_kv_cache(a->cache);
    if (rc != GMLP_OK) return rc;
    rc = check_kv_attention(a->B, a->T, a->n_q_heads, a->cache.n_kv_heads, a->table_width, a->cache.page_size);
    if (rc != GMLP_OK) return rc;
    if (a->q_start == nullptr && (a->q_len < 1 || a->B * a->q_len != a->T)) return GMLP_ERR_SHAPE;
    const float scale_log2 = a->scale * 1.4426950408889634f;                 // exponentials are powers of two
    if (!(scale_log2 > 0x1p-120f) || !(scale_log2 - scale_log2 == 0.0f)) return GMLP_ERR_FLAGS;
    if (a->B == 0 || a->T == 0) return GMLP_OK;
    if (!a->Q || !a->O || !a->block_table || !a->lengths) return GMLP_ERR_NULL;
    if (!aligned16(a->Q) || !aligned16(a->O) || (reinterpret_cast<uintptr_t>(a->block_table) & 3u) || (reinterpret_cast<uintptr_t>(a->lengths) & 3u) ||
        (reinterpret_cast<uintptr_t>(a->q_start) & 3u) || (reinterpret_cast<uintptr_t>(a->workspace) & 255u))
        return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    const int ratio = a->n_q_heads / a->cache.n_kv_heads;
    const uint64_t need = kv_attention_workspace(a->T, a->n_q_heads, a->cache.n_kv_heads, a->cache.head_dim, dev->sm_count);
    if (a->workspace == nullptr) return GMLP_ERR_NULL;
    if (a->workspace_bytes < need) return GMLP_ERR_WORKSPACE;
    claim_workspace(dev, static_cast<const uint8_t*>(a->workspace), need, nullptr, 0);
    gmlp::KvAttnArgs k{};
    k.O = static_cast<bf16*>(a->O);
    k.v = static_cast<const bf16*>(a->cache.v);
    k.table = static_cast<const int32_t*>(a->block_table);
    k.lengths = static_cast<const int32_t*>(a->lengths);
    k.q_start = static_cast<const int32_t*>(a->q_start);
    k.workspace = static_cast<uint8_t*>(a->workspace);
    k.B = (int)a->B;
    k.T = (int)a->T;
    k.Hq = a->n_q_heads;
    k.Hkv = a->cache.n_kv_heads;
    k.ratio = ratio;
    k.width = (int)a->table_width;
    k.page_size = a->cache.page_size;
    k.n_pages = (int)a->cache.n_pages;
    k.q_len = a->q_len;
    k.causal = (a->flags & GMLP_KV_CAUSAL) != 0;
    k.scale_log2 = scale_log2;
    k.tile_pos = 128 / ratio;
    k.box = a->cache.page_size & -a->cache.page_size;
    if (k.box > gmlp::kKvBlock) k.box = gmlp::kKvBlock;
    const int q_pos = a->T < k.tile_pos ? (int)a->T : k.tile_pos, D = a->cache.head_dim;
    // Where a request has more than 256 rows (a big item's) on average, most belong to big items, and these run better in the kernel that has no
    // code for few ones (a chunk of 2048 237 us with, 226 without; 40 single tokens and three chunks of 500, 143 rows on average, 234 and 246).
    // The host knows neither the lengths nor which rows belong to a request: padded rows count, and a chunk beside single tokens over many more
    // keys may take the kernel without few items although most of the work is theirs.
    const bool few = a->T * ratio <= 256 * a->B;
    k.few_pos = few ? gmlp::kKvFew / ratio : 0;                              // 0: none
    const int few_pos = k.few_pos == 0 ? q_pos : (a->T < k.few_pos ? (int)a->T : k.few_pos);
    k.q_bytes = ratio * q_pos * D * 2;
    k.q_few_bytes = ratio * few_pos * D * 2;
    k.slot_rows = kv_slot_rows(a->T, ratio);
    k.min_stretch = 768;
    const uint64_t cache_rows = (uint64_t)a->cache.n_pages * (uint64_t)k.Hkv * (uint64_t)k.page_size;
    CUtensorMap tmQ, tmQfew, tmK, tmV;
    if (!encode_kv_query(&tmQ, a->Q, D, k.Hq, a->T, ratio, q_pos) || !encode_kv_query(&tmQfew, a->Q, D, k.Hq, a->T, ratio, few_pos) ||
        !encode_2d(&tmK, a->cache.k, (uint64_t)D, cache_rows, 64, (uint32_t)k.box) ||
        !encode_2d(&tmV, a->cache.v, (uint64_t)D, cache_rows, 64, (uint32_t)k.box))
        return GMLP_ERR_LAUNCH;
    prof_begin(st);
    // no item is long enough to be cut where the table has few pages
    const int mode = a->T <= k.few_pos ? gmlp::kKvFewItem : (a->T <= k.tile_pos ? gmlp::kKvSmallItem : gmlp::kKvBigItem);
    const bool join = gmlp::kv_start(mode) + a->table_width * k.page_size * gmlp::kv_key(mode) > gmlp::kKvSnap;
    const bool long_items = a->table_width * k.page_size > gmlp::kKvFewSum * gmlp::kKvBlock;
    rc = D == 128 ? launch_kv_attention<128>(dev, tmQ, tmQfew, tmK, tmV, k, few, long_items, join, st)
                  : launch_kv_attention<64>(dev, tmQ, tmQfew, tmK, tmV, k, few, long_items, join, st);
    if (rc != GMLP_OK) return rc;
    return finish_checked(dev, a->flags, st);
}
