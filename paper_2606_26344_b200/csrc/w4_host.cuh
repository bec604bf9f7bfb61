// Host side of the 4-bit weight operators: checks, launch shapes, launches.  Included by api.cu inside its namespace.

enum { kW4Stream = 0, kW4Tile = 1, kW4Umma = 2 };
struct W4Plan {
    int kind;                                        // the kernel, kW4Stream, kW4Tile or kW4Umma
    int nt, ctas, threads, group_warps;
    int m_cta, m_parts, wr_log2, cluster;            // tile and umma kernels
    uint32_t smem;
};
inline int w4_k_blocks(int64_t K) { return (int)((K + 255) / 256) * 2; }      // of 128 rows, an even number
constexpr uint32_t kW4SmemMost = 224 * 1024;

// Launch shape of one product: `n16` column tiles (gated: of each matrix), K in `KB` blocks of 128, groups of G.
W4Plan w4_plan(int M, int terms, int KB, int n16, bool gated, int G, int sms) {
    W4Plan p{};
    const int rows = M * terms;
    // The persistent kernel, where all of X fits beside the rings.
    if (rows <= 16) {
        const uint64_t smem = gmlp::w4_stream_bytes(rows, KB, G);
        if (smem <= kW4SmemMost) {
            p.kind = kW4Stream;
            p.nt = rows <= 8 ? 1 : 2;
            p.threads = gmlp::kW4StreamThreads;
            // eight warps a tile where K is long or there are few tiles, else four (fewer hand-overs of sums)
            p.group_warps = KB >= 64 || n16 <= sms ? 8 : 4;
            p.ctas = n16 < sms ? n16 : sms;
            p.m_cta = M;
            p.m_parts = p.cluster = 1;
            p.smem = (uint32_t)smem;
            return p;
        }
    }
    // tcgen05 for more than 16 rows where its groups of 128 columns fill most of the GPU, in one wave or with K of 4096 or more
    // (1024 x 14336 at M = 64: 10.4 us against 18.5 for the tiles; 1024 x 28672 at M = 20, two short waves: 18.4 against 12.9), or where K
    // is long enough to pay for a cluster (14336 x 4096 at M = 64: 34.6 against 52; 4096 x 4096: 22.1 against 17.4); else tiles.
    const int groups128 = gated ? (n16 + 3) / 4 : (n16 + 7) / 8, ctas128 = groups128 * ((rows + 63) / 64);
    p.kind = rows > 16 && ((ctas128 >= 96 && (ctas128 <= sms || KB >= 32)) || (ctas128 >= 32 && KB >= 64)) ? kW4Umma : kW4Tile;
    const int rows_most = p.kind == kW4Umma ? 64 : 32;
    p.m_parts = (rows + rows_most - 1) / rows_most;
    p.m_cta = (M + p.m_parts - 1) / p.m_parts;
    p.m_parts = (M + p.m_cta - 1) / p.m_cta;
    const int rows_cta = p.m_cta * terms;
    p.cluster = 1;
    if (p.kind == kW4Umma) {
        p.nt = rows_cta <= 32 ? 4 : 8;               // rows are padded to 32 or 64
        // K over a cluster of up to four while the CTAs fit one wave, as long as each keeps eight k-blocks
        while (p.cluster < 4 && groups128 * p.m_parts <= cluster_capacity_estimate(p.cluster + 1, sms) && KB >= 8 * (p.cluster + 1)) ++p.cluster;
        p.ctas = groups128 * p.cluster;
        p.threads = gmlp::kW4UmmaThreads;
        p.smem = gmlp::w4_umma_smem(8 * p.nt);
        return p;
    }
    p.nt = (rows_cta + 7) / 8;
    const int units = gated ? n16 : (n16 + 1) / 2;
    // Column groups per CTA: few, so that a CTA's warps share long ranges of K and their sums stay in the CTA, unless there are
    // columns enough to fill the GPU with more (each group reads its CTA's copy of X).
    p.wr_log2 = rows_cta <= 16 ? 0 : (units * p.m_parts >= 4 * sms ? 2 : 1);
    const int WR = 1 << p.wr_log2, WK = 8 >> p.wr_log2, groups = (units + WR - 1) / WR;
    // K over a cluster only where the CTAs would leave a third of the SMs idle: its hand-over costs about two microseconds
    while (p.cluster < 4 && 3 * groups * p.m_parts * p.cluster <= 2 * sms && KB >= 2 * WK * (p.cluster + 1)) ++p.cluster;
    p.ctas = groups * p.cluster;
    p.threads = gmlp::kW4Threads;
    p.smem = gmlp::w4_tile_smem(p.nt, rows_cta, WK, G);
    return p;
}

typedef void (*W4Kernel)(gmlp::W4GemmArgs);
typedef void (*W4UmmaKernel)(gmlp::W4GemmArgs, CUtensorMap);
template <int NT>
W4Kernel w4_stream_kernel_for(int G, bool gated) {
    if (gated) return G == 32 ? gmlp::w4_stream_kernel<NT, 32, true> : (G == 64 ? gmlp::w4_stream_kernel<NT, 64, true> : gmlp::w4_stream_kernel<NT, 128, true>);
    return G == 32 ? gmlp::w4_stream_kernel<NT, 32, false> : (G == 64 ? gmlp::w4_stream_kernel<NT, 64, false> : gmlp::w4_stream_kernel<NT, 128, false>);
}
template <int NT>
W4Kernel w4_tile_kernel_for(int G, bool gated) {
    if (gated) return G == 32 ? gmlp::w4_tile_kernel<NT, 32, true> : (G == 64 ? gmlp::w4_tile_kernel<NT, 64, true> : gmlp::w4_tile_kernel<NT, 128, true>);
    return G == 32 ? gmlp::w4_tile_kernel<NT, 32, false> : (G == 64 ? gmlp::w4_tile_kernel<NT, 64, false> : gmlp::w4_tile_kernel<NT, 128, false>);
}
template <int RPAD>
W4UmmaKernel w4_umma_kernel_for(int G, bool gated) {
    if (gated) return G == 32 ? gmlp::w4_umma_kernel<RPAD, 32, true> : (G == 64 ? gmlp::w4_umma_kernel<RPAD, 64, true> : gmlp::w4_umma_kernel<RPAD, 128, true>);
    return G == 32 ? gmlp::w4_umma_kernel<RPAD, 32, false> : (G == 64 ? gmlp::w4_umma_kernel<RPAD, 64, false> : gmlp::w4_umma_kernel<RPAD, 128, false>);
}

int check_w4_matrix(const gmlp_w4_matrix& w) {
    if (w.reserved != 0) return GMLP_ERR_FLAGS;
    if (w.group != 32 && w.group != 64 && w.group != 128) return GMLP_ERR_SHAPE;
    if (w.K <= 0 || w.N <= 0 || w.K > kW4MaxDim || w.N > kW4MaxDim || w.K % w.group != 0) return GMLP_ERR_SHAPE;
    if (w.codes == nullptr || w.scales == nullptr) return GMLP_ERR_NULL;
    if (!aligned16(w.codes) || !aligned16(w.scales) || !aligned16(w.zeros)) return GMLP_ERR_ALIGN;
    return GMLP_OK;
}
inline gmlp::W4Operand w4_operand(const gmlp_w4_matrix& w) {
    return {static_cast<const uint8_t*>(w.codes), static_cast<const bf16*>(w.scales), static_cast<const uint8_t*>(w.zeros)};
}

// One launch chained to its predecessor by programmatic dependent launch.
template <typename... P, typename... A>
int launch_chained(void (*kernel)(P...), dim3 grid, unsigned threads, uint32_t smem, int cluster, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) != cudaSuccess) return GMLP_ERR_LAUNCH;
    GMLP_CHECK_LAUNCH();
    return GMLP_OK;
}

int launch_w4_gemm(DeviceState* dev, const gmlp_w4_matrix& w0, const gmlp_w4_matrix* w1, const bf16* X, int terms, bf16* out,
                   int64_t M, gmlp::GateAct act, bool early, cudaStream_t st) {
    const int K = (int)w0.K, N = (int)w0.N, KB = w4_k_blocks(K), n16 = (N + 15) / 16;
    const bool gated = w1 != nullptr;
    const W4Plan p = w4_plan((int)M, terms, KB, n16, gated, w0.group, dev->sm_count);
    W4Kernel kernel = nullptr;
    W4UmmaKernel umma = nullptr;
    int row = 0;                                     // of the kernels, for the attribute below
    if (p.kind == kW4Stream) {
        kernel = p.nt == 1 ? w4_stream_kernel_for<1>(w0.group, gated) : w4_stream_kernel_for<2>(w0.group, gated);
        row = p.nt - 1;
    } else if (p.kind == kW4Umma) {
        umma = p.nt == 4 ? w4_umma_kernel_for<32>(w0.group, gated) : w4_umma_kernel_for<64>(w0.group, gated);
        row = p.nt == 4 ? 2 : 3;
    } else {
        switch (p.nt) {
            case 1: kernel = w4_tile_kernel_for<1>(w0.group, gated); break;
            case 2: kernel = w4_tile_kernel_for<2>(w0.group, gated); break;
            case 3: kernel = w4_tile_kernel_for<3>(w0.group, gated); break;
            default: kernel = w4_tile_kernel_for<4>(w0.group, gated); break;
        }
        row = 3 + p.nt;
    }
    const int slot = row * 6 + (gated ? 3 : 0) + (w0.group == 32 ? 0 : (w0.group == 64 ? 1 : 2));
    if (!dev->w4_attr_set[slot]) {
        const void* f = umma != nullptr ? reinterpret_cast<const void*>(umma) : reinterpret_cast<const void*>(kernel);
        if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kW4SmemMost) != cudaSuccess) return GMLP_ERR_LAUNCH;
        dev->w4_attr_set[slot] = true;
    }
    gmlp::W4GemmArgs a{};
    a.w[0] = w4_operand(w0);
    a.w[1] = gated ? w4_operand(*w1) : a.w[0];
    a.X = X;
    a.out = out;
    a.M = (int)M;
    a.K = K;
    a.N = N;
    a.KB = KB;
    a.n16 = n16;
    a.terms = terms;
    a.m_cta = p.m_cta;
    a.cluster = p.cluster;
    a.group_warps = p.group_warps;
    a.wr_log2 = p.wr_log2;
    a.early = early ? 1 : 0;
    a.act = act;
    const dim3 grid((unsigned)p.ctas, (unsigned)p.m_parts);
    if (umma == nullptr) return launch_chained(kernel, grid, (unsigned)p.threads, p.smem, p.cluster, st, a);
    CUtensorMap tmX;                                 // rows of X in boxes of 64 k; two terms: a box each
    if (!encode_2d(&tmX, X, (uint64_t)K, (uint64_t)M * terms, 64, (uint32_t)(8 * p.nt / terms))) return GMLP_ERR_LAUNCH;
    return launch_chained(umma, grid, (unsigned)p.threads, p.smem, p.cluster, st, a, tmX);
}

int finish_checked(DeviceState* dev, uint32_t flags, cudaStream_t st) {
    if (!(flags & GMLP_FLAG_CHECKED)) return GMLP_OK;
    if (cudaStreamSynchronize(st) != cudaSuccess) return GMLP_ERR_LAUNCH;
    const int s = read_device_status();
    if (s == 0) return GMLP_OK;
    forget_counters(dev);                            // the word may be an earlier gmlp_forward's, cut short by a time-out
    return status_error(s);
}

int w4_matmul_impl(const gmlp_w4_matmul_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_w4_matmul_args) || (a->flags & ~(uint32_t)GMLP_FLAG_CHECKED)) return GMLP_ERR_FLAGS;
    int rc = check_w4_matrix(a->W);
    if (rc != GMLP_OK) return rc;
    if (a->M < 0 || a->M > gmlp::kW4MaxM) return GMLP_ERR_SHAPE;
    if (a->M == 0) return GMLP_OK;
    if (!a->X || !a->Y) return GMLP_ERR_NULL;
    if (!aligned16(a->X) || !aligned16(a->Y)) return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    prof_begin(st);
    rc = launch_w4_gemm(dev, a->W, nullptr, static_cast<const bf16*>(a->X), 1, static_cast<bf16*>(a->Y), a->M, kSilu, false, st);
    if (rc != GMLP_OK) return rc;
    prof_mark("w4_matmul", st);
    return finish_checked(dev, a->flags, st);
}

uint64_t w4_forward_workspace(int64_t M, int64_t d_model, int64_t d_ff, uint32_t flags) {
    if (M < 0 || M > gmlp::kW4MaxM || d_model <= 0 || d_ff <= 0 || d_model > kW4MaxDim || d_ff > kW4MaxDim) return 0;
    const uint64_t xn = (flags & GMLP_FLAG_RMSNORM) ? align256((uint64_t)M * d_model * 4) : 0;
    return xn + align256((uint64_t)M * d_ff * 4);
}

int w4_forward_impl(const gmlp_w4_args* a) {
    if (a == nullptr) return GMLP_ERR_NULL;
    const uint32_t known = GMLP_FLAG_CHECKED | GMLP_FLAG_RMSNORM | GMLP_FLAG_ACT_SWISH | GMLP_FLAG_ACT_GLU | GMLP_FLAG_ACT_GELU;
    if (a->struct_bytes != sizeof(gmlp_w4_args) || (a->flags & ~known) || a->reserved != 0) return GMLP_ERR_FLAGS;
    gmlp::GateAct act;
    if (!gate_act_from(a->flags, a->act_beta, &act)) return GMLP_ERR_FLAGS;
    int rc = GMLP_OK;
    for (const gmlp_w4_matrix* w : {&a->Wg, &a->Wu, &a->Wd}) {
        rc = check_w4_matrix(*w);
        if (rc != GMLP_OK) return rc;
    }
    const int64_t d_model = a->Wg.K, d_ff = a->Wg.N;
    if (a->Wu.K != d_model || a->Wu.N != d_ff || a->Wd.K != d_ff || a->Wd.N != d_model || a->Wu.group != a->Wg.group ||
        (a->Wu.zeros == nullptr) != (a->Wg.zeros == nullptr) || a->M < 0 || a->M > gmlp::kW4MaxM)
        return GMLP_ERR_SHAPE;
    if (a->M == 0) return GMLP_OK;
    if (!a->X || !a->Y || !a->workspace) return GMLP_ERR_NULL;
    if (!aligned16(a->X) || !aligned16(a->Y) || !aligned16(a->rms_gain)) return GMLP_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(a->workspace) & 255u) return GMLP_ERR_ALIGN;
    if (a->workspace_bytes < w4_forward_workspace(a->M, d_model, d_ff, a->flags)) return GMLP_ERR_WORKSPACE;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    uint8_t* ws = static_cast<uint8_t*>(a->workspace);
    const bool norm = (a->flags & GMLP_FLAG_RMSNORM) != 0;
    claim_workspace(dev, ws, w4_forward_workspace(a->M, d_model, d_ff, a->flags), nullptr, 0);
    bf16* Xn = reinterpret_cast<bf16*>(ws);
    bf16* H = reinterpret_cast<bf16*>(ws + (norm ? align256((uint64_t)a->M * d_model * 4) : 0));
    const bf16* X = static_cast<const bf16*>(a->X);
    prof_begin(st);
    if (norm) {
        rc = launch_chained(gmlp::w4_norm_kernel, dim3((unsigned)a->M), gmlp::kRmsThreads, 0, 1, st, X,
                            static_cast<const bf16*>(a->rms_gain), Xn, (int)a->M, (int)d_model, a->rms_eps);
        if (rc != GMLP_OK) return rc;
        prof_mark("w4_norm", st);
    }
    // the call's first kernel waits for everything before the call; later kernels may fetch their weights at once
    rc = launch_w4_gemm(dev, a->Wg, &a->Wu, norm ? Xn : X, norm ? 2 : 1, H, a->M, act, norm, st);
    if (rc != GMLP_OK) return rc;
    prof_mark("w4_gate_up", st);
    rc = launch_w4_gemm(dev, a->Wd, nullptr, H, 2, static_cast<bf16*>(a->Y), a->M, kSilu, true, st);
    if (rc != GMLP_OK) return rc;
    prof_mark("w4_down", st);
    return finish_checked(dev, a->flags, st);
}

// kind: gmlp::kW4From* to pack, -1 to unpack
int w4_layout_impl(const gmlp_w4_layout_args* a, int kind) {
    if (a == nullptr) return GMLP_ERR_NULL;
    if (a->struct_bytes != sizeof(gmlp_w4_layout_args) || (a->flags & ~(uint32_t)(GMLP_FLAG_CHECKED | GMLP_FLAG_WEIGHTS_OUT_IN)))
        return GMLP_ERR_FLAGS;
    int rc = check_w4_matrix(a->m);
    if (rc != GMLP_OK) return rc;
    if (!a->W || (kind == gmlp::kW4FromCodes && (!a->scales || (a->zeros == nullptr) != (a->m.zeros == nullptr)))) return GMLP_ERR_NULL;
    // read and written element by element, bf16 but for the codes that pack reads
    if ((kind != gmlp::kW4FromCodes && (reinterpret_cast<uintptr_t>(a->W) & 1u)) ||
        (kind == gmlp::kW4FromCodes && (reinterpret_cast<uintptr_t>(a->scales) & 1u)))
        return GMLP_ERR_ALIGN;
    DeviceState* dev = current_device(&rc);
    if (dev == nullptr) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(a->stream);
    const int K = (int)a->m.K, N = (int)a->m.N, G = a->m.group, out_in = (a->flags & GMLP_FLAG_WEIGHTS_OUT_IN) ? 1 : 0;
    const dim3 grid((unsigned)(((N + 15) / 16 * 16 + 127) / 128), (unsigned)w4_k_blocks(K));
    uint8_t* codes = static_cast<uint8_t*>(const_cast<void*>(a->m.codes));
    bf16* scales = static_cast<bf16*>(const_cast<void*>(a->m.scales));
    uint8_t* zeros = static_cast<uint8_t*>(const_cast<void*>(a->m.zeros));
    const bf16* s_in = static_cast<const bf16*>(a->scales);
    const uint8_t* z_in = static_cast<const uint8_t*>(a->zeros);
    if (kind < 0)
        rc = launch_chained(gmlp::w4_unpack_kernel, grid, 128, 0, 1, st, codes, scales, zeros, static_cast<bf16*>(a->W), out_in, K, N, G);
    else if (kind == gmlp::kW4FromCodes)
        rc = launch_chained(gmlp::w4_pack_kernel<gmlp::kW4FromCodes>, grid, 128, 0, 1, st, a->W, out_in, s_in, z_in, codes, scales, zeros, K, N, G);
    else if (zeros == nullptr)
        rc = launch_chained(gmlp::w4_pack_kernel<gmlp::kW4FromBf16>, grid, 128, 0, 1, st, a->W, out_in, s_in, z_in, codes, scales, zeros, K, N, G);
    else
        rc = launch_chained(gmlp::w4_pack_kernel<gmlp::kW4FromBf16Zeros>, grid, 128, 0, 1, st, a->W, out_in, s_in, z_in, codes, scales, zeros, K, N, G);
    if (rc != GMLP_OK) return rc;
    return finish_checked(dev, a->flags, st);
}
