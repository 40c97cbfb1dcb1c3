// Host side of the LM-head operators beside the CAT loss: cat_logprob_fwd / cat_logprob_bwd and
// cat_topk_kd_loss_fwd_bwd.  Included at the end of cat_api.cu, whose planning, tensor-map and launch helpers it uses.
#pragma once

namespace {

static_assert(CAT_TOPK_MAX == lp::MAX_TOP && lp::MAX_TOP == lp::THREADS, "one thread per list entry");

// ------------------------------------------------------------------------------ log probabilities
struct LpPlan {
    long long Ts;          // rows per slab
    long long ldz;         // row pitch of the logits slab
    long long ld_g;        // row pitch of the group maxima
    int group;             // columns per maximum (lp::GroupOf)
    bool skinny;           // few rows: the kernel of skinny.cuh
    int n_slabs;
    int S;                 // vocabulary splits of a full slab (the most any slab uses)
    size_t off_m, off_l, off_u, off_id, off_g, off_z, total;
};

// Vocabulary splits of the fp32 forward product: about four CTAs per SM.
int f32_splits(long long rows, long long V) {
    long long S = cdiv(4 * kPlanSMs, cdiv(rows, f32::TM));
    const long long num_n = cdiv(V, f32::TN);
    if (S > num_n) S = num_n;
    return static_cast<int>(S > kMaxSplits ? kMaxSplits : S);
}
int head_splits(const cat_shape* s, long long rows) {
    return s->in_dtype == CAT_BF16 ? fwd_splits(rows, s->V) : f32_splits(rows, s->V);
}

// Up to 128 rows go to the kernel of skinny.cuh.  Whole calls with 20 alternatives, GEMM of tc_gemm.cuh (and its pass over W for the norms) / that
// kernel, in us: 2048 x 128256 267 / 101 for one row, 202 / 115 for 64, 213 / 131 for 128; 1024 x 151936 170 / 81, 145 / 87, 149 / 103.
bool use_skinny(const cat_shape* s) { return s->in_dtype == CAT_BF16 && s->T <= skinny::MAX_ROWS; }

// Vocabulary entries per tile of that kernel: the height whose tiles, dealt to the SMs, leave the busiest the least to read.
int skinny_tile_rows(long long V) {
    int best = 128;
    long long most = cdiv(cdiv(V, 128), kPlanSMs) * 128;
    for (int r = 96; r >= 64; r -= 32) {
        const long long x = cdiv(cdiv(V, r), kPlanSMs) * r;
        if (x < most) { most = x; best = r; }
    }
    return best;
}

template <int TPW, int HALVES, int SUB>
int launch_skinny_as(const CUtensorMap& tmW, const CUtensorMap& tmH, const skinny::Params& plan, int* status, int grid, cudaStream_t st) {
    skinny::Params p = plan;
    p.stages = (skinny::SMEM_BYTES - 1024 - 8192) / ((SUB * p.tile_rows + p.n) * tc::BK * 2);
    if (p.stages > skinny::MAX_STAGES) p.stages = skinny::MAX_STAGES;
    auto kern = skinny::logits_kernel<TPW, HALVES, SUB>;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(kern, skinny::SMEM_BYTES, allowed)) return CAT_ERR_CUDA;
    const int threads = 64 + 128 * HALVES + (p.gmax != nullptr ? skinny::NORM_THREADS : 0);
    kern<<<static_cast<unsigned>(grid), threads, skinny::SMEM_BYTES, st>>>(tmW, tmH, p, status);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}

// Logits of all T <= 128 rows: part_m/l/u [*n_parts][T], group maxima and slab.
int launch_skinny(const cat_shape* s, const LpPlan& plan, const void* H, const void* W, bool top, uint8_t* ws, int sm_count, int* n_parts,
                  cudaStream_t st) {
    skinny::Params p;
    memset(&p, 0, sizeof(p));
    p.part_m = reinterpret_cast<float*>(ws + plan.off_m);
    p.part_l = reinterpret_cast<float*>(ws + plan.off_l);
    p.part_u = reinterpret_cast<float*>(ws + plan.off_u);
    p.part_id = reinterpret_cast<int*>(ws + plan.off_id);
    if (top) {
        p.gmax = reinterpret_cast<float*>(ws + plan.off_g);
        p.zs = reinterpret_cast<__half*>(ws + plan.off_z);
        p.w_sq = reinterpret_cast<int*>(ws + kNormOffset);
    }
    p.part_stride = plan.Ts; p.ld_g = plan.ld_g; p.ldz = plan.ldz;
    p.T = static_cast<int>(s->T); p.V = static_cast<int>(s->V);
    p.n = static_cast<int>(cdiv(s->T, 16) * 16);
    p.tile_rows = skinny_tile_rows(s->V);
    p.n_tiles = static_cast<int>(cdiv(s->V, p.tile_rows));
    p.num_kb = static_cast<int>(cdiv(s->d, tc::BK));
    p.wait_ns = tc::WAIT_LIMIT_NS;
    CUtensorMap tmW, tmH;
    if (tmap_k_major(&tmW, W, s->V, s->d, s->ldW, p.tile_rows) != CAT_OK) return CAT_ERR_CUDA;
    if (tmap_k_major(&tmH, H, s->T, s->d, s->ldH, p.n) != CAT_OK) return CAT_ERR_CUDA;
    int grid = sm_count < kPlanSMs ? sm_count : kPlanSMs;
    if (p.n_tiles < grid) grid = p.n_tiles;
    *n_parts = grid;
    int* status = reinterpret_cast<int*>(ws);
    if (s->T <= 32) return launch_skinny_as<32, 1, 1>(tmW, tmH, p, status, grid, st);
    if (s->T <= 64) return launch_skinny_as<32, 2, 2>(tmW, tmH, p, status, grid, st);
    return launch_skinny_as<64, 2, 2>(tmW, tmH, p, status, grid, st);
}

LpPlan plan_lp(const cat_shape* s, int top_k) {
    LpPlan p;
    const bool bf16 = s->in_dtype == CAT_BF16;
    const long long tile = bf16 ? tile_m() : f32::TM;
    p.group = bf16 ? tc::LP_GROUP : f32::TN;
    p.ldz = cdiv(s->V, 256) * 256;
    p.ld_g = bf16 ? cdiv(s->V, tc::BN) * (tc::BN / tc::LP_GROUP) : cdiv(cdiv(s->V, f32::TN), 4) * 4;
    p.Ts = s->T;
    if (top_k > 0) {
        const long long mib = s->slab_mib > 0 ? s->slab_mib : kDefaultFusedSlabMiB;
        long long cap = (mib << 20) / (p.ldz * (bf16 ? 2 : 4)) / tile * tile;
        if (cap < tile) cap = tile;
        if (cap < s->T) p.Ts = cdiv(cdiv(s->T, cdiv(s->T, cap)), tile) * tile;      // slabs of even height
    }
    p.skinny = use_skinny(s);
    if (p.skinny) p.Ts = s->T;
    p.n_slabs = static_cast<int>(cdiv(s->T, p.Ts));
    p.S = head_splits(s, p.Ts);
    const long long rest = s->T - (p.n_slabs - 1) * p.Ts;
    if (head_splits(s, rest) > p.S) p.S = head_splits(s, rest);
    if (p.skinny) p.S = kPlanSMs;                // one part per CTA
    size_t off = kHeaderBytes;
    p.off_m = off; off = align256(off + sizeof(float) * p.S * p.Ts);
    p.off_l = off; off = align256(off + sizeof(float) * p.S * p.Ts);
    p.off_u = off; off = align256(off + sizeof(float) * p.S * p.Ts);
    p.off_id = off; off = align256(off + sizeof(int) * p.S * p.Ts);
    p.off_g = off; if (top_k > 0) off = align256(off + sizeof(float) * static_cast<size_t>(p.Ts) * p.ld_g);
    p.off_z = off; if (top_k > 0) off = align256(off + (bf16 ? 2 : 4) * static_cast<size_t>(p.Ts) * p.ldz);
    p.total = off;
    return p;
}

// Up to this many rows, with more than a few alternatives, get the row kernel's large CTAs.  Whole calls with them / with small ones, in us: 200 rows of
// 2048 x 128256, k = 64: 228 / 278; 58 of 272 x 2915, 20: 21.0 / 23.0; 296 of 1024 x 20000, 20: 53.7 / 55.8, 297: 59.9 / 55.8; one of 2048 x 128256,
// 4: 97.4 / 95.5; 200 of 1024 x 20000, 1: 45.1 / 43.6; 67 of 1024 x 151936, 4: 84.0 / 85.9.
constexpr long long kFewRows = 2 * kPlanSMs, kFewAlternatives = 4;

template <class TI, class TZ, bool TOP>
int launch_lp_rows(const cat_shape* s, const LpPlan& plan, const TI* H, const TI* W, long long r0, long long rws, int S, uint8_t* ws,
                   const int64_t* labels, const uint8_t* valid, int top_k, float* logp, float* lse, float* entropy,
                   int64_t* top_ids, float* top_logp, cudaStream_t st) {
    lp::RowParams<TI, TZ> rp;
    memset(&rp, 0, sizeof(rp));
    rp.part_m = reinterpret_cast<float*>(ws + plan.off_m);
    rp.part_l = reinterpret_cast<float*>(ws + plan.off_l);
    rp.part_u = reinterpret_cast<float*>(ws + plan.off_u);
    rp.part_id = reinterpret_cast<int*>(ws + plan.off_id);
    rp.part_stride = s->in_dtype == CAT_BF16 ? plan.Ts : rws;
    rp.S = S;
    rp.H = H; rp.W = W; rp.ldH = s->ldH; rp.ldW = s->ldW;
    rp.d = static_cast<int>(s->d); rp.V = static_cast<int>(s->V);
    rp.labels = labels ? reinterpret_cast<const long long*>(labels) + r0 : nullptr;
    rp.valid = valid ? valid + r0 : nullptr;
    rp.logp = logp ? logp + r0 : nullptr;
    rp.lse = lse + r0;
    rp.entropy = entropy + r0;
    if (TOP) {
        rp.w_sq = reinterpret_cast<const int*>(ws + kNormOffset);
        rp.zs = reinterpret_cast<const TZ*>(ws + plan.off_z);
        rp.ldz = plan.ldz;
        rp.gmax = reinterpret_cast<const float*>(ws + plan.off_g);
        rp.ld_g = plan.ld_g;
        rp.n_g = static_cast<int>(cdiv(s->V, plan.group));
        rp.k = top_k;
        rp.top_ids = reinterpret_cast<long long*>(top_ids) + r0 * top_k;
        rp.top_logp = top_logp + r0 * top_k;
    }
    // launched ahead of the logits kernel's end, for which it waits: a decoding step is short enough for the 2 us to show
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rws), 1, 1);
    const bool few = rws <= kFewRows && top_k > kFewAlternatives;
    cfg.blockDim = dim3(few ? lp::RT_FEW : lp::RT_MANY, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t err = few ? cudaLaunchKernelEx(&cfg, lp::row_kernel<TI, TZ, TOP, lp::RT_FEW>, rp)
                                : cudaLaunchKernelEx(&cfg, lp::row_kernel<TI, TZ, TOP, lp::RT_MANY>, rp);
    if (err != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
    return CAT_OK;
}

// The longest row of W, ahead of the logits GEMM or beside it (see lp::norm_kernel).
template <bool BESIDE>
int launch_norms(const cat_shape* s, const __nv_bfloat16* W, int n_groups, int* w_sq, int sm_count, cudaStream_t st) {
    auto kern = lp::norm_kernel<BESIDE>;
    if (BESIDE) {      // a kernel that prefers another split of shared memory and L1 than the GEMM's would wait for the GEMM's CTAs to leave their SMs
        static std::atomic<unsigned long long> done{0};
        int dev = -1;
        if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
        const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
        if (bit == 0 || (done.load(std::memory_order_relaxed) & bit) == 0) {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) {
                cudaGetLastError();
                return CAT_ERR_CUDA;
            }
            done.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(BESIDE ? sm_count : 2 * sm_count), 1, 1);
    cfg.blockDim = dim3(lp::NORM_THREADS<BESIDE>, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = BESIDE ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kern, W, static_cast<long long>(s->ldW), static_cast<int>(s->d), static_cast<int>(s->V), n_groups, w_sq) !=
        cudaSuccess) {
        cudaGetLastError();
        return CAT_ERR_CUDA;
    }
    return CAT_OK;
}
// From this many rows on the GEMM is long enough for the pass beside it (figures at lp::norm_kernel).
constexpr long long kNormsBesideRows = 1024;

template <bool TOP>
int lp_slab(const cat_shape* s, const LpPlan& plan, const CUtensorMap& tmW, const void* H, const void* W, long long r0, long long rws,
            uint8_t* ws, const int64_t* labels, const uint8_t* valid, int top_k, float* logp, float* lse, float* entropy,
            int64_t* top_ids, float* top_logp, int sm_count, cudaStream_t st) {
    const int S = head_splits(s, rws);
    float* part_m = reinterpret_cast<float*>(ws + plan.off_m);
    float* part_l = reinterpret_cast<float*>(ws + plan.off_l);
    float* part_u = reinterpret_cast<float*>(ws + plan.off_u);
    if (s->in_dtype == CAT_BF16) {
        const __nv_bfloat16* Hs = static_cast<const __nv_bfloat16*>(H) + r0 * s->ldH;
        if (plan.skinny) {
            int n_parts = 0;
            const int rc = launch_skinny(s, plan, H, W, TOP, ws, sm_count, &n_parts, st);
            if (rc != CAT_OK) return rc;
            return launch_lp_rows<__nv_bfloat16, __half, TOP>(s, plan, Hs, static_cast<const __nv_bfloat16*>(W), r0, rws, n_parts, ws,
                                                              labels, valid, top_k, logp, lse, entropy, top_ids, top_logp, st);
        }
        CUtensorMap tmH, tmZ;
        if (tmap_a(&tmH, Hs, rws, s->d, s->ldH) != CAT_OK) return CAT_ERR_CUDA;
        if (TOP && tmap_out(&tmZ, ws + plan.off_z, rws, s->V, plan.ldz) != CAT_OK) return CAT_ERR_CUDA;
        const tc::Sched sched = make_sched(rws, s->V, s->d, S, band_tiles(s->d), 0);
        typename tc::EpiLp<TOP>::Params ep;
        ep.part_m = part_m; ep.part_l = part_l; ep.part_u = part_u; ep.part_id = reinterpret_cast<int*>(ws + plan.off_id); ep.part_stride = plan.Ts;
        ep.gmax = reinterpret_cast<float*>(ws + plan.off_g); ep.ld_g = plan.ld_g;
        ep.T = static_cast<int>(rws); ep.V = static_cast<int>(s->V);
        const __nv_bfloat16* Wb = static_cast<const __nv_bfloat16*>(W);
        int* w_sq = reinterpret_cast<int*>(ws + kNormOffset);
        const bool norms = TOP && r0 == 0, beside = rws >= kNormsBesideRows;
        int rc = norms && !beside ? launch_norms<false>(s, Wb, S, w_sq, sm_count, st) : CAT_OK;
        if (rc != CAT_OK) return rc;
        rc = launch_tc<0, 0, tc::EpiLp<TOP>>(tmH, tmW, sched, ep, reinterpret_cast<int*>(ws), sm_count, st, TOP ? &tmZ : nullptr);
        if (rc == CAT_OK && norms && beside) rc = launch_norms<true>(s, Wb, S, w_sq, sm_count, st);
        if (rc != CAT_OK) return rc;
        return launch_lp_rows<__nv_bfloat16, __half, TOP>(s, plan, Hs, Wb, r0, rws, S, ws, labels, valid,
                                                          top_k, logp, lse, entropy, top_ids, top_logp, st);
    }
    const float* Hs = static_cast<const float*>(H) + r0 * s->ldH;
    f32::Operands op;
    op.A = Hs; op.sAm = s->ldH; op.sAk = 1; op.B = static_cast<const float*>(W); op.sBk = 1; op.sBn = s->ldW;
    op.M = static_cast<int>(rws); op.N = static_cast<int>(s->V); op.Kd = static_cast<int>(s->d); op.n_groups = S;
    f32::EpiParams ep;
    memset(&ep, 0, sizeof(ep));
    ep.part_m = part_m; ep.part_l = part_l; ep.part_u = part_u; ep.part_id = reinterpret_cast<int*>(ws + plan.off_id); ep.V = static_cast<int>(s->V);
    if (TOP) {
        ep.zs = reinterpret_cast<float*>(ws + plan.off_z); ep.ld_z = plan.ldz;
        ep.gmax = reinterpret_cast<float*>(ws + plan.off_g); ep.ld_g = plan.ld_g;
        if (r0 == 0) ep.w_sq = reinterpret_cast<int*>(ws + kNormOffset);
    }
    const dim3 grid(static_cast<unsigned>(cdiv(rws, f32::TM)), static_cast<unsigned>(S));
    f32::gemm_kernel<f32::FWD, true, true><<<grid, f32::THREADS, 0, st>>>(op, ep);
    if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
    return launch_lp_rows<float, float, TOP>(s, plan, Hs, static_cast<const float*>(W), r0, rws, S, ws, labels, valid, top_k, logp, lse,
                                             entropy, top_ids, top_logp, st);
}

// ------------------------------------------------------------------------------ distillation from top logits
int check_topk_kd(const cat_topk_kd_desc* k) {
    if (!k) return CAT_ERR_NULL;
    if (k->L <= 0 || k->L >= (1ll << 31) || k->k < 1 || k->k > CAT_TOPK_MAX || k->ld < k->k) return CAT_ERR_SHAPE;
    if (!(k->beta >= 0.f && k->beta <= 3.0e38f)) return CAT_ERR_SHAPE;
    if (k->renormalize != 0 && k->renormalize != 1) return CAT_ERR_SHAPE;
    return CAT_OK;
}

// Row slabs of the fp32 operators: the logits of whole draft blocks, as many as the cap allows.
FusedPlan plan_fused_f32(const cat_shape* s) {
    FusedPlan f;
    memset(&f, 0, sizeof(f));
    f.ldz = cdiv(s->V, 8) * 8;
    const long long mib = s->slab_mib > 0 ? s->slab_mib : kDefaultFusedSlabMiB;
    long long cap = (mib << 20) / (f.ldz * 4) / s->K * s->K;
    const long long least = cdiv(f32::TM, s->K) * s->K;          // whole blocks that fill a row tile
    if (cap < least) cap = least;
    f.Ts = cap < s->T ? cap : s->T;
    f.n_slabs = static_cast<int>(cdiv(s->T, f.Ts));
    f.warp_scan = s->K <= 32 && (s->K & (s->K - 1)) == 0;
    f.S_max = 1;
    for (long long r0 = 0; r0 < s->T; r0 += f.Ts) {
        const long long rws = (s->T - r0) < f.Ts ? (s->T - r0) : f.Ts;
        const int S = f32_splits(rws, s->V);
        if (S > f.S_max) f.S_max = S;
        f.n_row_ctas += static_cast<int>(cdiv(f.warp_scan ? rws : rws / s->K, rows::ROW_THREADS));
    }
    size_t off = kHeaderBytes;
    f.off_part_m = off;   off = align256(off + sizeof(float) * f.S_max * f.Ts);
    f.off_part_l = off;   off = align256(off + sizeof(float) * f.S_max * f.Ts);
    f.off_z_label = off;  off = align256(off + sizeof(float) * s->T);
    f.off_row_ce = off;   off = align256(off + sizeof(float) * s->T);
    f.off_partials = off; off = align256(off + sizeof(rows::CtaPartial) * f.n_row_ctas);
    f.off_ref = off;      off = align256(off + sizeof(float) * s->T);
    f.off_hs = off;       off = align256(off + sizeof(float) * static_cast<size_t>(f.Ts) * static_cast<size_t>(s->d));
    f.off_z = off;        off = align256(off + sizeof(float) * static_cast<size_t>(f.Ts) * f.ldz);
    f.total = off;
    return f;
}

struct TkPlan {
    FusedPlan f;
    int ld_zt;             // k + 1 logits per row: the list's and the label's
    size_t off_valid, off_zt, off_kd_row, off_id, off_u, off_m1, off_l1, off_part, total;
};

TkPlan plan_tk(const cat_shape* s, int k) {
    TkPlan p;
    if (s->in_dtype == CAT_BF16) {
        p.f = plan_fused(s, false);
    } else {
        p.f = plan_fused_f32(s);
    }
    p.ld_zt = k + 1;
    size_t off = align256(p.f.total);
    p.off_valid = off;  off = align256(off + static_cast<size_t>(s->T));
    p.off_zt = off;     off = align256(off + sizeof(float) * static_cast<size_t>(p.f.Ts) * p.ld_zt);
    p.off_kd_row = off; off = align256(off + sizeof(float) * s->T);
    p.off_id = off;     off = align256(off + sizeof(int) * p.f.S_max * (s->in_dtype == CAT_BF16 ? s->T : 1));
    p.off_u = off;      off = align256(off + sizeof(float) * p.f.S_max * (s->in_dtype == CAT_BF16 ? s->T : 1));
    p.off_m1 = off;     off = align256(off + sizeof(float) * s->T);
    p.off_l1 = off;     off = align256(off + sizeof(float) * s->T);
    p.off_part = off;
    if (s->in_dtype == CAT_BF16) {
        const long long lo = lo_rows_of(s->T);
        const size_t full = dh_part_bytes(lo > 0 ? 2 * lo : p.f.Ts < s->T ? p.f.Ts : s->T, s->d, s->V, lo > 0);
        const size_t rest = dh_part_bytes(s->T - (p.f.n_slabs - 1) * p.f.Ts, s->d, s->V);
        off += full > rest ? full : rest;
    } else {
        off += kF32PartBytes;
    }
    p.total = off;
    return p;
}

// dH[r0 : r0 + rws, :] = scale dz W and dW (+)= scale dz^T Hw of one row slab; Hw: the slab's rows of H with pitch ldHw.  lo > 0: dz in
// two terms (kTwoTermRows).  rest, sparse: what the rounding left of the labels' entries (kLabelRestRows), without scale.  dw_sum: the sum over
// the slabs goes there ([V, d], fp32) and dW is left alone.
int slab_grads(const cat_shape* s, const FusedPlan& f, const void* W, const void* Hw, long long ldHw, void* zs, uint8_t* ws, long long r0,
               long long rws, long long lo, bool first, bool last, const float* scale, float* part, void* dH, void* dW, int accumulate_dW, int sm_count,
               cudaStream_t st, const lp::LabelRest* rest = nullptr, const tc::SparseTerms<true>* sparse = nullptr,
               float* dw_sum = nullptr) {
    const int V = static_cast<int>(s->V), d = static_cast<int>(s->d), R = static_cast<int>(rws);
    if (s->in_dtype != CAT_BF16) {
        const int rc = launch_f32_dh(static_cast<float*>(zs), f.ldz, static_cast<const float*>(W), s->ldW, R, d, V, scale,
                                     static_cast<float*>(dH) + r0 * s->ldH, s->ldH, false, part, st);
        if (rc != CAT_OK) return rc;
        return launch_f32_dw(static_cast<float*>(zs), f.ldz, static_cast<const float*>(Hw), ldHw, V, d, R, scale,
                             dw_sum ? dw_sum : static_cast<float*>(dW), dw_sum ? s->d : s->ldW, !first || (accumulate_dW && !dw_sum), part, st);
    }
    int* status = reinterpret_cast<int*>(ws);
    CUtensorMap tmZ_k, tmZ_mn, tmW_mn, tmH_mn;
    const long long all = lo > 0 ? 2 * lo : rws;         // rows of dz, with its second terms
    if (tmap_a(&tmZ_k, zs, all, s->V, f.ldz) != CAT_OK || tmap_mn_major(&tmZ_mn, zs, all, s->V, f.ldz) != CAT_OK ||
        tmap_mn_major(&tmW_mn, W, s->V, s->d, s->ldW) != CAT_OK || tmap_mn_major(&tmH_mn, Hw, all, s->d, ldHw) != CAT_OK)
        return CAT_ERR_CUDA;
    const int rc = launch_dh(tmZ_k, tmW_mn, rws, s->d, s->V, scale, static_cast<__nv_bfloat16*>(dH) + r0 * s->ldH, s->ldH, part, status,
                             sm_count, st, lo, rest);
    if (rc != CAT_OK) return rc;
    tc::EpiOut::Params ep;
    memset(&ep, 0, sizeof(ep));
    ep.alpha = scale; ep.M = V; ep.N = d;
    float* dw_acc = reinterpret_cast<float*>(ws + f.off_dw_acc);
    if (dw_sum || s->dW_dtype == CAT_F32) {
        ep.out_f32 = dw_sum ? dw_sum : static_cast<float*>(dW); ep.ld_out = dw_sum ? s->d : s->ldW;
        if (!first || (accumulate_dW && !dw_sum)) { ep.add_f32 = ep.out_f32; ep.ld_add = ep.ld_out; }
    } else {        // bf16 dW: several slabs are summed in fp32 scratch and rounded once at the end
        if (first) {
            if (accumulate_dW) { ep.add_bf16 = static_cast<const __nv_bfloat16*>(dW); ep.ld_add = s->ldW; }
        } else {
            ep.add_f32 = dw_acc; ep.ld_add = s->d;
        }
        if (last) { ep.out_bf16 = static_cast<__nv_bfloat16*>(dW); ep.ld_out = s->ldW; }
        else { ep.out_f32 = dw_acc; ep.ld_out = s->d; }
    }
    const tc::Sched sched = make_sched(s->V, s->d, all, 0, 1, 1);
    if (sparse == nullptr) return launch_out<1, 1>(tmZ_mn, tmH_mn, sched, ep, status, sm_count, st);
    tc::EpiOutT<true>::Params sp;
    memset(&sp, 0, sizeof(sp));
    static_cast<tc::SparseTerms<true>&>(sp) = *sparse;
    sp.add_f32 = ep.add_f32; sp.add_bf16 = ep.add_bf16; sp.out_f32 = ep.out_f32; sp.out_bf16 = ep.out_bf16;
    sp.ld_add = ep.ld_add; sp.ld_out = ep.ld_out; sp.M = ep.M; sp.N = ep.N; sp.alpha = ep.alpha;
    return launch_out<1, 1, true>(tmZ_mn, tmH_mn, sched, sp, status, sm_count, st);
}

template <class TI>
int tk_core(const cat_shape* s, const cat_topk_kd_desc* desc, const TkPlan& plan, const TI* H, const TI* W, const int64_t* labels,
            const uint8_t* valid, const int64_t* top_ids, const float* top_logp, const int64_t* block_start, const float* conf_ext,
            const float* grad_loss, float* loss, float* lse, float* conf, float* weight, cat_stats* stats, void* dH, void* dW,
            int accumulate_dW, uint8_t* ws, int sm_count, cudaStream_t st) {
    constexpr bool BF16 = sizeof(TI) == 2;
    const FusedPlan& f = plan.f;
    int* status = reinterpret_cast<int*>(ws);
    float* scale = reinterpret_cast<float*>(ws + kScaleOffset);
    int* n_bad = reinterpret_cast<int*>(ws + kBadOffset);
    float* part_m = reinterpret_cast<float*>(ws + f.off_part_m);
    float* part_l = reinterpret_cast<float*>(ws + f.off_part_l);
    float* z_label = reinterpret_cast<float*>(ws + f.off_z_label);
    float* row_ce = reinterpret_cast<float*>(ws + f.off_row_ce);
    float* ref = reinterpret_cast<float*>(ws + f.off_ref);
    float* zt = reinterpret_cast<float*>(ws + plan.off_zt);
    float* kd_row = reinterpret_cast<float*>(ws + plan.off_kd_row);
    int* part_id = reinterpret_cast<int*>(ws + plan.off_id);
    float* part_u = reinterpret_cast<float*>(ws + plan.off_u);
    float* m1 = reinterpret_cast<float*>(ws + plan.off_m1);
    float* l1 = reinterpret_cast<float*>(ws + plan.off_l1);
    unsigned char* ok = ws + plan.off_valid;
    TI* Hz = reinterpret_cast<TI*>(ws + f.off_hs);
    rows::CtaPartial* partials = reinterpret_cast<rows::CtaPartial*>(ws + f.off_partials);
    void* zs = ws + f.off_z;
    const int T = static_cast<int>(s->T), V = static_cast<int>(s->V), d = static_cast<int>(s->d), K = s->K;
    const long long* y = reinterpret_cast<const long long*>(labels);
    tk::Lists lists;
    lists.ids = reinterpret_cast<const long long*>(top_ids); lists.logp = top_logp;
    lists.block_start = reinterpret_cast<const long long*>(block_start);
    lists.ld = desc->ld; lists.k = desc->k; lists.K = K; lists.V = V; lists.renorm = desc->renormalize;

    CUtensorMap tmW_k;
    if (BF16 && tmap_b(&tmW_k, W, s->V, s->d, s->ldW) != CAT_OK) return CAT_ERR_CUDA;
    tk::begin_kernel<<<1, 1024, 0, st>>>(y, valid, lists.block_start, T, K, V, desc->L, grad_loss, ok, scale, n_bad, status,
                                         static_cast<int>(kHeaderBytes / sizeof(int)));
    if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
    int cta0 = 0;
    for (int sl = 0; sl < f.n_slabs; ++sl) {
        const long long r0 = static_cast<long long>(sl) * f.Ts;
        const long long rws = (s->T - r0) < f.Ts ? (s->T - r0) : f.Ts;
        const int S = head_splits(s, rws);
        const TI* Hs = H + r0 * s->ldH;
        const long long lo = BF16 ? lo_rows_of(s->T) : 0;
        const unsigned grid_rows = static_cast<unsigned>(lo > 0 ? lo : rws);
        tk::gather_kernel<TI><<<grid_rows, tk::THREADS, 0, st>>>(Hs, s->ldH, W, s->ldW, d, y, ok, lists, r0, static_cast<int>(rws),
                                                                 static_cast<int>(lo), zt, plan.ld_zt, ref, Hz);
        if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
        rows::RowParams rp;
        memset(&rp, 0, sizeof(rp));
        tk::MergeParams<TI> mp;
        if (BF16) {
            CUtensorMap tmH_k, tmZ_out;
            if (tmap_a(&tmH_k, Hs, rws, s->d, s->ldH) != CAT_OK || tmap_out(&tmZ_out, zs, rws, s->V, f.ldz) != CAT_OK) return CAT_ERR_CUDA;
            tc::EpiFwdRef::Params ep;
            ep.labels = y + r0; ep.part_m = part_m + r0; ep.part_l = part_l + r0; ep.z_label = z_label + r0; ep.ref = ref + r0;
            ep.part_u = part_u + r0; ep.part_id = part_id + r0; ep.part_stride = T; ep.T = static_cast<int>(rws); ep.V = V;
            const int rc = launch_tc<0, 0, tc::EpiFwdRef>(tmH_k, tmW_k, make_sched(rws, s->V, s->d, S, band_tiles(s->d), 0), ep, status,
                                                          sm_count, st, &tmZ_out);
            if (rc != CAT_OK) return rc;
            mp.part_m = ep.part_m; mp.part_l = ep.part_l; mp.part_u = ep.part_u; mp.part_id = ep.part_id; mp.part_stride = T;
        } else {
            f32::Operands op;
            op.A = reinterpret_cast<const float*>(Hs); op.sAm = s->ldH; op.sAk = 1;
            op.B = reinterpret_cast<const float*>(W); op.sBk = 1; op.sBn = s->ldW;
            op.M = static_cast<int>(rws); op.N = V; op.Kd = d; op.n_groups = S;
            f32::EpiParams ep;
            memset(&ep, 0, sizeof(ep));
            ep.labels = y + r0; ep.part_m = part_m; ep.part_l = part_l; ep.z_label = z_label + r0; ep.V = V;
            ep.zs = static_cast<float*>(zs); ep.ld_z = f.ldz;
            f32::gemm_kernel<f32::FWD, true, true><<<dim3(static_cast<unsigned>(cdiv(rws, f32::TM)), static_cast<unsigned>(S)), f32::THREADS, 0, st>>>(op, ep);
            mp.part_m = part_m; mp.part_l = part_l; mp.part_u = nullptr; mp.part_id = nullptr; mp.part_stride = rws;
        }
        mp.S = S; mp.H = Hs; mp.W = W; mp.ldH = s->ldH; mp.ldW = s->ldW; mp.d = d; mp.V = V; mp.labels = y + r0; mp.valid = ok + r0;
        mp.z_exact = zt + lists.k; mp.ld_exact = plan.ld_zt; mp.z_label = z_label + r0; mp.m1 = m1 + r0; mp.l1 = l1 + r0;
        mp.rows = static_cast<int>(rws);
        tk::merge_kernel<TI><<<static_cast<unsigned>(cdiv(rws, tk::WARPS)), tk::THREADS, 0, st>>>(mp);
        if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
        rp.part_m = m1 + r0; rp.part_l = l1 + r0; rp.part_stride = rws;
        // lse, confidence (Eq. 9), CAT weights (Eq. 10), cross-entropy partials of the slab's blocks
        rp.z_label = z_label + r0; rp.labels = y + r0; rp.valid = ok + r0; rp.conf_ext = conf_ext ? conf_ext + r0 : nullptr;
        rp.lse = lse + r0; rp.conf = conf + r0; rp.weight = weight + r0; rp.row_ce = row_ce + r0; rp.partials = partials + cta0;
        rp.T = static_cast<int>(rws); rp.V = V; rp.K = K; rp.S = 1;
        rp.fixed_decay = s->weight_mode == CAT_WEIGHT_FIXED_DECAY; rp.gamma = s->decay_gamma;
        int n_ctas;
        if (f.warp_scan) {
            n_ctas = static_cast<int>(cdiv(rws, rows::ROW_THREADS));
            rows::row_kernel<true><<<n_ctas, rows::ROW_THREADS, 0, st>>>(rp);
        } else {
            n_ctas = static_cast<int>(cdiv(rws / K, rows::ROW_THREADS));
            rows::row_kernel<false><<<static_cast<unsigned>(cdiv(rws, rows::ROW_THREADS)), rows::ROW_THREADS, 0, st>>>(rp);
            rows::block_scan_kernel<<<n_ctas, rows::ROW_THREADS, 0, st>>>(rp);
        }
        cta0 += n_ctas;
        tk::dz_kernel<!BF16><<<grid_rows, tk::THREADS, 0, st>>>(Hs, s->ldH, W, s->ldW, d, m1, zs, f.ldz, y, ok, lists, r0, static_cast<int>(rws), static_cast<int>(lo), lse,
                                                                weight, zt, plan.ld_zt, ref, desc->beta, kd_row, V);
        if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
        const int rc = slab_grads(s, f, W, Hz, s->d, zs, ws, r0, rws, lo, sl == 0, sl == f.n_slabs - 1, scale, reinterpret_cast<float*>(ws + plan.off_part), dH, dW, accumulate_dW,
                                  sm_count, st);
        if (rc != CAT_OK) return rc;
    }
    tk::end_kernel<<<1, 1024, 0, st>>>(partials, cta0, T / K, kd_row, T, desc->beta, loss, reinterpret_cast<rows::StatsOut*>(stats), n_bad, status);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}

// ------------------------------------------------------------------------------ gradients of the log probabilities
// By row slabs, as cat_topk_kd_loss_fwd_bwd: per slab recomputed logits -> dz, the closing entries (which need whole rows), dH of the slab's rows, dW
// summed over the slabs.
struct LpBwdPlan {
    FusedPlan f;
    long long lo;          // rows before the second terms of dz, or 0
    bool rest;             // labels' entries of dz to more than bf16 (kLabelRestRows)
    size_t off_rest, off_part, off_dw_sum, total;
};

LpBwdPlan plan_lp_bwd(const cat_shape* s) {
    LpBwdPlan p;
    const bool bf16 = s->in_dtype == CAT_BF16;
    p.f = bf16 ? plan_fused(s, false) : plan_fused_f32(s);
    p.lo = bf16 ? lo_rows_of(s->T) : 0;                  // a slab is never lower than 128 rows
    p.rest = bf16 && p.lo == 0 && s->T <= kLabelRestRows;
    size_t off = align256(p.f.total);
    p.off_rest = off;  if (p.rest) off = align256(off + 4 * sizeof(float) * static_cast<size_t>(s->T));
    p.off_part = off;
    if (bf16) {
        const size_t full = dh_part_bytes(p.lo > 0 ? 2 * p.lo : p.f.Ts < s->T ? p.f.Ts : s->T, s->d, s->V, p.lo > 0 || p.rest);
        const size_t last = dh_part_bytes(s->T - (p.f.n_slabs - 1) * p.f.Ts, s->d, s->V, p.rest);
        off += full > last ? full : last;
    } else {
        off += kF32PartBytes;
    }
    // what several slabs add to a dW that is accumulated into: summed first, so that dW takes one rounding whatever the slabs
    off = align256(off);
    p.off_dw_sum = p.f.dw_acc ? p.f.off_dw_acc : off;
    if (p.f.n_slabs > 1 && !p.f.dw_acc) off = align256(off + sizeof(float) * static_cast<size_t>(s->V) * static_cast<size_t>(s->d));
    p.total = off;
    return p;
}

struct LpGrads {
    const int64_t* labels;
    const uint8_t* valid;
    const float *lse, *entropy, *grad_logp, *grad_entropy;
};

template <class TI>
int lp_bwd_core(const cat_shape* s, const LpBwdPlan& plan, const TI* H, const TI* W, const LpGrads& a, TI* dH, void* dW, int accumulate_dW,
                uint8_t* ws, int sm_count, cudaStream_t st) {
    constexpr bool BF16 = sizeof(TI) == 2;
    const FusedPlan& f = plan.f;
    int* status = reinterpret_cast<int*>(ws);
    void* dz = ws + f.off_z;
    TI* Hz = reinterpret_cast<TI*>(ws + f.off_hs);
    float* part_sum = reinterpret_cast<float*>(ws + f.off_part_m);
    int* part_col = reinterpret_cast<int*>(ws + f.off_part_l);
    float* dz_label = reinterpret_cast<float*>(ws + f.off_z_label);
    int* closing = reinterpret_cast<int*>(ws + f.off_ref);
    const int d = static_cast<int>(s->d), V = static_cast<int>(s->V);
    const bool copy_H = a.valid != nullptr || plan.lo > 0;
    float* dw_sum = accumulate_dW && f.n_slabs > 1 ? reinterpret_cast<float*>(ws + plan.off_dw_sum) : nullptr;
    CUtensorMap tmW_k;
    if (BF16 && tmap_b(&tmW_k, W, s->V, s->d, s->ldW) != CAT_OK) return CAT_ERR_CUDA;
    for (int sl = 0; sl < f.n_slabs; ++sl) {
        const long long r0 = static_cast<long long>(sl) * f.Ts;
        const long long rws = (s->T - r0) < f.Ts ? (s->T - r0) : f.Ts;
        const long long all = plan.lo > 0 ? 2 * plan.lo : rws;             // rows of dz, with its second terms
        const TI* Hs = H + r0 * s->ldH;
        const long long* labels = a.labels ? reinterpret_cast<const long long*>(a.labels) + r0 : nullptr;
        const uint8_t* valid = a.valid ? a.valid + r0 : nullptr;
        const float *lse = a.lse + r0, *entropy = a.entropy ? a.entropy + r0 : nullptr;
        const float *gl = a.grad_logp ? a.grad_logp + r0 : nullptr, *ge = a.grad_entropy ? a.grad_entropy + r0 : nullptr;
        if (copy_H) {
            lp::copy_rows_kernel<TI><<<static_cast<unsigned>(all), lp::THREADS, 0, st>>>(Hs, s->ldH, d, static_cast<int>(rws), valid,
                                                                                         static_cast<int>(plan.lo), Hz);
            if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
        }
        lp::LabelRest rest{nullptr, labels, nullptr, s->ldW};
        tc::SparseTerms<true> sparse{};
        if (BF16) {
            const int S = fwd_splits(rws, s->V);
            CUtensorMap tmH_k, tmDz_out;
            if (tmap_a(&tmH_k, Hs, rws, s->d, s->ldH) != CAT_OK || tmap_out(&tmDz_out, dz, all, s->V, f.ldz) != CAT_OK) return CAT_ERR_CUDA;
            tc::EpiDzLp::Params zp;
            zp.labels = labels; zp.valid = valid; zp.lse = lse; zp.entropy = entropy; zp.grad_logp = gl; zp.grad_entropy = ge;
            zp.part_sum = part_sum; zp.part_col = part_col; zp.part_stride = s->T; zp.dz_label = dz_label;
            zp.T = static_cast<int>(rws); zp.V = V; zp.lo_rows = static_cast<int>(plan.lo);
            const int rc = launch_tc<0, 0, tc::EpiDzLp>(tmH_k, tmW_k, make_sched(rws, s->V, s->d, S, band_tiles(s->d), 0), zp, status, sm_count, st,
                                                        &tmDz_out);
            if (rc != CAT_OK) return rc;
            lp::CloseParams cp;
            memset(&cp, 0, sizeof(cp));
            cp.labels = labels; cp.valid = valid; cp.grad_logp = gl; cp.part_sum = part_sum; cp.part_col = part_col; cp.part_stride = s->T; cp.S = S;
            cp.dz_label = dz_label; cp.dz = static_cast<__nv_bfloat16*>(dz); cp.ldz = f.ldz;
            cp.T = static_cast<int>(rws); cp.V = V; cp.lo = static_cast<int>(plan.lo);
            if (plan.rest && gl) {
                cp.rest = reinterpret_cast<float*>(ws + plan.off_rest);
                cp.key = reinterpret_cast<int*>(cp.rest + s->T); cp.from = cp.key + s->T; cp.coef = cp.rest + 3 * s->T;
                rest.rest = cp.rest; rest.W = reinterpret_cast<const __nv_bfloat16*>(W);
                sparse.key = cp.key; sparse.from = cp.from; sparse.coef = cp.coef;
                sparse.src = reinterpret_cast<const __nv_bfloat16*>(Hs); sparse.ld_src = s->ldH; sparse.n = static_cast<int>(rws);
            }
            lp::close_kernel<<<static_cast<unsigned>(cdiv(rws, lp::WARPS)), lp::THREADS, 0, st>>>(cp);
        } else {
            f32::Operands op;
            f32::EpiParams ep;
            memset(&ep, 0, sizeof(ep));
            op.A = reinterpret_cast<const float*>(Hs); op.sAm = s->ldH; op.sAk = 1;
            op.B = reinterpret_cast<const float*>(W); op.sBk = 1; op.sBn = s->ldW;
            op.M = static_cast<int>(rws); op.N = V; op.Kd = d;
            op.n_groups = static_cast<int>(cdiv(V, f32::TN) < 65535 ? cdiv(V, f32::TN) : 65535);       // a grid's second extent ends there
            ep.labels = labels; ep.valid = valid; ep.lse = lse; ep.entropy = entropy; ep.grad_logp = gl; ep.grad_entropy = ge;
            ep.closing = closing; ep.dz = static_cast<float*>(dz); ep.ld_dz = f.ldz; ep.V = V;
            if (cudaMemsetAsync(closing, 0xFF, sizeof(int) * rws, st) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
            f32::gemm_kernel<f32::DZ, true, true><<<dim3(static_cast<unsigned>(cdiv(rws, f32::TM)), static_cast<unsigned>(op.n_groups)), f32::THREADS, 0, st>>>(op, ep);
            f32::close_kernel<<<static_cast<unsigned>(rws), 256, 0, st>>>(static_cast<float*>(dz), f.ldz, V, closing);
        }
        if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
        const int rc = slab_grads(s, f, W, copy_H ? Hz : Hs, copy_H ? s->d : s->ldH, dz, ws, r0, rws, plan.lo, sl == 0, sl == f.n_slabs - 1, nullptr,
                                  reinterpret_cast<float*>(ws + plan.off_part), dH, dW, accumulate_dW, sm_count, st, rest.rest ? &rest : nullptr,
                                  sparse.key ? &sparse : nullptr, dw_sum);
        if (rc != CAT_OK) return rc;
    }
    if (dw_sum) {
        const bool four = s->d % 4 == 0 && s->ldW % 4 == 0;
        const long long ctas = cdiv(s->V * (four ? s->d / 4 : s->d), lp::THREADS * 4);
        const unsigned grid = static_cast<unsigned>(ctas < 65535 ? ctas : 65535);
        if (s->dW_dtype == CAT_BF16) lp::add_sum_kernel<4><<<grid, lp::THREADS, 0, st>>>(dw_sum, s->V, d, static_cast<__nv_bfloat16*>(dW), s->ldW);
        else if (four) lp::add_sum_kernel<4><<<grid, lp::THREADS, 0, st>>>(dw_sum, s->V, d, static_cast<float*>(dW), s->ldW);
        else lp::add_sum_kernel<1><<<grid, lp::THREADS, 0, st>>>(dw_sum, s->V, d, static_cast<float*>(dW), s->ldW);
        if (cudaGetLastError() != cudaSuccess) return CAT_ERR_CUDA;
    }
    return CAT_OK;
}

}  // namespace

extern "C" {

size_t cat_logprob_workspace_bytes(const cat_shape* shape, int top_k, int pass) {
    if (!shape) return 0;
    cat_shape one = per_position_shape(shape);
    one.dW_dtype = shape->dW_dtype;
    if (check_shape(&one) != CAT_OK || top_k < 0 || top_k > CAT_TOPK_MAX) return 0;
    if (pass == 0) return plan_lp(&one, top_k).total;
    if (pass == 1) return plan_lp_bwd(&one).total;
    return 0;
}

int cat_logprob_fwd(const cat_shape* shape, const void* H, const void* W, const int64_t* labels, const uint8_t* valid, int32_t top_k,
                    float* logp, float* lse, float* entropy, int64_t* top_ids, float* top_logp, void* workspace,
                    size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !H || !W || !lse || !entropy || (labels == nullptr) != (logp == nullptr)) return CAT_ERR_NULL;
    const cat_shape one = per_position_shape(shape);
    const int sc = check_shape(&one);
    if (sc != CAT_OK) return sc;
    if (top_k < 0 || top_k > CAT_TOPK_MAX) return CAT_ERR_SHAPE;
    if (top_k > 0 && (!top_ids || !top_logp)) return CAT_ERR_NULL;
    const size_t in_al = one.in_dtype == CAT_BF16 ? 16 : 4;
    if (misaligned(H, in_al) || misaligned(W, in_al) || misaligned(labels, 8) || misaligned(logp, 4) || misaligned(lse, 4) ||
        misaligned(entropy, 4) || misaligned(top_ids, 8) || misaligned(top_logp, 4))
        return CAT_ERR_ALIGN;
    const LpPlan plan = plan_lp(&one, top_k);
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.total) return CAT_ERR_WORKSPACE;
    int sm_count = 0;
    const int dc = check_device(&sm_count);
    if (dc != CAT_OK) return dc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    CUtensorMap tmW;
    memset(&tmW, 0, sizeof(tmW));
    if (one.in_dtype == CAT_BF16 && tmap_b(&tmW, W, one.V, one.d, one.ldW) != CAT_OK) return CAT_ERR_CUDA;
    if (cudaMemsetAsync(ws, 0, kHeaderBytes, st) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
    for (int sl = 0; sl < plan.n_slabs; ++sl) {
        const long long r0 = static_cast<long long>(sl) * plan.Ts;
        const long long rws = (one.T - r0) < plan.Ts ? (one.T - r0) : plan.Ts;
        const int rc = top_k > 0 ? lp_slab<true>(&one, plan, tmW, H, W, r0, rws, ws, labels, valid, top_k, logp, lse, entropy, top_ids,
                                                 top_logp, sm_count, st)
                                 : lp_slab<false>(&one, plan, tmW, H, W, r0, rws, ws, labels, valid, 0, logp, lse, entropy, nullptr,
                                                  nullptr, sm_count, st);
        if (rc != CAT_OK) return rc;
    }
    return CAT_OK;
}

int cat_logprob_bwd(const cat_shape* shape, const void* H, const void* W, const int64_t* labels, const uint8_t* valid, const float* lse,
                    const float* entropy, const float* grad_logp, const float* grad_entropy, void* dH, void* dW, int accumulate_dW,
                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !H || !W || !lse || !dH || !dW || (grad_logp && !labels) || (grad_entropy && !entropy)) return CAT_ERR_NULL;
    cat_shape one = per_position_shape(shape);
    one.dW_dtype = shape->dW_dtype;
    const int sc = check_shape(&one);
    if (sc != CAT_OK) return sc;
    const bool bf16 = one.in_dtype == CAT_BF16;
    const size_t in_al = bf16 ? 16 : 4;
    if (misaligned(H, in_al) || misaligned(W, in_al) || misaligned(dH, in_al) || misaligned(dW, 16) || misaligned(labels, 8) ||
        misaligned(lse, 4) || misaligned(entropy, 4) || misaligned(grad_logp, 4) || misaligned(grad_entropy, 4))
        return CAT_ERR_ALIGN;
    const LpBwdPlan plan = plan_lp_bwd(&one);
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.total) return CAT_ERR_WORKSPACE;
    int sm_count = 0;
    const int dc = check_device(&sm_count);
    if (dc != CAT_OK) return dc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (cudaMemsetAsync(ws, 0, kHeaderBytes, st) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
    LpGrads a;
    a.labels = labels; a.valid = valid; a.lse = lse; a.entropy = entropy; a.grad_logp = grad_logp; a.grad_entropy = grad_entropy;
    return bf16 ? lp_bwd_core<__nv_bfloat16>(&one, plan, static_cast<const __nv_bfloat16*>(H), static_cast<const __nv_bfloat16*>(W), a,
                                             static_cast<__nv_bfloat16*>(dH), dW, accumulate_dW, ws, sm_count, st)
                : lp_bwd_core<float>(&one, plan, static_cast<const float*>(H), static_cast<const float*>(W), a, static_cast<float*>(dH), dW,
                                     accumulate_dW, ws, sm_count, st);
}

size_t cat_topk_kd_workspace_bytes(const cat_shape* shape, const cat_topk_kd_desc* desc) {
    if (check_shape(shape) != CAT_OK || check_topk_kd(desc) != CAT_OK) return 0;
    return plan_tk(shape, desc->k).total;
}

int cat_topk_kd_loss_fwd_bwd(const cat_shape* shape, const cat_topk_kd_desc* desc, const void* H, const void* W, const int64_t* labels,
                             const uint8_t* valid, const int64_t* top_ids, const float* top_logp, const int64_t* block_start,
                             const float* conf_ext, const float* grad_loss, float* loss, float* lse, float* conf, float* weight,
                             cat_stats* stats, void* dH, void* dW, int accumulate_dW, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
    if (!shape || !desc || !H || !W || !labels || !top_ids || !top_logp || !loss || !lse || !conf || !weight || !dH || !dW)
        return CAT_ERR_NULL;
    int rc = check_shape(shape);
    if (rc == CAT_OK) rc = check_topk_kd(desc);
    if (rc != CAT_OK) return rc;
    const size_t in_al = shape->in_dtype == CAT_BF16 ? 16 : 4;
    if (misaligned(H, in_al) || misaligned(W, in_al) || misaligned(dH, in_al) || misaligned(dW, 16) || misaligned(labels, 8) ||
        misaligned(top_ids, 8) || misaligned(top_logp, 4) || misaligned(block_start, 8) || misaligned(conf_ext, 4) ||
        misaligned(grad_loss, 4) || misaligned(loss, 4) || misaligned(lse, 4) || misaligned(conf, 4) || misaligned(weight, 4) ||
        misaligned(stats, 8))
        return CAT_ERR_ALIGN;
    const TkPlan plan = plan_tk(shape, desc->k);
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.total) return CAT_ERR_WORKSPACE;
    int sm_count = 0;
    rc = check_device(&sm_count);
    if (rc != CAT_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (shape->in_dtype == CAT_BF16)
        return tk_core<__nv_bfloat16>(shape, desc, plan, static_cast<const __nv_bfloat16*>(H), static_cast<const __nv_bfloat16*>(W), labels,
                                      valid, top_ids, top_logp, block_start, conf_ext, grad_loss, loss, lse, conf, weight, stats, dH, dW,
                                      accumulate_dW, ws, sm_count, st);
    return tk_core<float>(shape, desc, plan, static_cast<const float*>(H), static_cast<const float*>(W), labels, valid, top_ids, top_logp,
                          block_start, conf_ext, grad_loss, loss, lse, conf, weight, stats, dH, dW, accumulate_dW, ws, sm_count, st);
}

}  // extern "C"
