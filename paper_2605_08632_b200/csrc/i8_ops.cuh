// Host side of the operators on an 8-bit head: cat_i8_quantize, cat_i8_linear_fwd / _bwd and cat_i8_ce_fwd / _bwd.  Included at the end
// of cat_api.cu, whose planning and launch helpers it uses.
#pragma once
#include "i8_grad.cuh"
#include "i8_head.cuh"
#include "i8_skinny.cuh"

namespace {

constexpr size_t kMostOffset = 64;       // header: largest scale of the head, in i8::MOST_PARTS parts
static_assert(kMostOffset + sizeof(int) * i8::MOST_PARTS <= kClaimsOffset, "between the status and the claims");

enum I8Pass { kI8Linear = 0, kI8LinearBwd = 1, kI8Ce = 2, kI8CeBwd = 3 };

int check_i8(const cat_i8_shape* s, int pass) {
    if (!s) return CAT_ERR_NULL;
    if (s->T <= 0 || s->d <= 0 || s->V <= 0 || s->T >= (1ll << 31) || s->V >= (1ll << 31) || s->d > 65536) return CAT_ERR_SHAPE;
    if (s->ldX < s->d || s->ldW < s->d || s->slab_mib < 0) return CAT_ERR_SHAPE;
    if (s->x_dtype != CAT_BF16 && s->x_dtype != CAT_F32) return CAT_ERR_DTYPE;
    if (s->ldW % 16 != 0) return CAT_ERR_ALIGN;
    if (pass == kI8Linear || pass == kI8LinearBwd) {
        if (s->ldY < s->V) return CAT_ERR_SHAPE;
        if (s->y_dtype != CAT_BF16 && s->y_dtype != CAT_F32) return CAT_ERR_DTYPE;
        if (s->ldY % (s->y_dtype == CAT_BF16 ? 8 : 4) != 0) return CAT_ERR_ALIGN;
    }
    if (pass == kI8LinearBwd || pass == kI8CeBwd) {
        if (s->x_dtype != CAT_BF16 || (pass == kI8LinearBwd && s->y_dtype != CAT_BF16)) return CAT_ERR_DTYPE;
        if (s->lddX < s->d) return CAT_ERR_SHAPE;
        if (s->d % 8 != 0 || s->lddX % 8 != 0) return CAT_ERR_ALIGN;
    }
    return CAT_OK;
}

struct I8Plan {
    long long ldq;         // row pitch of the tokens' integers
    long long Ts;          // rows per slab
    long long ldz;
    int S;                 // splits of the vocabulary
    bool skinny;           // a few tokens: the kernel of i8_skinny.cuh
    bool widen;            // gradient: from a widened copy of the head; else widened on its way (i8_grad.cuh)
    size_t off_q, off_s, off_m, off_l, off_zy, off_factor, off_w16, off_part, off_z, total;
};

// How grad_kernel goes about its rows: units of columns per CTA, tiles of rows, and the parts its CTAs cut the vocabulary into: about 500 ns per slice of
// the longest part, four slices' worth for filling the ring, the parts written out and read back.
struct GradPlan {
    bool head_m;
    int units, tiles, n, num_kb, parts;
};
GradPlan plan_grad(long long rows, long long d, long long V) {
    GradPlan p;
    p.head_m = rows > 256;
    p.units = p.head_m ? 1 : 2;
    p.tiles = rows > 128 ? 2 : 1;
    p.n = rows > 128 && !p.head_m ? 128 : static_cast<int>(cdiv(cdiv(rows, p.tiles), 16) * 16);
    p.num_kb = static_cast<int>(cdiv(V, i8::GRAD_SLICE));
    const long long tiles = cdiv(d, i8::GRAD_COLS * p.units);
    const double out = static_cast<double>(rows) * static_cast<double>(d) * 3.0e-6;           // slices' worth of time per part
    double best_cost = 1e300;
    p.parts = 1;
    for (long long g = 1; g <= kPlanSMs && g <= p.num_kb; ++g) {
        const double cost = static_cast<double>(cdiv(tiles * g, kPlanSMs)) * static_cast<double>(cdiv(p.num_kb, g) + 4) + out * static_cast<double>(g);
        if (cost < best_cost) { best_cost = cost; p.parts = static_cast<int>(g); }
    }
    return p;
}
// Rows of a pass of it: one pass, or two of even height.
long long grad_pass_rows(long long rows) { return rows <= i8::GRAD_ROWS ? rows : cdiv(cdiv(rows, 2), 16) * 16; }

// Whether the gradient goes by a widened copy of the head: for more rows than two passes take, and where the copy is small against the rows' work.
// dX in us, copy / widened on its way.  One pass, heads of 1024 x 8000, 1024 x 32000, 2048 x 32000, 1024 x 151936: 16 rows 19 / 13, 42 / 21, 74 / 32, 154 / 61; 300 rows
// 20 / 20, 51 / 33, 95 / 52, 194 / 106; 400 rows 22 / 25, 54 / 39, 97 / 62, 198 / 125.  Two passes: 512 rows of 1024 x 8000 21 / 39, of 1024 x 32000 54 / 62, of
// 1024 x 50000 79 / 78, of 2048 x 32000 96 / 86, of 1024 x 151936 204 / 166; 600 rows of 2048 x 32000 109 / 103; 768 rows of 2048 x 32000 112 / 121, of 2048 x 64000
// 211 / 205, of 1024 x 151936 253 / 241; 860 rows of 1024 x 151936 294 / 259, of 4096 x 128000 1000 / 808.  Around the limit of 100 M weights, heads of 1024 x 80000,
// 1024 x 100000, 1024 x 120000: 656 rows 136 / 129, 169 / 158, 198 / 180; 704 rows 137 / 138, 171 / 170, 200 / 194; 768 rows 139 / 141, 173 / 174, 203 / 198; 832 rows of
// the first two 163 / 146, 203 / 180.  (The limit holds for 700 to 768 rows; below and above, smaller heads would gain 5 to 10 % from the two passes.)
bool use_widened_copy(long long rows, long long d, long long V) {
    const long long weights = d * V;
    return rows > 2 * i8::GRAD_ROWS || (rows > 640 && weights <= 100'000'000) || (rows > i8::GRAD_ROWS && weights <= 50'000'000) ||
           (rows > 300 && weights <= (1ll << 23));
}

size_t dx_part_bytes(long long rows, long long d, long long V, bool widen) {
    if (widen) return dh_part_bytes(rows, d, V);
    const long long most = grad_pass_rows(rows);
    const size_t full = sizeof(float) * plan_grad(most, d, V).parts * static_cast<size_t>(most) * d;
    const size_t rest = rows > most ? sizeof(float) * plan_grad(rows - most, d, V).parts * static_cast<size_t>(rows - most) * d : 0;
    return align256(full > rest ? full : rest);
}

I8Plan plan_i8(const cat_i8_shape* s, int pass) {
    I8Plan p;
    memset(&p, 0, sizeof(p));
    p.ldq = cdiv(s->d, 16) * 16;
    p.Ts = s->T;
    p.skinny = s->T <= i8::SKINNY_ROWS;
    p.widen = use_widened_copy(s->T, s->d, s->V);
    size_t off = kHeaderBytes;
    if (pass != kI8LinearBwd) {
        p.off_q = off; off = align256(off + static_cast<size_t>(s->T) * p.ldq);
        p.off_s = off; off = align256(off + sizeof(float) * s->T);
    }
    if (pass == kI8Ce) {
        p.S = fwd_splits(s->T, s->V);
        const size_t parts = p.skinny ? kPlanSMs : 2 * p.S;           // one per CTA, or two per split
        p.off_m = off; off = align256(off + sizeof(float) * parts * s->T);
        p.off_l = off; off = align256(off + sizeof(float) * parts * s->T);
        p.off_zy = off; off = align256(off + sizeof(float) * s->T);
    }
    if (pass == kI8CeBwd) {
        p.ldz = cdiv(s->V, 256) * 256;
        const long long mib = s->slab_mib > 0 ? s->slab_mib : kDefaultFusedSlabMiB;
        long long cap = (mib << 20) / (p.ldz * 2) / tile_m() * tile_m();
        if (cap < tile_m()) cap = tile_m();
        if (cap < s->T) p.Ts = cdiv(cdiv(s->T, cdiv(s->T, cap)), tile_m()) * tile_m();       // slabs of even height
        p.off_factor = off; off = align256(off + sizeof(float) * s->T);
        p.off_z = off; off = align256(off + 2 * static_cast<size_t>(p.Ts) * p.ldz);
    }
    if (pass == kI8LinearBwd || pass == kI8CeBwd) {
        p.off_w16 = off; if (p.widen) off = align256(off + 2 * static_cast<size_t>(s->V) * s->d);
        const size_t full = dx_part_bytes(p.Ts, s->d, s->V, p.widen), rest = dx_part_bytes(s->T - (cdiv(s->T, p.Ts) - 1) * p.Ts, s->d, s->V, p.widen);
        p.off_part = off; off += full > rest ? full : rest;
    }
    p.total = off;
    return p;
}

// A launch that may start ahead of the end of the kernel before it, for which it waits itself.
template <class... P, class... A>
int launch_ahead(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
    return CAT_OK;
}

template <class T, int WARPS>
void launch_quantize_rows(const T* X, long long rows, long long d, long long ldX, int8_t* Xq, long long ldq, long long pad, float* scale,
                          const i8::CallSetup& setup, int more, bool whole, cudaStream_t st) {
    constexpr int FEW = i8::MOST_EIGHTS / 2;
    const unsigned ctas = static_cast<unsigned>(cdiv(rows, i8::THREADS / 32 / WARPS) + more);
    auto kern = !whole                   ? i8::quantize_rows_kernel<T, WARPS, FEW, true>
                : d > 256 * FEW * WARPS ? i8::quantize_rows_kernel<T, WARPS, i8::MOST_EIGHTS, false> : i8::quantize_rows_kernel<T, WARPS, FEW, false>;
    kern<<<ctas, i8::THREADS, 0, st>>>(X, ldX, static_cast<int>(rows), static_cast<int>(d), Xq, ldq, static_cast<int>(pad), scale, setup);
}

// Rows of whole eights on 16-byte boundaries, up to 16384 long, and others up to 8192 long are read once, by one warp each or, where they are long or few, by
// up to eight: the head of 128256 x 2048 113 us, by a CTA per row that reads them twice 346; 151936 rows of 1003 bf16 values 144 and 414.
template <class T>
int launch_quantize(const T* X, long long rows, long long d, long long ldX, int8_t* Xq, long long ldq, long long pad, float* scale, const i8::CallSetup& setup,
                    cudaStream_t st) {
    const int more = setup.sw ? i8::MOST_PARTS : 0;
    const bool whole = d % 8 == 0 && ldX * sizeof(T) % 16 == 0 && !misaligned(X, 16);
    const long long per_warp = 256 * (whole ? i8::MOST_EIGHTS : i8::MOST_EIGHTS / 2);
    if (d <= 8 * per_warp && ldq % 8 == 0 && !misaligned(Xq, 8)) {
        int warps = 1;
        while (warps < 8 && (d > per_warp * warps || (rows * warps < 8 * kPlanSMs && d > 256 * warps))) warps *= 2;
        if (warps == 1) launch_quantize_rows<T, 1>(X, rows, d, ldX, Xq, ldq, pad, scale, setup, more, whole, st);
        else if (warps == 2) launch_quantize_rows<T, 2>(X, rows, d, ldX, Xq, ldq, pad, scale, setup, more, whole, st);
        else if (warps == 4) launch_quantize_rows<T, 4>(X, rows, d, ldX, Xq, ldq, pad, scale, setup, more, whole, st);
        else launch_quantize_rows<T, 8>(X, rows, d, ldX, Xq, ldq, pad, scale, setup, more, whole, st);
    } else {
        i8::quantize_kernel<T><<<static_cast<unsigned>(rows + more), i8::THREADS, 0, st>>>(X, ldX, static_cast<int>(rows), static_cast<int>(d), Xq, ldq,
                                                                                           static_cast<int>(pad), scale, setup);
    }
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}
int quantize(const void* X, int dtype, long long rows, long long d, long long ldX, int8_t* Xq, long long ldq, long long pad, float* scale,
             const i8::CallSetup& setup, cudaStream_t st) {
    return dtype == CAT_BF16 ? launch_quantize(static_cast<const __nv_bfloat16*>(X), rows, d, ldX, Xq, ldq, pad, scale, setup, st)
                             : launch_quantize(static_cast<const float*>(X), rows, d, ldX, Xq, ldq, pad, scale, setup, st);
}

i8::CallSetup header_setup(uint8_t* ws) {
    i8::CallSetup setup = {};
    setup.header = reinterpret_cast<int*>(ws);
    setup.header_ints = kHeaderBytes / sizeof(int);
    return setup;
}

// What every pass begins with: the checks that are alike, the header cleared and the tokens as integers where there are any.
int begin_i8(const cat_i8_shape* s, int pass, const I8Plan& plan, const void* X, const int8_t* Wq, const float* w_scale, void* workspace,
             size_t workspace_bytes, int* sm_count, i8::Head* h, cudaStream_t st) {
    if (misaligned(X, s->x_dtype == CAT_BF16 ? 2 : 4) || misaligned(Wq, 16) || misaligned(w_scale, 16)) return CAT_ERR_ALIGN;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.total) return CAT_ERR_WORKSPACE;
    const int dc = check_device(sm_count);
    if (dc != CAT_OK) return dc;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    h->xq = reinterpret_cast<int8_t*>(ws + plan.off_q); h->ldq = plan.ldq;
    h->sx = reinterpret_cast<float*>(ws + plan.off_s);
    h->wq = Wq; h->sw = w_scale; h->ldw = s->ldW;
    h->T = static_cast<int>(s->T); h->V = static_cast<int>(s->V); h->d = static_cast<int>(s->d);
    if (pass == kI8LinearBwd) return CAT_OK;
    i8::CallSetup setup = header_setup(ws);
    if (pass == kI8CeBwd) { setup.sw = w_scale; setup.V = h->V; setup.most = reinterpret_cast<int*>(ws + kMostOffset); }
    return quantize(X, s->x_dtype, s->T, s->d, s->ldX, reinterpret_cast<int8_t*>(ws + plan.off_q), plan.ldq, plan.ldq,
                    reinterpret_cast<float*>(ws + plan.off_s), setup, st);
}

// 8-bit operand [rows][d] with row pitch ld bytes: boxes of 128 bytes x box_rows, swizzled as the tensor cores want them, or of any width as they are.
int tmap_i8(CUtensorMap* m, const void* base, long long rows, long long d, long long ld, int box_rows, int as_is = 0) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return CAT_ERR_CUDA;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(as_is > 0 ? as_is : 2 * tc::BK), static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          as_is > 0 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CAT_OK : CAT_ERR_CUDA;
}

// The product of h's tokens and head through epilogue Epi: n_groups runs of vocabulary tiles per row tile.
template <class Epi>
int launch_i8(const i8::Head& h, const typename Epi::Params& ep, int n_groups, int* status, int sm_count, cudaStream_t st, const CUtensorMap* out) {
    CUtensorMap tmX, tmW;
    if (tmap_i8(&tmX, h.xq, h.T, h.d, h.ldq, tc::BM) != CAT_OK || tmap_i8(&tmW, h.wq, h.V, h.d, h.ldw, tc::BN / cta_group()) != CAT_OK) return CAT_ERR_CUDA;
    const long long slices = cdiv(h.d, 2);             // a 64-wide slice of 16-bit operands is 128 integers
    return launch_tc<0, 0, Epi>(tmX, tmW, make_sched(h.T, h.V, slices, n_groups, band_tiles(slices), 0), ep, status, sm_count, st, out);
}

int launch_add_parts(const float* part, int g, long long stride, long long rows, long long d, const float* factor, __nv_bfloat16* dX, long long lddX, cudaStream_t st) {
    return launch_ahead(i8::add_parts_kernel, dim3(static_cast<unsigned>(rows), static_cast<unsigned>(cdiv(d, i8::PART_COLS)), 1), i8::THREADS, 0, st, part, g, stride,
                        static_cast<int>(d), factor, dX, lddX);
}

// dX[r, :] = factor[r] sum_v A[r, v] W16[v, :], A [rows, V] and W16 [V, d] of the type Epi multiplies; the vocabulary in parts for few rows.
template <class Epi>
int launch_dx(const void* A, long long ldA, const uint16_t* w16, long long rows, long long d, long long V, const float* factor, __nv_bfloat16* dX, long long lddX,
              float* part, int* status, int sm_count, cudaStream_t st) {
    CUtensorMap tmA, tmW, tmO;
    if (tmap_a(&tmA, A, rows, V, ldA) != CAT_OK || tmap_mn_major(&tmW, w16, V, d, d) != CAT_OK) return CAT_ERR_CUDA;
    const int g = dh_parts(rows, d, V);
    tc::Sched sched = make_sched(rows, d, V, 0, 1, 1);
    typename Epi::Params ep;
    memset(&ep, 0, sizeof(ep));
    ep.N = static_cast<int>(d);
    if (g == 1) {
        ep.row_scale = factor; ep.M = static_cast<int>(rows); ep.out_bf16 = dX; ep.ld_out = lddX; ep.staged = 2;
        if (tmap_out(&tmO, dX, rows, d, lddX) != CAT_OK) return CAT_ERR_CUDA;
        return launch_tc<0, 1, Epi>(tmA, tmW, sched, ep, status, sm_count, st, &tmO);
    }
    const long long padded = sched.m_real * tile_m();
    sched.k_splits = g;
    sched.num_m_tiles = sched.m_real * g;
    sched.n_items = sched.num_m_tiles * sched.n_groups;
    ep.M = static_cast<int>(padded * g); ep.out_f32 = part; ep.ld_out = d; ep.staged = 1;
    if (tmap_out_f32(&tmO, part, ep.M, d, d) != CAT_OK) return CAT_ERR_CUDA;
    const int rc = launch_tc<0, 1, Epi>(tmA, tmW, sched, ep, status, sm_count, st, &tmO);
    if (rc != CAT_OK) return rc;
    return launch_add_parts(part, g, padded * d, rows, d, factor, dX, lddX, st);
}

template <int MODE, int TPW>
int launch_skinny_i8_as(const CUtensorMap& tmW, const CUtensorMap& tmX, i8::SkinnyParams p, int* status, int grid, cudaStream_t st) {
    p.stages = (skinny::SMEM_BYTES - 1024 - 8192) / ((i8::SUB * p.tile_rows + p.n) * 128);
    if (p.stages > skinny::MAX_STAGES) p.stages = skinny::MAX_STAGES;
    auto kern = i8::skinny_kernel<MODE, TPW>;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(kern, skinny::SMEM_BYTES, allowed)) return CAT_ERR_CUDA;
    return launch_ahead(kern, dim3(static_cast<unsigned>(grid), 1, 1), i8::SKINNY_THREADS, skinny::SMEM_BYTES, st, tmW, tmX, p, status);
}

// Up to 128 tokens against the head in the manner of MODE; p holds what that needs besides the sizes.
template <int MODE>
int launch_skinny_i8(i8::SkinnyParams p, int* status, int sm_count, int* n_parts, cudaStream_t st) {
    p.n = static_cast<int>(cdiv(p.h.T, 16) * 16);
    p.tile_rows = skinny_tile_rows(p.h.V);
    p.n_tiles = static_cast<int>(cdiv(p.h.V, p.tile_rows));
    p.num_kb = static_cast<int>(cdiv(p.h.d, 128));
    p.wait_ns = tc::WAIT_LIMIT_NS;
    CUtensorMap tmW, tmX;
    if (tmap_i8(&tmW, p.h.wq, p.h.V, p.h.d, p.h.ldw, p.tile_rows) != CAT_OK || tmap_i8(&tmX, p.h.xq, p.h.T, p.h.d, p.h.ldq, p.n) != CAT_OK) return CAT_ERR_CUDA;
    int grid = sm_count < kPlanSMs ? sm_count : kPlanSMs;
    if (p.n_tiles < grid) grid = p.n_tiles;
    if (n_parts) *n_parts = grid;
    if (p.h.T <= 64) return launch_skinny_i8_as<MODE, 32>(tmW, tmX, p, status, grid, st);
    return launch_skinny_i8_as<MODE, 64>(tmW, tmX, p, status, grid, st);
}

template <bool SCALED, int TMEM, int UNITS, bool HEAD_M>
int launch_grad_as(const CUtensorMap& tmW, const CUtensorMap& tmA, const i8::GradParams& p, int* status, dim3 grid, cudaStream_t st) {
    auto kern = i8::grad_kernel<SCALED, TMEM, UNITS, HEAD_M>;
    static std::atomic<unsigned long long> allowed{0};
    if (!allow_smem(kern, i8::GRAD_SMEM, allowed)) return CAT_ERR_CUDA;
    if (p.first) {           // what the head or dY comes from may still be running: no launch ahead of that
        kern<<<grid, i8::GRAD_THREADS, i8::GRAD_SMEM, st>>>(tmW, tmA, p, status);
        return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
    }
    return launch_ahead(kern, grid, i8::GRAD_THREADS, i8::GRAD_SMEM, st, tmW, tmA, p, status);
}

// dX[r, :] = factor[r] sum_v A[r, v] W[v, :] of one pass, the head widened on its way.  first: the call's inputs are all that it reads.
template <bool SCALED>
int launch_grad_pass(const i8::Head& h, const void* A, long long ldA, const float* factor, __nv_bfloat16* dX, long long lddX, float* part, bool first, int* status,
                     cudaStream_t st) {
    const GradPlan plan = plan_grad(h.T, h.d, h.V);
    i8::GradParams p;
    p.sw = h.sw; p.part = part; p.T = h.T; p.V = h.V; p.d = h.d;
    p.n = plan.n; p.tiles = plan.tiles; p.num_kb = plan.num_kb;
    const int a_bytes = plan.n * 128, slack = plan.n < 128 ? 128 * 128 - a_bytes : 0;           // the last slot's MMA reads 128 rows
    p.stages = (i8::GRAD_SMEM - 1024 - i8::GRAD_WIDE * plan.units * 2 * i8::GRAD_UNIT_BYTES - slack) / (plan.units * i8::GRAD_UNIT_BYTES + plan.tiles * a_bytes);
    if (p.stages > i8::GRAD_MAX_STAGES) p.stages = i8::GRAD_MAX_STAGES;
    p.first = first;
    p.wait_ns = tc::WAIT_LIMIT_NS;
    CUtensorMap tmW, tmA;
    if (tmap_i8(&tmW, h.wq, h.V, h.d, h.ldw, i8::GRAD_SLICE, i8::GRAD_COLS * plan.units) != CAT_OK || tmap_k_major(&tmA, A, h.T, h.V, ldA, p.n) != CAT_OK) return CAT_ERR_CUDA;
    const dim3 grid(static_cast<unsigned>(cdiv(h.d, i8::GRAD_COLS * plan.units)), static_cast<unsigned>(plan.parts), 1);
    const int rc = plan.head_m       ? launch_grad_as<SCALED, 512, 1, true>(tmW, tmA, p, status, grid, st)
                   : plan.tiles == 2 ? launch_grad_as<SCALED, 512, 2, false>(tmW, tmA, p, status, grid, st)
                                     : launch_grad_as<SCALED, 256, 2, false>(tmW, tmA, p, status, grid, st);
    if (rc != CAT_OK) return rc;
    return launch_add_parts(part, plan.parts, static_cast<long long>(h.T) * h.d, h.T, h.d, factor, dX, lddX, st);
}

template <bool SCALED>
int launch_grad(const i8::Head& h, const void* A, long long ldA, const float* factor, __nv_bfloat16* dX, long long lddX, float* part, int* status, cudaStream_t st) {
    const long long step = grad_pass_rows(h.T);
    for (long long r0 = 0; r0 < h.T; r0 += step) {
        i8::Head hp = h;
        hp.T = static_cast<int>(h.T - r0 < step ? h.T - r0 : step);
        const int rc = launch_grad_pass<SCALED>(hp, static_cast<const uint16_t*>(A) + r0 * ldA, ldA, factor ? factor + r0 : nullptr, dX + r0 * lddX, lddX, part,
                                                SCALED && r0 == 0, status, st);
        if (rc != CAT_OK) return rc;
    }
    return CAT_OK;
}

template <bool SCALED>
int launch_widen(const i8::Head& h, uint16_t* w16, const i8::CallSetup& setup, int sm_count, cudaStream_t st) {
    const int per_row = h.d / 8;
    i8::widen_kernel<SCALED><<<static_cast<unsigned>(8 * sm_count), i8::THREADS, 0, st>>>(h.wq, h.ldw, h.sw, static_cast<long long>(h.V) * per_row, per_row,
                                                                                          h.d, w16, setup);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}

}  // namespace

extern "C" {

int cat_i8_quantize(const void* X, int32_t dtype, int64_t rows, int64_t d, int64_t ldX, int8_t* Xq, int64_t ldXq, float* scale,
                    void* cuda_stream) {
    if (!X || !Xq || !scale) return CAT_ERR_NULL;
    if (rows <= 0 || rows >= (1ll << 31) || d <= 0 || d >= (1ll << 31) || ldX < d || ldXq < d) return CAT_ERR_SHAPE;
    if (dtype != CAT_BF16 && dtype != CAT_F32) return CAT_ERR_DTYPE;
    if (misaligned(X, dtype == CAT_BF16 ? 2 : 4) || misaligned(scale, 4)) return CAT_ERR_ALIGN;
    int sm_count = 0;
    const int dc = check_device(&sm_count);
    if (dc != CAT_OK) return dc;
    return quantize(X, dtype, rows, d, ldX, Xq, ldXq, d, scale, i8::CallSetup{}, static_cast<cudaStream_t>(cuda_stream));
}

size_t cat_i8_workspace_bytes(const cat_i8_shape* shape, int pass) {
    if (pass < kI8Linear || pass > kI8CeBwd || check_i8(shape, pass) != CAT_OK) return 0;
    return plan_i8(shape, pass).total;
}

int cat_i8_linear_fwd(const cat_i8_shape* shape, const void* X, const int8_t* Wq, const float* w_scale, const float* bias, void* Y,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !X || !Wq || !w_scale || !Y) return CAT_ERR_NULL;
    const int sc = check_i8(shape, kI8Linear);
    if (sc != CAT_OK) return sc;
    if (misaligned(Y, 16) || misaligned(bias, 16)) return CAT_ERR_ALIGN;
    const I8Plan plan = plan_i8(shape, kI8Linear);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int sm_count = 0;
    i8::Head h;
    const int rc = begin_i8(shape, kI8Linear, plan, X, Wq, w_scale, workspace, workspace_bytes, &sm_count, &h, st);
    if (rc != CAT_OK) return rc;
    int* status = static_cast<int*>(workspace);
    if (plan.skinny) {
        i8::SkinnyParams p;
        memset(&p, 0, sizeof(p));
        p.h = h; p.bias = bias; p.Y = Y; p.ldY = shape->ldY;
        return shape->y_dtype == CAT_F32 ? launch_skinny_i8<i8::SKINNY_F32>(p, status, sm_count, nullptr, st)
                                         : launch_skinny_i8<i8::SKINNY_BF16>(p, status, sm_count, nullptr, st);
    }
    const long long whole = h.V >= 32 ? h.V / 32 * 32 : 4;        // nothing is sent where there is no whole chunk
    CUtensorMap tmY;
    if (shape->y_dtype == CAT_F32) {
        if (tmap_out_f32(&tmY, Y, h.T, whole, shape->ldY) != CAT_OK) return CAT_ERR_CUDA;
        return launch_i8<i8::EpiLinear<true>>(h, {h.sx, h.sw, bias, Y, shape->ldY, h.T, h.V}, fwd_splits(h.T, h.V), status, sm_count, st, &tmY);
    }
    if (tmap_out(&tmY, Y, h.T, whole, shape->ldY) != CAT_OK) return CAT_ERR_CUDA;
    return launch_i8<i8::EpiLinear<false>>(h, {h.sx, h.sw, bias, Y, shape->ldY, h.T, h.V}, fwd_splits(h.T, h.V), status, sm_count, st, &tmY);
}

int cat_i8_linear_bwd(const cat_i8_shape* shape, const void* dY, const int8_t* Wq, const float* w_scale, void* dX,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !dY || !Wq || !w_scale || !dX) return CAT_ERR_NULL;
    const int sc = check_i8(shape, kI8LinearBwd);
    if (sc != CAT_OK) return sc;
    if (misaligned(dY, 16) || misaligned(dX, 16)) return CAT_ERR_ALIGN;
    const I8Plan plan = plan_i8(shape, kI8LinearBwd);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int sm_count = 0;
    i8::Head h;
    const int rc = begin_i8(shape, kI8LinearBwd, plan, nullptr, Wq, w_scale, workspace, workspace_bytes, &sm_count, &h, st);
    if (rc != CAT_OK) return rc;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (!plan.widen)
        return launch_grad<true>(h, dY, shape->ldY, nullptr, static_cast<__nv_bfloat16*>(dX), shape->lddX, reinterpret_cast<float*>(ws + plan.off_part),
                                 reinterpret_cast<int*>(ws), st);
    uint16_t* w16 = reinterpret_cast<uint16_t*>(ws + plan.off_w16);
    const int wc = launch_widen<true>(h, w16, header_setup(ws), sm_count, st);
    if (wc != CAT_OK) return wc;
    return launch_dx<i8::EpiOutBehind>(dY, shape->ldY, w16, shape->T, shape->d, shape->V, nullptr, static_cast<__nv_bfloat16*>(dX), shape->lddX,
                                 reinterpret_cast<float*>(ws + plan.off_part), reinterpret_cast<int*>(ws), sm_count, st);
}

int cat_i8_ce_fwd(const cat_i8_shape* shape, const void* X, const int8_t* Wq, const float* w_scale, const int64_t* labels,
                  const uint8_t* valid, float* nll, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !X || !Wq || !w_scale || !labels || !nll || !lse) return CAT_ERR_NULL;
    const int sc = check_i8(shape, kI8Ce);
    if (sc != CAT_OK) return sc;
    if (misaligned(labels, 8) || misaligned(nll, 4) || misaligned(lse, 4)) return CAT_ERR_ALIGN;
    const I8Plan plan = plan_i8(shape, kI8Ce);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int sm_count = 0;
    i8::Head h;
    const int rc = begin_i8(shape, kI8Ce, plan, X, Wq, w_scale, workspace, workspace_bytes, &sm_count, &h, st);
    if (rc != CAT_OK) return rc;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    float *part_m = reinterpret_cast<float*>(ws + plan.off_m), *part_l = reinterpret_cast<float*>(ws + plan.off_l),
          *z_label = reinterpret_cast<float*>(ws + plan.off_zy);
    const long long* y = reinterpret_cast<const long long*>(labels);
    int* status = reinterpret_cast<int*>(ws);
    int parts = 2 * plan.S, gc;
    if (plan.skinny) {
        i8::SkinnyParams p;
        memset(&p, 0, sizeof(p));
        p.h = h; p.labels = y; p.part_m = part_m; p.part_l = part_l; p.z_label = z_label;
        gc = launch_skinny_i8<i8::SKINNY_CE>(p, status, sm_count, &parts, st);
    } else {
        i8::EpiCe::Params ep;
        ep.sx = h.sx; ep.sw = h.sw; ep.labels = y; ep.part_m = part_m; ep.part_l = part_l; ep.z_label = z_label; ep.parts = parts; ep.T = h.T; ep.V = h.V;
        gc = launch_i8<i8::EpiCe>(h, ep, plan.S, status, sm_count, st, nullptr);
    }
    if (gc != CAT_OK) return gc;
    return launch_ahead(i8::merge_kernel, dim3(static_cast<unsigned>(cdiv(h.T, i8::THREADS / 32)), 1, 1), i8::THREADS, 0, st, static_cast<const float*>(part_m),
                        static_cast<const float*>(part_l), static_cast<const float*>(z_label), parts, h.T, h.V, y, valid, nll, lse);
}

int cat_i8_ce_bwd(const cat_i8_shape* shape, const void* X, const int8_t* Wq, const float* w_scale, const int64_t* labels,
                  const uint8_t* valid, const float* nll, const float* lse, const float* grad_nll, void* dX,
                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!shape || !X || !Wq || !w_scale || !labels || !nll || !lse || !grad_nll || !dX) return CAT_ERR_NULL;
    const int sc = check_i8(shape, kI8CeBwd);
    if (sc != CAT_OK) return sc;
    if (misaligned(labels, 8) || misaligned(nll, 4) || misaligned(lse, 4) || misaligned(grad_nll, 4) || misaligned(dX, 16)) return CAT_ERR_ALIGN;
    const I8Plan plan = plan_i8(shape, kI8CeBwd);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int sm_count = 0;
    i8::Head h;
    const int rc = begin_i8(shape, kI8CeBwd, plan, X, Wq, w_scale, workspace, workspace_bytes, &sm_count, &h, st);
    if (rc != CAT_OK) return rc;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int* most = reinterpret_cast<int*>(ws + kMostOffset);
    float* factor = reinterpret_cast<float*>(ws + plan.off_factor);
    __half* dz = reinterpret_cast<__half*>(ws + plan.off_z);
    const long long* y = reinterpret_cast<const long long*>(labels);
    uint16_t* w16 = reinterpret_cast<uint16_t*>(ws + plan.off_w16);
    float* part = reinterpret_cast<float*>(ws + plan.off_part);
    int* status = reinterpret_cast<int*>(ws);
    if (plan.widen) {
        const int wc = launch_widen<false>(h, w16, i8::CallSetup{}, sm_count, st);
        if (wc != CAT_OK) return wc;
    }
    for (long long r0 = 0; r0 < shape->T; r0 += plan.Ts) {
        i8::Head hs = h;
        hs.T = static_cast<int>(shape->T - r0 < plan.Ts ? shape->T - r0 : plan.Ts);
        hs.xq += r0 * plan.ldq; hs.sx += r0;
        const uint8_t* on = valid ? valid + r0 : nullptr;
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(dX) + r0 * shape->lddX;
        int gc;
        if (plan.skinny) {
            i8::SkinnyParams p;
            memset(&p, 0, sizeof(p));
            p.h = hs; p.Y = dz; p.ldY = plan.ldz; p.labels = y; p.valid = on; p.nll = nll; p.lse = lse; p.g = grad_nll; p.most = most; p.factor = factor;
            gc = launch_skinny_i8<i8::SKINNY_DZ>(p, status, sm_count, nullptr, st);
        } else {
            CUtensorMap tmZ;
            if (tmap_out(&tmZ, dz, hs.T, hs.V, plan.ldz) != CAT_OK) return CAT_ERR_CUDA;
            i8::EpiDz::Params ep;
            ep.sx = hs.sx; ep.sw = hs.sw; ep.labels = y + r0; ep.valid = on; ep.nll = nll + r0; ep.lse = lse + r0; ep.g = grad_nll + r0;
            ep.most = most; ep.factor = factor + r0; ep.T = hs.T; ep.V = hs.V;
            gc = launch_i8<i8::EpiDz>(hs, ep, fwd_splits(hs.T, hs.V), status, sm_count, st, &tmZ);
        }
        if (gc != CAT_OK) return gc;
        gc = plan.widen ? launch_dx<i8::EpiOutHalf>(dz, plan.ldz, w16, hs.T, hs.d, hs.V, factor + r0, out, shape->lddX, part, status, sm_count, st)
                        : launch_grad<false>(hs, dz, plan.ldz, factor + r0, out, shape->lddX, part, status, st);
        if (gc != CAT_OK) return gc;
    }
    return CAT_OK;
}

}  // extern "C"
