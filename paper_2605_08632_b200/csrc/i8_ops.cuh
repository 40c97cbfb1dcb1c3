// Host side of the operators on an 8-bit head: cat_i8_quantize, cat_i8_linear_fwd / _bwd and cat_i8_ce_fwd / _bwd.  Included at the end
// of cat_api.cu, whose planning and launch helpers it uses.
#pragma once

namespace {

constexpr size_t kMostOffset = 64;       // header: largest scale of the head

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
    int S;                 // parts of the vocabulary
    size_t off_q, off_s, off_m, off_l, off_zy, off_factor, off_z, total;
};

I8Plan plan_i8(const cat_i8_shape* s, int pass) {
    I8Plan p;
    memset(&p, 0, sizeof(p));
    p.ldq = cdiv(s->d, 16) * 16;
    p.S = static_cast<int>(cdiv(s->V, i8::TILE));
    size_t off = kHeaderBytes;
    if (pass != kI8LinearBwd) {
        p.off_q = off; off = align256(off + static_cast<size_t>(s->T) * p.ldq);
        p.off_s = off; off = align256(off + sizeof(float) * s->T);
    }
    if (pass == kI8Ce) {
        p.off_m = off; off = align256(off + sizeof(float) * p.S * s->T);
        p.off_l = off; off = align256(off + sizeof(float) * p.S * s->T);
        p.off_zy = off; off = align256(off + sizeof(float) * s->T);
    }
    if (pass == kI8CeBwd) {
        p.ldz = cdiv(s->V, 256) * 256;
        const long long mib = s->slab_mib > 0 ? s->slab_mib : kDefaultFusedSlabMiB;
        long long cap = (mib << 20) / (p.ldz * 2) / tile_m() * tile_m();
        if (cap < tile_m()) cap = tile_m();
        p.Ts = cap < s->T ? cap : s->T;
        p.off_factor = off; off = align256(off + sizeof(float) * s->T);
        p.off_z = off; off = align256(off + 2 * static_cast<size_t>(p.Ts) * p.ldz);
    }
    p.total = off;
    return p;
}

template <class T>
int launch_quantize(const void* X, long long rows, long long d, long long ldX, int8_t* Xq, long long ldq, long long pad, float* scale, cudaStream_t st) {
    i8::quantize_kernel<T><<<static_cast<unsigned>(rows), i8::THREADS, 0, st>>>(static_cast<const T*>(X), ldX, static_cast<int>(d), Xq, ldq,
                                                                                static_cast<int>(pad), scale);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}
int quantize(const void* X, int dtype, long long rows, long long d, long long ldX, int8_t* Xq, long long ldq, long long pad, float* scale,
             cudaStream_t st) {
    return dtype == CAT_BF16 ? launch_quantize<__nv_bfloat16>(X, rows, d, ldX, Xq, ldq, pad, scale, st)
                             : launch_quantize<float>(X, rows, d, ldX, Xq, ldq, pad, scale, st);
}

// What every pass begins with: the checks that are alike, the header cleared, the tokens as integers.
int begin_i8(const cat_i8_shape* s, int pass, const I8Plan& plan, const void* X, const int8_t* Wq, const float* w_scale, void* workspace,
             size_t workspace_bytes, int* sm_count, i8::Head* h, cudaStream_t st) {
    if (misaligned(X, s->x_dtype == CAT_BF16 ? 2 : 4) || misaligned(Wq, 16) || misaligned(w_scale, 4)) return CAT_ERR_ALIGN;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < plan.total) return CAT_ERR_WORKSPACE;
    const int dc = check_device(sm_count);
    if (dc != CAT_OK) return dc;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (cudaMemsetAsync(ws, 0, kHeaderBytes, st) != cudaSuccess) { cudaGetLastError(); return CAT_ERR_CUDA; }
    h->xq = reinterpret_cast<int8_t*>(ws + plan.off_q); h->ldq = plan.ldq;
    h->sx = reinterpret_cast<float*>(ws + plan.off_s);
    h->wq = Wq; h->sw = w_scale; h->ldw = s->ldW;
    h->T = static_cast<int>(s->T); h->V = static_cast<int>(s->V); h->d = static_cast<int>(s->d);
    if (pass == kI8LinearBwd) return CAT_OK;
    return quantize(X, s->x_dtype, s->T, s->d, s->ldX, reinterpret_cast<int8_t*>(ws + plan.off_q), plan.ldq, plan.ldq,
                    reinterpret_cast<float*>(ws + plan.off_s), st);
}

dim3 i8_grid(long long rows, long long cols) { return dim3(static_cast<unsigned>(cdiv(cols, i8::TILE)), static_cast<unsigned>(cdiv(rows, i8::TILE))); }

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
    return quantize(X, dtype, rows, d, ldX, Xq, ldXq, d, scale, static_cast<cudaStream_t>(cuda_stream));
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
    if (misaligned(Y, 16) || misaligned(bias, 4)) return CAT_ERR_ALIGN;
    const I8Plan plan = plan_i8(shape, kI8Linear);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int sm_count = 0;
    i8::Head h;
    const int rc = begin_i8(shape, kI8Linear, plan, X, Wq, w_scale, workspace, workspace_bytes, &sm_count, &h, st);
    if (rc != CAT_OK) return rc;
    const bool f32 = shape->y_dtype == CAT_F32;
    i8::linear_kernel<<<i8_grid(h.T, h.V), i8::THREADS, 0, st>>>(h, bias, f32 ? static_cast<float*>(Y) : nullptr,
                                                                 f32 ? nullptr : static_cast<__nv_bfloat16*>(Y), shape->ldY);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
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
    i8::dx_kernel<<<i8_grid(h.T, h.d), i8::THREADS, 0, st>>>(nullptr, static_cast<const __nv_bfloat16*>(dY), shape->ldY, nullptr, h,
                                                             static_cast<__nv_bfloat16*>(dX), shape->lddX);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
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
    i8::ce_kernel<<<i8_grid(h.T, h.V), i8::THREADS, 0, st>>>(h, y, part_m, part_l, z_label);
    i8::merge_kernel<<<static_cast<unsigned>(cdiv(h.T, i8::THREADS)), i8::THREADS, 0, st>>>(part_m, part_l, z_label, plan.S, h.T, h.T, h.V, y, valid, nll, lse);
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
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
    i8::largest_scale_kernel<<<static_cast<unsigned>(cdiv(h.V, 8 * i8::THREADS)), i8::THREADS, 0, st>>>(w_scale, h.V, most);
    for (long long r0 = 0; r0 < shape->T; r0 += plan.Ts) {
        i8::Head hs = h;
        hs.T = static_cast<int>(shape->T - r0 < plan.Ts ? shape->T - r0 : plan.Ts);
        hs.xq += r0 * plan.ldq; hs.sx += r0;
        i8::ce_dz_kernel<<<i8_grid(hs.T, h.V), i8::THREADS, 0, st>>>(hs, y + r0, valid ? valid + r0 : nullptr, nll + r0, lse + r0, grad_nll + r0, most,
                                                                     dz, plan.ldz, factor + r0);
        i8::dx_kernel<<<i8_grid(hs.T, h.d), i8::THREADS, 0, st>>>(dz, nullptr, plan.ldz, factor + r0, hs,
                                                                  static_cast<__nv_bfloat16*>(dX) + r0 * shape->lddX, shape->lddX);
    }
    return cudaGetLastError() == cudaSuccess ? CAT_OK : CAT_ERR_CUDA;
}

}  // extern "C"
