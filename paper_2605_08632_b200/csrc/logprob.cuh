// Log probabilities of given tokens, entropy and top alternatives of the rows of softmax(H W^T), and their
// gradients, without a stored T x V matrix.
//
//   z = H W^T,  lse = log sum_v exp z,  logp = z[y] - lse,  entropy = lse - sum_v p z = log l - u / l,
//   l = sum_v exp(z - m),  u = sum_v exp(z - m) (z - m)    (one pass, running maximum m)
//
// Forward: the logits GEMM (tc_gemm.cuh) with an epilogue that keeps (m, l, u) per row and vocabulary split.
// With alternatives wanted it also writes the row slab's logits as fp16 and the fp32 maximum of every run of 32
// columns; row_kernel then finds the top k among the few columns that can be in it (see there).
// Bound by the tensor cores for many rows and by reading W for few.
//
// Backward: the logits are recomputed per vocabulary slab and leave the GEMM as
//   dz[v] = gl ([v = y] - p) - ge p (log p + entropy)
// for upstream gradients gl (of logp) and ge (of the entropy); the dH and dW contractions follow.
#pragma once
#include "rowops.cuh"
#include "tc_gemm.cuh"

namespace cat {
namespace tc {

constexpr int LP_GROUP = 32;             // columns per maximum that the epilogue keeps (one TMEM chunk)
constexpr float LP_LOW = -1.0e30f;       // "no column yet": finite, so that 0 * (LP_LOW - m) is 0 and not NaN

// index of the first of 32 values that equals x (the last if none does)
__device__ __forceinline__ int first_at(const float (&f)[32], float x) {
    int at = 31;
#pragma unroll
    for (int i = 30; i >= 0; --i) at = f[i] == x ? i : at;
    return at;
}

// Softmax statistics with entropy, and the row's largest logit's column.  TOP: also the slab's logits as fp16 distances from the
// maximum of their 32-column group, and those maxima in fp32.
template <bool TOP>
struct EpiLp {
    struct Params {
        float* part_m;             // [n_groups][part_stride] running max of each (row, vocabulary split)
        float* part_l;             // sum exp(z - m)
        float* part_u;             // sum exp2(x) x with x = (z - m) log2 e
        int* part_id;              // first column that holds the maximum
        float* gmax;               // [T][ld_g] maximum of columns [32 g, 32 g + 32)   (TOP)
        long long ld_g;            // 8 * vocabulary tiles
        long long part_stride;
        int T;
        int V;
    };
    struct State {
        float m_run, l_run, u_run;
        int id;
        int row;
    };
    __device__ static __forceinline__ void begin_item(const Params&, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * BM + row_in_tile;
        s.m_run = LP_LOW;
        s.l_run = 0.f;
        s.u_run = 0.f;
        s.id = 0;
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, uint32_t taddr, OutStage& o) {
        const int col0 = n_tile * BN;
        const int ncols = min(BN, p.V - col0);
        float g[BN / LP_GROUP];
#pragma unroll
        for (int i = 0; i < BN / LP_GROUP; ++i) g[i] = LP_LOW;
#pragma unroll 1
        for (int c = 0; c < BN / 32; ++c) {
            if (c * 32 >= ncols) break;
            if (TOP && (c & 1) == 0) o.begin();
            uint32_t v[32];
            ptx::tmem_ld_32x32(taddr + c * 32, v);
            ptx::tmem_ld_wait();
            float f[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
            const int live = ncols - c * 32;
            if (live < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live) f[i] = LP_LOW;
            }
            float cmax = ptx::max3_f32(f[0], f[1], f[2]);
#pragma unroll
            for (int i = 3; i + 1 < 32; i += 2) cmax = ptx::max3_f32(cmax, f[i], f[i + 1]);
            cmax = fmaxf(cmax, f[31]);
            if (cmax > s.m_run) s.id = col0 + c * 32 + first_at(f, cmax);
            if (TOP) {
                // the slab keeps z - (maximum of the group): the group's largest logit stays exact, its neighbours near it
#pragma unroll
                for (int i = 0; i < BN / LP_GROUP; ++i)
                    if (i == c) g[i] = cmax;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    o.put((c & 1) * 4 + q, ptx::pack_f16x2_sat(f[q * 8 + 0] - cmax, f[q * 8 + 1] - cmax),
                          ptx::pack_f16x2_sat(f[q * 8 + 2] - cmax, f[q * 8 + 3] - cmax),
                          ptx::pack_f16x2_sat(f[q * 8 + 4] - cmax, f[q * 8 + 5] - cmax),
                          ptx::pack_f16x2_sat(f[q * 8 + 6] - cmax, f[q * 8 + 7] - cmax));
                if ((c & 1) != 0 || (c + 1) * 32 >= ncols) o.flush(col0 + (c >> 1) * 64);
            }
            const float m_new = fmaxf(s.m_run, cmax);
            const float mb = m_new * LOG2E;
            const uint64_t l2e2 = ptx::pack_f32x2(LOG2E, LOG2E), nmb2 = ptx::pack_f32x2(-mb, -mb);
            uint64_t sum2 = ptx::pack_f32x2(0.f, 0.f), u2 = sum2;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint64_t x2 = ptx::fma_f32x2(ptx::pack_f32x2(f[2 * i], f[2 * i + 1]), l2e2, nmb2);
                float x0, x1;
                ptx::unpack_f32x2(x2, x0, x1);
                const uint64_t e2 = ptx::pack_f32x2(ptx::ex2_approx(x0), ptx::ex2_approx(x1));
                sum2 = ptx::add_f32x2(sum2, e2);
                u2 = ptx::fma_f32x2(e2, x2, u2);
            }
            float s0, s1, u0, u1;
            ptx::unpack_f32x2(sum2, s0, s1);
            ptx::unpack_f32x2(u2, u0, u1);
            // move the running sums to the new maximum: u(m') = e^(m - m') (u(m) + (m - m') l(m))
            const float dm = (s.m_run - m_new) * LOG2E;
            const float sc = ptx::ex2_approx(dm);
            s.u_run = fmaf(sc, fmaf(dm, s.l_run, s.u_run), u0 + u1);
            s.l_run = fmaf(s.l_run, sc, s0 + s1);
            s.m_run = m_new;
        }
        if (TOP && s.row < p.T) {
            float4* out = reinterpret_cast<float4*>(p.gmax + static_cast<size_t>(s.row) * p.ld_g + n_tile * (BN / LP_GROUP));
            out[0] = make_float4(g[0], g[1], g[2], g[3]);
            out[1] = make_float4(g[4], g[5], g[6], g[7]);
        }
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return TOP ? p.T : 0; }
    __device__ static __forceinline__ void end_item(const Params& p, const State& s, int group) {
        if (s.row < p.T) {
            const size_t at = static_cast<size_t>(group) * p.part_stride + s.row;
            p.part_m[at] = s.m_run;
            p.part_l[at] = s.l_run;
            p.part_u[at] = s.u_run;
            p.part_id[at] = s.id;
        }
    }
};

// Backward: dz of the current vocabulary slab, rounded to bf16 once (the operand type of the two contractions).
struct EpiDzLp {
    struct Params {
        const long long* labels;       // [T]; nullptr without grad_logp
        const unsigned char* valid;    // [T] or nullptr
        const float* lse;              // [T]
        const float* entropy;          // [T]; nullptr without grad_entropy
        const float* grad_logp;        // [T] or nullptr
        const float* grad_entropy;     // [T] or nullptr
        int T;
        int V;
        int v0;
    };
    struct State {
        float l2;                      // lse * log2 e
        float ca, cb;                  // dz = p (ca + cb log2 p) + gl [v = y]
        float gl;
        int y_rel;
        bool on;                       // the row takes part; one that does not gets zeros whatever its logits are
        int row;
    };
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * BM + row_in_tile;
        s.l2 = 0.f;
        s.ca = s.cb = s.gl = 0.f;
        s.y_rel = -1;
        s.on = s.row < p.T && (p.valid == nullptr || p.valid[s.row] != 0);
        if (s.on) {
            s.l2 = p.lse[s.row] * LOG2E;
            if (p.grad_logp) {
                const long long y = p.labels[s.row];
                if (y >= 0 && y < p.V) {
                    s.y_rel = static_cast<int>(y) - p.v0;
                    s.gl = p.grad_logp[s.row];
                    s.ca = -s.gl;
                }
            }
            if (p.grad_entropy) {
                const float ge = p.grad_entropy[s.row];
                s.ca = fmaf(-ge, p.entropy[s.row], s.ca);
                s.cb = -ge * 0.6931471805599453f;
            }
        }
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, uint32_t taddr, OutStage& o) {
        const int col0 = n_tile * BN;
        const int ncols = min(BN, p.V - p.v0 - col0);
#pragma unroll 1
        for (int c = 0; c < BN / 32; ++c) {
            if (c * 32 >= ncols) break;
            if ((c & 1) == 0) o.begin();
            uint32_t v[32];
            ptx::tmem_ld_32x32(taddr + c * 32, v);
            ptx::tmem_ld_wait();
            float f[32];
            const int live = ncols - c * 32;
            const uint64_t l2e2 = ptx::pack_f32x2(LOG2E, LOG2E), nl2 = ptx::pack_f32x2(-s.l2, -s.l2);
            const uint64_t ca2 = ptx::pack_f32x2(s.ca, s.ca), cb2 = ptx::pack_f32x2(s.cb, s.cb);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint64_t x2 = ptx::fma_f32x2(ptx::pack_f32x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), l2e2, nl2);
                float x0, x1;
                ptx::unpack_f32x2(x2, x0, x1);
                const uint64_t p2 = ptx::pack_f32x2(ptx::ex2_approx(x0), ptx::ex2_approx(x1));
                ptx::unpack_f32x2(ptx::mul_f32x2(p2, ptx::fma_f32x2(cb2, x2, ca2)), f[2 * i], f[2 * i + 1]);
            }
            const int rel = s.y_rel - (col0 + c * 32);
            if (rel >= 0 && rel < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == rel) f[i] += s.gl;
            }
            if (live < 32 || !s.on) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live || !s.on) f[i] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o.put((c & 1) * 4 + q, ptx::pack_bf16x2(f[q * 8 + 0], f[q * 8 + 1]), ptx::pack_bf16x2(f[q * 8 + 2], f[q * 8 + 3]),
                      ptx::pack_bf16x2(f[q * 8 + 4], f[q * 8 + 5]), ptx::pack_bf16x2(f[q * 8 + 6], f[q * 8 + 7]));
            if ((c & 1) != 0 || (c + 1) * 32 >= ncols) o.flush(col0 + (c >> 1) * 64);
        }
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return p.T; }
    __device__ static __forceinline__ void end_item(const Params&, const State&, int) {}
};

}  // namespace tc

namespace lp {

constexpr int THREADS = 256;
constexpr int WARPS = THREADS / 32;
constexpr int MAX_TOP = 256;            // CAT_TOPK_MAX
constexpr int CAP = 1024;               // candidate columns held at a time

// H[r, :] . W[v, :] by one warp, every lane gets the sum.  bf16 products are exact in fp32 (16 significant bits), fp32
// products in fp64; the sums are taken in fp64 and always in the same order, so equal rows of W give equal logits.
__device__ __forceinline__ double warp_dot(const __nv_bfloat16* h, const __nv_bfloat16* w, int d, int lane) {
    const uint4* hv = reinterpret_cast<const uint4*>(h);
    const uint4* wv = reinterpret_cast<const uint4*>(w);
    double acc = 0.0;
#pragma unroll 4
    for (int i = lane; i < d / 8; i += 32) {
        const uint4 a = __ldg(hv + i), b = __ldg(wv + i);
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 fa = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&aw[j]));
            const float2 fb = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&bw[j]));
            acc += static_cast<double>(fa.x * fb.x);
            acc += static_cast<double>(fa.y * fb.y);
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
    return acc;
}
__device__ __forceinline__ double warp_dot(const float* h, const float* w, int d, int lane) {
    double acc = 0.0;
#pragma unroll 4
    for (int i = lane; i < d; i += 32) acc = fma(static_cast<double>(__ldg(h + i)), static_cast<double>(__ldg(w + i)), acc);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
    return acc;
}

// What the slab says of column v of a group whose maximum is gm: its logit up to `err`, plus the GEMM's own error.  fp16 slabs hold
// the distance from the maximum (half a step: 2^-11 of it, or 2^-25), fp32 slabs the logit itself.
__device__ __forceinline__ float stored(const __half* z, float gm, long long v, float& err) {
    const float dist = __half2float(z[v]);
    err = fmaf(-dist, 0.00048828125f, 3.0e-8f);
    return gm + dist;
}
__device__ __forceinline__ float stored(const float* z, float, long long v, float& err) {
    err = 0.f;
    return z[v];
}
template <class TZ>
struct GroupOf { static constexpr int value = tc::LP_GROUP; };
template <>
struct GroupOf<float> { static constexpr int value = 64; };       // columns per tile of the fp32 GEMM
// Error of a logit of the GEMM relative to the row's largest: one addition of 16 products (tensor cores) or one (fp32) at a time, each off
// by at most 2^-23 of a running sum that is taken to stay within twice that logit.
__device__ __forceinline__ float gemm_error(const __half*, int d) { return static_cast<float>(d / 16 + 8) * 2.384185791015625e-7f; }
__device__ __forceinline__ float gemm_error(const float*, int d) { return static_cast<float>(d + 8) * 2.384185791015625e-7f; }

template <class TI, class TZ>
struct RowParams {
    const float* part_m;           // [S][part_stride]
    const float* part_l;
    const float* part_u;
    const int* part_id;
    long long part_stride;
    int S;
    const TI* H;                   // rows of this slab
    const TI* W;
    long long ldH, ldW;
    int d, V;
    const long long* labels;       // [T] or nullptr
    const unsigned char* valid;    // [T] or nullptr
    float* logp;                   // [T] or nullptr
    float* lse;                    // [T]
    float* entropy;                // [T]
    // alternatives
    const TZ* zs;                  // [T][ldz] logits of the slab
    long long ldz;
    const float* gmax;             // [T][ld_g]
    long long ld_g;
    int n_g;                       // groups of GroupOf<TZ> columns
    int k;
    long long* top_ids;            // [T][k]
    float* top_logp;               // [T][k]
};

struct Shared {
    float red[2][WARPS];
    int count[2][WARPS];
    int n_cand;
    float lse;
    int id_max;
    double z_max, z_label;
    double z[CAP];                 // exact logits, where `err` says so
    float approx[CAP];
    float err[CAP];                // how far approx may be off; EXACT: z is known; OUT: not among the k largest
    int id[CAP];
    double z_keep[MAX_TOP];
    int id_keep[MAX_TOP];
};
constexpr float EXACT = -1.f, OUT = -2.f;

__device__ __forceinline__ float block_max(float x, float* red) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) x = fmaxf(x, red[i]);
    return x;
}

// A number that at least k of n values reach, and few more than k: bisection between the least and the largest of them.  The values
// are kept in registers when they fit.  big = largest |value|.
constexpr int KEPT = 20;
template <class F>
__device__ __forceinline__ float near_kth(F value, int n, int k, Shared& sh, float& big) {
    float v[KEPT];
    const bool fits = n <= KEPT * THREADS;
    float hi = -INFINITY, nlo = -INFINITY;
    if (fits) {
#pragma unroll
        for (int j = 0; j < KEPT; ++j) {
            const int i = j * THREADS + threadIdx.x;
            v[j] = i < n ? value(i) : -INFINITY;
            if (i < n) { hi = fmaxf(hi, v[j]); nlo = fmaxf(nlo, -v[j]); }
        }
    } else {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const float x = value(i);
            hi = fmaxf(hi, x);
            nlo = fmaxf(nlo, -x);
        }
    }
    hi = block_max(hi, sh.red[0]);
    float lo = -block_max(nlo, sh.red[1]);
    big = fmaxf(fabsf(hi), fabsf(lo));
    if (n <= k) return lo;
    for (int it = 0; it < 24; ++it) {
        const float mid = 0.5f * lo + 0.5f * hi;
        if (!(mid > lo && mid < hi)) break;
        int c = 0;
        if (fits) {
#pragma unroll
            for (int j = 0; j < KEPT; ++j) c += v[j] >= mid ? 1 : 0;
        } else {
            for (int i = threadIdx.x; i < n; i += THREADS) c += value(i) >= mid ? 1 : 0;
        }
        c = __reduce_add_sync(0xffffffffu, c);
        if ((threadIdx.x & 31) == 0) sh.count[it & 1][threadIdx.x >> 5] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) c += sh.count[it & 1][i];
        if (c >= k) {
            lo = mid;
            if (c <= k + k / 4 + 2) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// Exact logits of candidates [from, n) and the order of all n of them; the first k go to the front of the keep list.
template <class TI, class TZ>
__device__ __forceinline__ int settle(const RowParams<TI, TZ>& p, const TI* h, Shared& sh, int from, int n) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int c = from + warp; c < n; c += WARPS) {
        const double z = warp_dot(h, p.W + static_cast<long long>(sh.id[c]) * p.ldW, p.d, lane);
        if (lane == 0) sh.z[c] = z;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += THREADS) {
        const double z = sh.z[c];
        const int id = sh.id[c];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += (sh.z[j] > z || (sh.z[j] == z && sh.id[j] < id)) ? 1 : 0;
        if (rank < p.k) { sh.z_keep[rank] = z; sh.id_keep[rank] = id; }
    }
    __syncthreads();
    return n < p.k ? n : p.k;
}

// The same from the approximate logits, with exact ones only for candidates that their errors leave in doubt against another, and for
// those that the slab's fp16 has rounded (not the largest of their group): their values are returned.
template <class TI, class TZ>
__device__ __forceinline__ int settle_close(const RowParams<TI, TZ>& p, const TI* h, Shared& sh, int n, float eps) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned doubt = 0;                       // bit i: candidate threadIdx.x + i * THREADS needs its exact logit
    unsigned out = 0;
    static_assert(CAP / THREADS <= 32, "one bit per candidate of a thread");
    for (int i = 0, c = threadIdx.x; c < n; ++i, c += THREADS) {
        const float z = sh.approx[c], e = sh.err[c];
        int above = 0;
        bool near = false;
        for (int j = 0; j < n; ++j) {
            const float gap = sh.approx[j] - z, both = sh.err[j] + e;
            above += gap > both ? 1 : 0;
            near |= j != c && fabsf(gap) <= both;
        }
        if (above >= p.k) out |= 1u << i;
        else if (near || e > eps + 4.0e-8f) doubt |= 1u << i;
    }
    __syncthreads();
    for (int i = 0, c = threadIdx.x; c < n; ++i, c += THREADS) {
        if (out >> i & 1u) sh.err[c] = OUT;
        else if (doubt >> i & 1u) sh.err[c] = EXACT;
    }
    __syncthreads();
    for (int c = warp; c < n; c += WARPS) {
        if (sh.err[c] != EXACT) continue;
        const double z = warp_dot(h, p.W + static_cast<long long>(sh.id[c]) * p.ldW, p.d, lane);
        if (lane == 0) sh.z[c] = z;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += THREADS) {
        const float ec = sh.err[c];
        if (ec == OUT) continue;
        const int id = sh.id[c];
        const double z = ec == EXACT ? sh.z[c] : static_cast<double>(sh.approx[c]);
        int rank = 0;
        for (int j = 0; j < n; ++j) {
            const float ej = sh.err[j];
            if (ej == OUT || j == c) continue;
            // two in doubt against each other are both exact
            if (ec == EXACT && ej == EXACT) rank += (sh.z[j] > z || (sh.z[j] == z && sh.id[j] < id)) ? 1 : 0;
            else rank += sh.approx[j] > sh.approx[c] ? 1 : 0;
        }
        if (rank < p.k) { sh.z_keep[rank] = id == sh.id_max ? sh.z_max : z; sh.id_keep[rank] = id; }
    }
    __syncthreads();
    return n < p.k ? n : p.k;
}

// One CTA per row: merges the split partials (lse, entropy), the label's log probability, and the top k.
//
// lse.  The tensor cores' additions truncate, so a logit that is far from 0 comes out a few 1e-6 of itself too small.  In a row that
// is sure of a token that token's logit makes up lse, so the largest logit is taken again as an fp64 sum and the row's sums
// are corrected by the difference; the label's logit is such a sum too.
//
// Top k.  Any k group maxima are k logits of the row, so a number t that k group maxima reach is a lower bound of the row's k-th
// largest logit, and only columns at or above t, less the GEMM's error, can be among the k largest.  They are looked
// up in the slab: a few groups of it are read, not the row.  The order is that of the exact products: candidates whose approximate
// logits are closer than their errors are compared by fp64 sums (a gather of W for about one in twenty of them; taking all of them
// again cost 0.7 ms for 8192 rows of k = 64, a quarter of the GEMM), and equal logits go to the lower id.
// More than CAP candidates (a row of zeros, many equal rows of W) are settled batch by batch by exact sums.
template <class TI, class TZ, bool TOP>
__global__ void __launch_bounds__(THREADS) row_kernel(const RowParams<TI, TZ> p) {
    __shared__ Shared sh;
    const long long r = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (p.valid != nullptr && p.valid[r] == 0) {
        if (threadIdx.x == 0) {
            p.lse[r] = 0.f;
            p.entropy[r] = 0.f;
            if (p.logp) p.logp[r] = 0.f;
        }
        if (TOP)
            for (int i = threadIdx.x; i < p.k; i += THREADS) { p.top_ids[r * p.k + i] = -1; p.top_logp[r * p.k + i] = -INFINITY; }
        return;
    }
    const TI* h = p.H + r * p.ldH;
    if (warp == 0) {
        // merge the split partials; sums over splits in a fixed order
        float m = tc::LP_LOW;
        int id = 0;
        for (int s = lane; s < p.S; s += 32) {
            const float x = p.part_m[s * p.part_stride + r];
            if (x > m) { m = x; id = p.part_id[s * p.part_stride + r]; }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, off);
            const int oid = __shfl_xor_sync(0xffffffffu, id, off);
            if (om > m || (om == m && oid < id)) { m = om; id = oid; }
        }
        float l = 0.f, u = 0.f;
        for (int s = lane; s < p.S; s += 32) {
            const size_t at = s * p.part_stride + r;
            const float dm = (p.part_m[at] - m) * tc::LOG2E;
            const float e = exp2f(dm), ls = p.part_l[at];
            l = fmaf(e, ls, l);
            u = fmaf(e, fmaf(dm, ls, p.part_u[at]), u);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, off);
            u += __shfl_xor_sync(0xffffffffu, u, off);
        }
        const double z_max = warp_dot(h, p.W + static_cast<long long>(id) * p.ldW, p.d, lane);
        if (lane == 0) {
            // the largest logit entered as exp(0) = 1 and 0; it is exp(x) and x exp(x) with its exact distance x from m
            const float x = static_cast<float>(z_max - static_cast<double>(m));
            if (fabsf(x) < 1.f) {
                l += expm1f(x);
                u = fmaf(x * tc::LOG2E, expf(x), u);
            }
            const float logl = logf(l);
            const float lse = m + logl;
            sh.lse = lse;
            sh.id_max = id;
            sh.z_max = z_max;
            p.lse[r] = lse;
            const float ent = logl - 0.6931471805599453f * u / l;
            p.entropy[r] = ent < 0.f ? 0.f : ent + (lse - lse);      // NaN for a row that is not finite
        }
    } else if (warp == 1 && p.logp != nullptr) {
        const long long y = p.labels[r];
        double zy = 0.0;
        if (y >= 0 && y < p.V) zy = warp_dot(h, p.W + y * p.ldW, p.d, lane);
        if (lane == 0) sh.z_label = zy;
    }
    __syncthreads();
    const float lse = sh.lse;
    if (p.logp != nullptr && threadIdx.x == 0) {
        const long long y = p.labels[r];
        p.logp[r] = (y >= 0 && y < p.V) ? static_cast<float>(sh.z_label - static_cast<double>(lse)) : 0.f;
    }
    if (!TOP) return;
    long long* ids_out = p.top_ids + r * p.k;
    float* lp_out = p.top_logp + r * p.k;
    if (!isfinite(lse)) {
        for (int i = threadIdx.x; i < p.k; i += THREADS) { ids_out[i] = -1; lp_out[i] = NAN; }
        return;
    }
    const float* g = p.gmax + r * p.ld_g;
    const TZ* z = p.zs + r * p.ldz;
    constexpr int group = GroupOf<TZ>::value;
    // With few groups per alternative their maxima bound little (or there are not k of them): go by the logits themselves.
    float big;
    const float t = p.n_g >= 4 * p.k ? near_kth([&](int i) { return g[i]; }, p.n_g, p.k, sh, big)
                                     : near_kth([&](int i) { float e; return stored(z, g[i / group], i, e); }, p.V, p.k, sh, big);
    const float eps = big * gemm_error(z, p.d);
    // a bound taken over stored logits may lie their rounding (2^-11 of the row's span) too high
    const float thr = t - 2.f * eps - (p.n_g >= 4 * p.k ? 0.f : 1.0e-3f * big);
    if (threadIdx.x == 0) sh.n_cand = 0;
    __syncthreads();
    auto look = [&](int gi) {      // one warp appends the candidates of one group
        const float gm = g[gi];
        for (int o = 0; o < group; o += 32) {
            const long long col = static_cast<long long>(gi) * group + o + lane;
            float e, x;
            x = stored(z, gm, col < p.V ? col : 0, e);
            const bool in = col < p.V && x + e >= thr;
            const unsigned hit = __ballot_sync(0xffffffffu, in);
            if (hit == 0) continue;
            int at = 0;
            if (lane == 0) at = atomicAdd(&sh.n_cand, __popc(hit));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(hit & ((1u << lane) - 1u));
            if (in && at < CAP) { sh.id[at] = static_cast<int>(col); sh.approx[at] = x; sh.err[at] = eps + e; }
        }
    };
    for (int g0 = warp * 32; g0 < p.n_g; g0 += THREADS) {
        const int gi = g0 + lane;
        unsigned todo = __ballot_sync(0xffffffffu, gi < p.n_g && g[gi < p.n_g ? gi : 0] >= thr);
        while (todo) {
            const int b = __ffs(todo) - 1;
            todo &= todo - 1;
            look(g0 + b);
        }
    }
    __syncthreads();
    int kept;
    if (sh.n_cand <= CAP) {
        kept = settle_close(p, h, sh, sh.n_cand, eps);
    } else {
        // many logits within the error of the k-th.  A row of zeros has them all equal: ids 0, 1, ...
        bool nz = false;
        for (int i = threadIdx.x; i < p.d; i += THREADS) nz |= static_cast<float>(h[i]) != 0.f;
        if (!__syncthreads_or(nz ? 1 : 0)) {
            kept = p.k < p.V ? p.k : p.V;
            for (int i = threadIdx.x; i < kept; i += THREADS) { sh.z_keep[i] = 0.0; sh.id_keep[i] = i; }
            __syncthreads();
        } else {
            // otherwise batch by batch, one group per warp and step, the k best so far carried along
            kept = 0;
            int n = 0;
            for (int g0 = 0; g0 < p.n_g; g0 += WARPS) {
                if (threadIdx.x == 0) sh.n_cand = n;
                __syncthreads();
                const int gi = g0 + warp;
                if (gi < p.n_g && g[gi] >= thr) look(gi);
                __syncthreads();
                n = sh.n_cand;
                const bool last = g0 + WARPS >= p.n_g;
                if (n > CAP - WARPS * 64 || last) {
                    kept = settle(p, h, sh, kept, n);
                    for (int i = threadIdx.x; i < kept; i += THREADS) { sh.z[i] = sh.z_keep[i]; sh.id[i] = sh.id_keep[i]; }
                    n = kept;
                }
                __syncthreads();
            }
        }
    }
    for (int i = threadIdx.x; i < p.k; i += THREADS) {
        ids_out[i] = i < kept ? sh.id_keep[i] : -1;
        lp_out[i] = i < kept ? static_cast<float>(sh.z_keep[i] - static_cast<double>(lse)) : -INFINITY;
    }
}

// dH = scale * (part 0 + part 1 + ...), in that order, in bf16.  One CTA per row; `stride` elements from part to part.
__global__ void __launch_bounds__(THREADS) add_parts_kernel(const float* part, int n, long long stride, int d, const float* scale,
                                                            __nv_bfloat16* out, long long ld) {
    const long long r = blockIdx.x;
    const float a = scale ? *scale : 1.f;
    for (int i = threadIdx.x; i < d / 4; i += THREADS) {
        const float4* src = reinterpret_cast<const float4*>(part + r * d) + i;
        float4 s = __ldcs(src);
#pragma unroll 4
        for (int g = 1; g < n; ++g) {
            const float4 x = __ldcs(src + g * (stride / 4));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        uint2 o;
        o.x = ptx::pack_bf16x2(a * s.x, a * s.y);
        o.y = ptx::pack_bf16x2(a * s.z, a * s.w);
        *reinterpret_cast<uint2*>(out + r * ld + 4 * i) = o;
    }
}

// Copy of H with the rows that take no part set to zero: the dW contraction meets them with dz = 0, and 0 times
// whatever padding a caller left there (NaN, infinity) must add nothing.
template <class TI>
__global__ void __launch_bounds__(THREADS) masked_copy_kernel(const TI* H, long long ldH, int d, const unsigned char* valid,
                                                              TI* out) {
    const long long r = blockIdx.x;
    const bool on = valid == nullptr || valid[r] != 0;
    constexpr int PER = 16 / sizeof(TI);
    if (sizeof(TI) == 2) {
        const uint4* src = reinterpret_cast<const uint4*>(H + r * ldH);
        uint4* dst = reinterpret_cast<uint4*>(out + r * d);
        for (int i = threadIdx.x; i < d / PER; i += THREADS) dst[i] = on ? src[i] : make_uint4(0u, 0u, 0u, 0u);
    } else {
        for (int i = threadIdx.x; i < d; i += THREADS) out[r * d + i] = on ? H[r * ldH + i] : static_cast<TI>(0);
    }
}

}  // namespace lp
}  // namespace cat
