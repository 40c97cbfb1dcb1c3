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
// Backward: the logits are recomputed per row slab and leave the GEMM as
//   dz[v] = gl ([v = y] - p) - ge p (log p + entropy)
// for upstream gradients gl (of logp) and ge (of the entropy); close_kernel writes the entry of a token that has most of the row's probability, and
// the dH and dW contractions follow.
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

// (three chains: one alone is 16 dependent steps)
__device__ __forceinline__ float max_of(const float (&f)[32]) {
    float a = ptx::max3_f32(f[0], f[1], f[2]), b = ptx::max3_f32(f[3], f[4], f[5]), c = ptx::max3_f32(f[6], f[7], f[8]);
#pragma unroll
    for (int i = 9; i + 5 < 32; i += 6) {
        a = ptx::max3_f32(a, f[i], f[i + 1]);
        b = ptx::max3_f32(b, f[i + 2], f[i + 3]);
        c = ptx::max3_f32(c, f[i + 4], f[i + 5]);
    }
    a = ptx::max3_f32(a, f[27], f[28]);
    b = ptx::max3_f32(b, f[29], f[30]);
    return ptx::max3_f32(a, b, fmaxf(c, f[31]));
}

// l = sum exp(z - m) and u = sum exp2(x) x, x = (z - m) log2 e, with m the largest logit so far.
struct RunningSums {
    float m, l, u;
    __device__ __forceinline__ void clear() { m = LP_LOW; l = 0.f; u = 0.f; }
    // 32 logits whose largest is cmax
    __device__ __forceinline__ void add(const float (&f)[32], float cmax) {
        const float m_new = fmaxf(m, cmax);
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
        // the sums so far, moved to the new maximum: u(m') = e^(m - m') (u(m) + (m - m') l(m))
        const float dm = (m - m_new) * LOG2E;
        const float sc = ptx::ex2_approx(dm);
        u = fmaf(sc, fmaf(dm, l, u), u0 + u1);
        l = fmaf(l, sc, s0 + s1);
        m = m_new;
    }
};

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
        RunningSums r;
        int id;
        int row;
    };
    __device__ static __forceinline__ void begin_item(const Params&, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * BM + row_in_tile;
        s.r.clear();
        s.id = 0;
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, uint32_t taddr, OutStage& o) {
        const int col0 = n_tile * BN;
        const int ncols = min(BN, p.V - col0);
        float g[BN / LP_GROUP];
#pragma unroll
        for (int i = 0; i < BN / LP_GROUP; ++i) g[i] = LP_LOW;
        walk_tile(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            if (TOP && (c & 1) == 0) o.begin();
            float f[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
            const int live = ncols - c * 32;
            if (live < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live) f[i] = LP_LOW;
            }
            const float cmax = max_of(f);
            if (cmax > s.r.m) s.id = col0 + c * 32 + first_at(f, cmax);
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
            s.r.add(f, cmax);
        });
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
            p.part_m[at] = s.r.m;
            p.part_l[at] = s.r.l;
            p.part_u[at] = s.r.u;
            p.part_id[at] = s.id;
        }
    }
};

template <>
struct LetsNextStart<EpiLp<true>> { static constexpr bool value = true; };

// Backward: dz of the row slab, rounded to bf16 once (the operand type of the two contractions).
//
// The row's closing entry.  In a row that is sure of a token, that token's entry gl (1 - p) - ge p (log p + entropy) is small against its terms,
// and the rounding of lse alone, 1e-6 of p, would be a tenth of it at 1 - p = 1e-5.  A row of dz sums to zero, so that entry is the others' sum with
// the sign turned, as exact as they are.  It is left out here (at most one token has p above CLOSING), the others are summed per vocabulary
// split, and close_kernel writes it.
constexpr float CLOSING = -0.75f;        // log2 p
struct EpiDzLp {
    struct Params {
        const long long* labels;       // [T]; nullptr without grad_logp
        const unsigned char* valid;    // [T] or nullptr
        const float* lse;              // [T]
        const float* entropy;          // [T]; nullptr without grad_entropy
        const float* grad_logp;        // [T] or nullptr
        const float* grad_entropy;     // [T] or nullptr
        float* part_sum;               // [n_groups][part_stride] sum of the entries but the closing one
        int* part_col;                 // the closing entry's column, or -1
        long long part_stride;
        float* dz_label;               // [T] the label's entry before its rounding, unless it is the closing one
        int T;
        int V;
        int lo_rows;                   // > 0: also what the rounding leaves, as row lo_rows + r (a multiple of 32, >= T)
    };
    struct State {
        float l2;                      // lse * log2 e
        float ca, cb;                  // dz = p (ca + cb log2 p), and gl more at the label
        float gl;
        float sum;
        int col;
        int y;
        bool on;                       // the row takes part; one that does not gets zeros whatever its logits are
        int row;
    };
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * BM + row_in_tile;
        s.l2 = 0.f;
        s.ca = s.cb = s.gl = s.sum = 0.f;
        s.y = s.col = -1;
        s.on = s.row < p.T && (p.valid == nullptr || p.valid[s.row] != 0);
        if (s.on) {
            s.l2 = p.lse[s.row] * LOG2E;
            if (p.grad_logp) {
                const long long y = p.labels[s.row];
                if (y >= 0 && y < p.V) {
                    s.y = static_cast<int>(y);
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
        const int ncols = min(BN, p.V - col0);
        walk_tile(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            if ((c & 1) == 0) {
                if (p.lo_rows == 0) o.begin();
                else o.begin_both();
            }
            float f[32];
            const int live = ncols - c * 32;
            const uint64_t l2e2 = ptx::pack_f32x2(LOG2E, LOG2E), nl2 = ptx::pack_f32x2(-s.l2, -s.l2);
            const uint64_t ca2 = ptx::pack_f32x2(s.ca, s.ca), cb2 = ptx::pack_f32x2(s.cb, s.cb);
            float xmax = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint64_t x2 = ptx::fma_f32x2(ptx::pack_f32x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), l2e2, nl2);
                float x0, x1;
                ptx::unpack_f32x2(x2, x0, x1);
                xmax = ptx::max3_f32(xmax, x0, x1);
                const uint64_t p2 = ptx::pack_f32x2(ptx::ex2_approx(x0), ptx::ex2_approx(x1));
                ptx::unpack_f32x2(ptx::mul_f32x2(p2, ptx::fma_f32x2(cb2, x2, ca2)), f[2 * i], f[2 * i + 1]);
            }
            if (live < 32 || !s.on) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live || !s.on) f[i] = 0.f;
            }
            const int rel = s.y - (col0 + c * 32);
            if (rel >= 0 && rel < 32) {
                float at = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == rel) at = f[i] += s.gl;
                p.dz_label[s.row] = at;
            }
            if (xmax > CLOSING && s.on) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < live && fmaf(__uint_as_float(v[i]), LOG2E, -s.l2) > CLOSING && s.col < 0) {
                        s.col = col0 + c * 32 + i;
                        f[i] = 0.f;
                    }
            }
            uint64_t sum2 = ptx::pack_f32x2(f[0], f[1]), sum2b = ptx::pack_f32x2(f[2], f[3]);
#pragma unroll
            for (int i = 4; i < 32; i += 4) {
                sum2 = ptx::add_f32x2(sum2, ptx::pack_f32x2(f[i], f[i + 1]));
                sum2b = ptx::add_f32x2(sum2b, ptx::pack_f32x2(f[i + 2], f[i + 3]));
            }
            float s0, s1;
            ptx::unpack_f32x2(ptx::add_f32x2(sum2, sum2b), s0, s1);
            s.sum += s0 + s1;
            const bool closes = (c & 1) != 0 || (c + 1) * 32 >= ncols;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) hi[i] = ptx::pack_bf16x2(f[q * 8 + 2 * i], f[q * 8 + 2 * i + 1]);
                o.put((c & 1) * 4 + q, hi[0], hi[1], hi[2], hi[3]);
                if (p.lo_rows > 0) {
                    uint32_t lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        lo[i] = ptx::pack_bf16x2(f[q * 8 + 2 * i] - __uint_as_float(hi[i] << 16), f[q * 8 + 2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u));
                    o.put_other((c & 1) * 4 + q, lo[0], lo[1], lo[2], lo[3]);
                }
            }
            if (closes) {
                if (p.lo_rows == 0) o.flush(col0 + (c >> 1) * 64);
                else o.flush_both(col0 + (c >> 1) * 64, p.lo_rows);
            }
        });
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return p.lo_rows > 0 ? p.lo_rows : p.T; }
    __device__ static __forceinline__ void end_item(const Params& p, const State& s, int group) {
        if (s.row < p.T) {
            const size_t at = static_cast<size_t>(group) * p.part_stride + s.row;
            p.part_sum[at] = s.sum;
            p.part_col[at] = s.col;
        }
    }
};

}  // namespace tc

namespace lp {

constexpr int THREADS = 256;
constexpr int WARPS = THREADS / 32;
constexpr int MAX_TOP = 256;            // CAT_TOPK_MAX
constexpr int CAP = 512;                // candidate columns held at a time
// Threads RT of a row kernel's CTA: its phases wait more than they work, so with many rows small CTAs, eight to an SM; with rows for two CTAs
// an SM at most, large ones, which have four times as many exact logits under way.
constexpr int RT_MANY = 128, RT_FEW = 512;

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

// The same as an fp32 sum (four chains per lane), for where nothing is ordered by it: converting every product to fp64 costs 16 lanes
// a clock.
__device__ __forceinline__ float warp_dot_f32(const __nv_bfloat16* h, const __nv_bfloat16* w, int d, int lane) {
    const uint4* hv = reinterpret_cast<const uint4*>(h);
    const uint4* wv = reinterpret_cast<const uint4*>(w);
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = lane; i < d / 8; i += 32) {
        const uint4 a = __ldg(hv + i), b = __ldg(wv + i);
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 fa = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&aw[j]));
            const float2 fb = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&bw[j]));
            acc[j] = fmaf(fa.x, fb.x, acc[j]);
            acc[j] = fmaf(fa.y, fb.y, acc[j]);
        }
    }
    float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    return sum;
}
__device__ __forceinline__ float warp_dot_f32(const float* h, const float* w, int d, int lane) {
    return static_cast<float>(warp_dot(h, w, d, lane));
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
template <class TI>
__device__ __forceinline__ void prefetch_row(const TI* row, int d, int lane) {
    constexpr int LINE = 128 / sizeof(TI);
    for (int i = lane * LINE; i < d; i += 32 * LINE) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
}
template <class TZ>
struct GroupOf { static constexpr int value = tc::LP_GROUP; };
template <>
struct GroupOf<float> { static constexpr int value = 64; };       // columns per tile of the fp32 GEMM
// Error of a logit of the GEMM as a share of |h| |w|, the product of the norms, which no partial sum of h w exceeds.  (A share of the logit
// itself bounds nothing where the sum cancels: with channels of +-1000 the sums pass through 1000 on their way to a logit of 1.)
// Tensor cores: 16 products at a time, each of the 17 addends cut to 2^-25 of the power of two below the largest, the sum to 2^-23:
// 21 * 2^-25 a step (seen on a B200 with sums of a large term and many small ones).  fp32: runs of 256, each addition rounded to 2^-24.
// 8 steps more cover the roundings of what is made of the logits here.
__device__ __forceinline__ float gemm_error(const __half*, int d) { return static_cast<float>(d / 16 + 9) * (21.f * 0x1p-25f); }
__device__ __forceinline__ float gemm_error(const float*, int d) { return static_cast<float>(min(d, 256) + d / 256 + 9) * 0x1p-24f; }
// The same of warp_dot_f32: four chains of 2 ceil(d / 256) additions a lane, seven more to join them.
__device__ __forceinline__ float dot_error(int d) { return static_cast<float>(2 * ((d + 255) / 256) + 9) * 0x1p-24f; }
// The norm of a vector of d elements from the fp32 sum of their squares, rounded up: what the squares lost below the range, d 2^-126 at most,
// is added, and 1e-3 covers the roundings of the sum (chains of up to 2^12 additions).  Squares past the range give infinity: then every
// candidate is in doubt.
__device__ __forceinline__ float norm_above(float sum_sq, int d) {
    const float x = sqrtf(fmaf(static_cast<float>(d), 0x1p-126f, sum_sq)) * 1.001f;
    return x >= 0.f ? x : INFINITY;
}
// acc + the squares of two bf16 numbers, from above: the upper one is taken with the lower one's bits behind its own, which makes its
// square larger by up to 2^-6 of it and saves an instruction of four.
__device__ __forceinline__ float add_squares(float acc, uint32_t two) {
    const float a = __uint_as_float(two << 16), b = __uint_as_float(two);
    return fmaf(b, b, fmaf(a, a, acc));
}
__device__ __forceinline__ float add_squares(float acc, const uint4& x) {
    return add_squares(add_squares(add_squares(add_squares(acc, x.x), x.y), x.z), x.w);
}
// whether one of eight bf16 numbers is not zero
__device__ __forceinline__ bool any_of(const uint4& x) { return ((x.x | x.y | x.z | x.w) & 0x7fff7fffu) != 0; }
// The least sum of squares of a vector that is not zero, whatever its squares lose below the range: a sum of 0 means a vector of zeros.
constexpr float NOT_ZERO = 0x1p-126f;
// sum of the squares of a row, by one warp
__device__ __forceinline__ float warp_squares(const __nv_bfloat16* row, int d, int lane) {
    const uint4* v = reinterpret_cast<const uint4*>(row);
    constexpr int BATCH = 8;      // loads under way together
    const int n = d / 8;
    float sum = 0.f;
    int i = lane;
    for (; i + 32 * (BATCH - 1) < n; i += 32 * BATCH) {
        uint4 x[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) x[j] = __ldg(v + i + 32 * j);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) sum += add_squares(0.f, x[j]);
    }
#pragma unroll 4
    for (; i < n; i += 32) sum = add_squares(sum, __ldg(v + i));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if (sum == 0.f) {
        bool any = false;
        for (i = lane; i < n; i += 32) any |= any_of(__ldg(v + i));
        if (__any_sync(0xffffffffu, any)) sum = NOT_ZERO;
    }
    return sum;
}
__device__ __forceinline__ float warp_squares(const float* row, int d, int lane) {
    float sum = 0.f;
#pragma unroll 4
    for (int i = lane; i < d; i += 32) { const float x = __ldg(row + i); sum = fmaf(x, x, sum) + (x != 0.f ? NOT_ZERO : 0.f); }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    return sum;
}
// Raises *most, a float >= 0 held as its bits, to x; NaN counts as infinity.  The largest of many does not depend on their order.
__device__ __forceinline__ void raise_to(int* most, float x) {
    atomicMax(most, __float_as_int(x >= 0.f ? x : INFINITY));
}

// The largest sum of squares of a row of W, which row_kernel's bound wants.
//   BESIDE: launched behind the logits GEMM, whose CTAs let it start as soon as they all run.  They leave it 2 KB of shared memory and 28 KB of L1,
//     so that it reads at 1 to 1.7 TB/s: hidden behind a GEMM of many rows.  It ends after the GEMM, so that what follows may take its end for both.
//   otherwise ahead of the GEMM, alone, at the rate of a copy.  Its CTAs walk the GEMM's vocabulary groups (n_groups of them, in tiles of BN)
//     from back to front, so that what the GEMM reads first is in the L2.
// Whole calls with k = 20, beside / ahead, in us: 129 rows of 2048 x 128256 503 / 204, 700 561 / 422, 1100 513 / 624, 4000 1610 / 1853; 600 of 1024 x 151936
// 348 / 285, 1100 429 / 435, 2000 651 / 629.
template <bool BESIDE>
constexpr int NORM_THREADS = BESIDE ? 256 : 512;      // beside: what the registers that the GEMM leaves a quarter of an SM allow
template <bool BESIDE>
__global__ void __launch_bounds__(NORM_THREADS<BESIDE>) norm_kernel(const __nv_bfloat16* W, long long ldW, int d, int V, int n_groups, int* most) {
    constexpr int WARPS = NORM_THREADS<BESIDE> / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long n_tiles = (V + tc::BN - 1) / tc::BN;
    float mx = 0.f;
    for (int g = blockIdx.x % n_groups; g < n_groups; g += gridDim.x) {
        const int sharers = gridDim.x <= n_groups ? 1 : (gridDim.x - g + n_groups - 1) / n_groups;       // CTAs of this group
        const long long v0 = g * n_tiles / n_groups * tc::BN, v1 = min(static_cast<long long>(V), (g + 1) * n_tiles / n_groups * tc::BN);
        for (long long v = v1 - 1 - (blockIdx.x / n_groups) * WARPS - warp; v >= v0; v -= sharers * WARPS) {
            const float x = warp_squares(W + v * ldW, d, lane);
            mx = x <= mx ? mx : x;         // NaN stays
        }
    }
    if (lane == 0) raise_to(most, mx);
    if (BESIDE) asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <class TI, class TZ>
struct RowParams {
    const float* part_m;           // [S][part_stride]
    const float* part_l;
    const float* part_u;
    const int* part_id;            // nullptr: the largest logit is found through gmax and zs
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
    const int* w_sq;               // largest sum of squares of a row of W (float bits)
    const TZ* zs;                  // [T][ldz] logits of the slab
    long long ldz;
    const float* gmax;             // [T][ld_g]
    long long ld_g;
    int n_g;                       // groups of GroupOf<TZ> columns
    int k;
    long long* top_ids;            // [T][k]
    float* top_logp;               // [T][k]
};

template <int RT>
struct Shared {
    static constexpr int RW = RT / 32;
    float red[2][RW];
    int count[2][RW];
    int n_cand, n_near, n_rest, n_tied;
    float m, l, u, logl;
    float h_sq;                    // sum of the squares of the row of H
    int id_max;
    double z_max, z_label;
    double z[CAP];                 // logits summed again, where `err` says so
    float approx[CAP];
    float err[CAP];                // how far approx may be off; DOUBT, SUMMED: z is known; OUT: not among the k largest
    int id[CAP];
    double z_keep[MAX_TOP];
    int id_keep[MAX_TOP];
    int near[CAP];                 // groups that may hold candidates; then the candidates in doubt, and from the end the others
    float near_max[CAP];           // those groups' maxima
    int above[CAP], close[CAP];    // per candidate: others certainly above it, others within the errors
};
constexpr float DOUBT = -1.f, OUT = -2.f, SUMMED = -3.f;

template <int RW>
__device__ __forceinline__ float block_max(float x, float (&red)[RW]) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < RW; ++i) x = fmaxf(x, red[i]);
    return x;
}

// A bound that at least k of the values reach, and few more than k, from the largest values of each thread's four shares of them (best,
// -infinity for an empty share): any k of those are k of the values.  Bisection between the least and the largest, until at most
// k + k / 16 + 1 shares reach it (k = 64 of 4008 values: about 75 values do).  LP_LOW when fewer than k shares hold a value.  big: largest |value| there is.
template <int RT>
__device__ __forceinline__ float near_kth(const float (&best)[4], float least, int k, Shared<RT>& sh, float& big) {
    constexpr int RW = RT / 32;
    const float mine = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
    float hi = block_max(mine, sh.red[0]);
    big = fmaxf(fabsf(hi), fabsf(block_max(-least, sh.red[1])));
    const bool one = k <= RT / 4;                   // the threads' own largest values will do
    float low = mine;
    if (!one) {
#pragma unroll
        for (int j = 0; j < 4; ++j) low = fminf(low, best[j]);
    }
    float lo = -block_max(-low, sh.red[0]);         // -infinity with an empty share: the loop below counts from LP_LOW then
    lo = fmaxf(lo, tc::LP_LOW);
    const int enough = k + k / 16 + 1;
    auto count = [&](float x, int it) {
        if (one) return __syncthreads_count(mine >= x);
        int c = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) c += best[j] >= x ? 1 : 0;
        c = __reduce_add_sync(0xffffffffu, c);
        if ((threadIdx.x & 31) == 0) sh.count[it & 1][threadIdx.x >> 5] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int i = 0; i < RW; ++i) c += sh.count[it & 1][i];
        return c;
    };
    if (lo == tc::LP_LOW) {      // some share is empty: are there k at all?
        if (count(lo, 1) < k) return lo;
        lo = fmaxf(lo, -big);
    }
    for (int it = 0; it < 24; ++it) {
        const float mid = 0.5f * lo + 0.5f * hi;
        if (!(mid > lo && mid < hi)) break;
        const int c = count(mid, it);
        if (c >= k) {
            lo = mid;
            if (c <= enough) break;
        } else {
            hi = mid;
        }
    }
    return lo;
}

// The share of itself that the row's largest logit came out too small, by which its other logits, bf16 sums of as many terms, are taken to be off
// as well (their truncations add up to the same share of each within about a tenth).  Only where truncation of that logit itself explains it: a
// sum that passes through larger numbers is off by something else, which says nothing about the others.
__device__ __forceinline__ float off_share(float off, float m, int d) {
    return m > 1.f && off > 0.f && off <= gemm_error(static_cast<const __half*>(nullptr), d) * m ? off / m : 0.f;
}
template <class TI, class S>
__device__ __forceinline__ float off_share(const S& sh, int d) {
    return sizeof(TI) == 2 ? off_share(static_cast<float>(sh.z_max - static_cast<double>(sh.m)), sh.m, d) : 0.f;
}

// z - lse.  In a row that is sure of its token this is the logarithm of 1 + a little, of which lse rounded to fp32 would leave few places.
template <class S>
__device__ __forceinline__ float log_prob(double z, const S& sh) {
    return static_cast<float>((z - static_cast<double>(sh.m)) - static_cast<double>(sh.logl));
}

// lse and entropy from the merged sums and the exact largest logit, and the label's log probability; one thread.
template <class TI, class TZ, int RT>
__device__ __forceinline__ void finish_row(const RowParams<TI, TZ>& p, long long r, Shared<RT>& sh) {
    // the largest logit entered as exp(0) = 1 and 0; it is exp(x) and x exp(x) with its exact distance x from m
    float l = sh.l, u = sh.u;
    const float x = static_cast<float>(sh.z_max - static_cast<double>(sh.m));
    // l with the others' logits corrected too, to first order: the share times their sum of exp(z - m) z.  The entropy's two parts stay as
    // they were summed: there the share cancels but for itself times the logits' variance.
    float lc = fmaf(off_share<TI>(sh, p.d), fmaf(0.6931471805599453f, u, sh.m * (l - 1.f)), l);
    if (fabsf(x) < 1.f) {
        lc += expm1f(x);
        l += expm1f(x);
        u = fmaf(x * tc::LOG2E, expf(x), u);
    }
    const float logl = logf(lc), lse = sh.m + logl;
    sh.logl = logl;
    p.lse[r] = lse;
    const float ent = logf(l) - 0.6931471805599453f * u / l;
    p.entropy[r] = ent < 0.f ? 0.f : ent + (lse - lse);      // NaN for a row that is not finite
    if (p.logp != nullptr) {
        const long long y = p.labels[r];
        p.logp[r] = (y >= 0 && y < p.V) ? log_prob(y == sh.id_max ? sh.z_max : sh.z_label, sh) : 0.f;
    }
}

// The two logits of a row that are always taken exactly, by one warp each: which = 0 the largest, 1 the label's.
template <class TI, class TZ, int RT>
__device__ __forceinline__ void exact_one(const RowParams<TI, TZ>& p, const TI* h, long long r, Shared<RT>& sh, int which) {
    const int lane = threadIdx.x & 31;
    if (which == 0) {
        const double z = warp_dot(h, p.W + static_cast<long long>(sh.id_max) * p.ldW, p.d, lane);
        if (lane == 0) sh.z_max = z;
    } else if (p.logp != nullptr) {
        const long long y = p.labels[r];
        if (y >= 0 && y < p.V && y != sh.id_max) {
            const double z = warp_dot(h, p.W + y * p.ldW, p.d, lane);
            if (lane == 0) sh.z_label = z;
        }
    }
}

// Exact logits of candidates [from, n) and the order of all n of them; the first k go to the front of the keep list.
template <class TI, class TZ, int RT>
__device__ __forceinline__ int settle(const RowParams<TI, TZ>& p, const TI* h, Shared<RT>& sh, int from, int n) {
    constexpr int RW = RT / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int c = from + warp; c < n; c += RW) {
        const double z = warp_dot(h, p.W + static_cast<long long>(sh.id[c]) * p.ldW, p.d, lane);
        if (lane == 0) sh.z[c] = z;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += RT) {
        const double z = sh.z[c];
        const int id = sh.id[c];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += (sh.z[j] > z || (sh.z[j] == z && sh.id[j] < id)) ? 1 : 0;
        if (rank < p.k) { sh.z_keep[rank] = z; sh.id_keep[rank] = id; }
    }
    __syncthreads();
    return n < p.k ? n : p.k;
}

// The same, ordered by the approximate logits.  Candidates that their errors (eps and what the slab's rounding adds) leave in doubt against another
// are summed again, in fp32 (off by eps32 at most); those still in doubt against each other, in fp64, which takes eight times as long.
//
// The values.  A bf16 logit of 20 that comes out 3e-6 of itself too small would be off by more than its log probability has
// places for.  With few rows every value is an fp32 sum over d.  With many only values in doubt and values that the slab's fp16 has rounded (not
// the largest of their group) are summed, each a gather of a row of W, and the others are corrected by the share of itself that the largest
// logit is off (see finish_row).
template <class TI, class TZ, int RT>
__device__ __forceinline__ int settle_close(const RowParams<TI, TZ>& p, const TI* h, long long r, Shared<RT>& sh, int n, float eps, float eps32) {
    constexpr int RW = RT / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long y = p.logp != nullptr ? p.labels[r] : -1;
    if (RT == RT_FEW)
        for (int c = warp; c < n; c += RW) prefetch_row(p.W + static_cast<long long>(sh.id[c]) * p.ldW, p.d, lane);
    // Several threads share a candidate while there are threads to share: each looks at its part of the others.
    const int parts = n <= RT / 2 ? RT / (n > 0 ? n : 1) : 1;
    const int part = threadIdx.x / (n > 0 ? n : 1), per = (n + parts - 1) / parts;
    for (int c = threadIdx.x; c < n; c += RT) { sh.above[c] = 0; sh.close[c] = 0; }
    if (threadIdx.x == 0) sh.n_near = sh.n_rest = sh.n_tied = 0;
    // every place is written below, but where a logits kernel that timed out has left norms that bound nothing
    for (int c = threadIdx.x; c < p.k; c += RT) { sh.z_keep[c] = -INFINITY; sh.id_keep[c] = -1; }
    __syncthreads();
    for (int c = parts > 1 ? threadIdx.x - part * n : threadIdx.x; c < n && (parts == 1 || part < parts); c += parts > 1 ? CAP : RT) {
        const float z = sh.approx[c], e = sh.err[c];
        const int j0 = parts > 1 ? part * per : 0, j1 = parts > 1 ? min(n, j0 + per) : n;
        int above = 0, near = 0;
#pragma unroll 8
        for (int j = j0; j < j1; ++j) {
            const float gap = sh.approx[j] - z, both = sh.err[j] + e;
            above += gap > both ? 1 : 0;
            near += fabsf(gap) <= both ? 1 : 0;       // itself among them
        }
        if (above) atomicAdd(&sh.above[c], above);
        if (near) atomicAdd(&sh.close[c], near);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += RT) {
        if (sh.above[c] >= p.k) {
            sh.err[c] = OUT;
            sh.approx[c] = -INFINITY;
        } else if (sh.close[c] > 1) {
            sh.err[c] = DOUBT;
            sh.near[atomicAdd(&sh.n_near, 1)] = c;
        } else if (sizeof(TI) == 2 && sh.id[c] != sh.id_max && sh.id[c] != y &&
                   (RT == RT_FEW || sh.err[c] - eps > 4.0e-8f)) {
            sh.err[c] = SUMMED;
            sh.near[CAP - 1 - atomicAdd(&sh.n_rest, 1)] = c;
        }
        sh.above[c] = 0;
    }
    __syncthreads();
    const int n_doubt = sh.n_near, n_rest = sh.n_rest;
    for (int i = warp; i < n_doubt + 2 + n_rest; i += RW) {
        if (i < 2) {
            exact_one(p, h, r, sh, i);
        } else {
            const int c = i < n_doubt + 2 ? sh.near[i - 2] : sh.near[CAP - 1 - (i - n_doubt - 2)];
            const TI* w = p.W + static_cast<long long>(sh.id[c]) * p.ldW;
            const double z = sizeof(TI) == 2 ? static_cast<double>(warp_dot_f32(h, w, p.d, lane)) : warp_dot(h, w, p.d, lane);
            if (lane == 0) sh.z[c] = z;
        }
    }
    if (sizeof(TI) == 2 && n_doubt > 1) {
        __syncthreads();
        for (int i = threadIdx.x; i < n_doubt; i += RT) {
            const int c = sh.near[i];
            const float z = static_cast<float>(sh.z[c]);
            bool tied = false;
            for (int j = 0; j < n_doubt; ++j) tied |= j != i && fabsf(static_cast<float>(sh.z[sh.near[j]]) - z) <= 2.f * eps32;
            if (tied) sh.close[atomicAdd(&sh.n_tied, 1)] = c;
        }
        __syncthreads();
        const int n_tied = sh.n_tied;
        for (int i = warp; i < n_tied; i += RW) {
            const int c = sh.close[i];
            const double z = warp_dot(h, p.W + static_cast<long long>(sh.id[c]) * p.ldW, p.d, lane);
            if (lane == 0) sh.z[c] = z;
        }
    }
    for (int c = parts > 1 ? threadIdx.x - part * n : threadIdx.x; c < n && (parts == 1 || part < parts); c += parts > 1 ? CAP : RT) {
        const float zc = sh.approx[c];
        const int j0 = parts > 1 ? part * per : 0, j1 = parts > 1 ? min(n, j0 + per) : n;
        int rank = 0;
#pragma unroll 8
        for (int j = j0; j < j1; ++j) rank += sh.approx[j] > zc ? 1 : 0;
        if (rank) atomicAdd(&sh.above[c], rank);
    }
    __syncthreads();
    if (threadIdx.x == RT - 1) finish_row(p, r, sh);
    const float share = off_share<TI>(sh, p.d);
    for (int c = threadIdx.x; c < n; c += RT) {
        const float ec = sh.err[c], zc = sh.approx[c];
        if (ec == OUT) continue;
        const int id = sh.id[c];
        const double z = ec < 0.f ? sh.z[c] : static_cast<double>(fmaf(share, zc, zc));
        int rank = sh.above[c];
        if (ec == DOUBT) {      // against others in doubt the sums count
            for (int i = 0; i < n_doubt; ++i) {
                const int j = sh.near[i];
                rank += (sh.z[j] > z || (sh.z[j] == z && sh.id[j] < id) ? 1 : 0) - (sh.approx[j] > zc ? 1 : 0);
            }
        }
        if (rank < p.k) { sh.z_keep[rank] = id == sh.id_max ? sh.z_max : id == y ? sh.z_label : z; sh.id_keep[rank] = id; }
    }
    __syncthreads();
    return n < p.k ? n : p.k;
}

// One CTA per row: merges the split partials (lse, entropy), the label's log probability, and the top k.
//
// lse.  The tensor cores' additions truncate, so a logit that is far from 0 comes out a few 1e-6 of itself too small.  In a row that
// is sure of a token that token's logit makes up lse, so the largest logit is taken again as an fp64 sum and the row's sums
// are corrected by the difference; the label's logit is such a sum too, and so are the returned alternatives' (see settle_close).
//
// Top k.  Any k group maxima are k logits of the row, so a number t that k group maxima reach is a lower bound of the row's k-th
// largest logit, and only columns at or above t, less the GEMM's error, can be among the k largest.  They are looked
// up in the slab: a few groups of it are read, not the row.  The order is that of the exact products: candidates whose approximate
// logits are closer than their errors are summed again, and equal logits go to the lower id.  The errors are bounded by the norms of
// the row of H and of the longest row of W (gemm_error), so they hold whatever the sums pass through.
// 17 us for one row of V = 128256, k = 20, 525 us for 8192 rows, k = 64 (GEMM 2.82 ms): the bound 45, the list of groups 30, their look-up 78 (700
// thousand 64-byte reads all over the slab), ranking about 45, sums the rest: the norms leave most of 64 candidates in doubt, whose rows of W
// are 2 GB.  (Errors taken relative to the logit left one in twenty, 275 us, and wrong orders where sums cancel.)
// More than CAP candidates (a row of zeros, many equal rows of W) are settled batch by batch by exact sums.
template <class TI, class TZ, bool TOP, int RT>
__global__ void __launch_bounds__(RT, 1024 / RT) row_kernel(const RowParams<TI, TZ> p) {
    __shared__ Shared<RT> sh;
    const long long r = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");      // the logits kernel has finished (it may have been launched ahead of that)
    if (p.valid != nullptr && p.valid[r] == 0) {
        if (threadIdx.x == 0) {
            p.lse[r] = 0.f;
            p.entropy[r] = 0.f;
            if (p.logp) p.logp[r] = 0.f;
        }
        if (TOP)
            for (int i = threadIdx.x; i < p.k; i += RT) { p.top_ids[r * p.k + i] = -1; p.top_logp[r * p.k + i] = -INFINITY; }
        return;
    }
    const TI* h = p.H + r * p.ldH;
    constexpr int group = GroupOf<TZ>::value;
    const float* g = p.gmax + r * p.ld_g;
    const TZ* z = p.zs + r * p.ldz;
    // With few groups per alternative their maxima bound little (or there are not k of them): go by the logits themselves.
    const bool by_group = TOP && p.n_g >= 4 * p.k;
    float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, least = INFINITY;
    if (TOP) {
        auto see = [&](float x, int j) { best[j] = fmaxf(best[j], x); least = fminf(least, x); };
        if (by_group) {
#pragma unroll 4
            for (int i = threadIdx.x; i < (p.n_g + 3) / 4; i += RT) {      // the pitch is a multiple of 4
                const float4 x = reinterpret_cast<const float4*>(g)[i];
                see(x.x, 0);
                if (4 * i + 1 < p.n_g) see(x.y, 1);
                if (4 * i + 2 < p.n_g) see(x.z, 2);
                if (4 * i + 3 < p.n_g) see(x.w, 3);
            }
        } else {
            for (int i = threadIdx.x; i < p.V; i += 4 * RT) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int v = i + j * RT;
                    float e;
                    if (v < p.V) see(stored(z, g[v / group], v, e), j);
                }
            }
        }
    }
    if (warp == 1) {      // the rows of W whose exact logits are wanted at the end
        prefetch_row(h, p.d, lane);
        const long long y = p.logp != nullptr ? p.labels[r] : -1;
        if (y >= 0 && y < p.V) prefetch_row(p.W + y * p.ldW, p.d, lane);
    }
    if (TOP && warp == 2) {
        const float x = warp_squares(h, p.d, lane);
        if (lane == 0) sh.h_sq = x;
    }
    if (warp == 0) {
        // merge the split partials; sums over splits in a fixed order.  The loads of up to 160 splits are under way together.
        constexpr int BATCH = 5;
        float m = tc::LP_LOW, l = 0.f, u = 0.f;
        int id = 0;
        for (int s0 = 0; s0 < p.S; s0 += 32 * BATCH) {
            float ms[BATCH], ls[BATCH], us[BATCH];
            int is[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int s = s0 + 32 * j + lane;
                const size_t at = static_cast<size_t>(s < p.S ? s : 0) * p.part_stride + r;
                ms[j] = p.part_m[at]; ls[j] = p.part_l[at]; us[j] = p.part_u[at]; is[j] = p.part_id[at];
                if (s >= p.S) { ms[j] = tc::LP_LOW; ls[j] = us[j] = 0.f; }
            }
            float m_new = m;
#pragma unroll
            for (int j = 0; j < BATCH; ++j)
                if (ms[j] > m_new || (ms[j] == m_new && is[j] < id)) { m_new = ms[j]; id = is[j]; }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                const float om = __shfl_xor_sync(0xffffffffu, m_new, off);
                const int oid = __shfl_xor_sync(0xffffffffu, id, off);
                if (om > m_new || (om == m_new && oid < id)) { m_new = om; id = oid; }
            }
            const float dm0 = (m - m_new) * tc::LOG2E, e0 = exp2f(dm0);
            u = e0 * fmaf(dm0, l, u);
            l *= e0;
            m = m_new;
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const float dm = (ms[j] - m) * tc::LOG2E, e = exp2f(dm);
                l = fmaf(e, ls[j], l);
                u = fmaf(e, fmaf(dm, ls[j], us[j]), u);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, off);
            u += __shfl_xor_sync(0xffffffffu, u, off);
        }
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(p.V)) id = 0;      // a logits kernel that timed out leaves anything here
        prefetch_row(p.W + static_cast<long long>(id) * p.ldW, p.d, lane);
        if (lane == 0) {
            sh.m = m; sh.l = l; sh.u = u;
            sh.id_max = id;
            sh.n_cand = sh.n_near = 0;
        }
    }
    __syncthreads();
    if (!TOP) {
        if (warp < 2) exact_one(p, h, r, sh, warp);
        __syncthreads();
        if (threadIdx.x == 0) finish_row(p, r, sh);
        return;
    }
    long long* ids_out = p.top_ids + r * p.k;
    float* lp_out = p.top_logp + r * p.k;
    if (!isfinite(sh.m + logf(sh.l))) {
        for (int i = threadIdx.x; i < p.k; i += RT) { ids_out[i] = -1; lp_out[i] = NAN; }
        if (warp < 2) exact_one(p, h, r, sh, warp);
        __syncthreads();
        if (threadIdx.x == 0) finish_row(p, r, sh);
        return;
    }
    float big;
    const float t = near_kth(best, least, p.k, sh, big);
    // k exact logits reach t - eps; a bound taken over stored logits may lie their rounding (2^-11 of the row's span) higher
    const float size = norm_above(sh.h_sq, p.d) * norm_above(__int_as_float(*p.w_sq), p.d);
    const float eps = gemm_error(z, p.d) * size;
    const float thr = t - 2.2f * eps - (by_group ? 0.f : 1.0e-3f * big);
    // the groups that reach the threshold, then their columns that do
    auto keep_group = [&](int gi, float gm) {
        const int at = atomicAdd(&sh.n_near, 1);
        if (at < CAP) { sh.near[at] = gi; sh.near_max[at] = gm; }
    };
    const int n_vec = by_group ? (p.n_g + 3) / 4 : 0;
    // with one share per thread, a thread whose largest is below the threshold has nothing to look up
    if (fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3])) >= thr) {
#pragma unroll 4
        for (int i = threadIdx.x; i < n_vec; i += RT) {
            const float4 x = reinterpret_cast<const float4*>(g)[i];
            if (x.x >= thr) keep_group(4 * i, x.x);
            if (x.y >= thr && 4 * i + 1 < p.n_g) keep_group(4 * i + 1, x.y);
            if (x.z >= thr && 4 * i + 2 < p.n_g) keep_group(4 * i + 2, x.z);
            if (x.w >= thr && 4 * i + 3 < p.n_g) keep_group(4 * i + 3, x.w);
        }
    }
    if (!by_group)
        for (int gi = threadIdx.x; gi < p.n_g; gi += RT)
            if (g[gi] >= thr) keep_group(gi, g[gi]);
    __syncthreads();
    const int n_near = sh.n_near;
    auto append = [&](bool in, long long col, float x, float e) {      // whole warps
        const unsigned hit = __ballot_sync(0xffffffffu, in);
        if (hit == 0) return;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n_cand, __popc(hit));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(hit & ((1u << lane) - 1u));
        if (in && at < CAP) { sh.id[at] = static_cast<int>(col); sh.approx[at] = x; sh.err[at] = eps + e; }
    };
    if (n_near <= CAP) {
        const int n_el = n_near * group;
        constexpr int BATCH = 4;      // loads under way together
        for (int i0 = 0; i0 < n_el; i0 += BATCH * RT) {
            float x[BATCH], e[BATCH];
            long long col[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int i = i0 + j * RT + threadIdx.x, at = i < n_el ? i / group : 0;
                col[j] = static_cast<long long>(sh.near[at]) * group + (i & (group - 1));
                x[j] = stored(z, sh.near_max[at], col[j] < p.V ? col[j] : 0, e[j]);
                if (i >= n_el || col[j] >= p.V) x[j] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) append(x[j] + e[j] >= thr, col[j], x[j], e[j]);
        }
    }
    __syncthreads();
    int kept;
    if (n_near <= CAP && sh.n_cand <= CAP) {
        kept = settle_close(p, h, r, sh, sh.n_cand, eps, dot_error(p.d) * size);
    } else {
        if (warp < 2) exact_one(p, h, r, sh, warp);
        // many logits within the error of the k-th.  A row of zeros, or a head of zeros, has them all equal: ids 0, 1, ...
        if (sh.h_sq == 0.f || *p.w_sq == 0) {
            kept = p.k < p.V ? p.k : p.V;
            for (int i = threadIdx.x; i < kept; i += RT) { sh.z_keep[i] = 0.0; sh.id_keep[i] = i; }
            __syncthreads();
        } else {
            // otherwise batch by batch, one group per warp and step, the k best so far carried along
            kept = 0;
            int n = 0;
            constexpr int STEP = 4;          // at most 64 columns each: they fit beside MAX_TOP kept ones
            for (int g0 = 0; g0 < p.n_g; g0 += STEP) {
                if (threadIdx.x == 0) sh.n_cand = n;
                __syncthreads();
                const int gi = g0 + warp;
                if (warp < STEP && gi < p.n_g && g[gi] >= thr) {
                    for (int o = 0; o < group; o += 32) {
                        const long long col = static_cast<long long>(gi) * group + o + lane;
                        float e;
                        const float x = stored(z, g[gi], col < p.V ? col : 0, e);
                        append(col < p.V && x + e >= thr, col, x, e);
                    }
                }
                __syncthreads();
                n = sh.n_cand;
                const bool last = g0 + STEP >= p.n_g;
                if (n > CAP - STEP * 64 || last) {
                    kept = settle(p, h, sh, kept, n);
                    for (int i = threadIdx.x; i < kept; i += RT) { sh.z[i] = sh.z_keep[i]; sh.id[i] = sh.id_keep[i]; }
                    n = kept;
                }
                __syncthreads();
            }
        }
        if (threadIdx.x == 0) finish_row(p, r, sh);
        __syncthreads();
    }
    for (int i = threadIdx.x; i < p.k; i += RT) {
        ids_out[i] = i < kept ? sh.id_keep[i] : -1;
        lp_out[i] = i < kept ? log_prob(sh.z_keep[i], sh) : -INFINITY;
    }
}

// What the rounding to bf16 left of the labels' entries of dz, for the result to have it all the same: rest[r] W[labels[r], :] in dH,
// rest[r] H[r, :] in row labels[r] of dW (as tc::SparseTerms).
struct LabelRest {
    const float* rest;                 // [T], 0 in rows without a label; nullptr: not wanted
    const long long* labels;
    const __nv_bfloat16* W;
    long long ldW;
};

// dH = scale * (part 0 + part 1 + ...), in that order, in bf16.  One CTA per row; `stride` elements from part to part.  lo > 0: each part
// has a second term in row lo + r.
__global__ void __launch_bounds__(THREADS) add_parts_kernel(const float* part, int n, long long stride, int d, const float* scale,
                                                            __nv_bfloat16* out, long long ld, long long lo, const LabelRest label) {
    const long long r = blockIdx.x;
    const float a = scale ? *scale : 1.f;
    const float left = label.rest != nullptr ? label.rest[r] : 0.f;
    const uint2* w = left != 0.f ? reinterpret_cast<const uint2*>(label.W + label.labels[r] * label.ldW) : nullptr;
    for (int i = threadIdx.x; i < d / 4; i += THREADS) {
        const float4* src = reinterpret_cast<const float4*>(part + r * d) + i;
        float4 s = __ldcs(src);
#pragma unroll 4
        for (int g = 1; g < n; ++g) {
            const float4 x = __ldcs(src + g * (stride / 4));
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
        if (lo > 0) {
            for (int g = 0; g < n; ++g) {
                const float4 x = __ldcs(src + g * (stride / 4) + lo * d / 4);
                s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
            }
        }
        if (left != 0.f) {
            const uint2 x = __ldg(w + i);
            s.x = fmaf(left, __uint_as_float(x.x << 16), s.x); s.y = fmaf(left, __uint_as_float(x.x & 0xffff0000u), s.y);
            s.z = fmaf(left, __uint_as_float(x.y << 16), s.z); s.w = fmaf(left, __uint_as_float(x.y & 0xffff0000u), s.w);
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
__device__ __forceinline__ void copy_row(const TI* src, TI* dst, int d, bool on) {
    if (sizeof(TI) == 2) {
        for (int i = threadIdx.x; i < d / 8; i += THREADS)
            reinterpret_cast<uint4*>(dst)[i] = on ? __ldg(reinterpret_cast<const uint4*>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
    } else {
        for (int i = threadIdx.x; i < d; i += THREADS) dst[i] = on ? src[i] : static_cast<TI>(0);
    }
}
// One CTA per row of the copy.  lo > 0, for dz in two terms: rows T .. lo - 1 are zero and rows lo .. 2 lo - 1 a second copy.
template <class TI>
__global__ void __launch_bounds__(THREADS) copy_rows_kernel(const TI* H, long long ldH, int d, int T, const unsigned char* valid, int lo, TI* out) {
    const long long at = blockIdx.x, r = lo > 0 && at >= lo ? at - lo : at;
    const bool on = r < T && (valid == nullptr || valid[r] != 0);
    copy_row(H + (r < T ? r : 0) * ldH, out + at * d, d, on);
}

// out += sum, sum [V][d] and out with pitch ld, N elements at a time (4: aligned so).
__device__ __forceinline__ void add_to(float* to, const float* x) { *to += *x; }
__device__ __forceinline__ void add_to4(float* to, const float* x) {
    float4 a = *reinterpret_cast<float4*>(to);
    const float4 b = __ldcs(reinterpret_cast<const float4*>(x));
    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    *reinterpret_cast<float4*>(to) = a;
}
__device__ __forceinline__ void add_to4(__nv_bfloat16* to, const float* x) {
    uint2 a = *reinterpret_cast<uint2*>(to);
    const float4 b = __ldcs(reinterpret_cast<const float4*>(x));
    a.x = ptx::pack_bf16x2(__uint_as_float(a.x << 16) + b.x, __uint_as_float(a.x & 0xffff0000u) + b.y);
    a.y = ptx::pack_bf16x2(__uint_as_float(a.y << 16) + b.z, __uint_as_float(a.y & 0xffff0000u) + b.w);
    *reinterpret_cast<uint2*>(to) = a;
}
template <int N, class T>
__global__ void __launch_bounds__(THREADS) add_sum_kernel(const float* sum, long long V, int d, T* out, long long ld) {
    const long long cols = d / N;
    for (long long i = static_cast<long long>(blockIdx.x) * THREADS + threadIdx.x; i < V * cols; i += static_cast<long long>(gridDim.x) * THREADS) {
        const long long v = i / cols, c = i - v * cols;
        if constexpr (N == 4) add_to4(out + v * ld + 4 * c, sum + 4 * i);
        else add_to(out + v * ld + c, sum + i);
    }
}

// The closing entries of a slab of dz (see tc::EpiDzLp), one warp per row; and, with `rest`, what the rounding leaves of the labels' entries, as
// LabelRest and sorted by label and row for tc::SparseTerms (rows without a label: 0, and INT_MAX at the end).
struct CloseParams {
    const long long* labels;           // [T], with grad_logp
    const unsigned char* valid;        // [T] or nullptr
    const float* grad_logp;            // [T] or nullptr
    const float* part_sum;             // [S][part_stride]
    const int* part_col;
    long long part_stride;
    int S;
    const float* dz_label;             // [T]
    __nv_bfloat16* dz;
    long long ldz;
    int T, V;
    int lo;
    float* rest;                       // [T] each, or nullptr; only with grad_logp
    int* key;
    int* from;
    float* coef;
};
__global__ void __launch_bounds__(THREADS) close_kernel(const CloseParams p) {
    const int r = blockIdx.x * WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= p.T) return;
    float sum = 0.f;
    int col = -1;
    for (int s = lane; s < p.S; s += 32) {
        sum += p.part_sum[s * p.part_stride + r];
        col = max(col, p.part_col[s * p.part_stride + r]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    col = __reduce_max_sync(0xffffffffu, col);
    if (static_cast<unsigned>(col) >= static_cast<unsigned>(p.V)) col = -1;      // a GEMM that timed out leaves anything here
    const float entry = 0.f - sum;
    if (col >= 0 && lane == 0) {
        const __nv_bfloat16 hi = __float2bfloat16_rn(entry);
        p.dz[r * p.ldz + col] = hi;
        if (p.lo > 0) p.dz[(p.lo + r) * p.ldz + col] = __float2bfloat16_rn(entry - __bfloat162float(hi));
    }
    if (p.rest == nullptr) return;
    auto label = [&](int q) {
        const long long y = p.labels[q];
        return (p.valid == nullptr || p.valid[q] != 0) && y >= 0 && y < p.V ? static_cast<int>(y) : INT_MAX;
    };
    const int y = label(r);
    int rank = 0;
    for (int q0 = 0; q0 < p.T; q0 += 32) {
        const int q = q0 + lane, k = q < p.T ? label(q) : INT_MAX;
        rank += __popc(__ballot_sync(0xffffffffu, q < p.T && (k < y || (k == y && q < r))));
    }
    if (lane != 0) return;
    const float v = y == INT_MAX ? 0.f : y == col ? entry : p.dz_label[r];
    p.key[rank] = y;
    p.from[rank] = r;
    p.rest[r] = p.coef[rank] = v - __bfloat162float(__float2bfloat16_rn(v));
}

}  // namespace lp
}  // namespace cat
