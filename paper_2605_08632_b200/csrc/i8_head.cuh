// Operators on an LM head kept in 8 bits: rows held as integers with a scale each, the product of such rows, and the softmax cross
// entropy over it.
//
//   xq = 127 x / max |x| rounded to integers, sx = max |x| / 127;   z[t, v] = sx[t] sw[v] sum_i xq[t, i] wq[v, i]
//   with o = log sum_{v != y} exp z:   nll = log(1 + exp(o - z_y)),   lse = z_y + nll,   1 - p_y = 1 - exp(-nll)
//   dz[v] = g (1 - p_y) (exp(z_v - o) - [v = y]),    dX = (dz sw) Wq
//
// The label is kept out of the softmax sum because a row that is sure of it has lse - z_y and 1 - p_y far below lse's own rounding.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "logprob.cuh"
#include "ptx.cuh"
#include "tc_gemm.cuh"

namespace cat {
namespace i8 {

constexpr int THREADS = 256;
constexpr float LOW2 = -3.4028234664e38f;        // "no column yet", in units of log2: finite, so that LOW2 - LOW2 is 0, and below every logit
constexpr float NEAR_HALF = 0.49998f;   // a distance from an integer that is 2^-16 short of a half, or more: what decides it is past binary32

// ------------------------------------------------------------------------------ rows to integers
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// 127 x / most to the nearest integer, halves to the even one, exactly.  inv = 127 / most; the product x inv is off by less than 2^-16, so only where it
// comes that near to a half is more to be known: on which side of the odd number m = 2 (half) 254 x / most lies.  a + e is m most
// exactly, and the fma's result is exact because its two sides nearly cancel.
__device__ __forceinline__ float past_half(float x, float most, float n, float off) {
    const float side = off < 0.f ? -1.f : 1.f, m = fmaf(2.f, n, side);
    const float a = m * most, e = fmaf(m, most, -a), d = fmaf(254.f, x, -a);
    const bool beyond = side > 0.f ? d > e : d < e, odd = (static_cast<int>(n) & 1) != 0;
    return beyond || (d == e && odd) ? n + side : n;
}
// rows whose largest value is too small or too large for that: 127 x is exact in 64 bits, and no quotient of a 31-bit by a 24-bit number is within
// 2^-53 of a half without being one
__device__ __noinline__ int exact_steps(float x, float most) { return static_cast<int>(rint(127.0 * static_cast<double>(x) / static_cast<double>(most))); }
__device__ __forceinline__ float inverse_step(float most) { return most > 1.0e-30f && most < 1.0e30f ? 127.f / most : 0.f; }
__device__ __forceinline__ int steps_of(float x, float inv, float most) {
    if (inv == 0.f) return exact_steps(x, most);
    const float n = rintf(x * inv), off = fmaf(x, inv, -n);
    return static_cast<int>(fabsf(off) < NEAR_HALF ? n : past_half(x, most, n, off));
}

// What else the kernel that makes a call's tokens into integers does: it clears the workspace's header and finds the largest finite |scale| of the
// head, in MOST_PARTS parts.  Kept out of launches of their own: a small call is mostly the time between kernels.
constexpr int MOST_PARTS = 32;
struct CallSetup {
    int* header;           // status and worker claims, or nullptr
    int header_ints;
    const float* sw;       // scales of the head, or nullptr: MOST_PARTS more CTAs
    int V;
    int* most;             // [MOST_PARTS] float bits, inside the header (not cleared)
};
__device__ __forceinline__ void set_up_call(const CallSetup& c, int part) {
    if (part < 0) {
        if (c.header != nullptr && blockIdx.x == 0)
            for (int i = threadIdx.x; i < c.header_ints; i += THREADS) {
                int* at = c.header + i;
                if (c.most == nullptr || at < c.most || at >= c.most + MOST_PARTS) *at = 0;
            }
        return;
    }
    __shared__ unsigned s_part[THREADS / 32];
    unsigned bits = 0;
    for (long long v = static_cast<long long>(part) * THREADS + threadIdx.x; v < c.V; v += MOST_PARTS * THREADS) {
        const unsigned x = __float_as_uint(c.sw[v]) & 0x7fffffffu;
        if (x < 0x7f800000u) bits = max(bits, x);
    }
    bits = __reduce_max_sync(0xffffffffu, bits);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = bits;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < THREADS / 32; ++i) bits = max(bits, s_part[i]);
        c.most[part] = static_cast<int>(bits);
    }
}

// Rows of any length and alignment, one CTA each.
template <class T>
__global__ void __launch_bounds__(THREADS) quantize_kernel(const T* X, long long ldX, int rows, int d, int8_t* Xq, long long ldq, int pad, float* scale,
                                                           const CallSetup setup) {
    __shared__ unsigned s_most[THREADS / 32];
    const long long r = blockIdx.x;
    ptx::launch_dependents();
    set_up_call(setup, r < rows ? -1 : static_cast<int>(r) - rows);
    if (r >= rows) return;
    const T* x = X + r * ldX;
    unsigned bits = 0;                      // of |x|: ordered like the values, infinities and NaN above them
    const unsigned n = static_cast<unsigned>(d), n_out = static_cast<unsigned>(pad);          // an index may step past 2^31
    for (unsigned i = threadIdx.x; i < n; i += THREADS) bits = max(bits, __float_as_uint(to_float(x[i])) & 0x7fffffffu);
    bits = __reduce_max_sync(0xffffffffu, bits);
    if ((threadIdx.x & 31) == 0) s_most[threadIdx.x >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) bits = max(bits, s_most[i]);
    const float most = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u, any = finite && bits != 0u;
    const float inv = any ? inverse_step(most) : 0.f;
    int8_t* q = Xq + r * ldq;
    for (unsigned i = threadIdx.x; i < n_out; i += THREADS) q[i] = any && i < n ? static_cast<int8_t>(steps_of(to_float(x[i]), inv, most)) : 0;
    if (threadIdx.x == 0) scale[r] = finite ? most / 127.f : __uint_as_float(0x7fc00000u);
}

// Eight neighbouring values, 16 or 32 bytes.
template <class T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
    uint4 x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void clear() { x = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void set(const uint32_t* w) { x = make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ unsigned most() const {          // of |x|, as float bits
        const unsigned m = __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
    __device__ __forceinline__ void values(float (&f)[8]) const {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = __ldg(reinterpret_cast<const float4*>(p));
        b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void set(const uint32_t* w) {
        a = make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
        b = make_float4(__uint_as_float(w[4]), __uint_as_float(w[5]), __uint_as_float(w[6]), __uint_as_float(w[7]));
    }
    __device__ __forceinline__ void values(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
        f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ unsigned most() const {
        float f[8];
        values(f);
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
        return m;
    }
};

// Eight values at any address of their type: the whole 16-byte pieces around them, moved into place.  [lo, hi): the matrix; a piece that reaches past it (at
// its first and last value only) is put together value by value.  Values from `count` on are zero.
template <class T>
__device__ __forceinline__ Eight<T> eight_at(const T* x, int count, uintptr_t lo, uintptr_t hi) {
    constexpr int WORDS = 2 * sizeof(T), PIECES = WORDS / 4 + 1;          // of the eight; 16-byte pieces that they may touch
    const uintptr_t at = reinterpret_cast<uintptr_t>(x), base = at & ~static_cast<uintptr_t>(15);
    const unsigned shift = static_cast<unsigned>(at - base);
    uint32_t w[4 * PIECES];
#pragma unroll
    for (int g = 0; g < PIECES; ++g) {
        const uintptr_t p = base + 16 * g;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (p < at + count * sizeof(T)) {
            if (p >= lo && p + 16 <= hi) {
                v = __ldg(reinterpret_cast<const uint4*>(p));
            } else {
                uint32_t part[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < static_cast<int>(16 / sizeof(T)); ++j) {
                    const uintptr_t e = p + j * sizeof(T);
                    if (e >= lo && e < hi) {
                        if (sizeof(T) == 4) part[j & 3] = __ldg(reinterpret_cast<const uint32_t*>(e));
                        else part[(j >> 1) & 3] |= static_cast<uint32_t>(__ldg(reinterpret_cast<const uint16_t*>(e))) << (16 * (j & 1));
                    }
                }
                v = make_uint4(part[0], part[1], part[2], part[3]);
            }
        }
        w[4 * g] = v.x; w[4 * g + 1] = v.y; w[4 * g + 2] = v.z; w[4 * g + 3] = v.w;
    }
#pragma unroll
    for (int k = 8; k >= 4; k -= 4)                                       // by two words, by one
        if (shift & k) {
#pragma unroll
            for (int j = 0; j + k / 4 < 4 * PIECES; ++j) w[j] = w[j + k / 4];
        }
    if (sizeof(T) == 2 && (shift & 2)) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], 16);
    }
#pragma unroll
    for (int j = 0; j < WORDS; ++j) {
        if (sizeof(T) == 4) w[j] = j < count ? w[j] : 0u;
        else w[j] = 2 * j + 1 < count ? w[j] : 2 * j < count ? w[j] & 0xffffu : 0u;
    }
    Eight<T> r;
    r.set(w);
    return r;
}

// steps_of for eight values, as far as binary32 goes; `open`: one of them is too near to a half for that.  Adding 1.5 2^23 rounds to the nearest integer,
// halves to the even one, and leaves it in the low bits.
//   bf16: with 8-bit significands, 127 x / most is a half exactly or off it by 1 / (254 * 255) of itself or more.  The binary32 product, off by 2^-22,
//   is rounded to 20 bits first (Veltkamp's splitting), which makes halves of all that are ones, and moves none of the others across one.
//   fp32: the distance to the integer says whether a half is near.
template <class T>
__device__ __forceinline__ uint2 eight_steps(const float (&x)[8], float inv, bool& open) {
    constexpr float MAGIC = 12582912.f;
    const uint64_t inv2 = ptx::pack_f32x2(inv, inv), magic2 = ptx::pack_f32x2(MAGIC, MAGIC), minus2 = ptx::pack_f32x2(-1.f, -1.f);
    uint32_t m[8];
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint64_t x2 = ptx::pack_f32x2(x[i], x[i + 1]);
        uint64_t t2;
        if (sizeof(T) == 2) {
            const uint64_t p2 = ptx::mul_f32x2(x2, inv2), c2 = ptx::mul_f32x2(p2, ptx::pack_f32x2(17.f, 17.f));
            const uint64_t hi2 = ptx::fma_f32x2(ptx::fma_f32x2(p2, minus2, c2), minus2, c2);          // c - (c - p): 20 bits of p
            t2 = ptx::add_f32x2(hi2, magic2);
        } else {
            t2 = ptx::fma_f32x2(x2, inv2, magic2);
            float off0, off1;
            ptx::unpack_f32x2(ptx::fma_f32x2(x2, inv2, ptx::fma_f32x2(t2, minus2, magic2)), off0, off1);
            far = ptx::max3_f32(far, fabsf(off0), fabsf(off1));
        }
        float t0, t1;
        ptx::unpack_f32x2(t2, t0, t1);
        m[i] = __float_as_uint(t0);
        m[i + 1] = __float_as_uint(t1);
    }
    open = far >= NEAR_HALF;
    return make_uint2(__byte_perm(__byte_perm(m[0], m[1], 0x0040), __byte_perm(m[2], m[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(m[4], m[5], 0x0040), __byte_perm(m[6], m[7], 0x0040), 0x5410));
}
// eight values that binary32 alone does not settle, read once more; a call of its own, so that its registers are not the kernel's
template <class T>
__device__ __noinline__ void settle_eight(const T* x, int8_t* q, int count, float inv, float most) {
#pragma unroll 1
    for (int i = 0; i < count; ++i) q[i] = static_cast<int8_t>(steps_of(to_float(x[i]), inv, most));
}

// Rows of up to 256 EIGHTS WARPS values: WARPS warps each, one pass, the values kept in registers.  ANY: of any length and at any address, else whole eights
// on 16-byte boundaries.  The integers' rows begin on 8-byte boundaries.  Bound by HBM
// where rows are many; four CTAs on an SM keep enough loads under way (128256 x 2048: 113 us, 7.0 TB/s; before halves were settled
// without a branch 155 with four, 177 with three, 184 with five).
constexpr int MOST_EIGHTS = 8;           // per lane
template <class T, int WARPS, int EIGHTS, bool ANY>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 || EIGHTS < MOST_EIGHTS ? 4 : 2) quantize_rows_kernel(const T* X, long long ldX, int rows, int d, int8_t* Xq, long long ldq, int pad, float* scale,
                                                                const CallSetup setup) {
    constexpr int PER_CTA = THREADS / 32 / WARPS;
    __shared__ unsigned s_most[THREADS / 32];
    const int row_ctas = static_cast<int>((static_cast<unsigned>(rows) + PER_CTA - 1u) / PER_CTA);
    ptx::launch_dependents();
    set_up_call(setup, static_cast<int>(blockIdx.x) < row_ctas ? -1 : static_cast<int>(blockIdx.x) - row_ctas);
    if (static_cast<int>(blockIdx.x) >= row_ctas) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r = static_cast<long long>(blockIdx.x) * PER_CTA + warp / WARPS;
    const int first = (warp % WARPS) * 32 + lane, n = ANY ? (d + 7) >> 3 : d >> 3;        // this lane's eights: first + 32 WARPS i
    const bool on = r < rows;
    Eight<T> x[EIGHTS];
    unsigned bits = 0;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(X), hi = reinterpret_cast<uintptr_t>(X + (rows - 1) * ldX + d);
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) {
        const int g = first + 32 * WARPS * i;
        if (!on || g >= n) x[i].clear();
        else if (!ANY) x[i].load(X + r * ldX + 8 * g);
        else x[i] = eight_at(X + r * ldX + 8 * g, min(8, d - 8 * g), lo, hi);
    }
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) bits = max(bits, x[i].most());
    bits = __reduce_max_sync(0xffffffffu, bits);
    if (WARPS > 1) {
        if (lane == 0) s_most[warp] = bits;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WARPS; ++i) bits = max(bits, s_most[warp / WARPS * WARPS + i]);
    }
    if (!on) return;
    const float most = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u, any = finite && bits != 0u;
    const float inv = any ? inverse_step(most) : 0.f;
    int8_t* q = Xq + r * ldq;
    unsigned open = 0;                   // eights still to be settled
#pragma unroll
    for (int i = 0; i < EIGHTS; ++i) {
        const int g = first + 32 * WARPS * i;
        if (g >= n) break;
        float f[8];
        x[i].values(f);
        bool near;
        uint2 b = eight_steps<T>(f, inv, near);
        if (!any) b = make_uint2(0u, 0u);
        if (!ANY || 8 * g + 8 <= pad) {
            *reinterpret_cast<uint2*>(q + 8 * g) = b;
        } else {                         // the last ones of a row whose padding is not to be written
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (8 * g + j < d) q[8 * g + j] = static_cast<int8_t>((j < 4 ? b.x >> (8 * j) : b.y >> (8 * j - 32)) & 255u);
        }
        open |= near || inv == 0.f ? 1u << i : 0u;
    }
    if (any) {
        while (open != 0) {
            const int g = first + 32 * WARPS * (__ffs(open) - 1);
            open &= open - 1;
            settle_eight(X + r * ldX + 8 * g, q + 8 * g, ANY ? min(8, d - 8 * g) : 8, inv, most);
        }
    }
    if (warp % WARPS == 0 && lane == 0) {
        if (pad > 8 * n) *reinterpret_cast<uint2*>(q + 8 * n) = make_uint2(0u, 0u);          // the other half of 16 bytes
        scale[r] = finite ? most / 127.f : __uint_as_float(0x7fc00000u);
    }
}

struct Head {
    const int8_t* xq;      // [T][ldq]
    const float* sx;       // [T]
    const int8_t* wq;      // [V][ldw]
    const float* sw;       // [V]
    long long ldq, ldw;
    int T, V, d;
};

// ------------------------------------------------------------------------------ epilogues of the 8-bit product
// The GEMM of tc_gemm.cuh on integers (kind::i8, exact int32 sums, twice the bf16 rate).  A tile is done in half the time, so two sets of four
// warps share its columns.
using OutStage1 = tc::OutStageOf<1>;

// Chunks of 32 columns of this warp's half of a tile, body(c, v) for each that holds columns below ncols: the next one is on its way from
// tensor memory while the warp works on one.
template <class F>
__device__ __forceinline__ void walk_half(uint32_t taddr, int ncols, F&& body) {
    const int c0 = ((threadIdx.x - 64) >> 7) * 4;
    if (c0 * 32 >= ncols) return;
    uint32_t a[32], b[32];
    ptx::tmem_ld_32x32(taddr + c0 * 32, a);
#pragma unroll 1
    for (int c = c0; c < c0 + 4 && c * 32 < ncols; c += 2) {
        ptx::tmem_ld_wait(a);
        ptx::tmem_ld_32x32(taddr + (c + 1) * 32, b);
        body(c, a);
        ptx::tmem_ld_wait(b);
        if (c + 2 < c0 + 4) ptx::tmem_ld_32x32(taddr + (c + 2) * 32, a);
        if ((c + 1) * 32 < ncols) body(c + 1, b);
    }
    ptx::tmem_ld_wait();
}

// The scales (or biases) of the 128 columns of a warp's half of a tile, four to a lane: column 32 j + lane.  They are fetched one tile ahead and handed
// round by shuffles; loads of the same addresses by all lanes, chunk by chunk, waited for L2 every time (loss of 300 x 1024 x 151936 85 us).
struct Columns {
    float x[4];
    __device__ __forceinline__ void load(const float* p, int n_tile, int V) {
        const int col = n_tile * tc::BN + static_cast<int>((threadIdx.x - 64) >> 7) * 128 + static_cast<int>(threadIdx.x & 31);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = col + 32 * j < V ? __ldg(p + col + 32 * j) : 0.f;
    }
    // this lane's value of chunk c
    __device__ __forceinline__ float chunk(int c) const {
        const int j = c & 3;
        return j < 2 ? (j == 0 ? x[0] : x[1]) : (j == 2 ? x[2] : x[3]);
    }
};

// integer sums times the channels' scales, `mine` the lane's
__device__ __forceinline__ void scaled(const uint32_t (&v)[32], float mine, float (&f)[32]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2)
        ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(__int2float_rn(static_cast<int>(v[i])), __int2float_rn(static_cast<int>(v[i + 1]))),
                                         ptx::pack_f32x2(__shfl_sync(0xffffffffu, mine, i), __shfl_sync(0xffffffffu, mine, i + 1))), f[i], f[i + 1]);
}

// The product itself.  Bound by the traffic between L2 and the SMs where outputs are large: 1000 x 1024 x 151936 139 us, without stores 111.  Whole chunks of 32 columns leave through shared memory and TMA stores (the tensor map ends with them: a store that is cut
// off at the vocabulary's end would still write whole 16 bytes), the last ones from the threads.
template <bool F32>
struct EpiLinear {
    struct Params {
        const float* sx;       // [T]
        const float* sw;       // [V]
        const float* bias;     // [V] or nullptr
        void* Y;               // [T][ldY]
        long long ldY;
        int T, V;
    };
    struct State {
        Columns w, b;
        float sx;
        int row;
    };
    __device__ static __forceinline__ void ahead(const Params& p, State& s, int n_tile) {
        s.w.load(p.sw, n_tile, p.V);
        if (p.bias != nullptr) s.b.load(p.bias, n_tile, p.V);
    }
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * tc::BM + row_in_tile;
        s.sx = s.row < p.T ? p.sx[s.row] : 0.f;
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, int n_next, uint32_t taddr, OutStage1& o) {
        const int col0 = n_tile * tc::BN;
        const int ncols = min(tc::BN, p.V - col0);
        const Columns w = s.w, b = s.b;
        ahead(p, s, n_next);
        walk_half(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            float f[32];
            scaled(v, w.chunk(c), f);
            if (p.bias != nullptr) {
                const float mine = b.chunk(c);
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = __fadd_rn(__fmul_rn(f[i], s.sx), __shfl_sync(0xffffffffu, mine, i));
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] *= s.sx;
            }
            const int live = ncols - c * 32;
            if (live < 32) {
                if (!F32 && (c & 1) != 0) o.flush(col0 + (c >> 1) * 64);          // the chunk before, with whatever is beside it
                if (s.row < p.T) {
                    const long long at = s.row * p.ldY + col0 + c * 32;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (i >= live) continue;
                        if (F32) static_cast<float*>(p.Y)[at + i] = f[i];
                        else static_cast<__nv_bfloat16*>(p.Y)[at + i] = __float2bfloat16(f[i]);
                    }
                }
                return;
            }
            if (F32) {
                o.begin();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    o.put(j, __float_as_uint(f[4 * j]), __float_as_uint(f[4 * j + 1]), __float_as_uint(f[4 * j + 2]), __float_as_uint(f[4 * j + 3]));
                o.flush(col0 + c * 32);
            } else {
                if ((c & 1) == 0) o.begin();
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    o.put((c & 1) * 4 + q, ptx::pack_bf16x2(f[q * 8 + 0], f[q * 8 + 1]), ptx::pack_bf16x2(f[q * 8 + 2], f[q * 8 + 3]),
                          ptx::pack_bf16x2(f[q * 8 + 4], f[q * 8 + 5]), ptx::pack_bf16x2(f[q * 8 + 6], f[q * 8 + 7]));
                if ((c & 1) != 0 || live == 32) o.flush(col0 + (c >> 1) * 64);
            }
        });
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return p.T; }
    __device__ static __forceinline__ void end_item(const Params&, const State&, int) {}
};

// log2 e times a row's scale.  Columns that are not to count are at -infinity, and times this have to stay there: where the scale is 0 (rows of zeros, and rows
// whose largest value is so small that its 127th rounds to 0, with integers up to 127) it is the smallest number that is not, which leaves logits of 0 to within
// 2^-149 of their integer sums times the channel's scale.
__device__ __forceinline__ float log2_scale(float sx) { return sx == 0.f ? __uint_as_float(1u) : sx * tc::LOG2E; }

// Largest logit but the label's and the sum of the exponentials relative to it, in units of log2, and the label's logit.  The largest is rounded up, so
// that no exponent is above 0: rounded to nearest, a logit of 1e10 has one of up to 500 itself.
struct RowSums {
    float m, l;            // running maximum and sum
    float a;               // log2 e times the row's scale
    __device__ __forceinline__ void clear(float sx) { m = LOW2; l = 0.f; a = log2_scale(sx); }
    // 32 columns (without the row's scale), those that are not to count at -infinity
    __device__ __forceinline__ void add(const float (&f)[32]) {
        const float m_new = fmaxf(m, __fmul_ru(tc::max_of(f), a));
        const uint64_t a2 = ptx::pack_f32x2(a, a), nm2 = ptx::pack_f32x2(-m_new, -m_new);
        uint64_t sum2 = ptx::pack_f32x2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x0, x1;
            ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(f[2 * i], f[2 * i + 1]), a2, nm2), x0, x1);
            sum2 = ptx::add_f32x2(sum2, ptx::pack_f32x2(ptx::ex2_approx(x0), ptx::ex2_approx(x1)));
        }
        float s0, s1;
        ptx::unpack_f32x2(sum2, s0, s1);
        l = fmaf(l, ptx::ex2_approx(m - m_new), s0 + s1);
        m = m_new;
    }
};

// Cross entropy.  8192 x 2048 x 128256: 1240 us, 3.5 P operations a second, 2 % above the product without an epilogue; 8192 x 1024 x 151936: 846 us, 14 %.
struct EpiCe {
    struct Params {
        const float* sx;           // [T]
        const float* sw;           // [V]
        const long long* labels;   // [T]
        float* part_m;             // [T][parts]
        float* part_l;
        float* z_label;            // [T], in units of log2
        int parts;                 // 2 n_groups
        int T, V;
    };
    struct State {
        Columns w;
        RowSums r;
        int y, row;
    };
    __device__ static __forceinline__ void ahead(const Params& p, State& s, int n_tile) { s.w.load(p.sw, n_tile, p.V); }
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * tc::BM + row_in_tile;
        s.y = -1;
        float sx = 0.f;
        if (s.row < p.T) {
            sx = p.sx[s.row];
            const long long y = p.labels[s.row];
            if (y >= 0 && y < p.V) s.y = static_cast<int>(y);
        }
        s.r.clear(sx);
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, int n_next, uint32_t taddr, OutStage1&) {
        const int col0 = n_tile * tc::BN;
        const int ncols = min(tc::BN, p.V - col0);
        const Columns w = s.w;
        ahead(p, s, n_next);
        walk_half(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            float f[32];
            const int live = ncols - c * 32;
            scaled(v, w.chunk(c), f);
            if (live < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live) f[i] = -INFINITY;
            }
            const int rel = s.y - (col0 + c * 32);
            if (rel >= 0 && rel < 32) {
                float zy = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == rel) { zy = f[i]; f[i] = -INFINITY; }
                p.z_label[s.row] = zy * s.r.a;
            }
            s.r.add(f);
        });
    }
    __device__ static __forceinline__ int out_rows(const Params&) { return 0; }
    __device__ static __forceinline__ void end_item(const Params& p, const State& s, int group) {
        if (s.row >= p.T) return;
        const long long at = static_cast<long long>(s.row) * p.parts + 2 * group + static_cast<int>((threadIdx.x - 64) >> 7);
        p.part_m[at] = s.r.m;
        p.part_l[at] = s.r.l;
    }
};

// The parts of each row, [T][S], and what follows from them; z_label is read for rows with a label only.  One warp per row: its lanes share the parts out
// and are joined in a fixed order.
__global__ void __launch_bounds__(THREADS) merge_kernel(const float* part_m, const float* part_l, const float* z_label, int S, int T, int V,
                                                        const long long* labels, const unsigned char* valid, float* nll, float* lse) {
    const int lane = threadIdx.x & 31, r = blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
    ptx::grid_dependency_wait();
    if (r >= T) return;
    const float *pm = part_m + static_cast<long long>(r) * S, *pl = part_l + static_cast<long long>(r) * S;
    float m = LOW2;
    for (int s = lane; s < S; s += 32) m = fmaxf(m, pm[s]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    float l = 0.f;
    for (int s = lane; s < S; s += 32) l = fmaf(pl[s], exp2f(pm[s] - m), l);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if (lane != 0) return;
    if (m > LOW2 && l < 0x1p-126f) l = 0x1p-126f;          // past 1e9 the largest logit may lie so far below its rounded value that its own exponential is 0
    if (valid != nullptr && valid[r] == 0) {
        nll[r] = lse[r] = 0.f;
        return;
    }
    constexpr float LN2 = 0.693147180559945309f;
    const long long y = labels[r];
    if (y < 0 || y >= V) {
        nll[r] = 0.f;
        lse[r] = LN2 * (m + log2f(l));
        return;
    }
    const float zy = z_label[r], over = LN2 * ((m - zy) + log2f(l));
    const float n = over > 0.f ? over + log1pf(expf(-over)) : log1pf(expf(over));
    nll[r] = n;
    lse[r] = fmaf(LN2, zy, n);
}

// ------------------------------------------------------------------------------ gradient
// 2^k with (largest scale) 2^k in [2^14, 2^15), and 2^-k.  All lanes of a warp.
__device__ __forceinline__ void fit_half(const int* most, float& up, float& down) {
    static_assert(MOST_PARTS == 32, "one part per lane");
    int e = __reduce_max_sync(0xffffffffu, most[threadIdx.x & 31]) >> 23;       // its biased exponent
    e = e < 20 ? 20 : e > 250 ? 250 : e;
    up = __uint_as_float(static_cast<unsigned>(254 + 14 - e) << 23);
    down = __uint_as_float(static_cast<unsigned>(e - 14) << 23);
}

struct RowGrad {
    float others2;     // log2 sum of the others' exponentials
    float factor;      // g (1 - p_y)
    int y;
    bool on;
};
__device__ __forceinline__ RowGrad row_grad(int r, int T, int V, const long long* labels, const unsigned char* valid, const float* nll, const float* lse,
                                            const float* g) {
    RowGrad a{0.f, 0.f, -1, false};
    if (r >= T || (valid != nullptr && valid[r] == 0)) return a;
    const long long y = labels[r];
    if (y < 0 || y >= V) return a;
    const float rest = -expm1f(-nll[r]);                // 1 - p_y
    a.y = static_cast<int>(y);
    a.factor = g[r] * rest;
    a.on = !(rest < 1.0e-37f);                          // nothing left to tell the others apart: no gradient
    if (!a.on) { a.factor = 0.f; return a; }
    a.others2 = (lse[r] + logf(rest)) * tc::LOG2E;
    return a;
}

// exp(z_v - o) sw_v 2^k, and -sw_y 2^k at the label, as fp16: the rest of the row's factor is applied behind the contraction.  Half precision's 11 bits
// keep the rounding of a row's few large terms below that of the bf16 result (bf16 terms: rows of dX off by up to 2^-8 more).  With the largest scale at
// 2^14 or more, terms from 2^-28 of it up have those bits; smaller ones are off by up to 2^-39 of it.
struct EpiDz {
    struct Params {
        const float* sx;
        const float* sw;
        const long long* labels;
        const unsigned char* valid;
        const float* nll;
        const float* lse;
        const float* g;            // [T] upstream
        const int* most;           // [MOST_PARTS] bits of the largest scale
        float* factor;             // [T] out: g (1 - p_y) 2^-k
        int T, V;
    };
    struct State {
        Columns w;
        RowGrad q;
        float a, up, down;
        int row;
    };
    __device__ static __forceinline__ void ahead(const Params& p, State& s, int n_tile) { s.w.load(p.sw, n_tile, p.V); }
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * tc::BM + row_in_tile;
        s.q = row_grad(s.row, p.T, p.V, p.labels, p.valid, p.nll, p.lse, p.g);
        s.a = log2_scale(s.row < p.T ? p.sx[s.row] : 0.f);
        fit_half(p.most, s.up, s.down);
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, int n_next, uint32_t taddr, OutStage1& o) {
        const int col0 = n_tile * tc::BN;
        const int ncols = min(tc::BN, p.V - col0);
        const Columns w = s.w;
        ahead(p, s, n_next);
        const uint64_t a2 = ptx::pack_f32x2(s.a, s.a), no2 = ptx::pack_f32x2(-s.q.others2, -s.q.others2);
        walk_half(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            if ((c & 1) == 0) o.begin();
            const float mine = w.chunk(c), up = mine * s.up;
            float f[32];
            scaled(v, mine, f);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                float x0, x1;
                ptx::unpack_f32x2(ptx::fma_f32x2(ptx::pack_f32x2(f[i], f[i + 1]), a2, no2), x0, x1);
                ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(ptx::ex2_approx(x0), ptx::ex2_approx(x1)),
                                                 ptx::pack_f32x2(__shfl_sync(0xffffffffu, up, i), __shfl_sync(0xffffffffu, up, i + 1))), f[i], f[i + 1]);
            }
            const int rel = s.q.y - (col0 + c * 32);
            const float at_label = -__shfl_sync(0xffffffffu, up, rel & 31);
            if (rel >= 0 && rel < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == rel) f[i] = at_label;
            }
            if (!s.q.on) {
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o.put((c & 1) * 4 + q, ptx::pack_f16x2_sat(f[q * 8 + 0], f[q * 8 + 1]), ptx::pack_f16x2_sat(f[q * 8 + 2], f[q * 8 + 3]),
                      ptx::pack_f16x2_sat(f[q * 8 + 4], f[q * 8 + 5]), ptx::pack_f16x2_sat(f[q * 8 + 6], f[q * 8 + 7]));
            if ((c & 1) != 0 || (c + 1) * 32 >= ncols) o.flush(col0 + (c >> 1) * 64);
        });
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return p.T; }
    __device__ static __forceinline__ void end_item(const Params& p, const State& s, int group) {
        if (group == 0 && threadIdx.x < 192 && s.row < p.T) p.factor[s.row] = s.q.factor * s.down;
    }
};

// Two neighbouring ones of four integers, which come with 128 added (0 .. 255), as fp16: a byte behind 0x64 is 1024 + byte, the widely published way to widen bytes.
__device__ __forceinline__ __half2 widened(uint32_t biased, int pair) {
    const uint32_t w = __byte_perm(biased, 0x64646464u, pair ? 0x4342 : 0x4140);
    return __hsub2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0x6480)));       // - 1152
}

// The head as the 16-bit operand of the gradient's contraction: its integers in fp16 (exact; the cross entropy's terms are fp16 with the scale in them), or
// scale * integer in bf16, as an upstream dY is.  That rounding is a choice: dX is 2.4e-3 off, 1.7e-3 of it dX's own rounding.  Terms dY * scale in fp16, relative to
// each row's largest, would leave 1.7e-3, at a pass over dY for those maxima and a copy of it (some 140 us more at the rate of memory for 1000 x 151936, beside
// 360), and lose what lies far below the largest; bf16 holds upstream gradients of any range.
// 86 us for 1024 x 151936 (466 MB, 5.4 TB/s), 120 for 2048 x 128256 (6.6 TB/s): one load under way per thread, and divisions, keep shorter rows off the rate
// of memory.  (Beside the product of the gradient's terms, on what that leaves of the SMs, it does not fit: the step of 4096 rows 2.8 -> 3.4 ms.)
template <bool SCALED>
__global__ void __launch_bounds__(THREADS) widen_kernel(const int8_t* wq, long long ldw, const float* sw, long long units, int per_row, int d, uint16_t* out,
                                                        const CallSetup setup) {
    ptx::launch_dependents();
    set_up_call(setup, -1);
    for (long long u = blockIdx.x * static_cast<long long>(THREADS) + threadIdx.x; u < units; u += static_cast<long long>(gridDim.x) * THREADS) {
        const long long v = u / per_row;
        const int i = static_cast<int>(u - v * per_row) * 8;              // 8 integers: d is a multiple of 8
        const uint2 x = *reinterpret_cast<const uint2*>(wq + v * ldw + i);
        uint32_t r[4];
        const uint32_t b[2] = {x.x ^ 0x80808080u, x.y ^ 0x80808080u};    // 0 .. 255
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __half2 h = widened(b[j >> 1], j & 1);
            if (SCALED) {
                const float2 f = __half22float2(h);
                const float s = sw[v];
                r[j] = ptx::pack_bf16x2(f.x * s, f.y * s);
            } else {
                r[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        *reinterpret_cast<uint4*>(out + v * d + i) = make_uint4(r[0], r[1], r[2], r[3]);
    }
}

// Parts of a contraction, added in a fixed order; the row's factor; one rounding.  A CTA has 256 columns of a row, four threads share the parts of four of them:
// one by one they are mostly waited for (37 parts of 64 x 1024: 12 us by a thread each).
constexpr int PART_COLS = 256, PART_SHARES = 4;
__global__ void __launch_bounds__(THREADS) add_parts_kernel(const float* part, int g, long long stride, int d, const float* factor, __nv_bfloat16* out, long long ld) {
    __shared__ float4 s_sum[PART_SHARES - 1][PART_COLS / 4];
    const long long r = blockIdx.x;
    const int t = threadIdx.x & (PART_COLS / 4 - 1), share = threadIdx.x / (PART_COLS / 4), i = blockIdx.y * PART_COLS + t * 4;
    ptx::grid_dependency_wait();
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < d) {
#pragma unroll 4
        for (int k = share; k < g; k += PART_SHARES) {
            const float4 x = *reinterpret_cast<const float4*>(part + k * stride + r * d + i);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
    }
    if (share > 0) s_sum[share - 1][t] = s;
    __syncthreads();
    if (share > 0 || i >= d) return;
#pragma unroll
    for (int k = 0; k < PART_SHARES - 1; ++k) {
        const float4 x = s_sum[k][t];
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const float f = factor ? factor[r] : 1.f;
    *reinterpret_cast<uint2*>(out + r * ld + i) = make_uint2(ptx::pack_bf16x2(s.x * f, s.y * f), ptx::pack_bf16x2(s.z * f, s.w * f));
}

// the plain output of a contraction of fp16 operands, and of bf16 ones, behind other kernels of the call
struct EpiOutHalf : tc::EpiOutT<false> {};
struct EpiOutBehind : tc::EpiOutT<false> {};

}  // namespace i8

namespace tc {
template <bool F32>
struct OperandOf<i8::EpiLinear<F32>> { static constexpr Operand value = Operand::I8; };
template <>
struct OperandOf<i8::EpiCe> { static constexpr Operand value = Operand::I8; };
template <>
struct OperandOf<i8::EpiDz> { static constexpr Operand value = Operand::I8; };
template <>
struct OperandOf<i8::EpiOutHalf> { static constexpr Operand value = Operand::F16; };
template <bool F32>
struct EpiSets<i8::EpiLinear<F32>> { static constexpr int value = 2; };
template <>
struct StartsAhead<i8::EpiOutHalf> { static constexpr bool value = true; };
template <>
struct StartsAhead<i8::EpiOutBehind> { static constexpr bool value = true; };
template <bool F32>
struct StartsAhead<i8::EpiLinear<F32>> { static constexpr bool value = true; };
template <>
struct StartsAhead<i8::EpiCe> { static constexpr bool value = true; };
template <>
struct StartsAhead<i8::EpiDz> { static constexpr bool value = true; };
template <>
struct LetsNextStart<i8::EpiCe> { static constexpr bool value = true; };       // merge_kernel
template <bool F32>
struct LooksAhead<i8::EpiLinear<F32>> { static constexpr bool value = true; };
template <>
struct LooksAhead<i8::EpiCe> { static constexpr bool value = true; };
template <>
struct LooksAhead<i8::EpiDz> { static constexpr bool value = true; };
template <>
struct EpiSets<i8::EpiCe> { static constexpr int value = 2; };
template <>
struct EpiSets<i8::EpiDz> { static constexpr int value = 2; };
}  // namespace tc
}  // namespace cat
