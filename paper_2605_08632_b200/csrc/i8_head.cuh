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

#include "ptx.cuh"
#include "tc_gemm.cuh"

namespace cat {
namespace i8 {

constexpr int THREADS = 256;
constexpr float LOW2 = -1.0e30f;        // "no column yet", in units of log2: finite, so that LOW2 - LOW2 is 0

// ------------------------------------------------------------------------------ rows to integers
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// 127 x / most to the nearest integer, halves to the even one, exactly: the binary32 product is off by less than 2^-16, and what lies
// that near to a half is decided by the quotient in 64 bits (127 x is exact there, and no quotient of a 31-bit by a 24-bit number is
// within 2^-53 of a half without being one).  inv = 127 / most, or 0 where that is out of range.
__device__ __forceinline__ int steps_of(float x, float inv, float most) {
    const float t = x * inv;
    const float n = rintf(t);
    if (inv != 0.f && fabsf(t - n) < 0.4999f) return static_cast<int>(n);
    return static_cast<int>(rint(127.0 * static_cast<double>(x) / static_cast<double>(most)));
}

// One CTA per row.
template <class T>
__global__ void __launch_bounds__(THREADS) quantize_kernel(const T* X, long long ldX, int d, int8_t* Xq, long long ldq, int pad, float* scale) {
    __shared__ unsigned s_most[THREADS / 32];
    const long long r = blockIdx.x;
    const T* x = X + r * ldX;
    unsigned bits = 0;                      // of |x|: ordered like the values, infinities and NaN above them
    for (int i = threadIdx.x; i < d; i += THREADS) bits = max(bits, __float_as_uint(to_float(x[i])) & 0x7fffffffu);
    bits = __reduce_max_sync(0xffffffffu, bits);
    if ((threadIdx.x & 31) == 0) s_most[threadIdx.x >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) bits = max(bits, s_most[i]);
    const float most = __uint_as_float(bits);
    const bool finite = bits < 0x7f800000u, any = finite && bits != 0u;
    const float inv = any && most > 1.0e-30f ? 127.f / most : 0.f;
    int8_t* q = Xq + r * ldq;
    for (int i = threadIdx.x; i < pad; i += THREADS) q[i] = any && i < d ? static_cast<int8_t>(steps_of(to_float(x[i]), inv, most)) : 0;
    if (threadIdx.x == 0) scale[r] = finite ? most / 127.f : __uint_as_float(0x7fc00000u);
}

// ------------------------------------------------------------------------------ a plain product, 64 x 64 outputs per CTA
constexpr int TILE = 64;

struct Head {
    const int8_t* xq;      // [T][ldq], zeros past d
    const float* sx;       // [T]
    const int8_t* wq;      // [V][ldw]
    const float* sw;       // [V]
    long long ldq, ldw;
    int T, V, d;
};

__device__ __forceinline__ int four_bytes(const int8_t* row, int k, int d) {
    if (k + 4 <= d) return *reinterpret_cast<const int*>(row + k);
    int v = 0;
    for (int i = 0; i < 4; ++i)
        if (k + i < d) v |= (static_cast<int>(row[k + i]) & 255) << (8 * i);
    return v;
}

__device__ __forceinline__ void tile_sums(const Head& h, int r0, int c0, int (&acc)[4][4]) {
    __shared__ int sa[TILE][17], sb[TILE][17];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int k0 = 0; k0 < h.d; k0 += 64) {
        for (int i = threadIdx.x; i < TILE * 16; i += THREADS) {
            const int row = i >> 4, w = i & 15, k = k0 + 4 * w;
            sa[row][w] = r0 + row < h.T && k < h.d ? four_bytes(h.xq + (r0 + row) * h.ldq, k, h.d) : 0;
            sb[row][w] = c0 + row < h.V && k < h.d ? four_bytes(h.wq + (c0 + row) * h.ldw, k, h.d) : 0;
        }
        __syncthreads();
        for (int w = 0; w < 16; ++w)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = __dp4a(sa[ty * 4 + a][w], sb[tx * 4 + b][w], acc[a][b]);
        __syncthreads();
    }
}

__global__ void __launch_bounds__(THREADS) linear_kernel(const Head h, const float* bias, float* Yf, __nv_bfloat16* Yb, long long ldY) {
    const int c0 = blockIdx.x * TILE, r0 = blockIdx.y * TILE;
    int acc[4][4] = {};
    tile_sums(h, r0, c0, acc);
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int r = r0 + (threadIdx.x >> 4) * 4 + a, c = c0 + (threadIdx.x & 15) * 4 + b;
            if (r >= h.T || c >= h.V) continue;
            float y = __int2float_rn(acc[a][b]) * h.sw[c] * h.sx[r];
            if (bias) y += bias[c];
            if (Yf) Yf[r * ldY + c] = y;
            else Yb[r * ldY + c] = __float2bfloat16(y);
        }
}

// log2 e times a row's scale; a row of zeros has logits 0 whatever this is, and -infinity times it has to stay -infinity.
__device__ __forceinline__ float log2_scale(float sx) { return sx == 0.f ? tc::LOG2E : sx * tc::LOG2E; }

// Largest logit but the label's and the sum relative to it, per row and tile of the vocabulary, in units of log2.
__global__ void __launch_bounds__(THREADS) ce_kernel(const Head h, const long long* labels, float* part_m, float* part_l, float* z_label) {
    const int c0 = blockIdx.x * TILE, r0 = blockIdx.y * TILE;
    int acc[4][4] = {};
    tile_sums(h, r0, c0, acc);
    for (int a = 0; a < 4; ++a) {
        const int r = r0 + (threadIdx.x >> 4) * 4 + a;
        const float s = log2_scale(r < h.T ? h.sx[r] : 0.f);
        const long long y = r < h.T ? labels[r] : -1;
        float z[4], m = LOW2, l = 0.f;
        for (int b = 0; b < 4; ++b) {
            const int c = c0 + (threadIdx.x & 15) * 4 + b;
            z[b] = c < h.V ? __int2float_rn(acc[a][b]) * h.sw[c] * s : -INFINITY;
            if (r < h.T && c < h.V && c == y) { z_label[r] = z[b]; z[b] = -INFINITY; }
            m = fmaxf(m, z[b]);
        }
        for (int off = 8; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
        for (int b = 0; b < 4; ++b) l += exp2f(z[b] - m);
        for (int off = 8; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        if (r < h.T && (threadIdx.x & 15) == 0) {
            part_m[static_cast<long long>(blockIdx.x) * h.T + r] = m;
            part_l[static_cast<long long>(blockIdx.x) * h.T + r] = l;
        }
    }
}

// The parts of each row in order, and what follows from them; z_label is read for rows with a label only.
__global__ void __launch_bounds__(THREADS) merge_kernel(const float* part_m, const float* part_l, const float* z_label, int S, long long stride, int T, int V,
                                                        const long long* labels, const unsigned char* valid, float* nll, float* lse) {
    const int r = blockIdx.x * THREADS + threadIdx.x;
    if (r >= T) return;
    if (valid != nullptr && valid[r] == 0) {
        nll[r] = lse[r] = 0.f;
        return;
    }
    float m = LOW2;
    for (int s = 0; s < S; ++s) m = fmaxf(m, part_m[s * stride + r]);
    float l = 0.f;
    for (int s = 0; s < S; ++s) l = fmaf(part_l[s * stride + r], exp2f(part_m[s * stride + r] - m), l);
    constexpr double LN2 = 0.69314718055994530942;
    const double others = LN2 * (static_cast<double>(m) + log2(static_cast<double>(l)));
    const long long y = labels[r];
    if (y < 0 || y >= V) {
        nll[r] = 0.f;
        lse[r] = static_cast<float>(others);
        return;
    }
    const double zy = LN2 * static_cast<double>(z_label[r]), over = others - zy;
    const double n = over > 0.0 ? over + log1p(exp(-over)) : log1p(exp(over));
    nll[r] = static_cast<float>(n);
    lse[r] = static_cast<float>(zy + n);
}

// ------------------------------------------------------------------------------ gradient
// Largest finite |scale| of the head, as float bits raised from 0.
__global__ void __launch_bounds__(THREADS) largest_scale_kernel(const float* sw, int V, int* most) {
    unsigned bits = 0;
    for (int v = blockIdx.x * THREADS + threadIdx.x; v < V; v += gridDim.x * THREADS) {
        const unsigned b = __float_as_uint(sw[v]) & 0x7fffffffu;
        if (b < 0x7f800000u) bits = max(bits, b);
    }
    bits = __reduce_max_sync(0xffffffffu, bits);
    if ((threadIdx.x & 31) == 0) atomicMax(most, static_cast<int>(bits));
}

// 2^k with most 2^k in [2^14, 2^15), and 2^-k
__device__ __forceinline__ void fit_half(int most_bits, float& up, float& down) {
    int e = most_bits >> 23;                            // biased exponent of the largest scale
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

// exp(z_v - o) sw_v 2^k, and -sw_y 2^k at the label, as fp16
__global__ void __launch_bounds__(THREADS) ce_dz_kernel(const Head h, const long long* labels, const unsigned char* valid, const float* nll, const float* lse,
                                                        const float* g, const int* most, __half* dz, long long ldz, float* factor) {
    const int c0 = blockIdx.x * TILE, r0 = blockIdx.y * TILE;
    int acc[4][4] = {};
    tile_sums(h, r0, c0, acc);
    float up, down;
    fit_half(*most, up, down);
    for (int a = 0; a < 4; ++a) {
        const int r = r0 + (threadIdx.x >> 4) * 4 + a;
        if (r >= h.T) continue;
        const RowGrad q = row_grad(r, h.T, h.V, labels, valid, nll, lse, g);
        const float s = log2_scale(h.sx[r]);
        if (blockIdx.x == 0 && (threadIdx.x & 15) == 0) factor[r] = q.factor * down;
        for (int b = 0; b < 4; ++b) {
            const int c = c0 + (threadIdx.x & 15) * 4 + b;
            if (c >= h.V) continue;
            float x = 0.f;
            if (q.on) x = c == q.y ? -h.sw[c] * up : exp2f(fmaf(__int2float_rn(acc[a][b]) * h.sw[c], s, -q.others2)) * (h.sw[c] * up);
            dz[r * ldz + c] = __float2half(x);
        }
    }
}

// dX[r, i] = factor[r] sum_v A[r, v] wq[v, i]: A the fp16 terms above, or dY sw
__global__ void __launch_bounds__(THREADS) dx_kernel(const __half* dz, const __nv_bfloat16* dY, long long ldA, const float* factor, const Head h,
                                                     __nv_bfloat16* dX, long long ldX) {
    __shared__ float sa[TILE][17], sb[16][TILE + 1];
    const int c0 = blockIdx.x * TILE, r0 = blockIdx.y * TILE;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < h.V; k0 += 16) {
        for (int i = threadIdx.x; i < TILE * 16; i += THREADS) {
            const int row = i >> 4, k = k0 + (i & 15);
            float a = 0.f;
            if (r0 + row < h.T && k < h.V) a = dz ? __half2float(dz[(r0 + row) * ldA + k]) : __bfloat162float(dY[(r0 + row) * ldA + k]) * h.sw[k];
            sa[row][i & 15] = a;
            const int kb = k0 + i / TILE, c = c0 + i % TILE;
            sb[i / TILE][i % TILE] = kb < h.V && c < h.d ? static_cast<float>(h.wq[kb * h.ldw + c]) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sa[ty * 4 + a][k], sb[k][tx * 4 + b], acc[a][b]);
        __syncthreads();
    }
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int r = r0 + ty * 4 + a, c = c0 + tx * 4 + b;
            if (r < h.T && c < h.d) dX[r * ldX + c] = __float2bfloat16(acc[a][b] * (factor ? factor[r] : 1.f));
        }
}

}  // namespace i8
}  // namespace cat
