// fp32 products of the LM-head operators beside the CAT loss (fp32 inputs: FFMA throughout, precise expf), with their epilogues:
//   FWD   logits of a row slab: softmax partials (max, sum exp, entropy sum, first column of the maximum), optional logits
//         and maxima of 64-column tiles
//   DZ    recomputed logits turned into dz of cat_logprob_bwd
//   OUT   alpha * A B, plus an addend
// One 64 x 64 tile per CTA of 128 threads, 8 x 4 outputs each, 16-deep slices double buffered in shared memory with the next slice in
// registers meanwhile: per slice step three 16-byte shared loads feed 32 FFMA (a 4 x 4 tile per thread, as in simt.cuh, feeds 16 from two,
// and reached a sixth of the FFMA rate).  The sum over k is taken in runs of 256, added up in a second accumulator: the rounding of a
// sum over 4096 vocabulary entries grows with 256 + 16 instead of 4096 terms.  Outputs with few tiles have their contraction cut into
// parts (gridDim.z), summed in order by add_kernel.
// Measured, 512 rows x 256 x 4096 (1.07 GFLOP a product): forward 52 us, dH 50 us, dW 45 us, 20 to 24 TFLOP/s: one or two CTAs' worth of
// tiles per SM, so latency and not the FFMA rate (74 TFLOP/s) bounds them; simt.cuh's kernel takes 106, 880 and 127 us.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace cat {
namespace f32 {

constexpr int TM = 64, TN = 64, TK = 16, THREADS = 128;
constexpr int RUN = 256 / TK;            // slices per run of the sum
constexpr float LOG2E = 1.4426950408889634f;
constexpr float CLOSING = -0.5f;         // log p from which on close_kernel writes the entry: at most one token of a row
constexpr float LOW = -1.0e30f;          // "no column yet": finite, so that 0 * (LOW - m) is 0

enum { FWD = 0, DZ = 1, OUT = 2 };

struct Operands {
    const float* A;          // element (m, k) at A[m * sAm + k * sAk]; one of the strides is 1
    const float* B;          // element (k, n) at B[k * sBk + n * sBn]; one of the strides is 1
    long long sAm, sAk, sBk, sBn;
    int M, N, Kd;
    int n_groups;            // gridDim.y; group g covers n-tiles [g * nt / n_groups, (g + 1) * nt / n_groups)
};

struct EpiParams {
    const long long* labels;     // FWD: may be nullptr; DZ: nullptr without grad_logp
    int V;
    // FWD
    float* part_m;               // [n_groups][M]
    float* part_l;
    float* part_u;               // sum exp2(x) x, x = (z - max) log2 e; nullptr (with part_id) = not wanted
    int* part_id;
    float* z_label;              // or nullptr
    float* zs;                   // [M][ld_z] logits, or nullptr
    float* gmax;                 // [M][ld_g] maxima of the tiles, or nullptr
    int* w_sq;                   // raised to the largest sum of squares of a row of W (float bits), or nullptr
    long long ld_z, ld_g;
    // DZ: dz = gl ([v = y] - p) - ge p (log p + entropy); rows with valid = 0 get zeros
    const unsigned char* valid;
    const float* lse;
    const float* entropy;
    const float* grad_logp;
    const float* grad_entropy;
    int* closing;                // [M] raised to the column of the entry that close_kernel writes; -1 on entry
    float* dz;
    long long ld_dz;
    // OUT
    const float* alpha;          // device scalar or nullptr
    const float* add;            // or nullptr; only with one part
    float* out;                  // part p of several: out + p * part_stride, neither scaled nor added to
    long long ld_add, ld_out, part_stride;
};

// One TK-deep slice of a 64-row operand into registers: row r of the tile (its k along lanes when k is contiguous, its rows otherwise).
template <bool KC>
__device__ __forceinline__ void fetch(const float* base, long long s_row, long long s_k, int row0, int n_rows, int k0, int Kd, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = i * THREADS + threadIdx.x;
        const int k = k0 + (KC ? e & (TK - 1) : e >> 6), row = row0 + (KC ? e >> 4 : e & 63);
        v[i] = (row < n_rows && k < Kd) ? base[row * s_row + k * s_k] : 0.f;
    }
}
template <bool KC>
__device__ __forceinline__ void put(float (*s)[TM + 4], const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = i * THREADS + threadIdx.x;
        s[KC ? e & (TK - 1) : e >> 6][KC ? e >> 4 : e & 63] = v[i];
    }
}

template <int MODE, bool A_KC, bool B_KC>
__global__ void __launch_bounds__(THREADS, 4) gemm_kernel(const Operands op, const EpiParams ep) {
    static_assert(TM == TN && TM * TK == 8 * THREADS, "eight elements of either operand per thread and slice");
    __shared__ __align__(16) float As[2][TK][TM + 4];
    __shared__ __align__(16) float Bs[2][TK][TN + 4];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int m0 = blockIdx.x * TM;
    const int n_tiles = (op.N + TN - 1) / TN;
    const int g = blockIdx.y;
    const int nt0 = static_cast<int>((static_cast<long long>(g) * n_tiles) / op.n_groups);
    const int nt1 = static_cast<int>((static_cast<long long>(g + 1) * n_tiles) / op.n_groups);
    const int slices = (op.Kd + TK - 1) / TK;
    const int ks0 = static_cast<int>((static_cast<long long>(blockIdx.z) * slices) / gridDim.z);
    const int ks1 = static_cast<int>((static_cast<long long>(blockIdx.z + 1) * slices) / gridDim.z);

    // Sums of squares of B's columns (rows of W) as the slices pass: a thread's eight elements of a slice belong to columns 8 i + threadIdx.x / 16,
    // and 16 lanes share a column.  By the first row tile's CTAs alone.
    const bool squares = MODE == FWD && B_KC && ep.w_sq != nullptr && blockIdx.x == 0;
    float most = 0.f;
    // running sums of the tile's rows over the group's tiles (kept here, not in registers: the 16 threads of a row all need them)
    __shared__ float s_m[TM], s_l[TM], s_u[TM];
    __shared__ int s_id[TM];
    if (MODE == FWD && tx == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { s_m[ty * 8 + i] = LOW; s_l[ty * 8 + i] = s_u[ty * 8 + i] = 0.f; s_id[ty * 8 + i] = 0; }
    }
    for (int nt = nt0; nt < nt1; ++nt) {
        const int n0 = nt * TN;
        float total[8][4] = {}, acc[8][4] = {};
        float av[8], bv[8], sq[8] = {};
        auto add_squares = [&] {
            if (squares) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sq[i] = fmaf(bv[i], bv[i], sq[i]) + (bv[i] != 0.f ? 0x1p-126f : 0.f);      // 0 for zeros alone
            }
        };
        fetch<A_KC>(op.A, op.sAm, op.sAk, m0, op.M, ks0 * TK, op.Kd, av);
        fetch<B_KC>(op.B, op.sBn, op.sBk, n0, op.N, ks0 * TK, op.Kd, bv);
        __syncthreads();              // the previous tile's last slice has been read
        put<A_KC>(As[0], av);
        put<B_KC>(Bs[0], bv);
        add_squares();
        __syncthreads();
        for (int ks = ks0, run = 0; ks < ks1; ++ks) {
            const int buf = (ks - ks0) & 1;
            if (ks + 1 < ks1) {
                fetch<A_KC>(op.A, op.sAm, op.sAk, m0, op.M, (ks + 1) * TK, op.Kd, av);
                fetch<B_KC>(op.B, op.sBn, op.sBk, n0, op.N, (ks + 1) * TK, op.Kd, bv);
            }
#pragma unroll
            for (int kk = 0; kk < TK; ++kk) {
                const float4 a0 = *reinterpret_cast<const float4*>(&As[buf][kk][ty * 8]);
                const float4 a1 = *reinterpret_cast<const float4*>(&As[buf][kk][ty * 8 + 4]);
                const float4 b = *reinterpret_cast<const float4*>(&Bs[buf][kk][tx * 4]);
                const float a[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    acc[i][0] = fmaf(a[i], b.x, acc[i][0]);
                    acc[i][1] = fmaf(a[i], b.y, acc[i][1]);
                    acc[i][2] = fmaf(a[i], b.z, acc[i][2]);
                    acc[i][3] = fmaf(a[i], b.w, acc[i][3]);
                }
            }
            if (++run == RUN || ks + 1 == ks1) {
                run = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) { total[i][j] += acc[i][j]; acc[i][j] = 0.f; }
            }
            if (ks + 1 < ks1) {
                put<A_KC>(As[buf ^ 1], av);
                put<B_KC>(Bs[buf ^ 1], bv);
                add_squares();
                __syncthreads();
            }
        }
        if (squares) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) sq[i] += __shfl_xor_sync(0xffffffffu, sq[i], off);
                most = sq[i] <= most ? most : sq[i];        // NaN stays
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = m0 + ty * 8 + i, at = ty * 8 + i;
            if (MODE == FWD) {
                int y = -1;
                if (row < op.M && ep.labels) {
                    const long long yy = ep.labels[row];
                    if (yy >= 0 && yy < ep.V) y = static_cast<int>(yy);
                }
                float cmax = LOW;
                int id = op.N;
#pragma unroll
                for (int j = 3; j >= 0; --j) {
                    const int col = n0 + tx * 4 + j;
                    if (col >= op.N) continue;
                    if (total[i][j] >= cmax) { cmax = total[i][j]; id = col; }
                    if (col == y && ep.z_label != nullptr) ep.z_label[row] = total[i][j];
                    if (ep.zs != nullptr && row < op.M) ep.zs[row * ep.ld_z + col] = total[i][j];
                }
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) {
                    const float om = __shfl_xor_sync(0xffffffffu, cmax, off);
                    const int oid = __shfl_xor_sync(0xffffffffu, id, off);
                    if (om > cmax || (om == cmax && oid < id)) { cmax = om; id = oid; }
                }
                if (ep.gmax != nullptr && tx == 0 && row < op.M) ep.gmax[row * ep.ld_g + nt] = cmax;
                __syncwarp();
                const float m_old = s_m[at], l_old = s_l[at], u_old = s_u[at];
                const float m_new = fmaxf(m_old, cmax);
                float sum = 0.f, us = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (n0 + tx * 4 + j >= op.N) continue;
                    const float e = expf(total[i][j] - m_new);
                    sum += e;
                    us = fmaf(e, (total[i][j] - m_new) * LOG2E, us);
                }
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, off);
                    us += __shfl_xor_sync(0xffffffffu, us, off);
                }
                const float sc = expf(m_old - m_new);
                __syncwarp();
                if (tx == 0) {
                    if (cmax > m_old && id < op.N) s_id[at] = id;
                    s_u[at] = fmaf(sc, fmaf((m_old - m_new) * LOG2E, l_old, u_old), us);
                    s_l[at] = fmaf(l_old, sc, sum);
                    s_m[at] = m_new;
                }
            } else if (row < op.M) {
                float gl = 0.f, ca = 0.f, cb = 0.f, lse = 0.f;
                int y = -1;
                bool on = false;
                if (MODE == DZ) {
                    on = ep.valid == nullptr || ep.valid[row] != 0;
                    if (on) {
                        lse = ep.lse[row];
                        const long long yy = ep.grad_logp ? ep.labels[row] : -1;
                        if (yy >= 0 && yy < ep.V) { y = static_cast<int>(yy); gl = ep.grad_logp[row]; ca = -gl; }
                        if (ep.grad_entropy) { cb = -ep.grad_entropy[row]; ca = fmaf(cb, ep.entropy[row], ca); }
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int col = n0 + tx * 4 + j;
                    if (col >= op.N) continue;
                    if (MODE == DZ) {
                        const float x = total[i][j] - lse;
                        const float v = fmaf(expf(x), fmaf(cb, x, ca), col == y ? gl : 0.f);
                        ep.dz[row * ep.ld_dz + col] = on ? v : 0.f;
                        if (on && x > CLOSING) atomicMax(ep.closing + row, col);
                    } else if (gridDim.z > 1) {
                        ep.out[blockIdx.z * ep.part_stride + row * ep.ld_out + col] = total[i][j];
                    } else {
                        float v = (ep.alpha ? *ep.alpha : 1.f) * total[i][j];
                        if (ep.add) v += ep.add[row * ep.ld_add + col];
                        ep.out[row * ep.ld_out + col] = v;
                    }
                }
            }
        }
    }
    if (squares && tx == 0) atomicMax(ep.w_sq, __float_as_int(most >= 0.f ? most : INFINITY));
    if (MODE == FWD && tx == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = m0 + ty * 8 + i;
            if (row >= op.M) continue;
            const size_t at = static_cast<size_t>(g) * op.M + row;
            const int q = ty * 8 + i;
            ep.part_m[at] = s_m[q];
            ep.part_l[at] = s_l[q];
            if (ep.part_u != nullptr) { ep.part_u[at] = s_u[q]; ep.part_id[at] = s_id[q]; }
        }
    }
}

// The entry of a token that has most of its row's probability, one CTA per row.  A row of dz sums to zero, so it is the others' sum with the sign
// turned: as exact as they are, where gl (1 - p) of a row that is sure of its label keeps the rounding of z and lse (1e-6 of lse) against 1 - p.
__global__ void __launch_bounds__(256) close_kernel(float* dz, long long ld, int V, const int* closing) {
    __shared__ float s_sum[8];
    const long long row = blockIdx.x;
    const int y = closing[row];
    if (y < 0) return;
    float* z = dz + row * ld;
    float sum = 0.f;
    for (int v = threadIdx.x; v < V; v += 256) sum += v == y ? 0.f : z[v];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 1; i < 8; ++i) sum += s_sum[i];
        z[y] = 0.f - sum;
    }
}

// out = alpha * (part 0 + part 1 + ...) [+ add], in that order.
__global__ void __launch_bounds__(256) add_kernel(const float* part, int n, long long stride, int rows, int cols, const float* alpha,
                                                  const float* add, long long ld_add, float* out, long long ld_out) {
    const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<long long>(rows) * cols) return;
    const long long r = i / cols, c = i - r * cols;
    float s = part[i];
    for (int g = 1; g < n; ++g) s += part[g * stride + i];
    s *= alpha ? *alpha : 1.f;
    if (add) s += add[r * ld_add + c];
    out[r * ld_out + c] = s;
}

}  // namespace f32
}  // namespace cat
