// Distillation from a teacher's stored top logits, under the CAT weight: per draft row
//   weight * (beta * CE + KD),   KD = sum_i p_i (log p_i - z[id_i] + lse)
// over the row's list (id_i, log p_i), i < k, in the place of the full distribution of kd.cuh:
//   dz[v] = weight ((beta + sum_i p_i) q_v - beta [v = y] - sum_i p_i [v = id_i]).
// One row slab at a time: gather_kernel (the logits at the list's ids, fp32, and the slab's reference), the logits GEMM,
// which keeps z - ref in 16 bits, the row kernel of rowops.cuh, dz_kernel (z -> dz in place) and the dH and dW contractions.
//
// Why the slab holds logits and is turned into dz by a pass of its own (4 bytes per logit, bound by HBM), although
// cat_loss_fwd_bwd gets by without one: there the row's factor a[r] has to ride on H in the dW contraction, and
// rounding a[r] H[r, :] to bf16 costs as much as rounding dz.  Here dz is rounded to bf16 once, and H not at all.
// 16384 rows of 2048 x 128256, k = 16, per step: the three GEMMs 17.6 ms, dz 1.4 ms (6.1 TB/s), gather 0.24 ms (1.1 GB of W rows, 4.7 TB/s).
// Running dz of one block of rows beside the logits GEMM of the next, in extra warps, was tried: the GEMM, which
// takes all that the L2 can feed it, slowed down by three quarters of what the overlap saved.
#pragma once
#include "logprob.cuh"
#include <type_traits>

namespace cat {
namespace tc {

// Softmax statistics (as EpiFwdT), the label's logit, and z - ref in 16 bits: a whole number of steps of 2^-9 nats from -48, up to
// +80.  ref is the largest of the logits that the list and the label name, so softmax is below e^-48 times a named token's where it is
// cut off below, and above only logits that exceed every named one by 80 nats are cut, which dz_kernel takes again.  The steps put a relative error of at most 2^-10
// on softmax, 5.6e-4 rms, wherever it lies; fp16 would put 2^-12 |z - ref| there, 2.3e-3 rms in the bulk 8 to 16 nats below the top,
// which is more than the rounding of dz.
constexpr float STEPS = 512.f;           // per nat

constexpr float LOW_END = -48.f;         // the range's lower end: step 0
constexpr float TOP_STEP = 65535.f;

// two logits as steps, rounded and clamped, into the halves of a word.  The saturating fma clamps to the range as a share of it, and adding
// 2^23 leaves the whole number of steps in the low bits: two instructions a logit on the fma pipe, where clamping by min and max takes
// four, two of them at half the rate.  base = -(ref + LOW_END) STEPS / TOP_STEP.
__device__ __forceinline__ uint32_t pack_steps(float a, float b, float base) {
    const uint32_t x = __float_as_uint(fmaf(__saturatef(fmaf(a, STEPS / TOP_STEP, base)), TOP_STEP, 8388608.f));
    const uint32_t y = __float_as_uint(fmaf(__saturatef(fmaf(b, STEPS / TOP_STEP, base)), TOP_STEP, 8388608.f));
    return __byte_perm(x, y, 0x5410);
}
struct EpiFwdRef {
    struct Params {
        const long long* labels;   // [T]
        float* part_m;             // [n_groups][part_stride]
        float* part_l;
        float* part_u;             // see RunningSums
        int* part_id;              // first column that holds the maximum
        float* z_label;            // [T]
        const float* ref;          // [T]
        long long part_stride;
        int T;
        int V;
    };
    struct State {
        RunningSums r;
        float base;                // see pack_steps
        int id;
        int y;
        int row;
    };
    __device__ static __forceinline__ void begin_item(const Params& p, State& s, int m_tile, int row_in_tile) {
        s.row = m_tile * BM + row_in_tile;
        s.r.clear();
        s.id = 0;
        s.base = 0.f;
        s.y = -1;
        if (s.row < p.T) {
            const long long y = p.labels[s.row];
            if (y >= 0 && y < p.V) s.y = static_cast<int>(y);
            s.base = -(p.ref[s.row] + LOW_END) * (STEPS / TOP_STEP);
        }
    }
    __device__ static __forceinline__ void tile(const Params& p, State& s, int n_tile, uint32_t taddr, OutStage& o) {
        const int col0 = n_tile * BN;
        const int ncols = min(BN, p.V - col0);
        walk_tile(taddr, ncols, [&](int c, uint32_t (&v)[32]) {
            if ((c & 1) == 0) o.begin();
            float f[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
            const int live = ncols - c * 32;
            if (live < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i >= live) f[i] = LP_LOW;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o.put((c & 1) * 4 + q, pack_steps(f[q * 8 + 0], f[q * 8 + 1], s.base), pack_steps(f[q * 8 + 2], f[q * 8 + 3], s.base),
                      pack_steps(f[q * 8 + 4], f[q * 8 + 5], s.base), pack_steps(f[q * 8 + 6], f[q * 8 + 7], s.base));
            if ((c & 1) != 0 || (c + 1) * 32 >= ncols) o.flush(col0 + (c >> 1) * 64);
            const int rel = s.y - (col0 + c * 32);
            if (rel >= 0 && rel < 32) {
                float zy = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == rel) zy = f[i];
                p.z_label[s.row] = zy;
            }
            const float cmax = max_of(f);
            if (cmax > s.r.m) s.id = col0 + c * 32 + first_at(f, cmax);
            s.r.add(f, cmax);
        });
    }
    __device__ static __forceinline__ int out_rows(const Params& p) { return p.T; }
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

}  // namespace tc

namespace tk {

using lp::MAX_TOP;
using lp::THREADS;
using lp::WARPS;
constexpr float LOG2E = 1.4426950408889634f;

// First launch of a call, one CTA: the workspace header cleared, the rows that take part (mask bit set, label a token id, teacher position
// exists), g / N, and the unmasked rows whose label is no token id, counted (the kernels that follow know only the rows that take part).
__global__ void __launch_bounds__(1024) begin_kernel(const long long* labels, const unsigned char* valid, const long long* block_start, int T,
                                                     int K, int V, long long L, const float* grad_loss, unsigned char* valid_eff,
                                                     float* scale, int* n_bad, int* header, int header_words) {
    __shared__ int sh[32], sh_bad[32];
    for (int i = threadIdx.x; i < header_words; i += 1024) header[i] = 0;
    int n = 0, bad = 0;
#pragma unroll 4
    for (int r = threadIdx.x; r < T; r += 1024) {
        const long long y = labels[r];
        const int b = r / K;
        const long long t = block_start ? block_start[b] + (r - b * K) : r;
        const bool mask = valid == nullptr || valid[r] != 0, token = y >= 0 && y < V;
        const bool on = mask && token && t >= 0 && t < L;
        valid_eff[r] = on ? 1 : 0;
        n += on ? 1 : 0;
        bad += mask && !token ? 1 : 0;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    bad = __reduce_add_sync(0xffffffffu, bad);
    if ((threadIdx.x & 31) == 0) { sh[threadIdx.x >> 5] = n; sh_bad[threadIdx.x >> 5] = bad; }
    __syncthreads();
    if (threadIdx.x == 0) {
        int tot = 0, tot_bad = 0;
        for (int w = 0; w < 32; ++w) { tot += sh[w]; tot_bad += sh_bad[w]; }
        *n_bad = tot_bad;
        const float g = grad_loss ? *grad_loss : 1.f;
        *scale = tot > 0 ? g / static_cast<float>(tot) : 0.f;
    }
}

// Last launch, one CTA: loss = {beta ce + kd, ce, kd} with ce and kd the sums over rows over N (fp64, in a fixed order), and the statistics.
__global__ void __launch_bounds__(1024) end_kernel(const rows::CtaPartial* partials, int n_partials, int n_blocks, const float* kd_row, int T,
                                                   float beta, float* loss, rows::StatsOut* stats, const int* n_bad, const int* status) {
    __shared__ double s_d[4][32];
    __shared__ long long s_n[32];
    double d[4] = {0.0, 0.0, 0.0, 0.0};       // loss, weight, weight * conf, kd
    long long n = 0;                          // valid rows
    for (int i = threadIdx.x; i < n_partials; i += 1024) {
        const rows::CtaPartial q = partials[i];
        d[0] += q.loss; d[1] += q.sum_w; d[2] += q.sum_wc; n += q.n_valid;
    }
#pragma unroll 4
    for (int r = threadIdx.x; r < T; r += 1024) d[3] += static_cast<double>(kd_row[r]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] += __shfl_down_sync(0xffffffffu, d[j], off);
        n += __shfl_down_sync(0xffffffffu, n, off);
    }
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        for (int j = 0; j < 4; ++j) s_d[j][warp] = d[j];
        s_n[warp] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; ++w) {
            for (int j = 0; j < 4; ++j) d[j] += s_d[j][w];
            n += s_n[w];
        }
        const double N = n > 0 ? static_cast<double>(n) : 1.0;
        const float ce = n > 0 ? static_cast<float>(d[0] / N) : 0.f, kd = n > 0 ? static_cast<float>(d[3] / N) : 0.f;
        loss[0] = beta * ce + kd;
        loss[1] = ce;
        loss[2] = kd;
        if (stats) {
            stats->n_valid = n;
            stats->n_bad_labels = *n_bad;
            stats->sum_weight = static_cast<float>(d[1]);
            stats->est_accept_len = n_blocks > 0 ? static_cast<float>(d[2] / n_blocks) : 0.f;
            stats->device_status = *status;
            stats->reserved = 0;
        }
    }
}

// The teacher's lists: position t's entries are (ids[t * ld + i], logp[t * ld + i]), i < k.
struct Lists {
    const long long* ids;
    const float* logp;
    const long long* block_start;  // [T / K] or nullptr: row r reads position r
    long long ld;
    int k;
    int K;
    int V;
    int renorm;
    __device__ __forceinline__ long long position(long long r) const {
        return block_start ? block_start[r / K] + (r - (r / K) * K) : r;
    }
    // entry i counts iff its id is a token and its log probability is above -infinity (NaN counts, and shows)
    __device__ __forceinline__ bool entry(long long t, int i, long long& id, float& lp) const {
        id = ids[t * ld + i];
        lp = logp[t * ld + i];
        return id >= 0 && id < V && !(lp == -INFINITY);
    }
};

// One CTA per row of the slab: z[r, id_i] as fp32 for every counting entry of its list (one warp per dot product), ref[r],
// the largest of them and of the label's logit (0 for a row that takes no part), and the row's copy in Hz: the dW contraction's
// operand, in which a row that takes no part is zero whatever H holds there.
template <class TI>
__global__ void __launch_bounds__(THREADS) gather_kernel(const TI* H, long long ldH, const TI* W, long long ldW, int d,
                                                         const long long* labels, const unsigned char* valid_eff, Lists lists,
                                                         long long row0, int rows, int lo, float* zt, int ld_zt, float* ref, TI* Hz) {
    __shared__ float s_max[WARPS];
    const long long r = row0 + blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool pad = static_cast<int>(blockIdx.x) >= rows;            // dz in two terms: the grid goes on to `lo` rows
    const TI* h = H + (pad ? 0 : static_cast<long long>(blockIdx.x)) * ldH;
    const bool on = !pad && valid_eff[r] != 0;
    lp::copy_row(h, Hz + static_cast<long long>(blockIdx.x) * d, d, on);
    if (lo > 0) lp::copy_row(h, Hz + (static_cast<long long>(blockIdx.x) + lo) * d, d, on);
    if (pad) return;
    if (!valid_eff[r]) {
        if (threadIdx.x == 0) ref[r] = 0.f;
        return;
    }
    const long long t = lists.position(r);
    float mx = -INFINITY;
    for (int i = warp; i <= lists.k; i += WARPS) {
        long long id = -1;
        float lp;
        if (i == lists.k) id = labels[r];
        else if (!lists.entry(t, i, id, lp)) continue;
        const float z = lp::warp_dot_f32(h, W + id * ldW, d, lane);
        if (lane == 0) zt[static_cast<long long>(blockIdx.x) * ld_zt + i] = z;
        mx = fmaxf(mx, z);
    }
    if (lane == 0) s_max[warp] = mx;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 1; i < WARPS; ++i) mx = fmaxf(mx, s_max[i]);
        ref[r] = fabsf(mx) < 1.0e30f ? mx : 0.f;
    }
}

// Merges the vocabulary splits of a row's (max, sum exp) into one pair for the row kernel (one warp per row), and corrects the sum for the
// largest logit and the label's, which are known exactly (nearly: as fp32 sums): the tensor cores' additions truncate, and a token of
// high probability makes up lse (see lp::row_kernel).  z_label is replaced by the exact label logit.
template <class TI>
struct MergeParams {
    const float* part_m;           // [S][part_stride]
    const float* part_l;
    const float* part_u;           // with part_id
    const int* part_id;            // nullptr: fp32 logits, nothing to correct
    long long part_stride;
    int S;
    const TI* H;
    const TI* W;
    long long ldH, ldW;
    int d, V;
    const long long* labels;
    const unsigned char* valid;
    const float* z_exact;          // [rows] at pitch ld_exact: the label's logit, of rows that take part
    long long ld_exact;
    float* z_label;                // [rows] the GEMM's on entry
    float* m1;
    float* l1;
    int rows;
};
template <class TI>
__global__ void __launch_bounds__(THREADS) merge_kernel(const MergeParams<TI> p) {
    const int r = blockIdx.x * WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= p.rows) return;
    float m = -INFINITY;
    int id = 0;
    for (int s = lane; s < p.S; s += 32) {
        const float x = p.part_m[s * p.part_stride + r];
        if (x > m) { m = x; id = p.part_id ? p.part_id[s * p.part_stride + r] : 0; }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, off);
        const int oid = __shfl_xor_sync(0xffffffffu, id, off);
        if (om > m || (om == m && oid < id)) { m = om; id = oid; }
    }
    float l = 0.f, zl = 0.f;       // sum exp(z - m), and exp(z - m) z
    for (int s = lane; s < p.S; s += 32) {
        const float ms = p.part_m[s * p.part_stride + r], e = expf(ms - m), ls = p.part_l[s * p.part_stride + r];
        l = fmaf(e, ls, l);
        if (p.part_id) zl = fmaf(e, fmaf(0.6931471805599453f, p.part_u[s * p.part_stride + r], ms * ls), zl);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, off);
        zl += __shfl_xor_sync(0xffffffffu, zl, off);
    }
    if (p.valid[r]) {
        const float zy = p.z_exact[r * p.ld_exact];
        if (p.part_id && static_cast<unsigned>(id) < static_cast<unsigned>(p.V)) {      // a GEMM that timed out leaves anything here
            const bool is_label = p.labels[r] == id;
            const float z = is_label ? zy : lp::warp_dot_f32(p.H + r * p.ldH, p.W + id * p.ldW, p.d, lane);
            const float x = z - m, ly = p.z_label[r];
            zl -= m;
            if (fabsf(x) < 1.f) l += expm1f(x);
            if (!is_label) {
                const float e = expf(ly - m);
                zl = fmaf(-e, ly, zl);
                if (fabsf(zy - ly) < 1.f) l = fmaf(e, expm1f(zy - ly), l);
            }
            // the others, taken to be off by the same share of themselves as the largest (see lp::off_share)
            l = fmaf(lp::off_share(x, m, p.d), zl, l);
        }
        __syncwarp();
        if (lane == 0) p.z_label[r] = zy;
    }
    if (lane == 0) { p.m1[r] = m; p.l1[r] = l; }
}

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
__device__ __forceinline__ float block_sum(float x, float* red) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < WARPS; ++i) x += red[i];
    return x;
}

// One CTA per row of the slab: the row's KD value, and the stored logits turned into dz in place.  Dense part
// weight (beta + sum p) q from the stored z - ref; the entries at the label and at the list's ids from their fp32
// logits, an id that stands in the list twice with the sum of its probabilities.
// fp32 slabs (fp32 inputs) hold z itself and leave as fp32 dz.  In a row whose largest logit, m1, lies past the slab's range above all that the list
// and the label name, the logits that were cut off there are summed again.
//
// The closing entry.  Where a named token has nearly all of the row's probability, its entry (beta + mass) q - sub is small against its terms, and
// the rounding of lse, 1e-6 of q, stands against 1 - q.  A row of dz sums to zero (sum q = 1), so that entry is taken as the others' sum with
// the sign turned, off by the same share as they are: 2^-10 at most for bf16, which is less than the rounding of lse from 1 - q = 2^-10 down.
template <bool F32>
__global__ void __launch_bounds__(THREADS) dz_kernel(const std::conditional_t<F32, float, __nv_bfloat16>* H, long long ldH,
                                                     const std::conditional_t<F32, float, __nv_bfloat16>* W, long long ldW, int d, const float* m1,
                                                     void* zs, long long ldz, const long long* labels, const unsigned char* valid_eff,
                                                     Lists lists, long long row0, int rows, int lo, const float* lse, const float* weight,
                                                     const float* zt, int ld_zt, const float* ref, float beta, float* kd_row,
                                                     int V) {
    __shared__ float s_red[WARPS];
    __shared__ float s_p[MAX_TOP];
    __shared__ int s_id[MAX_TOP];
    __shared__ int s_close;
    constexpr float CLOSING = F32 ? -0.5f : -0.0009765625f;        // log q
    const long long r = row0 + blockIdx.x;
    uint4* row = reinterpret_cast<uint4*>(static_cast<unsigned short*>(zs) + static_cast<size_t>(blockIdx.x) * ldz);
    float* row32 = static_cast<float*>(zs) + static_cast<size_t>(blockIdx.x) * ldz;
    const int groups = static_cast<int>(ldz / 8);
    // what rounding to bf16 leaves, with dz in two terms
    uint4* rest = lo > 0 ? row + static_cast<size_t>(lo) * (ldz / 8) : nullptr;
    if (static_cast<int>(blockIdx.x) >= rows || !valid_eff[r]) {
        if (lo > 0)
            for (int g = threadIdx.x; g < groups; g += THREADS) rest[g] = make_uint4(0u, 0u, 0u, 0u);
        if (F32) for (int v = threadIdx.x; v < V; v += THREADS) row32[v] = 0.f;
        else for (int g = threadIdx.x; g < groups; g += THREADS) row[g] = make_uint4(0u, 0u, 0u, 0u);
        if (threadIdx.x == 0 && static_cast<int>(blockIdx.x) < rows) kd_row[r] = 0.f;
        return;
    }
    const long long t = lists.position(r);
    const float lse_r = lse[r], w = weight[r];
    const int y = static_cast<int>(labels[r]);
    const float* zr = zt + static_cast<long long>(blockIdx.x) * ld_zt;
    // the list: thread i holds entry i (k <= MAX_TOP = THREADS)
    const int i = threadIdx.x;
    long long id = -1;
    float lp = -INFINITY, z_i = 0.f;
    const bool there = i < lists.k && lists.entry(t, i, id, lp);
    if (there) z_i = zr[i];
    if (i == 0) s_close = -1;
    __syncthreads();
    if (there && z_i - lse_r > CLOSING) s_close = static_cast<int>(id);
    if (i == 0 && zr[lists.k] - lse_r > CLOSING) s_close = y;
    __syncthreads();
    const int close = s_close;
    // what the slab holds at the named tokens, for their part of the dense sum
    float held = 0.f, held_y = 0.f;
    if (close >= 0) {
        auto at = [&](long long v) { return F32 ? row32[v] : static_cast<float>(reinterpret_cast<const unsigned short*>(row)[v]); };
        if (there) held = at(id);
        if (i == 0) held_y = at(y);
    }
    if (lists.renorm) {
        const float m = block_max(there ? lp : -INFINITY, s_red);
        const float l = block_sum(there ? expf(lp - m) : 0.f, s_red);
        if (there) lp = lp - m - logf(l);
    }
    const float p_i = there ? expf(lp) : 0.f;
    const float mass = block_sum(p_i, s_red);
    // 0 (log 0 - ...) = 0: a probability that underflows adds nothing
    const float kd = block_sum(there && p_i != 0.f ? p_i * (lp - (z_i - lse_r)) : 0.f, s_red);
    if (i < MAX_TOP) {
        s_p[i] = p_i;
        s_id[i] = there ? static_cast<int>(id) : -1;
    }
    if (i == 0) kd_row[r] = w * kd;
    const float wm = w * (beta + mass);
    const float off = F32 ? 0.f : (ref[r] + (tc::LOW_END + 64.f) - lse_r) * LOG2E;
    // the dense part from what the slab holds: z, or steps from the lower end (less 2^15, the middle of the range)
    auto dense = [&](float x) { return F32 ? wm * expf(x - lse_r) : wm * ptx::ex2_approx(fmaf(x - 32768.f, LOG2E / tc::STEPS, off)); };
    float sum = 0.f;               // of the row's dense entries but the closing one, with one
    if (F32)
        for (int v = threadIdx.x; v < V; v += THREADS) {
            const float x = dense(row32[v]);
            row32[v] = x;
            if (v != close) sum += x;
        }
    else if (m1[r] - ref[r] > tc::LOW_END + tc::TOP_STEP / tc::STEPS - 0.1f) {
        if constexpr (!F32) {
            const int lane = threadIdx.x & 31;
            const __nv_bfloat16* h = H + static_cast<long long>(blockIdx.x) * ldH;
            for (int g0 = threadIdx.x - lane; g0 < groups; g0 += THREADS) {      // whole warps
                const int g = g0 + lane;
                const uint4 in = g < groups ? row[g] : make_uint4(0u, 0u, 0u, 0u);
                const uint32_t zw[4] = {in.x, in.y, in.z, in.w};
                float x[8];
                unsigned cut = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t n = j & 1 ? zw[j >> 1] >> 16 : zw[j >> 1] & 0xffffu;
                    x[j] = g * 8 + j < V ? wm * ptx::ex2_approx(fmaf(__uint_as_float(n | 0x4b000000u) - 8421376.f, LOG2E / tc::STEPS, off)) : 0.f;
                    cut |= n == 0xffffu && g * 8 + j < V ? 1u << j : 0u;
                }
                for (unsigned lanes = __ballot_sync(0xffffffffu, cut != 0); lanes != 0; lanes &= lanes - 1) {
                    const int src = __ffs(lanes) - 1;
                    for (unsigned at = __shfl_sync(0xffffffffu, cut, src); at != 0; at &= at - 1) {
                        const int j = __ffs(at) - 1;
                        const float z = lp::warp_dot_f32(h, W + (static_cast<long long>(g0 + src) * 8 + j) * ldW, d, lane);
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (lane == src && q == j) x[q] = wm * expf(z - lse_r);
                    }
                }
                if (g < groups) {
                    uint32_t o[4], left[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        o[j] = ptx::pack_bf16x2(x[2 * j], x[2 * j + 1]);
                        left[j] = ptx::pack_bf16x2(x[2 * j] - __uint_as_float(o[j] << 16), x[2 * j + 1] - __uint_as_float(o[j] & 0xffff0000u));
                    }
                    row[g] = make_uint4(o[0], o[1], o[2], o[3]);
                    if (lo > 0) rest[g] = make_uint4(left[0], left[1], left[2], left[3]);
                }
            }
        }
    } else {
        // four loads in flight a thread: slabs of few rows fill the SMs with too few warps to cover the memory's latency with one
        constexpr int AHEAD = 4;
        for (int g0 = threadIdx.x; g0 < groups; g0 += AHEAD * THREADS) {
            uint4 in[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (g0 + u * THREADS < groups) in[u] = __ldcs(row + g0 + u * THREADS);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int g = g0 + u * THREADS;
                if (g >= groups) break;
                const uint32_t zw[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
                uint32_t o[4], left[4];
                const int col = g * 8;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // steps from the middle of the range: the low bits of 2^23, and that much taken off exactly
                    const float n0 = __uint_as_float((zw[j] & 0xffffu) | 0x4b000000u) - 8421376.f;
                    const float n1 = __uint_as_float((zw[j] >> 16) | 0x4b000000u) - 8421376.f;
                    const float a = col + 2 * j < V ? wm * ptx::ex2_approx(fmaf(n0, LOG2E / tc::STEPS, off)) : 0.f;
                    const float b = col + 2 * j + 1 < V ? wm * ptx::ex2_approx(fmaf(n1, LOG2E / tc::STEPS, off)) : 0.f;
                    o[j] = ptx::pack_bf16x2(a, b);
                    if (lo > 0) left[j] = ptx::pack_bf16x2(a - __uint_as_float(o[j] << 16), b - __uint_as_float(o[j] & 0xffff0000u));
                    if (close >= 0) sum += (col + 2 * j != close ? a : 0.f) + (col + 2 * j + 1 != close ? b : 0.f);
                }
                row[g] = make_uint4(o[0], o[1], o[2], o[3]);
                if (lo > 0) rest[g] = make_uint4(left[0], left[1], left[2], left[3]);
            }
        }
    }
    __syncthreads();
    auto put = [&](long long at, float x) {
        if (F32) row32[at] = x;
        else {
            const __nv_bfloat16 hi = __float2bfloat16_rn(x);
            reinterpret_cast<__nv_bfloat16*>(row)[at] = hi;
            if (lo > 0) reinterpret_cast<__nv_bfloat16*>(rest)[at] = __float2bfloat16_rn(x - __bfloat162float(hi));
        }
    };
    if (there) {
        float sub = p_i;
        bool first = true;
        for (int j = 0; j < lists.k; ++j) {
            if (j == i || s_id[j] != static_cast<int>(id)) continue;
            first &= j > i;
            sub += s_p[j];
        }
        if (id == y) sub += beta;
        if (first && id != close) {
            const float x = w * ((beta + mass) * expf(z_i - lse_r) - sub);
            put(id, x);
            sum += x - dense(held);
        }
    }
    bool listed = false;
    for (int j = threadIdx.x; j < lists.k; j += THREADS) listed |= s_id[j] == y;
    if (!__syncthreads_or(listed ? 1 : 0) && threadIdx.x == 0 && y != close) {
        const float x = w * ((beta + mass) * expf(zr[lists.k] - lse_r) - beta);
        put(y, x);
        sum += x - dense(held_y);
    }
    if (close >= 0) {
        sum = block_sum(sum, s_red);
        if (threadIdx.x == 0) put(close, 0.f - sum);
    }
}

}  // namespace tk
}  // namespace cat
