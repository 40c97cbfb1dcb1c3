// The logits of a few rows (a decoding step: 1 to 128 hidden states) over the whole vocabulary, with softmax statistics, entropy sums and
// the material for the top alternatives.  All there is to do is to read W once, so this kernel is built around that:
//
//   * operands swapped: W's rows are the M side of tcgen05.mma (128 vocabulary entries per tile), the hidden states the N
//     side (rows rounded up to 16), so that no tensor-core or shared-memory work is spent on padding H to 256 rows;
//   * one CTA per SM, tiles of `tile_rows` vocabulary entries dealt round robin, a ring of W slices that fills the shared memory: 120 to
//     150 KB of W in flight per SM (the GEMM of tc_gemm.cuh has 96 KB), which is what the memory's latency asks for;
//   * an accumulator lane is a vocabulary entry and a column a hidden state: a warp turns 32 x 32 logits over in shared memory, after
//     which a thread holds 32 neighbouring logits of one hidden state and goes on like the epilogue of logprob.cuh.  (Reducing
//     across the lanes instead, one redux and five shuffles per hidden state, took 125 us for 67 rows of 1024 x 151936;
//     this way 61 us.)  Running sums stay in registers over all tiles of the CTA; warps and CTAs are merged at the end;
//   * with alternatives, four more warps sum the squares of W's rows as their slices pass, for the bound on the logits' errors
//     (lp::gemm_error): the longest row is known without another pass over W.
// Measured, with alternatives: one row of 2048 x 128256 (W 525 MB) 82 us, 6.4 TB/s, the rate of a plain copy; 67 rows of 1024 x 151936 (311 MB)
// 70 us, 4.4 TB/s: the slices of H share the ring, start and end of the launch are a seventh of it, and the squares hold every slice for
// a while longer (61 us without them).
#pragma once
#include "logprob.cuh"

namespace cat {
namespace skinny {

using tc::BK;
constexpr int MAX_ROWS = 128;
constexpr int MAX_STAGES = 12;
constexpr int SMEM_BYTES = 180 * 1024;       // ring, with the slack to align it

struct Ctl {
    unsigned long long full[MAX_STAGES];
    unsigned long long empty[MAX_STAGES];
    unsigned long long tfull[2];
    unsigned long long tempty[2];
    unsigned long long drain;
    uint32_t tmem_base;
    volatile int abort;
};

struct Params {
    float* part_m;        // [gridDim.x][part_stride]
    float* part_l;
    float* part_u;
    int* part_id;
    float* gmax;          // [T][ld_g] maxima of 32 neighbouring columns; nullptr (and zs) without alternatives
    __half* zs;           // [T][ldz] logits as distances from those maxima
    int* w_sq;            // raised to the largest sum of squares of a row of W (float bits)
    long long part_stride, ld_g, ldz;
    int T, V;
    int n;                // rows of H in a tile of it: T rounded up to 16
    int tile_rows;        // vocabulary entries per tile: 64, 96 or 128
    int n_tiles;
    int num_kb;           // 64-wide slices of d
    int stages;
    unsigned long long wait_ns;
};

// TPW: hidden states a warp looks after; HALVES: sets of four epilogue warps (HALVES * TPW >= T); SUB: W tiles that a slice of H is
// loaded for.  With many rows the slices of H take as much of the ring as those of W; two tiles per slice of H leave more of it to W.
// Threads: 64 + 128 HALVES, and NORM_THREADS more with alternatives.
constexpr int NORM_THREADS = 128;
template <int TPW, int HALVES, int SUB>
__global__ void __launch_bounds__(64 + 128 * HALVES + NORM_THREADS, 1)
logits_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmH, const Params p, int* status) {
    constexpr int COLS = TPW * HALVES;                       // accumulator columns (a power of two >= 32)
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ Ctl ctl;
    __shared__ float s_m[4][COLS], s_l[4][COLS], s_u[4][COLS];
    __shared__ int s_id[4][COLS];
    __shared__ float s_turn[4 * HALVES][32 * 33];
    const uint32_t ring = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_bytes = static_cast<uint32_t>(p.n) * BK * 2;
    // the slot of a W slice holds its tile_rows rows; the MMA reads 128, the last ones out of whatever follows, into accumulator
    // lanes that nobody looks at (the last slot is followed by 8 KB of slack)
    const uint32_t a_bytes = static_cast<uint32_t>(p.tile_rows) * BK * 2;
    const uint32_t stage_bytes = SUB * a_bytes + b_bytes;
    if (threadIdx.x == 0) {
        ptx::prefetch_tmap(&tmW);
        ptx::prefetch_tmap(&tmH);
        for (int i = 0; i < p.stages; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl.empty[i]), p.gmax != nullptr ? 1 + NORM_THREADS / 32 : 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.tfull[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl.tempty[i]), 4 * HALVES);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl.drain), 1);
        ctl.abort = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc<2 * SUB * COLS>(ptx::smem_u32(&ctl.tmem_base));
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl.tmem_base;
    volatile int* abort = &ctl.abort;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0, issued = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < p.n_tiles && ok; t += SUB * gridDim.x) {
                for (int kb = 0; kb < p.num_kb; ++kb) {
                    if (!tc::wait_bounded(ptx::smem_u32(&ctl.empty[stage]), phase ^ 1u, abort, status, p.wait_ns)) { ok = false; break; }
                    const uint32_t full = ptx::smem_u32(&ctl.full[stage]), dst = ring + stage * stage_bytes;
                    const int n_sub = SUB == 1 || t + static_cast<int>(gridDim.x) >= p.n_tiles ? 1 : SUB;      // the last round may have one tile
                    ptx::mbar_arrive_expect_tx(full, n_sub * a_bytes + b_bytes);
                    for (int j = 0; j < n_sub; ++j)
                        ptx::tma_load_2d(dst + j * a_bytes, &tmW, kb * BK, (t + j * static_cast<int>(gridDim.x)) * p.tile_rows, full);
                    ptx::tma_load_2d(dst + SUB * a_bytes, &tmH, kb * BK, 0, full);
                    ++issued;
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok) {      // aborted: let the copies already issued land before the CTA exits
                const int back = issued < p.stages ? issued : p.stages;
                for (int i = 0; i < back; ++i) {
                    const int q = issued - 1 - i;
                    tc::wait_bounded<true>(ptx::smem_u32(&ctl.full[q % p.stages]), (q / p.stages) & 1u, abort, status, tc::DRAIN_LIMIT_NS);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = ptx::idesc_bf16_f32(128, p.n, 0, 0);
            int stage = 0;
            uint32_t phase = 0, acc = 0, acc_phase = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < p.n_tiles && ok; t += SUB * gridDim.x) {
                if (!tc::wait_bounded(ptx::smem_u32(&ctl.tempty[acc]), acc_phase ^ 1u, abort, status, p.wait_ns)) { ok = false; break; }
                ptx::tc_fence_after();
                for (int kb = 0; kb < p.num_kb; ++kb) {
                    if (!tc::wait_bounded(ptx::smem_u32(&ctl.full[stage]), phase, abort, status, p.wait_ns)) { ok = false; break; }
                    ptx::tc_fence_after();
                    const uint32_t at = ring + stage * stage_bytes;
                    const uint64_t ad = ptx::smem_desc_sw128(at, 16, 1024), bd = ptx::smem_desc_sw128(at + SUB * a_bytes, 16, 1024);
                    const int n_sub = SUB == 1 || t + static_cast<int>(gridDim.x) >= p.n_tiles ? 1 : SUB;
                    for (int i = 0; i < n_sub; ++i)
#pragma unroll
                        for (int j = 0; j < BK / 16; ++j)
                            ptx::umma_bf16(tmem + (acc * SUB + i) * COLS, ad + i * (a_bytes >> 4) + 2 * j, bd + 2 * j, idesc, (kb | j) != 0 ? 1u : 0u);
                    ptx::umma_commit(ptx::smem_u32(&ctl.empty[stage]));
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
                if (!ok) break;
                ptx::umma_commit(ptx::smem_u32(&ctl.tfull[acc]));
                acc ^= 1u;
                if (acc == 0) acc_phase ^= 1u;
            }
            if (!ok) {      // aborted: no MMA may be in flight when TMEM is freed
                ptx::umma_commit(ptx::smem_u32(&ctl.drain));
                tc::wait_bounded<true>(ptx::smem_u32(&ctl.drain), 0, abort, status, tc::DRAIN_LIMIT_NS);
            }
        }
        __syncwarp();
    } else if (warp >= 2 + 4 * HALVES) {
        // Squares of W's rows: the rows of a round's tiles lie one behind the other in the slot, and a thread takes every 128th.  A row's 16-byte
        // pieces are read in an order of the lane's own, so that eight lanes meet eight different banks (the swizzle only moves pieces
        // within a row).
        const int i = threadIdx.x - (64 + 128 * HALVES);
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        float most = 0.f;
        for (int t = blockIdx.x; t < p.n_tiles && ok; t += SUB * gridDim.x) {
            float sq[SUB];
#pragma unroll
            for (int j = 0; j < SUB; ++j) sq[j] = 0.f;
            const int n_rows = (SUB == 1 || t + static_cast<int>(gridDim.x) >= p.n_tiles ? 1 : SUB) * p.tile_rows;
            for (int kb = 0; kb < p.num_kb; ++kb) {
                ok = tc::wait_bounded(ptx::smem_u32(&ctl.full[stage]), phase, abort, status, p.wait_ns);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < SUB; ++j) {
                    const int q = j * NORM_THREADS + i;
                    if (q >= n_rows) break;
                    const uint32_t row = ring + stage * stage_bytes + q * (BK * 2);
                    uint4 x[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) ptx::ld_shared_v4(row + ((c ^ (lane & 7)) << 4), x[c]);
                    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < 8; ++c) a[c & 3] = lp::add_squares(a[c & 3], x[c]);
                    const float sum = (a[0] + a[1]) + (a[2] + a[3]);
                    sq[j] += sum;
                    if (sum == 0.f) {
                        bool any = false;
#pragma unroll
                        for (int c = 0; c < 8; ++c) any |= lp::any_of(x[c]);
                        if (any) sq[j] += lp::NOT_ZERO;
                    }
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl.empty[stage]));
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
#pragma unroll
            for (int j = 0; j < SUB; ++j) most = sq[j] <= most ? most : sq[j];        // NaN stays
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, most, off);
            most = o <= most ? most : o;
        }
        if (lane == 0) lp::raise_to(p.w_sq, most);
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const int tok0 = half * TPW;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        float* turn = s_turn[warp - 2];
        tc::RunningSums sums[TPW / 32];          // of hidden state tok0 + 32 c + lane, over this warp's vocabulary entries
        int id[TPW / 32];
#pragma unroll
        for (int i = 0; i < TPW / 32; ++i) { sums[i].clear(); id[i] = 0; }
        uint32_t acc = 0, acc_phase = 0;
        bool ok = true;
        for (int t0 = blockIdx.x; t0 < p.n_tiles; t0 += SUB * gridDim.x) {
            ok = tc::wait_bounded(ptx::smem_u32(&ctl.tfull[acc]), acc_phase, abort, status, p.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            for (int j = 0, t = t0; j < SUB && t < p.n_tiles; ++j, t += gridDim.x) {
                const int v0 = t * p.tile_rows + quarter * 32;
                const bool in_tile = quarter * 32 < p.tile_rows && v0 < p.V;        // the warp has vocabulary entries
#pragma unroll
                for (int c = 0; c < TPW / 32; ++c) {
                    const int tok = tok0 + c * 32;
                    if (!in_tile || tok >= p.T) continue;
                    uint32_t raw[32];
                    ptx::tmem_ld_32x32(lanes + (acc * SUB + j) * COLS + tok, raw);
                    ptx::tmem_ld_wait();
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 32; ++i) turn[i * 33 + lane] = __uint_as_float(raw[i]);
                    __syncwarp();
                    float f[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[i] = turn[lane * 33 + i];
                    const int live = p.V - v0;
                    if (live < 32) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= live) f[i] = tc::LP_LOW;
                    }
                    const float g = tc::max_of(f);
                    if (g > sums[c].m) id[c] = v0 + tc::first_at(f, g);
                    sums[c].add(f, g);
                    if (p.gmax != nullptr && tok + lane < p.T) {
                        p.gmax[static_cast<long long>(tok + lane) * p.ld_g + (v0 >> 5)] = g;
                        // the pitch covers whole groups of 32 columns, so the last one may be written past the vocabulary
                        uint4* out = reinterpret_cast<uint4*>(p.zs + static_cast<long long>(tok + lane) * p.ldz + v0);
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            out[q] = make_uint4(ptx::pack_f16x2_sat(f[q * 8 + 0] - g, f[q * 8 + 1] - g), ptx::pack_f16x2_sat(f[q * 8 + 2] - g, f[q * 8 + 3] - g),
                                                ptx::pack_f16x2_sat(f[q * 8 + 4] - g, f[q * 8 + 5] - g), ptx::pack_f16x2_sat(f[q * 8 + 6] - g, f[q * 8 + 7] - g));
                    }
                }
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl.tempty[acc]));
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        }
#pragma unroll
        for (int c = 0; c < TPW / 32; ++c) {
            s_m[quarter][tok0 + c * 32 + lane] = sums[c].m;
            s_l[quarter][tok0 + c * 32 + lane] = sums[c].l;
            s_u[quarter][tok0 + c * 32 + lane] = sums[c].u;
            s_id[quarter][tok0 + c * 32 + lane] = id[c];
        }
        asm volatile("bar.sync 1, %0;" ::"n"(128 * HALVES) : "memory");
        const int i = threadIdx.x - 64;
        if (ok && i < p.T) {      // four quarters of the tile -> one entry per CTA
            float mm = s_m[0][i];
            int at_max = s_id[0][i];
#pragma unroll
            for (int q = 1; q < 4; ++q)
                if (s_m[q][i] > mm || (s_m[q][i] == mm && s_id[q][i] < at_max)) { mm = s_m[q][i]; at_max = s_id[q][i]; }
            float ll = 0.f, uu = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float dm = (s_m[q][i] - mm) * tc::LOG2E, sc = exp2f(dm);
                uu += sc * fmaf(dm, s_l[q][i], s_u[q][i]);
                ll = fmaf(sc, s_l[q][i], ll);
            }
            const long long at = blockIdx.x * p.part_stride + i;
            p.part_m[at] = mm;
            p.part_l[at] = ll;
            p.part_u[at] = uu;
            p.part_id[at] = at_max;
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<2 * SUB * COLS>(tmem);
    }
}

}  // namespace skinny
}  // namespace cat
