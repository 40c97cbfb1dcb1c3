// A few tokens (1 to 128, a decoding step or a small batch) against the whole 8-bit head: logits, the parts of the cross entropy, or the terms
// of its gradient.  All there is to do is to read the head once.  As in skinny.cuh the head's rows are the M side of tcgen05.mma (kind::i8), tiles are
// dealt round robin to one CTA per SM, and a ring of its slices fills the shared memory; a slice of 128 bytes holds 128 integers here.
//
// An accumulator lane is a vocabulary entry, so its scale is one value per thread.  Logits and gradient terms leave in that layout (32 neighbouring
// entries of one token per store); for the softmax sums a warp turns 32 x 32 of them over in shared memory.
//
// The kernel starts while the tokens are still being made into integers by the kernel before it: the head's first slices are fetched meanwhile.
#pragma once
#include "i8_head.cuh"
#include "skinny.cuh"

namespace cat {
namespace i8 {

enum SkinnyMode { SKINNY_BF16, SKINNY_F32, SKINNY_CE, SKINNY_DZ };
constexpr int SKINNY_ROWS = 128;

struct SkinnyParams {
    Head h;
    const float* bias;               // logits; or nullptr
    void* Y;                         // logits [T][ldY], or fp16 gradient terms
    long long ldY;
    const long long* labels;         // cross entropy and its gradient
    const unsigned char* valid;      // gradient
    const float *nll, *lse, *g;
    const int* most;
    float* factor;
    float *part_m, *part_l, *z_label;      // [T][gridDim.x] parts, [T]
    int n;                           // tokens rounded up to 16
    int tile_rows;                   // vocabulary entries per tile: 64, 96 or 128
    int n_tiles, num_kb, stages;
    unsigned long long wait_ns;
};

// TPW: tokens a warp looks after, a multiple of 32; HALVES sets of four epilogue warps; SUB tiles of the head per slice of the tokens, even for one token (32 us
// for 1 x 1024 x 151936 with one tile and one set, 29 with two).
constexpr int HALVES = 2, SUB = 2;
constexpr int SKINNY_THREADS = 64 + 128 * HALVES;
template <int MODE, int TPW>
__global__ void __launch_bounds__(SKINNY_THREADS, 1)
skinny_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const SkinnyParams p, int* status) {
    constexpr int COLS = TPW * HALVES;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ skinny::Ctl ctl;
    __shared__ float4 s_tok[COLS];                                       // what a token's column needs
    __shared__ float s_m[4][MODE == SKINNY_CE ? COLS : 1], s_l[4][MODE == SKINNY_CE ? COLS : 1];
    __shared__ float s_turn[MODE == SKINNY_CE ? 4 * HALVES : 1][32 * 33];
    const uint32_t ring = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_bytes = static_cast<uint32_t>(p.n) * 128;
    const uint32_t a_bytes = static_cast<uint32_t>(p.tile_rows) * 128;       // the MMA reads 128 rows, the last ones into lanes that nobody looks at
    const uint32_t stage_bytes = SUB * a_bytes + b_bytes;
    if (threadIdx.x == 0) {
        ptx::prefetch_tmap(&tmW);
        ptx::prefetch_tmap(&tmX);
        for (int i = 0; i < p.stages; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl.empty[i]), 1);
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
            bool ok = true, ready = false;
            // slice `kb` of round t: the head's part, the tokens' part
            const auto load_w = [&](int t, int kb, int s) {
                const uint32_t full = ptx::smem_u32(&ctl.full[s]), dst = ring + s * stage_bytes;
                const int n_sub = t + static_cast<int>(gridDim.x) >= p.n_tiles ? 1 : SUB;      // the last round may have one tile
                ptx::mbar_arrive_expect_tx(full, n_sub * a_bytes + b_bytes);
                for (int j = 0; j < n_sub; ++j) ptx::tma_load_2d(dst + j * a_bytes, &tmW, kb * 128, (t + j * static_cast<int>(gridDim.x)) * p.tile_rows, full);
            };
            const auto load_x = [&](int kb, int s) { ptx::tma_load_2d(ring + s * stage_bytes + SUB * a_bytes, &tmX, kb * 128, 0, ptx::smem_u32(&ctl.full[s])); };
            for (int t = blockIdx.x; t < p.n_tiles && ok; t += SUB * gridDim.x) {
                for (int kb = 0; kb < p.num_kb; ++kb) {
                    if (!ready && issued == p.stages) {          // the ring's first fill: the head alone, then the tokens
                        ptx::grid_dependency_wait();
                        for (int i = 0; i < issued; ++i) load_x(i % p.num_kb, i);
                        ready = true;
                    }
                    if (!tc::wait_bounded(ptx::smem_u32(&ctl.empty[stage]), phase ^ 1u, abort, status, p.wait_ns)) { ok = false; break; }
                    load_w(t, kb, stage);
                    if (ready) load_x(kb, stage);
                    ++issued;
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ready) {
                ptx::grid_dependency_wait();
                for (int i = 0; i < issued; ++i) load_x(i % p.num_kb, i);
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
            const uint32_t idesc = ptx::idesc_i8_s32(128, p.n);
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
                    const int n_sub = t + static_cast<int>(gridDim.x) >= p.n_tiles ? 1 : SUB;
                    for (int i = 0; i < n_sub; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            ptx::umma_i8(tmem + (acc * SUB + i) * COLS, ad + i * (a_bytes >> 4) + 2 * j, bd + 2 * j, idesc, (kb | j) != 0 ? 1u : 0u);
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
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const int T = p.h.T;
        const auto token = [&](int c) { return (c * HALVES + half) * 32; };      // first token of this warp's chunk c: dealt in turn, so that no set idles
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
        ptx::grid_dependency_wait();
        float up = 0.f, down = 0.f;
        if (MODE == SKINNY_DZ) fit_half(p.most, up, down);
        for (int t = threadIdx.x - 64; t < COLS; t += 128 * HALVES) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (t < T) {
                v.x = MODE == SKINNY_BF16 || MODE == SKINNY_F32 ? p.h.sx[t] : log2_scale(p.h.sx[t]);
                if (MODE == SKINNY_CE) {
                    const long long y = p.labels[t];
                    v.y = __int_as_float(y >= 0 && y < p.h.V ? static_cast<int>(y) : -1);
                }
                if (MODE == SKINNY_DZ) {
                    const RowGrad q = row_grad(t, T, p.h.V, p.labels, p.valid, p.nll, p.lse, p.g);
                    v.y = __int_as_float(q.y);
                    v.z = -q.others2;
                    v.w = q.on ? 1.f : 0.f;
                    if (blockIdx.x == 0) p.factor[t] = q.factor * down;
                }
            }
            s_tok[t] = v;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(128 * HALVES) : "memory");
        RowSums sums[TPW / 32];          // of token token(c) + lane, over this warp's vocabulary entries
        int label[TPW / 32];
        if (MODE == SKINNY_CE) {
#pragma unroll
            for (int c = 0; c < TPW / 32; ++c) {
                const float4 v = s_tok[token(c) + lane];
                sums[c].m = LOW2; sums[c].l = 0.f; sums[c].a = v.x;
                label[c] = token(c) + lane < T ? __float_as_int(v.y) : -1;
            }
        }
        uint32_t acc = 0, acc_phase = 0;
        bool ok = true;
        // the scales (and biases) of a round's entries are fetched a round ahead
        const auto scale_at = [&](const float* x, int t) {
            const int v = t * p.tile_rows + quarter * 32 + lane;
            return x != nullptr && t < p.n_tiles && quarter * 32 < p.tile_rows && v < p.h.V ? __ldg(x + v) : 0.f;
        };
        float w_next[SUB], b_next[SUB];
#pragma unroll
        for (int j = 0; j < SUB; ++j) {
            w_next[j] = scale_at(p.h.sw, blockIdx.x + j * gridDim.x);
            b_next[j] = MODE <= SKINNY_F32 ? scale_at(p.bias, blockIdx.x + j * gridDim.x) : 0.f;
        }
        for (int t0 = blockIdx.x; t0 < p.n_tiles; t0 += SUB * gridDim.x) {
            float w[SUB], b[SUB];
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                w[j] = w_next[j]; b[j] = b_next[j];
                w_next[j] = scale_at(p.h.sw, t0 + (SUB + j) * gridDim.x);
                if (MODE <= SKINNY_F32) b_next[j] = scale_at(p.bias, t0 + (SUB + j) * gridDim.x);
            }
            ok = tc::wait_bounded(ptx::smem_u32(&ctl.tfull[acc]), acc_phase, abort, status, p.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                const int t = t0 + j * static_cast<int>(gridDim.x);
                const int v0 = t * p.tile_rows + quarter * 32, v = v0 + lane;
                const bool in_tile = t < p.n_tiles && quarter * 32 < p.tile_rows && v0 < p.h.V;        // the warp has vocabulary entries
#pragma unroll
                for (int c = 0; c < TPW / 32; ++c) {
                    const int tok = token(c);
                    if (!in_tile || tok >= T) continue;
                    uint32_t raw[32];
                    ptx::tmem_ld_32x32(lanes + (acc * SUB + j) * COLS + tok, raw);
                    ptx::tmem_ld_wait(raw);
                    if (MODE == SKINNY_CE) {
                        float* turn = s_turn[warp - 2];
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 32; ++i) turn[i * 33 + lane] = v < p.h.V ? __int2float_rn(static_cast<int>(raw[i])) * w[j] : -INFINITY;
                        __syncwarp();
                        float f[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = turn[lane * 33 + i];
                        const int rel = label[c] - v0;
                        if (rel >= 0 && rel < 32) {
                            float zy = 0.f;
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (i == rel) { zy = f[i]; f[i] = -INFINITY; }
                            p.z_label[tok + lane] = zy * sums[c].a;
                        }
                        sums[c].add(f);
                    } else {
                        const int live = min(32, T - tok);
                        if (v < p.h.V) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                if (i >= live) break;
                                const float f = __int2float_rn(static_cast<int>(raw[i])) * w[j];
                                const long long at = static_cast<long long>(tok + i) * p.ldY + v;
                                if (MODE == SKINNY_DZ) {
                                    const float4 s = s_tok[tok + i];
                                    float x = ptx::ex2_approx(fmaf(f, s.x, s.z)) * (w[j] * up);
                                    if (__float_as_int(s.y) == v) x = -w[j] * up;
                                    if (s.w == 0.f) x = 0.f;
                                    static_cast<uint16_t*>(p.Y)[at] = static_cast<uint16_t>(ptx::pack_f16x2_sat(x, 0.f));
                                } else {
                                    const float y = __fadd_rn(__fmul_rn(f, s_tok[tok + i].x), b[j]);
                                    if (MODE == SKINNY_F32) static_cast<float*>(p.Y)[at] = y;
                                    else static_cast<__nv_bfloat16*>(p.Y)[at] = __float2bfloat16(y);
                                }
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl.tempty[acc]));
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        }
        if (MODE == SKINNY_CE) {
#pragma unroll
            for (int c = 0; c < TPW / 32; ++c) {
                s_m[quarter][token(c) + lane] = sums[c].m;
                s_l[quarter][token(c) + lane] = sums[c].l;
            }
            asm volatile("bar.sync 1, %0;" ::"n"(128 * HALVES) : "memory");
            const int i = threadIdx.x - 64;
            if (ok && i < T) {      // four quarters of the tiles -> one entry per CTA
                float m = s_m[0][i], l = 0.f;
#pragma unroll
                for (int q = 1; q < 4; ++q) m = fmaxf(m, s_m[q][i]);
#pragma unroll
                for (int q = 0; q < 4; ++q) l = fmaf(s_l[q][i], exp2f(s_m[q][i] - m), l);
                p.part_m[i * gridDim.x + blockIdx.x] = m;
                p.part_l[i * gridDim.x + blockIdx.x] = l;
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<2 * SUB * COLS>(tmem);
    }
}

}  // namespace i8
}  // namespace cat
