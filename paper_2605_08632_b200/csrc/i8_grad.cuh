// Gradient of the tokens of a small batch through the 8-bit head: dX^T[i, t] = sum_v W[v, i] A[t, v], A the 16-bit terms of the cross entropy's
// gradient (fp16, W the integers) or an upstream dY (bf16, W = scale * integer rounded to bf16).
//
// The tensor cores multiply no 8-bit by 16-bit operands, so the head has to be widened; a copy of it in memory (widen_kernel) is written and read again for
// 4 bytes per weight, against 1 to read it as it is.  With few rows that copy costs more than the product, so here the head is widened on its way:
//   * a CTA owns 128 columns of dX and a part of the vocabulary; its slices of the head, 64 entries x 128 columns in 8 bits, arrive by TMA beside
//     the same 64 columns of A;
//   * two groups of four warps take turns to turn a slice into 16 bits, in the swizzled layout of an MN-major operand (the tensor core transposes it): the
//     head is the M side, 128 columns, the rows of the batch the N side (two MMAs for more than 256);
//   * one fp32 tile of 128 x rows stays in tensor memory over the whole part; the parts are added in order by add_parts_kernel.
// Bound by reading the head for up to about 128 rows, by the shared memory's bandwidth above (operands, slices in and out of it).
#pragma once
#include "i8_head.cuh"

namespace cat {
namespace i8 {

constexpr int GRAD_ROWS = 512;
constexpr int GRAD_SLICE = 64;                       // vocabulary entries
constexpr int GRAD_COLS = 128;                       // columns of dX per CTA
constexpr int GRAD_WIDE = 4;                         // widened slices in flight
constexpr int GRAD_W_BYTES = GRAD_SLICE * GRAD_COLS;
constexpr int GRAD_WIDE_BYTES = 2 * GRAD_W_BYTES;
constexpr int GRAD_MAX_STAGES = 10;
constexpr int GRAD_SMEM = 226 * 1024;
constexpr int GRAD_THREADS = 320;

struct GradCtl {
    unsigned long long full[GRAD_MAX_STAGES], empty[GRAD_MAX_STAGES];
    unsigned long long wide_full[GRAD_WIDE], wide_empty[GRAD_WIDE];
    unsigned long long done, drain;
    uint32_t tmem_base;
    volatile int abort;
};

struct GradParams {
    const float* sw;       // [V]
    float* part;           // [gridDim.y][T][d]
    int T, V, d;
    int n;                 // rows per MMA, a multiple of 16
    int mmas;              // 1 or 2
    int num_kb;            // slices of the vocabulary
    int stages;
    unsigned long long wait_ns;
};

template <bool SCALED, int TMEM>
__global__ void __launch_bounds__(GRAD_THREADS, 1)
grad_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA, const GradParams p, int* status) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ GradCtl ctl;
    const uint32_t wide = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, ring = wide + GRAD_WIDE * GRAD_WIDE_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t b_bytes = static_cast<uint32_t>(p.n) * 128, stage_bytes = GRAD_W_BYTES + p.mmas * b_bytes;
    const int kb0 = static_cast<int>(static_cast<long long>(blockIdx.y) * p.num_kb / gridDim.y);
    const int slices = static_cast<int>((static_cast<long long>(blockIdx.y) + 1) * p.num_kb / gridDim.y) - kb0;
    if (threadIdx.x == 0) {
        ptx::prefetch_tmap(&tmW);
        ptx::prefetch_tmap(&tmA);
        for (int i = 0; i < p.stages; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl.empty[i]), 1);
        }
        for (int i = 0; i < GRAD_WIDE; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.wide_full[i]), 4);
            ptx::mbar_init(ptx::smem_u32(&ctl.wide_empty[i]), 1);
        }
        ptx::mbar_init(ptx::smem_u32(&ctl.done), 1);
        ptx::mbar_init(ptx::smem_u32(&ctl.drain), 1);
        ctl.abort = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        ptx::tmem_alloc<TMEM>(ptx::smem_u32(&ctl.tmem_base));
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = ctl.tmem_base;
    volatile int* abort = &ctl.abort;

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            int issued = 0;
            for (int i = 0; i < slices; ++i) {
                const int s = i % p.stages;
                if (!tc::wait_bounded(ptx::smem_u32(&ctl.empty[s]), ((i / p.stages) & 1) ^ 1u, abort, status, p.wait_ns)) { ok = false; break; }
                const uint32_t full = ptx::smem_u32(&ctl.full[s]), dst = ring + s * stage_bytes;
                const int v = (kb0 + i) * GRAD_SLICE;
                ptx::mbar_arrive_expect_tx(full, stage_bytes);
                ptx::tma_load_2d(dst, &tmW, blockIdx.x * GRAD_COLS, v, full);
                if (i == 0) ptx::grid_dependency_wait();        // A comes from the kernel before this one
                for (int j = 0; j < p.mmas; ++j) ptx::tma_load_2d(dst + GRAD_W_BYTES + j * b_bytes, &tmA, v, j * p.n, full);
                ++issued;
            }
            if (!ok) {      // aborted: let the copies already issued land before the CTA exits
                const int back = issued < p.stages ? issued : p.stages;
                for (int k = 0; k < back; ++k) {
                    const int i = issued - 1 - k;
                    tc::wait_bounded<true>(ptx::smem_u32(&ctl.full[i % p.stages]), (i / p.stages) & 1u, abort, status, tc::DRAIN_LIMIT_NS);
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = SCALED ? ptx::idesc_bf16_f32(128, p.n, 1, 0) : ptx::idesc_f16_f32(128, p.n, 1, 0);
            bool ok = true;
            for (int i = 0; i < slices; ++i) {
                const int s = i % p.stages, w = i % GRAD_WIDE;
                if (!tc::wait_bounded(ptx::smem_u32(&ctl.wide_full[w]), (i / GRAD_WIDE) & 1u, abort, status, p.wait_ns) ||
                    !tc::wait_bounded(ptx::smem_u32(&ctl.full[s]), (i / p.stages) & 1u, abort, status, p.wait_ns)) { ok = false; break; }
                ptx::tc_fence_after();
                const uint64_t ad = ptx::smem_desc_sw128(wide + w * GRAD_WIDE_BYTES, tc::MN_ATOM_BYTES, 1024);
                const uint32_t b = ring + s * stage_bytes + GRAD_W_BYTES;
                for (int m = 0; m < p.mmas; ++m) {
                    const uint64_t bd = ptx::smem_desc_sw128(b + m * b_bytes, 16, 1024);
#pragma unroll
                    for (int j = 0; j < GRAD_SLICE / 16; ++j)
                        ptx::umma_bf16(tmem + m * p.n, ad + j * (2048 >> 4), bd + 2 * j, idesc, (i | j) != 0 ? 1u : 0u);
                }
                ptx::umma_commit(ptx::smem_u32(&ctl.empty[s]));
                ptx::umma_commit(ptx::smem_u32(&ctl.wide_empty[w]));
            }
            ptx::umma_commit(ok ? ptx::smem_u32(&ctl.done) : ptx::smem_u32(&ctl.drain));
            if (!ok) tc::wait_bounded<true>(ptx::smem_u32(&ctl.drain), 0, abort, status, tc::DRAIN_LIMIT_NS);      // no MMA may be in flight when TMEM is freed
        }
        __syncwarp();
    } else {
        const int group = (warp - 2) >> 2, t = threadIdx.x - 64 - 128 * group;
        const int piece = t & 7, row0 = t >> 3;             // 16 columns of every 16th entry
        bool ok = true;
        float next[4];
        const auto scales_of = [&](int i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = (kb0 + i) * GRAD_SLICE + row0 + 16 * q;
                next[q] = i < slices && v < p.V ? __ldg(p.sw + v) : 0.f;
            }
        };
        if (SCALED) scales_of(group);
        for (int i = group; i < slices; i += 2) {
            const int s = i % p.stages, w = i % GRAD_WIDE;
            float scale[4];
            if (SCALED) {
#pragma unroll
                for (int q = 0; q < 4; ++q) scale[q] = next[q];
                scales_of(i + 2);
            }
            ok = tc::wait_bounded(ptx::smem_u32(&ctl.full[s]), (i / p.stages) & 1u, abort, status, p.wait_ns) &&
                 tc::wait_bounded(ptx::smem_u32(&ctl.wide_empty[w]), ((i / GRAD_WIDE) & 1) ^ 1u, abort, status, p.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const uint32_t src = ring + s * stage_bytes, dst = wide + w * GRAD_WIDE_BYTES + (piece >> 2) * tc::MN_ATOM_BYTES;
            uint4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) ptx::ld_shared_v4(src + (row0 + 16 * q) * GRAD_COLS + piece * 16, x[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = row0 + 16 * q;
                const uint32_t in[4] = {x[q].x ^ 0x80808080u, x[q].y ^ 0x80808080u, x[q].z ^ 0x80808080u, x[q].w ^ 0x80808080u};     // 0 .. 255
                uint32_t r[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t pair = __byte_perm(in[j >> 1], 0x64646464u, (j & 1) ? 0x4342 : 0x4140);                          // fp16 1024 + byte
                    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&pair), __half2half2(__ushort_as_half(0x6480)));         // - 1152
                    if (SCALED) {
                        const float2 f = __half22float2(h);
                        r[j] = ptx::pack_bf16x2(f.x * scale[q], f.y * scale[q]);
                    } else {
                        r[j] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
                // 16-byte pieces 2 (piece & 3) and the one after it of a 128-byte row, swizzled; the second half of the lanes begins with the odd one, so
                // that eight lanes write to eight different banks
                const int odd = piece >> 2, c = 2 * (piece & 3);
                const uint32_t line = dst + row * 128;
                ptx::st_shared_v4(line + (((c + odd) ^ (row & 7)) << 4), odd ? r[4] : r[0], odd ? r[5] : r[1], odd ? r[6] : r[2], odd ? r[7] : r[3]);
                ptx::st_shared_v4(line + (((c + 1 - odd) ^ (row & 7)) << 4), odd ? r[0] : r[4], odd ? r[1] : r[5], odd ? r[2] : r[6], odd ? r[3] : r[7]);
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl.wide_full[w]));
        }
        if (ok) {
            ok = tc::wait_bounded(ptx::smem_u32(&ctl.done), 0, abort, status, p.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
        }
        if (ok) {
            ptx::tc_fence_after();
            const int quarter = warp & 3, i0 = blockIdx.x * GRAD_COLS + quarter * 32, i = i0 + lane;
            float* out = p.part + static_cast<long long>(blockIdx.y) * p.T * p.d + i;
            for (int r0 = group * 32; r0 < p.T; r0 += 64) {
                uint32_t v[32];
                ptx::tmem_ld_32x32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + r0, v);
                ptx::tmem_ld_wait(v);
                if (i < p.d) {
#pragma unroll
                    for (int q = 0; q < 32; ++q)
                        if (r0 + q < p.T) out[static_cast<long long>(r0 + q) * p.d] = __uint_as_float(v[q]);
                }
            }
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc<TMEM>(tmem);
    }
}

}  // namespace i8
}  // namespace cat
