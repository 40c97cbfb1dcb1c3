// Gradient of the tokens of a small batch (up to 448 rows a pass) through the 8-bit head: dX[t, i] = sum_v A[t, v] W[v, i], A the 16-bit terms of the cross entropy's
// gradient (fp16, W the integers) or an upstream dY (bf16, W = scale * integer rounded to bf16: why, at widen_kernel).
//
// The tensor cores multiply no 8-bit by 16-bit operands, so the head has to be widened; a copy of it in memory (widen_kernel) is written and read again for
// 4 bytes per weight, against 1 to read it as it is.  With few rows that copy costs more than the product, so here the head is widened on its way:
//   * a CTA owns 256 columns of dX (128 for more than 256 rows) and a part of the vocabulary; its slices of the head, 64 entries x 128 columns in 8 bits,
//     arrive by TMA beside the same entries' columns of A;
//   * two groups of four warps take turns to turn a stage's slices into 16 bits, in the swizzled layout of an MN-major operand (the tensor core
//     transposes it);
//   * the fp32 tile of rows x columns stays in tensor memory over the whole part; the parts are added in order by add_parts_kernel.
// Up to 256 rows: they are the M side, in tiles of 128 however few there are, and the head the N side, 256 columns (an MMA with 128 columns of the head
// as M side and a few rows as N side takes as long: 16 rows of 1024 x 151936 68 us that way, 63 this).  Above, where A leaves room for 128 columns
// only, those are the M side and the rows the N side of two MMAs, in steps of 32 rows (300 rows 106 us, with rows as M side 169).  More rows than fit
// three stages go in two passes.
// Bound by the handshakes around each 64 entries (barriers, commits) rather than by memory or the tensor cores: about 1000 cycles per slice.
#pragma once
#include "i8_head.cuh"

namespace cat {
namespace i8 {

constexpr int GRAD_ROWS = 448;                       // a stage of 128 columns and so many rows fits three times
constexpr int GRAD_SLICE = 64;                       // vocabulary entries of a stage
constexpr int GRAD_COLS = 128;                       // columns of dX of a unit
constexpr int GRAD_UNIT_BYTES = GRAD_SLICE * GRAD_COLS;
constexpr int GRAD_WIDE = 2;                         // buffers of a stage's widened units, one for each group of warps
constexpr int GRAD_MAX_STAGES = 8;
constexpr int GRAD_SMEM = 226 * 1024;
constexpr int GRAD_THREADS = 320;

struct GradCtl {
    unsigned long long full[GRAD_MAX_STAGES], empty[GRAD_MAX_STAGES];
    unsigned long long wide_full[GRAD_WIDE];
    unsigned long long done, drain;
    uint32_t tmem_base;
    volatile int abort;
};

struct GradParams {
    const float* sw;       // [V]
    float* part;           // [gridDim.y][T][d]
    int T, V, d;
    int n;                 // rows of A per box, a multiple of 16: up to 128, or with the head as M side up to 256
    int tiles;             // boxes of them
    int num_kb;            // slices of the vocabulary
    int stages;            // 3 or more: see the widened buffers
    int first;             // no kernel of the call runs before this one
    unsigned long long wait_ns;
};

// UNITS: units per CTA side by side.  HEAD_M: the head is the M side.
template <bool SCALED, int TMEM, int UNITS, bool HEAD_M>
__global__ void __launch_bounds__(GRAD_THREADS, 1)
grad_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA, const GradParams p, int* status) {
    constexpr int N = UNITS * GRAD_COLS;           // columns of dX
    static_assert(!HEAD_M || UNITS == 1, "128 columns are an M side");
    constexpr int WIDE_BYTES = GRAD_WIDE * UNITS * 2 * GRAD_UNIT_BYTES;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ GradCtl ctl;
    const uint32_t wide = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u, ring = wide + WIDE_BYTES;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the slot of a tile of A holds its n rows; as M side the MMA reads 128, the last ones out of whatever follows, into accumulator lanes that nobody looks at
    const uint32_t a_bytes = static_cast<uint32_t>(p.n) * 128, stage_bytes = UNITS * GRAD_UNIT_BYTES + p.tiles * a_bytes;
    const int kb0 = static_cast<int>(static_cast<long long>(blockIdx.y) * p.num_kb / gridDim.y);
    const int n_iter = static_cast<int>((static_cast<long long>(blockIdx.y) + 1) * p.num_kb / gridDim.y) - kb0;
    const int col0 = blockIdx.x * N;
    if (threadIdx.x == 0) {
        // where this is the call's first kernel, it clears the status: long before a wait of any CTA can run out
        if (p.first && blockIdx.x == 0 && blockIdx.y == 0) *status = 0;
        ptx::prefetch_tmap(&tmW);
        ptx::prefetch_tmap(&tmA);
        for (int i = 0; i < p.stages; ++i) {
            ptx::mbar_init(ptx::smem_u32(&ctl.full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&ctl.empty[i]), 1);
        }
        for (int i = 0; i < GRAD_WIDE; ++i) ptx::mbar_init(ptx::smem_u32(&ctl.wide_full[i]), 4);
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
            int issued = 0, s = 0;
            uint32_t phase = 0, dst = ring;
            for (int i = 0; i < n_iter; ++i) {
                if (!tc::wait_bounded(ptx::smem_u32(&ctl.empty[s]), phase ^ 1u, abort, status, p.wait_ns)) { ok = false; break; }
                const uint32_t full = ptx::smem_u32(&ctl.full[s]);
                const int v = (kb0 + i) * GRAD_SLICE;
                ptx::mbar_arrive_expect_tx(full, stage_bytes);
                ptx::tma_load_2d(dst, &tmW, col0, v, full);
                if (i == 0) ptx::grid_dependency_wait();        // A comes from the kernel before this one
                for (int j = 0; j < p.tiles; ++j) ptx::tma_load_2d(dst + UNITS * GRAD_UNIT_BYTES + j * a_bytes, &tmA, v, j * (HEAD_M ? p.n : 128), full);
                ++issued;
                dst += stage_bytes;
                if (++s == p.stages) { s = 0; phase ^= 1u; dst = ring; }
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
            const uint32_t idesc = SCALED ? ptx::idesc_bf16_f32(128, HEAD_M ? p.n : N, HEAD_M, !HEAD_M) : ptx::idesc_f16_f32(128, HEAD_M ? p.n : N, HEAD_M, !HEAD_M);
            const uint64_t wd0 = ptx::smem_desc_sw128(wide, tc::MN_ATOM_BYTES, 1024);
            bool ok = true;
            int s = 0, w = 0;
            uint32_t phase = 0, w_phase = 0, a = ring + UNITS * GRAD_UNIT_BYTES;
            for (int i = 0; i < n_iter; ++i) {
                if (!tc::wait_bounded(ptx::smem_u32(&ctl.wide_full[w]), w_phase, abort, status, p.wait_ns) ||
                    !tc::wait_bounded(ptx::smem_u32(&ctl.full[s]), phase, abort, status, p.wait_ns)) { ok = false; break; }
                ptx::tc_fence_after();
                const uint64_t wd = wd0 + static_cast<uint64_t>(w * (UNITS * 2 * GRAD_UNIT_BYTES >> 4));
                for (int m = 0; m < p.tiles; ++m) {
                    const uint64_t ad = ptx::smem_desc_sw128(a + m * a_bytes, 16, 1024);
#pragma unroll
                    for (int j = 0; j < GRAD_SLICE / 16; ++j) {
                        const uint64_t w_at = wd + j * (2048 >> 4), a_at = ad + 2 * j;
                        ptx::umma_bf16(tmem + m * (HEAD_M ? p.n : N), HEAD_M ? w_at : a_at, HEAD_M ? a_at : w_at, idesc, (i | j) != 0 ? 1u : 0u);
                    }
                }
                ptx::umma_commit(ptx::smem_u32(&ctl.empty[s]));
                a += stage_bytes;
                if (++s == p.stages) { s = 0; phase ^= 1u; a = ring + UNITS * GRAD_UNIT_BYTES; }
                if (++w == GRAD_WIDE) { w = 0; w_phase ^= 1u; }
            }
            ptx::umma_commit(ok ? ptx::smem_u32(&ctl.done) : ptx::smem_u32(&ctl.drain));
            if (!ok) tc::wait_bounded<true>(ptx::smem_u32(&ctl.drain), 0, abort, status, tc::DRAIN_LIMIT_NS);      // no MMA may be in flight when TMEM is freed
        }
        __syncwarp();
    } else {
        const int group = (warp - 2) >> 2, t = threadIdx.x - 64 - 128 * group;
        const int piece = t & 7, row0 = t >> 3;             // 16 columns of every 16th entry
        // A lane's 16 columns are 16-byte pieces 2 (piece & 3) and the one after it of a 128-byte row, swizzled by the row (the same for all of its rows); the
        // second half of the lanes begins with the odd one, so that eight lanes write to eight different banks.
        const int odd = piece >> 2, c = 2 * (piece & 3);
        const uint32_t from = row0 * N + piece * 16, to = odd * tc::MN_ATOM_BYTES + row0 * 128;
        const uint32_t first = to + (((c + odd) ^ (row0 & 7)) << 4), second = to + (((c + 1 - odd) ^ (row0 & 7)) << 4);
        bool ok = true;
        float next[4];
        const auto scales_of = [&](int i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = (kb0 + i) * GRAD_SLICE + row0 + 16 * q;
                next[q] = i < n_iter && v < p.V ? __ldg(p.sw + v) : 0.f;
            }
        };
        if (SCALED) scales_of(group);
        const int w = group;
        int s = group;
        uint32_t phase = 0;
        // A widened buffer is free again when the stage that it was made from is: with more stages than buffers that barrier cannot complete once more before
        // the buffer is filled anew.  (A commit of its own costs the issuing thread 170 cycles.)
        uint32_t free_bar = 0, free_phase = 0;
        for (int i = group; i < n_iter; i += 2) {
            float scale[4];
            if (SCALED) {
#pragma unroll
                for (int q = 0; q < 4; ++q) scale[q] = next[q];
                scales_of(i + 2);
            }
            // In this order.  A wait names one of two phases, so it holds only where the phase before has completed for sure; with an odd number of stages the
            // slot's last slice was the other group's, whose copy may still be under way when this group comes here.  Once the MMAs of slice i - 2 are
            // done, so are those of i - stages, which waited for that copy.  (The other way round a group could take a slot for filled that still held
            // slice i - 3, and widened that: seen in one call in 30 to 150 with 449 rows of 2048 x 25001.)
            if (i >= 2) ok = tc::wait_bounded(free_bar, free_phase, abort, status, p.wait_ns);
            ok = ok && tc::wait_bounded(ptx::smem_u32(&ctl.full[s]), phase, abort, status, p.wait_ns);
            free_bar = ptx::smem_u32(&ctl.empty[s]);
            free_phase = phase;
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const uint32_t src = ring + s * stage_bytes + u * GRAD_COLS + from, dst = wide + (w * UNITS + u) * (2 * GRAD_UNIT_BYTES);
                uint4 x[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) ptx::ld_shared_v4(src + q * 16 * N, x[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t in[4] = {x[q].x ^ 0x80808080u, x[q].y ^ 0x80808080u, x[q].z ^ 0x80808080u, x[q].w ^ 0x80808080u};     // 0 .. 255
                    uint32_t r[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const __half2 h = widened(in[j >> 1], j & 1);
                        if (SCALED) {
                            const float2 f = __half22float2(h);
                            r[j] = ptx::pack_bf16x2(f.x * scale[q], f.y * scale[q]);
                        } else {
                            r[j] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                    ptx::st_shared_v4(dst + first + q * 2048, odd ? r[4] : r[0], odd ? r[5] : r[1], odd ? r[6] : r[2], odd ? r[7] : r[3]);
                    ptx::st_shared_v4(dst + second + q * 2048, odd ? r[0] : r[4], odd ? r[1] : r[5], odd ? r[2] : r[6], odd ? r[3] : r[7]);
                }
            }
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&ctl.wide_full[w]));
            s += 2;
            if (s >= p.stages) { s -= p.stages; phase ^= 1u; }
        }
        if (ok) {
            ok = tc::wait_bounded(ptx::smem_u32(&ctl.done), 0, abort, status, p.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
        }
        if (ok) {
            ptx::tc_fence_after();
            const int quarter = warp & 3;
            const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
            if (HEAD_M) {                    // a lane is a column
                const int i = col0 + quarter * 32 + lane;
                float* out = p.part + static_cast<long long>(blockIdx.y) * p.T * p.d + i;
                for (int r0 = group * 32; r0 < p.T; r0 += 64) {
                    uint32_t v[32];
                    ptx::tmem_ld_32x32(lanes + r0, v);
                    ptx::tmem_ld_wait(v);
                    if (i < p.d) {
#pragma unroll
                        for (int q = 0; q < 32; ++q)
                            if (r0 + q < p.T) out[static_cast<long long>(r0 + q) * p.d] = __uint_as_float(v[q]);
                    }
                }
            }
            // a lane is a row: 32 x 32 are turned over in the memory of the widened units (64 KB there), so that a store covers 128 bytes of one row
            float* turn = reinterpret_cast<float*>(smem_raw + (wide - ptx::smem_u32(smem_raw))) + (warp - 2) * (32 * 33);
            for (int m = 0; !HEAD_M && m < p.tiles; ++m) {
                const int r0 = m * 128 + quarter * 32, rows = min(32, p.T - r0);
                float* out = p.part + (static_cast<long long>(blockIdx.y) * p.T + r0) * p.d + col0 + lane;
#pragma unroll 1
                for (int c = group * (N / 2); c < (group + 1) * (N / 2) && col0 + c < p.d && rows > 0; c += 32) {
                    uint32_t v[32];
                    ptx::tmem_ld_32x32(lanes + m * N + c, v);
                    ptx::tmem_ld_wait(v);
                    __syncwarp();
#pragma unroll
                    for (int q = 0; q < 32; ++q) turn[lane * 33 + q] = __uint_as_float(v[q]);
                    __syncwarp();
                    if (col0 + c + lane < p.d) {
#pragma unroll 8
                        for (int q = 0; q < rows; ++q) out[static_cast<long long>(q) * p.d + c] = turn[q * 33 + lane];
                    }
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
