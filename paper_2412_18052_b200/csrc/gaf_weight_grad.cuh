// Weight gradient of a linear layer from an 8-bit checkpoint of its input: gaf_linear_weight_grad.
//
//     dW[n, m] = base[n, m] + sum over tokens t of dy[t, n] * x[t, m]        x: the values of the codes
//
// 2 T N M operations on the 5th-generation tensor cores.  The tokens are the contraction axis, so both operands are
// "MN-major": a row of either matrix is one step of the contraction.  The accumulator's 128 lanes are 128 columns m, the width of one
// block of codes: a token has one scale per tile, and since the scale is a power of two, the values of the codes are exact in
// bfloat16.  The codes are widened on their way through shared memory (8 bits cross the L2, not 16).
//
// Accuracy.  A tensor core adds to its binary32 accumulator by cutting off, not by rounding; over many steps that pulls a sum
// towards zero.  A chain therefore ends after kWgChunk tokens, and the chains are added, rounded to nearest, in registers of the epilogue's
// warps while the next one runs in the other half of tensor memory.
//
// A CTA's warps (persistent; one CTA per SM):
//   warps 0-7    epilogue: chains out of tensor memory into registers, the tile's result to global memory
//   warps 8-11   widen codes: 16 at a time from the copied tile into the swizzled layout that the tensor core reads
//   warp 12      tensor copies (TMA) of both matrices into a ring, bounded waits
//   warp 13      issues the MMAs
#pragma once

#include "gaf_gram_tc.cuh"
#include "gaf_layer_device.cuh"

namespace gaf {

constexpr int kWgM = 128, kWgN = 256, kWgK = 64;        // tile of dW, tokens per step
constexpr int kWgStages = 4, kWgWide = 3;               // rings: copied steps, widened steps
constexpr int kWgChunk = 256;                           // tokens per chain
constexpr int kWgChunkSteps = kWgChunk / kWgK;
constexpr int kWgDyBytes = kWgK * kWgN * 2, kWgCodeBytes = kWgK * kWgM, kWgWideBytes = kWgK * kWgM * 2;
constexpr int kWgSmem = kWgStages * (kWgDyBytes + kWgCodeBytes) + kWgWide * kWgWideBytes + 1024;
constexpr int kWgThreads = 512;
constexpr int kWgTmemCols = 512;

struct WeightGradArgs {
    const unsigned char *scales;
    const void *base;
    void *dweight;
    float *partials;            // [split][N][M], when the tokens are split
    Control *ctl;
    int64_t T, N, M, blocks;    // blocks: scale bytes of a row
    int terms;                  // 1; or 3: binary32 dy as the sum of three bfloat16 matrices, below one another
    int64_t steps_per_term;     // ceil(T / kWgK)
    int64_t tiles_m, tiles_n, splits, steps_per_split;      // (a multiple of kWgChunkSteps)
    unsigned int spin_limit;
    int test_extra_arrival;     // test hook: the first barrier expects an arrival that never comes
};

struct WgShared {
    uint64_t full[kWgStages], empty[kWgStages];         // copied steps
    uint64_t wide_full[kWgWide], wide_empty[kWgWide];   // widened steps
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drained;
    uint32_t tmem_base;
    volatile int abort_flag;
};

// Operand with the contraction axis outermost: swizzle atoms of 64 elements (128 bytes) by 8 tokens; the next 8 tokens are 1024 bytes
// on, the next 64 elements one column of atoms, kWgK * 128 bytes.
__device__ __forceinline__ uint64_t wg_desc(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)((kWgK * 128) >> 4) << 16;           // between atoms along the 64-element axis
    d |= (uint64_t)(1024 >> 4) << 32;                   // between groups of 8 tokens
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;                             // 128-byte swizzle
    return d;
}
// bf16 x bf16 -> f32, both operands MN-major, M = 128, N = 256.
constexpr uint32_t kWgInstrDesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(kWgN >> 3) << 17) |
                                  ((uint32_t)(kWgM >> 4) << 24);

__device__ __forceinline__ void wg_mma(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(kWgInstrDesc), "r"(accumulate)
        : "memory");
}

// Four codes (bytes of w) as bfloat16 numbers 2^120 times too small: e4m3 and bfloat16 have their fields in the same order, so a
// sign-extended code, four bits up, without the copies of its sign, is the number with its exponent counted from another origin; subnormal codes
// become subnormal numbers.  (Codes of NaN need another way.)
__device__ __forceinline__ void wg_widen4(unsigned int w, unsigned int &lo, unsigned int &hi) {
    asm("prmt.b32 %0, %1, %1, 0x9180;" : "=r"(lo) : "r"(w));        // (selector bit 3: the byte's sign, eight times)
    asm("prmt.b32 %0, %1, %1, 0xB3A2;" : "=r"(hi) : "r"(w));
    lo = (lo << 4) & 0x87F087F0u;
    hi = (hi << 4) & 0x87F087F0u;
}
__device__ __forceinline__ unsigned int wg_mul2(unsigned int a, unsigned int b) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const unsigned int *>(&r);
}
__device__ __forceinline__ unsigned int wg_power2(int e) {      // 2^e twice, e in -126..127
    const unsigned int p = (unsigned int)(e + 127) << 7;
    return p | (p << 16);
}

// A work item: one tile of dW and one range of steps.
struct WgItem { int64_t m0, n0, split, step0, step1; };
__device__ __forceinline__ WgItem wg_item(const WeightGradArgs &a, int64_t item) {
    WgItem w;
    const int64_t tiles = a.tiles_m * a.tiles_n, steps = a.terms * a.steps_per_term;
    w.split = item / tiles;
    const int64_t tile = item - w.split * tiles;
    w.n0 = (tile / a.tiles_m) * kWgN;
    w.m0 = (tile % a.tiles_m) * kWgM;
    w.step0 = w.split * a.steps_per_split;
    w.step1 = min(steps, w.step0 + a.steps_per_split);
    return w;
}

// `dy_map`: {N, terms x rows of a term} of bfloat16, box {64, kWgK}, 128-byte swizzle; `code_map`: {M, T} of bytes, box {kWgM, kWgK}.  Both
// fill what lies outside with zeros.  G: type of dW (of the partial sums: float).
template <typename G>
__global__ void __launch_bounds__(kWgThreads, 1)
weight_grad_kernel(const __grid_constant__ WeightGradArgs a, const __grid_constant__ CUtensorMap dy_map,
                   const __grid_constant__ CUtensorMap code_map) {
    extern __shared__ unsigned char wg_dyn[];
    __shared__ WgShared sh;
    unsigned char *const smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(wg_dyn) + 1023) & ~uintptr_t(1023));
    unsigned char *const dy_ring = smem, *const wide_ring = dy_ring + kWgStages * kWgDyBytes,
                         *const code_ring = wide_ring + kWgWide * kWgWideBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t n_items = a.tiles_m * a.tiles_n * a.splits;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kWgStages; ++s) {
            tc_mbar_init(&sh.full[s], 1 + (s == 0 && a.test_extra_arrival ? 1 : 0));
            tc_mbar_init(&sh.empty[s], 1);
        }
        for (int s = 0; s < kWgWide; ++s) {
            tc_mbar_init(&sh.wide_full[s], 128);
            tc_mbar_init(&sh.wide_empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            tc_mbar_init(&sh.acc_full[b], 1);
            tc_mbar_init(&sh.acc_empty[b], 256);
        }
        tc_mbar_init(&sh.drained, 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc_smem_u32(&sh.tmem_base)), "r"(kWgTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    grid_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) a.ctl->status = 0;

    // 4 x 128 threads with 128 registers each: 2 x 184 + 80 + 64 = 512
    if (warp < 8) {
        // ------------------------------------------------------------ epilogue ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        int64_t chain = 0;
        bool alive = true;
        for (int64_t item = blockIdx.x; item < n_items && alive; item += gridDim.x) {
            const WgItem w = wg_item(a, item);
            float sum[128];
#pragma unroll
            for (int j = 0; j < 128; ++j) sum[j] = 0.f;
            for (int64_t step = w.step0; step < w.step1; step += kWgChunkSteps, ++chain) {
                const int buf = (int)(chain & 1);
                if (!tc_mbar_wait_warp(&sh.acc_full[buf], (uint32_t)((chain >> 1) & 1), &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                tc_fence_after_sync();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t r[32];
                    tc_tmem_ld32(taddr + (uint32_t)(buf * kWgN + g * 32), r);
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[g * 32 + j] += __uint_as_float(r[j]);
                }
                tc_fence_before_sync();
                tc_mbar_arrive(&sh.acc_empty[buf]);
            }
            if (!alive) break;
            const int64_t m = w.m0 + quarter * 32 + lane, n0 = w.n0 + half * 128;
            if (m < a.M) {
                if (a.splits > 1) {
                    float *const out = a.partials + (w.split * a.N + n0) * a.M + m;
#pragma unroll
                    for (int j = 0; j < 128; ++j)
                        if (n0 + j < a.N) out[j * a.M] = sum[j];
                } else {
                    const G *const base = static_cast<const G *>(a.base);
                    G *const out = static_cast<G *>(a.dweight) + n0 * a.M + m;
#pragma unroll
                    for (int j = 0; j < 128; ++j)
                        if (n0 + j < a.N) out[j * a.M] = from_float<G>(base ? sum[j] + to_float<G>(base[(n0 + j) * a.M + m]) : sum[j]);
                }
            }
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------ widening ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        const int tid = threadIdx.x - 256;
        const int j = tid & 7, row0 = tid >> 3;          // 16 codes j of the rows row0, row0 + 16, ..
        // (half of the lanes write their two pieces in the other order: no two of eight lanes in the same banks)
        const int swap = j >> 2;
        uint32_t step_i = 0;                             // steps so far
        bool alive = true;
        for (int64_t item = blockIdx.x; item < n_items && alive; item += gridDim.x) {
            const WgItem w = wg_item(a, item);
            const unsigned char *const scale0 = a.scales + w.m0 / kCodeBlock;
            // scale bytes of a step are fetched one step ahead
            unsigned int next[4];
            auto fetch = [&](int64_t step) {
                const int64_t t0 = (step % a.steps_per_term) * kWgK + row0;
#pragma unroll
                for (int k = 0; k < 4; ++k) next[k] = step < w.step1 && t0 + 16 * k < a.T ? scale0[(t0 + 16 * k) * a.blocks] : 127u;
            };
            fetch(w.step0);
            for (int64_t step = w.step0; step < w.step1; ++step, ++step_i) {
                const int s = step_i % kWgStages, o = step_i % kWgWide;
                unsigned int scale[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) scale[k] = next[k];
                fetch(step + 1);
                if (!tc_mbar_wait_warp(&sh.full[s], (step_i / kWgStages) & 1u, &sh.abort_flag, a.spin_limit) ||
                    (step_i >= kWgWide &&
                     !tc_mbar_wait_warp(&sh.wide_empty[o], (step_i / kWgWide - 1) & 1u, &sh.abort_flag, a.spin_limit))) { alive = false; break; }
                const unsigned char *const codes = code_ring + s * kWgCodeBytes;
                unsigned char *const wide = wide_ring + o * kWgWideBytes + (j >> 2) * (kWgK * 128);
                uint4 c[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = *reinterpret_cast<const uint4 *>(codes + (row0 + 16 * k) * kWgM + j * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned int in[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
                    unsigned int out[8];
                    unsigned int nan = 0u;
#pragma unroll
                    for (int q = 0; q < 4; ++q) nan |= (in[q] & 0x7F7F7F7Fu) + 0x01010101u;
                    if (nan & 0x80808080u) {             // rare: some code is NaN
                        const float f = scale_of_byte(scale[k]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float2 x = value_pair((unsigned short)in[q]), y = value_pair((unsigned short)(in[q] >> 16));
                            out[2 * q] = pack_bf16x2(x.x * f, x.y * f);
                            out[2 * q + 1] = pack_bf16x2(y.x * f, y.y * f);
                        }
                    } else {
                        // 2^(e + 120) in one multiplication where that is a number, else 2^120 first
                        const int e = (int)scale[k] - 127;
                        const unsigned int f = e <= 7 ? wg_power2(max(e + 120, -126)) : wg_power2(120);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            wg_widen4(in[q], out[2 * q], out[2 * q + 1]);
                            out[2 * q] = wg_mul2(out[2 * q], f);
                            out[2 * q + 1] = wg_mul2(out[2 * q + 1], f);
                        }
                        if (e > 7) {
                            const unsigned int f2 = (scale[k] << 7) | (scale[k] << 23);
#pragma unroll
                            for (int q = 0; q < 8; ++q) out[q] = wg_mul2(out[q], f2);
                        }
                    }
                    const int row = row0 + 16 * k;
                    unsigned char *const line = wide + row * 128;
                    const int chunk = (2 * j) & 7;
                    const uint4 p0 = make_uint4(out[0], out[1], out[2], out[3]), p1 = make_uint4(out[4], out[5], out[6], out[7]);
                    *reinterpret_cast<uint4 *>(line + (((chunk + swap) ^ (row & 7)) << 4)) = swap ? p1 : p0;
                    *reinterpret_cast<uint4 *>(line + (((chunk + 1 - swap) ^ (row & 7)) << 4)) = swap ? p0 : p1;
                }
                tc_fence_async_smem();                   // the tensor core reads through the asynchronous proxy
                tc_mbar_arrive(&sh.wide_full[o]);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 12) {
            // -------------------------------------------------------- copies ----
            if (lane == 0) {
                uint32_t step_i = 0;
                bool alive = true;
                for (int64_t item = blockIdx.x; item < n_items && alive; item += gridDim.x) {
                    const WgItem w = wg_item(a, item);
                    for (int64_t step = w.step0; step < w.step1; ++step, ++step_i) {
                        const int s = step_i % kWgStages;
                        if (step_i >= kWgStages &&
                            !tc_mbar_wait(&sh.empty[s], (step_i / kWgStages - 1) & 1u, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        const int32_t t0 = (int32_t)((step % a.steps_per_term) * kWgK), y0 = (int32_t)(step * kWgK);
                        tc_mbar_arrive_expect_tx(&sh.full[s], kWgDyBytes + kWgCodeBytes);
                        tc_tma_load_2d(tc_smem_u32(code_ring + s * kWgCodeBytes), &code_map, (int32_t)w.m0, t0, &sh.full[s]);
#pragma unroll
                        for (int k = 0; k < kWgN / 64; ++k)
                            tc_tma_load_2d(tc_smem_u32(dy_ring + s * kWgDyBytes + k * (kWgK * 128)), &dy_map, (int32_t)(w.n0 + 64 * k), y0, &sh.full[s]);
                    }
                }
                // what is in flight lands before the CTA ends, also after a wait gave up
                for (uint32_t i = step_i > kWgStages ? step_i - kWgStages : 0; i < step_i; ++i)
                    for (unsigned int spin = 0; spin < a.spin_limit; ++spin)
                        if (tc_mbar_try(&sh.full[i % kWgStages], (i / kWgStages) & 1u, 2000u)) break;
            }
            __syncwarp();
        } else if (warp == 13) {
            // -------------------------------------------------------- MMA -------
            if (lane == 0) {
                uint32_t step_i = 0;
                int64_t chain = 0;
                bool alive = true;
                for (int64_t item = blockIdx.x; item < n_items && alive; item += gridDim.x) {
                    const WgItem w = wg_item(a, item);
                    for (int64_t step = w.step0; step < w.step1; ++step, ++step_i) {
                        const int s = step_i % kWgStages, o = step_i % kWgWide;
                        const int in_chain = (int)((step - w.step0) % kWgChunkSteps), buf = (int)(chain & 1);
                        if (in_chain == 0 && chain >= 2 &&
                            !tc_mbar_wait(&sh.acc_empty[buf], (uint32_t)((chain / 2 - 1) & 1), &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        if (!tc_mbar_wait(&sh.full[s], (step_i / kWgStages) & 1u, &sh.abort_flag, a.spin_limit) ||
                            !tc_mbar_wait(&sh.wide_full[o], (step_i / kWgWide) & 1u, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        tc_fence_after_sync();
                        const uint64_t da = wg_desc(tc_smem_u32(wide_ring + o * kWgWideBytes)), db = wg_desc(tc_smem_u32(dy_ring + s * kWgDyBytes));
#pragma unroll
                        for (int k = 0; k < kWgK / 16; ++k)       // 16 tokens = 2048 bytes on
                            wg_mma(tmem + (uint32_t)(buf * kWgN), da + (uint64_t)(k * 128), db + (uint64_t)(k * 128), in_chain || k ? 1u : 0u);
                        tc_commit(&sh.empty[s]);
                        tc_commit(&sh.wide_empty[o]);
                        if (in_chain == kWgChunkSteps - 1 || step + 1 == w.step1) {
                            tc_commit(&sh.acc_full[buf]);
                            ++chain;
                        }
                    }
                }
                // tensor memory is not freed under MMAs in flight
                tc_commit(&sh.drained);
                for (unsigned int spin = 0; spin < a.spin_limit; ++spin)
                    if (tc_mbar_try(&sh.drained, 0u, 2000u)) break;
            }
            __syncwarp();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 13) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kWgTmemCols) : "memory");
    if (sh.abort_flag && threadIdx.x == 0) atomicOr(&a.ctl->status, kStatusTimeoutBit);
}

// dW = base + the splits' sums in order.  Four elements per thread.
struct WgJoinArgs {
    const float *partials;
    const void *base;
    void *dweight;
    int64_t elements, splits;
};
template <typename G>
__global__ void __launch_bounds__(256) weight_grad_join_kernel(const WgJoinArgs a) {
    const int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    grid_wait();
    const G *const base = static_cast<const G *>(a.base);
    G *const out = static_cast<G *>(a.dweight);
    const int n = (int)min((int64_t)4, a.elements - e0);
    if (n <= 0) return;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if ((a.elements & 3) == 0) {                        // the splits' matrices start on 16-byte boundaries
        for (int64_t s = 0; s < a.splits; ++s) {
            const float4 p = __ldcg(reinterpret_cast<const float4 *>(a.partials + s * a.elements + e0));
            v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        }
    } else {
        for (int64_t s = 0; s < a.splits; ++s)
            for (int i = 0; i < n; ++i) v[i] += __ldcg(a.partials + s * a.elements + e0 + i);
    }
    for (int i = 0; i < n; ++i) out[e0 + i] = from_float<G>(base ? v[i] + to_float<G>(base[e0 + i]) : v[i]);
}

// dy laid out anew where tensor copies cannot read it as it is, as matrices below one another whose rows start on 16-byte boundaries.
// Binary32 as three bfloat16 matrices that add up to it: dy = hi + mid + lo, each the rest rounded to nearest (8 bits a time; exact
// while no term is below bfloat16's subnormals); bfloat16 rows at other distances as one.  Term k is rows k * rows .. + T of `out`; the
// rows from T on are zero.
struct WgTermsArgs {
    const void *dy;
    __nv_bfloat16 *out;
    int64_t stride, T, N, rows, pitch;
};
template <typename T>
__global__ void __launch_bounds__(256) weight_grad_terms_kernel(const WgTermsArgs a) {
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    grid_wait();
    if (c >= a.pitch) return;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float x = row < a.T && c < a.N ? to_float<T>(static_cast<const T *>(a.dy)[row * a.stride + c]) : 0.f;
        const bool finite = (__float_as_uint(x) & 0x7FFFFFFFu) < kInfBits;
#pragma unroll
        for (int k = 0; k < kTerms; ++k) {
            // (near the largest binary32 number the nearest bfloat16 is infinite: the largest finite one leaves a rest that still fits)
            float h = rounded<__nv_bfloat16>(x);
            if (finite && (__float_as_uint(h) & 0x7FFFFFFFu) >= kInfBits) h = copysignf(__uint_as_float(0x7F7F0000u), x);
            a.out[(k * a.rows + row) * a.pitch + c] = __float2bfloat16_rn(h);
            x = finite ? x - h : 0.f;
        }
    }
}

}  // namespace gaf
