// Weight gradient of a linear layer from an 8-bit checkpoint of its input: gaf_linear_weight_grad.
//
//     dW[n, m] = base[n, m] + sum over tokens t of dy[t, n] * x[t, m]        x: the values of the codes
//
// 2 T N M operations on the 5th-generation tensor cores.  The tokens are the contraction axis, so both operands are
// "MN-major": a row of either matrix is one step of the contraction.  The accumulator's lanes are columns m; the 128 of a CTA are
// one block of codes: a token has one scale per tile, and since the scale is a power of two, the values of the codes are exact in
// bfloat16.  The codes are widened on their way through shared memory (8 bits cross the L2, not 16).
//
// Two CTAs on neighbouring SMs work on one tile of 256 m by 256 n (cta_group::2): each widens the codes of its own 128 m and
// copies half of dy's columns, which the tensor cores of both read.  A tile of one CTA alone (128 x 256) would read 1.7 times as much
// through the L2 and through shared memory (2381 us against 1430 at the size below, both with one barrier ring).  Per step of 128 tokens,
// 1024 clocks of the tensor core, an SM's shared memory takes in 48 KB of copies, is read for 16 KB and written 32 KB by widening, and read for
// 64 KB by the MMAs: 160 of the 128 bytes a clock that it has, so that the tensor cores cannot be busy for more than four fifths of the time.
//
// Measured at T = 16384, N = M = 4096, dW in binary32: 463 us with random data (1.19 PFLOP/s, 0.71 of the measured cuBLAS burst, 0.85 of
// its rate under the power limit), 381 us in short runs; tensor pipe active 78 % of the
// cycles.  T = 300, N = M = 768: 10.2 us, two launches.  T = 4096, N = M = 4096: 118 us, with binary32 dy (three terms) 366 us.  T = 4096,
// N = 50,257, M = 768: 278 us in aligned rows, 1146 us in dense ones, which are laid out anew first.
//
// Accuracy.  A tensor core adds to its binary32 accumulator by cutting off, not by rounding; over many steps that pulls a sum
// towards zero.  A chain therefore ends after kWgChunk tokens, and the chains are added, rounded to nearest, in registers of the epilogue's
// warps while the next one runs in the other half of tensor memory.
//
// A CTA's warps (persistent; one CTA per SM):
//   warps 0-7    epilogue: chains out of tensor memory into registers, the tile's result to global memory
//   warps 8-15   widen codes: 16 at a time from the copied step into the swizzled layout that the tensor cores read
//   warp 16      tensor copies (TMA) of dy
//   warp 17      issues the MMAs (in the pair's first CTA; in the second it tells the first what is ready)
//   warp 18      tensor copies of the codes
//   warp 19      copies of their scale bytes (the aligned word that holds each)
// An arrival on a barrier costs tens of clocks, one after the other: wherever a step is handed on, one lane of a warp arrives.  And it
// waits for the loads that its thread has in flight: the widening warps have none (scale bytes that they fetched a step ahead themselves
// cost 0.7 us a step), the scales come by asynchronous copies.
// Three rings: codes, whose places are free again as soon as they are in registers, widened codes, and dy, both free when the MMAs have
// read them.  (One ring for codes and dy kept a step's codes until its MMAs were done: copy, widening and MMAs together
// take 4000 clocks, and five steps in flight left 800 a step.)  Every wait is bounded.
#pragma once

#include "gaf_gram_tc.cuh"
#include "gaf_layer_device.cuh"

namespace gaf {

constexpr int kWgM = 128, kWgN = 256, kWgK = 128;        // a CTA's part of a tile of dW, tokens per step
constexpr int kWgPairM = 2 * kWgM;                      // the pair's tile: 256 x 256
constexpr int kWgRing = 3, kWgCodeRing = 2;             // steps in the rings: dy and widened codes; codes
constexpr int kWgChunk = 512;                           // tokens per chain
constexpr int kWgChunkSteps = kWgChunk / kWgK;
constexpr int kWgDyBytes = kWgK * (kWgN / 2) * 2, kWgCodeBytes = kWgK * kWgM, kWgWideBytes = kWgK * kWgM * 2;
constexpr int kWgSmem = kWgRing * (kWgDyBytes + kWgWideBytes) + kWgCodeRing * kWgCodeBytes + 1024;
constexpr uint32_t kWgScalesAhead = 1;                  // steps whose scales are in flight (less than the ring holds)
constexpr int kWgThreads = 640;
constexpr int kWgNapEpilogue = 400, kWgNapWiden = 0, kWgNapCopy = 100, kWgNapMma = 0;
constexpr int kWgTmemCols = 512;
constexpr unsigned int kWgSpinLimit = 1u << 23;         // attempts of tens of clocks each: a third of a second or more

struct WeightGradArgs {
    const unsigned char *scales;
    const void *base;
    void *dweight;
    float *partials;            // [split][tile][n][m], of the tiles whose tokens are split
    Control *ctl;
    int64_t N, M, scale_bytes;
    int T, blocks;              // blocks: scale bytes of a row
    int steps, steps_per_term;  // steps of kWgK tokens; of each of the matrices that add up to dy
    int tiles_m, items;         // items of work: whole tiles, then the parts of the others
    int whole, rest;            // tiles that are done whole, and the others
    int steps_per_split;
    unsigned int spin_limit;
    int test_extra_arrival;     // test hook: the first barrier expects an arrival that never comes
};

struct WgShared {
    uint64_t code_full[kWgCodeRing], code_empty[kWgCodeRing];
    uint64_t dy_full[kWgRing], wide_full[kWgRing], done[kWgRing];  // done: the MMAs have read dy and the widened codes
    uint64_t other[kWgRing];                            // the second CTA's steps that are ready for the MMAs, in the first one
    uint32_t told[kWgRing];                             // where the second CTA's words go
    uint64_t acc_full[2], acc_empty[2];                 // chains (acc_empty: of both CTAs, in the first one)
    uint64_t drained;
    uint32_t scale[kWgCodeRing][kWgK];                  // the word that holds each token's scale byte
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
// bf16 x bf16 -> f32, both operands MN-major, M = 256 over the pair, N = 256.
constexpr uint32_t kWgInstrDesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(kWgN >> 3) << 17) |
                                  ((uint32_t)(kWgPairM >> 4) << 24);

__device__ __forceinline__ void wg_mma(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(kWgInstrDesc), "r"(accumulate)
        : "memory");
}
// All MMAs issued so far arrive, once complete, on the barrier at this place in both CTAs' shared memory.
__device__ __forceinline__ void wg_commit_both(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(tc_smem_u32(bar)),
                 "h"((unsigned short)3)
                 : "memory");
}
__device__ __forceinline__ void wg_commit_own(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(tc_smem_u32(bar)) : "memory");
}
// The address, in the pair's first CTA, of what is at this place here; and an arrival there.
__device__ __forceinline__ uint32_t wg_in_first(const void *p) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(tc_smem_u32(p)));
    return r;
}
// 4-byte asynchronous copy that reads the first `src_bytes` (0..4) bytes and fills up with zeros.
__device__ __forceinline__ void wg_copy4(uint32_t dst_smem, const void *src, uint32_t src_bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst_smem), "l"(src), "r"(src_bytes) : "memory");
}
// One lane of the warp, always the same.
__device__ __forceinline__ bool wg_elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// Bounded waits.  An attempt returns within tens of clocks whether or not the phase is complete, and a warp that polls takes issue
// slots from the widening warps: who can afford it sleeps between attempts (`nap` nanoseconds).  A warp polls, and arrives, without
// branching on the lane: after `if (lane == 0) ..` it went on in two parts, and executed everything twice (1223 -> 868 us at 16384 x 4096 x 4096).
// kCluster: for barriers that the other CTA's threads count on.
template <bool kCluster = false>
__device__ __forceinline__ uint32_t wg_try(uint64_t *bar, uint32_t parity) {
    uint32_t ok;
    if (kCluster)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(tc_smem_u32(bar)), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(tc_smem_u32(bar)), "r"(parity)
            : "memory");
    return ok;
}
template <int nap, typename Attempt>
__device__ __forceinline__ bool wg_wait_until(Attempt &&attempt, volatile int *abort_flag, unsigned int limit) {
    for (unsigned int spin = 0; spin < limit; ++spin) {
        if (attempt()) return true;
        if (nap > 0) __nanosleep(nap);
        if ((spin & 15u) == 15u && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}
template <int nap>
__device__ __forceinline__ bool wg_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag, unsigned int limit) {
    return wg_wait_until<nap>([&] { return wg_try(bar, parity) != 0u; }, abort_flag, limit);
}
// A warp's wait for all barriers that `attempt` tries.  Every lane polls every one of them: a vote orders no memory, so that a lane may read
// only what a barrier guards that it has polled itself.
template <int nap, typename Attempt>
__device__ __forceinline__ bool wg_wait_warp(Attempt &&attempt, volatile int *abort_flag, unsigned int limit) {
    return __all_sync(0xFFFFFFFFu, wg_wait_until<nap>(attempt, abort_flag, limit)) != 0;
}
// One lane's arrival for its whole warp.
__device__ __forceinline__ void wg_arrive_warp(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(tc_smem_u32(bar)) : "memory");
}
// An arrival at this place in the pair's first CTA that hands on what the fences of tcgen05 order: that this warp has read tensor memory.
__device__ __forceinline__ void wg_arrive_warp_in_first(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n\t}" ::"r"(wg_in_first(bar)) : "memory");
}
// One lane tells the first CTA what this CTA has in shared memory: a word stored there asynchronously, whose 4 bytes complete the barrier's phase with
// release semantics at cluster scope.  (An arrival with release semantics takes hundreds of clocks a step: 581 us where this took 488, at the size above, before the waits became what they are.)
__device__ __forceinline__ void wg_tell_first(uint32_t *word, uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xFFFFFFFF;\n\t"
        "@p st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];\n\t}" ::"r"(wg_in_first(word)), "r"(1u), "r"(wg_in_first(bar))
        : "memory");
}
// 32 lanes x 8 columns of accumulators.
__device__ __forceinline__ void wg_tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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
// Not zero if one of 16 codes is NaN, or the scale above 2^7 (then the factor of wg_widen16 is no number).
__device__ __forceinline__ unsigned int wg_unusual(const uint4 &c, unsigned int scale) {
    const unsigned int n = ((c.x & 0x7F7F7F7Fu) + 0x01010101u) | ((c.y & 0x7F7F7F7Fu) + 0x01010101u) | ((c.z & 0x7F7F7F7Fu) + 0x01010101u) |
                           ((c.w & 0x7F7F7F7Fu) + 0x01010101u);
    return (n & 0x80808080u) | (unsigned int)(scale > 134u);
}
// 16 codes and their scale byte as bfloat16 numbers: one multiplication by 2^(e + 120).
__device__ __forceinline__ void wg_widen16(const uint4 &c, unsigned int scale, unsigned int (&out)[8]) {
    const unsigned int in[4] = {c.x, c.y, c.z, c.w}, f = (scale + 120u) * 0x00800080u;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        wg_widen4(in[q], out[2 * q], out[2 * q + 1]);
        out[2 * q] = wg_mul2(out[2 * q], f);
        out[2 * q + 1] = wg_mul2(out[2 * q + 1], f);
    }
}
// The same for any codes and scale: by 2^127 first where 2^(e + 120) is no number, and codes of NaN become NaN.  (A value beyond
// bfloat16's range becomes infinite, which no code that was packed does.)
__device__ __forceinline__ void wg_widen16_any(const uint4 &c, unsigned int scale, unsigned int (&out)[8]) {
    const unsigned int in[4] = {c.x, c.y, c.z, c.w};
    const unsigned int f1 = min(scale + 120u, 254u) * 0x00800080u, f2 = scale > 134u ? (scale - 7u) * 0x00800080u : 0x3F803F80u;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        wg_widen4(in[q], out[2 * q], out[2 * q + 1]);
#pragma unroll
        for (int h = 2 * q; h < 2 * q + 2; ++h) {
            const unsigned int nan = __vcmpeq2(out[h] & 0x7FFF7FFFu, 0x07F007F0u);
            out[h] = wg_mul2(wg_mul2(out[h], f1), f2) | (nan & 0x7FFF7FFFu);
        }
    }
}

// A work item: one tile of dW and one range of steps.
struct WgItem { int m0, n0, part, step0, step1; };              // m0: of this CTA's half; part: place among the partial sums, or -1
__device__ __forceinline__ WgItem wg_item(const WeightGradArgs &a, int item, int rank) {
    WgItem w;
    int tile = item;
    w.part = item - a.whole;
    w.step0 = 0;
    w.step1 = a.steps;
    if (w.part >= 0) {
        const int split = w.part / a.rest;
        tile = a.whole + w.part - split * a.rest;
        w.step0 = split * a.steps_per_split;
        w.step1 = min(a.steps, w.step0 + a.steps_per_split);
    }
    const int tn = tile / a.tiles_m;
    w.n0 = tn * kWgN;
    w.m0 = (tile - tn * a.tiles_m) * kWgPairM + rank * kWgM;
    return w;
}

// `dy_map`: {N, rows of all terms} of bfloat16, box {64, kWgK}, 128-byte swizzle; `code_map`: {M, T} of bytes, box {kWgM, kWgK}, the
// same swizzle.  Both fill what lies outside with zeros.  G: type of dW (of the partial sums: float).
template <typename G>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWgThreads, 1)
weight_grad_kernel(const __grid_constant__ WeightGradArgs a, const __grid_constant__ CUtensorMap dy_map,
                   const __grid_constant__ CUtensorMap code_map) {
    extern __shared__ unsigned char wg_dyn[];
    __shared__ WgShared sh;
    unsigned char *const smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(wg_dyn) + 1023) & ~uintptr_t(1023));
    unsigned char *const dy_ring = smem, *const wide_ring = dy_ring + kWgRing * kWgDyBytes,
                         *const code_ring = wide_ring + kWgRing * kWgWideBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kWgCodeRing; ++s) {
            // codes, scales
            tc_mbar_init(&sh.code_full[s], 2 + (s == 0 && a.test_extra_arrival ? 1 : 0));
            tc_mbar_init(&sh.code_empty[s], 8);          // the widening warps
        }
        for (int s = 0; s < kWgRing; ++s) {
            tc_mbar_init(&sh.dy_full[s], 1);
            tc_mbar_init(&sh.wide_full[s], 8);
            tc_mbar_init(&sh.done[s], 1);
            tc_mbar_init(&sh.other[s], 1);               // (armed for the next word)
        }
        for (int b = 0; b < 2; ++b) {
            tc_mbar_init(&sh.acc_full[b], 1);
            tc_mbar_init(&sh.acc_empty[b], 16);
        }
        tc_mbar_init(&sh.drained, 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < kWgRing; ++s) tc_mbar_arrive_expect_tx(&sh.other[s], sizeof(uint32_t));
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc_smem_u32(&sh.tmem_base)), "r"(kWgTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    grid_wait();

    // 5 x 128 threads with 96 registers each: 2 x 160 + 2 x 48 + 64 = 480 (nothing spills: what a thread stores to local memory, its
    // fence for the tensor cores would wait for)
    if (warp < 8) {
        // ------------------------------------------------------------ epilogue ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        uint32_t chain = 0;
        bool alive = true;
        for (int item = pair; item < a.items && alive; item += pairs) {
            const WgItem w = wg_item(a, item, rank);
            float sum[128];
#pragma unroll
            for (int j = 0; j < 128; ++j) sum[j] = 0.f;
            for (int step = w.step0; step < w.step1; step += kWgChunkSteps, ++chain) {
                const uint32_t buf = chain & 1u;
                if (!wg_wait_warp<kWgNapEpilogue>([&] { return wg_try(&sh.acc_full[buf], (chain >> 1) & 1u) != 0u; }, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                tc_fence_after_sync();
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    uint32_t r[8];
                    wg_tmem_ld8(taddr + buf * kWgN + (uint32_t)(g * 8), r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[g * 8 + j] += __uint_as_float(r[j]);
                }
                tc_fence_before_sync();
                __syncwarp();
                wg_arrive_warp_in_first(&sh.acc_empty[buf]);
            }
            if (!alive) break;
            if (w.part >= 0) {
                float *const out = a.partials + ((int64_t)w.part * kWgN + half * 128) * kWgPairM + rank * kWgM + quarter * 32 + lane;
#pragma unroll
                for (int j = 0; j < 128; ++j) out[j * kWgPairM] = sum[j];
                continue;
            }
            const int64_t m = w.m0 + quarter * 32 + lane, n0 = w.n0 + half * 128;
            if (m < a.M) {
                const int n = (int)min((int64_t)128, a.N - n0);
                const G *const base = static_cast<const G *>(a.base);
                G *const out = static_cast<G *>(a.dweight) + n0 * a.M + m;
#pragma unroll
                for (int j = 0; j < 128; ++j)
                    if (j < n) out[j * a.M] = from_float<G>(base ? sum[j] + to_float<G>(base[(n0 + j) * a.M + m]) : sum[j]);
            }
        }
    } else if (warp < 16) {
        // ------------------------------------------------------------ widening ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        constexpr int kRows = 64, kUnits = kWgK / kRows;         // rows of the warps at a time
        // A unit is 16 codes of a row.  Four lanes take the four units of half a row (64 codes, one swizzle atom of the widened step), the four
        // lanes next to them those of the row whose number differs by 5: then neither the codes (swizzled by the copy) nor what is written
        // meets another lane's banks.  A warp takes 8 rows at a time.
        const int j = lane & 3, pair_of = lane >> 3, row = ((pair_of & 3) ^ ((lane & 4) ? 5 : 0)) + (warp - 8) * 8;
        const uint32_t code_at = (uint32_t)(row * kWgM + ((j ^ (row & 7)) << 4));                   // first half of the row; the second: ^ 64
        const uint32_t at0 = (uint32_t)(row * 128 + ((2 * j) ^ (row & 7)) * 16), at1 = (uint32_t)(row * 128 + ((2 * j + 1) ^ (row & 7)) * 16);
        int s = 0, o = 0;
        uint32_t full_phase = 0, wide_phase = 1;         // (the first round finds every widened step's place free)
        bool alive = true;
        for (int item = pair; item < a.items && alive; item += pairs) {
            const WgItem w = wg_item(a, item, rank);
            // (a multiple of 4 tokens further on, a scale byte lies at the same place of its word)
            const int shift = ((row * a.blocks + w.m0 / kCodeBlock) & 3) * 8;
            for (int step = w.step0; step < w.step1; ++step) {
                // (the codes, and the place they go to)
                if (!wg_wait_warp<kWgNapWiden>([&] { const uint32_t x = wg_try(&sh.code_full[s], full_phase), y = wg_try(&sh.done[o], wide_phase); return (x & y) != 0u; },
                                               &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                const unsigned char *const codes = code_ring + s * kWgCodeBytes;
                unsigned char *const wide = wide_ring + o * kWgWideBytes;
                uint4 c[2 * kUnits];
                unsigned int e[kUnits], unusual = 0u;
#pragma unroll
                for (int k = 0; k < kUnits; ++k) {
                    c[2 * k] = *reinterpret_cast<const uint4 *>(codes + code_at + k * kRows * kWgM);
                    c[2 * k + 1] = *reinterpret_cast<const uint4 *>(codes + (code_at ^ 64u) + k * kRows * kWgM);
                    e[k] = (sh.scale[s][row + k * kRows] >> shift) & 0xFFu;
                }
                __syncwarp();
                wg_arrive_warp(&sh.code_empty[s]);
#pragma unroll
                for (int k = 0; k < 2 * kUnits; ++k) unusual |= wg_unusual(c[k], e[k >> 1]);
                if (unusual == 0u) {
#pragma unroll
                    for (int k = 0; k < 2 * kUnits; ++k) {
                        unsigned int v[8];
                        wg_widen16(c[k], e[k >> 1], v);
                        unsigned char *const to = wide + (k & 1) * (kWgK * 128) + (k >> 1) * kRows * 128;
                        *reinterpret_cast<uint4 *>(to + at0) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4 *>(to + at1) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 2 * kUnits; ++k) {
                        unsigned int v[8];
                        wg_widen16_any(c[k], e[k >> 1], v);
                        unsigned char *const to = wide + (k & 1) * (kWgK * 128) + (k >> 1) * kRows * 128;
                        *reinterpret_cast<uint4 *>(to + at0) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4 *>(to + at1) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                }
                __syncwarp();
                wg_arrive_warp(&sh.wide_full[o]);
                if (++s == kWgCodeRing) { s = 0; full_phase ^= 1u; }
                if (++o == kWgRing) { o = 0; wide_phase ^= 1u; }
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 16) {
            // ------------------------------------------------- copies of dy ----
            if (lane == 0) {
                int s = 0;
                uint32_t phase = 1, issued = 0;          // (every place is free at first)
                bool alive = true;
                for (int item = pair; item < a.items && alive; item += pairs) {
                    const WgItem w = wg_item(a, item, rank);
                    const int n0 = w.n0 + rank * (kWgN / 2);
                    for (int step = w.step0; step < w.step1; ++step, ++issued) {
                        if (!wg_wait<kWgNapCopy>(&sh.done[s], phase, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        tc_mbar_arrive_expect_tx(&sh.dy_full[s], kWgDyBytes);
#pragma unroll
                        for (int k = 0; k < kWgN / 128; ++k)
                            tc_tma_load_2d(tc_smem_u32(dy_ring + s * kWgDyBytes + k * (kWgK * 128)), &dy_map, n0 + 64 * k, step * kWgK, &sh.dy_full[s]);
                        if (++s == kWgRing) { s = 0; phase ^= 1u; }
                    }
                }
                // what is in flight lands before the CTA ends, also after a wait gave up
                for (uint32_t i = issued > kWgRing ? issued - kWgRing : 0; i < issued; ++i)
                    for (unsigned int spin = 0; spin < min(a.spin_limit, kTcSpinLimit); ++spin)
                        if (tc_mbar_try(&sh.dy_full[i % kWgRing], (i / kWgRing) & 1u, 2000u)) break;
            }
            __syncwarp();
        } else if (warp == 17) {
            // -------------------------------------------------------- MMA -------
            // A wait costs some 250 clocks even when there is nothing to wait for, of which attempts issued one behind the other share most (three lanes that poll a
            // barrier each, and meet at a warp barrier: 11.2 us at 300 x 768 x 768 instead of 10.2).  The warp stays together (the MMAs' operands are in uniform
            // registers then) and one elected lane issues.
            int o = 0;
            uint32_t phase = 0, chain = 0;
            bool alive = true;
            if (rank == 0) {
                const uint64_t da = wg_desc(tc_smem_u32(wide_ring)), db = wg_desc(tc_smem_u32(dy_ring));
                for (int item = pair; item < a.items && alive; item += pairs) {
                    const WgItem w = wg_item(a, item, rank);
                    int in_chain = 0;
                    for (int step = w.step0; step < w.step1; ++step) {
                        const uint32_t buf = chain & 1u;
                        if (in_chain == 0 && !wg_wait_warp<kWgNapMma>([&] { return wg_try<true>(&sh.acc_empty[buf], ((chain >> 1) & 1u) ^ 1u) != 0u; }, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        if (!wg_wait_warp<kWgNapMma>([&] {
                                const uint32_t x = wg_try<true>(&sh.other[o], phase), y = wg_try(&sh.wide_full[o], phase), z = wg_try(&sh.dy_full[o], phase);
                                return (x & y & z) != 0u;
                            }, &sh.abort_flag, a.spin_limit)) {
                            alive = false;
                            break;
                        }
                        tc_fence_async_smem();                   // (see the second CTA's part below)
                        tc_fence_after_sync();
                        const bool last = in_chain == kWgChunkSteps - 1 || step + 1 == w.step1;
                        if (wg_elected()) {
                            tc_mbar_arrive_expect_tx(&sh.other[o], sizeof(uint32_t));
                            const uint64_t a0 = da + (uint64_t)(o * (kWgWideBytes / 16)), b0 = db + (uint64_t)(o * (kWgDyBytes / 16));
#pragma unroll
                            for (int k = 0; k < kWgK / 16; ++k)       // 16 tokens = 2048 bytes on
                                wg_mma(tmem + buf * kWgN, a0 + (uint64_t)(k * 128), b0 + (uint64_t)(k * 128), in_chain || k ? 1u : 0u);
                            wg_commit_both(&sh.done[o]);
                            if (last) wg_commit_both(&sh.acc_full[buf]);
                        }
                        __syncwarp();
                        ++in_chain;
                        if (last) {
                            ++chain;
                            in_chain = 0;
                        }
                        if (++o == kWgRing) { o = 0; phase ^= 1u; }
                    }
                }
                // tensor memory is not freed, and no shared memory left, under MMAs in flight
                if (wg_elected()) {
                    wg_commit_own(&sh.drained);
                    for (unsigned int spin = 0; spin < min(a.spin_limit, kTcSpinLimit); ++spin)
                        if (tc_mbar_try(&sh.drained, 0u, 2000u)) break;
                }
                __syncwarp();
            } else {
                // The second CTA's steps, told to the first.  The tensor cores read shared memory through the asynchronous proxy; the
                // fence between the two proxies stands here and before the MMAs, in threads that have nothing in flight: in each of the
                // widening threads it would wait for that thread's own stores.
                for (int item = pair; item < a.items && alive; item += pairs) {
                    const WgItem w = wg_item(a, item, rank);
                    for (int step = w.step0; step < w.step1; ++step) {
                        if (!wg_wait_warp<kWgNapMma>([&] { const uint32_t y = wg_try(&sh.wide_full[o], phase), z = wg_try(&sh.dy_full[o], phase); return (y & z) != 0u; },
                                                     &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        tc_fence_async_smem();
                        wg_tell_first(&sh.told[o], &sh.other[o]);
                        if (++o == kWgRing) { o = 0; phase ^= 1u; }
                    }
                }
            }
        } else if (warp == 18) {
            // ------------------------------------------------- copies of codes ----
            if (lane == 0) {
                int s = 0;
                uint32_t phase = 1, issued = 0;
                bool alive = true;
                for (int item = pair; item < a.items && alive; item += pairs) {
                    const WgItem w = wg_item(a, item, rank);
                    int t_step = w.step0 % a.steps_per_term;
                    for (int step = w.step0; step < w.step1; ++step, ++issued) {
                        if (!wg_wait<kWgNapCopy>(&sh.code_empty[s], phase, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
                        tc_mbar_arrive_expect_tx(&sh.code_full[s], kWgCodeBytes);
                        tc_tma_load_2d(tc_smem_u32(code_ring + s * kWgCodeBytes), &code_map, w.m0, t_step * kWgK, &sh.code_full[s]);
                        if (++t_step == a.steps_per_term) t_step = 0;
                        if (++s == kWgCodeRing) { s = 0; phase ^= 1u; }
                    }
                }
                for (uint32_t i = issued > kWgCodeRing ? issued - kWgCodeRing : 0; i < issued; ++i)
                    for (unsigned int spin = 0; spin < min(a.spin_limit, kTcSpinLimit); ++spin)
                        if (tc_mbar_try(&sh.code_full[i % kWgCodeRing], (i / kWgCodeRing) & 1u, 2000u)) break;
            }
            __syncwarp();
        } else {
            // ------------------------------------------------- copies of scales ----
            int s = 0, told = 0;                         // told: place of the oldest step whose scales have not been announced
            uint32_t phase = 1, issued = 0;
            bool alive = true;
            auto tell = [&] {
                __syncwarp();
                wg_arrive_warp(&sh.code_full[told]);
                if (++told == kWgCodeRing) told = 0;
            };
            for (int item = pair; item < a.items && alive; item += pairs) {
                const WgItem w = wg_item(a, item, rank);
                const int block = w.m0 / kCodeBlock;
                int t_step = w.step0 % a.steps_per_term;
                // this lane's first word of a step (of a block past the last one: the first word of all, of which nothing is read)
                const unsigned char *from = a.scales + (block < a.blocks ? ((int64_t)t_step * (kWgK * a.blocks) + lane * a.blocks + block) & ~int64_t(3) : 0);
                const int per_step = block < a.blocks ? kWgK * a.blocks : 0, per_row = per_step / kWgK;
                for (int step = w.step0; step < w.step1; ++step) {
                    const int rows = block < a.blocks ? a.T - t_step * kWgK : 0;         // of the tokens that remain
                    if (!wg_wait_warp<kWgNapCopy>([&] { return wg_try(&sh.code_empty[s], phase) != 0u; }, &sh.abort_flag, a.spin_limit)) { alive = false; break; }
#pragma unroll
                    for (int k = 0; k < kWgK / 32; ++k) {
                        const unsigned char *const word = from + 32 * k * per_row;
                        const bool in = lane + 32 * k < rows;
                        // (the last word of all may be a part)
                        wg_copy4(tc_smem_u32(&sh.scale[s][lane + 32 * k]), in ? word : a.scales,
                                 in ? (uint32_t)min((int64_t)4, a.scale_bytes - (word - a.scales)) : 0u);
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    if (++issued > kWgScalesAhead) {
                        asm volatile("cp.async.wait_group %0;" ::"n"(kWgScalesAhead) : "memory");
                        tell();
                    }
                    from += per_step;
                    if (++t_step == a.steps_per_term) { t_step = 0; from -= (int64_t)per_step * a.steps_per_term; }
                    if (++s == kWgCodeRing) { s = 0; phase ^= 1u; }
                }
            }
            tc_cp_async_wait_all();
            for (uint32_t k = 0; k < (issued < kWgScalesAhead ? issued : kWgScalesAhead); ++k) tell();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    // neither CTA leaves, or frees its tensor memory, while the other's MMAs or arrivals can still reach it
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    tc_fence_after_sync();
    if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kWgTmemCols) : "memory");
    if (sh.abort_flag && threadIdx.x == 0) a.ctl->layer_status = kLayerTimeout;
}

// dW = base + the parts' sums in order, of the tiles whose tokens were split.  Four elements of a row per thread.
constexpr int kWgJoinElements = 1024;           // per CTA
struct WgJoinArgs {
    const float *partials;
    const void *base;
    void *dweight;
    int64_t N, M;
    int splits, tiles_m, whole, rest;
};
template <typename G>
__global__ void __launch_bounds__(kWgJoinElements / 4) weight_grad_join_kernel(const WgJoinArgs a) {
    constexpr int kCtas = kWgPairM * kWgN / kWgJoinElements;
    const int r = blockIdx.x / kCtas, e0 = (blockIdx.x % kCtas) * kWgJoinElements + threadIdx.x * 4;
    const int tile = a.whole + r, tn = tile / a.tiles_m;
    const int64_t n = (int64_t)tn * kWgN + e0 / kWgPairM, m = (int64_t)(tile - tn * a.tiles_m) * kWgPairM + e0 % kWgPairM;
    grid_wait();
    if (n >= a.N || m >= a.M) return;
    const float *p = a.partials + (int64_t)r * (kWgPairM * kWgN) + e0;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s, p += (int64_t)a.rest * (kWgPairM * kWgN)) {
        const float4 f = __ldcg(reinterpret_cast<const float4 *>(p));
        v[0] += f.x; v[1] += f.y; v[2] += f.z; v[3] += f.w;
    }
    const G *const base = static_cast<const G *>(a.base);
    G *const out = static_cast<G *>(a.dweight) + n * a.M + m;
    const int left = (int)min((int64_t)4, a.M - m);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) out[i] = from_float<G>(base ? v[i] + to_float<G>(base[n * a.M + m + i]) : v[i]);
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
