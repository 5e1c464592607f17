// Root-mean-square norm with the residual's addition, and its backward pass: gaf_rms_norm and gaf_rms_norm_grad.
//
//     h = x + residual (rounded to the matrices' type)      r = 1 / sqrt(mean h^2 + eps)      y = h r w
//     dx = residual_grad + r (w dy - h r^2 mean(w dy h))     dw = sum over rows of dy h r
//
// Both are bound by memory (16384 x 4096 bfloat16: forward with residual and coded result 96 to 100 us, 6.0 to 6.3 TB/s, with h's checkpoint too 113 us; backward from an 8-bit checkpoint with a
// residual's gradient 90 us, 5.2 TB/s, issue slots half taken).  A row is held in registers between its reduction and its results, so that everything is read and
// written once: R threads of a CTA share a row, up to S tiles of 256 columns per warp.
#pragma once

#include "gaf_layer_device.cuh"

namespace gaf {

constexpr int kNormMaxWidth = 16384;
constexpr int kNormThreads = 128;               // threads of a CTA whose rows take fewer

__host__ __device__ constexpr int norm_threads(int R) { return R > kNormThreads ? R : kNormThreads; }

// Sum over the R threads of a row, the same in all of them.  `scratch`: two sets of 32 floats, used in turn, so that one barrier per
// sum is enough.
template <int R>
__device__ __forceinline__ float row_sum(float v, float *scratch, int turn) {
    v = warp_sum(v);
    if (R == 32) return v;
    float *const s = scratch + 32 * (turn & 1);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    const int first = (threadIdx.x / R) * (R / 32);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < R / 32; ++w) sum += s[first + w];
    return sum;
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    unsigned char *y_codes, *y_scales, *h_codes, *h_scales;
    float *rstd;
    int64_t x_stride, residual_stride, y_codes_stride, h_codes_stride;
    int64_t T, d, blocks;
    float eps;
    int coded_y;                // y holds the values of its codes
};

template <typename T, bool VEC, int R, int S>
__global__ void __launch_bounds__(norm_threads(R)) rms_norm_kernel(const NormArgs a) {
    __shared__ float scratch[64];
    const int lane = threadIdx.x & 31, w_row = (threadIdx.x % R) >> 5;
    const int64_t row = (int64_t)blockIdx.x * (norm_threads(R) / R) + threadIdx.x / R;
    // (rows past the end take part in the barriers and touch nothing)
    const int64_t d = row < a.T ? a.d : 0;
    grid_wait();
    float v[S][8], ss = 0.f;
    {
        Share<T> sx[S], sr[S];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
            load_tile<VEC>(static_cast<const T *>(a.x) + row * a.x_stride + c, lane, d - c, sx[s]);
            if (a.residual) load_tile<VEC>(static_cast<const T *>(a.residual) + row * a.residual_stride + c, lane, d - c, sr[s]);
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
            sx[s].get(v[s]);
            if (a.residual) {
                float r[8];
                sr[s].get(r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[s][i] = rounded<T>(v[s][i] + r[i]);
                if (a.h) store_tile<VEC>(static_cast<T *>(a.h) + row * a.d + c, lane, d - c, v[s]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(v[s][i], v[s][i], ss);
        }
    }
    const float r = 1.0f / sqrtf(row_sum<R>(ss, scratch, 0) / (float)a.d + a.eps);
    if (a.rstd && threadIdx.x % R == 0 && row < a.T) a.rstd[row] = r;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
        unsigned int code[2];
        int e[2];
        if (a.h_codes) {
            encode_tile<VEC>(v[s], code, e);
            store_codes<VEC>(a.h_codes + row * a.h_codes_stride + c, a.h_scales + row * a.blocks + c / kCodeBlock, lane, d - c, code, e);
        }
        if (a.y || a.y_codes) {
            float w[8], y[8];
            load_tile<VEC>(static_cast<const T *>(a.weight) + c, lane, d - c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[s][i] * r * w[i];
            if (a.y_codes) {
                encode_tile<VEC>(y, code, e);
                store_codes<VEC>(a.y_codes + row * a.y_codes_stride + c, a.y_scales + row * a.blocks + c / kCodeBlock, lane, d - c, code, e);
                if (a.coded_y) decode8(code, power_of_two(e[0]), power_of_two(e[1]), y);
            }
            if (a.y) store_tile<VEC>(static_cast<T *>(a.y) + row * a.d + c, lane, d - c, y);
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *weight, *residual_grad;
    const unsigned char *h_codes, *h_scales;
    const float *rstd;
    void *dx;
    float *partials;            // [CTA][d]: sums over the CTA's rows
    int64_t dy_stride, h_stride, codes_stride, residual_grad_stride;
    int64_t T, d, blocks;
};

// Rows are dealt round-robin to the CTAs; each keeps its columns' sums for the weight's gradient in registers and leaves them in
// `partials`, which norm_grad_finish_kernel adds up in CTA order.
// (__grid_constant__: arguments of 128 bytes or less are otherwise copied to registers at the start, of which there are none to spare: 104 us instead of 90 for
// 16384 x 4096 bfloat16 from codes.)
template <typename T, bool VEC, bool CODED, int R, int S>
__global__ void __launch_bounds__(norm_threads(R)) rms_norm_grad_kernel(const __grid_constant__ NormGradArgs a) {
    constexpr int kRows = norm_threads(R) / R;          // rows that a CTA has in hand
    __shared__ float scratch[64];
    __shared__ float columns[kRows > 1 ? S * (R / 32) * kTile : 1];
    const int lane = threadIdx.x & 31, w_row = (threadIdx.x % R) >> 5, sub = threadIdx.x / R;
    float dw[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[s][i] = 0.f;
    Share<T> s_w[S], s_dy[S], s_h[CODED ? 1 : S], s_res[S];
    CodeShare s_code[CODED ? S : 1];
    float r = 0.f;
    auto load = [&](int64_t row) {
        const int64_t d = row < a.T ? a.d : 0;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
            load_tile<VEC>(static_cast<const T *>(a.dy) + row * a.dy_stride + c, lane, d - c, s_dy[s]);
            if constexpr (CODED)
                load_codes<VEC>(a.h_codes + row * a.codes_stride + c, a.h_scales + row * a.blocks + c / kCodeBlock, lane, d - c, s_code[s]);
            else
                load_tile<VEC>(static_cast<const T *>(a.h) + row * a.h_stride + c, lane, d - c, s_h[s]);
        }
        r = row < a.T ? a.rstd[row] : 0.f;
    };
    grid_wait();
    // (Nothing: a border that the compiler moves no loads across.  Without it 16384 x 4096 from codes takes 92 us in bfloat16 instead of 90, 8192 x 4096 in
    // binary32 95 instead of 88.)
    if (blockIdx.x == 0 && threadIdx.x == 0) asm volatile("" ::: "memory");
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + sub;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
        load_tile<VEC>(static_cast<const T *>(a.weight) + c, lane, a.d - c, s_w[s]);
    }
    // the next row in flight while this one is summed and written: not in binary32, whose rows take all registers (16384 x 4096, without a
    // residual's gradient: 142 us; with the next row in flight it was 185 against 165 us, in bfloat16 76 against 85 us)
    constexpr bool kAhead = sizeof(T) == 2;
    if (kAhead) load(row);
    int turn = 0;
    // (all rows of a CTA take part in the barriers until the first is past the end)
#pragma unroll 1
    for (; row - sub < a.T; row += step, ++turn) {
        const int64_t d = row < a.T ? a.d : 0;
        if (!kAhead) load(row);
        const float r_row = r;
        float wdy[S][8], n[S][8], q = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
            float dy[8], w[8];
            s_dy[s].get(dy);
            if constexpr (CODED) s_code[s].get(n[s]); else s_h[s].get(n[s]);
            s_w[s].get(w);
            if (a.residual_grad)
                load_tile<VEC>(static_cast<const T *>(a.residual_grad) + row * a.residual_grad_stride + c, lane, d - c, s_res[s]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[s][i] *= r_row;
                dw[s][i] = fmaf(dy[i], n[s][i], dw[s][i]);
                wdy[s][i] = dy[i] * w[i];
                q = fmaf(wdy[s][i], n[s][i], q);
            }
        }
        if (kAhead) load(row + step);
        const float mean = row_sum<R>(q, scratch, turn) / (float)a.d;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = r_row * (wdy[s][i] - n[s][i] * mean);
            if (a.residual_grad) {
                float g[8];
                s_res[s].get(g);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] += g[i];
            }
            store_tile<VEC>(static_cast<T *>(a.dx) + row * a.d + c, lane, d - c, o);
        }
    }
    grid_release();
    // the CTA's rows side by side are added in order
    float *const out = a.partials + (int64_t)blockIdx.x * a.d;
    if (kRows > 1) {
        for (int k = 0; k < kRows; ++k) {
            if (sub == k) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    float *const p = columns + (s * (R / 32) + w_row) * kTile;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float *const at = p + tile_column<VEC>(lane, i);
                        dw[s][i] = k == 0 ? dw[s][i] : dw[s][i] + *at;
                        *at = dw[s][i];
                    }
                }
            }
            __syncthreads();
        }
        if (sub != kRows - 1) return;
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t c = (int64_t)(s * (R / 32) + w_row) * kTile;
        store_tile<VEC>(out + c, lane, a.d - c, dw[s]);
    }
}

// dw = base + the sum of `n` rows of partials, in binary64, row groups in order.
constexpr int kNormFinishGroups = 16;
struct NormFinishArgs {
    const float *partials;
    const void *base;
    void *dweight;
    int n;
    int64_t d;
};
template <typename G>
__global__ void __launch_bounds__(32 * kNormFinishGroups) norm_grad_finish_kernel(const NormFinishArgs a) {
    __shared__ double part[kNormFinishGroups][32];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    grid_wait();
    double sum = 0.0;
    if (c < a.d) {
        const int per = (a.n + kNormFinishGroups - 1) / kNormFinishGroups;
        const int end = min(a.n, (group + 1) * per);
#pragma unroll 8
        for (int k = group * per; k < end; ++k) sum += (double)__ldcg(a.partials + (int64_t)k * a.d + c);
    }
    part[group][lane] = sum;
    __syncthreads();
    if (group == 0 && c < a.d) {
        for (int g = 1; g < kNormFinishGroups; ++g) sum += part[g][lane];
        if (a.base) sum += (double)to_float<G>(static_cast<const G *>(a.base)[c]);
        static_cast<G *>(a.dweight)[c] = from_float<G>((float)sum);
    }
}

}  // namespace gaf
