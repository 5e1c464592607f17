// Building blocks of the layers' kernels: how a warp holds a stretch of a row, and the 8-bit code of a block of 128 elements.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gaf_device.cuh"

namespace gaf {

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ------------------------------------------------------------------ tiles ---
// A warp works on tiles of 256 consecutive columns of a row, 8 elements per lane.  VEC (every row starts on a 16-byte boundary
// and has a multiple of 8 columns): lane l holds columns 8 l .. 8 l + 7, moved 16 bytes at a time.  Otherwise element i of
// lane l is column 32 i + l, so that a warp's accesses are contiguous at any width and stride.
constexpr int kTile = 256;

template <bool VEC>
__device__ __forceinline__ int tile_column(int lane, int i) { return VEC ? lane * 8 + i : i * 32 + lane; }

__device__ __forceinline__ void unpack_bf16x8(const uint4 &r, float (&v)[8]) {
    const unsigned int w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = bf16_bits_to_float(w[k] & 0xFFFFu);
        v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ unsigned int pack_bf16x2(float lo, float hi) {       // round to nearest even
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned int *>(&p);
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
// A value as it comes back from a buffer of type T.
template <typename T> __device__ __forceinline__ float rounded(float v) { return to_float<T>(from_float<T>(v)); }

// One lane's share of a tile as it was loaded: bfloat16 stays packed, so that loads in flight cost half the registers.
template <typename T> struct Share;
template <> struct Share<float> {
    float v[8];
    __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i];
    }
};
template <> struct Share<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void get(float (&o)[8]) const { unpack_bf16x8(r, o); }
};

// 32 bytes of one lane, in one access where the address allows it: a warp's two accesses of 16 bytes per lane would each touch half of
// every 32-byte sector.
__device__ __forceinline__ void load8_f32(const float *q, float (&v)[8]) {
    if ((reinterpret_cast<uintptr_t>(q) & 31u) == 0) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "l"(q)
                     : "memory");
    } else {
        const float4 a = reinterpret_cast<const float4 *>(q)[0], b = reinterpret_cast<const float4 *>(q)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
__device__ __forceinline__ void store8_f32(float *q, const float (&v)[8]) {
    if ((reinterpret_cast<uintptr_t>(q) & 31u) == 0) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
                     "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
    } else {
        reinterpret_cast<float4 *>(q)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(q)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// `p`: the tile's first column; `left` columns of the row remain from there on.  What lies past them is zero.
template <bool VEC>
__device__ __forceinline__ void load_tile(const float *p, int lane, int64_t left, Share<float> &s) {
    if (VEC) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s.v[i] = 0.f;
        if (lane * 8 < left) load8_f32(p + lane * 8, s.v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) s.v[i] = i * 32 + lane < left ? p[i * 32 + lane] : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void load_tile(const __nv_bfloat16 *p, int lane, int64_t left, Share<__nv_bfloat16> &s) {
    if (VEC) {
        s.r = lane * 8 < left ? *reinterpret_cast<const uint4 *>(p + lane * 8) : make_uint4(0u, 0u, 0u, 0u);
    } else {
        const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
        unsigned int w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i * 32 + lane < left ? q[i * 32 + lane] : 0u;
        s.r = make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void load_tile(const T *p, int lane, int64_t left, float (&v)[8]) {
    Share<T> s;
    load_tile<VEC>(p, lane, left, s);
    s.get(v);
}
template <bool VEC>
__device__ __forceinline__ void store_tile(float *p, int lane, int64_t left, const float (&v)[8]) {
    if (VEC) {
        if (lane * 8 < left) store8_f32(p + lane * 8, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i * 32 + lane < left) p[i * 32 + lane] = v[i];
    }
}
template <bool VEC>
__device__ __forceinline__ void store_tile(__nv_bfloat16 *p, int lane, int64_t left, const float (&v)[8]) {
    if (VEC) {
        if (lane * 8 < left) *reinterpret_cast<uint4 *>(p + lane * 8) = pack_bf16x8(v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i * 32 + lane < left) p[i * 32 + lane] = __float2bfloat16_rn(v[i]);
    }
}

// ------------------------------------------------------------------ codes ---
// A block of 128 consecutive elements of a row (the last one of a row may be shorter) is held as e4m3 codes and one power of two:
// with a the largest finite magnitude, the exponent is the smallest e in [-120, 120] with a <= 448 * 2^e, a code is x 2^-e
// rounded to nearest even, and its value code * 2^e.  A power of two loses no more than a free scale would (e4m3 is a floating format:
// the relative step is the same anywhere above its subnormals) and makes the values exact in bfloat16: the tensor cores can
// multiply them without another rounding.  From -120 on every step of a block, 2^-9 2^e, is a bfloat16 number; at 120 codes stop at
// 240, for 256 * 2^120 would be infinite.  What is not finite becomes the code of NaN and has no say in its block's exponent.
constexpr int kCodeBlock = 128;
constexpr int kCodeMinExp = -120, kCodeMaxExp = 120;
constexpr unsigned int kInfBits = 0x7F800000u;

// 448 = 1.75 * 2^8: the exponent is that of a, less 8, and one more if a's mantissa is above 1.75.
__device__ __forceinline__ int code_exponent(unsigned int magnitude_bits) {
    const int e = (int)((magnitude_bits + 0x1FFFFFu) >> 23) - 135;
    return e < kCodeMinExp ? kCodeMinExp : (e > kCodeMaxExp ? kCodeMaxExp : e);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned int)(e + 127) << 23); }  // -126..127
__device__ __forceinline__ unsigned char code_scale_byte(int e) { return (unsigned char)(e + 127); }
// (any byte is a power of two, 2^-127 and 2^128 among them)
__device__ __forceinline__ float scale_of_byte(unsigned int b) {
    return b == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23);
}

__device__ __forceinline__ unsigned short code_pair(float lo, float hi) {
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 value_pair(unsigned short codes) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(codes, __NV_E4M3);
    return __half22float2(__half2(h));
}

// Largest magnitudes among a lane's elements, as bits: m[0] of elements 0..3 and m[1] of 4..7 (VEC: m[0] of all).
template <bool VEC>
__device__ __forceinline__ void magnitudes(const float (&v)[8], unsigned int (&m)[2]) {
    m[0] = m[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m[VEC ? 0 : i >> 2] = max(m[VEC ? 0 : i >> 2], __float_as_uint(v[i]) & 0x7FFFFFFFu);
}
// Codes of a warp's tile (two blocks).  m: as above.  c: the lane's 8 codes in order.  e[0], e[1]: the exponents of the blocks of elements 0..3
// and 4..7 (VEC: both the block of all 8).  Every lane of the warp has to call.
template <bool VEC>
__device__ __forceinline__ void encode_tile(const float (&v)[8], unsigned int (&m)[2], unsigned int (&c)[2], int (&e)[2]) {
#pragma unroll
    for (int o = VEC ? 8 : 16; o > 0; o >>= 1) {
        m[0] = max(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], o));
        if (!VEC) m[1] = max(m[1], __shfl_xor_sync(0xFFFFFFFFu, m[1], o));
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
    if (__any_sync(0xFFFFFFFFu, max(m[0], m[1]) >= kInfBits)) {       // rare: something is not finite
        m[0] = m[1] = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned int b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
            if (b >= kInfBits) x[i] = __uint_as_float(0x7FC00000u);
            else m[VEC ? 0 : i >> 2] = max(m[VEC ? 0 : i >> 2], b);
        }
#pragma unroll
        for (int o = VEC ? 8 : 16; o > 0; o >>= 1) {
            m[0] = max(m[0], __shfl_xor_sync(0xFFFFFFFFu, m[0], o));
            if (!VEC) m[1] = max(m[1], __shfl_xor_sync(0xFFFFFFFFu, m[1], o));
        }
    }
    e[0] = code_exponent(m[0]);
    e[1] = VEC ? e[0] : code_exponent(m[1]);
    const float s0 = power_of_two(-e[0]), s1 = VEC ? s0 : power_of_two(-e[1]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= i < 4 ? s0 : s1;
    if (max(e[0], e[1]) == kCodeMaxExp) {                              // rare; (a NaN passes both comparisons)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (e[i >> 2] != kCodeMaxExp) continue;
            if (x[i] > 240.f) x[i] = 240.f;
            if (x[i] < -240.f) x[i] = -240.f;
        }
    }
    c[0] = (unsigned int)code_pair(x[0], x[1]) | ((unsigned int)code_pair(x[2], x[3]) << 16);
    c[1] = (unsigned int)code_pair(x[4], x[5]) | ((unsigned int)code_pair(x[6], x[7]) << 16);
}
template <bool VEC>
__device__ __forceinline__ void encode_tile(const float (&v)[8], unsigned int (&c)[2], int (&e)[2]) {
    unsigned int m[2];
    magnitudes<VEC>(v, m);
    encode_tile<VEC>(v, m, c, e);
}
// The same of a share as it was loaded (v: its elements): packed bfloat16 are compared two at a time.
template <bool VEC>
__device__ __forceinline__ void encode_share(const Share<float> &s, float (&v)[8], unsigned int (&c)[2], int (&e)[2]) {
    s.get(v);
    encode_tile<VEC>(v, c, e);
}
template <bool VEC>
__device__ __forceinline__ void encode_share(const Share<__nv_bfloat16> &s, float (&v)[8], unsigned int (&c)[2], int (&e)[2]) {
    s.get(v);
    const unsigned int p = __vmaxu2(s.r.x & 0x7FFF7FFFu, s.r.y & 0x7FFF7FFFu), q = __vmaxu2(s.r.z & 0x7FFF7FFFu, s.r.w & 0x7FFF7FFFu);
    unsigned int m[2];
    if (VEC) {
        const unsigned int r = __vmaxu2(p, q);
        m[0] = max(r << 16, r & 0xFFFF0000u);
        m[1] = 0u;
    } else {
        m[0] = max(p << 16, p & 0xFFFF0000u);
        m[1] = max(q << 16, q & 0xFFFF0000u);
    }
    encode_tile<VEC>(v, m, c, e);
}
// What a lane's 8 codes stand for; s0, s1: the scales of elements 0..3 and 4..7.
__device__ __forceinline__ void decode8(const unsigned int (&c)[2], float s0, float s1, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = value_pair((unsigned short)(c[k >> 1] >> (16 * (k & 1))));
        const float s = k < 2 ? s0 : s1;
        v[2 * k] = f.x * s;
        v[2 * k + 1] = f.y * s;
    }
}

// Writes a tile's codes and scale bytes.  `codes`: the tile's first code; `scales`: the tile's first scale byte.
template <bool VEC>
__device__ __forceinline__ void store_codes(unsigned char *codes, unsigned char *scales, int lane, int64_t left,
                                            const unsigned int (&c)[2], const int (&e)[2]) {
    if (VEC) {
        if (lane * 8 < left) *reinterpret_cast<uint2 *>(codes + lane * 8) = make_uint2(c[0], c[1]);
        if ((lane & 15) == 0 && lane * 8 < left) scales[lane >> 4] = code_scale_byte(e[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i * 32 + lane < left) codes[i * 32 + lane] = (unsigned char)(c[i >> 2] >> (8 * (i & 3)));
        if (lane < 2 && lane * kCodeBlock < left) scales[lane] = code_scale_byte(lane == 0 ? e[0] : e[1]);
    }
}
// One lane's codes of a tile and the scales of its elements 0..3 and 4..7.
struct CodeShare {
    unsigned int c[2];
    unsigned int s;             // the two scale bytes
    __device__ __forceinline__ void get(float (&v)[8]) const { decode8(c, scale_of_byte(s & 0xFFu), scale_of_byte(s >> 8), v); }
};
template <bool VEC>
__device__ __forceinline__ void load_codes(const unsigned char *codes, const unsigned char *scales, int lane, int64_t left,
                                           CodeShare &s) {
    s.c[0] = s.c[1] = 0u;
    s.s = 0x7F7Fu;
    if (VEC) {
        if (lane * 8 < left) {
            const uint2 r = *reinterpret_cast<const uint2 *>(codes + lane * 8);
            s.c[0] = r.x;
            s.c[1] = r.y;
            s.s = scales[lane >> 4] * 0x101u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i * 32 + lane < left) s.c[i >> 2] |= (unsigned int)codes[i * 32 + lane] << (8 * (i & 3));
        if (left > 0) s.s = scales[0] | ((left > kCodeBlock ? scales[1] : 0x7Fu) << 8);
    }
}

// -------------------------------------------------------------- reductions --

__device__ __forceinline__ float warp_sum(float v) {        // the same sum in every lane
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

}  // namespace gaf
