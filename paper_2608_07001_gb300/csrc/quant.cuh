// quant.cuh -- rows of a quantised cache: d codes of e4m3 and one scale 2^e.
//
// e is the smallest integer of [-120, 119] with max |x| <= 448 2^e over the
// row's finite values, 448 the largest code; a code is x 2^-e rounded to
// nearest even (NaN for what is not finite, +-448 above 448 2^119).  A power of two scales
// without a rounding of its own, and a floating code keeps its 4 significant bits
// wherever in the range the row ends, so a finer scale would gain nothing.  The
// value code 2^e has 4 bits and lies between 2^-129 and 1.75 2^127: exact in bf16
// and fp32, and written again it comes back as it was.  A byte holds e + 127.
#pragma once

#include "serve.cuh"

#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

namespace gkv {
namespace serve {

struct E4m3 { uint8_t bits; };                 // storage of a quantised pool

__device__ __forceinline__ float finite_size(float x) {
    const float a = fabsf(x);
    return a <= FLT_MAX ? a : 0.f;
}

// e + 127 from the largest finite size: its exponent p with 1.m <= 1.75, one more above (the sum carries), less 8.
__device__ __forceinline__ int row_scale_byte(float top) {
    return min(max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8, 7), 246);
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float inverse_of(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Codes of two values times inv, the first in the low byte.
__device__ __forceinline__ uint32_t codes2(float x, float y, float inv) {
    x = fabsf(x) <= FLT_MAX ? x * inv : NAN;
    y = fabsf(y) <= FLT_MAX ? y * inv : NAN;
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t codes4(const float *x, float inv) {
    return codes2(x[0], x[1], inv) | codes2(x[2], x[3], inv) << 16;
}

// The two codes in the low half of c as numbers.
__device__ __forceinline__ float2 values2(uint32_t c) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The largest of `n` lanes (a power of two, all of one row), in each of them.  The other lanes of the warp may be elsewhere.
template <int N>
__device__ __forceinline__ float row_max(float x) {
    const int lane = threadIdx.x & 31;
    const unsigned mask = N == 32 ? 0xffffffffu : ((1u << (N & 31)) - 1) << (lane & ~(N - 1));
#pragma unroll
    for (int o = N / 2; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor_sync(mask, x, o));
    return x;
}

// 16 bytes of a row: 4 or 8 numbers.
__device__ __forceinline__ void unpack16(uint4 u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x);
    x[1] = __uint_as_float(u.y);
    x[2] = __uint_as_float(u.z);
    x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(uint4 u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
template <int N>
__device__ __forceinline__ float top_of(const float (&x)[N]) {
    float m = finite_size(x[0]);
#pragma unroll
    for (int i = 1; i < N; i++) m = fmaxf(m, finite_size(x[i]));
    return m;
}
// Their codes, at 4 or 8 bytes.
__device__ __forceinline__ void put_codes(uint8_t *p, const float (&x)[4], float inv) {
    *reinterpret_cast<uint32_t *>(p) = codes4(x, inv);
}
__device__ __forceinline__ void put_codes(uint8_t *p, const float (&x)[8], float inv) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(codes4(x, inv), codes4(x + 4, inv));
}

}  // namespace serve
}  // namespace gkv
