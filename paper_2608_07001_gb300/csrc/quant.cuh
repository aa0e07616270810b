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

#include <type_traits>

namespace gkv {
namespace serve {

struct E4m3 { uint8_t bits; };                 // storage of a quantised pool

__device__ __forceinline__ float finite_size(float x) {
    const float a = fabsf(x);
    return a <= FLT_MAX ? a : 0.f;
}

// e + 127 from the bits of the largest finite size: its exponent p with 1.m <= 1.75, one more above (the sum carries), less 8.
__device__ __forceinline__ int row_scale_byte(uint32_t top) {
    return min(max((int)((top + 0x1fffffu) >> 23) - 8, 7), 246);
}
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float inverse_of(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Codes of two values times inv, the first in the low byte.
__device__ __forceinline__ uint32_t codes2(float x, float y, float inv) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y * inv), "f"(x * inv));
    return r;
}
__device__ __forceinline__ uint32_t codes4(const float *x, float inv) {
    return codes2(x[0], x[1], inv) | codes2(x[2], x[3], inv) << 16;
}

// The two codes in the low half of c, as f16 (exact) and as numbers.
__device__ __forceinline__ uint32_t f16x2_codes(uint32_t c) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
    return h;
}
__device__ __forceinline__ float2 values2(uint32_t c) {
    const uint32_t h = f16x2_codes(c);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
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
// The size of a number as its bits without the sign: ordered as the sizes are, infinity and NaN above all others.
constexpr uint32_t kInfBits = 0x7f800000u;
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float (&x)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
}
template <int N>
__device__ __forceinline__ uint32_t top_finite_bits(const float (&x)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) m = max(m, __float_as_uint(finite_size(x[i])));
    return m;
}
// The largest of N lanes (a power of two, all of one row), in each of them.  The other lanes of the warp may be elsewhere.
template <int N>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    const int lane = threadIdx.x & 31;
    const unsigned mask = N == 32 ? 0xffffffffu : ((1u << (N & 31)) - 1) << (lane & ~(N - 1));
#pragma unroll
    for (int o = N / 2; o >= 1; o >>= 1) x = max(x, __shfl_xor_sync(mask, x, o));
    return x;
}
// The scale byte of a row of which LANES lanes hold N numbers each; those that are not finite become NaN.
template <int LANES, int N>
__device__ __forceinline__ int row_scale(float (&x)[N]) {
    uint32_t top = row_max<LANES>(top_bits(x));
    if (top >= kInfBits) {                     // the row's lanes together
#pragma unroll
        for (int i = 0; i < N; i++)
            if (!(fabsf(x[i]) <= FLT_MAX)) x[i] = NAN;
        top = row_max<LANES>(top_finite_bits(x));
    }
    return row_scale_byte(top);
}
// Their codes, at 4 or 8 bytes.
__device__ __forceinline__ void put_codes(uint8_t *p, const float *x, float inv, std::integral_constant<int, 4>) {
    *reinterpret_cast<uint32_t *>(p) = codes4(x, inv);
}
__device__ __forceinline__ void put_codes(uint8_t *p, const float *x, float inv, std::integral_constant<int, 8>) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(codes4(x, inv), codes4(x + 4, inv));
}
template <int N>
__device__ __forceinline__ float top_of(const float (&x)[N]) { return __uint_as_float(top_finite_bits(x)); }

}  // namespace serve
}  // namespace gkv
