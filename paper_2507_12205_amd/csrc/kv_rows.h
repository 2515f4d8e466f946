// Rows of the paged cache as a group of lanes has them, eight values to a lane: how they come from a view and go to one, and how they
// become codes.
//   8 bits: s = max|x| / 127 (FP32),                      code = rint(x / s),        x ~ s * code
//   4 bits: z = min x, s = (max x - z) / 15 (both FP16),  code = rint((x - z) / s),  x ~ z + s * code
//           (s is the next smaller FP16 value where z + 15 s would not be one)
// The steps are computed and applied in FP32; 4-bit codes are taken with the step and the lowest value as they are kept, in 16 bits, so that
// nothing but the code itself is rounded.  NaN counts as 0 and what is beyond FP16's largest value as that: a code stands for a finite value.
#ifndef ECSPMV_KV_ROWS_H
#define ECSPMV_KV_ROWS_H

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "serve.h"

namespace ecs {

__device__ __forceinline__ float to_float(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }
__device__ __forceinline__ uint32_t to_half(float f) { return __half_as_ushort(__float2half_rn(f)); }

struct Eight {
    uint32_t w[4];
    __device__ __forceinline__ uint32_t get(int i) const { return (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu; }
};

__device__ __forceinline__ Eight load_eight(const View &v, uint32_t wide, uint32_t token, uint32_t head, uint32_t at)
{
    const uint16_t *p = v.data + (int64_t)token * v.token_stride + (int64_t)head * v.head_stride + (int64_t)at * v.dim_stride;
    Eight e;
    if (wide) {
        const uint4 t = *reinterpret_cast<const uint4 *>(p);
        e.w[0] = t.x, e.w[1] = t.y, e.w[2] = t.z, e.w[3] = t.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) e.w[i] = (uint32_t)p[(2 * i) * v.dim_stride] | (uint32_t)p[(2 * i + 1) * v.dim_stride] << 16;
    }
    return e;
}

__device__ __forceinline__ void store_eight(const View &v, uint32_t wide, uint32_t token, uint32_t head, uint32_t at, const Eight &e)
{
    uint16_t *p = v.data + (int64_t)token * v.token_stride + (int64_t)head * v.head_stride + (int64_t)at * v.dim_stride;
    if (wide) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i * v.dim_stride] = (uint16_t)e.get(i);
    }
}

// The codes and the step of a row that 2^lanes_shift neighbouring lanes have, N values each in pieces of eight that start at at[...] of the row (a piece
// that starts beyond it is none), to where they lie; `valid`: whether the row has a place.  All lanes of the row come here.  WIDE: values need not be FP16
// values, so that the lowest one is rounded to what is kept of it.  `turned`: a row that has been rotated; its 4-bit step is the range times 1/15, as a
// program gets it that divides by a number in FP32 tensor operations (where the quotient lies between two FP16 values, it may be the other one).
template <int BITS, bool WIDE, int N>
__device__ __forceinline__ void store_codes(float (&x)[N], uint8_t *codes, uint8_t *steps, const uint32_t (&at)[N / 8], uint32_t dim, uint32_t lanes_shift,
                                            bool valid, bool turned = false)
{
    float low = 65504.0f, high = -65504.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -65504.0f), 65504.0f);
        if (N == 8 || at[i / 8] < dim) {
            low = fminf(low, x[i]);
            high = fmaxf(high, x[i]);
        }
    }
    if (N == 8 && at[0] >= dim) low = 65504.0f, high = -65504.0f;         // a lane without values
    for (uint32_t o = 1u; o < 1u << lanes_shift; o <<= 1) {
        low = fminf(low, __shfl_xor(low, (int)o, 64));
        high = fmaxf(high, __shfl_xor(high, (int)o, 64));
    }
    if constexpr (BITS == 8) {
        const float most = fmaxf(-low, high), step = most / 127.0f, inv = most > 0.0f ? 1.0f / most * 127.0f : 0.0f;
#pragma unroll
        for (int k = 0; k < N / 8; ++k) {
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (int)fminf(fmaxf(rintf(x[8 * k + i] * inv), -127.0f), 127.0f);
                w[i >> 2] |= ((uint32_t)c & 0xFFu) << (8 * (i & 3));
            }
            if (valid && (N == 8 || at[k] < dim)) *reinterpret_cast<uint2 *>(codes + at[k]) = make_uint2(w[0], w[1]);
        }
        if (valid && at[0] == 0) *reinterpret_cast<float *>(steps) = step;
    } else {
        const uint32_t low_bits = to_half(low);
        uint32_t step_bits;
        if constexpr (WIDE) {
            low = to_float(low_bits);
            const float range = fmaxf(high - low, 0.0f);                   // (rounded up, the lowest value may be above the largest)
            float product = range * (1.0f / 15.0f);
            asm("" : "+v"(product));                                       // (a product in FP32: not one that is rounded to FP16 at once)
            step_bits = to_half(turned ? product : range / 15.0f);
        } else {
            step_bits = to_half((high - low) / 15.0f);
        }
        if (fmaf(15.0f, to_float(step_bits), low) >= 65520.0f) --step_bits;  // (rounded up, and the last code would be infinity in FP16)
        const float step = to_float(step_bits), inv = step > 0.0f ? 1.0f / step : 0.0f;
#pragma unroll
        for (int k = 0; k < N / 8; ++k) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= (uint32_t)fminf(fmaxf(rintf((x[8 * k + i] - low) * inv), 0.0f), 15.0f) << (4 * i);
            if (valid && (N == 8 || at[k] < dim)) *reinterpret_cast<uint32_t *>(codes + (at[k] >> 1)) = w;
        }
        if (valid && at[0] == 0) *reinterpret_cast<uint32_t *>(steps) = step_bits | low_bits << 16;
    }
}

}  // namespace ecs
#endif
