// The paged cache of keys and values: quantised as it is written, and read back.
//
// A row is what one token has in one head: dim values.  Eight of them go through a lane (one 128-bit access where the rows of k
// and v allow it, else value by value), a row takes the next power of two of dim / 8 lanes, and its largest (and smallest) value
// is found by exchanges between these lanes, so that every value is read once and every code written once: a row is one trip to
// memory, and what bounds it is how many rows are under way (8191 tokens, 8 heads of 128: 16 bits 14.4 us, 67 MB at 4.6 TB/s; 8 bits
// 15.8, 4 bits 15.1; read back 11.9, 10.8, 10.5.  One lane for k's and v's row together: 14.4, 15.3, 14.9 and 11.9, 10.8, 9.4, but 8
// tokens of 40 heads 3.7 -> 5.1).
//   8 bits: s = max|x| / 127 (FP32),                      code = rint(x / s),        x ~ s * code
//   4 bits: z = min x, s = (max x - z) / 15 (both FP16),  code = rint((x - z) / s),  x ~ z + s * code
//           (s is the next smaller FP16 value where z + 15 s would not be one)
// The steps are computed and applied in FP32; 4-bit codes are taken with the step as it is kept, in 16 bits, so that nothing but the
// code itself is rounded.  NaN counts as 0 and infinities as the largest FP16 value: a code stands for a finite value.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "serve.h"

namespace {

using ecs::Cache;
using ecs::KvArgs;
using ecs::View;

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

// Which row a lane works on.  Rows are taken 2^run_shift neighbouring tokens of one head after another: a workgroup's codes then lie side
// by side in the cache (with the heads of one token after another every row went to a place of its own, 64 bytes of 4-bit codes and 4 of
// steps: 8191 tokens, 8 heads of 128, written in 16.4 us).  k and v are the two halves of the grid.
struct Row {
    bool of_v, valid;
    uint32_t token, head, at, lane;       // at: its first value
    uint64_t place;                       // row of the cache
    __device__ __forceinline__ Row(const KvArgs &a)
    {
        const uint32_t lanes = 1u << a.lanes_shift;
        const uint32_t in_block = threadIdx.x >> a.lanes_shift, per_block = blockDim.x >> a.lanes_shift;
        const uint32_t r = blockIdx.x * per_block + in_block;
        of_v = blockIdx.y != 0;
        lane = threadIdx.x & (lanes - 1u);
        at = 8u * lane;
        const uint32_t turn = r >> a.run_shift, first = turn / a.cache.heads;
        head = turn - first * a.cache.heads;
        const uint32_t mine = (first << a.run_shift) + (r & ((1u << a.run_shift) - 1u));
        const bool some = mine < a.tokens;
        token = min(mine, a.tokens - 1u);
        const int64_t slot = a.slots[token];
        valid = some && slot >= 0 && slot < (int64_t)a.cache.pages << a.cache.page_shift && at < a.cache.dim;
        const uint64_t page = (uint64_t)slot >> a.cache.page_shift, off = (uint64_t)slot & ((1u << a.cache.page_shift) - 1u);
        place = ((page * a.cache.heads + head) << a.cache.page_shift) + off;
        inside = some && at < a.cache.dim;
    }
    bool inside;                          // this lane has values, whether or not the slot is one of the cache's
};

template <int BITS>
__global__ __launch_bounds__(256) void kv_write_kernel(const KvArgs a)
{
    const Row r(a);
    const View &from = r.of_v ? a.v : a.k;
    Eight e = {};
    if (r.inside) e = load_eight(from, r.of_v ? a.v_wide : a.k_wide, r.token, r.head, r.at);       // (not waiting for the slot)
    uint8_t *codes = (r.of_v ? a.cache.v : a.cache.k) + r.place * a.cache.row_bytes;
    uint8_t *steps = (r.of_v ? a.cache.v_step : a.cache.k_step) + r.place * 4u;
    if constexpr (BITS == 16) {
        if (r.valid) *reinterpret_cast<uint4 *>(codes + 2u * r.at) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
        return;
    }
    float x[8], low = 65504.0f, high = -65504.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = to_float(e.get(i));
        x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -65504.0f), 65504.0f);
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
    }
    if (r.at >= a.cache.dim) low = 65504.0f, high = -65504.0f;            // a lane without values
    for (uint32_t o = 1u; o < 1u << a.lanes_shift; o <<= 1) {
        low = fminf(low, __shfl_xor(low, (int)o, 64));
        high = fmaxf(high, __shfl_xor(high, (int)o, 64));
    }
    if constexpr (BITS == 8) {
        const float most = fmaxf(-low, high), step = most / 127.0f, inv = most > 0.0f ? 1.0f / most * 127.0f : 0.0f;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (int)fminf(fmaxf(rintf(x[i] * inv), -127.0f), 127.0f);
            w[i >> 2] |= ((uint32_t)c & 0xFFu) << (8 * (i & 3));
        }
        if (r.valid) {
            *reinterpret_cast<uint2 *>(codes + r.at) = make_uint2(w[0], w[1]);
            if (r.lane == 0) *reinterpret_cast<float *>(steps) = step;
        }
    } else {
        uint32_t step_bits = to_half((high - low) / 15.0f);
        if (fmaf(15.0f, to_float(step_bits), low) >= 65520.0f) --step_bits;  // (rounded up, and the last code would be infinity in FP16)
        const float step = to_float(step_bits), inv = step > 0.0f ? 1.0f / step : 0.0f;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w |= (uint32_t)fminf(fmaxf(rintf((x[i] - low) * inv), 0.0f), 15.0f) << (4 * i);
        if (r.valid) {
            *reinterpret_cast<uint32_t *>(codes + (r.at >> 1)) = w;
            if (r.lane == 0) *reinterpret_cast<uint32_t *>(steps) = step_bits | to_half(low) << 16;
        }
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void kv_read_kernel(const KvArgs a)
{
    const Row r(a);
    if (!r.inside) return;
    Eight e = {};                                                         // a slot that is none: zeros
    if (r.valid) {
        const uint8_t *codes = (r.of_v ? a.cache.v : a.cache.k) + r.place * a.cache.row_bytes;
        const uint8_t *steps = (r.of_v ? a.cache.v_step : a.cache.k_step) + r.place * 4u;
        if constexpr (BITS == 16) {
            const uint4 t = *reinterpret_cast<const uint4 *>(codes + 2u * r.at);
            e.w[0] = t.x, e.w[1] = t.y, e.w[2] = t.z, e.w[3] = t.w;
        } else if constexpr (BITS == 8) {
            const uint2 t = *reinterpret_cast<const uint2 *>(codes + r.at);
            const float step = *reinterpret_cast<const float *>(steps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (int)(int8_t)((i < 4 ? t.x : t.y) >> (8 * (i & 3)));
                e.w[i >> 1] |= to_half((float)c * step) << (16 * (i & 1));
            }
        } else {
            const uint32_t t = *reinterpret_cast<const uint32_t *>(codes + (r.at >> 1));
            const uint32_t s = *reinterpret_cast<const uint32_t *>(steps);
            const float step = to_float(s & 0xFFFFu), low = to_float(s >> 16);
#pragma unroll
            for (int i = 0; i < 8; ++i)      // (a 4-bit code times an 11-bit step is exact: rounded once in FP32, once to FP16)
                e.w[i >> 1] |= to_half(fmaf((float)((t >> (4 * i)) & 15u), step, low)) << (16 * (i & 1));
        }
    }
    store_eight(r.of_v ? a.v : a.k, r.of_v ? a.v_wide : a.k_wide, r.token, r.head, r.at, e);
}

template <auto K16, auto K8, auto K4>
int launch(const KvArgs &a, void *stream)
{
    const uint32_t per_block = 256u >> a.lanes_shift, runs = (a.tokens + (1u << a.run_shift) - 1u) >> a.run_shift;
    const uint64_t rows = ((uint64_t)runs * a.cache.heads) << a.run_shift;
    const uint32_t grid = (uint32_t)((rows + per_block - 1u) / per_block);
    switch (a.cache.bits) {
    case 16: return ecs::launch_args<K16>(a, grid, 2, 1, 256, stream);
    case 8: return ecs::launch_args<K8>(a, grid, 2, 1, 256, stream);
    default: return ecs::launch_args<K4>(a, grid, 2, 1, 256, stream);
    }
}

}  // namespace

namespace ecs {

int launch_kv_write(const KvArgs &a, void *stream)
{
    return launch<kv_write_kernel<16>, kv_write_kernel<8>, kv_write_kernel<4>>(a, stream);
}

int launch_kv_read(const KvArgs &a, void *stream)
{
    return launch<kv_read_kernel<16>, kv_read_kernel<8>, kv_read_kernel<4>>(a, stream);
}

}  // namespace ecs
