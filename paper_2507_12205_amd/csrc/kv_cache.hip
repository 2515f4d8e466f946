// The paged cache of keys and values: quantised as it is written, and read back.
//
// A row is what one token has in one head: dim values.  Eight of them go through a lane (one 128-bit access where the rows of k
// and v allow it, else value by value), a row takes the next power of two of dim / 8 lanes, and its largest (and smallest) value
// is found by exchanges between these lanes, so that every value is read once and every code written once: a row is one trip to
// memory, and what bounds it is how many rows are under way (8191 tokens, 8 heads of 128: 16 bits 14.4 us, 67 MB at 4.6 TB/s; 8 bits
// 15.8, 4 bits 15.1; read back 11.9, 10.8, 10.5.  One lane for k's and v's row together: 14.4, 15.3, 14.9 and 11.9, 10.8, 9.4, but 8
// tokens of 40 heads 3.7 -> 5.1).
// Codes and steps: kv_rows.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "kv_rows.h"
#include "serve.h"

namespace {

using ecs::Cache;
using ecs::Eight;
using ecs::KvArgs;
using ecs::View;
using ecs::load_eight;
using ecs::store_eight;
using ecs::to_float;
using ecs::to_half;

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
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_float(e.get(i));
        ecs::store_codes<BITS, false>(x, codes, steps, {r.at}, a.cache.dim, a.lanes_shift, r.valid);
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
