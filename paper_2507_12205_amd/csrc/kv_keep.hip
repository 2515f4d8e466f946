// The rows of an accepted path, which lie where their nodes were written, moved to follow one another: key first + path[i] of a sequence
// becomes its key first + i, in the caches of many layers at once.
//
// path[i] >= i (a path grows): a row lies behind every place that rows before it go to, so that rows which are copied in order stay whole.  A
// thread copies one piece of a row, the same one of every row of its sequence, head and layer, eight of them under way at once: nobody else
// reads or writes these places, and there is nothing to wait for.  Bits are copied as they are.
//
// What bounds it are four trips to memory, one after the other (how many and where, pages, rows, their new places), and rows that lie apart: five
// rows of 40 heads of 128 in 40 layers, 16 bits, 4.5 us (4 MB read and 4 written); four of 8 heads of 128 of 32 sequences in 32 layers, 4 bits, 7.9 (65536
// rows of 64 and 4 bytes; several rows at once in a workgroup, all read before any is written: 8.3).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "serve.h"

namespace {

using ecs::KeepArgs;

constexpr uint32_t kThreads = 256, kAtOnce = 8;
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));

// `count` pieces from `at` to `to` (of them, the i-th at `base` + [i] * bytes), in order
template <class Piece>
__device__ __forceinline__ void copy_rows(uint8_t *base, const uint64_t (*rows)[2], uint32_t count, uint32_t bytes)
{
    for (uint32_t i = 0; i < count; i += kAtOnce) {
        Piece x[kAtOnce];
        uint64_t to[kAtOnce];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t j = min(i + u, count - 1u);
            to[u] = rows[j][1];
            x[u] = *reinterpret_cast<const Piece *>(base + rows[j][0] * bytes);
        }
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u)
            if (i + u < count) *reinterpret_cast<Piece *>(base + to[u] * bytes) = x[u];
    }
}

template <class Piece>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(const KeepArgs a)
{
    __shared__ uint64_t rows[kThreads][2];                                // from, to: rows of the cache (of head 0)
    __shared__ uint32_t counts[kThreads / 64];
    const uint32_t seq = blockIdx.y, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t pieces = a.row_bytes / (uint32_t)sizeof(Piece);
    const uint32_t layer = blockIdx.x / a.blocks, work = (blockIdx.x - layer * a.blocks) * kThreads + tid;
    const uint32_t each = pieces + a.steps;                               // a head's pieces of codes, and its step
    const uint32_t head = work / each, piece = work - head * each;
    const ecs::KeepArgs::Tensors &t = a.layer[layer >> 1];
    uint8_t *codes = (layer & 1u) ? t.v : t.k, *steps = (layer & 1u) ? t.v_step : t.k_step;

    const uint32_t n = (uint32_t)min(max(a.accepted[seq], 0), (int32_t)a.nodes);
    const int64_t first = a.first[seq], places = (int64_t)a.max_pages << a.page_shift;
    const int32_t *path = a.path + (int64_t)seq * a.path_stride, *table = a.table + (int64_t)seq * a.table_stride;
    for (uint32_t i0 = 0; i0 < n; i0 += kThreads) {
        // where the next rows are and go; those that lie right, or nowhere, are left out
        uint64_t from = 0, to = 0;
        bool moves = false;
        if (i0 + tid < n) {
            const int32_t node = path[i0 + tid];
            const int64_t x = first + node, y = first + i0 + tid;
            if (node > (int32_t)(i0 + tid) && first >= 0 && x < places) {
                const uint32_t px = (uint32_t)table[x >> a.page_shift], py = (uint32_t)table[y >> a.page_shift];
                const uint32_t mask = (1u << a.page_shift) - 1u;
                moves = px < a.pages && py < a.pages;
                from = (((uint64_t)px * a.heads) << a.page_shift) + ((uint32_t)x & mask);
                to = (((uint64_t)py * a.heads) << a.page_shift) + ((uint32_t)y & mask);
            }
        }
        const uint64_t some = __ballot(moves);
        if (lane == 0) counts[wave] = (uint32_t)__popcll(some);
        __syncthreads();
        uint32_t at = (uint32_t)__popcll(some & ((1ull << lane) - 1ull)), count = 0;
#pragma unroll
        for (uint32_t w = 0; w < kThreads / 64u; ++w) {
            at += w < wave ? counts[w] : 0u;
            count += counts[w];
        }
        if (moves) rows[at][0] = from, rows[at][1] = to;
        __syncthreads();
        if (count && head < a.heads) {
            const uint64_t head_row = (uint64_t)head << a.page_shift;
            if (piece < pieces)
                copy_rows<Piece>(codes + head_row * a.row_bytes + piece * sizeof(Piece), rows, count, a.row_bytes);
            else
                copy_rows<uint32_t>(steps + 4u * head_row, rows, count, 4u);
        }
        __syncthreads();
    }
}

}  // namespace

namespace ecs {

int launch_kv_keep(KeepArgs &a, uint32_t layers, uint32_t batch, void *stream)
{
    const uint32_t piece = a.row_bytes % 16u == 0 ? 16u : 8u;
    a.blocks = (a.heads * (a.row_bytes / piece + a.steps) + kThreads - 1u) / kThreads;
    return piece == 16u ? launch_args<kv_keep_kernel<words4>>(a, 2u * layers * a.blocks, batch, 1, kThreads, stream)
                        : launch_args<kv_keep_kernel<words2>>(a, 2u * layers * a.blocks, batch, 1, kThreads, stream);
}

}  // namespace ecs
