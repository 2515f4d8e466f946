// New tokens into the paged cache with their positions in them: keys (and queries) are rotated, pair by pair of their first values,
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair,
// keys and values become codes and go to their places, queries go to where the caller wants them.  One launch.
//
// A row is what one token has in one head of q, k or v.  A lane has 16 values of it, two pieces of eight: both halves of eight pairs, or 16
// neighbouring values, so that nothing is exchanged between lanes but a row's least and largest value.  A workgroup takes up to 16
// neighbouring tokens and some heads of them, in q the heads of a token after one another, as they lie, in k and v (and in q that lies as columns)
// the tokens of a head, as they come to lie in the cache.  The turns of these tokens are worked out once, by all of its threads, and lie in LDS for all of
// its rows.  What bounds it is memory: 8191 tokens, 64/8 heads of 128, 16 bits 77 us, 336 MB at 4.3 TB/s, 8 bits 81, 4 bits 79 (eight values a lane
// with their partners' from another lane, q in the order of k and v: 95, 99, 99); 8 tokens, 12/12 heads of 64 as columns, 4.0.  In heads of 80 five of
// a row's eight lanes have values: 8191 tokens, 32/32 heads, 16 bits 84 us, 252 MB at 3.0 TB/s; with 20 of the 40 pairs 98, as partners then come
// through LDS, value by value (kAnywhere; where the pairs' number is no multiple of 8).
//
// An angle is a product in 64 bits (of position 10^6, 32 bits would leave 0.03 of an angle), and so are its cosine and sine, which are then
// rounded to 32; the rotated values stay in 32 bits until they are rounded once, to FP16 or to a code.  The two products of a pair are
// rounded each: a code next to its border is then the one that a program gets which rotates in FP32 operations of its own.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "kernel_handle.h"
#include "kv_rows.h"
#include "serve.h"

namespace {

using ecs::AppendArgs;
using ecs::Eight;
using ecs::to_float;
using ecs::to_half;

constexpr uint32_t kThreads = 256, kRun = 16;                            // tokens of a workgroup, if there are more than 8

// Cosine and sine of x turns, by their series around the nearest quarter of a turn: |y| <= pi / 4, what is left out is below 3e-14
__device__ __forceinline__ void turn(double x, float &c, float &s)
{
    x -= rint(x);
    const double quarter = rint(4.0 * x), y = (x - 0.25 * quarter) * 6.283185307179586477, z = y * y;
    const double si = y * (1.0 + z * (-1.0 / 6 + z * (1.0 / 120 + z * (-1.0 / 5040 + z * (1.0 / 362880 + z * (-1.0 / 39916800 + z * (1.0 / 6227020800)))))));
    const double co = 1.0 + z * (-1.0 / 2 + z * (1.0 / 24 + z * (-1.0 / 720 + z * (1.0 / 40320 + z * (-1.0 / 3628800 + z * (1.0 / 479001600 + z * (-1.0 / 87178291200)))))));
    const int q = (int)quarter;                                           // -2 ... 2
    c = (float)((q & 1) ? ((q & 2) ? si : -si) : ((q & 2) ? -co : co));
    s = (float)((q & 1) ? ((q & 2) ? -co : co) : ((q & 2) ? -si : si));
}

// a c + b s, each product rounded by itself
__device__ __forceinline__ float turned(float a, float c, float b, float s)
{
#pragma clang fp contract(off)
    const float x = a * c, y = b * s;
    return x + y;
}

// The run of tokens of workgroup x of n: neighbouring runs, which share lines of memory where tokens lie in columns, on the same die (every eighth
// workgroup) one after another: 8191 tokens, 64/8 heads of 128 in columns, 16 bits 240 us without, 174 with
__device__ __forceinline__ uint32_t run_of(uint32_t x, uint32_t n)
{
    const uint32_t die = x & 7u;
    return die * (n >> 3) + min(die, n & 7u) + (x >> 3);
}

// A value of 16 neighbouring tokens, of which there are `count`, where tokens lie after one another
__device__ __forceinline__ void load_column(const uint16_t *p, uint32_t count, Eight (&e)[2])
{
    if (count >= kRun) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint4 w = *reinterpret_cast<const uint4 *>(p + 8 * k);
            e[k] = Eight{{w.x, w.y, w.z, w.w}};
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kRun; ++i)
            if (i < count) e[i / 8].w[i % 8 / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    }
}
__device__ __forceinline__ void store_column(uint16_t *p, uint32_t count, const uint32_t (&w)[8])
{
    if (count >= kRun) {
#pragma unroll
        for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4 *>(p + 8 * k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < kRun; ++i)
            if (i < count) p[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
    }
}

// How the pairs of a head lie in a lane's pieces: halves of eight pairs, neighbours, or halves that begin anywhere (their partners are looked up)
enum { kHalves, kNeighbours, kAnywhere };

template <int BITS, int PAIRS, bool COLUMNS>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float turns[];            // [token of the run][cos, sin][pair]
    __shared__ uint4 rows_lds[PAIRS == kAnywhere ? 2 * kThreads : 1];     // two pieces of every lane
    const uint32_t tid = threadIdx.x, first = (a.q_wide && a.k_wide && a.v_wide ? blockIdx.x : run_of(blockIdx.x, gridDim.x)) << a.run_shift;
    const uint32_t run = min(1u << a.run_shift, a.tokens - first);
    // heads of q, or heads of k and then of v
    const bool of_q = blockIdx.y < a.q_blocks;
    const uint32_t all = of_q ? a.q_heads : 2u * a.cache.heads, head0 = (blockIdx.y - (of_q ? 0u : a.q_blocks)) * a.heads_per_block;
    const uint32_t heads = min(a.heads_per_block, all - head0), rows = heads << a.run_shift;
    const uint32_t lane = tid & ((1u << a.lanes_shift) - 1u), dim = a.cache.dim, pairs = a.pairs, pad = (pairs + 3u) & ~3u;
    const uint32_t per_pass = kThreads >> a.lanes_shift;
    const bool by_token = of_q && a.q_wide;                               // one token's heads after another (else they lie as columns)
    // where this lane's pieces start, and its first pair
    uint32_t at[2] = {16u * lane, 16u * lane + 8u};
    if (PAIRS == kHalves && lane < pairs / 8u) at[0] = 8u * lane, at[1] = 8u * lane + pairs;
    const uint32_t pair0 = 8u * lane;

    // Where tokens lie in columns, a thread brings one value of 16 tokens, and the rows of a pass are put together in LDS (rows of 16-byte pieces, one more
    // than they need).  By rows, a lane reads its values one by one: 64/8 heads of 128, 16 bits, 8191 tokens so 158 us, 8184 by columns 108, 16/16 heads of 256,
    // 4001 tokens 125, 4000 62.  A run has 32 bytes of each line of 128, and three barriers to a pass: wavefronts wait for 56 % of their time (rows: 77 us; a
    // run of 64 tokens would take whole lines, and four times the LDS for its turns).  Columns that start off 16 bytes are read by rows, value by value, 4.6
    // times the memory instructions (by columns all the same 263 for 176: 8191 tokens, up to 32 heads).
    const bool columns = COLUMNS && (of_q ? a.q_columns : a.kv_columns), columns_out = of_q && columns && a.q_out_columns;
    const uint32_t tile_row = 32u << a.lanes_shift, tile_step = tile_row + 16u;         // bytes
    uint8_t *tile = reinterpret_cast<uint8_t *>(turns + 2u * pad * (1u << a.run_shift));
    const uint32_t column = tid & ((16u << a.lanes_shift) - 1u), column_head = tid >> (a.lanes_shift + 4u);
    uint8_t *tile_column = tile + kRun * column_head * tile_step + 2u * column;

    struct Rows {
        uint32_t head, token;
        bool inside, of_v;
        int64_t slot;
        Eight e[2];
    };
    auto ask = [&](uint32_t pass) {                                       // sends the loads of this lane's row of a pass off
        Rows r;
        const uint32_t i = pass * per_pass + (tid >> a.lanes_shift);
        const uint32_t in_run = by_token ? i / heads : i & ((1u << a.run_shift) - 1u);
        r.head = head0 + (by_token ? i - in_run * heads : i >> a.run_shift);
        r.inside = i < rows && in_run < run;
        r.token = first + min(in_run, run - 1u);
        r.of_v = !of_q && r.head >= a.cache.heads;
        if (r.of_v) r.head -= a.cache.heads;
        r.slot = of_q ? 0 : a.slots[r.token];
        if (columns) {
            r.e[0] = r.e[1] = Eight{};
            const uint32_t of = pass * (per_pass / kRun) + column_head, head = head0 + of;
            if (of < heads && column < dim) {
                const bool of_v = !of_q && head >= a.cache.heads;
                const ecs::View &v = of_q ? a.q : of_v ? a.v : a.k;
                load_column(v.data + first + (int64_t)(of_v ? head - a.cache.heads : head) * v.head_stride + (int64_t)column * v.dim_stride, run, r.e);
            }
            return r;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            r.e[k] = Eight{};
            if (r.inside && at[k] < dim)
                r.e[k] = ecs::load_eight(of_q ? a.q : r.of_v ? a.v : a.k, of_q ? a.q_wide : r.of_v ? a.v_wide : a.k_wide, r.token, r.head, at[k]);
        }
        return r;
    };
    Rows next = ask(0);

    if (of_q || head0 < a.cache.heads) {                                  // (values alone need no turns)
        for (uint32_t i = tid; i < run * pairs; i += kThreads) {
            const uint32_t t = i / pairs, p = i - t * pairs;
            float c, s;
            turn((double)a.position[first + t] * a.frequency[p] * 0.15915494309189533577, c, s);
            turns[(2u * t) * pad + p] = c;
            turns[(2u * t + 1u) * pad + p] = s;
        }
    }
    __syncthreads();

    for (uint32_t pass = 0; pass * per_pass < rows; ++pass) {
        Rows r = next;
        if (columns) {
            __syncthreads();                                              // (what the last pass left has been read)
#pragma unroll
            for (uint32_t i = 0; i < kRun; ++i) *reinterpret_cast<uint16_t *>(tile_column + i * tile_step) = (uint16_t)r.e[i / 8].get(i % 8);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 w = at[k] < dim ? *reinterpret_cast<const uint4 *>(tile + (tid >> a.lanes_shift) * tile_step + 2u * at[k]) : uint4{};
                r.e[k] = Eight{{w.x, w.y, w.z, w.w}};
            }
        }
        if ((pass + 1u) * per_pass < rows) next = ask(pass + 1u);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = to_float(r.e[i / 8].get(i % 8));
        const float *cosine = turns + 2u * (r.token - first) * pad, *sine = cosine + pad;
        if constexpr (PAIRS == kAnywhere) {                               // partners in any lane of the row: through LDS
#pragma unroll
            for (int k = 0; k < 2; ++k) rows_lds[2u * tid + k] = make_uint4(r.e[k].w[0], r.e[k].w[1], r.e[k].w[2], r.e[k].w[3]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const uint16_t *row = reinterpret_cast<const uint16_t *>(rows_lds + 2u * (tid - lane));
            if (!r.of_v) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t d = 16u * lane + i;
                    if (d < 2u * pairs) {
                        const bool upper = d >= pairs;
                        const uint32_t pair = upper ? d - pairs : d;
                        x[i] = turned(x[i], cosine[pair], to_float(row[upper ? pair : d + pairs]), upper ? sine[pair] : -sine[pair]);
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();                              // (the next pass writes there)
        } else if (!r.of_v && pair0 < pairs) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t p = pair0 + i;
                if (PAIRS == kNeighbours && p >= pairs) break;
                const int u = PAIRS == kNeighbours ? 2 * i : i, v = PAIRS == kNeighbours ? 2 * i + 1 : i + 8;
                const float c = cosine[p], s = sine[p], y = x[u];
                x[u] = turned(y, c, x[v], -s);
                x[v] = turned(y, s, x[v], c);
            }
        }
        const uint64_t places = (uint64_t)a.cache.pages << a.cache.page_shift;
        const bool valid = r.inside && !of_q && (uint64_t)r.slot < places;
        const uint64_t page = (uint64_t)r.slot >> a.cache.page_shift, off = (uint64_t)r.slot & ((1u << a.cache.page_shift) - 1u);
        const uint64_t place = ((page * a.cache.heads + r.head) << a.cache.page_shift) + off;
        uint8_t *codes = (r.of_v ? a.cache.v : a.cache.k) + place * a.cache.row_bytes;
        if (BITS == 16 || of_q) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                Eight e;
#pragma unroll
                for (int i = 0; i < 4; ++i) e.w[i] = to_half(x[8 * k + 2 * i]) | to_half(x[8 * k + 2 * i + 1]) << 16;
                if (r.of_v) e = r.e[k];                                   // (bit for bit, NaN too)
                if (at[k] < dim) {
                    if (columns_out)
                        *reinterpret_cast<uint4 *>(tile + (tid >> a.lanes_shift) * tile_step + 2u * at[k]) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
                    else if (of_q && r.inside)
                        ecs::store_eight(a.q_out, a.q_out_wide, r.token, r.head, at[k], e);
                    if (valid) *reinterpret_cast<uint4 *>(codes + 2u * at[k]) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
                }
            }
        }
        if (columns_out) {
            __syncthreads();
            const uint32_t of = pass * (per_pass / kRun) + column_head;
            uint32_t w[kRun / 2];
#pragma unroll
            for (uint32_t i = 0; i < kRun; ++i) {
                const uint32_t h = *reinterpret_cast<const uint16_t *>(tile_column + i * tile_step);
                w[i / 2] = (i & 1) ? w[i / 2] | h << 16 : h;
            }
            if (of < heads && column < dim)
                store_column(a.q_out.data + first + (int64_t)(head0 + of) * a.q_out.head_stride + (int64_t)column * a.q_out.dim_stride, run, w);
        }
        if constexpr (BITS < 16)
            if (!of_q)
                ecs::store_codes<BITS, true>(x, codes, (r.of_v ? a.cache.v_step : a.cache.k_step) + 4u * place, at, dim, a.lanes_shift, valid, !r.of_v && pairs != 0u);
    }
}

template <int BITS, bool COLUMNS>
int launch_pairs(const AppendArgs &a, uint32_t gx, uint32_t gy, uint32_t lds, void *stream)
{
    if (a.neighbours) return ecs::launch_args<kv_append_kernel<BITS, kNeighbours, COLUMNS>>(a, gx, gy, 1, kThreads, stream, lds);
    if (a.pairs % 8u == 0) return ecs::launch_args<kv_append_kernel<BITS, kHalves, COLUMNS>>(a, gx, gy, 1, kThreads, stream, lds);
    return ecs::launch_args<kv_append_kernel<BITS, kAnywhere, COLUMNS>>(a, gx, gy, 1, kThreads, stream, lds);
}
template <int BITS>
int launch_columns(const AppendArgs &a, uint32_t gx, uint32_t gy, uint32_t lds, void *stream)
{
    return a.q_columns || a.kv_columns ? launch_pairs<BITS, true>(a, gx, gy, lds, stream) : launch_pairs<BITS, false>(a, gx, gy, lds, stream);
}

}  // namespace

namespace ecs {

int launch_kv_append(AppendArgs &a, void *stream)
{
    a.lanes_shift = a.cache.dim <= 16u ? 0u : a.cache.dim <= 32u ? 1u : a.cache.dim <= 64u ? 2u : a.cache.dim <= 128u ? 3u : 4u;
    const uint32_t run = 1u << a.run_shift, runs = (a.tokens + run - 1u) / run, heads = a.q_heads + 2u * a.cache.heads;
    const uint32_t a_pass = std::max(1u, (kThreads >> a.lanes_shift) / run);
    auto in_columns = [&](const View &v, uint32_t wide) {
        return run == kRun && !wide && v.token_stride == 1 && v.head_stride % 8 == 0 && v.dim_stride % 8 == 0 && (uintptr_t)v.data % 16u == 0;
    };
    if (a.q_heads == 0) a.q_wide = 1u;                                    // (no queries: as good as rows)
    a.q_columns = a.q_heads && in_columns(a.q, a.q_wide);
    a.q_out_columns = a.q_heads && in_columns(a.q_out, a.q_out_wide);
    a.kv_columns = in_columns(a.k, a.k_wide) && in_columns(a.v, a.v_wide);
    // (in columns four runs share a line, and have to be at the same heads to share it in a die's cache: 8184 tokens, 64/8 heads of 128, 16 bits, with
    // up to 32 heads 145.7 us, 16 118.5, 8 108.3, 4 114.3, 2 134.6; 8191 of them 174, 166, 158, 158)
    const uint32_t most_heads = a.q_wide && a.k_wide && a.v_wide ? heads : 8u;
    // Some more workgroups than the chip holds at once, each with as many heads as that leaves it (8191 tokens, 64/8 heads, 16 bits: from 512 on 99.7 us,
    // 768 91.9, 1024 78.5, 1280 77.5, 2048 82.3, 8192 97.6)
    a.heads_per_block = std::max({a_pass, heads / 32768u + 1u, (uint32_t)std::min<uint64_t>(most_heads, (uint64_t)runs * heads / 1280u)});
    a.q_blocks = (a.q_heads + a.heads_per_block - 1u) / a.heads_per_block;
    const uint32_t gy = a.q_blocks + (2u * a.cache.heads + a.heads_per_block - 1u) / a.heads_per_block;
    // a pass has 256 >> lanes_shift rows
    const uint32_t tile = a.q_columns || a.kv_columns ? (kThreads >> a.lanes_shift) * ((32u << a.lanes_shift) + 16u) : 0u;
    const uint32_t lds = 2u * run * ((a.pairs + 3u) & ~3u) * (uint32_t)sizeof(float) + tile;
    return a.cache.bits == 16u ? launch_columns<16>(a, runs, gy, lds, stream)
           : a.cache.bits == 8u ? launch_columns<8>(a, runs, gy, lds, stream)
                                : launch_columns<4>(a, runs, gy, lds, stream);
}

}  // namespace ecs
