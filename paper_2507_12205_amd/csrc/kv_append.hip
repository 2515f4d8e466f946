// New tokens into the paged cache with their positions in them: keys (and queries) are rotated, pair by pair of their first values,
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair,
// keys and values become codes and go to their places, queries go to where the caller wants them.  One launch.
//
// A row is what one token has in one head of q, k or v.  A lane has 16 values of it, two pieces of eight: both halves of eight pairs, or 16
// neighbouring values, so that nothing is exchanged between lanes but a row's least and largest value.  A workgroup takes up to 16
// neighbouring tokens and some heads of them, in q the heads of a token after one another, as they lie, in k and v (and in q that lies as columns)
// the tokens of a head, as they come to lie in the cache.  The turns of these tokens are worked out once, by all of its threads, and lie in LDS for all of
// its rows.  What bounds it is memory: 8191 tokens, 64/8 heads of 128, 16 bits 77 us, 336 MB at 4.3 TB/s, 8 bits 81, 4 bits 79 (eight values a lane
// with their partners' from another lane, q in the order of k and v: 95, 99, 99); 8 tokens, 12/12 heads of 64 as columns, 4.0.
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

constexpr uint32_t kThreads = 256;

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
// workgroup) one after another: 8191 tokens, 64/8 heads of 128 in columns, 16 bits 240 us without, 176 with
__device__ __forceinline__ uint32_t run_of(uint32_t x, uint32_t n)
{
    const uint32_t die = x & 7u;
    return die * (n >> 3) + min(die, n & 7u) + (x >> 3);
}

// How the pairs of a head lie in a lane's pieces: halves of eight pairs, neighbours, or halves that begin anywhere (their partners are looked up)
enum { kHalves, kNeighbours, kAnywhere };

template <int BITS, int PAIRS>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a)
{
    extern __shared__ float turns[];                                      // [token of the run][cos, sin][pair]
    __shared__ uint4 rows_lds[PAIRS == kAnywhere ? 2 * kThreads : 1];     // two pieces of every lane
    const uint32_t tid = threadIdx.x, first = (a.q_wide && a.k_wide && a.v_wide ? blockIdx.x : run_of(blockIdx.x, gridDim.x)) << a.run_shift, run = min(1u << a.run_shift, a.tokens - first);
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
                    if (of_q && r.inside) ecs::store_eight(a.q_out, a.q_out_wide, r.token, r.head, at[k], e);
                    if (valid) *reinterpret_cast<uint4 *>(codes + 2u * at[k]) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
                }
            }
        }
        if constexpr (BITS < 16)
            if (!of_q)
                ecs::store_codes<BITS, true>(x, codes, (r.of_v ? a.cache.v_step : a.cache.k_step) + 4u * place, at, dim, a.lanes_shift, valid);
    }
}

template <int BITS>
int launch_pairs(const AppendArgs &a, uint32_t gx, uint32_t gy, uint32_t lds, void *stream)
{
    if (a.neighbours) return ecs::launch_args<kv_append_kernel<BITS, kNeighbours>>(a, gx, gy, 1, kThreads, stream, lds);
    if (a.pairs % 8u == 0) return ecs::launch_args<kv_append_kernel<BITS, kHalves>>(a, gx, gy, 1, kThreads, stream, lds);
    return ecs::launch_args<kv_append_kernel<BITS, kAnywhere>>(a, gx, gy, 1, kThreads, stream, lds);
}

}  // namespace

namespace ecs {

int launch_kv_append(AppendArgs &a, void *stream)
{
    a.lanes_shift = a.cache.dim <= 16u ? 0u : a.cache.dim <= 32u ? 1u : a.cache.dim <= 64u ? 2u : a.cache.dim <= 128u ? 3u : 4u;
    const uint32_t run = 1u << a.run_shift, runs = (a.tokens + run - 1u) / run, heads = a.q_heads + 2u * a.cache.heads;
    const uint32_t a_pass = std::max(1u, (kThreads >> a.lanes_shift) / run);
    // Some more workgroups than the chip holds at once, each with as many heads as that leaves it (8191 tokens, 64/8 heads, 16 bits: from 512 on 99.7 us,
    // 768 91.9, 1024 78.5, 1280 77.5, 2048 82.3, 8192 97.6)
    a.heads_per_block = std::max({a_pass, heads / 32768u + 1u, (uint32_t)std::min<uint64_t>(heads, (uint64_t)runs * heads / 1280u)});
    a.q_blocks = (a.q_heads + a.heads_per_block - 1u) / a.heads_per_block;
    const uint32_t gy = a.q_blocks + (2u * a.cache.heads + a.heads_per_block - 1u) / a.heads_per_block;
    const uint32_t lds = 2u * run * ((a.pairs + 3u) & ~3u) * (uint32_t)sizeof(float);
    return a.cache.bits == 16u ? launch_pairs<16>(a, runs, gy, lds, stream)
           : a.cache.bits == 8u ? launch_pairs<8>(a, runs, gy, lds, stream)
                                : launch_pairs<4>(a, runs, gy, lds, stream);
}

}  // namespace ecs
