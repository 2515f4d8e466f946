// New tokens into the paged cache with their positions in them: keys (and queries) are rotated, pair by pair of their first values,
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * frequency of the pair,
// keys and values become codes and go to their places, queries go to where the caller wants them.  One launch.
//
// A row is what one token has in one head of q, k or v; as in kv_cache.hip a lane has eight neighbouring values of it.  A workgroup takes
// up to 16 neighbouring tokens and some heads of them: the turns of these tokens are worked out once, by all of its threads, and lie in
// LDS for all of its rows.  An angle is a product in 64 bits (of position 10^6, 32 bits would leave 0.03 of an angle), and so are its cosine and
// sine, which are then rounded to 32; the rotated values stay in 32 bits until they are rounded once, to FP16 or to a code.  The two products of
// a pair are rounded each: a code next to its border is then the one that a program gets which rotates in FP32 operations of its own.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <algorithm>

#include "kernel_handle.h"
#include "kv_rows.h"
#include "serve.h"

namespace {

using ecs::AppendArgs;
using ecs::Eight;
using ecs::View;
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

template <int BITS>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a)
{
    extern __shared__ float turns[];                                      // [token of the run][cos, sin][pair]
    const uint32_t tid = threadIdx.x, first = blockIdx.x << a.run_shift, run = min(1u << a.run_shift, a.tokens - first);
    const uint32_t heads = a.q_heads + 2u * a.cache.heads, head0 = blockIdx.y * a.heads_per_block, head1 = min(head0 + a.heads_per_block, heads);
    const uint32_t lane = tid & ((1u << a.lanes_shift) - 1u), at = 8u * lane, dim = a.cache.dim;
    const uint32_t per_pass = kThreads >> a.lanes_shift, rows = (head1 - head0) << a.run_shift;
    const uint32_t pairs = a.pairs, pad = (pairs + 3u) & ~3u;

    struct Rows {
        uint32_t head, token, kind;                                       // kind: 0 q, 1 k, 2 v
        bool inside;
        int64_t slot;
        Eight e;
    };
    auto ask = [&](uint32_t pass) {                                       // sends the loads of this lane's row of a pass off
        Rows r;
        const uint32_t i = pass * per_pass + (tid >> a.lanes_shift), in_run = i & ((1u << a.run_shift) - 1u);
        r.head = head0 + (i >> a.run_shift);
        r.inside = i < rows && in_run < run && at < dim;
        r.token = first + min(in_run, run - 1u);
        r.kind = r.head < a.q_heads ? 0u : r.head < a.q_heads + a.cache.heads ? 1u : 2u;
        r.head -= r.kind == 0u ? 0u : r.kind == 1u ? a.q_heads : a.q_heads + a.cache.heads;
        r.slot = a.slots[r.token];
        r.e = Eight{};
        if (r.inside) r.e = ecs::load_eight(r.kind == 0u ? a.q : r.kind == 1u ? a.k : a.v, r.kind == 0u ? a.q_wide : r.kind == 1u ? a.k_wide : a.v_wide,
                                            r.token, r.head, at);
        return r;
    };
    Rows next = ask(0);

    if (head0 < a.q_heads + a.cache.heads) {                              // (values alone need no turns)
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
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_float(r.e.get(i));
        const float *cosine = turns + 2u * (r.token - first) * pad, *sine = cosine + pad;
        if (a.neighbours) {
            if (r.kind < 2u) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t p = at / 2u + i;
                    if (p < pairs) {
                        const float c = cosine[p], s = sine[p], u = x[2 * i], v = x[2 * i + 1];
                        x[2 * i] = turned(u, c, v, -s);
                        x[2 * i + 1] = turned(u, s, v, c);
                    }
                }
            }
        } else if ((pairs & 7u) == 0u) {                                  // a lane's values have their partners in one other lane
            const bool upper = at >= pairs;
            const uint32_t from = upper ? lane - pairs / 8u : lane + pairs / 8u;
            const int source = (int)((tid & 63u) - lane + (at < 2u * pairs ? from : lane));
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__shfl((int)r.e.w[i], source, 64);
            if (r.kind < 2u && at < 2u * pairs) {
                const uint32_t p = upper ? at - pairs : at;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = cosine[p + i], s = upper ? sine[p + i] : -sine[p + i];
                    x[i] = turned(x[i], c, to_float((i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu), s);
                }
            }
        } else if (r.kind < 2u && r.inside) {                             // partners anywhere: read where they lie (before anything is written)
            const View &from = r.kind == 0u ? a.q : a.k;
            const uint16_t *p = from.data + (int64_t)r.token * from.token_stride + (int64_t)r.head * from.head_stride;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t d = at + i;
                if (d < 2u * pairs) {
                    const bool upper = d >= pairs;
                    const uint32_t pair = upper ? d - pairs : d;
                    const float c = cosine[pair], s = upper ? sine[pair] : -sine[pair];
                    x[i] = turned(x[i], c, to_float(p[(int64_t)(upper ? pair : d + pairs) * from.dim_stride]), s);
                }
            }
        }
        const uint64_t places = (uint64_t)a.cache.pages << a.cache.page_shift;
        const bool valid = r.inside && r.kind != 0u && (uint64_t)r.slot < places;
        const uint64_t page = (uint64_t)r.slot >> a.cache.page_shift, off = (uint64_t)r.slot & ((1u << a.cache.page_shift) - 1u);
        const uint64_t place = ((page * a.cache.heads + r.head) << a.cache.page_shift) + off;
        if (BITS == 16 || r.kind == 0u) {
            Eight e;
#pragma unroll
            for (int i = 0; i < 4; ++i) e.w[i] = to_half(x[2 * i]) | to_half(x[2 * i + 1]) << 16;
            if (r.kind == 2u) e = r.e;                                    // (bit for bit, NaN too)
            if (r.kind == 0u) {
                if (r.inside) ecs::store_eight(a.q_out, a.q_out_wide, r.token, r.head, at, e);
            } else if (valid) {
                *reinterpret_cast<uint4 *>((r.kind == 1u ? a.cache.k : a.cache.v) + place * a.cache.row_bytes + 2u * at) =
                    make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
            }
        }
        if constexpr (BITS < 16)
            if (r.kind != 0u)                                             // (a row's lanes are of one kind)
                ecs::store_codes<BITS, true>(x, (r.kind == 1u ? a.cache.k : a.cache.v) + place * a.cache.row_bytes,
                                       (r.kind == 1u ? a.cache.k_step : a.cache.v_step) + 4u * place, at, dim, a.lanes_shift, valid);
    }
}

}  // namespace

namespace ecs {

static uint32_t append_lds_bytes(uint32_t run_shift, uint32_t pairs) { return (2u << run_shift) * ((pairs + 3u) & ~3u) * (uint32_t)sizeof(float); }

int launch_kv_append(AppendArgs &a, void *stream)
{
    const uint32_t runs = (a.tokens + (1u << a.run_shift) - 1u) >> a.run_shift, heads = a.q_heads + 2u * a.cache.heads;
    const uint32_t a_pass = std::max(1u, kThreads >> a.lanes_shift >> a.run_shift);
    a.heads_per_block = std::max({a_pass, heads / 65535u + 1u, (uint32_t)std::min<uint64_t>(heads, (uint64_t)runs * heads / 4096u)});
    const uint32_t gy = (heads + a.heads_per_block - 1u) / a.heads_per_block;
    const uint32_t lds = append_lds_bytes(a.run_shift, a.pairs);
    switch (a.cache.bits) {
    case 16: return launch_args<kv_append_kernel<16>>(a, runs, gy, 1, kThreads, stream, lds);
    case 8: return launch_args<kv_append_kernel<8>>(a, runs, gy, 1, kThreads, stream, lds);
    default: return launch_args<kv_append_kernel<4>>(a, runs, gy, 1, kThreads, stream, lds);
    }
}

}  // namespace ecs
