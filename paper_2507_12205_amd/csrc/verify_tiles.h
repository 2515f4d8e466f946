// Drawing a token from weights over a vocabulary: the first one whose running sum passes a bound.  Tiles of 1024 neighbouring tokens are added
// up by many workgroups; one workgroup then finds the tile, and in it the token, from running sums.  Everything is in 64 bits: the answer is a
// whole number, and sums in 32 bits would give another token for another order of additions (at 32000 tokens about one in thirty).
#ifndef ECSPMV_VERIFY_TILES_H
#define ECSPMV_VERIFY_TILES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ecs {

constexpr uint32_t kThreads = 256, kTile = 1024, kMaxTiles = 1024;           // up to 2^20 tokens
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));      // rows start where they start

// A lane's values of a row in a tile: [k][i] is token 1024 tile + 256 k + 4 lane + i, zero beyond the vocabulary
__device__ __forceinline__ void load_tile(const float *p, uint32_t vocab, uint32_t tile, uint32_t lane, float4u (&a)[4])
{
    const uint32_t first = tile * kTile + 4u * lane;
    const bool whole = (tile + 1u) * kTile <= vocab;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t v = first + 256u * k;
        a[k] = float4u{0, 0, 0, 0};
        if (whole || v + 4u <= vocab) {
            a[k] = *reinterpret_cast<const float4u *>(p + v);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (v + i < vocab) a[k][i] = p[v + i];
        }
    }
}

__device__ __forceinline__ double wave_incl_scan(double v, uint32_t lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(v, o, 64);
        if (lane >= (uint32_t)o) v += t;
    }
    return v;
}

// W::tile gives a lane its weights of a tile, as load_tile orders them
template <class W>
__device__ __forceinline__ double tile_sum(const W &w, uint32_t tile, uint32_t lane)
{
    double v[4][4], s = 0.0;
    w.tile(tile, lane, v);
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) s += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    return s;
}

struct Drawing {
    double sum[kMaxTiles], wave_total[kThreads / 64], before;
    uint32_t found_tile, last_tile, token_id;
};

// The first token whose running sum passes u times the sum of all weights, in every thread of the workgroup; -1 where no weight is above zero.
// `sums`: the tiles' sums; W::reduced: whether something was taken off the weights, W::restore: without it, for where that leaves nothing.
template <class W>
__device__ __forceinline__ int32_t draw_token(W &w, const double *sums, double u, uint32_t vocab, Drawing &s)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, tiles = (vocab + kTile - 1u) / kTile;
    for (uint32_t t = tid; t < tiles; t += kThreads) s.sum[t] = sums[t];
    double total = 0.0;
    for (int attempt = 0; attempt < 2; ++attempt) {                         // twice only where what was taken off leaves nothing
        if (tid == 0) s.found_tile = 0xFFFFFFFFu, s.last_tile = 0;
        __syncthreads();
        // running sums over the tiles: every thread takes neighbouring ones
        const uint32_t per = (tiles + kThreads - 1u) / kThreads, t0 = min(tid * per, tiles), t1 = min(t0 + per, tiles);
        double mine = 0.0;
        for (uint32_t t = t0; t < t1; ++t) mine += s.sum[t];
        const double run = wave_incl_scan(mine, lane);
        if (lane == 63u) s.wave_total[wave] = run;
        __syncthreads();
        double off = 0.0;
        total = 0.0;
        for (uint32_t k = 0; k < kThreads / 64u; ++k) {
            if (k < wave) off += s.wave_total[k];
            total += s.wave_total[k];
        }
        if (total > 0.0) {
            const double bound = u * total, start = off + (run - mine);
            double c = start;
            uint32_t hit = 0xFFFFFFFFu, last = 0xFFFFFFFFu;
            for (uint32_t t = t0; t < t1; ++t) {
                c += s.sum[t];
                if (s.sum[t] > 0.0) {
                    last = t;
                    if (hit == 0xFFFFFFFFu && c > bound) hit = t;
                }
            }
            if (hit != 0xFFFFFFFFu) atomicMin(&s.found_tile, hit);
            if (last != 0xFFFFFFFFu) atomicMax(&s.last_tile, last);
            __syncthreads();
            const uint32_t tile = s.found_tile != 0xFFFFFFFFu ? s.found_tile : s.last_tile;
            if (tile >= t0 && tile < t1) {
                double b = start;
                for (uint32_t t = t0; t < tile; ++t) b += s.sum[t];
                s.before = b;
            }
            __syncthreads();
            if (wave == 0) {
                double v[4][4], four[4], sums_to[4], done = s.before;             // 256 tokens after another
                w.tile(tile, lane, v);
                uint32_t token = 0xFFFFFFFFu, some = 0;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) sums_to[k] = four[k] = (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
#pragma unroll
                for (int o = 1; o < 64; o <<= 1)                             // the four scans side by side
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        const double t = __shfl_up(sums_to[k], o, 64);
                        if (lane >= (uint32_t)o) sums_to[k] += t;
                    }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    double cum = done + (sums_to[k] - four[k]);
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        cum += v[k][i];
                        const uint32_t id = tile * kTile + 256u * k + 4u * lane + i;
                        if (v[k][i] > 0.0) some = id + 1u;
                        if (token == 0xFFFFFFFFu && cum > bound && v[k][i] > 0.0) token = id;
                    }
                    done += __shfl(sums_to[k], 63, 64);
                }
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) {
                    token = min(token, (uint32_t)__shfl_xor((int)token, o, 64));
                    some = max(some, (uint32_t)__shfl_xor((int)some, o, 64));
                }
                if (lane == 0) s.token_id = token != 0xFFFFFFFFu ? token : some - 1u;
            }
            __syncthreads();
            break;
        }
        if (!w.reduced()) break;
        w.restore();
        for (uint32_t t = wave; t < tiles; t += kThreads / 64u) {
            const double added = tile_sum(w, t, lane);
            if (lane == 0) s.sum[t] = added;
        }
        __syncthreads();                                                    // (and s.wave_total has been read)
    }
    return total > 0.0 ? (int32_t)s.token_id : -1;
}

}  // namespace ecs
#endif
