// The check of drafted tokens: which are accepted, and the token that follows them.
//
// Draft i is accepted while u_i * q_i(x_i) < p_i(x_i).  With n accepted, the next token is drawn from w = max(p_n - q_n, 0) after a
// refusal and from w = p_n where every draft was accepted: it is the first v whose running sum w_0 + ... + w_v passes u * sum(w).
// Differences and sums are in 64 bits: the answer is a whole number, and sums in 32 bits would give another token for another order
// of additions (at 32000 tokens about one in thirty).
//
// Two launches.  The first adds up tiles of 1024 neighbouring tokens of the one row of p and q that counts, eight tiles to a workgroup,
// eight 128-bit loads of each lane on their way; the second finds the tile and then the token from running sums.  What bounds it are the
// trips to memory, one after the other: count, drafts, their probabilities, the row; sums, the tile.  1 sequence over 32000 tokens 11.0 us,
// 32 over 128256 17 us (33 MB).  One workgroup for each sequence and one launch (a compute unit by itself brings some 35 GB/s) took 11.2
// and 31.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "serve.h"

namespace {

using ecs::VerifyArgs;

constexpr uint32_t kThreads = 256, kTile = 1024, kMaxTiles = 1024;           // up to 2^20 tokens
constexpr uint32_t kTilesPerBlock = 8;

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));      // rows start where they start

struct Weights {
    const float *p, *q;       // q: null where nothing is taken off
    uint32_t skip, vocab;     // skip: a draft without probabilities of its own, which was certain of this token
    __device__ __forceinline__ double weight(uint32_t v, float a, float b) const
    {
        const double w = (double)a - (double)b;
        return w > 0.0 && v != skip ? w : 0.0;                              // (NaN counts as 0)
    }
    // the weights of this lane in a tile: [k][i] is token 1024 tile + 256 k + 4 lane + i
    __device__ __forceinline__ void tile(uint32_t t, uint32_t lane, double (&w)[4][4]) const
    {
        float4u a[4], b[4];
        const uint32_t first = t * kTile + 4u * lane;
        const bool whole = (t + 1u) * kTile <= vocab;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t v = first + 256u * k;
            a[k] = b[k] = float4u{0, 0, 0, 0};
            if (whole || v + 4u <= vocab) {
                a[k] = *reinterpret_cast<const float4u *>(p + v);
                if (q) b[k] = *reinterpret_cast<const float4u *>(q + v);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (v + i < vocab) {
                        a[k][i] = p[v + i];
                        if (q) b[k][i] = q[v + i];
                    }
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[k][i] = weight(first + 256u * k + i, a[k][i], b[k][i]);
    }
};

__device__ __forceinline__ double wave_incl_scan(double v, uint32_t lane)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(v, o, 64);
        if (lane >= (uint32_t)o) v += t;
    }
    return v;
}

// How many drafts of a sequence stand, in every thread; `shared`: a word of LDS
__device__ __forceinline__ uint32_t accepted_drafts(const VerifyArgs &a, uint32_t seq, uint32_t count, uint32_t *shared)
{
    const float *p = a.target + seq * a.target_seq, *q = a.draft ? a.draft + seq * a.draft_seq : nullptr;
    const int32_t *x = a.drafted + (size_t)seq * a.drafts;
    const float *u = a.uniform + (size_t)seq * (a.drafts + 1u);
    if (threadIdx.x == 0) *shared = count;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) {
        const int32_t t = x[i];
        bool ok = false;                                                    // a token that is none is refused
        if (t >= 0 && (uint32_t)t < a.vocab) {
            const float pt = p[i * a.target_row + t], qt = q ? q[i * a.draft_row + t] : 1.0f;
            ok = u[i] * qt < pt;
        }
        if (!ok) atomicMin(shared, i);
    }
    __syncthreads();
    return *shared;
}

__device__ __forceinline__ uint32_t drafts_of(const VerifyArgs &a, uint32_t seq)
{
    return a.count ? (uint32_t)min(max(a.count[seq], 0), (int32_t)a.drafts) : a.drafts;
}

__device__ __forceinline__ Weights weights_of(const VerifyArgs &a, uint32_t seq, uint32_t n, uint32_t count)
{
    const bool refused = n < count;
    return {a.target + seq * a.target_seq + n * a.target_row, refused && a.draft ? a.draft + seq * a.draft_seq + n * a.draft_row : nullptr,
            refused && !a.draft ? (uint32_t)a.drafted[(size_t)seq * a.drafts + n] : 0xFFFFFFFFu, a.vocab};
}

__device__ __forceinline__ double tile_sum(const Weights &w, uint32_t tile, uint32_t lane)
{
    double v[4][4], s = 0.0;
    w.tile(tile, lane, v);
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) s += (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    return s;
}

// sums[seq][tiles + 1]: the tiles' sums, then the number of accepted drafts
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(const VerifyArgs a)
{
    __shared__ uint32_t shared;
    const uint32_t seq = blockIdx.y, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t count = drafts_of(a, seq), n = accepted_drafts(a, seq, count, &shared);
    const Weights w = weights_of(a, seq, n, count);
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    double *sums = a.sums + (size_t)seq * (tiles + 1u);
#pragma unroll
    for (uint32_t k = 0; k < kTilesPerBlock / (kThreads / 64u); ++k) {
        const uint32_t t = blockIdx.x * kTilesPerBlock + k * (kThreads / 64u) + wave;
        if (t >= tiles) break;
        const double s = tile_sum(w, t, lane);
        if (lane == 0) sums[t] = s;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) sums[tiles] = (double)n;
}

__global__ __launch_bounds__(kThreads) void verify_token_kernel(const VerifyArgs a)
{
    __shared__ double sum[kMaxTiles], wave_total[kThreads / 64], before;
    __shared__ uint32_t found_tile, last_tile, token_id;
    const uint32_t seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    const double *sums = a.sums + (size_t)seq * (tiles + 1u);
    const uint32_t count = drafts_of(a, seq), n = min((uint32_t)sums[tiles], count);
    const double u = (double)a.uniform[(size_t)seq * (a.drafts + 1u) + a.drafts];
    for (uint32_t t = tid; t < tiles; t += kThreads) sum[t] = sums[t];
    Weights w = weights_of(a, seq, n, count);
    double total = 0.0;
    for (int attempt = 0; attempt < 2; ++attempt) {                         // twice only where p - q leaves nothing: then from p
        if (tid == 0) found_tile = 0xFFFFFFFFu, last_tile = 0;
        __syncthreads();
        // running sums over the tiles: every thread takes neighbouring ones
        const uint32_t per = (tiles + kThreads - 1u) / kThreads, t0 = min(tid * per, tiles), t1 = min(t0 + per, tiles);
        double mine = 0.0;
        for (uint32_t t = t0; t < t1; ++t) mine += sum[t];
        const double run = wave_incl_scan(mine, lane);
        if (lane == 63u) wave_total[wave] = run;
        __syncthreads();
        double off = 0.0;
        total = 0.0;
        for (uint32_t k = 0; k < kThreads / 64u; ++k) {
            if (k < wave) off += wave_total[k];
            total += wave_total[k];
        }
        if (total > 0.0) {
            const double bound = u * total, start = off + (run - mine);
            double c = start;
            uint32_t hit = 0xFFFFFFFFu, last = 0xFFFFFFFFu;
            for (uint32_t t = t0; t < t1; ++t) {
                c += sum[t];
                if (sum[t] > 0.0) {
                    last = t;
                    if (hit == 0xFFFFFFFFu && c > bound) hit = t;
                }
            }
            if (hit != 0xFFFFFFFFu) atomicMin(&found_tile, hit);
            if (last != 0xFFFFFFFFu) atomicMax(&last_tile, last);
            __syncthreads();
            const uint32_t tile = found_tile != 0xFFFFFFFFu ? found_tile : last_tile;
            if (tile >= t0 && tile < t1) {
                double b = start;
                for (uint32_t t = t0; t < tile; ++t) b += sum[t];
                before = b;
            }
            __syncthreads();
            if (wave == 0) {
                double v[4][4], s[4], sums_to[4], done = before;             // 256 tokens after another
                w.tile(tile, lane, v);
                uint32_t token = 0xFFFFFFFFu, some = 0;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) sums_to[k] = s[k] = (v[k][0] + v[k][1]) + (v[k][2] + v[k][3]);
#pragma unroll
                for (int o = 1; o < 64; o <<= 1)                             // the four scans side by side
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        const double t = __shfl_up(sums_to[k], o, 64);
                        if (lane >= (uint32_t)o) sums_to[k] += t;
                    }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    double cum = done + (sums_to[k] - s[k]);
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
                if (lane == 0) token_id = token != 0xFFFFFFFFu ? token : some - 1u;
            }
            __syncthreads();
            break;
        }
        if (!w.q && w.skip == 0xFFFFFFFFu) break;
        w.q = nullptr;
        w.skip = 0xFFFFFFFFu;
        for (uint32_t t = wave; t < tiles; t += kThreads / 64u) {
            const double s = tile_sum(w, t, lane);
            if (lane == 0) sum[t] = s;
        }
        __syncthreads();                                                    // (and wave_total has been read)
    }
    const int32_t *x = a.drafted + (size_t)seq * a.drafts;
    int32_t *out = a.tokens + (size_t)seq * (a.drafts + 1u);
    for (uint32_t i = tid; i <= a.drafts; i += kThreads) out[i] = i < n ? x[i] : i == n && total > 0.0 ? (int32_t)token_id : -1;
    if (tid == 0) a.accepted[seq] = (int32_t)n;
}

}  // namespace

namespace ecs {

uint64_t verify_work_bytes(uint32_t batch, uint32_t vocab) { return (uint64_t)batch * ((vocab + kTile - 1u) / kTile + 1u) * sizeof(double); }

int launch_verify(const VerifyArgs &a, uint32_t batch, void *stream)
{
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    const int e = launch_args<verify_sums_kernel>(a, (tiles + kTilesPerBlock - 1u) / kTilesPerBlock, batch, 1, kThreads, stream);
    return e ? e : launch_args<verify_token_kernel>(a, batch, 1, 1, kThreads, stream);
}

}  // namespace ecs
