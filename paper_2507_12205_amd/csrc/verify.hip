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
#include "verify_tiles.h"

namespace {

using ecs::VerifyArgs;
using ecs::float4u;
using ecs::kThreads;
using ecs::kTile;
using ecs::tile_sum;

constexpr uint32_t kTilesPerBlock = 8;

struct Weights {
    const float *p, *q;       // q: null where nothing is taken off
    uint32_t skip, vocab;     // skip: a draft without probabilities of its own, which was certain of this token
    __device__ __forceinline__ double weight(uint32_t v, float a, float b) const
    {
        const double w = (double)a - (double)b;
        return w > 0.0 && v != skip ? w : 0.0;                              // (NaN counts as 0)
    }
    __device__ __forceinline__ void tile(uint32_t t, uint32_t lane, double (&w)[4][4]) const
    {
        float4u a[4], b[4] = {};
        ecs::load_tile(p, vocab, t, lane, a);
        if (q) ecs::load_tile(q, vocab, t, lane, b);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[k][i] = weight(t * kTile + 4u * lane + 256u * k + i, a[k][i], b[k][i]);
    }
    __device__ __forceinline__ bool reduced() const { return q || skip != 0xFFFFFFFFu; }
    __device__ __forceinline__ void restore()
    {
        q = nullptr;
        skip = 0xFFFFFFFFu;
    }
};

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
    __shared__ ecs::Drawing shared;
    const uint32_t seq = blockIdx.x, tid = threadIdx.x;
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    const double *sums = a.sums + (size_t)seq * (tiles + 1u);
    const uint32_t count = drafts_of(a, seq), n = min((uint32_t)sums[tiles], count);
    const double u = (double)a.uniform[(size_t)seq * (a.drafts + 1u) + a.drafts];
    Weights w = weights_of(a, seq, n, count);
    const int32_t token = ecs::draw_token(w, sums, u, a.vocab, shared);
    const int32_t *x = a.drafted + (size_t)seq * a.drafts;
    int32_t *out = a.tokens + (size_t)seq * (a.drafts + 1u);
    for (uint32_t i = tid; i <= a.drafts; i += kThreads) out[i] = i < n ? x[i] : i == n ? token : -1;
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
