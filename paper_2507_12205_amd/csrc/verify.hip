// The check of drafted tokens: which are accepted, and the token that follows them.
//
// Draft i is accepted while u_i * q_i(x_i) < p_i(x_i).  With n accepted, the next token is drawn from w = max(p_n - q_n, 0) after a
// refusal and from w = p_n where every draft was accepted: it is the first v whose running sum w_0 + ... + w_v passes u * sum(w).
// Differences and sums are in 64 bits: the answer is a whole number, and sums in 32 bits would give another token for another order
// of additions (at 32000 tokens about one in thirty).
//
// One workgroup per sequence; each wavefront adds up tiles of 256 neighbouring tokens, whose sums stay in LDS; the tile and then the
// token are found from running sums.  One pass over one row of p and of q.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "serve.h"

namespace {

using ecs::VerifyArgs;

constexpr uint32_t kThreads = 1024, kTile = 256, kMaxTiles = 4096;          // up to 2^20 tokens

struct Weights {
    const float *p, *q;       // q: null where nothing is taken off
    uint32_t skip, vocab;     // skip: a draft without probabilities of its own, which was certain of this token
    __device__ __forceinline__ double get(uint32_t v) const
    {
        if (v >= vocab || v == skip) return 0.0;
        const double w = (double)p[v] - (q ? (double)q[v] : 0.0);
        return w > 0.0 ? w : 0.0;                                           // (NaN counts as 0)
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

__global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyArgs a)
{
    __shared__ double tile_sum[kMaxTiles];
    __shared__ double wave_total[kThreads / 64];
    __shared__ uint32_t refused, found_tile, last_token;
    __shared__ double before;
    const uint32_t seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t count = a.count ? (uint32_t)min(max(a.count[seq], 0), (int32_t)a.drafts) : a.drafts;
    const float *p = a.target + seq * a.target_seq, *q = a.draft ? a.draft + seq * a.draft_seq : nullptr;
    const int32_t *x = a.drafted + (size_t)seq * a.drafts;
    const float *u = a.uniform + (size_t)seq * (a.drafts + 1u);
    if (tid == 0) refused = count;
    __syncthreads();
    for (uint32_t i = tid; i < count; i += kThreads) {
        const int32_t t = x[i];
        bool ok = false;                                                    // a token that is none is refused
        if (t >= 0 && (uint32_t)t < a.vocab) {
            const float pt = p[i * a.target_row + t], qt = q ? q[i * a.draft_row + t] : 1.0f;
            ok = u[i] * qt < pt;
        }
        if (!ok) atomicMin(&refused, i);
    }
    __syncthreads();
    const uint32_t n = refused;
    Weights w = {p + n * a.target_row, n < count && q ? q + n * a.draft_row : nullptr, n < count && !q ? (uint32_t)x[n] : 0xFFFFFFFFu, a.vocab};
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    double total = 0.0;
    for (int attempt = 0; attempt < 2; ++attempt) {                         // twice only where p - q leaves nothing: then from p
        for (uint32_t t = wave; t < tiles; t += kThreads / 64u) {
            double s = 0.0;
#pragma unroll
            for (uint32_t k = 0; k < kTile / 64u; ++k) s += w.get(t * kTile + 64u * k + lane);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
            if (lane == 0) tile_sum[t] = s;
        }
        __syncthreads();
        // running sums over the tiles: every thread takes neighbouring ones
        const uint32_t per = (tiles + kThreads - 1u) / kThreads, t0 = min(tid * per, tiles), t1 = min(t0 + per, tiles);
        double mine = 0.0;
        for (uint32_t t = t0; t < t1; ++t) mine += tile_sum[t];
        double run = wave_incl_scan(mine, lane);
        if (lane == 63u) wave_total[wave] = run;
        if (tid == 0) found_tile = 0xFFFFFFFFu, last_token = 0;
        __syncthreads();
        double off = 0.0;
        total = 0.0;
        for (uint32_t k = 0; k < kThreads / 64u; ++k) {
            if (k < wave) off += wave_total[k];
            total += wave_total[k];
        }
        if (total > 0.0) {
            const double bound = (double)u[a.drafts] * total;
            double c = off + run - mine;
            uint32_t hit = 0xFFFFFFFFu, last = 0xFFFFFFFFu;
            for (uint32_t t = t0; t < t1; ++t) {
                const double next = c + tile_sum[t];
                if (tile_sum[t] > 0.0) last = t;
                if (hit == 0xFFFFFFFFu && tile_sum[t] > 0.0 && next > bound) hit = t;
                c = next;
            }
            if (hit != 0xFFFFFFFFu) atomicMin(&found_tile, hit);
            if (last != 0xFFFFFFFFu) atomicMax(&last_token, last);
            __syncthreads();
            const uint32_t tile = found_tile != 0xFFFFFFFFu ? found_tile : last_token;
            if (tile >= t0 && tile < t1) {
                double b = off + run - mine;
                for (uint32_t t = t0; t < tile; ++t) b += tile_sum[t];
                before = b;
            }
            __syncthreads();
            if (wave == 0) {
                double v[kTile / 64u], s = 0.0;                              // four neighbouring tokens per lane
#pragma unroll
                for (uint32_t k = 0; k < kTile / 64u; ++k) s += v[k] = w.get(tile * kTile + (kTile / 64u) * lane + k);
                double cum = before + wave_incl_scan(s, lane) - s;
                uint32_t token = 0xFFFFFFFFu, some = 0;
#pragma unroll
                for (uint32_t k = 0; k < kTile / 64u; ++k) {
                    cum += v[k];
                    const uint32_t id = tile * kTile + (kTile / 64u) * lane + k;
                    if (v[k] > 0.0) some = id + 1u;
                    if (token == 0xFFFFFFFFu && cum > bound && v[k] > 0.0) token = id;
                }
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) {
                    token = min(token, (uint32_t)__shfl_xor((int)token, o, 64));
                    some = max(some, (uint32_t)__shfl_xor((int)some, o, 64));
                }
                if (lane == 0) last_token = token != 0xFFFFFFFFu ? token : some - 1u;
            }
            __syncthreads();
            break;
        }
        if (!w.q && w.skip == 0xFFFFFFFFu) break;
        w.q = nullptr;
        w.skip = 0xFFFFFFFFu;
        __syncthreads();                                                    // tile_sum and wave_total have been read
    }
    int32_t *out = a.tokens + (size_t)seq * (a.drafts + 1u);
    for (uint32_t i = tid; i <= a.drafts; i += kThreads) out[i] = i < n ? x[i] : i == n && total > 0.0 ? (int32_t)last_token : -1;
    if (tid == 0) a.accepted[seq] = (int32_t)n;
}

}  // namespace

namespace ecs {

int launch_verify(const VerifyArgs &a, uint32_t batch, void *stream)
{
    return launch_args<verify_kernel>(a, batch, 1, 1, kThreads, stream);
}

}  // namespace ecs
