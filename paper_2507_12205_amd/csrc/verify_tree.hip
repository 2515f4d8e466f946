// The check of a tree of drafted tokens: which path of it is accepted, and the token that follows it.
//
// At a node (first the token before the tree) its children are asked in order.  A child x is accepted while u * S < p(x), where p are the
// target's probabilities after the node and S = 1 - (the p of the children that were refused): the probability that a token drawn from
// p is x, given that it is none of those.  With a child accepted the walk goes on there; without, the next token is drawn from p without the
// refused tokens.  So every token has the target's probability, however the tree was made.  S, sums and comparisons are in 64 bits.
//
// A child comes after its parent, so that one pass over the nodes in order is the whole walk: 64 nodes in the lanes of a wavefront, a ballot
// for the children of the node that it is at.  Everything that the walk needs of p is asked for at once, before it starts.
//
// Two launches, as for drafts in a row (verify.hip): the first adds up tiles of the row that counts, each workgroup after a walk of its
// own, one of which writes down in the workspace what came of it; the second draws the token and writes the outputs, which may so lie where
// the tree and its random numbers do: all walks have ended by then, and the second launch reads none of these.  What bounds it are the trips
// to memory, one after the other: the tree, its p, the row; the sums, the tile.  26 nodes over 32000 tokens 12.1 us, 32 sequences of up to 63
// over 128256 16.6 (with a second walk in the second launch instead of the first one's result 12.3 and 18.3).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernel_handle.h"
#include "serve.h"
#include "verify_tiles.h"

namespace {

using ecs::VerifyTreeArgs;
using ecs::float4u;
using ecs::kThreads;
using ecs::kTile;
using ecs::kMostNodes;

constexpr uint32_t kTilesPerBlock = 8;

struct Walk {
    int32_t token[kMostNodes], parent[kMostNodes];
    float p[kMostNodes], u[kMostNodes];
    int32_t path[kMostNodes], gone[kMostNodes];                             // accepted nodes; tokens refused at the last of them
    uint32_t accepted, refused;
};

// p of a row without the tokens in `gone`
struct Weights {
    const float *p;
    const int32_t *gone;                                                    // in LDS
    uint32_t refused, vocab;
    __device__ __forceinline__ void tile(uint32_t t, uint32_t lane, double (&w)[4][4]) const
    {
        float4u a[4];
        ecs::load_tile(p, vocab, t, lane, a);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[k][i] = a[k][i] > 0.0f ? (double)a[k][i] : 0.0;        // (NaN counts as 0)
        for (uint32_t j = 0; j < refused; ++j) {
            const uint32_t x = (uint32_t)gone[j];
            if (x / kTile != t) continue;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (x % kTile == 256u * k + 4u * lane + i) w[k][i] = 0.0;
        }
    }
    __device__ __forceinline__ bool reduced() const { return refused != 0; }
    __device__ __forceinline__ void restore() { refused = 0; }
};

// Goes down the tree of a sequence; every thread sees the result
__device__ __forceinline__ void walk_tree(const VerifyTreeArgs &a, uint32_t seq, Walk &s)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u;
    const uint32_t count = a.count ? (uint32_t)min(max(a.count[seq], 0), (int32_t)a.nodes) : a.nodes;
    const float *target = a.target + seq * a.target_seq;
    for (uint32_t i = tid; i < a.nodes; i += kThreads) {                    // (all of them: not waiting for the count)
        const size_t at = (size_t)seq * a.nodes + i;
        const int32_t parent = a.parent[at], x = a.drafted[at];
        const bool below = parent >= -1 && parent < (int32_t)i, is_token = x >= 0 && (uint32_t)x < a.vocab;
        s.parent[i] = below ? parent : -2;                                  // a node without a place in the tree: never reached
        s.token[i] = is_token ? x : -1;                                     // what is no token is refused, and takes nothing
        s.u[i] = a.uniform[(size_t)seq * (a.nodes + 1u) + i];
        s.p[i] = below && is_token ? target[(int64_t)(parent + 1) * a.target_row + x] : 0.0f;
    }
    __syncthreads();
    if (tid < 64u) {
        int32_t at = -1;
        uint32_t n = 0, refused = 0;
        double left = 1.0;
        for (uint32_t i0 = 0; i0 < count; i0 += 64u) {
            const uint32_t i = i0 + lane;
            const int32_t parent = i < count ? s.parent[i] : -2, token = i < count ? s.token[i] : -1;
            const float p = i < count ? s.p[i] : 0.0f, u = i < count ? s.u[i] : 0.0f;
            bool dead = false;                                              // asked already, or the same token was refused here
            for (uint32_t j = 0; j < refused; ++j) dead |= parent == at && token == s.gone[j];
            for (;;) {
                const uint64_t children = __ballot(parent == at && !dead);
                if (!children) break;
                const int j = __ffsll((unsigned long long)children) - 1;
                const float pj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), j));
                const float uj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u), j));
                const int32_t x = __builtin_amdgcn_readlane(token, j);
                if (x >= 0 && (double)uj * left < (double)pj) {
                    at = (int32_t)(i0 + j);
                    if (lane == 0) s.path[n] = at;
                    ++n;
                    refused = 0;
                    left = 1.0;
                    dead = false;                                           // (the nodes here that hang on `at` come after it)
                } else {
                    left -= pj > 0.0f ? (double)pj : 0.0;
                    dead |= lane == (uint32_t)j;
                    if (x >= 0) {
                        if (lane == 0) s.gone[refused] = x;
                        ++refused;
                        dead |= parent == at && token == x;
                    }
                }
            }
            asm volatile("" ::: "memory");                                  // s.gone is read by all lanes
        }
        if (lane == 0) s.accepted = n, s.refused = refused;
    }
    __syncthreads();
}

// What a walk leaves for the second launch, behind a sequence's sums: accepted, refused, the row of p that counts, the next token's random number; the
// accepted nodes, each with its token in its last 20 bits, and then the refused tokens (no node is both, so that they are no more than the nodes)
struct Left {
    int32_t accepted, refused, row;
    float u;
    int32_t list[];
};
constexpr uint32_t kTokenBits = 20;
static_assert(kMostNodes <= 1u << (31 - kTokenBits) && ecs::kMaxTiles * kTile <= 1u << kTokenBits, "a node and its token in one word");
__device__ __forceinline__ uint32_t sequence_bytes(uint32_t nodes, uint32_t vocab)
{
    return (vocab + kTile - 1u) / kTile * 8u + (uint32_t)sizeof(Left) + (nodes + 1u) / 2u * 8u;
}

__global__ __launch_bounds__(kThreads) void verify_tree_sums_kernel(const VerifyTreeArgs a)
{
    __shared__ Walk s;
    const uint32_t seq = blockIdx.y, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    walk_tree(a, seq, s);
    const uint32_t n = s.accepted, refused = s.refused, tiles = (a.vocab + kTile - 1u) / kTile;
    const int32_t row = n ? s.path[n - 1u] + 1 : 0;
    double *sums = reinterpret_cast<double *>(a.work + (size_t)seq * sequence_bytes(a.nodes, a.vocab));
    const Weights w = {a.target + seq * a.target_seq + row * a.target_row, s.gone, refused, a.vocab};
#pragma unroll
    for (uint32_t k = 0; k < kTilesPerBlock / (kThreads / 64u); ++k) {
        const uint32_t t = blockIdx.x * kTilesPerBlock + k * (kThreads / 64u) + wave;
        if (t >= tiles) break;
        const double sum = ecs::tile_sum(w, t, lane);
        if (lane == 0) sums[t] = sum;
    }
    if (blockIdx.x) return;
    Left *left = reinterpret_cast<Left *>(sums + tiles);
    if (tid == 0) {
        left->accepted = (int32_t)n, left->refused = (int32_t)refused, left->row = row;
        left->u = a.uniform[(size_t)seq * (a.nodes + 1u) + a.nodes];
    }
    for (uint32_t i = tid; i < n + refused; i += kThreads)
        left->list[i] = i < n ? s.path[i] << kTokenBits | s.token[s.path[i]] : s.gone[i - n];
}

__global__ __launch_bounds__(kThreads) void verify_tree_token_kernel(const VerifyTreeArgs a)
{
    __shared__ int32_t list[kMostNodes];
    __shared__ ecs::Drawing shared;
    const uint32_t seq = blockIdx.x, tid = threadIdx.x, tiles = (a.vocab + kTile - 1u) / kTile;
    const double *sums = reinterpret_cast<const double *>(a.work + (size_t)seq * sequence_bytes(a.nodes, a.vocab));
    const Left *left = reinterpret_cast<const Left *>(sums + tiles);
    const uint32_t n = (uint32_t)left->accepted, refused = (uint32_t)left->refused;
    for (uint32_t i = tid; i < a.nodes; i += kThreads) list[i] = left->list[i];          // (all that there is room for: not waiting for how many)
    Weights w = {a.target + seq * a.target_seq + left->row * a.target_row, list + n, refused, a.vocab};
    const int32_t token = ecs::draw_token(w, sums, (double)left->u, a.vocab, shared);   // (a barrier before `list` is read)
    int32_t *tokens = a.tokens + (size_t)seq * (a.nodes + 1u), *path = a.path + (size_t)seq * a.nodes;
    for (uint32_t i = tid; i <= a.nodes; i += kThreads) {
        const int32_t node = i < n ? list[i] : -1;
        tokens[i] = i < n ? node & ((1 << kTokenBits) - 1) : i == n ? token : -1;
        if (i < a.nodes) path[i] = i < n ? node >> kTokenBits : -1;
    }
    if (tid == 0) a.accepted[seq] = (int32_t)n;
}

}  // namespace

namespace ecs {

uint64_t verify_tree_work_bytes(uint32_t batch, uint32_t nodes, uint32_t vocab)
{
    return (uint64_t)batch * ((uint64_t)((vocab + kTile - 1u) / kTile) * 8u + 16u + (nodes + 1u) / 2u * 8u);
}

int launch_verify_tree(const VerifyTreeArgs &a, uint32_t batch, void *stream)
{
    const uint32_t tiles = (a.vocab + kTile - 1u) / kTile;
    const int e = launch_args<verify_tree_sums_kernel>(a, (tiles + kTilesPerBlock - 1u) / kTilesPerBlock, batch, 1, kThreads, stream);
    return e ? e : launch_args<verify_tree_token_kernel>(a, batch, 1, 1, kThreads, stream);
}

}  // namespace ecs
