// Attention of new tokens over the paged cache of keys and values.
//
// For a head of the cache, the rows are the (token, head of its group) pairs of a sequence's new tokens: row r is token r / group,
// head r % group of the group.  A row sees the keys up to its own place, p = kv_len - new + token:
//   o_r = sum_{j <= p} exp(t_j - m) v_j / sum_{j <= p} exp(t_j - m),   t_j = scale * q_r . k_j,   m = max t_j
// in one pass over the keys: m and both sums are carried along, and what was added up under an older m is scaled by exp(m_old - m_new).
//
// With ECS_TREE the new tokens are the nodes of a tree: a row sees every key before the first of them, and of the new ones those whose bits
// are set in its token's words (from there on the sum is over j that are seen).  The kernels are the same but for what is hidden in tiles that
// new tokens reach into.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>
#include <algorithm>
#include <type_traits>

#include "kernel_handle.h"
#include "serve.h"

namespace {

using ecs::AttentionArgs;

#ifdef ECS_TREE
constexpr bool kTree = true;
#else
constexpr bool kTree = false;
#endif
template <bool TREE>
using ArgsOf = std::conditional_t<TREE, ecs::AttentionTreeArgs, AttentionArgs>;

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kNone = -__builtin_inff();

// a register as two FP16 values and back
__device__ __forceinline__ half2v as_half2(uint32_t w) { return __builtin_bit_cast(half2v, w); }
__device__ __forceinline__ uint32_t as_word(half2v h) { return __builtin_bit_cast(uint32_t, h); }
__device__ __forceinline__ half8v as_half8(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint4 t = make_uint4(a, b, c, d);
    return __builtin_bit_cast(half8v, t);
}

template <int BYTES>
struct Raw {
    uint32_t w[BYTES < 4 ? 1 : BYTES / 4];
    __device__ __forceinline__ void load(const uint8_t *p)
    {
        if constexpr (BYTES == 2) {
            w[0] = *reinterpret_cast<const uint16_t *>(p);
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else if constexpr (BYTES == 8) {
            const uint2 t = *reinterpret_cast<const uint2 *>(p);
            w[0] = t.x, w[1] = t.y;
        } else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const uint4 t = reinterpret_cast<const uint4 *>(p)[i];
                w[4 * i] = t.x, w[4 * i + 1] = t.y, w[4 * i + 2] = t.z, w[4 * i + 3] = t.w;
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (uint32_t &x : w) x = 0;
    }
};

// Codes as FP16 values, exactly: the code goes into the last bits of 1024, which is then taken off.
__device__ __forceinline__ uint32_t minus(uint32_t w, _Float16 c) { return as_word(as_half2(w) - half2v{c, c}); }
// a constant in a register, where an instruction that has two would need two: the mask and what it is joined with
__device__ __forceinline__ uint32_t held(uint32_t x)
{
    asm("" : "+v"(x));
    return x;
}
// (w & mask) | bits in one instruction
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) { return (w & held(mask)) | held(bits); }
// two bytes (in the low halves of 16 bits each, the sign bit flipped) of 8-bit codes
__device__ __forceinline__ uint32_t from_bytes(uint32_t w) { return minus(w | 0x64006400u, (_Float16)1152.0f); }
// bytes `first` and `first` + 1 of a word, the sign bits flipped
__device__ __forceinline__ uint32_t from_bytes_of(uint32_t w, int first)
{
    return minus(__builtin_amdgcn_perm(held(0x64646464u), w, first ? 0x04030402u : 0x04010400u), (_Float16)1152.0f);
}
// two nibbles, in bits 0-3 and 16-19; less 8, and the lowest value of a row is taken 8 steps higher (low_of): sums of products with
// rounded weights then cancel less
__device__ __forceinline__ uint32_t from_nibbles(uint32_t w) { return minus(and_or(w, 0x000F000Fu, 0x64006400u), (_Float16)1032.0f); }
// those in bits 4-7 and 20-23, without a shift: whole numbers of the values from 64 to 80
__device__ __forceinline__ uint32_t from_high_nibbles(uint32_t w) { return minus(and_or(w, 0x00F000F0u, 0x54005400u), (_Float16)72.0f); }

// 8 neighbouring codes of a key as eight FP16 values, in 4 bits 16 too large: the code is the first four bits behind the leading one of a
// value in [16, 32), and q's sum times 16 steps comes off a score.  (Of 1032, which q's sum would come off without the shift that this takes,
// FP32 is left with too little: a score of 128 terms off by up to 1e-3 where q has a mean; taken off the codes instead, 8 tokens over 32768
// keys in 4 bits take 59.8 us in the place of 58.3, 16 x 1 token of up to 8192 33.7 of 31.6.)  With 4 bits they come in the order
// 0 4 1 5 2 6 3 7 (slot_dim): the values of q are put in the same order, and the order of a sum's terms is free.
template <int BITS>
__device__ __forceinline__ half8v key_values(const uint32_t *w)
{
    if constexpr (BITS == 16) {
        return as_half8(w[0], w[1], w[2], w[3]);
    } else if constexpr (BITS == 8) {
        const uint32_t a = w[0] ^ 0x80808080u, b = w[1] ^ 0x80808080u;
        return as_half8(from_bytes_of(a, 0), from_bytes_of(a, 2), from_bytes_of(b, 0), from_bytes_of(b, 2));
    } else {
        auto two = [](uint32_t x) { return and_or(x, 0x03C003C0u, 0x4C004C00u); };
        return as_half8(two(w[0] << 6), two(w[0] << 2), two(w[0] >> 2), two(w[0] >> 6));
    }
}
template <int BITS>
__device__ __forceinline__ constexpr int slot_dim(int i) { return BITS == 4 ? (i >> 1) + 4 * (i & 1) : i; }

// The i-th of a lane's values of eight keys as an operand: key r in slot r
template <int BITS, class R>
__device__ __forceinline__ half8v value_column(const R (&v)[8], int i)
{
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if constexpr (BITS == 16) {
            o[p] = __builtin_amdgcn_perm(v[2 * p + 1].w[i >> 1], v[2 * p].w[i >> 1], (i & 1) ? 0x07060302u : 0x05040100u);
        } else if constexpr (BITS == 8) {
            const uint32_t s = 0x0C040C00u + 0x00010001u * (uint32_t)(i & 3);
            o[p] = from_bytes(__builtin_amdgcn_perm(v[2 * p + 1].w[i >> 2], v[2 * p].w[i >> 2], s) ^ 0x00800080u);
        } else {
            const uint32_t s = 0x0C040C00u + 0x00010001u * (uint32_t)((i >> 1) & 3);
            const uint32_t t = __builtin_amdgcn_perm(v[2 * p + 1].w[i >> 3], v[2 * p].w[i >> 3], s);
            o[p] = (i & 1) ? from_high_nibbles(t) : from_nibbles(t);
        }
    }
    return as_half8(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ float half_to_float(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }

// A value whose further use is worked out where it stands: in a loop, what follows from it is not kept in registers from before
__device__ __forceinline__ uint32_t here(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// The share of a part of the softmax's sums whose maximum is m, where the largest of all is `top`: above zero, as weights are, so that an infinity
// which the part has met stays one; 0 where it has met no key
__device__ __forceinline__ float share_of(float m, float top)
{
    return m == kNone ? 0.0f : fmaxf(__builtin_amdgcn_exp2f(m - top), 1.17549435e-38f);
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_inff(); }
__device__ __forceinline__ bool half_finite(uint32_t h) { return (h & 0x7C00u) != 0x7C00u; }

// A result as FP16.  It is a mean of values, so that what is finite here and past FP16's largest value is so by rounding only.
__device__ __forceinline__ _Float16 to_result(float x)
{
    const float most = 65504.0f;
    const float y = __builtin_amdgcn_fmed3f(x, -most, most);
    return (_Float16)(finite(x) ? y : x);
}

// the larger of a lane's value and that of the lane 32 (16) away, without LDS
__device__ __forceinline__ float max_over_32(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// the step of a 4-bit row, and what its code 8 stands for
__device__ __forceinline__ float step_of(uint32_t w) { return half_to_float(w & 0xFFFFu); }
__device__ __forceinline__ float low_of(uint32_t w) { return fmaf(8.0f, step_of(w), half_to_float(w >> 16)); }

// The power of two above a step, as an exponent; no less than -32 (the smallest step is 2^-31, a row of equal values has none)
__device__ __forceinline__ float reach_of(float step) { return fmaxf((float)((int)(__float_as_uint(step) >> 23) - 126), -32.0f); }

constexpr float kLeastStep = 2.3283064e-10f;          // 2^-32: of a row whose codes are all 0

// A sequence's part of the arguments
struct Sequence {
    uint32_t first, new_tokens, len;      // first token in q, how many, keys in all
    const int32_t *table;
    __device__ __forceinline__ Sequence(const AttentionArgs &a, uint32_t b)
    {
        const int32_t total = (int32_t)a.tokens;
        const int32_t s = min(max(a.q_start[b], 0), total), e = min(max(a.q_start[b + 1], s), total);
        first = (uint32_t)s;
        new_tokens = min((uint32_t)(e - s), a.max_new);
        const uint64_t most = (uint64_t)a.max_pages << a.cache.page_shift;
        len = (uint32_t)min((uint64_t)max(a.kv_len[b], 0), most);
        behind = (int32_t)len - (e - s);
        table = a.table + (int64_t)b * a.table_stride;
    }
    int32_t behind;                       // keys before the first new token (negative: the first tokens see nothing)
};

// Which of 32 keys a token of a tree sees: bit i is key `key0` + i, of `end` keys in all, the first new one of them `behind`
__device__ __forceinline__ uint32_t seen_bits(const ecs::AttentionTreeArgs &a, uint32_t token, uint32_t key0, int32_t behind, uint32_t end)
{
    const uint32_t *words = a.seen + (int64_t)token * a.seen_stride, count = a.seen_words;
    const int32_t first = (int32_t)key0 - behind;                  // the new token that is key0 (negative: keys before the tree)
    const uint32_t at = (uint32_t)max(first, 0) >> 5;
    const uint64_t pair = (uint64_t)(at + 1u < count ? words[at + 1u] : 0u) << 32 | (at < count ? words[at] : 0u);
    const uint32_t before = (uint32_t)min(max(-first, 0), 32);
    const uint32_t bits = first >= 0 ? (uint32_t)(pair >> (first & 31)) : (uint32_t)(pair << before | ((1ull << before) - 1u));
    const uint32_t left = end > key0 ? end - key0 : 0u;
    return left < 32u ? bits & ((1u << left) - 1u) : bits;
}

// ---- what a workgroup takes of several sequences' rows and keys -----------------------------------------------------------------------------
//
// For rows that all see all keys, the work of a sequence is (tiles of its rows) x (tiles of its keys).  Sequences differ in both, and the host
// sees neither, so that the workgroups of a launch are dealt out here, by every one of them for itself: with each sequence's keys cut into
// pieces of L tiles at most, L is the least length (but for a few steps of halving) at which all pieces find a workgroup.
// (us by equal numbers of splits for all / by this, all else as it was then: 16 trees of up to 16 nodes over up to 8192 keys, 64/8 heads of 128, 8 bits,
// 98.7 / 85.8; eight of up to 49 over up to 2000, 32 heads of 80, 4 bits, 61.2 / 41.8.)

// inclusive results over the lanes of an operation whose neutral element is all zeros
template <class T, class F>
__device__ __forceinline__ T lanes_scan(T v, F with)
{
    auto step = [&](auto from, auto rows) {
        const int t = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(from)::value, decltype(rows)::value, 0xF, false);
        v = with(v, __builtin_bit_cast(T, t));
    };
    typedef std::integral_constant<int, 0xF> all;
    step(std::integral_constant<int, 0x111>(), all());             // from 1, 2, 4, 8 lanes before, of 16
    step(std::integral_constant<int, 0x112>(), all());
    step(std::integral_constant<int, 0x114>(), all());
    step(std::integral_constant<int, 0x118>(), all());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());      // from the last lane of the 16, the 32 before
    step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xC>());
    return v;
}
__device__ __forceinline__ uint32_t sums_to(uint32_t v)
{
    return lanes_scan(v, [](uint32_t x, uint32_t y) { return x + y; });
}
template <class T>
__device__ __forceinline__ T last_lane(T v)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

struct Share {
    uint32_t seq, tile, split, splits;    // splits == 0: nothing
    uint32_t base;                        // balanced: where the sequence's partial results start, in rows of all heads of the cache
};

// Keys up to which sequences are left whole: what a split saves has to be more than the join and its launch take.  us in a graph, whole / split: 16 rows,
// four sequences of 8 tokens, 32 heads of 128, 768 keys FP16 12.9 / 14.4, 8 bits 12.9 / 12.0, 4 bits 12.4 / 14.4, 908 keys 15.0 / 17.6, 15.9 / 14.7, 14.2 / 13.8; one
// of 8, 508 keys 9.5 / 11.7, 908 14.9 / 12.6; rows that share keys in LDS, FP16, eight sequences of 30 tokens, 430 keys 16.8 / 19.9, four, 530 17.7 / 19.6, one
// of 64, 704 19.0 / 15.9; 4 bits, one of 40, 540 keys 21.2 / 16.1.
__host__ __device__ constexpr uint32_t whole_keys(bool few_rows, bool codes) { return few_rows ? 768u : codes ? 256u : 512u; }

template <uint32_t ROWS, uint32_t KEYS, uint32_t HALF, uint32_t WHOLE>
__device__ __forceinline__ Share share_of_work(const ecs::AttentionTreeArgs &a, bool first_wave)
{
    const uint32_t slot = blockIdx.y + gridDim.y * blockIdx.z;     // (blockIdx.x: the head)
    if (slot >= a.slots) return {0, 0, 0, 0, 0};
    if (!a.balanced) {
        const uint32_t item = slot / a.splits;
        return {item / a.row_tiles, item % a.row_tiles, slot % a.splits, a.splits, 0};
    }
    const uint32_t lane = threadIdx.x & 63u, b = min(lane, a.batch - 1u);
    const Sequence s(a, b);
    const uint32_t rows = lane < a.batch ? s.new_tokens * a.group : 0u, items = (rows + ROWS - 1u) / ROWS;
    const uint32_t tiles_of_keys = lane < a.batch ? max((s.len + KEYS - 1u) / KEYS, 1u) : 1u;
    // what a tile of keys costs: HALF sixteenths where rows are half of a tile's at most
    const uint32_t keys = HALF == 16u || rows > ROWS / 2u ? tiles_of_keys : max(tiles_of_keys * HALF / 16u, 1u);
    const uint32_t all = last_lane(sums_to(items));
    const uint32_t longest = last_lane(lanes_scan(keys, [](uint32_t x, uint32_t y) { return max(x, y); }));
    const float work = last_lane(lanes_scan((float)items * (float)keys, [](float x, float y) { return x + y; }));
    auto pieces = [&](uint32_t length) { return (keys + length - 1u) / length; };
    // as many pieces as the chip has workgroups at once, or, with more tiles of rows than that, as it has in whole rounds
    const uint32_t goal = min(a.slots, max((all + a.at_once - 1u) / a.at_once, 1u) * a.at_once);
    // the least length there could be, and one at which it works out: work / length + all <= goal (in case FP32 says otherwise: no pieces)
    uint32_t low = longest <= WHOLE / KEYS ? longest : max((uint32_t)(work / (float)goal), 256u / KEYS), length = longest;
    if (goal > all) {
        const uint32_t enough = max((uint32_t)(work / (float)(goal - all)) + 1u, low);
        if (last_lane(sums_to(items * pieces(enough))) <= goal) length = min(length, enough);
    }
    for (int step = 0; step < 5 && low < length; ++step) {
        const uint32_t middle = (low + length) / 2u;
        if (last_lane(sums_to(items * pieces(middle))) <= goal)
            length = middle;
        else
            low = middle + 1u;
    }
    const uint32_t mine = pieces(length), to = sums_to(items * mine), rows_to = sums_to(rows * mine);
    const uint32_t before = to - items * mine, rows_before = rows_to - rows * mine;
    // (rows that would lie behind the workspace: starts that are not in order)
    const uint32_t splits = mine > 1u && rows_to > a.part_rows ? 0u : mine;
    if (first_wave && slot == 0 && blockIdx.x == 0) a.plan[lane] = {splits, rows_before, lane < a.batch ? s.first : 0xFFFFFFFFu, s.new_tokens};
    const uint32_t seq = (uint32_t)__popcll(__ballot(to <= slot));
    if (seq >= a.batch) return {0, 0, 0, 0, 0};
    const uint32_t in = slot - (uint32_t)__builtin_amdgcn_readlane((int)before, (int)seq);
    const uint32_t tiles = (uint32_t)__builtin_amdgcn_readlane((int)items, (int)seq), split = in / tiles;
    return {seq, in - split * tiles, split, (uint32_t)__builtin_amdgcn_readlane((int)splits, (int)seq),
            (uint32_t)__builtin_amdgcn_readlane((int)rows_before, (int)seq)};
}

// The page of a key, a number that is one whatever the table holds
__device__ __forceinline__ uint32_t page_of(const AttentionArgs &a, const int32_t *table, uint32_t key)
{
    return min((uint32_t)table[key >> a.cache.page_shift], a.cache.pages - 1u);
}

// ---- up to 16 rows per workgroup, its four wavefronts on different keys ------------------------------------------------------------
//
// A wavefront takes 32 keys at a time.  Keys times q: the keys are the rows of the matrix product's result and the 16 rows of q its
// columns, so that lane l has column l % 16 and of each 16 keys the four 4 (l / 16) ... + 3.  These are what the second product, V^T
// times the weights, reads of the weights in that lane, if its sum over 32 keys is taken in the order that the first one left: the
// weights never leave their lane.  V comes as it lies in memory, 8 keys times DP / 16 values per lane, and is turned round in
// registers; its columns are dealt to the products as DP / 16 per lane, the i-th product has values i of every lane.
//
// What bounds it is reading the cache, and with one token to a sequence the two trips (lengths and pages, then keys) before the first key and
// the join after the last, some 15 us together: one token over 200 keys, 12 heads of 64, 4.8 us; 16 sequences of up to 8192 keys, 8 heads
// of 128 in 8 bits, 144 MB, 40 us; 8 tokens over 32768 keys, 40 heads of 128 in FP16, 671 MB, 126 us, 5.3 TB/s.  16 rows because that is
// the least that a matrix instruction takes; four wavefronts on keys of their own need no barrier before the end.
template <int BITS, int DP, bool PAD, bool TREE>
__global__ __launch_bounds__(256, BITS == 4 ? (DP > 128 ? 2 : DP > 64 ? 3 : 4) : DP > 128 ? 1 : 2) void attention_rows_kernel(const ArgsOf<TREE> a)
{
    constexpr int kSteps = DP / 32, VD = DP / 16;
    constexpr int KB = BITS == 16 ? 8 : BITS == 8 || PAD || DP == 64 ? 16 : 32;       // neighbouring values of a key in a lane
    constexpr int kLoads = DP / 4 / KB;
    typedef Raw<KB * BITS / 8> KeyRaw;
    typedef Raw<VD * BITS / 8> ValueRaw;
    constexpr int kRow = DP + 4;
    __shared__ float lds_o[4][16][kRow];
    __shared__ float lds_ml[4][16][2];

    const uint32_t tid = threadIdx.x, lane = tid & 63u, j = lane & 15u, g = lane >> 4;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    uint32_t tile = blockIdx.x / a.splits, split = blockIdx.x - tile * a.splits, head = blockIdx.y, seq = blockIdx.z, splits = a.splits, base = 0;
    if constexpr (TREE) {
        head = blockIdx.x;
        const Share mine = share_of_work<16, 32, 16, whole_keys(true, BITS < 16)>(a, tid < 64u);
        tile = mine.tile, split = mine.split, seq = mine.seq, splits = mine.splits, base = mine.base;
        if (splits == 0) return;
    }
    const Sequence s(a, seq);
    const uint32_t rows = s.new_tokens * a.group, row0 = 16u * tile;
    if (row0 >= rows) return;
    const uint32_t dim = PAD ? a.cache.dim : DP;

    // this lane's row, and the keys that rows of the tile see
    const uint32_t row = min(row0 + j, rows - 1u), token = row / a.group;
    const int32_t seen = min(s.behind + (int32_t)token + 1, (int32_t)s.len);             // keys that this row sees
    const uint32_t last_row = min(row0 + 15u, rows - 1u);
    const int32_t end_i = TREE ? (int32_t)s.len : min(s.behind + (int32_t)(last_row / a.group) + 1, (int32_t)s.len);
    const uint32_t end = end_i > 0 ? (uint32_t)end_i : 0u;
    const int32_t all_see = TREE ? s.behind : s.behind + (int32_t)(row0 / a.group) + 1;  // keys that every row sees

    const uint32_t tiles = (end + 31u) >> 5, per = (tiles + splits - 1u) / splits;
    const uint32_t t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);
    const uint32_t page_mask = (1u << a.cache.page_shift) - 1u;
    const uint64_t page_rows = (uint64_t)a.cache.heads << a.cache.page_shift, head_rows = (uint64_t)head << a.cache.page_shift;

    f32x4 acc[VD];
#pragma unroll
    for (int i = 0; i < VD; ++i) acc[i] = f32x4{0, 0, 0, 0};
    // m: the maximum that weights are taken against, of t, with steps of t plus the key's reach_of(step of V): weights times steps, which go to
    // the products as FP16, then stay in its range, and the largest of what this row sees are the ones that keep their bits, whatever steps
    // lie beside them.  m may lie up to 8 below the true maximum, weights then go to 2^8, and what was added up is seldom scaled
    float m = kNone, m_true = kNone, l = 0.0f, z_acc = 0.0f;
    bool odd = false;                                              // values that are not finite were left out

    // The keys of the next round are asked for as soon as this round's have been multiplied, its values before that: both are on their way
    // while the softmax is worked out.
    uint32_t page_list = 0;                                       // lane 2 i + h: the page of the h-th 16 keys of the i-th of 32 rounds
    uint64_t at[2], at_next[2] = {0, 0};                          // first row of each 16 keys in the cache
    KeyRaw k[2][kLoads];
    uint32_t ks[8] = {};
    auto request_k = [&](uint32_t t) {
        const uint32_t round = (t - t0 - wave) >> 2;
        // keys beyond the last one are read from where the last one is
        auto key_of = [&](uint32_t tile, uint32_t h) { return min(32u * tile + 16u * h, (end - 1u) & ~15u); };
        if ((round & 31u) == 0) {
            page_list = page_of(a, s.table, key_of(t + 4u * (lane >> 1), lane & 1u));
            asm volatile("" : "+v"(page_list));                   // waited for here, and not by every round
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)page_list, (int)(2u * (round & 31u) + h));
            at_next[h] = (uint64_t)page * page_rows + head_rows + (key_of(t, h) & page_mask);
            const uint8_t *p = a.cache.k + at_next[h] * a.cache.row_bytes + (j * a.cache.row_bytes + g * (KB * BITS / 8));
#pragma unroll
            for (int x = 0; x < kLoads; ++x) {
                if (!PAD || (uint32_t)(x * 4 * KB) + g * KB < dim)
                    k[h][x].load(p + x * (4 * KB * BITS / 8));
                else
                    k[h][x].clear();
            }
            if constexpr (BITS < 16) {
                const uint4 x = *reinterpret_cast<const uint4 *>(a.cache.k_step + 4u * (at_next[h] + 4u * g));
                ks[4 * h] = x.x, ks[4 * h + 1] = x.y, ks[4 * h + 2] = x.z, ks[4 * h + 3] = x.w;
            }
        }
    };
    if (t0 + wave < t1) request_k(t0 + wave);

    half8v q[kSteps];
    float q_sum = 0.0f;
    {
        const uint16_t *p = a.q.data + (int64_t)(s.first + token) * a.q.token_stride +
                            (int64_t)(head * a.group + (row - token * a.group)) * a.q.head_stride;
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
            const uint32_t d0 = (uint32_t)(t / (KB / 8)) * (4u * KB) + g * KB + 8u * (t % (KB / 8));
            const bool in = !PAD || d0 < dim;
            uint32_t w[4] = {0, 0, 0, 0};
            if (in) {
                if (a.q_wide) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(p + d0);
                    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i >> 1] |= (uint32_t)p[(int64_t)(d0 + i) * a.q.dim_stride] << (16 * (i & 1));
                }
            }
            uint32_t o[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = slot_dim<BITS>(i);
                const uint32_t h = (d & 1) ? w[d >> 1] >> 16 : w[d >> 1] & 0xFFFFu;
                o[i >> 1] |= h << (16 * (i & 1));
                if constexpr (BITS == 4) q_sum += half_to_float(h);
            }
            q[t] = as_half8(o[0], o[1], o[2], o[3]);
        }
        if constexpr (BITS == 4) {
            q_sum += __shfl_xor(q_sum, 16, 64);
            q_sum += __shfl_xor(q_sum, 32, 64);
        }
    }

    for (uint32_t t = t0 + wave; t < t1; t += 4u) {
        const uint32_t key0 = 32u * t;
        at[0] = at_next[0], at[1] = at_next[1];
        ValueRaw v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const uint8_t *p = a.cache.v + at[r >> 2] * a.cache.row_bytes + ((4u * g + (r & 3)) * a.cache.row_bytes + j * (VD * BITS / 8));
            if (!PAD || j * VD < dim)
                v[r].load(p);
            else
                v[r].clear();
        }
        uint32_t vs[8] = {};
        if constexpr (BITS < 16) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 y = *reinterpret_cast<const uint4 *>(a.cache.v_step + 4u * (at[h] + 4u * g));
                vs[4 * h] = y.x, vs[4 * h + 1] = y.y, vs[4 * h + 2] = y.z, vs[4 * h + 3] = y.w;
            }
        }
        __builtin_amdgcn_sched_barrier(0);

        float w[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 c = {0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                constexpr int kPer = KB / 8;                       // steps that a load feeds
                c = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_values<BITS>(&k[h][t / kPer].w[(t % kPer) * (BITS / 4)]), q[t], c, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float d = c[r];
                if constexpr (BITS == 8) d *= __uint_as_float(ks[4 * h + r]);
                if constexpr (BITS == 4) d = fmaf(fmaf(-24.0f, q_sum, d), step_of(ks[4 * h + r]), q_sum * low_of(ks[4 * h + r]));
                w[4 * h + r] = d * a.scale_log2;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (t + 4u < t1) request_k(t + 4u);
        __builtin_amdgcn_sched_barrier(0);
        const bool some_hidden = (int32_t)(key0 + 32u) > all_see || key0 + 32u > end;
        if (some_hidden) {
            if constexpr (TREE) {
                const uint32_t bits = seen_bits(a, s.first + token, key0, s.behind, end) >> (4u * g);
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (!(bits >> ((r < 4 ? 0 : 16) + (r & 3)) & 1u)) {
                        w[r] = kNone;
                        if constexpr (BITS < 16) vs[r] = 0u;       // (a node that was left out may have a step that is none)
                    }
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int32_t key = (int32_t)(key0 + (r < 4 ? 0u : 16u) + 4u * g + (r & 3));
                    if (key >= seen) w[r] = kNone;
                }
            }
        }
        float most = kNone, step[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if constexpr (BITS < 16) {
                if (some_hidden && key0 + (r < 4 ? 0u : 16u) + 4u * g + (r & 3) >= end) vs[r] = 0u;
                step[r] = BITS == 8 ? __uint_as_float(vs[r]) : step_of(vs[r]);
                most = fmaxf(most, w[r] + reach_of(step[r]));
            } else {
                most = fmaxf(most, w[r]);
            }
        }
        const float m_new = m_true = fmaxf(m_true, max_over_32(max_over_16(most)));
        if (const bool far = m_new > m + 8.0f; __any((int)far)) {
            const float alpha = far ? __builtin_amdgcn_exp2f(m - m_new) : 1.0f;       // (0 where nothing was seen before)
            m = far ? m_new : m;                                   // a row goes by its own scores alone
            l *= alpha;
            z_acc *= alpha;
#pragma unroll
            for (int i = 0; i < VD; ++i) acc[i] *= alpha;
        }
        const float base = m == kNone ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            w[r] = __builtin_amdgcn_exp2f(w[r] - base);
            sum += w[r];
            if constexpr (BITS == 4) z_acc = fmaf(w[r], low_of(vs[r]), z_acc);
            if constexpr (BITS < 16) w[r] *= step[r];
        }
        l += sum;

        if constexpr (BITS == 16) {
            if (some_hidden) {
                // Keys that no row of the tile sees may hold anything; and where V is not finite, a weight of 0 has to stay without
                // effect on the rows that do not see it: such values are left out of the product.
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const uint32_t key = key0 + (r < 4 ? 0u : 16u) + 4u * g + (r & 3);
#pragma unroll
                    for (uint32_t &x : v[r].w) {
                        x = key < end ? x : 0u;
                        const uint32_t keep = (half_finite(x) ? 0xFFFFu : 0u) | (half_finite(x >> 16) ? 0xFFFF0000u : 0u);
                        odd |= keep != 0xFFFFFFFFu;
                        x &= keep;
                    }
                }
            }
        }
        // The weights as FP16 and what that leaves out, also as FP16: the matrix instructions have time for both, and the result is then as
        // exact as sums in FP32 (rounded once its error is 1.4 times that).  What is left out is that of the very value in pw: converted a
        // second time, a weight times its step may round the other way, with the product of both rounded first or not.
        uint32_t pw[4], pr[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            pw[p] = as_word(half2v{(_Float16)w[2 * p], (_Float16)w[2 * p + 1]});
            asm("" : "+v"(pw[p]));
            const half2v o = as_half2(pw[p]);
            pr[p] = as_word(half2v{(_Float16)(w[2 * p] - (float)o[0]), (_Float16)(w[2 * p + 1] - (float)o[1])});
        }
        const half8v weights = as_half8(pw[0], pw[1], pw[2], pw[3]), rest = as_half8(pr[0], pr[1], pr[2], pr[3]);
#pragma unroll
        for (int i = 0; i < VD; ++i) {
            const half8v column = value_column<BITS>(v, i);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(column, weights, acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(column, rest, acc[i], 0, 0, 0);
        }
    }

    if constexpr (BITS == 16) {
        // Where V was not finite, the sum of what was not is the result: weights are above zero, but in FP16, or the second part of one, they
        // may be zero or less.  Rare, and not fast.  (With a weight of NaN, l is NaN too.)
#pragma unroll
        for (int i = 0; i < VD; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                odd |= !finite(acc[i][r]);
                acc[i][r] = finite(acc[i][r]) ? acc[i][r] : 0.0f;
            }
        if (__any((int)odd)) {
            for (uint32_t t = t0 + wave; t < t1; t += 4u)
#pragma unroll 1
                for (uint32_t key = 32u * t; key < min(32u * t + 32u, end); ++key) {
                    if constexpr (TREE) {
                        if (!(seen_bits(a, s.first + token, key, s.behind, end) & 1u)) continue;
                    } else {
                        if ((int32_t)key >= seen) continue;
                    }
                    const uint64_t at = (uint64_t)page_of(a, s.table, key) * page_rows + head_rows + (key & page_mask);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t d = VD * (4u * g + r);
                        if (PAD && d >= dim) continue;
                        ValueRaw x;
                        x.load(a.cache.v + at * a.cache.row_bytes + 2u * d);
#pragma unroll
                        for (int i = 0; i < VD; ++i) {
                            const uint32_t v = (i & 1) ? x.w[i >> 1] >> 16 : x.w[i >> 1] & 0xFFFFu;
                            acc[i][r] += half_finite(v) ? 0.0f : half_to_float(v);
                        }
                    }
                }
        }
    }

    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if constexpr (BITS == 4) {
        z_acc += __shfl_xor(z_acc, 16, 64);
        z_acc += __shfl_xor(z_acc, 32, 64);
    }
    // the four wavefronts' results meet in LDS
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < VD; i += 4) {
            f32x4 o = {acc[i][r], acc[i + 1][r], acc[i + 2][r], acc[i + 3][r]};
            if constexpr (BITS == 4) o = o + z_acc;
            *reinterpret_cast<f32x4 *>(&lds_o[wave][j][VD * (4u * g + r) + i]) = o;
        }
    if (g == 0) lds_ml[wave][j][0] = m, lds_ml[wave][j][1] = l;
    __syncthreads();

    const uint32_t n = tid >> 4, d0 = VD * (tid & 15u);
    if (row0 + n >= rows || d0 >= dim) return;
    float most = kNone, total = 0.0f, share[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) most = fmaxf(most, lds_ml[x][n][0]);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        share[x] = share_of(lds_ml[x][n][0], most);
        total += share[x] * lds_ml[x][n][1];
    }
    float o[VD];
#pragma unroll
    for (int i = 0; i < VD; ++i) {
        o[i] = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) o[i] += share[x] * lds_o[x][n][d0 + i];
    }
    const uint32_t out_row = row0 + n, out_token = out_row / a.group, out_head = head * a.group + (out_row - out_token * a.group);
    if (splits == 1u) {
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        uint16_t *p = a.out.data + (int64_t)(s.first + out_token) * a.out.token_stride + (int64_t)out_head * a.out.head_stride;
#pragma unroll
        for (int i = 0; i < VD; i += 2) {
            const half2v h = {to_result(o[i] * inv), to_result(o[i + 1] * inv)};
            if (a.out_wide) {
                *reinterpret_cast<uint32_t *>(p + d0 + i) = as_word(h);
            } else {
                p[(int64_t)(d0 + i) * a.out.dim_stride] = (uint16_t)as_word(h);
                p[(int64_t)(d0 + i + 1) * a.out.dim_stride] = (uint16_t)(as_word(h) >> 16);
            }
        }
    } else {
        uint64_t at = ((uint64_t)split * a.tokens + s.first + out_token) * a.q_heads + out_head;
        if constexpr (TREE)
            if (a.balanced) at = ((uint64_t)base + split * rows + out_row) * a.cache.heads + head;
#pragma unroll
        for (int i = 0; i < VD; i += 4) *reinterpret_cast<f32x4 *>(a.part_o + at * dim + d0 + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
        if ((tid & 15u) == 0) a.part_ml[2 * at] = most, a.part_ml[2 * at + 1] = total;
    }
}

// ---- 128 rows per workgroup, 32 for each of its wavefronts, which share the keys through LDS -----------------------------------------
//
// Tiles of KT keys and values lie in LDS twice: one is computed with while the next one is on its way, FP16 straight from memory to LDS, 8-
// and 4-bit codes through registers, where they become FP16 values (exact whole numbers; their steps are applied to the products'
// results and to the weights).  As above the keys are the rows of the first product, 32 x 32 at a time, a lane has column l % 32 and of
// each 8 keys the four 4 (l / 32) ... + 3, and the weights stay in their lane; the second product's V^T comes from LDS through its
// transposing read, four keys of a column per lane.
// Pieces of 16 bytes are swapped within a row by the key's number, so that a wavefront's reads spread over all banks: of K, 16 lanes
// read the same piece of 16 rows; of V, 64 bytes of 8 rows.
//
// The weights go to the second product as one FP16 value, 2^-11 of each, where the kernel above has a second one for what that leaves out: the
// error against 64 bits is 2.9e-4 of the result in place of the 2.1e-4 that its own rounding to FP16 makes.  Here the matrix instructions are
// half of the time, and a second part costs what it takes (us by one / by two: 2048 tokens over 4096 keys, heads of 128, FP16 132 / 171, 8 bits 164 /
// 194, 4 bits 168 / 202; 512 over 9098 108 / 133; five of up to 333 over 3000, heads of 80, 68 / 80, 4 bits 78 / 86).  With FP16 the sum of the weights is
// that of the rounded ones.  Trees of up to 64 rows wait for the keys and values of FP16, so that a second part costs them nothing there, and they have it
// (64 nodes of heads of 128, one tree over 32768 keys 131.3 / 132.5, four over 8000 112.2 / 111.1).  It is not free with 257 nodes (16000 keys, 32/8 heads, 95.5 /
// 124.4), heads of 256 (192 nodes over 8000 45.9 / 50.3) and codes (four of 64 over 8000, 8 bits 83.5 / 93.9, 4 bits 77.6 / 87.4; sixteen of up to 16 over up to
// 8192, 8 bits, 76.0 / 83.8), which are rounded by up to 2^-8 of their row's largest value, 2^-5 of its range in 4 bits, when they are written.
//
// 2048 tokens over 4096 keys, 32 heads of 128, FP16: 121 - 127 us, 810 - 850 TFLOP/s of the products that the mask leaves (a large matrix
// product alone reaches 1140 - 1229 here).  A wavefront's products and its softmax follow one another, and those of the two wavefronts of a SIMD overlap only in
// part; without the loads it would take 98 - 107.  32 rows to a wavefront: with 64 the accumulators moved between the two halves
// of the register file (208 us).  Softmax and products of neighbouring halves interleaved in one wavefront took 123 us here, but 122 for
// 110 where 512 tokens see 9098 keys, 105 for 71 with five sequences in FP16 and 402 for 158 in 4 bits.
template <int RC>
__device__ __forceinline__ uint32_t k_swap(uint32_t key) { return RC >= 16 ? key & 15u : (key / (16 / RC)) & (RC - 1u); }
template <int RC>
__device__ __forceinline__ uint32_t v_swap(uint32_t key) { return RC >= 16 ? (key & 3u) << 2 : RC == 8 ? (key & 2u) << 1 : 0u; }

// eight 4-bit codes, less 8, in their own order, or as they come
template <bool SLOTS>
__device__ __forceinline__ uint4 nibble_values(uint32_t w)
{
    const uint32_t a = from_nibbles(w), b = from_high_nibbles(w), c = from_nibbles(w >> 8), d = from_high_nibbles(w >> 8);    // 0 4, 1 5, 2 6, 3 7
    if constexpr (SLOTS) return make_uint4(a, b, c, d);
    return make_uint4(__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(d, c, 0x05040100u),
                      __builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u));
}
// eight codes of 8 or 4 bits as FP16 values
template <int BITS, bool SLOTS>
__device__ __forceinline__ uint4 code_values(const Raw<BITS> &r)
{
    if constexpr (BITS == 8) {
        const uint32_t a = r.w[0] ^ 0x80808080u, b = r.w[1] ^ 0x80808080u;
        return make_uint4(from_bytes_of(a, 0), from_bytes_of(a, 2), from_bytes_of(b, 0), from_bytes_of(b, 2));
    } else {
        return nibble_values<SLOTS>(r.w[0]);
    }
}

//
// With ON_KEYS == 2 a workgroup has 64 rows, and two wavefronts share 32 of them: each works on half of a tile's keys, and their results meet
// in LDS at the end.  Where the rows of a tree's tile of 128 are 64 or fewer, its workgroup does the same if keys and values are codes (16 trees of up to 16
// nodes over up to 8192 keys, 64/8 heads of 128, 8 bits: 83.8 us without, 78.9 with; FP16 has not the registers): a tile of keys then costs 0.72 of what it
// costs otherwise (128 and 64 rows, sixteen sequences of one length, 127 and 91 us), and shares are dealt out by that (9/16 85.6, 13/16 81.2).
//
// With trees, codes' weights have the step of their values in the exponent: p step = 2^(score + log2 step), the running maximum is that of these
// exponents, and the sum of the weights that of p step / step.  A multiplication and an addition fewer for each score (of some seven beside the
// exponential): the same trees in 8 bits 81.1 -> 76.3 us, 8 x 49 of 2000 in 4 bits 40.0 -> 38.5.  The logarithm, of at most 32 in size, is off by some 2^-19 of it,
// and a weight by 2^-19.5 of itself above and below the line alike.  A row of equal values has no step: 2^-32 stands for it, its codes are 0.
// In 4 bits eight codes are left in the order in which two masks and a shift take them apart, in LDS and in the accumulators, and the lanes' results put in order
// at the end: 8 x 49 of 2000 38.8 -> 36.9.
template <int BITS, int DP, bool TREE, int ON_KEYS>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void attention_chunk_kernel(const ArgsOf<TREE> a)
{
    constexpr int RC = DP <= 32 ? 4 : DP <= 64 ? 8 : DP <= 128 ? 16 : 32;              // 16-byte pieces of a row in LDS
    constexpr int KT = RC == 32 && ON_KEYS == 1 ? 32 : 64, kSteps = DP / 16, kTiles = DP / 32;
    constexpr uint32_t kRows = 128 / ON_KEYS;
    constexpr bool kByRows = TREE && ON_KEYS == 1 && BITS < 16 && DP <= 128;           // a tile of 64 rows or fewer is worked on as with ON_KEYS == 2
    constexpr bool kStepInExponent = TREE && BITS < 16;            // (of V; lds_step has 1 / step and low / step of it)
    constexpr bool kSlots = TREE && BITS == 4;                     // dims in LDS in the order 0 4 1 5 2 6 3 7 (slot_dim) of each eight
    constexpr int kGroups = KT / 16;                                                   // a wavefront brings 16 keys; with 32, of K or of V
    constexpr int kIssues = RC / 4;                                                    // accesses per lane for 16 rows
    // (four objects and not two of twice the size: a read of LDS then waits for what is on its way into the same object only)
    __shared__ uint4 lds_k0[KT * RC], lds_k1[KT * RC], lds_v0[KT * RC], lds_v1[KT * RC];
    __shared__ float lds_step[2][2][2][KT];                                            // [buffer][k, v][step, low][key]
    __shared__ float lds_reach[2][BITS < 16 ? KT : 1];                                 // reach_of a key's step of V, or its logarithm
    __shared__ uint32_t lds_odd[2];
    __shared__ float lds_mlz[2][3][32];                                                // of the second of two wavefronts that share rows

    const uint32_t tid = threadIdx.x, lane = tid & 63u, n = lane & 31u, h = lane >> 5;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    // the last rows see the most keys: their workgroups start first.  Where all workgroups run at once (two on a compute unit, one that
    // starts early beside one that starts late), the second half goes the other way, so that each pair has the same to do.
    uint32_t tile = blockIdx.y / a.splits, head = blockIdx.x, split = blockIdx.y % a.splits, seq = blockIdx.z, splits = a.splits, base = 0;
    if (TREE)
        ;
    else if (tile < (a.row_tiles + 1u) / 2u || gridDim.x * gridDim.y * gridDim.z > 512u)
        tile = a.row_tiles - 1u - tile;
    else
        tile -= (a.row_tiles + 1u) / 2u;
    if constexpr (TREE) {
        const Share mine = share_of_work<kRows, KT, kByRows ? 11 : 16, whole_keys(false, BITS < 16)>(a, tid < 64u);
        tile = mine.tile, split = mine.split, seq = mine.seq, splits = mine.splits, base = mine.base;
        if (splits == 0) return;
    }
    const Sequence s(a, seq);
    const uint32_t rows = s.new_tokens * a.group, row0 = kRows * tile;
    if (row0 >= rows) return;
    const uint32_t dim = a.cache.dim, pieces = dim / 8u;

    auto work = [&](auto shared_by) {                              // by how many wavefronts rows are shared
        constexpr int kShared = decltype(shared_by)::value, kHalves = KT / 32 / kShared;                           // halves of a tile: of a wavefront
        constexpr int kParts = kShared == 2 && BITS == 16 && DP <= 128 ? 2 : 1;            // FP16 values that a weight goes to the second product as
        const uint32_t wave_row = row0 + 32u * (wave % (4u / kShared)), half0 = kHalves * (wave / (4u / kShared));     // first row, first half of a tile
        const uint32_t row = min(wave_row + n, rows - 1u), token = row / a.group;
        const int32_t seen = min(s.behind + (int32_t)token + 1, (int32_t)s.len);
        auto sees = [&](uint32_t r) -> int32_t {                                           // keys up to the last one that row r sees
            return TREE ? (int32_t)s.len : max(min(s.behind + (int32_t)(min(r, rows - 1u) / a.group) + 1, (int32_t)s.len), 0);
        };
        const uint32_t end = (uint32_t)sees(row0 + kRows - 1u);                                  // of the workgroup
        const uint32_t all_see = TREE ? (uint32_t)max(s.behind, 0) : (uint32_t)sees(row0);
        const uint32_t wave_end = wave_row < rows ? (uint32_t)sees(wave_row + 31u) : 0u;

        half8v q[kSteps];
        float q_sum = 0.0f;
        {
            const uint16_t *p = a.q.data + (int64_t)(s.first + token) * a.q.token_stride +
                                (int64_t)(head * a.group + (row - token * a.group)) * a.q.head_stride;
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const uint32_t d0 = 16u * t + 8u * h;
                uint32_t w[4] = {0, 0, 0, 0};
                if (d0 < dim) {
                    if (a.q_wide) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(p + d0);
                        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i >> 1] |= (uint32_t)p[(int64_t)(d0 + i) * a.q.dim_stride] << (16 * (i & 1));
                    }
                }
                if (a.scale_log2 < 0.0f)                               // the largest score is the one with the largest product
#pragma unroll
                    for (uint32_t &x : w) x ^= 0x80008000u;
                if constexpr (BITS == 4)
#pragma unroll
                    for (int i = 0; i < 4; ++i) q_sum += half_to_float(w[i] & 0xFFFFu) + half_to_float(w[i] >> 16);
                q[t] = !kSlots ? as_half8(w[0], w[1], w[2], w[3])
                               : as_half8(__builtin_amdgcn_perm(w[2], w[0], 0x05040100u), __builtin_amdgcn_perm(w[2], w[0], 0x07060302u),
                                          __builtin_amdgcn_perm(w[3], w[1], 0x05040100u), __builtin_amdgcn_perm(w[3], w[1], 0x07060302u));
            }
            if constexpr (BITS == 4) q_sum += __shfl_xor(q_sum, 32, 64);
        }
        // (a scale of 0 as the least there is: a hidden key's score, minus infinity, stays that)
        const float scale = a.scale_log2 == 0.0f ? 1.17549435e-38f : fabsf(a.scale_log2), by = BITS == 16 ? scale : 1.0f;

        const uint32_t tiles = (end + KT - 1u) / KT, per = (tiles + splits - 1u) / splits;
        const uint32_t t0 = min(split * per, tiles), t1 = min(t0 + per, tiles);
        const uint32_t page_mask = (1u << a.cache.page_shift) - 1u;
        const uint64_t page_rows = (uint64_t)a.cache.heads << a.cache.page_shift, head_rows = (uint64_t)head << a.cache.page_shift;
        const uint32_t group16 = kGroups == 4 ? wave : wave & 1u;
        const bool brings_k = kGroups == 4 || wave < 2u, brings_v = kGroups == 4 || wave >= 2u;

        if (pieces < (uint32_t)RC)
            for (uint32_t i = tid; i < KT * RC; i += 256u)             // what is beyond dim stays zero
                lds_k0[i] = lds_k1[i] = lds_v0[i] = lds_v1[i] = make_uint4(0, 0, 0, 0);
        if (tid < 2u) lds_odd[tid] = 0;
        __syncthreads();

        // Bringing tile t into buffer b, this wavefront's 16 keys of it: request() sends the loads off, arrive() waits for them and writes what
        // has come through registers.
        Raw<BITS> raw_k[BITS < 16 ? kIssues : 1], raw_v[BITS < 16 ? kIssues : 1];
        uint32_t raw_step = 0;
        auto first_key = [&](uint32_t t) { return min(t * KT + 16u * group16, (end - 1u) & ~15u); };      // (beyond the end: the last 16 keys again)
        uint32_t page_list = 0;                                        // lane i: the page of this wavefront's keys in the i-th tile of 64
        auto request = [&](uint32_t t, auto buffer) {
            const int b = buffer;
            uint4 *lds_k = b ? lds_k1 : lds_k0, *lds_v = b ? lds_v1 : lds_v0;
            if (((t - t0) & 63u) == 0) {
                page_list = page_of(a, s.table, first_key(t + lane));
                asm volatile("" : "+v"(page_list));                    // waited for here, where it happens, and not by every tile
            }
            const uint32_t key = first_key(t);
            const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)page_list, (int)((t - t0) & 63u));
            const uint64_t at = (uint64_t)page * page_rows + head_rows + (key & page_mask);
            const uint8_t *kp = a.cache.k + at * a.cache.row_bytes, *vp = a.cache.v + at * a.cache.row_bytes;
            const uint32_t self = here(lane);
            auto bring = [&](auto whole) {                             // whole: dim fills the rows of LDS
#pragma unroll
                for (int i = 0; i < kIssues; ++i) {
                    const uint32_t r = (64u * i + self) / RC, c = self % RC;             // row of the 16, piece
                    const uint32_t row = decltype(whole)::value ? r * (2u * DP) : r * a.cache.row_bytes;
                    if constexpr (BITS == 16) {
                        const uint32_t to = (16u * group16) * RC + 64u * i;
                        if (const uint32_t from = c ^ k_swap<RC>(16u * group16 + r); brings_k && (decltype(whole)::value || from < pieces))
                            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(kp + (row + 16u * from)),
                                                             (__attribute__((address_space(3))) void *)(&lds_k[to]), 16, 0, 0);
                        if (const uint32_t from = c ^ v_swap<RC>(16u * group16 + r); brings_v && (decltype(whole)::value || from < pieces))
                            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(vp + (row + 16u * from)),
                                                             (__attribute__((address_space(3))) void *)(&lds_v[to]), 16, 0, 0);
                    } else {
                        const uint32_t from = row + min(c, pieces - 1u) * BITS;
                        if (brings_k) raw_k[i].load(kp + from);
                        if (brings_v) raw_v[i].load(vp + from);
                    }
                }
            };
            if (BITS == 16 && DP == 8 * RC && pieces == RC)
                bring(std::true_type{});
            else
                bring(std::false_type{});
            if constexpr (BITS < 16)                                   // lanes 0 ... 15 the steps of the keys, 16 ... 31 those of the values
                raw_step = *reinterpret_cast<const uint32_t *>(((self & 16u) ? a.cache.v_step : a.cache.k_step) + 4u * (at + (self & 15u)));
        };
        auto arrive = [&](uint32_t t, auto buffer) {
            const int b = buffer;
            uint4 *lds_k = b ? lds_k1 : lds_k0, *lds_v = b ? lds_v1 : lds_v0;
            const uint32_t key0 = t * KT + 16u * group16, self = here(lane);
            if constexpr (BITS == 16) {
                __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): what went straight to LDS is there
                asm volatile("" ::: "memory");
                if ((t + 1u) * KT > all_see && brings_v) {
                    // Some rows do not see all of this tile.  What no row sees may be anything: zeros; and values that are not finite are
                    // left out here, so that a weight of 0 makes nothing of them (they are added at the end in the rows that see them).
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < kIssues; ++i) {
                        const uint32_t x = 64u * i + self, at = (16u * group16) * RC + x;
                        uint4 v = lds_v[at];
                        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (uint32_t &y : w) {
                            y = key0 + x / RC < end ? y : 0u;
                            const uint32_t keep = (half_finite(y) ? 0xFFFFu : 0u) | (half_finite(y >> 16) ? 0xFFFF0000u : 0u);
                            odd |= keep != 0xFFFFFFFFu;
                            y &= keep;
                        }
                        lds_v[at] = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (odd) lds_odd[b] = 1u;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kIssues; ++i) {
                    const uint32_t x = 64u * i + self, r = x / RC, c = x % RC, kk = 16u * group16 + r;
                    if (c < pieces) {
                        if (brings_k) lds_k[kk * RC + (c ^ k_swap<RC>(kk))] = code_values<BITS, kSlots>(raw_k[i]);
                        if (brings_v) lds_v[kk * RC + (c ^ v_swap<RC>(kk))] = code_values<BITS, kSlots>(raw_v[i]);
                    }
                }
                const bool in = key0 + (lane & 15u) < end;
                float step = !in ? 0.0f : BITS == 8 ? __uint_as_float(raw_step) : step_of(raw_step);
                float low = !in || BITS == 8 ? 0.0f : low_of(raw_step);
                float f = lane < 16u ? scale : 1.0f, reach = reach_of(step);
                if constexpr (kStepInExponent)
                    if (lane >= 16u) {
                        // What is not finite goes into the exponent alone, and so to the rows that see the key: a node that was left out may have a
                        // step that is none.  (8-bit steps below the least count as that: 127 of it are less than half of FP16's least value.)
                        const bool none = !(finite(step) && finite(low));
                        if (none || step < kLeastStep) low += 8.0f * kLeastStep, step = kLeastStep;
                        reach = none ? __builtin_nanf("") : __builtin_amdgcn_logf(step);
                        f = __builtin_amdgcn_rcpf(step);
                        if (none) low = 0.0f;
                        step = 1.0f;
                    }
                if (lane < 32u) {
                    lds_step[b][lane >> 4][0][16u * group16 + (lane & 15u)] = f * step;
                    if constexpr (BITS == 4) lds_step[b][lane >> 4][1][16u * group16 + (lane & 15u)] = f * low;
                    if (lane >= 16u) lds_reach[b][16u * group16 + (lane & 15u)] = reach;
                }
            }
        };

        auto hold = []() {                                             // (with codes there are not the registers for it)
            if constexpr (BITS == 16) __builtin_amdgcn_sched_barrier(0);
        };
        typedef float f32x16 __attribute__((ext_vector_type(16)));
        f32x16 acc[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[i][x] = 0.0f;
        // m: the maximum that weights are taken against, as in the kernel for few rows; it may lie up to 8 below the true one
        float m = kNone, m_true = kNone, l = 0.0f, z_acc = 0.0f;

        auto compute = [&](uint32_t t, auto buffer) {
            const int b = buffer;
            const uint4 *lds_k = b ? lds_k1 : lds_k0, *lds_v = b ? lds_v1 : lds_v0;
            const uint32_t key0 = t * KT;
            const bool masked = key0 + KT > all_see;                   // not all rows see all of the tile
            float w[16 * kHalves];
            // What is read of K and V is asked for a few products ahead, V's first half before the weights are worked out.  (Left to the
            // compiler, the reads come pair by pair right before their products, and a wavefront waits for each: 140 us
            // in the place of 133 for 2048 tokens over 4096 keys.)
            half8v kf[kHalves][kSteps];
            const uint32_t key_n = here(n);
            auto read_k = [&](int y) {
#pragma unroll
                for (int x = 0; x < kHalves; ++x) {
                    const uint32_t key = 32u * (half0 + x) + key_n;
                    kf[x][y] = __builtin_bit_cast(half8v, lds_k[key * RC + ((2u * y + h) ^ k_swap<RC>(key))]);
                }
            };
            constexpr int kAhead = kSteps < 4 ? kSteps : 4;
#pragma unroll
            for (int y = 0; y < kAhead; ++y) read_k(y);
            hold();
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            const uint32_t i16 = lane & 15u, sub = (lane >> 4) & 1u;   // a lane of 16: row i16 / 4 of four keys, values 4 (i16 % 4) ... + 3
            constexpr int kReads = 4 * kHalves * kTiles;               // [16 keys][8 of them][32 values]
            s16x4 vf[kReads];
            auto read_v = [&](int i) {
                const int x = i / (2 * kTiles), y = i % (2 * kTiles) / 2, e = i % 2;
                const uint32_t key = 32u * half0 + 16u * x + 8u * e + 4u * h + i16 / 4u;
                const uint32_t c = 4u * y + 2u * sub + ((i16 >> 1) & 1u);
                const uint4 *p = &lds_v[key * RC + (c ^ v_swap<RC>(key))];
                vf[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(reinterpret_cast<const uint2 *>(p) + (i16 & 1u)));
            };
            f32x16 c[kHalves];
#pragma unroll
            for (int x = 0; x < kHalves; ++x) c[x] = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int y = 0; y < kSteps; ++y) {
#pragma unroll
                for (int x = 0; x < kHalves; ++x) c[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[x][y], q[y], c[x], 0, 0, 0);
                if (y + kAhead < kSteps) read_k(y + kAhead);
                if (y >= kSteps - kAhead)
#pragma unroll
                    for (int i = (y + kAhead - kSteps) * (kReads / 2) / kAhead; i < (y + 1 + kAhead - kSteps) * (kReads / 2) / kAhead; ++i) read_v(i);
                hold();
            }
#pragma unroll
            for (int i = 0; i < 16 * kHalves; ++i) w[i] = c[i / 16][i % 16];
            if constexpr (BITS < 16) {
#pragma unroll
                for (int i = 0; i < 16 * kHalves; i += 4) {            // (the steps of the keys have the scale in them)
                    const uint32_t key = 32u * half0 + 8u * (i / 4) + 4u * h;
                    const f32x4 step = *reinterpret_cast<const f32x4 *>(&lds_step[b][0][0][key]);
                    if constexpr (kStepInExponent) {
                        f32x4 more = *reinterpret_cast<const f32x4 *>(&lds_reach[b][key]);
                        if constexpr (BITS == 4) {
                            const f32x4 low = *reinterpret_cast<const f32x4 *>(&lds_step[b][0][1][key]);
#pragma unroll
                            for (int r = 0; r < 4; ++r) more[r] = fmaf(low[r], q_sum, more[r]);
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[i + r] = fmaf(w[i + r], step[r], more[r]);
                    } else if constexpr (BITS == 4) {
                        const f32x4 low = *reinterpret_cast<const f32x4 *>(&lds_step[b][0][1][key]) * q_sum;
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[i + r] = fmaf(w[i + r], step[r], low[r]);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) w[i + r] *= step[r];
                    }
                }
            }
            if (TREE && masked) {
                if constexpr (TREE)
#pragma unroll
                    for (int x = 0; x < kHalves; ++x) {
                        const uint32_t bits = seen_bits(a, here(s.first + token), key0 + 32u * (half0 + x), s.behind, end) >> (4u * h);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(bits >> (8 * (i / 4) + (i & 3)) & 1u)) w[16 * x + i] = kNone;
                    }
            } else if (masked) {
                int32_t left = seen - (int32_t)(key0 + 32u * half0 + 4u * h);
                asm volatile("" : "+v"(left));                         // (kept a branch: few tiles take it)
#pragma unroll
                for (int i = 0; i < 16 * kHalves; ++i)
                    if (8 * (i / 4) + (i & 3) >= left) w[i] = kNone;
            }
            float most = kNone;
            if constexpr (BITS == 16 || kStepInExponent) {
#pragma unroll
                for (int i = 0; i < 16 * kHalves; ++i) most = fmaxf(most, w[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 16 * kHalves; i += 4) {
                    const f32x4 reach = *reinterpret_cast<const f32x4 *>(&lds_reach[b][32u * half0 + 8u * (i / 4) + 4u * h]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, w[i + r] + reach[r]);
                }
            }
            const float m_new = m_true = fmaxf(m_true, max_over_32(most) * by);
            if (const bool far = m_new > m + 8.0f; __any((int)far)) {
                const float alpha = far ? __builtin_amdgcn_exp2f(m - m_new) : 1.0f;       // (0 where nothing was seen before)
                m = far ? m_new : m;                                   // a row goes by its own scores alone
                l *= alpha;
                z_acc *= alpha;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc[i] *= alpha;
            }
            const float base = m == kNone ? 0.0f : m;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 16 * kHalves; ++i) {
                w[i] = __builtin_amdgcn_exp2f(BITS == 16 ? fmaf(w[i], by, -base) : w[i] - base);
                if constexpr (kParts == 2 || (BITS < 16 && !kStepInExponent)) sum += w[i];  // (with FP16 in one part the rounded ones are added up, below)
            }
            if constexpr (BITS < 16) {
#pragma unroll
                for (int i = 0; i < 16 * kHalves; i += 4) {
                    const uint32_t key = 32u * half0 + 8u * (i / 4) + 4u * h;
                    const f32x4 step = *reinterpret_cast<const f32x4 *>(&lds_step[b][1][0][key]);
                    if constexpr (BITS == 4) {
                        const f32x4 low = *reinterpret_cast<const f32x4 *>(&lds_step[b][1][1][key]);
#pragma unroll
                        for (int r = 0; r < 4; ++r) z_acc = fmaf(w[i + r], low[r], z_acc);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if constexpr (kStepInExponent)
                            sum = fmaf(w[i + r], step[r], sum);
                        else
                            w[i + r] *= step[r];
                }
            }
            half8v weights[2 * kHalves], rest[2 * kHalves];
#pragma unroll
            for (int x = 0; x < 2 * kHalves; ++x) {
                uint32_t o[4], e[4] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[i] = as_word(half2v{(_Float16)w[8 * x + 2 * i], (_Float16)w[8 * x + 2 * i + 1]});
                    if constexpr (kParts == 2) {                   // what that leaves out, as in the kernel for few rows
                        asm("" : "+v"(o[i]));
                        const half2v p = as_half2(o[i]);
                        e[i] = as_word(half2v{(_Float16)(w[8 * x + 2 * i] - (float)p[0]), (_Float16)(w[8 * x + 2 * i + 1] - (float)p[1])});
                    } else if constexpr (BITS == 16) {
                        sum = __builtin_amdgcn_fdot2(as_half2(o[i]), half2v{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
                    }
                }
                weights[x] = as_half8(o[0], o[1], o[2], o[3]);
                rest[x] = as_half8(e[0], e[1], e[2], e[3]);
            }
            l += sum;
#pragma unroll
            for (int x = 0; x < 2 * kHalves; ++x)
#pragma unroll
                for (int y = 0; y < kTiles; ++y) {
                    const int at = x * kTiles + y;
                    const uint2 lo = __builtin_bit_cast(uint2, vf[2 * at]), hi = __builtin_bit_cast(uint2, vf[2 * at + 1]);
                    acc[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_half8(lo.x, lo.y, hi.x, hi.y), weights[x], acc[y], 0, 0, 0);
                    if constexpr (kParts == 2) acc[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_half8(lo.x, lo.y, hi.x, hi.y), rest[x], acc[y], 0, 0, 0);
                    if (2 * at + 1 + kReads / 2 < kReads) {
                        read_v(2 * at + kReads / 2);
                        read_v(2 * at + 1 + kReads / 2);
                        hold();
                    }
                }
        };

        auto step = [&](uint32_t t, auto buffer, auto other) {
            if (t + 1u < t1) request(t + 1u, other);
            if (t * KT < wave_end) compute(t, buffer);
            if (t + 1u < t1) arrive(t + 1u, other);
            __syncthreads();
        };
        if (t0 < t1) {
            const std::integral_constant<int, 0> first;
            const std::integral_constant<int, 1> second;
            request(t0, first);
            arrive(t0, first);
            __syncthreads();
            if constexpr (BITS == 16) {
                for (uint32_t t = t0; t < t1; t += 2u) {
                    step(t, first, second);
                    if (t + 1u < t1) step(t + 1u, second, first);
                }
            } else {                                                   // (nothing goes straight to LDS: one copy of the code, and fewer registers)
                for (uint32_t t = t0, b = 0; t < t1; ++t, b ^= 1u) step(t, (int)b, (int)(b ^ 1u));
            }
        }

        if constexpr (BITS == 16) {
            // Where V was not finite, as in the kernel for few rows
            bool odd = (lds_odd[0] | lds_odd[1]) != 0u;
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    odd |= !finite(acc[y][i]);
                    acc[y][i] = finite(acc[y][i]) ? acc[y][i] : 0.0f;
                }
            if (__any((int)odd)) {
                const uint32_t last = min(t1 * KT, end);
#pragma unroll 1
                for (uint32_t key = t0 * KT; key < last; ++key) {
                    if constexpr (TREE) {
                        if (!(seen_bits(a, s.first + token, key, s.behind, end) & 1u)) continue;
                    } else {
                        if ((int32_t)key >= seen) continue;
                    }
                    const uint64_t at = (uint64_t)page_of(a, s.table, key) * page_rows + head_rows + (key & page_mask);
                    const uint16_t *vp = reinterpret_cast<const uint16_t *>(a.cache.v + at * a.cache.row_bytes);
#pragma unroll
                    for (int y = 0; y < kTiles; ++y)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t d = 32u * y + 8u * (i / 4) + 4u * h + (i & 3);
                            if (d < dim && !half_finite(vp[d])) acc[y][i] += half_to_float(vp[d]);
                        }
                }
            }
        }

        l += __shfl_xor(l, 32, 64);
        if constexpr (BITS == 4) z_acc += __shfl_xor(z_acc, 32, 64);
        if constexpr (kShared == 2) {
            // the second half's results to the wavefront that has the first (the last tile has been waited for by all)
            const uint32_t pair = wave & 1u;
            uint4 *to = pair ? lds_v0 : lds_k0;
            if (wave >= 2u) {
#pragma unroll
                for (int y = 0; y < kTiles; ++y)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        to[64u * (4 * y + i) + lane] = __builtin_bit_cast(uint4, f32x4{acc[y][4 * i], acc[y][4 * i + 1], acc[y][4 * i + 2], acc[y][4 * i + 3]});
                if (h == 0) lds_mlz[pair][0][n] = m, lds_mlz[pair][1][n] = l, lds_mlz[pair][2][n] = z_acc;
            }
            __syncthreads();
            if (wave >= 2u) return;
            const float other = lds_mlz[pair][0][n], top = fmaxf(m, other), f0 = share_of(m, top), f1 = share_of(other, top);
            m = top;
            l = f0 * l + f1 * lds_mlz[pair][1][n];
            z_acc = f0 * z_acc + f1 * lds_mlz[pair][2][n];
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 o = __builtin_bit_cast(f32x4, to[64u * (4 * y + i) + lane]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[y][4 * i + r] = f0 * acc[y][4 * i + r] + f1 * o[r];
                }
        }
        if constexpr (kSlots)                                          // a lane's 0 4 1 5 or 2 6 3 7 become 0 1 2 3 or 4 5 6 7
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const auto even = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[y][i]), __float_as_uint(acc[y][i + 1]), false, false);
                    const auto odd = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[y][i + 2]), __float_as_uint(acc[y][i + 3]), false, false);
                    acc[y][i] = __uint_as_float(even[0]), acc[y][i + 1] = __uint_as_float(odd[0]);
                    acc[y][i + 2] = __uint_as_float(even[1]), acc[y][i + 3] = __uint_as_float(odd[1]);
                }
        const uint32_t out_row = wave_row + n;
        if (out_row >= rows) return;
        const uint32_t out_head = head * a.group + (row - token * a.group);
        if (splits == 1u) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t *p = a.out.data + (int64_t)(s.first + token) * a.out.token_stride + (int64_t)out_head * a.out.head_stride;
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint32_t d = 32u * y + 8u * (i / 4) + 4u * h;
                    if (d >= dim) continue;
                    uint32_t o[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        o[r] = as_word(half2v{to_result((acc[y][i + 2 * r] + z_acc) * inv), to_result((acc[y][i + 2 * r + 1] + z_acc) * inv)});
                    if (a.out_wide) {
                        *reinterpret_cast<uint2 *>(p + d) = make_uint2(o[0], o[1]);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) p[(int64_t)(d + r) * a.out.dim_stride] = (uint16_t)(o[r >> 1] >> (16 * (r & 1)));
                    }
                }
        } else {
            uint64_t at = ((uint64_t)split * a.tokens + s.first + token) * a.q_heads + out_head;
            if constexpr (TREE)
                if (a.balanced) at = ((uint64_t)base + split * rows + out_row) * a.cache.heads + head;
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint32_t d = 32u * y + 8u * (i / 4) + 4u * h;
                    if (d < dim)
                        *reinterpret_cast<f32x4 *>(a.part_o + at * dim + d) =
                            f32x4{acc[y][i] + z_acc, acc[y][i + 1] + z_acc, acc[y][i + 2] + z_acc, acc[y][i + 3] + z_acc};
                }
            if (h == 0) a.part_ml[2 * at] = m, a.part_ml[2 * at + 1] = l;
        }
    };
    if constexpr (kByRows) {
        if (rows - row0 <= 64u)
            work(std::integral_constant<int, 2>());
        else
            work(std::integral_constant<int, 1>());
    } else {
        work(std::integral_constant<int, ON_KEYS>());
    }
}

// ---- joining the splits ----------------------------------------------------------------------------------------------------------------
//
// For each (token, head) the parts of its splits, each taken to the largest of their maxima:
//   o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s
// What bounds it is the trip to memory, so that what a row needs is asked for at once and rows are many to a compute unit.
//
// Where a row's parts are: the s-th is row first + s * step of the partial results.  With shares of several sequences by their lengths
// a row belongs to one of them, whose splits and place the first launch has written down.
struct Parts {
    uint64_t first, step;
    uint32_t splits;                      // 0: nothing to join
};

template <bool TREE, uint32_t LANES>
__device__ __forceinline__ Parts parts_of(const ArgsOf<TREE> &a, uint32_t token, uint32_t head)
{
    if constexpr (TREE) {
        if (a.balanced) {
            // the last sequence that starts at this token or before it, for each of the wavefront's rows
            const uint32_t lane = threadIdx.x & 63u;
            const ecs::AttentionTreeArgs::Words mine = a.plan[lane];
            uint32_t b = 0;
#pragma unroll
            for (uint32_t r = 0; r < 64u; r += LANES) {
                const uint32_t of = (uint32_t)__builtin_amdgcn_readlane((int)token, (int)r);
                const uint32_t count = (uint32_t)__popcll(__ballot(mine.z <= of));
                if (lane >= r) b = max(count, 1u) - 1u;
            }
            const uint32_t splits = (uint32_t)__shfl((int)mine.x, (int)b, 64), base = (uint32_t)__shfl((int)mine.y, (int)b, 64);
            const uint32_t first = (uint32_t)__shfl((int)mine.z, (int)b, 64), news = (uint32_t)__shfl((int)mine.w, (int)b, 64);
            const uint32_t in = token - first, rows = news * a.group;
            if (token < first || in >= news || splits < 2u) return {0, 0, 0};
            const uint32_t of_cache = head / a.group, row = in * a.group + (head - of_cache * a.group);
            return {((uint64_t)base + row) * a.cache.heads + of_cache, (uint64_t)rows * a.cache.heads, splits};
        }
    }
    return {(uint64_t)token * a.q_heads + head, (uint64_t)a.tokens * a.q_heads, a.splits};
}

// Few rows: a workgroup for each, its wavefronts on different splits.
template <bool TREE>
__global__ __launch_bounds__(256) void attention_join_splits_kernel(const ArgsOf<TREE> a)
{
    __shared__ float lds_o[4][256];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, dim = a.cache.dim;
    const uint32_t r = blockIdx.x, token = r / a.q_heads, head = r - token * a.q_heads;
    if ((int32_t)token < a.q_start[0] || (int32_t)token >= a.q_start[a.batch]) return;            // of no sequence (the whole workgroup)
    const Parts parts = parts_of<TREE, 64>(a, token, head);
    if (TREE && parts.splits == 0) return;
    const uint64_t row = parts.first, step = parts.step;
    const uint32_t splits = TREE ? parts.splits : a.splits;
    float l = 0.0f, o[4] = {0, 0, 0, 0}, top = kNone;
    // 64 splits at a time: a lane looks at one, its share goes to the others by readlane, so that all that is waited for is two trips
    for (uint32_t first = 0; first < splits; first += 64u) {
        const uint32_t s = first + lane;
        const float2 ml = s < splits ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * (row + s * step)) : make_float2(kNone, 0.0f);
        float m = ml.x;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
        m = fmaxf(m, top);
        const float before = share_of(top, m);
        top = m;
        const float share = share_of(ml.x, m);
        l = l * before + share * ml.y;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= before;
        const uint32_t count = min(splits - first, 64u);
        for (uint32_t k = wave; k < count; k += 16u) {             // four splits of this wavefront on their way
            float x[4][4], f[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) {
                const uint32_t at = min(k + 4u * u, count - 1u);
                f[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(share), (int)at));
                if (k + 4u * u >= count) f[u] = 0.0f;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) x[u][i] = lane + 64u * i < dim ? a.part_o[(row + (first + at) * step) * dim + lane + 64u * i] : 0.0f;
            }
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u)
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) o[i] = f[u] == 0.0f ? o[i] : fmaf(f[u], x[u][i], o[i]);
        }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);    // (every wavefront has looked at all of them)
#pragma unroll
    for (int i = 0; i < 4; ++i) lds_o[wave][lane + 64u * i] = o[i];
    __syncthreads();
    if (tid >= dim) return;
    const float sum = lds_o[0][tid] + lds_o[1][tid] + lds_o[2][tid] + lds_o[3][tid];
    a.out.data[(int64_t)token * a.out.token_stride + (int64_t)head * a.out.head_stride + (int64_t)tid * a.out.dim_stride] =
        __builtin_bit_cast(uint16_t, to_result(l == 0.0f ? 0.0f : sum / l));
}

// Many rows, which have few splits: L lanes for each, four values a lane, four splits on their way.
template <int L, bool TREE>
__global__ __launch_bounds__(256) void attention_join_rows_kernel(const ArgsOf<TREE> a)
{
    const uint32_t r = blockIdx.x * (256u / L) + threadIdx.x / L, d = 4u * (threadIdx.x % L), dim = a.cache.dim;
    const uint32_t token = r / a.q_heads, head = r - token * a.q_heads;
    const Parts parts = parts_of<TREE, L>(a, token, head);         // (by the whole wavefront)
    if (token >= a.tokens || d >= dim) return;
    const int32_t first = a.q_start[0], last = a.q_start[a.batch];
    const uint64_t row = parts.first, step = parts.step;
    const uint32_t splits = TREE ? parts.splits : a.splits;
    if (TREE && splits == 0) return;
    float l = 0.0f, top = kNone;
    f32x4 o = {0, 0, 0, 0};
    for (uint32_t s = 0; s < splits; s += 4u) {
        float2 ml[4];
        f32x4 x[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint64_t at = row + min(s + u, splits - 1u) * step;
            ml[u] = *reinterpret_cast<const float2 *>(a.part_ml + 2 * at);
            x[u] = *reinterpret_cast<const f32x4 *>(a.part_o + at * dim + d);
        }
        float m = top;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) m = fmaxf(m, ml[u].x);    // (the last one, read again, changes nothing)
        const float before = share_of(top, m);
        top = m;
        l *= before;
        o *= before;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            if (s + u >= splits) continue;
            // (a split without a maximum has added up nothing, or scores that are all NaN: its sums are then NaN, and have to stay)
            const float share = share_of(ml[u].x, m);
            l = fmaf(share, ml[u].y, l);
            o += share * x[u];
        }
    }
    if ((int32_t)token < first || (int32_t)token >= last) return;  // of no sequence
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t *p = a.out.data + (int64_t)token * a.out.token_stride + (int64_t)head * a.out.head_stride;
    const uint32_t w0 = as_word(half2v{to_result(o[0] * inv), to_result(o[1] * inv)});
    const uint32_t w1 = as_word(half2v{to_result(o[2] * inv), to_result(o[3] * inv)});
    if (a.out_wide) {
        *reinterpret_cast<uint2 *>(p + d) = make_uint2(w0, w1);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[(int64_t)(d + i) * a.out.dim_stride] = (uint16_t)((i < 2 ? w0 : w1) >> (16 * (i & 1)));
    }
}

template <int BITS>
int launch_rows(const ArgsOf<kTree> &a, void *stream)
{
#ifdef ECS_TREE
    const uint32_t gx = a.cache.heads, gy = std::min(a.slots, 32768u), gz = (a.slots + gy - 1u) / gy;
#else
    const uint32_t gx = a.row_tiles * a.splits, gy = a.cache.heads, gz = a.batch;
#endif
    switch (a.cache.dim) {
    case 64: return ecs::launch_args<attention_rows_kernel<BITS, 64, false, kTree>>(a, gx, gy, gz, 256, stream);
    case 128: return ecs::launch_args<attention_rows_kernel<BITS, 128, false, kTree>>(a, gx, gy, gz, 256, stream);
    case 256: return ecs::launch_args<attention_rows_kernel<BITS, 256, false, kTree>>(a, gx, gy, gz, 256, stream);
    default: break;
    }
    if (a.cache.dim < 64) return ecs::launch_args<attention_rows_kernel<BITS, 64, true, kTree>>(a, gx, gy, gz, 256, stream);
    if (a.cache.dim < 128) return ecs::launch_args<attention_rows_kernel<BITS, 128, true, kTree>>(a, gx, gy, gz, 256, stream);
    return ecs::launch_args<attention_rows_kernel<BITS, 256, true, kTree>>(a, gx, gy, gz, 256, stream);
}

template <int BITS, int ON_KEYS>
int launch_chunk(const ArgsOf<kTree> &a, void *stream)
{
#ifdef ECS_TREE
    const uint32_t gx = a.cache.heads, gy = std::min(a.slots, 32768u), gz = (a.slots + gy - 1u) / gy;
#else
    const uint32_t gx = a.cache.heads, gy = a.row_tiles * a.splits, gz = a.batch;
#endif
    const uint32_t width = (a.cache.dim + 31u) / 32u;
    switch (width) {
    case 1: return ecs::launch_args<attention_chunk_kernel<BITS, 32, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
    case 2: return ecs::launch_args<attention_chunk_kernel<BITS, 64, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
    case 3: return ecs::launch_args<attention_chunk_kernel<BITS, 96, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
    case 4: return ecs::launch_args<attention_chunk_kernel<BITS, 128, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
    default: break;
    }
    if constexpr (!kTree || ON_KEYS == 2) {                        // (of trees, wider heads have 64 rows to a workgroup: plan_attention_tree)
        if (width == 5u) return ecs::launch_args<attention_chunk_kernel<BITS, 160, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
        if (width == 6u) return ecs::launch_args<attention_chunk_kernel<BITS, 192, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
        if (width == 7u) return ecs::launch_args<attention_chunk_kernel<BITS, 224, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
        return ecs::launch_args<attention_chunk_kernel<BITS, 256, kTree, ON_KEYS>>(a, gx, gy, gz, 256, stream);
    }
    return (int)hipErrorInvalidValue;
}

template <int BITS>
int launch_bits(const ArgsOf<kTree> &a, void *stream)
{
#ifdef ECS_TREE
    if (a.chunk == 2u) return launch_chunk<BITS, 2>(a, stream);
#endif
    return a.chunk ? launch_chunk<BITS, 1>(a, stream) : launch_rows<BITS>(a, stream);
}

int launch_join(const ArgsOf<kTree> &a, void *stream)
{
    // (us by a workgroup / by some lanes for each row: 320 rows of 25 splits 129 / 134, 1024 of 8 46.2 / 46.0; four bits, 1000 tokens of 32
    // heads, two splits, by a wavefront 95, by 32 lanes 86)
    const uint32_t rows = a.tokens * a.q_heads;
    if (rows < 2048u) return ecs::launch_args<attention_join_splits_kernel<kTree>>(a, rows, 1, 1, 256, stream);
    if (a.cache.dim <= 64u) return ecs::launch_args<attention_join_rows_kernel<16, kTree>>(a, (rows + 15u) / 16u, 1, 1, 256, stream);
    if (a.cache.dim <= 128u) return ecs::launch_args<attention_join_rows_kernel<32, kTree>>(a, (rows + 7u) / 8u, 1, 1, 256, stream);
    return ecs::launch_args<attention_join_rows_kernel<64, kTree>>(a, (rows + 3u) / 4u, 1, 1, 256, stream);
}

}  // namespace

namespace ecs {

#ifndef ECS_TREE
// Rows of a workgroup, and how many workgroups are wanted, in the kernel for few rows and in the one whose rows share keys in LDS
constexpr uint32_t kFewRows = 16, kFewWanted = 1024, kChunkRows = 128, kChunkWanted = 512;
// (token, head) rows per head of the cache up to which the kernel for few rows takes a call (figures at plan_attention)
static uint64_t rows_of_16(uint32_t dim, uint32_t bits) { return dim <= 128u && bits == 16u ? 16u : bits == 4u ? 64u : 32u; }
static uint64_t splits_of_keys(uint64_t max_kv) { return (max_kv + 255u) / 256u; }

AttentionPlan plan_attention(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint64_t tokens, uint32_t max_new,
                             uint64_t max_kv)
{
    AttentionPlan p = {};
    const uint64_t rows = (uint64_t)max_new * group;
    // 128 rows that share their keys in LDS, or 16 a workgroup that each bring them: us by 16 / by 128, 24 rows on 8003 keys of four
    // sequences, heads of 128, 32.3 / 29.0, in 8 bits 32.8 / 35.7, in 4 28.2 / 38.9; 48 rows 66 / 33, 45.5 / 41.5, 37.4 / 45.5; 64 rows on
    // 564 keys 36 / 23, 29.7 / 25.6, 24.1 / 28.9; heads of 256, 32 rows, 17.5 / 27.5.
    p.chunk = rows > rows_of_16(dim, bits);
    const uint64_t per_tile = p.chunk ? kChunkRows : kFewRows;
    p.row_tiles = (uint32_t)((rows + per_tile - 1u) / per_tile);
    const uint64_t blocks = (uint64_t)p.row_tiles * kv_heads * batch;
    // Enough workgroups for the chip, and two rounds of 32 keys for each wavefront of a split (four tiles of 64 for a workgroup).  More and
    // smaller ones cost more in partial results than they gain (us by 512 / 1024 workgroups of 128 rows: 1024 tokens over 2048, heads of
    // 128, 54 / 69, 512 over 9098 111 / 131, 200 over 2000 of three sequences, 4 bits, 52 / 61; 1024 / 2048 of 16 rows: 8 tokens over 32768
    // 129 / 136, in 8 bits 77 / 89).  Several sequences whose chunks just fill the chip are split in two all the same: otherwise the
    // longest one's workgroups are what the others wait for.  That is a bet on lengths that differ, which the host does not see (heads of 128, whole / in
    // two, FP16, 8 and 4 bits: five of up to 333 tokens over up to 3000 keys 91 / 83, 108 / 115, 112 / 88, other lengths 80 / 74, 103 / 84, 109 / 87;
    // five of one length 128 / 147, 150 / 166, 151 / 169).  With more workgroups than the chip holds at once the next one starts where one ends, and two
    // splits cost in both cases (eight sequences 97 / 100, 149 / 155, 136 / 151, of one length 208 / 226; twelve 147 / 167, 189 / 190, 157 / 160).
    const uint64_t wanted = p.chunk ? kChunkWanted : kFewWanted, by_keys = splits_of_keys(max_kv);
    uint64_t by_chip = blocks ? wanted / blocks : 1u;
    if (p.chunk && batch > 1u && by_chip == 1u) by_chip = 2u;
    p.splits = (uint32_t)std::max<uint64_t>(1u, std::min(by_chip, by_keys));
    if (p.splits > 1u) p.work_bytes = (uint64_t)p.splits * tokens * kv_heads * group * (dim + 2u) * sizeof(float);
    return p;
}

// Of trees.  Rows per workgroup: 16 that bring their keys themselves, or 64 or 128 that share them in LDS; us by 16 / 64 / 128 (heads of 128 where not
// said): 32 rows on up to 8000 keys of four sequences FP16 - / 75 / 80, 8 bits 45.6 / 54.0 / -, 4 bits 48 / 69 / -; 40 on 3000, 4 bits, 72.9 / 68.5 / -; 64 on
// 8000, 8 bits, - / 77 / 87, 4 bits 72 / 64 / -; 100 on 4000, FP16, - / 34.5 / 37.5; 128 on 8192 of sixteen, 8 bits, - / 156 / 125, FP16 equal; heads of 256,
// 128 rows on 8000, FP16, - / 39.5 / 46.8, 192 of four, 8 bits, - / 27.5 / 36.6.
constexpr uint32_t kHalfRows = 64;
static uint32_t tree_rows_of_16(uint32_t dim, uint32_t bits) { return dim <= 128u && bits == 16u ? kFewRows : 2u * kFewRows; }

TreePlan plan_attention_tree(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint32_t max_new, uint64_t tokens,
                             uint64_t max_kv)
{
    TreePlan t = {};
    const uint64_t rows = (uint64_t)max_new * group;
    t.chunk = rows <= tree_rows_of_16(dim, bits) ? 0u : dim > 128u || rows <= kHalfRows ? 2u : 1u;
    const uint32_t per_tile = t.chunk == 0u ? kFewRows : t.chunk == 1u ? kChunkRows : kHalfRows;
    t.row_tiles = (uint32_t)((rows + per_tile - 1u) / per_tile);
    // Pieces for the workgroups that the chip holds at once, by the kernels' registers and LDS (heads of 256, 8 tokens over 8000 keys in FP16: by 1024
    // workgroups 22.3 us, by 256 20.1; two of up to 8000 in 8 bits, heads of 128, 1024 41.5, 768 37.9)
    const uint64_t resident = t.chunk ? (dim > 128u ? 256u : 512u) : dim <= 64u ? 1024u : dim <= 128u ? 768u : bits == 4u ? 512u : 256u;
    const uint64_t at_once = resident / kv_heads, items = (uint64_t)batch * t.row_tiles;
    t.splits = 1;
    t.slots = items;
    if (batch > kTreeSequences) {                                  // (more sequences than the lanes of a wavefront: equal splits for all)
        t.splits = (uint32_t)std::max<uint64_t>(1u, std::min(at_once / std::max<uint64_t>(items, 1u), splits_of_keys(max_kv)));
        t.slots = items * t.splits;
        if (t.splits > 1u) t.work_bytes = (uint64_t)t.splits * tokens * kv_heads * group * (dim + 2u) * sizeof(float);
    } else if (max_kv > whole_keys(t.chunk == 0u, bits < 16u) && (batch > 1u ? items < 2u * at_once : items < at_once)) {
        // (one sequence with a tile of rows for every workgroup, and several that fill the chip twice over, are left whole)
        t.balanced = 1;
        t.at_once = (uint32_t)at_once;
        t.slots = std::max(items, at_once);
        t.part_rows = (uint32_t)std::min<uint64_t>(t.slots * per_tile, splits_of_keys(max_kv) * std::min<uint64_t>(tokens, (uint64_t)batch * max_new) * group);
        t.work_bytes = kTreePlanBytes + (uint64_t)t.part_rows * kv_heads * (dim + 2u) * sizeof(float);
    }
    return t;
}

uint64_t most_attention_work(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint64_t tokens, uint32_t max_new,
                             uint64_t max_kv)
{
    // A workgroup takes up to per_tile rows, and there are splits only while they are no more than `wanted` (twice that where two splits are the
    // least, and for trees of several sequences): so many rows of partial results at most, whatever the call; and no more splits than the keys allow.
    const uint64_t few = rows_of_16(dim, bits), by_keys = splits_of_keys(max_kv);
    uint64_t most = 0;
    if (group <= few) most = (uint64_t)kFewWanted * kFewRows * (batch > 1u ? 2u : 1u);
    if ((uint64_t)max_new * group > tree_rows_of_16(dim, bits)) most = std::max<uint64_t>(most, (uint64_t)kChunkWanted * kChunkRows * (batch > 1u ? 2u : 1u));
    if (by_keys <= 1u) return 0;
    const uint64_t rows = std::min<uint64_t>(tokens, (uint64_t)batch * max_new) * kv_heads * group;
    return kTreePlanBytes + std::min(most, by_keys * rows) * (dim + 2u) * sizeof(float);
}

int launch_attention(const AttentionArgs &a, void *stream)
#else
int launch_attention_tree(const AttentionTreeArgs &a, void *stream)
#endif
{
    const int e = a.cache.bits == 16 ? launch_bits<16>(a, stream) : a.cache.bits == 8 ? launch_bits<8>(a, stream) : launch_bits<4>(a, stream);
    return e || !a.joins() ? e : launch_join(a, stream);
}

}  // namespace ecs
