// Arguments and host-callable launches of the kernels around the products: the paged cache of keys and values (kv_cache.hip),
// attention over it (attention.hip) and the check of drafted tokens (verify.hip).  Each launch returns a hipError_t value as int.
#ifndef ECSPMV_SERVE_H
#define ECSPMV_SERVE_H

#include <stddef.h>
#include <stdint.h>

namespace ecs {

// (token, head, element) -> data[token * token_stride + head * head_stride + element * dim_stride]
struct View {
    uint16_t *data;
    int64_t token_stride, head_stride, dim_stride;
};

// [page][head][place in the page][head_dim] codes, [page][head][place] steps
struct Cache {
    uint8_t *k, *v, *k_step, *v_step;
    uint32_t pages, heads, page_shift, dim;
    uint32_t bits, row_bytes;             // bytes of one token's codes of one head
};

struct KvArgs {
    Cache cache;
    View k, v;
    const int64_t *slots;
    uint32_t tokens, lanes_shift;         // log2 of the lanes that share a row
    uint32_t run_shift;                   // log2 of the neighbouring tokens of a head that follow one another
    uint32_t k_wide, v_wide;              // rows of k, v are 16-byte pieces
};
int launch_kv_write(const KvArgs &a, void *stream);
int launch_kv_read(const KvArgs &a, void *stream);

struct AppendArgs {
    Cache cache;
    View q, q_out, k, v;
    const int64_t *slots;
    const int32_t *position;
    const double *frequency;              // of each pair
    uint32_t tokens, q_heads, pairs, neighbours;
    uint32_t lanes_shift, run_shift;      // as in KvArgs, but a lane has 16 values
    uint32_t heads_per_block, q_blocks;   // heads of q, or of k and v, that a workgroup takes; workgroups for q
    uint32_t q_wide, q_out_wide, k_wide, v_wide;
    uint32_t q_columns, q_out_columns, kv_columns;              // tokens follow one another, from aligned places on: runs of 16 go through LDS
};
int launch_kv_append(AppendArgs &a, void *stream);                         // (chooses lanes_shift, heads_per_block, q_blocks, columns)

constexpr uint32_t kKeepLayers = 64;      // of a launch
struct KeepArgs {
    struct Tensors {
        uint8_t *k, *v, *k_step, *v_step;
    } layer[kKeepLayers];
    const int32_t *first, *path, *accepted, *table;
    int64_t path_stride, table_stride;
    uint32_t nodes, max_pages;
    uint32_t pages, heads, page_shift, row_bytes;
    uint32_t steps, blocks;               // whether rows have steps; workgroups to the keys or values of a layer
};
int launch_kv_keep(KeepArgs &a, uint32_t layers, uint32_t batch, void *stream);

struct AttentionArgs {
    Cache cache;
    View q, out;
    const int32_t *q_start, *kv_len, *table;
    int64_t table_stride;
    float *part_o, *part_ml;              // partial results of the splits (splits > 1)
    uint32_t tokens, q_heads, group;      // group: heads of q per head of the cache
    uint32_t batch, max_pages, max_new;
    uint32_t chunk, row_tiles, splits;    // chunk: 128 rows per workgroup instead of 16 (2, with trees: 64)
    uint32_t q_wide, out_wide;
    float scale_log2;                     // scale * log2(e)
    bool joins() const { return splits > 1u; }
};
struct AttentionPlan {
    uint32_t chunk, row_tiles, splits;
    uint64_t work_bytes;
};
AttentionPlan plan_attention(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint64_t tokens, uint32_t max_new,
                             uint64_t max_kv);
// the most that a call of no more sequences, tokens, new tokens of one and places asks for, if q has no rows beyond batch * max_new
uint64_t most_attention_work(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint64_t tokens, uint32_t max_new,
                             uint64_t max_kv);
int launch_attention(const AttentionArgs &a, void *stream);

constexpr uint32_t kTreeSequences = 64;   // that are dealt out by their lengths
constexpr uint32_t kTreePlanBytes = 16 * kTreeSequences;                  // of the workspace: four words for each
struct TreePlan : AttentionPlan {
    uint64_t slots;                       // workgroups to a head
    uint32_t balanced, part_rows;         // shares by the sequences' lengths; rows of partial results that there is room for
    uint32_t at_once;                     // balanced: workgroups to a head that the chip has at once
};
TreePlan plan_attention_tree(uint32_t batch, uint32_t kv_heads, uint32_t group, uint32_t dim, uint32_t bits, uint32_t max_new, uint64_t tokens,
                             uint64_t max_kv);
struct AttentionTreeArgs : AttentionArgs {
    const uint32_t *seen;                 // bit i of a token's words: it sees its sequence's i-th new token
    int64_t seen_stride;                  // words from one token to the next
    uint32_t seen_words;                  // words that count
    uint32_t slots, balanced, part_rows, at_once;               // as planned
    struct alignas(16) Words {
        uint32_t x, y, z, w;
    } *plan;                              // where shares are balanced, of each sequence: splits, first row of its partial results, first token, tokens
    bool joins() const { return balanced || splits > 1u; }
};
int launch_attention_tree(const AttentionTreeArgs &a, void *stream);

struct VerifyArgs {
    const float *target, *draft, *uniform;
    const int32_t *drafted, *count;
    int32_t *tokens, *accepted;
    int64_t target_seq, target_row, draft_seq, draft_row;      // strides in elements
    uint32_t drafts, vocab;
    double *sums;                         // verify_work_bytes
};
uint64_t verify_work_bytes(uint32_t batch, uint32_t vocab);
int launch_verify(const VerifyArgs &a, uint32_t batch, void *stream);

constexpr uint32_t kMostNodes = 1024;
struct VerifyTreeArgs {
    const float *target, *uniform;
    const int32_t *drafted, *parent, *count;
    int32_t *tokens, *path, *accepted;
    int64_t target_seq, target_row;       // strides in elements
    uint32_t nodes, vocab;
    uint8_t *work;                        // verify_tree_work_bytes
};
uint64_t verify_tree_work_bytes(uint32_t batch, uint32_t nodes, uint32_t vocab);
int launch_verify_tree(const VerifyTreeArgs &a, uint32_t batch, void *stream);

}  // namespace ecs
#endif
