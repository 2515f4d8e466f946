// C ABI around the products (see include/ecspmv.h): argument checks of the cache, the attention over it and the check of drafted
// tokens, in a row and in trees.  Nothing here allocates or can throw.
#include <cstdint>
#include <cstring>

#include "../../include/ecspmv.h"
#include "serve.h"
#include "status.h"

namespace {

template <class T>
int copy_struct(const T *from, T &to)
{
    std::memset(&to, 0, sizeof(T));
    if (!from || from->struct_size < sizeof(uint32_t)) return ECSPMV_ERR_INVALID;
    std::memcpy(&to, from, from->struct_size < sizeof(T) ? from->struct_size : sizeof(T));
    return ECSPMV_OK;
}

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1u)) == 0; }

int check_cache(const ecspmv_kv_cache_t *from, ecs::Cache &c)
{
    ecspmv_kv_cache_t t;
    const int s = copy_struct(from, t);
    if (s) return s;
    if (t.bits != 16 && t.bits != 8 && t.bits != 4) return ECSPMV_ERR_UNSUPPORTED;
    if (!t.k || !t.v || t.pages < 1 || t.heads < 1) return ECSPMV_ERR_INVALID;
    if (t.page_size < 16 || t.page_size > 1024 || (t.page_size & (t.page_size - 1))) return ECSPMV_ERR_UNSUPPORTED;
    if (t.head_dim < 16 || t.head_dim > 256 || t.head_dim % 16) return ECSPMV_ERR_UNSUPPORTED;
    if (t.pages > 0x7fffffff || t.heads > 65535) return ECSPMV_ERR_UNSUPPORTED;
    if (!aligned(t.k, 16) || !aligned(t.v, 16)) return ECSPMV_ERR_INVALID;
    if (t.bits != 16 && (!t.k_step || !t.v_step || !aligned(t.k_step, 16) || !aligned(t.v_step, 16))) return ECSPMV_ERR_INVALID;
    c.k = static_cast<uint8_t *>(t.k);
    c.v = static_cast<uint8_t *>(t.v);
    c.k_step = static_cast<uint8_t *>(t.k_step);
    c.v_step = static_cast<uint8_t *>(t.v_step);
    c.pages = (uint32_t)t.pages;
    c.heads = (uint32_t)t.heads;
    c.page_shift = (uint32_t)__builtin_ctz((unsigned)t.page_size);
    c.dim = (uint32_t)t.head_dim;
    c.bits = (uint32_t)t.bits;
    c.row_bytes = c.dim * c.bits / 8u;
    return ECSPMV_OK;
}

int check_view(const ecspmv_view_t *from, ecs::View &v, uint32_t &wide)
{
    if (!from || !from->data || !aligned(from->data, 2)) return ECSPMV_ERR_INVALID;
    v.data = static_cast<uint16_t *>(from->data);
    v.token_stride = from->token_stride;
    v.head_stride = from->head_stride;
    v.dim_stride = from->dim_stride;
    wide = v.dim_stride == 1 && v.token_stride % 8 == 0 && v.head_stride % 8 == 0 && aligned(v.data, 16);
    return ECSPMV_OK;
}

// Whether an output's values all have a place of their own, as far as a stride of 0 tells
bool spread_out(const ecspmv_view_t &v, int64_t tokens, int64_t heads)
{
    return (v.token_stride != 0 || tokens <= 1) && (v.head_stride != 0 || heads <= 1) && v.dim_stride != 0;
}

// log2 of the neighbouring tokens of a head that follow one another
uint32_t run_of_tokens(uint32_t tokens)
{
    uint32_t shift = 0;
    while ((1u << shift) < tokens && shift < 4u) ++shift;
    return shift;
}

int kv_call(const ecspmv_kv_cache_t *cache, const ecspmv_view_t *k, const ecspmv_view_t *v, const int64_t *d_slots, int64_t tokens,
            void *stream, int (*launch)(const ecs::KvArgs &, void *))
{
    ecs::KvArgs a;
    std::memset(&a, 0, sizeof(a));
    int s = check_cache(cache, a.cache);
    if (s) return s;
    if (tokens < 0) return ECSPMV_ERR_INVALID;
    if (tokens == 0) return ECSPMV_OK;
    if ((s = check_view(k, a.k, a.k_wide)) || (s = check_view(v, a.v, a.v_wide))) return s;
    if (!d_slots || !aligned(d_slots, 8)) return ECSPMV_ERR_INVALID;
    if (tokens > 0x7fffffff || ((uint64_t)tokens + 16u) * a.cache.heads > 0x7fffffffu) return ECSPMV_ERR_UNSUPPORTED;
    a.slots = d_slots;
    a.tokens = (uint32_t)tokens;
    while ((8u << a.lanes_shift) < a.cache.dim) ++a.lanes_shift;
    a.run_shift = run_of_tokens(a.tokens);
    return ecs::hip_status(launch(a, stream));
}

int check_attention(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *from, ecs::AttentionArgs &a, ecs::AttentionPlan &plan,
                    ecspmv_attention_t &t)
{
    std::memset(&a, 0, sizeof(a));
    int s = check_cache(cache, a.cache);
    if (s || (s = copy_struct(from, t))) return s;
    if (t.q_heads < 1 || (uint32_t)t.q_heads % a.cache.heads || t.tokens < 0 || t.batch < 0 || t.max_pages < 0 || t.max_new < 0)
        return ECSPMV_ERR_INVALID;
    if (t.batch > 65535 || t.tokens > 0x7fffffff || (uint64_t)t.tokens * (uint64_t)t.q_heads > 0x7fffffffu) return ECSPMV_ERR_UNSUPPORTED;
    a.tokens = (uint32_t)t.tokens;
    a.q_heads = (uint32_t)t.q_heads;
    a.group = a.q_heads / a.cache.heads;
    a.batch = (uint32_t)t.batch;
    a.max_pages = (uint32_t)t.max_pages;
    a.max_new = (uint32_t)t.max_new < a.tokens ? (uint32_t)t.max_new : a.tokens;
    if ((uint64_t)a.max_pages << a.cache.page_shift > 0x7fffffffu) return ECSPMV_ERR_UNSUPPORTED;
    plan = ecs::plan_attention(a.batch, a.cache.heads, a.group, a.cache.dim, a.cache.bits, a.tokens, a.max_new,
                               (uint64_t)a.max_pages << a.cache.page_shift);
    a.chunk = plan.chunk;
    a.row_tiles = plan.row_tiles;
    if ((uint64_t)plan.row_tiles * plan.splits > 65535u) return ECSPMV_ERR_UNSUPPORTED;          // (8 million rows: a grid's second dimension)
    a.splits = plan.splits;
    return ECSPMV_OK;
}

// What both attentions look at before they launch; `need`: bytes of the workspace
int check_tensors(const ecspmv_attention_t &t, uint64_t need, void *d_work, size_t work_bytes, ecs::AttentionArgs &args)
{
    int s;
    if ((s = check_view(&t.q, args.q, args.q_wide)) || (s = check_view(&t.out, args.out, args.out_wide))) return s;
    if (!t.q_start || !t.kv_len || !aligned(t.q_start, 4) || !aligned(t.kv_len, 4)) return ECSPMV_ERR_INVALID;
    if (args.max_pages && (!t.page_table || !aligned(t.page_table, 4) || t.table_stride < t.max_pages)) return ECSPMV_ERR_INVALID;
    if (need && (!d_work || !aligned(d_work, 16))) return ECSPMV_ERR_INVALID;
    if (work_bytes < need) return ECSPMV_ERR_TOO_SMALL;
    args.q_start = t.q_start;
    args.kv_len = t.kv_len;
    args.table = t.page_table;
    args.table_stride = t.table_stride;
    args.scale_log2 = t.scale * 1.44269504088896340736f;
    return ECSPMV_OK;
}

int check_attention_tree(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *from, ecs::AttentionTreeArgs &a, ecs::TreePlan &plan,
                         ecspmv_attention_t &t)
{
    std::memset(&a, 0, sizeof(a));
    ecs::AttentionPlan rows;
    const int s = check_attention(cache, from, a, rows, t);
    if (s) return s;
    plan = ecs::plan_attention_tree(a.batch, a.cache.heads, a.group, a.cache.dim, a.cache.bits, a.max_new, a.tokens,
                                    (uint64_t)a.max_pages << a.cache.page_shift);
    if (plan.slots > 0x7fffffffu) return ECSPMV_ERR_UNSUPPORTED;
    a.chunk = plan.chunk;
    a.row_tiles = plan.row_tiles;
    a.splits = plan.splits;
    a.slots = (uint32_t)plan.slots;
    a.balanced = plan.balanced;
    a.part_rows = plan.part_rows;
    a.at_once = plan.at_once;
    a.seen_words = (a.max_new + 31u) / 32u;
    return ECSPMV_OK;
}

bool nothing_to_compute(const ecs::AttentionArgs &a) { return a.tokens == 0 || a.batch == 0 || a.max_new == 0; }

int check_verify(const ecspmv_verify_t *from, ecspmv_verify_t &t)
{
    const int s = copy_struct(from, t);
    if (s) return s;
    if (t.batch < 0 || t.drafts < 0 || t.vocab < 1) return ECSPMV_ERR_INVALID;
    if (t.batch > 65535 || t.vocab > 1 << 20 || t.drafts > 1 << 20) return ECSPMV_ERR_UNSUPPORTED;
    return ECSPMV_OK;
}

int check_verify_tree(const ecspmv_verify_tree_t *from, ecspmv_verify_tree_t &t)
{
    const int s = copy_struct(from, t);
    if (s) return s;
    if (t.batch < 0 || t.nodes < 0 || t.vocab < 1) return ECSPMV_ERR_INVALID;
    if (t.batch > 65535 || t.vocab > 1 << 20 || t.nodes > (int32_t)ecs::kMostNodes) return ECSPMV_ERR_UNSUPPORTED;
    return ECSPMV_OK;
}

}  // namespace

extern "C" {

int ecspmv_kv_write(const ecspmv_kv_cache_t *cache, const ecspmv_view_t *k, const ecspmv_view_t *v, const int64_t *d_slots,
                    int64_t tokens, void *stream)
{
    return kv_call(cache, k, v, d_slots, tokens, stream, ecs::launch_kv_write);
}

int ecspmv_kv_read(const ecspmv_kv_cache_t *cache, const int64_t *d_slots, int64_t tokens, const ecspmv_view_t *k,
                   const ecspmv_view_t *v, void *stream)
{
    return kv_call(cache, k, v, d_slots, tokens, stream, ecs::launch_kv_read);
}

int ecspmv_kv_append(const ecspmv_kv_cache_t *cache, const ecspmv_view_t *k, const ecspmv_view_t *v, const int64_t *d_slots, int64_t tokens,
                     const ecspmv_rotary_t *rotary, void *stream)
{
    ecs::AppendArgs a;
    std::memset(&a, 0, sizeof(a));
    ecspmv_rotary_t t;
    int s = check_cache(cache, a.cache);
    if (s || (s = copy_struct(rotary, t))) return s;
    if (t.rotary_dim < 0 || t.rotary_dim % 2 || t.rotary_dim > (int32_t)a.cache.dim || t.q_heads < 0 || tokens < 0) return ECSPMV_ERR_INVALID;
    if (t.neighbours != 0 && t.neighbours != 1) return ECSPMV_ERR_UNSUPPORTED;
    if (tokens == 0) return ECSPMV_OK;
    if ((s = check_view(k, a.k, a.k_wide)) || (s = check_view(v, a.v, a.v_wide))) return s;
    if (t.q_heads && ((s = check_view(&t.q, a.q, a.q_wide)) || (s = check_view(&t.q_out, a.q_out, a.q_out_wide)))) return s;
    if (t.q_heads && !spread_out(t.q_out, tokens, t.q_heads)) return ECSPMV_ERR_INVALID;
    // (other workgroups read k and v while q_out is written)
    if (t.q_heads && (t.q_out.data == k->data || t.q_out.data == v->data)) return ECSPMV_ERR_INVALID;
    if (!d_slots || !aligned(d_slots, 8)) return ECSPMV_ERR_INVALID;
    if (t.rotary_dim && (!t.frequency || !aligned(t.frequency, 8) || !t.position || !aligned(t.position, 4))) return ECSPMV_ERR_INVALID;
    if (tokens > 1 << 27 || t.q_heads > 65535 || ((uint64_t)tokens + 16u) * (2u * a.cache.heads + (uint32_t)t.q_heads) > 0x7fffffffu)
        return ECSPMV_ERR_UNSUPPORTED;
    a.slots = d_slots;
    a.position = t.position;
    a.frequency = t.frequency;
    a.tokens = (uint32_t)tokens;
    a.q_heads = (uint32_t)t.q_heads;
    a.pairs = (uint32_t)t.rotary_dim / 2u;
    a.neighbours = (uint32_t)t.neighbours;
    a.run_shift = run_of_tokens(a.tokens);
    return ecs::hip_status(ecs::launch_kv_append(a, stream));
}

int ecspmv_kv_keep(const ecspmv_kv_cache_t *const *caches, int32_t count, const ecspmv_keep_t *from, void *stream)
{
    ecspmv_keep_t t;
    int s = copy_struct(from, t);
    if (s) return s;
    if (count < 0 || t.batch < 0 || t.nodes < 0 || t.max_pages < 0 || (count && !caches)) return ECSPMV_ERR_INVALID;
    if (t.batch > 65535) return ECSPMV_ERR_UNSUPPORTED;
    ecs::KeepArgs a;
    std::memset(&a, 0, sizeof(a));
    ecs::Cache all, one;
    for (int32_t i = 0; i < count; ++i) {                                  // every one of them before anything is launched
        if ((s = check_cache(caches[i], one))) return s;
        if (i == 0) all = one;
        if (one.pages != all.pages || one.heads != all.heads || one.page_shift != all.page_shift || one.dim != all.dim || one.bits != all.bits)
            return ECSPMV_ERR_INVALID;
    }
    if (count == 0 || t.batch == 0 || t.nodes == 0 || t.max_pages == 0) return ECSPMV_OK;
    if ((uint64_t)t.max_pages << all.page_shift > 0x7fffffffu) return ECSPMV_ERR_UNSUPPORTED;
    const void *needed[] = {t.first, t.path, t.accepted, t.page_table};
    for (const void *p : needed)
        if (!p || !aligned(p, 4)) return ECSPMV_ERR_INVALID;
    if (t.table_stride < t.max_pages || t.path_stride < t.nodes) return ECSPMV_ERR_INVALID;
    a.first = t.first;
    a.path = t.path;
    a.accepted = t.accepted;
    a.table = t.page_table;
    a.path_stride = t.path_stride;
    a.table_stride = t.table_stride;
    a.nodes = (uint32_t)t.nodes;
    a.max_pages = (uint32_t)t.max_pages;
    a.pages = all.pages;
    a.heads = all.heads;
    a.page_shift = all.page_shift;
    a.row_bytes = all.row_bytes;
    a.steps = all.bits != 16u;
    for (int32_t i = 0; i < count;) {
        uint32_t layers = 0;
        for (; i < count && layers < ecs::kKeepLayers; ++i, ++layers) {
            if ((s = check_cache(caches[i], one))) return s;
            a.layer[layers] = {one.k, one.v, one.k_step, one.v_step};
        }
        if ((s = ecs::hip_status(ecs::launch_kv_keep(a, layers, (uint32_t)t.batch, stream)))) return s;
    }
    return ECSPMV_OK;
}

int ecspmv_attention_workspace(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *a, size_t *bytes)
{
    if (!bytes) return ECSPMV_ERR_INVALID;
    ecs::AttentionArgs args;
    ecs::AttentionPlan plan;
    ecspmv_attention_t t;
    const int s = check_attention(cache, a, args, plan, t);
    if (s) return s;
    *bytes = (size_t)plan.work_bytes;
    return ECSPMV_OK;
}

int ecspmv_attention_workspace_most(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *a, size_t *bytes)
{
    if (!bytes) return ECSPMV_ERR_INVALID;
    ecs::AttentionArgs args;
    ecs::AttentionPlan plan;
    ecspmv_attention_t t;
    const int s = check_attention(cache, a, args, plan, t);
    if (s) return s;
    const uint64_t most = ecs::most_attention_work(args.batch, args.cache.heads, args.group, args.cache.dim, args.cache.bits, args.tokens,
                                                   args.max_new, (uint64_t)args.max_pages << args.cache.page_shift);
    *bytes = (size_t)(most > plan.work_bytes ? most : plan.work_bytes);
    return ECSPMV_OK;
}

int ecspmv_attention(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *a, void *d_work, size_t work_bytes, void *stream)
{
    ecs::AttentionArgs args;
    ecs::AttentionPlan plan;
    ecspmv_attention_t t;
    int s = check_attention(cache, a, args, plan, t);
    if (s) return s;
    if (nothing_to_compute(args)) return ECSPMV_OK;
    if ((s = check_tensors(t, plan.work_bytes, d_work, work_bytes, args))) return s;
    args.part_o = static_cast<float *>(d_work);
    args.part_ml = args.part_o + (uint64_t)plan.splits * args.tokens * args.q_heads * args.cache.dim;
    return ecs::hip_status(ecs::launch_attention(args, stream));
}

int ecspmv_attention_tree_workspace(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *a, size_t *bytes)
{
    if (!bytes) return ECSPMV_ERR_INVALID;
    ecs::AttentionTreeArgs args;
    ecs::TreePlan plan;
    ecspmv_attention_t t;
    const int s = check_attention_tree(cache, a, args, plan, t);
    if (s) return s;
    *bytes = (size_t)plan.work_bytes;
    return ECSPMV_OK;
}

int ecspmv_attention_tree(const ecspmv_kv_cache_t *cache, const ecspmv_attention_t *a, const uint32_t *d_seen, int64_t seen_stride, void *d_work,
                          size_t work_bytes, void *stream)
{
    ecs::AttentionTreeArgs args;
    ecs::TreePlan plan;
    ecspmv_attention_t t;
    int s = check_attention_tree(cache, a, args, plan, t);
    if (s) return s;
    if (nothing_to_compute(args)) return ECSPMV_OK;
    if ((s = check_tensors(t, plan.work_bytes, d_work, work_bytes, args))) return s;
    if (!spread_out(t.out, t.tokens, t.q_heads)) return ECSPMV_ERR_INVALID;
    if (!d_seen || !aligned(d_seen, 4) || seen_stride < (int64_t)args.seen_words) return ECSPMV_ERR_INVALID;
    args.seen = d_seen;
    args.seen_stride = seen_stride;
    uint8_t *work = static_cast<uint8_t *>(d_work);
    args.plan = reinterpret_cast<ecs::AttentionTreeArgs::Words *>(work);
    args.part_o = reinterpret_cast<float *>(work + (plan.balanced ? ecs::kTreePlanBytes : 0u));
    args.part_ml = args.part_o + (plan.balanced ? (uint64_t)plan.part_rows * args.cache.heads : (uint64_t)plan.splits * args.tokens * args.q_heads) *
                                     args.cache.dim;
    return ecs::hip_status(ecs::launch_attention_tree(args, stream));
}

int ecspmv_verify_workspace(const ecspmv_verify_t *from, size_t *bytes)
{
    ecspmv_verify_t t;
    const int s = check_verify(from, t);
    if (s) return s;
    if (!bytes) return ECSPMV_ERR_INVALID;
    *bytes = (size_t)ecs::verify_work_bytes((uint32_t)t.batch, (uint32_t)t.vocab);
    return ECSPMV_OK;
}

int ecspmv_verify(const ecspmv_verify_t *from, void *d_work, size_t work_bytes, void *stream)
{
    ecspmv_verify_t t;
    const int s = check_verify(from, t);
    if (s) return s;
    if (t.batch == 0) return ECSPMV_OK;
    if (!d_work || !aligned(d_work, 8)) return ECSPMV_ERR_INVALID;
    if (work_bytes < ecs::verify_work_bytes((uint32_t)t.batch, (uint32_t)t.vocab)) return ECSPMV_ERR_TOO_SMALL;
    if (!t.target || !t.uniform || !t.tokens || !t.accepted || (t.drafts && !t.drafted)) return ECSPMV_ERR_INVALID;
    const void *all[] = {t.target, t.draft, t.uniform, t.drafted, t.count, t.tokens, t.accepted};
    for (const void *p : all)
        if (!aligned(p, 4)) return ECSPMV_ERR_INVALID;
    ecs::VerifyArgs a;
    std::memset(&a, 0, sizeof(a));
    a.target = t.target;
    a.draft = t.draft;
    a.uniform = t.uniform;
    a.drafted = t.drafted;
    a.count = t.count;
    a.tokens = t.tokens;
    a.accepted = t.accepted;
    a.target_seq = t.target_seq;
    a.target_row = t.target_row;
    a.draft_seq = t.draft_seq;
    a.draft_row = t.draft_row;
    a.drafts = (uint32_t)t.drafts;
    a.vocab = (uint32_t)t.vocab;
    a.sums = static_cast<double *>(d_work);
    return ecs::hip_status(ecs::launch_verify(a, (uint32_t)t.batch, stream));
}

int ecspmv_verify_tree_workspace(const ecspmv_verify_tree_t *from, size_t *bytes)
{
    ecspmv_verify_tree_t t;
    const int s = check_verify_tree(from, t);
    if (s) return s;
    if (!bytes) return ECSPMV_ERR_INVALID;
    *bytes = (size_t)ecs::verify_tree_work_bytes((uint32_t)t.batch, (uint32_t)t.nodes, (uint32_t)t.vocab);
    return ECSPMV_OK;
}

int ecspmv_verify_tree(const ecspmv_verify_tree_t *from, void *d_work, size_t work_bytes, void *stream)
{
    ecspmv_verify_tree_t t;
    const int s = check_verify_tree(from, t);
    if (s) return s;
    if (t.batch == 0) return ECSPMV_OK;
    if (!d_work || !aligned(d_work, 8)) return ECSPMV_ERR_INVALID;
    if (work_bytes < ecs::verify_tree_work_bytes((uint32_t)t.batch, (uint32_t)t.nodes, (uint32_t)t.vocab)) return ECSPMV_ERR_TOO_SMALL;
    if (!t.target || !t.uniform || !t.tokens || !t.accepted || (t.nodes && (!t.drafted || !t.parent || !t.path))) return ECSPMV_ERR_INVALID;
    const void *all[] = {t.target, t.uniform, t.drafted, t.parent, t.count, t.tokens, t.path, t.accepted};
    for (const void *p : all)
        if (!aligned(p, 4)) return ECSPMV_ERR_INVALID;
    ecs::VerifyTreeArgs a;
    std::memset(&a, 0, sizeof(a));
    a.target = t.target;
    a.uniform = t.uniform;
    a.drafted = t.drafted;
    a.parent = t.parent;
    a.count = t.count;
    a.tokens = t.tokens;
    a.path = t.path;
    a.accepted = t.accepted;
    a.target_seq = t.target_seq;
    a.target_row = t.target_row;
    a.nodes = (uint32_t)t.nodes;
    a.vocab = (uint32_t)t.vocab;
    a.work = static_cast<uint8_t *>(d_work);
    return ecs::hip_status(ecs::launch_verify_tree(a, (uint32_t)t.batch, stream));
}

}  // extern "C"
