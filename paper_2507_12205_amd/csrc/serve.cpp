// C ABI around the products (see include/ecspmv.h): argument checks of the cache, the attention over it and the check of drafted
// tokens.  Nothing here allocates or can throw.
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
    while ((1u << a.run_shift) < a.tokens && a.run_shift < 4u) ++a.run_shift;
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

int check_verify(const ecspmv_verify_t *from, ecspmv_verify_t &t)
{
    const int s = copy_struct(from, t);
    if (s) return s;
    if (t.batch < 0 || t.drafts < 0 || t.vocab < 1) return ECSPMV_ERR_INVALID;
    if (t.batch > 65535 || t.vocab > 1 << 20 || t.drafts > 1 << 20) return ECSPMV_ERR_UNSUPPORTED;
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
    if (args.tokens == 0 || args.batch == 0 || args.max_new == 0) return ECSPMV_OK;          // nothing to compute
    if ((s = check_view(&t.q, args.q, args.q_wide)) || (s = check_view(&t.out, args.out, args.out_wide))) return s;
    if (!t.q_start || !t.kv_len || !aligned(t.q_start, 4) || !aligned(t.kv_len, 4)) return ECSPMV_ERR_INVALID;
    if (args.max_pages && (!t.page_table || !aligned(t.page_table, 4) || t.table_stride < t.max_pages)) return ECSPMV_ERR_INVALID;
    if (plan.work_bytes && (!d_work || !aligned(d_work, 16))) return ECSPMV_ERR_INVALID;
    if (work_bytes < plan.work_bytes) return ECSPMV_ERR_TOO_SMALL;
    args.q_start = t.q_start;
    args.kv_len = t.kv_len;
    args.table = t.page_table;
    args.table_stride = t.table_stride;
    args.part_o = static_cast<float *>(d_work);
    args.part_ml = args.part_o + (uint64_t)plan.splits * args.tokens * args.q_heads * args.cache.dim;
    args.scale_log2 = t.scale * 1.44269504088896340736f;
    return ecs::hip_status(ecs::launch_attention(args, stream));
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

}  // extern "C"
