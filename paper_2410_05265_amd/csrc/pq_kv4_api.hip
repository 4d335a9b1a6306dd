// C entry points of the paged 4-bit KV cache: argument checking only; every kernel goes to the caller's stream.
#include "pq_kv4.h"

#include <float.h>
#include <math.h>

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + b_bytes && y < x + a_bytes;
}

bool page_size_ok(int32_t ps) { return ps >= 16 && ps <= 1024 && (ps & (ps - 1)) == 0; }

// The sizes of a cache, without its pointers.
int check_cache_shape(const pq_kv4_cache* c)
{
    if (!c) return PQ_ERR_NULL;
    if (!page_size_ok(c->page_size) || c->n_pages < 1 || c->n_pages > INT32_MAX || c->n_kv_heads < 1) return PQ_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return PQ_ERR_UNSUPPORTED;
    if (c->group != 0 && c->group != 32 && c->group != 64 && c->group != 128) return PQ_ERR_SHAPE;
    if (c->group > c->head_dim) return PQ_ERR_SHAPE;
    return PQ_OK;
}

int check_cache(const pq_kv4_cache* c, pq::kv4::Cache* out)
{
    if (const int rc = check_cache_shape(c); rc != PQ_OK) return rc;
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale) return PQ_ERR_NULL;
    const uintptr_t steps = c->group ? 16 : 4;
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, steps) || !aligned(c->v_scale, steps)) return PQ_ERR_ALIGN;
    *out = {static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->v_codes), c->k_scale, c->v_scale, c->n_pages, c->n_kv_heads,
            __builtin_ctz((unsigned)c->page_size)};
    return PQ_OK;
}

// The sizes of an attention call: tokens of a request count as int32, and a launch holds at most 2^32 threads.
bool attention_sizes_ok(int64_t T, int32_t B, int32_t n_heads, int32_t max_q, int32_t table_pages, const pq_kv4_cache* c)
{
    return T >= 0 && B >= 0 && n_heads >= 1 && n_heads % c->n_kv_heads == 0 && T < 1 << 30 && T * n_heads < 1 << 30 && (int64_t)B * c->n_kv_heads < 1 << 21 &&
           max_q >= 1 && table_pages >= 1 && (int64_t)table_pages * c->page_size < 1 << 30;
}

}  // namespace

extern "C" {

int pq_kv4_slots(const int32_t* kv_len, const int32_t* q_len, int32_t B, int32_t* block_table, int32_t table_pages,
                 const int32_t* free_pages, int32_t n_free, const int32_t* taken, int32_t page_size, int64_t T, int32_t position_offset,
                 int32_t* cu_q, int32_t* kv_len_out, int32_t* positions, int64_t* slots, int32_t* taken_out, void* stream)
{
    if (B < 0 || B >= 1 << 26 || T < 0 || T > INT32_MAX || table_pages < 1 || n_free < 0 || position_offset < 0 || !page_size_ok(page_size)) return PQ_ERR_SHAPE;
    if ((B > 0 && (!kv_len || !q_len || !block_table || !kv_len_out)) || (n_free > 0 && !free_pages) || !cu_q || !taken_out ||
        (T > 0 && (!positions || !slots)))
        return PQ_ERR_NULL;
    for (const void* p : {(const void*)kv_len, (const void*)q_len, (const void*)block_table, (const void*)free_pages, (const void*)taken,
                          (const void*)cu_q, (const void*)kv_len_out, (const void*)positions, (const void*)taken_out})
        if (!aligned(p, 4)) return PQ_ERR_ALIGN;
    if (!aligned(slots, 8)) return PQ_ERR_ALIGN;
    // workgroups read the lengths while others write
    const size_t b4 = (size_t)B * 4, t4 = (size_t)T * 4;
    const struct { const void* p; size_t bytes; } written[] = {{block_table, b4 * table_pages}, {cu_q, b4 + 4}, {kv_len_out, b4}, {positions, t4}, {slots, 2 * t4}, {taken_out, 4}},
                                                  read[] = {{kv_len, b4}, {q_len, b4}, {free_pages, (size_t)n_free * 4}, {taken, 4}};
    for (const auto& w : written)
        for (const auto& r : read)
            if (overlap(w.p, w.bytes, r.p, r.bytes)) return PQ_ERR_UNSUPPORTED;
    return pq::kv4::launch_slots(kv_len, q_len, B, block_table, table_pages, free_pages, n_free, taken, __builtin_ctz((unsigned)page_size),
                                 (int32_t)T, position_offset, cu_q, kv_len_out, positions, slots, taken_out, static_cast<hipStream_t>(stream));
}

int pq_kv4_append(const void* qkv_f16, int64_t row_stride, int64_t T, int32_t n_heads, const int32_t* positions, const int64_t* slots,
                  const void* q_weight_f16, const void* k_weight_f16, float eps, const float* cos_sin, int64_t max_positions,
                  int32_t rotary_dim, int32_t interleaved, int32_t rotate, float clip, const pq_kv4_cache* cache, void* q_out_f16,
                  void* stream)
{
    pq::kv4::Cache c;
    if (const int rc = check_cache(cache, &c); rc != PQ_OK) return rc;
    const int64_t heads = (int64_t)n_heads + 2ll * c.n_kv_heads, D = cache->head_dim;
    if (T < 0 || n_heads < 1 || n_heads % c.n_kv_heads != 0 || heads > 65535 || T >= 1 << 25 || T * heads > INT32_MAX) return PQ_ERR_SHAPE;
    if (row_stride < heads * D || row_stride % 8 != 0) return PQ_ERR_SHAPE;
    if (cos_sin && (max_positions < 1 || rotary_dim < 16 || rotary_dim > D || rotary_dim % 16 != 0)) return PQ_ERR_SHAPE;
    if (!isfinite(eps) || eps < 0.0f) return PQ_ERR_SHAPE;
    if (!(isfinite(clip) && clip > 0.0f && clip <= 1.0f)) return PQ_ERR_SCALE;
    if (T == 0) return PQ_OK;
    if (!qkv_f16 || !slots || !q_out_f16 || (cos_sin && !positions)) return PQ_ERR_NULL;
    if (!aligned(qkv_f16, 16) || !aligned(q_out_f16, 16) || !aligned(q_weight_f16, 16) || !aligned(k_weight_f16, 16) || !aligned(cos_sin, 16) ||
        !aligned(positions, 4) || !aligned(slots, 8))
        return PQ_ERR_ALIGN;
    if (overlap(qkv_f16, (size_t)((T - 1) * row_stride + heads * D) * 2, q_out_f16, (size_t)(T * n_heads * D) * 2)) return PQ_ERR_UNSUPPORTED;
    // (the reciprocal root takes subnormal numbers for zero; beside the least square of an fp16 number, 2^-48, no smaller eps shows)
    if (eps > 0.0f && eps < FLT_MIN) eps = FLT_MIN;
    const pq::kv4::AppendArgs a = {static_cast<const __half*>(qkv_f16), row_stride, T, n_heads, positions, slots,
                                   static_cast<const __half*>(q_weight_f16), static_cast<const __half*>(k_weight_f16), eps, cos_sin,
                                   max_positions, rotary_dim, interleaved, clip, c, static_cast<__half*>(q_out_f16)};
    return pq::kv4::launch_append(a, cache->head_dim, cache->group, rotate != 0, static_cast<hipStream_t>(stream));
}

size_t pq_kv4_attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t max_q, int32_t table_pages, const pq_kv4_cache* cache)
{
    if (check_cache_shape(cache) != PQ_OK || T <= 0 || B <= 0 || !attention_sizes_ok(T, B, n_heads, max_q, table_pages, cache)) return 0;
    return pq::kv4::attention_workspace_bytes(T, B, n_heads, cache->n_kv_heads, cache->head_dim, max_q, (int64_t)table_pages * cache->page_size);
}

int pq_kv4_attention(const void* q_f16, int64_t row_stride, int64_t T, int32_t n_heads, const int32_t* cu_q, const int32_t* kv_len,
                     int32_t B, int32_t max_q, const int32_t* block_table, int32_t table_pages, const pq_kv4_cache* cache,
                     const void* prefix_k_f16, const void* prefix_v_f16, int32_t n_prefix, float softmax_scale, int32_t causal,
                     void* out_f16, void* workspace, size_t workspace_bytes, void* stream)
{
    pq::kv4::Cache c;
    if (const int rc = check_cache(cache, &c); rc != PQ_OK) return rc;
    const int64_t D = cache->head_dim;
    if (!attention_sizes_ok(T, B, n_heads, max_q, table_pages, cache) || n_prefix < 0 || n_prefix > 1024) return PQ_ERR_SHAPE;
    if (row_stride < n_heads * D || row_stride % 8 != 0) return PQ_ERR_SHAPE;
    if (!(isfinite(softmax_scale) && softmax_scale > 0.0f)) return PQ_ERR_SCALE;
    if (T == 0 || B == 0) return PQ_OK;
    if (!q_f16 || !cu_q || !kv_len || !block_table || !out_f16 || (n_prefix > 0 && (!prefix_k_f16 || !prefix_v_f16))) return PQ_ERR_NULL;
    if (!aligned(q_f16, 16) || !aligned(out_f16, 16) || !aligned(prefix_k_f16, 16) || !aligned(prefix_v_f16, 16) || !aligned(cu_q, 4) ||
        !aligned(kv_len, 4) || !aligned(block_table, 4))
        return PQ_ERR_ALIGN;
    if (overlap(q_f16, (size_t)((T - 1) * row_stride + n_heads * D) * 2, out_f16, (size_t)(T * n_heads * D) * 2)) return PQ_ERR_UNSUPPORTED;
    const size_t need = pq_kv4_attention_workspace_bytes(T, B, n_heads, max_q, table_pages, cache);
    if (!workspace || workspace_bytes < need) return PQ_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return PQ_ERR_ALIGN;
    const pq::kv4::AttentionArgs a = {static_cast<const __half*>(q_f16), row_stride, T, n_heads, n_heads / c.n_kv_heads, cu_q, kv_len, B,
                                      block_table, table_pages, c, static_cast<const __half*>(prefix_k_f16),
                                      static_cast<const __half*>(prefix_v_f16), n_prefix, softmax_scale, causal,
                                      static_cast<__half*>(out_f16)};
    return pq::kv4::launch_attention(a, cache->head_dim, cache->group, max_q, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
