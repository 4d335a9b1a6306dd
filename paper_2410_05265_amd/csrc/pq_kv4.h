// Internal declarations of the paged 4-bit KV cache: its addressing, and the launchers behind the pq_kv4_* entry points.
#pragma once

#include "pq_internal.h"

namespace pq {
namespace kv4 {

// A page holds page_size tokens of every head: [n_pages, n_kv_heads, page_size, head_dim / 2] bytes, and with dynamic steps
// [n_pages, n_kv_heads, page_size, head_dim / group] floats.  A head's part of a page lies in one piece, so whoever reads one head
// reads whole cache lines (a token's 64 bytes of 128 channels between those of other heads would be half lines).
struct Cache {
    uint8_t* k_codes;
    uint8_t* v_codes;
    float* k_scale;
    float* v_scale;
    int64_t n_pages;
    int32_t n_kv_heads;
    int32_t log2_page;      // of page_size
};

struct AppendArgs {
    const __half* qkv;
    int64_t row_stride;
    int64_t T;
    int32_t n_heads;
    const int32_t* positions;
    const int64_t* slots;
    const __half* q_weight;
    const __half* k_weight;
    float eps;
    const float* cos_sin;
    int64_t max_positions;
    int32_t rotary_dim;
    int32_t interleaved;
    float clip;
    Cache cache;
    __half* q_out;
};

struct AttentionArgs {
    const __half* q;
    int64_t row_stride;
    int64_t T;
    int32_t n_heads;
    int32_t heads_per_kv;
    const int32_t* cu_q;
    const int32_t* kv_len;
    int32_t B;
    const int32_t* table;
    int32_t table_pages;
    Cache cache;
    const __half* prefix_k;
    const __half* prefix_v;
    int32_t n_prefix;
    float softmax_scale;
    int32_t causal;
    __half* out;
};

int launch_slots(const int32_t* kv_len, const int32_t* q_len, int32_t B, int32_t* block_table, int32_t table_pages,
                 const int32_t* free_pages, int32_t n_free, const int32_t* taken, int32_t log2_page, int32_t T, int32_t position_offset,
                 int32_t* cu_q, int32_t* kv_len_out, int32_t* positions, int64_t* slots, int32_t* taken_out, hipStream_t st);
int launch_append(const AppendArgs& a, int32_t head_dim, int32_t group, bool rotate, hipStream_t st);

size_t attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, int64_t capacity);
int launch_attention(const AttentionArgs& a, int32_t head_dim, int32_t group, int32_t max_q, void* ws, hipStream_t st);

}  // namespace kv4
}  // namespace pq
