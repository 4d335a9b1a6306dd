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
    // What rows see of a history (Masked kernels): its first `sinks` tokens and the last `window` before the row's own end, and of a tree's
    // nodes those of its mask, uint32 [T, words] (null: no trees).
    const uint32_t* tree;
    int32_t words;
    int32_t window;         // 1 .. kWidestWindow
    int32_t sinks;
};
constexpr int32_t kWidestWindow = (1 << 30) - 1;       // (no table holds as many tokens)

constexpr int kMostNodes = 256;         // of a tree: eight words of mask

int launch_slots(const int32_t* kv_len, const int32_t* q_len, int32_t B, int32_t* block_table, int32_t table_pages,
                 const int32_t* free_pages, int32_t n_free, const int32_t* taken, int32_t log2_page, int32_t T, int32_t position_offset,
                 int32_t* cu_q, int32_t* kv_len_out, int32_t* positions, int64_t* slots, int32_t* taken_out, hipStream_t st);
int launch_append(const AppendArgs& a, int32_t head_dim, int32_t group, bool rotate, hipStream_t st);

struct AcceptArgs {
    const int32_t* tokens;
    const int32_t* parents;
    const int32_t* chosen;
    const int32_t* cu_q;
    const int32_t* kv_len;
    int32_t B;
    int32_t T;
    int32_t words;
    int32_t depth;
    const int32_t* table;
    int32_t table_pages;
    int32_t log2_page;
    int32_t* free_pages;
    int32_t n_free;
    const int32_t* taken;
    int32_t* accepted;
    int32_t* next_token;
    int32_t* path;
    int32_t* kv_len_out;
    int64_t* from_slots;
    int64_t* to_slots;
    int32_t* taken_out;
};

int launch_tree(const int32_t* parents, const int32_t* cu_q, const int32_t* kv_len, int32_t B, int32_t T, int32_t words, int32_t position_offset,
                uint32_t* mask, int32_t* positions, hipStream_t st);
int launch_accept(const AcceptArgs& a, hipStream_t st);
int launch_keep(const int64_t* from_slots, const int64_t* to_slots, int32_t B, int32_t width, const pq_kv4_cache* caches, int32_t n_caches, hipStream_t st);

// What the host knows of the histories: the table's tokens, and where kernels look at windows and trees what rows see of them.
struct Histories {
    int64_t table;
    bool masked;
    int32_t window, sinks;
    // Tokens of one that up to `tokens` rows see, at most.
    int64_t seen_by(int64_t tokens) const
    {
        const int64_t most = (int64_t)window + sinks + tokens + 128;
        return masked && most < table ? most : table;
    }
};
size_t attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, const Histories& h);
int launch_attention(const AttentionArgs& a, int32_t head_dim, int32_t group, int32_t max_q, bool masked, void* ws, hipStream_t st);

}  // namespace kv4
}  // namespace pq
