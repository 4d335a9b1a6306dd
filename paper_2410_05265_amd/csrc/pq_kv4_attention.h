// What the attention kernels over the paged 4-bit cache share.
//
//     out_i = sum_t p_it v_t / sum_t p_it,    p_it = exp2(c k_t . q_i - m_i),    c = softmax_scale * log2(e)
//
// over the prefix tokens and the cached ones that query i sees (Eq. 3 of the paper: the prefix in full precision in front of the
// quantized keys and values).  Scores are computed transposed, S^T = K Q^T: a lane then holds scores of one query, their maximum and sum
// stay within the lane, and the probabilities lie in its registers as the second product O^T = V^T P^T wants them.
//
// Codes as fp16 operands: u = code + 8 (one exclusive or for eight) moved to bits 4 to 7 of each half is the subnormal number u * 2^-20,
// which the matrix instructions take exactly: a mask and at most one shift for two codes, no subtraction.  The offset leaves by itself:
// K (u - 8) q starts its sum at -8 sum(q) 2^-20, and sum p (u - 8) = sum p u - 8 sum p, where sum p is the cached tokens' part of the
// softmax's own denominator (of the rounded probabilities that the product uses); the prefix tokens' values have no offset.  Over n
// tokens of like weight the sum with the offset is some 2 sqrt(n) times the one without, and its roundings as many times larger, so the
// kernel for few rows takes it off every 64 tiles, and the one for many rows has values without it in its operands.  (At bits 0 to 3 the products lose low bits against the accumulator: 6e-7 of the largest
// sum, at bits 4 to 7 none were lost.)
//
// Probabilities are rounded to fp16 relative to a reference m that lags behind the running maximum: it moves only when a score passes it by
// 14 (p <= 2^14), and then to 6 above which 2^6 = p stands.  p keeps fp16's full precision down to 2^-20 of the largest, the accumulators are
// rescaled only when the reference moves, by a power of two, and the denominator sums what was rounded: where one token has all the weight its
// rounding leaves again.  With dynamic steps the product takes weights p * step, rounded once, a rounding for every group of channels; the
// denominator then sums p as it is: the sum of rounded p would be a second, independent error, sqrt(3) instead of sqrt(2) times the rounding of
// the fp16 result where one token has the weight (measured over histories of 1 to 2000 tokens: 1.40 to 1.45, static steps 1.0 to 1.44).  That is
// over many rows; where a call has few of them these errors do not average out, and the kernel for few rows takes large weights as two fp16
// numbers each.
#pragma once

#include "pq_kv4.h"

namespace pq {
namespace kv4 {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int kTileRows = 256;           // rows of a workgroup of the kernel for many queries

// Where a call may hold requests of more rows than kSmallRows, those take the tile kernel and the others the row kernel.  Row | tile kernel
// alone, us, 32 heads of 128 on 8, with 128, 192 and 256 rows: one request of 33000 tokens 62 | 73, 62 | 72, 75 | 73; 8 of 2000 to 4000 51 | 59,
// 57 | 47, 69 | 49; 64 of 1000 to 2000 139 | 129, 177 | 122, 221 | 126, with a step to 32 channels 261 | 262, 373 | 264, 485 | 266.  (Of several
// requests the row kernel is launched for the others as well, 8 us; many requests of 129 to 192 rows would gain from a lower border all the
// same, a single one would lose.)
constexpr int kSmallRows = 192;

constexpr float kNothing = -1e30f;       // reference before the first score (a score is above -2^20)
constexpr float kMost = 14.0f, kBack = 6.0f;
constexpr float kUnit = 0x1.0p20f;       // a code as operand is u * 2^-20
constexpr uint32_t kNibble = 0x00F000F0u, kOffset = 0x88888888u;

// Codes j and j + 4 of a dword (already offset to 0..15) as two fp16 operands.
template <int J> __device__ __forceinline__ uint32_t operand(uint32_t u)
{
    if constexpr (J == 0) return (u << 4) & kNibble;
    else if constexpr (J == 1) return u & kNibble;
    else if constexpr (J == 2) return (u >> 4) & kNibble;
    else return (u >> 8) & kNibble;
}

// Eight codes of a key as an operand: channels in the order 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ v8h key_operand(uint32_t codes)
{
    const uint32_t u = codes ^ kOffset;
    const v4u r = {operand<0>(u), operand<1>(u), operand<2>(u), operand<3>(u)};
    return __builtin_bit_cast(v8h, r);
}

// Eight fp16 values in that order.
__device__ __forceinline__ v8h in_key_order(const v4u d)
{
    const v4u r = {__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u),
                   __builtin_amdgcn_perm(d[3], d[1], 0x05040100u), __builtin_amdgcn_perm(d[3], d[1], 0x07060302u)};
    return __builtin_bit_cast(v8h, r);
}

__device__ __forceinline__ uint32_t two_halves(float a, float b)
{
    const v2h h = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, h);
}

// (Cuts off what `to` has no bits for instead of rounding: over a long history a denominator so added was 2^-24 too small for each addition,
// 3e-4 after 32768 tokens, and eight times as much in a static step's offset.  So only a tile's own weights are added with it.)
__device__ __forceinline__ float add_halves(uint32_t pair, float to)
{
    const v2h one = {(_Float16)1.0f, (_Float16)1.0f};
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, pair), one, to, false);
}

// A value's dynamic step, times a probability of zero, is zero: one that is not finite (of a token with an infinite value) counts as the
// largest number, so that who sees the token leaves fp16's range, and who does not is not touched.
__device__ __forceinline__ float finite_step(float s) { return fmaxf(fminf(s, __FLT_MAX__), 0.0f); }

// 1 / x of a power of two.
__device__ __forceinline__ float inverse(float x) { return __uint_as_float(0x7F000000u - __float_as_uint(x)); }

// A request as the kernels see it: nothing that lies on the device takes them out of bounds.  Its rows may end with the call's (T), its history
// with the table; what a row sees is counted from the whole lengths all the same.
struct Request {
    int32_t start, q_len, n;     // first row, rows, cached tokens within the table
    int32_t sees;                // causal: tokens that the first row sees, of any number (may be negative); a later one as many more
};

constexpr int64_t kMostTokens = 1 << 30;                   // (no table is that long)
__device__ __forceinline__ Request request(const AttentionArgs& a, int b)
{
    Request r;
    const int64_t begin = a.cu_q[b], end = max((int64_t)a.cu_q[b + 1], begin);
    const int64_t from = min(max(begin, (int64_t)0), a.T), to = min(max(end, from), a.T), capacity = (int64_t)a.table_pages << a.cache.log2_page;
    int64_t kv = max(a.kv_len[b], 0);
    if (kv >= kMostTokens) kv = capacity;                  // (no length: as many as there may be)
    r.start = (int32_t)from;
    r.q_len = (int32_t)(to - from);
    r.n = (int32_t)min(kv, capacity);
    r.sees = (int32_t)min(max(kv - (end - 1 - from), -kMostTokens), kMostTokens);
    return r;
}

// Tokens that row `token` of a request sees, and those that every row from it on sees.
__device__ __forceinline__ int sees(const AttentionArgs& a, const Request& r, int token)
{
    return a.causal ? min(max(r.sees + token, 0), r.n) : r.n;
}

// ---- Windows, and trees of drafted tokens: the kernels' variants with `Masked` among their parameters.
//
// A request of at most 32 * words rows is a tree, of which c = sees - 1 tokens lie in front: row i sees t < c with t < sinks or t >= c + |mask_i| - window,
// and node j, the token c + j, if its mask says so.  Any other is a chain: row i sees t < sees + i with t < sinks or t >= sees + i - window.
struct Masked;

__device__ __forceinline__ bool is_tree(const AttentionArgs& a, const Request& r) { return a.tree != nullptr && r.q_len <= 32 * a.words; }

// Tokens that a row sees: t < limit with t < sinks or t >= lo; of a tree's the nodes behind are in its mask.
struct Row { int limit, lo; };

// Word w of the mask of a row: nodes that there are.
__device__ __forceinline__ uint32_t mask_word(const AttentionArgs& a, const Request& r, int token, int w)
{
    if (w < 0 || w >= a.words) return 0;
    const int nodes = r.q_len - 32 * w;
    const uint32_t there = nodes >= 32 ? ~0u : nodes > 0 ? (1u << nodes) - 1 : 0u;
    return a.tree[(int64_t)(r.start + token) * a.words + w] & there;
}

// Nodes first .. first + 31 (first may be negative) in a row's mask.
__device__ __forceinline__ uint32_t mask_bits(const AttentionArgs& a, const Request& r, int token, int first)
{
    const int w = first >> 5;
    return __builtin_amdgcn_alignbit(mask_word(a, r, token, w + 1), mask_word(a, r, token, w), first & 31);
}

__device__ __forceinline__ Row masked_row(const AttentionArgs& a, const Request& r, int token)
{
    if (!is_tree(a, r)) return {min(max(r.sees + token, 0), r.n), max(r.sees + token - a.window, 0)};
    const int c = r.sees - 1;
    int nodes = 0;
    if (a.window < kWidestWindow) {
        for (int w = 0; w < a.words; ++w) nodes += __builtin_popcount(mask_word(a, r, token, w));
    }
    return {min(max(c, 0), r.n), max(c - a.window + nodes, 0)};
}

// What the rows of tokens first .. last of a request see, as far as no mask has to be read.
struct Seen {
    int all;       // every row sees the tokens before it, but for the window
    int any;       // no row sees one from it on
    int lo, lo_top;    // tokens before lo that are no sinks are seen by no row, those from lo_top on are hidden by no row's window
};
__device__ __forceinline__ Seen masked_rows(const AttentionArgs& a, const Request& r, int first, int last)
{
    if (is_tree(a, r)) {
        const int c = r.sees - 1;
        return {min(max(c, 0), r.n), min(max(c + r.q_len, 0), r.n), min(max(c - a.window, 0), r.n), max(c - a.window + r.q_len, 0)};
    }
    return {min(max(r.sees + first, 0), r.n), min(max(r.sees + last, 0), r.n), min(max(r.sees + first - a.window, 0), r.n),
            max(r.sees + last - a.window, 0)};
}

// A history in tiles of SIZE tokens, without those that only hold tokens between the sinks and the window: tile number i of what is left.
template <int SIZE> struct Tiles {
    int front, gap;                                // tiles of the sinks, and those left out behind them
    __device__ __forceinline__ Tiles(const AttentionArgs& a, int lo) : front((int)(((int64_t)a.sinks + SIZE - 1) / SIZE)), gap(max(lo / SIZE - front, 0)) {}
    __device__ __forceinline__ int at(int i) const { return i + (i >= front ? gap : 0); }
    __device__ __forceinline__ int count(int end) const         // of the tokens before `end`
    {
        const int all = (end + SIZE - 1) / SIZE;
        return all <= front ? all : max(all - gap, front);
    }
};

// Requests of more than small_rows rows (tokens times query heads of a key/value head); the others are the row kernel's.
size_t tiles_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int64_t capacity);
int launch_attention_tiles(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, float* partial, hipStream_t st);
size_t masked_tiles_workspace_bytes(int64_t T, int32_t B, int32_t per_kv, int32_t head_dim, int small_rows);

}  // namespace kv4
}  // namespace pq
