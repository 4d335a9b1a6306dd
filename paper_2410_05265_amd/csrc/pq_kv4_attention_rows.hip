// Attention over the paged 4-bit cache for few queries of a request: decoded tokens, and some drafted ones.
//
// The queries of a request that share a key/value head (its tokens times the heads of the group) are the columns of the matrix instructions,
// 16 or 32 of them (CB blocks of 16), so that up to as many read every code once.  Bound by HBM: 128 bytes of codes for a token and head of
// 128 channels.  One token each of 64 requests of up to 8192 cached ones, 32 heads on 8: 356 MB in 72 us and 4.6 for the second kernel, where
// a kernel that only reads as many bytes in a row takes 56.  One request of 1537 tokens: 7 us and 4, all latency.
//
// Work is cut over the histories, in units of kTile tokens of one request, head and tile of rows.  All units of the call lie one after another,
// and every wavefront takes an equal run of them, whatever the requests' lengths are: a run that covers a history whole writes its outputs,
// one that begins or ends inside a history leaves a partial sum (at most two to a wavefront), and a second small kernel adds those, in the
// order of the wavefronts.  Wavefronts never wait for one another: with runs to a workgroup, and its four wavefronts' sums joined behind
// barriers, the ends of histories cost a tenth of the time.  The lengths are read on the device, so a captured call follows them.
//
// A wavefront takes 32 tokens at a time.  Their codes go from memory straight into its ring of kDepth places in LDS, so three tiles are on
// their way without a register; a lane then reads 16 bytes of a token's key codes (its part of every step of the first product), and 4
// bytes of each of eight tokens' value codes: an 8 x 8 block, whose transposition is a byte permutation of two tokens.
#include "pq_kv4_attention_plan.h"

#define PQ_INLINE __attribute__((always_inline))

namespace pq {
namespace kv4 {
namespace {

__device__ __forceinline__ v4f product(const v8h& a, const v8h& b, const v4f& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 32;                          // tokens of a wavefront's step: a unit
constexpr int kDepth = 4;                          // places of a wavefront's ring
// Two workgroups to a CU: 128 of its 160 KiB of LDS with 128 channels (32 to 40 KiB with 64, where registers would allow three).  (Three with three places, where the registers allow them: 64 requests of up to 8192
// tokens 84.1 us against 82.4, 24 x 32 heads of up to 2300 42.5 against 43.4, 3 requests of up to 131072 93.8 against 86.4.)
constexpr int kPerCu = 2, kGroups = 256 * kPerCu;
constexpr float kLeast = 0x1.0p-80f;               // smallest reference of value weights (dynamic steps)

// Units of every tile of a request's rows: those of all its tokens, with MASKED of those that one of its rows may see.
template <bool MASKED>
__device__ __forceinline__ int64_t units_of_tile(const AttentionArgs& a, const Request& r)
{
    if constexpr (MASKED) {
        const Seen s = masked_rows(a, r, 0, max(r.q_len - 1, 0));
        return max(Tiles<kTile>(a, s.lo).count(s.any), 1);
    }
    return r.n > 0 ? (r.n + kTile - 1) / kTile : 1;
}

// Histories of a request: heads x tiles of rows; none if it has more than small_rows rows.
template <int ROWS>
__device__ __forceinline__ int tiles_of(const AttentionArgs& a, const Request& r, int small_rows)
{
    const int64_t rows = (int64_t)r.q_len * a.heads_per_kv;
    return rows > small_rows ? 0 : (int)((rows + ROWS - 1) / ROWS);
}

__device__ __forceinline__ int64_t divided(int64_t x, int64_t by)
{
    if (((x | by) >> 32) == 0) return (uint32_t)x / (uint32_t)by;      // a third of the instructions
    return x / by;
}

// The requests' histories and units: each lane of the calling wavefront sums a run of requests.
struct Plan {
    int64_t total, before, own;          // units: all, those before this lane's requests, and theirs
    int64_t items, items_before;         // histories
    int first, last;                     // this lane's requests
    Request r;                           // the last of them
};

template <int ROWS, bool MASKED>
__device__ __forceinline__ Plan plan(const AttentionArgs& a, int small_rows, int lane)
{
    Plan p;
    const int each = (a.B + 63) / 64;
    p.first = min(lane * each, a.B);
    p.last = min(p.first + each, a.B);
    p.own = 0;
    p.r = {0, 0, 0, 0};
    int64_t items = 0;
    for (int b = p.first; b < p.last; ++b) {
        p.r = request(a, b);
        const int64_t n = (int64_t)tiles_of<ROWS>(a, p.r, small_rows) * a.cache.n_kv_heads;
        items += n;
        p.own += n * units_of_tile<MASKED>(a, p.r);
    }
    int64_t units_incl = p.own, items_incl = items;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t u = __shfl_up(units_incl, d, 64), i = __shfl_up(items_incl, d, 64);
        if (lane >= d) {
            units_incl += u;
            items_incl += i;
        }
    }
    p.before = units_incl - p.own;
    p.total = __shfl(units_incl, 63, 64);
    p.items_before = items_incl - items;
    p.items = __shfl(items_incl, 63, 64);
    return p;
}

// A history, as the kernel that adds partial sums takes it: `parts` wavefronts from `worker` on have some of it (one: it is done); the
// first one's sum lies at its second place, if `second`.
struct Item {
    int worker, parts, second, start, rows, head, row0, unused;
};

// 16 or 4 bytes of every lane from memory straight into LDS, lane after lane from lds_addr (wavefront-uniform) on; `once`: past the caches.
__device__ __forceinline__ void to_lds16_once(const void* src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds_addr)) : "memory");
}
__device__ __forceinline__ void to_lds16(const void* src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds_addr)) : "memory");
}
__device__ __forceinline__ void to_lds4(const void* src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds_addr)) : "memory");
}

__device__ __forceinline__ v4u in_halves(const float (&w)[8])
{
    return (v4u){two_halves(w[0], w[1]), two_halves(w[2], w[3]), two_halves(w[4], w[5]), two_halves(w[6], w[7])};
}
// What fp16 leaves of eight weights, in fp16: with it 22 bits of each.
__device__ __forceinline__ v4u rest_in_halves(const float (&w)[8])
{
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = w[i] - (float)(_Float16)w[i];
    return in_halves(rest);
}
// (Their own sum first: add_halves.)
__device__ __forceinline__ float add_eight(const v4u& w, float to) { return to + add_halves(w[3], add_halves(w[2], add_halves(w[1], add_halves(w[0], 0.0f)))); }

template <int D, int G, bool DYNAMIC, int CB>
struct Shape {
    static constexpr int NG = D / G, KS = G / 32, CH = G / 16, ROWS = 16 * CB;
    static constexpr int CODES = kTile * D / 2;                          // bytes of a tile's keys, and of its values
    static constexpr int SLOT = 2 * CODES + (DYNAMIC ? 256 * NG : 0);
    static constexpr int LOADS = 2 * CODES / 1024 + (DYNAMIC ? NG : 0);  // of a tile
    static constexpr size_t kLds = (size_t)kWaves * kDepth * SLOT;
};

template <int D, int G, bool DYNAMIC, int CB, typename... KIND>
__global__ __launch_bounds__(kThreads, kPerCu) void k_kv4_attention_rows(AttentionArgs a, float* partial, Item* items, int64_t most_items, int small_rows)
{
    constexpr bool MASKED = sizeof...(KIND) > 0;
    typedef Shape<D, G, DYNAMIC, CB> S;
    constexpr int NG = S::NG, KS = S::KS, CH = S::CH, ROWS = S::ROWS;
    extern __shared__ __align__(256) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int log2_page = a.cache.log2_page, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv;
    const uint8_t* const ring = lds + wave * kDepth * S::SLOT;
    const uint32_t ring_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)ring;

    const Plan p = plan<ROWS, MASKED>(a, small_rows, lane);
    // Codes that one wavefront reads once go past the caches, where they would push out each other and, from call to call, themselves: a call's
    // history from 64 MiB on (356 MB 82 -> 73.5 us, 148 MB 43.2 -> 39.8, 342 MB with dynamic steps 84.5 -> 79.9); below, they may be in the
    // memory-side cache still, where a program has few caches: three in turn, through the caches | past them, 32 MB 18.5 | 19.1, 59 MB 26.5 |
    // 27.8, and 27 MB with dynamic steps 23.4 | 24.6; thirty-two in turn 16 MB 16.3 | 15.9, 32 MB 20.0 | 19.4, 59 MB 28.4 | 27.9.
    const bool stream = p.total * (2 * S::CODES) > 64 << 20;
    // (place 0 holds their count; only rows that lie in two requests, from a cu_q that does not ascend, make more than there are places)
    if (blockIdx.x == 0 && threadIdx.x == 0) items[0].parts = (int)min(p.items, most_items);
    // the first `more` runs have one unit more
    const int64_t workers = min((int64_t)gridDim.x * kWaves, p.total);
    const int worker = xcd_run(blockIdx.x, gridDim.x) * kWaves + wave;
    if (worker >= workers) return;
    const int64_t each = divided(p.total, workers), more = p.total - each * workers;
    const int64_t range = each * worker + min((int64_t)worker, more), range_end = range + each + (worker < more ? 1 : 0);
    auto worker_of = [&](int64_t unit) PQ_INLINE {
        return unit < more * (each + 1) ? divided(unit, each + 1) : more + divided(unit - more * (each + 1), each);
    };

    // the request that the run begins in, its first unit and its first history
    int b;
    int64_t base, item_base;
    Request r;
    {
        const bool mine = p.before <= range && range < p.before + p.own;
        int at = p.first;
        int64_t u = p.before, i = p.items_before;
        r = p.r;
        if (mine && p.last - p.first > 1) {
            for (; at < p.last; ++at) {
                r = request(a, at);
                const int64_t n = (int64_t)tiles_of<ROWS>(a, r, small_rows) * Hkv;
                const int64_t units = n * units_of_tile<MASKED>(a, r);
                if (range < u + units) break;
                u += units;
                i += n;
            }
        }
        const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));
        b = __builtin_amdgcn_readfirstlane(__shfl(at, from, 64));
        base = __shfl(u, from, 64);
        item_base = __shfl(i, from, 64);
        r.start = __builtin_amdgcn_readfirstlane(__shfl(r.start, from, 64));
        r.q_len = __builtin_amdgcn_readfirstlane(__shfl(r.q_len, from, 64));
        r.n = __builtin_amdgcn_readfirstlane(__shfl(r.n, from, 64));
        r.sees = __builtin_amdgcn_readfirstlane(__shfl(r.sees, from, 64));
    }

    for (int64_t u0 = range; u0 < range_end;) {
        const int tiles = tiles_of<ROWS>(a, r, small_rows);
        const int64_t per = units_of_tile<MASKED>(a, r), whole = per * tiles * Hkv;
        if (u0 >= base + whole) {                  // (requests without queries, or with many, have no units)
            base += whole;
            item_base += (int64_t)tiles * Hkv;
            r = request(a, ++b);
            continue;
        }
        const int64_t item = divided(u0 - base, per), from_unit = u0 - base - item * per, take = min(range_end - u0, per - from_unit);
        const int head = __builtin_amdgcn_readfirstlane((int)item / tiles), tile = __builtin_amdgcn_readfirstlane((int)item % tiles);
        const int rows = r.q_len * per_kv;
        const int first_token = tile * ROWS / per_kv, last_token = min((tile * ROWS + ROWS - 1) / per_kv, r.q_len - 1);
        const bool tree = MASKED && is_tree(a, r);
        Seen seen;                                 // (lo: of the request, lo_top: of this tile's rows)
        if constexpr (MASKED) {
            seen = masked_rows(a, r, first_token, last_token);
            seen.lo = masked_rows(a, r, 0, 0).lo;
        } else {
            seen = {sees(a, r, first_token), sees(a, r, last_token), 0, 0};
        }
        const int all_see = seen.all, any_sees = seen.any;     // tokens before all_see need no mask, but for a window's
        const Tiles<kTile> left_in(a, MASKED ? seen.lo : 0);
        const int from = (int)(from_unit * kTile), to = (int)min((from_unit + take) * kTile, (int64_t)any_sees);
        auto start_of = [&](int i) PQ_INLINE -> int { return MASKED ? left_in.at((int)from_unit + i) * kTile : from + i * kTile; };
        if (from_unit == 0 && lane == 0 && item_base + item < most_items)
            items[1 + item_base + item] = {worker, take == per ? 1 : (int)worker_of(u0 + per - 1) - worker + 1, u0 == range ? 0 : 1, r.start, rows, head,
                                           tile * ROWS, 0};

        // ---- codes on their way
        const int32_t* table = a.table + (int64_t)b * a.table_pages;
        int ids_from = -64, ids = 0;
        const int count = __builtin_amdgcn_readfirstlane(MASKED ? max((int)min(from_unit + take, (int64_t)left_in.count(any_sees)) - (int)from_unit, 0)
                                                                : from < to ? (to - from + kTile - 1) / kTile : 0);
        uint32_t bad_bits = 0;                     // two bits for each place of the ring: blocks of 16 tokens whose page is none
        auto fetch = [&](int i) PQ_INLINE {
            const int t0 = start_of(i), place = i % kDepth;
            int64_t first[2];                      // of the blocks, in this head's part of the cache
            bad_bits &= ~(3u << (2 * place));
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const int t = t0 + 16 * blk, page_at = t >> log2_page;
                if (page_at >= ids_from + 64) {
                    ids_from = page_at;
                    ids = table[min(page_at + lane, a.table_pages - 1)];
                }
                const int page = __builtin_amdgcn_readlane(ids, page_at - ids_from);
                const bool bad = (uint32_t)page >= (uint64_t)a.cache.n_pages || page_at >= a.table_pages;
                bad_bits |= (bad ? 1u : 0u) << (2 * place + blk);
                first[blk] = (((int64_t)(bad ? 0 : page) * Hkv + head) << log2_page) + (t & ((1 << log2_page) - 1));
            }
            const uint32_t to_addr = ring_addr + place * S::SLOT;
            auto codes = [&](auto to_lds) PQ_INLINE {
                if constexpr (D == 128) {
#pragma unroll
                    for (int blk = 0; blk < 2; ++blk) {
                        to_lds(a.cache.k_codes + first[blk] * 64 + 16 * lane, to_addr + 1024 * blk);
                        to_lds(a.cache.v_codes + first[blk] * 64 + 16 * lane, to_addr + S::CODES + 1024 * blk);
                    }
                } else {                           // 32 lanes to a block
                    const int64_t at = (lane < 32 ? first[0] : first[1]) * 32 + 16 * (lane & 31);
                    to_lds(a.cache.k_codes + at, to_addr);
                    to_lds(a.cache.v_codes + at, to_addr + S::CODES);
                }
            };
            if (stream && tiles == 1) codes([](const void* src, uint32_t to) PQ_INLINE { to_lds16_once(src, to); });
            else codes([](const void* src, uint32_t to) PQ_INLINE { to_lds16(src, to); });
            if constexpr (DYNAMIC) {
#pragma unroll
                for (int j = 0; j < NG; ++j) {     // step e of the tile's 32 NG: token e / NG, group e % NG
                    const int e = 32 * j + (lane & 31), t = e / NG;
                    const int64_t at = ((t < 16 ? first[0] : first[1]) + (t & 15)) * NG + e % NG;
                    to_lds4((lane < 32 ? a.cache.k_scale : a.cache.v_scale) + at, to_addr + 2 * S::CODES + 256 * j);
                }
            }
        };
        // ---- queries: channels as the keys' operands have them
        v4u raw[CB][NG * KS];
        int limit[CB], lo[CB];                     // tokens that the lane's query sees: before limit, those of no sink from lo on
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int row = min(tile * ROWS + 16 * c + col, rows - 1), token = row / per_kv, q_head = head * per_kv + row % per_kv;
            if constexpr (MASKED) {
                const Row see = masked_row(a, r, token);
                limit[c] = see.limit;
                lo[c] = see.lo;
            } else {
                limit[c] = sees(a, r, token);
                lo[c] = 0;
            }
            const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
#pragma unroll
            for (int i = 0; i < NG * KS; ++i) raw[c][i] = *reinterpret_cast<const v4u*>(src + i / KS * G + quarter * (G / 4) + 8 * (i % KS));
        }
        const bool prefix = a.n_prefix > 0 && from_unit == 0;
        const int early = prefix ? kDepth - 2 : kDepth;    // (the prefix tokens' values take the other two places)
        for (int i = 0; i < min(count, early); ++i) fetch(i);
        v8h q[CB][NG * KS];
        float c0[CB][NG];
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const v4u minus8 = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v4f z = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    q[c][g * KS + s] = in_key_order(raw[c][g * KS + s]);
                    z = product(__builtin_bit_cast(v8h, minus8), q[c][g * KS + s], z);
                }
                c0[c][g] = z[0];
            }
        }
        const float scale = a.softmax_scale * 1.44269504088896341f;
        float c1 = scale * kUnit, v_step = 1.0f;
        if constexpr (!DYNAMIC) {
            c1 *= a.cache.k_scale[head];
            v_step = a.cache.v_scale[head];
        }

        float m[CB], l[CB];                        // l: of this lane's tokens
        float l_free[CB];                          // static steps: of tokens whose values' offset is not in o (prefix), or no longer
        v4f o[CB][NG * CH];
        float ref[CB][NG], lw[CB][NG];             // dynamic steps: weights p * step are rounded relative to ref
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            m[c] = kNothing;
            l[c] = l_free[c] = 0.0f;
#pragma unroll
            for (int i = 0; i < NG * CH; ++i) o[c][i] = (v4f){0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                ref[c][g] = kLeast;
                lw[c][g] = 0.0f;
            }
        }

        // exp2(c1 x + bias - m) of the scores x [16 (i / 4) + 4 quarter + i % 4]; the reference m follows the largest, what is there is rescaled.
        auto probabilities = [&](int c, float (&x)[8], float c1, float bias) PQ_INLINE -> float {
            float most = x[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) most = fmaxf(most, x[i]);
            most = fmaf(most, c1, bias);
            if (__builtin_amdgcn_ballot_w64(most > m[c] + kMost) != 0) {
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float to_m = most > m[c] + kMost ? ceilf(most) - kBack : m[c];
                const float alpha = __builtin_amdgcn_exp2f(m[c] - to_m);
                m[c] = to_m;
                l[c] *= alpha;
                if constexpr (DYNAMIC) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const float at = ref[c][g] * alpha, f = at >= kLeast ? 1.0f : at * (1.0f / kLeast);
                        ref[c][g] = fmaxf(at, kLeast);
                        lw[c][g] *= f;
#pragma unroll
                        for (int i = 0; i < CH; ++i) o[c][g * CH + i] *= f;
                    }
                } else {
                    l_free[c] *= alpha;
#pragma unroll
                    for (int i = 0; i < NG * CH; ++i) o[c][i] *= alpha;
                }
            }
            const float minus = bias - m[c];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c1, minus));
            if constexpr (DYNAMIC) l[c] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            return __builtin_amdgcn_exp2f(most - m[c]);
        };

        // ---- prefix tokens, by the run that begins the history
        if (prefix) {
            const uint32_t to_addr = ring_addr + (kDepth - 2) * S::SLOT;
            const __half* const values = reinterpret_cast<const __half*>(ring + (kDepth - 2) * S::SLOT);
            static_assert(2 * S::SLOT >= kTile * D * 2, "32 tokens in fp16");
            for (int t0 = 0; t0 < a.n_prefix; t0 += kTile) {
#pragma unroll
                for (int i = 0; i < kTile * D * 2 / 1024; ++i) {
                    const int at = 1024 * i + 16 * lane, t = min(t0 + at / (2 * D), a.n_prefix - 1);
                    to_lds16(reinterpret_cast<const uint8_t*>(a.prefix_v + ((int64_t)t * Hkv + head) * D) + at % (2 * D), to_addr + 1024 * i);
                }
                float x[CB][8];
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const int t = min(t0 + 16 * blk + col, a.n_prefix - 1);
                    const __half* src = a.prefix_k + ((int64_t)t * Hkv + head) * D;
                    v4f z[CB];
#pragma unroll
                    for (int c = 0; c < CB; ++c) z[c] = (v4f){0, 0, 0, 0};
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int s = 0; s < KS; ++s) {
                            const v8h w = in_key_order(*reinterpret_cast<const v4u*>(src + g * G + quarter * (G / 4) + 8 * s));
#pragma unroll
                            for (int c = 0; c < CB; ++c) z[c] = product(w, q[c][g * KS + s], z[c]);
                        }
                    const int left = a.n_prefix - (t0 + 16 * blk + 4 * quarter);
#pragma unroll
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[c][4 * blk + i] = i < left ? z[c][i] : -INFINITY;
                }
                v4u pr[CB], rest[CB];
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    probabilities(c, x[c], scale, 0.0f);
                    pr[c] = in_halves(x[c]);
                    rest[c] = rest_in_halves(x[c]);
                    if constexpr (!DYNAMIC) l[c] = add_eight(rest[c], add_eight(pr[c], l[c]));
                }
                wait_vm<0>();
#pragma unroll
                for (int i = 0; i < NG * CH; ++i) {
                    const int ch = i / CH * G + CH * col + i % CH;
                    v8h w;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        w[k] = *reinterpret_cast<const _Float16*>(values + (16 * (k >> 2) + 4 * quarter + (k & 3)) * D + ch);
#pragma unroll
                    for (int c = 0; c < CB; ++c) o[c][i] = product(w, __builtin_bit_cast(v8h, rest[c]), product(w, __builtin_bit_cast(v8h, pr[c]), o[c][i]));
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read before the next values, or codes, take their place)
            }
            // in units of a code; their sum of p apart, so that no offset is added here to be taken off again: its rounding would be 2^-21 of
            // a step, and where these tokens have the weight their values may be far smaller
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const float times = DYNAMIC ? 1.0f / (kUnit * kLeast) : 1.0f / (kUnit * v_step);
#pragma unroll
                for (int i = 0; i < NG * CH; ++i) o[c][i] *= times;
#pragma unroll
                for (int g = 0; g < NG; ++g) ref[c][g] = kLeast;
                if constexpr (!DYNAMIC) {
                    l_free[c] = l[c];
                    l[c] = 0.0f;
                }
            }
            for (int i = early; i < min(count, kDepth); ++i) fetch(i);
        }

        // ---- the history
        for (int i = 0; i < count; ++i) {
            const int t0 = start_of(i), place = i % kDepth;
            // until this tile is there; those behind it may be on their way
            const int behind = min(count - 1 - i, kDepth - 1);
            if (behind == 3) wait_vm<3 * S::LOADS>();
            else if (behind == 2) wait_vm<2 * S::LOADS>();
            else if (behind == 1) wait_vm<S::LOADS>();
            else wait_vm<0>();
            const uint8_t* const kc = ring + place * S::SLOT;
            const uint8_t* const vc = kc + S::CODES;
            const bool bad0 = (bad_bits >> (2 * place)) & 1, bad1 = (bad_bits >> (2 * place + 1)) & 1;
            const bool masked = t0 + kTile > all_see || bad0 || bad1 || (MASKED && t0 < seen.lo_top && t0 + kTile > a.sinks);
            uint32_t k[2][NG * KS], v[8][NG];
            v4f ks[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1], vs[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1];
            // (steps of four tokens, NG each, one after another; every 32 steps of keys are followed by 32 of values)
            auto steps = [&](int blk, int j) PQ_INLINE {
                const int e = (16 * blk + 4 * quarter) * NG + 4 * j;
                return kc + 2 * S::CODES + e / 32 * 256 + e % 32 * 4;
            };
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const uint8_t* src = kc + (16 * blk + col) * (D / 2) + g * (G / 2) + quarter * (G / 8);
                    if constexpr (KS == 4) {
                        const v4u w = *reinterpret_cast<const v4u*>(src);
#pragma unroll
                        for (int s = 0; s < 4; ++s) k[blk][g * KS + s] = w[s];
                    } else if constexpr (KS == 2) {
                        const v2u w = *reinterpret_cast<const v2u*>(src);
                        k[blk][g * KS] = w[0];
                        k[blk][g * KS + 1] = w[1];
                    } else {
                        k[blk][g] = *reinterpret_cast<const uint32_t*>(src);
                    }
                    if constexpr (DYNAMIC) ks[blk][g] = *reinterpret_cast<const v4f*>(steps(blk, g));
                }
            auto values = [&]() PQ_INLINE {
#pragma unroll
                for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint8_t* from_v = vc + (16 * blk + 4 * quarter + j) * (D / 2) + g * (G / 2) + col * (G / 32);
                            if constexpr (KS == 4) v[4 * blk + j][g] = *reinterpret_cast<const uint32_t*>(from_v);
                            else if constexpr (KS == 2) v[4 * blk + j][g] = *reinterpret_cast<const uint16_t*>(from_v);
                            else v[4 * blk + j][g] = *from_v;
                        }
                        if constexpr (DYNAMIC) vs[blk][g] = *reinterpret_cast<const v4f*>(steps(blk, g) + 128);
                    }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // read before the next tile takes this place
                if (i + kDepth < count) fetch(i + kDepth);
            };
            // (four groups, or two and two blocks of rows: keys and values at once would not fit the registers)
            constexpr bool kLater = NG * CB >= 4;
            if constexpr (!kLater) values();

            float x[CB][8], top[CB];               // top: the largest of this lane's x, or of its column's
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    v4f z[CB];
#pragma unroll
                    for (int c = 0; c < CB; ++c) z[c] = (v4f){0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < KS; ++s) {
                        const v8h w = key_operand(k[blk][g * KS + s]);
#pragma unroll
                        for (int c = 0; c < CB; ++c) z[c] = product(w, q[c][g * KS + s], z[c]);
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float& to_x = x[c][4 * blk + j];
                            if constexpr (DYNAMIC) to_x = fmaf(z[c][j] + c0[c][g], ks[blk][(j * NG + g) / 4][(j * NG + g) % 4], g == 0 ? 0.0f : to_x);
                            else to_x = z[c][j];
                        }
                }
            if (masked) {
#pragma unroll
                for (int c = 0; c < CB; ++c) {
                    const int left = limit[c] - (t0 + 4 * quarter);
                    if constexpr (MASKED) {        // a bit for each of 32 tokens from this lane's first on
                        auto below = [](int n) PQ_INLINE -> uint32_t { return n <= 0 ? 0 : n >= 32 ? ~0u : (1u << n) - 1; };
                        uint32_t see = below(left) & (~below(lo[c] - (t0 + 4 * quarter)) | below(a.sinks - (t0 + 4 * quarter)));
                        if (tree && t0 + kTile > all_see)          // nodes of its mask, behind the limit
                            see |= (mask_bits(a, r, min(tile * ROWS + 16 * c + col, rows - 1) / per_kv, t0 - (r.sees - 1)) >> (4 * quarter)) & ~below(left);
                        if (bad0) see &= 0xFFFF0000u;
                        if (bad1) see &= 0x0000FFFFu;
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[c][j] = (see >> (16 * (j >> 2) + (j & 3))) & 1 ? x[c][j] : -INFINITY;
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (16 * (j >> 2) + (j & 3) >= left || (j < 4 ? bad0 : bad1)) x[c][j] = -INFINITY;
                }
            }
#pragma unroll
            for (int c = 0; c < CB; ++c) top[c] = probabilities(c, x[c], c1, DYNAMIC ? 0.0f : c0[c][0] * c1);
            if constexpr (kLater) values();
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v4u pr[CB];
                float w[CB][8];                            // the product's weights
                // Up to 32 rows in one block: where a weight is more than its lane has added up so far, what fp16 leaves of this tile's weights is
                // multiplied as well, so that a weight which is more than half of a sum is never rounded to 11 bits.  Errors in multiples of those
                // of rounding the exact result, without | with it, median and largest: 3 requests of up to 131072 tokens, dynamic steps, 30 sets
                // of inputs 1.39, 1.62 | 1.11, 1.34, one token of one request 1.36, 1.52 | 1.00, 1.00, drafted tokens 1.42, 1.45 | 1.01, 1.07.
                // It costs 75.8 -> 78.5 us, 11.7 -> 11.9, 23.1 -> 24.5; 64 requests of up to 8192 tokens 73.4 -> 75.  (Always: 73 -> 77.5.  More
                // rows make an average that needs none: 1.41, and steps to 32 channels would take 7 % longer.)
                bool large = false;
                const bool split = CB == 1 && tiles <= 2;
                if constexpr (!DYNAMIC) {
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[c][j] = x[c][j];
                        pr[c] = in_halves(w[c]);
                        if (split) large |= __builtin_amdgcn_ballot_w64(top[c] > l[c]) != 0;
                        l[c] = add_eight(pr[c], l[c]);
                    }
                } else {
                    float step[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) step[j] = vs[j >> 2][((j & 3) * NG + g) / 4][((j & 3) * NG + g) % 4];
                    if (masked) {
                        // what lies behind the last token may be anything, and what only later queries see may be infinite: neither must
                        // meet a probability of zero as it is
                        const int left = r.n - (t0 + 4 * quarter);
#pragma unroll
                        for (int j = 0; j < 8; ++j) step[j] = 16 * (j >> 2) + (j & 3) >= left || (j < 4 ? bad0 : bad1) ? 0.0f : finite_step(step[j]);
                        asm volatile("");          // (a branch: computed for every tile it costs one of 32 channels to a step 5 %)
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        float most = 0.0f;
                        const float inv = inverse(ref[c][g]);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            w[c][j] = x[c][j] * inv * step[j];
                            most = fmaxf(most, w[c][j]);
                        }
                        if (__builtin_amdgcn_ballot_w64(most > 0x1.0p14f) != 0) {
                            most = fmaxf(most, __shfl_xor(most, 16, 64));
                            most = fmaxf(most, __shfl_xor(most, 32, 64));
                            const int up = most > 0x1.0p14f ? ilogbf(most) - (int)kBack : 0;
                            const float f = ldexpf(1.0f, -up);
                            ref[c][g] = ldexpf(ref[c][g], up);
                            lw[c][g] *= f;
                            most *= f;
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[c][j] *= f;
#pragma unroll
                            for (int j = 0; j < CH; ++j) o[c][g * CH + j] *= f;
                        }
                        pr[c] = in_halves(w[c]);
                        if (split) large |= __builtin_amdgcn_ballot_w64(most > lw[c][g]) != 0;
                        lw[c][g] = add_eight(pr[c], lw[c][g]);
                    }
                }
                uint32_t low[4], high[4];                  // codes of tokens 2 j and 2 j + 1
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    low[j] = __builtin_amdgcn_perm(v[2 * j + 1][g], v[2 * j][g], 0x05040100u) ^ kOffset;
                    if constexpr (CH == 8) high[j] = __builtin_amdgcn_perm(v[2 * j + 1][g], v[2 * j][g], 0x07060302u) ^ kOffset;
                }
                auto products = [&](const v4u (&p)[CB]) PQ_INLINE {
                    static_for<0, CH>([&](auto J) PQ_INLINE {
                        constexpr int j = decltype(J)::value;
                        v4u u;
#pragma unroll
                        for (int n = 0; n < 4; ++n) u[n] = operand<(j & 3)>(j < 4 ? low[n] : high[n]);
#pragma unroll
                        for (int c = 0; c < CB; ++c)
                            o[c][g * CH + j] = product(__builtin_bit_cast(v8h, u), __builtin_bit_cast(v8h, p[c]), o[c][g * CH + j]);
                    });
                };
                products(pr);
                if (large) {
                    v4u rest[CB];
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        rest[c] = rest_in_halves(w[c]);
                        if constexpr (DYNAMIC) lw[c][g] = add_eight(rest[c], lw[c][g]);
                        else l[c] = add_eight(rest[c], l[c]);
                    }
                    products(rest);
                }
            }
            // The codes' offset is taken off every 64 tiles: over n tokens of like weight it is some 2 sqrt(n) times the values' sum, and its
            // roundings would pass the result's own after a few thousand tokens in a row.
            if (i % 64 == 63) {
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        float& sum = DYNAMIC ? lw[c][g] : l[c];
                        float all = sum + __shfl_xor(sum, 16, 64);
                        all += __shfl_xor(all, 32, 64);
                        all *= 8.0f / kUnit;
#pragma unroll
                        for (int j = 0; j < CH; ++j) o[c][g * CH + j] -= all;
                        if constexpr (!DYNAMIC) l_free[c] += sum;
                        sum = 0.0f;
                    }
            }
        }

        // ---- results.  Block j of a group holds channels CH * row + j: a lane's rows 4 quarter .. + 3 are 4 CH channels in a row.
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            l[c] += __shfl_xor(l[c], 16, 64);
            l[c] += __shfl_xor(l[c], 32, 64);
            float l_all = l[c];
            if constexpr (!DYNAMIC) {
                l_free[c] += __shfl_xor(l_free[c], 16, 64);
                l_all += l_free[c] + __shfl_xor(l_free[c], 32, 64);
            }
            const int row = tile * ROWS + 16 * c + col;
            const bool live = row < rows;
            const float f = take == per ? (l_all > 0.0f ? v_step / l_all : 0.0f) : v_step;
            float* const part = partial + (((int64_t)worker * 2 + (u0 == range ? 0 : 1)) * ROWS + 16 * c + col) * (D + 4);
            __half* const dst = a.out + ((int64_t)(r.start + min(row, rows - 1) / per_kv) * a.n_heads + head * per_kv + min(row, rows - 1) % per_kv) * D;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float times = kUnit * f, minus = 8.0f * l[c] * f;
                if constexpr (DYNAMIC) {
                    float lw_all = lw[c][g] + __shfl_xor(lw[c][g], 16, 64);
                    lw_all += __shfl_xor(lw_all, 32, 64);
                    times = kUnit * ref[c][g] * f;
                    minus = 8.0f * lw_all * ref[c][g] * f;
                }
                const int ch = g * G + 4 * CH * quarter;
                if (!live) continue;
                if (take == per) {
#pragma unroll
                    for (int i = 0; i < 4 * CH; i += 8) {
                        v4u w;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            w[j] = two_halves(fmaf(o[c][g * CH + (i + 2 * j) % CH][(i + 2 * j) / CH], times, -minus),
                                              fmaf(o[c][g * CH + (i + 2 * j + 1) % CH][(i + 2 * j + 1) / CH], times, -minus));
                        *reinterpret_cast<v4u*>(dst + ch + i) = w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4 * CH; i += 4) {
                        v4f w;
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = fmaf(o[c][g * CH + (i + j) % CH][(i + j) / CH], times, -minus);
                        *reinterpret_cast<v4f*>(part + 4 + ch + i) = w;
                    }
                }
            }
            if (live && take != per && quarter == 0) {
                part[0] = m[c];
                part[1] = l_all;
            }
        }
        u0 += take;
    }
}

// Row `row` of one history that was cut, by a wavefront: two channels (one of 64) and one part's maximum and sum to a lane.
template <int D> struct Joined {
    float top = kNothing, sum = 0.0f, acc[D / 64] = {};
};

// The next COUNT or fewer parts.  All their loads are on their way before the first is used: one after another they would take a microsecond
// each, and a second one if they waited for the maxima.
template <int D, int COUNT>
__device__ __forceinline__ void add_parts(Joined<D>& j, const float* __restrict__ first, int64_t step, int64_t second, int n0, int n, int lane)
{
    constexpr int kEach = D / 64;
    float x[COUNT][kEach];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const int at = n0 + min(i, n - 1);
        const float* src = first + at * step + (at == 0 ? second : 0) + 4 + kEach * lane;
#pragma unroll
        for (int k = 0; k < kEach; ++k) x[i][k] = src[k];
    }
    const int mine = n0 + min(lane, n - 1);
    const float* const head = first + mine * step + (mine == 0 ? second : 0);
    const float m = lane < n ? head[0] : kNothing, l = lane < n ? head[1] : 0.0f;
    float to = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) to = fmaxf(to, __shfl_xor(to, d, 64));
    to = fmaxf(to, j.top);
    const float old = __builtin_amdgcn_exp2f(j.top - to), f = lane < n ? __builtin_amdgcn_exp2f(m - to) : 0.0f;
    float part = l * f;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) part += __shfl_xor(part, d, 64);
    j.sum = fmaf(j.sum, old, part);
#pragma unroll
    for (int k = 0; k < kEach; ++k) j.acc[k] *= old;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const float fi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), i));
#pragma unroll
        for (int k = 0; k < kEach; ++k) j.acc[k] = fmaf(x[i][k], fi, j.acc[k]);
    }
    j.top = to;
}

// Parts n0 .. end - 1 of a row.  (MASKED: in more sizes, fewer loads that are not wanted: 16 requests of 8 nodes over 4000 tokens 38.7 -> 37.0 us, one of
// 26 over 3000 25.1 -> 24.5.)
template <int D, int CB, bool MASKED = false>
__device__ __forceinline__ Joined<D> add_up(const float* __restrict__ partial, const Item& item, int row, int n0, int end, int lane)
{
    constexpr int ROWS = 16 * CB;
    Joined<D> j;
    const float* const first = partial + ((int64_t)item.worker * 2 * ROWS + row) * (D + 4);
    const int64_t step = 2 * ROWS * (D + 4), second = item.second ? ROWS * (D + 4) : 0;
    for (; end - n0 > 8; n0 += 64) {
        const int n = min(end - n0, 64);
        if (MASKED && n > 32 && n <= 48) add_parts<D, 48>(j, first, step, second, n0, n, lane);
        else if (n > 32) add_parts<D, 64>(j, first, step, second, n0, n, lane);
        else if (MASKED && n <= 16) add_parts<D, 16>(j, first, step, second, n0, n, lane);
        else add_parts<D, 32>(j, first, step, second, n0, n, lane);
    }
    if (n0 < end) add_parts<D, 8>(j, first, step, second, n0, end - n0, lane);
    return j;
}

template <int D>
__device__ __forceinline__ void write_joined(const AttentionArgs& a, const Joined<D>& j, const Item& item, int row, int lane)
{
    constexpr int kEach = D / 64;
    const float f = j.sum > 0.0f ? 1.0f / j.sum : 0.0f;
    const int at_row = item.row0 + row, per_kv = a.heads_per_kv;
    __half* dst = a.out + ((int64_t)(item.start + at_row / per_kv) * a.n_heads + item.head * per_kv + at_row % per_kv) * D + kEach * lane;
    if constexpr (kEach == 2) *reinterpret_cast<__half2*>(dst) = __floats2half2_rn(j.acc[0] * f, j.acc[1] * f);
    else *dst = __float2half_rn(j.acc[0] * f);
}

// Adds the partial sums of the histories that were cut: a workgroup takes four rows of one, one to a wavefront.
constexpr int kJoinGroups = 1 << 16;     // (there may be more histories than a launch can have workgroups)
template <int D, int CB, bool MASKED>
__device__ __forceinline__ void join_items(const AttentionArgs& a, const float* __restrict__ partial, const Item* __restrict__ items, uint32_t group, uint32_t groups)
{
    const int lane = threadIdx.x & 63, row = blockIdx.y * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int count = items[0].parts;
    Item item = items[1 + group];                                        // (of the last call, or nothing, from the count on)
    for (int64_t i = group; i < count; i += groups) {
        if (i != group) item = items[1 + i];
        if (item.parts > 1 && item.row0 + row < item.rows) write_joined<D>(a, add_up<D, CB, MASKED>(partial, item, row, 0, item.parts, lane), item, row, lane);
    }
}
template <int D, int CB>
__global__ __launch_bounds__(kThreads) void k_kv4_attention_join(AttentionArgs a, const float* __restrict__ partial, const Item* __restrict__ items)
{
    join_items<D, CB, false>(a, partial, items, blockIdx.x, gridDim.x);
}

// The same with a workgroup to a row, each of its wavefronts adding a quarter of the parts.
template <int D, int CB>
__device__ __forceinline__ void join_items_together(const AttentionArgs& a, const float* __restrict__ partial, const Item* __restrict__ items, uint32_t group, uint32_t groups)
{
    constexpr int kEach = D / 64;
    __shared__ float quarters[kWaves][2 + kEach][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = blockIdx.y;
    const int count = items[0].parts;
    for (int64_t i = group; i < count; i += groups) {
        const Item item = items[1 + i];
        if (item.parts <= 1 || item.row0 + row >= item.rows) continue;
        const int each = (item.parts + kWaves - 1) / kWaves, from = min(wave * each, item.parts);
        Joined<D> j = add_up<D, CB, true>(partial, item, row, from, min(from + each, item.parts), lane);
        quarters[wave][0][lane] = j.top;
        quarters[wave][1][lane] = j.sum;
#pragma unroll
        for (int k = 0; k < kEach; ++k) quarters[wave][2 + k][lane] = j.acc[k];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const float top = quarters[w][0][lane], to = fmaxf(j.top, top), old = __builtin_amdgcn_exp2f(j.top - to), f = __builtin_amdgcn_exp2f(top - to);
                j.top = to;
                j.sum = fmaf(j.sum, old, quarters[w][1][lane] * f);
#pragma unroll
                for (int k = 0; k < kEach; ++k) j.acc[k] = fmaf(j.acc[k], old, quarters[w][2 + k][lane] * f);
            }
            write_joined<D>(a, j, item, row, lane);
        }
        __syncthreads();                           // (read before the next item's)
    }
}

// Behind the masked row kernel; where the tile kernel comes then (runs > 0), one workgroup more makes its plan meanwhile.  Few histories, of many parts
// each, are joined by workgroups together.  A wavefront | a workgroup to a row, us of the whole call, 32 heads of 128 on 8: one token over 1600
// tokens (8 histories) 13.5 | 12.1, over 12000 33.1 | 20.9, over 50000 36.4 | 27.7; 8 nodes over 12000 (24) 28.2 | 24.0; four requests' tokens over
// 12000 (40) 25.0 | 22.4; 26 nodes over 3000 (56) 25.4 | 26.0; four requests of 26 over 4000 (over 200) 29.9 | 32.9.
constexpr int kFewItems = 48;
template <int D, int CB, bool TOGETHER>
__global__ __launch_bounds__(kThreads) void k_kv4_attention_join_masked(AttentionArgs a, const float* __restrict__ partial, const Item* __restrict__ items, RunPlan p,
                                                                        int runs, int small_rows)
{
    const uint32_t plans = runs > 0 ? 1 : 0;
    if (blockIdx.x < plans) {
        if (blockIdx.y == 0) make_plan<kThreads>(a, p, runs, small_rows);
    } else if constexpr (TOGETHER) {
        join_items_together<D, CB>(a, partial, items, blockIdx.x - plans, gridDim.x - plans);
    } else {
        join_items<D, CB, true>(a, partial, items, blockIdx.x - plans, gridDim.x - plans);
    }
}

// What a call has at most: histories (of 16 rows), and workgroups with something to do.
struct Most {
    int64_t items, units, groups;
};
Most at_most(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int64_t capacity, int small_rows)
{
    const int64_t by_rows = T * (n_heads / n_kv_heads) / 16 + B, by_requests = ((int64_t)small_rows + 15) / 16 * B;
    const int64_t items = (by_rows < by_requests ? by_rows : by_requests) * n_kv_heads, units = items * ((capacity + kTile - 1) / kTile);
    return {items, units, (units + kWaves - 1) / kWaves};
}

// Scratch memory: partial sums, two to a wavefront, then the list of histories.
size_t partial_bytes(int64_t groups, int32_t head_dim, int blocks)
{
    return (size_t)(groups < kGroups ? groups : kGroups) * kWaves * 2 * 16 * blocks * (head_dim + 4) * sizeof(float);
}

template <int D, int G, bool DYNAMIC, int CB, typename... KIND>
int launch(const AttentionArgs& a, int small_rows, int64_t capacity, void* ws, const TilePlan* tiles, hipStream_t st)
{
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t lds = Shape<D, G, DYNAMIC, CB>::kLds;
    const auto kernel = k_kv4_attention_rows<D, G, DYNAMIC, CB, KIND...>;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, allowed); rc != PQ_OK) return rc;
    const Most most = at_most(a.T, a.B, a.n_heads, a.cache.n_kv_heads, capacity, small_rows);
    const int64_t groups = most.groups < kGroups ? most.groups : kGroups;
    float* const partial = static_cast<float*>(ws);
    Item* const items = reinterpret_cast<Item*>(static_cast<uint8_t*>(ws) + partial_bytes(most.groups, D, CB));
    kernel<<<(unsigned)groups, kThreads, lds, st>>>(a, partial, items, most.items, small_rows);
    const unsigned joins = (unsigned)(most.items < kJoinGroups ? most.items : kJoinGroups);
    if constexpr (sizeof...(KIND) > 0) {
        const TilePlan then = tiles ? *tiles : TilePlan{};
        const unsigned groups = joins + (tiles ? 1 : 0);
        if (most.items <= kFewItems) k_kv4_attention_join_masked<D, CB, true><<<dim3(groups, 16 * CB), kThreads, 0, st>>>(a, partial, items, then.plan, then.runs, small_rows);
        else k_kv4_attention_join_masked<D, CB, false><<<dim3(groups, 4 * CB), kThreads, 0, st>>>(a, partial, items, then.plan, then.runs, small_rows);
    } else {
        k_kv4_attention_join<D, CB><<<dim3(joins, 4 * CB), kThreads, 0, st>>>(a, partial, items);
    }
    return hip_status(hipGetLastError());
}

// Column blocks: two where requests have more than 16 rows and the histories of 16 rows may be more than 48 units for every wavefront (the host
// knows the table, not the lengths: under a table far longer than the histories the choice is two); with less to do, twice the runs of half
// the work are faster.  One | two, us, 32 heads of 128 on 8: 16 requests of 2000 to 4000 tokens with 20 rows 36 | 34, 32 rows (32000 units) 37 |
// 40, 64 rows 50 | 48, 128 rows (128000) 78 | 66; 64 requests with 20 rows (up to 128000) 81 | 66, 32 rows 84 | 78, 128 rows 261 | 197; one of
// 131072 with 48 rows (98000) 85 | 75; one step to a head, 64 requests, 128 rows 297 | 229.  Four groups of dynamic steps would not fit the
// registers twice (16 requests, 64 rows 64 | 85; 64 requests, 128 rows 326 | 339).  The masked kernel's two blocks with a step to 64 channels spill 8
// registers and are worth it: 64 trees of up to 3000 tokens, one | two blocks, 96, 104, 128 and 160 rows 232 | 180, 256 | 218, 318 | 241, 362 | 271.
int blocks_for(int32_t max_q, int32_t per_kv, int64_t units) { return (int64_t)max_q * per_kv > 16 && units > 48 * kGroups * kWaves ? 2 : 1; }

// The masked tile kernel cuts its work into equal runs and leaves out wavefronts without rows, so it is worth its launches earlier, where a
// call has much to do.  Row | tile kernel, us, trees, 32 heads of 128 on 8, with 64, 104, 128 and 192 rows: 64 requests of up to 3000 tokens 94 | 115,
// 128 | 126, 154 | 131, 205 | 159, with a step to 32 channels 161 | 253, 238 | 266, 293 | 283, 400 | 323; 16 of 4000 46 | 54, 66 | 62, 61 | 57,
// 74 | 66; with less to do, 4 of 4000, 29 | 35, 30 | 38, 37 | 39, 43 | 47, one of 3000 23 | 33, 26 | 36, 27 | 36, 29 | 43.  Just above the border, with
// 108, 112, 120 and 160 rows, 64 requests of up to 3000: static steps 172 | 135, 166 | 129, 178 | 137, 200 | 164; one step to 128 channels 190 | 177,
// 193 | 182, 198 | 185, 239 | 224; to 64 222 | 212, 220 | 208, 231 | 219, 271 | 262; to 32 311 | 279, 351 | 312, 370 | 298, 439 | 340.  16 of 4000:
// 67 | 59, 69 | 61, 67 | 59, 82 | 75; 78 | 78, 78 | 81, 75 | 78, 89 | 92; 89 | 90, 92 | 96, 90 | 92, 97 | 103; 115 | 114, 121 | 120, 134 | 122, 131 | 115.
constexpr int kMaskedSmallRows = 104;
constexpr int64_t kMuch = 4096;          // steps of 64 tokens, of all requests and heads
int border_for(int32_t B, int32_t n_kv_heads, int32_t per_kv, const Histories& h)
{
    return h.masked && (int64_t)B * n_kv_heads * h.seen_by(kSmallRows / per_kv) >= 64 * kMuch ? kMaskedSmallRows : kSmallRows;
}
bool takes_tiles(int32_t max_q, int32_t per_kv, int border) { return (int64_t)max_q * per_kv > border; }
// A single request is the tile kernel's whatever its rows are: the two launches that would find nothing to do take 4 us (1024 tokens of one
// prompt, 32 heads on 8: 38 us with them, 34 without); with the masked one, which spreads a single row's steps over all workgroups as well, also some
// that see little, four steps to a workgroup at most.  Two row launches more | all rows in tiles, us, one prompt and B - 1 tokens, 32 heads of 128 on 8,
// by the tokens' steps in all: 54 steps (B 2, window 256) prompts of 300, 1500 and 3100 47 | 42, 54 | 46, 75 | 69; 590 (B 5, 1000) 49 | 41, 75 | 67,
// 108 | 103; 872 (B 17, 256) 49 | 41, 57 | 56, 81 | 63; 1090 (B 5, 2000) 54 | 48, 97 | 96, 155 | 151; 2180 (B 9, 2000) 56 | 56, 101 | 87, 158 | 161; 4360
// (B 17, 2000) 61 | 71, 107 | 120, 164 | 180.  (A prompt of 2000 tokens is 256 tiles and heads, one to a run and none cut, and any more cut them: 46 | 54.)
// Trees of 26 gain longer, their rows fill more of a tile: beside 300 tokens 750 steps 66 | 51, 4125 98 | 74, 11625 153 | 131.
int small_rows_for(int32_t max_q, int32_t per_kv, int32_t B, int32_t n_kv_heads, const Histories& h)
{
    const int border = border_for(B, n_kv_heads, per_kv, h);
    if (!takes_tiles(max_q, per_kv, border)) return INT32_MAX;
    const bool little = h.masked && (int64_t)(B - 1) * n_kv_heads * h.seen_by(border / per_kv) <= 64 * 4 * 256;
    return B == 1 || little ? 0 : border;
}

size_t rows_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, int small_rows, const Histories& h)
{
    if (small_rows == 0) return 0;
    const Most most = at_most(T, B, n_heads, n_kv_heads, h.seen_by(max_q), small_rows);
    return (partial_bytes(most.groups, head_dim, blocks_for(max_q, n_heads / n_kv_heads, most.units)) + (size_t)(most.items + 1) * sizeof(Item) + 255) & ~(size_t)255;
}

template <int CB, typename... KIND>
int launch_rows(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, int64_t capacity, void* ws, const TilePlan* tiles, hipStream_t st)
{
    if (head_dim == 64) {
        if (group == 0) return launch<64, 64, false, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
        if (group == 32) return launch<64, 32, true, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
        return launch<64, 64, true, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
    }
    if (group == 0) return launch<128, 128, false, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
    if (group == 32) return launch<128, 32, true, 1, KIND...>(a, small_rows, capacity, ws, tiles, st);
    if (group == 64) return launch<128, 64, true, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
    return launch<128, 128, true, CB, KIND...>(a, small_rows, capacity, ws, tiles, st);
}

}  // namespace

size_t attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, const Histories& h)
{
    const int32_t per_kv = n_heads / n_kv_heads;
    const int small_rows = small_rows_for(max_q, per_kv, B, n_kv_heads, h);
    size_t all = rows_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, max_q, small_rows, h);
    if (small_rows != INT32_MAX)
        all += h.masked ? masked_tiles_workspace_bytes(T, B, per_kv, head_dim, small_rows) : tiles_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, h.table);
    return all > 256 ? all : 256;                  // (0 says that the sizes are refused)
}

int launch_attention(const AttentionArgs& a, int32_t head_dim, int32_t group, int32_t max_q, bool masked, void* ws, hipStream_t st)
{
    const Histories h = {(int64_t)a.table_pages << a.cache.log2_page, masked, a.window, a.sinks};
    const int small_rows = small_rows_for(max_q, a.heads_per_kv, a.B, a.cache.n_kv_heads, h);
    uint8_t* const tiles_ws = static_cast<uint8_t*>(ws) + rows_workspace_bytes(a.T, a.B, a.n_heads, a.cache.n_kv_heads, head_dim, max_q, small_rows, h);
    const bool some_tiles = small_rows != INT32_MAX;
    if (some_tiles && !masked) {
        const int rc = launch_attention_tiles(a, head_dim, group, small_rows, reinterpret_cast<float*>(tiles_ws), st);
        if (rc != PQ_OK || small_rows == 0) return rc;
    }
    const TilePlan plan = some_tiles && masked ? plan_of(a, head_dim, group, small_rows, tiles_ws) : TilePlan{};
    if (masked && small_rows == 0) return launch_masked_tiles(a, head_dim, group, small_rows, plan, false, st);
    const int64_t capacity = h.seen_by(max_q), units = at_most(a.T, a.B, a.n_heads, a.cache.n_kv_heads, capacity, small_rows).units;
    const bool one = blocks_for(max_q, a.heads_per_kv, units) == 1;
    auto rows = [&](auto launch) { return launch(a, head_dim, group, small_rows, capacity, ws, some_tiles ? &plan : nullptr, st); };
    if (!masked) return one ? rows(launch_rows<1>) : rows(launch_rows<2>);
    const int rc = one ? rows(launch_rows<1, Masked>) : rows(launch_rows<2, Masked>);
    return rc != PQ_OK || !some_tiles ? rc : launch_masked_tiles(a, head_dim, group, small_rows, plan, true, st);
}

}  // namespace kv4
}  // namespace pq
