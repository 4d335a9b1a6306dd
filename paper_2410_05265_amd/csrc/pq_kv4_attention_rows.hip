// Attention over the paged 4-bit cache for few queries of a request: decoded tokens, and some drafted ones.
//
// The queries of a request that share a key/value head (its tokens times the heads of the group) are the columns of the matrix instructions,
// 16 or 32 of them (CB blocks of 16), so that up to as many read every code once.  Bound by HBM: 128 bytes of codes for a token and head of
// 128 channels.
//
// Work is cut over the histories, in units of kUnitTokens tokens of one request, head and tile of rows.  All units of the call lie one after
// another, and every workgroup takes an equal run of them, whatever the requests' lengths are: a run that covers a history whole writes
// its outputs, one that begins or ends inside a history leaves a partial sum (at most two to a workgroup), and a second small kernel
// adds those, in the order of the workgroups.  The lengths are read on the device, so a captured call follows them.
//
// A wavefront takes 32 tokens at a time.  Their codes go from memory straight into its ring of kDepth places in LDS, so three tiles are on
// their way without a register; a lane then reads 16 bytes of a token's key codes (its part of every step of the first product), and 4
// bytes of each of eight tokens' value codes: an 8 x 8 block, whose transposition is a byte permutation of two tokens.
#include "pq_kv4_attention.h"

#define PQ_INLINE __attribute__((always_inline))

namespace pq {
namespace kv4 {
namespace {

__device__ __forceinline__ v4f product(const v8h& a, const v8h& b, const v4f& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 32;                          // tokens of a wavefront's step
constexpr int kUnitTokens = kTile * kWaves;
constexpr int kDepth = 4;                          // places of a wavefront's ring
constexpr int kWorkers = 512;                      // two workgroups to a CU, as their LDS allows
constexpr float kLeast = 0x1.0p-80f;               // smallest reference of value weights (dynamic steps)

__device__ __forceinline__ int64_t units_of_tile(const Request& r) { return r.n > 0 ? (r.n + kUnitTokens - 1) / kUnitTokens : 1; }

// Units of a request: (heads x tiles of rows) x units of its history; none if it has more than small_rows rows.
template <int ROWS>
__device__ __forceinline__ int64_t units_of(const AttentionArgs& a, const Request& r, int small_rows, int& tiles)
{
    const int64_t rows = (int64_t)r.q_len * a.heads_per_kv;
    tiles = rows > small_rows ? 0 : (int)((rows + ROWS - 1) / ROWS);
    return units_of_tile(r) * tiles * a.cache.n_kv_heads;
}

// The requests' units: each lane of the calling wavefront sums a run of requests.
struct Plan {
    int64_t total, before;      // all units; those before this lane's requests
    int64_t own;
    int first, last;            // this lane's requests
};

template <int ROWS>
__device__ __forceinline__ Plan plan(const AttentionArgs& a, int small_rows, int lane)
{
    Plan p;
    const int each = (a.B + 63) / 64;
    p.first = min(lane * each, a.B);
    p.last = min(p.first + each, a.B);
    p.own = 0;
    for (int b = p.first; b < p.last; ++b) {
        int tiles;
        p.own += units_of<ROWS>(a, request(a, b), small_rows, tiles);
    }
    int64_t incl = p.own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(incl, d, 64);
        if (lane >= d) incl += v;
    }
    p.before = incl - p.own;
    p.total = __shfl(incl, 63, 64);
    return p;
}

// The request that unit u (below the total) belongs to, and its first unit.
template <int ROWS>
__device__ __forceinline__ int find_request(const AttentionArgs& a, const Plan& p, int small_rows, int64_t u, int64_t& base)
{
    const bool mine = p.before <= u && u < p.before + p.own;
    int b = p.first;
    int64_t first = p.before;
    if (mine) {
        for (; b < p.last; ++b) {
            int tiles;
            const int64_t n = units_of<ROWS>(a, request(a, b), small_rows, tiles);
            if (u < first + n) break;
            first += n;
        }
    }
    const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));
    base = __shfl(first, from, 64);
    return __builtin_amdgcn_readfirstlane(__shfl(b, from, 64));
}

// 16 or 4 bytes of every lane from memory straight into LDS, lane after lane from lds_addr (wavefront-uniform) on.
__device__ __forceinline__ void to_lds16(const void* src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(lds_addr) : "memory");
}
__device__ __forceinline__ void to_lds4(const void* src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(lds_addr) : "memory");
}

template <int D, int G, bool DYNAMIC, int CB>
struct Shape {
    static constexpr int NG = D / G, KS = G / 32, CH = G / 16, ROWS = 16 * CB;
    static constexpr int CODES = kTile * D / 2;                          // bytes of a tile's keys, and of its values
    static constexpr int SLOT = 2 * CODES + (DYNAMIC ? 256 * NG : 0);
    static constexpr int LOADS = 2 * CODES / 1024 + (DYNAMIC ? NG : 0);  // of a tile
    static constexpr int PITCH = D + 4;                                  // floats of a row between the wavefronts' sums
    static constexpr int RING = kWaves * kDepth * SLOT, SUMS = kWaves * ROWS * PITCH * 4;
    static constexpr size_t kLds = (RING > SUMS ? RING : SUMS) + kWaves * ROWS * 8;
};

template <int D, int G, bool DYNAMIC, int CB>
__global__ __launch_bounds__(kThreads, 2) void k_kv4_attention_rows(AttentionArgs a, float* partial, int workers, int small_rows)
{
    typedef Shape<D, G, DYNAMIC, CB> S;
    constexpr int NG = S::NG, KS = S::KS, CH = S::CH, ROWS = S::ROWS;
    extern __shared__ __align__(256) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int log2_page = a.cache.log2_page, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv;
    float* const sums = reinterpret_cast<float*>(lds);                   // (over the rings)
    float* const sum_m = reinterpret_cast<float*>(lds + S::kLds - kWaves * ROWS * 8);
    float* const sum_l = sum_m + kWaves * ROWS;
    const uint8_t* const ring = lds + wave * kDepth * S::SLOT;
    const uint32_t ring_addr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)ring;

    const Plan p = plan<ROWS>(a, small_rows, lane);
    const int64_t total = p.total;
    const int active = (int)min((int64_t)workers, total);
    const int worker = xcd_run(blockIdx.x, gridDim.x);
    if (worker >= active) return;
    const int64_t range = total * worker / active, range_end = total * (worker + 1) / active;
    int64_t base;                                  // first unit of request b
    int b = find_request<ROWS>(a, p, small_rows, range, base);

    for (int64_t u0 = range; u0 < range_end;) {
        int tiles;
        const Request r = request(a, b);
        const int64_t whole = units_of<ROWS>(a, r, small_rows, tiles), per = units_of_tile(r);
        if (u0 >= base + whole) {                  // (requests without queries, or with many, have no units)
            base += whole;
            ++b;
            continue;
        }
        const int64_t item = (u0 - base) / per, from_unit = (u0 - base) % per, take = min(range_end - u0, per - from_unit);
        const int head = __builtin_amdgcn_readfirstlane((int)(item / tiles)), tile = __builtin_amdgcn_readfirstlane((int)(item % tiles));
        const int rows = r.q_len * per_kv;
        const int first_token = tile * ROWS / per_kv, last_token = min((tile * ROWS + ROWS - 1) / per_kv, r.q_len - 1);
        const int all_see = a.causal ? r.n - (r.q_len - 1 - first_token) : r.n;         // tokens before this one need no mask
        const int any_sees = a.causal ? r.n - (r.q_len - 1 - last_token) : r.n;
        const int from = (int)(from_unit * kUnitTokens), to = (int)min((from_unit + take) * kUnitTokens, (int64_t)max(any_sees, 0));

        // ---- codes on their way: this wavefront's tiles are from + 32 wave + 128 i
        const int32_t* table = a.table + (int64_t)b * a.table_pages;
        int ids_from = -64, ids = 0;
        const int t_first = from + wave * kTile;
        const int count = __builtin_amdgcn_readfirstlane(t_first < to ? (to - t_first + kUnitTokens - 1) / kUnitTokens : 0);
        uint32_t bad_bits = 0;                     // two bits for each place of the ring: blocks of 16 tokens whose page is none
        auto fetch = [&](int i) PQ_INLINE {
            const int t0 = t_first + i * kUnitTokens, place = i % kDepth;
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
            if constexpr (D == 128) {
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    to_lds16(a.cache.k_codes + first[blk] * 64 + 16 * lane, to_addr + 1024 * blk);
                    to_lds16(a.cache.v_codes + first[blk] * 64 + 16 * lane, to_addr + S::CODES + 1024 * blk);
                }
            } else {                               // 32 lanes to a block
                const int64_t at = (lane < 32 ? first[0] : first[1]) * 32 + 16 * (lane & 31);
                to_lds16(a.cache.k_codes + at, to_addr);
                to_lds16(a.cache.v_codes + at, to_addr + S::CODES);
            }
            if constexpr (DYNAMIC) {
#pragma unroll
                for (int j = 0; j < NG; ++j) {     // step e of the tile's 32 NG: token e / NG, group e % NG
                    const int e = 32 * j + (lane & 31), t = e / NG;
                    const int64_t at = ((t < 16 ? first[0] : first[1]) + (t & 15)) * NG + e % NG;
                    to_lds4((lane < 32 ? a.cache.k_scale : a.cache.v_scale) + at, to_addr + 2 * S::CODES + 256 * j);
                }
            }
        };
        const bool prefix = a.n_prefix > 0 && from_unit == 0 && wave == 0;
        const int early = prefix ? kDepth / 2 : kDepth;    // (the prefix tokens' values take the other places)
        for (int i = 0; i < min(count, early); ++i) fetch(i);

        // ---- queries: channels as the keys' operands have them
        v8h q[CB][NG * KS];
        float c0[CB][NG];
        int limit[CB];                             // tokens that the lane's query sees
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int row = min(tile * ROWS + 16 * c + col, rows - 1), token = row / per_kv, q_head = head * per_kv + row % per_kv;
            limit[c] = a.causal ? max(r.n - (r.q_len - 1 - token), 0) : r.n;
            const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
            const v4u minus8 = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v4f z = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    q[c][g * KS + s] = in_key_order(*reinterpret_cast<const v4u*>(src + g * G + quarter * (G / 4) + 8 * s));
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
        v4f o[CB][NG * CH];
        float ref[CB][NG], lw[CB][NG];             // dynamic steps: weights p * step are rounded relative to ref
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            m[c] = kNothing;
            l[c] = 0.0f;
#pragma unroll
            for (int i = 0; i < NG * CH; ++i) o[c][i] = (v4f){0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                ref[c][g] = kLeast;
                lw[c][g] = 0.0f;
            }
        }

        // exp2(c1 x + bias - m) of the scores x [16 (i / 4) + 4 quarter + i % 4]; the reference m follows the largest, what is there is rescaled.
        auto probabilities = [&](int c, float (&x)[8], float c1, float bias, v4u& pr) PQ_INLINE {
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
#pragma unroll
                    for (int i = 0; i < NG * CH; ++i) o[c][i] *= alpha;
                }
            }
            const float minus = bias - m[c];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c1, minus));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pr[i] = two_halves(x[2 * i], x[2 * i + 1]);
                l[c] = add_halves(pr[i], l[c]);
            }
        };

        // ---- prefix tokens, by the first wavefront of the run that begins the history
        if (prefix) {
            const uint32_t to_addr = ring_addr + kDepth / 2 * S::SLOT;
            const __half* const values = reinterpret_cast<const __half*>(ring + kDepth / 2 * S::SLOT);
            static_assert(kDepth / 2 * S::SLOT >= kTile * D * 2, "32 tokens in fp16");
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
                v4u pr[CB];
#pragma unroll
                for (int c = 0; c < CB; ++c) probabilities(c, x[c], scale, 0.0f, pr[c]);
                wait_vm<0>();
#pragma unroll
                for (int i = 0; i < NG * CH; ++i) {
                    const int ch = i / CH * G + CH * col + i % CH;
                    v8h w;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        w[k] = *reinterpret_cast<const _Float16*>(values + (16 * (k >> 2) + 4 * quarter + (k & 3)) * D + ch);
#pragma unroll
                    for (int c = 0; c < CB; ++c) o[c][i] = product(w, __builtin_bit_cast(v8h, pr[c]), o[c][i]);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (read before the next values, or codes, take their place)
            }
            // as if they were codes: sum p v = step (unit acc - 8 sum p) has to hold
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                float l_all = l[c] + __shfl_xor(l[c], 16, 64);
                l_all += __shfl_xor(l_all, 32, 64);
                const float times = DYNAMIC ? 1.0f / (kUnit * kLeast) : 1.0f / (kUnit * v_step), plus = DYNAMIC ? 0.0f : 8.0f / kUnit * l_all;
#pragma unroll
                for (int i = 0; i < NG * CH; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[c][i][k] = fmaf(o[c][i][k], times, plus);
#pragma unroll
                for (int g = 0; g < NG; ++g) ref[c][g] = kLeast;
            }
            for (int i = early; i < min(count, kDepth); ++i) fetch(i);
        }

        // ---- the history
        for (int i = 0; i < count; ++i) {
            const int t0 = t_first + i * kUnitTokens, place = i % kDepth;
            // until this tile is there; those behind it may be on their way
            const int behind = min(count - 1 - i, kDepth - 1);
            if (behind == kDepth - 1) wait_vm<(kDepth - 1) * S::LOADS>();
            else if (behind == 2) wait_vm<2 * S::LOADS>();
            else if (behind == 1) wait_vm<S::LOADS>();
            else wait_vm<0>();
            const uint8_t* const kc = ring + place * S::SLOT;
            const uint8_t* const vc = kc + S::CODES;
            const bool bad0 = (bad_bits >> (2 * place)) & 1, bad1 = (bad_bits >> (2 * place + 1)) & 1;
            const bool masked = t0 + kTile > all_see || bad0 || bad1;
            uint32_t k[2][NG * KS], v[8][NG];
            v4f ks[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1], vs[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1];
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
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint8_t* from_v = vc + (16 * blk + 4 * quarter + j) * (D / 2) + g * (G / 2) + col * (G / 32);
                        if constexpr (KS == 4) v[4 * blk + j][g] = *reinterpret_cast<const uint32_t*>(from_v);
                        else if constexpr (KS == 2) v[4 * blk + j][g] = *reinterpret_cast<const uint16_t*>(from_v);
                        else v[4 * blk + j][g] = *from_v;
                    }
                }
            if constexpr (DYNAMIC) {
                // steps of four tokens, NG each, one after another; every 32 steps of keys are followed by 32 of values
#pragma unroll
                for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const int e = (16 * blk + 4 * quarter) * NG + 4 * j;
                        const uint8_t* src = kc + 2 * S::CODES + e / 32 * 256 + e % 32 * 4;
                        ks[blk][j] = *reinterpret_cast<const v4f*>(src);
                        vs[blk][j] = *reinterpret_cast<const v4f*>(src + 128);
                    }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // read before the next tile takes this place
            if (i + kDepth < count) fetch(i + kDepth);

            float x[CB][8];
            v4u pr[CB];
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
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (16 * (j >> 2) + (j & 3) >= left || (j < 4 ? bad0 : bad1)) x[c][j] = -INFINITY;
                }
            }
#pragma unroll
            for (int c = 0; c < CB; ++c) probabilities(c, x[c], c1, DYNAMIC ? 0.0f : c0[c][0] * c1, pr[c]);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                if constexpr (DYNAMIC) {
                    float step[8];
                    const int left = r.n - (t0 + 4 * quarter);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = (j & 3) * NG + g;
                        step[j] = vs[j >> 2][e / 4][e % 4];
                        // what lies behind the last token may be anything: it must not meet a probability of zero
                        if (masked && (16 * (j >> 2) + (j & 3) >= left || (j < 4 ? bad0 : bad1))) step[j] = 0.0f;
                    }
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        float w[8], most = 0.0f;
                        const float inv = 1.0f / ref[c][g];              // a power of two
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            w[j] = x[c][j] * inv * step[j];
                            most = fmaxf(most, w[j]);
                        }
                        if (__builtin_amdgcn_ballot_w64(most > 0x1.0p14f) != 0) {
                            most = fmaxf(most, __shfl_xor(most, 16, 64));
                            most = fmaxf(most, __shfl_xor(most, 32, 64));
                            const int up = most > 0x1.0p14f ? ilogbf(most) - (int)kBack : 0;
                            const float f = ldexpf(1.0f, -up);
                            ref[c][g] = ldexpf(ref[c][g], up);
                            lw[c][g] *= f;
#pragma unroll
                            for (int j = 0; j < 8; ++j) w[j] *= f;
#pragma unroll
                            for (int j = 0; j < CH; ++j) o[c][g * CH + j] *= f;
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            pr[c][j] = two_halves(w[2 * j], w[2 * j + 1]);
                            lw[c][g] = add_halves(pr[c][j], lw[c][g]);
                        }
                    }
                }
                uint32_t low[4], high[4];                  // codes of tokens 2 j and 2 j + 1
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    low[j] = __builtin_amdgcn_perm(v[2 * j + 1][g], v[2 * j][g], 0x05040100u) ^ kOffset;
                    if constexpr (CH == 8) high[j] = __builtin_amdgcn_perm(v[2 * j + 1][g], v[2 * j][g], 0x07060302u) ^ kOffset;
                }
                static_for<0, CH>([&](auto J) PQ_INLINE {
                    constexpr int j = decltype(J)::value;
                    v4u w;
#pragma unroll
                    for (int n = 0; n < 4; ++n) w[n] = operand<(j & 3)>(j < 4 ? low[n] : high[n]);
#pragma unroll
                    for (int c = 0; c < CB; ++c)
                        o[c][g * CH + j] = product(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, pr[c]), o[c][g * CH + j]);
                });
            }
        }

        // ---- the four wavefronts' sums become one
        __syncthreads();                           // (they lie over the rings)
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            l[c] += __shfl_xor(l[c], 16, 64);
            l[c] += __shfl_xor(l[c], 32, 64);
            if (quarter == 0) {
                sum_m[wave * ROWS + 16 * c + col] = m[c];
                sum_l[wave * ROWS + 16 * c + col] = l[c];
            }
            const bool live = tile * ROWS + 16 * c + col < rows;
            float* const dst = sums + (wave * ROWS + 16 * c + col) * S::PITCH;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float times = kUnit, minus = 8.0f * l[c];
                if constexpr (DYNAMIC) {
                    float lw_all = lw[c][g] + __shfl_xor(lw[c][g], 16, 64);
                    lw_all += __shfl_xor(lw_all, 32, 64);
                    times = kUnit * ref[c][g];
                    minus = 8.0f * lw_all * ref[c][g];
                }
                // block j of a group holds channels CH * row + j: a lane's rows 4 quarter .. + 3 are 4 CH channels in a row
                if (live) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < CH; ++j) dst[g * G + CH * (4 * quarter + i) + j] = fmaf(o[c][g * CH + j][i], times, -minus);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            constexpr int kEach = D / 16;
            const int out_row = 16 * c + (tid >> 4), d0 = (tid & 15) * kEach, at_row = tile * ROWS + out_row;
            if (at_row < rows) {
                float top = sum_m[out_row], sum = 0.0f, acc[kEach];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sum_m[w * ROWS + out_row]);
#pragma unroll
                for (int i = 0; i < kEach; ++i) acc[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(sum_m[w * ROWS + out_row] - top);
                    sum = fmaf(sum_l[w * ROWS + out_row], f, sum);
#pragma unroll
                    for (int i = 0; i < kEach; ++i) acc[i] = fmaf(sums[(w * ROWS + out_row) * S::PITCH + d0 + i], f * v_step, acc[i]);
                }
                if (take == per) {
                    const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
                    __half* dst = a.out + ((int64_t)(r.start + at_row / per_kv) * a.n_heads + head * per_kv + at_row % per_kv) * D + d0;
#pragma unroll
                    for (int i = 0; i < kEach; i += 2) *reinterpret_cast<__half2*>(dst + i) = __floats2half2_rn(acc[i] * f, acc[i + 1] * f);
                } else {
                    const int64_t slot = (int64_t)worker * 2 + (u0 == range ? 0 : 1);
                    float* dst = partial + (slot * ROWS + out_row) * (D + 4);
#pragma unroll
                    for (int i = 0; i < kEach; ++i) dst[4 + d0 + i] = acc[i];
                    if (d0 == 0) {
                        dst[0] = top;
                        dst[1] = sum;
                    }
                }
            }
        }
        __syncthreads();
        u0 += take;
    }
}

// Adds the partial sums of the histories that were cut: a workgroup takes the one that the border before its worker's run is the first to cut.
template <int D, int CB>
__global__ __launch_bounds__(kThreads) void k_kv4_attention_join(AttentionArgs a, const float* __restrict__ partial, int workers, int small_rows)
{
    constexpr int ROWS = 16 * CB, kEach = D / 16;
    const int tid = threadIdx.x, lane = tid & 63;
    const Plan p = plan<ROWS>(a, small_rows, lane);
    const int64_t total = p.total;
    const int active = (int)min((int64_t)workers, total), worker = blockIdx.x + 1;
    if (worker >= active) return;
    auto start_of = [&](int w) { return total * w / active; };
    const int64_t border = start_of(worker);
    int64_t base;
    const int b = find_request<ROWS>(a, p, small_rows, border, base);
    const Request r = request(a, b);
    int tiles;
    units_of<ROWS>(a, r, small_rows, tiles);
    const int64_t per = units_of_tile(r), item = (border - base) / per, first = base + item * per, last = first + per;
    if (first == border || first < start_of(worker - 1)) return;       // not cut here, or by an earlier border as well
    const int head = (int)(item / tiles), tile = (int)(item % tiles), rows = r.q_len * a.heads_per_kv;
#pragma unroll
    for (int c = 0; c < CB; ++c) {
        const int row = 16 * c + (tid >> 4), d0 = (tid & 15) * kEach, at_row = tile * ROWS + row;
        if (at_row >= rows) continue;
        float top = kNothing, sum = 0.0f, acc[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) acc[i] = 0.0f;
        for (int w = worker - 1; w < active && start_of(w) < last; ++w) {
            const int64_t slot = (int64_t)w * 2 + (start_of(w) >= first ? 0 : 1);
            const float* src = partial + (slot * ROWS + row) * (D + 4);
            const float m = src[0], to = fmaxf(top, m);
            const float f = __builtin_amdgcn_exp2f(top - to), g = __builtin_amdgcn_exp2f(m - to);
            sum = fmaf(sum, f, src[1] * g);
#pragma unroll
            for (int i = 0; i < kEach; ++i) acc[i] = fmaf(acc[i], f, src[4 + d0 + i] * g);
            top = to;
        }
        const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
        __half* dst = a.out + ((int64_t)(r.start + at_row / a.heads_per_kv) * a.n_heads + head * a.heads_per_kv + at_row % a.heads_per_kv) * D + d0;
#pragma unroll
        for (int i = 0; i < kEach; i += 2) *reinterpret_cast<__half2*>(dst + i) = __floats2half2_rn(acc[i] * f, acc[i + 1] * f);
    }
}

template <int D, int G, bool DYNAMIC, int CB>
int launch(const AttentionArgs& a, int workers, int small_rows, float* partial, hipStream_t st)
{
    static std::atomic<uint64_t> allowed{0};
    constexpr size_t lds = Shape<D, G, DYNAMIC, CB>::kLds;
    const auto kernel = k_kv4_attention_rows<D, G, DYNAMIC, CB>;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, allowed); rc != PQ_OK) return rc;
    kernel<<<workers, kThreads, lds, st>>>(a, partial, workers, small_rows);
    if (workers > 1) k_kv4_attention_join<D, CB><<<workers - 1, kThreads, 0, st>>>(a, partial, workers, small_rows);
    return hip_status(hipGetLastError());
}

// As many as the call can have units at most (tiles of 16 rows), up to the GPU's places.
int workers_for(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int64_t capacity)
{
    const int64_t tiles = T * (n_heads / n_kv_heads) / 16 + B, units = tiles * n_kv_heads * ((capacity + kUnitTokens - 1) / kUnitTokens);
    return (int)(units < kWorkers ? units : kWorkers);
}

// Column blocks: one, if it holds every request's rows (max_q is right, or more tiles of rows are taken).
int blocks_for(int32_t max_q, int32_t per_kv) { return (int64_t)max_q * per_kv <= 16 ? 1 : 2; }

size_t rows_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, int64_t capacity)
{
    const size_t rows = (size_t)workers_for(T, B, n_heads, n_kv_heads, capacity) * 2 * 16 * blocks_for(max_q, n_heads / n_kv_heads);
    return (rows * (head_dim + 4) * sizeof(float) + 255) & ~(size_t)255;
}

template <int CB>
int launch_rows(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, float* partial, hipStream_t st)
{
    const int workers = workers_for(a.T, a.B, a.n_heads, a.cache.n_kv_heads, (int64_t)a.table_pages << a.cache.log2_page);
    if (head_dim == 64) {
        if (group == 0) return launch<64, 64, false, CB>(a, workers, small_rows, partial, st);
        if (group == 32) return launch<64, 32, true, CB>(a, workers, small_rows, partial, st);
        return launch<64, 64, true, CB>(a, workers, small_rows, partial, st);
    }
    if (group == 0) return launch<128, 128, false, CB>(a, workers, small_rows, partial, st);
    if (group == 32) return launch<128, 32, true, CB>(a, workers, small_rows, partial, st);
    if (group == 64) return launch<128, 64, true, CB>(a, workers, small_rows, partial, st);
    return launch<128, 128, true, CB>(a, workers, small_rows, partial, st);
}

// Requests of up to this many rows take the row kernel where the call may hold larger ones.
constexpr int kSmallRows = 64;

bool takes_tiles(int32_t max_q, int32_t per_kv) { return (int64_t)max_q * per_kv > kSmallRows; }

}  // namespace

size_t attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, int64_t capacity)
{
    const size_t rows = rows_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, max_q, capacity);
    return rows + (takes_tiles(max_q, n_heads / n_kv_heads) ? tiles_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, capacity) : 0);
}

int launch_attention(const AttentionArgs& a, int32_t head_dim, int32_t group, int32_t max_q, void* ws, hipStream_t st)
{
    float* const partial = static_cast<float*>(ws);
    const bool tiles = takes_tiles(max_q, a.heads_per_kv);
    const int small_rows = tiles ? kSmallRows : INT32_MAX;
    if (tiles) {
        const size_t rows = rows_workspace_bytes(a.T, a.B, a.n_heads, a.cache.n_kv_heads, head_dim, max_q, (int64_t)a.table_pages << a.cache.log2_page);
        if (const int rc = launch_attention_tiles(a, head_dim, group, small_rows, partial + rows / sizeof(float), st); rc != PQ_OK) return rc;
    }
    return blocks_for(max_q, a.heads_per_kv) == 1 ? launch_rows<1>(a, head_dim, group, small_rows, partial, st)
                                                  : launch_rows<2>(a, head_dim, group, small_rows, partial, st);
}

}  // namespace kv4
}  // namespace pq
