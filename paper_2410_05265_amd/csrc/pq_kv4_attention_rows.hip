// Attention over the paged 4-bit cache for few queries of a request: decoded tokens, and some drafted ones.
//
// The queries of a request that share a key/value head (its tokens times the heads of the group) are the 16 columns of the matrix
// instructions; up to 16 of them read every code once.  Bound by HBM: 128 bytes of codes for a token and head of 128 channels.
//
// Work is cut over the histories, in units of kUnitTokens tokens of one request, head and tile of 16 rows.  All units of the call lie one after
// another, and every workgroup takes an equal run of them, whatever the requests' lengths are: a run that covers a history whole writes
// its outputs, one that begins or ends inside a history leaves a partial sum (at most two to a workgroup), and a second small kernel
// adds those, in the order of the workgroups.  The lengths are read on the device, so a captured call follows them.
//
// A wavefront takes 32 tokens at a time: codes of the tile after next are on their way while one is multiplied.  A lane reads 16 bytes of a
// token's key codes (its part of every step of the first product), and 4 bytes of each of eight tokens' value codes: an 8 x 8 block, whose
// transposition is a byte permutation of two tokens.
#include "pq_kv4_attention.h"

namespace pq {
namespace kv4 {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRows = 16;
constexpr int kTile = 32;                          // tokens of a wavefront's step
constexpr int kUnitTokens = kTile * kWaves;
constexpr int kWorkers = 1024;                     // four workgroups to a CU
constexpr float kLeast = 0x1.0p-80f;               // smallest reference of value weights (dynamic steps)

__device__ __forceinline__ int64_t units_of_tile(const Request& r) { return r.n > 0 ? (r.n + kUnitTokens - 1) / kUnitTokens : 1; }

// Units of a request: (heads x tiles of rows) x units of its history; none if it has more than small_rows rows.
__device__ __forceinline__ int64_t units_of(const AttentionArgs& a, const Request& r, int small_rows, int& tiles)
{
    const int64_t rows = (int64_t)r.q_len * a.heads_per_kv;
    tiles = rows > small_rows ? 0 : (int)((rows + kRows - 1) / kRows);
    return units_of_tile(r) * tiles * a.cache.n_kv_heads;
}

// The requests' units: each lane of the calling wavefront sums a run of requests.
struct Plan {
    int64_t total, before;      // all units; those before this lane's requests
    int64_t own;
    int first, last;            // this lane's requests
};

__device__ __forceinline__ Plan plan(const AttentionArgs& a, int small_rows, int lane)
{
    Plan p;
    const int each = (a.B + 63) / 64;
    p.first = min(lane * each, a.B);
    p.last = min(p.first + each, a.B);
    p.own = 0;
    for (int b = p.first; b < p.last; ++b) {
        int tiles;
        p.own += units_of(a, request(a, b), small_rows, tiles);
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

struct Shared {
    float o[kWaves][kRows][128];
    float m[kWaves][kRows], l[kWaves][kRows];
};

template <int D, int G, bool DYNAMIC>
struct Codes {
    static constexpr int NG = D / G, KS = G / 32;
    uint32_t k[2][NG * KS];
    uint32_t v[8][NG];
    float ks[DYNAMIC ? 2 : 1][DYNAMIC ? 4 * NG : 1], vs[DYNAMIC ? 2 : 1][DYNAMIC ? 4 * NG : 1];
    bool bad[2];                                   // a block of 16 tokens whose page is none
};

template <int D, int G, bool DYNAMIC>
__global__ __launch_bounds__(kThreads, DYNAMIC ? 2 : 3) void k_kv4_attention_rows(AttentionArgs a, float* partial, int workers, int small_rows)
{
    constexpr int NG = D / G, KS = G / 32, CH = G / 16;
    typedef Codes<D, G, DYNAMIC> C;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int log2_page = a.cache.log2_page, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv;

    const Plan p = plan(a, small_rows, lane);
    const int64_t total = p.total;
    const int active = (int)min((int64_t)workers, total);
    const int worker = xcd_run(blockIdx.x, gridDim.x);
    if (worker >= active) return;
    const int64_t range = total * worker / active, range_end = total * (worker + 1) / active;

    int b;
    int64_t base;                                  // first unit of request b
    {
        const bool mine = p.before <= range && range < p.before + p.own;
        int at = p.first;
        int64_t u = p.before;
        if (mine) {
            for (; at < p.last; ++at) {
                int tiles;
                const int64_t n = units_of(a, request(a, at), small_rows, tiles);
                if (range < u + n) break;
                u += n;
            }
        }
        const int from = __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine));
        b = __builtin_amdgcn_readfirstlane(__shfl(at, from, 64));
        base = __shfl(u, from, 64);
    }

    for (int64_t u0 = range; u0 < range_end;) {
        int tiles;
        const Request r = request(a, b);
        const int64_t whole = units_of(a, r, small_rows, tiles), per = units_of_tile(r);
        if (u0 >= base + whole) {                  // (requests without queries, or with many, have no units)
            base += whole;
            ++b;
            continue;
        }
        const int64_t item = (u0 - base) / per, from_unit = (u0 - base) % per, take = min(range_end - u0, per - from_unit);
        const int head = __builtin_amdgcn_readfirstlane((int)(item / tiles)), tile = __builtin_amdgcn_readfirstlane((int)(item % tiles));
        const int rows = r.q_len * per_kv;
        const int row = tile * kRows + col;
        const bool live = row < rows;
        const int token = live ? row / per_kv : r.q_len - 1, q_head = head * per_kv + (live ? row % per_kv : 0);
        const int back = r.q_len - 1 - token;      // queries of the request behind this one
        const int limit = a.causal ? max(r.n - back, 0) : r.n;
        const int first_token = tile * kRows / per_kv, last_token = min((tile * kRows + kRows - 1) / per_kv, r.q_len - 1);
        const int all_see = a.causal ? r.n - (r.q_len - 1 - first_token) : r.n;         // tokens before this one need no mask
        const int any_sees = a.causal ? r.n - (r.q_len - 1 - last_token) : r.n;
        const int from = (int)(from_unit * kUnitTokens), to = (int)min((from_unit + take) * kUnitTokens, (int64_t)max(any_sees, 0));

        // queries: channels as the keys' operands have them
        v8h q[NG * KS];
        {
            const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    q[g * KS + s] = in_key_order(*reinterpret_cast<const v4u*>(src + g * G + quarter * (G / 4) + 8 * s));
        }
        v4f c0[NG];
        {
            const v4u minus8 = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                c0[g] = (v4f){0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    c0[g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, minus8), q[g * KS + s], c0[g], 0, 0, 0);
            }
        }
        const float scale = a.softmax_scale * 1.44269504088896341f;
        float c1 = scale * kUnit, v_step = 1.0f;
        if constexpr (!DYNAMIC) {
            c1 *= a.cache.k_scale[head];
            v_step = a.cache.v_scale[head];
        }

        float m = kNothing, l = 0.0f;              // l: this lane's tokens
        v4f o[NG * CH];
        float ref[NG], lw[NG];                     // dynamic steps: weights p * step are rounded relative to ref
#pragma unroll
        for (int i = 0; i < NG * CH; ++i) o[i] = (v4f){0, 0, 0, 0};
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            ref[g] = kLeast;
            lw[g] = 0.0f;
        }

        // Scores x (times c, without the reference) to probabilities relative to m; rescales what is there if m moves.
        auto probabilities = [&](float (&x)[2][4]) {
            float most = x[0][0];
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, x[i >> 2][i & 3]);
            if (__builtin_amdgcn_ballot_w64(most > m + kMost) != 0) {
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float to_m = most > m + kMost ? ceilf(most) - kBack : m;
                const float alpha = __builtin_amdgcn_exp2f(m - to_m);
                m = to_m;
                l *= alpha;
                if constexpr (DYNAMIC) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const float at = ref[g] * alpha, f = at >= kLeast ? 1.0f : at * (1.0f / kLeast);
                        ref[g] = fmaxf(at, kLeast);
                        lw[g] *= f;
#pragma unroll
                        for (int i = 0; i < CH; ++i) o[g * CH + i] *= f;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NG * CH; ++i) o[i] *= alpha;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = __builtin_amdgcn_exp2f(x[i >> 2][i & 3] - m);
        };

        // prefix tokens, by the first wavefront of the run that begins the history
        if (a.n_prefix > 0 && from_unit == 0 && wave == 0) {
            for (int t0 = 0; t0 < a.n_prefix; t0 += kTile) {
                float x[2][4];
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    const int t = min(t0 + 16 * blk + col, a.n_prefix - 1);
                    const __half* src = a.prefix_k + ((int64_t)t * Hkv + head) * D;
                    v4f s4 = {0, 0, 0, 0};
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int s = 0; s < KS; ++s)
                            s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                                in_key_order(*reinterpret_cast<const v4u*>(src + g * G + quarter * (G / 4) + 8 * s)), q[g * KS + s], s4, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[blk][i] = t0 + 16 * blk + 4 * quarter + i < a.n_prefix ? s4[i] * scale : -INFINITY;
                }
                probabilities(x);
                v4u pr;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    pr[i] = two_halves(x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1]);
                    l = add_halves(pr[i], l);
                }
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int j = 0; j < CH; ++j) {
                        v8h w;
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int t = min(t0 + 16 * (k >> 2) + 4 * quarter + (k & 3), a.n_prefix - 1);
                            w[k] = *reinterpret_cast<const _Float16*>(a.prefix_v + ((int64_t)t * Hkv + head) * D + g * G + CH * col + j);
                        }
                        o[g * CH + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w, __builtin_bit_cast(v8h, pr), o[g * CH + j], 0, 0, 0);
                    }
            }
            // as if they were codes: sum p v = step (unit acc - 8 sum p) has to hold
            float l_all = l + __shfl_xor(l, 16, 64);
            l_all += __shfl_xor(l_all, 32, 64);
            const float times = DYNAMIC ? 1.0f / (kUnit * kLeast) : 1.0f / (kUnit * v_step), plus = DYNAMIC ? 0.0f : 8.0f / kUnit * l_all;
#pragma unroll
            for (int i = 0; i < NG * CH; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[i][k] = fmaf(o[i][k], times, plus);
            if constexpr (DYNAMIC) {
#pragma unroll
                for (int g = 0; g < NG; ++g) ref[g] = kLeast;
            }
        }

        // ---- the history
        const int32_t* table = a.table + (int64_t)b * a.table_pages;
        int ids_from = -64, ids = 0;
        auto load = [&](int t0, C& c) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const int t = t0 + 16 * blk, page_at = t >> log2_page;
                if (page_at >= ids_from + 64) {
                    ids_from = page_at;
                    ids = table[min(page_at + lane, a.table_pages - 1)];
                }
                int page = __builtin_amdgcn_readlane(ids, page_at - ids_from);
                c.bad[blk] = (uint32_t)page >= (uint64_t)a.cache.n_pages || page_at >= a.table_pages;
                page = c.bad[blk] ? 0 : page;
                const int64_t first = (((int64_t)page * Hkv + head) << log2_page) + (t & ((1 << log2_page) - 1));
                const uint8_t* kc = a.cache.k_codes + first * (D / 2);
                const uint8_t* vc = a.cache.v_codes + first * (D / 2);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const uint8_t* src = kc + col * (D / 2) + g * (G / 2) + quarter * (G / 8);
                    if constexpr (KS == 4) {
                        const v4u w = *reinterpret_cast<const v4u*>(src);
#pragma unroll
                        for (int s = 0; s < 4; ++s) c.k[blk][g * KS + s] = w[s];
                    } else if constexpr (KS == 2) {
                        const v2u w = *reinterpret_cast<const v2u*>(src);
                        c.k[blk][g * KS] = w[0];
                        c.k[blk][g * KS + 1] = w[1];
                    } else {
                        c.k[blk][g] = *reinterpret_cast<const uint32_t*>(src);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint8_t* vs = vc + (4 * quarter + i) * (D / 2) + g * (G / 2) + col * (G / 32);
                        if constexpr (KS == 4) c.v[4 * blk + i][g] = *reinterpret_cast<const uint32_t*>(vs);
                        else if constexpr (KS == 2) c.v[4 * blk + i][g] = *reinterpret_cast<const uint16_t*>(vs);
                        else c.v[4 * blk + i][g] = *vs;
                    }
                }
                if constexpr (DYNAMIC) {
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        const v4f x = *reinterpret_cast<const v4f*>(a.cache.k_scale + (first + 4 * quarter) * NG + 4 * i);
                        const v4f y = *reinterpret_cast<const v4f*>(a.cache.v_scale + (first + 4 * quarter) * NG + 4 * i);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            c.ks[blk][4 * i + k] = x[k];
                            c.vs[blk][4 * i + k] = y[k];
                        }
                    }
                }
            }
        };
        auto multiply = [&](int t0, const C& c) {
            float x[2][4];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                v4f s4[NG];
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    s4[g] = c0[g];
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        s4[g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_operand(c.k[blk][g * KS + s]), q[g * KS + s], s4[g], 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (DYNAMIC) {
                        float sum = 0.0f;
#pragma unroll
                        for (int g = 0; g < NG; ++g) sum = fmaf(s4[g][i], c.ks[blk][i * NG + g], sum);
                        x[blk][i] = sum * c1;
                    } else {
                        x[blk][i] = s4[0][i] * c1;
                    }
                }
            }
            const bool masked = t0 + kTile > all_see || c.bad[0] || c.bad[1];
            if (masked) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t0 + 16 * (i >> 2) + 4 * quarter + (i & 3) >= limit || c.bad[i >> 2]) x[i >> 2][i & 3] = -INFINITY;
            }
            probabilities(x);
            v4u pr;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pr[i] = two_halves(x[i >> 1][2 * (i & 1)], x[i >> 1][2 * (i & 1) + 1]);
                l = add_halves(pr[i], l);
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                if constexpr (DYNAMIC) {
                    float w[8], most = 0.0f;
                    const float inv = 1.0f / ref[g];       // a power of two
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float step = c.vs[i >> 2][(i & 3) * NG + g];
                        if (masked && (t0 + 16 * (i >> 2) + 4 * quarter + (i & 3) >= r.n || c.bad[i >> 2])) step = 0.0f;
                        w[i] = x[i >> 2][i & 3] * inv * step;
                        most = fmaxf(most, w[i]);
                    }
                    if (__builtin_amdgcn_ballot_w64(most > 0x1.0p14f) != 0) {
                        most = fmaxf(most, __shfl_xor(most, 16, 64));
                        most = fmaxf(most, __shfl_xor(most, 32, 64));
                        const int up = most > 0x1.0p14f ? ilogbf(most) - (int)kBack : 0;
                        const float f = ldexpf(1.0f, -up);
                        ref[g] = ldexpf(ref[g], up);
                        lw[g] *= f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] *= f;
#pragma unroll
                        for (int i = 0; i < CH; ++i) o[g * CH + i] *= f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        pr[i] = two_halves(w[2 * i], w[2 * i + 1]);
                        lw[g] = add_halves(pr[i], lw[g]);
                    }
                }
                uint32_t low[4], high[4];                  // codes of tokens 2 i and 2 i + 1
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x0 = c.v[2 * i][g], x1 = c.v[2 * i + 1][g];
                    low[i] = __builtin_amdgcn_perm(x1, x0, 0x05040100u) ^ kOffset;
                    if constexpr (CH == 8) high[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302u) ^ kOffset;
                }
                static_for<0, CH>([&](auto J) {
                    constexpr int j = decltype(J)::value;
                    v4u w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = operand<(j & 3)>(j < 4 ? low[i] : high[i]);
                    o[g * CH + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, w), __builtin_bit_cast(v8h, pr), o[g * CH + j], 0, 0, 0);
                });
            }
        };
        {
            C c[2];
            int t = from + wave * kTile;
            if (t < to) load(t, c[0]);
            while (t < to) {
                if (t + kUnitTokens < to) load(t + kUnitTokens, c[1]);
                multiply(t, c[0]);
                t += kUnitTokens;
                if (t >= to) break;
                if (t + kUnitTokens < to) load(t + kUnitTokens, c[0]);
                multiply(t, c[1]);
                t += kUnitTokens;
            }
        }

        // ---- the four wavefronts' sums become one
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (lane < kRows) {
            sh.m[wave][lane] = m;
            sh.l[wave][lane] = l;
        }
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float times = kUnit, minus = 8.0f * l;
            if constexpr (DYNAMIC) {
                float lw_all = lw[g] + __shfl_xor(lw[g], 16, 64);
                lw_all += __shfl_xor(lw_all, 32, 64);
                times = kUnit * ref[g];
                minus = 8.0f * lw_all * ref[g];
            }
            // block j of a group holds channels CH * row + j: a lane's rows 4 quarter .. + 3 are 4 CH channels in a row
            if (live) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < CH; ++j)
                        sh.o[wave][col][g * G + CH * (4 * quarter + i) + j] = fmaf(o[g * CH + j][i], times, -minus);
            }
        }
        __syncthreads();
        {
            constexpr int kEach = D / 16;
            const int out_row = tid >> 4, d0 = (tid & 15) * kEach, at_row = tile * kRows + out_row;
            if (at_row < rows) {
                float top = sh.m[0][out_row], sum = 0.0f, acc[kEach];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sh.m[w][out_row]);
#pragma unroll
                for (int i = 0; i < kEach; ++i) acc[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = __builtin_amdgcn_exp2f(sh.m[w][out_row] - top);
                    sum = fmaf(sh.l[w][out_row], f, sum);
#pragma unroll
                    for (int i = 0; i < kEach; ++i) acc[i] = fmaf(sh.o[w][out_row][d0 + i], f * v_step, acc[i]);
                }
                if (take == per) {
                    const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
                    __half* dst = a.out + ((int64_t)(r.start + at_row / per_kv) * a.n_heads + head * per_kv + at_row % per_kv) * D + d0;
#pragma unroll
                    for (int i = 0; i < kEach; i += 2) *reinterpret_cast<__half2*>(dst + i) = __floats2half2_rn(acc[i] * f, acc[i + 1] * f);
                } else {
                    const int64_t slot = (int64_t)worker * 2 + (u0 == range ? 0 : 1);
                    float* dst = partial + (slot * kRows + out_row) * (D + 4);
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

// Adds the partial sums of every row whose history was cut: one wavefront to a row and head.
template <int D>
__global__ __launch_bounds__(kThreads) void k_kv4_attention_join(AttentionArgs a, const float* __restrict__ partial, int workers, int small_rows)
{
    const int lane = threadIdx.x & 63;
    const int64_t index = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (index >= a.T * a.n_heads) return;
    const int64_t at = index / a.n_heads;
    const int q_head = (int)(index % a.n_heads), head = q_head / a.heads_per_kv;
    const Plan p = plan(a, small_rows, lane);
    // the request that this row belongs to
    int b = -1;
    int64_t base = 0, u = p.before;
    for (int i = p.first; i < p.last; ++i) {
        int tiles;
        const Request r = request(a, i);
        if (b < 0 && at >= r.start && at < (int64_t)r.start + r.q_len) {
            b = i;
            base = u;
        }
        u += units_of(a, r, small_rows, tiles);
    }
    const uint64_t found = __builtin_amdgcn_ballot_w64(b >= 0);
    if (found == 0) return;
    const int from = __builtin_ctzll(found);
    b = __shfl(b, from, 64);
    base = __shfl(base, from, 64);
    const Request r = request(a, b);
    int tiles;
    units_of(a, r, small_rows, tiles);
    if (tiles == 0) return;
    const int64_t per = units_of_tile(r), total = p.total;
    const int row = (int)(at - r.start) * a.heads_per_kv + q_head % a.heads_per_kv;
    const int64_t first = base + ((int64_t)head * tiles + row / kRows) * per, last = first + per - 1;
    const int active = (int)min((int64_t)workers, total);
    const int w0 = (int)(((first + 1) * active - 1) / total), w1 = (int)(((last + 1) * active - 1) / total);
    if (w0 == w1) return;                          // written by the workgroup that took it whole
    float top = kNothing, sum = 0.0f, x = 0.0f, y = 0.0f;
    for (int w = w0; w <= w1; ++w) {
        const int64_t slot = (int64_t)w * 2 + (total * w / active >= first ? 0 : 1);
        const float* src = partial + (slot * kRows + row % kRows) * (D + 4);
        const float m = src[0], l = src[1], to = fmaxf(top, m);
        const float f = __builtin_amdgcn_exp2f(top - to), g = __builtin_amdgcn_exp2f(m - to);
        sum = fmaf(sum, f, l * g);
        if constexpr (D == 128) {
            x = fmaf(x, f, src[4 + 2 * lane] * g);
            y = fmaf(y, f, src[5 + 2 * lane] * g);
        } else {
            x = fmaf(x, f, src[4 + lane] * g);
        }
        top = to;
    }
    const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
    __half* dst = a.out + (at * a.n_heads + q_head) * D;
    if constexpr (D == 128) *reinterpret_cast<__half2*>(dst + 2 * lane) = __floats2half2_rn(x * f, y * f);
    else dst[lane] = __float2half_rn(x * f);
}

template <int D, int G, bool DYNAMIC>
int launch(const AttentionArgs& a, int workers, int small_rows, float* partial, hipStream_t st)
{
    k_kv4_attention_rows<D, G, DYNAMIC><<<workers, kThreads, 0, st>>>(a, partial, workers, small_rows);
    k_kv4_attention_join<D><<<(unsigned)((a.T * a.n_heads + kWaves - 1) / kWaves), kThreads, 0, st>>>(a, partial, workers, small_rows);
    return hip_status(hipGetLastError());
}

int workers_for(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int64_t capacity)
{
    const int64_t tiles = T * (n_heads / n_kv_heads) / kRows + B, units = tiles * n_kv_heads * ((capacity + kUnitTokens - 1) / kUnitTokens);
    return (int)(units < kWorkers ? units : kWorkers);
}

size_t rows_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int64_t capacity)
{
    const size_t bytes = (size_t)workers_for(T, B, n_heads, n_kv_heads, capacity) * 2 * kRows * (head_dim + 4) * sizeof(float);
    return (bytes + 255) & ~(size_t)255;
}

int launch_rows(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, float* partial, hipStream_t st)
{
    const int workers = workers_for(a.T, a.B, a.n_heads, a.cache.n_kv_heads, (int64_t)a.table_pages << a.cache.log2_page);
    if (head_dim == 64) {
        if (group == 0) return launch<64, 64, false>(a, workers, small_rows, partial, st);
        if (group == 32) return launch<64, 32, true>(a, workers, small_rows, partial, st);
        return launch<64, 64, true>(a, workers, small_rows, partial, st);
    }
    if (group == 0) return launch<128, 128, false>(a, workers, small_rows, partial, st);
    if (group == 32) return launch<128, 32, true>(a, workers, small_rows, partial, st);
    if (group == 64) return launch<128, 64, true>(a, workers, small_rows, partial, st);
    return launch<128, 128, true>(a, workers, small_rows, partial, st);
}

// Requests of up to this many rows take the row kernel where the call may hold larger ones.
constexpr int kSmallRows = 64;

bool takes_tiles(int32_t max_q, int32_t per_kv) { return (int64_t)max_q * per_kv > kSmallRows; }

}  // namespace

size_t attention_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_q, int64_t capacity)
{
    const size_t rows = rows_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, capacity);
    return rows + (takes_tiles(max_q, n_heads / n_kv_heads) ? tiles_workspace_bytes(T, B, n_heads, n_kv_heads, head_dim, capacity) : 0);
}

int launch_attention(const AttentionArgs& a, int32_t head_dim, int32_t group, int32_t max_q, void* ws, hipStream_t st)
{
    float* const partial = static_cast<float*>(ws);
    if (!takes_tiles(max_q, a.heads_per_kv)) return launch_rows(a, head_dim, group, INT32_MAX, partial, st);
    const size_t rows = rows_workspace_bytes(a.T, a.B, a.n_heads, a.cache.n_kv_heads, head_dim, (int64_t)a.table_pages << a.cache.log2_page);
    const int rc = launch_attention_tiles(a, head_dim, group, kSmallRows, partial + rows / sizeof(float), st);
    return rc == PQ_OK ? launch_rows(a, head_dim, group, kSmallRows, partial, st) : rc;
}

}  // namespace kv4
}  // namespace pq
