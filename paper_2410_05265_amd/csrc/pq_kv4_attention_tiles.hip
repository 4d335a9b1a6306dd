// Attention over the paged 4-bit cache for many queries of a request: prompts, and chunks of them.
//
// Bound by the matrix instructions: 4 D operations for every query, head and token that it sees, the codes read once per 256 rows.  A workgroup
// takes 256 rows (a request's tokens times the query heads that share a key/value head), each wavefront 64 of them, two blocks of 32
// columns: a fragment read from LDS feeds two instructions.  One wavefront to a SIMD, so that 128 accumulators, 64 registers of queries and
// the scores of two tiles fit.  A step is a tile of 64 tokens: its codes are expanded once per workgroup, into fp16 operands in LDS (the
// expansion by every wavefront for itself would be four times the vector instructions, which are what the matrix instructions wait
// for here: exponentials, maxima and sums of 64 scores a lane).  The scores of the next tile are multiplied while the probabilities of this
// one are formed, and the codes after next are on their way.
//
// Where a call has few tiles of rows, the histories are cut into `splits` parts; their sums go through scratch memory and a second kernel.
#include "pq_kv4_attention.h"

namespace pq {
namespace kv4 {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = kTileRows, kCols = 64;      // rows of a workgroup and of a wavefront
constexpr int kTile = 64;                         // tokens of a step
constexpr float kLeast = 0x1.0p-80f;

// Which tile of rows: the index-th of all requests that this kernel takes, a request's last tile (the one that sees most) first.
struct Where {
    int b, tile;        // b < 0: there is no such tile
    Request r;
};

__device__ __forceinline__ int tiles_of(const AttentionArgs& a, const Request& r, int small_rows)
{
    const int64_t rows = (int64_t)r.q_len * a.heads_per_kv;
    return rows <= small_rows ? 0 : (int)((rows + kRows - 1) / kRows);
}

__device__ __forceinline__ Where find_tile(const AttentionArgs& a, int64_t index, int small_rows, int lane)
{
    const int each = (a.B + 63) / 64, first = min(lane * each, a.B), last = min(first + each, a.B);
    int64_t own = 0;
    for (int b = first; b < last; ++b) own += tiles_of(a, request(a, b), small_rows);
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(incl, d, 64);
        if (lane >= d) incl += v;
    }
    const bool mine = incl - own <= index && index < incl;
    const uint64_t found = __builtin_amdgcn_ballot_w64(mine);
    Where w = {-1, 0, {0, 0, 0}};
    if (found == 0) return w;
    int b = first, tile = 0;
    if (mine) {
        int64_t u = incl - own;
        for (; b < last; ++b) {
            const int n = tiles_of(a, request(a, b), small_rows);
            if (index < u + n) {
                tile = (int)(u + n - 1 - index);
                break;
            }
            u += n;
        }
    }
    const int from = __builtin_ctzll(found);
    w.b = __builtin_amdgcn_readfirstlane(__shfl(b, from, 64));
    w.tile = __builtin_amdgcn_readfirstlane(__shfl(tile, from, 64));
    w.r = request(a, w.b);
    return w;
}

// Row `at` of the accumulators as a channel: channels of a group lie so in LDS that neighbouring threads of the expansion write
// neighbouring places.
template <int G> __device__ __forceinline__ constexpr int channel_of(int at)
{
    const int g = at / G, in = at % G;
    return g * G + 8 * (in % (G / 8)) + in / (G / 8);
}

template <int D, int G, bool DYNAMIC>
struct Lds {
    static constexpr int NG = D / G;
    v4u k[2][kTile][D / 8];              // [token][eight channels], the place exchanged with bits of the token
    v2u v[2][kTile / 16][2][D][2];       // [16 tokens][half of the lanes][channel]: eight tokens in the order of the probabilities
    float ks[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1][kTile], vs[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1][kTile];
    int bad[4][4];                       // of the last tiles: blocks of 16 tokens whose page is none
};

template <int D, int G, bool DYNAMIC>
__global__ __launch_bounds__(kThreads, 1) void k_kv4_attention_tiles(AttentionArgs a, float* partial, int splits, int small_rows)
{
    constexpr int NG = D / G, KS = D / 16, KSG = G / 16, DB = D / 32, DBG = G / 32;
    extern __shared__ __align__(256) uint8_t raw_lds[];
    typedef Lds<D, G, DYNAMIC> L;
    L& sh = *reinterpret_cast<L*>(raw_lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int log2_page = a.cache.log2_page, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv;
    const int head = blockIdx.x % Hkv, split = (blockIdx.x / Hkv) % splits;
    const int64_t index = blockIdx.x / Hkv / splits;
    const Where at = find_tile(a, index, small_rows, lane);
    if (at.b < 0) return;
    const Request r = at.r;
    const int rows = r.q_len * per_kv, row0 = at.tile * kRows;
    const int last_token = min((row0 + kRows - 1) / per_kv, r.q_len - 1);
    const int visible = max(a.causal ? r.n - (r.q_len - 1 - last_token) : r.n, 0);
    const int all_tiles = (visible + kTile - 1) / kTile;
    const int begin = (int)((int64_t)all_tiles * split / splits), end = (int)((int64_t)all_tiles * (split + 1) / splits);

    // this lane's queries
    int limit[2], wave_sees = r.n;           // tokens that all of the wavefront's rows see
    v8h q[2][KS];
    float c0[2][NG];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int row = min(row0 + wave * kCols + 32 * c + col, rows - 1);
        const int token = row / per_kv, q_head = head * per_kv + row % per_kv;
        limit[c] = a.causal ? max(r.n - (r.q_len - 1 - token), 0) : r.n;
        const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[c][s] = in_key_order(*reinterpret_cast<const v4u*>(src + 16 * s + 8 * half));
    }
    if (a.causal) wave_sees = r.n - (r.q_len - 1 - min(row0 + wave * kCols, rows - 1) / per_kv);
    {
        const v4u minus8 = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v16f z = {};
#pragma unroll
                for (int s = 0; s < KSG; ++s)
                    z = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, minus8), q[c][g * KSG + s], z, 0, 0, 0);
                c0[c][g] = z[0];
            }
    }
    const float scale = a.softmax_scale * 1.44269504088896341f;
    float c1 = scale * kUnit, v_step = 1.0f;
    if constexpr (!DYNAMIC) {
        c1 *= a.cache.k_scale[head];
        v_step = a.cache.v_scale[head];
    }

    float m[2] = {kNothing, kNothing}, l[2] = {0.0f, 0.0f};
    float ref[2][NG], lw[2][NG];
    v16f o[2][DB];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int i = 0; i < DB; ++i) o[c][i] = (v16f){};
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            ref[c][g] = kLeast;
            lw[c][g] = 0.0f;
        }
    }

    // The reference follows the largest score of a column block (times c, both halves of the lanes); what is there is rescaled.
    auto follow = [&](int c, float most) {
        if (__builtin_amdgcn_ballot_w64(most > m[c] + kMost) == 0) return;
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        const float to_m = most > m[c] + kMost ? ceilf(most) - kBack : m[c];
        const float alpha = __builtin_amdgcn_exp2f(m[c] - to_m);
        m[c] = to_m;
        l[c] *= alpha;
        if constexpr (DYNAMIC) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float x = ref[c][g] * alpha, f = x >= kLeast ? 1.0f : x * (1.0f / kLeast);
                ref[c][g] = fmaxf(x, kLeast);
                lw[c][g] *= f;
#pragma unroll
                for (int i = 0; i < DBG; ++i) o[c][g * DBG + i] *= f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < DB; ++i) o[c][i] *= alpha;
        }
    };

    // ---- the history: wavefront w loads and expands tokens 16 w .. 16 w + 15 of every tile
    const int32_t* table = a.table + (int64_t)at.b * a.table_pages;
    auto page_of = [&](int tile) { return table[min((tile * kTile + 16 * wave) >> log2_page, a.table_pages - 1)]; };
    auto is_bad = [&](int tile, int page) {
        return (uint32_t)page >= (uint64_t)a.cache.n_pages || ((tile * kTile + 16 * wave) >> log2_page) >= a.table_pages;
    };
    auto first_token = [&](int tile, int page) {   // of this wavefront's block, in this head's part of the cache
        const int64_t from = is_bad(tile, page) ? 0 : page;
        return ((from * Hkv + head) << log2_page) + ((tile * kTile + 16 * wave) & ((1 << log2_page) - 1));
    };
    struct KeyCodes { uint32_t w[D / 32]; float s[DYNAMIC ? NG : 1]; int bad; };
    struct ValueCodes { uint32_t w[4]; float s[DYNAMIC ? NG : 1]; };
    auto load_keys = [&](int tile, int page, KeyCodes& x) {
        const int64_t first = first_token(tile, page);
        const uint8_t* src = a.cache.k_codes + (first + (lane >> 2)) * (D / 2) + (lane & 3) * (D / 8);
        if constexpr (D == 128) {
            const v4u w = *reinterpret_cast<const v4u*>(src);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.w[i] = w[i];
        } else {
            const v2u w = *reinterpret_cast<const v2u*>(src);
            x.w[0] = w[0];
            x.w[1] = w[1];
        }
        if constexpr (DYNAMIC) {                   // lane: token lane / 4, group lane % 4
            if ((lane & 3) < NG) x.s[0] = a.cache.k_scale[(first + (lane >> 2)) * NG + (lane & 3)];
        }
        x.bad = is_bad(tile, page);
    };
    // (four tokens x eight channels to a lane; heads of 64 channels: four channels)
    auto load_values = [&](int tile, int page, ValueCodes& x) {
        const int64_t first = first_token(tile, page);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint8_t* src = a.cache.v_codes + (first + 4 * (lane >> 4) + i) * (D / 2) + (lane & 15) * (D / 32);
            if constexpr (D == 128) x.w[i] = *reinterpret_cast<const uint32_t*>(src);
            else x.w[i] = *reinterpret_cast<const uint16_t*>(src);
        }
        if constexpr (DYNAMIC) {
            if ((lane & 3) < NG) x.s[0] = a.cache.v_scale[(first + (lane >> 2)) * NG + (lane & 3)];
        }
    };
    auto expand_keys = [&](int tile, const KeyCodes& x) {
        const int t = 16 * wave + (lane >> 2), buf = tile & 1;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            sh.k[buf][t][((lane & 3) * (D / 32) + i) ^ (t & 7)] = __builtin_bit_cast(v4u, key_operand(x.w[i]));
        if constexpr (DYNAMIC) {
            if ((lane & 3) < NG) sh.ks[buf][lane & 3][t] = x.s[0];
        }
        if (lane == 0) sh.bad[tile & 3][wave] = x.bad;
    };
    auto expand_values = [&](int tile, const ValueCodes& x) {
        // four tokens: 8 (quad / 2) + 4 (quad % 2) of the block; the lanes' half quad % 2, the first or second four of its eight
        const int quad = lane >> 4, c = lane & 15, buf = tile & 1;
        constexpr int C = D / 16;
        const uint32_t low[2] = {__builtin_amdgcn_perm(x.w[1], x.w[0], 0x05040100u) ^ kOffset, __builtin_amdgcn_perm(x.w[3], x.w[2], 0x05040100u) ^ kOffset};
        const uint32_t high[2] = {__builtin_amdgcn_perm(x.w[1], x.w[0], 0x07060302u) ^ kOffset, __builtin_amdgcn_perm(x.w[3], x.w[2], 0x07060302u) ^ kOffset};
        static_for<0, C>([&](auto J) {
            constexpr int j = decltype(J)::value;
            const uint32_t* const w = j < 4 ? low : high;
            const v2u y = {operand<(j & 3)>(w[0]), operand<(j & 3)>(w[1])};
            // channel C c + j, at the place that channel_of gives back
            const int ch = C * c + j, g = ch / G, in = ch % G, place = g * G + (in % 8) * (G / 8) + in / 8;
            sh.v[buf][wave][quad & 1][place][quad >> 1] = y;
        });
        if constexpr (DYNAMIC) {
            // what lies behind the last token may be anything: it must not meet a probability of zero
            if ((lane & 3) < NG) sh.vs[buf][lane & 3][16 * wave + (lane >> 2)] = tile * kTile + 16 * wave + (lane >> 2) < r.n ? x.s[0] : 0.0f;
        }
    };

    auto scores = [&](int buf, v16f (&s)[2][2]) {      // [32 tokens][columns]
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            if constexpr (DYNAMIC) {
                s[tb][0] = (v16f){};
                s[tb][1] = (v16f){};
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                v16f z[2] = {{}, {}};
#pragma unroll
                for (int k = g * KSG; k < (g + 1) * KSG; ++k) {
                    const int t = 32 * tb + col;
                    const v8h w = __builtin_bit_cast(v8h, sh.k[buf][t][(2 * k + half) ^ (t & 7)]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) z[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w, q[c][k], z[c], 0, 0, 0);
                }
                if constexpr (DYNAMIC) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const v4f step = *reinterpret_cast<const v4f*>(&sh.ks[buf][g][32 * tb + 8 * i + 4 * half]);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int c = 0; c < 2; ++c) s[tb][c][4 * i + j] = fmaf(z[c][4 * i + j] + c0[c][g], step[j], s[tb][c][4 * i + j]);
                    }
                } else {
                    s[tb][0] = z[0];
                    s[tb][1] = z[1];
                }
            }
        }
    };

    // exp2(c1 score + bias - m), rounded, and their sum
    auto probabilities = [&](v16f (&s)[2][2], float c1, const float (&bias)[2], v4u (&p)[2][4]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float most = -INFINITY;
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, s[tb][c][i]);
            follow(c, fmaf(most, c1, bias[c]));
            const float minus = bias[c] - m[c];
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    s[tb][c][i] = __builtin_amdgcn_exp2f(fmaf(s[tb][c][i], c1, minus));
                    s[tb][c][i + 1] = __builtin_amdgcn_exp2f(fmaf(s[tb][c][i + 1], c1, minus));
                    const uint32_t two = two_halves(s[tb][c][i], s[tb][c][i + 1]);
                    p[c][2 * tb + (i >> 3)][(i & 7) >> 1] = two;
                    l[c] = add_halves(two, l[c]);
                }
        }
    };
    auto mask = [&](int tile, v16f (&s)[2][2]) {
        const int* bad = sh.bad[tile & 3];
        const int b0 = __builtin_amdgcn_readfirstlane(bad[0]), b1 = __builtin_amdgcn_readfirstlane(bad[1]), b2 = __builtin_amdgcn_readfirstlane(bad[2]),
                  b3 = __builtin_amdgcn_readfirstlane(bad[3]);
        if (tile * kTile + kTile <= wave_sees && !(b0 | b1 | b2 | b3)) return;
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int none = tb == 0 ? (i < 8 ? b0 : b1) : (i < 8 ? b2 : b3);
                    if (tile * kTile + 32 * tb + 8 * (i >> 2) + 4 * half + (i & 3) >= limit[c] || none) s[tb][c][i] = -INFINITY;
                }
    };
    // dynamic steps: the weights p * step of one group, rounded relative to ref
    auto weights = [&](int buf, int g, const v16f (&s)[2][2], v4u (&p)[2][4]) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float inv = 1.0f / ref[c][g];
            float w[2][16], most = 0.0f;
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const v4f step = *reinterpret_cast<const v4f*>(&sh.vs[buf][g][32 * tb + 8 * i + 4 * half]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // (a token that is not seen weighs nothing, whatever its step is)
                        w[tb][4 * i + j] = s[tb][c][4 * i + j] > 0.0f ? s[tb][c][4 * i + j] * inv * step[j] : 0.0f;
                        most = fmaxf(most, w[tb][4 * i + j]);
                    }
                }
            if (__builtin_amdgcn_ballot_w64(most > 0x1.0p14f) != 0) {
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const int up = most > 0x1.0p14f ? ilogbf(most) - (int)kBack : 0;
                const float f = ldexpf(1.0f, -up);
                ref[c][g] = ldexpf(ref[c][g], up);
                lw[c][g] *= f;
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i >> 4][i & 15] *= f;
#pragma unroll
                for (int i = 0; i < DBG; ++i) o[c][g * DBG + i] *= f;
            }
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                const uint32_t two = two_halves(w[i >> 4][i & 15], w[i >> 4][(i & 15) + 1]);
                p[c][i >> 3][(i & 7) >> 1] = two;
                lw[c][g] = add_halves(two, lw[c][g]);
            }
        }
    };
    auto multiply = [&](int buf, int first, int count, const v4u (&p)[2][4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int d = first; d < first + count; ++d) {
                const v8h w = *reinterpret_cast<const v8h*>(&sh.v[buf][k][half][32 * d + col][0]);
#pragma unroll
                for (int c = 0; c < 2; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w, __builtin_bit_cast(v8h, p[c][k]), o[c][d], 0, 0, 0);
            }
    };

    // ---- prefix tokens: as a tile of their own, in fp16
    if (a.n_prefix > 0 && split == 0) {
        float keep[2][NG];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                keep[c][g] = c0[c][g];
                c0[c][g] = 0.0f;
            }
        for (int t0 = 0; t0 < a.n_prefix; t0 += kTile) {
            __syncthreads();
            for (int i = tid; i < kTile * (D / 8); i += kThreads) {
                const int t = i / (D / 8), c = i % (D / 8);
                const int64_t at = ((int64_t)min(t0 + t, a.n_prefix - 1) * Hkv + head) * D + 8 * c;
                sh.k[0][t][c ^ (t & 7)] = __builtin_bit_cast(v4u, in_key_order(*reinterpret_cast<const v4u*>(a.prefix_k + at)));
                const v4u x = *reinterpret_cast<const v4u*>(a.prefix_v + at);
                // token t of its 16: 8 (t / 8) + 4 (half of the lanes) + t % 4
                const int in16 = t & 15;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int ch = 8 * c + j, place = ch / G * G + (ch % G % 8) * (G / 8) + ch % G / 8;
                    __half* dst = reinterpret_cast<__half*>(&sh.v[0][t >> 4][(in16 >> 2) & 1][place][in16 >> 3]);
                    dst[in16 & 3] = reinterpret_cast<const __half*>(&x)[j];
                }
            }
            if constexpr (DYNAMIC) {
                if (tid < kTile) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) sh.ks[0][g][tid] = 1.0f;
                }
            }
            __syncthreads();
            v16f s[2][2];
            v4u p[2][4];
            scores(0, s);
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (t0 + 32 * tb + 8 * (i >> 2) + 4 * half + (i & 3) >= a.n_prefix) s[tb][c][i] = -INFINITY;
            const float none[2] = {0.0f, 0.0f};
            probabilities(s, scale, none, p);
            multiply(0, 0, DB, p);
        }
        __syncthreads();
        // as if they were codes: sum p v = step (unit acc - 8 sum p) has to hold
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float l_all = l[c] + __shfl_xor(l[c], 32, 64);
            const float times = DYNAMIC ? 1.0f / (kUnit * kLeast) : 1.0f / (kUnit * v_step), plus = DYNAMIC ? 0.0f : 8.0f / kUnit * l_all;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[c][d][i] = fmaf(o[c][d][i], times, plus);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                ref[c][g] = kLeast;
                c0[c][g] = keep[c][g];
            }
        }
    }

    if (begin < end) {
        KeyCodes kx;
        ValueCodes vx;
        int page1, page2;                          // of the tile whose values, and of that whose keys are loaded next
        const float bias[2] = {DYNAMIC ? 0.0f : c0[0][0] * c1, DYNAMIC ? 0.0f : c0[1][0] * c1};
        {
            const int page = page_of(begin);
            page1 = page_of(begin + 1);
            load_keys(begin, page, kx);
            load_values(begin, page, vx);
            page2 = page_of(begin + 2);
            expand_keys(begin, kx);
            load_keys(begin + 1, page1, kx);
        }
        // Keys of tile i + 1 and values of tile i are in LDS behind the barrier; keys of i + 2 and values of i + 1 in registers.
        if constexpr (DYNAMIC) {
            expand_values(begin, vx);
            load_values(begin + 1, page1, vx);
            for (int i = begin; i < end; ++i) {
                __syncthreads();
                v16f s[2][2];
                v4u p[2][4];
                const int page3 = page_of(i + 3);
                scores(i & 1, s);
                expand_keys(i + 1, kx);
                load_keys(i + 2, page2, kx);
                mask(i, s);
                probabilities(s, c1, bias, p);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    weights(i & 1, g, s, p);
                    multiply(i & 1, g * DBG, DBG, p);
                }
                expand_values(i + 1, vx);
                load_values(i + 2, page2, vx);
                page2 = page3;
            }
        } else {
            v16f s[2][2];
            __syncthreads();
            scores(begin & 1, s);
            expand_keys(begin + 1, kx);
            load_keys(begin + 2, page2, kx);
            expand_values(begin, vx);
            load_values(begin + 1, page1, vx);
            for (int i = begin; i < end; ++i) {
                __syncthreads();
                v16f next[2][2];
                v4u p[2][4];
                const int page3 = page_of(i + 3);
                mask(i, s);
                scores((i + 1) & 1, next);         // (behind the last tile: of whatever lies there, and not used)
                probabilities(s, c1, bias, p);
                multiply(i & 1, 0, DB, p);
                expand_keys(i + 2, kx);
                load_keys(i + 3, page3, kx);
                expand_values(i + 1, vx);
                load_values(i + 2, page2, vx);
                page2 = page3;
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c >> 1][c & 1] = next[c >> 1][c & 1];
            }
        }
    }

    // ---- results
    float l_all[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) l_all[c] = l[c] + __shfl_xor(l[c], 32, 64);
    float times[2][NG], minus[2][NG];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            if constexpr (DYNAMIC) {
                times[c][g] = kUnit * ref[c][g];
                minus[c][g] = 8.0f * ref[c][g] * (lw[c][g] + __shfl_xor(lw[c][g], 32, 64));
            } else {
                times[c][g] = kUnit * v_step;
                minus[c][g] = 8.0f * v_step * l_all[c];
            }
        }
    if (splits > 1) {
        // [slot][row of the accumulators, maximum, sum][256 rows]: neighbouring lanes write neighbouring floats
        float* dst = partial + ((index * Hkv + head) * splits + split) * (int64_t)(D + 2) * kRows + wave * kCols + col;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    dst[(32 * d + 8 * (i >> 2) + 4 * half + (i & 3)) * kRows + 32 * c] = fmaf(o[c][d][i], times[c][d / DBG], -minus[c][d / DBG]);
            if (half == 0) {
                dst[D * kRows + 32 * c] = m[c];
                dst[(D + 1) * kRows + 32 * c] = l_all[c];
            }
        }
        return;
    }
    __syncthreads();
    __half* const lines = reinterpret_cast<__half*>(raw_lds) + wave * kCols * (D + 8);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float f = l_all[c] > 0.0f ? 1.0f / l_all[c] : 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                lines[(32 * c + col) * (D + 8) + channel_of<G>(32 * d + 8 * (i >> 2) + 4 * half + (i & 3))] =
                    __float2half_rn(fmaf(o[c][d][i], times[c][d / DBG], -minus[c][d / DBG]) * f);
    }
    // (each wavefront its own rows: what it reads here it has written itself)
    constexpr int kPer = D / 8;                    // lanes to a row
    for (int i = lane / kPer; i < kCols; i += 64 / kPer) {
        const int row = row0 + wave * kCols + i;
        if (row < rows)
            *reinterpret_cast<v4u*>(a.out + ((int64_t)(r.start + row / per_kv) * a.n_heads + head * per_kv + row % per_kv) * D + 8 * (lane % kPer)) =
                *reinterpret_cast<const v4u*>(lines + i * (D + 8) + 8 * (lane % kPer));
    }
}

// Adds the parts of a tile's rows: a workgroup takes 64 rows, a wavefront a quarter of the channels.
template <int D, int G>
__global__ __launch_bounds__(kThreads) void k_kv4_attention_join_tiles(AttentionArgs a, const float* __restrict__ partial, int splits, int small_rows)
{
    __shared__ __align__(16) __half lines[64][D + 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, Hkv = a.cache.n_kv_heads;
    const int head = blockIdx.x % Hkv;
    const int64_t index = blockIdx.x / Hkv;
    const Where at = find_tile(a, index, small_rows, lane);
    if (at.b < 0) return;
    const int rows = at.r.q_len * a.heads_per_kv, row0 = at.tile * kRows + blockIdx.y * 64;
    if (row0 >= rows) return;
    const int64_t size = (int64_t)(D + 2) * kRows;
    const float* src = partial + (index * Hkv + head) * splits * size + blockIdx.y * 64 + lane;
    float top = kNothing, sum = 0.0f;
    for (int s = 0; s < splits; ++s) top = fmaxf(top, src[s * size + D * kRows]);
    float acc[D / 4];
#pragma unroll
    for (int i = 0; i < D / 4; ++i) acc[i] = 0.0f;
    for (int s = 0; s < splits; ++s) {
        const float f = __builtin_amdgcn_exp2f(src[s * size + D * kRows] - top);
        sum = fmaf(src[s * size + (D + 1) * kRows], f, sum);
#pragma unroll
        for (int i = 0; i < D / 4; ++i) acc[i] = fmaf(src[s * size + (wave * (D / 4) + i) * kRows], f, acc[i]);
    }
    const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int i = 0; i < D / 4; ++i) lines[lane][channel_of<G>(wave * (D / 4) + i)] = __float2half_rn(acc[i] * f);
    __syncthreads();
    constexpr int kPer = D / 8;
    for (int i = tid / kPer; i < 64; i += kThreads / kPer) {
        const int row = row0 + i;
        if (row < rows)
            *reinterpret_cast<v4u*>(a.out + ((int64_t)(at.r.start + row / a.heads_per_kv) * a.n_heads + head * a.heads_per_kv + row % a.heads_per_kv) * D +
                                    8 * (tid % kPer)) = *reinterpret_cast<const v4u*>(&lines[i][8 * (tid % kPer)]);
    }
}

int64_t tiles_at_most(int64_t T, int32_t B, int32_t per_kv) { return T * per_kv / kRows + B; }

// Parts of a history: as many as bring the tiles to the compute units, and no longer than to leave each some tiles of tokens.
int splits_for(int64_t tiles, int32_t n_kv_heads, int64_t capacity)
{
    const int64_t groups = tiles * n_kv_heads;
    int64_t s = 512 / (groups > 0 ? groups : 1);
    const int64_t most = capacity / (8 * kTile);
    if (s > most) s = most;
    return s > 1 ? (int)s : 1;
}

template <int D, int G, bool DYNAMIC>
int launch(const AttentionArgs& a, int64_t tiles, int splits, int small_rows, float* partial, hipStream_t st)
{
    static std::atomic<uint64_t> allowed{0};
    const size_t out = (size_t)kWaves * kCols * (D + 8) * 2, lds = sizeof(Lds<D, G, DYNAMIC>) > out ? sizeof(Lds<D, G, DYNAMIC>) : out;
    const auto kernel = k_kv4_attention_tiles<D, G, DYNAMIC>;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, allowed); rc != PQ_OK) return rc;
    const int Hkv = a.cache.n_kv_heads;
    kernel<<<(unsigned)(tiles * Hkv * splits), kThreads, lds, st>>>(a, partial, splits, small_rows);
    if (splits > 1) k_kv4_attention_join_tiles<D, G><<<dim3((unsigned)(tiles * Hkv), kRows / 64), kThreads, 0, st>>>(a, partial, splits, small_rows);
    return hip_status(hipGetLastError());
}

}  // namespace

size_t tiles_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int64_t capacity)
{
    const int64_t tiles = tiles_at_most(T, B, n_heads / n_kv_heads);
    const int splits = splits_for(tiles, n_kv_heads, capacity);
    return splits > 1 ? (size_t)(tiles * n_kv_heads * splits) * kRows * (head_dim + 2) * sizeof(float) : 0;
}

int launch_attention_tiles(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, float* partial, hipStream_t st)
{
    const int64_t tiles = tiles_at_most(a.T, a.B, a.heads_per_kv);
    const int splits = splits_for(tiles, a.cache.n_kv_heads, (int64_t)a.table_pages << a.cache.log2_page);
    if (head_dim == 64) {
        if (group == 0) return launch<64, 64, false>(a, tiles, splits, small_rows, partial, st);
        if (group == 32) return launch<64, 32, true>(a, tiles, splits, small_rows, partial, st);
        return launch<64, 64, true>(a, tiles, splits, small_rows, partial, st);
    }
    if (group == 0) return launch<128, 128, false>(a, tiles, splits, small_rows, partial, st);
    if (group == 32) return launch<128, 32, true>(a, tiles, splits, small_rows, partial, st);
    if (group == 64) return launch<128, 64, true>(a, tiles, splits, small_rows, partial, st);
    return launch<128, 128, true>(a, tiles, splits, small_rows, partial, st);
}

}  // namespace kv4
}  // namespace pq
