// Attention over the paged 4-bit cache for many queries of a request: prompts, and chunks of them.
//
// Bound by the matrix instructions: 4 D operations for every query, head and token that it sees, the codes read once per 256 rows.  A workgroup
// of eight wavefronts takes 256 rows (a request's tokens times the query heads that share a key/value head), each wavefront 32 of them, the
// columns of the matrix instructions.  A step is a tile of 64 tokens: its codes are expanded once per workgroup into fp16 operands in LDS,
// keys by four wavefronts and values by the other four (the expansion by every wavefront for itself would be eight times the vector
// instructions, which are scarce beside the exponentials), while the codes after next are on their way.  Two wavefronts share a SIMD: one's
// exponentials run beside the other's products.  (Four wavefronts of 64 columns with 512 registers each needed fewer reads of LDS and spilled:
// 1.8 times as long.)  500 queries over 33000 tokens, 64 heads on 8: 537 GFLOP in 510 us, 1050 TFLOP/s (a library product of fp16 matrices:
// 1171), matrix pipe busy 48 % of the cycles at 2.0 GHz.  4 prompts of up to 4096 tokens, 32 heads on 8: 314 GFLOP in 363 us, 870 TFLOP/s:
// a workgroup's start and end take as long as five of its steps, of which it has 26 on average, and 5 % of the products meet the mask.
//
// Where a call has few tiles of rows, the histories are cut into `splits` parts; their sums go through scratch memory and a second kernel.
#include "pq_kv4_attention.h"

#define PQ_INLINE __attribute__((always_inline))

namespace pq {
namespace kv4 {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kThreads = 512, kWaves = 8;
constexpr int kRows = kTileRows, kCols = 32;      // rows of a workgroup and of a wavefront
constexpr int kTile = 64;                         // tokens of a step
constexpr int kPrefixTile = 32;
constexpr int kJoinThreads = 256;
constexpr float kLeast = 0x1.0p-80f;

__device__ __forceinline__ v16f product(const v8h& a, const v8h& b, const v16f& c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

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

// For many requests: `starts`, tiles before each request and in all.  A workgroup that walks over the requests itself reads all of them, and
// there may be as many workgroups; with this list it reads some ten or twenty entries.  Without | with it, us, 4 heads of 128 on one, 60
// queries each over 200 tokens: 256 requests 32 | 34, 512 61 | 60, 1024 124 | 107, 2048 361 | 221, 16384 9700 | 1520, 65536 136000 | 5900.
constexpr int kManyRequests = 512;
constexpr int kStartThreads = 1024;
__global__ __launch_bounds__(kStartThreads) void k_kv4_attention_tile_starts(AttentionArgs a, int32_t* starts, int small_rows)
{
    __shared__ int64_t sums[kStartThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, each = (a.B + kStartThreads - 1) / kStartThreads;
    const int first = min(tid * each, a.B), last = min(first + each, a.B);
    int64_t own = 0;
    for (int b = first; b < last; ++b) own += tiles_of(a, request(a, b), small_rows);
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(incl, d, 64);
        if (lane >= d) incl += v;
    }
    if (lane == 63) sums[tid >> 6] = incl;
    __syncthreads();
    int64_t at = incl - own;
    for (int w = 0; w < tid >> 6; ++w) at += sums[w];
    auto saturate = [](int64_t v) PQ_INLINE { return (int32_t)min(v, (int64_t)INT32_MAX); };   // (of rows that lie in several requests)
    for (int b = first; b < last; ++b) {
        starts[b] = saturate(at);
        at += tiles_of(a, request(a, b), small_rows);
    }
    if (tid == kStartThreads - 1) starts[a.B] = saturate(at);
}

__device__ __forceinline__ Where find_tile(const AttentionArgs& a, int64_t index, int small_rows, const int32_t* __restrict__ starts, int lane)
{
    if (starts != nullptr) {
        if (index >= starts[a.B]) return {-1, 0, {0, 0, 0, 0}};
        int lo = 0, hi = a.B - 1;                  // the first request that ends behind the index
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (starts[mid + 1] > index) hi = mid;
            else lo = mid + 1;
        }
        const Request r = request(a, lo);
        const int n = tiles_of(a, r, small_rows), tile = n - 1 - (int)(index - starts[lo]);
        return {tile >= 0 && tile < n ? lo : -1, tile, r};
    }
    const int each = (a.B + 63) / 64, first = min(lane * each, a.B), last = min(first + each, a.B);
    Request r = {0, 0, 0, 0};                       // the last of this lane's; up to 64 requests are read once
    int64_t own = 0;
    for (int b = first; b < last; ++b) {
        r = request(a, b);
        own += tiles_of(a, r, small_rows);
    }
    int64_t incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(incl, d, 64);
        if (lane >= d) incl += v;
    }
    const bool mine = incl - own <= index && index < incl;
    const uint64_t found = __builtin_amdgcn_ballot_w64(mine);
    if (found == 0) return {-1, 0, r};
    int b = first, tile = (int)(incl - 1 - index);
    if (mine && last - first > 1) {
        int64_t u = incl - own;
        for (; b < last; ++b) {
            r = request(a, b);
            const int n = tiles_of(a, r, small_rows);
            if (index < u + n) {
                tile = (int)(u + n - 1 - index);
                break;
            }
            u += n;
        }
    }
    const int from = __builtin_ctzll(found);
    auto lanes = [&](int v) PQ_INLINE { return __builtin_amdgcn_readlane(v, from); };
    return {lanes(b), lanes(tile), {lanes(r.start), lanes(r.q_len), lanes(r.n), lanes(r.sees)}};
}

// Row `at` of the accumulators as a channel: channels of a group lie so in LDS that neighbouring threads of the expansion write
// neighbouring places.
template <int G> __device__ __forceinline__ constexpr int channel_of(int at)
{
    const int in = at % G;
    return at - in + 8 * (in % (G / 8)) + in / (G / 8);
}
template <int G> __device__ __forceinline__ constexpr int place_of(int channel)
{
    const int in = channel % G;
    return channel - in + (in % 8) * (G / 8) + in / 8;
}

// Operands of codes, u * 2^-20, without their offset: (u - 8) * 2^-20, exact in fp16.  For values its roundings would be many times the result's
// own over a long history of like weights (500 queries over 33000 tokens, 24 sets of inputs: errors of 1.45 times the rounding of the exact result
// at the median, 1.65 at most, without it 1.38 and 1.41; it costs 516 -> 519 us).  For keys with dynamic steps it would cost an addition to every
// score; here it is taken off once for all eight wavefronts.
template <int N, typename V> __device__ __forceinline__ V without_offset(const V& x)
{
    typedef _Float16 halves __attribute__((ext_vector_type(N)));
    return __builtin_bit_cast(V, __builtin_bit_cast(halves, x) - (halves)(_Float16)0x1.0p-17f);
}

template <int D, int G, bool DYNAMIC>
struct Lds {
    static constexpr int NG = D / G;
    v4u k[2][kTile][D / 8 + 1];          // [token][eight channels]; tokens an odd number of 16 bytes apart, so that eight of them meet all banks
    v2u v[2][kTile / 16][2][D][2];       // [16 tokens][half of the lanes][channel]: eight tokens in the order of the probabilities
    float ks[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1][kTile], vs[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1][kTile];
    float vs_most[DYNAMIC ? 2 : 1][DYNAMIC ? NG : 1][4];     // largest of a block of 16 tokens
    int bad[2][4];                       // blocks of 16 tokens whose page is none
};

// Two workgroups to a CU where 128 registers do: one's start and end, and its waits at the barriers, beside the other's products (64 channels,
// static steps, 32 heads on 8, one | two: 4 prompts of up to 4096 tokens 232 | 206 us, 4 of 4096 390 | 357, 300 queries each over up to 4000 64 |
// 65, 500 over 33000 178 | 184; with dynamic steps what does not fit is spilled: to 64 channels 347 | 422, 500 over 33000 277 | 531).
template <int D, int G, bool DYNAMIC>
__global__ __launch_bounds__(kThreads, D == 64 && !DYNAMIC ? 4 : 2) void k_kv4_attention_tiles(AttentionArgs a, float* partial, const int32_t* __restrict__ starts, int splits, int small_rows)
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
    const Where at = find_tile(a, index, small_rows, starts, lane);
    if (at.b < 0) return;
    const Request r = at.r;
    const int rows = r.q_len * per_kv, row0 = at.tile * kRows;
    const int last_token = min((row0 + kRows - 1) / per_kv, r.q_len - 1);
    const int visible = __builtin_amdgcn_readfirstlane(sees(a, r, last_token));        // (a division leaves it in a vector register)
    const int all_tiles = (visible + kTile - 1) / kTile;
    const int begin = (int)((int64_t)all_tiles * split / splits), end = (int)((int64_t)all_tiles * (split + 1) / splits);

    // this lane's query
    int limit, wave_sees;                    // tokens that it sees, and that all of the wavefront's see
    v8h q[KS];
    float c0 = 0.0f;                         // -8 sum(q): the codes' offset (dynamic steps: the operands are without it)
    {
        const int row = min(row0 + wave * kCols + col, rows - 1);
        const int token = row / per_kv, q_head = head * per_kv + row % per_kv;
        limit = sees(a, r, token);
        wave_sees = __builtin_amdgcn_readfirstlane(sees(a, r, min(row0 + wave * kCols, rows - 1) / per_kv));
        const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8h*>(src + 16 * s + 8 * half);
    }
    // ---- the history: wavefronts w and w + 4 load and expand keys and values of tokens 16 w .. 16 w + 15 of every tile
    const int32_t* table = a.table + (int64_t)at.b * a.table_pages;
    const int block = wave & 3;
    const bool keys = wave < 4;
    struct Codes { v4u w; float s; int bad; };
    auto page_of = [&](int tile) PQ_INLINE { return table[min((tile * kTile + 16 * block) >> log2_page, a.table_pages - 1)]; };
    auto load = [&](int tile, int page, Codes& x) PQ_INLINE {
        const int t = tile * kTile + 16 * block;
        x.bad = (uint32_t)page >= (uint64_t)a.cache.n_pages || (t >> log2_page) >= a.table_pages;
        const int64_t from = x.bad ? 0 : page, first = ((from * Hkv + head) << log2_page) + (t & ((1 << log2_page) - 1));
        // (one vector, set as a whole on both sides: an array's members went through scratch memory in every step)
        if (keys) {                                // D / 4 channels of a token to a lane
            const uint8_t* src = a.cache.k_codes + (first + (lane >> 2)) * (D / 2) + (lane & 3) * (D / 8);
            if constexpr (D == 128) {
                x.w = *reinterpret_cast<const v4u*>(src);
            } else {
                const v2u w = *reinterpret_cast<const v2u*>(src);
                x.w = (v4u){w[0], w[1], 0, 0};
            }
        } else {                                   // D / 16 channels of four tokens
            auto token = [&](int i) PQ_INLINE -> uint32_t {
                const uint8_t* src = a.cache.v_codes + (first + 4 * (lane >> 4) + i) * (D / 2) + (lane & 15) * (D / 32);
                if constexpr (D == 128) return *reinterpret_cast<const uint32_t*>(src);
                else return *reinterpret_cast<const uint16_t*>(src);
            };
            x.w = (v4u){token(0), token(1), token(2), token(3)};
        }
        if constexpr (DYNAMIC) {                   // lane: token lane / 4, group lane % 4
            if ((lane & 3) < NG) x.s = (keys ? a.cache.k_scale : a.cache.v_scale)[(first + (lane >> 2)) * NG + (lane & 3)];
        }
    };
    auto expand = [&](int tile, int buf, const Codes& x) PQ_INLINE {
        const int t = 16 * block + (lane >> 2);
        if (keys) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) sh.k[buf][t][(lane & 3) * (D / 32) + i] =
                DYNAMIC ? without_offset<8>(__builtin_bit_cast(v4u, key_operand(x.w[i]))) : __builtin_bit_cast(v4u, key_operand(x.w[i]));
            if (lane == 0) sh.bad[buf][block] = x.bad;
            if constexpr (DYNAMIC) {
                if ((lane & 3) < NG) sh.ks[buf][lane & 3][t] = x.s;
            }
        } else {
            // four tokens: 8 (quad / 2) + 4 (quad % 2) of the block; the lanes' half quad % 2, the first or second four of its eight
            const int quad = lane >> 4, c = lane & 15;
            uint32_t low[2], high[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                low[i] = __builtin_amdgcn_perm(x.w[2 * i + 1], x.w[2 * i], 0x05040100u) ^ kOffset;
                if constexpr (D == 128) high[i] = __builtin_amdgcn_perm(x.w[2 * i + 1], x.w[2 * i], 0x07060302u) ^ kOffset;
            }
            static_for<0, D / 16>([&](auto J) PQ_INLINE {
                constexpr int j = decltype(J)::value;
                const uint32_t* const w = j < 4 ? low : high;
                const v2u y = {operand<(j & 3)>(w[0]), operand<(j & 3)>(w[1])};
                sh.v[buf][block][quad & 1][place_of<G>(D / 16 * c + j)][quad >> 1] = without_offset<4>(y);
            });
            if constexpr (DYNAMIC) {
                // what lies behind the last token, or in no page, may be anything, and what only later queries see may be infinite: neither
                // must meet a probability of zero as it is
                const float step = tile * kTile + t < r.n && !x.bad ? finite_step(x.s) : 0.0f;
                float most = step;
#pragma unroll
                for (int d = 4; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
                if ((lane & 3) < NG) sh.vs[buf][lane & 3][t] = step;
                if (lane < NG) sh.vs_most[buf][lane][block] = most;
            }
        }
    };

    Codes next;
    int page = 0;
    if (begin < end) {                             // (on their way while the queries are and the prefix tokens are taken)
        load(begin, page_of(begin), next);
        page = page_of(begin + 1);
    }

    // ---- prefix tokens, in tiles of 32: a thread's token and eight channels of it
    const bool prefix = a.n_prefix > 0 && split == 0;
    const int prefix_t = tid / (D / 8), prefix_c = tid % (D / 8);
    v4u prefix_k = {}, prefix_v = {};
    auto load_prefix = [&](int t0) PQ_INLINE {
        if (prefix_t >= kPrefixTile) return;
        const int64_t from = ((int64_t)min(t0 + prefix_t, a.n_prefix - 1) * Hkv + head) * D + 8 * prefix_c;
        prefix_k = *reinterpret_cast<const v4u*>(a.prefix_k + from);
        prefix_v = *reinterpret_cast<const v4u*>(a.prefix_v + from);
    };
    if (prefix) load_prefix(0);

#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = in_key_order(__builtin_bit_cast(v4u, q[s]));
    if constexpr (!DYNAMIC) {
        const v4u minus8 = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
        v16f z = {};
#pragma unroll
        for (int s = 0; s < KS; ++s) z = product(__builtin_bit_cast(v8h, minus8), q[s], z);
        c0 = z[0];
    }

    const float scale = a.softmax_scale * 1.44269504088896341f;
    float c1 = scale * kUnit, v_step = 1.0f;
    if constexpr (!DYNAMIC) {
        c1 *= a.cache.k_scale[head];
        v_step = a.cache.v_scale[head];
    }

    float m = kNothing, l = 0.0f;
    float ref[NG];                           // dynamic steps: weights p * step are rounded relative to ref
    v16f o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) o[i] = (v16f){};
#pragma unroll
    for (int g = 0; g < NG; ++g) ref[g] = kLeast;

    // exp2(c1 x + bias - m) of a tile's scores.  The reference m follows the largest; what is there is rescaled.
    auto probabilities = [&](auto& x, float c1, float bias, auto& p) PQ_INLINE {
        constexpr int N = sizeof(x) / sizeof(x[0]);
        float most = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
        most = fmaf(most, c1, bias);
        if (__builtin_amdgcn_ballot_w64(most > m + kMost) != 0) {
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float to_m = most > m + kMost ? ceilf(most) - kBack : m;
            const float alpha = __builtin_amdgcn_exp2f(m - to_m);
            m = to_m;
            l *= alpha;
            if constexpr (DYNAMIC) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float y = ref[g] * alpha, f = y >= kLeast ? 1.0f : y * (1.0f / kLeast);
                    ref[g] = fmaxf(y, kLeast);
#pragma unroll
                    for (int i = 0; i < DBG; ++i) o[g * DBG + i] *= f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < DB; ++i) o[i] *= alpha;
            }
        }
        const float minus = bias - m;
        float own = 0.0f;                          // (this tile's first: add_halves)
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c1, minus));
            x[i + 1] = __builtin_amdgcn_exp2f(fmaf(x[i + 1], c1, minus));
            const uint32_t two = two_halves(x[i], x[i + 1]);
            p[i >> 3][(i & 7) >> 1] = two;
            if constexpr (DYNAMIC) own += x[i] + x[i + 1];         // (the product rounds weights, and not these)
            else own = add_halves(two, own);
        }
        l += own;
    };
    // dynamic steps: the weights p * step of one group, rounded relative to ref, which moves as m does
    auto weights = [&](int buf, int g, const float (&x)[32], float most_x, v4u (&p)[4]) PQ_INLINE {
        const v4f most4 = *reinterpret_cast<const v4f*>(&sh.vs_most[buf][g][0]);
        const float most_step = fmaxf(fmaxf(most4[0], most4[1]), fmaxf(most4[2], most4[3]));
        // no weight is larger than this product
        if (__builtin_amdgcn_ballot_w64(most_x * most_step > 0x1.0p14f * ref[g]) != 0) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const v4f step = *reinterpret_cast<const v4f*>(&sh.vs[buf][g][2 * i + 4 * half]);
#pragma unroll
                for (int j = 0; j < 4; ++j) most = fmaxf(most, x[i + j] * step[j]);
            }
            most = fmaxf(most, __shfl_xor(most, 32, 64)) * inverse(ref[g]);
            const int up = most > 0x1.0p14f ? ilogbf(most) - (int)kBack : 0;
            const float f = ldexpf(1.0f, -up);
            ref[g] = ldexpf(ref[g], up);
#pragma unroll
            for (int i = 0; i < DBG; ++i) o[g * DBG + i] *= f;
        }
        const float inv = inverse(ref[g]);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const v4f step = *reinterpret_cast<const v4f*>(&sh.vs[buf][g][2 * i + 4 * half]);
            p[i >> 3][(i & 7) >> 1] = two_halves(x[i] * inv * step[0], x[i + 1] * inv * step[1]);
            p[i >> 3][((i & 7) >> 1) + 1] = two_halves(x[i + 2] * inv * step[2], x[i + 3] * inv * step[3]);
        }
    };
    // scores x of a tile [token 32 tb + 8 (i / 4) + 4 half + i % 4], in units of a code (dynamic: of 2^20 steps)
    auto scores = [&](int buf, auto& x) PQ_INLINE {
        constexpr int TB = sizeof(x) / sizeof(x[0]) / 16;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) {
                v16f z = {};
#pragma unroll
                for (int k = 0; k < KSG; ++k)
                    z = product(__builtin_bit_cast(v8h, sh.k[buf][32 * tb + col][2 * (g * KSG + k) + half]), q[g * KSG + k], z);
                if constexpr (DYNAMIC) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const v4f step = *reinterpret_cast<const v4f*>(&sh.ks[buf][g][32 * tb + 2 * i + 4 * half]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float& to = x[16 * tb + i + j];
                            to = g == 0 ? z[i + j] * step[j] : fmaf(z[i + j], step[j], to);
                        }
                    }
                    // (computed here, and not sunk to where the scores are used: all groups' products and steps would not fit the registers)
#pragma unroll
                    for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(x[16 * tb + i]));
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[16 * tb + i] = z[i];
                }
            }
        }
    };
    auto multiply = [&](int buf, int first, int count, const auto& p) PQ_INLINE {
#pragma unroll
        for (int k = 0; k < (int)(sizeof(p) / sizeof(p[0])); ++k)
#pragma unroll
            for (int d = first; d < first + count; ++d)
                o[d] = product(*reinterpret_cast<const v8h*>(&sh.v[buf][k][half][32 * d + col][0]), __builtin_bit_cast(v8h, p[k]), o[d]);
    };

    // ---- prefix tokens, in fp16 where the codes' operands lie
    if (prefix) {
        for (int t0 = 0; t0 < a.n_prefix; t0 += kPrefixTile) {
            __syncthreads();
            if (prefix_t < kPrefixTile) {
                const int t = prefix_t, in16 = t & 15;             // token t of its 16: 8 (t / 8) + 4 (half of the lanes) + t % 4
                sh.k[0][t][prefix_c] = __builtin_bit_cast(v4u, in_key_order(prefix_k));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __half* dst = reinterpret_cast<__half*>(&sh.v[0][t >> 4][(in16 >> 2) & 1][place_of<G>(8 * prefix_c + j)][in16 >> 3]);
                    dst[in16 & 3] = reinterpret_cast<const __half*>(&prefix_v)[j];
                }
            }
            if constexpr (DYNAMIC) {
                if (tid < kPrefixTile) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) sh.ks[0][g][tid] = 1.0f;
                }
            }
            if (t0 + kPrefixTile < a.n_prefix) load_prefix(t0 + kPrefixTile);
            __syncthreads();
            float x[kPrefixTile / 2];
            v4u p[kPrefixTile / 16];
            scores(0, x);
            const int left = a.n_prefix - t0 - 4 * half;
#pragma unroll
            for (int i = 0; i < kPrefixTile / 2; ++i)
                if (8 * (i >> 2) + (i & 3) >= left) x[i] = -INFINITY;
            probabilities(x, scale, 0.0f, p);
            multiply(0, 0, DB, p);
        }
        __syncthreads();
        // in units of a code
        const float times = DYNAMIC ? 1.0f / (kUnit * kLeast) : 1.0f / (kUnit * v_step);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= times;
#pragma unroll
        for (int g = 0; g < NG; ++g) ref[g] = kLeast;
    }

    if (begin < end) {
        const float bias = c0 * c1;
        expand(begin, 0, next);
        load(begin + 1, page, next);
        page = page_of(begin + 2);
        for (int i = begin; i < end; ++i) {
            const int buf = (i - begin) & 1;
            __syncthreads();                       // tile i is in LDS; nobody reads tile i - 1 any more
            const int page_after = page_of(i + 3);
            float x[32];
            v4u p[4];
            scores(buf, x);
            expand(i + 1, buf ^ 1, next);
            load(i + 2, page, next);
            page = page_after;
            // what rows do not see, or has no page
            if (i * kTile + kTile > wave_sees ||
                __builtin_amdgcn_readfirstlane(sh.bad[buf][0] | sh.bad[buf][1] | sh.bad[buf][2] | sh.bad[buf][3]) != 0) {
                const int left = limit - (i * kTile + 4 * half);
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (8 * (j >> 2) + (j & 3) >= left || sh.bad[buf][j >> 3]) x[j] = -INFINITY;
            }
            probabilities(x, c1, bias, p);
            if constexpr (DYNAMIC) {
                float most_x = x[0];
#pragma unroll
                for (int i = 1; i < 32; ++i) most_x = fmaxf(most_x, x[i]);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    weights(buf, g, x, most_x, p);
                    multiply(buf, g * DBG, DBG, p);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                multiply(buf, 0, DB, p);
            }
        }
    }

    // ---- results
    const float l_all = l + __shfl_xor(l, 32, 64);
    float times[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) times[g] = kUnit * (DYNAMIC ? ref[g] : v_step);
    if (splits > 1) {
        // [slot][row of the accumulators, maximum, sum][256 rows]: neighbouring lanes write neighbouring floats
        float* dst = partial + ((index * Hkv + head) * splits + split) * (int64_t)(D + 2) * kRows + wave * kCols + col;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                dst[(32 * d + 8 * (i >> 2) + 4 * half + (i & 3)) * kRows] = o[d][i] * times[d / DBG];
        if (half == 0) {
            dst[D * kRows] = m;
            dst[(D + 1) * kRows] = l_all;
        }
        return;
    }
    __syncthreads();
    __half* const lines = reinterpret_cast<__half*>(raw_lds) + wave * kCols * (D + 8);
    const float f = l_all > 0.0f ? 1.0f / l_all : 0.0f;
    if constexpr (G >= 64) {                       // a lane holds eight channels in a row, 16 bytes
        constexpr int kStep = G / 8, kOver = 16 / kStep;           // rows of the accumulators between them, of them in one block
#pragma unroll
        for (int d0 = 0; d0 < DB; d0 += DBG)
#pragma unroll
            for (int i0 = 0; i0 < 16 / (2 * kOver); ++i0) {
                v4u w;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float y[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int d = d0 + (e + k) / (2 * kOver), i = i0 + (e + k) % (2 * kOver) * (16 / (2 * kOver));
                        y[k] = o[d][i] * times[d / DBG] * f;
                    }
                    w[e / 2] = two_halves(y[0], y[1]);
                }
                *reinterpret_cast<v4u*>(lines + col * (D + 8) + channel_of<G>(32 * d0 + 8 * (i0 >> 2) + 4 * half + (i0 & 3))) = w;
            }
    } else {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                lines[col * (D + 8) + channel_of<G>(32 * d + 8 * (i >> 2) + 4 * half + (i & 3))] =
                    __float2half_rn(o[d][i] * times[d / DBG] * f);
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
__global__ __launch_bounds__(kJoinThreads) void k_kv4_attention_join_tiles(AttentionArgs a, const float* __restrict__ partial, const int32_t* __restrict__ starts, int splits,
                                                                            int small_rows)
{
    __shared__ __align__(16) __half lines[64][D + 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, Hkv = a.cache.n_kv_heads;
    const int head = blockIdx.x % Hkv;
    const int64_t index = blockIdx.x / Hkv;
    const Where at = find_tile(a, index, small_rows, starts, lane);
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
    for (int i = tid / kPer; i < 64; i += kJoinThreads / kPer) {
        const int row = row0 + i;
        if (row < rows)
            *reinterpret_cast<v4u*>(a.out + ((int64_t)(at.r.start + row / a.heads_per_kv) * a.n_heads + head * a.heads_per_kv + row % a.heads_per_kv) * D +
                                    8 * (tid % kPer)) = *reinterpret_cast<const v4u*>(&lines[i][8 * (tid % kPer)]);
    }
}

// Tiles of rows, at most.  Of several requests only those of more than 192 rows come here, and R such rows are at most 2 R / 257 tiles
// (two of 257): requests that decode beside a prompt do not count as a tile each.
int64_t tiles_at_most(int64_t T, int32_t B, int32_t per_kv)
{
    const int64_t by_requests = (T * per_kv + (int64_t)(kRows - 1) * B) / kRows, by_rows = 2 * T * per_kv / (kRows + 1);
    static_assert(2 * (kSmallRows + 1) >= kRows + 1, "one tile of the fewest rows");
    return B == 1 || by_requests < by_rows ? by_requests : by_rows > 1 ? by_rows : 1;
}

// Parts of a history, of at least eight tiles of tokens each where the table is as long as the history (the host knows the table; parts of
// shorter ones are shorter, or empty).  Several requests differ in length: about two workgroups to a CU even that
// out (B 4, 300 queries each over up to 4000 tokens, 32 on 8 heads: one part 127 us, two 103, three 112).  The parts of one request are
// alike: as many as fill whole rounds of one workgroup to a CU, which is what its registers allow, with eight tiles' time for what every
// workgroup does once (500 queries over 33000 tokens, 64 on 8 heads: one part 910 us, two 534, four 541; 64 queries over 131072, 32 on 8
// heads: 16 parts 269, 32 173, 64 202; 400 queries over 20000, 8 heads on one: 19 parts 75, 39 91).
int splits_for(int64_t tiles, int32_t B, int32_t n_kv_heads, int64_t capacity)
{
    const int64_t groups = tiles * n_kv_heads, steps = capacity / kTile, most = steps / 8 < 512 / groups ? steps / 8 : 512 / groups;
    if (most <= 1) return 1;
    if (B > 1) return (int)most;
    int best = 1;
    double least = 1e30;
    for (int s = 1; s <= (int)most; ++s) {
        const double time = (double)((groups * s + 255) / 256) * ((double)steps / s + 8.0);
        if (time < least) {
            least = time;
            best = s;
        }
    }
    return best;
}

template <int D, int G, bool DYNAMIC>
int launch(const AttentionArgs& a, int64_t tiles, int splits, int small_rows, float* partial, const int32_t* starts, hipStream_t st)
{
    static std::atomic<uint64_t> allowed{0};
    const size_t out = (size_t)kWaves * kCols * (D + 8) * 2, lds = sizeof(Lds<D, G, DYNAMIC>) > out ? sizeof(Lds<D, G, DYNAMIC>) : out;
    const auto kernel = k_kv4_attention_tiles<D, G, DYNAMIC>;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, allowed); rc != PQ_OK) return rc;
    const int Hkv = a.cache.n_kv_heads;
    kernel<<<(unsigned)(tiles * Hkv * splits), kThreads, lds, st>>>(a, partial, starts, splits, small_rows);
    if (splits > 1) k_kv4_attention_join_tiles<D, G><<<dim3((unsigned)(tiles * Hkv), kRows / 64), kJoinThreads, 0, st>>>(a, partial, starts, splits, small_rows);
    return hip_status(hipGetLastError());
}

// Scratch memory: partial sums, then the list of starts.
size_t tiles_partial_bytes(int64_t tiles, int splits, int32_t n_kv_heads, int32_t head_dim)
{
    return splits > 1 ? (size_t)(tiles * n_kv_heads * splits) * kRows * (head_dim + 2) * sizeof(float) : 0;
}

}  // namespace

size_t tiles_workspace_bytes(int64_t T, int32_t B, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int64_t capacity)
{
    const int64_t tiles = tiles_at_most(T, B, n_heads / n_kv_heads);
    const int splits = splits_for(tiles, B, n_kv_heads, capacity);
    return tiles_partial_bytes(tiles, splits, n_kv_heads, head_dim) + (B > kManyRequests ? ((size_t)(B + 1) * sizeof(int32_t) + 255) & ~(size_t)255 : 0);
}

int launch_attention_tiles(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, float* partial, hipStream_t st)
{
    const int64_t tiles = tiles_at_most(a.T, a.B, a.heads_per_kv);
    const int splits = splits_for(tiles, a.B, a.cache.n_kv_heads, (int64_t)a.table_pages << a.cache.log2_page);
    int32_t* starts = nullptr;
    if (a.B > kManyRequests) {
        starts = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(partial) + tiles_partial_bytes(tiles, splits, a.cache.n_kv_heads, head_dim));
        k_kv4_attention_tile_starts<<<1, kStartThreads, 0, st>>>(a, starts, small_rows);
    }
    if (head_dim == 64) {
        if (group == 0) return launch<64, 64, false>(a, tiles, splits, small_rows, partial, starts, st);
        if (group == 32) return launch<64, 32, true>(a, tiles, splits, small_rows, partial, starts, st);
        return launch<64, 64, true>(a, tiles, splits, small_rows, partial, starts, st);
    }
    if (group == 0) return launch<128, 128, false>(a, tiles, splits, small_rows, partial, starts, st);
    if (group == 32) return launch<128, 32, true>(a, tiles, splits, small_rows, partial, starts, st);
    if (group == 64) return launch<128, 64, true>(a, tiles, splits, small_rows, partial, starts, st);
    return launch<128, 128, true>(a, tiles, splits, small_rows, partial, starts, st);
}

}  // namespace kv4
}  // namespace pq
