// A step's queries, keys and values on their way into attention: per-head RMS norm, position rotation and Hadamard rotation (App. B
// "Online Rotation", R3) of queries and keys, and the 4-bit codes of keys and values in the slots of a paged cache (Table 1: per-head
// static steps of O2, group-wise dynamic ones of O1), in one pass over the fused projection's output.
//
//     queries, keys:  y = x / sqrt(mean x^2 + eps) * w;   (y_a, y_b) <- (y_a cos - y_b sin, y_b cos + y_a sin);   z = H_D y / sqrt(D)
//     values:         z = x
//     queries leave as fp16(z); codes = clamp(round_half_even(z / step), -8, 7)
//
// The codes are those of the definition in double precision.  They are computed in fp32; where a quotient lies nearer to a border
// k + 1/2 than the error of the fp32 path can reach, its head vector is computed again in fp64 (a few in a thousand), so neither the
// order of the fp32 sums nor their contraction shows in the cache.
//
// Bound by HBM: 2 bytes of every channel in, 2 out for queries and half a byte for keys and values (8192 tokens x 48 heads of 128: 180 MB in
// 44 us, 4.1 TB/s, where a copy of as many bytes takes 35); with norms and dynamic steps (2111 tokens x 80 heads: 81 MB in 26 us) by no one
// thing: vector instructions issue in 39 % of the cycles, and the wavefronts are a round and a fifth of what the card holds; a step of 64
// tokens by its launch and three dependent loads (4.5 us).  A lane holds eight channels (16 bytes), D / 8 lanes a head, a wavefront the same
// head of 8 or 4 consecutive tokens: one kind of work to a wavefront, the step and the norm's weights are read once, and in a page the tokens
// of a head lie one after another.  The four wavefronts of a workgroup take four neighbouring heads of these tokens, which share the rows of
// the table of angles.
#include "pq_kv4.h"
#include "pq_rotate.h"

namespace pq {
namespace kv4 {
namespace {

constexpr int kThreads = 256;

template <int B> __device__ __forceinline__ float from_lane_xor(float v) { return rq::lane_xor<B>(v); }
template <int B> __device__ __forceinline__ double from_lane_xor(double v) { return __shfl_xor(v, 1 << B, 64); }

// Over the lanes of 2^BITS neighbours.
template <int BITS, typename F> __device__ __forceinline__ F sum_lanes(F v)
{
    static_for<0, BITS>([&](auto B) { v += from_lane_xor<decltype(B)::value>(v); });
    return v;
}
template <int BITS, typename F> __device__ __forceinline__ F max_lanes(F v)
{
    static_for<0, BITS>([&](auto B) { v = max(v, from_lane_xor<decltype(B)::value>(v)); });
    return v;
}

// What a lane knows about its eight channels of a query or key, the same for the fp32 and the fp64 path.
struct Lane {
    float x[8];
    float w[8];           // the norm's weight, or 1
    float cs[8], sn[8];   // cosine and sine of each channel's angle, the sine with the sign it enters with
    int partner;          // lane whose channels turn with this one's (halves of less than a head)
    bool turns;           // whether these channels turn
};

// Which channels turn together: none; neighbours; those half a head apart, in lanes one bit apart; those half of rotary_dim apart.
enum Turn { kNone, kPairs, kHalfHead, kHalves };

template <int LOG2_D> __device__ __forceinline__ constexpr double inv_sqrt()       // 1 / sqrt(D)
{
    static_assert(LOG2_D == 6 || LOG2_D == 7, "heads of 64 or 128 channels");
    return LOG2_D == 6 ? 0.125 : 0.08838834764831845;
}

// Everything is linear in the norm's factor, which is left to the caller: v times the return value is what was asked for.  In fp32 the Hadamard
// rotation's values carry the sign of rq::lane_sign as well, which whoever takes them multiplies in.
template <typename F, int LOG2_D, bool ROTATE>
__device__ __forceinline__ F turn(const Lane& c, bool norm, Turn rope, F eps, int lane, F (&v)[8])
{
    F scale = 1;
    constexpr int kLaneBits = LOG2_D - 3;
    constexpr bool kExact = std::is_same<F, double>::value;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (F)c.x[i];
    if (norm) {
        F sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i] * v[i];
        sum = sum_lanes<kLaneBits>(sum);
        const F mean = sum * (F)(1.0 / (1 << LOG2_D)) + eps;
        if constexpr (kExact) scale = 1.0 / sqrt(mean);
        else scale = __builtin_amdgcn_rsqf(mean);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= (F)c.w[i];
    }
    if (rope != kNone) {
        F other[8];
        if (rope == kHalfHead) {
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = from_lane_xor<kLaneBits - 1>(v[i]);
        } else if (rope == kHalves) {
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = __shfl(v[i], c.partner, 64);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) other[i] = v[i ^ 1];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const F turned = v[i] * (F)c.cs[i] + other[i] * (F)c.sn[i];
            v[i] = c.turns ? turned : v[i];        // (not by a sine of zero: an infinity would reach its neighbour)
        }
    }
    if constexpr (ROTATE) {
        if constexpr (!kExact) {
            rq::reg_stages8(v, 3);
            static_for<0, kLaneBits>([&](auto B) { rq::lane_stage<decltype(B)::value>(v, lane); });
        } else {
            static_for<0, 3>([&](auto S) {
                constexpr int d = 1 << decltype(S)::value;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((i & d) == 0) {
                        const F a = v[i], b = v[i + d];
                        v[i] = a + b;
                        v[i + d] = a - b;
                    }
            });
            static_for<0, kLaneBits>([&](auto B) {
                constexpr int b = decltype(B)::value;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const F p = from_lane_xor<b>(v[i]);
                    v[i] = (lane >> b) & 1 ? p - v[i] : p + v[i];
                }
            });
        }
    }
    return scale;
}

// Codes of eight quotients, and whether one of them is nearer than `near` to a border between two codes.
__device__ __forceinline__ uint32_t codes8(const float (&t)[8], float near, bool& suspect)
{
    uint32_t s = 0;
    suspect = false;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        const float c = __builtin_amdgcn_fmed3f(t[i], -8.0f, 7.0f), r = c + rq::kMagic;
        suspect |= !(fabsf(c - (r - rq::kMagic)) <= 0.5f - near);     // (no bound, from a NaN in the vector: all of it)
        s = (s << 4) + __float_as_uint(r);
    }
    return (s - rq::kMagicSum) ^ 0x88888888u;
}

__device__ __forceinline__ uint32_t codes8(const double (&t)[8])
{
    uint32_t s = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) s = (s << 4) | ((uint32_t)(int)fmin(fmax(rint(t[i]), -8.0), 7.0) & 15u);
    return s;
}

__device__ __forceinline__ void halves_to_floats(const v4i raw, float (&v)[8])
{
    const __half2* h = reinterpret_cast<const __half2*>(&raw);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(h[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// A head's static step.  (Both addresses are read before one is chosen: a choice between two members of the arguments kept these in scratch
// memory, 16 bytes of every lane, a fifth of what a long prompt's call wrote.)
__device__ __forceinline__ float head_step(const AppendArgs& a, bool is_value, int kv_head)
{
    const float* const of_keys = a.cache.k_scale;
    const float* const of_values = a.cache.v_scale;
    return (is_value ? of_values : of_keys)[kv_head];
}

// Stores the codes of a wavefront's vectors, and the steps where they are dynamic.
template <int LOG2_D, int LOG2_GROUP>
__device__ __forceinline__ void store_codes(const AppendArgs& a, bool is_value, int64_t token, int c, uint32_t codes, float step)
{
    constexpr int D = 1 << LOG2_D, kGroupBits = LOG2_GROUP ? LOG2_GROUP - 3 : LOG2_D - 3;
    reinterpret_cast<uint32_t*>((is_value ? a.cache.v_codes : a.cache.k_codes) + token * (D / 2))[c] = codes;
    if constexpr (LOG2_GROUP != 0) {
        if ((c & ((1 << kGroupBits) - 1)) == 0) (is_value ? a.cache.v_scale : a.cache.k_scale)[token * (D >> LOG2_GROUP) + (c >> kGroupBits)] = step;
    }
}

// Codes (and steps) of key or value vectors by the definition in fp64, for those vectors of the wavefront that `wanted` has a lane of.
template <int LOG2_D, int LOG2_GROUP, bool ROTATE>
__device__ __forceinline__ void append_exact(const AppendArgs& a, Lane& ln, Turn rope, int head, int64_t token0, uint64_t wanted, int lane)
{
    constexpr int kLanes = (1 << LOG2_D) / 8, kLaneBits = LOG2_D - 3;
    constexpr int kGroupBits = LOG2_GROUP ? LOG2_GROUP - 3 : kLaneBits;
    const int c = lane & (kLanes - 1), Hkv = a.cache.n_kv_heads;
    const bool is_value = head >= a.n_heads + Hkv;
    const int kv_head = head - a.n_heads - (is_value ? Hkv : 0);
    double d[8];
    if (is_value) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = (double)ln.x[i];
    } else {
        if (a.k_weight) halves_to_floats(*reinterpret_cast<const v4i*>(a.k_weight + 8 * c), ln.w);
        const double scale = turn<double, LOG2_D, ROTATE>(ln, a.k_weight != nullptr, rope, (double)a.eps, lane, d) * (ROTATE ? inv_sqrt<LOG2_D>() : 1.0);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] *= scale;
    }
    float step;
    if constexpr (LOG2_GROUP == 0) {
        step = head_step(a, is_value, kv_head);
    } else {
        double most = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmax(most, fabs(d[i]));
        step = (float)((double)a.clip * max_lanes<kGroupBits>(most) / 7.0);
        if (!(step > 0.0f)) step = 1.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] /= (double)step;
    if ((wanted >> (lane & ~(kLanes - 1))) & ((1ull << kLanes) - 1))
        store_codes<LOG2_D, LOG2_GROUP>(a, is_value, token0 + ((int64_t)kv_head << a.cache.log2_page), c, codes8(d), step);
}

// The head vectors of one head of the wavefront's tokens: a query's channels, or the codes of a key or value.  Returns the lanes whose
// codes the fp32 path cannot decide; their vectors are left to append_exact.
template <int LOG2_D, int LOG2_GROUP, bool ROTATE>
__device__ __forceinline__ uint64_t append_head(const AppendArgs& a, Lane& ln, Turn rope, const v4i raw, int head, __half* q_row, int64_t token0, bool live, bool first, int lane)
{
    constexpr int D = 1 << LOG2_D, kLanes = D / 8, kLaneBits = LOG2_D - 3;
    constexpr int kGroupBits = LOG2_GROUP ? LOG2_GROUP - 3 : kLaneBits;
    const int c = lane & (kLanes - 1), Hkv = a.cache.n_kv_heads;
    const bool is_query = head < a.n_heads, is_value = head >= a.n_heads + Hkv;
    const bool norm = !is_value && (is_query ? a.q_weight : a.k_weight) != nullptr;
    // (a wavefront's heads ascend: queries, then keys)
    if (norm && (first || head - kThreads / 64 < a.n_heads != is_query))
        halves_to_floats(*reinterpret_cast<const v4i*>((is_query ? a.q_weight : a.k_weight) + 8 * c), ln.w);
    halves_to_floats(raw, ln.x);
    float unit = ROTATE && !is_value ? (float)inv_sqrt<LOG2_D>() : 1.0f;
    const float sign = ROTATE && !is_value ? rq::lane_sign(lane, kLaneBits) : 1.0f;

    float v[8];
    if (is_value) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ln.x[i];
    } else {
        unit *= turn<float, LOG2_D, ROTATE>(ln, norm, rope, a.eps, lane, v);
    }
    if (is_query) {
        const float m = unit * sign;
        v4i o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(v[2 * i] * m, v[2 * i + 1] * m);
            o[i] = *reinterpret_cast<const int*>(&h);
        }
        if (live) *reinterpret_cast<v4i*>(q_row + head * D) = o;
        return 0;
    }

    const int kv_head = head - a.n_heads - (is_value ? Hkv : 0);
    const int64_t token = token0 + ((int64_t)kv_head << a.cache.log2_page);       // of this head in the cache
    float step;
    if constexpr (LOG2_GROUP == 0) {
        step = head_step(a, is_value, kv_head);
    } else {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
        step = (float)((double)a.clip * ((double)max_lanes<kGroupBits>(most) * unit) / 7.0);
        if (!(step > 0.0f)) step = 1.0f;
    }
    const float mult = unit / step * sign;
    float t8[8], norm2 = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t8[i] = v[i] * mult;
        norm2 = fmaf(t8[i], t8[i], norm2);
    }
    // The multiplier and its product are off by 2^-22 of a quotient, 2^-19 at the end of the range.  The norm's weights, position rotation and
    // butterflies: each rounds by 2^-24 of the vector's length at most and what follows passes it on (the rotations are orthogonal up to a
    // factor), ten such roundings in all, and the norm's factor itself is within 8.5 * 2^-24 of its value (half the 12 roundings of the sum
    // of squares, half of the mean's, the reciprocal root's 2^-23), 8.5 * 2^-21 at the end of the range: with the first less than 2^-17.
    float near = 0x1.0p-17f;
    if (!is_value) near += 0x1.0p-20f * __builtin_amdgcn_sqrtf(sum_lanes<kLaneBits>(norm2));
    bool suspect;
    const uint32_t codes = codes8(t8, near, suspect);
    const uint64_t found = __builtin_amdgcn_ballot_w64(suspect && live);
    // (by vector: what a token gets does not depend on its neighbours)
    if (live && ((found >> (lane & ~(kLanes - 1))) & ((1ull << kLanes) - 1)) == 0) store_codes<LOG2_D, LOG2_GROUP>(a, is_value, token, c, codes, step);
    return found;
}

// One head to a wavefront, or (MANY) eight, every fourth one: then what belongs to the token (its place, its angles) is read once for
// them, the next head's values are on their way while one is turned, and the vectors for the fp64 path wait to the end, so that their
// registers are not held in the loop.  (Five wavefronts to a SIMD are asked for: left alone, static steps take 120 registers and four, 8192
// tokens x 48 heads 48.3 us instead of 46.)
constexpr int kMany = 8;
template <int LOG2_D, int LOG2_GROUP, bool ROTATE, bool MANY>
__global__ __launch_bounds__(kThreads, MANY ? 5 : 1) void k_kv4_append(AppendArgs a)
{
    constexpr int D = 1 << LOG2_D, kLanes = D / 8, kTokens = 64 / kLanes, kStride = kThreads / 64;
    const int lane = threadIdx.x & 63, c = lane & (kLanes - 1), heads = a.n_heads + 2 * a.cache.n_kv_heads;
    constexpr int each = MANY ? kMany : 1;
    int head = blockIdx.y * (kStride * each) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (head >= heads) return;                                           // whole wavefronts; nothing synchronises the workgroup
    const int64_t t = (int64_t)blockIdx.x * kTokens + lane / kLanes, row = min(t, a.T - 1);
    const __half* src = a.qkv + row * a.row_stride + 8 * c;
    auto load = [&](int h) { return __builtin_nontemporal_load(reinterpret_cast<const v4i*>(src + (int64_t)h * D)); };
    v4i raw = load(head);
    const int64_t slot = a.slots[row];
    const bool live = t < a.T && slot >= 0 && slot < a.cache.n_pages << a.cache.log2_page;
    if (__builtin_amdgcn_ballot_w64(live) == 0) return;
    __half* const q_row = a.q_out + row * a.n_heads * D + 8 * c;
    // head 0's place in the cache; a head further on lies a page further
    const int64_t token0 = (((slot >> a.cache.log2_page) * a.cache.n_kv_heads) << a.cache.log2_page) + (slot & ((1ll << a.cache.log2_page) - 1));

    Lane ln;
    Turn rope = kNone;
    if (a.cos_sin != nullptr && head < a.n_heads + a.cache.n_kv_heads) {
        const int half = a.rotary_dim / 2;
        const int64_t position = min(max((int64_t)a.positions[row], (int64_t)0), a.max_positions - 1);
        const float* cs = a.cos_sin + position * a.rotary_dim;
        const bool turns = ln.turns = 8 * c < a.rotary_dim;
        ln.partner = lane;
        if (a.interleaved) {
            rope = kPairs;
            const float4 x = *reinterpret_cast<const float4*>(cs + (turns ? 4 * c : 0)), y = *reinterpret_cast<const float4*>(cs + half + (turns ? 4 * c : 0));
            const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ln.cs[2 * i] = ln.cs[2 * i + 1] = xs[i];
                ln.sn[2 * i] = -ys[i];
                ln.sn[2 * i + 1] = ys[i];
            }
        } else {
            rope = a.rotary_dim == D ? kHalfHead : kHalves;
            const bool first = 8 * c < half;
            const int at = turns ? (first ? 8 * c : 8 * c - half) : 0;
            if (turns) ln.partner = first ? lane + half / 8 : lane - half / 8;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const float4 x = *reinterpret_cast<const float4*>(cs + at + i), y = *reinterpret_cast<const float4*>(cs + half + at + i);
                const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    ln.cs[i + k] = xs[k];
                    ln.sn[i + k] = first ? -ys[k] : ys[k];
                }
            }
        }
    }
    if constexpr (!MANY) {
        const uint64_t found = append_head<LOG2_D, LOG2_GROUP, ROTATE>(a, ln, rope, raw, head, q_row, token0, live, true, lane);
        if (found != 0) append_exact<LOG2_D, LOG2_GROUP, ROTATE>(a, ln, rope, head, token0, found, lane);
        return;
    }
    __shared__ uint64_t suspects[kStride][kMany];                   // of each wavefront's own
    const int first_head = head, wave = threadIdx.x >> 6, end = min(heads, head + kStride * each);
    uint32_t asked = 0;
#pragma unroll 1
    for (int j = 0;; ++j) {
        const v4i now = raw;
        if (head + kStride < end) raw = load(head + kStride);
        const uint64_t found = append_head<LOG2_D, LOG2_GROUP, ROTATE>(a, ln, rope, now, head, q_row, token0, live, j == 0, lane);
        if (found != 0) {
            asked |= 1u << j;
            suspects[wave][j] = found;
        }
        head += kStride;
        if (head >= end) break;
    }
#pragma unroll 1
    for (; asked != 0; asked &= asked - 1) {
        const int j = __builtin_ctz(asked);
        const int again = first_head + j * kStride;
        halves_to_floats(load(again), ln.x);
        // (what derives from these is computed here, and not once in front of the loop, where it would hold twice their registers)
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(ln.cs[i]), "+v"(ln.sn[i]));
        append_exact<LOG2_D, LOG2_GROUP, ROTATE>(a, ln, rope, again, token0, suspects[wave][j], lane);
    }
}

template <int LOG2_D, int LOG2_GROUP, bool ROTATE>
int launch(const AppendArgs& a, hipStream_t st)
{
    constexpr int kTokens = 64 / ((1 << LOG2_D) / 8);
    const int64_t blocks = (a.T + kTokens - 1) / kTokens;
    const int heads = a.n_heads + 2 * a.cache.n_kv_heads;
    // Eight heads to a wavefront once one to each would be more than about two wavefronts to every place on the card (5 to 8 a SIMD, 1024
    // SIMDs).  One | eight, us: 48 heads of 128, static steps, 200 tokens 5.0 | 7.8, 1000 (12000 wavefronts) 10.1 | 12.5, 2000 15.2 | 16.5, 8192
    // 50 | 46, 16000 99 | 85; 80 heads with dynamic steps and norms: 512 tokens (10240) 10.8 | 13.1, 800 13.8 | 15.4, 1000 17.0 | 16.5, 8000
    // 97 | 74; 48 heads of 64: 2000 tokens (12000) 9.5 | 11.9, 8000 26.2 | 26.2.  (The border is the lowest of any kind's: static steps without
    // norms gain from about 40000 wavefronts on and lose up to a tenth between.)  With twelve a step of 64 tokens takes twice as long.
    const bool many = blocks * heads > 12288;
    const int each = 4 * (many ? kMany : 1);                             // heads of a workgroup
    const dim3 grid((unsigned)blocks, (unsigned)((heads + each - 1) / each));
    if (many) k_kv4_append<LOG2_D, LOG2_GROUP, ROTATE, true><<<grid, kThreads, 0, st>>>(a);
    else k_kv4_append<LOG2_D, LOG2_GROUP, ROTATE, false><<<grid, kThreads, 0, st>>>(a);
    return hip_status(hipGetLastError());
}

template <int LOG2_D, int LOG2_GROUP>
int launch(const AppendArgs& a, bool rotate, hipStream_t st)
{
    return rotate ? launch<LOG2_D, LOG2_GROUP, true>(a, st) : launch<LOG2_D, LOG2_GROUP, false>(a, st);
}

}  // namespace

int launch_append(const AppendArgs& a, int32_t head_dim, int32_t group, bool rotate, hipStream_t st)
{
    if (head_dim == 64) {
        if (group == 0) return launch<6, 0>(a, rotate, st);
        if (group == 32) return launch<6, 5>(a, rotate, st);
        return launch<6, 6>(a, rotate, st);
    }
    if (group == 0) return launch<7, 0>(a, rotate, st);
    if (group == 32) return launch<7, 5>(a, rotate, st);
    if (group == 64) return launch<7, 6>(a, rotate, st);
    return launch<7, 7>(a, rotate, st);
}

}  // namespace kv4
}  // namespace pq
