// Codes of accepted tokens to their places, in all layers of a model: token after token, every head's D / 2 bytes of keys and of values, and
// with dynamic steps D / group floats of each.
//
// A wavefront takes one request in one layer, all its heads or some of them.  Its entries stay in their order: what an entry reads is read
// before it, or one behind it, is written, so an entry may write where an earlier one read (the way of accepted tokens, which only move
// forward).  It is bound by memory, by the number of pieces rather than their bytes.
#include "pq_kv4.h"

namespace pq {
namespace kv4 {
namespace {

constexpr int kMostLayers = 96;          // of a launch: their addresses are its arguments
constexpr int kMostWidth = 256;

// Heads are shared out to wavefronts of their own until there are this many: with 8 heads in 80 layers one request's 64 entries 9.5 -> 5.6 us,
// 256 of them with 4 steps each 46 -> 11; 16 requests with 32 heads in 32 layers 17.2 -> 10.8.  48 requests with 6 entries in 80 layers:
// 16.1 us for 368 640 pieces of 64 bytes and their steps, read and written, nearly each in a line of its own.
constexpr int kWavefronts = 4096;
constexpr int kMostHeads = 1 << 16;      // of a wavefront: what it has to move is counted in 32 bits, 256 entries of up to four pieces each

struct Layers {
    struct {
        uint8_t* codes[2];
        float* steps[2];
    } of[kMostLayers];
};

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// NG: steps of a token and head, 0 if they are static.
template <int D, int NG>
__global__ __launch_bounds__(64) void k_kv4_keep(Layers layers, const int64_t* __restrict__ from_slots, const int64_t* __restrict__ to_slots, int B, int width,
                                                 int64_t n_slots, int n_kv_heads, int heads, int log2_page)
{
    __shared__ int64_t from_s[kMostWidth], to_s[kMostWidth];       // places of the entries that move, in tokens of head 0
    const int lane = threadIdx.x;
    constexpr int kPieces = D / 32;                                // 16 bytes of a token's codes
    for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
        int count = 0;
        for (int i0 = 0; i0 < width; i0 += 64) {
            const int i = i0 + lane;
            const int64_t from = i < width ? from_slots[b * width + i] : -1, to = i < width ? to_slots[b * width + i] : -1;
            const bool moves = from >= 0 && from < n_slots && to >= 0 && to < n_slots && from != to;
            const uint64_t all = __builtin_amdgcn_ballot_w64(moves);
            const int64_t in = (1ll << log2_page) - 1;
            if (moves) {
                const int at = count + __builtin_popcountll(all & ((1ull << lane) - 1));
                from_s[at] = (((from >> log2_page) * n_kv_heads) << log2_page) + (from & in);
                to_s[at] = (((to >> log2_page) * n_kv_heads) << log2_page) + (to & in);
            }
            count += __builtin_popcountll(all);
        }
        __syncthreads();
        const auto& layer = layers.of[blockIdx.y];
        const int head0 = (int)blockIdx.z * heads, n_heads = min(heads, n_kv_heads - head0);
        // head after head, in each entry after entry, its pieces
        const int pieces = count * kPieces;
        for (int x = lane; x < pieces * n_heads; x += 64) {
            const int head = head0 + x / pieces, entry = x % pieces / kPieces, piece = x % kPieces;
            const int64_t shift = (int64_t)head << log2_page, from = (from_s[entry] + shift) * (D / 2) + 16 * piece, to = (to_s[entry] + shift) * (D / 2) + 16 * piece;
            const v4u k = *reinterpret_cast<const v4u*>(layer.codes[0] + from), v = *reinterpret_cast<const v4u*>(layer.codes[1] + from);
            asm volatile("" ::: "memory");
            *reinterpret_cast<v4u*>(layer.codes[0] + to) = k;
            *reinterpret_cast<v4u*>(layer.codes[1] + to) = v;
        }
        if constexpr (NG > 0) {
            const int steps = count * NG;
            for (int x = lane; x < steps * n_heads; x += 64) {
                const int head = head0 + x / steps, entry = x % steps / NG, g = x % NG;
                const int64_t shift = (int64_t)head << log2_page, from = (from_s[entry] + shift) * NG + g, to = (to_s[entry] + shift) * NG + g;
                const float k = layer.steps[0][from], v = layer.steps[1][from];
                asm volatile("" ::: "memory");
                layer.steps[0][to] = k;
                layer.steps[1][to] = v;
            }
        }
        __syncthreads();
    }
}

template <int D, int NG>
void launch(const Layers& layers, int n, const int64_t* from_slots, const int64_t* to_slots, int32_t B, int32_t width, const pq_kv4_cache& c, hipStream_t st)
{
    const int groups = B < 1 << 16 ? B : 1 << 16;
    const int64_t parts = kWavefronts / ((int64_t)groups * n);
    const int shared = parts < 2 ? c.n_kv_heads : parts >= c.n_kv_heads ? 1 : (int)((c.n_kv_heads + parts - 1) / parts);
    const int heads = shared < kMostHeads ? shared : kMostHeads;
    k_kv4_keep<D, NG><<<dim3((unsigned)groups, (unsigned)n, (unsigned)(((int64_t)c.n_kv_heads + heads - 1) / heads)), 64, 0, st>>>(
        layers, from_slots, to_slots, B, width, c.n_pages * c.page_size, c.n_kv_heads, heads, __builtin_ctz((unsigned)c.page_size));
}

}  // namespace

int launch_keep(const int64_t* from_slots, const int64_t* to_slots, int32_t B, int32_t width, const pq_kv4_cache* caches, int32_t n_caches, hipStream_t st)
{
    for (int32_t first = 0; first < n_caches; first += kMostLayers) {
        const int n = n_caches - first < kMostLayers ? n_caches - first : kMostLayers;
        Layers layers = {};
        for (int i = 0; i < n; ++i) {
            const pq_kv4_cache& c = caches[first + i];
            layers.of[i] = {{static_cast<uint8_t*>(c.k_codes), static_cast<uint8_t*>(c.v_codes)}, {c.k_scale, c.v_scale}};
        }
        const pq_kv4_cache& c = caches[0];
        const int ng = c.group ? c.head_dim / c.group : 0;
        if (c.head_dim == 64) (ng == 0 ? launch<64, 0> : ng == 1 ? launch<64, 1> : launch<64, 2>)(layers, n, from_slots, to_slots, B, width, c, st);
        else (ng == 0 ? launch<128, 0> : ng == 1 ? launch<128, 1> : ng == 2 ? launch<128, 2> : launch<128, 4>)(layers, n, from_slots, to_slots, B, width, c, st);
        if (const int rc = hip_status(hipGetLastError()); rc != PQ_OK) return rc;
    }
    return PQ_OK;
}

}  // namespace kv4
}  // namespace pq
