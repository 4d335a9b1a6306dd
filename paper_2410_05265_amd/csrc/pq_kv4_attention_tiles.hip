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
#include "pq_kv4_attention_plan.h"

#define PQ_INLINE __attribute__((always_inline))

namespace pq {
namespace kv4 {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kThreads = 512, kWaves = 8;
constexpr int kRows = kTileRows, kCols = 32;      // rows of a workgroup and of a wavefront
constexpr int kTile = 64;                         // tokens of a step
static_assert(kTile == kPlanStep, "units");
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
    return row_tiles_of(a, r, small_rows);
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

// Runs: a workgroup to a CU, two where registers let two run there (64 channels, static steps; 9 registers are spilled then).  One | two, us, 32 heads on
// 8: 2 prompts of up to 6000, window 1024 182 | 170, 4 of 4000, window 512 179 | 163, 8 chunks of 500 behind 3500, window 1024 80 | 72, one of 12000,
// window 4096 503 | 462; 32 trees of 64 over up to 6000 130 | 125, 64 of 40 over up to 3000 136 | 121, 16 of 64 over 20000 261 | 243.  Where there is
// little for them all, two lose: one prompt of 600, window 256 32 | 39, one tree of 64 over 8000 with 64 heads 44 | 52.
template <int D, bool DYNAMIC> constexpr int kRuns = D == 64 && !DYNAMIC ? 512 : 256;

// What the kernels are given beside the call's arguments: scratch memory, and how it is used.
template <typename... KIND> struct Work {
    float* partial;
    const int32_t* starts;       // tiles before each request, null: not listed
    int splits, small_rows;
};
template <> struct Work<Masked> {
    RunPlan plan;
};
struct PlainParts { float* partial; const int32_t* starts; int splits, small_rows; };
struct MaskedParts { float* partial; const Start* starts; int splits, small_rows; };
__device__ __forceinline__ PlainParts parts_of(const Work<>& w) { return {w.partial, w.starts, w.splits, w.small_rows}; }
__device__ __forceinline__ MaskedParts parts_of(const Work<Masked>& w) { return {w.plan.partial, w.plan.starts, 0, 0}; }
__device__ __forceinline__ Cut* cuts_of(const Work<>&) { return nullptr; }
__device__ __forceinline__ Cut* cuts_of(const Work<Masked>& w) { return w.plan.cuts; }
__device__ __forceinline__ const RowTile* tiles_of(const Work<>&) { return nullptr; }
__device__ __forceinline__ const RowTile* tiles_of(const Work<Masked>& w) { return w.plan.tiles; }

// What lies there, as scalars: where a branch goes by it, and barriers stand behind the branch, the wavefronts go whole.
// (Words of 64-bit members and pointers: as `int` the compiler might take them for other memory than the members that were written.)
typedef int word_of_any __attribute__((may_alias));
template <typename T> __device__ __forceinline__ T for_all(const T* from)
{
    T v;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i)
        reinterpret_cast<word_of_any*>(&v)[i] = __builtin_amdgcn_readfirstlane(reinterpret_cast<const word_of_any*>(from)[i]);
    return v;
}

constexpr int kPlanThreads = 1024;       // (alone; beside the row kernel's second one it has that one's)
__global__ __launch_bounds__(kPlanThreads) void k_kv4_attention_plan(AttentionArgs a, RunPlan p, int runs, int small_rows)
{
    make_plan<kPlanThreads>(a, p, runs, small_rows);
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
template <int D, int G, bool DYNAMIC, typename... KIND>
__global__ __launch_bounds__(kThreads, D == 64 && !DYNAMIC ? 4 : 2) void k_kv4_attention_tiles(AttentionArgs given, Work<KIND...> work)
{
    constexpr bool MASKED = sizeof...(KIND) > 0;
    [[maybe_unused]] const auto [partial, starts, splits, small_rows] = parts_of(work);
    constexpr int NG = D / G, KS = D / 16, KSG = G / 16, DB = D / 32, DBG = G / 32;
    extern __shared__ __align__(256) uint8_t raw_lds[];
    typedef Lds<D, G, DYNAMIC> L;
    L& sh = *reinterpret_cast<L*>(raw_lds);
    const int worker = MASKED ? xcd_run(blockIdx.x, gridDim.x) : 0;
    [[maybe_unused]] Cut* const cuts = cuts_of(work);
    [[maybe_unused]] const RowTile* const row_tiles = tiles_of(work);
    // Codes on their way run from one tile of rows into the next: where the steps of the one and the other find theirs.
    struct Source {
        const int32_t* table;
        int head, n, gap, unused;
    };
    // What a wavefront keeps from tile to tile.  It lies in LDS, for each of its own: the compiler orders loads and products by the registers that are
    // left, and with this in scalar ones it read every operand right in front of its product (a step of 2.1 us took 2.5).
    struct Held {
        Start run;
        RowTile tile;            // what comes then
        Source now, then;
    };
    __shared__ Held held_by[kWaves];
    if constexpr (MASKED) {
        Held& held = held_by[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
        const Start run = for_all(starts + worker);
        if (run.tile < 0) return;
        held.run = run;
        held.tile = for_all(row_tiles + run.tile);
    }
    struct Codes { v4u w; float s; int bad, left; };               // left: tokens from the tile's first on
    Codes next;
    int page = 0, first_buf = 0;
    bool primed = false, ahead = false;
    while (true) {
    // (read anew for every tile of rows: kept, the arguments alone take half of the scalar registers)
    auto arguments = [&]() PQ_INLINE -> const AttentionArgs& {
        if constexpr (!MASKED) return given;
        uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(at));
        return *(const AttentionArgs*)(const __attribute__((address_space(4))) AttentionArgs*)at;
    };
    const AttentionArgs& a = arguments();
    const int log2_page = a.cache.log2_page, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv, left_front = MASKED ? Tiles<kTile>(a, 0).front : 0;
    int tid = threadIdx.x;
    if constexpr (MASKED) asm volatile("" : "+v"(tid));            // (what comes from it is not kept from one tile to the next: registers)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    int head = blockIdx.x % Hkv, split = MASKED ? 0 : (blockIdx.x / Hkv) % splits, begin, end;
    const int64_t index = MASKED ? 0 : blockIdx.x / Hkv / splits;
    bool cut = MASKED ? false : splits > 1;        // its sums go through scratch memory
    Where at;
    int more_units = 0, next_index = 0, next_head = 0, gap = 0;
    Held& held = held_by[wave];
    if constexpr (MASKED) {
        Start run = for_all(&held.run);
        const RowTile row_tile = for_all(&held.tile);
        if (run.length <= 0) return;
        if (!primed) __syncthreads();              // (nobody reads the last tile's operands any more)
        at = {row_tile.b, row_tile.tile, row_tile.r};
        head = run.head;
        const int units = units_of(row_tile.steps), take = (int)min((int64_t)(units - run.unit), run.length), last = run.unit + take;
        if (last <= kTileUnits) return;            // (the run ends in front of its first step)
        begin = max(run.unit - kTileUnits, 0);
        end = min(last - kTileUnits, row_tile.steps);
        cut = begin > 0 || last < units;
        split = begin;
        held.now = {a.table + (int64_t)at.b * a.table_pages, head, at.r.n, row_tile.gap, 0};
        if (begin == 0 && cut && tid == 0) {
            int parts = 1;
            for (int64_t left = units - last; left > 0; left -= run.each) ++parts;
            cuts[worker] = {parts, at.r.start, at.r.q_len * per_kv, head, at.tile * kRows, {0, 0, 0}};
        }
        walk_on(run, row_tile, take, Hkv);
        held.run = run;
        more_units = (int)min(run.length, (int64_t)kTileUnits + 1);
        next_index = run.tile;
        next_head = run.head;
        gap = row_tile.gap;
    } else {
        at = find_tile(a, index, small_rows, starts, lane);
        if (at.b < 0) return;
    }
    const Request r = at.r;
    const int rows = r.q_len * per_kv, row0 = at.tile * kRows;
    const bool tree = MASKED && is_tree(a, r);
    const bool live = !MASKED || row0 + wave * kCols < rows;      // some of the wavefront's rows are there
    if constexpr (!MASKED) {
        const int last_token = min((row0 + kRows - 1) / per_kv, r.q_len - 1);
        const int visible = __builtin_amdgcn_readfirstlane(sees(a, r, last_token));    // (a division leaves it in a vector register)
        const int all_tiles = (visible + kTile - 1) / kTile;
        begin = (int)((int64_t)all_tiles * split / splits);
        end = (int)((int64_t)all_tiles * (split + 1) / splits);
    }

    // this lane's query
    int limit, wave_sees;                    // tokens that it sees, and that all of the wavefront's see
    int hidden = 0, wave_hidden = 0, row_token;    // a window: those before it that are no sinks it does not see, and some of the wavefront's do not
    v8h q[KS];
    float c0 = 0.0f;                         // -8 sum(q): the codes' offset (dynamic steps: the operands are without it)
    {
        const int row = min(row0 + wave * kCols + col, rows - 1);
        const int token = row / per_kv, q_head = head * per_kv + row % per_kv;
        row_token = token;
        if constexpr (MASKED) {
            const Row see = masked_row(a, r, token);
            const Seen wave_rows = masked_rows(a, r, min(row0 + wave * kCols, rows - 1) / per_kv, min(row0 + wave * kCols + kCols - 1, rows - 1) / per_kv);
            limit = see.limit;
            hidden = see.lo;
            wave_sees = __builtin_amdgcn_readfirstlane(wave_rows.all);
            wave_hidden = __builtin_amdgcn_readfirstlane(wave_rows.lo_top);
        } else {
            limit = sees(a, r, token);
            wave_sees = __builtin_amdgcn_readfirstlane(sees(a, r, min(row0 + wave * kCols, rows - 1) / per_kv));
        }
        const __half* src = a.q + (int64_t)(r.start + token) * a.row_stride + (int64_t)q_head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const v8h*>(src + 16 * s + 8 * half);
    }
    // What a tile of rows needs beside the steps is asked for at once: queries, prefix tokens, pages, the tile that comes then.  One after another
    // these waits took as long as two steps.
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

    // ---- the history: wavefronts w and w + 4 load and expand keys and values of tokens 16 w .. 16 w + 15 of every tile
    const int block = wave & 3;
    const bool keys = wave < 4;
    auto fetch = [&](int64_t first, Codes& x) PQ_INLINE {          // 16 tokens from this one of the head's on
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
    const int32_t* const table = a.table + (int64_t)at.b * a.table_pages;
    auto page_of = [&](int tile) PQ_INLINE { return table[min((tile * kTile + 16 * block) >> log2_page, a.table_pages - 1)]; };
    auto load = [&](int tile, int page, Codes& x) PQ_INLINE {
        const int t = tile * kTile + 16 * block;
        x.bad = (uint32_t)page >= (uint64_t)a.cache.n_pages || (t >> log2_page) >= a.table_pages;
        x.left = r.n - tile * kTile;
        const int64_t from = x.bad ? 0 : page;
        fetch(((from * Hkv + head) << log2_page) + (t & ((1 << log2_page) - 1)), x);
    };
    // MASKED: step i is tile i, or lies behind the gap; steps from `end` on are the next item's first two.  64 pages are looked up at once, and a lane
    // read where one is used.  (A page carried from step to step through the outer loop was waited for at once, and what is computed for every step
    // is kept short: twice the scalar instructions made a step of 2.1 us 2.6.)
    int load_tile = 0, ids_from = 0;               // the last tile that is on its way; slots of pages from ids_from on, and which are none
    int64_t slots = 0;
    uint64_t none = 0;
    int then_page = 0;                             // lanes 0 and 1: of the next item's first two steps
    auto tile_of = [&](int step, int gap) PQ_INLINE { return step + (step >= left_front ? gap : 0); };
    auto page_at = [&](int tile) PQ_INLINE { return (tile * kTile + 16 * block) >> log2_page; };
    auto look_up = [&](int from, int page, int head) PQ_INLINE {
        const int at = from + lane;
        const bool bad = (uint32_t)page >= (uint64_t)a.cache.n_pages || at >= a.table_pages;
        slots = ((int64_t)(bad ? 0 : page) * Hkv + head) << log2_page;
        none = __builtin_amdgcn_ballot_w64(bad);
        ids_from = from;
    };
    auto load_step = [&](int i, Codes& x) PQ_INLINE {
        const int in = (1 << log2_page) - 1;
        if (i >= end) {
            if (!ahead) return;                    // (nothing comes then)
            const Source then = for_all(&held.then);
            const int tile = tile_of(i - end, then.gap), page = __builtin_amdgcn_readlane(then_page, i - end);
            x.bad = (uint32_t)page >= (uint64_t)a.cache.n_pages || page_at(tile) >= a.table_pages;
            x.left = then.n - tile * kTile;
            fetch(((int64_t)((x.bad ? 0 : page) * (int64_t)Hkv + then.head) << log2_page) + ((tile * kTile + 16 * block) & in), x);
            return;
        }
        load_tile = i == left_front ? i + gap : load_tile + 1;
        const int at = page_at(load_tile);
        if ((uint32_t)(at - ids_from) >= 64) {
            const Source now = for_all(&held.now);
            look_up(at, now.table[min(at + lane, a.table_pages - 1)], now.head);
        }
        x.bad = (int)(none >> (at - ids_from)) & 1;
        x.left = r.n - load_tile * kTile;
        const uint32_t low = __builtin_amdgcn_readlane((int)(uint32_t)slots, at - ids_from), high = __builtin_amdgcn_readlane((int)(slots >> 32), at - ids_from);
        fetch((int64_t)((uint64_t)high << 32 | low) + ((load_tile * kTile + 16 * block) & in), x);
    };
    auto expand = [&](int buf, const Codes& x) PQ_INLINE {
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
                const float step = t < x.left && !x.bad ? finite_step(x.s) : 0.0f;
                float most = step;
#pragma unroll
                for (int d = 4; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
                if ((lane & 3) < NG) sh.vs[buf][lane & 3][t] = step;
                if (lane < NG) sh.vs_most[buf][lane][block] = most;
            }
        }
    };

    if constexpr (MASKED) {
        load_tile = tile_of(begin + (primed ? 1 : 0), gap) - (primed ? 0 : 1);
        const int from = max(page_at(load_tile), 0), page = begin < end ? table[min(from + lane, a.table_pages - 1)] : 0;
        RowTile next_tile = {};
        if (more_units > 0) next_tile = for_all(row_tiles + next_index);
        held.tile = next_tile;
        look_up(from, page, head);
        // the last steps load the first two of the next tile's
        ahead = end - begin >= 2 && more_units > kTileUnits && next_tile.steps > 0;
        if (begin < end && !primed) load_step(begin, next);
        if (ahead) {
            const int32_t* const then_table = a.table + (int64_t)next_tile.b * a.table_pages;
            held.then = {then_table, next_head, next_tile.r.n, next_tile.gap, 0};
            then_page = then_table[min(page_at(tile_of(lane & 1, next_tile.gap)), a.table_pages - 1)];
        }
    } else if (begin < end) {                      // (on their way while the queries are and the prefix tokens are taken)
        load(begin, page_of(begin), next);
        page = page_of(begin + 1);
    }


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
    const int spare = MASKED && primed ? first_buf ^ 1 : 0;       // (the other one holds the first tile)
    if (prefix) {
        for (int t0 = 0; t0 < a.n_prefix; t0 += kPrefixTile) {
            __syncthreads();
            if (prefix_t < kPrefixTile) {
                const int t = prefix_t, in16 = t & 15;             // token t of its 16: 8 (t / 8) + 4 (half of the lanes) + t % 4
                sh.k[spare][t][prefix_c] = __builtin_bit_cast(v4u, in_key_order(prefix_k));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __half* dst = reinterpret_cast<__half*>(&sh.v[spare][t >> 4][(in16 >> 2) & 1][place_of<G>(8 * prefix_c + j)][in16 >> 3]);
                    dst[in16 & 3] = reinterpret_cast<const __half*>(&prefix_v)[j];
                }
            }
            if constexpr (DYNAMIC) {
                if (tid < kPrefixTile) {
#pragma unroll
                    for (int g = 0; g < NG; ++g) sh.ks[DYNAMIC ? spare : 0][g][tid] = 1.0f;
                }
            }
            if (t0 + kPrefixTile < a.n_prefix) load_prefix(t0 + kPrefixTile);
            __syncthreads();
            float x[kPrefixTile / 2];
            v4u p[kPrefixTile / 16];
            if (MASKED && !live) continue;
            scores(spare, x);
            const int left = a.n_prefix - t0 - 4 * half;
#pragma unroll
            for (int i = 0; i < kPrefixTile / 2; ++i)
                if (8 * (i >> 2) + (i & 3) >= left) x[i] = -INFINITY;
            probabilities(x, scale, 0.0f, p);
            multiply(spare, 0, DB, p);
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
        if constexpr (!MASKED) {
            expand(0, next);
            load(begin + 1, page, next);
            page = page_of(begin + 2);
        } else if (!primed) {
            first_buf = 0;
            expand(0, next);
            load_step(begin + 1, next);
        }
        int tile = MASKED ? tile_of(begin, gap) - 1 : begin - 1;
        auto history = [&](auto live_rows) PQ_INLINE {
        constexpr bool LIVE = decltype(live_rows)::value;          // (else the wavefront only loads and expands for the others)
        for (int i = begin; i < end; ++i) {
            const int buf = (MASKED ? first_buf + i - begin : i - begin) & 1;
            __syncthreads();                       // tile i is in LDS; nobody reads tile i - 1 any more
            const int page_after = MASKED ? 0 : page_of(i + 3);
            tile = MASKED && i == left_front ? i + gap : tile + 1;
            const int t0 = tile * kTile;
            float x[32];
            v4u p[4];
            if constexpr (LIVE) scores(buf, x);
            expand(buf ^ 1, next);
            if constexpr (MASKED) load_step(i + 2, next);
            else load(i + 2, page, next);
            page = page_after;
            if constexpr (!LIVE) continue;
            // what rows do not see, or has no page
            if (t0 + kTile > wave_sees || (MASKED && t0 < wave_hidden && t0 + kTile > a.sinks) ||
                __builtin_amdgcn_readfirstlane(sh.bad[buf][0] | sh.bad[buf][1] | sh.bad[buf][2] | sh.bad[buf][3]) != 0) {
                const int left = limit - (t0 + 4 * half);
                if constexpr (MASKED) {            // a bit for each of 64 tokens from this lane's first on (a branch for every score took 2 us)
                    auto below = [](int n) PQ_INLINE -> uint64_t { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; };
                    uint64_t see = below(left) & (~below(hidden - (t0 + 4 * half)) | below(a.sinks - (t0 + 4 * half)));
                    if (tree && t0 + kTile > wave_sees) {          // nodes of its mask, behind the limit
                        const uint32_t low = mask_bits(a, r, row_token, t0 - (r.sees - 1)), high = mask_bits(a, r, row_token, t0 + 32 - (r.sees - 1));
                        see |= (((uint64_t)high << 32 | low) >> (4 * half)) & ~below(left);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (sh.bad[buf][k]) see &= ~(0xFFFFull << (16 * k));
                    const uint32_t see_low = (uint32_t)see, see_high = (uint32_t)(see >> 32);
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = ((j < 16 ? see_low : see_high) >> ((8 * (j >> 2) + (j & 3)) & 31)) & 1 ? x[j] : -INFINITY;
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (8 * (j >> 2) + (j & 3) >= left || sh.bad[buf][j >> 3]) x[j] = -INFINITY;
                }
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
        };
        if constexpr (MASKED) {
            if (live) history(std::true_type{});
            else history(std::false_type{});
            first_buf = (first_buf + end - begin) & 1;
            primed = ahead;
        } else {
            history(std::true_type{});
        }
    } else if constexpr (MASKED) {
        primed = false;
    }

    // ---- results
    const float l_all = l + __shfl_xor(l, 32, 64);
    float times[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) times[g] = kUnit * (DYNAMIC ? ref[g] : v_step);
    if (cut) {
        // [slot][row of the accumulators, maximum, sum][256 rows]: neighbouring lanes write neighbouring floats
        if (MASKED && !live) continue;
        float* dst = partial + (MASKED ? 2 * worker + (split == 0 ? 1 : 0) : (index * Hkv + head) * splits + split) * (int64_t)(D + 2) * kRows + wave * kCols + col;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                dst[(32 * d + 8 * (i >> 2) + 4 * half + (i & 3)) * kRows] = o[d][i] * times[d / DBG];
        if (half == 0) {
            dst[D * kRows] = m;
            dst[(D + 1) * kRows] = l_all;
        }
        if constexpr (MASKED) continue;
        return;
    }
    if constexpr (!MASKED) __syncthreads();
    __half* const lines = reinterpret_cast<__half*>(raw_lds + (MASKED ? sizeof(L) : 0)) + wave * kCols * (D + 8);      // (the next tile's operands may be there)
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
    if constexpr (!MASKED) return;
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

// The same for the tiles that runs have cut: a workgroup takes 64 rows and 64 channels of one, a thread 16 channels of a row.  The loads of four
// parts are on their way at once (one after another, and 32 channels to a thread: 10 tiles of rows x 8 heads in four parts each 32 us).
template <int D, int G>
__global__ __launch_bounds__(kJoinThreads) void k_kv4_attention_join_runs(AttentionArgs a, RunPlan p)
{
    constexpr int kAtOnce = 4, kChannels = 16;
    const Cut cut = p.cuts[blockIdx.x];
    const int lane = threadIdx.x & 63, in_tile = blockIdx.y * 64 + lane, row = cut.row0 + in_tile;
    if (cut.parts <= 0 || cut.row0 + (int)blockIdx.y * 64 >= cut.rows) return;
    const int channel0 = blockIdx.z * 64 + kChannels * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // part 0 lies at its workgroup's second place, the others at the first of theirs
    const int64_t size = (int64_t)(D + 2) * kRows;
    const float* const first = p.partial + blockIdx.x * 2 * size + in_tile;
    float top = kNothing, sum = 0.0f, acc[kChannels] = {};
    for (int s0 = 0; s0 < cut.parts; s0 += kAtOnce) {
        float m[kAtOnce], l[kAtOnce], x[kAtOnce][kChannels];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int s = min(s0 + k, cut.parts - 1);
            const float* const src = first + (2 * s + (s == 0 ? 1 : 0)) * size;
            m[k] = src[D * kRows];
            l[k] = src[(D + 1) * kRows];
            if (s0 + k >= cut.parts) l[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < kChannels; ++i) x[k][i] = src[place_of<G>(channel0 + i) * kRows];
        }
        float to = top;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) to = fmaxf(to, m[k]);
        const float old = __builtin_amdgcn_exp2f(top - to);
        top = to;
        sum *= old;
#pragma unroll
        for (int i = 0; i < kChannels; ++i) acc[i] *= old;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float f = s0 + k < cut.parts ? __builtin_amdgcn_exp2f(m[k] - to) : 0.0f;
            sum = fmaf(l[k], f, sum);
#pragma unroll
            for (int i = 0; i < kChannels; ++i) acc[i] = fmaf(x[k][i], f, acc[i]);
        }
    }
    if (row >= cut.rows) return;
    const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
    __half* const dst = a.out + ((int64_t)(cut.start + row / a.heads_per_kv) * a.n_heads + cut.head * a.heads_per_kv + row % a.heads_per_kv) * D + channel0;
#pragma unroll
    for (int i = 0; i < kChannels; i += 8) {
        v4u w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = two_halves(acc[i + 2 * j] * f, acc[i + 2 * j + 1] * f);
        *reinterpret_cast<v4u*>(dst + i) = w;
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

template <int D, int G, bool DYNAMIC, typename... KIND>
int launch(const AttentionArgs& a, int64_t groups, const Work<KIND...>& work, hipStream_t st)
{
    static std::atomic<uint64_t> allowed{0};
    const size_t out = (size_t)kWaves * kCols * (D + 8) * 2, in = sizeof(Lds<D, G, DYNAMIC>), lds = sizeof...(KIND) > 0 ? in + out : in > out ? in : out;
    const auto kernel = k_kv4_attention_tiles<D, G, DYNAMIC, KIND...>;
    if (const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, allowed); rc != PQ_OK) return rc;
    kernel<<<(unsigned)groups, kThreads, lds, st>>>(a, work);
    return hip_status(hipGetLastError());
}

template <int D, int G, bool DYNAMIC>
int launch_plain(const AttentionArgs& a, int64_t groups, const Work<>& work, hipStream_t st)
{
    if (const int rc = launch<D, G, DYNAMIC>(a, groups * work.splits, work, st); rc != PQ_OK) return rc;
    if (work.splits > 1)
        k_kv4_attention_join_tiles<D, G><<<dim3((unsigned)groups, kRows / 64), kJoinThreads, 0, st>>>(a, work.partial, work.starts, work.splits, work.small_rows);
    return hip_status(hipGetLastError());
}

template <int D, int G, bool DYNAMIC>
int launch_masked(const AttentionArgs& a, const Work<Masked>& work, hipStream_t st)
{
    constexpr int runs = kRuns<D, DYNAMIC>;
    if (const int rc = launch<D, G, DYNAMIC, Masked>(a, runs, work, st); rc != PQ_OK) return rc;
    k_kv4_attention_join_runs<D, G><<<dim3(runs, kRows / 64, D / 64), kJoinThreads, 0, st>>>(a, work.plan);
    return hip_status(hipGetLastError());
}

// Scratch memory: partial sums, then the list of starts.
size_t tiles_partial_bytes(int64_t tiles, int splits, int32_t n_kv_heads, int32_t head_dim)
{
    return splits > 1 ? (size_t)(tiles * n_kv_heads * splits) * kRows * (head_dim + 2) * sizeof(float) : 0;
}

size_t up_to_256(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
// The masked variant's scratch memory, at `ws`; its size.
size_t lay_out(RunPlan* p, void* ws, int64_t most_tiles, int32_t B, int32_t head_dim)
{
    uint8_t* const base = static_cast<uint8_t*>(ws);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up_to_256(bytes);
        return base + here;
    };
    p->starts = reinterpret_cast<Start*>(take(kMostRuns * sizeof(Start)));
    p->cuts = reinterpret_cast<Cut*>(take(kMostRuns * sizeof(Cut)));
    p->tiles = reinterpret_cast<RowTile*>(take((size_t)most_tiles * sizeof(RowTile)));
    p->units_before = reinterpret_cast<int64_t*>(take(most_tiles > kFewestPlanThreads ? (size_t)(most_tiles + 1) * sizeof(int64_t) : 0));
    p->tiles_before = reinterpret_cast<int32_t*>(take(B > kFewestPlanThreads ? (size_t)(B + 1) * sizeof(int32_t) : 0));
    p->partial = reinterpret_cast<float*>(take((size_t)(head_dim == 64 ? kMostRuns : 256) * 2 * kRows * (head_dim + 2) * sizeof(float)));
    p->most_tiles = (int)most_tiles;
    return at;
}

}  // namespace

size_t masked_tiles_workspace_bytes(int64_t T, int32_t B, int32_t per_kv, int32_t head_dim, int small_rows)
{
    RunPlan p;
    return lay_out(&p, nullptr, masked_tiles_at_most(T, B, per_kv, small_rows), B, head_dim);
}

TilePlan plan_of(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, void* ws)
{
    TilePlan t;
    lay_out(&t.plan, ws, masked_tiles_at_most(a.T, a.B, a.heads_per_kv, small_rows), a.B, head_dim);
    t.runs = head_dim == 128 ? kRuns<128, false> : group == 0 ? kRuns<64, false> : kRuns<64, true>;
    return t;
}

int launch_masked_tiles(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, const TilePlan& plan, bool made, hipStream_t st)
{
    if (!made) {
        k_kv4_attention_plan<<<1, kPlanThreads, 0, st>>>(a, plan.plan, plan.runs, small_rows);
        if (const int rc = hip_status(hipGetLastError()); rc != PQ_OK) return rc;
    }
    const Work<Masked> w = {plan.plan};
    if (head_dim == 64) {
        if (group == 0) return launch_masked<64, 64, false>(a, w, st);
        if (group == 32) return launch_masked<64, 32, true>(a, w, st);
        return launch_masked<64, 64, true>(a, w, st);
    }
    if (group == 0) return launch_masked<128, 128, false>(a, w, st);
    if (group == 32) return launch_masked<128, 32, true>(a, w, st);
    if (group == 64) return launch_masked<128, 64, true>(a, w, st);
    return launch_masked<128, 128, true>(a, w, st);
}

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
    const int64_t groups = tiles * a.cache.n_kv_heads;
    const Work<> w = {partial, starts, splits, small_rows};
    if (head_dim == 64) {
        if (group == 0) return launch_plain<64, 64, false>(a, groups, w, st);
        if (group == 32) return launch_plain<64, 32, true>(a, groups, w, st);
        return launch_plain<64, 64, true>(a, groups, w, st);
    }
    if (group == 0) return launch_plain<128, 128, false>(a, groups, w, st);
    if (group == 32) return launch_plain<128, 32, true>(a, groups, w, st);
    if (group == 64) return launch_plain<128, 64, true>(a, groups, w, st);
    return launch_plain<128, 128, true>(a, groups, w, st);
}

}  // namespace kv4
}  // namespace pq
