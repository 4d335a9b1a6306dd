// What the masked attention kernels for many rows are told before they start: the tiles of rows, and where each workgroup's run begins.
#pragma once
#include "pq_kv4_attention.h"

namespace pq {
namespace kv4 {

constexpr int kPlanStep = 64;            // tokens of a step

__device__ __forceinline__ int row_tiles_of(const AttentionArgs& a, const Request& r, int small_rows)
{
    const int64_t rows = (int64_t)r.q_len * a.heads_per_kv;
    return rows <= small_rows ? 0 : (int)((rows + kTileRows - 1) / kTileRows);
}

// ---- The masked variant's work is cut into runs.  What a tile of rows sees differs more there (windows, trees beside prompts), and so do the
// requests: all steps of the call, request after request, in each head after head and tile of rows after tile, lie one after another, and every
// workgroup takes an equal run of them, whatever the lengths are (a chiplet's workgroups read neighbouring rows' tokens of one head: with the
// heads inside the tiles the codes missed its L2, prompts took 1.4 times as long).  A tile and head that a run covers whole is written as it is;
// of one that is cut, the workgroups leave partial sums (at most two each), and a second kernel adds them.  The tiles and where the runs begin are
// listed by one workgroup in front: planned by every workgroup for itself they cost 40 us of code that is run once and has to come from memory.
// Alone that is a launch of 7 us; where the row kernel runs too, its second kernel has the workgroup beside it (32 trees of up to 64 nodes over up
// to 6001 tokens 167 -> 161 us, 8 trees beside a prompt 117 -> 108).

// A run is counted in units: a tile and head has one for every step and kTileUnits in front, for what it takes beside its steps (queries, prefix,
// results; without them a run of many short tiles took up to 1.3 times as long as one of few long ones).
constexpr int kTileUnits = 5;

// A tile of rows: `steps` of 64 tokens (0: it sees nothing), of which those from Tiles::front on lie `gap` further.
struct RowTile {
    int b, tile, of, steps, gap;         // of: tiles of the request, as far as they are listed
    Request r;
};
__device__ __forceinline__ int units_of(int steps) { return kTileUnits + max(steps, 1); }
// Of a workgroup, its first unit: of a tile and head; tile < 0: it has none.
struct Start {
    int tile, head, unit, unused;
    int64_t length, each;        // units of the run, and of one that is not the last
};
// A tile that was cut, by the workgroup that began it: `parts` workgroups from it on have some of it (0: none was).
struct Cut {
    int parts, start, rows, head, row0, unused[3];
};
constexpr int kMostRuns = 512, kFewestUnits = 7;

// A run goes on to the tile and head behind `t`, of whose units it has taken `take`: the request's next tile, or its first one of the next head.
__device__ __forceinline__ void walk_on(Start& run, const RowTile& t, int take, int n_kv_heads)
{
    run.length -= take;
    run.unit = 0;
    ++run.tile;
    if (t.tile + 1 == t.of && run.head + 1 < n_kv_heads) {
        ++run.head;
        run.tile -= t.of;
    } else if (t.tile + 1 == t.of) {
        run.head = 0;
    }
}

// Tiles of requests of more than small_rows rows, at most: 256 rows of one at least, or the rows of a smaller one.
inline int64_t masked_tiles_at_most(int64_t T, int32_t B, int32_t per_kv, int small_rows)
{
    const int64_t rows = T * per_kv, by_requests = rows / kTileRows + B, fewest = small_rows + 1 < (kTileRows + 1) / 2 ? small_rows + 1 : (kTileRows + 1) / 2;
    const int64_t by_rows = rows / fewest + 1;
    return by_requests < by_rows ? by_requests : by_rows;
}

// Scratch memory of the masked variant.
struct RunPlan {
    Start* starts;               // [kMostRuns]
    Cut* cuts;                   // [kMostRuns]
    RowTile* tiles;              // [most_tiles]
    int64_t* units_before;       // [most_tiles + 1], of one head
    int32_t* tiles_before;       // [B + 1], of each request
    float* partial;              // two places for each run
    int most_tiles;
};
struct TilePlan {
    RunPlan plan;
    int runs;
};
// Of a call, with its scratch memory at `ws`; the tile kernel and what joins its parts, with the plan in front unless it is `made`.
TilePlan plan_of(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, void* ws);
int launch_masked_tiles(const AttentionArgs& a, int32_t head_dim, int32_t group, int small_rows, const TilePlan& plan, bool made, hipStream_t st);
constexpr int kFewestPlanThreads = 256;            // of the workgroups that make plans: lists for more entries are in scratch memory

// Inclusive sum over the workgroup; `all`: the sum.
template <int THREADS> __device__ __forceinline__ int64_t sum_up(int64_t v, int64_t* sums, int tid, int64_t& all)
{
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(v, d, 64);
        if (lane >= d) v += x;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    all = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) v += sums[w];
        all += sums[w];
    }
    return v;
}
// The last place whose entry is at most x.
template <typename T> __device__ __forceinline__ int place_in(const T* list, int n, int64_t x)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (list[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Tiles of rows and starts of runs, by one workgroup.
template <int THREADS> __device__ __forceinline__ void make_plan(const AttentionArgs& a, const RunPlan& p, int runs, int small_rows)
{
    static_assert(THREADS >= kFewestPlanThreads, "lists");
    __shared__ int64_t sums[THREADS / 64], few_units[THREADS + 1];
    __shared__ int32_t few_tiles[THREADS + 1];
    const int tid = threadIdx.x, Hkv = a.cache.n_kv_heads, per_kv = a.heads_per_kv;
    int32_t* const tiles_before = a.B <= THREADS ? few_tiles : p.tiles_before;
    const int each = (a.B + THREADS - 1) / THREADS, first = min(tid * each, a.B), last = min(first + each, a.B);
    int64_t own = 0, all;
    for (int b = first; b < last; ++b) own += row_tiles_of(a, request(a, b), small_rows);
    int64_t at = sum_up<THREADS>(own, sums, tid, all) - own;
    for (int b = first; b < last; ++b) {
        tiles_before[b] = (int32_t)min(at, (int64_t)INT32_MAX);
        if (last - first > 1) at += row_tiles_of(a, request(a, b), small_rows);
    }
    // (only rows that lie in two requests, from a cu_q that does not ascend, make more than there are places: then the last ones are in no list)
    const int tiles = (int)min(all, (int64_t)p.most_tiles);
    int64_t* const units_before = tiles <= THREADS ? few_units : p.units_before;
    __syncthreads();
    int64_t total = 0;
    for (int t0 = 0; t0 < tiles; t0 += THREADS) {
        const int t = t0 + tid;
        int64_t units = 0, sum;
        if (t < tiles) {
            // (the last of the requests that begin there: those in front of it have no tiles)
            const int b = place_in(tiles_before, a.B, t);
            const Request r = request(a, b);
            const int tile = t - tiles_before[b], row0 = tile * kTileRows;
            const Seen seen = masked_rows(a, r, row0 / per_kv, min((row0 + kTileRows - 1) / per_kv, r.q_len - 1));
            const Tiles<kPlanStep> left(a, seen.lo);
            const int count = left.count(seen.any);
            p.tiles[t] = {b, tile, min(row_tiles_of(a, r, small_rows), tiles - tiles_before[b]), count, left.gap, r};
            units = units_of(count);
        }
        const int64_t incl = sum_up<THREADS>(units, sums, tid, sum);
        if (t < tiles) units_before[t] = total + incl - units;
        total += sum;
    }
    if (tid == 0) units_before[tiles] = total;
    __syncthreads();
    const int64_t units = total * Hkv, length = max((units + runs - 1) / runs, (int64_t)kFewestUnits);
    for (int run = tid; run < runs; run += THREADS) {
        p.cuts[run].parts = 0;
        const int64_t begin = length * run;
        Start s = {-1, 0, 0, 0, min(length, units - begin), length};
        if (begin < units) {
            int lo = 0, hi = a.B - 1;                  // the request
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (units_before[min(tiles_before[mid], tiles)] * Hkv <= begin) lo = mid;
                else hi = mid - 1;
            }
            const int first_tile = tiles_before[lo], end_tile = lo + 1 < a.B ? min(tiles_before[lo + 1], tiles) : tiles;
            const int64_t base = units_before[first_tile], one = units_before[end_tile] - base, in = begin - base * Hkv;
            s.head = (int)(in / one);
            const int64_t at_unit = base + in - s.head * one;
            s.tile = first_tile + place_in(units_before + first_tile, end_tile - first_tile, at_unit);
            s.unit = (int)(at_unit - units_before[s.tile]);
        }
        p.starts[run] = s;
    }
}

}  // namespace kv4
}  // namespace pq
