// The plan of the masked attention kernels for many rows (make_plan), and the way of their workgroups through its list, on the CPU: one fiber to a
// thread of the workgroup, which goes on when all have come to a barrier.  HIP source, its host side alone; nothing is launched.
//
// For each case: no list is written behind its end, every entry that a workgroup asks for is one that was listed, and all units of the listed tiles,
// for every head, are taken once.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <ucontext.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <random>
#include <vector>

namespace group {
struct Index { int x, y, z; };
int threads, now;
Index index() { return {now, 0, 0}; }
std::vector<ucontext_t> fibers;
std::vector<std::vector<char>> stacks;
std::vector<int64_t> said;
std::vector<bool> done;
ucontext_t outside;
std::function<void()> body;

void barrier() { swapcontext(&fibers[now], &outside); }
int64_t shuffle_up(int64_t v, int d, int width)
{
    said[now] = v;
    barrier();
    const int64_t x = now % width >= d ? said[now - d] : v;
    barrier();
    return x;
}
void enter()
{
    body();
    done[now] = true;
    swapcontext(&fibers[now], &outside);
}
void run(int n, std::function<void()> f)
{
    threads = n;
    body = std::move(f);
    fibers.resize(n);
    stacks.resize(n);
    said.assign(n, 0);
    done.assign(n, false);
    for (int t = 0; t < n; ++t) {
        stacks[t].resize(32768);
        getcontext(&fibers[t]);
        fibers[t].uc_stack.ss_sp = stacks[t].data();
        fibers[t].uc_stack.ss_size = stacks[t].size();
        fibers[t].uc_link = nullptr;
        makecontext(&fibers[t], enter, 0);
    }
    while (true) {
        int ended = 0;
        for (now = 0; now < n; ++now) {
            if (!done[now]) swapcontext(&outside, &fibers[now]);
            ended += done[now];
        }
        if (ended == n) return;
        if (ended != 0) {
            std::puts("some threads ended in front of a barrier of the others");
            std::exit(1);
        }
    }
}
}  // namespace group

#undef __device__
#undef __shared__
#define __device__ __attribute__((host)) __attribute__((device))
#define __shared__ static
#define threadIdx group::index()
#define __syncthreads group::barrier
#define __shfl_up group::shuffle_up
using std::max;
using std::min;
#include "../paper_2410_05265_amd/csrc/pq_kv4_attention_plan.h"
#undef threadIdx

using namespace pq::kv4;

namespace {

std::string_view what;
bool fail(const char* why, long long a = 0, long long b = 0)
{
    std::printf("%.*s: %s (%lld, %lld)\n", (int)what.size(), what.data(), why, a, b);
    return false;
}

template <typename T> struct List {
    std::vector<T> all;
    size_t n;
    explicit List(size_t count) : all(count + 64), n(count) { std::memset((void*)all.data(), 0x5A, all.size() * sizeof(T)); }
    bool kept() const
    {
        const char* const at = reinterpret_cast<const char*>(all.data() + n);
        return std::all_of(at, at + 64 * sizeof(T), [](char c) { return c == 0x5A; });
    }
};

struct Case {
    std::vector<int32_t> cu, kv;
    int T, Hkv, per_kv, table_pages, log2_page, words, window, sinks, small_rows, runs;
};

template <int THREADS> bool check(const Case& c)
{
    const int B = (int)c.kv.size();
    AttentionArgs a = {};
    a.T = c.T;
    a.n_heads = c.Hkv * c.per_kv;
    a.heads_per_kv = c.per_kv;
    a.cu_q = c.cu.data();
    a.kv_len = c.kv.data();
    a.B = B;
    a.table_pages = c.table_pages;
    a.cache.n_kv_heads = c.Hkv;
    a.cache.log2_page = c.log2_page;
    a.cache.n_pages = 1000;
    a.causal = 1;
    a.tree = c.words ? reinterpret_cast<const uint32_t*>(&a) : nullptr;        // (the plan reads no masks)
    a.words = c.words;
    a.window = c.window;
    a.sinks = c.sinks;
    const int64_t most = masked_tiles_at_most(c.T, B, c.per_kv, c.small_rows);
    List<Start> starts(kMostRuns);
    List<Cut> cuts(kMostRuns);
    List<RowTile> tiles(most);
    List<int64_t> units_before(most > kFewestPlanThreads ? most + 1 : 0);
    List<int32_t> tiles_before(B > kFewestPlanThreads ? B + 1 : 0);
    const RunPlan p = {starts.all.data(), cuts.all.data(), tiles.all.data(), units_before.all.data(), tiles_before.all.data(), nullptr, (int)most};
    group::run(THREADS, [&] { make_plan<THREADS>(a, p, c.runs, c.small_rows); });
    if (!starts.kept() || !cuts.kept() || !tiles.kept() || !units_before.kept() || !tiles_before.kept()) return fail("a list is written behind its end");

    int64_t all = 0, units = 0;
    for (int b = 0; b < B; ++b) all += row_tiles_of(a, request(a, b), c.small_rows);
    const int listed = (int)std::min(all, most);
    std::vector<int64_t> taken((size_t)listed * c.Hkv, 0);
    for (int t = 0; t < listed; ++t) {
        const RowTile& x = tiles.all[t];
        if (x.b < 0 || x.b >= B || x.tile < 0 || (int64_t)x.tile * kTileRows >= (int64_t)x.r.q_len * c.per_kv) return fail("no tile of rows", t, x.tile);
        if (x.r.start < 0 || x.r.start + x.r.q_len > c.T) return fail("rows that there are not", t, x.r.start);
        units += (int64_t)units_of(x.steps) * c.Hkv;
    }
    int64_t total = 0;
    for (int run = 0; run < c.runs; ++run) {
        Start at = starts.all[run];
        if (at.tile < 0) continue;
        while (at.length > 0) {
            if (at.tile < 0 || at.tile >= listed || at.head < 0 || at.head >= c.Hkv) return fail("an entry that was not listed", at.tile, listed);
            const RowTile& x = tiles.all[at.tile];
            const int take = (int)std::min((int64_t)(units_of(x.steps) - at.unit), at.length);
            if (take <= 0) return fail("a run that does not go on", run, at.unit);
            taken[(size_t)at.tile * c.Hkv + at.head] += take;
            total += take;
            walk_on(at, x, take, c.Hkv);
        }
    }
    if (total != units) return fail("units that no run has, or two", total, units);
    for (int t = 0; t < listed; ++t)
        for (int h = 0; h < c.Hkv; ++h)
            if (taken[(size_t)t * c.Hkv + h] != units_of(tiles.all[t].steps)) return fail("a tile that is not taken whole", t, h);
    return true;
}

bool both(const Case& c) { return check<256>(c) && check<1024>(c); }

}  // namespace

int main()
{
    bool ok = true;
    auto with = [&](std::string_view name, std::vector<int32_t> cu, int T, int per_kv, int Hkv) {
        what = name;
        Case c = {cu, std::vector<int32_t>(cu.size() - 1, 9000), T, Hkv, per_kv, 200, 6, 0, 1000, 4, 0, 256};
        for (int small_rows : {0, 104, 192})
            for (int words : {0, 8})
                for (int runs : {256, 512}) {
                    c.small_rows = small_rows;
                    c.words = words;
                    c.runs = runs;
                    ok = both(c) && ok;
                }
    };
    with("one prompt", {0, 6400}, 6400, 4, 8);
    with("prompts", {0, 1000, 1000, 1300, 6400}, 6400, 4, 8);
    with("more rows than the call has", {0, 1000, 7000, 9000}, 6400, 4, 8);
    with("the same rows twice", {0, 6400, 0, 6400}, 6400, 4, 8);
    with("the same rows twice, few heads", {0, 1000, 0, 1000}, 1000, 4, 8);
    with("rows many times over", {0, 3000, 5, 2900, 17, 3000, 0, 3000, 2990, 3000}, 3000, 1, 3);
    with("rows in front of the first", {-5000, 300, -7, 1000, 40, 600}, 1000, 8, 1);
    for (int B : {255, 256, 257, 1023, 1024, 1025}) {                              // the lists' two places
        what = "many requests";
        Case c = {{0}, {}, 0, 2, 1, 200, 4, 1, 70, 3, 104, 512};
        std::mt19937 rng(B);
        for (int b = 0; b < B; ++b) {
            const int q = b % 3 == 0 ? rng() % 3 : 105 + rng() % 300;
            c.cu.push_back(c.cu.back() + q);
            c.kv.push_back(q + rng() % 500);
        }
        c.T = c.cu.back() - 7;
        ok = both(c) && ok;
    }
    what = "any cu_q";
    for (int seed = 0; seed < 300; ++seed) {
        std::mt19937 rng(seed);
        const int B = 1 + rng() % 12, T = 1 + rng() % (seed % 2 ? 600 : 20000);
        Case c = {{}, {}, T, (int)(1 + rng() % 8), (int)(1 + rng() % 8), (int)(1 + rng() % 300), (int)(4 + rng() % 4), (int)(rng() % 9),
                  (int)(1 + rng() % (seed % 3 ? 300 : 1 << 30)), (int)(rng() % 200), seed % 5 == 0 ? 0 : seed % 5 == 1 ? 192 : 104, seed % 4 ? 256 : 512};
        for (int b = 0; b <= B; ++b) c.cu.push_back((int32_t)(rng() % (2 * T)) - T / 4);
        if (seed % 7 == 0) std::sort(c.cu.begin(), c.cu.end());
        for (int b = 0; b < B; ++b) c.kv.push_back(rng() % 9 == 0 ? INT32_MAX - (int)(rng() % 3) : (int32_t)(rng() % 30000) - 100);
        ok = (seed % 16 ? check<256>(c) : both(c)) && ok;
    }
    if (ok) std::puts("kv4_plan_walk: ok");
    return ok ? 0 : 1;
}
