// Trees of drafted tokens: masks and positions from parents, and the walk along the branch that the model's own choices follow.
//
//     A(i) = {i} + A(parent of i)   (a root's: {i}),    mask of row i = the set A(i),    position = offset + c + |A(i)| - 1,
//
// c tokens of the request lying in front of its rows.  A few kilobytes: what counts are launches and the loads that wait for one another.  A
// wavefront takes a request; its parents lie in LDS, where every lane walks from its own nodes up to their roots.  One tree of 26 nodes 2.6 us, 250
// of up to 64 beside 6 prompts 4.2; the walk through those 4.5, and 3.7 for their pages.
#include "pq_kv4.h"

namespace pq {
namespace kv4 {
namespace {

constexpr int kNodesOfLane = kMostNodes / 64, kMostWords = kMostNodes / 32;
constexpr int kMostGroups = 1 << 16;

// A request's rows, those below T of them, and the tokens in front of them.
struct Rows {
    int start, count;
    int64_t before;
};

__device__ __forceinline__ Rows rows_of(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ kv_len, int b, int T)
{
    const int64_t begin = cu_q[b], end = max((int64_t)cu_q[b + 1], begin), from = min(max(begin, (int64_t)0), (int64_t)T), to = min(max(end, from), (int64_t)T);
    return {(int)from, (int)(to - from), max((int64_t)max(kv_len[b], 0) - (end - begin), (int64_t)0)};
}

__device__ __forceinline__ int32_t saturate(int64_t v) { return (int32_t)min(v, (int64_t)INT32_MAX); }

__global__ __launch_bounds__(64) void k_kv4_tree(const int32_t* __restrict__ parents, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ kv_len,
                                                 int B, int T, int words, int position_offset, uint32_t* __restrict__ mask, int32_t* __restrict__ positions)
{
    __shared__ int parent_s[kMostNodes];
    const int lane = threadIdx.x, slice = blockIdx.y * 64 + lane, threads = gridDim.y * 64;
    auto no_row = [&](int64_t t) {
        positions[t] = 0;
        for (int w = 0; w < words; ++w) mask[t * words + w] = 0;
    };
    for (int b = blockIdx.x; b <= B; b += gridDim.x) {
        if (b == B) {                              // rows of no request
            const int64_t first = B > 0 ? min(max(cu_q[0], 0), T) : T, last = B > 0 ? max(cu_q[B], 0) : 0;
            for (int64_t t = slice; t < first; t += threads) no_row(t);
            for (int64_t t = last + slice; t < T; t += threads) no_row(t);
            break;
        }
        const Rows r = rows_of(cu_q, kv_len, b, T);
        if (r.count > 32 * words) {                // a prompt
            for (int64_t i = slice; i < r.count; i += threads) {
                const int64_t t = r.start + i;
                positions[t] = saturate(position_offset + r.before + i);
                for (int w = 0; w < words; ++w) mask[t * words + w] = 0;
            }
            continue;
        }
        if (blockIdx.y != 0) continue;
        for (int i = lane; i < r.count; i += 64) {
            const int p = parents[r.start + i];
            parent_s[i] = p >= 0 && p < i ? p : -1;
        }
        __syncthreads();
        for (int i = lane; i < r.count; i += 64) {
            uint32_t m[kMostWords] = {};
            int nodes = 0;
            for (int at = i; at >= 0; at = parent_s[at]) {         // (a parent lies in front: it ends)
#pragma unroll
                for (int w = 0; w < kMostWords; ++w) m[w] |= at >> 5 == w ? 1u << (at & 31) : 0u;
                ++nodes;
            }
            const int64_t t = r.start + i;
            positions[t] = saturate(position_offset + r.before + nodes - 1);
#pragma unroll
            for (int w = 0; w < kMostWords; ++w)
                if (w < words) mask[t * words + w] = m[w];
        }
        __syncthreads();                           // (read before the next request takes their place)
    }
}

// The walk of one request, by one wavefront:  node 0, then of the node that was accepted last the lowest child whose token the model chose there.
struct Walk {
    int chosen[kMostNodes], path[kMostNodes];
};

__device__ __forceinline__ int64_t slot_of(const AcceptArgs& a, int b, int64_t token)
{
    const int64_t col = token >> a.log2_page;
    const int page = col < a.table_pages ? a.table[(int64_t)b * a.table_pages + col] : -1;
    return page >= 0 ? ((int64_t)page << a.log2_page) + (token & ((1 << a.log2_page) - 1)) : -1;
}

__device__ __forceinline__ void walk(const AcceptArgs& a, int b, Walk& s, int lane)
{
    const Rows r = rows_of(a.cu_q, a.kv_len, b, a.T);
    int kept = r.count, next = -1, found = 0;
    if (r.count > 32 * a.words) {                  // a prompt stays whole
        next = a.chosen[r.start + r.count - 1];
    } else if (r.count > 0) {
        int parent[kNodesOfLane], token[kNodesOfLane];
#pragma unroll
        for (int k = 0; k < kNodesOfLane; ++k) {
            const int i = 64 * k + lane;
            parent[k] = token[k] = -1;
            if (i < r.count) {
                parent[k] = a.parents[r.start + i];
                token[k] = a.tokens[r.start + i];
                s.chosen[i] = a.chosen[r.start + i];
            }
            if (parent[k] >= i) parent[k] = -1;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (one wavefront: what its lanes wrote is there)
        int at = 0;
        while (true) {
            next = __builtin_amdgcn_readfirstlane(s.chosen[at]);
            if (lane == 0) s.path[found] = at;
            if (++found >= a.depth) break;
            int child = -1;
#pragma unroll
            for (int k = kNodesOfLane - 1; k >= 0; --k) {
                const uint64_t fits = __builtin_amdgcn_ballot_w64(parent[k] == at && token[k] == next);
                if (fits != 0) child = 64 * k + __builtin_ctzll(fits);
            }
            if (child < 0) break;
            at = child;
        }
        kept = found;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    if (lane == 0) {
        a.accepted[b] = kept;
        a.next_token[b] = next;
        a.kv_len_out[b] = saturate(r.before + kept);
    }
    for (int i = lane; i < a.depth; i += 64) {
        const int node = i < found ? s.path[i] : -1;
        int64_t from = -1, to = -1;
        if (node >= 0 && node != i) {
            from = slot_of(a, b, r.before + node);
            to = slot_of(a, b, r.before + i);
            if (from < 0 || to < 0) from = to = -1;
        }
        const int64_t place = (int64_t)b * a.depth + i;
        a.path[place] = node;
        a.from_slots[place] = from;
        a.to_slots[place] = to;
    }
}

// Pages behind what the requests keep, back to the free list: with r of them and `top` pages of the list given out, the k-th goes to place
// top - 1 - k and top - r stay given out.  One workgroup, a request to a thread.
constexpr int kBackThreads = 1024;
__device__ __forceinline__ void give_back(const AcceptArgs& a, int64_t* sums)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int top = a.n_free > 0 ? min(max(*a.taken, 0), a.n_free) : 0;
    const int mask = (1 << a.log2_page) - 1;
    int64_t given = 0;
    for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
        const int b = b0 + tid;
        int from = 0, to = 0;
        int64_t own = 0;
        const int32_t* row = a.table;
        if (b < a.B) {
            row = a.table + (int64_t)b * a.table_pages;
            from = (int)min(((int64_t)a.kv_len_out[b] + mask) >> a.log2_page, (int64_t)a.table_pages);
            to = (int)min(((int64_t)max(a.kv_len[b], 0) + mask) >> a.log2_page, (int64_t)a.table_pages);
            for (int c = from; c < to; ++c) own += row[c] >= 0;
        }
        int64_t incl = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t v = __shfl_up(incl, d, 64);
            if (lane >= d) incl += v;
        }
        if (lane == 63) sums[wave] = incl;
        __syncthreads();
        int64_t k = given + incl - own;
        for (int w = 0; w < waves; ++w) {
            if (w < wave) k += sums[w];
            given += sums[w];
        }
        for (int c = from; c < to; ++c) {
            if (row[c] < 0) continue;
            if (k < top) a.free_pages[top - 1 - k] = row[c];
            ++k;
        }
        __syncthreads();
    }
    if (tid == 0) *a.taken_out = (int)max((int64_t)top - given, (int64_t)0);
}

__global__ __launch_bounds__(64) void k_kv4_accept(AcceptArgs a)
{
    __shared__ Walk s;
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) walk(a, b, s, threadIdx.x);
}

__global__ __launch_bounds__(kBackThreads) void k_kv4_give_back(AcceptArgs a)
{
    __shared__ int64_t sums[kBackThreads / 64];
    give_back(a, sums);
}

// Both in one launch while one workgroup's 16 wavefronts do for all walks: one request's 26 nodes 8.6 -> 5.5 us, 24 of 64 nodes 11.0 -> 8.0;
// at 48 both take 10, at 128 the one workgroup 22 and the two launches 10.  (32 of 256 nodes: 13.2 against 12.)
constexpr int kFewRequests = 24;
__global__ __launch_bounds__(kBackThreads) void k_kv4_accept_few(AcceptArgs a)
{
    __shared__ Walk s[kBackThreads / 64];
    __shared__ int64_t sums[kBackThreads / 64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int b = wave; b < a.B; b += kBackThreads / 64) walk(a, b, s[wave], threadIdx.x & 63);
    __threadfence_block();
    __syncthreads();                               // (lengths that other wavefronts wrote)
    give_back(a, sums);
}

}  // namespace

int launch_tree(const int32_t* parents, const int32_t* cu_q, const int32_t* kv_len, int32_t B, int32_t T, int32_t words, int32_t position_offset,
                uint32_t* mask, int32_t* positions, hipStream_t st)
{
    const int groups = B + 1 < kMostGroups ? B + 1 : kMostGroups;
    // prompts and padding: about four rows to a thread
    int64_t slices = ((int64_t)T / groups + 255) / 256;
    const int64_t most = groups < 2048 ? 2048 / groups : 1;
    slices = slices < 1 ? 1 : slices > most ? most : slices;
    k_kv4_tree<<<dim3((unsigned)groups, (unsigned)slices), 64, 0, st>>>(parents, cu_q, kv_len, B, T, words, position_offset, mask, positions);
    return hip_status(hipGetLastError());
}

int launch_accept(const AcceptArgs& a, hipStream_t st)
{
    if (a.B <= kFewRequests) {
        k_kv4_accept_few<<<1, kBackThreads, 0, st>>>(a);
        return hip_status(hipGetLastError());
    }
    k_kv4_accept<<<a.B < kMostGroups ? a.B : kMostGroups, 64, 0, st>>>(a);
    k_kv4_give_back<<<1, kBackThreads, 0, st>>>(a);
    return hip_status(hipGetLastError());
}

}  // namespace kv4
}  // namespace pq
