// Block table, slots and positions of a step's new tokens, from the requests' lengths.
//
//     before_b = min(W, ceil(kv_b / ps)),  after_b = min(W, ceil((kv_b + q_b) / ps)),  need_b = after_b - before_b,
//     first_b  = taken + sum of need over the requests before b,
//     table[b, before_b + i] = free_pages[first_b + i]           (-1 past the end of the list)
//     cu_q[b]  = sum of q over the requests before b,
//     token cu_q[b] + i:  position = offset + kv_b + i,  slot = table[b, (kv_b + i) / ps] * ps + (kv_b + i) % ps  (-1 without a page).
//
// A few kilobytes to a few megabytes: what counts is that it is one launch (3 us for 64 decoded tokens, 7 for 1500 requests with some
// 150000 tokens, 1.9 MB: two dependent rounds of loads and a launch).  Every workgroup sums the requests before its own itself
// (two integers of each, from the caches), then places its own by scans of one wavefront, kChunk at a time, and its threads walk over
// their tokens as one sequence.  blockIdx.y divides that sequence: one long prompt is written by many workgroups.  There are no more than
// kMostGroups workgroups along the requests, so that what they read in front of their own stays in proportion to the requests: beyond
// 16 * kMostGroups of them each takes several chunks.
// No workgroup reads what another writes: pages given out in this call are looked up in the free list, not in the table.
#include "pq_kv4.h"

namespace pq {
namespace kv4 {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 16;       // requests that a workgroup places at a time
constexpr int kMostGroups = 2048;

struct Request {
    int64_t kv, q;
    int32_t before, need;
};

__device__ __forceinline__ Request request(const int32_t* kv_len, const int32_t* q_len, int b, int W, int log2_page)
{
    Request r;
    r.kv = max(kv_len[b], 0);
    r.q = max(q_len[b], 0);
    const int64_t mask = (1ll << log2_page) - 1;
    const int64_t before = (r.kv + mask) >> log2_page, after = (r.kv + r.q + mask) >> log2_page;
    r.before = (int32_t)min(before, (int64_t)W);
    r.need = (int32_t)min(after, (int64_t)W) - r.before;
    return r;
}

__device__ __forceinline__ int32_t saturate(int64_t v) { return (int32_t)min(v, (int64_t)INT32_MAX); }

__global__ __launch_bounds__(kThreads) void k_kv4_slots(const int32_t* __restrict__ kv_len, const int32_t* __restrict__ q_len, int B,
                                                        int32_t* table, int W, const int32_t* __restrict__ free_pages, int n_free,
                                                        const int32_t* taken, int log2_page, int T, int position_offset, int32_t* cu_q,
                                                        int32_t* kv_len_out, int32_t* positions, int64_t* slots, int32_t* taken_out, int chunks)
{
    __shared__ int64_t wave_q[kThreads / 64], wave_need[kThreads / 64];
    __shared__ int64_t start_s[kChunk + 1], first_s[kChunk];       // of the workgroup's requests: cu_q and place in the free list
    __shared__ int64_t kv_s[kChunk];
    __shared__ int32_t before_s[kChunk], need_s[kChunk];
    const int tid = threadIdx.x, lane = tid & 63;
    const int own_first = blockIdx.x * chunks * kChunk, own_end = min(own_first + chunks * kChunk, B);

    int64_t q_sum = 0, need_sum = 0;
    for (int b = tid; b < own_first; b += kThreads) {
        const Request r = request(kv_len, q_len, b, W, log2_page);
        q_sum += r.q;
        need_sum += r.need;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        q_sum += __shfl_xor(q_sum, d, 64);
        need_sum += __shfl_xor(need_sum, d, 64);
    }
    if (lane == 0) {
        wave_q[tid >> 6] = q_sum;
        wave_need[tid >> 6] = need_sum;
    }
    __syncthreads();
    int64_t start = 0, first = 0;                                  // of the next chunk, in the first wavefront
    if (tid < 64) {
        first = taken ? *taken : 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            start += wave_q[w];
            first += wave_need[w];
        }
    }
    const int slice = blockIdx.y * kThreads + tid, threads = gridDim.y * kThreads;
    for (int b0 = own_first;; b0 += kChunk) {
        const int own = min(kChunk, own_end - b0);                 // (none if there are no requests)
        if (tid < 64) {
            Request r = {0, 0, 0, 0};
            if (lane < own) r = request(kv_len, q_len, b0 + lane, W, log2_page);
            int64_t q_incl = r.q, need_incl = r.need;
#pragma unroll
            for (int d = 1; d < kChunk; d <<= 1) {
                const int64_t a = __shfl_up(q_incl, d, 64), c = __shfl_up(need_incl, d, 64);
                if (lane >= d) {
                    q_incl += a;
                    need_incl += c;
                }
            }
            if (lane < kChunk) {
                start_s[lane] = start + q_incl - r.q;
                first_s[lane] = first + need_incl - r.need;
                kv_s[lane] = r.kv;
                before_s[lane] = r.before;
                need_s[lane] = r.need;
                if (lane == kChunk - 1) start_s[kChunk] = start + q_incl;
            }
            if (lane < own && blockIdx.y == 0) {
                cu_q[b0 + lane] = saturate(start + q_incl - r.q);
                kv_len_out[b0 + lane] = saturate(r.kv + r.q);
            }
            if (lane == kChunk - 1 && blockIdx.y == 0 && b0 + own == B) {
                cu_q[B] = saturate(start + q_incl);
                *taken_out = saturate(first + need_incl);
            }
            start += __shfl(q_incl, kChunk - 1, 64);
            first += __shfl(need_incl, kChunk - 1, 64);
        }
        __syncthreads();

        // new entries of the table: one wavefront to a request
        for (int j = slice >> 6; j < own; j += threads >> 6) {
            const int64_t from = first_s[j];
            for (int i = lane; i < need_s[j]; i += 64) {
                const int64_t at = from + i;
                table[(int64_t)(b0 + j) * W + before_s[j] + i] = at >= 0 && at < n_free ? free_pages[at] : -1;
            }
        }
        // tokens
        const int64_t begin = start_s[0], end = min(start_s[kChunk], (int64_t)T);
        for (int64_t t = begin + slice; t < end; t += threads) {
            int j = 0;
#pragma unroll
            for (int d = kChunk / 2; d >= 1; d >>= 1) j += start_s[j + d] <= t ? d : 0;
            const int64_t at = kv_s[j] + t - start_s[j], col = at >> log2_page;
            int64_t page = -1;
            if (col < before_s[j]) {
                page = table[(int64_t)(b0 + j) * W + col];
            } else if (col < before_s[j] + need_s[j]) {
                const int64_t i = first_s[j] + col - before_s[j];
                if (i >= 0 && i < n_free) page = free_pages[i];
            }
            positions[t] = saturate(position_offset + at);
            slots[t] = page >= 0 ? (page << log2_page) + (at & ((1ll << log2_page) - 1)) : -1;
        }
        // rows behind the last request
        if (b0 + own == B) {
            for (int64_t t = start_s[kChunk] + slice; t < T; t += threads) {
                positions[t] = 0;
                slots[t] = -1;
            }
        }
        if (b0 + kChunk >= own_end) break;
        __syncthreads();                                           // (read before the next chunk takes their place)
    }
}

}  // namespace

int launch_slots(const int32_t* kv_len, const int32_t* q_len, int32_t B, int32_t* block_table, int32_t table_pages,
                 const int32_t* free_pages, int32_t n_free, const int32_t* taken, int32_t log2_page, int32_t T, int32_t position_offset,
                 int32_t* cu_q, int32_t* kv_len_out, int32_t* positions, int64_t* slots, int32_t* taken_out, hipStream_t st)
{
    const int all = B > 0 ? (B + kChunk - 1) / kChunk : 1, chunks = (all + kMostGroups - 1) / kMostGroups, groups = (all + chunks - 1) / chunks;
    // about four tokens to a thread, and no more than eight workgroups to a CU in all
    const int64_t per_group = ((int64_t)T + groups - 1) / groups;
    int64_t slices = (per_group + 4 * kThreads - 1) / (4 * kThreads), most = kMostGroups / groups;
    if (most < 1) most = 1;
    if (slices < 1) slices = 1;
    if (slices > most) slices = most;
    k_kv4_slots<<<dim3((unsigned)groups, (unsigned)slices), kThreads, 0, st>>>(kv_len, q_len, B, block_table, table_pages, free_pages, n_free,
                                                                               taken, log2_page, T, position_offset, cu_q, kv_len_out, positions,
                                                                               slots, taken_out, chunks);
    return hip_status(hipGetLastError());
}

}  // namespace kv4
}  // namespace pq
