// Page tables and slot maps of the paged latent cache, built on the GPU from the requests' lengths.
//
// Request b holds len_b tokens in ceil(len_b / page) pages (block_table[b, 0 ..)) and adds new_b more in this step.  The
// pages it lacks come off the top of a stack of free pages, request by request in index order.  With
//     held_b = ceil(len_b / page),  need_b = ceil((len_b + new_b) / page)
//     cu_b = sum_{a < b} new_a,     off_b = sum_{a < b} (need_a - held_a)
// column held_b + k of row b becomes free_pages[n_free - 1 - (off_b + k)], and the new token number i of request b is
// row cu_b + i of the step: position len_b + i, slot block_table[b, position / page] * page + position % page.
//
// Integer work of a few hundred kilobytes: what it costs is launches and latency, so it is one kernel.  Every block
// computes both prefix sums itself (n is thousands at most; that is a few microseconds of redundant work instead of
// a second launch or a grid-wide wait), keeps them in shared memory, and fills its share of the rows by binary search.
// Measured: 48 requests with a token each 3.4 us, 1024 requests with 130 thousand new tokens 5.8 us (1 MB written; the rest is latency).
#pragma once
#include "sm100_ptx.cuh"

namespace laga {

constexpr int kPlanThreads = 512;
constexpr int kPlanMaxRequests = 8192;                       // two prefix arrays of 4 bytes per request in shared memory
constexpr unsigned kStatusCachePlan = 0x50000000u;           // | what did not fit
enum { kPlanBadLength = 1, kPlanNoPages = 2, kPlanNoColumns = 3, kPlanNoRows = 4 };

struct CachePlanArgs {
    const int *seq_lens, *new_lens;        // [n]
    int n, page_shift, columns;
    int* block_table;                      // [n, columns]
    const int *free_pages, *n_free;
    int free_capacity, max_tokens;
    int *slots, *positions;                // [max_tokens]
    int *cu_new, *seq_lens_out, *n_free_out;
    unsigned* status;
};

// last index i in [0, n) with start[i] <= t; `start` is non-decreasing with start[0] = 0
__device__ __forceinline__ int plan_find(const int* start, int n, int t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads)
cache_plan_kernel(const CachePlanArgs a) {
    extern __shared__ int plan_smem[];
    int* cu = plan_smem;                   // [n + 1] new tokens before request b
    int* off = plan_smem + a.n + 1;        // [n + 1] new pages before request b
    __shared__ long long warp_tokens[kPlanThreads / 32], warp_pages[kPlanThreads / 32];
    __shared__ int bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int page = 1 << a.page_shift;
    const long long capacity = static_cast<long long>(a.columns) << a.page_shift;
    if (tid == 0) bad = 0;
    __syncthreads();

    // both prefix sums, a contiguous run of requests per thread; 64-bit sums, so that no set of lengths wraps around
    const int run = (a.n + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min(a.n, tid * run), b1 = min(a.n, b0 + run);
    long long tokens = 0, pages = 0;
    int fault = 0;
    for (int b = b0; b < b1; ++b) {
        const long long len = a.seq_lens[b], add = a.new_lens[b];
        if (len < 0 || add < 0) { fault = kPlanBadLength; continue; }
        if (len + add > capacity) { fault = kPlanNoColumns; continue; }
        tokens += add;
        pages += ((len + add + page - 1) >> a.page_shift) - ((len + page - 1) >> a.page_shift);
    }
    if (fault) atomicMax(&bad, fault);
    long long it = tokens, ip = pages;     // inclusive scans inside the warp
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, it, d), p = __shfl_up_sync(0xffffffffu, ip, d);
        if (lane >= d) { it += t; ip += p; }
    }
    if (lane == 31) { warp_tokens[warp] = it; warp_pages[warp] = ip; }
    __syncthreads();
    long long before_t = it - tokens, before_p = ip - pages, total_t = 0, total_p = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        if (w < warp) { before_t += warp_tokens[w]; before_p += warp_pages[w]; }
        total_t += warp_tokens[w];
        total_p += warp_pages[w];
    }
    const int n_free = *a.n_free;
    int why = bad;
    if (!why && (n_free < 0 || n_free > a.free_capacity)) why = kPlanBadLength;
    if (!why && total_p > n_free) why = kPlanNoPages;
    if (!why && total_t > a.max_tokens) why = kPlanNoRows;
    const bool first = blockIdx.x == 0;
    if (why) {      // nothing is taken: the state comes back as it was, and no row has a slot
        const int stride = gridDim.x * kPlanThreads;
        for (int t = blockIdx.x * kPlanThreads + tid; t < a.max_tokens; t += stride) { a.slots[t] = -1; a.positions[t] = 0; }
        if (first) {
            for (int b = tid; b < a.n; b += kPlanThreads) { a.cu_new[b] = 0; a.seq_lens_out[b] = a.seq_lens[b]; }
            if (tid == 0) { a.cu_new[a.n] = 0; *a.n_free_out = n_free; *a.status = kStatusCachePlan | why; }
        }
        return;
    }
    for (int b = b0; b < b1; ++b) {
        const int len = a.seq_lens[b], add = a.new_lens[b];
        cu[b] = static_cast<int>(before_t);
        off[b] = static_cast<int>(before_p);
        if (first) { a.cu_new[b] = static_cast<int>(before_t); a.seq_lens_out[b] = len + add; }
        before_t += add;
        before_p += ((static_cast<long long>(len) + add + page - 1) >> a.page_shift) - ((static_cast<long long>(len) + page - 1) >> a.page_shift);
    }
    if (tid == 0) {
        cu[a.n] = static_cast<int>(total_t);
        off[a.n] = static_cast<int>(total_p);
        if (first) { a.cu_new[a.n] = static_cast<int>(total_t); *a.n_free_out = n_free - static_cast<int>(total_p); *a.status = 0u; }
    }
    __syncthreads();
    const int stride = gridDim.x * kPlanThreads, start = blockIdx.x * kPlanThreads + tid;
    const int n_tokens = static_cast<int>(total_t), n_pages = static_cast<int>(total_p);
    for (int k = start; k < n_pages; k += stride) {
        const int b = plan_find(off, a.n, k);
        const int held = static_cast<int>((static_cast<long long>(a.seq_lens[b]) + page - 1) >> a.page_shift);
        a.block_table[static_cast<size_t>(b) * a.columns + held + (k - off[b])] = a.free_pages[n_free - 1 - k];
    }
    for (int t = start; t < a.max_tokens; t += stride) {
        int slot = -1, position = 0;
        if (t < n_tokens) {
            const int b = plan_find(cu, a.n, t);
            const int len = a.seq_lens[b];
            position = len + (t - cu[b]);
            const int column = position >> a.page_shift;
            const int held = static_cast<int>((static_cast<long long>(len) + page - 1) >> a.page_shift);
            // a page of this step is read from the stack: its table entry may be another block's to write
            const int p = column < held ? a.block_table[static_cast<size_t>(b) * a.columns + column]
                                        : a.free_pages[n_free - 1 - (off[b] + column - held)];
            const long long s = (static_cast<long long>(p) << a.page_shift) + (position & (page - 1));
            slot = p >= 0 && s <= 0x7fffffffll ? static_cast<int>(s) : -1;
        }
        a.slots[t] = slot;
        a.positions[t] = position;
    }
}

}  // namespace laga
