// uq_plan.hpp -- block tables and slot maps of a ragged step from its lengths
// (uq_plan_tokens of include/uq.h), part of the uq_quantize.hip translation
// unit.
//
// Two exclusive prefix sums over the sequences, of their token rows and of the
// pages they take, decide everything; a row's sequence is found by a binary
// search in the first.  Every block makes both sums itself, in LDS, and then
// does its share of the rows and of the new page-table entries, so that one
// launch without any exchange between blocks suffices.  A new page's id is
// read from the free list, never from a page-table entry that another block
// writes.  The sums saturate one above the limit they are compared with, which
// keeps them in 32 bits (saturating addition of non-negative values is
// associative).  Bound by launch latency: 5.0 us for 64 sequences of one token,
// 6.8 us for 300 sequences and 32768 rows (0.5 MB).
#pragma once

#include "uq_device.hpp"
#include "uq_internal.hpp"

namespace uq {

constexpr int kPlanThreads = 256;

__device__ __forceinline__ int sat_add(int a, int b, int most) {
    const int s = a + b;   // both at most 2^29
    return s < most ? s : most;
}

// Inclusive saturating scan over the block of one value per thread.
__device__ __forceinline__ int block_scan(int x, int most, int* wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_up(x, s);
        if (lane >= s) x = sat_add(x, o, most);
    }
    __syncthreads();   // an earlier scan's sums are read
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x = sat_add(x, wave_sums[w], most);
    return x;
}

// The last index i of a[0 .. n - 1] (ascending, a[0] <= x) with a[i] <= x.
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads) plan_tokens_kernel(PlanParams p) {
    // first token row and first free-list entry of every sequence
    extern __shared__ int lds[];
    int* row0 = lds;
    int* entry0 = lds + p.batch + 1;
    __shared__ int wave_sums[kPlanThreads / 64];
    __shared__ int totals[2];
    const int tid = threadIdx.x;
    const int cap = int(p.num_tokens);
    // sequences per thread, in order
    const int per = (p.batch + kPlanThreads - 1) / kPlanThreads;
    const int b0 = tid * per < p.batch ? tid * per : p.batch;
    const int b1 = b0 + per < p.batch ? b0 + per : p.batch;
    auto length = [](int x) { return x > 0 ? x : 0; };
    int rows = 0;
    for (int b = b0; b < b1; ++b) {
        const int n = length(p.new_lens[b]);
        rows = sat_add(rows, n < cap + 1 ? n : cap + 1, cap + 1);
    }
    int end = block_scan(rows, cap + 1, wave_sums);
    if (tid == kPlanThreads - 1) totals[0] = end < cap ? end : cap;
    // the exclusive sum: the previous thread's inclusive one (saturated sums
    // cannot be subtracted)
    __shared__ int before[kPlanThreads];
    before[tid] = end;
    __syncthreads();
    int start = tid > 0 ? before[tid - 1] : 0;
    int pages = 0;
    for (int b = b0; b < b1; ++b) {
        const int h = length(p.cached_lens[b]), n = length(p.new_lens[b]);
        row0[b] = start;
        start = sat_add(start, n < cap + 1 ? n : cap + 1, cap + 1);
        const int64_t total = (int64_t(h) + n + kPage - 1) / kPage, held = (int64_t(h) + kPage - 1) / kPage;
        const bool fits = total <= p.max_pages_per_seq && start <= cap;
        const int need = fits ? int(total - held < p.num_free + 1 ? total - held : p.num_free + 1) : 0;
        entry0[b] = need;   // replaced by the sum below
        pages = sat_add(pages, need, p.num_free + 1);
    }
    end = block_scan(pages, p.num_free + 1, wave_sums);
    __syncthreads();
    before[tid] = end;
    __syncthreads();
    int entry = tid > 0 ? before[tid - 1] : 0;
    int refused = 0, taken = 0;
    for (int b = b0; b < b1; ++b) {
        const int need = entry0[b];
        const int h = length(p.cached_lens[b]), n = length(p.new_lens[b]);
        const int64_t total = (int64_t(h) + n + kPage - 1) / kPage;
        const bool fits = total <= p.max_pages_per_seq && sat_add(row0[b], n < cap + 1 ? n : cap + 1, cap + 1) <= cap;
        const bool ok = fits && (need == 0 || sat_add(entry, need, p.num_free + 1) <= p.num_free);
        // a refused sequence keeps its place in the sum; the sign bit marks it
        entry0[b] = ok ? entry : entry | int(0x80000000u);
        if (ok) taken += need;
        refused += ok ? 0 : 1;
        entry = sat_add(entry, need, p.num_free + 1);
        if (blockIdx.x == 0) {
            p.context_lens[b] = ok ? h + n : 0;
            p.cu_seqlens[b] = row0[b] < cap ? row0[b] : cap;
        }
    }
    // the pages of all admitted sequences: admitted ones are a prefix of those
    // that need any, so their sum is the last admitted entry's end
    int all = block_scan(taken, p.num_free + 1, wave_sums);
    if (tid == kPlanThreads - 1) totals[1] = all;
    if (blockIdx.x == 0) {
        const int r = block_scan(refused, 0x3FFFFFFF, wave_sums);
        if (tid == kPlanThreads - 1) {
            p.cu_seqlens[p.batch] = totals[0];
            p.result[0] = totals[0];
            p.result[1] = all;
            p.result[2] = r;
        }
    }
    __syncthreads();
    const int used = totals[0], got = totals[1];
    const int step = int(gridDim.x) * kPlanThreads;
    // token rows
    for (int t = blockIdx.x * kPlanThreads + tid; t < cap; t += step) {
        int seq = -1, pos = 0;
        int64_t slot = -1;
        if (t < used) {
            seq = last_not_above(row0, p.batch, t);
            const int h = length(p.cached_lens[seq]);
            // (a refused sequence's position may pass 32 bits: it wraps, and is not used)
            pos = int(unsigned(h) + unsigned(t - row0[seq]));
            const int e = entry0[seq];
            if (e >= 0) {
                const int held = (h + kPage - 1) / kPage, pg = pos / kPage;
                const int page = pg >= held ? p.free_pages[e + pg - held]
                                            : p.page_table[int64_t(seq) * p.max_pages_per_seq + pg];
                slot = int64_t(page) * kPage + pos % kPage;
            }
        }
        p.seq_ids[t] = seq;
        p.positions[t] = pos;
        p.slots[t] = slot;
    }
    // new page-table entries: entry j of the free list goes to the last admitted
    // sequence whose first entry is at most j
    for (int j = blockIdx.x * kPlanThreads + tid; j < got; j += step) {
        int lo = 0, hi = p.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((entry0[mid] & 0x7FFFFFFF) <= j) lo = mid; else hi = mid;
        }
        const int held = (length(p.cached_lens[lo]) + kPage - 1) / kPage;
        p.page_table[int64_t(lo) * p.max_pages_per_seq + held + j - (entry0[lo] & 0x7FFFFFFF)] = p.free_pages[j];
    }
}

hipError_t launch_plan_tokens(const PlanParams& p, hipStream_t stream) {
    // a row (or entry) per thread, up to two blocks per CU
    const int64_t work = p.num_tokens > p.num_free ? p.num_tokens : p.num_free;
    int64_t blocks = (work + kPlanThreads - 1) / kPlanThreads;
    blocks = blocks < 1 ? 1 : blocks < 2 * kNumCus ? blocks : 2 * kNumCus;
    const unsigned lds = unsigned(2 * p.batch + 1) * sizeof(int);
    hipLaunchKernelGGL(plan_tokens_kernel, dim3(unsigned(blocks)), dim3(kPlanThreads), lds, stream, p);
    return hipGetLastError();
}

}  // namespace uq
