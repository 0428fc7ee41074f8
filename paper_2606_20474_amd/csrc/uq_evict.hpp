// uq_evict.hpp -- eviction from the FP4 cache by accumulated attention weight
// (uq_select_tokens and uq_compact_kv of include/uq.h; uq_weights.hpp has
// uq_token_weights), part of the uq_quantize.hip translation unit.
#pragma once

#include "uq_device.hpp"
#include "uq_internal.hpp"

namespace uq {

// ---------------------------------------------------------------------------
// Which tokens stay.  Of a row (sequence, KV head) with more tokens than the
// budget: the first `sinks`, the last `recent`, and of those between the ones with
// the largest weights, of equal ones the first.  The weight of the last one that
// stays is found by its bits, most significant first, from counts of the keys
// (floats as integers of the same order) that begin with the bits found so far.

constexpr int kSelectThreads = 1024;

// A float's bits as an unsigned integer of the same order; -0 equals 0, and a NaN is
// below every number.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = f32_bits(w + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads) select_tokens_kernel(SelectParams p) {
    constexpr int kBins = 2048, kWaves = kSelectThreads / 64;
    __shared__ int bins[kBins];
    __shared__ int wave_sum[2][kWaves];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = int(blockIdx.x / unsigned(p.heads));
    int n = p.context_lens[b];
    n = n < p.max_context ? n : p.max_context;
    n = n > 0 ? n : 0;
    const float* w = p.weights + int64_t(blockIdx.x) * p.width;
    int32_t* kept = p.kept + int64_t(blockIdx.x) * p.budget;
    if (blockIdx.x % unsigned(p.heads) == 0 && tid == 0) p.kept_lens[b] = n < p.budget ? n : p.budget;
    if (n <= p.budget) {
        for (int i = tid; i < p.budget; i += kSelectThreads) kept[i] = i < n ? i : -1;
        return;
    }
    // the tokens that compete, and how many of them stay
    const int lo = p.sinks, hi = n - p.recent;
    const int want = p.budget - p.sinks - p.recent;
    uint32_t prefix = 0;    // the bits found
    int above = 0;          // competing keys above every key that begins with them
    int shift = 32;
    // (want == 0: no key is above the largest one, and no equal one stays)
    for (int pass = 0; pass < 3 && want > 0; ++pass) {
        const int width = pass == 2 ? 10 : 11;
        const int before = shift;
        shift -= width;
        for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
        __syncthreads();
        for (int t = lo + tid; t < hi; t += kSelectThreads) {
            const uint32_t key = weight_key(w[t]);
            if (before == 32 || key >> before == prefix) atomicAdd(&bins[(key >> shift) & ((1u << width) - 1)], 1);
        }
        __syncthreads();
        // the largest bin with at least want - above keys in it and above it: thread i
        // holds bins 2 i and 2 i + 1, from the top
        const int top = kBins - 1 - 2 * tid;
        const int c0 = bins[top], c1 = bins[top - 1];
        int sum = c0 + c1;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int o = __shfl_up(sum, s);
            if (lane >= s) sum += o;
        }
        if (lane == 63) wave_sum[0][wave] = sum;
        __syncthreads();
        int prior = 0;
        for (int i = 0; i < wave; ++i) prior += wave_sum[0][i];
        const int end = above + prior + sum, mid = end - c1, start = mid - c0;
        if (start < want && end >= want) {
            found[0] = mid >= want ? top : top - 1;
            found[1] = mid >= want ? start : mid;
        }
        __syncthreads();
        prefix = (prefix << width) | uint32_t(found[0]);
        above = found[1];
        __syncthreads();
    }
    // every key above `prefix` stays, and the first `ties` equal to it
    const uint32_t least = want > 0 ? prefix : 0xFFFFFFFFu;
    const int ties = want > 0 ? want - above : 0;
    // a wave takes a run of tokens: counts first, then the indices
    const int run = ((n + kSelectThreads - 1) / kSelectThreads) * 64;
    const int from = wave * run < n ? wave * run : n, to = from + run < n ? from + run : n;
    auto kind = [&](int t, bool& sure, bool& equal) {
        sure = equal = false;
        if (t < to) {
            const bool fixed = t < lo || t >= hi;
            const uint32_t key = fixed ? 0u : weight_key(w[t]);
            sure = fixed || key > least;
            equal = !fixed && key == least;
        }
    };
    int nsure = 0, nequal = 0;
    for (int t = from; t < to; t += 64) {
        bool sure, equal;
        kind(t + lane, sure, equal);
        nsure += __builtin_popcountll(__builtin_amdgcn_ballot_w64(sure));
        nequal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(equal));
    }
    if (lane == 0) {
        wave_sum[0][wave] = nsure;
        wave_sum[1][wave] = nequal;
    }
    __syncthreads();
    int s0 = 0, e0 = 0;
    for (int i = 0; i < wave; ++i) {
        s0 += wave_sum[0][i];
        e0 += wave_sum[1][i];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    for (int t = from; t < to; t += 64) {
        bool sure, equal;
        kind(t + lane, sure, equal);
        const uint64_t sm = __builtin_amdgcn_ballot_w64(sure), em = __builtin_amdgcn_ballot_w64(equal);
        const int s = s0 + __builtin_popcountll(sm & below), e = e0 + __builtin_popcountll(em & below);
        const int at = s + (e < ties ? e : ties);
        if ((sure || (equal && e < ties)) && at < p.budget) kept[at] = t + lane;
        s0 += __builtin_popcountll(sm);
        e0 += __builtin_popcountll(em);
    }
}

hipError_t launch_select_tokens(const SelectParams& p, hipStream_t stream) {
    hipLaunchKernelGGL(select_tokens_kernel, dim3(unsigned(p.batch * p.heads)), dim3(kSelectThreads), 0, stream, p);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The kept tokens to the front of their pages, in place and in order.  A token
// never moves up (the i-th kept one stands at i or behind), so a block that takes a
// (sequence, KV head) in chunks of tokens may write a chunk once it has read it:
// what later chunks read lies behind.  Tokens that stay where they are are not
// touched.

constexpr int kCompactThreads = 256;

template <int D>
__global__ void __launch_bounds__(kCompactThreads) compact_kv_kernel(CompactParams p) {
    constexpr int NT = kCompactThreads, G = D / 32;
    constexpr int TOK = 64;                           // tokens of a chunk
    constexpr int KU = TOK * G / NT, VU = TOK * (D / 8) / NT, SU = TOK * G * 2 / NT;   // units per thread
    static_assert(KU * NT == TOK * G || KU == 0, "");
    constexpr int KR = KU > 0 ? KU : 1, SR = SU > 0 ? SU : 1;
    const int tid = threadIdx.x;
    if (blockIdx.x == unsigned(p.batch * p.heads)) {
        // page ids behind the kept tokens, in sequence order
        __shared__ int sums[NT];
        int base = 0;
        for (int b0 = 0; b0 < p.batch; b0 += NT) {
            const int b = b0 + tid;
            int first = 0, count = 0;
            if (b < p.batch) {
                const int most = p.max_pages_per_seq * kPage;
                int n = p.context_lens[b], k = p.kept_lens[b];
                n = n < 0 ? 0 : n < most ? n : most;
                k = k < 0 ? 0 : k < n ? k : n;
                first = (k + kPage - 1) / kPage;
                count = (n + kPage - 1) / kPage - first;
            }
            sums[tid] = count;
            __syncthreads();
            for (int s = 1; s < NT; s <<= 1) {
                const int o = tid >= s ? sums[tid - s] : 0;
                __syncthreads();
                sums[tid] += o;
                __syncthreads();
            }
            const int all = sums[NT - 1];
            const int at = base + sums[tid] - count;
            if (p.freed_pages != nullptr)
                for (int i = 0; i < count; ++i) p.freed_pages[at + i] = p.page_table[int64_t(b) * p.max_pages_per_seq + first + i];
            base += all;
            __syncthreads();
        }
        if (tid == 0) *p.freed_count = base;
        return;
    }
    const int b = int(blockIdx.x / unsigned(p.heads)), h = int(blockIdx.x % unsigned(p.heads));
    const int most = p.max_pages_per_seq * kPage;
    int len = p.kept_lens[b];
    len = len < 0 ? 0 : len < p.budget ? len : p.budget;
    len = len < most ? len : most;
    const int32_t* kept = p.kept + int64_t(blockIdx.x) * p.budget;
    const int32_t* table = p.page_table + int64_t(b) * p.max_pages_per_seq;
    float* w = p.weights != nullptr ? p.weights + int64_t(blockIdx.x) * p.width : nullptr;
    __shared__ int64_t src_tile[TOK], dst_tile[TOK];   // (page, head) index, -1: nothing to move
    __shared__ int src_at[TOK];
    for (int c0 = 0; c0 < len; c0 += TOK) {
        float wv = 0.f;
        int from = 0;
        if (tid < TOK) {
            const int to = c0 + tid;
            int64_t d = -1, s = -1;
            if (to < len) {
                from = kept[to];
                from = from < to ? to : from < most ? from : most - 1;
                if (from != to) {
                    const int sp = table[from / kPage], dp = table[to / kPage];
                    s = (sp >= 0 && sp < p.num_pages ? int64_t(sp) : 0) * p.heads + h;
                    d = dp >= 0 && dp < p.num_pages ? int64_t(dp) * p.heads + h : -1;
                    if (w != nullptr && from < p.width) wv = w[from];
                }
            }
            src_tile[tid] = s;
            dst_tile[tid] = d;
            src_at[tid] = from % kPage;
        }
        __syncthreads();
        u32x4 kc[KR];
        uint32_t vc[VU];
        uint8_t sc[SR];
#pragma unroll
        for (int u = 0; u < KR; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), g = i / TOK;
            if (g < G && dst_tile[t] >= 0)
                kc[u] = *reinterpret_cast<const u32x4*>(p.codes + src_tile[t] * (16 * D) + (g * kPage + src_at[t]) * 16);
        }
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), e = i / TOK;
            if (dst_tile[t] >= 0)
                vc[u] = *reinterpret_cast<const uint32_t*>(p.codes + src_tile[t] * (16 * D) + 8 * D +
                                                           ((src_at[t] >> 2) * (D / 8) + e) * 16 + (src_at[t] & 3) * 4);
        }
#pragma unroll
        for (int u = 0; u < SR; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), g = i / TOK;
            if (g < 2 * G && dst_tile[t] >= 0) sc[u] = p.scales[src_tile[t] * D + g * kPage + src_at[t]];
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): the chunk is read
        __syncthreads();
#pragma unroll
        for (int u = 0; u < KR; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), g = i / TOK, a = (c0 + t) & (kPage - 1);
            if (g < G && dst_tile[t] >= 0)
                *reinterpret_cast<u32x4*>(p.codes + dst_tile[t] * (16 * D) + (g * kPage + a) * 16) = kc[u];
        }
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), e = i / TOK, a = (c0 + t) & (kPage - 1);
            if (dst_tile[t] >= 0)
                *reinterpret_cast<uint32_t*>(p.codes + dst_tile[t] * (16 * D) + 8 * D + ((a >> 2) * (D / 8) + e) * 16 + (a & 3) * 4) = vc[u];
        }
#pragma unroll
        for (int u = 0; u < SR; ++u) {
            const int i = tid + u * NT, t = i & (TOK - 1), g = i / TOK, a = (c0 + t) & (kPage - 1);
            if (g < 2 * G && dst_tile[t] >= 0) p.scales[dst_tile[t] * D + g * kPage + a] = sc[u];
        }
        if (w != nullptr && tid < TOK && c0 + tid < len && from != c0 + tid && c0 + tid < p.width) w[c0 + tid] = wv;
        __syncthreads();
    }
    if (w != nullptr) {
        int n = p.context_lens[b];
        n = n < most ? n : most;
        n = n < p.width ? n : p.width;
        for (int t = len + tid; t < n; t += NT) w[t] = 0.f;
    }
}

hipError_t launch_compact_kv(const CompactParams& p, hipStream_t stream) {
    const dim3 grid{unsigned(p.batch * p.heads) + (p.freed_count != nullptr ? 1u : 0u)}, block{unsigned(kCompactThreads)};
    if (p.head_dim == 64) hipLaunchKernelGGL(compact_kv_kernel<64>, grid, block, 0, stream, p);
    else if (p.head_dim == 128) hipLaunchKernelGGL(compact_kv_kernel<128>, grid, block, 0, stream, p);
    else hipLaunchKernelGGL(compact_kv_kernel<256>, grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace uq
