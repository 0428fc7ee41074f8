// uq_extend.hpp -- attention of several new queries per sequence over the FP4
// cache (uq_extend_attention of include/uq.h), part of the uq_decode.hip
// translation unit.
//
// With m queries at the end of a context of n tokens, query i at position
// n - m + i, and G query heads per KV head, a row is a (query, head of the KV
// head) pair, row r = query r / G, head r % G: all rows of a (sequence, KV head)
// read the same keys and values, so a block takes M of them and walks the
// visible context once in tiles of 8192 / d tokens.
//
//   scores    S^T = K Q^T on v_mfma_scale_f32_32x32x64_f8f6f4: FP4 keys with
//             their scale bytes as operand A (rows = tokens), the rotated FP8
//             queries as operand B (columns = rows of the block).  A lane then
//             holds 16 tokens of one row, so the softmax needs no exchange
//             between lanes but one (lanes l and l ^ 32 share a row).
//   softmax   in the log2 domain, relative to a running reference with a lazy
//             rescale, sums per lane until the end.
//   values    O^T += V^T P^T on v_mfma_f32_32x32x16_f16.  The scores leave the
//             QK instruction in the order in which P enters as operand B (the
//             token of a k index is free as long as V's operand uses the same
//             order), so P stays in registers.  V is decoded once per block and
//             tile into FP16 in LDS, transposed to operand order.
//
// M = 256 (4 waves of 64 rows; 128 at d = 256, where the accumulators leave room
// for 32 rows per wave): a decoded tile serves as many rows as registers hold.  A wave
// of d = 128 takes all 256 VGPRs, two waves per SIMD.  For sequences of at most 64
// rows per KV head the four waves take tiles of their own instead, each all the
// rows, and are joined at the end; long contexts with few rows are split over blocks
// (extend_shape in uq_api.hip has the rules and both sides' times).
//
// What bounds it: the issue of the softmax's and the decode's vector instructions
// beside the matrix instructions.  8192 new tokens of 64 heads over 4, d = 128: 0.82 ms a
// pass among others (0.92 on a GPU that idled before), 1.35 PFLOP/s for the 1.1e12 flops
// that causality leaves; the matrix cores are busy 46 % of the time and vector
// instructions issue 72 % of it.  5 tokens of 64 heads over 8 in 16 sequences of 8k to
// 24k: 117 us a pass, 2.2 TB/s of codes and scales, the four waves' work on 64 rows of
// which 40 are used (vector 52 %, matrix 18 %, 37 % of the waves' time waiting with two
// waves per SIMD).
//
// FP16 holds P with 11 significant bits from 2^-14 on, its range ending at 2^16, and the
// sum counts weights that FP16 would lose.  So a row's weights are relative to a
// reference 7 or more below its largest score, whose weight is 2^7 to 2^15 then, and
// where the heavy tokens' values are small the reference follows the scores down: the row's
// sum and accumulators are fp32 and hold what lies behind, up to 2^80 of it.
//
// A code times 2^E is exact in FP16 for E in [-23, 13].  So the values of each block of
// 32 channels are taken relative to an exponent of their own, v 2^-e, and the
// accumulators hold O 2^-e: e is 8 below the largest scale exponent when it is set (in
// the first tile), and set again, the accumulators rescaled, when a tile's largest
// passes e + 13.  Values more than 2^31 below the largest of their 32 channels that the
// block has seen are lost.
#pragma once

#include "uq_device.hpp"
#include "uq_internal.hpp"
#include "uq_quad.hpp"

namespace uq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// A weight of the binade [2^k, 2^(k+1)) loses 2^-11 2^k on average when it is cut to
// 11 significant bits, a share of 2^-11 / (2 ln 2) over log-uniform weights: log2 of
// one plus that, and the inverse of one plus that.  (A weight of 1, lifted and cut,
// is 1 again.)
constexpr float kLift = 5.08057e-4f;
constexpr float kLower = 0.99964790f;

// The reference of a row's weights, in powers of two.  It moves up when a score of 32
// tokens is more than kUp above it, to kLead below that score.  It moves down to the
// largest of the 32 when that is more than kDown below it and the row's average so far is
// less than kSmall in some 32 channels, where the largest scale is 2^8 or more: the heavy
// tokens' values are small then, and light ones count.  Down by at most kDepth and only
// while the row's sum is below 2^kDepth, so that the accumulators (at most 2^16 times the
// sum) stay finite.
constexpr float kLead = 7.0f, kUp = kLead + kLazyRescale, kDown = -9.0f;
constexpr float kSmall = 32.0f;
constexpr float kDepth = 40.0f, kDeep = 0x1p40f;
// A wave looks for low scores while it has credit: 1 for each 32 tokens, at most
// kCredit, less kCostMoved for each 32 with a lane below kDown where a row moved down and
// kCostIdle where none did.  (Scores of a standard deviation of 4, 6 and 12 in powers of
// two, 8192 new tokens of 64 heads: 867, 857 and 855 us, 840, 824 and 840 without looking,
// 930, 1016 and 1060 when looking at every 32 and whatever the values.)
constexpr int kCredit = 64, kCostMoved = 8, kCostIdle = 64;

constexpr int kNoBase = -512;   // no exponent yet: every scale is above it

// Tokens per tile: one 16-byte unit of K and one of V for each of 256 threads.
template <int D> constexpr int extend_tile() { return 8192 / D; }

// CROSS, below: the queries have no order and see their whole context
// (uq_cross_attention); every row then stands at the last token.  Kernels of their own, so that
// those with causality keep their registers.  8 sequences of 100 to 900 queries over 3k to 14k tokens, 64
// heads over 8: 500 us a pass, 1.21 PFLOP/s; 16 of 5 queries over 1500, 16 heads of 64 over 16, 27 us.

// Where a block's rows stand and which tiles they see.
struct ExtendRows {
    int b;              // sequence
    int first, count;   // its first token row in q, number of queries
    int row0;           // first row of the block
    int n_ctx;          // context length
    int sink_tiles;     // tiles of the first tokens, ahead of the others
    int tile0;          // first of the other tiles
    int tiles;          // all of them
    int split;          // the block's share of the tiles
    int share;          // tokens per split, or 0: p.splits equal ones
};

// Tiles that rows with positions lo .. hi see.
template <int TT>
__device__ __forceinline__ void extend_tiles(const ExtendParams& p, int lo, int hi, ExtendRows& r) {
    const int end = hi + 1;
    const int last = end > 0 ? (end + TT - 1) / TT : 0;
    r.sink_tiles = 0;
    r.tile0 = 0;
    if (p.window > 0) {
        const int from = lo - p.window + 1;   // the first row's window, the earliest
        r.tile0 = from > 0 ? from / TT : 0;
        const int sinks = p.sinks < end ? p.sinks : end;
        r.sink_tiles = sinks > 0 ? (sinks + TT - 1) / TT : 0;
        if (r.sink_tiles >= r.tile0) r.sink_tiles = r.tile0 = 0;
    }
    r.tiles = r.sink_tiles + (last > r.tile0 ? last - r.tile0 : 0);
}

__device__ __forceinline__ int extend_first(const ExtendParams& p, int b) {
    const int x = p.cu_seqlens[b];
    return x < 0 ? 0 : x < p.num_tokens ? x : p.num_tokens;
}
__device__ __forceinline__ int extend_context(const ExtendParams& p, int b) {
    int n = p.context_lens[b];
    n = n < p.max_context ? n : p.max_context;
    return n > 0 ? n : 0;
}

// Tiles per split of a row block with `tiles` of them: of a number of splits, or of
// `share` tokens each.
template <int TT>
__device__ __forceinline__ int extend_per_split(int tiles, int splits, int share) {
    const int per = share > 0 ? (share - 1) / TT + 1 : (tiles + splits - 1) / splits;
    return per > 4 ? per : 4;
}

// Row block `at` of the batch, M rows each, the blocks of one sequence from its
// last rows (the longest) to its first.  False: there is none.  Wave-uniform;
// every wave of the block finds it alone, 64 sequences at a time.
template <int M>
__device__ __forceinline__ bool extend_find(const ExtendParams& p, int at, ExtendRows& r) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
        const int b = b0 + lane;
        int first = 0, count = 0;
        if (b < p.batch) {
            first = extend_first(p, b);
            count = extend_first(p, b + 1) - first;
            count = count > 0 ? count : 0;
        }
        const int blocks = int((int64_t(count) * p.group + M - 1) / M);
        int sum = blocks;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int o = __shfl_up(sum, s);
            if (lane >= s) sum += o;
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > at);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            r.b = b0 + l;
            r.first = __builtin_amdgcn_readlane(first, l);
            r.count = __builtin_amdgcn_readlane(count, l);
            const int n = __builtin_amdgcn_readlane(blocks, l);
            const int i = at - before - (__builtin_amdgcn_readlane(sum, l) - n);
            r.row0 = (n - 1 - i) * M;
            r.n_ctx = __builtin_amdgcn_readfirstlane(extend_context(p, r.b));
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The same with the row blocks of all sequences (at most 64, one per lane) in
// descending order of their last position, to a 32nd of the longest context: blocks
// of different sequences differ by the whole context, and a long one that starts
// last leaves the others' CUs idle.  above(j): blocks that end at or past the j-th
// 32nd; `at` falls into the largest j with more than `at` of them.
template <int M, bool CROSS>
__device__ __forceinline__ bool extend_find_longest(const ExtendParams& p, int at, ExtendRows& r) {
    const int lane = threadIdx.x & 63;
    int first = 0, count = 0, n = 0;
    if (lane < p.batch) {
        first = extend_first(p, lane);
        count = extend_first(p, lane + 1) - first;
        count = count > 0 ? count : 0;
        n = extend_context(p, lane);
    }
    const int blocks = int((int64_t(count) * p.group + M - 1) / M);
    const int start = n - count;
    auto total = [&](int x) {
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s);
        return __builtin_amdgcn_readfirstlane(x);
    };
    int top = n;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_xor(top, s);
        top = top > o ? top : o;
    }
    const int width = __builtin_amdgcn_readfirstlane(top) / 32 + 1;
    auto above = [&](int j) {
        const int64_t from = int64_t(j) * width;
        if (CROSS) return j == 0 || from < n ? blocks : 0;
        if (j == 0 || from <= start) return blocks;
        return from >= n ? 0 : blocks - int((from - start) * p.group / M);
    };
    if (total(blocks) <= at) return false;
    int lo = 0, hi = 32;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (total(above(mid)) > at) lo = mid; else hi = mid;
    }
    const int longer = above(hi), here = above(lo) - longer;
    const int rank = at - total(longer);
    int sum = here;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_up(sum, s);
        if (lane >= s) sum += o;
    }
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > rank));
    r.b = l;
    r.first = __builtin_amdgcn_readlane(first, l);
    r.count = __builtin_amdgcn_readlane(count, l);
    r.n_ctx = __builtin_amdgcn_readlane(n, l);
    const int i = rank - __builtin_amdgcn_readlane(sum - here, l);
    r.row0 = (__builtin_amdgcn_readlane(blocks - longer, l) - 1 - i) * M;
    return true;
}

// Block `at` where every row block has p.splits of them.
template <int M, bool CROSS>
__device__ __forceinline__ bool extend_find_split(const ExtendParams& p, int at, ExtendRows& r) {
    r.split = at % p.splits;
    r.share = 0;
    return p.longest_first ? extend_find_longest<M, CROSS>(p, at / p.splits, r) : extend_find<M>(p, at / p.splits, r);
}

// Row block and split `at` of a batch (at most 64 sequences, one per lane, no
// window) whose contexts are split into shares of the same length: the smallest
// whose blocks fit p.row_blocks, tried from the mean on in steps of a 16th, and at
// least a p.splits-th of the longest context, as a row has no more partials.  TT, TA:
// tokens per tile of a sequence whose rows, or tokens (p.alone_rows), the waves split.
template <int M, int TT, int TA>
__device__ __forceinline__ bool extend_find_share(const ExtendParams& p, int at, ExtendRows& r) {
    const int lane = threadIdx.x & 63;
    int first = 0, count = 0, n = 0;
    if (lane < p.batch) {
        first = extend_first(p, lane);
        count = extend_first(p, lane + 1) - first;
        count = count > 0 ? count : 0;
        n = extend_context(p, lane);
    }
    const int blocks = int((int64_t(count) * p.group + M - 1) / M);
    const bool alone = count * p.group <= p.alone_rows;
    int top = blocks > 0 ? n : 0;
    float tokens = float(n) * float(blocks);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_xor(top, s);
        top = top > o ? top : o;
        tokens += __shfl_xor(tokens, s);
    }
    top = __builtin_amdgcn_readfirstlane(top);
    const float mean = tokens / float(p.row_blocks);
    int share = top / p.splits + 1;
    if (mean > float(share)) share = __builtin_amdgcn_readfirstlane(mean < float(top) ? int(mean) : top);
    int parts, sum;
    while (true) {
        const int tiles = n > 0 ? (n - 1) / (alone ? TA : TT) + 1 : 0;
        const int per = alone ? extend_per_split<TA>(0, 1, share) : extend_per_split<TT>(0, 1, share);
        parts = tiles > per ? (tiles + per - 1) / per : 1;
        sum = blocks * parts;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int o = __shfl_up(sum, s);
            if (lane >= s) sum += o;
        }
        if (share >= top || __builtin_amdgcn_readlane(sum, 63) <= p.row_blocks) break;
        const int step = share / 16 + 1;
        share = step < top - share ? share + step : top;
    }
    r.share = share;
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum > at);
    if (past == 0) return false;
    const int l = __builtin_ctzll(past);
    r.b = l;
    r.first = __builtin_amdgcn_readlane(first, l);
    r.count = __builtin_amdgcn_readlane(count, l);
    r.n_ctx = __builtin_amdgcn_readlane(n, l);
    const int of = __builtin_amdgcn_readlane(parts, l), all = __builtin_amdgcn_readlane(blocks, l);
    const int i = at - (__builtin_amdgcn_readlane(sum, l) - all * of);
    r.row0 = (all - 1 - i / of) * M;
    r.split = i % of;
    return true;
}

// Positions of a row block's first and last row.
template <int M, bool CROSS>
__device__ __forceinline__ void extend_span(const ExtendParams& p, const ExtendRows& r, int& lo, int& hi) {
    if constexpr (CROSS) {
        lo = hi = r.n_ctx - 1;
        return;
    }
    const int last = r.row0 + M < r.count * p.group ? r.row0 + M - 1 : r.count * p.group - 1;
    lo = r.n_ctx - r.count + r.row0 / p.group;
    hi = r.n_ctx - r.count + last / p.group;
}

// One 16-byte unit of a page's V codes (4 tokens x 8 channels, the tokens' scales in
// sc) as eight pairs of dwords: of each channel the 4 tokens in FP16.
__device__ __forceinline__ void decode_unit(const u32x4& v, const float (&sc)[4], uint2 (&out)[8]) {
    uint32_t w[4][4];   // [token][channel pair]
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t d = v[t];
        w[t][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, sc[t], 0));
        w[t][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, sc[t], 1));
        w[t][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, sc[t], 2));
        w[t][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, sc[t], 3));
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        out[2 * c] = make_uint2(__builtin_amdgcn_perm(w[1][c], w[0][c], 0x05040100u),
                                __builtin_amdgcn_perm(w[3][c], w[2][c], 0x05040100u));
        out[2 * c + 1] = make_uint2(__builtin_amdgcn_perm(w[1][c], w[0][c], 0x07060302u),
                                    __builtin_amdgcn_perm(w[3][c], w[2][c], 0x07060302u));
    }
}

// One column of the accumulators, channel 32 c + 8 (i / 4) + 4 half + i % 4 in
// acc[c][q][i] with lanes l and l ^ 32 sharing it, to channel 32 c + 16 (i / 8) + 8
// half + i % 8: runs of 8 channels per lane, for the stores.  On the way, with
// `rotate`, the rotation R: the halves' exchange brings both values of a pair of
// its stage (width 4) into one lane.
template <int CB, int NQ>
__device__ __forceinline__ void gather_columns(v16f (&acc)[CB][NQ], int q, bool rotate) {
#pragma clang fp contract(off)
    auto stage = [&](int h) {
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (i & h) continue;
                const float a = acc[c][q][i], b = acc[c][q][i + h];
                acc[c][q][i] = a + b;
                acc[c][q][i + h] = a - b;
            }
    };
    if (rotate) {
        stage(1);
        stage(2);
        stage(4);
        stage(8);
#pragma unroll
        for (int h = 1; h < CB; h <<= 1)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                if (c & h) continue;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float a = acc[c][q][i], b = acc[c + h][q][i];
                    acc[c][q][i] = a + b;
                    acc[c + h][q][i] = a - b;
                }
            }
    }
    const float r = rotate ? inv_sqrt_d<32 * CB>() : 1.0f;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i & 4) continue;
            float a = acc[c][q][i], b = acc[c][q][i + 4];
            swap32(a, b);   // lane l: both halves' values of acc[i] (l < 32) or of acc[i + 4]
            acc[c][q][i] = rotate ? (a + b) * r : a;
            acc[c][q][i + 4] = rotate ? (a - b) * r : b;
        }
}

// n / group, exact for n < 2^28.
__device__ __forceinline__ int div_group(const ExtendParams& p, int n) {
    return p.group == 1 ? n : int(__umulhi(unsigned(n), p.group_magic));
}

// The wave's 32 NQ query rows from row0 on, as FP8 in operand order at `qs`: a quad
// of lanes per row, 16 rows at a time, all loads in flight before the first
// rotation.
template <int DT, int D, int NQ>
__device__ __forceinline__ void stage_queries(const ExtendParams& p, const ExtendRows& r, int hk, int row0, uint8_t* qs) {
    constexpr int NG = D / 32, KS = D / 64;
    const int lane = threadIdx.x & 63, L = lane & 3;
    const int rows = r.count * p.group;
    // the rows of a pass together fill 64 registers, 128 at head size 256
    constexpr int PASS = D == 64 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < 2 * NQ; i += PASS) {
        float x[DT == 3 ? 1 : PASS][NG][8];
        uint2 w[PASS][NG];
#pragma unroll
        for (int u = 0; u < PASS; ++u) {
            // (rows past the last: that one again, so that no load waits for a branch)
            int row = row0 + 16 * (i + u) + (lane >> 2);
            row = row < rows ? row : rows - 1;
            const int tok = div_group(p, row);
            const int64_t elem = int64_t(r.first + tok) * p.q_stride + int64_t(hk * p.group + row - tok * p.group) * D + 8 * L;
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                if constexpr (DT == 3) w[u][j] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.q) + elem + 32 * j);
                else load_x8<DT>(p.q, elem + 32 * j, x[u][j]);
            }
        }
#pragma unroll
        for (int u = 0; u < PASS; ++u) {
            if constexpr (DT != 3) {
                wht_quad<NG>(x[u], L);
#pragma unroll
                for (int j = 0; j < NG; ++j)
                    w[u][j] = make_uint2(e4m3x4(x[u][j][0], x[u][j][1], x[u][j][2], x[u][j][3]),
                                         e4m3x4(x[u][j][4], x[u][j][5], x[u][j][6], x[u][j][7]));
            }
            const int rr = 16 * (i + u) + (lane >> 2);   // row of the wave
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                const int c = 32 * j + 8 * L;
                const int dst = ((rr >> 5) * KS + (c >> 6)) * 2048 + (((c >> 4) & 1) * 32 + (rr & 31)) * 32 + ((c >> 5) & 1) * 16 + (c & 15);
                *reinterpret_cast<uint2*>(qs + dst) = w[u][j];
            }
        }
    }
}

// Two parts of a row, references m and sums l: the first becomes both, and the
// share of the second in it is returned.
__device__ __forceinline__ float join_share(float& m, float& l, float m2, float l2) {
    const float top = __builtin_fmaxf(m, m2);
    const float a = l * __builtin_amdgcn_exp2f(m - top), b = l2 * __builtin_amdgcn_exp2f(m2 - top);
    m = top;
    l = a + b;
    return b > 0.f ? b / l : 0.f;
}

// Tokens per tile and shared memory of a walk.  ALONE: a wave walks tiles of its
// own (one in W), with buffers of its own.
template <int D, int W, bool ALONE> struct ExtendShape {
    static constexpr int CB = D / 32;
    static constexpr int TT = !ALONE ? extend_tile<D>() : D == 64 ? 64 : 32;
    // decoded values of a tile: [page][32 channels][half][8 channels][channel][8 tokens].
    // The loads take 16 bytes per lane, lane = channel; the stores 16 bytes (of a
    // channel) per lane, lane = octet of channels.  Octets 144 bytes and the 32-channel
    // blocks 16 banks apart: 8 lanes of either meet in no bank.
    static constexpr int kVOctet = 8 * 16 + 16;
    static constexpr int kVRow = 4 * kVOctet + 32;
    static_assert(2 * kVRow % 128 == 64 && kVOctet % 128 == 16, "bank layout");
    static constexpr int kVt = TT / kPage * CB * 2 * kVRow;
    static constexpr int kK = TT * D / 2;                 // K codes of a tile
    static constexpr int kKs = TT / kPage * D / 2;        // and their scales
    static constexpr int kBuffers = ALONE ? 1 : 2;
    static constexpr int kState = 16 + 8 * CB;            // grow, top, base
    static constexpr int kWalker = kBuffers * (kVt + kK + kKs) + kState;
    static constexpr int kLds = (ALONE ? W : 1) * kWalker;
};

// The walk of a block over tiles first_tile .. last_tile - 1, NQ blocks of 32 rows per
// wave, W waves: of different rows that share each tile, or (ALONE) of the same
// rows, every wave with tiles of its own.  Per tile a thread moves 16-byte units of
// K and of V: loaded into registers while the tile before is computed (the page ids
// one tile earlier still), stored to LDS after it, K as it is and V decoded.  Two
// buffers and one barrier per tile; a wave alone needs one buffer and none.
template <int D, int NQ, int W, bool ALONE, bool CROSS>
__device__ __forceinline__ void extend_walk(const ExtendParams& p, ExtendRows r, int hk, uint8_t* smem) {
    using Shape = ExtendShape<D, W, ALONE>;
    constexpr int TT = Shape::TT, CB = Shape::CB, kVRow = Shape::kVRow, kVOctet = Shape::kVOctet;
    constexpr int M = 32 * NQ * (ALONE ? 1 : W);   // rows of the block
    constexpr int NT = ALONE ? 64 : 64 * W;        // threads that share a tile
    constexpr int KS = D / 64;                     // k steps of QK^T
    constexpr int kPageUnits = D / 2;              // 16-byte units of a page's K, and of its V
    constexpr int kUnits = TT / kPage * kPageUnits;
    constexpr int UR = (kUnits + NT - 1) / NT;
    constexpr int STEP = ALONE ? W : 1;            // tiles from one of this walker's to the next
    static_assert(32 * NQ * D * (ALONE ? 1 : W) <= Shape::kBuffers * Shape::kVt, "the query operand is staged in the value buffers");
    static_assert(kUnits % 64 == 0 && kUnits % NT % 64 == 0, "units go to whole waves");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int uw = ALONE ? 0 : wave;               // wave among those that share a tile
    const int half = lane >> 5, col = lane & 31;
    uint8_t* const mine = smem + (ALONE ? wave : 0) * Shape::kWalker;
    auto vt = [&](int slot) { return mine + slot * Shape::kVt; };
    auto kt = [&](int slot) { return mine + Shape::kBuffers * Shape::kVt + slot * Shape::kK; };
    auto kst = [&](int slot) { return mine + Shape::kBuffers * (Shape::kVt + Shape::kK) + slot * Shape::kKs; };
    int* const grow = reinterpret_cast<int*>(mine + Shape::kWalker - Shape::kState);   // a scale above FP16's range in the tile
    int* const top = grow + 4;     // largest scale byte of the tile, per 32 channels (when one grows)
    int* const base = top + CB;    // scale byte the values are relative to: 127 + e
    // the waves that share a tile; a wave's own LDS accesses are in order
    auto sync = [&]() {
        if constexpr (ALONE) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        } else {
            __syncthreads();
        }
    };

    int lo, hi;
    extend_span<M, CROSS>(p, r, lo, hi);
    extend_tiles<TT>(p, lo, hi, r);
    int first_tile = 0, last_tile = r.tiles;
    bool whole = true;
    if (p.splits > 1) {
        const int per = extend_per_split<TT>(r.tiles, p.splits, r.share);
        whole = r.tiles <= per;
        first_tile = r.split * per;
        last_tile = first_tile + per < r.tiles ? first_tile + per : r.tiles;
        if (first_tile >= last_tile && r.split != 0) return;
    }
    const int rows = r.count * p.group;       // of the sequence and KV head

    // ---- queries: rotated and cast to FP8 (unless they are), to the lane order
    // of the B operand: k step s, lane (row, half): bytes 0..15 are channels
    // 64 s + 16 half .., 16..31 are 64 s + 32 + 16 half ..
    uint8_t* qs = vt(0) + uw * (32 * NQ * D);
    const int w_row0 = r.row0 + uw * (32 * NQ);
    if (p.q_dtype == 0) stage_queries<0, D, NQ>(p, r, hk, w_row0, qs);
    else if (p.q_dtype == 1) stage_queries<1, D, NQ>(p, r, hk, w_row0, qs);
    else if (p.q_dtype == 2) stage_queries<2, D, NQ>(p, r, hk, w_row0, qs);
    else stage_queries<3, D, NQ>(p, r, hk, w_row0, qs);
    const int wtid = ALONE ? lane : tid;
    if (wtid < 2) grow[wtid] = 0;
    if (wtid < CB) {
        top[wtid] = 0;
        base[wtid] = kNoBase;
    }
    sync();
    v8i qop[NQ][KS];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const uint4* src = reinterpret_cast<const uint4*>(qs + (q * KS + s) * 2048 + lane * 32);
            const uint4 a = src[0], c = src[1];
            qop[q][s] = v8i{int(a.x), int(a.y), int(a.z), int(a.w), int(c.x), int(c.y), int(c.z), int(c.w)};
        }
    sync();

    // the wave's first and last position (a wave without rows only moves tiles)
    const bool busy = w_row0 < rows;
    const int w_last = w_row0 + 32 * NQ < rows ? w_row0 + 32 * NQ - 1 : rows - 1;
    const int w_lo = CROSS ? hi : r.n_ctx - r.count + w_row0 / p.group, w_hi = CROSS ? hi : r.n_ctx - r.count + w_last / p.group;

    const int32_t* pt_row = p.page_table + int64_t(r.b) * p.max_pages_per_seq;
    const int n_pages = (hi + kPage) / kPage;   // pages up to the last that holds a visible token
    auto token_of = [&](int t) { return TT * (t < r.sink_tiles ? t : t - r.sink_tiles + r.tile0); };

    // ---- this thread's part of a tile: unit tid + u NT, `in` of its page; the first
    // D / 8 units of a page also move 4 of its K scales each.  A page takes whole
    // waves from head size 128 on: its id and addresses are scalars then.
    int32_t ids[UR];
    u32x4 kcode[UR], vcode[UR];
    uint32_t vscale[UR], kscale[UR];
    int my_base = kNoBase;      // base[] of its units' channels
    constexpr bool kWavePages = kPageUnits % 64 == 0;
    // The lane, computed anew in each tile: addresses that follow from it are then
    // made where they are used instead of living in registers through the walk (with
    // them the accumulators did not fit, and every spilled one waited for the
    // loads of the next tile).
    auto fresh_lane = [&]() {
        unsigned l = unsigned(lane);
        asm volatile("" : "+v"(l));
        return l;
    };
    auto unit_page = [&](unsigned l, int u) {
        return kWavePages ? (64 * uw + u * NT) / kPageUnits : int(64 * uw + u * NT + l) / kPageUnits;
    };
    auto unit_in = [&](unsigned l, int u) {
        return kWavePages ? unsigned((64 * uw + u * NT) % kPageUnits) + l : (64u * uw + u * NT + l) % kPageUnits;
    };
    auto has_unit = [&](int u) { return (u + 1) * NT <= kUnits || 64 * uw + u * NT < kUnits; };   // whole waves
    auto load_ids = [&](int tile) {
        const unsigned l = fresh_lane();
        const int page0 = token_of(tile) / kPage;
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            // (pages past the last visible token's: that one again, masked)
            const int v = page0 + unit_page(l, u);
            ids[u] = pt_row[v < n_pages ? v : n_pages - 1];
        }
    };
    auto load_tile = [&]() {
        const unsigned l = fresh_lane();
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (!has_unit(u)) continue;
            const int32_t id = clamp_ids(kWavePages ? __builtin_amdgcn_readfirstlane(ids[u]) : ids[u], p.num_pages);
            const int64_t ph = int64_t(id) * p.num_kv_heads + hk;
            const unsigned in = unit_in(l, u);
            const uint8_t* codes = p.codes + ph * (16 * D);
            const uint8_t* scales = p.scales + ph * D;
            kcode[u] = *reinterpret_cast<const u32x4*>(codes + 16 * in);
            vcode[u] = *reinterpret_cast<const u32x4*>(codes + 8 * D + 16 * in);
            vscale[u] = *reinterpret_cast<const uint32_t*>(scales + D / 2 + (in % (D / 8) >> 2) * 16 + 4 * (in / (D / 8)));
            if (in < D / 8) kscale[u] = *reinterpret_cast<const uint32_t*>(scales + 4 * in);
        }
    };
    auto store_k = [&](int slot) {
        const unsigned l = fresh_lane();
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (!has_unit(u)) continue;
            const unsigned in = unit_in(l, u);
            *reinterpret_cast<u32x4*>(kt(slot) + 16 * (64 * uw + u * NT + l)) = kcode[u];
            if (in < D / 8) *reinterpret_cast<uint32_t*>(kst(slot) + unit_page(l, u) * (D / 2) + 4 * in) = kscale[u];
        }
    };
    // The scale bytes of unit u; tokens that no row of the block sees may hold
    // anything, so theirs become 0.
    static_assert(NT % (D / 8) == 0, "a thread's units are of the same channels");
    auto octet = [&](unsigned l) { return int(l % (D / 8)); };   // (D / 8 divides 64)
    const int seen_from = p.window > 0 ? lo - p.window + 1 : 0;
    auto unit_scales = [&](unsigned l, int tile, int u) {
        const int tok0 = token_of(tile), tok = tok0 + kPage * unit_page(l, u) + 4 * int(unit_in(l, u) / (D / 8));
        uint32_t sc = vscale[u];
        if (tok0 + TT - 1 > hi || (tok0 < seen_from && tok0 + TT > p.sinks)) {
            // seen by some row: up to the last, and in the first row's window or a first token
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (!((tok + t <= hi) & ((tok + t >= seen_from) | (tok + t < p.sinks)))) sc &= ~(0xFFu << (8 * t));
        }
        return sc;
    };
    // Decodes this thread's units into the value buffer, relative to my_base; true
    // if a scale is above the range.
    auto store_v = [&](int tile, int slot) {
        bool above = false;
        const unsigned l = fresh_lane();
        const int oct = octet(l);
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (!has_unit(u)) continue;
            const int pg = unit_page(l, u), tq = int(unit_in(l, u) / (D / 8));
            const uint32_t bytes = unit_scales(l, tile, u);
            // the float 2^(byte - base): the byte at a float's exponent, moved by 127 - base
            // and 0 below the exponent range (a byte above base + 13 may leave it, and
            // the tile is decoded again)
            const uint32_t k23 = 23u;
            const int b[4] = {int(f32_bits(byte_scale0(bytes, k23))), int(f32_bits(byte_scale1(bytes, k23))),
                              int(f32_bits(byte_scale2(bytes, k23))), int(f32_bits(byte_scale3(bytes, k23)))};
            const int shift = (127 - my_base) * (1 << 23), limit = (my_base + 13 < 255 ? my_base + 13 : 255) * (1 << 23);
            float sc[4];
            int most = b[0];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                most = most > b[t] ? most : b[t];
                const int e = int(uint32_t(b[t]) + uint32_t(shift));
                sc[t] = bits_f32(uint32_t(e > 0 ? e : 0));
            }
            above = above || most > limit;
            uint2 out[8];
            decode_unit(vcode[u], sc, out);
            uint8_t* dst = vt(slot) + ((pg * CB + (oct >> 2)) * 2 + (tq & 1)) * kVRow + kVOctet * (oct & 3);
            if constexpr (D <= 128) {
                // the lane of tq ^ 2, D / 4 lanes away, has the other 4 tokens of the 16 bytes:
                // the two exchange, and each stores 4 of the 8 channels (8-byte stores
                // meet in a bank four at a time and took the LDS 4 times as long)
                dst += (tq >> 1) * 64;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint2 a = out[i], b = out[i + 4];
                    const auto x = D == 128 ? __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false)
                                            : __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);
                    const auto y = D == 128 ? __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false)
                                            : __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
                    *reinterpret_cast<uint4*>(dst + 16 * i) = make_uint4(x[0], y[0], x[1], y[1]);
                }
            } else {
                // (that lane is one of another wave)
#pragma unroll
                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint2*>(dst + 8 * (tq >> 1) + 16 * i) = out[i];
            }
        }
        return above;
    };

    const float sl2 = p.scale_log2;
    constexpr float kNoMax = -1e30f;
    float m_run[NQ], l_run[NQ];
    v16f acc[CB][NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        m_run[q] = kNoMax;
        l_run[q] = 0.f;
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[c][q] = v16f(0.f);
    }
    bool big_max = false;   // wave-uniform: a reference of magnitude 2^20 or more (see decode_kernel)

    int credit = kCredit;   // for looking down, wave-uniform

    // Tiles of 128 tokens (head size 64): of one that is partly hidden only the 32s with a
    // visible token are computed, and only those with a hidden one masked (two prompts of
    // 4099, 64 heads over 8, window 1024: 198 us a pass, 245 without; 128: 83, 135; no
    // window: the same).  With tiles of 64 (head size 128) windows gain, 307 us against 321
    // and 135 against 157, and chunks behind long contexts lose, 2314 against 2292: not there.
    constexpr bool kPick = TT > 64;
    auto clear_of = [&](int from, int n) {
        return from + n - 1 <= w_lo && (p.window == 0 || from > w_hi - p.window || from + n <= p.sinks);
    };
    // The wave's rows against the tile in `slot`; `clear`: every row sees all 32 tokens.
    // Masks, rescaling and large maxima are one branch, so that the rest is one
    // block of instructions, in which the exponentials of the second 16 tokens run
    // beside the products of the first.
    auto compute = [&](int tok0, int slot) {
        const unsigned l = fresh_lane(), lh = l >> 5, lc = l & 31;
        const uint8_t* v_at = vt(slot) + lh * kVRow + 16 * lc + (kVOctet - 128) * (lc >> 3);
        const uint8_t* k_at = kt(slot) + (lc >> 4) * (8 * D) + (lh * 16 + (lc & 15)) * 16;
        const uint8_t* s_at = kst(slot) + (lc >> 4) * (D / 2) + lh * 16 + (lc & 15);
        v16f s[NQ];
        auto scores = [&](int tb) {
            uint4 ka[KS];
            int ksc[KS];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                ka[k] = *reinterpret_cast<const uint4*>(k_at + tb * (16 * D) + k * 512);
                ksc[k] = s_at[tb * D + k * 32];
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) s[q] = v16f(0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const v8i a = {int(ka[k].x), int(ka[k].y), int(ka[k].z), int(ka[k].w), 0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < NQ; ++q)
                    s[q] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, qop[q][k], s[q], 4, 0, 0, ksc[k], 0, 127);
            }
        };
        auto tokens = [&](int tb, bool clear) {
            auto load_v = [&](int mm, uint4 (&v)[CB]) {
#pragma unroll
                for (int c = 0; c < CB; ++c) v[c] = *reinterpret_cast<const uint4*>(v_at + ((2 * tb + mm) * CB + c) * 2 * kVRow);
            };
            auto max_of = [&](int q) {
                float mx = __builtin_fmaxf(__builtin_fmaxf(s[q][0], s[q][1]), s[q][2]);
#pragma unroll
                for (int i = 3; i < 15; i += 2) mx = __builtin_fmaxf(__builtin_fmaxf(mx, s[q][i]), s[q][i + 1]);
                return __builtin_fmaxf(mx, s[q][15]);
            };
            auto move = [&](int q, float to) {
                const float alpha = __builtin_amdgcn_exp2f(m_run[q] - to);
                l_run[q] *= alpha;
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[c][q] *= alpha;
                m_run[q] = to;
            };
            // The references of rows with low scores, moved down; true if one was.  (Both lanes
            // of a row decide alike; one that sees none of the 32 stays.)
            auto follow_down = [&]() {
                bool any = false;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    float a = max_of(q), b = a, la = l_run[q], lb = la, least = __builtin_inff();
                    swap32(a, b);
                    swap32(la, lb);
                    const float mloc = __builtin_fmaxf(a, b) * sl2, sum = la + lb;
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        float oa = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) oa = __builtin_fmaxf(oa, __builtin_fabsf(acc[c][q][i]));
                        float ob = oa;
                        swap32(oa, ob);
                        least = __builtin_fminf(least, __builtin_fmaxf(oa, ob));
                    }
                    const bool down = mloc < m_run[q] + kDown && mloc > -__builtin_inff() && sum < kDeep && least < sum * kSmall;
                    if (down) move(q, __builtin_fmaxf(mloc, m_run[q] - kDepth));
                    any = any || __builtin_amdgcn_ballot_w64(down) != 0;
                }
                return any;
            };
            // half the width of the scores' range: kDown .. kUp, or without credit all below kUp
            // (2^20: a score that low adds nothing)
            const bool follow = credit > 0;
            const float width = follow ? 0.5f * (kUp - kDown) : 0x1p20f;
            credit = credit < kCredit ? credit + 1 : credit;
            bool moves = !clear || big_max;
#pragma unroll
            for (int q = 0; q < NQ; ++q)
                moves = __builtin_amdgcn_ballot_w64(__builtin_fabsf(__builtin_fmaf(max_of(q), sl2, (width - kUp) - m_run[q])) > width) != 0 ||
                        moves;
            float scale = sl2, shift[NQ];
            if (__builtin_expect(moves, 0)) {
                big_max = false;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    if (!clear) {
                        // element i: token 8 (i / 4) + 4 half + i % 4 of the 32; it is seen when 0 <=
                        // position - token < window, or among the first tokens
                        const int tok = tok0 + 32 * tb + 4 * int(lh), row = w_row0 + 32 * q + int(lc);
                        const int pos = row >= rows ? -1 : CROSS ? r.n_ctx - 1 : r.n_ctx - r.count + div_group(p, row);
                        const unsigned reach = p.window > 0 ? unsigned(p.window) : 0x80000000u;
                        const int sinks = pos + 1 < p.sinks ? pos + 1 : p.sinks;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int tt = tok + 8 * (i >> 2) + (i & 3);
                            const bool seen = (unsigned(pos - tt) < reach) | (tt < sinks);
                            s[q][i] = seen ? s[q][i] : -__builtin_inff();
                        }
                    }
                    float a = max_of(q), b = a;
                    swap32(a, b);
                    const float mloc = __builtin_fmaxf(a, b) * sl2;
                    if (mloc > m_run[q] + kUp) move(q, mloc - kLead);
                    big_max = big_max || __builtin_amdgcn_ballot_w64(__builtin_fabsf(m_run[q]) >= 0x1p20f && m_run[q] != kNoMax) != 0;
                }
                if (follow) {
                    bool low = false;
#pragma unroll
                    for (int q = 0; q < NQ; ++q) {
                        const float a = max_of(q);
                        low = low || __builtin_amdgcn_ballot_w64(a * sl2 < m_run[q] + kDown && a > -__builtin_inff()) != 0;
                    }
                    if (low) credit -= follow_down() ? kCostMoved : kCostIdle;
                }
            }
#pragma unroll
            for (int q = 0; q < NQ; ++q) shift[q] = kLift - m_run[q];
            if (__builtin_expect(big_max, 0)) {
                // the difference to the rounded product, as m_run is one less kLead
#pragma clang fp contract(off)
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[q][i] = s[q][i] * sl2 - m_run[q];
                    shift[q] = kLift;
                }
                scale = 1.f;
            }
            // P of tokens 16 mm .. 16 mm + 15 as operand B, cut to FP16 (the conversion that
            // rounds to nearest takes twice as long, and the sum of pairs by a dot product
            // shuts out the matrix instructions).  kLift, in the shift, makes up for the
            // mean of what is cut; the sum, of the lifted weights, is lowered at the end.
            auto weights = [&](int mm, uint4 (&ph)[NQ]) {
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][8 * mm + 2 * i], scale, shift[q]));
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][8 * mm + 2 * i + 1], scale, shift[q]));
                        w[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));
                        l_run[q] += x + y;
                    }
                    ph[q] = uint4{w[0], w[1], w[2], w[3]};
                }
            };
            auto values = [&](const uint4 (&v)[CB], const uint4 (&ph)[NQ]) {
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
                        acc[c][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, v[c]),
                                                                           __builtin_bit_cast(v8h, ph[q]), acc[c][q], 0, 0, 0);
            };
            uint4 p0[NQ], p1[NQ], va[CB], vb[CB];
            load_v(0, va);
            weights(0, p0);
            load_v(1, vb);
            values(va, p0);
            weights(1, p1);
            values(vb, p1);
        };
        const bool clear = clear_of(tok0, TT);
        // of a tile that is not clear only the 32s that a row of the wave sees
        int tb_from = 0, tb_end = TT / 32;
        if (kPick && !clear) {
            tb_end = (w_hi - tok0) / 32 + 1;
            if (p.window > 0) {
                const int from = w_lo - p.window + 1 - tok0;   // first token of the windows, in the tile
                if (tok0 >= p.sinks) tb_from = from > 0 ? from / 32 : 0;
                else if (from >= TT) tb_end = (p.sinks - tok0 + 31) / 32 < tb_end ? (p.sinks - tok0 + 31) / 32 : tb_end;
            }
        }
        scores(0);
#pragma unroll
        for (int tb = 0; tb < TT / 32; ++tb) {
            if (!kPick || (tb >= tb_from && tb < tb_end)) tokens(tb, kPick ? clear || clear_of(tok0 + 32 * tb, 32) : clear);
            if (tb + 1 < TT / 32) scores(tb + 1);
        }
    };

    // The exponents from the largest scales of the tile whose units this thread
    // holds, the accumulators rescaled to them.
    auto set_base = [&](int tile) {
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (!has_unit(u)) continue;
            const uint32_t bytes = unit_scales(lane, tile, u);
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicMax(&top[octet(lane) >> 2], int((bytes >> (8 * i)) & 0xFFu));
        }
        sync();
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int old = base[c], now = top[c] - 8 > old ? top[c] - 8 : old;
            const float f = old == kNoBase ? 0.0f : __builtin_ldexpf(1.0f, old - now);   // (1 where nothing changes)
#pragma unroll
            for (int q = 0; q < NQ; ++q) acc[c][q] *= f;
        }
        my_base = top[octet(lane) >> 2] - 8 > my_base ? top[octet(lane) >> 2] - 8 : my_base;
        sync();
        if (wtid < CB) {
            base[wtid] = top[wtid] - 8 > base[wtid] ? top[wtid] - 8 : base[wtid];
            top[wtid] = 0;
        }
    };

    // ---- the walk.  While a tile is computed, the walker's next is on its way into
    // registers and the page ids of the one after too.  (Past the last tile in pages
    // that exist.)  Nobody is left in the tile before the last when a tile is stored
    // to its buffers.
    if constexpr (ALONE) first_tile += wave;
    if (first_tile < last_tile) {
        load_ids(first_tile);
        load_tile();
        load_ids(first_tile + STEP);
        set_base(first_tile);
    }
    for (int t = first_tile, slot = 0; t < last_tile; t += STEP, slot ^= ALONE ? 0 : 1) {
        store_k(slot);
        if (store_v(t, slot)) grow[slot] = 1;
        sync();
        if (__builtin_expect(grow[slot] != 0, 0)) {
            // rare: a scale above the range.  The tile is decoded again.
            sync();
            if (wtid == 0) grow[slot] = 0;
            set_base(t);
            store_v(t, slot);
            sync();
        }
        load_tile();
        load_ids(t + 2 * STEP);
        const int tok0 = token_of(t);
        // tiles past the wave's last row, or before its windows and after the sinks
        if (!busy || tok0 > w_hi || (p.window > 0 && tok0 + TT <= w_lo - p.window + 1 && tok0 >= p.sinks)) continue;
        compute(tok0, slot);
    }

    // ---- the row's sum over both halves, the accumulators divided by it and back to
    // O, then the row itself or its partial.  (Parts of a row are averages with their
    // sums as weights, so that no finite result overflows on the way.)
    if (!ALONE && !busy) return;
    float back[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c) back[c] = base[c] == kNoBase ? 0.0f : __builtin_ldexpf(1.0f, base[c] - 127);
    float l_row[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        float a = l_run[q], b = l_run[q];
        swap32(a, b);
        l_row[q] = (a + b) * kLower;
        const float inv = l_row[q] > 0.f ? 1.0f / l_row[q] : 0.f;   // a row that sees nothing is 0
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[c][q] = acc[c][q] * inv * back[c];
    }
    if constexpr (ALONE) {
        // the waves' parts of the rows, one after another through LDS into wave 0's
        float4* const part = reinterpret_cast<float4*>(smem);
        float2* const ml = reinterpret_cast<float2*>(smem + CB * NQ * 4 * 1024);
        static_assert(CB * NQ * 4 * 1024 + NQ * 512 <= Shape::kLds, "a wave's part fits");
        for (int w = 1; w < W; ++w) {
            __syncthreads();
            if (wave == w) {
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
#pragma unroll
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            part[((q * CB + c) * 4 + i) * 64 + lane] =
                                make_float4(acc[c][q][4 * i], acc[c][q][4 * i + 1], acc[c][q][4 * i + 2], acc[c][q][4 * i + 3]);
                    ml[q * 64 + lane] = make_float2(m_run[q], l_row[q]);
                }
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float2 o = ml[q * 64 + lane];
                    const float g = join_share(m_run[q], l_row[q], o.x, o.y);
#pragma unroll
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 x = part[((q * CB + c) * 4 + i) * 64 + lane];
                            acc[c][q][4 * i] = acc[c][q][4 * i] * (1.0f - g) + x.x * g;
                            acc[c][q][4 * i + 1] = acc[c][q][4 * i + 1] * (1.0f - g) + x.y * g;
                            acc[c][q][4 * i + 2] = acc[c][q][4 * i + 2] * (1.0f - g) + x.z * g;
                            acc[c][q][4 * i + 3] = acc[c][q][4 * i + 3] * (1.0f - g) + x.w * g;
                        }
                }
            }
        }
        if (wave != 0) return;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const float l = l_row[q];
        const int row = w_row0 + 32 * q + col;
        const int tok = div_group(p, row);
        const int64_t out_row = int64_t(r.first + tok) * p.num_q_heads + hk * p.group + (row - tok * p.group);
        if (!whole) {
            if (row < rows) {
                const int64_t part = int64_t(r.split) * p.num_tokens * p.num_q_heads + out_row;
#pragma unroll
                for (int c = 0; c < CB; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4*>(p.part_acc + part * D + 32 * c + 8 * i + 4 * half) =
                            make_float4(acc[c][q][4 * i], acc[c][q][4 * i + 1], acc[c][q][4 * i + 2], acc[c][q][4 * i + 3]);
                if (half == 0) *reinterpret_cast<float2*>(p.part_ml + part * 2) = make_float2(m_run[q], l);
            }
            continue;
        }
        gather_columns(acc, q, p.rotate_v != 0);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                const v16f& o = acc[c][q];
                const int64_t at = out_row * D + 32 * c + 2 * i + 8 * half;
                if (row >= rows) continue;
                if (p.out_dtype == 0) {
                    float4* dst = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
                    dst[0] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    dst[1] = make_float4(o[i + 4], o[i + 5], o[i + 6], o[i + 7]);
                } else {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at) =
                        uint4{pack_bf16x2(o[i], o[i + 1]), pack_bf16x2(o[i + 2], o[i + 3]), pack_bf16x2(o[i + 4], o[i + 5]),
                              pack_bf16x2(o[i + 6], o[i + 7])};
                }
            }
    }
}

// MIXED: sequences with up to p.alone_rows rows of a KV head are walked by waves that
// split the tokens.  (Both walks in one kernel cost the other some registers, so it
// is a kernel of its own.)
template <int D, int NQ, int W, bool MIXED, bool CROSS>
__global__ void __launch_bounds__(64 * W, 2) extend_kernel(ExtendParams p) {
    constexpr int kTogetherLds = ExtendShape<D, W, false>::kLds, kAloneLds = MIXED ? ExtendShape<D, W, true>::kLds : 0;
    __shared__ __attribute__((aligned(16))) uint8_t smem[kTogetherLds > kAloneLds ? kTogetherLds : kAloneLds];
    const int hk = int(blockIdx.x % unsigned(p.num_kv_heads));
    const int rest = int(blockIdx.x / unsigned(p.num_kv_heads));
    constexpr int M = 32 * NQ * W;
    ExtendRows r;
    if constexpr (MIXED) {
        if (p.share != nullptr) {
            const bool found = extend_find_share<M, extend_tile<D>(), ExtendShape<D, W, true>::TT>(p, rest, r);
            if (blockIdx.x == 0 && threadIdx.x == 0) *p.share = r.share;   // for the join
            if (!found) return;
        } else if (!extend_find_split<M, CROSS>(p, rest, r)) {
            return;
        }
        if (r.count * p.group <= p.alone_rows) {
            extend_walk<D, 2, W, true, CROSS>(p, r, hk, smem);
            return;
        }
    } else if (!extend_find_split<M, CROSS>(p, rest, r)) {
        return;
    }
    extend_walk<D, NQ, W, false, CROSS>(p, r, hk, smem);
}

// Joins the partials of every (token, query head): 16 lanes per row, N channels
// each.
template <int D, int M, bool CROSS>
__global__ void __launch_bounds__(256) extend_merge_kernel(ExtendParams p) {
    constexpr int N = D / 16;
    const int L = threadIdx.x & 15;
    const int64_t row = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4);
    const int t = int(row / p.num_q_heads);
    if (t >= p.num_tokens) return;   // whole 16-lane rows
    const int hq = int(row - int64_t(t) * p.num_q_heads);
    // the sequence of token row t: the last that starts at or before it
    int lo = 0, hi = p.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (extend_first(p, mid) <= t) lo = mid; else hi = mid;
    }
    ExtendRows r;
    r.b = lo;
    r.first = extend_first(p, lo);
    r.count = extend_first(p, lo + 1) - r.first;
    if (t < r.first || t >= r.first + r.count) return;
    r.n_ctx = extend_context(p, lo);
    r.row0 = ((t - r.first) * p.group + hq % p.group) / M * M;
    int plo, phi;
    extend_span<M, CROSS>(p, r, plo, phi);
    constexpr int TT = extend_tile<D>(), TA = ExtendShape<D, 4, true>::TT;
    const int share = p.share != nullptr ? *p.share : 0;
    int per;
    if (r.count * p.group <= p.alone_rows) {
        extend_tiles<TA>(p, plo, phi, r);
        per = extend_per_split<TA>(r.tiles, p.splits, share);
    } else {
        extend_tiles<TT>(p, plo, phi, r);
        per = extend_per_split<TT>(r.tiles, p.splits, share);
    }
    if (r.tiles <= per) return;   // written by the first launch
    const int parts = (r.tiles + per - 1) / per;
    const int64_t step = int64_t(p.num_tokens) * p.num_q_heads;
    float m = -3e38f, l = 0.f, o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
#pragma unroll 4
    for (int s = 0; s < parts; ++s) {
        const int64_t at = s * step + row;
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
        float a[N];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(p.part_acc + at * D + N * L + 4 * i);
            a[4 * i] = v.x;
            a[4 * i + 1] = v.y;
            a[4 * i + 2] = v.z;
            a[4 * i + 3] = v.w;
        }
        const float g = join_share(m, l, ml.x, ml.y);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * (1.0f - g) + a[i] * g;
    }
    if (p.rotate_v) wht_x<N>(o, L);
    const int64_t at = row * D + N * L;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        if (p.out_dtype == 0)
            *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at + 4 * i) =
                make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        else
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at + 4 * i) =
                make_uint2(pack_bf16x2(o[4 * i], o[4 * i + 1]), pack_bf16x2(o[4 * i + 2], o[4 * i + 3]));
    }
}

template <int D, int NQ, int W, bool CROSS>
static hipError_t launch_extend_with(const ExtendParams& p, hipStream_t stream) {
    const dim3 grid{unsigned(int64_t(p.row_blocks) * p.num_kv_heads * (p.share != nullptr ? 1 : p.splits))}, block{64u * W};
    if (p.alone_rows > 0) {
        if constexpr (D <= 128) launch_kernel(extend_kernel<D, NQ, W, true, CROSS>, grid, block, stream, p);
        else return hipErrorInvalidValue;   // (not asked for)
    } else {
        launch_kernel(extend_kernel<D, NQ, W, false, CROSS>, grid, block, stream, p);
    }
    if (p.splits > 1) {
        const int64_t rows = int64_t(p.num_tokens) * p.num_q_heads;
        hipLaunchKernelGGL((extend_merge_kernel<D, 32 * NQ * W, CROSS>), dim3(unsigned((rows + 15) / 16)), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

int extend_block_rows(int head_dim) { return head_dim == 256 ? 128 : 256; }
int extend_alone_rows(int head_dim) { return head_dim == 256 ? 0 : 64; }

template <bool CROSS>
static hipError_t launch_extend_as(const ExtendParams& p, hipStream_t stream) {
    if (p.head_dim == 64) return launch_extend_with<64, 2, 4, CROSS>(p, stream);
    if (p.head_dim == 128) return launch_extend_with<128, 2, 4, CROSS>(p, stream);
    return launch_extend_with<256, 1, 4, CROSS>(p, stream);
}

hipError_t launch_extend(const ExtendParams& p, hipStream_t stream) {
    return p.cross ? launch_extend_as<true>(p, stream) : launch_extend_as<false>(p, stream);
}

}  // namespace uq
