// uq_weights.hpp -- the attention weight of every cached token (uq_token_weights
// of include/uq.h), part of the uq_quantize.hip translation unit.
//
// A row is a (query, query head of a KV head) pair of a sequence, row r = query
// r / G, head r % G.  Its scores s_t over the visible tokens give the softmax
// weights p_t = 2^(c s_t - m) / l, c = scale log2 e, and token t gets the sum of
// its weights over all rows.  Weights of different rows add up only when they are
// normalised, so the keys are read twice:
//
//   token_norms   m and l of every row.  A wave holds 16 NB rows as operand B and
//                 walks the tokens of a chunk; keys are operand A, so a lane sees
//                 4 tokens of one row and needs no exchange until the end.
//   token_sums    the sums.  A wave holds P units of keys as operand B and walks
//                 the rows, which are operand A: a lane sees 4 rows of one token
//                 and adds in its register.
//
// A page's key tile is [channels / 32][token][16 bytes], which is operand order of
// v_mfma_scale_f32_16x16x128_f8f6f4 (lane: token l % 16, 32 channels l / 16), and so
// are its scale bytes: keys go from memory to the matrix instruction with one
// 16-byte load per lane and no LDS.  FP8 query rows are two such loads.  Head size
// 64 takes two pages into one operand and half of the query operand is zero; head
// size 256 takes two instructions per page.
//
// Every sum has a fixed order: results do not depend on what else runs.
#pragma once

#include "uq_device.hpp"
#include "uq_internal.hpp"

namespace uq {

constexpr float kNoRow = -1e30f;      // reference of a row that has seen no token
constexpr float kMaskedRow = 3e38f;   // reference that makes every weight 0
constexpr float kRefSlack = 8.0f;     // powers of two a score may pass the reference
constexpr float kBigRef = 0x1p20f;    // from here on c s is rounded before the reference is taken off

// Keys of 16 tokens (32 at head size 64) as operand bytes.
template <int D> struct KeyUnit {
    static constexpr int kSteps = D == 256 ? 2 : 1;
    static constexpr int kPages = D == 64 ? 2 : 1;
    static constexpr int kTiles = kPages;            // 16x16 results per 16 rows
    static constexpr int kTokens = kPage * kPages;
    u32x4 code[kSteps];
    int scale[kSteps];
};

// 16 rows of FP8 queries as operand bytes.
template <int D> struct RowUnit {
    u32x4 lo[D == 256 ? 2 : 1], hi[D == 64 ? 1 : D == 256 ? 2 : 1];
};

__device__ __forceinline__ v8i join_halves(const u32x4& a, const u32x4& b) {
    return v8i{int(a[0]), int(a[1]), int(a[2]), int(a[3]), int(b[0]), int(b[1]), int(b[2]), int(b[3])};
}

// The row operand of result tile `tile` and step `s`.
template <int D>
__device__ __forceinline__ v8i row_operand(const RowUnit<D>& q, int tile, int s) {
    const u32x4 none = {0u, 0u, 0u, 0u};
    if constexpr (D == 64) return tile == 0 ? join_halves(q.lo[0], none) : join_halves(none, q.lo[0]);
    else return join_halves(q.lo[s], q.hi[s]);
}
template <int D>
__device__ __forceinline__ v8i key_operand(const KeyUnit<D>& k, int s) {
    const u32x4 none = {0u, 0u, 0u, 0u};
    return join_halves(k.code[s], none);
}

// Scores of 16 tokens (tile of the unit) against 16 rows: result row = token,
// column = row (TOKEN_ROWS), or the other way round.
template <int D, bool TOKEN_ROWS>
__device__ __forceinline__ v4f unit_scores(const KeyUnit<D>& k, const RowUnit<D>& q, int tile) {
    v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KeyUnit<D>::kSteps; ++i) {
        const v8i ko = key_operand<D>(k, i), qo = row_operand<D>(q, tile, i);
        if constexpr (TOKEN_ROWS)
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ko, qo, s, 4, 0, 0, k.scale[i], 0, 127);
        else
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(qo, ko, s, 0, 4, 0, 127, 0, k.scale[i]);
    }
    return s;
}

// A sequence's rows: its last `use` queries, first token row `first`, and context n.
struct WeightsSeq {
    int first, use, n;
};
__device__ __forceinline__ WeightsSeq weights_seq(const WeightsParams& p, int b) {
    auto row = [&](int i) {
        const int x = p.cu_seqlens[i];
        return x < 0 ? 0 : x < p.num_tokens ? x : p.num_tokens;
    };
    const int from = row(b), end = row(b + 1);
    int use = end > from ? end - from : 0;
    if (p.last > 0 && use > p.last) use = p.last;
    int n = p.context_lens[b];
    n = n < p.max_context ? n : p.max_context;
    return {end - use, use, n > 0 ? n : 0};
}
// Position of a sequence's first query; query i stands i behind it, or with no
// order all at the last token.
__device__ __forceinline__ int first_position(const WeightsParams& p, const WeightsSeq& s) {
    return p.causal ? s.n - s.use : s.n - 1;
}
// Index of a sequence's first row in the per-row arrays.
__device__ __forceinline__ int64_t first_row(const WeightsParams& p, int b, const WeightsSeq& s, int hk) {
    return int64_t(hk) * p.rows_per_head + int64_t(p.by_seq ? b * p.last : s.first) * p.group;
}
__device__ __forceinline__ int weights_div(const WeightsParams& p, int n) {
    return p.group == 1 ? n : int(__umulhi(unsigned(n), p.group_magic));   // exact for n < 2^28
}

// Items of the batch in ascending order, 64 sequences at a time, one per lane: a
// wave's items ascend, so that every sequence is looked at once.
struct ItemFinder {
    int b0 = -64, before = 0, all = 0;
    int items = 0, sum = 0;      // of this lane's sequence, and up to it
    WeightsSeq seq = {0, 0, 0};
    template <class COUNT>
    __device__ __forceinline__ bool find(const WeightsParams& p, int at, COUNT count, int& b, int& idx, WeightsSeq& s) {
        const int lane = threadIdx.x & 63;
        while (at >= before + all) {
            before += all;
            b0 += 64;
            if (b0 >= p.batch) return false;
            seq = {0, 0, 0};
            if (b0 + lane < p.batch) seq = weights_seq(p, b0 + lane);
            items = b0 + lane < p.batch ? count(seq) : 0;
            sum = items;
#pragma unroll
            for (int i = 1; i < 64; i <<= 1) {
                const int o = __shfl_up(sum, i);
                if (lane >= i) sum += o;
            }
            all = __builtin_amdgcn_readlane(sum, 63);
        }
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + sum > at));
        b = b0 + l;
        idx = at - before - __builtin_amdgcn_readlane(sum - items, l);
        s = {__builtin_amdgcn_readlane(seq.first, l), __builtin_amdgcn_readlane(seq.use, l),
             __builtin_amdgcn_readlane(seq.n, l)};
        return true;
    }
};

// Page ids of a sequence, 64 at a time.
struct PageIds {
    int ids = 0, from = -1;
    __device__ __forceinline__ void load(const WeightsParams& p, int b, int page, int pages) {
        const int i = page + int(threadIdx.x & 63);
        from = page;
        ids = p.page_table[int64_t(b) * p.max_pages_per_seq + (i < pages ? i : pages - 1)];
        ids = ids >= 0 && int64_t(ids) < p.num_pages ? ids : 0;
    }
    __device__ __forceinline__ int at(int page) const { return __builtin_amdgcn_readlane(ids, page - from); }
};

// Unit `u` of a sequence (its pages among the loaded ids): tokens at n and behind
// may never have been written, and their scale bytes become 0.
template <int D>
__device__ __forceinline__ void load_keys(const WeightsParams& p, const PageIds& ids, int hk, int u, int pages, KeyUnit<D>& k) {
    const int lane = threadIdx.x & 63;
    if constexpr (D == 64) {
        const int a = ids.at(2 * u), c = ids.at(2 * u + 1 < pages ? 2 * u + 1 : 2 * u);
        const int64_t ph = int64_t(lane < 32 ? a : c) * p.num_kv_heads + hk;
        k.code[0] = *reinterpret_cast<const u32x4*>(p.codes + ph * (16 * D) + 16 * (lane & 31));
        k.scale[0] = p.scales[ph * D + (lane & 31)];
    } else {
        const int64_t ph = int64_t(ids.at(u)) * p.num_kv_heads + hk;
        const uint8_t* codes = p.codes + ph * (16 * D);
        const uint8_t* scales = p.scales + ph * D;
#pragma unroll
        for (int i = 0; i < KeyUnit<D>::kSteps; ++i) {
            k.code[i] = *reinterpret_cast<const u32x4*>(codes + 1024 * i + 16 * lane);
            k.scale[i] = scales[64 * i + lane];
        }
    }
}
template <int D>
__device__ __forceinline__ void hide_unwritten(KeyUnit<D>& k, int u, int n) {
    const int lane = threadIdx.x & 63;
    const int t = u * KeyUnit<D>::kTokens + (D == 64 ? (lane >> 5) * kPage : 0) + (lane & 15);
#pragma unroll
    for (int i = 0; i < KeyUnit<D>::kSteps; ++i) k.scale[i] = t < n ? k.scale[i] : 0;
}

// The row that this lane holds of the 16 from r0 on, clamped to the last.
template <int D>
__device__ __forceinline__ void load_rows(const WeightsParams& p, const WeightsSeq& s, int hk, int r0, int rows, RowUnit<D>& q) {
    const int lane = threadIdx.x & 63;
    int r = r0 + (lane & 15);
    r = r < rows ? r : rows - 1;
    const int i = weights_div(p, r);
    const uint8_t* at = p.q + int64_t(s.first + i) * p.q_stride + int64_t(hk * p.group + r - i * p.group) * D + 16 * (lane >> 4);
    q.lo[0] = *reinterpret_cast<const u32x4*>(at);
    if constexpr (D >= 128) q.hi[0] = *reinterpret_cast<const u32x4*>(at + 64);
    if constexpr (D == 256) {
        q.lo[1] = *reinterpret_cast<const u32x4*>(at + 128);
        q.hi[1] = *reinterpret_cast<const u32x4*>(at + 192);
    }
}

// c s - m: fused, or where m is large from the rounded product, as m is one.
__device__ __forceinline__ float above_ref(float s, float c, float m, bool big) {
#pragma clang fp contract(off)
    return big ? s * c - m : __builtin_fmaf(s, c, -m);
}

// Row blocks of 16 NB rows times chunks of p.chunk tokens, a wave each: the row's
// reference and sum over the chunk, or (one chunk) the reference and 1 / sum.
template <int D, int NB>
__global__ void __launch_bounds__(256) token_norms_kernel(WeightsParams p) {
    using Unit = KeyUnit<D>;
    constexpr int TOK = Unit::kTokens, PF = 4;
    const int lane = threadIdx.x & 63, grp = lane >> 4;
    const int waves = int(gridDim.x) * 4;
    const int units_per_chunk = p.chunk / TOK;
    auto count = [&](const WeightsSeq& s) {
        const int rows = s.use * p.group;
        return p.num_kv_heads * ((rows + 16 * NB - 1) / (16 * NB)) * ((s.n + p.chunk - 1) / p.chunk);
    };
    ItemFinder items;
    int b, idx;
    WeightsSeq s;
    for (int at = int(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); items.find(p, at, count, b, idx, s);
         at += waves) {
        const int rows = s.use * p.group, blocks = (rows + 16 * NB - 1) / (16 * NB), chunks = (s.n + p.chunk - 1) / p.chunk;
        const int rest = idx / blocks, r0 = (idx - rest * blocks) * (16 * NB);
        const int hk = rest / chunks, chunk = rest - hk * chunks;
        const int pos0 = first_position(p, s);
        const int r1 = r0 + 16 * NB < rows ? r0 + 16 * NB - 1 : rows - 1;     // the block's last row
        const int lo = p.causal ? pos0 + weights_div(p, r0) : pos0, hi = p.causal ? pos0 + weights_div(p, r1) : pos0;
        RowUnit<D> q[NB];
        float m[NB], l[NB];
        int pos[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            load_rows<D>(p, s, hk, r0 + 16 * j, rows, q[j]);
            const int r = r0 + 16 * j + (lane & 15) < rows ? r0 + 16 * j + (lane & 15) : rows - 1;
            pos[j] = p.causal ? pos0 + weights_div(p, r) : pos0;
            m[j] = kNoRow;
            l[j] = 0.f;
        }
        // units of the chunk up to the last that a row of the block sees
        const int u0 = chunk * units_per_chunk;
        int u1 = hi >= 0 ? hi / TOK + 1 : 0;
        u1 = u1 < u0 + units_per_chunk ? u1 : u0 + units_per_chunk;
        const int pages = (s.n + kPage - 1) / kPage;
        bool big = false;
        auto use_unit = [&](const Unit& k, int u) {
#pragma unroll
            for (int t = 0; t < Unit::kTiles; ++t) {
                const int t0 = u * TOK + kPage * t;
                v4f x[NB];
                bool up = false;
#pragma unroll
                for (int j = 0; j < NB; ++j) x[j] = unit_scores<D, true>(k, q[j], t);
                if (t0 + kPage - 1 > lo) {
#pragma unroll
                    for (int j = 0; j < NB; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[j][i] = t0 + 4 * grp + i <= pos[j] ? x[j][i] : -__builtin_inff();
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float mx = __builtin_fmaxf(__builtin_fmaxf(x[j][0], x[j][1]), __builtin_fmaxf(x[j][2], x[j][3]));
                    up = up || mx * p.scale_log2 > m[j] + kRefSlack;
                }
                if (__builtin_amdgcn_ballot_w64(up) != 0) {
                    big = false;
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const float mx = __builtin_fmaxf(__builtin_fmaxf(x[j][0], x[j][1]), __builtin_fmaxf(x[j][2], x[j][3])) * p.scale_log2;
                        if (mx > m[j] + kRefSlack) {
                            l[j] *= __builtin_amdgcn_exp2f(m[j] - mx);
                            m[j] = mx;
                        }
                        big = big || __builtin_amdgcn_ballot_w64(__builtin_fabsf(m[j]) >= kBigRef && m[j] != kNoRow) != 0;
                    }
                }
                // (a row that has seen nothing yet: -inf - -1e30 is -inf still)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) l[j] += __builtin_amdgcn_exp2f(above_ref(x[j][i], p.scale_log2, m[j], big));
            }
        };
        for (int u = u0; u < u1;) {
            // up to 64 pages' ids at once
            PageIds ids;
            ids.load(p, b, u * Unit::kPages, pages);
            const int end = u + 64 / Unit::kPages < u1 ? u + 64 / Unit::kPages : u1;
            Unit cur[PF], nxt[PF];
#pragma unroll
            for (int i = 0; i < PF; ++i) load_keys<D>(p, ids, hk, u + i < end ? u + i : end - 1, pages, cur[i]);
            for (; u < end; u += PF) {
#pragma unroll
                for (int i = 0; i < PF; ++i) load_keys<D>(p, ids, hk, u + PF + i < end ? u + PF + i : end - 1, pages, nxt[i]);
#pragma unroll
                for (int i = 0; i < PF; ++i) {
                    if (u + i < end) {
                        hide_unwritten<D>(cur[i], u + i, s.n);
                        use_unit(cur[i], u + i);
                    }
                }
#pragma unroll
                for (int i = 0; i < PF; ++i) cur[i] = nxt[i];
            }
            u = end;
        }
        // the four lane groups' parts of a row
#pragma unroll
        for (int j = 0; j < NB; ++j) {
#pragma unroll
            for (int x = 16; x < 64; x <<= 1) {
                const float mo = __shfl_xor(m[j], x), lo2 = __shfl_xor(l[j], x);
                const float top = __builtin_fmaxf(m[j], mo);
                l[j] = l[j] * __builtin_amdgcn_exp2f(m[j] - top) + lo2 * __builtin_amdgcn_exp2f(mo - top);
                m[j] = top;
            }
            const int r = r0 + 16 * j + lane;
            if (lane < 16 && r < rows) {
                const int64_t row = first_row(p, b, s, hk) + r;
                if (p.chunks > 1) {
                    *reinterpret_cast<float2*>(p.parts + 2 * (int64_t(chunk) * p.rows_per_head * p.num_kv_heads + row)) = make_float2(m[j], l[j]);
                } else {
                    p.ref[row] = l[j] > 0.f ? m[j] : kMaskedRow;
                    p.inv[row] = l[j] > 0.f ? 1.0f / l[j] : 0.f;
                }
            }
        }
    }
}

// The chunks' references and sums of every row into one: 4 lanes per row.
__global__ void __launch_bounds__(256) token_norms_join_kernel(WeightsParams p) {
    const int64_t row = int64_t(blockIdx.x) * 64 + (threadIdx.x >> 2);
    const int64_t all = p.rows_per_head * p.num_kv_heads;
    if (row >= all) return;   // whole quads
    // the sequence of the row: the last that starts at or before it
    const int64_t in_head = row % p.rows_per_head;
    const int tok = int(in_head / p.group);
    int b;
    WeightsSeq s;
    bool real;
    if (p.by_seq) {
        b = tok / p.last;
        s = weights_seq(p, b);
        real = tok - b * p.last < s.use;
    } else {
        int lo = 0, hi = p.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu_seqlens[mid] <= tok) lo = mid; else hi = mid;
        }
        b = lo;
        s = weights_seq(p, b);
        real = tok >= s.first && tok < s.first + s.use;
    }
    if (!real) return;
    const int chunks = (s.n + p.chunk - 1) / p.chunk;
    float m = kNoRow, l = 0.f;
#pragma unroll 4
    for (int c = int(threadIdx.x & 3); c < chunks; c += 4) {
        const float2 x = *reinterpret_cast<const float2*>(p.parts + 2 * (c * all + row));
        const float top = __builtin_fmaxf(m, x.x);
        l = l * __builtin_amdgcn_exp2f(m - top) + x.y * __builtin_amdgcn_exp2f(x.x - top);
        m = top;
    }
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
        const float mo = __shfl_xor(m, x), lo2 = __shfl_xor(l, x);
        const float top = __builtin_fmaxf(m, mo);
        l = l * __builtin_amdgcn_exp2f(m - top) + lo2 * __builtin_amdgcn_exp2f(mo - top);
        m = top;
    }
    if ((threadIdx.x & 3) == 0) {
        p.ref[row] = l > 0.f ? m : kMaskedRow;
        p.inv[row] = l > 0.f ? 1.0f / l : 0.f;
    }
}

// Four floats at any 4-byte boundary.
struct __attribute__((packed, aligned(4))) Float4At4 {
    float v[4];
};

// Groups of P units of keys times splits of p.row_split rows, a wave each.
template <int D, int P>
__global__ void __launch_bounds__(256) token_sums_kernel(WeightsParams p) {
    using Unit = KeyUnit<D>;
    constexpr int TOK = Unit::kTokens, N = P * Unit::kTiles;
    const int lane = threadIdx.x & 63, grp = lane >> 4;
    const int waves = int(gridDim.x) * 4;
    auto splits_of = [&](const WeightsSeq& s) {
        const int rows = s.use * p.group;
        return rows > 0 ? (rows - 1) / p.row_split + 1 : 0;
    };
    auto count = [&](const WeightsSeq& s) { return p.num_kv_heads * splits_of(s) * ((s.n + P * TOK - 1) / (P * TOK)); };
    ItemFinder items;
    int b, idx;
    WeightsSeq s;
    for (int at = int(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); items.find(p, at, count, b, idx, s);
         at += waves) {
        const int groups = (s.n + P * TOK - 1) / (P * TOK), splits = splits_of(s), rows = s.use * p.group;
        const int rest = idx / groups, u0 = (idx - rest * groups) * P;
        const int hk = rest / splits, split = rest - hk * splits;
        const int pages = (s.n + kPage - 1) / kPage, last_unit = (s.n - 1) / TOK;
        PageIds ids;
        ids.load(p, b, u0 * Unit::kPages, pages);
        Unit k[P];
#pragma unroll
        for (int u = 0; u < P; ++u) load_keys<D>(p, ids, hk, u0 + u < last_unit ? u0 + u : last_unit, pages, k[u]);
        // this lane's tokens of the result: 4 lane groups write a quarter of the tiles each
        float* const out = p.splits > 1 ? p.parts + ((int64_t(split) * p.batch + b) * p.num_kv_heads + hk) * p.max_context
                                        : p.weights + (int64_t(b) * p.num_kv_heads + hk) * p.width;
        const int pos0 = first_position(p, s);
        const int tok0 = u0 * TOK, tok1 = tok0 + P * TOK - 1 < s.n ? tok0 + P * TOK - 1 : s.n - 1;
        // rows from `from` on see a token, from `clear` on all of them
        auto rows_to = [&](int t) {
            const int i = t - pos0;
            return !p.causal || i <= 0 ? 0 : (i < s.use ? i : s.use) * p.group;
        };
        int r0 = rows_to(tok0) & ~15;
        r0 = r0 > split * p.row_split ? r0 : split * p.row_split;
        const int end = (split + 1) * p.row_split < rows ? (split + 1) * p.row_split : rows;
        const int clear = rows_to(tok1);
        const int64_t base = first_row(p, b, s, hk);
        float acc[N];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll
        for (int u = 0; u < P; ++u) hide_unwritten<D>(k[u], u0 + u, s.n);
        RowUnit<D> q;
        Float4At4 ref, inv;
        auto load = [&](int r, RowUnit<D>& qq, Float4At4& a, Float4At4& c) {
            load_rows<D>(p, s, hk, r, rows, qq);
            a = *reinterpret_cast<const Float4At4*>(p.ref + base + r + 4 * grp);
            c = *reinterpret_cast<const Float4At4*>(p.inv + base + r + 4 * grp);
        };
        if (r0 < end) load(r0, q, ref, inv);
        for (; r0 < end; r0 += 16) {
            RowUnit<D> qn;
            Float4At4 refn, invn;
            load(r0 + 16 < end ? r0 + 16 : r0, qn, refn, invn);
            bool big = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (rows behind the last: memory that no row owns)
                const bool real = r0 + 4 * grp + i < rows;
                ref.v[i] = real ? ref.v[i] : kMaskedRow;
                inv.v[i] = real ? inv.v[i] : 0.f;
                big = big || (real && __builtin_fabsf(ref.v[i]) >= kBigRef);
            }
            big = __builtin_amdgcn_ballot_w64(big) != 0;
            const bool masked = r0 < clear;
#pragma unroll
            for (int u = 0; u < P; ++u)
#pragma unroll
                for (int t = 0; t < Unit::kTiles; ++t) {
                    const v4f x = unit_scores<D, false>(k[u], q, t);
                    float e[4];
                    if (__builtin_expect(masked || big, 0)) {
                        const int seen = rows_to((u0 + u) * TOK + kPage * t + (lane & 15));
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            e[i] = __builtin_amdgcn_exp2f(above_ref(x[i], p.scale_log2, ref.v[i], big));
                            e[i] = r0 + 4 * grp + i >= seen ? e[i] : 0.f;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], p.scale_log2, -ref.v[i]));
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[u * Unit::kTiles + t] = __builtin_fmaf(e[i], inv.v[i], acc[u * Unit::kTiles + t]);
                }
            q = qn;
            ref = refn;
            inv = invn;
        }
        // the four lane groups' rows of a token; group g writes tiles g, g + 4 ..
        float mine[(N + 3) / 4];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            acc[i] += __shfl_xor(acc[i], 16);
            acc[i] += __shfl_xor(acc[i], 32);
            mine[i / 4] = (i & 3) == 0 || grp == (i & 3) ? acc[i] : mine[i / 4];
        }
#pragma unroll
        for (int i = 0; i < (N + 3) / 4; ++i) {
            const int t = tok0 + kPage * (4 * i + grp) + (lane & 15);
            if (4 * i + grp < N && t < s.n) out[t] = p.splits > 1 ? mine[i] : out[t] + mine[i];
        }
    }
}

// The row splits' sums of a token, in their order, added to its weight.
__global__ void __launch_bounds__(256) token_sums_join_kernel(WeightsParams p) {
    const int bh = int(blockIdx.y);
    const int t = int(blockIdx.x) * 256 + int(threadIdx.x);
    const WeightsSeq s = weights_seq(p, bh / p.num_kv_heads);
    const int rows = s.use * p.group, splits = rows > 0 ? (rows - 1) / p.row_split + 1 : 0;
    if (t >= s.n || splits == 0) return;
    float sum = 0.f;
    for (int i = 0; i < splits; ++i) sum += p.parts[(int64_t(i) * gridDim.y + bh) * p.max_context + t];
    p.weights[int64_t(bh) * p.width + t] += sum;
}

template <int D>
static void launch_token_weights_d(const WeightsParams& p, hipStream_t stream) {
    const dim3 block{256u};
    const dim3 norms{unsigned(p.norm_blocks)}, sums{unsigned(p.sum_blocks)};
    if (p.row_units == 1) hipLaunchKernelGGL((token_norms_kernel<D, 1>), norms, block, 0, stream, p);
    else if (p.row_units == 2) hipLaunchKernelGGL((token_norms_kernel<D, 2>), norms, block, 0, stream, p);
    else if (p.row_units == 4 || D == 256) hipLaunchKernelGGL((token_norms_kernel<D, 4>), norms, block, 0, stream, p);
    else hipLaunchKernelGGL((token_norms_kernel<D, (D == 256 ? 4 : 8)>), norms, block, 0, stream, p);
    if (p.chunks > 1) {
        const int64_t rows = p.rows_per_head * p.num_kv_heads;
        hipLaunchKernelGGL(token_norms_join_kernel, dim3(unsigned((rows + 63) / 64)), block, 0, stream, p);
    }
    if (p.key_units == 2) hipLaunchKernelGGL((token_sums_kernel<D, 2>), sums, block, 0, stream, p);
    else hipLaunchKernelGGL((token_sums_kernel<D, (D == 128 ? 8 : 4)>), sums, block, 0, stream, p);
    if (p.splits > 1)
        hipLaunchKernelGGL(token_sums_join_kernel, dim3(unsigned((p.max_context + 255) / 256), unsigned(p.batch * p.num_kv_heads)), block,
                           0, stream, p);
}

hipError_t launch_token_weights(const WeightsParams& p, hipStream_t stream) {
    if (p.head_dim == 64) launch_token_weights_d<64>(p, stream);
    else if (p.head_dim == 128) launch_token_weights_d<128>(p, stream);
    else launch_token_weights_d<256>(p, stream);
    return hipGetLastError();
}

}  // namespace uq
