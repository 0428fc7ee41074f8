// uq_rows.hpp -- the rows around the cache (uq_norm_rope, uq_norm_rope_write,
// uq_read_kv of include/uq.h), part of the uq_quantize.hip translation unit:
// one head vector of D = 32 NG channels per quad of lanes, lane L holding
// channels 32 j + 8 L + i in x[j][i], as in quantize_kv_kernel.
//
// Norm and position rotation are written with explicit fused operations and
// no contraction, so that every kernel gets the same bits for the same row.
#pragma once

#include "uq_device.hpp"
#include "uq_internal.hpp"

namespace uq {

// y = x * rsqrt(mean(x^2) + eps) * w.  The squares are summed along the lane's
// channels, then over the quad.
template <int NG>
__device__ __forceinline__ void norm_quad(float (&x)[NG][8], const float* w, float eps, int L) {
#pragma clang fp contract(off)
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[j][i], x[j][i], s);
    s = s + quad_xor<1>(s);
    s = s + quad_xor<2>(s);
    const float r = __builtin_amdgcn_rsqf(s * (1.0f / float(32 * NG)) + eps);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        float g[8];
        load_x8<0>(w, 32 * j + 8 * L, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = (x[j][i] * r) * g[i];
    }
}

// (a, b) <- (a c - b s, b c + a s).
__device__ __forceinline__ void rotate_pair(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
    const float p = b * s, q = a * s;
    const float ya = __builtin_fmaf(a, c, -p);
    b = __builtin_fmaf(b, c, q);
    a = ya;
}

// Pairs (c, c + 32 H), c < 32 H: both in this lane.
template <int NG, int H>
__device__ __forceinline__ void rope_in_lane(float (&x)[NG][8], const float* cs, int L) {
    if constexpr (2 * H <= NG) {
#pragma unroll
        for (int j = 0; j < H; ++j) {
            float c[8], s[8];
            load_x8<0>(cs, 32 * j + 8 * L, c);
            load_x8<0>(cs, 32 * H + 32 * j + 8 * L, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) rotate_pair(x[j][i], x[j + H][i], c[i], s[i]);
        }
    }
}

// Pairs (c, c + 8 S), c < 8 S, S 1 or 2: lanes L and L ^ S of the quad, in
// x[0]; with S = 1 only lanes 0 and 1 take part.  The whole quad executes this.
template <int S, int NG>
__device__ __forceinline__ void rope_across(float (&x)[NG][8], const float* cs, int L) {
    float c[8], s[8];
    load_x8<0>(cs, 8 * (L & (S - 1)), c);
    load_x8<0>(cs, 8 * S + 8 * (L & (S - 1)), s);
    const bool upper = (L & S) != 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float o = quad_xor<S>(x[0][i]);
        float a = upper ? o : x[0][i], b = upper ? x[0][i] : o;
        rotate_pair(a, b, c[i], s[i]);
        if (L < 2 * S) x[0][i] = upper ? b : a;
    }
}

// cs: the position's row of the table, rot / 2 cosines, then the sines.
template <int NG>
__device__ __forceinline__ void rope_quad(float (&x)[NG][8], const float* cs, int rot, bool interleaved, int L) {
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            const int c0 = 32 * j + 8 * L;   // this lane's 8 channels, 4 pairs (rot is a multiple of 8)
            if (c0 < rot) {
                float c[4], s[4];
                load_x4<0>(cs, c0 / 2, c);
                load_x4<0>(cs, rot / 2 + c0 / 2, s);
#pragma unroll
                for (int i = 0; i < 4; ++i) rotate_pair(x[j][2 * i], x[j][2 * i + 1], c[i], s[i]);
            }
        }
        return;
    }
    if (rot == 64) rope_in_lane<NG, 1>(x, cs, L);
    else if (rot == 128) rope_in_lane<NG, 2>(x, cs, L);
    else if (rot == 192) rope_in_lane<NG, 3>(x, cs, L);
    else if (rot == 256) rope_in_lane<NG, 4>(x, cs, L);
    else if (rot == 32) rope_across<2, NG>(x, cs, L);
    else if (rot == 16) rope_across<1, NG>(x, cs, L);
}

// Eight fp32 values as elements e .. e + 7 of a buffer of dtype DT (0 f32, 1
// bf16, 2 f16, rounded to nearest), 16-byte aligned for the 16-bit types.
__device__ __forceinline__ void store_x8(void* base, int64_t elem, int dt, const float (&x)[8]) {
    if (dt == 0) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + elem);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (dt == 1) {
                const v2bf h = {__bf16(x[2 * i]), __bf16(x[2 * i + 1])};
                w[i] = __builtin_bit_cast(uint32_t, h);
            } else {
                typedef _Float16 v2h __attribute__((ext_vector_type(2)));
                const v2h h = {_Float16(x[2 * i]), _Float16(x[2 * i + 1])};
                w[i] = __builtin_bit_cast(uint32_t, h);
            }
        }
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + elem) = uint4{w[0], w[1], w[2], w[3]};
    }
}

// Norm and rotation of the vector a quad holds (token t, weight w or nullptr).
template <int NG>
__device__ __forceinline__ void norm_rope_quad(float (&x)[NG][8], const NormRopeParams& p, int64_t t, const float* w,
                                               int L) {
    if (w != nullptr) norm_quad<NG>(x, w, p.eps, L);
    if (p.rot > 0) {
        int pos = p.positions[t];
        pos = pos < 0 ? 0 : pos < p.max_position ? pos : p.max_position - 1;
        rope_quad<NG>(x, p.cos_sin + int64_t(pos) * p.rot, p.rot, p.interleaved != 0, L);
    }
}

// Norm and rotation of q and k rows; with a cache (WRITE) K's result and V go
// into it, and a FP8 query is rotated like the keys and cast.  The first
// q_blocks blocks take 64 (token, query head) vectors each, heads fastest, so
// that a wave reads 16 heads of a token from one run of memory and one row
// of the table; the others 64 (token, kv head) vectors of k in the same
// order, or (WRITE) the units of quantize_kv_kernel: 16 tokens of one kv head
// per wave, whose stores then fill a page's tiles.
//
// Bound by memory: 16381 tokens, 64 query heads to FP8 and 8 KV heads to the cache
// at d = 128, 487 MB, take 116 us (4.2 TB/s; a copy moves 5.0); 8191 tokens of 64 + 8
// heads at d = 64 rotated to FP16 rows, 151 MB, 30 us; 32 tokens, as a decode step
// writes them, 5 us, a launch.  More than three waves per SIMD need V in the registers
// after K is done with them (130 us with both at once; five waves' worth of spills
// are none); several heads per quad, the weights and angles loaded once for all,
// gave 126 us.
template <int DT, int NG, bool WRITE>
__global__ void __launch_bounds__(256, NG <= 4 ? 5 : 2) norm_rope_kernel(NormRopeParams p, QuantizeParams c) {
    constexpr int D = 32 * NG;
    const int L = threadIdx.x & 3;
    float x[NG][8];
    if (blockIdx.x < p.q_blocks || !WRITE) {
        const bool isk = blockIdx.x >= p.q_blocks;
        const int heads = isk ? p.num_kv_heads : p.num_q_heads;
        const unsigned vec = (blockIdx.x - (isk ? p.q_blocks : 0u)) * 64u + (threadIdx.x >> 2);
        const unsigned t = vec / unsigned(heads);
        if (t >= p.num_tokens) return;   // whole quads
        const int h = int(vec - t * unsigned(heads));
        const int64_t row = int64_t(t) * (isk ? p.k_stride : p.q_stride) + int64_t(h) * D + 8 * L;
#pragma unroll
        for (int j = 0; j < NG; ++j) load_x8<DT>(isk ? p.k : p.q, row + 32 * j, x[j]);
        norm_rope_quad<NG>(x, p, t, isk ? p.k_weight : p.q_weight, L);
        const int64_t out = int64_t(vec) * D + 8 * L;
        if (p.out_dtype == 3) {
            wht_quad<NG>(x, L);
#pragma unroll
            for (int j = 0; j < NG; ++j)
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.q_out) + out + 32 * j) =
                    make_uint2(e4m3x4(x[j][0], x[j][1], x[j][2], x[j][3]), e4m3x4(x[j][4], x[j][5], x[j][6], x[j][7]));
        } else {
#pragma unroll
            for (int j = 0; j < NG; ++j) store_x8(isk ? p.k_out : p.q_out, out + 32 * j, p.out_dtype, x[j]);
        }
        return;
    }
    if constexpr (WRITE) {
        const unsigned wi = (blockIdx.x - p.q_blocks) * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int h = int(wi % unsigned(c.num_kv_heads));
        const int64_t t = int64_t(wi / unsigned(c.num_kv_heads)) * 16 + ((threadIdx.x & 63) >> 2);
        if (t >= c.num_tokens) return;
        const int64_t row = t * c.token_stride + int64_t(h) * D + 8 * L;
        const int64_t slot = c.slot_mapping[t];
        float xv[NG][8];
#pragma unroll
        for (int j = 0; j < NG; ++j) load_x8<DT>(c.k, row + 32 * j, x[j]);
        int64_t page;
        int off;
        const bool valid = page_of_slot(c, slot, page, off);
        if (!valid) return;
        norm_rope_quad<NG>(x, p, t, p.k_weight, L);
        const int64_t ph = page * c.num_kv_heads + h;
        uint8_t* kc = c.codes + ph * (16 * D);
        uint8_t* ks = c.scales + ph * D;
        uint32_t w[NG], b[NG];
        quantize_xq<NG>(x, L, c.c, true, w, b, [&](float (&y)[NG][8]) {
#pragma unroll
            for (int j = 0; j < NG; ++j) load_x8<DT>(c.k, row + 32 * j, y[j]);
            norm_rope_quad<NG>(y, p, t, p.k_weight, L);
        });
        store_k_quad<NG>(kc, ks, off, L, w, b);
#pragma unroll
        for (int j = 0; j < NG; ++j) load_x8<DT>(c.v, row + 32 * j, xv[j]);
        quantize_xq<NG>(xv, L, c.c, c.rotate_v != 0, w, b, [&](float (&y)[NG][8]) {
#pragma unroll
            for (int j = 0; j < NG; ++j) load_x8<DT>(c.v, row + 32 * j, y[j]);
        });
        store_v_quad<NG>(kc + 8 * D, ks + D / 2, off, L, w, b);
    }
}

// Stored tokens back to rows: the writer's quad reads the dwords it would
// write, decodes them by the hardware conversion and rotates the vector back
// (R is its own inverse).  Units of 16 tokens of one kv head per wave, kv head
// fastest, as the writer's.  Bound by memory: 65530 tokens of 8 heads at d = 128 to
// BF16 rows, 340 MB of which four fifths are written, take 76 to 81 us (4.2 to 4.5
// TB/s; a copy moves 5.0).
template <int NG>
__global__ void __launch_bounds__(256) read_kv_kernel(QuantizeParams c, void* k_out, void* v_out, int dt) {
    constexpr int D = 32 * NG;
    const int L = threadIdx.x & 3;
    const unsigned wi = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = int(wi % unsigned(c.num_kv_heads));
    const int64_t t = int64_t(wi / unsigned(c.num_kv_heads)) * 16 + ((threadIdx.x & 63) >> 2);
    if (t >= c.num_tokens) return;   // whole quads
    int64_t page;
    int off;
    if (!page_of_slot(c, c.slot_mapping[t], page, off)) return;
    const int64_t ph = page * c.num_kv_heads + h;
    const uint8_t* kc = c.codes + ph * (16 * D);
    const uint8_t* ks = c.scales + ph * D;
    const int64_t out = (t * c.num_kv_heads + h) * D + 8 * L;
    uint32_t w[2][NG];
    float sc[2][NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        w[0][j] = *reinterpret_cast<const uint32_t*>(kc + (j * kPage + off) * 16 + 4 * L);
        sc[0][j] = ue8m0_to_f32(ks[j * kPage + off]);
        w[1][j] = *reinterpret_cast<const uint32_t*>(kc + 8 * D + ((off >> 2) * (D / 8) + 4 * j + L) * 16 + (off & 3) * 4);
        sc[1][j] = ue8m0_to_f32(ks[D / 2 + j * kPage + off]);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        void* dst = kv ? v_out : k_out;
        if (dst == nullptr) continue;
        float x[NG][8];
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kv][j], sc[kv][j], 0);
            const v2f b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kv][j], sc[kv][j], 1);
            const v2f d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kv][j], sc[kv][j], 2);
            const v2f e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kv][j], sc[kv][j], 3);
            x[j][0] = a[0]; x[j][1] = a[1]; x[j][2] = b[0]; x[j][3] = b[1];
            x[j][4] = d[0]; x[j][5] = d[1]; x[j][6] = e[0]; x[j][7] = e[1];
        }
        if (kv == 0 || c.rotate_v) wht_quad<NG>(x, L);
#pragma unroll
        for (int j = 0; j < NG; ++j) store_x8(dst, out + 32 * j, dt, x[j]);
    }
}

static int64_t kv_units(const QuantizeParams& c) { return (c.num_tokens + 15) / 16 * c.num_kv_heads; }

template <int NG, bool WRITE>
static void launch_norm_rope_ng(const NormRopeParams& p, const QuantizeParams& c, int dtype, unsigned blocks,
                                hipStream_t stream) {
    const dim3 grid{blocks}, block{256u};
    if (dtype == 0) hipLaunchKernelGGL((norm_rope_kernel<0, NG, WRITE>), grid, block, 0, stream, p, c);
    else if (dtype == 1) hipLaunchKernelGGL((norm_rope_kernel<1, NG, WRITE>), grid, block, 0, stream, p, c);
    else hipLaunchKernelGGL((norm_rope_kernel<2, NG, WRITE>), grid, block, 0, stream, p, c);
}

hipError_t launch_norm_rope(NormRopeParams p, const QuantizeParams* c, int head_dim, int dtype, hipStream_t stream) {
    const int64_t qb = (p.num_tokens * p.num_q_heads + 63) / 64;
    const int64_t kb = c != nullptr ? (kv_units(*c) + 3) / 4 : (p.num_tokens * p.num_kv_heads + 63) / 64;
    if (qb + kb == 0) return hipSuccess;
    p.q_blocks = unsigned(qb);
    const unsigned blocks = unsigned(qb + kb);
    const QuantizeParams none{};
    if (c != nullptr) {
        if (head_dim == 64) launch_norm_rope_ng<2, true>(p, *c, dtype, blocks, stream);
        else if (head_dim == 128) launch_norm_rope_ng<4, true>(p, *c, dtype, blocks, stream);
        else launch_norm_rope_ng<8, true>(p, *c, dtype, blocks, stream);
    } else {
        if (head_dim == 64) launch_norm_rope_ng<2, false>(p, none, dtype, blocks, stream);
        else if (head_dim == 128) launch_norm_rope_ng<4, false>(p, none, dtype, blocks, stream);
        else launch_norm_rope_ng<8, false>(p, none, dtype, blocks, stream);
    }
    return hipGetLastError();
}

hipError_t launch_read_kv(const QuantizeParams& c, void* k_out, void* v_out, int dtype, hipStream_t stream) {
    const int64_t units = kv_units(c);
    if (units == 0) return hipSuccess;
    const dim3 grid{unsigned((units + 3) / 4)}, block{256u};
    if (c.head_dim == 64) hipLaunchKernelGGL(read_kv_kernel<2>, grid, block, 0, stream, c, k_out, v_out, dtype);
    else if (c.head_dim == 128) hipLaunchKernelGGL(read_kv_kernel<4>, grid, block, 0, stream, c, k_out, v_out, dtype);
    else hipLaunchKernelGGL(read_kv_kernel<8>, grid, block, 0, stream, c, k_out, v_out, dtype);
    return hipGetLastError();
}

}  // namespace uq
