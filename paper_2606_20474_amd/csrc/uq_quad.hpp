// uq_quad.hpp -- the rotation R of a head vector held by a quad of lanes, D / 4
// channels per lane (the writer, the rows around the cache, the queries of
// uq_extend_attention).
#pragma once

#include "uq_device.hpp"

namespace uq {

// Lane exchange inside a quad (4 consecutive lanes) with DPP quad_perm:
// partner lane L^1 or L^2.
template <int S>
__device__ __forceinline__ float quad_xor(float x) {
    constexpr int ctrl = S == 1 ? 0xB1 : 0x4E;   // quad_perm [1,0,3,2] / [2,3,0,1]
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), ctrl, 0xF, 0xF, true));
}

// One cross-lane butterfly stage for the 8 values of a lane, partner L^S:
// y <- dpp(y) * t + y, one v_fmac_f32 per value with the partner lane's
// value as a DPP (quad_perm) operand (the compiler does not fold the DPP move
// into this tied instruction itself).  s_nop 1 first: a DPP read needs two
// wait states after a VALU write of its register, and inside the block no
// register is read after it is written.  All 64 lanes are active.
#define UQ_FMAC_DPP(P, i) "v_fmac_f32_dpp %" #i ", %" #i ", %8 quad_perm:" P " row_mask:0xf bank_mask:0xf bound_ctrl:1\n\t"
#define UQ_FMAC_DPP8(P)                                                                                          \
    "s_nop 1\n\t" UQ_FMAC_DPP(P, 0) UQ_FMAC_DPP(P, 1) UQ_FMAC_DPP(P, 2) UQ_FMAC_DPP(P, 3) UQ_FMAC_DPP(P, 4)      \
        UQ_FMAC_DPP(P, 5) UQ_FMAC_DPP(P, 6) UQ_FMAC_DPP(P, 7)
template <int S>
__device__ __forceinline__ void quad_stage8(float (&y)[8], float t) {
    if constexpr (S == 1) {
        asm volatile(UQ_FMAC_DPP8("[1,0,3,2]")
                     : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]), "+v"(y[4]), "+v"(y[5]), "+v"(y[6]), "+v"(y[7])
                     : "v"(t));
    } else {
        asm volatile(UQ_FMAC_DPP8("[2,3,0,1]")
                     : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]), "+v"(y[4]), "+v"(y[5]), "+v"(y[6]), "+v"(y[7])
                     : "v"(t));
    }
}
#undef UQ_FMAC_DPP8
#undef UQ_FMAC_DPP

// The rotation in its plain form: each cross-lane stage moves the partner's
// value (DPP) and combines it with one fma, fma(s, x, o) = x + o or o - x.
// wht_quad below gives the same values with one instruction per value and
// stage, except for the signs of exact zeros when the input vector is all
// zero; quantize_xq falls back to this form for such vectors.
template <int NG>
__device__ __forceinline__ void wht_quad_plain(float (&x)[NG][8], int L) {
#pragma clang fp contract(off)
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) {
#pragma unroll
        for (int j = 0; j < NG; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i & h) continue;
                const float a = x[j][i], b = x[j][i + h];
                x[j][i] = a + b;
                x[j][i + h] = a - b;
            }
        }
    }
    const float s1 = (L & 1) ? -1.0f : 1.0f;
    const float s2 = (L & 2) ? -1.0f : 1.0f;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = __builtin_fmaf(s1, x[j][i], quad_xor<1>(x[j][i]));
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = __builtin_fmaf(s2, x[j][i], quad_xor<2>(x[j][i]));
#pragma unroll
    for (int h = 1; h < NG; h <<= 1) {
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            if (j & h) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = x[j][i], b = x[j + h][i];
                x[j][i] = a + b;
                x[j + h][i] = a - b;
            }
        }
    }
    const float r = inv_sqrt_d<32 * NG>();
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = x[j][i] * r;
}

// The rotation of one head vector of D = 32 NG channels held by 4 lanes of
// a quad: lane L holds channels 32j + 8L + i in x[j][i] (j < NG, i < 8).
// The stages run in the order of the format (widths 1, 2, 4, ..., D/2): 1,
// 2, 4 inside a lane over i, 8 and 16 across lanes L^1, L^2, then 32, 64
// (and 128 for D = 256) inside a lane over j; each maps (a, b) to
// (a + b, a - b) in fp32, then one multiply by fl32(1/sqrt(D)).  The values
// equal those of the 16-lane form wht_x bit for bit.
//
// The two cross-lane stages take one instruction per value,
// v_fmac_f32 with the partner's value as a DPP operand: y <- dpp(y) * t + y
// with t = +-1 per lane.  The upper lane of a pair needs o - x but a single
// form gives it x - o, so it keeps the negated value (every fp32 rounding is
// symmetric under negation) and its sign sigma is tracked: t1 = sigma after
// the first stage, and since both lanes of a second-stage pair carry the
// same sigma, t2 makes the second stage right up to sign too; the final
// multiply by sigma * fl32(1/sqrt(D)) (exact) restores every value.
// Negation symmetry fails at exact zeros only: an exact cancellation gives
// +0 whatever the signs.  The reference form yields -0 only from a subtree
// of zeros, and every output depends on all inputs, so for an input that is
// not all zero every zero output is +0: the final step is fma(y, sigma r,
// +0), which keeps every nonzero result (and the sign of an underflow) and
// turns every exact zero into +0.  An all-zero input is left to
// wht_quad_plain.
template <int NG>
__device__ __forceinline__ void wht_quad(float (&x)[NG][8], int L) {
#pragma clang fp contract(off)
#pragma unroll
    for (int h = 1; h < 8; h <<= 1) {
#pragma unroll
        for (int j = 0; j < NG; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i & h) continue;
                const float a = x[j][i], b = x[j][i + h];
                x[j][i] = a + b;
                x[j][i + h] = a - b;
            }
        }
    }
    const float t1 = (L & 1) ? -1.0f : 1.0f;
    const float t2 = (L & 2) ? -1.0f : 1.0f;
#pragma unroll
    for (int j = 0; j < NG; ++j) quad_stage8<1>(x[j], t1);
#pragma unroll
    for (int j = 0; j < NG; ++j) quad_stage8<2>(x[j], t2);
#pragma unroll
    for (int h = 1; h < NG; h <<= 1) {
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            if (j & h) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = x[j][i], b = x[j + h][i];
                x[j][i] = a + b;
                x[j + h][i] = a - b;
            }
        }
    }
    const float r = inv_sqrt_d<32 * NG>() * (t1 * t2);
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = __builtin_fmaf(x[j][i], r, 0.0f);
}

}  // namespace uq
