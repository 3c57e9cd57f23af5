// Blocked cache of keys and values held in 4 or 8 bits: format, layout and
// the arithmetic that both directions and the attention share.
//
// A block holds block_tokens tokens of every head.  Its memory is
// [block][head][unit], a unit being 16 tokens of one head, both keys and
// values with their scales, contiguous (KvUnit::BYTES, a multiple of 16): the
// attention moves whole units with one bulk copy each, whatever the block's
// length.  Inside a unit the codes lie in the order in which the lanes of a
// warp hold the 16 x 16 A operand of an mma (lane = 4 g + c):
//   keys    lane (g, c) has the dims [c D/4, (c+1) D/4) of tokens g and g + 8
//   values  lane (g, c) has the dims [g D/8, (g+1) D/8) of tokens 2c, 2c + 1,
//           2c + 8, 2c + 9
// so that a lane's loads from shared memory are 16 bytes each, consecutive
// lanes at consecutive addresses, and no code moves between lanes.
//
// 4 bits: a 32-bit word is 8 consecutive dims, dim 2i in nibble i and dim
// 2i + 1 in nibble i + 4 (i < 4): (w >> 4i) & 0x000f000f is an adjacent pair in
// two 16-bit halves.  A nibble is code + 8, code in -7..7.  Per 16 dims one scale
// byte b: e = (1 + (b & 15) / 16) 2^((b >> 4) - 15); per token and head one
// byte T + 127; the value is code e 2^T: 3 bits times 5 bits times a power of two,
// exact in fp16 (scaled) and in bf16.
// 8 bits: a byte is code + 128; per token and head the scale as bf16 bits.
#pragma once

#include <cuda_fp16.h>

#include "ak_common.cuh"

namespace ak {

constexpr int KV_UNIT = 16;        // tokens of a unit
constexpr int KV_T_MIN = -100, KV_T_MAX = 125;

template <int BITS, int D>
struct KvUnit {
    static_assert(BITS == 4 || BITS == 8, "4 or 8 bits");
    static_assert(D == 64 || D == 128 || D == 256, "head widths");
    static constexpr int GROUPS = D / 16;
    static constexpr int CODES = KV_UNIT * D * BITS / 8;
    static constexpr int K_CODES = 0, V_CODES = CODES;
    // 4 bits: scale bytes, then the exponents; 8 bits: bf16 scales
    static constexpr int SCALES = BITS == 4 ? KV_UNIT * GROUPS : KV_UNIT * 2;
    static constexpr int K_SCALES = 2 * CODES, V_SCALES = 2 * CODES + SCALES;
    static constexpr int K_EXP = V_SCALES + SCALES, V_EXP = K_EXP + KV_UNIT;   // 4 bits only
    static constexpr int BYTES = 2 * CODES + 2 * SCALES + (BITS == 4 ? 2 * KV_UNIT : 0);
    static_assert(BYTES % 16 == 0, "bulk copies of whole units");

    // Byte offset of the codes of 16 consecutive dims from d0 (a multiple of
    // 16) of token t: keys lie contiguous (8 or 16 bytes) ...
    __host__ __device__ static constexpr int k_code(int t, int d0) {
        const int j = t >> 3, lane = (t & 7) * 4 + d0 / (D / 4), at = (d0 % (D / 4)) * BITS / 8;
        constexpr int per = D / 4 * BITS / 8;   // bytes a lane has of one token
        if (per == 8) return K_CODES + lane * 16 + j * 8 + at;
        constexpr int chunks = per / 16 > 0 ? per / 16 : 1;
        return K_CODES + ((j * chunks + at / 16) * 32 + lane) * 16 + at % 16;
    }
    // ... values too, but in 8 consecutive dims from d0 (a multiple of 8): at D = 64
    // 16 dims belong to two lanes.
    __host__ __device__ static constexpr int v_code(int t, int d0) {
        const int j = t >> 3, i = t & 1, lane = (d0 / (D / 8)) * 4 + ((t & 7) >> 1);
        const int at = (d0 % (D / 8)) * BITS / 8;
        constexpr int per = D / 8 * BITS / 8;
        if (per == 4) return V_CODES + lane * 16 + (j * 2 + i) * 4 + at;
        if (per == 8) return V_CODES + (j * 32 + lane) * 16 + i * 8 + at;
        constexpr int chunks = per / 16 > 0 ? per / 16 : 1;
        return V_CODES + (((j * 2 + i) * chunks + at / 16) * 32 + lane) * 16 + at % 16;
    }
    // 4 bits: the scale byte of group gr (16 dims) of token t
    __host__ __device__ static constexpr int k_scale(int t, int gr) {
        constexpr int per = D / 64;             // groups a lane has of one token
        return K_SCALES + (((t & 7) * 4 + gr / per) * 2 + (t >> 3)) * per + gr % per;
    }
    __host__ __device__ static constexpr int v_scale(int t, int gr) {
        return V_SCALES + (gr * 4 + ((t & 7) >> 1)) * 4 + (t >> 3) * 2 + (t & 1);
    }
    // index of token t among the exponents (4 bits) or the bf16 scales (8 bits)
    __host__ __device__ static constexpr int k_row(int t) { return (t & 7) * 2 + (t >> 3); }
    __host__ __device__ static constexpr int v_row(int t) {
        return ((t & 7) >> 1) * 4 + (t >> 3) * 2 + (t & 1);
    }
};

inline int64_t kv_unit_bytes(int bits, int dim) {
    return bits == 4 ? (int64_t)KV_UNIT * dim + 2 * dim + 2 * KV_UNIT
                     : (int64_t)2 * KV_UNIT * dim + 4 * KV_UNIT;
}

// ------------------------------------------------------------------ arithmetic
// Largest T with 7 * 2^T <= a, from a's exponent and mantissa (1.75 = 7/4),
// clamped; a finite, >= 0.
__device__ __forceinline__ int kv_row_exp(float a) {
    const uint32_t u = __float_as_uint(a);
    const int t = (int)(u >> 23) - 127 - 2 - ((u & 0x7fffffu) < 0x600000u ? 1 : 0);
    return max(KV_T_MIN, min(KV_T_MAX, t));
}
__device__ __forceinline__ float pow2i(int e) {   // -126 <= e <= 127
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
// a / den rounded to the nearest with `keep` mantissa bits dropped, ties to
// even: the fp32 quotient is within half an ulp, and where it lies exactly
// between two results the exact remainder says on which side the quotient is.
// Returns the result's fp32 bits >> keep.
__device__ __forceinline__ uint32_t kv_round_quotient(float a, float den, float times, int keep) {
    const float q = __fdiv_rn(a, den);
    const float rem = fmaf(-den, q, a);
    const uint32_t u = __float_as_uint(q * times);   // times: a power of two
    const uint32_t low = u & ((1u << keep) - 1u), half = 1u << (keep - 1);
    const bool up = low > half || (low == half && (rem > 0.f || (rem == 0.f && ((u >> keep) & 1u))));
    return (u >> keep) + (up ? 1u : 0u);
}
// The scale byte of a group whose largest magnitude is ag, in a row of exponent T.
__device__ __forceinline__ uint32_t kv_scale_byte(float ag, int T) {
    const int b = (int)kv_round_quotient(ag, 7.f, pow2i(-T), 19) - (112 << 4);
    return (uint32_t)max(0, min(255, b));
}
__device__ __forceinline__ float kv_scale_of(uint32_t b) {
    return __uint_as_float((b + (112u << 4)) << 19);
}
// The bf16 bits of the 8-bit format's scale of a row of largest magnitude a.
__device__ __forceinline__ uint32_t kv_scale_bf16(float a) {
    return max(kv_round_quotient(a, 127.f, 1.f, 16), (uint32_t)(KV_T_MIN + 127) << 7);
}
// round(x / s), ties to even, clamped to +-top.  x * inv is within an ulp of the
// quotient, so its rounding is off by one step at most, and the remainder
// x - c s (exact: s has at most 8 significant bits) says so.
__device__ __forceinline__ int kv_code(float x, float s, float inv, int top) {
    float c = rintf(x * inv);
    const float d = fmaf(-c, s, x), h = 0.5f * s;
    const bool odd = ((int)c) & 1;
    if (d > h || (d == h && odd)) c += 1.f;
    else if (d < -h || (d == -h && odd)) c -= 1.f;
    return max(-top, min(top, (int)c));
}
// What is stored of an input: NaN as 0, infinities as the largest fp32.
__device__ __forceinline__ float kv_finite(float x) {
    return x != x ? 0.f : fminf(fmaxf(x, -3.402823466e38f), 3.402823466e38f);
}

}  // namespace ak
