// Rotation of rows to their positions: what the caches' append kernels share.
//
// Of a row's first `rotary` values pair i, (x[i], x[i + rotary / 2]) or, interleaved,
// (x[2i], x[2i + 1]), becomes (a c - b s, b c + a s) with c and s from the tables' row of the
// token's position: fp32, both products and the sum rounded (no fused multiply-add, so that
// the stored codes are defined to the bit; two pairs an instruction were faster and came out fused).
// A thread turns 16 values: eight whole pairs, so that query rows can be turned in place.  Tables come
// from L1: the heads of a token share a row of them.
#pragma once

#include <cuda_fp16.h>

#include "ak_common.cuh"

namespace ak {

struct RotateArgs {
    const int64_t *positions;
    const float *cos, *sin;            // [table_rows][rotary / 2]
    int64_t table_rows;
    const void *q;                     // or NULL
    void *q_out;
    int64_t q_row, q_head, o_row, o_head;
    int rotary, q_heads;
    bool pairs;                        // interleaved
    bool wide;                         // 16-byte loads and stores of q and q_out are aligned
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __half &y) { y = __float2half_rn(x); }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16 &y) { y = __float2bfloat16_rn(x); }

// Two adjacent values, 16-bit ones in one conversion.
__device__ __forceinline__ void pair_from_f32(float a, float b, float *y) { y[0] = a, y[1] = b; }
__device__ __forceinline__ void pair_from_f32(float a, float b, __half *y) { *(__half2 *)y = __floats2half2_rn(a, b); }
__device__ __forceinline__ void pair_from_f32(float a, float b, __nv_bfloat16 *y) {
    *(__nv_bfloat162 *)y = __floats2bfloat162_rn(a, b);
}

// N (8 or 16) consecutive values, as they are: what is converted later keeps no instruction waiting
// before the loads behind it.
template <int N, bool WIDE, typename T>
__device__ __forceinline__ void load_raw(const T *src, T *raw) {
    if constexpr (WIDE) {
#pragma unroll
        for (int w = 0; w < N * (int)sizeof(T) / 16; ++w) ((int4 *)raw)[w] = __ldcs((const int4 *)src + w);
    } else {
#pragma unroll
        for (int w = 0; w < N; ++w) raw[w] = src[w];
    }
}
template <int N, bool WIDE, typename T>
__device__ __forceinline__ void load_run(const T *src, float *f) {
    alignas(16) T raw[N];
    load_raw<N, WIDE>(src, raw);
#pragma unroll
    for (int w = 0; w < N; ++w) f[w] = to_f32(raw[w]);
}
template <int N, bool WIDE, typename T>
__device__ __forceinline__ void store_run(T *dst, const float *f) {
    alignas(16) T raw[N];
#pragma unroll
    for (int w = 0; w < N; w += 2) pair_from_f32(f[w], f[w + 1], raw + w);
    if constexpr (WIDE) {
#pragma unroll
        for (int w = 0; w < (int)sizeof(raw) / 16; ++w) __stcs((int4 *)dst + w, ((const int4 *)raw)[w]);
    } else {
#pragma unroll
        for (int w = 0; w < N; ++w) dst[w] = raw[w];
    }
}
// Whether a token's position is in the tables; one that is not is recorded.
__device__ __forceinline__ bool rotate_at(const RotateArgs &a, int64_t pos, int *status) {
    if (pos >= 0 && pos < a.table_rows) return true;
    set_status(status, AKASHIC_EDEVICE);
    return false;
}
// The table entries of eight consecutive pairs (rows of a multiple of 16 floats: 16-byte
// aligned where the tables are).
__device__ __forceinline__ void rotate_table(const RotateArgs &a, int64_t pos, int pair0, float (&c)[8],
                                             float (&s)[8]) {
    const int64_t at = pos * (a.rotary / 2) + pair0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        *(float4 *)(c + 4 * w) = __ldg((const float4 *)(a.cos + at) + w);
        *(float4 *)(s + 4 * w) = __ldg((const float4 *)(a.sin + at) + w);
    }
}
__device__ __forceinline__ float turn_a(float a, float b, float c, float s) {
    return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
}
__device__ __forceinline__ float turn_b(float a, float b, float c, float s) {
    return __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
}
// Pairs [8u, 8u + 8) of a row: side by side where interleaved, else eight first members and eight
// second ones.
template <bool WIDE, typename T>
__device__ __forceinline__ void load_unit(const RotateArgs &a, const T *src, int u, T *raw) {
    if (a.pairs) {
        load_raw<16, WIDE>(src + 16 * u, raw);
    } else {
        load_raw<8, WIDE>(src + 8 * u, raw);
        load_raw<8, WIDE>(src + a.rotary / 2 + 8 * u, raw + 8);
    }
}
template <typename T>
__device__ __forceinline__ void turn_unit(const RotateArgs &a, const T *raw, int u, int64_t pos, float (&f)[16]) {
    float c[8], s[8];
    rotate_table(a, pos, 8 * u, c, s);
#pragma unroll
    for (int w = 0; w < 16; ++w) f[w] = to_f32(raw[w]);
    if (a.pairs) {
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const float x = f[2 * w], y = f[2 * w + 1];
            f[2 * w] = turn_a(x, y, c[w], s[w]), f[2 * w + 1] = turn_b(x, y, c[w], s[w]);
        }
    } else {
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const float x = f[w], y = f[w + 8];
            f[w] = turn_a(x, y, c[w], s[w]), f[w + 8] = turn_b(x, y, c[w], s[w]);
        }
    }
}
// Unit u (16 values) of a query row: turned, or, behind the rotated values, copied.
// pos < 0: a row of no token, zeros.
template <bool WIDE, typename T>
__device__ __forceinline__ void load_query(const RotateArgs &a, const T *src, int u, T *raw) {
    if (16 * u < a.rotary) load_unit<WIDE>(a, src, u, raw);
    else load_raw<16, WIDE>(src + 16 * u, raw);
}
template <bool WIDE, typename T>
__device__ __forceinline__ void store_query(const RotateArgs &a, const T *raw, T *dst, int u, int64_t pos) {
    float f[16];
    const bool turned = 16 * u < a.rotary;
    if (pos < 0) {
#pragma unroll
        for (int w = 0; w < 16; ++w) f[w] = 0.f;
    } else if (turned) {
        turn_unit(a, raw, u, pos, f);
    } else {
#pragma unroll
        for (int w = 0; w < 16; ++w) f[w] = to_f32(raw[w]);
    }
    if (turned && !a.pairs) {
        store_run<8, WIDE>(dst + 8 * u, f);
        store_run<8, WIDE>(dst + a.rotary / 2 + 8 * u, f + 8);
    } else {
        store_run<16, WIDE>(dst + 16 * u, f);
    }
}
// Values [d0, d0 + 16) of a row, turned where they are among the rotated ones (rotary a multiple
// of 32: d0's values are then all first or all second members).
template <bool WIDE, typename T>
__device__ __forceinline__ void turn_group(const RotateArgs &a, const T *src, int d0, int64_t pos, float (&f)[16]) {
    load_run<16, WIDE>(src + d0, f);
    if (d0 >= a.rotary) return;
    const int half = a.rotary / 2;
    if (a.pairs) {
        alignas(16) T raw[16];
        load_unit<WIDE>(a, src, d0 / 16, raw);
        turn_unit(a, raw, d0 / 16, pos, f);
        return;
    }
    const bool second = d0 >= half;
    float other[16];
    load_run<16, WIDE>(src + (second ? d0 - half : d0 + half), other);
#pragma unroll
    for (int k = 0; k < 16; k += 8) {
        float c[8], s[8];
        rotate_table(a, pos, (second ? d0 - half : d0) + k, c, s);
#pragma unroll
        for (int w = 0; w < 8; ++w)
            f[k + w] = second ? turn_b(other[k + w], f[k + w], c[w], s[w]) : turn_a(f[k + w], other[k + w], c[w], s[w]);
    }
}

// Checks the rotation of a call of n tokens and takes it over (false: *why says what is wrong).
int dtype_size(int32_t dtype);   // bytes, 0: no type of rows
bool rotate_args(const akashic_mem_rotation_t *r, int width, int size, int64_t n, RotateArgs *a, const char **why);

}  // namespace ak
