// Writing rows of keys and values into the quantised cache, and reading them
// back (format and layout: ak_kv.cuh).
//
// Both are one pass over the dense rows, bound by memory.  A thread has 16
// consecutive dims of one row: the scale group of the 4-bit format, so that only
// the row's largest magnitude needs its neighbours (D / 16 lanes of the warp).
// Writing has keys and values in the two halves of the grid, reading both in one thread, which
// then looks up its slot once: 16384 tokens 16.3 us and 19.1 in halves.  Writing in
// one thread took 13.5 us instead of 14.7 for 8192 tokens, but 2.3 instead of 1.9 for one,
// which every decoded token is.
// Measured (8 heads, D = 128, 4 bits, bf16): 8192 tokens written in 14.7 us, read in 8.8
// (43 MB: 2.9 and 4.9 TB/s), 16384 read in 16.3 (5.3); a single token 1.9 and 1.6 us.
// Instructions bound the writing: 25 a value (the exactly rounded quotient and code some ten, the rest
// loads' conversions, checks for what is not finite, maxima, addresses), three of four issue slots. Its
// stores touch 11 sectors a request, as a row's values lie in pieces 64 bytes apart; L2 is 27 % busy.
// Nibbles cost the reading.
#include <stdarg.h>
#include <stdio.h>

#include "ak_attend.cuh"
#include "ak_rotate.cuh"

namespace ak {

akashic_status_t kv_fail(akashic_status_t code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

akashic_status_t kv_check_config(const akashic_mem_kv_config_t *c, const char *who) {
    if (!c) return kv_fail(AKASHIC_EINVAL, "%s: NULL config", who);
    if (c->bits != 4 && c->bits != 8) return kv_fail(AKASHIC_EINVAL, "%s: bits must be 4 or 8", who);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return kv_fail(AKASHIC_EINVAL, "%s: head_dim must be 64, 128 or 256", who);
    if (c->heads < 1 || c->heads > KV_MAX_HEADS)
        return kv_fail(AKASHIC_EINVAL, "%s: heads must be in [1, %d]", who, KV_MAX_HEADS);
    if (c->block_tokens < KV_UNIT || c->block_tokens > 4096 || c->block_tokens % KV_UNIT)
        return kv_fail(AKASHIC_EINVAL, "%s: block_tokens must be a multiple of 16 in [16, 4096]", who);
    if (c->n_blocks < 1 || c->n_blocks > 0x7fffffffLL / (c->block_tokens / KV_UNIT))
        return kv_fail(AKASHIC_EINVAL, "%s: n_blocks must be >= 1, with at most 2^31 - 1 units of 16 tokens", who);
    if (c->n_blocks * (c->block_tokens / KV_UNIT) > 0xfffffffeLL / c->heads)
        return kv_fail(AKASHIC_EINVAL, "%s: more than 2^32 - 2 units of 16 tokens and a head", who);
    if (c->device < 0) return kv_fail(AKASHIC_EINVAL, "%s: device must be >= 0", who);
    return AKASHIC_OK;
}

// The caller's device made current for the call, and put back.
KvDevice::KvDevice(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    ok = prev == dev || cudaSetDevice(dev) == cudaSuccess;
    if (!ok) cudaGetLastError();
    changed = ok && prev != dev;
}
KvDevice::~KvDevice() {
    if (changed && prev >= 0) cudaSetDevice(prev);
}

namespace {

struct KvRows {
    const akashic_mem_kv_config_t *cfg;
    unsigned char *cache;
    const void *in[2];             // write: k, v
    void *out[2];                  // read: k, v (contiguous)
    int64_t row_stride[2], head_stride[2];
    const int64_t *slots;
    int32_t *tags;
    const int32_t *new_tags;
    int *status;
    int64_t n;
    bool wide;                     // 16-byte loads and stores are aligned
    RotateArgs turn;               // write with rotation
};

struct KvPlace {
    int64_t unit;                  // of the cache, -1: none
    int token;
};
// Where slot `s` of head h lies; an index out of range is recorded and skipped.
__device__ __forceinline__ KvPlace kv_place(int64_t s, int h, int heads, uint32_t units,
                                            uint32_t per_block, int *status) {
    if (s == -1) return {-1, 0};
    if (s < 0 || (s >> 4) >= (int64_t)units) {
        set_status(status, AKASHIC_EDEVICE);
        return {-1, 0};
    }
    const uint32_t u = (uint32_t)(s >> 4), b = u / per_block;
    return {((int64_t)b * heads + h) * per_block + (u - b * per_block), (int)(s & 15)};
}

// The 16 codes of a group, biased to be positive, `bits` wide and in the cache's
// order (ak_kv.cuh).  q = x / s correctly rounded (one Newton step on x inv); where
// x / s is a whole number and a half q is just that, and otherwise it is on the
// same side of it: for 16-bit inputs x and s (c + 1/2) have at most 19 bits, so they
// differ by 2^-19 relative or not at all; for fp32 the remainder is looked at.
// 1.5 2^23 + bias added rounds half to even and leaves the code in the low bits; the
// words are sums of these shifted into place, less the constants' sum.  No clamp:
// |x / s| stays below 7.3 and 127.3.
template <typename T, int BITS>
__device__ __forceinline__ void kv_codes(const float (&f)[16], float s, uint32_t (&w)[BITS / 2]) {
    constexpr int TOP = BITS == 4 ? 7 : 127, PER = 32 / BITS;
    constexpr float BASE = 12582912.f + (TOP + 1);
    const float inv = __frcp_rn(s);
    float worst = 0.f;
#pragma unroll
    for (int i = 0; i < BITS / 2; ++i) {
        w[i] = 0;
        uint32_t less = 0;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const float x = f[i * PER + p], q0 = x * inv;
            const float m = fmaf(fmaf(-q0, s, x), inv, q0) + BASE;
            if constexpr (sizeof(T) == 4) worst = fmaxf(worst, fabsf(fmaf(BASE - m, s, x)));
            const int at = BITS == 4 ? 4 * (p >> 1) + 16 * (p & 1) : 8 * p;
            w[i] += __float_as_uint(m) << at;
            less += 0x4b400000u << at;
        }
        w[i] -= less;
    }
    if (sizeof(T) == 4 && worst > 0.5f * s) {
#pragma unroll
        for (int i = 0; i < BITS / 2; ++i) {
            w[i] = 0;
#pragma unroll
            for (int p = 0; p < PER; ++p)
                w[i] |= (uint32_t)(kv_code(f[i * PER + p], s, inv, TOP) + TOP + 1)
                        << (BITS == 4 ? 4 * (p >> 1) + 16 * (p & 1) : 8 * p);
        }
    }
}

// TURN: keys are rotated to their positions on the way, in fp32, and the grid's third layer rotates
// the query rows of the same tokens (`tokens_q` at a time).  A thread reads its group and the group of the
// other members of its pairs, which a second thread of the row reads too (L1): exchanging them between
// lanes would tie the split to the rotated width.  Measured (8192 tokens, 8 heads, D = 128, 4 bits, bf16):
// 23 us where writing alone takes 16, with 32 query heads 48 (178 MB: 3.7 TB/s); the layers one beside the
// other instead of one after the other took the same time, and four heads a thread twice that.  A single
// token with 32 query heads: 3 us.
template <typename T, int BITS, int D, bool WIDE, bool TURN>
__global__ void __launch_bounds__(256)
k_kv_write(unsigned char *__restrict__ cache, const T *__restrict__ k, const T *__restrict__ v,
           int64_t k_row, int64_t k_head, int64_t v_row, int64_t v_head,
           const int64_t *__restrict__ slots, int32_t *__restrict__ tags,
           const int32_t *__restrict__ new_tags, int64_t n, int heads, uint32_t units,
           uint32_t per_block, int tokens, int *status, const RotateArgs turn, int tokens_q) {
    using U = KvUnit<BITS, D>;
    constexpr int G = U::GROUPS;
    griddep_wait();
    if constexpr (TURN) {
        if (blockIdx.y == 2) {
            for (int64_t i0 = (int64_t)blockIdx.x * tokens_q; i0 < n; i0 += (int64_t)gridDim.x * tokens_q) {
                const uint32_t total = (uint32_t)min((int64_t)tokens_q, n - i0) * turn.q_heads * G;
                for (uint32_t x = threadIdx.x; x < total; x += 256) {
                    const uint32_t row = x / G, ti = row / (uint32_t)turn.q_heads, h = row - ti * turn.q_heads;
                    const int64_t i = i0 + ti, slot = slots[i];
                    int64_t pos = turn.positions[i];
                    const T *src = (const T *)turn.q + i * turn.q_row + h * turn.q_head;
                    T *dst = (T *)turn.q_out + i * turn.o_row + h * turn.o_head;
                    alignas(16) T raw[16];         // (on its way before the slot and the position are known)
                    if (turn.wide) load_query<true>(turn, src, x % G, raw);
                    else load_query<false>(turn, src, x % G, raw);
                    if (kv_place(slot, 0, heads, units, per_block, status).unit < 0 || !rotate_at(turn, pos, status))
                        pos = -1;
                    if (turn.wide) store_query<true>(turn, raw, dst, x % G, pos);
                    else store_query<false>(turn, raw, dst, x % G, pos);
                }
            }
            return;
        }
    }
    const bool is_v = blockIdx.y;
    const T *base = is_v ? v : k;
    const int64_t row_stride = is_v ? v_row : k_row, head_stride = is_v ? v_head : k_head;
    for (int64_t i0 = (int64_t)blockIdx.x * tokens; i0 < n; i0 += (int64_t)gridDim.x * tokens) {
        const uint32_t total = (uint32_t)min((int64_t)tokens, n - i0) * heads * G;
        // the bound is rounded up to whole warps: the row's lanes meet in shuffles
        for (uint32_t x = threadIdx.x; x < ((total + 31) & ~31u); x += 256) {
            const uint32_t row = x / G, gr = x % G, ti = row / (uint32_t)heads, h = row - ti * heads;
            const int64_t i = i0 + ti, slot = x < total ? slots[i] : -1;
            KvPlace at = kv_place(slot, h, heads, units, per_block, status);
            int64_t pos = 0;
            if constexpr (TURN) {
                pos = x < total ? turn.positions[i] : 0;
                if (at.unit >= 0 && !rotate_at(turn, pos, status)) at.unit = -1;
            }
            float f[16];
#pragma unroll
            for (int w = 0; w < 16; ++w) f[w] = 0.f;
            if (TURN && !is_v && at.unit >= 0) {
                turn_group<WIDE>(turn, base + i * row_stride + h * head_stride, gr * 16, pos, f);
            } else if (at.unit >= 0) {
                const T *src = base + i * row_stride + h * head_stride + gr * 16;
                alignas(16) T raw[16];
                if constexpr (WIDE) {
#pragma unroll
                    for (int w = 0; w < (int)sizeof(raw) / 16; ++w)
                        ((int4 *)raw)[w] = __ldcs((const int4 *)src + w);
                } else {
#pragma unroll
                    for (int w = 0; w < 16; ++w) raw[w] = src[w];
                }
#pragma unroll
                for (int w = 0; w < 16; ++w) f[w] = to_f32(raw[w]);
            }
            float ag = 0.f, odd = 0.f;         // odd: not 0 with a NaN or an infinity
#pragma unroll
            for (int w = 0; w < 16; ++w) ag = fmaxf(ag, fabsf(f[w])), odd = fmaf(f[w], 0.f, odd);
            if (odd != 0.f) {
                ag = 0.f;
#pragma unroll
                for (int w = 0; w < 16; ++w) f[w] = kv_finite(f[w]), ag = fmaxf(ag, fabsf(f[w]));
            }
            float a = ag;
#pragma unroll
            for (int o = G / 2; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
            if (at.unit < 0) continue;
            unsigned char *dst = cache + at.unit * U::BYTES;
            const int t = at.token, d0 = gr * 16;
            uint32_t w[BITS / 2];
            if constexpr (BITS == 4) {
                const int E = kv_row_exp(a);
                const uint32_t b = kv_scale_byte(ag, E);
                if (TURN && !is_v) kv_codes<float, 4>(f, kv_scale_of(b) * pow2i(E), w);
                else kv_codes<T, 4>(f, kv_scale_of(b) * pow2i(E), w);
                if (is_v) {
                    if (U::v_code(0, 8) == U::v_code(0, 0) + 4)
                        *(uint2 *)(dst + U::v_code(t, d0)) = make_uint2(w[0], w[1]);
                    else {
                        *(uint32_t *)(dst + U::v_code(t, d0)) = w[0];
                        *(uint32_t *)(dst + U::v_code(t, d0 + 8)) = w[1];
                    }
                    dst[U::v_scale(t, gr)] = (unsigned char)b;
                    if (gr == 0) dst[U::V_EXP + U::v_row(t)] = (unsigned char)(E + 127);
                } else {
                    *(uint2 *)(dst + U::k_code(t, d0)) = make_uint2(w[0], w[1]);
                    dst[U::k_scale(t, gr)] = (unsigned char)b;
                    if (gr == 0) dst[U::K_EXP + U::k_row(t)] = (unsigned char)(E + 127);
                }
            } else {
                const uint32_t sb = kv_scale_bf16(a);
                if (TURN && !is_v) kv_codes<float, 8>(f, __uint_as_float(sb << 16), w);
                else kv_codes<T, 8>(f, __uint_as_float(sb << 16), w);
                if (is_v) {
                    if (U::v_code(0, 8) == U::v_code(0, 0) + 8)
                        *(uint4 *)(dst + U::v_code(t, d0)) = make_uint4(w[0], w[1], w[2], w[3]);
                    else {
                        *(uint2 *)(dst + U::v_code(t, d0)) = make_uint2(w[0], w[1]);
                        *(uint2 *)(dst + U::v_code(t, d0 + 8)) = make_uint2(w[2], w[3]);
                    }
                    if (gr == 0) ((uint16_t *)(dst + U::V_SCALES))[U::v_row(t)] = (uint16_t)sb;
                } else {
                    *(uint4 *)(dst + U::k_code(t, d0)) = make_uint4(w[0], w[1], w[2], w[3]);
                    if (gr == 0) ((uint16_t *)(dst + U::K_SCALES))[U::k_row(t)] = (uint16_t)sb;
                }
            }
            if (tags && !is_v && h == 0 && gr == 0) tags[slot] = new_tags ? new_tags[i] : 0;
        }
    }
}

// code * s with code = biased - bias, exact: the biased code put under 2^23 and taken
// away again (an integer conversion runs at a quarter of the rate).
template <int BIAS>
__device__ __forceinline__ float kv_value(uint32_t biased, float s) {
    return s * (__uint_as_float(0x4b000000u | biased) - (8388608.f + BIAS));
}
template <typename T, int BITS, int D, bool WIDE>
__global__ void __launch_bounds__(256)
k_kv_read(const unsigned char *__restrict__ cache, T *__restrict__ k, T *__restrict__ v,
          const int64_t *__restrict__ slots, int64_t n, int heads, uint32_t units,
          uint32_t per_block, int tokens, int *status) {
    using U = KvUnit<BITS, D>;
    constexpr int G = U::GROUPS;
    griddep_wait();
    for (int64_t i0 = (int64_t)blockIdx.x * tokens; i0 < n; i0 += (int64_t)gridDim.x * tokens) {
        const uint32_t total = (uint32_t)min((int64_t)tokens, n - i0) * heads * G;
        for (uint32_t x = threadIdx.x; x < total; x += 256) {
            const uint32_t row = x / G, gr = x % G, ti = row / (uint32_t)heads, h = row - ti * heads;
            const int d0 = gr * 16;
            const KvPlace at = kv_place(slots[i0 + ti], h, heads, units, per_block, status);
            const int t = at.token;
            // both rows' codes and scales on their way before the arithmetic
            uint32_t w[2][BITS / 2];
            float s[2] = {0.f, 0.f};
            if (at.unit >= 0) {
                const unsigned char *src = cache + at.unit * U::BYTES;
                if constexpr (BITS == 4) {
                    const uint2 q = *(const uint2 *)(src + U::k_code(t, d0));
                    w[0][0] = q.x, w[0][1] = q.y;
                    if (U::v_code(0, 8) == U::v_code(0, 0) + 4) {
                        const uint2 y = *(const uint2 *)(src + U::v_code(t, d0));
                        w[1][0] = y.x, w[1][1] = y.y;
                    } else {
                        w[1][0] = *(const uint32_t *)(src + U::v_code(t, d0));
                        w[1][1] = *(const uint32_t *)(src + U::v_code(t, d0 + 8));
                    }
                    s[0] = kv_scale_of(src[U::k_scale(t, gr)]) * pow2i((int)src[U::K_EXP + U::k_row(t)] - 127);
                    s[1] = kv_scale_of(src[U::v_scale(t, gr)]) * pow2i((int)src[U::V_EXP + U::v_row(t)] - 127);
                } else {
                    const uint4 q = *(const uint4 *)(src + U::k_code(t, d0));
                    const uint2 y0 = *(const uint2 *)(src + U::v_code(t, d0));
                    const uint2 y1 = *(const uint2 *)(src + U::v_code(t, d0 + 8));
                    w[0][0] = q.x, w[0][1] = q.y, w[0][2] = q.z, w[0][3] = q.w;
                    w[1][0] = y0.x, w[1][1] = y0.y, w[1][2] = y1.x, w[1][3] = y1.y;
                    s[0] = __uint_as_float((uint32_t)((const uint16_t *)(src + U::K_SCALES))[U::k_row(t)] << 16);
                    s[1] = __uint_as_float((uint32_t)((const uint16_t *)(src + U::V_SCALES))[U::v_row(t)] << 16);
                }
            }
#pragma unroll
            for (int is_v = 0; is_v < 2; ++is_v) {
                alignas(16) T raw[16];
#pragma unroll
                for (int p = 0; p < 16; ++p) {
                    float f = 0.f;
                    if (at.unit >= 0)
                        f = BITS == 4 ? kv_value<8>((w[is_v][p >> 3] >> (4 * ((p & 7) >> 1) + 16 * (p & 1))) & 15u, s[is_v])
                                      : kv_value<128>((w[is_v][p >> 2] >> (8 * (p & 3))) & 255u, s[is_v]);
                    from_f32(f, raw[p]);
                }
                T *dst = (is_v ? v : k) + i0 * heads * D + (int64_t)x * 16;
                if constexpr (WIDE) {
#pragma unroll
                    for (int q = 0; q < (int)sizeof(raw) / 16; ++q)
                        __stcs((int4 *)dst + q, ((const int4 *)raw)[q]);
                } else {
#pragma unroll
                    for (int p = 0; p < 16; ++p) dst[p] = raw[p];
                }
            }
        }
    }
}

// A CTA takes `tokens` at a time: enough for its 256 threads, or a single one where the
// heads fill them.
int kv_tokens(int heads, int groups) {
    const int t = 256 / (heads * groups);
    return t > 1 ? t : 1;
}
unsigned kv_grid(int64_t n, int tokens) {
    const int64_t want = ceil_div(n, (int64_t)tokens), most = (int64_t)device_sm_count() * 16;
    return (unsigned)(want < most ? want : most);
}

template <typename T, int BITS, int D, bool TURN>
cudaError_t launch_write(const KvRows &r, cudaStream_t st) {
    const int tokens = kv_tokens(r.cfg->heads, D / 16);
    const uint32_t per = (uint32_t)(r.cfg->block_tokens / KV_UNIT);
    const uint32_t units = (uint32_t)(r.cfg->n_blocks * per);
    auto *kernel = r.wide ? k_kv_write<T, BITS, D, true, TURN> : k_kv_write<T, BITS, D, false, TURN>;
    unsigned grid = kv_grid(r.n, tokens), layers = 2;
    int tokens_q = 1;
    if (TURN && r.turn.q) {
        tokens_q = kv_tokens(r.turn.q_heads, D / 16);
        const unsigned want = kv_grid(r.n, tokens_q);
        grid = want > grid ? want : grid, layers = 3;
    }
    return launch_pdl(kernel, dim3(grid, layers), dim3(256), 0, st, r.cache, (const T *)r.in[0],
                      (const T *)r.in[1], r.row_stride[0], r.head_stride[0], r.row_stride[1], r.head_stride[1],
                      r.slots, r.tags, r.new_tags, r.n, r.cfg->heads, units, per, tokens, r.status, r.turn, tokens_q);
}
template <typename T, int BITS, int D>
cudaError_t launch_read(const KvRows &r, cudaStream_t st) {
    const int tokens = kv_tokens(r.cfg->heads, D / 16);
    const uint32_t per = (uint32_t)(r.cfg->block_tokens / KV_UNIT);
    const uint32_t units = (uint32_t)(r.cfg->n_blocks * per);
    auto *kernel = r.wide ? k_kv_read<T, BITS, D, true> : k_kv_read<T, BITS, D, false>;
    return launch_pdl(kernel, dim3(kv_grid(r.n, tokens)), dim3(256), 0, st, r.cache, (T *)r.out[0],
                      (T *)r.out[1], r.slots, r.n, r.cfg->heads, units, per, tokens, r.status);
}

enum KvCall { KV_WRITE, KV_READ, KV_APPEND };
template <typename T, int BITS, int D>
cudaError_t launch_rows(const KvRows &r, cudaStream_t st, KvCall call) {
    return call == KV_WRITE  ? launch_write<T, BITS, D, false>(r, st)
           : call == KV_READ ? launch_read<T, BITS, D>(r, st)
                             : launch_write<T, BITS, D, true>(r, st);
}
template <typename T, int BITS>
cudaError_t launch_rows_dim(const KvRows &r, cudaStream_t st, KvCall call) {
    switch (r.cfg->head_dim) {
    case 64: return launch_rows<T, BITS, 64>(r, st, call);
    case 128: return launch_rows<T, BITS, 128>(r, st, call);
    default: return launch_rows<T, BITS, 256>(r, st, call);
    }
}
template <typename T>
cudaError_t launch_rows_bits(const KvRows &r, cudaStream_t st, KvCall call) {
    return r.cfg->bits == 4 ? launch_rows_dim<T, 4>(r, st, call) : launch_rows_dim<T, 8>(r, st, call);
}

akashic_status_t run_rows(const char *who, const KvRows &r, int32_t dtype, void *stream, KvCall call) {
    KvDevice dev(r.cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "%s: device %d cannot be made current", who, r.cfg->device);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == AKASHIC_DTYPE_BF16   ? launch_rows_bits<__nv_bfloat16>(r, st, call)
                          : dtype == AKASHIC_DTYPE_FP16 ? launch_rows_bits<__half>(r, st, call)
                                                        : launch_rows_bits<float>(r, st, call);
    if (e != cudaSuccess) return kv_fail(AKASHIC_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return AKASHIC_OK;
}

}  // namespace

int dtype_size(int32_t dtype) {
    return dtype == AKASHIC_DTYPE_FP32 ? 4 : dtype == AKASHIC_DTYPE_BF16 || dtype == AKASHIC_DTYPE_FP16 ? 2 : 0;
}

bool rotate_args(const akashic_mem_rotation_t *r, int width, int size, int64_t n, RotateArgs *a, const char **why) {
    // neighbouring rows or heads of q_out that share memory; q in place with other strides
    const bool rows = n > 1, heads = r->q_heads > 1;
    auto close = [&](int64_t stride) { return stride > -width && stride < width; };
    const bool over = r->q && ((rows && close(r->q_out_row_stride)) || (heads && close(r->q_out_head_stride)) ||
                               (r->q == r->q_out && ((rows && r->q_row_stride != r->q_out_row_stride) ||
                                                     (heads && r->q_head_stride != r->q_out_head_stride))));
    *why = r->rotary_dim < 32 || r->rotary_dim % 32 || r->rotary_dim > width
               ? "rotary_dim must be a multiple of 32, at most the row's width"
           : r->table_rows < 1                        ? "table_rows must be >= 1"
           : !r->positions || !r->cos || !r->sin      ? "NULL positions or table"
           : ((uintptr_t)r->cos | (uintptr_t)r->sin) & 15u || (uintptr_t)r->positions & 7u
               ? "tables must be 16-byte aligned, positions to their element"
           : !r->q != !r->q_out                       ? "q and q_out come together"
           : r->q && (r->q_heads < 1 || r->q_heads > KV_MAX_HEADS * KV_MAX_HEADS)
               ? "q_heads must be in [1, 2^20]"
           : ((uintptr_t)r->q | (uintptr_t)r->q_out) & (uintptr_t)(size - 1)
               ? "q and q_out must be aligned to their element"
           : over ? "rows of q_out must not overlap, nor rows of q, but for those that they replace"
                  : nullptr;
    if (*why) return false;
    a->positions = r->positions, a->cos = r->cos, a->sin = r->sin;
    a->table_rows = r->table_rows, a->rotary = r->rotary_dim, a->pairs = r->interleaved != 0;
    a->q = r->q, a->q_out = r->q_out, a->q_heads = r->q_heads;
    a->q_row = r->q_row_stride, a->q_head = r->q_head_stride;
    a->o_row = r->q_out_row_stride, a->o_head = r->q_out_head_stride;
    a->wide = !(((uintptr_t)r->q | (uintptr_t)r->q_out |
                 (uintptr_t)((r->q_row_stride | r->q_head_stride | r->q_out_row_stride | r->q_out_head_stride) * size)) & 15u);
    return true;
}

}  // namespace ak

using namespace ak;

extern "C" akashic_status_t akashic_mem_kv_cache_bytes(const akashic_mem_kv_config_t *cfg,
                                                       int64_t *bytes) {
    set_last_error("");
    if (akashic_status_t s = kv_check_config(cfg, "kv_cache_bytes")) return s;
    if (!bytes) return kv_fail(AKASHIC_EINVAL, "kv_cache_bytes: NULL bytes");
    const int64_t units = cfg->n_blocks * (cfg->block_tokens / KV_UNIT);
    *bytes = units * cfg->heads * kv_unit_bytes(cfg->bits, cfg->head_dim);
    return AKASHIC_OK;
}

namespace {

akashic_status_t kv_write_rows(const char *who, const akashic_mem_kv_config_t *cfg, void *cache, int32_t *tags,
                               const void *k, int64_t k_row_stride, int64_t k_head_stride, const void *v,
                               int64_t v_row_stride, int64_t v_head_stride, int32_t dtype, int64_t n,
                               const int64_t *slots, const int32_t *new_tags, const akashic_mem_rotation_t *rot,
                               int32_t *status, void *stream, KvCall call) {
    set_last_error("");
    if (akashic_status_t s = kv_check_config(cfg, who)) return s;
    const int size = dtype_size(dtype);
    if (!size) return kv_fail(AKASHIC_EINVAL, "%s: dtype must be BF16, FP16 or FP32", who);
    if (n < 0 || n > 0x7fffffffLL) return kv_fail(AKASHIC_EINVAL, "%s: n must be in [0, 2^31-1]", who);
    if (call == KV_APPEND && !rot) return kv_fail(AKASHIC_EINVAL, "%s: NULL rotation", who);
    if (n == 0) return AKASHIC_OK;
    if (!cache || !k || !v || !slots) return kv_fail(AKASHIC_EINVAL, "%s: NULL argument", who);
    if ((uintptr_t)cache & 15u) return kv_fail(AKASHIC_EINVAL, "%s: cache must be 16-byte aligned", who);
    if (((uintptr_t)k | (uintptr_t)v) & (uintptr_t)(size - 1))
        return kv_fail(AKASHIC_EINVAL, "%s: k and v must be aligned to their element", who);
    if ((uintptr_t)slots & 7u || ((uintptr_t)tags | (uintptr_t)new_tags) & 3u)
        return kv_fail(AKASHIC_EINVAL, "%s: slots and tags must be aligned to their element", who);
    if (new_tags && !tags) return kv_fail(AKASHIC_EINVAL, "%s: new_tags needs the cache's tags", who);
    KvRows r = {};
    const char *why = nullptr;
    if (call == KV_APPEND && !rotate_args(rot, cfg->head_dim, size, n, &r.turn, &why))
        return kv_fail(AKASHIC_EINVAL, "%s: %s", who, why);
    r.cfg = cfg;
    r.cache = (unsigned char *)cache;
    r.in[0] = k, r.in[1] = v;
    r.row_stride[0] = k_row_stride, r.row_stride[1] = v_row_stride;
    r.head_stride[0] = k_head_stride, r.head_stride[1] = v_head_stride;
    r.slots = slots, r.tags = tags, r.new_tags = new_tags, r.status = status, r.n = n;
    r.wide = !(((uintptr_t)k | (uintptr_t)v |
                (uintptr_t)((k_row_stride | k_head_stride | v_row_stride | v_head_stride) * size)) & 15u);
    return run_rows(who, r, dtype, stream, call);
}

}  // namespace

extern "C" akashic_status_t akashic_mem_kv_write(
    const akashic_mem_kv_config_t *cfg, void *cache, int32_t *tags, const void *k,
    int64_t k_row_stride, int64_t k_head_stride, const void *v, int64_t v_row_stride,
    int64_t v_head_stride, int32_t dtype, int64_t n, const int64_t *slots,
    const int32_t *new_tags, int32_t *status, void *stream) {
    return kv_write_rows("kv_write", cfg, cache, tags, k, k_row_stride, k_head_stride, v, v_row_stride, v_head_stride,
                         dtype, n, slots, new_tags, nullptr, status, stream, KV_WRITE);
}

extern "C" akashic_status_t akashic_mem_kv_append(
    const akashic_mem_kv_config_t *cfg, void *cache, int32_t *tags, const void *k,
    int64_t k_row_stride, int64_t k_head_stride, const void *v, int64_t v_row_stride,
    int64_t v_head_stride, int32_t dtype, int64_t n, const int64_t *slots,
    const int32_t *new_tags, const akashic_mem_rotation_t *rotation, int32_t *status, void *stream) {
    return kv_write_rows("kv_append", cfg, cache, tags, k, k_row_stride, k_head_stride, v, v_row_stride, v_head_stride,
                         dtype, n, slots, new_tags, rotation, status, stream, KV_APPEND);
}

extern "C" akashic_status_t akashic_mem_kv_read(const akashic_mem_kv_config_t *cfg,
                                                const void *cache, const int64_t *slots, int64_t n,
                                                int32_t dtype, void *k, void *v, int32_t *status,
                                                void *stream) {
    set_last_error("");
    if (akashic_status_t s = kv_check_config(cfg, "kv_read")) return s;
    const int size = dtype_size(dtype);
    if (!size) return kv_fail(AKASHIC_EINVAL, "kv_read: dtype must be BF16, FP16 or FP32");
    if (n < 0 || n > 0x7fffffffLL) return kv_fail(AKASHIC_EINVAL, "kv_read: n must be in [0, 2^31-1]");
    if (n == 0) return AKASHIC_OK;
    if (!cache || !k || !v || !slots) return kv_fail(AKASHIC_EINVAL, "kv_read: NULL argument");
    if ((uintptr_t)cache & 15u) return kv_fail(AKASHIC_EINVAL, "kv_read: cache must be 16-byte aligned");
    if (((uintptr_t)k | (uintptr_t)v) & (uintptr_t)(size - 1))
        return kv_fail(AKASHIC_EINVAL, "kv_read: k and v must be aligned to their element");
    if ((uintptr_t)slots & 7u) return kv_fail(AKASHIC_EINVAL, "kv_read: slots must be aligned to their element");
    KvRows r = {};
    r.cfg = cfg;
    r.cache = (unsigned char *)cache;
    r.out[0] = k, r.out[1] = v;
    r.slots = slots, r.status = status, r.n = n;
    r.wide = !(((uintptr_t)k | (uintptr_t)v) & 15u);
    return run_rows("kv_read", r, dtype, stream, KV_READ);
}
