// The latent cache: rows of one latent vector and one rotated key a token rounded into their
// slots, and the entry points of the attention that reads them.
//
// Appending is one pass over the rows, bound by memory: a thread 16 values (of the rotated part eight
// pairs), the query rows of the same tokens in the grid's second layer.  Measured (bf16, R = 512, P = 64):
// 16384 rows without a rotation 8.2 us (38 MB), with it 10.5, with 16 query heads 23 (109 MB: 4.7 TB/s);
// 48 rows with 64 query heads 2.3 us.
#include "ak_latent.cuh"
#include "ak_rotate.cuh"

namespace ak {

namespace {

// What is stored of a value: NaN as 0, what is beyond the type's range as its largest.
template <typename S>
__device__ __forceinline__ float latent_finite(float x) {
    const float most = is_bf16<S> ? 3.38953139e38f : 65504.f;
    return x != x ? 0.f : fminf(fmaxf(x, -most), most);
}

template <typename T, typename S, bool WIDE>
__global__ void __launch_bounds__(256)
k_latent_append(S *__restrict__ cache, const T *__restrict__ latent, const T *__restrict__ rope, int64_t l_row,
                int64_t r_row, const int64_t *__restrict__ slots, int32_t *__restrict__ tags,
                const int32_t *__restrict__ new_tags, int64_t n, int64_t rows, int R, int P, int *status,
                const RotateArgs turn) {
    griddep_wait();
    const bool query = blockIdx.y;
    const int per = query ? P / 16 * turn.q_heads : (R + P) / 16;      // threads a token
    const int64_t total = n * per;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < total; x += (int64_t)gridDim.x * 256) {
        const int64_t i = total < 0x7fffffff ? (uint32_t)x / (uint32_t)per : x / per;
        const int u = (int)(x - i * per);
        const int64_t slot = slots[i];
        const int64_t pos = turn.positions ? turn.positions[i] : 0;
        const int y = u - R / 16;              // unit of the rotated part
        alignas(16) T raw[16];                 // (on its way before the slot and the position are known)
        if (query) {
            const T *src = (const T *)turn.q + i * turn.q_row + u / (P / 16) * turn.q_head;
            if (turn.wide) load_query<true>(turn, src, u % (P / 16), raw);
            else load_query<false>(turn, src, u % (P / 16), raw);
        } else if (y < 0) {
            load_raw<16, WIDE>(latent + i * l_row + 16 * u, raw);
        } else if (turn.positions) {
            load_unit<WIDE>(turn, rope + i * r_row, y, raw);
        } else {
            load_raw<16, WIDE>(rope + i * r_row + 16 * y, raw);
        }
        bool have = slot != -1;
        if (have && (slot < 0 || slot >= rows)) {
            set_status(status, AKASHIC_EDEVICE);
            have = false;
        }
        if (query) {
            if (have) have = rotate_at(turn, pos, status);
            T *dst = (T *)turn.q_out + i * turn.o_row + u / (P / 16) * turn.o_head;
            if (turn.wide) store_query<true>(turn, raw, dst, u % (P / 16), have ? pos : -1);
            else store_query<false>(turn, raw, dst, u % (P / 16), have ? pos : -1);
            continue;
        }
        if (have && turn.positions) have = rotate_at(turn, pos, status);
        if (!have) continue;
        S *dst = cache + slot * (R + P);
        float f[16];
        if (y >= 0 && turn.positions) {
            turn_unit(turn, raw, y, pos, f);
        } else {
#pragma unroll
            for (int w = 0; w < 16; ++w) f[w] = to_f32(raw[w]);
        }
#pragma unroll
        for (int w = 0; w < 16; ++w) f[w] = latent_finite<S>(f[w]);
        if (y >= 0 && turn.positions && !turn.pairs) {
            store_run<8, true>(dst + R + 8 * y, f);
            store_run<8, true>(dst + R + P / 2 + 8 * y, f + 8);
        } else {
            store_run<16, true>(dst + 16 * u, f);
        }
        if (tags && u == 0) tags[slot] = new_tags ? new_tags[i] : 0;
    }
}

struct LatentRows {
    const akashic_mem_latent_config_t *cfg;
    void *cache;
    const void *latent, *rope;
    int64_t l_row, r_row;
    const int64_t *slots;
    int32_t *tags;
    const int32_t *new_tags;
    int64_t n;
    int *status;
    bool wide;
    RotateArgs turn;
};

template <typename T, typename S>
cudaError_t launch_append(const LatentRows &r, cudaStream_t st) {
    auto *kernel = r.wide ? k_latent_append<T, S, true> : k_latent_append<T, S, false>;
    const int R = r.cfg->latent_dim, P = r.cfg->rope_dim;
    int64_t per = (R + P) / 16;
    if (r.turn.q && P / 16 * r.turn.q_heads > per) per = P / 16 * r.turn.q_heads;
    const int64_t want = ceil_div(r.n * per, (int64_t)256), most = (int64_t)device_sm_count() * 16;
    return launch_pdl(kernel, dim3((unsigned)(want < most ? want : most), r.turn.q ? 2 : 1), dim3(256), 0, st,
                      (S *)r.cache, (const T *)r.latent, (const T *)r.rope, r.l_row, r.r_row, r.slots, r.tags,
                      r.new_tags, r.n, r.cfg->n_blocks * r.cfg->block_tokens, R, P, r.status, r.turn);
}
template <typename T>
cudaError_t launch_append_to(const LatentRows &r, cudaStream_t st) {
    return r.cfg->dtype == AKASHIC_DTYPE_BF16 ? launch_append<T, __nv_bfloat16>(r, st)
                                              : launch_append<T, __half>(r, st);
}

akashic_status_t latent_check(const akashic_mem_latent_config_t *c, const char *who) {
    if (!c) return kv_fail(AKASHIC_EINVAL, "%s: NULL config", who);
    if (c->latent_dim != 128 && c->latent_dim != 256 && c->latent_dim != 512)
        return kv_fail(AKASHIC_EINVAL, "%s: latent_dim must be 128, 256 or 512", who);
    if (c->rope_dim != 32 && c->rope_dim != 64) return kv_fail(AKASHIC_EINVAL, "%s: rope_dim must be 32 or 64", who);
    if (c->dtype != AKASHIC_DTYPE_BF16 && c->dtype != AKASHIC_DTYPE_FP16)
        return kv_fail(AKASHIC_EINVAL, "%s: dtype must be BF16 or FP16", who);
    if (c->block_tokens < 16 || c->block_tokens > 4096 || c->block_tokens % 16)
        return kv_fail(AKASHIC_EINVAL, "%s: block_tokens must be a multiple of 16 in [16, 4096]", who);
    // (rows are coordinates of tensor maps; a tile beyond the last is one, too)
    if (c->n_blocks < 1 || c->n_blocks > (0x7fffffffLL - 8191) / c->block_tokens)
        return kv_fail(AKASHIC_EINVAL, "%s: n_blocks must be >= 1, with at most 2^31 - 2^13 tokens", who);
    if (c->device < 0) return kv_fail(AKASHIC_EINVAL, "%s: device must be >= 0", who);
    return AKASHIC_OK;
}

akashic_status_t attend_check(const akashic_mem_latent_config_t *cfg, const akashic_mem_latent_attend_t *a,
                              bool expanded, const char *who) {
    if (akashic_status_t s = latent_check(cfg, who)) return s;
    if (!a) return kv_fail(AKASHIC_EINVAL, "%s: NULL arguments", who);
    if (a->q_heads < 1 || a->q_heads > KV_MAX_HEADS)
        return kv_fail(AKASHIC_EINVAL, "%s: q_heads must be in [1, %d]", who, KV_MAX_HEADS);
    if (a->n_seq < 0 || a->n_q < 0 || a->max_blocks < 0)
        return kv_fail(AKASHIC_EINVAL, "%s: n_seq, n_q and max_blocks must be >= 0", who);
    if (a->max_blocks > 0x7fffff00LL / cfg->block_tokens)
        return kv_fail(AKASHIC_EINVAL, "%s: a list may hold fewer than 2^31 tokens", who);
    if ((int64_t)a->n_q * a->q_heads > 0x7fffffffLL)
        return kv_fail(AKASHIC_EINVAL, "%s: n_q x q_heads must be below 2^31", who);
    if (!a->q_start && a->n_seq > 0 && a->n_q % a->n_seq)
        return kv_fail(AKASHIC_EINVAL, "%s: without q_start, n_q must be a multiple of n_seq", who);
    if (!(a->scale - a->scale == 0.f) || a->scale == 0.f)
        return kv_fail(AKASHIC_EINVAL, "%s: scale must be finite and not 0", who);
    if (!a->tags != !a->q_tags) return kv_fail(AKASHIC_EINVAL, "%s: tags and q_tags come together", who);
    if (!expanded) return AKASHIC_OK;
    if ((a->nope_dim != 64 && a->nope_dim != 128) || (a->value_dim != 64 && a->value_dim != 128))
        return kv_fail(AKASHIC_EINVAL, "%s: nope_dim and value_dim must be 64 or 128", who);
    if (a->lse) return kv_fail(AKASHIC_EINVAL, "%s: the expanded form has no lse", who);
    // (before anything is multiplied by their product; what else a call needs of the scratch is 2 GB, or one head's)
    if (a->n_seq > 0 && a->n_q > 0 &&
        latent_seq_rows(a->max_blocks * cfg->block_tokens) > (0x7fffffffLL - 8192) / a->n_seq)
        return kv_fail(AKASHIC_EINVAL, "%s: sequences times the tokens of a list must be below 2^31", who);
    const int64_t st[2][2] = {{a->w_k_head_stride, a->w_k_row_stride}, {a->w_v_head_stride, a->w_v_row_stride}};
    for (auto &w : st)
        if (w[1] < cfg->latent_dim || w[1] % 8 || w[1] > (1 << 30) || w[0] < 0 || w[0] % w[1] ||
            (a->q_heads > 1 && w[0] / w[1] > (0x7fffffffLL - 256) / (a->q_heads - 1)))
            return kv_fail(AKASHIC_EINVAL,
                           "%s: rows of w_k and w_v must be evenly spaced, by a multiple of 8 from latent_dim on", who);
    return AKASHIC_OK;
}

akashic_status_t run_attend(const akashic_mem_latent_config_t *cfg, const void *cache,
                            const akashic_mem_latent_attend_t *a, void *scratch, int64_t scratch_bytes,
                            int32_t *status, void *stream, bool expanded, const char *who) {
    set_last_error("");
    if (akashic_status_t s = attend_check(cfg, a, expanded, who)) return s;
    if (a->n_seq == 0 || a->n_q == 0) return AKASHIC_OK;
    if (!cache || !a->q || !a->out || (!a->blocks && a->max_blocks) || (!scratch && scratch_bytes > 0) ||
        (expanded && (!a->w_k || !a->w_v)))
        return kv_fail(AKASHIC_EINVAL, "%s: NULL argument", who);
    if (((uintptr_t)cache | (uintptr_t)scratch | (uintptr_t)a->tags) & 15u ||
        (expanded && ((uintptr_t)a->w_k | (uintptr_t)a->w_v) & 15u))
        return kv_fail(AKASHIC_EINVAL, "%s: cache, tags, weights and scratch must be 16-byte aligned", who);
    if ((uintptr_t)a->out & 3u || (uintptr_t)a->q & 1u)
        return kv_fail(AKASHIC_EINVAL, "%s: out must be 4-byte aligned, q to its element", who);
    if ((uintptr_t)a->blocks & 7u ||
        ((uintptr_t)a->q_start | (uintptr_t)a->kv_len | (uintptr_t)a->prefix_len | (uintptr_t)a->q_tags |
         (uintptr_t)a->lse) & 3u)
        return kv_fail(AKASHIC_EINVAL, "%s: arrays must be aligned to their element", who);
    KvDevice dev(cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "%s: device %d cannot be made current", who, cfg->device);
    LatentParams p = {};
    AttendParams &b = p.a;
    b.cache = (const unsigned char *)cache;
    b.q = a->q, b.q_row = a->q_row_stride, b.q_head = a->q_head_stride;
    b.out = a->out, b.lse = a->lse;
    b.q_start = a->q_start, b.kv_len = a->kv_len, b.prefix = a->prefix_len;
    b.blocks = a->blocks, b.tags = a->tags, b.q_tags = a->q_tags, b.status = status;
    b.n_blocks = cfg->n_blocks, b.max_blocks = a->max_blocks;
    b.n_q = a->n_q, b.n_seq = a->n_seq, b.q_heads = a->q_heads;
    b.heads = expanded ? a->q_heads : 1, b.group = expanded ? 1 : a->q_heads;
    b.per_block = cfg->block_tokens / KV_UNIT;
    b.max_kv = (int)(a->max_blocks * cfg->block_tokens);
    b.causal = a->causal;
    b.scale = a->scale;
    b.out_wide = !((uintptr_t)a->out & 15u);
    b.q_wide = !(((uintptr_t)a->q | (uintptr_t)((a->q_row_stride | a->q_head_stride) * 2)) & 15u);
    p.R = cfg->latent_dim, p.P = cfg->rope_dim, p.bf16 = cfg->dtype == AKASHIC_DTYPE_BF16;
    if (expanded) {
        p.nope = a->nope_dim, p.value = a->value_dim;
        p.w_k = a->w_k, p.w_v = a->w_v;
        p.k_head = a->w_k_head_stride, p.k_row = a->w_k_row_stride;
        p.v_head = a->w_v_head_stride, p.v_row = a->w_v_row_stride;
    }
    const int64_t need = expanded ? latent_expanded_scratch(p) : latent_absorbed_scratch(p);
    if (scratch_bytes < need) return kv_fail(AKASHIC_EINVAL, "%s: scratch needs %lld bytes", who, (long long)need);
    const cudaError_t e = expanded ? launch_latent_expanded(p, scratch, (cudaStream_t)stream)
                                   : launch_latent_absorbed(p, scratch, (cudaStream_t)stream);
    if (e != cudaSuccess) return kv_fail(AKASHIC_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return AKASHIC_OK;
}

akashic_status_t attend_scratch(const akashic_mem_latent_config_t *cfg, const akashic_mem_latent_attend_t *a,
                                int64_t *bytes, bool expanded, const char *who) {
    set_last_error("");
    if (akashic_status_t s = attend_check(cfg, a, expanded, who)) return s;
    if (!bytes) return kv_fail(AKASHIC_EINVAL, "%s: NULL bytes", who);
    KvDevice dev(cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "%s: device %d cannot be made current", who, cfg->device);
    LatentParams p = {};
    p.a.n_q = a->n_q, p.a.n_seq = a->n_seq, p.a.q_heads = a->q_heads;
    p.a.max_kv = (int)(a->max_blocks * cfg->block_tokens);
    p.a.heads = expanded ? a->q_heads : 1, p.a.group = expanded ? 1 : a->q_heads;
    p.a.tags = a->tags, p.a.q_start = a->q_start;
    p.R = cfg->latent_dim, p.P = cfg->rope_dim;
    p.nope = a->nope_dim, p.value = a->value_dim;
    *bytes = a->n_seq == 0 || a->n_q == 0 ? 0 : expanded ? latent_expanded_scratch(p) : latent_absorbed_scratch(p);
    return AKASHIC_OK;
}

}  // namespace
}  // namespace ak

using namespace ak;

extern "C" akashic_status_t akashic_mem_latent_cache_bytes(const akashic_mem_latent_config_t *cfg, int64_t *bytes) {
    set_last_error("");
    if (akashic_status_t s = latent_check(cfg, "latent_cache_bytes")) return s;
    if (!bytes) return kv_fail(AKASHIC_EINVAL, "latent_cache_bytes: NULL bytes");
    *bytes = cfg->n_blocks * cfg->block_tokens * (cfg->latent_dim + cfg->rope_dim) * 2;
    return AKASHIC_OK;
}

extern "C" akashic_status_t akashic_mem_latent_append(
    const akashic_mem_latent_config_t *cfg, void *cache, int32_t *tags, const void *latent, int64_t latent_stride,
    const void *k_rope, int64_t k_rope_stride, int32_t dtype, int64_t n, const int64_t *slots, const int32_t *new_tags,
    const akashic_mem_rotation_t *rotation, int32_t *status, void *stream) {
    const char *who = "latent_append";
    set_last_error("");
    if (akashic_status_t s = latent_check(cfg, who)) return s;
    const int size = dtype_size(dtype);
    if (!size) return kv_fail(AKASHIC_EINVAL, "%s: dtype must be BF16, FP16 or FP32", who);
    if (n < 0 || n > 0x7fffffffLL) return kv_fail(AKASHIC_EINVAL, "%s: n must be in [0, 2^31-1]", who);
    if (n == 0) return AKASHIC_OK;
    if (!cache || !latent || !k_rope || !slots) return kv_fail(AKASHIC_EINVAL, "%s: NULL argument", who);
    if ((uintptr_t)cache & 15u) return kv_fail(AKASHIC_EINVAL, "%s: cache must be 16-byte aligned", who);
    if (((uintptr_t)latent | (uintptr_t)k_rope) & (uintptr_t)(size - 1) || (uintptr_t)slots & 7u ||
        ((uintptr_t)tags | (uintptr_t)new_tags) & 3u)
        return kv_fail(AKASHIC_EINVAL, "%s: arrays must be aligned to their element", who);
    if (new_tags && !tags) return kv_fail(AKASHIC_EINVAL, "%s: new_tags needs the cache's tags", who);
    LatentRows r = {};
    if (rotation) {
        const char *why = nullptr;
        if (rotation->rotary_dim != cfg->rope_dim)
            return kv_fail(AKASHIC_EINVAL, "%s: rotary_dim must be rope_dim", who);
        if (!rotate_args(rotation, cfg->rope_dim, size, n, &r.turn, &why))
            return kv_fail(AKASHIC_EINVAL, "%s: %s", who, why);
    }
    r.cfg = cfg, r.cache = cache, r.latent = latent, r.rope = k_rope;
    r.l_row = latent_stride, r.r_row = k_rope_stride;
    r.slots = slots, r.tags = tags, r.new_tags = new_tags, r.n = n, r.status = status;
    r.wide = !(((uintptr_t)latent | (uintptr_t)k_rope | (uintptr_t)((latent_stride | k_rope_stride) * size)) & 15u);
    KvDevice dev(cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "%s: device %d cannot be made current", who, cfg->device);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = dtype == AKASHIC_DTYPE_BF16   ? launch_append_to<__nv_bfloat16>(r, st)
                          : dtype == AKASHIC_DTYPE_FP16 ? launch_append_to<__half>(r, st)
                                                        : launch_append_to<float>(r, st);
    if (e != cudaSuccess) return kv_fail(AKASHIC_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return AKASHIC_OK;
}

extern "C" akashic_status_t akashic_mem_latent_attend_scratch(const akashic_mem_latent_config_t *cfg,
                                                              const akashic_mem_latent_attend_t *a, int64_t *bytes) {
    return attend_scratch(cfg, a, bytes, false, "latent_attend_scratch");
}
extern "C" akashic_status_t akashic_mem_latent_expanded_scratch(const akashic_mem_latent_config_t *cfg,
                                                                const akashic_mem_latent_attend_t *a, int64_t *bytes) {
    return attend_scratch(cfg, a, bytes, true, "latent_expanded_scratch");
}
extern "C" akashic_status_t akashic_mem_latent_attend(const akashic_mem_latent_config_t *cfg, const void *cache,
                                                      const akashic_mem_latent_attend_t *a, void *scratch,
                                                      int64_t scratch_bytes, int32_t *status, void *stream) {
    return run_attend(cfg, cache, a, scratch, scratch_bytes, status, stream, false, "latent_attend");
}
extern "C" akashic_status_t akashic_mem_latent_attend_expanded(const akashic_mem_latent_config_t *cfg,
                                                               const void *cache, const akashic_mem_latent_attend_t *a,
                                                               void *scratch, int64_t scratch_bytes, int32_t *status,
                                                               void *stream) {
    return run_attend(cfg, cache, a, scratch, scratch_bytes, status, stream, true, "latent_attend_expanded");
}
