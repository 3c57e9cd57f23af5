// Attention over the latent cache, the plain kernel: a warp a query row and head, one key at a
// time, everything in fp32.  The expanded form takes the query into the latent space and the
// result out of it: w_k^T q, then w_v o.
#include "ak_latent.cuh"

namespace ak {

namespace {

constexpr int MOST = 512 / 32;                 // latent values a lane

__device__ __forceinline__ float value16(const uint16_t *p, bool bf16) {
    return bf16 ? __bfloat162float(*(const __nv_bfloat16 *)p) : __half2float(*(const __half *)p);
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

__global__ void __launch_bounds__(256) k_latent_rows(const __grid_constant__ LatentParams lp, const bool expanded) {
    const AttendParams &p = lp.a;
    griddep_wait();
    const int lane = threadIdx.x & 31, per = lp.R / 32, T = p.per_block * KV_UNIT, wide = lp.R + lp.P;
    const int64_t all = (int64_t)p.n_q * p.q_heads;
    for (int64_t w = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; w < all; w += (int64_t)gridDim.x * 8) {
        const int row = (int)(w / p.q_heads), h = (int)(w - (int64_t)row * p.q_heads);
        int seq = -1;
        AttendSeq q = {};
        for (int s0 = 0; s0 < p.n_seq && seq < 0; s0 += 32) {
            AttendSeq x = {};
            if (s0 + lane < p.n_seq) x = attend_seq(p, s0 + lane);
            const unsigned in = __ballot_sync(0xffffffffu, s0 + lane < p.n_seq && row >= x.row0 && row < x.row0 + x.nq);
            if (in) seq = s0 + __ffs(in) - 1;
        }
        if (seq < 0) continue;
        q = attend_seq(p, seq);
        const uint16_t *src = (const uint16_t *)p.q + row * p.q_row + h * p.q_head;
        float ql[MOST] = {}, qr[2] = {}, o[MOST] = {};
        if (expanded) {
            for (int n = 0; n < lp.nope; ++n) {
                const float x = value16(src + n, lp.bf16);
                const uint16_t *wr = (const uint16_t *)lp.w_k + h * lp.k_head + n * lp.k_row;
#pragma unroll
                for (int i = 0; i < MOST; ++i)
                    if (i < per) ql[i] = fmaf(x, value16(wr + 32 * i + lane, lp.bf16), ql[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MOST; ++i)
                if (i < per) ql[i] = value16(src + 32 * i + lane, lp.bf16);
        }
        for (int i = 0; i < lp.P / 32; ++i) qr[i] = value16(src + (expanded ? lp.nope : lp.R) + 32 * i + lane, lp.bf16);
        const int limit = attend_limit(p, q, row - q.row0), tag = p.q_tags ? p.q_tags[row] : 0;
        float m = NEG, l = 0.f;
        for (int j = 0; j < limit; ++j) {
            const int64_t id = p.blocks[seq * p.max_blocks + j / T];
            if (id < 0 || id >= p.n_blocks) {
                if (id != -1) set_status(p.status, AKASHIC_EDEVICE);
                continue;
            }
            const int64_t slot = id * T + j % T;
            if (p.tags && (p.tags[slot] != tag || tag < 0)) continue;
            const uint16_t *c = (const uint16_t *)p.cache + slot * wide;
            float y[MOST], z = 0.f;
#pragma unroll
            for (int i = 0; i < MOST; ++i)
                if (i < per) y[i] = value16(c + 32 * i + lane, lp.bf16), z = fmaf(ql[i], y[i], z);
            for (int i = 0; i < lp.P / 32; ++i) z = fmaf(qr[i], value16(c + lp.R + 32 * i + lane, lp.bf16), z);
            z = warp_sum(z) * p.scale * LOG2E_F;
            const float top = fmaxf(m, z), down = ex2(m - top), e = ex2(z - top);
            m = top, l = l * down + e;
#pragma unroll
            for (int i = 0; i < MOST; ++i)
                if (i < per) o[i] = fmaf(o[i], down, e * y[i]);
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const int64_t dst = (int64_t)row * p.q_heads + h;
        auto put = [&](int64_t at, float x) {
            if (lp.bf16) ((__nv_bfloat16 *)p.out)[at] = __float2bfloat16_rn(x);
            else ((__half *)p.out)[at] = __float2half_rn(x);
        };
        if (expanded) {
            for (int n = 0; n < lp.value; ++n) {
                const uint16_t *wr = (const uint16_t *)lp.w_v + h * lp.v_head + n * lp.v_row;
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < MOST; ++i)
                    if (i < per) x = fmaf(o[i], value16(wr + 32 * i + lane, lp.bf16), x);
                x = warp_sum(x) * inv;
                if (lane == 0) put(dst * lp.value + n, x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MOST; ++i)
                if (i < per) put(dst * lp.R + 32 * i + lane, o[i] * inv);
            if (p.lse && lane == 0) p.lse[dst] = lse_of(m, l);
        }
    }
}

cudaError_t launch_rows(LatentParams &p, bool expanded, cudaStream_t st) {
    const int64_t want = ceil_div((int64_t)p.a.n_q * p.a.q_heads, (int64_t)8), most = (int64_t)device_sm_count() * 8;
    return launch_pdl(k_latent_rows, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, p, expanded);
}

}  // namespace

int64_t latent_absorbed_scratch(const LatentParams &) { return 0; }
int64_t latent_expanded_scratch(const LatentParams &) { return 0; }
cudaError_t launch_latent_absorbed(LatentParams &p, void *, cudaStream_t st) { return launch_rows(p, false, st); }
cudaError_t launch_latent_expanded(LatentParams &p, void *, cudaStream_t st) { return launch_rows(p, true, st); }

}  // namespace ak
