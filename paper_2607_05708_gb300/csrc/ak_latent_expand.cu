// The expanded form's keys and values: w_k c_j and w_v c_j of every token of every sequence, for a
// group of heads, into the caller's scratch, rounded to the cache's type (the attention multiplies them
// with operands of that type).
//
// One product a head and 128 tokens, tokens x R times R x (nope + value), on tcgen05: bound by the
// tensor cores, and beside them by the weights' way from L2.  A CTA keeps its tokens' rows (128 KB at R = 512)
// in shared memory for all heads of its share and streams the heads' weights past them, 64 of
// R at a time.  Two accumulators, so that one is rounded and written while the other is computed.
//
// Measured (18,600 tokens, 32 heads, R = 512, 128 + 128 dims): 156 GFLOP in 126 us, two thirds of a plain
// product's burst rate, the tensor pipe 52 % busy; the weights come from L2 once a tile of tokens, 1.8 GB
// at 14 TB/s.  Eight warps that write instead of four: no gain.  Pairs of CTAs would halve the weights' way.
#include <atomic>

#include "ak_latent.cuh"
#include "ak_umma.cuh"

namespace ak {

namespace {

template <int R>
struct Expand {
    static constexpr int TOK = 128, CHUNKS = R / 64;
    static constexpr int A_CHUNK = TOK * 128, A_BYTES = CHUNKS * A_CHUNK;
    static constexpr int W_BYTES = 256 * 128;            // 64 of R, of all rows of a head's weights
    static constexpr int STAGES = R == 512 ? 3 : 4;
    static constexpr int SMEM = 1024 + A_BYTES + STAGES * W_BYTES;
    static constexpr int WRITE = 4;                      // warps that write
    static constexpr int THREADS = 32 * (WRITE + 2);
};

// A share's place in the order (sequence, tile of 128 tokens, head).
struct ExpandCursor {
    int seq, tile, head, tiles;
};
__device__ __forceinline__ int expand_tiles(const AttendParams &p, int s) {
    return max(1, (attend_seq(p, s).kv + 127) / 128);    // (a sequence without tokens is read as one tile, too)
}

template <int R>
__global__ void __launch_bounds__(Expand<R>::THREADS, 1)
k_latent_expand(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap k_map,
                const __grid_constant__ CUtensorMap v_map, const __grid_constant__ LatentParams lp,
                const __grid_constant__ LatentSpace sp, const int box, const int n_rows) {
    using C = Expand<R>;
    constexpr int ST = C::STAGES;
    const AttendParams &p = lp.a;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *smem = (unsigned char *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    unsigned char *s_a = smem, *s_w = smem + C::A_BYTES;
    __shared__ uint64_t wfull[ST], wempty[ST], afull, aempty, tfull[2], tempty[2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int dead_word;
    volatile int *dead = &dead_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    griddep_wait();
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) mbar_init(&wfull[i], 1), mbar_init(&wempty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&tfull[i], 1), mbar_init(&tempty[i], C::WRITE);
        mbar_init(&afull, 1), mbar_init(&aempty, 1), mbar_init(&drained, 1);
        mbar_fence_init();
        dead_word = 0;
    }
    if (warp == 0) {
        tmem_alloc(&tmem_slot, 512);
        tmem_relinquish();
    }
    // ---- every CTA an equal share of all (tile, head): sums over runs of sequences
    int64_t *prefix = (int64_t *)s_w;      // (until the weights come)
    const int nt = C::THREADS, run = (p.n_seq + nt - 1) / nt;
    {
        int64_t sum = 0;
        for (int i = 0; i < run; ++i)
            if (tid * run + i < p.n_seq) sum += expand_tiles(p, tid * run + i);
        int64_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) prefix[warp] = incl;
        __syncthreads();
        int64_t before = 0;
        for (int w = 0; w < warp; ++w) before += prefix[w];
        __syncthreads();
        prefix[tid] = before + incl - sum;
        if (tid == nt - 1) prefix[nt] = before + incl;
    }
    __syncthreads();
    const int64_t total = prefix[nt] * sp.heads, per = (total + gridDim.x - 1) / gridDim.x;
    const int64_t first = per * blockIdx.x;
    const int64_t left = max((int64_t)0, min(per, total - first));
    ExpandCursor cur = {};
    if (left > 0) {
        const int64_t t = first / sp.heads;
        cur.head = (int)(first - t * sp.heads);
        int run_at = 0;
        for (int i = 0; i < nt; ++i)
            if (prefix[i] <= t) run_at = i;    // (runs without sequences come last)
        int64_t rest = t - prefix[run_at];
        cur.seq = run_at * run;
        // (a run's first sequence may be behind the last: then the one before it holds t)
        while (rest >= (cur.tiles = expand_tiles(p, cur.seq))) rest -= cur.tiles, ++cur.seq;
        cur.tile = (int)rest;
    }
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    auto next = [&](ExpandCursor &c) {         // true: another tile
        if (++c.head < sp.heads) return false;
        c.head = 0;
        if (++c.tile >= c.tiles) {
            c.tile = 0;
            if (++c.seq < p.n_seq) c.tiles = expand_tiles(p, c.seq);
        }
        return true;
    };
    const int rows_w = lp.nope + lp.value;

    if (warp == C::WRITE) {
        // ---------------- copying
        const int nb = C::TOK / box, T = p.per_block * KV_UNIT;
        uint32_t n_tile = 0, n_w = 0;
        bool ok = true, fresh = true;
        for (int64_t i = 0; i < left && ok; ++i) {
            if (fresh) {
                // the tile's tokens, 64 values a box, spread over the lanes
                const int tok = cur.tile * C::TOK + lane % nb * box, kv = attend_seq(p, cur.seq).kv;
                int y = n_rows;                // behind the last row: zeros
                if (tok < kv) {
                    const int b = tok / T;
                    const int64_t id = p.blocks[cur.seq * p.max_blocks + b];
                    if (id >= 0 && id < p.n_blocks) y = (int)(id * T + (tok - b * T));
                    else if (id != -1) set_status(p.status, AKASHIC_EDEVICE);
                }
                ok = wide_wait(&aempty, (n_tile & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(&afull, C::A_BYTES);
                __syncwarp();
                for (int x = lane; x < C::CHUNKS * nb; x += 32)          // (32 is a multiple of nb: x % nb = lane % nb)
                    tma_load_2d(s_a + x / nb * C::A_CHUNK + lane % nb * box * 128, &rows_map, &afull, x / nb * 64, y);
                ++n_tile;
            }
            const int h = sp.head0 + cur.head;
            for (int c = 0; c < C::CHUNKS; ++c, ++n_w) {
                const uint32_t st = n_w % ST;
                ok = wide_wait(&wempty[st], ((n_w / ST) & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect_tx(&wfull[st], rows_w * 128);
                    tma_load_2d(s_w + st * C::W_BYTES, &k_map, &wfull[st], c * 64, (int)(h * sp.k_step));
                    tma_load_2d(s_w + st * C::W_BYTES + lp.nope * 128, &v_map, &wfull[st], c * 64,
                                (int)(h * sp.v_step));
                }
                __syncwarp();
            }
            fresh = next(cur);
        }
        // nothing is on its way when the CTA ends (where a wait gave up; else all has been read)
        if (!ok && n_tile > 0) mbar_wait(&afull, (n_tile - 1) & 1, p.status);
        for (uint32_t i = 0; !ok && i < ST; ++i)
            if (n_w > i) mbar_wait(&wfull[i], ((n_w - i - 1) / ST) & 1, p.status);
        __syncwarp();
    } else if (warp == C::WRITE + 1) {
        // ---------------- issuing
        const uint32_t idesc = idesc_f16(rows_w, lp.bf16);
        const uint64_t a_at = desc64(desc_k(smem_u32(s_a))), w_at = desc64(desc_k(smem_u32(s_w)));
        uint32_t n_tile = 0, n_w = 0;
        bool ok = true, fresh = true;
        for (int64_t i = 0; i < left && ok; ++i) {
            if (fresh) ok = wide_wait(&afull, n_tile++ & 1, dead, p.status);
            const uint32_t acc = (uint32_t)i & 1;
            if (ok) ok = wide_wait(&tempty[acc], ((uint32_t)(i >> 1) & 1) ^ 1, dead, p.status);
            for (int c = 0; ok && c < C::CHUNKS; ++c, ++n_w) {
                const uint32_t st = n_w % ST;
                ok = wide_wait(&wfull[st], (n_w / ST) & 1, dead, p.status);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_ss(tmem + acc * 256, a_at + c * (C::A_CHUNK >> 4) + 2 * k,
                               w_at + st * (C::W_BYTES >> 4) + 2 * k, idesc, c > 0 || k > 0);
                    umma_commit(&wempty[st]);
                }
                __syncwarp();
            }
            if (!ok) break;
            fresh = next(cur);
            if (elect_one()) {
                umma_commit(&tfull[acc]);
                if (fresh) umma_commit(&aempty);
            }
            __syncwarp();
        }
        if (elect_one()) umma_commit(&drained);
        mbar_wait(&drained, 0, p.status);
        __syncwarp();
    } else {
        // ---------------- writing: a lane is token 32 warp + lane
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        const float most = lp.bf16 ? 3.38953139e38f : 65504.f;
        bool ok = true;
        for (int64_t i = 0; i < left && ok; ++i) {
            const uint32_t acc = (uint32_t)i & 1;
            ok = wide_wait(&tfull[acc], (uint32_t)(i >> 1) & 1, dead, p.status);
            if (!ok) break;
            tc_fence_after();
            const int64_t row = (int64_t)cur.head * sp.seq_rows * p.n_seq + (int64_t)cur.seq * sp.seq_rows +
                                cur.tile * C::TOK + warp * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < rows_w; c += 32) {
                uint32_t y[32];
                tmem_ld32(tmem + lanes + acc * 256 + c, y);
                tmem_ld_wait();
                uint32_t h[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    // (finite: a value that a row does not see meets a weight of 0)
                    const float a = fminf(fmaxf(__uint_as_float(y[2 * k]), -most), most);
                    const float b = fminf(fmaxf(__uint_as_float(y[2 * k + 1]), -most), most);
                    if (lp.bf16) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
                        h[k] = *(const uint32_t *)&v;
                    } else {
                        h[k] = pack_h2(a, b);
                    }
                }
                uint16_t *dst = c < lp.nope ? (uint16_t *)sp.k + row * lp.nope + c
                                            : (uint16_t *)sp.v + row * lp.value + (c - lp.nope);
#pragma unroll
                for (int k = 0; k < 16; k += 8)                // whole sectors
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 2 * k),
                                 "r"(h[k]), "r"(h[k + 1]), "r"(h[k + 2]), "r"(h[k + 3]), "r"(h[k + 4]),
                                 "r"(h[k + 5]), "r"(h[k + 6]), "r"(h[k + 7])
                                 : "memory");
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tempty[acc]);
            next(cur);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

template <int R>
cudaError_t run_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st) {
    using C = Expand<R>;
    auto *kernel = k_latent_expand<R>;
    // once a device (the attribute stays; another thread that comes first does the same)
    static std::atomic<bool> ready[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev].store(true, std::memory_order_release);
    }
    const CUtensorMapDataType type = p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap rows, k, v;
    e = latent_rows_map(p, 128, &rows);
    const uint64_t heads = (uint64_t)p.a.q_heads - 1;
    if (e == cudaSuccess)
        e = make_tmap_2d(&k, p.w_k, type, 2, R, sp.k_step * heads + p.nope, p.k_row * 2, 64, p.nope);
    if (e == cudaSuccess)
        e = make_tmap_2d(&v, p.w_v, type, 2, R, sp.v_step * heads + p.value, p.v_row * 2, 64, p.value);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(device_sm_count()), dim3(C::THREADS), C::SMEM, st, rows, k, v, p, sp,
                      latent_box(p, 128), (int)(p.a.n_blocks * p.a.per_block * KV_UNIT));
}

}  // namespace

cudaError_t launch_latent_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st) {
    return p.R == 128   ? run_expand<128>(p, sp, st)
           : p.R == 256 ? run_expand<256>(p, sp, st)
                        : run_expand<512>(p, sp, st);
}

}  // namespace ak
