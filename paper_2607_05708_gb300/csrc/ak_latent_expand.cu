// The expanded form's keys and values: w_k c_j and w_v c_j of every token of every sequence, for a
// group of heads, into the caller's scratch, rounded to the cache's type (the attention multiplies them
// with operands of that type).
//
// One product a head and 128 tokens, tokens x R times R x (nope + value), on tcgen05: bound by the
// tensor cores, and beside them by the weights' way from L2.  A CTA keeps its tokens' rows (128 KB at R = 512)
// in shared memory for all heads of its share and streams the heads' weights past them, 64 of
// R at a time.  Two accumulators, so that one is rounded and written while the other is computed.
//
// Measured (18,600 tokens, 32 heads, R = 512, 128 + 128 dims): 156 GFLOP in 102 us, 0.8 of a plain product's
// burst rate, the tensor pipe 69 % busy, 1.1 GB from L2.  A CTA alone took 127 us: a head's weights come from
// L2 once a tile of tokens, 1.8 GB at 14 TB/s.  Eight warps that write instead of four: no gain.
#include <atomic>

#include "ak_latent.cuh"
#include "ak_umma.cuh"

namespace ak {

namespace {

// PAIR: clusters of two CTAs, each with a tile of its own, w_k or w_v of a head and the results of its tile;
// the first one's products (cta_group::2) read both, so that weights come from L2 once for two tiles.
template <int R, bool PAIR>
struct Expand {
    static constexpr int TOK = 128, CHUNKS = R / 64;
    static constexpr int A_CHUNK = TOK * 128, A_BYTES = CHUNKS * A_CHUNK;
    static constexpr int CTAS = PAIR ? 2 : 1;            // that share a head's weights
    static constexpr int W_BYTES = 256 / CTAS * 128;     // 64 of R, of the CTA's rows of a head's weights
    static constexpr int STAGES = (R == 512 ? 3 : 4) * CTAS;
    static constexpr int SMEM = 1024 + A_BYTES + STAGES * W_BYTES;
    static constexpr int WRITE = 4;                      // warps that write
    static constexpr int THREADS = 32 * (WRITE + 2);
};

// A share's place in the order (CTAS tiles, head), of which a CTA has a tile.  Behind the last sequence: none.
struct ExpandCursor {
    int seq, tile, head, tiles;
};
__device__ __forceinline__ int expand_tiles(const AttendParams &p, int s) {
    return max(1, (attend_seq(p, s).kv + 127) / 128);    // (a sequence without tokens is read as one tile, too)
}

template <int R, bool PAIR>
__global__ void __launch_bounds__(Expand<R, PAIR>::THREADS, 1)
k_latent_expand(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap k_map,
                const __grid_constant__ CUtensorMap v_map, const __grid_constant__ LatentParams lp,
                const __grid_constant__ LatentSpace sp, const int box, const int n_rows) {
    using C = Expand<R, PAIR>;
    constexpr int ST = C::STAGES, G = C::CTAS;
    const AttendParams &p = lp.a;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *smem = (unsigned char *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    unsigned char *s_a = smem, *s_w = smem + C::A_BYTES;
    __shared__ uint64_t wfull[ST], wempty[ST], afull, aempty, tfull[2], tempty[2], drained;
    __shared__ uint32_t tmem_slot;
    __shared__ int dead_word;
    volatile int *dead = &dead_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const bool lead = rank == 0;               // issues the products
    griddep_wait();
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) mbar_init(&wfull[i], 1), mbar_init(&wempty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&tfull[i], 1), mbar_init(&tempty[i], G * C::WRITE);
        mbar_init(&afull, 1), mbar_init(&aempty, 1), mbar_init(&drained, 1);
        mbar_fence_init();
        dead_word = 0;
    }
    if (warp == 0) {
        if constexpr (PAIR) {
            tmem_alloc2(&tmem_slot, 512);
            tmem_relinquish2();
        } else {
            tmem_alloc(&tmem_slot, 512);
            tmem_relinquish();
        }
    }
    // ---- equal shares of all (CTAS tiles, head): sums over runs of sequences
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
    const int64_t tiles = prefix[nt], total = (tiles + G - 1) / G * sp.heads, shares = gridDim.x / G;
    const int64_t per = (total + shares - 1) / shares, first = per * (blockIdx.x / G);
    const int64_t left = max((int64_t)0, min(per, total - first));
    ExpandCursor cur = {p.n_seq, 0, 0, 1};
    if (left > 0) {
        const int64_t t = first / sp.heads * G + rank;
        cur.head = (int)(first % sp.heads);
        if (t < tiles) {
            int run_at = 0;
            for (int i = 0; i < nt; ++i)
                if (prefix[i] <= t) run_at = i;    // (runs without sequences come last)
            int64_t rest = t - prefix[run_at];
            cur.seq = run_at * run;
            // (a run's first sequence may be behind the last: then the one before it holds t)
            while (rest >= (cur.tiles = expand_tiles(p, cur.seq))) rest -= cur.tiles, ++cur.seq;
            cur.tile = (int)rest;
        }
    }
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();        // the other CTA's barriers are there
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    auto next = [&](ExpandCursor &c) {         // true: another tile
        if (++c.head < sp.heads) return false;
        c.head = 0;
        c.tile += G;
        while (c.seq < p.n_seq && c.tile >= c.tiles) {
            c.tile -= c.tiles;
            if (++c.seq < p.n_seq) c.tiles = expand_tiles(p, c.seq);
        }
        return true;
    };
    const int rows_w = lp.nope + lp.value;
    // a copy whose end the issuing CTA's barrier tells
    auto load = [&](unsigned char *to, const CUtensorMap *map, uint64_t *bar, int x, int y) {
        if (lead) tma_load_2d(to, map, bar, x, y);
        else tma_load_2d_pair(to, map, bar, 0, x, y);
    };

    if (warp == C::WRITE) {
        // ---------------- copying
        const int nb = C::TOK / box, T = p.per_block * KV_UNIT;
        uint32_t n_tile = 0, n_w = 0;
        bool ok = true, fresh = true;
        for (int64_t i = 0; i < left && ok; ++i) {
            if (fresh) {
                // the tile's tokens, 64 values a box, spread over the lanes
                const int tok = cur.tile * C::TOK + lane % nb * box;
                const int kv = cur.seq < p.n_seq ? attend_seq(p, cur.seq).kv : 0;
                int y = n_rows;                // behind the last row: zeros
                if (tok < kv) {
                    const int b = tok / T;
                    const int64_t id = p.blocks[cur.seq * p.max_blocks + b];
                    if (id >= 0 && id < p.n_blocks) y = (int)(id * T + (tok - b * T));
                    else if (id != -1) set_status(p.status, AKASHIC_EDEVICE);
                }
                ok = wide_wait(&aempty, (n_tile & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (lead && lane == 0) mbar_expect_tx(&afull, G * C::A_BYTES);
                __syncwarp();
                for (int x = lane; x < C::CHUNKS * nb; x += 32)          // (32 is a multiple of nb: x % nb = lane % nb)
                    load(s_a + x / nb * C::A_CHUNK + lane % nb * box * 128, &rows_map, &afull, x / nb * 64, y);
                ++n_tile;
            }
            const int h = sp.head0 + cur.head;
            for (int c = 0; c < C::CHUNKS; ++c, ++n_w) {
                const uint32_t st = n_w % ST;
                ok = wide_wait(&wempty[st], ((n_w / ST) & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (elect_one()) {
                    if (lead) mbar_expect_tx(&wfull[st], rows_w * 128);
                    unsigned char *to = s_w + st * C::W_BYTES;
                    if constexpr (PAIR) {
                        load(to, lead ? &k_map : &v_map, &wfull[st], c * 64, (int)(h * (lead ? sp.k_step : sp.v_step)));
                    } else {
                        tma_load_2d(to, &k_map, &wfull[st], c * 64, (int)(h * sp.k_step));
                        tma_load_2d(to + lp.nope * 128, &v_map, &wfull[st], c * 64, (int)(h * sp.v_step));
                    }
                }
                __syncwarp();
            }
            fresh = next(cur);
        }
        // nothing is on its way when the CTA ends (where a wait gave up; else all has been read); what the
        // other CTA's barriers tell of is given time instead
        if (!ok && lead) {
            if (n_tile > 0) mbar_wait(&afull, (n_tile - 1) & 1, p.status);
            for (uint32_t i = 0; i < ST; ++i)
                if (n_w > i) mbar_wait(&wfull[(n_w - i - 1) % ST], ((n_w - i - 1) / ST) & 1, p.status);
        }
        for (int i = 0; !ok && !lead && i < 200; ++i) __nanosleep(1000);
        __syncwarp();
    } else if (PAIR && warp == C::WRITE + 1 && !lead) {
        // (the other CTA issues the pair's products)
    } else if (warp == C::WRITE + 1) {
        // ---------------- issuing
        const uint32_t idesc = idesc_f16(rows_w, lp.bf16, 128 * G);
        const uint64_t a_at = desc64(desc_k(smem_u32(s_a))), w_at = desc64(desc_k(smem_u32(s_w)));
        auto commit = [&](uint64_t *bar) {
            if constexpr (PAIR) {
                umma2_commit(bar);
                umma2_commit_to(bar, 1);
            } else {
                umma_commit(bar);
            }
        };
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
                    for (int k = 0; k < 4; ++k) {
                        const uint64_t a = a_at + c * (C::A_CHUNK >> 4) + 2 * k;
                        const uint64_t w = w_at + st * (C::W_BYTES >> 4) + 2 * k;
                        if constexpr (PAIR) umma2_bf16(tmem + acc * 256, a, w, idesc, c > 0 || k > 0);
                        else mma_ss(tmem + acc * 256, a, w, idesc, c > 0 || k > 0);
                    }
                    commit(&wempty[st]);
                }
                __syncwarp();
            }
            if (!ok) break;
            fresh = next(cur);
            if (elect_one()) {
                commit(&tfull[acc]);
                if (fresh) commit(&aempty);
            }
            __syncwarp();
        }
        if (elect_one()) {
            if constexpr (PAIR) umma2_commit(&drained);
            else umma_commit(&drained);
        }
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
            const bool real = cur.seq < p.n_seq;
            const int64_t row = (int64_t)cur.head * sp.seq_rows * p.n_seq + (int64_t)cur.seq * sp.seq_rows +
                                cur.tile * C::TOK + warp * 32 + lane;
            // What a row does not see meets a weight of 0: what is stored of a value is finite.  A token one of whose
            // sums is no number (not finite: of weights that are not, of infinities of both signs) gets a key
            // that is none, so that the rows that see it, and no others, are NaN.  The key's first value is the last
            // to be written.  (Looked for by the largest size of 32 sums, so that the usual ones are not saturated
            // either: calls of one row over 18,600 tokens, 32 heads, R = 512 and 256, 180 and 158 us; by a chain of
            // products with 0 184 and 172; saturated without a look 181 and 160.)
            bool odd = false;                  // a sum that is not finite
#pragma unroll 1
            for (int c = rows_w - 32; real && c >= 0; c -= 32) {
                uint32_t y[32];
                tmem_ld32(tmem + lanes + acc * 256 + c, y);
                tmem_ld_wait();
                float top[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 32; k += 4)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        asm("max.NaN.abs.f32 %0, %0, %1, %2;"
                            : "+f"(top[i])
                            : "f"(__uint_as_float(y[k + 2 * i])), "f"(__uint_as_float(y[k + 2 * i + 1])));
                if (!(top[0] <= most && top[1] <= most)) {
                    odd = odd || !(top[0] < INFINITY && top[1] < INFINITY);
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        y[k] = __float_as_uint(fminf(fmaxf(__uint_as_float(y[k]), -most), most));
                }
                uint32_t h[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float a = __uint_as_float(y[2 * k]), b = __uint_as_float(y[2 * k + 1]);
                    if (lp.bf16) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
                        h[k] = *(const uint32_t *)&v;
                    } else {
                        h[k] = pack_h2(a, b);
                    }
                }
                if (c == 0 && odd) h[0] |= 0x7fffu;     // a NaN of either type
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
            if (lane == 0) {
                if (lead) mbar_arrive(&tempty[acc]);
                else mbar_arrive_remote(&tempty[acc], 0);
            }
            next(cur);
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) {
        cluster_sync();                        // neither leaves while the other may still need it
        tc_fence_after();
        if (warp == 0) tmem_dealloc2(tmem, 512);
    } else {
        tc_fence_after();
        if (warp == 0) tmem_dealloc(tmem, 512);
    }
}

template <int R, bool PAIR>
cudaError_t run_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st) {
    using C = Expand<R, PAIR>;
    auto *kernel = k_latent_expand<R, PAIR>;
    // the CTAs or pairs that fit on the GPU, once a device (another thread that comes first finds the same)
    static std::atomic<int> fit[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    int shares = dev < 64 ? fit[dev].load(std::memory_order_acquire) : 0;
    if (!shares) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) return e;
        shares = device_sm_count();
        if (PAIR) e = pairs_that_fit(kernel, C::THREADS, C::SMEM, &shares);
        if (e != cudaSuccess) return e;
        if (dev < 64) fit[dev].store(shares, std::memory_order_release);
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
    const int box = latent_box(p, 128), n_rows = (int)(p.a.n_blocks * p.a.per_block * KV_UNIT);
    if constexpr (PAIR) return launch_pairs(kernel, shares, C::THREADS, C::SMEM, st, rows, k, v, p, sp, box, n_rows);
    else return launch_pdl(kernel, dim3(shares), dim3(C::THREADS), C::SMEM, st, rows, k, v, p, sp, box, n_rows);
}
// Pairs where weights are widest and a CTA has PAIR_TILES products or more (by the lists' widths; lengths only the
// device knows).  Whole calls of 64 rows with pairs and without, us, by products a CTA: R = 512, 128 + 128 dims, 1:
// 36.5, 36.0; 5: 56.8, 59.1; 10: 87, 95; 20: 138, 155; 40: 223, 258.  R = 256: 1: 34.7, 33.3; 5: 50.6, 51.0; 10: 80,
// 82; 40: 199, 214.  R = 128: 10: 75.1, 74.5; 40: 191, 193.  R = 256, 64 + 64 dims: 10: 56.3, 55.9; 40: 148, 151.
constexpr int PAIR_TILES = 5;
template <int R>
cudaError_t run_expand_form(const LatentParams &p, const LatentSpace &sp, cudaStream_t st) {
    if constexpr (R >= 256)
        if (p.nope == 128 && p.value == 128 && sp.rows / 128 >= (int64_t)PAIR_TILES * device_sm_count())
            return run_expand<R, true>(p, sp, st);
    return run_expand<R, false>(p, sp, st);
}

}  // namespace

cudaError_t launch_latent_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st) {
    return p.R == 128   ? run_expand_form<128>(p, sp, st)
           : p.R == 256 ? run_expand_form<256>(p, sp, st)
                        : run_expand_form<512>(p, sp, st);
}

}  // namespace ak
