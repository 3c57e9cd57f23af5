// Expanded attention over the latent cache, on tcgen05: query rows of a head over its keys
// [w_k c | rotated key] and values w_v c, which ak_latent_expand.cu has left in the scratch (the rotated
// keys come from the cache, for all heads the same).
//
// 2 (nope + P + value) flops a visible pair bound it.  A CTA takes 256 query rows of a sequence and head,
// two row tiles of 128, and runs over tiles of 128 tokens:
//   copying warp   keys and values by tensor maps, in one ring; beside them which tokens are there,
//                  and their tags
//   issuing warp   S = Q K^T into tensor memory, O += P V with P from there.  While one row tile's
//                  scores are in the softmax, the tensor cores work on the other's
//   softmax warps  a thread a row, 64 scores at a time: maximum, weights and total need no shuffle.  P
//                  replaces its scores.  The maximum is raised, and O rescaled, only when a weight would
//                  grow by 2^8.  Weights are rounded to the cache's type, the type of the values that they
//                  multiply; totals add up the unrounded ones
// Tiles are shared out evenly over the CTAs (ak_attend.cuh); parts of an item are joined after it
// (ak_latent_join.cu).
//
// Measured (2 requests of 2048 rows behind 10240 tokens, 32 heads, 128 + 64 and 128 dims): 643 GFLOP in
// 510 us, two thirds of a plain matrix product's burst rate, the tensor pipe 58 % busy; by CTAs alone 517.  A
// step of 256 rows and 128 tokens takes 4300 cycles, its 40 products 2600 at the pipe's rate.  What did not
// help: scaling inside the exponent (32 instructions less of 220 for 64 scores); sixteen softmax warps, two a
// row (661 us for the call's 638: 18 warps leave 96 registers a thread); scores of 64 tokens at a time into
// the columns that the softmax has read, ahead of the weights (716: 24 products of N = 64 more).
#include <atomic>

#include "ak_latent.cuh"
#include "ak_umma.cuh"

namespace ak {

namespace {

constexpr int MIXED = -3;

// PAIR: clusters of two CTAs share an item of twice the rows.  Each has two row tiles of its own, the keys
// of half a tile's tokens and half the dims of its values; the first one's products (cta_group::2) read both
// halves, so that a product of scores reads 6 KB of a CTA's shared memory where it read 8.
template <int DN, int DV, bool PAIR>
struct WideLatent {
    static constexpr int CTAS = PAIR ? 2 : 1;
    static constexpr int TILE_ROWS = 128 * CTAS, ROWS = 2 * TILE_ROWS, TOK = 128, HALF = 64;
    static constexpr int CHUNK = TOK * 128;              // 64 values of 128 rows
    static constexpr int KC = DN / 64 + 1, VC = DV / 64; // chunks of a key, of a value
    static constexpr int Q_TILE = KC * CHUNK, Q_BYTES = 2 * Q_TILE;
    static constexpr int K_ROWS = TOK / CTAS, K_CHUNK = K_ROWS * 128;    // of a CTA
    static constexpr int K_BYTES = KC * K_CHUNK, V_BYTES = VC * CHUNK / CTAS;
    // Keys and values in one ring of chunks, tile by tile.  Two tiles where there is room; else (DN = DV = 128) eight
    // chunks of a tile's five: keys then wait for the values of the tile before the last, values for the scores of
    // the last, which are both over long before.  (Values in a buffer of their own waited for the
    // products with the ones before them: a step of 256 rows and 128 tokens 5000 cycles.)
    // Pairs have room for three tiles.
    static constexpr int TILE = KC + VC, SLOTS = Q_BYTES / CHUNK + 2 * TILE <= 14 ? 2 * TILE : 14 - Q_BYTES / CHUNK;
    static constexpr bool TWO = SLOTS == 2 * TILE;
    static_assert(PAIR || TWO || (KC == 3 && VC == 2 && SLOTS == 8), "what waits for what");
    static_assert(!PAIR || V_BYTES == CHUNK, "half the dims of a value are one chunk");
    static constexpr int DEEP = PAIR ? 3 : 2;            // tiles on their way
    __device__ static uint32_t slot(uint32_t tile, int chunk) { return (tile * TILE + chunk) % SLOTS; }
    // where a tile's chunk stands: of its keys, of its values
    __device__ static uint32_t key_at(uint32_t tile, int c) {
        return PAIR ? tile % DEEP * (K_BYTES + V_BYTES) + c * K_CHUNK : slot(tile, c) * CHUNK;
    }
    __device__ static uint32_t value_at(uint32_t tile, int c) {
        return PAIR ? tile % DEEP * (K_BYTES + V_BYTES) + K_BYTES : slot(tile, KC + c) * CHUNK;
    }
    static constexpr int METAS = 3;                      // tiles whose tags are kept
    static constexpr int SMEM = 1024 + Q_BYTES + (PAIR ? DEEP * (K_BYTES + V_BYTES) : SLOTS * CHUNK);
    static constexpr int SOFT = 8, THREADS = 32 * (SOFT + 2);
    static constexpr int S_COL = 2 * DV;                 // tensor memory: O, then S
    static_assert(S_COL + 2 * TOK <= 512, "tensor memory");
    // An item's beginning and end count as steps.  (2, 3, 4 of them: seven documents in a prompt of 6007 rows, 384
    // items, 98, 101, 102 us.)
    static constexpr int EXTRA = 2;
};

__device__ __forceinline__ void store_row32h(const LatentParams &lp, int64_t at, const uint32_t (&y)[32]) {
    uint32_t h[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const float a = latent_result(__uint_as_float(y[2 * k]), lp.bf16);
        const float b = latent_result(__uint_as_float(y[2 * k + 1]), lp.bf16);
        if (lp.bf16) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
            h[k] = *(const uint32_t *)&v;
        } else {
            h[k] = pack_h2(a, b);
        }
    }
    uint32_t *dst = (uint32_t *)((uint16_t *)lp.a.out + at);
    if (lp.a.out_wide) {
#pragma unroll
        for (int k = 0; k < 16; k += 4) *(uint4 *)(dst + k) = make_uint4(h[k], h[k + 1], h[k + 2], h[k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) dst[k] = h[k];
    }
}

template <int DN, int DV, bool PAIR>
__global__ void __launch_bounds__(WideLatent<DN, DV, PAIR>::THREADS, 1)
k_latent_wide(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap k_map,
              const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap q_map,
              const __grid_constant__ LatentParams lp, const __grid_constant__ LatentSpace sp, const int box,
              const int n_rows) {
    using C = WideLatent<DN, DV, PAIR>;
    constexpr int TOK = C::TOK, ROWS = C::ROWS, HT = C::HALF, ND = C::DEEP;
    const AttendParams &p = lp.a;          // (heads: those of the group; its first is sp.head0)
    extern __shared__ unsigned char raw_smem[];
    unsigned char *smem = (unsigned char *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    unsigned char *s_q = smem, *s_kv = smem + C::Q_BYTES;
    __shared__ uint64_t kfull[ND], kempty[ND], vfull[ND], vempty[ND], mfull[C::METAS];
    __shared__ uint64_t sfull[2], pfull[2][2], odone[2][2], qfull[2], qempty, drained;
    __shared__ alignas(16) int m_tag[C::METAS][TOK];
    __shared__ alignas(16) int m_group[C::METAS][TOK / 16];    // the tag of 16 tokens, MIXED: several
    __shared__ uint32_t m_there[C::METAS]; // of a tile: a bit every 16 tokens that are listed
    __shared__ uint32_t tmem_slot;
    __shared__ int dead_word;
    volatile int *dead = &dead_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u, share_at = blockIdx.x / C::CTAS;
    const bool lead = rank == 0;               // issues the products

    griddep_wait();
    if (tid == 0) {
        for (int i = 0; i < ND; ++i) {
            mbar_init(&kfull[i], 1), mbar_init(&kempty[i], 1);
            mbar_init(&vfull[i], 1), mbar_init(&vempty[i], 1);
        }
        for (int i = 0; i < C::METAS; ++i) mbar_init(&mfull[i], 1);
        for (int t = 0; t < 2; ++t) {
            // One a half: two may be under way, and a wait knows only the last phase from the one
            // before it.
            for (int b = 0; b < 2; ++b) mbar_init(&pfull[t][b], 4 * C::CTAS), mbar_init(&odone[t][b], 1);
            mbar_init(&sfull[t], 1), mbar_init(&qfull[t], lp.q_map ? 1 : 4);
        }
        mbar_init(&qempty, 1), mbar_init(&drained, 1);
        mbar_fence_init();
        dead_word = 0;
        if (lead) ((LatentJoin *)p.joins)[share_at] = {0, 0, 0};
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
    constexpr int ALL = 0x7fffffff;
    // (the plan stands in s_q until query rows come)
    const LatentShare share = latent_share(p, ROWS, TOK, C::EXTRA, (int64_t *)s_q, C::CTAS);
    const int64_t first = share.first, per = share.per;
    int left = share.left;
    AttendCursor cur = share.cur;
    fence_async_smem();                    // (copies write where the plan stood)
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();        // the other CTA's barriers are there
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const bool tags = p.tags != nullptr;
    // a copy whose end the issuing CTA's barrier tells
    auto load = [&](unsigned char *to, const CUtensorMap *map, uint64_t *bar, int x, int y) {
        if (lead) tma_load_2d(to, map, bar, x, y);
        else tma_load_2d_pair(to, map, bar, 0, x, y);
    };

    if (warp == C::SOFT) {
        // ---------------- copying
        const int nb = C::K_ROWS / box, T = p.per_block * KV_UNIT;
        uint32_t n_tile = 0, n_k = 0, n_v = 0, items = 0, q_tiles[2] = {0, 0};
        bool ok = true;
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            if (part.n <= 0) break;
            const int first_tile = part.from + (p.ranges ? p.ranges[attend_range_at(p, cur.q, cur.tile, ROWS)].x : 0);
            if (lp.q_map) {
                // query rows, a row tile's 64 values at a time (those behind the item's are others' or zeros: their
                // results are not written)
                const int rows = cur.q.nq - cur.tile * ROWS;
                ok = wide_wait(&qempty, (items++ & 1) ^ 1, dead, p.status);
                if (!ok) break;
                for (int t = 0; t < (rows > C::TILE_ROWS ? 2 : 1); ++t, __syncwarp()) {
                    ++q_tiles[t];
                    if (!elect_one()) continue;
                    const int y = cur.q.row0 + cur.tile * ROWS + t * C::TILE_ROWS + (int)rank * 128;
                    if (lead) mbar_expect_tx(&qfull[t], C::CTAS * C::Q_TILE);
                    for (int c = 0; c < C::KC; ++c) {
                        unsigned char *to = s_q + t * C::Q_TILE + c * C::CHUNK;
                        if (lead) tma_load_3d(to, &q_map, &qfull[t], c * 64, y, sp.head0 + cur.head);
                        else tma_load_3d_pair(to, &q_map, &qfull[t], 0, c * 64, y, sp.head0 + cur.head);
                    }
                }
            }
            const int64_t *list = p.blocks + cur.seq * p.max_blocks;
            // lane: the row of 16 tokens lane % 8 of a tile, -1: not listed
            auto place = [&](int i) {
                const int tok = (first_tile + i) * TOK + lane % 8 * 16;
                if (i >= part.n || tok >= cur.q.kv) return -1;
                const int b = tok / T;
                const int64_t id = list[b];
                if (id >= 0 && id < p.n_blocks) return (int)(id * T + (tok - b * T));
                if (id != -1) set_status(p.status, AKASHIC_EDEVICE);
                return -1;
            };
            // lane: the tags of four tokens
            auto tags_of = [&](int row) {
                const int r = __shfl_sync(0xffffffffu, row, lane / 4);
                return tags && r >= 0 ? *(const int4 *)(p.tags + (int64_t)r + lane % 4 * 4) : make_int4(-1, -1, -1, -1);
            };
            const int64_t at = ((int64_t)cur.head * p.n_seq + cur.seq) * sp.seq_rows;
            int next = place(0);
            int4 next_tags = tags_of(next);
            for (int i = 0; ok && i < part.n; ++i, ++n_tile) {
                const int row = next, tok = (first_tile + i) * TOK;
                const int4 tag = next_tags;
                next = place(i + 1);
                const uint32_t b = n_tile % ND, me = n_tile % C::METAS;
                // (a tile's meta goes where that of the third before it was: its weights came before the scores of
                // the tile after it, which came before the weights, and so the values, of the second before this)
                if (n_tile >= ND)
                    ok = wide_wait(C::TWO && !PAIR ? &kempty[b] : &vempty[b], (n_tile / ND - 1) & 1, dead, p.status);
                if (!ok) break;
                const uint32_t there = __ballot_sync(0xffffffffu, row >= 0) & 255u;
                if (tags) {
                    const int4 y = make_int4(max(tag.x, -1), max(tag.y, -1), max(tag.z, -1), max(tag.w, -1));
                    *(int4 *)&m_tag[me][4 * lane] = y;
                    int least = min(min(y.x, y.y), min(y.z, y.w)), most = max(max(y.x, y.y), max(y.z, y.w));
#pragma unroll
                    for (int o = 1; o < 4; o *= 2) {
                        least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
                        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                    }
                    if (lane % 4 == 0) m_group[me][lane / 4] = least == most ? least : MIXED;
                }
                if (lane == 0) m_there[me] = there;
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&mfull[me]);
                    if (lead) mbar_expect_tx(&kfull[b], C::CTAS * C::K_BYTES);
                }
                // the sequence's rows in the scratch end with its tiles: behind them zeros
                const int y = tok < max(cur.q.kv, 1) ? (int)(at + tok) : (int)sp.rows;
                const int box_row = __shfl_sync(0xffffffffu, row, ((int)rank * C::K_ROWS + lane % nb * box) / 16);
                __syncwarp();
                if (lane < nb)
                    load(s_kv + C::key_at(n_tile, C::KC - 1) + lane * box * 128, &rows_map, &kfull[b], lp.R,
                         box_row < 0 ? n_rows : box_row);
                else if (lane >= 16 && lane < 16 + C::KC - 1)
                    load(s_kv + C::key_at(n_tile, lane - 16), &k_map, &kfull[b], (lane - 16) * 64,
                         y + (int)rank * C::K_ROWS);
                ++n_k;
                next_tags = tags_of(next);
                if (!PAIR && C::TWO && n_tile > 1) ok = wide_wait(&vempty[b], (n_tile - 2) >> 1 & 1, dead, p.status);
                if (!PAIR && !C::TWO && n_tile > 0)
                    ok = wide_wait(&kempty[b ^ 1], (n_tile - 1) >> 1 & 1, dead, p.status);
                if (!ok) break;
                if (lead && lane == 0) mbar_expect_tx(&vfull[b], C::CTAS * C::V_BYTES);
                __syncwarp();
                if (lane < C::VC / C::CTAS)
                    load(s_kv + C::value_at(n_tile, lane), &v_map, &vfull[b], lane * 64 + (int)rank * (DV / 2), y);
                ++n_v;
            }
            left -= part.used;
            if (left > 0) attend_next(p, ROWS, TOK, C::EXTRA, 1, ALL, cur);
        }
        // nothing is on its way when the CTA ends (where a wait gave up; else all has been read); what the
        // other CTA's barriers tell of is given time instead
        for (int t = 0; !ok && lead && t < 2; ++t)
            if (q_tiles[t]) mbar_wait(&qfull[t], (q_tiles[t] - 1) & 1, p.status);
        for (uint32_t i = 0; !ok && lead && i < ND; ++i) {
            if (n_k > i) mbar_wait(&kfull[(n_k - i - 1) % ND], (n_k - i - 1) / ND & 1, p.status);
            if (n_v > i) mbar_wait(&vfull[(n_v - i - 1) % ND], (n_v - i - 1) / ND & 1, p.status);
        }
        for (int i = 0; !ok && !lead && i < 200; ++i) __nanosleep(1000);
        __syncwarp();
    } else if (PAIR && warp == C::SOFT + 1 && !lead) {
        // (the other CTA issues the pair's products)
    } else if (warp == C::SOFT + 1) {
        // ---------------- issuing
        const uint32_t id_s = idesc_f16(TOK, lp.bf16, C::TILE_ROWS);
        const uint32_t id_o = idesc_f16(DV, lp.bf16, C::TILE_ROWS) | IDESC_B_MN_MAJOR;
        const uint32_t id_half = idesc_f16(64, lp.bf16) | IDESC_B_MN_MAJOR;
        const uint64_t q_at = desc64(desc_k(smem_u32(s_q))), k_at = desc64(desc_k(smem_u32(s_kv)));
        const uint64_t v_at = desc64(desc_mn(smem_u32(s_kv), C::CHUNK));
        const int rope_steps = lp.P / 16;
        uint32_t n_tile = 0, q_phase = 0, tiles0 = 0, tiles1 = 0;      // tiles: of the row tile, so far
        bool ok = true;
        auto commit = [&](uint64_t *bar) {
            if constexpr (PAIR) {
                umma2_commit(bar);
                umma2_commit_to(bar, 1);
            } else {
                umma_commit(bar);
            }
        };
        auto product = [&](uint32_t d, uint64_t a, uint64_t b, bool add) {
            if constexpr (PAIR) umma2_bf16(d, a, b, id_s, add);
            else mma_ss(d, a, b, id_s, add);
        };
        // S of the item's tile i for row tile t; the row tiles share a tile's keys
        auto scores = [&](int t, int i, int mt, bool last) {
            const uint32_t x = n_tile + i;
            if (ok && t == 0) ok = wide_wait(&kfull[x % ND], x / ND & 1, dead, p.status);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = tmem + C::S_COL + t * TOK;
                const uint64_t qa = q_at + t * (C::Q_TILE >> 4);
#pragma unroll
                for (int c = 0; c < C::KC - 1; ++c) {
                    const uint64_t ka = k_at + (C::key_at(x, c) >> 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        product(d, qa + c * (C::CHUNK >> 4) + 2 * k, ka + 2 * k, c > 0 || k > 0);
                }
                const uint64_t ka = k_at + (C::key_at(x, C::KC - 1) >> 4);
                for (int k = 0; k < rope_steps; ++k)
                    product(d, qa + (C::KC - 1) * (C::CHUNK >> 4) + 2 * k, ka + 2 * k, true);
                commit(&sfull[t]);
                if (!PAIR && t == mt - 1) umma_commit(&kempty[x & 1]);
                if (t == mt - 1 && last) commit(&qempty);
            }
            __syncwarp();
        };
        auto values = [&](int t, int i, int b, int mt) {
            const uint32_t x = n_tile + i, c = (t ? tiles1 : tiles0) + i;
            if (ok && t == 0 && b == 0) ok = wide_wait(&vfull[x % ND], x / ND & 1, dead, p.status);
            if (ok) ok = wide_wait(&pfull[t][b], c & 1, dead, p.status);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t va = v_at + (C::value_at(x, 0) >> 4) + b * (HT * 128 >> 4);
                if (PAIR || C::VC == 1 || C::value_at(x, 1) == C::value_at(x, 0) + C::CHUNK) {
#pragma unroll
                    for (int k = 0; k < HT / 16; ++k) {
                        const uint32_t pa = tmem + C::S_COL + t * TOK + b * HT + k * 8;
                        const bool add = i > 0 || b > 0 || k > 0;
                        if constexpr (PAIR) mma2_ts(tmem + t * DV, pa, va + (2048 * k >> 4), id_o, add);
                        else mma_ts(tmem + t * DV, pa, va + (2048 * k >> 4), id_o, add);
                    }
                } else {
                    // the ring's end lies between the chunks: 64 values at a time
                    const uint64_t vb = v_at + (C::value_at(x, 1) >> 4) + b * (HT * 128 >> 4);
#pragma unroll
                    for (int k = 0; k < HT / 16; ++k) {
                        const uint32_t pa = tmem + C::S_COL + t * TOK + b * HT + k * 8;
                        mma_ts(tmem + t * DV, pa, va + (2048 * k >> 4), id_half, i > 0 || b > 0 || k > 0);
                        mma_ts(tmem + t * DV + 64, pa, vb + (2048 * k >> 4), id_half, i > 0 || b > 0 || k > 0);
                    }
                }
                commit(&odone[t][b]);
                if (t == mt - 1 && b == 1) commit(&vempty[x % ND]);
            }
            __syncwarp();
        };
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            const int n = part.n;
            if (n <= 0) break;
            const int mt = cur.q.nq * p.group - cur.tile * ROWS > C::TILE_ROWS ? 2 : 1;
            for (int t = 0; t < mt; ++t) {
                if (ok) ok = wide_wait(&qfull[t], q_phase >> t & 1, dead, p.status);
                q_phase ^= 1u << t;
                scores(t, 0, mt, n == 1);
            }
            for (int i = 0; ok && i < n; ++i) {
                for (int t = 0; t < mt; ++t) {
                    values(t, i, 0, mt);
                    values(t, i, 1, mt);
                    if (i + 1 < n) scores(t, i + 1, mt, i + 2 == n);
                }
            }
            tiles0 += n;
            if (mt > 1) tiles1 += n;
            n_tile += n;
            left -= part.used;
            if (left > 0) attend_next(p, ROWS, TOK, C::EXTRA, 1, ALL, cur);
        }
        if (elect_one()) {
            if constexpr (PAIR) umma2_commit(&drained);
            else umma_commit(&drained);
        }                                      // what was issued ends before the tensor memory goes
        mbar_wait(&drained, 0, p.status);
        __syncwarp();
    } else {
        // ---------------- softmax: a lane is row 32 (warp % 4) + lane of row tile t
        const int t = warp >> 2, rt = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t o_at = tmem + lanes + t * DV;
        const float f = p.scale * LOG2E_F;
        uint32_t n_tile = 0, tiles = 0;        // tiles: of this row tile, so far
        bool ok = true;
        int64_t done = 0;
        while (left > 0 && ok) {
            const AttendPart mine = attend_part(cur, left);
            const int n = mine.n;
            if (n <= 0) break;
            const AttendSeq sq = cur.q;
            const int row_first = cur.tile * ROWS, rows = min(ROWS, sq.nq - row_first);
            const int first_tile = mine.from + (p.ranges ? p.ranges[attend_range_at(p, sq, cur.tile, ROWS)].x : 0);
            // A weight is 2^shift where its score set the row's maximum, 2^(shift + M_SLACK) at most: within fp16's
            // range; a row's bf16 ones less than 1 in all, so that values near the type's largest add up to no
            // infinity.
            const float shift = lp.bf16 ? latent_off_bf16(sq.kv) : P_SHIFT;
            if (t == 0 || rows > C::TILE_ROWS) {
                const int head = sp.head0 + cur.head;
                if (!PAIR && !lp.q_map) {
                    // ---- the warp's 32 query rows, whose strides no tensor map has
                    const int g_all = (DN + lp.P) / 8;
                    for (int x = lane; x < 32 * g_all; x += 32) {
                        const int row = (warp & 3) * 32 + x / g_all, g = x % g_all;
                        uint4 z = make_uint4(0, 0, 0, 0);
                        if (t * 128 + row < rows)
                            z = load_row8((const uint16_t *)p.q + head * p.q_head + g * 8 +
                                          (int64_t)(sq.row0 + row_first + t * 128 + row) * p.q_row, p.q_wide);
                        *(uint4 *)(s_q + t * C::Q_TILE + (g >> 3) * C::CHUNK + row * 128 +
                                   (((g & 7) ^ (row & 7)) << 4)) = z;
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&qfull[t]);
                }
                const int tile_row = t * C::TILE_ROWS + (int)rank * 128, r = tile_row + rt;
                const bool real = r < rows;
                const int limit = real ? attend_limit(p, sq, row_first + r) : sq.kv;
                // a slot without a token has tag -1, and a row that sees none -2
                const int qt = real && tags ? p.q_tags[sq.row0 + row_first + r] : -2, qtag = qt < 0 ? -2 : qt;
                const int safe = attend_limit(p, sq, row_first + tile_row) - HT;
                float mm = 0.f, l = 0.f;
                bool unset = real;             // no key seen yet: mm = 0
                for (int i = 0; i < n; ++i, ++tiles) {
                    const uint32_t me = (n_tile + i) % C::METAS;
                    // (the scores first: a row tile that had no rows in the items before has not followed the
                    // other barrier, and by their time it can be in no later phase)
                    ok = wide_wait(&sfull[t], tiles & 1, dead, p.status);
                    if (ok) ok = wide_wait(&mfull[me], ((n_tile + i) / C::METAS) & 1, dead, p.status);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t there = m_there[me];
#pragma unroll 1
                    for (int b = 0; b < 2; ++b) {
                        const uint32_t s_at = tmem + lanes + C::S_COL + t * TOK + b * HT;
                        const int tok = (first_tile + i) * TOK + b * HT;
                        const uint32_t bits = there >> (4 * b) & 15u;
                        uint32_t x[HT];
                        auto pair = [&](int k) { return f2_pack(__uint_as_float(x[k]), __uint_as_float(x[k + 1])); };
                        tmem_ld32(s_at, *(uint32_t(*)[32])x);
                        tmem_ld32(s_at + 32, *(uint32_t(*)[32])(x + 32));
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < HT; k += 2) {
                            const float2 y = f2_open(f2_mul(pair(k), f2_pack(f, f)));
                            x[k] = __float_as_uint(y.x), x[k + 1] = __float_as_uint(y.y);
                        }
                        // Tags 16 tokens at a time: documents and chunks are longer, so that a row sees all of
                        // them or none (compared one by one a half took 2400 cycles, not 1100).
                        bool masked = tok > safe || bits != 15u;
                        int4 group = make_int4(0, 0, 0, 0);
                        if (tags) {
                            group = *(const int4 *)&m_group[me][4 * b];
                            const bool all = group.x == group.y && group.y == group.z && group.z == group.w &&
                                             group.x == qtag;
                            masked = masked || !__all_sync(0xffffffffu, all || !real);
                        }
                        if (masked) {
#pragma unroll
                            for (int u = 0; u < HT / 16; ++u) {
                                const int of = u == 0 ? group.x : u == 1 ? group.y : u == 2 ? group.z : group.w;
                                int end = bits >> u & 1u ? limit - tok - u * 16 : 0;
                                if (tags && of != MIXED && of != qtag) end = 0;
#pragma unroll
                                for (int k = 0; k < 16; ++k)
                                    if (k >= end) x[u * 16 + k] = 0xff800000u;
                                if (!tags || of != MIXED) continue;
#pragma unroll
                                for (int k = 0; k < 16; k += 4) {
                                    const int4 y = *(const int4 *)&m_tag[me][b * HT + u * 16 + k];
                                    x[u * 16 + k] = y.x == qtag ? x[u * 16 + k] : 0xff800000u;
                                    x[u * 16 + k + 1] = y.y == qtag ? x[u * 16 + k + 1] : 0xff800000u;
                                    x[u * 16 + k + 2] = y.z == qtag ? x[u * 16 + k + 2] : 0xff800000u;
                                    x[u * 16 + k + 3] = y.w == qtag ? x[u * 16 + k + 3] : 0xff800000u;
                                }
                            }
                        }
                        float tops[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) tops[k] = __uint_as_float(x[k]);
#pragma unroll
                        for (int k = 4; k < HT; k += 8)
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                tops[y] = fmaxf(fmaxf(tops[y], __uint_as_float(x[k + y])),
                                                k + 4 + y < HT ? __uint_as_float(x[k + 4 + y]) : -INFINITY);
                        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                        // the maximum is raised when a weight would pass 2^(shift + M_SLACK)
                        const bool rises = unset ? top > -INFINITY : top - mm > shift + M_SLACK;
                        const bool moves = __any_sync(0xffffffffu, rises);         // O changes its scale
                        float down = 1.f;
                        if (rises) {
                            down = unset ? 0.f : ex2(mm - (top - shift));
                            unset = false;
                            mm = top - shift;
                        }
                        uint64_t sum[2] = {0, 0};
                        uint32_t pk[HT / 2];
#pragma unroll
                        for (int k = 0; k < HT; k += 2) {
                            const float2 u = f2_open(f2_add(pair(k), f2_pack(-mm, -mm)));
                            const float e0 = ex2(u.x), e1 = ex2(u.y);
                            sum[k / 2 % 2] = f2_add(sum[k / 2 % 2], f2_pack(e0, e1));
                            if (lp.bf16) {
                                const __nv_bfloat162 w = __floats2bfloat162_rn(e0, e1);
                                pk[k / 2] = *(const uint32_t *)&w;
                            } else {
                                pk[k / 2] = pack_h2(e0, e1);
                            }
                        }
                        const float2 y = f2_open(f2_add(sum[0], sum[1]));
                        l = l * down + (y.x + y.y);
                        tmem_st32(s_at, pk);
                        if (i + b > 0 && moves) {
                            // once the products before have been added
                            ok = wide_wait(&odone[t][b ^ 1], (b ? tiles : tiles - 1) & 1, dead, p.status);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int d = 0; d < DV; d += 32) {
                                uint32_t z[32];
                                tmem_ld32(o_at + d, z);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 32; ++k) z[k] = __float_as_uint(__uint_as_float(z[k]) * down);
                                tmem_st32(o_at + d, z);
                            }
                        }
                        tmem_st_wait();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (lead) mbar_arrive(&pfull[t][b]);
                            else mbar_arrive_remote(&pfull[t][b], 0);
                        }
                    }
                    if (!ok) break;
                }
                if (ok) ok = wide_wait(&odone[t][1], (tiles - 1) & 1, dead, p.status);
                if (!ok) break;
                tc_fence_after();
                // ---- whole items are written, others left for the joining kernel
                const bool whole = n == cur.units;
                if (unset) mm = NEG;
                float *part = p.partial + ((int64_t)share_at * 2 + (mine.from == 0)) * attend_slot_floats(ROWS, DV);
                const float inv = l > 0.f ? 1.f / l : l;       // a NaN stays one
                const int64_t dst = (int64_t)(sq.row0 + row_first + r) * p.q_heads + head;
#pragma unroll 1
                for (int d = 0; d < DV; d += 32) {
                    uint32_t y[32];
                    tmem_ld32(o_at + d, y);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * inv);
                    if (!real) continue;
                    if (whole) {
                        store_row32h(lp, dst * DV + d, y);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *(uint4 *)(part + r * DV + d + k) = make_uint4(y[k], y[k + 1], y[k + 2], y[k + 3]);
                    }
                }
                if (!whole) {
                    part[ROWS * DV + r] = mm, part[ROWS * DV + ROWS + r] = l;
                    if (r == 0 && mine.from == 0)
                        ((LatentJoin *)p.joins)[share_at] = {
                            dst, rows, (int)((first + done - cur.unit + cur.units - 1) / per)};
                }
                tc_fence_before();
            }
            n_tile += n;
            left -= mine.used, done += mine.used;
            if (left > 0) attend_next(p, ROWS, TOK, C::EXTRA, 1, ALL, cur);
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

// Whether query rows come by a tensor map, whose strides are below 2^40 bytes.
bool q_spaced(const LatentParams &p) {
    const int64_t far = 1LL << 32;
    return p.a.q_wide && p.a.q_row > 0 && p.a.q_head > 0 && p.a.q_row < far && p.a.q_head < far;
}

// The CTAs or pairs that a call's steps are shared out to.
template <int DN, int DV, bool PAIR>
cudaError_t wide_shares(int *shares) {
    using C = WideLatent<DN, DV, PAIR>;
    auto *kernel = k_latent_wide<DN, DV, PAIR>;
    // once a device (another thread that comes first finds the same)
    static std::atomic<int> fit[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (*shares = fit[dev].load(std::memory_order_acquire)) > 0) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    *shares = device_sm_count();
    if (PAIR && e == cudaSuccess) e = pairs_that_fit(kernel, C::THREADS, C::SMEM, shares);
    if (e == cudaSuccess && dev < 64) fit[dev].store(*shares, std::memory_order_release);
    return e;
}

template <int DN, int DV, bool PAIR = false>
cudaError_t run_wide(LatentParams &p, const LatentSpace &sp, int shares, cudaStream_t st) {
    using C = WideLatent<DN, DV, PAIR>;
    auto *kernel = k_latent_wide<DN, DV, PAIR>;
    cudaError_t e = cudaSuccess;
    const CUtensorMapDataType type = p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap rows, k, v;
    e = latent_rows_map(p, C::K_ROWS, &rows);
    if (e == cudaSuccess) e = make_tmap_2d(&k, sp.k, type, 2, DN, (uint64_t)sp.rows, DN * 2, 64, C::K_ROWS);
    if (e == cudaSuccess) e = make_tmap_2d(&v, sp.v, type, 2, DV, (uint64_t)sp.rows, DV * 2, 64, C::TOK);
    CUtensorMap q = rows;
    p.q_map = q_spaced(p);
    if (e == cudaSuccess && p.q_map)
        p.q_map = make_tmap_3d(&q, p.a.q, type, DN + p.P, (uint64_t)p.a.n_q, p.a.q_row * 2, (uint64_t)p.a.q_heads,
                               p.a.q_head * 2, 64, 128) == cudaSuccess;
    if (PAIR && !p.q_map) e = cudaErrorInvalidValue;
    if (e != cudaSuccess) return e;
    const int box = latent_box(p, C::K_ROWS), n_rows = (int)(p.a.n_blocks * p.a.per_block * KV_UNIT);
    if constexpr (PAIR)
        return launch_pairs(kernel, shares, C::THREADS, C::SMEM, st, rows, k, v, q, p, sp, box, n_rows);
    else
        return launch_pdl(kernel, dim3(shares), dim3(C::THREADS), C::SMEM, st, rows, k, v, q, p, sp, box, n_rows);
}

constexpr int WIDE_ROWS = 256;
// Keys and values are stored 32 bytes at a time, and the caller's scratch need only be 16-byte aligned: they begin at
// the next whole line, for which the scratch has room.
constexpr int KEYS_AT = 128;
// The heads whose keys and values are in the scratch at a time: all, as far as these take 2 GB.
struct Plan {
    int64_t seq_rows, joins, ranges, partial, k, v;    // rows a sequence and head; bytes
    int heads, ctas;
};
Plan plan_of(const LatentParams &p) {
    Plan x;
    x.ctas = device_sm_count();
    x.seq_rows = latent_seq_rows(p.a.max_kv);
    const int64_t rows = x.seq_rows * p.a.n_seq, room = (2LL << 30) / (rows * (p.nope + p.value) * 2);
    const int64_t most = room < 1 ? 1 : room < p.a.q_heads ? room : p.a.q_heads;
    x.heads = (int)ceil_div((int64_t)p.a.q_heads, ceil_div((int64_t)p.a.q_heads, most));
    x.joins = latent_joins_bytes(x.ctas);
    x.ranges = p.a.tags ? ceil_div(attend_ranges(p.a.n_q, 1, p.a.n_seq, WIDE_ROWS) * 8, (int64_t)256) * 256 : 0;
    x.partial = x.ctas * 2 * attend_slot_floats(WIDE_ROWS, p.value) * 4;
    x.k = rows * x.heads * p.nope * 2, x.v = rows * x.heads * p.value * 2;
    return x;
}

// Pairs of CTAs where keys and values are widest, sequences have rows for them and lists are long: their products
// are faster, beginnings and ends of items slower.  The GPU's time of whole calls with pairs and without, us, sequences
// x rows / context, heads (R = 512): 1 x 1024 / 2048, 16: 60, 57; 4 x 1024 / 2048, 16: 131, 127; 1 x 4096 / 4096, 16: 137,
// 133; 4 x 1024 / 4096, 16: 208, 214; 4 x 1024 / 4096, 32: 356, 374; 4 x 512 / 6144, 32: 352, 366; 1 x 8192 / 8192, 16: 334,
// 331; 2 x 2048 / 8192, 32: 549, 582; 2 x 2048 / 10240, 32: 675, 725; 2 x 600 / 10240, 32: 415, 387; 1 x 2048 / 16384, 16:
// 308, 324; R = 256, 1 x 512 / 32768, 16: 227, 239.  From 4096 on what is gained or lost goes by how items fall on the
// CTAs; from 8192 on it is a gain in most.  Contexts shorter than their lists only the device knows: in lists of 8192,
// 4 x 1024 / 2048, 16: 131, 127; 16 x 700 / 700, 16: 172, 148; 8 x 512 / 512, 16: 80, 72.
constexpr int PAIR_ROWS = 512, PAIR_KV = 8192;
bool pairs_for(const LatentParams &p) {
    return p.nope == 128 && p.value == 128 && q_spaced(p) && p.a.n_q >= (int64_t)PAIR_ROWS * p.a.n_seq &&
           p.a.max_kv >= PAIR_KV;
}

}  // namespace

int64_t latent_expanded_scratch(const LatentParams &p) {
    const Plan x = plan_of(p);
    return x.joins + x.ranges + x.partial + KEYS_AT - 16 + x.k + x.v;
}

cudaError_t launch_latent_expanded(LatentParams &p, void *scratch, cudaStream_t st) {
    const Plan x = plan_of(p);
    unsigned char *at = (unsigned char *)scratch;
    AttendParams &a = p.a;
    LatentSpace sp = {};
    a.joins = (int4 *)at, at += x.joins;
    int2 *ranges = (int2 *)at;
    at += x.ranges;
    a.partial = (float *)at, at += x.partial;
    at = (unsigned char *)(((uintptr_t)at + KEYS_AT - 1) & ~(uintptr_t)(KEYS_AT - 1));
    sp.k = at, sp.v = at + x.k;            // (x.k: a multiple of 128 rows)
    sp.seq_rows = x.seq_rows;
    sp.k_step = p.k_head / p.k_row, sp.v_step = p.v_head / p.v_row;
    // (a pair's part has twice the rows, and there are at most half as many: the scratch is the same)
    const bool pair = pairs_for(p);
    const int rows = pair ? 2 * WIDE_ROWS : WIDE_ROWS;
    int shares = 0;
    cudaError_t e = pair                               ? wide_shares<128, 128, true>(&shares)
                    : p.nope == 64 && p.value == 64    ? wide_shares<64, 64, false>(&shares)
                    : p.nope == 64                     ? wide_shares<64, 128, false>(&shares)
                    : p.value == 64                    ? wide_shares<128, 64, false>(&shares)
                                                       : wide_shares<128, 128, false>(&shares);
    if (x.ranges && e == cudaSuccess) {
        a.ranges = ranges;
        e = launch_attend_ranges(a, 128, {rows, shares}, 1, 0x7fffffff, st);
    }
    for (int h = 0; e == cudaSuccess && h < a.q_heads; h += x.heads) {
        sp.head0 = h, sp.heads = a.heads = a.q_heads - h < x.heads ? a.q_heads - h : x.heads;
        sp.rows = x.seq_rows * a.n_seq * sp.heads;
        e = launch_latent_expand(p, sp, st);
        if (e == cudaSuccess)
            e = pair                            ? run_wide<128, 128, true>(p, sp, shares, st)
                : p.nope == 64 && p.value == 64 ? run_wide<64, 64>(p, sp, shares, st)
                : p.nope == 64                  ? run_wide<64, 128>(p, sp, shares, st)
                : p.value == 64                 ? run_wide<128, 64>(p, sp, shares, st)
                                                : run_wide<128, 128>(p, sp, shares, st);
        if (e == cudaSuccess) e = launch_latent_join(p, p.value, shares, rows, a.q_heads, st);
    }
    return e;
}

}  // namespace ak
