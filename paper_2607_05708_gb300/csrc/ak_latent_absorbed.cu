// Absorbed attention over the latent cache, on tcgen05.
//
// Every head reads the same rows [latent | rotated key], so a token's 2 (R + P) bytes meet
// 2 H (2R + P) flops: bytes bound it up to some 64 heads.  Rows of a tile are (query row, head) pairs,
// 16, 32 or 64 of them; a step is 64 tokens at R = 512, else 128.  The products are transposed,
//   S^T = K Q^T      M = tokens, N = rows, K = R + P
//   O^T += C^T P^T   M = 128 latent dims at a time, N = rows, K = tokens
// so that M is full whatever the number of heads, and the R x rows accumulators (4 x 64 columns of
// 128 lanes at R = 512) leave tensor memory for two S.  One copy of a tile in shared memory serves both
// products: as K it is K-major, as C^T the same bytes are MN-major.
//   a warp ahead   looks up the tiles' blocks
//   copying warp   query rows, then the tiles' boxes of tokens: rotated keys, and the latent dims 128 at
//                  a time; blocks that are not listed read as zeros
//   issuing warps  one the scores of the next tile, one O^T += of this one: one warp for both waited for
//                  the softmax of one tile while the next one's scores could have been under way
//   softmax warps  a thread a token and 16 rows.  Weights are relative to a reference of the row, not to its
//                  running maximum, and the reference is raised, O^T and the totals rescaled, only when a
//                  weight would pass 2^SLACK times that: maxima over tokens, which lie across the lanes, are
//                  then not needed tile by tile.  P^T goes to shared memory, MN-major.
// Tiles are shared out evenly over the CTAs (ak_attend.cuh); parts of an item are joined after it
// (ak_latent_join.cu).
//
// Measured (the GPU's time, with the join; R = 512, bf16): 64 requests of up to 8192 tokens, 32 heads, 74 us
// (337 MB: 50 at a copy's rate); 64 heads over 200,000 tokens 63 us (231 MB: 34); 5 drafted rows of 16
// requests, 40 heads, 71 us.  The kernel alone takes 71, 60 and 73 us under the profiler, which empties the caches,
// DRAM 61 and 49 % busy in the first two, the tensor pipe 20 and 32 %.  A step of 64 rows takes 2.6 to 3.5 thousand
// cycles (its products 2000, its bytes 3200 at DRAM's rate with all SMs); a beginning takes 5000, the first pass
// through cold instructions 10000, another item 5000, the join 8 to 12 us.
#include <atomic>

#include "ak_latent.cuh"
#include "ak_umma.cuh"

namespace ak {

namespace {

// Tokens of a tile.  At R = 512 two tiles of 128 have no room, and one and its successor's first chunks
// wait for each other (16 heads over 200,000 tokens 67 us, with tiles of 64 62; 64 heads do not fit at
// all); at R = 256 tiles of 64 only double the waits (44 us with tiles of 128, 48 with 64).
constexpr int tokens_of(int R) { return R == 512 ? 64 : 128; }

template <int R, int NR>
struct Absorbed {
    static constexpr int TOK = tokens_of(R);
    static constexpr int PAIRS = R / 128, CHUNKS = R / 64 + 1;
    static constexpr int CW = 16;                        // rows of a softmax thread
    static constexpr int SOFT = NR / CW * 4;             // softmax warps
    static constexpr int THREADS = 32 * (SOFT + 4);
    static constexpr int PAIR_BYTES = TOK * 256, ROPE_BYTES = TOK * 128;
    static constexpr int Q_BYTES = CHUNKS * NR * 128;
    // P^T: a row a token; 64 bytes of it, in the 64-byte swizzle, hold 32 rows' weights
    static constexpr int P_ROW = NR > 32 ? 128 : 64, P_BYTES = TOK * P_ROW;
    static constexpr int ROOM = 232448 - 1024 - 5120 - Q_BYTES - P_BYTES;
    static constexpr int TILES = ROOM / (PAIRS * PAIR_BYTES + ROPE_BYTES);     // whole tiles on their way
    static constexpr int ROPES = TILES < 1 ? 1 : TILES, STAGES = (ROOM - ROPES * ROPE_BYTES) / PAIR_BYTES;
    static_assert(STAGES > PAIRS, "a tile, and the next on its way");
    static constexpr int SMEM = 1024 + Q_BYTES + P_BYTES + ROPES * ROPE_BYTES + STAGES * PAIR_BYTES;
    static constexpr int S_COL = 256;                    // tensor memory: O^T, then two S^T
    static_assert(PAIRS * NR <= S_COL && S_COL + 2 * NR <= 512, "tensor memory");
    static constexpr int METAS = STAGES / PAIRS + 2;     // tiles whose places are known
    // An item's beginning and end (rows in, result out, an empty pipeline) count as steps.  (2, 4, 7 of
    // them: 5 drafted rows of 16 requests 108, 103, 104 us, 64 requests of 32 heads 91, 89, 89, when measured.)
    static constexpr int EXTRA = 4;
};

// A weight is 2^off where its score is the one that set the row's reference, and 2^(off + SLACK) at
// most.  fp16 has room for 2^15 and down to 2^-24.  bf16's weights are so small (latent_off_bf16) that a row's
// add up to less than 1 in all its parts: values near the type's largest then add up to no infinity.  Weights are
// rounded to the cache's type because a product's operands have one type; totals add up the unrounded ones.
constexpr float SLACK = M_SLACK;

// Whether any thread of the barrier's has `x`, for all of them.
__device__ __forceinline__ bool bar_any(int id, int threads, bool x) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %3, 0;\n\t"
        "barrier.cta.red.or.pred q, %1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"(id), "r"(threads), "r"((uint32_t)x)
        : "memory");
    return any != 0;
}
// v[c], c < N, combined over the warp's lanes: lane L has column L % N.
template <int N, typename F>
__device__ __forceinline__ float over_lanes(float (&v)[N], F f) {
    const int lane = threadIdx.x & 31;
    if constexpr (N == 16) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = f(v[j], __shfl_xor_sync(0xffffffffu, v[j], 16));
    }
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int j = 0; j < o; ++j) {
            const float keep = up ? v[j + o] : v[j], give = up ? v[j] : v[j + o];
            v[j] = f(keep, __shfl_xor_sync(0xffffffffu, give, o));
        }
    }
    return v[0];
}
template <int N>
__device__ __forceinline__ void tmem_ldn(uint32_t at, uint32_t (&r)[N]) {
    if constexpr (N == 32) tmem_ld32(at, r);
    else tmem_ld16(at, r);
}
template <int N>
__device__ __forceinline__ void tmem_stn(uint32_t at, const uint32_t (&r)[N]) {
    if constexpr (N == 32) tmem_st32(at, r);
    else tmem_st16(at, r);
}

template <int R, int NR>
__global__ void __launch_bounds__(Absorbed<R, NR>::THREADS, 1)
k_latent_absorbed(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap pair_map,
                  const __grid_constant__ CUtensorMap q_map, const __grid_constant__ LatentParams lp, const int box,
                  const int n_rows) {
    using C = Absorbed<R, NR>;
    constexpr int TOK = C::TOK, PAIRS = C::PAIRS, ST = C::STAGES, CW = C::CW, THR = 32 * C::SOFT;
    const AttendParams &p = lp.a;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *smem = (unsigned char *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    unsigned char *s_pair = smem, *s_rope = s_pair + ST * C::PAIR_BYTES, *s_p = s_rope + C::ROPES * C::ROPE_BYTES;
    unsigned char *s_q = s_p + C::P_BYTES;
    __shared__ uint64_t full[ST], empty[ST], rope_full[C::ROPES], rope_empty[C::ROPES];
    __shared__ uint64_t sfull[2], pfull[2], odone, qfull, qempty, mfull[C::METAS], mempty[C::METAS], drained[2];
    __shared__ int m_row[C::METAS][8];                   // first row of each of a tile's boxes, -1: none
    __shared__ alignas(16) float c_ref[NR], c_fac[NR];
    __shared__ alignas(16) int c_limit[NR], c_tag[NR];
    __shared__ float c_part[4][NR];
    __shared__ uint32_t tmem_slot;
    __shared__ int dead_word;
    volatile int *dead = &dead_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    griddep_wait();
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
        for (int i = 0; i < C::ROPES; ++i) mbar_init(&rope_full[i], 1), mbar_init(&rope_empty[i], 1);
        for (int i = 0; i < C::METAS; ++i) mbar_init(&mfull[i], 1), mbar_init(&mempty[i], 1);
        for (int i = 0; i < 2; ++i) mbar_init(&sfull[i], 1), mbar_init(&pfull[i], C::SOFT);
        mbar_init(&odone, 1), mbar_init(&qfull, lp.q_map ? 1 : C::SOFT), mbar_init(&qempty, 1);
        mbar_init(&drained[0], 1), mbar_init(&drained[1], 1);
        mbar_fence_init();
        dead_word = 0;
        if (!p.direct) ((LatentJoin *)p.joins)[blockIdx.x] = {0, 0, 0};
    }
    if (warp == 0) {
        tmem_alloc(&tmem_slot, 512);
        tmem_relinquish();
    }
    constexpr int ALL = 0x7fffffff;
    const LatentShare share = latent_share(p, NR, TOK, C::EXTRA, (int64_t *)s_q);      // (until it holds query rows)
    const int64_t first = share.first, per = share.per;
    int left = share.left;
    AttendCursor cur = share.cur;
    fence_async_smem();                    // (copies write where the plan stood)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    if (warp == C::SOFT) {
        // ---------------- copying
        const int nb = TOK / box;              // boxes of a chunk
        uint32_t n_tile = 0, n_pair = 0, n_rope = 0, items = 0;
        bool ok = true;
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            if (part.n <= 0) break;
            if (lp.q_map) {
                // query rows, evenly spaced in memory (those behind the item's are others' or zeros: their results
                // are not written)
                ok = wide_wait(&qempty, (items & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect_tx(&qfull, C::Q_BYTES);
                    for (int c = 0; c < C::CHUNKS; ++c)
                        tma_load_2d(s_q + c * NR * 128, &q_map, &qfull, c * 64, cur.q.row0 * p.group + cur.tile * NR);
                }
                __syncwarp();
                ++items;
            }
            for (int i = 0; ok && i < part.n; ++i, ++n_tile) {
                const uint32_t me = n_tile % C::METAS;
                ok = wide_wait(&mfull[me], (n_tile / C::METAS) & 1, dead, p.status);
                const int *rows = m_row[me];
                // the rotated keys first: their place is free before the others'
                const uint32_t sr = n_tile % C::ROPES;
                if (ok) ok = wide_wait(&rope_empty[sr], ((n_tile / C::ROPES) & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (elect_one()) {
                    mbar_expect_tx(&rope_full[sr], C::ROPE_BYTES);
                    for (int b = 0; b < nb; ++b)
                        tma_load_2d(s_rope + sr * C::ROPE_BYTES + b * box * 128, &rows_map, &rope_full[sr], R,
                                    rows[b] < 0 ? n_rows : rows[b]);
                }
                __syncwarp();
                ++n_rope;
                for (int k = 0; ok && k < PAIRS; ++k, ++n_pair) {
                    const uint32_t st = n_pair % ST;
                    ok = wide_wait(&empty[st], ((n_pair / ST) & 1) ^ 1, dead, p.status);
                    if (!ok) break;
                    if (elect_one()) {
                        unsigned char *to = s_pair + st * C::PAIR_BYTES;
                        mbar_expect_tx(&full[st], C::PAIR_BYTES);
                        // (rows behind the last one: zeros)
                        if (nb == 1) {
                            tma_load_3d(to, &pair_map, &full[st], 0, rows[0] < 0 ? n_rows : rows[0], 2 * k);
                        } else {
                            for (int b = 0; b < nb; ++b) {
                                const int y = rows[b] < 0 ? n_rows : rows[b];
                                tma_load_2d(to + b * box * 128, &rows_map, &full[st], k * 128, y);
                                tma_load_2d(to + C::ROPE_BYTES + b * box * 128, &rows_map, &full[st], k * 128 + 64, y);
                            }
                        }
                    }
                    __syncwarp();
                }
            }
            left -= part.used;
            if (left > 0) attend_next(p, NR, TOK, C::EXTRA, 1, ALL, cur);
        }
        // nothing is on its way when the CTA ends (where a wait gave up; else all has been read)
        if (!ok && items > 0) mbar_wait(&qfull, (items - 1) & 1, p.status);
        for (uint32_t i = 0; !ok && i < ST; ++i)
            if (n_pair > i) mbar_wait(&full[i], ((n_pair - i - 1) / ST) & 1, p.status);
        for (uint32_t i = 0; !ok && i < C::ROPES; ++i)
            if (n_rope > i) mbar_wait(&rope_full[i], ((n_rope - i - 1) / C::ROPES) & 1, p.status);
        __syncwarp();
    } else if (warp == C::SOFT + 2) {
        // ---------------- looking ahead: the tiles' places
        const int nb = TOK / box, T = p.per_block * KV_UNIT;
        uint32_t n_tile = 0;
        bool ok = true;
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            if (part.n <= 0) break;
            const int64_t *list = p.blocks + cur.seq * p.max_blocks;
            // lane: the row of box lane of a tile, -1: none
            auto place = [&](int i) {
                const int tok = (part.from + i) * TOK + lane * box;
                if (lane >= nb || i >= part.n || tok >= cur.q.kv) return -1;
                const int b = tok / T;
                const int64_t id = list[b];
                if (id >= 0 && id < p.n_blocks) return (int)(id * T + (tok - b * T));
                if (id != -1) set_status(p.status, AKASHIC_EDEVICE);
                return -1;
            };
            int next = place(0);
            for (int i = 0; i < part.n; ++i, ++n_tile) {
                const uint32_t me = n_tile % C::METAS;
                const int row = next;
                ok = wide_wait(&mempty[me], ((n_tile / C::METAS) & 1) ^ 1, dead, p.status);
                if (!ok) break;
                if (lane < nb) m_row[me][lane] = row;
                __syncwarp();
                if (lane == 0) mbar_arrive(&mfull[me]);
                next = place(i + 1);
            }
            left -= part.used;
            if (left > 0) attend_next(p, NR, TOK, C::EXTRA, 1, ALL, cur);
        }
    } else if (warp == C::SOFT + 1) {
        // ---------------- issuing S^T = K Q^T, of a tile once the weights of the one before the last are there
        const uint32_t id_s = idesc_f16(NR, lp.bf16, TOK);
        const uint64_t q_at = desc64(desc_k(smem_u32(s_q))), k_at = desc64(desc_k(smem_u32(s_pair)));
        const uint64_t r_at = desc64(desc_k(smem_u32(s_rope)));
        const int rope_steps = lp.P / 16;
        uint32_t t = 0, items = 0, x = 0;      // tiles and pairs since the kernel began
        bool ok = true;
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            if (part.n <= 0) break;
            ok = wide_wait(&qfull, items++ & 1, dead, p.status);
            for (int i = 0; ok && i < part.n; ++i, ++t) {
                const uint32_t d = tmem + C::S_COL + (t & 1) * NR, sr = t % C::ROPES;
                if (t > 1) ok = wide_wait(&pfull[t & 1], (t - 2) >> 1 & 1, dead, p.status);
                if (ok) ok = wide_wait(&rope_full[sr], (t / C::ROPES) & 1, dead, p.status);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    for (int y = 0; y < rope_steps; ++y)
                        mma_ss(d, r_at + sr * (C::ROPE_BYTES >> 4) + 2 * y,
                               q_at + ((C::CHUNKS - 1) * NR * 128 >> 4) + 2 * y, id_s, y > 0);
                    umma_commit(&rope_empty[sr]);
                }
                __syncwarp();
                for (int k = 0; k < PAIRS; ++k, ++x) {
                    const uint32_t st = x % ST;
                    ok = wide_wait(&full[st], (x / ST) & 1, dead, p.status);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t ka = k_at + st * (C::PAIR_BYTES >> 4), qa = q_at + k * (2 * NR * 128 >> 4);
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            mma_ss(d, ka + (y / 4) * (C::ROPE_BYTES >> 4) + 2 * (y % 4),
                                   qa + (y / 4) * (NR * 128 >> 4) + 2 * (y % 4), id_s, true);
                        if (k == PAIRS - 1) umma_commit(&sfull[t & 1]);
                        if (k == PAIRS - 1 && i == part.n - 1) umma_commit(&qempty);
                    }
                    __syncwarp();
                }
            }
            left -= part.used;
            if (left > 0) attend_next(p, NR, TOK, C::EXTRA, 1, ALL, cur);
        }
        if (elect_one()) umma_commit(&drained[0]);             // what was issued ends before the tensor memory goes
        mbar_wait(&drained[0], 0, p.status);
        __syncwarp();
    } else if (warp == C::SOFT + 3) {
        // ---------------- issuing O^T += C^T P^T
        const uint32_t id_o = idesc_f16(NR, lp.bf16) | IDESC_A_MN_MAJOR | IDESC_B_MN_MAJOR;
        const uint64_t v_at = desc64(desc_mn(smem_u32(s_pair), C::ROPE_BYTES));
        const uint64_t p_at = desc64(desc_mn(smem_u32(s_p), 0), C::P_ROW == 128 ? DESC_HI : DESC_HI_64);
        uint32_t t = 0;
        bool ok = true;
        while (left > 0 && ok) {
            const AttendPart part = attend_part(cur, left);
            if (part.n <= 0) break;
            for (int i = 0; i < part.n; ++i, ++t) {
                ok = wide_wait(&pfull[t & 1], t >> 1 & 1, dead, p.status);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll 1
                    for (int m = 0; m < PAIRS; ++m) {          // (short code: the first pass through it is a cold one)
                        const uint32_t st = (t * PAIRS + m) % ST;
                        const uint64_t va = v_at + st * (C::PAIR_BYTES >> 4);
#pragma unroll
                        for (int k = 0; k < TOK / 16; ++k)
                            mma_ss(tmem + m * NR, va + (2048 * k >> 4), p_at + (16 * C::P_ROW * k >> 4), id_o,
                                   i > 0 || k > 0);
                        umma_commit(&empty[st]);
                    }
                    umma_commit(&odone);
                    umma_commit(&mempty[t % C::METAS]);
                }
                __syncwarp();
            }
            left -= part.used;
            if (left > 0) attend_next(p, NR, TOK, C::EXTRA, 1, ALL, cur);
        }
        if (elect_one()) umma_commit(&drained[1]);
        mbar_wait(&drained[1], 0, p.status);
        __syncwarp();
    } else {
        // ---------------- softmax: a lane is token 32 (warp % 4) + lane, rows [c0, c0 + CW).  (Scores of M = 64
        // lie in the first 16 lanes of every 32.)
        const int quad = warp & 3, c0 = warp / 4 * CW, dim = quad * 32 + lane;
        const int key = TOK == 128 ? dim : quad * 16 + (lane & 15);
        const bool used = TOK == 128 || lane < 16;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const float f = p.scale * LOG2E_F;
        const bool tags = p.tags != nullptr;
        uint32_t n_tile = 0;
        // After a wait that gave up the warps wait for nothing more, but go on to the end: they meet at
        // barriers, which have no limit.
        bool ok = true;
        int64_t done = 0;
        while (left > 0) {
            const AttendPart mine = attend_part(cur, left);
            const int n = mine.n;
            if (n <= 0) break;
            const AttendSeq sq = cur.q;
            const int row_first = cur.tile * NR, rows = min(NR, sq.nq * p.group - row_first);
            const float off = lp.bf16 ? latent_off_bf16(sq.kv) : 7.f;
            if (!lp.q_map) {
                // ---- query rows whose strides no tensor map has
                for (int x = tid; x < NR * (R + lp.P) / 8; x += THR) {
                    const int r = x / ((R + lp.P) / 8), g = x - r * ((R + lp.P) / 8);
                    uint4 z = make_uint4(0, 0, 0, 0);
                    if (r < rows) {
                        const uint32_t at = row_first + r, i = at / (uint32_t)p.group;
                        z = load_row8((const uint16_t *)p.q + (int64_t)(sq.row0 + (int)i) * p.q_row +
                                      (int64_t)(at - i * p.group) * p.q_head + g * 8, p.q_wide);
                    }
                    *(uint4 *)(s_q + (g >> 3) * (NR * 128) + r * 128 + (((g & 7) ^ (r & 7)) << 4)) = z;
                }
            }
            named_bar(1, THR);                 // (the item before has been written)
            if (tid < NR) {
                const uint32_t at = row_first + min(tid, rows - 1);
                const int i = (int)(at / (uint32_t)p.group);
                c_ref[tid] = NEG;
                c_limit[tid] = attend_limit(p, sq, i);
                // a slot without a token has tag -1 here, and a row that sees none -2
                const int qt = tags ? p.q_tags[sq.row0 + i] : 0;
                c_tag[tid] = qt < 0 ? -2 : qt;
            }
            fence_async_smem();
            named_bar(1, THR);
            if (!lp.q_map && lane == 0) mbar_arrive(&qfull);
            const int safe = attend_limit(p, sq, row_first / p.group) - TOK;
            // heads of one query row have one tag: a token has it or not
            const bool one_tag = row_first / p.group == (row_first + rows - 1) / p.group;
            float l[CW];
#pragma unroll
            for (int c = 0; c < CW; ++c) l[c] = 0.f;
            for (int i = 0; i < n; ++i, ++n_tile) {
                const int tok = (mine.from + i) * TOK;
                ok = ok && wide_wait(&mfull[n_tile % C::METAS], (n_tile / C::METAS) & 1, dead, p.status);
                const int row = ok ? m_row[n_tile % C::METAS][key / box] : -1;
                bool have = row >= 0 && used;
                int tag = -1;
                if (tags && have) tag = max(-1, p.tags[(int64_t)row + key % box]);
                if (tags && one_tag) have = have && tag == c_tag[0];
                const bool masked = __any_sync(0xffffffffu, used && !have) || (tags && !one_tag) || tok > safe;
                ok = ok && wide_wait(&sfull[n_tile & 1], n_tile >> 1 & 1, dead, p.status);
                tc_fence_after();
                uint32_t raw[CW];
                tmem_ldn<CW>(tmem + lanes + C::S_COL + (n_tile & 1) * NR + c0, raw);
                tmem_ld_wait();
                float x[CW];
#pragma unroll
                for (int c = 0; c < CW; ++c) x[c] = __uint_as_float(raw[c]) * f;
                if (masked) {
                    const int j = have ? tok + key : 0x7fffffff;
#pragma unroll
                    for (int c = 0; c < CW; c += 4) {
                        const int4 lim = *(const int4 *)&c_limit[c0 + c];
                        x[c] = j < lim.x ? x[c] : -INFINITY;
                        x[c + 1] = j < lim.y ? x[c + 1] : -INFINITY;
                        x[c + 2] = j < lim.z ? x[c + 2] : -INFINITY;
                        x[c + 3] = j < lim.w ? x[c + 3] : -INFINITY;
                        if (!tags || one_tag) continue;
                        const int4 y = *(const int4 *)&c_tag[c0 + c];
                        x[c] = tag == y.x ? x[c] : -INFINITY;
                        x[c + 1] = tag == y.y ? x[c + 1] : -INFINITY;
                        x[c + 2] = tag == y.z ? x[c + 2] : -INFINITY;
                        x[c + 3] = tag == y.w ? x[c + 3] : -INFINITY;
                    }
                }
                if (TOK == 64) {
#pragma unroll
                    for (int c = 0; c < CW; ++c) x[c] = used ? x[c] : -INFINITY;
                }
                float most = -INFINITY;
#pragma unroll
                for (int c = 0; c < CW; c += 4) {
                    const float4 m = *(const float4 *)&c_ref[c0 + c];
                    most = fmaxf(fmaxf(most, x[c] - m.x), fmaxf(x[c + 1] - m.y, fmaxf(x[c + 2] - m.z, x[c + 3] - m.w)));
                }
                bool waited = false;           // for the products before
                if (bar_any(2, THR, most > off + SLACK)) {
                    // ---- a row's reference is raised: its maximum over the tile's tokens
                    float v[CW];
#pragma unroll
                    for (int c = 0; c < CW; ++c) v[c] = x[c];
                    const float top = over_lanes<CW>(v, [](float a, float b) { return fmaxf(a, b); });
                    if (lane < CW) c_part[quad][c0 + lane] = top;
                    named_bar(1, THR);
                    if (tid < NR) {
                        const float m = fmaxf(fmaxf(c_part[0][tid], c_part[1][tid]),
                                              fmaxf(c_part[2][tid], c_part[3][tid]));
                        const float was = c_ref[tid];
                        float now = was, fac = 1.f;
                        if (m - was > off + SLACK) now = m - off, fac = was == NEG ? 0.f : ex2(was - now);
                        c_ref[tid] = now, c_fac[tid] = fac;
                    }
                    named_bar(1, THR);
                    float fac[CW];
#pragma unroll
                    for (int c = 0; c < CW; c += 4) *(float4 *)&fac[c] = *(const float4 *)&c_fac[c0 + c];
#pragma unroll
                    for (int c = 0; c < CW; ++c) l[c] *= fac[c];
                    if (i > 0) {
                        ok = ok && wide_wait(&odone, (n_tile - 1) & 1, dead, p.status);
                        waited = true;
                        tc_fence_after();
#pragma unroll 1
                        for (int m = 0; m < PAIRS; ++m) {
                            uint32_t o[CW];
                            tmem_ldn<CW>(tmem + lanes + m * NR + c0, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int c = 0; c < CW; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * fac[c]);
                            tmem_stn<CW>(tmem + lanes + m * NR + c0, o);
                        }
                        tmem_st_wait();
                    }
                }
                uint32_t w[CW / 2];
#pragma unroll
                for (int c = 0; c < CW; c += 4) {
                    const float4 m = *(const float4 *)&c_ref[c0 + c];
                    const float e0 = ex2(x[c] - m.x), e1 = ex2(x[c + 1] - m.y), e2 = ex2(x[c + 2] - m.z),
                                e3 = ex2(x[c + 3] - m.w);
                    l[c] += e0, l[c + 1] += e1, l[c + 2] += e2, l[c + 3] += e3;
                    if (lp.bf16) {
                        const __nv_bfloat162 a = __floats2bfloat162_rn(e0, e1), b = __floats2bfloat162_rn(e2, e3);
                        w[c / 2] = *(const uint32_t *)&a, w[c / 2 + 1] = *(const uint32_t *)&b;
                    } else {
                        w[c / 2] = pack_h2(e0, e1), w[c / 2 + 1] = pack_h2(e2, e3);
                    }
                }
                if (!waited && n_tile > 0)     // P^T has been read
                    ok = ok && wide_wait(&odone, (n_tile - 1) & 1, dead, p.status);
#pragma unroll
                for (int c = 0; used && c < CW / 2; c += 4) {
                    const int ch = c0 / 8 + c / 4;       // 16 bytes of the token's weights
                    const int sw = C::P_ROW == 128 ? ch ^ (key & 7) : ch ^ (key >> 1 & 3);
                    *(uint4 *)(s_p + key * C::P_ROW + (sw << 4)) = make_uint4(w[c], w[c + 1], w[c + 2], w[c + 3]);
                }
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&pfull[n_tile & 1]);
            }
            // ---- totals
            if (left == mine.used) griddep_launch();
            const float sum = over_lanes<CW>(l, [](float a, float b) { return a + b; });
            if (lane < CW) c_part[quad][c0 + lane] = sum;
            ok = ok && wide_wait(&odone, (n_tile - 1) & 1, dead, p.status);
            named_bar(1, THR);
            tc_fence_after();
            // ---- whole items are written, others left for the joining kernel
            const bool whole = n == cur.units;
            float *part = p.partial + ((int64_t)blockIdx.x * 2 + (mine.from == 0)) * attend_slot_floats(NR, R);
            const int64_t dst = (int64_t)sq.row0 * p.group + row_first;
            if (tid < NR) {
                const float tot = (c_part[0][tid] + c_part[1][tid]) + (c_part[2][tid] + c_part[3][tid]);
                c_fac[tid] = tot > 0.f ? 1.f / tot : tot;      // a NaN stays one
                if (!whole) part[NR * R + tid] = c_ref[tid], part[NR * R + NR + tid] = tot;
                else if (tid < rows && p.lse) p.lse[dst + tid] = lse_of(c_ref[tid], tot);
                if (!whole && tid == 0 && mine.from == 0)
                    ((LatentJoin *)p.joins)[blockIdx.x] = {dst, rows,
                                                           (int)((first + done - cur.unit + cur.units - 1) / per)};
            }
            named_bar(1, THR);
            float inv[CW];
#pragma unroll
            for (int c = 0; c < CW; c += 4) *(float4 *)&inv[c] = *(const float4 *)&c_fac[c0 + c];
#pragma unroll 1
            for (int m = 0; m < PAIRS; ++m) {
                uint32_t o[CW];
                tmem_ldn<CW>(tmem + lanes + m * NR + c0, o);
                tmem_ld_wait();
                if (!whole) {
                    float *to = part + c0 * R + m * 128 + dim;
#pragma unroll
                    for (int c = 0; c < CW; ++c) to[c * R] = __uint_as_float(o[c]) * inv[c];
                } else {
                    uint16_t *to = (uint16_t *)p.out + (dst + c0) * R + m * 128 + dim;
#pragma unroll
                    for (int c = 0; c < CW; ++c)
                        if (c0 + c < rows) to[c * R] = round16(__uint_as_float(o[c]) * inv[c], lp.bf16);
                }
            }
            tc_fence_before();
            left -= mine.used, done += mine.used;
            if (left > 0) attend_next(p, NR, TOK, C::EXTRA, 1, ALL, cur);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

struct AbsorbedMaps {
    CUtensorMap rows, pairs, q;        // boxes of 64 values, of 128, of a tile's query rows
};
template <int R, int NR>
cudaError_t run_absorbed(const LatentParams &p, const AbsorbedMaps &m, int box, int n_rows, int ctas, cudaStream_t st) {
    using C = Absorbed<R, NR>;
    auto *kernel = k_latent_absorbed<R, NR>;
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
    return launch_pdl(kernel, dim3(ctas), dim3(C::THREADS), C::SMEM, st, m.rows, m.pairs, m.q, p, box, n_rows);
}
template <int R>
cudaError_t run_absorbed_rows(const LatentParams &p, const AbsorbedMaps &m, int box, int n_rows, int rows, int ctas,
                              cudaStream_t st) {
    return rows == 16   ? run_absorbed<R, 16>(p, m, box, n_rows, ctas, st)
           : rows == 32 ? run_absorbed<R, 32>(p, m, box, n_rows, ctas, st)
                        : run_absorbed<R, 64>(p, m, box, n_rows, ctas, st);
}

// Rows of a tile, from the sequences' rows on average: a tile costs about the same whatever its rows
// while bytes bound it, and fewer leave more room for tokens on their way.
int tile_rows(const LatentParams &p) {
    const int64_t rows = ceil_div((int64_t)p.a.n_q, (int64_t)p.a.n_seq) * p.a.q_heads;
    return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}

// Short lists and no more items than SMs: a CTA an item, no scratch and no joining kernel, up to as many steps one after
// the other as take the GPU no longer than a step a CTA and the join.  The GPU's time in this form and shared out,
// us, by steps, one request of 16 heads: R = 128, 4: 8.4, 12.1; 6: 10.0, 12.8; 8: 11.6, 13.6; 12: 14.9, 15.0; 16: 18.1,
// 16.2.  R = 256, 4: 9.4, 12.1; 6: 11.7, 12.6; 8: 14.0, 13.1.  R = 512, 4: 10.9, 12.5; 6: 13.6, 12.7; 8: 16.4, 13.3.  128
// heads, R = 512, 4: 13.8, 15.4; 6: 17.4, 15.8.  64 requests, R = 512, 6: 14.0, 20.8; 16: 28.0, 26.9.  A call one after
// the other, host and all: up to 8 steps 13 to 16 where shared out 22 to 24 (a launch and an allocation less).
constexpr int DIRECT_STEPS = 6;
int direct_tiles(const LatentParams &p, int sms) {
    if (p.a.q_start) return 0;
    const int64_t tiles = ceil_div((int64_t)p.a.n_q / p.a.n_seq * p.a.q_heads, (int64_t)tile_rows(p));
    const int steps = (int)ceil_div((int64_t)p.a.max_kv, (int64_t)tokens_of(p.R));
    return tiles * p.a.n_seq <= sms && steps <= DIRECT_STEPS ? (int)tiles : 0;
}

}  // namespace

int64_t latent_joins_bytes(int ctas) { return ceil_div((int64_t)ctas * 16, (int64_t)256) * 256; }

int64_t latent_absorbed_scratch(const LatentParams &p) {
    const int ctas = device_sm_count();
    if (direct_tiles(p, ctas)) return 0;
    return latent_joins_bytes(ctas) + (int64_t)ctas * 2 * attend_slot_floats(tile_rows(p), p.R) * 4;
}

int latent_box(const LatentParams &p, int most) {
    const int T = p.a.per_block * KV_UNIT;
    return (T & -T) < most ? (T & -T) : most;
}
cudaError_t latent_rows_map(const LatentParams &p, int most, CUtensorMap *map) {
    const uint64_t rows = (uint64_t)p.a.n_blocks * p.a.per_block * KV_UNIT, wide = p.R + p.P;
    return make_tmap_2d(map, p.a.cache, p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                        wide, rows, wide * 2, 64, (uint32_t)latent_box(p, most));
}

cudaError_t launch_latent_absorbed(LatentParams &p, void *scratch, cudaStream_t st) {
    const int rows = tile_rows(p), tok = tokens_of(p.R), box = latent_box(p, tok);
    int ctas = device_sm_count();
    p.a.direct = direct_tiles(p, ctas);
    if (p.a.direct) ctas = p.a.direct * p.a.n_seq;
    const int n_rows = (int)(p.a.n_blocks * p.a.per_block * KV_UNIT);
    if (!p.a.direct) {
        p.a.joins = (int4 *)scratch;
        p.a.partial = (float *)((unsigned char *)scratch + latent_joins_bytes(ctas));
    }
    const CUtensorMapDataType type = p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    AbsorbedMaps m;
    cudaError_t e = latent_rows_map(p, tok, &m.rows);
    if (e == cudaSuccess) e = make_tmap_cols(&m.pairs, p.a.cache, type, p.R, n_rows, (p.R + p.P) * 2, box, 2);
    if (e != cudaSuccess) return e;
    // rows of (row, head) evenly spaced
    p.q_map = p.a.q_wide && p.a.q_head > 0 && p.a.q_head < (1 << 30) && p.a.q_row == p.a.q_head * p.a.q_heads;
    m.q = m.rows;
    if (p.q_map)
        p.q_map = make_tmap_2d(&m.q, p.a.q, type, 2, p.R + p.P, (uint64_t)p.a.n_q * p.a.q_heads, p.a.q_head * 2, 64,
                               rows) == cudaSuccess;
    e = p.R == 128   ? run_absorbed_rows<128>(p, m, box, n_rows, rows, ctas, st)
        : p.R == 256 ? run_absorbed_rows<256>(p, m, box, n_rows, rows, ctas, st)
                     : run_absorbed_rows<512>(p, m, box, n_rows, rows, ctas, st);
    if (e != cudaSuccess || p.a.direct) return e;
    return launch_latent_join(p, p.R, ctas, rows, 1, st);
}

}  // namespace ak
