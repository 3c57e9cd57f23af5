// Attention of few query rows over the quantised cache (decoding, drafted
// tokens, queries over their retrieved chunks), and the joining of items
// whose steps several CTAs shared.
//
// The cache is read once and everything else is small: bytes bound it (146
// bytes a token and head at D = 128, 4 bits), and next to them the instructions
// that turn codes into fp16, about 1.4 a value.  So:
//  * the scores are computed transposed, S^T = K Q^T, and O^T = V^T P^T: the keys
//    and values are the 16-row operand A of mma.m16n8k16, the query rows (the
//    heads of a group) the 8 columns of B; 8 heads waste nothing, and a
//    unit's codes are turned into A fragments in the registers of the lane that
//    loaded them (ak_kv.cuh): no shuffle, no store to shared memory.  The tensor
//    memory path would want the fp16 tile written to shared memory first.
//  * a nibble n in the low bits of a half is the subnormal n 2^-24; one fused
//    multiply-add by e 2^15 and -8 e 2^-9 gives (n - 8) e 2^-9: one instruction
//    for two values.  Where that is below fp16's normal range it is rounded to
//    its steps of 2^-24, 2^-17 of the row's largest.  A key's 2^T goes to its
//    score, a value's to its weight, in fp32: a row's result depends on what it sees
//    alone.
//  * a warp has its own share of all units (16 tokens), brought by bulk copies
//    into its own ring across the items' ends, with its own running maximum, sum and
//    accumulators: no barrier in the loop.  Where a share begins or ends inside an
//    item, the parts are added up after it, first within the CTA.
//  * P is fp16, p 2^T in units of a power of two (R_SHIFT): those down to 2^-16 of the largest
//    so far keep 11 bits; sums, maxima and accumulators are fp32.  The maximum is raised only when a
//    score exceeds it by 2^8, so that the accumulators are rarely rescaled.
// Measured (one query row of 32 heads a sequence, 8 key/value heads, D = 128, 4 bits): 64
// sequences of 4096, 8192 and 16384 tokens 80, 134 and 241 us, so 5.7 TB/s (84 % of a
// copy) for what is added and 26 us beside it: the plan and the first fetches (8), the rings'
// filling and the warps' uneven ends, the join (4).  In the loop some 310 instructions a unit
// issue in 2.4 of 4 slots (ALU pipe 49 %): they, not the 75 KB in flight an SM, are next to
// the bytes.  8 heads of 700 tokens 13 us, of which 10 are there for 100 tokens too.
#include <atomic>

#include "ak_attend.cuh"
#include "ak_sm100.cuh"

namespace ak {

namespace {

constexpr int NW = 8;                         // warps of a CTA

__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                      uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}
template <int BITS, int D, int NB>
struct Narrow {
    using U = KvUnit<BITS, D>;
    static constexpr int ROWS = 8 * NB;
    // A step is what a warp works on at a time: two units where the registers allow,
    // so that waits, fetches and the checks of maxima and exponents come half as often.
    static constexpr int UPS = D <= 128 ? 2 : 1, STEP = UPS * KV_UNIT;
    static constexpr int STAGE = UPS * (U::BYTES + 64);  // a step's units, then their tags
    static constexpr int ACC = ROWS * D * 4;             // a warp's accumulators
    static constexpr int SMALL = NW * ROWS * 4 * 4 + 2 * NW * ROWS * 12 + 2 * NW * 48 + NW * 64 + 64;
    static_assert(NW * ACC >= (NW * 32 + 1) * 8, "the plan's sums lie where parts come later");
    static constexpr int WANT = (225 * 512 - NW * ACC - SMALL) / (NW * (STAGE + 16));
    static constexpr int MOST = (225 * 1024 - NW * ACC - SMALL) / (NW * (STAGE + 16));
    // two CTAs an SM where the rings of two stages leave room for it
    static constexpr bool TWO = WANT >= 2 && NB == 1 && D <= 128;
    static constexpr int NS_ = TWO ? WANT : MOST;
    static constexpr int NS = NS_ > 8 ? 8 : NS_;
    static_assert(NS >= 2, "a ring of two steps");
    static constexpr int RING = NS * STAGE;              // of a warp; at the end, its accumulators
    static_assert(RING >= ACC, "the last item's accumulators fit the ring");
    static constexpr int SMEM = NW * (RING + NS * 16) + NW * ACC + SMALL;
};

// Where a warp's fetching stands: the item, the steps of it that are the warp's share.
struct Fetch {
    AttendCursor cur;
    int i, n;
};

// A warp's part of an item, left for the joining of the CTA's warps.
struct Entry {
    int64_t start;                             // of the item, in all steps
    int seq, head, tile, unit, n, units;
};
static_assert(sizeof(Entry) <= 48 && sizeof(Fetch) <= 64, "Narrow::SMALL");

__device__ __forceinline__ int r_of(float rf) {  // R of 2^-R
    return 127 - (int)(__float_as_uint(rf) >> 23);
}

// A lane's part of the B fragments of a tile's query rows: row g of each 8, dims
// c D/4 + 4 kk + {0..3}.  bf16 rows are scaled by a power of two to a largest
// magnitude in [1, 2): exact but for values below 2^-14 of it.  Returns 1 / the scale.
template <int D>
__device__ __forceinline__ float load_query(const AttendParams &p, bool bf16, int64_t at, bool real,
                                            uint32_t (&f)[D / 16][2]) {
    const int c = threadIdx.x & 3;
    uint16_t raw[D / 4];
    const uint16_t *src = (const uint16_t *)p.q + at + c * (D / 4);
#pragma unroll
    for (int i = 0; i < D / 4; ++i) raw[i] = 0;
    if (real) {
        if (p.q_wide) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) *(uint4 *)(raw + 8 * i) = *(const uint4 *)(src + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < D / 4; ++i) raw[i] = src[i];
        }
    }
    if (!bf16) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            f[k][0] = raw[4 * k] | (uint32_t)raw[4 * k + 1] << 16;
            f[k][1] = raw[4 * k + 2] | (uint32_t)raw[4 * k + 3] << 16;
        }
        return 1.f;
    }
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < D / 4; ++i) a = fmaxf(a, fabsf(bf16_to_f32(raw[i])));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
    const int e = max(-126, min(126, (int)(__float_as_uint(a) >> 23) - 127));
    const float by = pow2i(-e);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        f[k][0] = pack_h2(bf16_to_f32(raw[4 * k]) * by, bf16_to_f32(raw[4 * k + 1]) * by);
        f[k][1] = pack_h2(bf16_to_f32(raw[4 * k + 2]) * by, bf16_to_f32(raw[4 * k + 3]) * by);
    }
    return pow2i(e);
}

// HEAVY: capped scores or a distance bias.  Compiled apart: their instructions in the loop, though
// jumped over, cost the others 3 % (64 sequences of up to 8192 tokens 89.4 and 86.5 us).
template <int BITS, int D, int NB, bool HEAVY>
__global__ void __launch_bounds__(NW * 32, Narrow<BITS, D, NB>::TWO ? 2 : 1)
k_attend_narrow(const __grid_constant__ AttendParams p, const bool bf16, const int lo, const int hi) {
    using C = Narrow<BITS, D, NB>;
    using U = typename C::U;
    constexpr int ROWS = C::ROWS, NS = C::NS, MT = D / 16, UPS = C::UPS, STEP = C::STEP;
    constexpr int UP = BITS == 4 ? 9 : 0;      // values are staged as v 2^-9 / 2^T
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, c = lane & 3;
    unsigned char *at = smem + NW * C::RING;
    int64_t *prefix = (int64_t *)at;           // until the warps have found their items
    float *heads = (float *)at;                           at += NW * C::ACC;
    Entry *entries = (Entry *)at;                         at += 2 * NW * sizeof(Entry);
    uint64_t *bar = (uint64_t *)at + warp * NS;           at += NW * NS * 8;
    Fetch *ahead = (Fetch *)at + warp;                    at += NW * sizeof(Fetch);
    unsigned char *listed = at + warp * NS * 2;           at += NW * NS * 4;
    float *em = (float *)at;                              at += 2 * NW * ROWS * 4;   // of entries
    float *el = (float *)at;                              at += 2 * NW * ROWS * 4;
    float *er = (float *)at;                              at += 2 * NW * ROWS * 4;
    float *slope = (float *)at + warp * ROWS;             at += NW * ROWS * 4;       // of rows
    int *limit = (int *)at + warp * ROWS;                 at += NW * ROWS * 4;
    int *pos = (int *)at + warp * ROWS;                   at += NW * ROWS * 4;
    int *qtag = (int *)at + warp * ROWS;
    unsigned char *ring = smem + warp * C::RING;

    griddep_wait();
    if (lane == 0)
        for (int i = 0; i < NS; ++i) mbar_init(bar + i, UPS);
    mbar_fence_init();
    if (lane < 2) entries[2 * warp + lane].seq = -1;
    if (tid == 0 && !p.direct) p.joins[blockIdx.x] = make_int4(-1, 0, 0, 0);
    // The warp's share: of all steps, or (p.direct) of the CTA's one item.
    AttendCursor cur = {};
    int64_t per, first;
    int left;
    if (p.direct) {
        cur.seq = blockIdx.x / p.heads, cur.head = blockIdx.x % p.heads;
        cur.q = attend_seq(p, cur.seq);
        cur.units = attend_units(p, cur.q, 0, ROWS, STEP);
        per = (cur.units + NW - 1) / NW;
        first = per * warp;
        cur.unit = (int)first;
        left = max(0, min((int)per, cur.units - cur.unit));
        __syncthreads();
    } else {
        attend_sums(p, ROWS, STEP, 0, lo, hi, prefix);
        const int64_t total = prefix[NW * 32], workers = (int64_t)gridDim.x * NW;
        per = max((int64_t)1, (total + workers - 1) / workers);
        first = per * (blockIdx.x * NW + warp);
        left = (int)max((int64_t)0, min(per, total - first));      // steps of this warp
        if (left > 0) cur = attend_find(p, ROWS, STEP, 0, lo, hi, prefix, first);
        __syncthreads();
    }

    // Fetching runs up to NS steps ahead of the work, across items.  Lane x looks up the x-th unit
    // from the present one, a warp's worth at a time, and copies it itself when
    // its turn comes.  Where fetching stands is kept in shared memory: it is needed
    // once a look-up only, and the registers are not there.
    constexpr int PER = 32 / UPS;              // steps of a look-up
    uint32_t my_unit = 0, my_slots = 0;        // this lane's unit of the cache, its slots / 16
    int my_state = 0;                          // 0: no token of it is seen, 1: by its tags, 3: all are
    int fetch_left = left, turn = 32, turn_end = 32, fetch_stage = 0;
    const bool tags = p.tags != nullptr;
    auto look_up = [&]() {
        AttendCursor x = ahead->cur;
        int i = ahead->i, n = ahead->n;        // steps of the item: done, this share's
        if (i == n) {
            attend_next(p, ROWS, STEP, 0, lo, hi, x);
            i = 0, n = min(x.units, fetch_left);
        }
        __syncwarp();
        const int steps = min(PER, n - i), u = (x.unit + i) * UPS + lane;
        if (lane == 0) *ahead = Fetch{x, i + steps, n};
        my_state = 0;
        if (lane < steps * UPS && u < (x.q.kv + KV_UNIT - 1) / KV_UNIT) {
            const int b = u / p.per_block, w = u - b * p.per_block;
            const int64_t id = p.blocks[x.seq * p.max_blocks + b];
            if (id >= 0 && id < p.n_blocks) {
                my_slots = (uint32_t)id * p.per_block + w;
                my_unit = ((uint32_t)id * p.heads + x.head) * p.per_block + w;
                my_state = tags ? 1 : 3;
                const int r0 = x.tile * ROWS, r1 = min(r0 + ROWS, x.q.nq * p.group) - 1;
                if (tags && r0 / p.group == r1 / p.group) {
                    // One query: a unit of other tags is not fetched, one of its tag needs no
                    // look at the tokens (a retrieved chunk has one tag).
                    const int qt = p.q_tags[x.q.row0 + r0 / p.group];
                    int same = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int4 y = ((const int4 *)p.tags)[(uint64_t)my_slots * 4 + k];
                        same += (y.x == qt) + (y.y == qt) + (y.z == qt) + (y.w == qt);
                    }
                    my_state = qt < 0 || same == 0 ? 0 : same == 16 ? 3 : 1;
                }
            } else if (id != -1) {
                set_status(p.status, AKASHIC_EDEVICE);
            }
        }
        turn = 0, turn_end = steps * UPS;
        __syncwarp();
    };
    // The lanes whose turn it is arrive on the stage's barrier and copy their units, by predicate:
    // the branches around this took a tenth of the step's instructions.
    auto fetch = [&](uint64_t *b, unsigned char *stage_at, unsigned char *flags, int j, bool turn_now) {
        const uint32_t bytes = my_state ? U::BYTES + (my_state == 1 ? 64 : 0) : 0;
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.u32 p, %0, 0;\n\t"
            "setp.ne.and.u32 q, %1, 0, p;\n\t"
            "@p st.shared.u8 [%2], %1;\n\t"
            "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%3], %4;\n\t"
            "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%5], [%6], %7, [%3];\n\t}" ::"r"(
                (uint32_t)turn_now),
            "r"((uint32_t)my_state), "r"(smem_u32(flags + j)), "r"(smem_u32(b)), "r"(bytes),
            "r"(smem_u32(stage_at) + j * U::BYTES), "l"(p.cache + (uint64_t)my_unit * U::BYTES), "n"(U::BYTES)
            : "memory");
        if (turn_now && my_state == 1)
            bulk_load(stage_at + UPS * U::BYTES + j * 64, p.tags + (uint64_t)my_slots * 16, 64, b);
    };
    auto issue = [&]() {
        if (fetch_left == 0) return;
        if (turn == turn_end) look_up();
        const int j = lane - turn;
        fetch(bar + fetch_stage, ring + fetch_stage * C::STAGE, listed + fetch_stage * 2, j, (unsigned)j < (unsigned)UPS);
        turn += UPS, --fetch_left;
        fetch_stage = fetch_stage + 1 == NS ? 0 : fetch_stage + 1;
    };
    if (left > 0) {
        if (lane == 0) *ahead = Fetch{cur, 0, min(cur.units - cur.unit, left)};
        __syncwarp();
        for (int i = 0; i < NS; ++i) issue();
    }

    bool ok = true;                            // no wait of this warp has expired
    uint32_t stage = 0, phase = 0;
    const float cap_l = p.cap * LOG2E_F;
    float o[NB][MT][4], mm[NB][2], l[NB][2];
    float rf[NB][2], rf_most;                  // 2^-R of the rows, the lane's largest
    int64_t done = 0;
    bool tail = false;                         // the accumulators hold the last item's part
    while (left > 0) {
        const int n = min(cur.units - cur.unit, left);
        const AttendSeq sq = cur.q;
        const int row_first = cur.tile * ROWS, rows = min(ROWS, sq.nq * p.group - row_first);

        // ---- the query rows
        __syncwarp();
        float f_own = 0.f;                     // lane r: row r's factor
        uint32_t qf[NB][MT][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int r = b * 8 + g, row = row_first + r;
            const int i = r < rows ? row / p.group : 0;
            const int hd = cur.head * p.group + (r < rows ? row - i * p.group : 0);
            const float f = load_query<D>(p, bf16, (sq.row0 + i) * p.q_row + hd * p.q_head, r < rows, qf[b]);
            if (c == 0) {
                slope[r] = r < rows && p.slopes ? p.slopes[hd] * LOG2E_F : 0.f;
                limit[r] = r < rows ? attend_limit(p, sq, i) : sq.kv;
                pos[r] = sq.kv - sq.nq + i;
                qtag[r] = r < rows && p.q_tags ? p.q_tags[sq.row0 + i] : -1;
            }
            const float x = __shfl_sync(0xffffffffu, f, (lane & 7) * 4);
            if (lane >> 3 == b) f_own = x;
        }
        __syncwarp();
        float qk[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r)
                qk[b][r] = __shfl_sync(0xffffffffu, f_own, b * 8 + 2 * c + r) * p.scale * LOG2E_F *
                           (BITS == 4 ? 512.f : 1.f);
        const int safe = limit[0] - STEP;   // keys below limit[0] are seen by every row

        uint32_t unset = (1u << (2 * NB)) - 1u;    // rows that have not seen a key yet: mm = 0
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int t = 0; t < MT; ++t) o[b][t][0] = o[b][t][1] = o[b][t][2] = o[b][t][3] = 0.f;
            mm[b][0] = mm[b][1] = 0.f, l[b][0] = l[b][1] = 0.f;
            rf[b][0] = rf[b][1] = rf_most = pow2i(-R_MIN);
        }

        int tok = cur.unit * STEP;
        for (int it = 0; ok && it < n; ++it, tok += STEP) {
            // (one answer for all lanes: one that gave up alone would leave the others in a shuffle)
            if (!__all_sync(0xffffffffu, mbar_test_wait(bar + stage, phase)) &&
                !__all_sync(0xffffffffu, mbar_wait(bar + stage, phase, p.status))) {
                ok = false;                    // the other copies still land: wait for them
                const int out = min(left - it, NS);
                for (int k = 1; k < out; ++k) {
                    stage = stage + 1 == NS ? 0 : stage + 1;
                    if (stage == 0) phase ^= 1;
                    mbar_wait(bar + stage, phase, p.status);
                }
                break;
            }
            const unsigned char *st = ring + stage * C::STAGE;
            const uint32_t have = UPS == 2 ? *(const uint16_t *)(listed + stage * 2) : listed[stage * 2];
            if (have) {
                // ---- S^T = K Q^T, per unit
                float s[UPS][NB][4], kf0[UPS], kf1[UPS];   // scales of the keys of tokens g, g + 8
#pragma unroll
                for (int j = 0; j < UPS; ++j) {
                const unsigned char *un = st + j * U::BYTES;
#pragma unroll
                for (int b = 0; b < NB; ++b) s[j][b][0] = s[j][b][1] = s[j][b][2] = s[j][b][3] = 0.f;
                auto keys = [&](int kk, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) mma16(s[j][b], a0, a1, a2, a3, qf[b][kk][0], qf[b][kk][1]);
                };
                if constexpr (BITS == 4) {
                    constexpr int W = D / 32, PER = D / 64;    // words and groups of a token
                    uint32_t w[2][W], sc[(2 * PER + 3) / 4];
                    if constexpr (D == 64) {
                        const uint4 x = *(const uint4 *)(un + U::K_CODES + lane * 16);
                        w[0][0] = x.x, w[0][1] = x.y, w[1][0] = x.z, w[1][1] = x.w;
                        sc[0] = *(const uint16_t *)(un + U::K_SCALES + lane * 2);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int q = 0; q < W / 4; ++q) {
                                const uint4 x = *(const uint4 *)(un + U::K_CODES + ((i * (W / 4) + q) * 32 + lane) * 16);
                                w[i][q * 4] = x.x, w[i][q * 4 + 1] = x.y, w[i][q * 4 + 2] = x.z, w[i][q * 4 + 3] = x.w;
                            }
                        if constexpr (D == 128) {
                            sc[0] = *(const uint32_t *)(un + U::K_SCALES + lane * 4);
                        } else {
                            const uint2 x = *(const uint2 *)(un + U::K_SCALES + lane * 8);
                            sc[0] = x.x, sc[1] = x.y;
                        }
                    }
                    const uint32_t ex = *(const uint16_t *)(un + U::K_EXP + g * 2);
                    kf0[j] = __uint_as_float((ex & 255u) << 23), kf1[j] = __uint_as_float((ex >> 8) << 23);
#pragma unroll
                    for (int gr = 0; gr < PER; ++gr) {
                        uint32_t sj[2], s4[2], cj[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int b = i * PER + gr;
                            const uint32_t by = (sc[b / 4] >> (8 * (b & 3))) & 255u;
                            sj[i] = by * 0x00400040u + 0x3c003c00u;
                            s4[i] = sj[i] - 0x10001000u;
                            cj[i] = h2mul(sj[i], H2_M2_21);
                        }
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            uint32_t h0[4], h1[4];
                            nibbles(w[0][gr * 2 + q], sj[0], s4[0], cj[0], h0);
                            nibbles(w[1][gr * 2 + q], sj[1], s4[1], cj[1], h1);
                            const int kk = (gr * 2 + q) * 2;
                            keys(kk, h0[0], h1[0], h0[1], h1[1]);
                            keys(kk + 1, h0[2], h1[2], h0[3], h1[3]);
                        }
                    }
                } else {
                    constexpr int CH = D / 64;                 // 16-byte chunks of a token
#pragma unroll
                    for (int q = 0; q < CH; ++q) {
                        const uint4 x = *(const uint4 *)(un + U::K_CODES + (q * 32 + lane) * 16);
                        const uint4 y = *(const uint4 *)(un + U::K_CODES + ((CH + q) * 32 + lane) * 16);
                        const uint32_t wx[4] = {x.x, x.y, x.z, x.w}, wy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            keys(q * 4 + i, h2add(__byte_perm(wx[i], 0x64646464u, 0x4140), H2_M1152),
                                 h2add(__byte_perm(wy[i], 0x64646464u, 0x4140), H2_M1152),
                                 h2add(__byte_perm(wx[i], 0x64646464u, 0x4342), H2_M1152),
                                 h2add(__byte_perm(wy[i], 0x64646464u, 0x4342), H2_M1152));
                    }
                    const uint32_t ks = *(const uint32_t *)(un + U::K_SCALES + g * 4);
                    kf0[j] = __uint_as_float(ks << 16), kf1[j] = __uint_as_float(ks & 0xffff0000u);
                }
                }

                // ---- scores in log2 units less the running maximum (mm = m - 6); what a row does not
                // see is -inf.  (The row's factor first: with the key's, 2^125 for a stored infinity,
                // it may be infinite, and a score of 0 then NaN.)
                const int *tg = (const int *)(st + UPS * U::BYTES);
                const bool masked = tok > safe || have != (UPS == 2 ? 0x303u : 3u);
                auto less = [](float a, float f, float m) {    // a f - m, a f rounded: at 2^24 and more its
                    // rounding error is 1 and more, and equal scores would not have equal weights
                    return BITS == 4 ? fmaf(a, f, -m) : __fsub_rn(__fmul_rn(a, f), m);   // (4 bits: exact)
                };
                float most = NEG;
#pragma unroll
                for (int j = 0; j < UPS; ++j) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        if constexpr (HEAVY) {
                            uint32_t x[4];
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                x[r] = __float_as_uint(s[j][b][r] * qk[b][r & 1] * (r < 2 ? kf0[j] : kf1[j]));
                            if (p.cap > 0.f) cap_scores<4>(x, cap_l);
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int col = b * 8 + 2 * c + (r & 1);
                                float &z = s[j][b][r];
                                z = __uint_as_float(x[r]);
                                if (p.slopes)
                                    z -= slope[col] * (float)abs(pos[col] - (tok + j * 16 + g + (r < 2 ? 0 : 8)));
                                z -= mm[b][r & 1];
                            }
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                s[j][b][r] = less(s[j][b][r] * qk[b][r & 1], r < 2 ? kf0[j] : kf1[j], mm[b][r & 1]);
                        }
                        if (masked) {
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int col = b * 8 + 2 * c + (r & 1), t = j * 16 + g + (r < 2 ? 0 : 8);
                                const uint32_t state = have >> (8 * j) & 3u;
                                const int tag = tg[t];         // (no branches: what is not there is not used)
                                const bool seen = (state != 0) & (tok + t < limit[col]) &
                                                  ((state == 3) | ((tag >= 0) & (tag == qtag[col])));
                                if (!seen) s[j][b][r] = -INFINITY;
                            }
                        }
                        most = fmaxf(fmaxf(most, s[j][b][0]), fmaxf(fmaxf(s[j][b][1], s[j][b][2]), s[j][b][3]));
                    }
                }
                // ---- the values' scales, of tokens g and g + 8
                float v[UPS][2], vmax = 0.f;
#pragma unroll
                for (int j = 0; j < UPS; ++j) {
                    const unsigned char *un = st + j * U::BYTES;
                    if constexpr (BITS == 4) {
                        v[j][0] = __uint_as_float((uint32_t)un[U::V_EXP + (g >> 1) * 4 + (g & 1)] << 23);
                        v[j][1] = __uint_as_float((uint32_t)un[U::V_EXP + (g >> 1) * 4 + 2 + (g & 1)] << 23);
                    } else {
                        const uint16_t *vs = (const uint16_t *)(un + U::V_SCALES) + (g >> 1) * 4 + (g & 1);
                        v[j][0] = __uint_as_float((uint32_t)vs[0] << 16), v[j][1] = __uint_as_float((uint32_t)vs[2] << 16);
                    }
                    // where no token was written there may be any bits: times a weight of 0
                    if (masked) v[j][0] = fminf(fabsf(v[j][0]), 1e38f), v[j][1] = fminf(fabsf(v[j][1]), 1e38f);
                    vmax = fmaxf(vmax, fmaxf(v[j][0], v[j][1]));
                }
                // ---- running maxima, and R.  Whether there is something to raise, a bound says that
                // takes in all of the lane's tokens and rows; by how much, a row's own.
                if (__any_sync(0xffffffffu, unset || most > P_SHIFT + M_SLACK ||
                                                ex2(most) * (vmax * rf_most) > (float)(1 << R_SLACK))) {
                    rf_most = 0.f;
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            float x = fmaxf(s[0][b][r], s[0][b][r + 2]);
                            if constexpr (UPS == 2) x = fmaxf(x, fmaxf(s[1][b][r], s[1][b][r + 2]));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                            x -= P_SHIFT;                      // the maximum's rise
                            const bool fresh = unset >> (2 * b + r) & 1u;
                            const bool rise = fresh ? x > -INFINITY : x > M_SLACK;
                            const int rr = r_of(rf[b][r]);
                            int rn = rr;
                            float o_down = 0.f;                // log2
                            if (rise) {                        // R falls by as much: O keeps its scale
                                unset &= ~(1u << (2 * b + r));
                                mm[b][r] += x;
#pragma unroll
                                for (int j = 0; j < UPS; ++j) s[j][b][r] -= x, s[j][b][r + 2] -= x;
                                l[b][r] *= fresh ? 0.f : ex2(-x);
                                rn = fresh ? R_MIN : max(R_MIN, rr - (int)fminf(ceilf(x), 300.f));
                                if (!fresh) o_down = -x;       // (a fresh row's O is 0)
                            }
                            float y = -INFINITY;               // the largest weight times its value's 2^T, log2
#pragma unroll
                            for (int j = 0; j < UPS; ++j)
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    y = fmaxf(y, s[j][b][r + 2 * i] + (float)((int)(__float_as_uint(v[j][i]) >> 23) - 127));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                            if (y > (float)(rn + R_SLACK)) rn = min(R_MAX, (int)ceilf(y) - R_SHIFT);
                            if (rise || rn != rr) {
                                const float2 f = ex2_wide(o_down + (float)(rr - rn));
                                rf[b][r] = pow2i(-rn);
#pragma unroll
                                for (int t = 0; t < MT; ++t)
                                    o[b][t][r] = o[b][t][r] * f.x * f.y, o[b][t][r + 2] = o[b][t][r + 2] * f.x * f.y;
                            }
                            rf_most = fmaxf(rf_most, rf[b][r]);
                        }
                }
                // ---- weights times their values' scales, and P^T as the B operand
                uint32_t pb[UPS][NB][2];
#pragma unroll
                for (int j = 0; j < UPS; ++j)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        float (&z)[4] = s[j][b];
#pragma unroll
                        for (int r = 0; r < 4; ++r) z[r] = ex2(z[r]);
                        l[b][0] += z[0] + z[2], l[b][1] += z[1] + z[3];
                        pb[j][b][0] = transpose8(pack_h2(z[0] * rf[b][0] * v[j][0], z[1] * rf[b][1] * v[j][0]));
                        pb[j][b][1] = transpose8(pack_h2(z[2] * rf[b][0] * v[j][1], z[3] * rf[b][1] * v[j][1]));
                    }

                // ---- O^T += V^T P^T
#pragma unroll
                for (int j = 0; j < UPS; ++j) {
                const unsigned char *un = st + j * U::BYTES;
                auto values = [&](int mt, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                    for (int b = 0; b < NB; ++b) mma16(o[b][mt], a0, a1, a2, a3, pb[j][b][0], pb[j][b][1]);
                };
                if constexpr (BITS == 4) {
                    constexpr int W = D / 64;                  // words a lane has of a token
                    uint32_t w[4][W];                          // tokens 2c, 2c + 1, 2c + 8, 2c + 9
                    if constexpr (W == 1) {
                        const uint4 x = *(const uint4 *)(un + U::V_CODES + lane * 16);
                        w[0][0] = x.x, w[1][0] = x.y, w[2][0] = x.z, w[3][0] = x.w;
                    } else if constexpr (W == 2) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint4 x = *(const uint4 *)(un + U::V_CODES + (i * 32 + lane) * 16);
                            w[2 * i][0] = x.x, w[2 * i][1] = x.y, w[2 * i + 1][0] = x.z, w[2 * i + 1][1] = x.w;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint4 x = *(const uint4 *)(un + U::V_CODES + (i * 32 + lane) * 16);
                            w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
                        }
                    }
                    constexpr int GL = D == 256 ? 2 : 1;       // groups a lane has of a token
#pragma unroll
                    for (int gl = 0; gl < GL; ++gl) {
                        const int gr = D == 64 ? g >> 1 : g * GL + gl;
                        const uint32_t x = *(const uint32_t *)(un + U::V_SCALES + (gr * 4 + c) * 4);
                        const uint32_t s0 = __byte_perm(x, 0, 0x4140) * 64u + 0x3c003c00u;
                        const uint32_t s1 = __byte_perm(x, 0, 0x4342) * 64u + 0x3c003c00u;
                        const uint32_t s04 = s0 - 0x10001000u, s14 = s1 - 0x10001000u;
                        const uint32_t c0 = h2mul(s0, H2_M2_21), c1 = h2mul(s1, H2_M2_21);
                        constexpr int WG = W / GL;             // words of a group
#pragma unroll
                        for (int q = 0; q < WG; ++q) {
                            const int i = gl * WG + q;
                            uint32_t x0[4], y0[4], x1[4], y1[4];
                            nibbles(__byte_perm(w[0][i], w[1][i], 0x5410), s0, s04, c0, x0);
                            nibbles(__byte_perm(w[0][i], w[1][i], 0x7632), s0, s04, c0, y0);
                            nibbles(__byte_perm(w[2][i], w[3][i], 0x5410), s1, s14, c1, x1);
                            nibbles(__byte_perm(w[2][i], w[3][i], 0x7632), s1, s14, c1, y1);
#pragma unroll
                            for (int t = 0; t < 4; ++t) values(i * 4 + t, x0[t], y0[t], x1[t], y1[t]);
                        }
                    }
                } else {
                    constexpr int W = D / 32;                  // words (4 dims) of a token
                    uint32_t w[4][W];
                    if constexpr (W == 2) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint4 x = *(const uint4 *)(un + U::V_CODES + (i * 32 + lane) * 16);
                            w[2 * i][0] = x.x, w[2 * i][1] = x.y, w[2 * i + 1][0] = x.z, w[2 * i + 1][1] = x.w;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int q = 0; q < W / 4; ++q) {
                                const uint4 x = *(const uint4 *)(un + U::V_CODES + ((i * (W / 4) + q) * 32 + lane) * 16);
                                w[i][q * 4] = x.x, w[i][q * 4 + 1] = x.y, w[i][q * 4 + 2] = x.z, w[i][q * 4 + 3] = x.w;
                            }
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t sel = half ? 0x7362 : 0x5140;
                            const uint32_t x = __byte_perm(w[0][i], w[1][i], sel);
                            const uint32_t y = __byte_perm(w[2][i], w[3][i], sel);
                            values(i * 2 + half,
                                   h2add(__byte_perm(x, 0x64646464u, 0x4140), H2_M1152),
                                   h2add(__byte_perm(x, 0x64646464u, 0x4342), H2_M1152),
                                   h2add(__byte_perm(y, 0x64646464u, 0x4140), H2_M1152),
                                   h2add(__byte_perm(y, 0x64646464u, 0x4342), H2_M1152));
                        }
                }
                }
            }
            __syncwarp();                      // the stage has been read
            issue();
            stage = stage + 1 == NS ? 0 : stage + 1;
            if (stage == 0) phase ^= 1;
        }

        // ---- the item, or this warp's part of it, is done
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (unset >> (2 * b + r) & 1u) mm[b][r] = NEG;
#pragma unroll
                for (int off = 4; off < 32; off <<= 1)
                    l[b][r] += __shfl_xor_sync(0xffffffffu, l[b][r], off);
            }
        if (n == cur.units) {                  // whole: written from here
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int x = b * 8 + 2 * c + r, row = row_first + x;
                    if (x >= rows) continue;
                    const int i = row / p.group;
                    const int64_t dst = (int64_t)(sq.row0 + i) * p.q_heads + cur.head * p.group + (row - i * p.group);
                    const float inv = l[b][r] > 0.f ? 1.f / l[b][r] : l[b][r];   // a NaN stays one
                    const int e = r_of(rf[b][r]) + UP;
                    const float up = pow2i(e / 2), up2 = pow2i(e - e / 2);
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        store_pair(p, bf16, dst * D + g * (D / 8) + 2 * t, o[b][t][r] * inv * up * up2,
                                   o[b][t][r + 2] * inv * up * up2);
                    if (g == 0 && p.lse) p.lse[dst] = lse_of(mm[b][r], l[b][r]);
                }
        } else {
            // the share begins or ends inside the item.  A part at the share's
            // beginning leaves the registers now, one at its end after the loop.
            tail = done != 0;
            const int e = 2 * warp + (tail ? 1 : 0);
            if (lane == 0)
                entries[e] = Entry{first + done - cur.unit, cur.seq, cur.head, cur.tile, cur.unit, n, cur.units};
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (g == 0) {
                        const int x = e * ROWS + b * 8 + 2 * c + r;
                        em[x] = mm[b][r], el[x] = l[b][r], er[x] = (float)r_of(rf[b][r]);
                    }
                    if (!tail)
#pragma unroll
                        for (int t = 0; t < MT; ++t)
                            *(float2 *)(heads + (warp * ROWS + b * 8 + 2 * c + r) * D + g * (D / 8) + 2 * t) =
                                make_float2(o[b][t][r], o[b][t][r + 2]);
                }
        }
        left -= n, done += n;
        if (left > 0) attend_next(p, ROWS, STEP, 0, lo, hi, cur);
    }
    if (tail) {
        // nothing is in flight any more: the ring takes the last item's part
        float *own = (float *)ring;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    *(float2 *)(own + (b * 8 + 2 * c + r) * D + g * (D / 8) + 2 * t) =
                        make_float2(o[b][t][r], o[b][t][r + 2]);
    }
    __syncthreads();
    // ---- parts of one item by several warps (neighbours in the order) are added up
    for (int e0 = 0; e0 < 2 * NW;) {
        const Entry a = entries[e0];
        if (a.seq < 0) {
            ++e0;
            continue;
        }
        int e1 = e0 + 1, end = a.unit + a.n;
        for (int e = e1; e < 2 * NW; ++e) {
            const Entry &x = entries[e];
            if (x.seq < 0) continue;
            if (x.start != a.start) break;
            e1 = e + 1, end = x.unit + x.n;
        }
        const AttendSeq sq = attend_seq(p, a.seq);
        const int row_first = a.tile * ROWS, rows = min(ROWS, sq.nq * p.group - row_first);
        const bool whole = a.unit == 0 && end == a.units;
        float *part = p.partial + ((int64_t)blockIdx.x * 2 + (a.unit == 0)) * attend_slot_floats(ROWS, D);
        for (int x = tid; x < ROWS * (D / 2); x += NW * 32) {
            const int r = x / (D / 2), d = x % (D / 2) * 2;
            // a part's sums are in units of its maximum's weight times 2^R: the largest of these
            // units, to a whole power of two, is the sum's
            float mx = NEG, rx = R_MIN, tot = 0.f, v0 = 0.f, v1 = 0.f;
            for (int e = e0; e < e1; ++e)
                if (entries[e].seq >= 0) mx = fmaxf(mx, em[e * ROWS + r]);
            for (int e = e0; e < e1; ++e)
                if (entries[e].seq >= 0) rx = fmaxf(rx, er[e * ROWS + r] + floorf(em[e * ROWS + r] - mx));
            for (int e = e0; e < e1; ++e) {
                if (entries[e].seq < 0) continue;
                const float z = em[e * ROWS + r] - mx, ft = ex2(z + (er[e * ROWS + r] - rx));
                const float *acc = e & 1 ? (const float *)(smem + (e >> 1) * C::RING) : heads + (e >> 1) * ROWS * D;
                const float2 y = *(const float2 *)(acc + r * D + d);
                tot += ex2(z) * el[e * ROWS + r];
                v0 += ft * y.x, v1 += ft * y.y;
            }
            const int up = (int)rx + UP;
            const float inv = tot > 0.f ? 1.f / tot : tot;
            if (!whole) {
                *(float2 *)(part + r * D + d) = make_float2(scale2(v0 * inv, up), scale2(v1 * inv, up));
                if (d == 0) part[ROWS * D + r] = mx, part[ROWS * D + ROWS + r] = tot;
            } else if (r < rows) {
                const int row = row_first + r, i = row / p.group;
                const int64_t dst = (int64_t)(sq.row0 + i) * p.q_heads + a.head * p.group + (row - i * p.group);
                store_pair(p, bf16, dst * D + d, scale2(v0 * inv, up), scale2(v1 * inv, up));
                if (d == 0 && p.lse) p.lse[dst] = lse_of(mx, tot);
            }
        }
        if (tid == 0 && a.unit == 0 && !whole)
            // the item begins here and ends in the share of a later CTA
            p.joins[blockIdx.x] = make_int4(a.seq, a.head, a.tile, (int)((a.start + a.units - 1) / per / NW));
        e0 = e1;
    }
}

// Items whose steps lay in several CTAs: the slots in the order of the CTAs, a CTA 8 rows
// of an item (256 rows in one CTA took 80 us).  The slots' factors first, then the
// sums, eight slots in flight.
constexpr int JOIN_ROWS = 8, JOIN_CTAS = 1024;     // of the kernel before, at most
template <int D>
__global__ void __launch_bounds__(256)
k_attend_join(const AttendParams p, const int rows, const bool bf16) {
    __shared__ float factor[JOIN_ROWS * JOIN_CTAS];    // a slot's share of the row's total
    griddep_wait();
    const int4 j = p.joins[blockIdx.x];
    if (j.x < 0) return;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const AttendSeq sq = attend_seq(p, j.x);
    const int real = min(rows, sq.nq * p.group - j.z * rows);
    const int parts = j.w - (int)blockIdx.x + 1;
    const int64_t floats = attend_slot_floats(rows, D);
    const float *base = p.partial + (int64_t)blockIdx.x * 2 * floats;
    auto slot = [&](int k) { return base + (k ? (int64_t)k * 2 : 1) * floats; };
    const int r0 = blockIdx.y * JOIN_ROWS, n = min(JOIN_ROWS, real - r0);
    if (n <= 0) return;
    if (warp < n) {
        const int r = r0 + warp;
        float mx = NEG, tot = 0.f;
        for (int k = lane; k < parts; k += 32) mx = fmaxf(mx, slot(k)[rows * D + r]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        for (int k = lane; k < parts; k += 32) {
            const float f = ex2(slot(k)[rows * D + r] - mx) * slot(k)[rows * D + rows + r];
            factor[warp * parts + k] = f;
            tot += f;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) tot += __shfl_xor_sync(0xffffffffu, tot, o);
        const float inv = tot > 0.f ? 1.f / tot : tot;         // a NaN stays one
        for (int k = lane; k < parts; k += 32) factor[warp * parts + k] *= inv;
        if (lane == 0) {
            const int row = j.z * rows + r, i = row / p.group;
            if (p.lse)
                p.lse[(int64_t)(sq.row0 + i) * p.q_heads + j.y * p.group + (row - i * p.group)] = lse_of(mx, tot);
        }
    }
    __syncthreads();
    for (int x = tid; x < n * (D / 4); x += 256) {
        const int r = x / (D / 4), d = x % (D / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < parts; ++k) {
            const float f = factor[r * parts + k];
            const float4 y = *(const float4 *)(slot(k) + (r0 + r) * D + d);
            v.x += f * y.x, v.y += f * y.y, v.z += f * y.z, v.w += f * y.w;
        }
        const int row = j.z * rows + r0 + r, i = row / p.group;
        const int64_t dst = (int64_t)(sq.row0 + i) * p.q_heads + j.y * p.group + (row - i * p.group);
        store_pair(p, bf16, dst * D + d, v.x, v.y);
        store_pair(p, bf16, dst * D + d + 2, v.z, v.w);
    }
}

template <int BITS, int D, int NB, bool HEAVY>
cudaError_t run_narrow(const AttendParams &p, int dtype, int ctas, int lo, int hi, cudaStream_t st) {
    using C = Narrow<BITS, D, NB>;
    auto *kernel = k_attend_narrow<BITS, D, NB, HEAVY>;
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
    return launch_pdl(kernel, dim3(ctas), dim3(NW * 32), C::SMEM, st, p, dtype == AKASHIC_DTYPE_BF16, lo, hi);
}
template <int BITS, int D, int NB>
cudaError_t run_narrow_kind(const AttendParams &p, int dtype, int ctas, int lo, int hi, cudaStream_t st) {
    return p.cap > 0.f || p.slopes ? run_narrow<BITS, D, NB, true>(p, dtype, ctas, lo, hi, st)
                                   : run_narrow<BITS, D, NB, false>(p, dtype, ctas, lo, hi, st);
}
template <int BITS, int D>
cudaError_t run_narrow_rows(const AttendParams &p, int dtype, const AttendShape &s, int lo, int hi,
                            cudaStream_t st) {
    if (s.rows == 8) return run_narrow_kind<BITS, D, 1>(p, dtype, s.ctas, lo, hi, st);
    if constexpr (D <= 128) return run_narrow_kind<BITS, D, 2>(p, dtype, s.ctas, lo, hi, st);
    return cudaErrorInvalidValue;
}
template <int BITS>
cudaError_t run_narrow_dim(const AttendParams &p, int dim, int dtype, const AttendShape &s, int lo,
                           int hi, cudaStream_t st) {
    return dim == 64 ? run_narrow_rows<BITS, 64>(p, dtype, s, lo, hi, st)
           : dim == 128 ? run_narrow_rows<BITS, 128>(p, dtype, s, lo, hi, st)
                        : run_narrow_rows<BITS, 256>(p, dtype, s, lo, hi, st);
}
template <int BITS>
int narrow_ctas(int dim) {                     // an SM's, of tiles of 8 rows
    return dim == 64 ? Narrow<BITS, 64, 1>::TWO + 1 : dim == 128 ? Narrow<BITS, 128, 1>::TWO + 1 : 1;
}

}  // namespace

AttendShape attend_narrow_shape(int bits, int dim, int max_rows, int sms) {
    AttendShape s;
    s.rows = max_rows <= 8 || dim == 256 ? 8 : 16;
    const int per = s.rows == 16 ? 1 : bits == 4 ? narrow_ctas<4>(dim) : narrow_ctas<8>(dim);
    s.ctas = sms * per;
    return s;
}

cudaError_t launch_attend_narrow(const AttendParams &p, int bits, int dim, int dtype,
                                 const AttendShape &shape, int lo, int hi, cudaStream_t st) {
    return bits == 4 ? run_narrow_dim<4>(p, dim, dtype, shape, lo, hi, st)
                     : run_narrow_dim<8>(p, dim, dtype, shape, lo, hi, st);
}

cudaError_t launch_attend_join(const AttendParams &p, int dtype, int dim, int ctas, int rows,
                               cudaStream_t st) {
    const bool bf16 = dtype == AKASHIC_DTYPE_BF16;
    auto *kernel = dim == 64 ? k_attend_join<64> : dim == 128 ? k_attend_join<128> : k_attend_join<256>;
    if (ctas > JOIN_CTAS) return cudaErrorInvalidValue;        // (a GPU of more than 512 SMs)
    return launch_pdl(kernel, dim3(ctas, (rows + JOIN_ROWS - 1) / JOIN_ROWS), dim3(256), 0, st, p, rows, bf16);
}

}  // namespace ak

using namespace ak;

namespace {

akashic_status_t attend_check(const akashic_mem_kv_config_t *cfg, const akashic_mem_kv_attend_t *a,
                              const char *who) {
    if (akashic_status_t s = kv_check_config(cfg, who)) return s;
    if (!a) return kv_fail(AKASHIC_EINVAL, "%s: NULL arguments", who);
    if (a->dtype != AKASHIC_DTYPE_BF16 && a->dtype != AKASHIC_DTYPE_FP16)
        return kv_fail(AKASHIC_EINVAL, "%s: dtype must be BF16 or FP16", who);
    if (a->q_heads < 1 || a->q_heads % cfg->heads || a->q_heads / cfg->heads > KV_MAX_HEADS)
        return kv_fail(AKASHIC_EINVAL, "%s: q_heads must be a multiple of heads, at most 1024 times it", who);
    if (a->n_seq < 0 || a->n_q < 0 || a->max_blocks < 0)
        return kv_fail(AKASHIC_EINVAL, "%s: n_seq, n_q and max_blocks must be >= 0", who);
    if (a->max_blocks > 0x7fffff00LL / cfg->block_tokens)
        return kv_fail(AKASHIC_EINVAL, "%s: a list may hold fewer than 2^31 tokens", who);
    if ((int64_t)a->n_q * a->q_heads > 0x7fffffffLL)
        return kv_fail(AKASHIC_EINVAL, "%s: n_q x q_heads must be below 2^31", who);
    if (!a->q_start && a->n_seq > 0 && a->n_q % a->n_seq)
        return kv_fail(AKASHIC_EINVAL, "%s: without q_start, n_q must be a multiple of n_seq", who);
    if (!(a->scale == a->scale) || !(a->scale - a->scale == 0.f))
        return kv_fail(AKASHIC_EINVAL, "%s: scale must be finite", who);
    if (!(a->cap >= 0.f) || !(a->cap - a->cap == 0.f) || (a->cap > 0.f && a->cap < 1.17549435e-38f))
        return kv_fail(AKASHIC_EINVAL, "%s: cap must be 0 or a normal positive number", who);
    if (!a->tags != !a->q_tags)
        return kv_fail(AKASHIC_EINVAL, "%s: tags and q_tags come together", who);
    return AKASHIC_OK;
}

// Which kernels a call launches.  Where all sequences have the same number of rows
// (query rows times group) one takes them all; else each takes the sequences on
// its side of wide_from() rows.
// Microseconds of the kernel for few rows and of the one for many, 4 bits, 2 key/value heads:
//   16 sequences of 5000 tokens, D = 128: 64 rows 52.0 and 45.3, 80 rows 67.5 and 46.0;
//       D = 256: 32 rows 63.5 and 61.4, 40 rows 82.5 and 62.9
//   1024 of 200 tokens, D = 128: 64 rows 199 and 210, 80 rows 283 and 219
// Where so few items share the GPU that more than 16 CTAs leave parts of one to be
// joined, and the work is little, the former stays ahead for longer:
//   one sequence of 20000, D = 128: 128 rows 40.8 and 41.4, 256 rows 53.1 and 47.0;
//       D = 256: 128 rows 64.5 and 63.1, 256 rows 99.6 and 64.9
//   one of 200000, D = 128: 64 rows 92.6 and 87.8, 128 rows 177 and 91.5
int wide_from(const akashic_mem_kv_config_t *cfg, const akashic_mem_kv_attend_t *a, int sms) {
    const int64_t items = (int64_t)a->n_seq * cfg->heads;
    const bool shared = items * 16 < sms && items * a->max_blocks * cfg->block_tokens < (1 << 17);
    return shared ? 129 : cfg->head_dim == 256 ? 33 : 65;
}
// Short lists and no more items than CTAs at once: a CTA an item, as planning and joining would
// take longer than the uneven shares (8 heads of 700 tokens 13.1 and 18.2 us, of 1400
// 17.2 and 18.7, of 2000 19.5 and 18.9).
constexpr int DIRECT_STEPS = 48;   // of 32 tokens: six a warp
struct AttendRoute {
    int from = 0;                                 // rows from which the kernel for many takes a sequence
    AttendShape narrow = {0, 0}, wide = {0, 0};   // ctas 0: not launched
    bool direct = false;                          // a CTA an item, nothing to join
    int64_t joins = 0, bytes = 0;                 // scratch: of the joins, in all
    int64_t narrow_floats = 0, ranges = 0;        // floats of the narrow slots, bytes of the ranges
};
AttendRoute route_of(const akashic_mem_kv_config_t *cfg, const akashic_mem_kv_attend_t *a) {
    AttendRoute r;
    const int64_t rows = (int64_t)a->n_q * (a->q_heads / cfg->heads);
    const int64_t most = a->q_start || a->n_seq == 0 ? rows : rows / a->n_seq;
    const int sms = device_sm_count(), from = r.from = wide_from(cfg, a, sms);
    if (a->q_start || most < from)
        r.narrow = attend_narrow_shape(cfg->bits, cfg->head_dim, (int)(most < from ? most : from - 1), sms);
    if (most >= from) r.wide = attend_wide_shape(cfg->head_dim, sms);
    const int64_t steps = ceil_div(a->max_blocks * cfg->block_tokens, (int64_t)32);
    r.direct = !a->q_start && most <= r.narrow.rows && (int64_t)a->n_seq * cfg->heads <= r.narrow.ctas && steps <= DIRECT_STEPS;
    if (r.direct) return r;                       // no scratch
    r.joins = ceil_div((int64_t)(r.narrow.ctas + r.wide.ctas) * 16, (int64_t)256) * 256;
    r.narrow_floats = r.narrow.ctas * 2 * attend_slot_floats(r.narrow.rows, cfg->head_dim);
    if (r.wide.ctas && a->tags)
        r.ranges = ceil_div(attend_ranges(a->n_q, a->q_heads / cfg->heads, a->n_seq, r.wide.rows) * 8, (int64_t)256) * 256;
    r.bytes = r.joins + r.ranges + (r.narrow_floats + r.wide.ctas * 2 * attend_slot_floats(r.wide.rows, cfg->head_dim)) * 4;
    return r;
}

}  // namespace

extern "C" akashic_status_t akashic_mem_kv_attend_scratch(const akashic_mem_kv_config_t *cfg,
                                                          const akashic_mem_kv_attend_t *a,
                                                          int64_t *bytes) {
    set_last_error("");
    if (akashic_status_t s = attend_check(cfg, a, "kv_attend_scratch")) return s;
    if (!bytes) return kv_fail(AKASHIC_EINVAL, "kv_attend_scratch: NULL bytes");
    KvDevice dev(cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "kv_attend_scratch: device %d cannot be made current", cfg->device);
    *bytes = route_of(cfg, a).bytes;
    return AKASHIC_OK;
}

extern "C" akashic_status_t akashic_mem_kv_attend(const akashic_mem_kv_config_t *cfg,
                                                  const void *cache,
                                                  const akashic_mem_kv_attend_t *a, void *scratch,
                                                  int64_t scratch_bytes, int32_t *status,
                                                  void *stream) {
    set_last_error("");
    if (akashic_status_t s = attend_check(cfg, a, "kv_attend")) return s;
    if (a->n_seq == 0 || a->n_q == 0) return AKASHIC_OK;
    if (!cache || !a->q || !a->out || (!a->blocks && a->max_blocks) || (!scratch && scratch_bytes > 0))
        return kv_fail(AKASHIC_EINVAL, "kv_attend: NULL argument");
    if (((uintptr_t)cache | (uintptr_t)scratch | (uintptr_t)a->tags) & 15u)
        return kv_fail(AKASHIC_EINVAL, "kv_attend: cache, tags and scratch must be 16-byte aligned");
    if ((uintptr_t)a->out & 3u || (uintptr_t)a->q & 1u)
        return kv_fail(AKASHIC_EINVAL, "kv_attend: out must be 4-byte aligned, q to its element");
    if ((uintptr_t)a->blocks & 7u || ((uintptr_t)a->q_start | (uintptr_t)a->kv_len | (uintptr_t)a->prefix_len |
                                      (uintptr_t)a->slopes | (uintptr_t)a->q_tags | (uintptr_t)a->lse) & 3u)
        return kv_fail(AKASHIC_EINVAL, "kv_attend: arrays must be aligned to their element");
    KvDevice dev(cfg->device);
    if (!dev.ok) return kv_fail(AKASHIC_ECUDA, "kv_attend: device %d cannot be made current", cfg->device);
    const AttendRoute r = route_of(cfg, a);
    if (scratch_bytes < r.bytes)
        return kv_fail(AKASHIC_EINVAL, "kv_attend: scratch needs %lld bytes", (long long)r.bytes);
    AttendParams p = {};
    p.cache = (const unsigned char *)cache;
    p.q = a->q, p.q_row = a->q_row_stride, p.q_head = a->q_head_stride;
    p.out = a->out, p.lse = a->lse;
    p.q_start = a->q_start, p.kv_len = a->kv_len, p.prefix = a->prefix_len;
    p.blocks = a->blocks, p.slopes = a->slopes, p.tags = a->tags, p.q_tags = a->q_tags;
    p.status = status;
    p.joins = (int4 *)scratch;
    p.partial = (float *)((unsigned char *)scratch + r.joins + r.ranges);
    p.n_blocks = cfg->n_blocks, p.max_blocks = a->max_blocks;
    p.n_q = a->n_q, p.n_seq = a->n_seq, p.q_heads = a->q_heads, p.heads = cfg->heads;
    p.group = a->q_heads / cfg->heads;
    p.per_block = cfg->block_tokens / KV_UNIT;
    p.max_kv = (int)(a->max_blocks * cfg->block_tokens);
    p.causal = a->causal;
    p.out_wide = !((uintptr_t)a->out & 15u);
    p.q_wide = !(((uintptr_t)a->q | (uintptr_t)((a->q_row_stride | a->q_head_stride) * 2)) & 15u);
    p.scale = a->scale != 0.f ? a->scale : 1.f / sqrtf((float)cfg->head_dim);
    p.cap = a->cap;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    if (r.narrow.ctas) {
        AttendShape shape = r.narrow;
        if (r.direct) p.direct = 1, shape.ctas = a->n_seq * cfg->heads;
        e = launch_attend_narrow(p, cfg->bits, cfg->head_dim, a->dtype, shape, 1, r.from - 1, st);
        if (e == cudaSuccess && !r.direct) e = launch_attend_join(p, a->dtype, cfg->head_dim, r.narrow.ctas, r.narrow.rows, st);
    }
    if (e == cudaSuccess && r.wide.ctas) {
        p.joins += r.narrow.ctas;
        p.partial += r.narrow_floats;
        p.direct = 0;
        if (r.ranges) {
            p.ranges = (const int2 *)((unsigned char *)scratch + r.joins);
            e = launch_attend_ranges(p, cfg->head_dim, r.wide, r.from, 0x7fffffff, st);
        }
        if (e == cudaSuccess)
            e = launch_attend_wide(p, cfg->bits, cfg->head_dim, a->dtype, r.wide, r.from, 0x7fffffff, st);
        if (e == cudaSuccess) e = launch_attend_join(p, a->dtype, cfg->head_dim, r.wide.ctas, r.wide.rows, st);
    }
    if (e != cudaSuccess)
        return kv_fail(AKASHIC_ECUDA, "kv_attend: launch failed: %s", cudaGetErrorString(e));
    return AKASHIC_OK;
}
