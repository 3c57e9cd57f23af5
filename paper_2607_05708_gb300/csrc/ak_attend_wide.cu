// Attention of many query rows (prompts, long drafts) over the quantised cache, on
// tcgen05.
//
// The products bound it: 4 D flops a visible pair.  A CTA takes 256 query rows (two
// M = 128 tiles; one at D = 256, where an accumulator fills half of the tensor memory) of a
// sequence and key/value head and runs over tiles of N = 128 tokens (64 at D = 256):
//   dequantising warps  a unit's codes from global memory into registers, from
//       there as fp16 into shared memory in the 128-byte swizzle: keys K-major,
//       values MN-major, which is the same layout (rows of tokens, 64 dims wide).
//       One pass serves both row tiles;
//   issuing thread      S = Q K^T into tensor memory, O += P V with P from there.  While
//       one row tile's scores are in the softmax, the tensor cores work on the
//       other's.  (At D = 256 on the next 64 tokens' scores; at D <= 128 S = 128 x 64
//       would take as long as 128 x 128: 75 and 64 cycles for 16 dims.)  It waits
//       by polling: mbarrier.try_wait costs some 200 cycles even on a phase that is over;
//   softmax warps       a thread a row, 64 scores at a time: maximum, weights and total
//       need no shuffle.  P (fp16) replaces its scores.  The maximum is raised,
//       and O rescaled, only when a weight would exceed 2^14.
// A 4-bit key or value is staged in fp16 as it is, c e 2^T (times 2^STAGE), where its row's T lies in a window
// (KEY_LO and so on); outside of it at the window's end, with the rest of its power of two as a factor, in
// fp32, of the key's scores or the value's weight.  8 bits: as codes, the scale the factor.  So a
// score and a weight depend on their own key and value alone, whatever else is in the tile, and
// a half of a tile whose factors are all 1 skips them.  Where fp16's normal range ends keys and
// values are rounded to 2^-17 of their own row's largest.  (Factors for all 4-bit rows: prompts of 2048 and
// 1600 rows 734 us for 710, capped 1060 for 932, though a word of codes takes 11 instructions for 9;
// with all values outside of the window 1134.)
// A weight times its value's factor is divided by the row's 2^R before it becomes fp16.  R goes by what the
// row has seen: raised, and O rescaled, only when a product would pass 2^14 (R_SLACK); 0 while all
// of the row's values have been within the window.
// Measured (4 bits): requests of 2048 and 1668 rows behind 10240 and 8341 tokens, 32 heads on 8, D = 128 (514
// GFLOP) 749 us, 0.69 PFLOP/s, and 1013 us with capped scores; some 3.4 us a step of 256 rows and
// 128 tokens, items' ends apart, of which the products are 1.06: scores, softmax and O += P V of a
// row tile follow each other, and tensor memory (O of two tiles, and S) has no room for a
// second S at D = 128.  One request of 2048 rows behind 8192 tokens: D = 64 272, 128 351, 256 869 us.
#include <stddef.h>

#include <atomic>

#include "ak_attend.cuh"
#include "ak_sm100.cuh"

namespace ak {

namespace {

template <int D>
struct Wide {
    static constexpr int MT = D == 256 ? 1 : 2;          // row tiles of 128
    static constexpr int ROWS = 128 * MT;
    static constexpr int N = D == 256 ? 64 : 128;        // tokens of a tile
    static constexpr int UNITS = N / KV_UNIT;
    static constexpr int HT = 64, HPT = N / HT;          // tokens the softmax takes at a time
    static constexpr int SN = MT == 2 ? N : HT;          // columns of S computed at once
    // Warps: softmax, dequantising, one that issues.  At D <= 128 the registers of five
    // warpgroups are split by need, so that a unit of a tile has a warp of its own.
    // For softmax, dequantising, the last one, a thread; together the 96 of the launch.  Requests
    // of 2048 and 1600 rows behind 10240 and 8000 tokens, 32 heads on 8, D = 128, us:
    //                    120, 80, 80   136, 80, 48   144, 72, 48   152, 64, 48   160, 56, 48
    //   4 bits                   691           711           712           710           706
    //   4 bits, capped           908           915           921           906           923
    //   8 bits                  1273          1001           929           782           786
    //   8 bits, capped          1672          1349          1280          1158          1117
    static constexpr int regs(int role) { return role == 0 ? 160 : role == 1 ? 56 : 48; }
    static constexpr bool SPLIT = MT == 2;
    static constexpr int SOFT = 4 * MT, DEQ = SPLIT ? 8 : 4;
    static constexpr int THREADS = 32 * (SOFT + DEQ + (SPLIT ? 4 : 1));
    static_assert(!SPLIT || 256 * (regs(0) + regs(1)) + 128 * regs(2) <= THREADS * 96, "registers");
    static_assert(UNITS == DEQ, "a dequantising warp has one unit of every tile");
    static constexpr int STAGES = 2;
    // An item's beginning and end (query rows in, result out, an empty pipeline: 7 to 10 us; a step
    // 3) count as steps: 0, 1, 2 and 3 of them 145, 124, 124 and 130 us for 7 documents in
    // 6007 tokens at D = 64, 8 bits; 177, 146, 143 and 149 at D = 128, 4 bits (L2 cold).
    static constexpr int EXTRA = 2;
    static constexpr int Q_BYTES = ROWS * D * 2, KV_BYTES = N * D * 2;
    static constexpr int S_COL = MT * D;                 // tensor memory: O, then S
    static constexpr uint32_t TMEM_COLS = 512;
    static_assert(S_COL + MT * 2 * HT <= 512, "tensor memory");
    static constexpr int SMEM = 1024 + Q_BYTES + 2 * STAGES * KV_BYTES;
};

// What the consumers of a tile need beside the operands.
template <int N>
struct alignas(16) Meta {           // pairs of its floats are read at once
    // The factors of the keys (times 2^-KEY_DOWN) and of the values, 1 where there is no token; 4 bits:
    // written where a unit has one that is not 1 (bent)
    float ksig[N], vsig[N];
    int tag[N];
    int tok;                        // first token
    // of each unit: the largest exponent of its values' factors, biased by 127, 0 if it has no
    // token; whether it is bent
    alignas(8) unsigned char vtop[N / KV_UNIT], bent[N / KV_UNIT];
};
// The windows of T.  Upwards 72 s (values8) has to stay in fp16's range; downwards a row's largest, 7 2^(T + STAGE), is
// 2^17 times the roundings where e is small (from T = -7 on all is exact).  Values: twelve powers of two
// only, so that the weights' smallest step times the window's largest value is small beside its
// smallest.
constexpr int STAGE = 2, KEY_LO = -10, KEY_HI = 6, VAL_LO = -10, VAL_HI = 2;
// Keys' factors are stored times 2^-KEY_DOWN, and the row's is multiplied by it where they are used: a key
// of T = 125 (a stored infinity) times any product of a query row stays in fp32's range.
template <int BITS>
constexpr int KEY_DOWN = BITS == 4 ? 26 : 12;
static_assert(offsetof(Meta<64>, ksig) % 8 == 0 && offsetof(Meta<64>, vsig) % 8 == 0 &&
                  offsetof(Meta<128>, ksig) % 8 == 0 && offsetof(Meta<128>, vsig) % 8 == 0 &&
                  offsetof(Meta<64>, tag) % 16 == 0 && offsetof(Meta<128>, tag) % 16 == 0,
              "pairs, and four tags");

// 32 registers to 32 consecutive columns of the thread's lane, and the wait.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// D[tmem] (+)= A[smem] B[smem]^T and D[tmem] (+)= A[tmem] B[smem], fp16, by the lane that
// has `go`.  The whole warp comes here, so that addresses stay in uniform registers
// (behind a branch on the lane an issue took 120 cycles and more; the product takes 64),
// and of a shared-memory descriptor (ak_sm100.cuh) only the low word changes.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void umma_ss(uint32_t go, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "mov.b64 x, {%2, %6};\n\t"
        "mov.b64 y, {%3, %6};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], x, y, %4, p;\n\t}" ::"r"(go),
        "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI)
        : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t go, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "mov.b64 y, {%3, %6};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], y, %4, p;\n\t}" ::"r"(go),
        "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI)
        : "memory");
}
__device__ __forceinline__ void umma_commit_if(uint32_t go, uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(go),
        "r"(smem_u32(bar))
        : "memory");
}
// Low words of the descriptors of K-major and MN-major tiles.
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return ((saddr & 0x3ffffu) >> 4) | 1u << 16; }
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t lbo) {
    return ((saddr & 0x3ffffu) >> 4) | (lbo >> 4) << 16;
}
// Instruction descriptor: D fp32, A and B fp16, M = 128.
constexpr uint32_t idesc_f16(int n) {
    return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// Bounded wait of a warp of one role; when any role's wait has expired the others give up too.  One
// answer for all lanes: a lane that gave up beside others that did not would leave them in
// their next shuffle.
__device__ __forceinline__ bool wide_wait(uint64_t *bar, uint32_t parity, volatile int *dead,
                                          int *status) {
    bool there = mbar_test_wait(bar, parity);
    for (uint32_t i = 0; !there && i < WAIT_LIMIT; ++i) {
        there = mbar_try_wait(bar, parity);
        if ((i & 255u) == 255u && *dead) break;
    }
    if (__all_sync(0xffffffffu, there)) return true;
    if (!there && !*dead) set_status(status, AKASHIC_ETIMEOUT);
    *dead = 1;
    return false;
}

// A unit's codes and scales as a lane holds them (ak_kv.cuh).
template <int BITS, int D>
struct UnitRegs {
    static constexpr int KC = D * BITS / 256, VC = KC;   // 16-byte loads
    uint4 k[KC], v[VC];
    uint32_t ks[BITS == 4 ? (D == 256 ? 2 : 1) : 1], vs[BITS == 4 ? (D == 256 ? 2 : 1) : 2];
    uint32_t ke, ve;
};
template <int BITS, int D>
__device__ __forceinline__ void load_keys(const unsigned char *un, bool have, UnitRegs<BITS, D> &r) {
    using U = KvUnit<BITS, D>;
    const int lane = threadIdx.x & 31, g = lane >> 2;
    if (!have) return;
#pragma unroll
    for (int i = 0; i < r.KC; ++i) r.k[i] = __ldg((const uint4 *)(un + U::K_CODES + (i * 32 + lane) * 16));
    if constexpr (BITS == 4) {
        if constexpr (D == 64) r.ks[0] = __ldg((const uint16_t *)(un + U::K_SCALES + lane * 2));
        else if constexpr (D == 128) r.ks[0] = __ldg((const uint32_t *)(un + U::K_SCALES + lane * 4));
        else {
            const uint2 x = __ldg((const uint2 *)(un + U::K_SCALES + lane * 8));
            r.ks[0] = x.x, r.ks[1] = x.y;
        }
        r.ke = __ldg((const uint16_t *)(un + U::K_EXP + g * 2));
    } else {
        r.ks[0] = __ldg((const uint32_t *)(un + U::K_SCALES + g * 4));
    }
}
template <int BITS, int D>
__device__ __forceinline__ void load_values(const unsigned char *un, bool have, UnitRegs<BITS, D> &r) {
    using U = KvUnit<BITS, D>;
    const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    if (!have) return;
#pragma unroll
    for (int i = 0; i < r.VC; ++i) r.v[i] = __ldg((const uint4 *)(un + U::V_CODES + (i * 32 + lane) * 16));
    if constexpr (BITS == 4) {
        constexpr int GL = D == 256 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < GL; ++i) {
            const int gr = D == 64 ? g >> 1 : g * GL + i;
            r.vs[i] = __ldg((const uint32_t *)(un + U::V_SCALES + (gr * 4 + c) * 4));
        }
        r.ve = __ldg((const uint32_t *)(un + U::V_EXP + c * 4));
    } else {
        const uint2 x = __ldg((const uint2 *)(un + U::V_SCALES + c * 8));
        r.vs[0] = x.x, r.vs[1] = x.y;
    }
}
// Where dims [d, d + 8) of token t lie in a tile of `rows` tokens (128-byte swizzle).
__device__ __forceinline__ uint4 *tile_chunk(unsigned char *tile, int rows, int t, int d) {
    return (uint4 *)(tile + (d >> 6) * (rows * 128) + t * 128 + ((((d & 63) >> 3) ^ (t & 7)) << 4));
}
// 2^(T + STAGE), T within the window, twice in fp16, from T + 127.
template <int LO, int HI>
__device__ __forceinline__ uint32_t window_h2(uint32_t biased) {
    static_assert(LO + STAGE >= -14 && HI + STAGE <= 15, "normal numbers");
    return (uint32_t)(min(max((int)biased, LO + 127), HI + 127) + STAGE - 112) * 0x04000400u;
}
// The values of a word of 8 nibbles, adjacent pairs: (n - 8) s, s = e 2^(T + STAGE) twice.  A nibble under 2^10 is
// 1024 + n, one of bits 4 to 7 under 2 (64 + n) / 32: (64 + n) / 32 times 32 s less 72 s in one rounding, and
// 72 s has nine bits.  (1032 s has 13: the others take two instructions.)
struct NibbleScale {
    uint32_t s, s32, c;
};
__device__ __forceinline__ void values8(uint32_t w, const NibbleScale &k, uint32_t (&h)[4]) {
    const uint32_t w8 = w >> 8;
    h[0] = h2mul(h2add((w & 0x000f000fu) | 0x64006400u, 0xe408e408u), k.s);               // - 1032
    h[1] = h2fma((w & 0x00f000f0u) | 0x40004000u, k.s32, k.c);
    h[2] = h2mul(h2add((w8 & 0x000f000fu) | 0x64006400u, 0xe408e408u), k.s);
    h[3] = h2fma((w8 & 0x00f000f0u) | 0x40004000u, k.s32, k.c);
}
// Of a scale byte, and of its row's 2^T (window_h2).
__device__ __forceinline__ NibbleScale nibble_scale(uint32_t by, uint32_t pow) {
    NibbleScale k;
    const uint32_t e = by * 0x00400040u + 0x14001400u;         // e 2^5
    k.s32 = h2mul(e, pow);
    k.s = h2mul(k.s32, 0x28002800u);                           // / 32
    k.c = h2mul(k.s32, 0xc080c080u);                           // times -72 / 32
    return k;
}
__device__ __forceinline__ uint4 codes8(uint32_t w0, uint32_t w1) {
    return make_uint4(h2add(__byte_perm(w0, 0x64646464u, 0x4140), H2_M1152),
                      h2add(__byte_perm(w0, 0x64646464u, 0x4342), H2_M1152),
                      h2add(__byte_perm(w1, 0x64646464u, 0x4140), H2_M1152),
                      h2add(__byte_perm(w1, 0x64646464u, 0x4342), H2_M1152));
}
__device__ __forceinline__ uint32_t word_of(const uint4 &x, int i) {
    return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
}

// 32 values of a result row; 16 bytes a store where out is so aligned (rows are).
__device__ __forceinline__ void store_row32(const AttendParams &p, bool bf16, int64_t at, const uint32_t (&y)[32]) {
    uint32_t h[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const float a = __uint_as_float(y[2 * k]), b = __uint_as_float(y[2 * k + 1]);
        if (bf16) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
            h[k] = *(const uint32_t *)&v;
        } else {
            h[k] = pack_h2(a, b);
        }
    }
    uint32_t *dst = (uint32_t *)((uint16_t *)p.out + at);
    if (p.out_wide) {
#pragma unroll
        for (int k = 0; k < 16; k += 4) *(uint4 *)(dst + k) = make_uint4(h[k], h[k + 1], h[k + 2], h[k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) dst[k] = h[k];
    }
}

template <int BITS, int D>
__global__ void __launch_bounds__(Wide<D>::THREADS, 1)
k_attend_wide(const __grid_constant__ AttendParams p, const bool bf16, const int lo, const int hi) {
    using C = Wide<D>;
    using U = KvUnit<BITS, D>;
    constexpr int N = C::N, MT = C::MT, ROWS = C::ROWS, ST = C::STAGES, HT = C::HT, HPT = C::HPT;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *smem = (unsigned char *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
    unsigned char *sq_ = smem, *sk = smem + C::Q_BYTES, *sv = sk + ST * C::KV_BYTES;
    __shared__ Meta<N> meta[ST];
    __shared__ uint64_t kfull[ST], vfull[ST], empty[ST];      // tiles: keys, values, both read
    __shared__ uint64_t sfull[MT][2], pfull[MT][2], odone[MT][2], qfull[MT], drained;
    __shared__ float qscale[ROWS];
    __shared__ uint32_t tmem_slot;
    __shared__ int dead_word;
    volatile int *dead = &dead_word;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    griddep_wait();
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(&kfull[i], 32 * C::DEQ);
            mbar_init(&vfull[i], 32 * C::DEQ);
            mbar_init(&empty[i], 1);
        }
        for (int t = 0; t < MT; ++t) {
            // One a buffer: two halves may be under way, and a wait knows only the
            // last phase from the one before it.
            for (int b = 0; b < 2; ++b) {
                mbar_init(&sfull[t][b], 1);
                mbar_init(&pfull[t][b], 4);
                mbar_init(&odone[t][b], 1);
            }
            mbar_init(&qfull[t], 4);
        }
        mbar_init(&drained, 1);
        mbar_fence_init();
        dead_word = 0;
        p.joins[blockIdx.x] = make_int4(-1, 0, 0, 0);
    }
    if (warp == 0) {
        tmem_alloc(&tmem_slot, C::TMEM_COLS);
        tmem_relinquish();
    }
    int64_t *prefix = (int64_t *)sq_;          // until the warps have found their items
    static_assert(C::Q_BYTES >= (C::THREADS + 1) * 8, "the plan's sums");
    attend_sums(p, ROWS, N, C::EXTRA, lo, hi, prefix);
    const int64_t total = prefix[C::THREADS];
    const int64_t per = max((int64_t)1, (total + gridDim.x - 1) / gridDim.x);
    const int64_t first = per * blockIdx.x;
    int left = (int)max((int64_t)0, min(per, total - first));
    AttendCursor cur = {};
    if (left > 0) cur = attend_find(p, ROWS, N, C::EXTRA, lo, hi, prefix, first);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const bool tags = p.tags != nullptr;

    if (warp >= C::SOFT && warp < C::SOFT + C::DEQ) {
        // ---------------- dequantising
        if constexpr (C::SPLIT) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::regs(1)));
        const int w = warp - C::SOFT, g = lane >> 2, c = lane & 3;
        const bool far = D == 128 && c >= 2, odd = D == 128 && (g & 1);    // (shared memory banks)
        uint32_t n_tile = 0;                   // tiles since the kernel began
        while (left > 0 && !__any_sync(0xffffffffu, *dead)) {
            const AttendPart part = attend_part(cur, left);
            const int n = part.n, units = (cur.q.kv + KV_UNIT - 1) / KV_UNIT;
            if (n <= 0) break;
            // the tile of the item's first step that is this CTA's
            const int first_tile = part.from + (p.ranges ? p.ranges[attend_range_at(p, cur.q, cur.tile, ROWS)].x : 0);
            const int64_t *list = p.blocks + cur.seq * p.max_blocks;
            int64_t my_unit = -1, my_slots = 0;
            auto look_up = [&](int i) {        // lane: this warp's unit of tile i + lane
                my_unit = -1;
                const int tile = i + lane;
                const int u = (first_tile + tile) * C::UNITS + w;
                if (tile < n && u < units) {
                    const int b = u / p.per_block, x = u - b * p.per_block;
                    const int64_t id = list[b];
                    if (id >= 0 && id < p.n_blocks) {
                        my_slots = id * p.per_block + x;
                        my_unit = (id * p.heads + cur.head) * p.per_block + x;
                    } else if (id != -1) {
                        set_status(p.status, AKASHIC_EDEVICE);
                    }
                }
            };
            UnitRegs<BITS, D> r;
            int64_t un = -1;                   // of the tile whose registers are being filled
            int tag_next = 0;
            auto places = [&](int i) {         // of tile i
                if (i % 32 == 0) look_up(i);
                un = __shfl_sync(0xffffffffu, my_unit, i % 32);
                if (tags) {                    // lane: the tag of the unit's token lane
                    const int64_t sl = __shfl_sync(0xffffffffu, my_slots, i % 32);
                    tag_next = un >= 0 && lane < 16 ? p.tags[sl * 16 + lane] : -1;
                }
            };
            places(0);
            load_keys<BITS, D>(p.cache + un * U::BYTES, un >= 0, r);
            load_values<BITS, D>(p.cache + un * U::BYTES, un >= 0, r);
            for (int i = 0; i < n; ++i, ++n_tile) {
                const int st = n_tile % ST, tok = (first_tile + i) * N;
                if (!wide_wait(&empty[st], ((n_tile / ST) & 1) ^ 1, dead, p.status)) break;
                Meta<N> &m = meta[st];
                const bool have = un >= 0;
                const int t0 = w * 16, lt = t0 + lane;     // the unit's first token in the tile, the lane's
                bool mine = have && lane < 16 && tok + lt < cur.q.kv;
                if (tags) {
                    mine = mine && tag_next >= 0;
                    if (lane < 16) m.tag[lt] = max(tag_next, -1);
                }
                const uint32_t ok = __ballot_sync(0xffffffffu, mine);      // the unit's valid tokens
                float kf = 1.f, vf = 1.f;      // the lane's token's factors
                bool bent = BITS == 8;         // one is not 1
                if (c < 2) {
                    uint32_t s = c ? r.ks[0] & 0xffff0000u : r.ks[0] << 16;
                    const bool valid = ok >> (g + 8 * c) & 1u;
                    if constexpr (BITS == 4) {
                        const int T = (int)(r.ke >> (8 * c) & 255u) - 127, rest = T - min(max(T, KEY_LO), KEY_HI);
                        s = (uint32_t)(rest + 127) << 23;
                        bent = valid && rest;
                    }
                    kf = valid ? __uint_as_float(s - ((uint32_t)KEY_DOWN<BITS> << 23)) : 1.f;
                }
                uint32_t vmax = 0;
                if (g < 4) {                   // lane: token 2c + (g & 1) + 8 (g >> 1)
                    const int t = 2 * c + (g & 1) + (g >> 1) * 8;
                    const bool valid = ok >> t & 1u;
                    uint32_t s = 0;
                    if constexpr (BITS == 4) {
                        const int T = (int)(r.ve >> (8 * g) & 255u) - 127, rest = T - min(max(T, VAL_LO), VAL_HI);
                        s = (uint32_t)(rest + 127) << 23;
                        bent = bent || (valid && rest);
                    } else {
                        s = (r.vs[g >> 1] >> (16 * (g & 1))) << 16;
                    }
                    vf = valid ? __uint_as_float(s) : 1.f;
                    if (valid) vmax = s >> 23;
                }
                if (__any_sync(0xffffffffu, bent)) {
                    vmax = __reduce_max_sync(0xffffffffu, vmax);
                    if (c < 2) m.ksig[t0 + g + 8 * c] = kf;
                    if (g < 4) m.vsig[t0 + 2 * c + (g & 1) + (g >> 1) * 8] = vf;
                    if (lane == 0) m.vtop[w] = (unsigned char)vmax, m.bent[w] = 1;
                } else if (lane == 0) {
                    m.vtop[w] = ok ? 127 : 0, m.bent[w] = 0;
                }
                if (w == 0 && lane == 0) m.tok = tok;
                // ---- keys
                unsigned char *kt_ = sk + st * C::KV_BYTES, *vt_ = sv + st * C::KV_BYTES;
                if (!have) {
                    // nothing listed: the products read zeros
                    for (int x = lane; x < 16 * (D / 8); x += 32)
                        *tile_chunk(kt_, N, t0 + x / (D / 8), x % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
                } else if constexpr (BITS == 4) {
                    constexpr int W = D / 32, PERG = D / 64;
                    const uint32_t kp[2] = {window_h2<KEY_LO, KEY_HI>(r.ke & 255u), window_h2<KEY_LO, KEY_HI>(r.ke >> 8 & 255u)};
                    if constexpr (D == 128) {
                        // lanes c and c + 2 meet in the same banks (64 dims apart): the
                        // latter take their two groups the other way round
                        r.ks[0] = __byte_perm(r.ks[0], 0, far ? 0x2301 : 0x3210);
#pragma unroll
                        for (int i2 = 0; i2 < 2; ++i2)
                            if (far) r.k[i2] = make_uint4(r.k[i2].z, r.k[i2].w, r.k[i2].x, r.k[i2].y);
                    }
#pragma unroll
                    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
                        for (int gr = 0; gr < PERG; ++gr) {
                            const int b = i2 * PERG + gr;
                            const uint32_t by = (r.ks[b / 4] >> (8 * (b & 3))) & 255u;
                            const NibbleScale s = nibble_scale(by, kp[i2]);
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const int x = gr * 2 + q;      // word of the token
                                const int at = D == 64 ? i2 * 2 + x : i2 * W + x;
                                uint32_t h[4];
                                values8(word_of(r.k[at / 4], at % 4), s, h);
                                *tile_chunk(kt_, N, t0 + g + 8 * i2, c * (D / 4) + (x ^ (far ? 2 : 0)) * 8) = make_uint4(h[0], h[1], h[2], h[3]);
                            }
                        }
                } else {
                    constexpr int CH = D / 64;
#pragma unroll
                    for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
                        for (int q = 0; q < CH; ++q) {
                            uint4 x = r.k[i2 * CH + q];
                            if (D == 128 && far) x = r.k[i2 * CH + (q ^ 1)];
                            const int d = c * (D / 4) + (q ^ (far ? 1 : 0)) * 16;
                            *tile_chunk(kt_, N, t0 + g + 8 * i2, d) = codes8(x.x, x.y);
                            *tile_chunk(kt_, N, t0 + g + 8 * i2, d + 8) = codes8(x.z, x.w);
                        }
                }
                if (i + 1 < n) {
                    places(i + 1);
                    load_keys<BITS, D>(p.cache + un * U::BYTES, un >= 0, r);
                }
                fence_async_smem();
                mbar_arrive(&kfull[st]);
                // ---- values
                if (!have) {
                    for (int x = lane; x < 16 * (D / 8); x += 32)
                        *tile_chunk(vt_, N, t0 + x / (D / 8), x % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
                } else {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int t = t0 + 2 * c + (x & 1) + (x >> 1) * 8;
                        if constexpr (BITS == 4) {
                            constexpr int W = D / 64, GL = D == 256 ? 2 : 1, WG = W / GL;
                            const uint32_t vp = window_h2<VAL_LO, VAL_HI>(r.ve >> (8 * x) & 255u);
#pragma unroll
                            for (int gl = 0; gl < GL; ++gl) {
                                const uint32_t by = (r.vs[gl] >> (8 * x)) & 255u;
                                const NibbleScale s = nibble_scale(by, vp);
#pragma unroll
                                for (int q = 0; q < WG; ++q) {
                                    const int i3 = gl * WG + q, at = x * W + i3;
                                    uint32_t h[4], word = word_of(r.v[at / 4], at % 4);
                                    if (D == 128 && odd) word = word_of(r.v[at / 4], (at ^ 1) % 4);
                                    values8(word, s, h);
                                    *tile_chunk(vt_, N, t, g * (D / 8) + (i3 ^ (odd ? 1 : 0)) * 8) = make_uint4(h[0], h[1], h[2], h[3]);
                                }
                            }
                        } else {
                            constexpr int W = D / 32;          // words of 4 dims
#pragma unroll
                            for (int q = 0; q < W; q += 2) {
                                const int at = x * W + q;
                                uint32_t w0 = word_of(r.v[at / 4], at % 4), w1 = word_of(r.v[at / 4], at % 4 + 1);
                                if (D == 128 && odd)
                                    w0 = word_of(r.v[at / 4], (at ^ 2) % 4), w1 = word_of(r.v[at / 4], (at ^ 2) % 4 + 1);
                                *tile_chunk(vt_, N, t, g * (D / 8) + (q ^ (odd ? 2 : 0)) * 4) = codes8(w0, w1);
                            }
                        }
                    }
                }
                if (i + 1 < n) load_values<BITS, D>(p.cache + un * U::BYTES, un >= 0, r);
                fence_async_smem();
                mbar_arrive(&vfull[st]);
            }
            left -= part.used;
            if (left > 0) attend_next(p, ROWS, N, C::EXTRA, lo, hi, cur);
        }
    } else if (warp >= C::SOFT + C::DEQ) {
        // ---------------- issuing
        if constexpr (C::SPLIT) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::regs(2)));
        if (warp == C::SOFT + C::DEQ) {
            constexpr uint32_t id_s = idesc_f16(C::SN), id_o = idesc_f16(D) | IDESC_B_MN_MAJOR;
            const uint32_t go = lane == 0;
            const uint32_t q_at = desc_k(smem_u32(sq_)), k_at = desc_k(smem_u32(sk)), v_at = desc_mn(smem_u32(sv), N * 128);
            uint32_t n_tile = 0, q_phase = 0, ph0 = 0, ph1 = 0;    // ph: halves of the row tile, so far
            bool ok = true;
            // S of half h of the item (its first tile: n_tile) for row tile t; at D <= 128
            // (h even) of the whole tile
            auto scores = [&](int t, int h) {
                const uint32_t x = n_tile + h / HPT, b = ((t ? ph1 : ph0) + h) & 1;
                if (!ok) return;
                // the row tiles share a tile's keys
                if (t == 0 && !(ok = wide_wait(&kfull[x % ST], (x / ST) & 1, dead, p.status))) return;
                tc_fence_after();
                const uint32_t qa = q_at + (t * 128 * D * 2 >> 4), ka = k_at + (x % ST) * (C::KV_BYTES >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    umma_ss(go, tmem + C::S_COL + (t * 2 + b) * HT, qa + ((k / 4) * (128 * 128) >> 4) + 2 * (k % 4),
                            ka + ((k / 4) * (N * 128) >> 4) + 2 * (k % 4), id_s, k > 0);
                umma_commit_if(go, &sfull[t][b]);
            };
            auto values = [&](int t, int h) {
                const uint32_t x = n_tile + h / HPT, c = (t ? ph1 : ph0) + h, b = c & 1;
                if (!ok) return;
                if (t == 0 && h % HPT == 0 && !(ok = wide_wait(&vfull[x % ST], (x / ST) & 1, dead, p.status))) return;
                if (!(ok = wide_wait(&pfull[t][b], c >> 1 & 1, dead, p.status))) return;
                tc_fence_after();
                const uint32_t va = v_at + (x % ST) * (C::KV_BYTES >> 4) + h % HPT * (HT * 128 >> 4);
#pragma unroll
                for (int k = 0; k < HT / 16; ++k)
                    umma_ts(go, tmem + t * D, tmem + C::S_COL + (t * 2 + b) * HT + k * 8, va + (2048 * k >> 4), id_o,
                            (h > 0 || k > 0) ? 1u : 0u);
                umma_commit_if(go, &odone[t][b]);
            };
            while (left > 0 && ok) {
                const AttendPart part = attend_part(cur, left);
                const int n = part.n, nh = n * HPT;
                if (n <= 0) break;
                const int mt = cur.q.nq * p.group - cur.tile * ROWS > 128 ? MT : 1;
                if constexpr (MT == 1) {
                    // Two buffers: scores once theirs is free (the weights before were taken
                    // by products issued before: they run in order), O += P V once the weights
                    // are there; whichever is ready.
                    if (ok) ok = wide_wait(&qfull[0], q_phase & 1, dead, p.status);
                    q_phase ^= 1u;
                    int s_next = 0, v_next = 0;
                    uint32_t polls = 0;
                    while (ok && v_next < nh) {
                        bool moved = false;
                        // (one answer for all lanes, as above)
                        if (s_next < nh && s_next - v_next <= 1 &&
                            __all_sync(0xffffffffu, mbar_test_wait(&kfull[(n_tile + s_next) % ST], ((n_tile + s_next) / ST) & 1))) {
                            scores(0, s_next++);
                            moved = true;
                        }
                        const uint32_t c = ph0 + v_next;
                        if (v_next < s_next && __all_sync(0xffffffffu, mbar_test_wait(&pfull[0][c & 1], c >> 1 & 1))) {
                            values(0, v_next);
                            umma_commit_if(go, &empty[(n_tile + v_next++) % ST]);
                            moved = true;
                        }
                        // a bounded wait, like the others (wide_wait)
                        polls = moved ? 0 : polls + 1;
                        if ((polls & 1023u) == 1023u && __any_sync(0xffffffffu, *dead)) ok = false;
                        if (polls >= SPIN_LIMIT) {
                            *dead = 1;
                            set_status(p.status, AKASHIC_ETIMEOUT);
                            ok = false;
                        }
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        if (!ok || t >= mt) break;
                        ok = wide_wait(&qfull[t], q_phase >> t & 1, dead, p.status);
                        q_phase ^= 1u << t;
                        scores(t, 0);
                    }
                    for (int h = 0; ok && h < nh; ++h)
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            if (t >= mt) break;
                            values(t, h);
                            if (h % HPT < HPT - 1) continue;
                            if (ok && t == mt - 1) umma_commit_if(go, &empty[(n_tile + h / HPT) % ST]);
                            if (h + 1 < nh) scores(t, h + 1);
                        }
                }
                ph0 += nh;
                if (mt > 1) ph1 += nh;
                n_tile += n;
                left -= part.used;
                if (left > 0) attend_next(p, ROWS, N, C::EXTRA, lo, hi, cur);
            }
            umma_commit_if(go, &drained);      // what was issued ends before the tensor memory goes
            mbar_wait(&drained, 0, p.status);
        }
        __syncwarp();
    } else {
        // ---------------- softmax: a lane is row 32 (warp % 4) + lane of row tile t
        if constexpr (C::SPLIT) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::regs(0)));
        const int t = warp >> 2, rt = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t o_at = tmem + lanes + t * D;
        const float cap_l = p.cap * LOG2E_F;
        const bool heavy = p.cap > 0.f || p.slopes || p.scale < 0.f;   // a mask of -inf wants a factor > 0
        uint32_t n_tile = 0, halves = 0;       // halves: of this row tile, so far
        bool ok = true;
        int64_t done = 0;
        while (left > 0 && ok) {
            const AttendPart mine = attend_part(cur, left);
            const int n = mine.n;
            if (n <= 0) break;
            const AttendSeq sq = cur.q;
            const int row_first = cur.tile * ROWS, rows = min(ROWS, sq.nq * p.group - row_first);
            const int r = t * 128 + rt;
            if (t == 0 || rows > 128) {
                // ---- the warp's 32 query rows, 16 bytes a lane: bf16 scaled by a power of two
                // to a largest magnitude in [1, 2)
                constexpr int CH = D / 8, RP = 32 / CH;
                constexpr int AT_ONCE = 4;             // (short code: it runs once an item, from a cold cache)
#pragma unroll 1
                for (int y0 = 0; y0 < CH; y0 += AT_ONCE) {
                    uint4 z[AT_ONCE];
#pragma unroll
                    for (int y = 0; y < AT_ONCE; ++y) {
                        const int row = t * 128 + (warp & 3) * 32 + (y0 + y) * RP + lane / CH;
                        const uint32_t at = row_first + min(row, rows - 1), i = at / (uint32_t)p.group;
                        const uint16_t *src = (const uint16_t *)p.q + (int64_t)(sq.row0 + (int)i) * p.q_row +
                                              (int64_t)(cur.head * p.group + (int)(at - i * p.group)) * p.q_head + lane % CH * 8;
                        if (p.q_wide) {
                            z[y] = *(const uint4 *)src;
                        } else {
                            alignas(16) uint16_t x[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) x[k] = src[k];
                            z[y] = *(const uint4 *)x;
                        }
                        if (row >= rows) z[y] = make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int y = 0; y < AT_ONCE; ++y) {
                        const int row = (warp & 3) * 32 + (y0 + y) * RP + lane / CH, ch = lane % CH;
                        float up = 1.f;
                        if (bf16) {
                            uint32_t w[4] = {z[y].x, z[y].y, z[y].z, z[y].w};
                            float a = 0.f;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                a = fmaxf(a, fmaxf(fabsf(__uint_as_float(w[k] << 16)), fabsf(__uint_as_float(w[k] & 0xffff0000u))));
#pragma unroll
                            for (int o = CH / 2; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
                            const int e = max(-126, min(126, (int)(__float_as_uint(a) >> 23) - 127));
                            const float by = pow2i(-e);
                            up = pow2i(e);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                w[k] = pack_h2(__uint_as_float(w[k] << 16) * by, __uint_as_float(w[k] & 0xffff0000u) * by);
                            z[y] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                        *tile_chunk(sq_ + t * 128 * D * 2, 128, row, ch * 8) = z[y];
                        if (ch == 0) qscale[t * 128 + row] = up;
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&qfull[t]);
                const bool real = r < rows;
                const int i = real ? (row_first + r) / p.group : 0;
                const int hd = cur.head * p.group + (real ? row_first + r - i * p.group : 0);
                const float qf = qscale[r] * p.scale * LOG2E_F * (BITS == 4 ? 1.f / (1 << STAGE) : 1.f);
                const int limit = real ? attend_limit(p, sq, i) : sq.kv, pos = sq.kv - sq.nq + i;
                const float slope = real && p.slopes ? p.slopes[hd] * LOG2E_F : 0.f;
                // a slot without a token has tag -1 here, and a row that sees none -2
                const int qt = real && p.q_tags ? p.q_tags[sq.row0 + i] : -2, qtag = qt < 0 ? -2 : qt;
                const int safe = attend_limit(p, sq, (row_first + t * 128) / p.group) - HT;

                float mm = 0.f, l = 0.f;
                bool unset = real;             // no key seen yet: mm = 0
                int rr = 0, tile_tok = 0;      // rr: R
                bool plain = BITS == 4;        // R is 0 for all rows of the warp
                bool big = false, any_big = false;         // the maximum has been beyond 2^20: the row's, one of the warp's
                for (int h = 0; h < n * HPT; ++h, ++halves) {
                    const uint32_t x_tile = n_tile + h / HPT, st = x_tile % ST, b = halves & 1;
                    const uint32_t s_at = tmem + lanes + C::S_COL + (t * 2 + b) * HT;
                    if (h % HPT == 0) {
                        // what the dequantising warps wrote beside the tile, while its scores
                        // are computed
                        // A row tile that had no rows in the items before has not followed the keys' barriers, and
                        // a wait by parity takes a phase two before for its own.  Its scores, of which it
                        // has seen every phase, come after their tile's keys, and nothing goes on to the
                        // phase after that without its weights.
                        if (t > 0 && h == 0) ok = wide_wait(&sfull[t][b], halves >> 1 & 1, dead, p.status);
                        if (ok) ok = wide_wait(&kfull[st], (x_tile / ST) & 1, dead, p.status);
                        tile_tok = meta[st].tok;
                        if (ok) ok = wide_wait(&sfull[t][b], halves >> 1 & 1, dead, p.status);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    const Meta<N> &m = meta[st];
                    const int half = h % HPT * HT, tok = tile_tok + half;
                    const uint32_t vtop = *(const uint32_t *)&m.vtop[half / KV_UNIT];
                    const uint32_t bends = BITS == 4 ? *(const uint32_t *)&m.bent[half / KV_UNIT] : 0x01010101u;
                    const bool flat = bends == 0;
                    if (BITS == 4 && !flat) {
                        // the keys' factors (short loops, here and below: what is rare costs the rest no registers)
#pragma unroll 1
                        for (int k0 = 0; k0 < HT; k0 += 8) {
                            const bool bent = bends >> (k0 / KV_UNIT * 8) & 1u;
                            uint32_t y[8];
                            tmem_ld8(s_at + k0, y);
                            tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                y[k] = __float_as_uint(__uint_as_float(y[k]) * (bent ? m.ksig[half + k0 + k] : pow2i(-KEY_DOWN<BITS>)));
                            tmem_st8(s_at + k0, y);
                        }
                        tmem_st_wait();
                    }
                    // (a byte of vtop is 0)
                    const bool masked = tags || tok > safe || ((vtop - 0x01010101u) & ~vtop & 0x80808080u);
                    uint32_t x[HT];
                    auto pair = [&](int k) { return f2_pack(__uint_as_float(x[k]), __uint_as_float(x[k + 1])); };
                    auto put = [&](int k, uint64_t v) {
                        const float2 y = f2_open(v);
                        x[k] = __float_as_uint(y.x), x[k + 1] = __float_as_uint(y.y);
                    };
                    tmem_ld32(s_at, *(uint32_t(*)[32])x);
                    tmem_ld32(s_at + 32, *(uint32_t(*)[32])(x + 32));
                    float f = flat ? qf : qf * pow2i(KEY_DOWN<BITS>);      // of the scores, log2 units
                    tmem_ld_wait();
                    if constexpr (BITS == 8)
#pragma unroll
                        for (int k = 0; k < HT; k += 2) put(k, f2_mul(pair(k), *(const uint64_t *)&m.ksig[half + k]));
                    if (heavy || masked) {
                        // in place, from here on the factor is 1
#pragma unroll
                        for (int k = 0; k < HT; k += 2) put(k, f2_mul(pair(k), f2_pack(f, f)));
                        f = 1.f;
                        if (p.cap > 0.f) cap_scores<HT>(x, cap_l);
                        if (p.slopes) {
                            const float away = (float)(pos - tok);
#pragma unroll
                            for (int k = 0; k < HT; ++k)
                                x[k] = __float_as_uint(fmaf(-slope, fabsf(away - (float)k), __uint_as_float(x[k])));
                        }
                        if (masked) {
#pragma unroll
                            for (int u = 0; u < HT / 16; ++u) {
                                const int end = vtop >> (8 * u) & 255u ? limit - tok - u * 16 : 0;
#pragma unroll
                                for (int k = 0; k < 16; ++k)
                                    if (k >= end) x[u * 16 + k] = 0xff800000u;
                                if (!tags) continue;
                                // (four at once and without a branch: one after the other, each
                                // behind the last one's branch, took 10 us a step)
#pragma unroll
                                for (int k = 0; k < 16; k += 4) {
                                    const int4 y = *(const int4 *)&m.tag[half + u * 16 + k];
                                    x[u * 16 + k] = y.x == qtag ? x[u * 16 + k] : 0xff800000u;
                                    x[u * 16 + k + 1] = y.y == qtag ? x[u * 16 + k + 1] : 0xff800000u;
                                    x[u * 16 + k + 2] = y.z == qtag ? x[u * 16 + k + 2] : 0xff800000u;
                                    x[u * 16 + k + 3] = y.w == qtag ? x[u * 16 + k + 3] : 0xff800000u;
                                }
                            }
                        }
                    }
                    float top = __uint_as_float(x[0]);
#pragma unroll
                    for (int k = 1; k < HT; ++k) top = fmaxf(top, __uint_as_float(x[k]));
                    top *= f;
                    // the maximum is raised when a weight would pass 2^14
                    const bool rises = unset ? top > -INFINITY : top - mm > P_SHIFT + M_SLACK;
                    bool moves = __any_sync(0xffffffffu, rises);               // O changes its scale
                    // Scores of 2^20 and more are rounded before the maximum is taken from them: of 2^33, x f
                    // unrounded is as much as 2^9 away from the maximum that is its own rounding.
                    if (moves) {
                        big = big || (rises && fabsf(top) > 1048576.f);
                        any_big = __any_sync(0xffffffffu, big);
                    }
                    if (any_big && !heavy && !masked) {
                        const float in = big ? f : 1.f;
                        f = big ? 1.f : f;
#pragma unroll
                        for (int k = 0; k < HT; k += 2) put(k, f2_mul(pair(k), f2_pack(in, in)));
                    }
                    float x_up = 0.f;
                    if (rises) {
                        x_up = unset ? INFINITY : top - P_SHIFT - mm;
                        unset = false;
                        mm = top - P_SHIFT;
                    }
                    const float down = ex2(-x_up);             // of what was summed so far
                    float2 od = make_float2(down, 1.f);        // of O, two factors
                    float n1 = -mm, unit = 1.f;
                    bool loop = false;
                    if (!(flat && plain)) {
                        // R: falls as the maximum rises, so that O keeps its scale, and is raised by what the row
                        // sees.  That there is nothing to look for the half's largest exponent says,
                        // whoever sees it.
                        int rn = rr;
                        if (x_up > 0.f) rn = x_up < INFINITY ? max(R_MIN, rr - (int)fminf(ceilf(x_up), 300.f)) : R_MIN;
                        float wm = top - mm;                   // the largest product, log2
                        if (!flat) {
                            const int t4 = max(max(vtop & 255u, vtop >> 8 & 255u), max(vtop >> 16 & 255u, vtop >> 24));
                            if (__any_sync(0xffffffffu, wm + (float)(t4 - 127) > (float)(rn + R_SLACK))) {
                                wm = -INFINITY;
                                tmem_st32(s_at, *(const uint32_t(*)[32])x);
                                tmem_st32(s_at + 32, *(const uint32_t(*)[32])(x + 32));
                                tmem_st_wait();
#pragma unroll 1
                                for (int k0 = 0; k0 < HT; k0 += 8) {
                                    const bool bent = bends >> (k0 / KV_UNIT * 8) & 1u;
                                    uint32_t y[8];
                                    tmem_ld8(s_at + k0, y);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int k = 0; k < 8; ++k) {              // (rounded as top - mm is)
                                        const int e = bent ? (int)(__float_as_uint(m.vsig[half + k0 + k]) >> 23) - 127 : 0;
                                        wm = fmaxf(wm, __fsub_rn(__fmul_rn(__uint_as_float(y[k]), f), mm) + (float)e);
                                    }
                                }
                            } else {
                                wm = -INFINITY;
                            }
                        }
                        if (wm > (float)(rn + R_SLACK))
                            rn = BITS == 4 && wm >= (float)(R_SHIFT - 1) && wm <= (float)R_SLACK ? 0 : min(R_MAX, (int)ceilf(wm) - R_SHIFT);
                        od = ex2_wide((float)(rr - rn) - (x_up < INFINITY ? x_up : 0.f));
                        moves = __any_sync(0xffffffffu, x_up != 0.f || rr != rn);
                        rr = rn;
                        plain = BITS == 4 && __all_sync(0xffffffffu, rr == 0);
                        // The weights over 2^R: the exponential of the score less both, or, where that could
                        // leave fp32's range (values beyond 2^64 or so, or below 2^-64) or the score swallows R,
                        // R as a factor.  (A row's own R and maximum decide how its weights are
                        // computed; a row that sees nothing has none.)
                        const bool far = !unset && (abs(rr) > 64 || big);
                        const int r_in = far || unset ? 0 : rr;
                        n1 = -mm - (float)r_in, unit = pow2i(r_in);
                        loop = __any_sync(0xffffffffu, far) || BITS == 4;
                        if (loop) {
                            const float rf = far ? pow2i(-rr) : 1.f;
                            float sum[4] = {0.f, 0.f, 0.f, 0.f};
                            tmem_st32(s_at, *(const uint32_t(*)[32])x);
                            tmem_st32(s_at + 32, *(const uint32_t(*)[32])(x + 32));
                            tmem_st_wait();
#pragma unroll 1
                            for (int k0 = 0; k0 < HT; k0 += 8) {
                                const bool bent = bends >> (k0 / KV_UNIT * 8) & 1u;
                                uint32_t y[8], w[4];
                                tmem_ld8(s_at + k0, y);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 8; k += 2) {
                                    const float e0 = ex2(fmaf(__uint_as_float(y[k]), f, n1)), e1 = ex2(fmaf(__uint_as_float(y[k + 1]), f, n1));
                                    sum[k % 4] += e0, sum[k % 4 + 1] += e1;
                                    w[k / 2] = pack_h2(e0 * rf * (bent ? m.vsig[half + k0 + k] : 1.f),
                                                       e1 * rf * (bent ? m.vsig[half + k0 + k + 1] : 1.f));
                                }
                                tmem_st4(s_at + k0 / 2, w);    // (over scores that have been read)
                            }
                            l = l * down + ((sum[0] + sum[2]) + (sum[1] + sum[3])) * unit;
                        }
                    }
                    if (!loop) {
                        uint64_t sum[2] = {0, 0};              // (in the order of the loop above)
                        const uint64_t n2 = f2_pack(n1, n1);
                        uint32_t pk[HT / 2];
#pragma unroll
                        for (int k = 0; k < HT; k += 2) {
                            const float2 u = f2_open(f2_fma(pair(k), f2_pack(f, f), n2));
                            uint64_t e2 = f2_pack(ex2(u.x), ex2(u.y));
                            sum[k / 2 % 2] = f2_add(sum[k / 2 % 2], e2);
                            if constexpr (BITS == 8) e2 = f2_mul(e2, *(const uint64_t *)&m.vsig[half + k]);
                            const float2 y = f2_open(e2);
                            pk[k / 2] = pack_h2(y.x, y.y);
                        }
                        const float2 y = f2_open(f2_add(sum[0], sum[1]));
                        l = l * down + (y.x + y.y) * unit;
                        tmem_st32(s_at, pk);
                    }
                    if (h > 0 && moves) {
                        // once the products before have been added
                        ok = wide_wait(&odone[t][b ^ 1], (halves - 1) >> 1 & 1, dead, p.status);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int d = 0; d < D; d += 32) {
                            uint32_t y[32];
                            tmem_ld32(o_at + d, y);
                            tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 32; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * od.x * od.y);
                            tmem_st32(o_at + d, y);
                        }
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&pfull[t][b]);
                }
                if (ok) ok = wide_wait(&odone[t][(halves - 1) & 1], (halves - 1) >> 1 & 1, dead, p.status);
                if (!ok) break;
                tc_fence_after();
                // ---- whole items are written, others left for the joining kernel
                const bool whole = n == cur.units;
                if (unset) mm = NEG;
                float *part = p.partial + ((int64_t)blockIdx.x * 2 + (mine.from == 0)) * attend_slot_floats(ROWS, D);
                const int up = rr - (BITS == 4 ? STAGE : 0);
                const float inv = l > 0.f ? 1.f / l : l, up0 = pow2i(up / 2), up1 = pow2i(up - up / 2);
                const int64_t dst = (int64_t)(sq.row0 + i) * p.q_heads + hd;
#pragma unroll 1
                for (int d = 0; d < D; d += 32) {
                    uint32_t y[32];
                    tmem_ld32(o_at + d, y);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * inv * up0 * up1);
                    if (!whole) {
                        if (real)
#pragma unroll
                        for (int k = 0; k < 32; k += 4)
                            *(uint4 *)(part + r * D + d + k) = make_uint4(y[k], y[k + 1], y[k + 2], y[k + 3]);
                    } else if (real) {
                        store_row32(p, bf16, dst * D + d, y);
                    }
                }
                if (!whole) {
                    part[ROWS * D + r] = mm, part[ROWS * D + ROWS + r] = l;
                    if (r == 0 && mine.from == 0)
                        p.joins[blockIdx.x] = make_int4(cur.seq, cur.head, cur.tile,
                                                        (int)((first + done - cur.unit + cur.units - 1) / per));
                } else if (real && p.lse) {
                    p.lse[dst] = lse_of(mm, l);
                }
                tc_fence_before();
            }
            n_tile += n;
            left -= mine.used, done += mine.used;
            if (left > 0) attend_next(p, ROWS, N, C::EXTRA, lo, hi, cur);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) tmem_dealloc(tmem, C::TMEM_COLS);
}

// With tags: the steps between the first and the last that hold a tag which some row of a
// tile has (documents packed one after the other: a document's rows look at its own
// part only).  A CTA a sequence: the range of tags of every step, then of every row tile,
// and the steps that overlap it.  Past RANGE_STEPS steps nothing is left out.
constexpr int RANGE_STEPS = 4096;
__global__ void __launch_bounds__(1024)
k_attend_ranges(const __grid_constant__ AttendParams p, int2 *ranges, const int rows, const int step, const int lo,
                const int hi) {
    __shared__ int2 have[RANGE_STEPS];         // the least and the greatest tag of a step
    griddep_wait();
    const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const AttendSeq q = attend_seq(p, s);
    if (!attend_takes(p, q, lo, hi)) return;
    const int steps = (q.kv + step - 1) / step, T = p.per_block * KV_UNIT;
    const bool small = steps <= RANGE_STEPS;
    const int warps = blockDim.x >> 5;
    for (int x = tid >> 5; small && x < steps; x += warps) {
        int2 r = make_int2(0x7fffffff, -1);
        const int j = x * step + 4 * lane;     // the lane's four tokens, of one block
        if (4 * lane < step && j < q.kv) {
            const int b = j / T;
            const int64_t id = p.blocks[s * p.max_blocks + b];
            if (id >= 0 && id < p.n_blocks) {
                const int4 y = *(const int4 *)(p.tags + id * T + (j - b * T));
                const int t[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (t[k] >= 0 && j + k < q.kv) r = make_int2(min(r.x, t[k]), max(r.y, t[k]));
            } else if (id != -1) {
                set_status(p.status, AKASHIC_EDEVICE);   // its step may be left out
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            r = make_int2(min(r.x, __shfl_xor_sync(0xffffffffu, r.x, o)), max(r.y, __shfl_xor_sync(0xffffffffu, r.y, o)));
        if (lane == 0) have[x] = r;
    }
    __syncthreads();
    const int tiles = attend_tiles(p, q, rows);
    for (int t = tid >> 5; t < tiles; t += warps) {            // a warp a row tile
        const uint32_t all = (uint32_t)q.nq * p.group, end = min((uint32_t)(t + 1) * rows, all) - 1u;
        const int i0 = (int)((uint32_t)t * rows / p.group), i1 = (int)(end / p.group);
        const int limit = (attend_limit(p, q, i1) + step - 1) / step;
        int2 want = make_int2(0x7fffffff, -1), r = make_int2(0, limit);
        for (int i = i0 + lane; i <= i1; i += 32) {
            const int y = p.q_tags[q.row0 + i];
            if (y >= 0) want = make_int2(min(want.x, y), max(want.y, y));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            want = make_int2(min(want.x, __shfl_xor_sync(0xffffffffu, want.x, o)),
                             max(want.y, __shfl_xor_sync(0xffffffffu, want.y, o)));
        if (small) {
            // 32 steps at a time from either side
            auto seen = [&](int x) {
                return __ballot_sync(0xffffffffu, x >= 0 && x < limit && have[x].x <= want.y && have[x].y >= want.x);
            };
            unsigned any = 0;
            for (; r.x < limit && !(any = seen(r.x + lane)); r.x += 32) {}
            r.x = any ? r.x + __ffs(any) - 1 : limit;
            any = 0;
            for (; r.y > r.x && !(any = seen(r.y - 1 - lane)); r.y -= 32) {}
            r.y = any ? r.y - __ffs(any) + 1 : r.x;
        }
        if (lane == 0)
            ranges[attend_range_at(p, q, t, rows)] = r;
    }
}

template <int BITS, int D>
cudaError_t run_wide(const AttendParams &p, int dtype, int ctas, int lo, int hi, cudaStream_t st) {
    using C = Wide<D>;
    auto *kernel = k_attend_wide<BITS, D>;
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
    return launch_pdl(kernel, dim3(ctas), dim3(C::THREADS), C::SMEM, st, p, dtype == AKASHIC_DTYPE_BF16, lo, hi);
}

}  // namespace

AttendShape attend_wide_shape(int dim, int sms) {
    return {dim == 256 ? Wide<256>::ROWS : Wide<128>::ROWS, sms};
}
cudaError_t launch_attend_ranges(const AttendParams &p, int dim, const AttendShape &shape, int lo, int hi,
                                 cudaStream_t st) {
    const int step = dim == 256 ? Wide<256>::N : Wide<128>::N;
    // a warp a step or row tile, as far as a CTA goes
    const int64_t most = max((int64_t)p.max_kv / step, (int64_t)p.n_q * p.group / p.n_seq / shape.rows);
    const int warps = (int)min((int64_t)32, max((int64_t)4, most));
    return launch_pdl(k_attend_ranges, dim3(p.n_seq), dim3(32 * warps), 0, st, p, (int2 *)p.ranges, shape.rows, step,
                      lo, hi);
}
cudaError_t launch_attend_wide(const AttendParams &p, int bits, int dim, int dtype,
                               const AttendShape &s, int lo, int hi, cudaStream_t st) {
    if (bits == 4)
        return dim == 64 ? run_wide<4, 64>(p, dtype, s.ctas, lo, hi, st)
               : dim == 128 ? run_wide<4, 128>(p, dtype, s.ctas, lo, hi, st)
                            : run_wide<4, 256>(p, dtype, s.ctas, lo, hi, st);
    return dim == 64 ? run_wide<8, 64>(p, dtype, s.ctas, lo, hi, st)
           : dim == 128 ? run_wide<8, 128>(p, dtype, s.ctas, lo, hi, st)
                        : run_wide<8, 256>(p, dtype, s.ctas, lo, hi, st);
}

}  // namespace ak
