// Attention over the quantised cache: what its kernels share.
#pragma once

#include "ak_kv.cuh"

namespace ak {

constexpr int KV_MAX_HEADS = 1024;

akashic_status_t kv_fail(akashic_status_t code, const char *fmt, ...);
akashic_status_t kv_check_config(const akashic_mem_kv_config_t *c, const char *who);

// Makes a device current for a call and puts the caller's back.
struct KvDevice {
    int prev = -1;
    bool ok = false, changed = false;
    explicit KvDevice(int dev);
    ~KvDevice();
};

// One call's arguments on the device.
struct AttendParams {
    const unsigned char *cache;
    const void *q;
    int64_t q_row, q_head;            // strides in elements
    void *out;                        // [n_q][q_heads][D]
    float *lse;                       // [n_q][q_heads] or NULL
    const int32_t *q_start;           // [n_seq + 1] or NULL: n_q / n_seq rows each
    const int32_t *kv_len;            // [n_seq] or NULL: all listed tokens
    const int32_t *prefix;            // [n_seq] or NULL
    const int64_t *blocks;            // [n_seq][max_blocks]
    const float *slopes;              // [q_heads] or NULL
    const int32_t *tags;              // one a slot, or NULL
    const int32_t *q_tags;            // [n_q] or NULL
    int *status;
    const int2 *ranges;               // many-row kernel with tags: each row tile's first and last
                                      // step (attend_range_at), or NULL
    float *partial;                   // unfinished items' results (PartialSlot)
    int4 *joins;                      // what the joining kernel has to join
    int64_t n_blocks, max_blocks;
    int n_q, n_seq, q_heads, heads, group;
    int per_block;                    // units of a block
    int max_kv;                       // tokens that the lists can hold
    int causal;
    int direct;                       // few-row kernel: CTA b has item b, sequences of one tile
    bool q_wide, out_wide;            // query rows, out: 16-byte aligned
    float scale, cap;                 // cap 0: none
};

// A sequence: its query rows and context.
struct AttendSeq {
    int row0, nq, kv, prefix, seq;
};
__device__ __forceinline__ AttendSeq attend_seq(const AttendParams &p, int s) {
    AttendSeq q;
    if (p.q_start) {
        const int a = p.q_start[s], b = p.q_start[s + 1];
        q.row0 = max(0, min(a, p.n_q));
        q.nq = max(0, min(b, p.n_q) - q.row0);
        if (a < 0 || b < a || b > p.n_q) set_status(p.status, AKASHIC_EDEVICE);
    } else {
        q.nq = p.n_q / p.n_seq;
        q.row0 = s * q.nq;
    }
    q.kv = p.max_kv;
    if (p.kv_len) {
        const int n = p.kv_len[s];
        if (n < 0 || n > p.max_kv) set_status(p.status, AKASHIC_EDEVICE);
        q.kv = max(0, min(n, p.max_kv));
    }
    q.prefix = p.prefix ? max(0, min(p.prefix[s], q.kv)) : 0;
    q.seq = s;
    return q;
}
// Keys [0, limit) may be seen by the row at place i of the sequence.
__device__ __forceinline__ int attend_limit(const AttendParams &p, const AttendSeq &q, int i) {
    return p.causal ? max(q.prefix, max(0, q.kv - q.nq + i + 1)) : q.kv;
}

// The work of a call: items (sequence, kv head, tile of `rows` query rows) in
// that order, each of attend_units() steps of `step` tokens, at least one (an
// item without keys still writes its rows).  A row of a tile is a query row of
// the sequence and one of the group's heads: r = i * group + head.
// (rows of a sequence, query rows times group, stay below 2^31)
__device__ __forceinline__ int attend_tiles(const AttendParams &p, const AttendSeq &q, int rows) {
    return (int)(((uint32_t)q.nq * (uint32_t)p.group + (uint32_t)rows - 1u) / (uint32_t)rows);
}
// Where a row tile's range stands: the sequences' tiles one after the other.
__host__ __device__ __forceinline__ int64_t attend_ranges(int64_t n_q, int group, int n_seq, int rows) {
    return n_q * group / rows + n_seq + 1;
}
__device__ __forceinline__ int attend_range_at(const AttendParams &p, const AttendSeq &q, int tile, int rows) {
    return (int)((uint32_t)q.row0 * (uint32_t)p.group / (uint32_t)rows) + q.seq + tile;
}
__device__ __forceinline__ int attend_units(const AttendParams &p, const AttendSeq &q, int tile,
                                            int rows, int step) {
    if (p.ranges) {
        const int2 r = p.ranges[attend_range_at(p, q, tile, rows)];
        return max(1, r.y - r.x);
    }
    const uint32_t all = (uint32_t)q.nq * (uint32_t)p.group;
    const uint32_t last = min((uint32_t)(tile + 1) * (uint32_t)rows, all) - 1u;
    const int end = attend_limit(p, q, (int)(last / (uint32_t)p.group));
    return max(1, (int)(((uint32_t)end + (uint32_t)step - 1u) / (uint32_t)step));
}
// Whether a kernel that takes sequences of [lo, hi] rows takes this one.
__device__ __forceinline__ bool attend_takes(const AttendParams &p, const AttendSeq &q, int lo, int hi) {
    const int n = q.nq * p.group;
    return n >= lo && n <= hi;
}
// The steps of one head of a sequence, and `extra` more an item: every lane's own (s, 0
// where it has none).
// A whole warp calls it: sequences of many tiles are summed up by all lanes.
__device__ __forceinline__ int64_t attend_seq_units(const AttendParams &p, const AttendSeq &q, bool have,
                                                    int rows, int step, int extra, int lo, int hi) {
    constexpr int FEW = 4;
    const int lane = threadIdx.x & 31;
    const int tiles = have && attend_takes(p, q, lo, hi) ? attend_tiles(p, q, rows) : 0;
    int64_t u = 0;
    if (tiles <= FEW)
        for (int t = 0; t < tiles; ++t) u += extra + attend_units(p, q, t, rows, step);
    for (unsigned many = __ballot_sync(0xffffffffu, tiles > FEW); many; many &= many - 1) {
        const int l = __ffs(many) - 1;
        const AttendSeq x = {__shfl_sync(0xffffffffu, q.row0, l), __shfl_sync(0xffffffffu, q.nq, l),
                             __shfl_sync(0xffffffffu, q.kv, l), __shfl_sync(0xffffffffu, q.prefix, l),
                             __shfl_sync(0xffffffffu, q.seq, l)};
        const int n = __shfl_sync(0xffffffffu, tiles, l);
        int64_t v = 0;
        for (int t = lane; t < n; t += 32) v += extra + attend_units(p, x, t, rows, step);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == l) u = v;
    }
    return u;
}

// Where a worker (a warp, or a CTA of the kernel for many rows) stands in the
// order of all items.
struct AttendCursor {
    int seq, head, tile, unit;        // unit: first step of the item that is the worker's, less
                                      // than 0 within the extra steps
    int units;                        // of the item
    AttendSeq q;
};

// Every worker takes an equal share of the steps of all items, so that a batch
// of very different lengths fills the GPU evenly.  An item's beginning and end count
// as `extra` steps, before its others.  All threads of the CTA sum
// up the sequences' steps (each a run of consecutive sequences); prefix[t], in
// shared memory, is the sum of the runs before thread t's, prefix[blockDim.x] all.
__device__ __forceinline__ void attend_sums(const AttendParams &p, int rows, int step, int extra,
                                            int lo, int hi, int64_t *prefix) {
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (p.n_seq + nt - 1) / nt;
    int64_t sum = 0;
    for (int i = 0; i < run; ++i) {
        const int s = tid * run + i;
        const bool have = s < p.n_seq;
        sum += attend_seq_units(p, attend_seq(p, have ? s : 0), have, rows, step, extra, lo, hi) * p.heads;
    }
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
    __syncthreads();
}
// The item in which step `first` (below the total) lies.  A whole warp calls it.
__device__ __forceinline__ AttendCursor attend_find(const AttendParams &p, int rows, int step, int extra,
                                                    int lo, int hi, const int64_t *prefix,
                                                    int64_t first) {
    const int nt = blockDim.x, lane = threadIdx.x & 31;
    const int run = (p.n_seq + nt - 1) / nt;
    AttendCursor c = {};
    int t = 0;                        // the last thread whose run begins at or before `first`
    for (int t0 = 0; t0 < nt; t0 += 32) {
        const unsigned before = __ballot_sync(0xffffffffu, prefix[t0 + lane] <= first);
        t = t0 + 31 - __clz(before);
        if (before != 0xffffffffu || first < prefix[t0 + 32]) break;
    }
    int64_t rest = first - prefix[t], one = 0;   // within that run
    for (int s0 = t * run;; s0 += 32) {
        const int s = s0 + lane;
        const bool have = s < p.n_seq;
        const int64_t w = attend_seq_units(p, attend_seq(p, have ? s : 0), have, rows, step, extra, lo, hi) * p.heads;
        int64_t incl = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        const unsigned in = __ballot_sync(0xffffffffu, rest < incl);
        if (in) {
            const int l = __ffs(in) - 1;
            c.seq = s0 + l;
            rest -= __shfl_sync(0xffffffffu, incl - w, l);
            one = __shfl_sync(0xffffffffu, w, l) / p.heads;
            break;
        }
        rest -= __shfl_sync(0xffffffffu, incl, 31);
        if (s0 >= p.n_seq) return c;  // not reached: first is below the total
    }
    c.q = attend_seq(p, c.seq);
    c.head = (int)(rest / one);
    rest -= c.head * one;
    // the tile, 32 at a time
    for (const int tiles = attend_tiles(p, c.q, rows); c.tile < tiles; c.tile += 32) {
        const int t = c.tile + lane;
        const int w = t < tiles ? extra + attend_units(p, c.q, t, rows, step) : 0;
        int64_t incl = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        const unsigned in = __ballot_sync(0xffffffffu, rest < incl);
        if (in) {
            const int l = __ffs(in) - 1;
            c.tile += l;
            c.units = __shfl_sync(0xffffffffu, w, l);
            rest -= __shfl_sync(0xffffffffu, incl, l) - c.units;
            c.units -= extra;
            break;
        }
        rest -= __shfl_sync(0xffffffffu, incl, 31);
    }
    c.unit = (int)rest - extra;
    return c;
}
// The next item (the caller knows that there is one).
__device__ __forceinline__ void attend_next(const AttendParams &p, int rows, int step, int extra,
                                            int lo, int hi, AttendCursor &c) {
    c.unit = -extra;
    if (++c.tile >= attend_tiles(p, c.q, rows)) {
        c.tile = 0;
        if (++c.head >= p.heads) {
            c.head = 0;
            do {
                c.q = attend_seq(p, ++c.seq);
            } while (c.seq + 1 < p.n_seq && !attend_takes(p, c.q, lo, hi));
        }
    }
    c.units = attend_units(p, c.q, c.tile, rows, step);
}

// What a share of `left` steps, extra ones counted, has of the cursor's item: n steps from
// `from`; n <= 0 where it ends within the extra ones.
struct AttendPart {
    int from, n, used;
};
__device__ __forceinline__ AttendPart attend_part(const AttendCursor &c, int left) {
    const int used = min(c.units - c.unit, left), from = max(c.unit, 0);
    return {from, used - (from - c.unit), used};
}

// An item whose steps lie in several CTAs' shares: each leaves its rows'
// results over its part, maxima and totals in a slot of the workspace (two a CTA: slot 0 for
// the item that began before its share, slot 1 for one that begins in it), the CTA in
// which the item begins notes it in joins, and the joining kernel adds the slots
// up in the order of the CTAs.
//   slot: float out[rows][D], m[rows] (log2 units), l[rows]
// (Results, not the weighted sums: of values near the largest fp32 those are infinite.)
__host__ __device__ __forceinline__ int64_t attend_slot_floats(int rows, int dim) {
    return (int64_t)rows * (dim + 2);
}

// ------------------------------------------------------------------ arithmetic
constexpr float NEG = -3.402823466e38f;       // "no score yet": below all scores, finite: no NaN from differences
constexpr float P_SHIFT = 6.f, M_SLACK = 8.f; // log2 units
// A row's weights, times their values' powers of two 2^T (8 bits: scales in [2^T, 2^(T+1))), are divided
// by 2^R before they become fp16.  R goes by the greatest of these products that the row has seen, not by
// tokens that it does not see or that weigh nothing: raised when one would pass 2^(R + R_SLACK),
// so that it comes to 2^(R_SHIFT - 1) to 2^(R_SHIFT + 1): fp16 then has room for the 2^8 by which weights may
// still grow, and values of eight times the size, and 2^-27 of the greatest as its smallest step.
// (With 6 and 13 for these two the many-row kernel looked for the greatest often: two capped prompts of 2048
// rows, all factors in use, 1300 us for 1159.)
// Within R_MIN and R_MAX 2^-R is a normal number.
constexpr int R_MIN = -126, R_MAX = 126, R_SLACK = 14, R_SHIFT = 3;

__device__ __forceinline__ uint32_t h2fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t h2mul(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t h2add(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 ex2_wide(float x) {   // 2^x as two factors, x from -252
    const float a = fmaxf(x, -126.f);
    return make_float2(ex2(a), ex2(fmaxf(x - a, -126.f)));
}
__device__ __forceinline__ float scale2(float x, int e) {   // x 2^e, |e| <= 252
    return x * pow2i(e / 2) * pow2i(e - e / 2);
}

__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 f2_open(uint64_t a) {
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(a));
    return d;
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// cap tanh(x / cap) of a lane's scores, in place (log2 units, like cap).  Where all of the
// warp's are within 0.7 cap: x q(t), t = (x / cap)^2 <= 1/2, q the polynomial of degree 5
// nearest to tanh(sqrt t) / sqrt t there in relative error (3.6e-8 with its coefficients in fp32; fitted
// by iteratively reweighted least squares), two scores an instruction.  Else
// 1 - 2 / (1 + e^(2y)), which alone would lose small scores under a large cap.
template <int N>
__device__ __forceinline__ void cap_scores(uint32_t (&x)[N], float cap) {
    const float c = 1.f / cap, c2 = 2.f * LOG2E_F * c;
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) most = fmaxf(most, fabsf(__uint_as_float(x[k])));
    if (__all_sync(0xffffffffu, most <= 0.7f * cap)) {
        const float q[6] = {1.f, -0.3333311080932617f, 0.13328056037425995f, -0.053502924740314484f,
                            0.019964739680290222f, -0.005034883972257376f};
        const uint64_t cc = f2_pack(c, c);
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            const uint64_t z = f2_pack(__uint_as_float(x[k]), __uint_as_float(x[k + 1]));
            const uint64_t y = f2_mul(z, cc), t = f2_mul(y, y);
            uint64_t v = f2_pack(q[5], q[5]);
#pragma unroll
            for (int i = 4; i >= 0; --i) v = f2_fma(v, t, f2_pack(q[i], q[i]));
            const float2 r = f2_open(f2_mul(v, z));
            x[k] = __float_as_uint(r.x), x[k + 1] = __float_as_uint(r.y);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            x[k] = __float_as_uint(cap * (1.f - __fdividef(2.f, 1.f + ex2(__uint_as_float(x[k]) * c2))));
    }
}

// Four adjacent-dim (or, after pairing, adjacent-token) pairs of a word of 8
// nibbles: pair i in h[i].  s: e 2^15 in both halves, s4: s 2^-4, c: -s 2^-21.
__device__ __forceinline__ void nibbles(uint32_t w, uint32_t s, uint32_t s4, uint32_t c,
                                        uint32_t (&h)[4]) {
    const uint32_t w8 = w >> 8;
    h[0] = h2fma(w & 0x000f000fu, s, c);
    h[1] = h2fma(w & 0x00f000f0u, s4, c);
    h[2] = h2fma(w8 & 0x000f000fu, s, c);
    h[3] = h2fma(w8 & 0x00f000f0u, s4, c);
}
constexpr uint32_t H2_M2_21 = 0x80088008u;   // -2^-21, twice
constexpr uint32_t H2_M1152 = 0xe480e480u;   // -1152, twice
// Two adjacent values of a result row, and its log-sum-exp.
__device__ __forceinline__ void store_pair(const AttendParams &p, bool bf16, int64_t at, float a, float b) {
    if (bf16)
        *(__nv_bfloat162 *)((__nv_bfloat16 *)p.out + at) = __floats2bfloat162_rn(a, b);
    else
        *(uint32_t *)((__half *)p.out + at) = pack_h2(a, b);
}
__device__ __forceinline__ float lse_of(float m, float total) {
    return total == 0.f ? -INFINITY : (m + log2f(total)) * 0.69314718055994530942f;
}

// ------------------------------------------------------------------ launches
// Joins what the `ctas` CTAs of a kernel with tiles of `rows` rows left.
cudaError_t launch_attend_join(const AttendParams &p, int dtype, int dim, int ctas, int rows,
                               cudaStream_t st);

// The kernels.  lo, hi: the numbers of rows (query rows times group) of the
// sequences that they take.
struct AttendShape {
    int rows, ctas;                   // rows of a tile, CTAs
};
AttendShape attend_narrow_shape(int bits, int dim, int max_rows, int sms);
cudaError_t launch_attend_narrow(const AttendParams &p, int bits, int dim, int dtype,
                                 const AttendShape &shape, int lo, int hi, cudaStream_t st);
AttendShape attend_wide_shape(int dim, int sms);
// Fills p.ranges (attend_ranges() entries) for the sequences that the kernel will take.
cudaError_t launch_attend_ranges(const AttendParams &p, int dim, const AttendShape &shape, int lo, int hi,
                                 cudaStream_t st);
cudaError_t launch_attend_wide(const AttendParams &p, int bits, int dim, int dtype,
                               const AttendShape &shape, int lo, int hi, cudaStream_t st);

}  // namespace ak
