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
    float *partial;                   // unfinished items' results (PartialSlot)
    int4 *joins;                      // what the joining kernel has to join
    int64_t n_blocks, max_blocks;
    int n_q, n_seq, q_heads, heads, group;
    int per_block;                    // units of a block
    int max_kv;                       // tokens that the lists can hold
    int causal;
    float scale, cap;                 // cap 0: none
};

// A sequence: its query rows and context.
struct AttendSeq {
    int row0, nq, kv, prefix;
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
__device__ __forceinline__ int attend_tiles(const AttendParams &p, const AttendSeq &q, int rows) {
    return (int)(((int64_t)q.nq * p.group + rows - 1) / rows);
}
__device__ __forceinline__ int attend_units(const AttendParams &p, const AttendSeq &q, int tile,
                                            int rows, int step) {
    const int64_t last = min((int64_t)(tile + 1) * rows, (int64_t)q.nq * p.group) - 1;
    const int end = attend_limit(p, q, (int)(last / p.group));
    return max(1, (end + step - 1) / step);
}
// Whether a kernel that takes sequences of [lo, hi] rows takes this one.
__device__ __forceinline__ int64_t attend_seq_units(const AttendParams &p, const AttendSeq &q,
                                                    int rows, int step, int lo, int hi) {
    const int64_t n = (int64_t)q.nq * p.group;
    if (n < lo || n > hi) return 0;
    const int tiles = attend_tiles(p, q, rows);
    int64_t u = 0;
    for (int t = 0; t < tiles; ++t) u += attend_units(p, q, t, rows, step);
    return u;
}

// Where a CTA stands in the order of all items.
struct AttendCursor {
    int seq, head, tile, unit;        // unit: first step of the item that is this CTA's
    int units;                        // of the item
    AttendSeq q;
};

// Every CTA takes an equal share [first, first + count) of the steps of all
// items, so that a batch of very different lengths fills the GPU evenly; it
// finds the share's first item by a scan over the sequences.  `per` is a
// CTA's share (a multiple of nothing in particular, at least min_per).
// All threads of the CTA call this; scratch: 34 int64 in shared memory.
__device__ __forceinline__ bool attend_plan(const AttendParams &p, int rows, int step, int lo,
                                            int hi, int min_per, int64_t *scratch, int64_t &first,
                                            int64_t &count, int64_t &per, AttendCursor &cur) {
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int warps = nt >> 5;
    int64_t sum = 0, mine = 0;
    for (int s = tid; s < p.n_seq; s += nt) {
        mine = attend_seq_units(p, attend_seq(p, s), rows, step, lo, hi) * p.heads;
        sum += mine;
    }
    int64_t x = sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) scratch[warp] = x;
    __syncthreads();
    int64_t total = 0;
    for (int w = 0; w < warps; ++w) total += scratch[w];
    per = (total + gridDim.x - 1) / gridDim.x;
    if (per < min_per) per = min_per;
    first = per * blockIdx.x;
    count = min(per, total - first);
    if (count <= 0) return false;
    // the sequence in whose range `first` lies
    int64_t base = 0;
    for (int s0 = 0; s0 < p.n_seq; s0 += nt) {
        const int s = s0 + tid;
        // with one round of the loop the first pass left this thread's sum
        int64_t w = p.n_seq <= nt ? mine
                    : s < p.n_seq ? attend_seq_units(p, attend_seq(p, s), rows, step, lo, hi) * p.heads
                                  : 0;
        if (s >= p.n_seq) w = 0;
        int64_t incl = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        __syncthreads();
        if (lane == 31) scratch[warp] = incl;
        __syncthreads();
        int64_t before = base, all = 0;
        for (int i = 0; i < warps; ++i) {
            if (i < warp) before += scratch[i];
            all += scratch[i];
        }
        const int64_t hi_ = before + incl, lo_ = hi_ - w;
        if (w > 0 && first >= lo_ && first < hi_) {
            scratch[32] = s;
            scratch[33] = first - lo_;
        }
        __syncthreads();
        if (first < base + all) break;
        base += all;
    }
    cur.seq = (int)scratch[32];
    int64_t rest = scratch[33];
    __syncthreads();
    cur.q = attend_seq(p, cur.seq);
    const int64_t one = attend_seq_units(p, cur.q, rows, step, lo, hi);
    cur.head = (int)(rest / one);
    rest -= cur.head * one;
    cur.tile = 0;
    cur.units = attend_units(p, cur.q, 0, rows, step);
    while (rest >= cur.units) {
        rest -= cur.units;
        cur.units = attend_units(p, cur.q, ++cur.tile, rows, step);
    }
    cur.unit = (int)rest;
    return true;
}
// The next item (the caller knows that there is one).
__device__ __forceinline__ void attend_next(const AttendParams &p, int rows, int step, int lo,
                                            int hi, AttendCursor &c) {
    c.unit = 0;
    if (++c.tile >= attend_tiles(p, c.q, rows)) {
        c.tile = 0;
        if (++c.head >= p.heads) {
            c.head = 0;
            do {
                c.q = attend_seq(p, ++c.seq);
            } while (c.seq + 1 < p.n_seq && ((int64_t)c.q.nq * p.group < lo ||
                                             (int64_t)c.q.nq * p.group > hi));
        }
    }
    c.units = attend_units(p, c.q, c.tile, rows, step);
}

// An item whose steps lie in several CTAs' shares: each leaves its rows'
// unnormalised sums, maxima and totals in a slot of the workspace (two a CTA: its
// first item, which may have begun before its share, and its last), the CTA
// in which the item begins notes it, and the joining kernel adds the slots up in
// the order of the CTAs.
//   slot: float acc[rows][D], m[rows] (log2 units), l[rows]
__host__ __device__ __forceinline__ int64_t attend_slot_floats(int rows, int dim) {
    return (int64_t)rows * (dim + 2);
}

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

}  // namespace ak
