// Attention over the latent cache: what its kernels share.
#pragma once

#include "ak_attend.cuh"
#include "ak_sm100.cuh"

namespace ak {

template <typename S>
constexpr bool is_bf16 = false;
template <>
constexpr bool is_bf16<__nv_bfloat16> = true;

// One call's arguments.  Absorbed: one key head, all query heads its group; expanded: a key head a
// query head.
struct LatentParams {
    AttendParams a;
    int R, P;                         // latent and rotated values of a row
    bool bf16;                        // else fp16
    bool q_map;                       // query rows come by a tensor map
    // expanded
    int nope, value;
    const void *w_k, *w_v;
    int64_t k_head, k_row, v_head, v_row;
};

// The power of two of a bf16 weight whose score set its row's reference: below 2^(-1 - M_SLACK) / kv, so that kv
// weights of 2^M_SLACK times that, the most one may have, add up to less than 1 (2^-16 for up to 127 tokens, 2^-23
// for 8192; fp32 holds 2^-86 of it at the longest context).  For scores within 2^24, beyond which fp32 tells a reference
// from one so much higher no longer.
__device__ __forceinline__ float latent_off_bf16(int kv) { return (float)(__clz(kv) - 33) - M_SLACK; }
// A result in the type's range.  It is a mean of finite values, which its weights' rounding can put half a step beyond
// the type's largest, and its own rounding then to infinity.  A NaN stays one.
__device__ __forceinline__ float latent_result(float x, bool bf16) {
    float y;
    asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(bf16 ? 3.38953139e38f : 65504.f));
    return y;
}
__device__ __forceinline__ uint16_t round16(float x, bool bf16) {
    x = latent_result(x, bf16);
    return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
}
// Eight values of a query row.
__device__ __forceinline__ uint4 load_row8(const uint16_t *src, bool wide) {
    if (wide) return *(const uint4 *)src;
    alignas(16) uint16_t h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = src[k];
    return *(const uint4 *)h;
}

// attend_seq with its loads side by side.
__device__ __forceinline__ AttendSeq latent_seq(const AttendParams &p, int s) {
    int a = 0, b = 0, n = p.max_kv, prefix = 0;
    if (p.q_start) a = __ldg(p.q_start + s), b = __ldg(p.q_start + s + 1);
    if (p.kv_len) n = __ldg(p.kv_len + s);
    if (p.prefix) prefix = __ldg(p.prefix + s);
    AttendSeq q;
    if (p.q_start) {
        q.row0 = max(0, min(a, p.n_q));
        q.nq = max(0, min(b, p.n_q) - q.row0);
    } else {
        q.nq = p.n_q / p.n_seq;
        q.row0 = s * q.nq;
    }
    q.kv = max(0, min(n, p.max_kv));
    q.prefix = max(0, min(prefix, q.kv));
    q.seq = s;
    if (a < 0 || b < a || b > p.n_q || n < 0 || n > p.max_kv) set_status(p.status, AKASHIC_EDEVICE);
    return q;
}

// attend_sums and attend_find in one where every thread has a sequence at most: the thread whose sequence
// has the CTA's first step knows where (3500 cycles less at a kernel's beginning).  All threads call it;
// prefix: blockDim.x + 1 words of shared memory.  first, left: the CTA's share.
struct LatentShare {
    AttendCursor cur;
    int64_t first, per;
    int left;
};
// ctas: that have one together.
__device__ __forceinline__ LatentShare latent_share(const AttendParams &p, int rows, int step, int extra,
                                                    int64_t *prefix, int ctas = 1) {
    constexpr int ALL = 0x7fffffff;
    __shared__ AttendCursor found;
    __shared__ int have_found;
    const int nt = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    LatentShare r;
    if (p.direct) {                            // a CTA an item: p.direct tiles a sequence
        const int s = blockIdx.x / p.direct;
        r.cur = {};
        r.cur.seq = s, r.cur.tile = blockIdx.x - s * p.direct, r.cur.q = latent_seq(p, s);
        r.cur.units = attend_units(p, r.cur.q, r.cur.tile, rows, step), r.cur.unit = -extra;
        r.first = 0, r.left = r.cur.units + extra, r.per = r.left;
        return r;
    }
    AttendSeq q = {};
    int64_t sum = 0, before = 0;
    const bool one = p.n_seq <= nt;
    if (tid == 0) have_found = 0;
    if (one) {
        const bool have = tid < p.n_seq;
        q = latent_seq(p, have ? tid : 0);
        sum = attend_seq_units(p, q, have, rows, step, extra, 1, ALL) * p.heads;
        int64_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) prefix[warp] = incl;
        __syncthreads();
        for (int w = 0; w < warp; ++w) before += prefix[w];
        __syncthreads();
        before += incl - sum;
        prefix[tid] = before;
        if (tid == nt - 1) prefix[nt] = before + sum;
        __syncthreads();
    } else {
        attend_sums(p, rows, step, extra, 1, ALL, prefix);
    }
    const int64_t total = prefix[nt], g = gridDim.x / ctas;
    r.per = total + g < 0x7fffffff ? max(1u, ((uint32_t)total + (uint32_t)g - 1u) / (uint32_t)g) : (total + g - 1) / g;
    r.first = r.per * (blockIdx.x / ctas);
    r.left = (int)max((int64_t)0, min(r.per, total - r.first));
    r.cur = {};
    if (r.left <= 0) return r;                 // (the whole CTA)
    if (one) {
        int64_t rest = r.first - before;
        if (rest >= 0 && rest < sum && attend_tiles(p, q, rows) <= 8 && sum < 0x7fffffff) {
            const int of_head = (int)sum / p.heads;
            AttendCursor c = {};
            c.seq = tid, c.q = q;
            c.head = (int)rest / of_head;
            int x = (int)rest - c.head * of_head;
            while (x >= (c.units = extra + attend_units(p, q, c.tile, rows, step))) x -= c.units, ++c.tile;
            c.units -= extra;
            c.unit = x - extra;
            found = c;
            have_found = 1;
        }
        __syncthreads();
        if (have_found) {
            r.cur = found;
            return r;
        }
    }
    r.cur = attend_find(p, rows, step, extra, 1, ALL, prefix, r.first);
    return r;
}

// What the joining kernel has to join, an entry a CTA of the kernel before: of an item that begins in its
// share and ends in another's the row of out (and lse) of its first row, its rows (0: none) and the last
// CTA.  From one of its rows to the next it is `step` rows of out.
struct alignas(16) LatentJoin {
    int64_t dst;
    int rows, last;
};

// Rows that the expanded form's scratch has for a sequence and head.
inline int64_t latent_seq_rows(int64_t tokens) { return ceil_div(tokens > 0 ? tokens : 1, (int64_t)128) * 128; }
// The expanded form's keys and values of a group of heads: row (head, sequence, token) at (head *
// n_seq + sequence) * seq_rows + token.
struct LatentSpace {
    void *k, *v;                      // [rows][nope], [rows][value]
    int64_t seq_rows, rows;           // seq_rows: latent_seq_rows; all rows: coordinates of tensor maps
    int64_t k_step, v_step;           // rows of w_k and w_v from one head to the next
    int head0, heads;
};

// Pairs of CTAs: how many fit on the GPU at a time, and a launch of so many.
template <typename K>
cudaError_t pairs_that_fit(K *kernel, int threads, size_t smem, int *pairs) {
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2, at.val.clusterDim.y = 1, at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(device_sm_count() & ~1)), cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem, cfg.attrs = &at, cfg.numAttrs = 1;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(pairs, kernel, &cfg);
    return e != cudaSuccess ? e : *pairs < 1 ? cudaErrorLaunchOutOfResources : cudaSuccess;
}
template <typename K, typename... Args>
cudaError_t launch_pairs(K *kernel, int pairs, int threads, size_t smem, cudaStream_t st, const Args &...args) {
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // see griddep_wait
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * pairs), cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem, cfg.stream = st, cfg.attrs = at, cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

// Scratch of the joins, the tokens of a box of the copies from the cache (boxes do not cross blocks), and
// the cache's tensor map: boxes of 64 values of at most
// `most` tokens.
int64_t latent_joins_bytes(int ctas);
int latent_box(const LatentParams &p, int most);
cudaError_t latent_rows_map(const LatentParams &p, int most, CUtensorMap *map);

cudaError_t launch_latent_join(const LatentParams &p, int dim, int ctas, int rows, int step, cudaStream_t st);

int64_t latent_absorbed_scratch(const LatentParams &p);
int64_t latent_expanded_scratch(const LatentParams &p);
cudaError_t launch_latent_absorbed(LatentParams &p, void *scratch, cudaStream_t st);
cudaError_t launch_latent_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st);
cudaError_t launch_latent_expanded(LatentParams &p, void *scratch, cudaStream_t st);

}  // namespace ak
