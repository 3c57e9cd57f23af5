// Items of the latent attention whose steps lay in several CTAs' shares: the parts' results, weighed and
// added in the order of the CTAs, so that results are the same bits every time.
//
// Items of few parts: a warp some rows of an item, whose parts' loads are then under way together (with a row a
// warp packed documents take 91.4 us, not 90.1, two prompts of 2048 rows 632 either way; 256 retrieved lists, of 16
// rows an item, 46.8, not 48.0).  Of many (a long
// sequence is one item in the shares of all CTAs): a CTA 128 values of a row, its parts in groups of threads
// that each add every so-manieth part up; 152 parts one after the other took 80 us.  The CTAs look for their
// rows among the items themselves: a CTA a row of what might be an item would be thousands that find none.
// Measured: 152 parts of 64 rows x 512, 12 us; 64 items of three or four such parts, 10 us; two prompts of 2048 rows and
// 32 heads 21; beginnings and latencies, not bytes, bound them.
#include "ak_latent.cuh"

namespace ak {

namespace {

constexpr int JOIN_THREADS = 512, JOIN_WARPS = JOIN_THREADS / 32;
constexpr int JOIN_CTAS = 1024;                // of the kernel before, at most
constexpr int FEW_PARTS = 32;                  // of an item whose rows take a warp each

template <int D>
__global__ void __launch_bounds__(JOIN_THREADS)
k_latent_join(const __grid_constant__ LatentParams lp, const int ctas, const int rows, const int step) {
    constexpr int RW = D < 128 ? 4 : 512 / D;  // rows of a warp where parts are few: four loads a lane are under way
    constexpr int WIDE = D < 128 ? D : 128, SLICES = D / WIDE, LANES = WIDE / 4, GROUPS = JOIN_THREADS / LANES;
    const AttendParams &p = lp.a;
    __shared__ int before[JOIN_CTAS + 1];      // rows, or runs of rows, of the items that begin in the CTAs before
    __shared__ int sums[JOIN_WARPS];
    __shared__ float factor[JOIN_CTAS], red[2][JOIN_WARPS];
    __shared__ float4 acc[JOIN_THREADS];
    griddep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // ---- the items, two CTAs' a thread
    const LatentJoin *joins = (const LatentJoin *)p.joins;
    auto rows_of = [&](int b) {
        if (b >= ctas) return 0;
        const LatentJoin j = joins[b];
        return j.last - b < FEW_PARTS ? (j.rows + JOIN_WARPS * RW - 1) / (JOIN_WARPS * RW) : j.rows * SLICES;
    };
    const int r0 = rows_of(2 * tid), r1 = rows_of(2 * tid + 1);
    int incl = r0 + r1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    for (int w = 0; w < warp; ++w) incl += sums[w];
    before[2 * tid] = incl - r0 - r1, before[2 * tid + 1] = incl - r1;
    if (tid == JOIN_THREADS - 1) before[JOIN_CTAS] = incl;
    __syncthreads();
    const int total = before[JOIN_CTAS];
    const int64_t floats = attend_slot_floats(rows, D);
    auto store = [&](int64_t at, float a, float b) {
        store_pair(p, lp.bf16, at, latent_result(a, lp.bf16), latent_result(b, lp.bf16));
    };
    for (int u = blockIdx.x; u < total; u += gridDim.x) {
        int lo = 0, hi = JOIN_CTAS;            // the last CTA with before <= u: the one whose item has row u
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (before[mid] <= u) lo = mid;
            else hi = mid;
        }
        const LatentJoin j = joins[lo];
        const int at = u - before[lo], parts = j.last - lo + 1;
        const float *base = p.partial + (int64_t)lo * 2 * floats;
        auto slot = [&](int k) { return base + (k ? (int64_t)k * 2 : 1) * floats; };
        if (parts <= FEW_PARTS) {
            const int rw = (at * JOIN_WARPS + warp) * RW, n = min(RW, j.rows - rw);
            if (n <= 0) continue;
            // lane: a part
            float f[RW], mx[RW], tot[RW];
#pragma unroll
            for (int y = 0; y < RW; ++y) {
                const bool have = lane < parts && y < n;
                mx[y] = have ? slot(lane)[rows * D + rw + y] : NEG;
                f[y] = have ? slot(lane)[rows * D + rows + rw + y] : 0.f;
            }
#pragma unroll
            for (int y = 0; y < RW; ++y) {
                const float m = mx[y];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) mx[y] = fmaxf(mx[y], __shfl_xor_sync(0xffffffffu, mx[y], o));
                f[y] = lane < parts ? ex2(m - mx[y]) * f[y] : 0.f;
                tot[y] = f[y];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) tot[y] += __shfl_xor_sync(0xffffffffu, tot[y], o);
            }
            constexpr int STRIPS = D > 128 ? D / 128 : 1;
            float4 v[RW][STRIPS];
#pragma unroll
            for (int y = 0; y < RW; ++y)
#pragma unroll
                for (int i = 0; i < STRIPS; ++i) v[y][i] = make_float4(0.f, 0.f, 0.f, 0.f);
            const bool mine = lane < D / 4;
#pragma unroll 2
            for (int k = 0; k < parts; ++k) {
                const float *src = slot(k) + rw * D + lane * 4;
                float4 x[RW][STRIPS];
#pragma unroll
                for (int y = 0; y < RW; ++y)
#pragma unroll
                    for (int i = 0; i < STRIPS; ++i)
                        x[y][i] = mine && y < n ? *(const float4 *)(src + y * D + i * 128)
                                                : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int y = 0; y < RW; ++y) {
                    const float fk = __shfl_sync(0xffffffffu, f[y], k);
#pragma unroll
                    for (int i = 0; i < STRIPS; ++i) {
                        v[y][i].x += fk * x[y][i].x, v[y][i].y += fk * x[y][i].y;
                        v[y][i].z += fk * x[y][i].z, v[y][i].w += fk * x[y][i].w;
                    }
                }
            }
#pragma unroll
            for (int y = 0; y < RW; ++y) {
                if (y >= n) continue;
                const int64_t dst = j.dst + (int64_t)(rw + y) * step;
                const float inv = tot[y] > 0.f ? 1.f / tot[y] : tot[y];        // a NaN stays one
#pragma unroll
                for (int i = 0; i < STRIPS; ++i)
                    if (mine) {
                        store(dst * D + lane * 4 + i * 128, v[y][i].x * inv, v[y][i].y * inv);
                        store(dst * D + lane * 4 + i * 128 + 2, v[y][i].z * inv, v[y][i].w * inv);
                    }
                if (lane == 0 && p.lse) p.lse[dst] = lse_of(mx[y], tot[y]);
            }
            continue;
        }
        // ---- the parts' weights
        const int r = at / SLICES, d0 = at % SLICES * WIDE;
        float mx = NEG, tot = 0.f;
        for (int k = tid; k < parts; k += JOIN_THREADS) mx = fmaxf(mx, slot(k)[rows * D + r]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if (lane == 0) red[0][warp] = mx;
        __syncthreads();
        for (int w = 0; w < JOIN_WARPS; ++w) mx = fmaxf(mx, red[0][w]);
        for (int k = tid; k < parts; k += JOIN_THREADS) {
            const float f = ex2(slot(k)[rows * D + r] - mx) * slot(k)[rows * D + rows + r];
            factor[k] = f;
            tot += f;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) tot += __shfl_xor_sync(0xffffffffu, tot, o);
        if (lane == 0) red[1][warp] = tot;
        __syncthreads();
        tot = 0.f;
        for (int w = 0; w < JOIN_WARPS; ++w) tot += red[1][w];
        const float inv = tot > 0.f ? 1.f / tot : tot;         // a NaN stays one
        // ---- the sum
        const int g = tid / LANES, d = d0 + tid % LANES * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = g; k < parts; k += GROUPS) {
            const float f = factor[k];
            const float4 y = *(const float4 *)(slot(k) + r * D + d);
            v.x += f * y.x, v.y += f * y.y, v.z += f * y.z, v.w += f * y.w;
        }
        acc[tid] = v;
        __syncthreads();
        if (g == 0) {
            for (int i = 1; i < GROUPS; ++i) {
                const float4 y = acc[i * LANES + tid];
                v.x += y.x, v.y += y.y, v.z += y.z, v.w += y.w;
            }
            const int64_t dst = j.dst + (int64_t)r * step;
            store(dst * D + d, v.x * inv, v.y * inv);
            store(dst * D + d + 2, v.z * inv, v.w * inv);
            if (tid == 0 && d0 == 0 && p.lse) p.lse[dst] = lse_of(mx, tot);
        }
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_latent_join(const LatentParams &p, int dim, int ctas, int rows, int step, cudaStream_t st) {
    if (ctas > JOIN_CTAS) return cudaErrorInvalidValue;        // (a GPU of more than 1024 SMs)
    auto *kernel = dim == 64    ? k_latent_join<64>
                   : dim == 128 ? k_latent_join<128>
                   : dim == 256 ? k_latent_join<256>
                                : k_latent_join<512>;
    return launch_pdl(kernel, dim3(2 * device_sm_count()), dim3(JOIN_THREADS), 0, st, p, ctas, rows, step);
}

}  // namespace ak
