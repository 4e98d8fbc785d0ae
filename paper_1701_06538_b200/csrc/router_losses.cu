// Losses of the router over all experts' probabilities, with their gradient: the balance loss f.P (Shazeer et al., 2017, in the form of Fedus et al., 2021) and
// the z loss (Zoph et al., 2022), over the whole batch or sequence by sequence. With p = softmax(logits), lse = log sum exp(logits), T_s the live tokens of sequence s, L all of them,
//   counts[s, j] = choices of expert j by them,   prob_sums[s, j] = sum of p_tj over them
//   balance = w_balance n / (k L) sum_s (1 / T_s) sum_j counts[s, j] prob_sums[s, j],   z = w_z / L sum_t lse_t^2
//   dlogits_tj = p_tj (c_j - sum_i c_i p_ti + 2 w_z lse_t / L),   c_j = w_balance n counts[s, j] / (k L T_s)      (counts are constants)
// Bound by memory: the logits are read once and the gradients written once. The counts are needed for every gradient and depend on topk_idx alone, which is small: they are
// made first, then one pass over the logits makes gradients and sums of probabilities together, and a last launch adds up the sums of its blocks. A block has
// consecutive tokens; where a sequence ends inside them it closes its sums and begins new ones: block c and sequence s leave theirs in place c + s, which no other two share.
// Sums are float in threads over a block's tokens and double over blocks, always in the same order.
#include <float.h>
#include <math_constants.h>

#include "block.cuh"

namespace moe {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int COUNT_CLUSTER = 8;  // blocks that count one sequence's choices together, where there are few sequences
constexpr int SUM_BLOCKS = 4 * 148;

struct Scratch {
    int32_t *live;     // [S] live tokens
    int32_t *ticket;   // blocks of the last launch that are done
    float *part;       // [chunks + S][n]
    double *z;         // [chunks] sums of lse^2
    double *balance;   // [SUM_BLOCKS]
};
int64_t rows_of_chunk(int64_t T) { return imax(8, cdiv(T, 4 * 148)); }
int64_t chunks_of(int64_t T) { return cdiv(imax(T, 1), rows_of_chunk(T)); }
Scratch scratch_at(Carver &cv, int64_t T, int32_t n, int32_t S) {
    Scratch s;
    s.live = cv.take<int32_t>(S);
    s.ticket = cv.take<int32_t>(1);
    s.part = cv.take<float>((chunks_of(T) + S) * n);
    s.z = cv.take<double>(chunks_of(T));
    s.balance = cv.take<double>(SUM_BLOCKS);
    return s;
}

// The tokens of a sequence: none from the last offset on and, whatever the offsets are, none outside the batch
__device__ __forceinline__ int2 tokens_of(const RouterLossArgs &a, int32_t s) {
    if (!a.offsets) return make_int2(0, (int32_t)a.T);
    const int32_t end = min(max(a.offsets[a.S], 0), (int32_t)a.T), from = min(max(a.offsets[s], 0), end), to = min(max(a.offsets[s + 1], 0), end);
    return make_int2(from, max(from, to));
}
__device__ __forceinline__ double sum_of_block(double v, double *sh) {  // of all threads, by all of them in the same order
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}

// Choices and live tokens of a sequence, by a cluster of blocks through each other's shared memory, or by one block
template <bool CLUSTER>
__global__ void __launch_bounds__(THREADS) router_counts_kernel(const RouterLossArgs a, const Scratch w) {
    extern __shared__ int32_t hist[];  // [n], and the live tokens
    const int32_t parts = CLUSTER ? COUNT_CLUSTER : 1, rank = CLUSTER ? blockIdx.x % COUNT_CLUSTER : 0, s = CLUSTER ? blockIdx.x / COUNT_CLUSTER : blockIdx.x;
    for (int32_t j = threadIdx.x; j <= a.n; j += THREADS) hist[j] = 0;
    __syncthreads();
    wait_previous_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.ticket = 0;
    const int2 t = tokens_of(a, s);
    const uint32_t k = (uint32_t)a.k;
    const int64_t end = (int64_t)t.y * k;
    int32_t live = 0;
#pragma unroll 4
    for (int64_t i = (int64_t)t.x * k + rank * THREADS + threadIdx.x; i < end; i += parts * THREADS) {
        const uint32_t token = (uint32_t)i / k;  // T k is below 2^31
        if (a.keep && !a.keep[token]) continue;
        live += (uint32_t)i == token * k;
        const int32_t e = a.topk_idx[i];
        if ((uint32_t)e < (uint32_t)a.n) atomicAdd(hist + e, 1);
    }
    live = __reduce_add_sync(0xffffffffu, live);
    if ((threadIdx.x & 31) == 0 && live) atomicAdd(hist + a.n, live);
    if constexpr (CLUSTER) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (int32_t j = rank * THREADS + threadIdx.x; j <= a.n; j += COUNT_CLUSTER * THREADS) {
            int32_t sum = 0;
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(hist + j);
#pragma unroll
            for (int32_t q = 0; q < COUNT_CLUSTER; ++q) {
                uint32_t there;
                int32_t v;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(q));
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(there) : "memory");
                sum += v;
            }
            if (j < a.n) a.counts[(int64_t)s * a.n + j] = sum;
            else w.live[s] = sum;
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");  // nobody leaves while it is read
    } else {
        __syncthreads();
        for (int32_t j = threadIdx.x; j <= a.n; j += THREADS) {
            if (j < a.n) a.counts[(int64_t)s * a.n + j] = hist[j];
            else w.live[s] = hist[j];
        }
    }
}

// Sums over the lanes of a row: a part of a warp, or the whole block (sh: a place per warp, twice)
template <int LANES> __device__ __forceinline__ float row_max(float v, float *sh) {
#pragma unroll
    for (int off = (LANES > 32 ? 32 : LANES) / 2; off > 0; off >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, v, off);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(o));
    }
    if constexpr (LANES > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(sh[w]));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ float2 row_sums(float2 v, float *sh) {
#pragma unroll
    for (int off = (LANES > 32 ? 32 : LANES) / 2; off > 0; off >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, off);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, off);
    }
    if constexpr (LANES > 32) {
        if ((threadIdx.x & 31) == 0) { sh[WARPS + (threadIdx.x >> 5)] = v.x; sh[2 * WARPS + (threadIdx.x >> 5)] = v.y; }
        __syncthreads();
        v = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { v.x += sh[WARPS + w]; v.y += sh[2 * WARPS + w]; }
    }
    return v;
}

template <int VEC> struct Columns;
template <> struct Columns<4> {
    float4 q;
    __device__ __forceinline__ void load(const float *p) { q = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<float4 *>(p) = q; }
    __device__ __forceinline__ float &operator[](int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
};
template <> struct Columns<1> {
    float q;
    __device__ __forceinline__ void load(const float *p) { q = *p; }
    __device__ __forceinline__ void store(float *p) const { *p = q; }
    __device__ __forceinline__ float &operator[](int) { return q; }
};

// LANES threads have a row, U vectors of VEC columns each
template <int LANES, int U, int VEC, bool GRAD>
__global__ void __launch_bounds__(THREADS) router_rows_kernel(const RouterLossArgs a, const Scratch w, int32_t chunk_rows) {
    constexpr int ROWS = THREADS / LANES;  // at a time
    extern __shared__ float sums[];        // [min(ROWS, WARPS)][n]
    __shared__ float sh[3 * WARPS];
    __shared__ double wide[WARPS];
    const int lane = threadIdx.x % LANES, place = threadIdx.x / LANES;
    const int32_t n = a.n;
    const int32_t first = (int32_t)blockIdx.x * chunk_rows, last = min(first + chunk_rows, (int32_t)a.T);
    wait_previous_kernel();
    auto column = [&](int u) { return (lane + u * LANES) * VEC; };
    // tokens that count, of all sequences
    double all = 0.0;
    for (int32_t s = threadIdx.x; s < a.S; s += THREADS) all += (double)w.live[s];
    all = sum_of_block(all, wide);
    const float by_z = all > 0.0 ? (float)(2.0 * (double)a.w_z / all) : 0.0f;
    // the sequence of the first token: the last one that begins at it or before
    int32_t s = 0;
    if (a.offsets) {
        int32_t lo = 0, hi = a.S;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (a.offsets[mid] <= first) lo = mid; else hi = mid;
        }
        s = lo;
    }
    double z = 0.0;
    auto zeros = [&](int32_t from, int32_t to) {  // rows outside all sequences
        if constexpr (GRAD)
            for (int64_t i = (int64_t)from * n + threadIdx.x; i < (int64_t)to * n; i += THREADS) a.dlogits[i] = 0.0f;
    };
    int32_t at = first;
    while (at < last) {
        if (s >= a.S) { zeros(at, last); break; }
        const int2 t = tokens_of(a, s);
        if (at < t.x) {  // (before the first sequence)
            const int32_t to = min(t.x, last);
            zeros(at, to);
            at = to;
            continue;
        }
        const int32_t end = min(t.y, last);
        if (end <= at) { ++s; continue; }
        const int32_t live = w.live[s];
        const float by = live > 0 ? (float)((double)a.w_balance * n / ((double)a.k * all * live)) : 0.0f;
        Columns<VEC> c[U], p[U];
        float lse2 = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                c[u][i] = column(u) + i < n ? (float)a.counts[(int64_t)s * n + column(u) + i] * by : 0.0f;
                p[u][i] = 0.0f;
            }
        for (int32_t base = at; base < end; base += ROWS) {
            const int32_t row = base + place;
            const bool in = row < end, live_row = in && (!a.keep || a.keep[row]);
            const float *x = a.logits + (int64_t)row * n;
            Columns<VEC> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[u][i] = -CUDART_INF_F;
                if (live_row && column(u) < n) v[u].load(x + column(u));
            }
            float top = -CUDART_INF_F;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(v[u][i]));
            top = row_max<LANES>(top, sh);
            const bool empty = top == -CUDART_INF_F;  // no expert left, or no row
            float2 two = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[u][i] = empty ? 0.0f : exp2f((v[u][i] - top) * 1.44269504088896340736f);
                    two.x += v[u][i];
                    two.y = fmaf(c[u][i], v[u][i], two.y);
                }
            two = row_sums<LANES>(two, sh);
            const float r = empty ? 0.0f : 1.0f / two.x, lse = empty ? 0.0f : top + logf(two.x);
            const float pull = fmaf(two.y, -r, by_z * lse);
            if (lane == 0) lse2 = fmaf(lse, lse, lse2);
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[u][i] *= r;
                    p[u][i] += v[u][i];
                    v[u][i] *= c[u][i] + pull;
                }
                if (GRAD && in && column(u) < n) v[u].store(a.dlogits + (int64_t)row * n + column(u));
            }
        }
        z += (double)lse2;
        // the block's sums of this sequence: rows of a warp, then warps
#pragma unroll
        for (int off = LANES; off < 32; off <<= 1)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) p[u][i] += __shfl_xor_sync(0xffffffffu, p[u][i], off);
        float *to = w.part + ((int64_t)blockIdx.x + s) * n;
        if constexpr (LANES > 32) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (column(u) < n) p[u].store(to + column(u));
        } else {
            __syncthreads();
            if ((threadIdx.x & 31) < LANES)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (column(u) < n) p[u].store(sums + (threadIdx.x >> 5) * n + column(u));
            __syncthreads();
            for (int32_t j = threadIdx.x; j < n; j += THREADS) {
                float v = sums[j];
#pragma unroll
                for (int q = 1; q < WARPS; ++q) v += sums[q * n + j];
                to[j] = v;
            }
        }
        at = end;
        if (at >= t.y) ++s;
    }
    z = sum_of_block(z, wide);
    if (threadIdx.x == 0) w.z[blockIdx.x] = z;
}

// prob_sums of a sequence's 32 columns from the chunks that it lies in, and the two losses by the last block to be done
__global__ void __launch_bounds__(THREADS) router_sums_kernel(const RouterLossArgs a, const Scratch w, int32_t chunk_rows, int32_t chunks) {
    __shared__ double wide[WARPS], cols[WARPS][32];
    __shared__ bool last_one;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t groups = (a.n + 31) / 32;
    wait_previous_kernel();
    double all = 0.0, balance = 0.0;
    for (int32_t s = threadIdx.x; s < a.S; s += THREADS) all += (double)w.live[s];
    all = sum_of_block(all, wide);
    for (int64_t item = blockIdx.x; item < (int64_t)a.S * groups; item += gridDim.x) {
        const int32_t s = (int32_t)(item / groups), j = (int32_t)(item % groups) * 32 + lane;
        const int2 t = tokens_of(a, s);
        double v = 0.0;
        if (t.y > t.x && j < a.n)
#pragma unroll 4
            for (int32_t c = t.x / chunk_rows + warp; c <= (t.y - 1) / chunk_rows; c += WARPS) v += (double)w.part[((int64_t)c + s) * a.n + j];
        __syncthreads();
        cols[warp][lane] = v;
        __syncthreads();
        if (warp == 0 && j < a.n) {
#pragma unroll
            for (int q = 1; q < WARPS; ++q) v += cols[q][lane];
            if (a.prob_sums) a.prob_sums[(int64_t)s * a.n + j] = (float)v;
            const int32_t live = w.live[s];
            if (live > 0) balance += v * (double)a.counts[(int64_t)s * a.n + j] / live;
        }
    }
    balance = sum_of_block(balance, wide);
    if (threadIdx.x == 0) {
        w.balance[blockIdx.x] = balance;
        __threadfence();
        last_one = atomicAdd(w.ticket, 1) == (int32_t)gridDim.x - 1;
    }
    __syncthreads();
    if (!last_one) return;
    __threadfence();
    balance = 0.0;
    double z = 0.0;
    for (int32_t i = threadIdx.x; i < (int32_t)gridDim.x; i += THREADS) balance += __ldcg(w.balance + i);
    for (int32_t i = threadIdx.x; i < chunks; i += THREADS) z += w.z[i];
    balance = sum_of_block(balance, wide);
    z = sum_of_block(z, wide);
    if (threadIdx.x == 0) {
        a.losses[0] = all > 0.0 ? (float)((double)a.w_balance * a.n / ((double)a.k * all) * balance) : 0.0f;
        a.losses[1] = all > 0.0 ? (float)((double)a.w_z / all * z) : 0.0f;
    }
}

template <int LANES, int U, int VEC> int32_t rows(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    const size_t bytes = LANES > 32 ? 0 : (size_t)WARPS * a.n * sizeof(float);  // at most 32 KiB
    const unsigned grid = (unsigned)chunks_of(a.T);
    const int32_t chunk = (int32_t)rows_of_chunk(a.T);
    if (a.dlogits) launch_kernel(router_rows_kernel<LANES, U, VEC, true>, grid, THREADS, bytes, st, a, w, chunk);
    else launch_kernel(router_rows_kernel<LANES, U, VEC, false>, grid, THREADS, bytes, st, a, w, chunk);
    MOE_LAUNCHED();
    return MOE_OK;
}
int32_t launch_rows(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    if (a.n % 4 == 0) {
        if (a.n <= 32) return rows<8, 1, 4>(a, w, st);
        if (a.n <= 64) return rows<16, 1, 4>(a, w, st);
        if (a.n <= 128) return rows<32, 1, 4>(a, w, st);
        if (a.n <= 256) return rows<32, 2, 4>(a, w, st);
        if (a.n <= 512) return rows<32, 4, 4>(a, w, st);
        if (a.n <= 1024) return rows<32, 8, 4>(a, w, st);
        if (a.n <= 2048) return rows<256, 2, 4>(a, w, st);
        return rows<256, 8, 4>(a, w, st);
    }
    if (a.n <= 32) return rows<32, 1, 1>(a, w, st);
    if (a.n <= 128) return rows<32, 4, 1>(a, w, st);
    if (a.n <= 512) return rows<32, 16, 1>(a, w, st);
    if (a.n <= 1024) return rows<32, 32, 1>(a, w, st);
    if (a.n <= 2048) return rows<256, 8, 1>(a, w, st);
    return rows<256, 32, 1>(a, w, st);
}

int32_t launch_counts(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    const size_t bytes = (size_t)(a.n + 1) * sizeof(int32_t);  // at most 32 KiB and a word
    // one block a sequence once there are enough of them for most SMs
    if (a.S * COUNT_CLUSTER > 148) {
        launch_kernel(router_counts_kernel<false>, dim3((unsigned)a.S), dim3(THREADS), bytes, st, a, w);
        MOE_LAUNCHED();
        return MOE_OK;
    }
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = COUNT_CLUSTER; attrs[0].val.clusterDim.y = 1; attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // as launch_kernel
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.S * COUNT_CLUSTER); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = bytes; cfg.stream = st;
    cfg.attrs = attrs; cfg.numAttrs = 2;
    cudaLaunchKernelEx(&cfg, router_counts_kernel<true>, a, w);
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace

int64_t router_losses_bytes(int64_t T, int32_t n, int32_t S) {
    Carver cv(nullptr);
    scratch_at(cv, T, n, S);
    return (int64_t)cv.off;
}

int32_t launch_router_losses(const RouterLossArgs &a, void *ws, cudaStream_t st) {
    Carver cv(ws);
    const Scratch w = scratch_at(cv, a.T, a.n, a.S);
    MOE_TRY(launch_counts(a, w, st));
    MOE_TRY(launch_rows(a, w, st));
    const int64_t items = (int64_t)a.S * cdiv(a.n, 32);
    launch_kernel(router_sums_kernel, dim3((unsigned)imin(items, SUM_BLOCKS)), dim3(THREADS), 0, st, a, w, (int32_t)rows_of_chunk(a.T), (int32_t)chunks_of(a.T));
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace moe
