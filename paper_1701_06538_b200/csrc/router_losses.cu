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
#include "pairs.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int COUNT_THREADS = 1024, COUNT_EACH = 8;  // choices a thread has on their way
constexpr int SUM_WARPS = 32, SUM_BLOCKS = 2 * 148;
constexpr int ROW_BLOCKS = 2 * 148;                  // two an SM (131072 x 128 with 4, 3 and 2, four rows at a time: 47.3, 41.0, 40.9 us; 20000 x 512: 35.0, 35.1, 31.3)

struct Scratch {
    int32_t *live;     // [S] live tokens
    int32_t *ticket;   // blocks of the last launch that are done
    float *part;       // [chunks + S][n]
    double *z;         // [chunks] sums of lse^2
    double *balance;   // [SUM_BLOCKS]
};
// Tokens of a block, a multiple of the most rows that a warp has at a time. (Multiples of 32: 477 x 376 of 324 sequences 47 us instead of 21, one after the other in 15 blocks; 4190 x 1276 39 instead
// of 30; 20000 x 512 33 instead of 32. Of 8: 477 x 376 25 us.)
constexpr int64_t CHUNK_ROWS = 4;
int64_t rows_of_chunk(int64_t T) { return cdiv(cdiv(imax(T, 1), ROW_BLOCKS), CHUNK_ROWS) * CHUNK_ROWS; }
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
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// Of N warps, for all of them, always in the same order. (By exchanges: a chain of additions in double is 30 of its latencies.) sh: a place per warp
template <int N> __device__ __forceinline__ double sum_of_block(double v, double *sh) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < N ? sh[threadIdx.x & 31] : 0.0);
}

// Choices and live tokens of a sequence into hist [n + 1], by `parts` blocks together. (The loads of COUNT_EACH choices go before what depends on them.)
__device__ __forceinline__ void count_choices(const RouterLossArgs &a, const Divisor &by_k, int32_t s, int32_t rank, int32_t parts, int32_t *hist) {
    const int2 t = tokens_of(a, s);
    const int32_t end = t.y * a.k, stride = parts * (int32_t)blockDim.x;  // T k is below 2^31
    int32_t live = 0;
    for (int64_t i = (int64_t)t.x * a.k + rank * blockDim.x + threadIdx.x; i < end; i += (int64_t)COUNT_EACH * stride) {
        int32_t e[COUNT_EACH], in_token[COUNT_EACH];
        bool in[COUNT_EACH];
#pragma unroll
        for (int q = 0; q < COUNT_EACH; ++q) {
            const int64_t at = i + (int64_t)q * stride;
            in[q] = at < end;
            e[q] = in[q] ? a.topk_idx[at] : -1;
            const int32_t token = by_k((int32_t)(in[q] ? at : 0), in_token[q]);
            if (a.keep && in[q]) in[q] = a.keep[token] != 0;
        }
#pragma unroll
        for (int q = 0; q < COUNT_EACH; ++q) {
            if (!in[q]) continue;
            live += in_token[q] == 0;
            if ((uint32_t)e[q] < (uint32_t)a.n) atomicAdd(hist + e[q], 1);
        }
    }
    live = __reduce_add_sync(0xffffffffu, live);
    if ((threadIdx.x & 31) == 0 && live) atomicAdd(hist + a.n, live);
}
// By a cluster of blocks through each other's shared memory, or by one block
template <bool CLUSTER>
__global__ void __launch_bounds__(COUNT_THREADS) router_counts_kernel(const RouterLossArgs a, const Scratch w, const Divisor by_k, int32_t parts) {
    extern __shared__ int32_t hist[];  // [n], and the live tokens
    const int32_t rank = CLUSTER ? blockIdx.x % parts : 0, s = CLUSTER ? blockIdx.x / parts : blockIdx.x;
    for (int32_t j = threadIdx.x; j <= a.n; j += COUNT_THREADS) hist[j] = 0;
    __syncthreads();
    wait_previous_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.ticket = 0;
    count_choices(a, by_k, s, rank, parts, hist);
    if constexpr (CLUSTER) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        for (int32_t j = rank * COUNT_THREADS + threadIdx.x; j <= a.n; j += parts * COUNT_THREADS) {
            int32_t sum = 0;
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(hist + j);
#pragma unroll 8
            for (int32_t q = 0; q < parts; ++q) {
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
        for (int32_t j = threadIdx.x; j <= a.n; j += COUNT_THREADS) {
            if (j < a.n) a.counts[(int64_t)s * a.n + j] = hist[j];
            else w.live[s] = hist[j];
        }
    }
}

__device__ __forceinline__ float larger(float a, float b) {  // a NaN stays
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
}
// N values over the lanes of a row at once, put together by `op`: in the first steps lanes give away half of their values, so that eight take seventeen exchanges with what tells
// all lanes, not forty. LANES is a part of a warp; or the whole block (N values of one row; sh: a place per warp and value)
template <int N, int LANES, typename Op> __device__ __forceinline__ void over_lanes(float (&s)[N], float *sh, Op op) {
    constexpr int L = LANES > 32 ? 32 : LANES;
    const int lane = threadIdx.x & 31;
    int off = L / 2, m = N / 2;
#pragma unroll
    for (; m >= 1; m >>= 1, off >>= 1) {
        const bool up = lane & off;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float keep = up ? s[i + m] : s[i], send = up ? s[i] : s[i + m];
            s[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, off));
        }
    }
    float t = s[0];
#pragma unroll
    for (; off >= 1; off >>= 1) t = op(t, __shfl_xor_sync(0xffffffffu, t, off));
    constexpr int EACH = L / N;
    if constexpr (LANES > 32) {
        __syncthreads();
        if (lane % EACH == 0) sh[(threadIdx.x >> 5) * N + lane / EACH] = t;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = sh[i];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) s[i] = op(s[i], sh[w * N + i]);
        }
    } else if constexpr (N > 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = __shfl_sync(0xffffffffu, t, i * EACH, L);
    } else {
        s[0] = t;
    }
}

__device__ __forceinline__ float power_of_two(float x) {  // the hardware's, to two units of the last place; 0 below float's smallest normal number
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// A thread's columns of a row as pairs: U vectors of VEC columns, LANES vectors apart
template <int LANES, int U, int VEC> struct Columns {
    static constexpr int H = U * VEC / 2;
    static_assert(U * VEC % 2 == 0, "pairs");
    int32_t n;
    int lane;
    bool in[U];
    __device__ __forceinline__ Columns(int32_t n_, int lane_) : n(n_), lane(lane_) {
#pragma unroll
        for (int u = 0; u < U; ++u) in[u] = (lane + u * LANES) * VEC < n;
    }
    __device__ __forceinline__ int32_t column(int e) const { return (lane + e / VEC * LANES) * VEC + e % VEC; }
    // row: of the thread's first column
    __device__ __forceinline__ void load(const float *row, float2 (&v)[H]) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            if constexpr (VEC == 4) {
                const float4 q = *reinterpret_cast<const float4 *>(row + u * (LANES * 4));
                v[2 * u] = make_float2(q.x, q.y);
                v[2 * u + 1] = make_float2(q.z, q.w);
            } else {
                (u & 1 ? v[u / 2].y : v[u / 2].x) = row[u * LANES];
            }
        }
    }
    __device__ __forceinline__ void store(float *row, const float2 (&v)[H]) const {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!in[u]) continue;
            if constexpr (VEC == 4) *reinterpret_cast<float4 *>(row + u * (LANES * 4)) = make_float4(v[2 * u].x, v[2 * u].y, v[2 * u + 1].x, v[2 * u + 1].y);
            else row[u * LANES] = u & 1 ? v[u / 2].y : v[u / 2].x;
        }
    }
};

// Rows first .. last - 1 by a block. LANES threads have R rows at a time, some pairs of columns of each, and the next R rows on their way.
template <int LANES, int U, int VEC, int R, bool GRAD>
__device__ __forceinline__ void router_rows(const RouterLossArgs &a, const Scratch &w, int32_t block, int32_t first, int32_t last, float *sums, double *wide, float *sh) {
    constexpr int ROWS = THREADS / LANES * R, H = U * VEC / 2;  // at a time
    constexpr float LOG2_E = 1.44269504088896340736f;
    const int place = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int32_t n = a.n;
    const Columns<LANES, U, VEC> mine(n, lane);
    // tokens that count, of all sequences
    double all = 0.0;
    if (a.S == 1) {
        all = (double)w.live[0];
    } else {
        for (int32_t s = threadIdx.x; s < a.S; s += THREADS) all += (double)w.live[s];
        all = sum_of_block<WARPS>(all, wide);
    }
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
        float2 next[R][H];
        int32_t row = at + place * R;  // the first of the rows to be fetched
        const int64_t from = (int64_t)row * n + mine.lane * VEC;
        const float *x_at = a.logits + from;
        float *d_at = GRAD ? a.dlogits + from : nullptr;
        auto fetch = [&]() {
            const float *x = x_at;
#pragma unroll
            for (int r = 0; r < R; ++r, x += n) {
#pragma unroll
                for (int h = 0; h < H; ++h) next[r][h] = both(-CUDART_INF_F);
                if (row + r < end && (!a.keep || a.keep[row + r])) mine.load(x, next[r]);
            }
            row += ROWS;
            x_at += (int64_t)ROWS * n;
        };
        fetch();
        float2 c[H], p[H];
        float lse2 = 0.0f;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int32_t j = mine.column(2 * h), i = mine.column(2 * h + 1);
            c[h] = make_float2(j < n ? (float)a.counts[(int64_t)s * n + j] * by : 0.0f, i < n ? (float)a.counts[(int64_t)s * n + i] * by : 0.0f);
            p[h] = both(0.0f);
        }
#pragma unroll 1
        for (int32_t left = end - at - place * R, base = at; base < end; base += ROWS, left -= ROWS) {  // left: rows from the first one of this turn on
            float2 v[R][H];
            float top[R], two[2 * R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                top[r] = larger(next[r][0].x, next[r][0].y);
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    v[r][h] = next[r][h];
                    if (h > 0) top[r] = larger(larger(v[r][h].x, v[r][h].y), top[r]);
                }
            }
            if (base + ROWS < end) fetch();
            over_lanes<R, LANES>(top, sh, larger);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (top[r] == -CUDART_INF_F) top[r] = 0.0f;  // no expert left, or no row: every power is 0
                float2 sum = both(0.0f), pull = both(0.0f);
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    const float2 t2 = mul2(fma2(v[r][h], both(1.0f), both(-top[r])), both(LOG2_E));
                    v[r][h] = make_float2(power_of_two(t2.x), power_of_two(t2.y));
                    sum = fma2(v[r][h], both(1.0f), sum);
                    pull = fma2(c[h], v[r][h], pull);
                }
                two[2 * r] = sum.x + sum.y;
                two[2 * r + 1] = pull.x + pull.y;
            }
            over_lanes<2 * R, LANES>(two, sh, [](float x, float y) { return x + y; });
            float *d = d_at;
#pragma unroll
            for (int r = 0; r < R; ++r, d += n) {
                const bool empty = two[2 * r] == 0.0f;
                const float by_sum = empty ? 0.0f : __fdividef(1.0f, two[2 * r]), lse = empty ? 0.0f : top[r] + logf(two[2 * r]);
                const float pull = fmaf(two[2 * r + 1], -by_sum, by_z * lse) * by_sum;
                lse2 = fmaf(lse, lse, lse2);
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    p[h] = fma2(v[r][h], both(by_sum), p[h]);
                    v[r][h] = mul2(v[r][h], fma2(c[h], both(by_sum), both(pull)));
                }
                if (GRAD && r < left) mine.store(d, v[r]);
            }
            if constexpr (GRAD) d_at += (int64_t)ROWS * n;
        }
        if (lane == 0) z += (double)lse2;
        // the block's sums of this sequence: rows of a warp, then warps
#pragma unroll
        for (int off = LANES; off < 32; off <<= 1)
#pragma unroll
            for (int h = 0; h < H; ++h) {
                p[h].x += __shfl_xor_sync(0xffffffffu, p[h].x, off);
                p[h].y += __shfl_xor_sync(0xffffffffu, p[h].y, off);
            }
        float *to = w.part + ((int64_t)block + s) * n;
        if constexpr (LANES > 32) {
            mine.store(to + lane * VEC, p);
        } else {
            __syncthreads();
            if ((threadIdx.x & 31) < LANES) mine.store(sums + (threadIdx.x >> 5) * n + lane * VEC, p);
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
    z = sum_of_block<WARPS>(z, wide);
    if (threadIdx.x == 0) w.z[block] = z;
}
template <int LANES, int U, int VEC, int R, bool GRAD>
__global__ void __launch_bounds__(THREADS, U * VEC <= 16 ? 2 : 1) router_rows_kernel(const RouterLossArgs a, const Scratch w, int32_t chunk_rows) {
    extern __shared__ __align__(16) float sums[];  // [WARPS][n]
    __shared__ float sh[2 * WARPS];
    __shared__ double wide[WARPS];
    const int32_t first = (int32_t)blockIdx.x * chunk_rows, last = min(first + chunk_rows, (int32_t)a.T);
    wait_previous_kernel();
    router_rows<LANES, U, VEC, R, GRAD>(a, w, blockIdx.x, first, last, sums, wide, sh);
}

// What `v`, of every warp's lanes' columns, comes to: prob_sums and the sequence's part of the balance loss
__device__ __forceinline__ double put_sums(const RouterLossArgs &a, const Scratch &w, int32_t s, int32_t j, double v) {
    if (j >= a.n) return 0.0;
    if (a.prob_sums) a.prob_sums[(int64_t)s * a.n + j] = (float)v;
    const int32_t live = w.live[s];
    return live > 0 ? v * (double)a.counts[(int64_t)s * a.n + j] / live : 0.0;
}
__device__ __forceinline__ void put_losses(const RouterLossArgs &a, double all, double balance, double z) {
    a.losses[0] = all > 0.0 ? (float)((double)a.w_balance * a.n / ((double)a.k * all) * balance) : 0.0f;
    a.losses[1] = all > 0.0 ? (float)((double)a.w_z / all * z) : 0.0f;
}
// prob_sums of a sequence's 32 columns from the chunks that it lies in, by the warps of a block together (their loads at once) or, where sequences are short, by one of them; and the
// two losses by the last block to be done
template <bool BLOCK>
__global__ void __launch_bounds__(SUM_WARPS * 32) router_sums_kernel(const RouterLossArgs a, const Scratch w, int32_t chunk_rows, int32_t chunks) {
    __shared__ double wide[SUM_WARPS], cols[SUM_WARPS][33];
    __shared__ bool last_one;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t groups = (a.n + 31) / 32;
    const int64_t items = (int64_t)a.S * groups;
    wait_previous_kernel();
    double balance = 0.0;
    for (int64_t item = BLOCK ? blockIdx.x : (int64_t)blockIdx.x * SUM_WARPS + warp; item < items; item += (int64_t)gridDim.x * (BLOCK ? 1 : SUM_WARPS)) {
        const int32_t s = (int32_t)(item / groups), j = (int32_t)(item % groups) * 32 + lane;
        const int2 t = tokens_of(a, s);
        double v = 0.0;
        if (t.y > t.x && j < a.n)
#pragma unroll 5
            for (int32_t c = t.x / chunk_rows + (BLOCK ? warp : 0); c <= (t.y - 1) / chunk_rows; c += BLOCK ? SUM_WARPS : 1) v += (double)w.part[((int64_t)c + s) * a.n + j];
        if constexpr (BLOCK) {
            __syncthreads();
            cols[warp][lane] = v;
            __syncthreads();
            v = warp_sum(cols[lane][warp]);  // of column `warp`
            if (lane == 0) balance += put_sums(a, w, s, j - lane + warp, v);
        } else {
            balance += put_sums(a, w, s, j, v);
        }
    }
    balance = sum_of_block<SUM_WARPS>(balance, wide);
    if (threadIdx.x == 0) {
        w.balance[blockIdx.x] = balance;
        __threadfence();
        last_one = atomicAdd(w.ticket, 1) == (int32_t)gridDim.x - 1;
    }
    __syncthreads();
    if (!last_one) return;
    __threadfence();
    balance = 0.0;
    double z = 0.0, all = 0.0;
    for (int32_t i = threadIdx.x; i < (int32_t)gridDim.x; i += SUM_WARPS * 32) balance += __ldcg(w.balance + i);
    for (int32_t i = threadIdx.x; i < chunks; i += SUM_WARPS * 32) z += w.z[i];
    for (int32_t s = threadIdx.x; s < a.S; s += SUM_WARPS * 32) all += (double)w.live[s];
    balance = warp_sum(balance);
    z = warp_sum(z);
    all = warp_sum(all);
    if (lane == 0) { cols[0][warp] = balance; cols[1][warp] = z; cols[2][warp] = all; }
    __syncthreads();
    if (warp > 0) return;
    balance = warp_sum(cols[0][lane]);
    z = warp_sum(cols[1][lane]);
    all = warp_sum(cols[2][lane]);
    if (lane == 0) put_losses(a, all, balance, z);
}

// Everything by one block, for a few rows
template <int LANES, int U, int VEC, int R, bool GRAD>
__global__ void __launch_bounds__(THREADS) router_small_kernel(const RouterLossArgs a, const Scratch w, const Divisor by_k) {
    extern __shared__ __align__(16) float sums[];  // [WARPS][n], and the counts [n + 1] of a sequence before
    __shared__ float sh[2 * WARPS];
    __shared__ double wide[WARPS];
    wait_previous_kernel();
    int32_t *hist = reinterpret_cast<int32_t *>(sums);
    for (int32_t s = 0; s < a.S; ++s) {
        for (int32_t j = threadIdx.x; j <= a.n; j += THREADS) hist[j] = 0;
        __syncthreads();
        count_choices(a, by_k, s, 0, 1, hist);
        __syncthreads();
        for (int32_t j = threadIdx.x; j <= a.n; j += THREADS) {
            if (j < a.n) a.counts[(int64_t)s * a.n + j] = hist[j];
            else w.live[s] = hist[j];
        }
        __syncthreads();
    }
    router_rows<LANES, U, VEC, R, GRAD>(a, w, 0, 0, (int32_t)a.T, sums, wide, sh);
    __syncthreads();
    double balance = 0.0, all = 0.0;
    for (int32_t i = threadIdx.x; i < a.S * a.n; i += THREADS) {
        const int32_t s = i / a.n, j = i - s * a.n;
        const int2 t = tokens_of(a, s);
        balance += put_sums(a, w, s, j, t.y > t.x ? (double)w.part[(int64_t)s * a.n + j] : 0.0);
    }
    for (int32_t s = threadIdx.x; s < a.S; s += THREADS) all += (double)w.live[s];
    balance = sum_of_block<WARPS>(balance, wide);
    all = sum_of_block<WARPS>(all, wide);
    if (threadIdx.x == 0) put_losses(a, all, balance, w.z[0]);
}

// One block: as many rows and columns as it has done while three launches follow one another (256 x 64 in a recorded graph 9.5 us by one, 13.0 by three; 16 x 1000 10.2 and 15.7; 512 x 64 14.0 and 13.7)
constexpr int64_t SMALL = 16384;
bool small(const RouterLossArgs &a) { return a.T * a.n <= SMALL && (int64_t)a.S * a.n <= SMALL && a.n <= 1024 && a.S <= 16; }

template <int LANES, int U, int VEC, int R> int32_t rows(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    const size_t bytes = LANES > 32 ? 0 : (size_t)WARPS * a.n * sizeof(float);  // at most 32 KiB
    if constexpr (LANES <= 32) {
        if (small(a)) {
            const size_t both = imax((int64_t)bytes, (a.n + 1) * 4);
            launch_kernel(a.dlogits ? router_small_kernel<LANES, U, VEC, R, true> : router_small_kernel<LANES, U, VEC, R, false>, dim3(1), dim3(THREADS), both, st, a, w, Divisor::of(a.k));
            MOE_LAUNCHED();
            return MOE_OK;
        }
    }
    launch_kernel(a.dlogits ? router_rows_kernel<LANES, U, VEC, R, true> : router_rows_kernel<LANES, U, VEC, R, false>, dim3((unsigned)chunks_of(a.T)), dim3(THREADS), bytes, st, a, w,
                  (int32_t)rows_of_chunk(a.T));
    MOE_LAUNCHED();
    return MOE_OK;
}
int32_t launch_rows(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    if (a.n % 4 == 0) {
        if (a.n <= 32) return rows<8, 1, 4, 4>(a, w, st);
        if (a.n <= 64) return rows<16, 1, 4, 4>(a, w, st);
        if (a.n <= 128) return rows<32, 1, 4, 4>(a, w, st);
        if (a.n <= 256) return rows<32, 2, 4, 4>(a, w, st);
        if (a.n <= 512) return rows<32, 4, 4, 1>(a, w, st);
        if (a.n <= 1024) return rows<32, 8, 4, 1>(a, w, st);
        if (a.n <= 2048) return rows<256, 2, 4, 1>(a, w, st);
        return rows<256, 8, 4, 1>(a, w, st);
    }
    if (a.n <= 32) return rows<16, 2, 1, 4>(a, w, st);
    if (a.n <= 128) return rows<32, 4, 1, 4>(a, w, st);
    if (a.n <= 512) return rows<32, 16, 1, 1>(a, w, st);
    if (a.n <= 1024) return rows<32, 32, 1, 1>(a, w, st);
    if (a.n <= 2048) return rows<256, 8, 1, 1>(a, w, st);
    return rows<256, 32, 1, 1>(a, w, st);
}

int32_t launch_counts(const RouterLossArgs &a, const Scratch &w, cudaStream_t st) {
    const size_t bytes = (size_t)(a.n + 1) * sizeof(int32_t);  // at most 32 KiB and a word
    // blocks for a sequence, so that most SMs have one (one each: 131072 x 128 of one sequence 96 us instead of 41, 32768 x 64 of eight 27.7 instead of 23.5, of 30 21.7 instead of 20.7)
    const int parts = a.S <= 9 ? 16 : a.S <= 18 ? 8 : a.S <= 37 ? 4 : a.S <= 74 ? 2 : 1;
    if (parts == 1) {
        launch_kernel(router_counts_kernel<false>, dim3((unsigned)a.S), dim3(COUNT_THREADS), bytes, st, a, w, Divisor::of(a.k), 1);
        MOE_LAUNCHED();
        return MOE_OK;
    }
    static PerDevice wide;
    const bool sixteen = wide.get([&]() {
        return cudaFuncSetAttribute(reinterpret_cast<const void *>(router_counts_kernel<true>), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess ? 1 : 0;
    }) > 0;
    if (!sixteen) return MOE_ERR_CUDA;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = parts; attrs[0].val.clusterDim.y = 1; attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // as launch_kernel
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.S * parts)); cfg.blockDim = dim3(COUNT_THREADS); cfg.dynamicSmemBytes = bytes; cfg.stream = st;
    cfg.attrs = attrs; cfg.numAttrs = 2;
    cudaLaunchKernelEx(&cfg, router_counts_kernel<true>, a, w, Divisor::of(a.k), parts);
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
    const bool one = small(a);
    if (!one) MOE_TRY(launch_counts(a, w, st));
    MOE_TRY(launch_rows(a, w, st));
    if (one) return MOE_OK;
    const int64_t items = (int64_t)a.S * cdiv(a.n, 32), chunk = rows_of_chunk(a.T);
    // A warp each where a sequence lies in four chunks or fewer for every turn that blocks would take. (131072 x 128, one sequence: blocks 41 us, warps 69; 32768 x 64 of 40: 21 and 24; 32768 x 256
    // of 61, two turns: 33.9 and 31.0; 8443 x 84 of 118: 20.8 and 19.3)
    const bool blocks = a.T > 4 * chunk * a.S * cdiv(items, SUM_BLOCKS);
    launch_kernel(blocks ? router_sums_kernel<true> : router_sums_kernel<false>, dim3((unsigned)imin(blocks ? items : cdiv(items, SUM_WARPS), SUM_BLOCKS)), dim3(SUM_WARPS * 32), 0, st, a, w,
                  (int32_t)chunk, (int32_t)chunks_of(a.T));
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace moe
