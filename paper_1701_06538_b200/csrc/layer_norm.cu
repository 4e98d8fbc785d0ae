// Layer norm (Ba, Kiros and Hinton, 2016) of the rows before a block, one pass over memory each way.
//   xn = (x - mean) r w + b,   r = (variance + eps)^-1/2,   mean and variance over the row's columns
// Backward, with n = (x - mean) r and u = dxn w:
//   dX = dres + r (u - mean(u) - n mean(u n)),   dw = sum of dxn n over the rows,   db = sum of dxn
// Bound by memory (a row's 7 or 13 operations an element are a tenth of what the cores do meanwhile). A team of warps has K rows at a time, a vector or a few of each
// in every thread, from the first sum to the store, and the next rows on their way: every thread copies what it will read itself, so that no barrier and no wait but its own
// stands between them. The variance is taken of the differences from the mean, a second sum over the team: the mean of squares less the square of the mean loses what a
// row's mean is larger than its spread. Sums are float in threads and teams, double over the blocks' sums of columns, in a fixed order.
#include "async_copy.cuh"
#include "block.cuh"
#include "pairs.cuh"
#include "vectors.cuh"

namespace moe {

namespace {

// Rows of a team on their way or in work (131072 x 1024 forward with 2, 3, 4 of them: 94.2, 95.9, 97.1 us; backward of 65536 x 1024 with 2, 3, 4: 85.8, 86.2, 87.0)
constexpr int STAGES = 2;

__device__ __forceinline__ float2 add2(float2 a, float2 b) { return fma2(a, both(1.0f), b); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// N sums over the threads of a team at once: in the first steps lanes give away half of their sums, so that four sums take seven exchanges and not twenty. Lane l is left with
// sum l / (32 / N). `sh` has a place per warp and sum, twice: who writes the next sums does so on the other side, and the barrier of those keeps it from coming round.
template <int N, bool ONE> __device__ __forceinline__ void sums_of_team(float (&s)[N], int warps, float *sh, int &side) {
    const int lane = threadIdx.x & 31;
    float t;
    if constexpr (N == 1) {
        t = warp_sum(s[0]);
    } else {
        int off = 16;
#pragma unroll
        for (int m = N / 2; m >= 1; m >>= 1, off >>= 1) {
            const bool up = lane & off;
#pragma unroll
            for (int i = 0; i < m; ++i) {
                const float keep = up ? s[i + m] : s[i], send = up ? s[i] : s[i + m];
                s[i] = keep + __shfl_xor_sync(0xffffffffu, send, off);
            }
        }
        t = s[0];
#pragma unroll
        for (; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    }
    constexpr int EACH = 32 / N;  // lanes of a sum
    if constexpr (ONE) {
        if constexpr (N == 1) s[0] = t;
        else
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = __shfl_sync(0xffffffffu, t, i * EACH);
        return;
    }
    const int warp = threadIdx.x >> 5, team = warp / warps;
    float *mine = sh + side * (16 * N);
    side ^= 1;
    if (lane % EACH == 0) mine[warp * N + lane / EACH] = t;
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.0f;
    const float *q = mine + team * warps * N;
    for (int w = 0; w < warps; ++w, q += N) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(q + i);
                s[i] += f.x; s[i + 1] += f.y; s[i + 2] += f.z; s[i + 3] += f.w;
            }
        } else if constexpr (N == 2) {
            const float2 f = *reinterpret_cast<const float2 *>(q);
            s[0] += f.x; s[1] += f.y;
        } else {
            s[0] += *q;
        }
    }
}

// Where a thread's vectors lie. Everything that a row or a stage further on needs is an addition.
template <typename T, int V> struct Places {
    int64_t first;        // bytes: row 0 of the team, the thread's first vector
    int64_t row_bytes;
    int32_t v_bytes;      // between the thread's vectors of a row
    bool in[V];           // which of them there are
    __device__ __forceinline__ Places(int32_t d, int lane, int threads) {
        const int32_t pieces = d / Vec<T>::N;
        first = 16 * (int64_t)lane;
        row_bytes = (int64_t)d * sizeof(T);
        v_bytes = 16 * threads;
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = lane + v * threads < pieces;
    }
};
template <typename T, int V> __device__ __forceinline__ void load_weights(const float *p, int lane, int threads, const Places<T, V> &at, float2 (&w)[V][Vec<T>::N / 2]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int i = 0; i < Vec<T>::N / 2; ++i) w[v][i] = both(0.0f);
        if (p && at.in[v]) load_floats(p + (int64_t)(lane + v * threads) * Vec<T>::N, w[v]);
    }
}

// ONE: a row is one warp's
template <typename T, int V, int K, int THREADS, int BLOCKS, bool ONE>
__global__ void __launch_bounds__(THREADS, BLOCKS) layer_norm_kernel(const LayerNormArgs a, int warps) {
    constexpr int N = Vec<T>::N, P = N / 2;
    extern __shared__ uint4 ring[];  // [stage][row of K][vector of V][thread of THREADS]
    __shared__ __align__(16) float sh[2 * 16 * K];
    int side = 0;
    const int threads = ONE ? 32 : warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads;
    const float by = 1.0f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * teams * K;
    int64_t row = ((int64_t)blockIdx.x * teams + threadIdx.x / threads) * K;
    const Places<T, V> at(a.d, lane, threads);
    wait_previous_kernel();  // (the weights too may be what the launch before writes: an optimiser's)
    const char *from = static_cast<const char *>(a.x) + at.first + row * at.row_bytes;
    char *to = static_cast<char *>(a.xn) + at.first + row * at.row_bytes;
    const int64_t step_bytes = step * at.row_bytes;
    int64_t ahead = row;  // the rows that are fetched next
    auto fetch = [&](int stage) {
        if (ahead < a.T) {
            const char *p = from;
#pragma unroll
            for (int k = 0; k < K; ++k, p += at.row_bytes)
                if (k == 0 || ahead + k < a.T)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (at.in[v]) copy16(ring + ((stage * K + k) * V + v) * THREADS + threadIdx.x, p + v * at.v_bytes);
        }
        copies_commit();
        from += step_bytes;
        ahead += step;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(s);
    float2 w[V][P], b[V][P];  // on their way together with the first rows
    load_weights<T, V>(a.w, lane, threads, at, w);
    load_weights<T, V>(a.b, lane, threads, at, b);
    int stage = 0;
    for (; row < a.T; row += step, to += step_bytes) {
        fetch(stage == 0 ? STAGES - 1 : stage - 1);
        copies_wait<STAGES - 1>();
        float2 x[K][V][P];
        float s[K], mean[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float2 sum = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Vec<T> raw;
                raw.raw = make_uint4(0u, 0u, 0u, 0u);
                if (at.in[v] && (k == 0 || row + k < a.T)) raw.raw = ring[((stage * K + k) * V + v) * THREADS + threadIdx.x];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    x[k][v][i] = raw.get(2 * i);
                    sum = add2(x[k][v][i], sum);
                }
            }
            s[k] = sum.x + sum.y;
        }
        sums_of_team<K, ONE>(s, warps, sh, side);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            mean[k] = s[k] * by;
            float2 sum = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    x[k][v][i] = add2(x[k][v][i], both(-mean[k]));
                    if (!at.in[v]) x[k][v][i] = both(0.0f);
                    sum = fma2(x[k][v][i], x[k][v][i], sum);
                }
            s[k] = sum.x + sum.y;
        }
        sums_of_team<K, ONE>(s, warps, sh, side);
        char *out = to;
#pragma unroll
        for (int k = 0; k < K; ++k, out += at.row_bytes) {
            if (k > 0 && row + k >= a.T) break;
            const float r = 1.0f / sqrtf(s[k] * by + a.eps);
            if (lane == 0) {
                if (a.mean) a.mean[row + k] = mean[k];
                if (a.rstd) a.rstd[row + k] = r;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!at.in[v]) break;
                Vec<T> o;
#pragma unroll
                for (int i = 0; i < P; ++i) o.set(2 * i, fma2(mul2(x[k][v][i], both(r)), w[v][i], b[v][i]));
                *reinterpret_cast<uint4 *>(out + v * at.v_bytes) = o.raw;
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
}

// Backward. Every thread adds up dxn n and dxn of its columns; at the end the block's teams are added up and its sums written. HELD: weights in registers; else, in the widest rows, read
// when they are wanted.
template <typename T, int V, int K, int THREADS, int BLOCKS, int S, bool ONE, bool RES, bool HELD>
__global__ void __launch_bounds__(THREADS, BLOCKS) layer_norm_grads_kernel(const LayerNormGradArgs a, int warps) {
    constexpr int N = Vec<T>::N, P = N / 2, TENSORS = RES ? 3 : 2;
    extern __shared__ uint4 ring[];  // [stage][tensor: x, dxn, dres][row of K][vector of V][thread of THREADS]
    __shared__ __align__(16) float sh[2 * 16 * 2 * K];
    int side = 0;
    const int threads = ONE ? 32 : warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads, team = threadIdx.x / threads;
    const float by = -1.0f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * teams * K;
    int64_t row = ((int64_t)blockIdx.x * teams + team) * K;
    const Places<T, V> at(a.d, lane, threads);
    wait_previous_kernel();
    float2 held[HELD ? V : 1][P];
    auto weights = [&](int v, float2 (&w)[P]) {
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = held[v][i];
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = both(0.0f);
            if (at.in[v]) load_floats(a.w + (int64_t)(lane + v * threads) * N, w);
        }
    };
    const int64_t offset = at.first + row * at.row_bytes, step_bytes = step * at.row_bytes;
    const char *x_from = static_cast<const char *>(a.x) + offset, *g_from = static_cast<const char *>(a.dxn) + offset, *res_from = static_cast<const char *>(a.dres) + offset;
    char *to = static_cast<char *>(a.dX) + offset;
    int64_t ahead = row;
    auto place = [&](int stage, int tensor, int k, int v) { return ring + (((stage * TENSORS + tensor) * K + k) * V + v) * THREADS + threadIdx.x; };
    auto fetch = [&](int stage) {
        if (ahead < a.T) {
            int64_t p = 0;
#pragma unroll
            for (int k = 0; k < K; ++k, p += at.row_bytes)
                if (k == 0 || ahead + k < a.T)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (at.in[v]) {
                            copy16(place(stage, 0, k, v), x_from + p + v * at.v_bytes);
                            copy16(place(stage, 1, k, v), g_from + p + v * at.v_bytes);
                            if constexpr (RES) copy16(place(stage, 2, k, v), res_from + p + v * at.v_bytes);
                        }
        }
        copies_commit();
        x_from += step_bytes; g_from += step_bytes; res_from += step_bytes;
        ahead += step;
    };
    float next_mean[K], next_r[K];  // of the rows to come: loaded a turn ahead
    auto statistics = [&](int64_t first) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            next_mean[k] = first + k < a.T ? a.mean[first + k] : 0.0f;
            next_r[k] = first + k < a.T ? a.rstd[first + k] : 0.0f;
        }
    };
    float2 dw[V][P], db[V][P];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < P; ++i) dw[v][i] = db[v][i] = both(0.0f);
#pragma unroll
    for (int i = 0; i < S; ++i) fetch(i);
    if constexpr (HELD) load_weights<T, V>(a.w, lane, threads, at, held);
    statistics(row);
    int stage = 0;
    for (; row < a.T; row += step, to += step_bytes) {
        float r[K], s[2 * K], off[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            r[k] = next_r[k];
            off[k] = -next_mean[k];
        }
        statistics(row + step);
        copies_wait<S - 1>();
        Vec<T> g[K][V];
        float2 n[K][V][P];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float2 first = both(0.0f), second = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Vec<T> x;
                x.raw = g[k][v].raw = make_uint4(0u, 0u, 0u, 0u);
                if (at.in[v] && (k == 0 || row + k < a.T)) {
                    x.raw = *place(stage, 0, k, v);
                    g[k][v].raw = *place(stage, 1, k, v);
                }
                float2 w[P];
                weights(v, w);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    n[k][v][i] = mul2(add2(x.get(2 * i), both(off[k])), both(r[k]));  // (x r - mean r loses what the mean is larger than the spread)
                    const float2 d = g[k][v].get(2 * i), u = mul2(d, w[i]);
                    first = add2(u, first);
                    second = fma2(u, n[k][v][i], second);
                    dw[v][i] = fma2(d, n[k][v][i], dw[v][i]);
                    db[v][i] = add2(d, db[v][i]);
                }
            }
            s[2 * k] = first.x + first.y;
            s[2 * k + 1] = second.x + second.y;
        }
        sums_of_team<2 * K, ONE>(s, warps, sh, side);
        char *out = to;
#pragma unroll
        for (int k = 0; k < K; ++k, out += at.row_bytes) {
            if (k > 0 && row + k >= a.T) break;
            const float m1 = s[2 * k] * by, m2 = s[2 * k + 1] * by;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!at.in[v]) break;
                float2 w[P];
                weights(v, w);
                Vec<T> res, o;
                if constexpr (RES) res.raw = *place(stage, 2, k, v);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 t = fma2(n[k][v][i], both(m2), fma2(g[k][v].get(2 * i), w[i], both(m1)));
                    if constexpr (RES) o.set(2 * i, fma2(t, both(r[k]), res.get(2 * i)));
                    else o.set(2 * i, mul2(t, both(r[k])));
                }
                *reinterpret_cast<uint4 *>(out + v * at.v_bytes) = o.raw;
            }
        }
        fetch(stage);  // each thread has read its own places
        stage = stage + 1 == S ? 0 : stage + 1;
    }
    // Sums of the block, team behind team through the ring, which has room for 2 d floats
    copies_wait<0>();
    float *all = reinterpret_cast<float *>(ring);
    for (int turn = 0; turn < teams; ++turn) {
        __syncthreads();
        if (team != turn) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!at.in[v]) break;
            float2 *to_w = reinterpret_cast<float2 *>(all + (int64_t)(lane + v * threads) * N), *to_b = reinterpret_cast<float2 *>(all + a.d + (int64_t)(lane + v * threads) * N);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                to_w[i] = turn ? add2(to_w[i], dw[v][i]) : dw[v][i];
                to_b[i] = turn ? add2(to_b[i], db[v][i]) : db[v][i];
            }
        }
    }
    __syncthreads();
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.d;
    for (int i = threadIdx.x; i < a.d / 2; i += blockDim.x) reinterpret_cast<float4 *>(part)[i] = reinterpret_cast<const float4 *>(all)[i];
}

// dw and db from the blocks' sums: 32 columns a block, a warp every 32nd part, its loads (ten at most) together
constexpr int COLUMN_WARPS = 32;
__global__ void __launch_bounds__(COLUMN_WARPS * 32) layer_norm_columns_kernel(const float *part, int32_t parts, int32_t d, float *dw, float *db) {
    wait_previous_kernel();
    __shared__ double sh[COLUMN_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t col = blockIdx.x * 32 + lane;
    double s = 0.0;
    if (col < 2 * d)
#pragma unroll 10
        for (int32_t p = warp; p < parts; p += COLUMN_WARPS) s += (double)part[(int64_t)p * 2 * d + col];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || col >= 2 * d) return;
#pragma unroll
    for (int q = 1; q < COLUMN_WARPS; ++q) s += sh[q][lane];
    if (col < d) dw[col] = (float)s;
    else if (db) db[col - d] = (float)s;
}

// A row's vectors: V of them in each thread of a team of up to 16 warps. As many a thread as there are registers for (no sums between warps for rows of up to 128 vectors), fewer
// where that leaves more than a fifth of a team's threads without work. (A tenth: 4681 x 1792 forward 11.4 us instead of 8.9, 3744 x 2240 16.0 instead of 10.3; backward of 6553 x 1280 17.8, not 19.9.)
struct Team { int V, warps, threads; };
Team team_of(int32_t d, int32_t act, int most) {
    const int64_t pieces = (int64_t)d * (int64_t)act_bytes(act) / 16;
    Team best = {0, 0, 0};
    double share = 0.0;
    for (int V = most; V >= 1; V /= 2) {
        const int64_t warps = cdiv(pieces, 32 * V);
        const double s = (double)pieces / (double)(32 * V * warps);
        if (warps > 16 || s <= share) continue;
        best = {V, (int)warps, (int)(32 * warps * (warps <= 8 ? 8 / warps : 1))};
        share = s;
        if (s >= 0.8) break;
    }
    return best;
}
Team forward_team(int32_t d, int32_t act) { return team_of(d, act, (int64_t)d * (int64_t)act_bytes(act) / 16 > 2048 ? 8 : 4); }
Team backward_team(int32_t d, int32_t act) {  // 16 elements of a row a thread, whose sums of columns take 32 registers; the widest rows have 32
    const int64_t pieces = (int64_t)d * (int64_t)act_bytes(act) / 16;
    const int most = act == MOE_BF16 ? 2 : 4;
    return team_of(d, act, pieces > 512 * most ? 2 * most : most);
}
// Rows of a team at a time: two vectors of a row and its gradient are what fits beside the sums of columns (bf16 backward of 65536 x 1024 with two rows of two: 121 us, with one 86)
constexpr int rows_at_once(int V, bool backward) { return backward ? (V == 1 ? 2 : 1) : V >= 4 ? 1 : 4 / V; }
// 512 threads an SM: two blocks, three of teams of five warps (7234 x 1160 forward with two 14.5 us, with three 11.6; backward 21.9 and 19.4), one of teams of more than eight.
// Backward of four vectors a thread: two, whose rings of 96 KiB an SM holds
int64_t blocks_of(int64_t T, const Team &t, bool backward) {
    return imin(cdiv(T, (int64_t)rows_at_once(t.V, backward) * (t.threads / (32 * t.warps))), 148 * imin(512 / t.threads, backward && t.V > 2 ? 2 : 3));
}

template <typename T, int V, int THREADS, bool ONE> int32_t forward(const LayerNormArgs &a, const Team &t, cudaStream_t st) {
    constexpr int K = rows_at_once(V, false), BYTES = STAGES * K * V * THREADS * 16;
    constexpr auto kernel = layer_norm_kernel<T, V, K, THREADS, 512 / THREADS, ONE>;
    static PerDevice allowed;
    if (!allow_shared(allowed, kernel, BYTES)) return MOE_ERR_CUDA;
    launch_kernel(kernel, dim3((unsigned)blocks_of(a.T, t, false)), dim3(t.threads), BYTES, st, a, t.warps);
    MOE_LAUNCHED();
    return MOE_OK;
}
int32_t columns(const LayerNormGradArgs &a, int32_t blocks, cudaStream_t st) {
    launch_kernel(layer_norm_columns_kernel, dim3((unsigned)cdiv(2 * a.d, 32)), dim3(COLUMN_WARPS * 32), 0, st, (const float *)a.part, blocks, a.d, a.dw, a.db);
    MOE_LAUNCHED();
    return MOE_OK;
}
template <typename T, int V, int THREADS, bool ONE, bool RES> int32_t backward(const LayerNormGradArgs &a, const Team &t, cudaStream_t st) {
    constexpr int K = rows_at_once(V, true), S = V == 8 ? 1 : STAGES, BYTES = S * (RES ? 3 : 2) * K * V * THREADS * 16;
    constexpr auto kernel = layer_norm_grads_kernel<T, V, K, THREADS, 512 / THREADS, S, ONE, RES, V * Vec<T>::N <= 16>;
    static PerDevice allowed;
    if (!allow_shared(allowed, kernel, BYTES)) return MOE_ERR_CUDA;
    const int64_t blocks = blocks_of(a.T, t, true);
    launch_kernel(kernel, dim3((unsigned)blocks), dim3(t.threads), BYTES, st, a, t.warps);
    MOE_LAUNCHED();
    return columns(a, (int32_t)blocks, st);
}
template <typename T, int V> int32_t forward_of(const LayerNormArgs &a, const Team &t, cudaStream_t st) {
    if (t.warps == 1) return forward<T, V, 256, true>(a, t, st);
    return t.threads <= 256 ? forward<T, V, 256, false>(a, t, st) : forward<T, V, 512, false>(a, t, st);
}
template <typename T, int V, bool RES> int32_t backward_of(const LayerNormGradArgs &a, const Team &t, cudaStream_t st) {
    if (t.warps == 1) return backward<T, V, 256, true, RES>(a, t, st);
    return t.threads <= 256 ? backward<T, V, 256, false, RES>(a, t, st) : backward<T, V, 512, false, RES>(a, t, st);
}
template <typename T> int32_t forward_any(const LayerNormArgs &a, const Team &t, cudaStream_t st) {
    if (t.V == 1) return forward_of<T, 1>(a, t, st);
    if (t.V == 2) return forward_of<T, 2>(a, t, st);
    if (t.V == 4) return forward_of<T, 4>(a, t, st);
    if constexpr (sizeof(T) == 4) return forward<T, 8, 512, false>(a, t, st);
    return MOE_ERR_UNSUPPORTED;  // (no such row: MOE_NORM_MAX_D)
}
template <typename T, bool RES> int32_t backward_any(const LayerNormGradArgs &a, const Team &t, cudaStream_t st) {
    if (t.V == 1) return backward_of<T, 1, RES>(a, t, st);
    if (t.V == 2) return backward_of<T, 2, RES>(a, t, st);
    if (t.V == 4) {
        if constexpr (sizeof(T) == 4) return backward_of<T, 4, RES>(a, t, st);
        return backward<T, 4, 512, false, RES>(a, t, st);
    }
    if constexpr (sizeof(T) == 4) return backward<T, 8, 512, false, RES>(a, t, st);
    return MOE_ERR_UNSUPPORTED;
}

}  // namespace

int64_t layer_norm_grad_floats(int64_t T, int32_t d, int32_t act) { return 2 * (int64_t)d * imax(1, blocks_of(T, backward_team(d, act), true)); }

int32_t launch_layer_norm(const LayerNormArgs &a, cudaStream_t st) {
    if (a.T == 0) return MOE_OK;
    const Team t = forward_team(a.d, a.act);
    return a.act == MOE_BF16 ? forward_any<bf16>(a, t, st) : forward_any<float>(a, t, st);
}

int32_t launch_layer_norm_grads(const LayerNormGradArgs &a, cudaStream_t st) {
    if (a.T == 0) return columns(a, 0, st);  // sums of nothing
    const Team t = backward_team(a.d, a.act);
    if (a.act == MOE_BF16) return a.dres ? backward_any<bf16, true>(a, t, st) : backward_any<bf16, false>(a, t, st);
    return a.dres ? backward_any<float, true>(a, t, st) : backward_any<float, false>(a, t, st);
}

}  // namespace moe
