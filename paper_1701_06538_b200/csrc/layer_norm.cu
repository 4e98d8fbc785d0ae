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

constexpr int FORWARD_STAGES = 3;  // rows of a team on their way or in work

// N sums over the threads of a team at once: in the first steps lanes give away half of their sums, so that eight sums take nine exchanges and not forty. Lane l is left with
// sum l / (32 / N). `sh` has a place per warp and sum, twice: who writes the next sums does so on the other side, and the barrier of those keeps it from coming round.
template <int N> __device__ __forceinline__ void sums_of_team(float (&s)[N], int warps, float *sh, int &side) {
    const int lane = threadIdx.x & 31;
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
    float t = s[0];
#pragma unroll
    for (; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    constexpr int EACH = 32 / N;  // lanes of a sum
    if (warps == 1) {
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
    for (int q = team * warps; q < (team + 1) * warps; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += mine[q * N + i];
}

// The weights of a thread's columns: in registers, or where a thread has more than two vectors of each row read when they are wanted
template <typename T, int V> struct Weights {
    static constexpr int P = Vec<T>::N / 2;
    static constexpr bool HELD = V <= 2;
    const float *at;
    float2 held[HELD ? V : 1][P];
    __device__ __forceinline__ Weights(const float *p, int first, int step, int pieces) : at(p) {
        if constexpr (HELD)
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int i = 0; i < P; ++i) held[v][i] = both(0.0f);
                if (p && first + v * step < pieces) load_floats<P>(p + (int64_t)(first + v * step) * Vec<T>::N, held[v]);
            }
    }
    __device__ __forceinline__ void get(int v, int q, float2 (&w)[P]) const {  // of vector q, the thread's v-th
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = held[v][i];
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = both(0.0f);
            if (at) load_floats<P>(at + (int64_t)q * Vec<T>::N, w);
        }
    }
};

template <typename T, int V, int K, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS) layer_norm_kernel(const LayerNormArgs a, int warps) {
    constexpr int N = Vec<T>::N, P = N / 2;
    extern __shared__ uint4 ring[];  // [stage][row of K][vector of V][thread]
    __shared__ float sh[2 * 16 * K];
    int side = 0;
    const int threads = warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads, wide = blockDim.x;
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * teams * K;
    int64_t row = ((int64_t)blockIdx.x * teams + threadIdx.x / threads) * K;
    const Weights<T, V> w(a.w, lane, threads, pieces), b(a.b, lane, threads, pieces);
    wait_previous_kernel();
    auto place = [&](int stage, int k, int v) { return ring + ((stage * K + k) * V + v) * wide + threadIdx.x; };
    auto fetch = [&](int stage, int64_t first) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (first + k < a.T && lane + v * threads < pieces)
                    copy16(place(stage, k, v), static_cast<const T *>(a.x) + (first + k) * a.d + (int64_t)(lane + v * threads) * N);
        copies_commit();
    };
#pragma unroll
    for (int s = 0; s < FORWARD_STAGES - 1; ++s) fetch(s, row + s * step);
    int stage = 0;
    for (; row < a.T; row += step) {
        fetch(stage == 0 ? FORWARD_STAGES - 1 : stage - 1, row + (FORWARD_STAGES - 1) * step);
        copies_wait<FORWARD_STAGES - 1>();
        Vec<T> x[K][V];
        float s[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float2 sum = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[k][v].raw = make_uint4(0u, 0u, 0u, 0u);
                if (lane + v * threads < pieces && row + k < a.T) x[k][v].raw = *place(stage, k, v);
#pragma unroll
                for (int i = 0; i < P; ++i) sum = fma2(x[k][v].get(2 * i), both(1.0f), sum);
            }
            s[k] = sum.x + sum.y;
        }
        sums_of_team<K>(s, warps, sh, side);
        float mean[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            mean[k] = s[k] * by;
            float2 sum = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane + v * threads < pieces)
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const float2 off = fma2(x[k][v].get(2 * i), both(1.0f), both(-mean[k]));
                        sum = fma2(off, off, sum);
                    }
            s[k] = sum.x + sum.y;
        }
        sums_of_team<K>(s, warps, sh, side);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (row + k >= a.T) break;
            const float r = 1.0f / sqrtf(s[k] * by + a.eps);
            if (lane == 0) {
                if (a.mean) a.mean[row + k] = mean[k];
                if (a.rstd) a.rstd[row + k] = r;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int q = lane + v * threads;
                if (q >= pieces) break;
                float2 wv[P], bv[P];
                w.get(v, q, wv);
                b.get(v, q, bv);
                Vec<T> o;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 off = fma2(x[k][v].get(2 * i), both(1.0f), both(-mean[k]));
                    o.set(2 * i, fma2(mul2(off, both(r)), wv[i], bv[i]));
                }
                store_vec<T>(a.xn, row + k, a.d, q, o);
            }
        }
        stage = stage + 1 == FORWARD_STAGES ? 0 : stage + 1;
    }
}

// Backward. Every thread adds up dxn n and dxn of its columns; at the end the block's teams are added up and its sums written.
template <typename T, int V, int K, int THREADS, int BLOCKS, int STAGES>
__global__ void __launch_bounds__(THREADS, BLOCKS) layer_norm_grads_kernel(const LayerNormGradArgs a, int warps) {
    constexpr int N = Vec<T>::N, P = N / 2;
    extern __shared__ uint4 ring[];  // [stage][tensor: x, dxn, dres][row of K][vector of V][thread]
    __shared__ float sh[2 * 16 * 2 * K];
    int side = 0;
    const int threads = warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads, wide = blockDim.x, team = threadIdx.x / threads;
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    const int64_t step = (int64_t)gridDim.x * teams * K;
    int64_t row = ((int64_t)blockIdx.x * teams + team) * K;
    const int tensors = a.dres ? 3 : 2;
    const Weights<T, V> w(a.w, lane, threads, pieces);
    wait_previous_kernel();
    auto place = [&](int stage, int tensor, int k, int v) { return ring + (((stage * tensors + tensor) * K + k) * V + v) * wide + threadIdx.x; };
    auto fetch = [&](int stage, int64_t first) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (first + k < a.T && lane + v * threads < pieces) {
                    const int64_t at = (first + k) * a.d + (int64_t)(lane + v * threads) * N;
                    copy16(place(stage, 0, k, v), static_cast<const T *>(a.x) + at);
                    copy16(place(stage, 1, k, v), static_cast<const T *>(a.dxn) + at);
                    if (tensors == 3) copy16(place(stage, 2, k, v), static_cast<const T *>(a.dres) + at);
                }
        copies_commit();
    };
    float2 dw[V][P], db[V][P];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < P; ++i) dw[v][i] = db[v][i] = both(0.0f);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) fetch(s, row + s * step);
    int stage = 0;
    for (; row < a.T; row += step) {
        float off[K], r[K], s[2 * K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            r[k] = row + k < a.T ? a.rstd[row + k] : 0.0f;
            off[k] = row + k < a.T ? -a.mean[row + k] * r[k] : 0.0f;
        }
        copies_wait<STAGES - 1>();
        Vec<T> x[K][V], g[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float2 first = both(0.0f), second = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[k][v].raw = g[k][v].raw = make_uint4(0u, 0u, 0u, 0u);
                const int q = lane + v * threads;
                if (q < pieces && row + k < a.T) {
                    x[k][v].raw = *place(stage, 0, k, v);
                    g[k][v].raw = *place(stage, 1, k, v);
                }
                float2 wv[P];
                if (Weights<T, V>::HELD || q < pieces) w.get(v, q, wv);
                else
#pragma unroll
                    for (int i = 0; i < P; ++i) wv[i] = both(0.0f);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 n = fma2(x[k][v].get(2 * i), both(r[k]), both(off[k])), d = g[k][v].get(2 * i), u = mul2(d, wv[i]);
                    first = fma2(u, both(1.0f), first);
                    second = fma2(u, n, second);
                    dw[v][i] = fma2(d, n, dw[v][i]);
                    db[v][i] = fma2(d, both(1.0f), db[v][i]);
                }
            }
            s[2 * k] = first.x + first.y;
            s[2 * k + 1] = second.x + second.y;
        }
        sums_of_team<2 * K>(s, warps, sh, side);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (row + k >= a.T) break;
            const float m1 = -s[2 * k] * by, m2 = -s[2 * k + 1] * by;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int q = lane + v * threads;
                if (q >= pieces) break;
                float2 wv[P];
                w.get(v, q, wv);
                Vec<T> res, o;
                if (tensors == 3) res.raw = *place(stage, 2, k, v);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 n = fma2(x[k][v].get(2 * i), both(r[k]), both(off[k]));
                    const float2 t = fma2(n, both(m2), fma2(g[k][v].get(2 * i), wv[i], both(m1)));
                    o.set(2 * i, tensors == 3 ? fma2(t, both(r[k]), res.get(2 * i)) : mul2(t, both(r[k])));
                }
                store_vec<T>(a.dX, row + k, a.d, q, o);
            }
        }
        fetch(stage, row + STAGES * step);  // each thread has read its own places
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    // Sums of the block: team behind team through the ring, which takes 2 d floats (4 bytes a column for every 32 of a row's 2-byte elements in it)
    copies_wait<0>();
    float *all = reinterpret_cast<float *>(ring);
    for (int turn = 0; turn < teams; ++turn) {
        __syncthreads();
        if (team != turn) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int q = lane + v * threads;
            if (q >= pieces) break;
            float2 *to = reinterpret_cast<float2 *>(all + (int64_t)q * N), *to_b = reinterpret_cast<float2 *>(all + a.d + (int64_t)q * N);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                to[i] = turn ? fma2(to[i], both(1.0f), dw[v][i]) : dw[v][i];
                to_b[i] = turn ? fma2(to_b[i], both(1.0f), db[v][i]) : db[v][i];
            }
        }
    }
    __syncthreads();
    float *part = a.part + (int64_t)blockIdx.x * 2 * a.d;
    for (int i = threadIdx.x; i < a.d / 2; i += blockDim.x) reinterpret_cast<float4 *>(part)[i] = reinterpret_cast<const float4 *>(all)[i];
}

// dw and db from the blocks' sums: 32 columns a block, a warp every sixteenth part
constexpr int COLUMN_WARPS = 16;
__global__ void __launch_bounds__(COLUMN_WARPS * 32) layer_norm_columns_kernel(const float *part, int32_t parts, int32_t d, float *dw, float *db) {
    wait_previous_kernel();
    __shared__ double sh[COLUMN_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t col = blockIdx.x * 32 + lane;
    double s = 0.0;
    if (col < 2 * d)
#pragma unroll 8
        for (int32_t p = warp; p < parts; p += COLUMN_WARPS) s += (double)part[(int64_t)p * 2 * d + col];
    sh[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || col >= 2 * d) return;
#pragma unroll
    for (int q = 1; q < COLUMN_WARPS; ++q) s += sh[q][lane];
    if (col < d) dw[col] = (float)s;
    else if (db) db[col - d] = (float)s;
}

// Vectors of a row in each thread of a team of up to 16 warps
struct Team { int V, K, warps, threads; };
Team team_of(int32_t d, int32_t act) {
    const int64_t pieces = (int64_t)d * (int64_t)act_bytes(act) / 16;
    Team t;
    t.V = pieces <= 256 ? 1 : pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8;
    t.K = t.V == 1 ? 4 : t.V == 2 ? 2 : 1;
    t.warps = (int)cdiv(pieces, 32 * t.V);
    t.threads = 32 * t.warps * (t.warps <= 8 ? 8 / t.warps : 1);
    return t;
}
// Blocks that an SM holds: of 256 threads four, or two with the backward pass's sums; of 512 threads one
int per_sm(const Team &t, bool backward) { return t.threads > 256 ? 1 : backward ? 2 : 4; }
int64_t blocks_of(int64_t T, const Team &t, bool backward) {
    return imin(cdiv(T, (int64_t)t.K * (t.threads / (32 * t.warps))), (int64_t)per_sm(t, backward) * 148);
}

template <typename T, int V, int K, int THREADS, int BLOCKS> int32_t forward(const LayerNormArgs &a, const Team &t, cudaStream_t st) {
    static PerDevice allowed;
    const int bytes = FORWARD_STAGES * K * V * t.threads * 16;
    if (!allow_shared(allowed, layer_norm_kernel<T, V, K, THREADS, BLOCKS>, FORWARD_STAGES * K * V * THREADS * 16)) return MOE_ERR_CUDA;
    launch_kernel(layer_norm_kernel<T, V, K, THREADS, BLOCKS>, dim3((unsigned)blocks_of(a.T, t, false)), dim3(t.threads), bytes, st, a, t.warps);
    MOE_LAUNCHED();
    return MOE_OK;
}
int32_t columns(const LayerNormGradArgs &a, int32_t blocks, cudaStream_t st) {
    launch_kernel(layer_norm_columns_kernel, dim3((unsigned)cdiv(2 * a.d, 32)), dim3(COLUMN_WARPS * 32), 0, st, (const float *)a.part, blocks, a.d, a.dw, a.db);
    MOE_LAUNCHED();
    return MOE_OK;
}
template <typename T, int V, int K, int THREADS, int BLOCKS, int STAGES> int32_t backward(const LayerNormGradArgs &a, const Team &t, cudaStream_t st) {
    static PerDevice allowed;
    const int bytes = STAGES * 3 * K * V * 16;  // a thread
    if (!allow_shared(allowed, layer_norm_grads_kernel<T, V, K, THREADS, BLOCKS, STAGES>, bytes * THREADS)) return MOE_ERR_CUDA;
    const int64_t blocks = blocks_of(a.T, t, true);
    launch_kernel(layer_norm_grads_kernel<T, V, K, THREADS, BLOCKS, STAGES>, dim3((unsigned)blocks), dim3(t.threads), (size_t)bytes * t.threads, st, a, t.warps);
    MOE_LAUNCHED();
    return columns(a, (int32_t)blocks, st);
}
template <typename T> int32_t forward_of(const LayerNormArgs &a, const Team &t, cudaStream_t st) {
    if (t.V == 1) return forward<T, 1, 4, 256, 4>(a, t, st);
    if (t.V == 2) return t.threads <= 256 ? forward<T, 2, 2, 256, 4>(a, t, st) : forward<T, 2, 2, 512, 1>(a, t, st);
    if (t.V == 4) return forward<T, 4, 1, 512, 1>(a, t, st);
    if constexpr (sizeof(T) == 4) return forward<T, 8, 1, 512, 1>(a, t, st);
    return MOE_ERR_UNSUPPORTED;  // (no such row: MOE_NORM_MAX_D)
}
template <typename T> int32_t backward_of(const LayerNormGradArgs &a, const Team &t, cudaStream_t st) {
    if (t.V == 1) return backward<T, 1, 4, 256, 2, 2>(a, t, st);
    if (t.V == 2) return t.threads <= 256 ? backward<T, 2, 2, 256, 2, 2>(a, t, st) : backward<T, 2, 2, 512, 1, 2>(a, t, st);
    if (t.V == 4) return backward<T, 4, 1, 512, 1, 2>(a, t, st);
    if constexpr (sizeof(T) == 4) return backward<T, 8, 1, 512, 1, 1>(a, t, st);
    return MOE_ERR_UNSUPPORTED;
}

}  // namespace

int64_t layer_norm_grad_floats(int64_t T, int32_t d, int32_t act) {
    return 2 * (int64_t)d * imax(1, blocks_of(T, team_of(d, act), true));
}

int32_t launch_layer_norm(const LayerNormArgs &a, cudaStream_t st) {
    if (a.T == 0) return MOE_OK;
    const Team t = team_of(a.d, a.act);
    return a.act == MOE_BF16 ? forward_of<bf16>(a, t, st) : forward_of<float>(a, t, st);
}

int32_t launch_layer_norm_grads(const LayerNormGradArgs &a, cudaStream_t st) {
    const Team t = team_of(a.d, a.act);
    if (a.T == 0) return columns(a, 0, st);  // sums of nothing
    return a.act == MOE_BF16 ? backward_of<bf16>(a, t, st) : backward_of<float>(a, t, st);
}

}  // namespace moe
