// The Muon step (Jordan et al., 2024) over a list of batches of matrices: momentum, the update orthogonalised by Newton-Schulz products, weights. For every matrix
//   m = momentum m + g,   u = g + momentum m  (or m),   X = u / (|u| + eps)  over its Frobenius norm,   then newton_schulz.cu
// Here: the two passes before the products, both bound by memory. The first makes m and the sums of u's squares, the second X, which needs the whole matrix' norm. u is made of the
// momentum as it is held, so that the second pass makes the same one again.
#include <float.h>
#include <math_constants.h>

#include <vector>

#include "muon.cuh"
#include "pairs.cuh"
#include "tc.cuh"
#include "vectors.cuh"

namespace moe {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, EACH = 8, TURNS = 4;
constexpr int CHUNK = THREADS * EACH * TURNS;  // elements of a block
constexpr int64_t MOST_X = (int64_t)1 << 30;   // bytes of X of a launch (one matrix at least)

struct Passes {
    double *part;     // [matrices][chunks] sums of squares
    __half *x;
    int32_t *done;    // [matrices]
    int32_t *next, *status;
    int32_t chunks, clear_status, nesterov;
    float momentum, eps, grad_scale;
    const moe_muon_rates *rates;
};

// Eight elements from p + at, or those of them that there are
template <typename T, bool VECTORS> __device__ __forceinline__ void load8(const T *p, int64_t at, int64_t live, float (&v)[EACH]) {
    if constexpr (VECTORS) {
        constexpr int N = Vec<T>::N;
#pragma unroll
        for (int i = 0; i < EACH / N; ++i) {
            Vec<T> q;
            q.raw = *reinterpret_cast<const uint4 *>(p + at + i * N);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 f = q.get(j);
                v[i * N + j] = f.x;
                v[i * N + j + 1] = f.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] = i < live ? to_f32(p[at + i]) : 0.0f;
    }
}
template <typename T, bool VECTORS> __device__ __forceinline__ void store8(T *p, int64_t at, int64_t live, const float (&v)[EACH]) {
    if constexpr (VECTORS) {
        constexpr int N = Vec<T>::N;
#pragma unroll
        for (int i = 0; i < EACH / N; ++i) {
            Vec<T> q;
#pragma unroll
            for (int j = 0; j < N; j += 2) q.set(j, make_float2(v[i * N + j], v[i * N + j + 1]));
            *reinterpret_cast<uint4 *>(p + at + i * N) = q.raw;
        }
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < live) p[at + i] = from_f32<T>(v[i]);
    }
}
template <typename T> __device__ __forceinline__ float held(float v) { return to_f32(from_f32<T>(v)); }

__device__ __forceinline__ double sum_of_block(double v, double *sh) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}

// Squares are added up in float over eight elements, then in double
template <typename GT, typename MT, bool VECTORS>
__device__ __forceinline__ double momentum_chunk(const GT *g, MT *m, int64_t at, int64_t end, float grad_scale, const Passes &k) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int64_t here = at + (int64_t)(i * THREADS + threadIdx.x) * EACH, live = end - here;
        if (live <= 0) break;
        float gv[EACH], mv[EACH];
        load8<GT, VECTORS>(g, here, live, gv);
        load8<MT, VECTORS>(m, here, live, mv);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            gv[j] *= grad_scale;
            mv[j] = held<MT>(fmaf(k.momentum, mv[j], gv[j]));
            const float u = k.nesterov ? fmaf(k.momentum, mv[j], gv[j]) : mv[j];
            s = fmaf(u, u, s);
        }
        store8<MT, VECTORS>(m, here, live, mv);
        sum += (double)s;
    }
    return sum;
}
template <bool VECTORS>
__global__ void __launch_bounds__(THREADS) muon_momentum_kernel(const __grid_constant__ MuonBatch b, const Passes k) {
    __shared__ double sh[WARPS];
    wait_previous_kernel();
    const int32_t matrix = blockIdx.x / k.chunks, chunk = blockIdx.x % k.chunks;
    if (threadIdx.x == 0 && chunk == 0) {
        k.done[matrix] = 0;
        if (matrix == 0) {
            *k.next = 0;
            if (k.clear_status) *k.status = 0;
        }
    }
    const int32_t i = b.entry_of(matrix);
    const MuonEntry &t = b.t[i];
    const int64_t each = (int64_t)b.rows * b.cols, first = (matrix - b.first[i]) * each, at = first + (int64_t)chunk * CHUNK, end = min(at + CHUNK, first + each);
    const float grad_scale = k.rates ? k.rates->grad_scale : k.grad_scale;
    double s;
    switch (t.kind & 6) {
        case 0: s = momentum_chunk<float, float, VECTORS>(static_cast<const float *>(t.g), static_cast<float *>(t.m), at, end, grad_scale, k); break;
        case 2: s = momentum_chunk<bf16, float, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<float *>(t.m), at, end, grad_scale, k); break;
        case 4: s = momentum_chunk<float, bf16, VECTORS>(static_cast<const float *>(t.g), static_cast<bf16 *>(t.m), at, end, grad_scale, k); break;
        default: s = momentum_chunk<bf16, bf16, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<bf16 *>(t.m), at, end, grad_scale, k); break;
    }
    s = sum_of_block(s, sh);
    if (threadIdx.x == 0) k.part[blockIdx.x] = s;
}

// X in rows of ld elements, zeros behind the columns: a block has CHUNK of them, a piece of eight a thread at a time
template <typename GT, typename MT, bool VECTORS>
__device__ __forceinline__ void normalise_chunk(const GT *g, const MT *m, int64_t first, __half *x, int64_t begin, int64_t pieces, int32_t cols, int32_t ld, float grad_scale, float by,
                                                const Passes &k) {
    const int32_t in_row = ld / EACH;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int64_t piece = begin + i * THREADS + threadIdx.x;
        if (piece >= pieces) break;
        const int32_t row = (int32_t)((uint32_t)piece / (uint32_t)in_row), col = ((int32_t)piece - row * in_row) * EACH, live = cols - col;
        uint32_t out[EACH / 2] = {0u, 0u, 0u, 0u};
        if (live > 0) {
            const int64_t at = first + (int64_t)row * cols + col;
            float gv[EACH], mv[EACH];
            load8<MT, VECTORS>(m, at, live, mv);
            if (k.nesterov) load8<GT, VECTORS>(g, at, live, gv);
#pragma unroll
            for (int j = 0; j < EACH; j += 2) {
                float u[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) u[q] = (k.nesterov ? fmaf(k.momentum, mv[j + q], gv[j + q] * grad_scale) : mv[j + q]) * by;
                const __half2 h = __floats2half2_rn(u[0], u[1]);
                out[j / 2] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(x + piece * EACH) = make_uint4(out[0], out[1], out[2], out[3]);
    }
}
template <bool VECTORS>
__global__ void __launch_bounds__(THREADS) muon_normalise_kernel(const __grid_constant__ MuonBatch b, const Passes k, int32_t blocks, int32_t ld) {
    __shared__ double sh[WARPS];
    wait_previous_kernel();
    const int32_t matrix = blockIdx.x / blocks, block = blockIdx.x % blocks;
    double s = 0.0;
    for (int32_t c = threadIdx.x; c < k.chunks; c += THREADS) s += k.part[(int64_t)matrix * k.chunks + c];
    s = sqrt(sum_of_block(s, sh)) + (double)k.eps;
    // a matrix whose norm is no finite number becomes NaN as a whole
    const float by = s <= (double)FLT_MAX ? (float)((double)MUON_UNIT / s) : CUDART_NAN_F;
    const int32_t i = b.entry_of(matrix);
    const MuonEntry &t = b.t[i];
    const int64_t first = (int64_t)(matrix - b.first[i]) * b.rows * b.cols, pieces = (int64_t)b.rows * (ld / EACH), begin = (int64_t)block * (CHUNK / EACH);
    __half *x = k.x + (int64_t)matrix * b.rows * ld;
    const float grad_scale = k.rates ? k.rates->grad_scale : k.grad_scale;
    switch (t.kind & 6) {
        case 0: normalise_chunk<float, float, VECTORS>(static_cast<const float *>(t.g), static_cast<const float *>(t.m), first, x, begin, pieces, b.cols, ld, grad_scale, by, k); break;
        case 2: normalise_chunk<bf16, float, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<const float *>(t.m), first, x, begin, pieces, b.cols, ld, grad_scale, by, k); break;
        case 4: normalise_chunk<float, bf16, VECTORS>(static_cast<const float *>(t.g), static_cast<const bf16 *>(t.m), first, x, begin, pieces, b.cols, ld, grad_scale, by, k); break;
        default: normalise_chunk<bf16, bf16, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<const bf16 *>(t.m), first, x, begin, pieces, b.cols, ld, grad_scale, by, k); break;
    }
}

int32_t check_tensor(const moe_muon_tensor &t) {
    if (t.count < 0 || t.count > (int64_t)1 << 24 || t.rows <= 0 || t.cols <= 0 || t.rows > MOE_MUON_MAX_SIDE || t.cols > MOE_MUON_MAX_SIDE) return MOE_ERR_INVALID_ARG;
    for (int32_t type : {t.w_type, t.g_type, t.m_type})
        if (type != MOE_F32 && type != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!(t.weight_decay >= 0.0f) || !(t.weight_decay <= FLT_MAX) || !(fabsf(t.scale) <= FLT_MAX)) return MOE_ERR_INVALID_ARG;
    if (t.count == 0) return MOE_OK;
    const void *all[] = {t.w, t.g, t.m};
    for (const void *p : all)
        if (!p || !aligned16(p)) return MOE_ERR_INVALID_ARG;
    if (t.master && (t.w_type != MOE_BF16 || !aligned16(t.master))) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// What is launched together: matrices of one shape, as many as X has room for
struct Launch {
    MuonBatch batch;
    int64_t matrices() const { return batch.first[batch.n]; }
};
// The tensors in launches, shape by shape as they come first; `run` is given each
template <typename Run> int32_t for_each_launch(const moe_muon_tensor *tensors, int32_t count, Run run) {
    std::vector<char> taken;
    try {
        taken.assign((size_t)count, 0);
    } catch (...) {
        return MOE_ERR_WORKSPACE;
    }
    Launch l;
    for (int32_t i = 0; i < count; ++i) {
        if (taken[i] || tensors[i].count == 0) continue;
        const int32_t rows = tensors[i].rows, cols = tensors[i].cols;
        const int64_t each = (int64_t)rows * cols, most = imin((int64_t)1 << 20, imax(1, MOST_X / ((int64_t)rows * muon_ld(cols) * 2)));
        l.batch.rows = rows; l.batch.cols = cols; l.batch.n = l.batch.first[0] = 0;
        auto flush = [&]() -> int32_t {
            if (l.batch.n == 0) return MOE_OK;
            MOE_TRY(run(l));
            l.batch.n = 0;
            return MOE_OK;
        };
        for (int32_t j = i; j < count; ++j) {
            const moe_muon_tensor &t = tensors[j];
            if (taken[j] || t.count == 0 || t.rows != rows || t.cols != cols) continue;
            taken[j] = 1;
            for (int64_t from = 0; from < t.count;) {
                if (l.batch.n == MUON_MAX_LIST || l.matrices() >= most) MOE_TRY(flush());
                const int64_t here = imin(t.count - from, most - (l.batch.n ? l.matrices() : 0)), at = from * each;
                auto on = [&](const void *p, int32_t type) { return static_cast<char *>(const_cast<void *>(p)) + at * (int64_t)act_bytes(type); };
                MuonEntry &e = l.batch.t[l.batch.n];
                e.w = on(t.w, t.w_type); e.g = on(t.g, t.g_type); e.m = on(t.m, t.m_type);
                e.master = t.master ? t.master + at : nullptr;
                e.scale = t.scale; e.decay = t.weight_decay;
                e.kind = (t.w_type == MOE_BF16 ? 1 : 0) | (t.g_type == MOE_BF16 ? 2 : 0) | (t.m_type == MOE_BF16 ? 4 : 0) | (t.master ? 8 : 0);
                l.batch.first[l.batch.n + 1] = l.batch.first[l.batch.n] + (int32_t)here;
                ++l.batch.n;
                from += here;
            }
        }
        MOE_TRY(flush());
    }
    return MOE_OK;
}
struct Scratch {
    int32_t *done, *next;
    double *part;
    __half *x;
    void *products;
};
Scratch scratch_of(Carver &cv, const Launch &l) {
    const int64_t each = (int64_t)l.batch.rows * l.batch.cols;
    Scratch s;
    s.next = cv.take<int32_t>(1);
    s.done = cv.take<int32_t>(l.matrices());
    s.part = cv.take<double>(l.matrices() * cdiv(each, CHUNK));
    s.x = cv.take<__half>(l.matrices() * l.batch.rows * muon_ld(l.batch.cols));
    s.products = cv.take_bytes(ns_scratch_bytes(l.batch.rows, l.batch.cols, l.matrices()));
    return s;
}

}  // namespace

int32_t muon_check(const moe_muon_tensor *tensors, int32_t count) {
    for (int32_t i = 0; i < count; ++i) MOE_TRY(check_tensor(tensors[i]));
    return MOE_OK;
}

int32_t muon_bytes(const moe_muon_tensor *tensors, int32_t count, int64_t *bytes) {
    *bytes = kWsHeader;
    return for_each_launch(tensors, count, [&](const Launch &l) -> int32_t {
        Carver cv(nullptr);
        cv.take_bytes(kWsHeader);
        scratch_of(cv, l);
        *bytes = imax(*bytes, (int64_t)cv.off);
        return MOE_OK;
    });
}

int32_t launch_muon(const moe_muon_tensor *tensors, int32_t count, const moe_muon_params &p, const moe_muon_rates *rates, void *ws, cudaStream_t st) {
    bool first = true;
    return for_each_launch(tensors, count, [&](const Launch &l) -> int32_t {
        Carver cv(ws);
        int32_t *status = static_cast<int32_t *>(cv.take_bytes(kWsHeader));
        const Scratch s = scratch_of(cv, l);
        const int64_t each = (int64_t)l.batch.rows * l.batch.cols, ld = muon_ld(l.batch.cols);
        Passes k = {};
        k.part = s.part; k.x = s.x; k.done = s.done; k.next = s.next; k.status = status;
        k.chunks = (int32_t)cdiv(each, CHUNK); k.clear_status = first; k.nesterov = p.nesterov;
        k.momentum = (float)p.momentum; k.eps = (float)p.eps; k.grad_scale = (float)p.grad_scale; k.rates = rates;
        const int64_t blocks = cdiv((int64_t)l.batch.rows * ld, CHUNK);
        if (l.matrices() * imax(blocks, k.chunks) > INT32_MAX) return MOE_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)(l.matrices() * k.chunks)), grid2((unsigned)(l.matrices() * blocks));
        // vectors of eight where every matrix, or every row, begins at one
        launch_kernel(each % EACH == 0 ? muon_momentum_kernel<true> : muon_momentum_kernel<false>, grid, dim3(THREADS), 0, st, l.batch, k);
        MOE_LAUNCHED();
        launch_kernel(l.batch.cols % EACH == 0 ? muon_normalise_kernel<true> : muon_normalise_kernel<false>, grid2, dim3(THREADS), 0, st, l.batch, k, (int32_t)blocks, (int32_t)ld);
        MOE_LAUNCHED();
        const NsWork w = {&l.batch, (int32_t)l.matrices(), p.steps, s.x, s.done, s.next, status, s.products, (float)p.lr, rates};
        MOE_TRY(launch_newton_schulz(w, st));
        first = false;
        return MOE_OK;
    });
}

}  // namespace moe
