// The whole Muon step of a small matrix, M up to 128, N up to 768 (the shorter and the longer side) and 49152 elements, by one block: momentum, norm, all Newton-Schulz products and the weights in one launch. See
// newton_schulz.cu for the products, their scaling and their diagonals.
//
// Bound by latency: 15 products, each of which needs the one before. X stays in shared memory, A and B in one place of it and accumulators in tensor memory, so that from product to product there
// is a barrier and not a way through L2 (8 experts of 64 x 128 and their gate: 31 us, by newton_schulz.cu 89; 40 of 72 x 520: 89 and 151).
//
// X is held as [N][128] whichever way the matrix lies, M columns and zeros behind them: 64-column pieces of 128-byte rows, 128-byte swizzle. A = X' X takes it MN-major twice, X B K-major by 128 rows
// of it at a time, whose accumulators lie beside each other in tensor memory, four at most; X B takes the place of X.
#include <type_traits>

#include "muon.cuh"
#include "muon_passes.cuh"
#include "pairs.cuh"
#include "short_wait.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr int THREADS = 512, WARPS = 16, MAX_TILES = 6;
constexpr int MAX_N = 128 * MAX_TILES;

__device__ __forceinline__ double block_sum(double v, double *sh) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sh[w];
    return s;
}
__device__ __forceinline__ uint64_t desc_columns(uint32_t addr, uint32_t piece_bytes) {  // MN-major, pieces of 64 columns piece_bytes apart
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(piece_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint32_t idesc_small(bool mn, int n) { return (1u << 4) | ((uint32_t)mn << 15) | ((uint32_t)mn << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24); }
__device__ __forceinline__ void unpack8(const uint4 &q, float2 (&v)[4]) {
    const __half2 *h = reinterpret_cast<const __half2 *>(&q);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __half22float2(h[i]);
}
__device__ __forceinline__ uint4 pack8(const float2 (&v)[4]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[i].x, v[i].y);
        u[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

struct Matrix {
    int64_t first;       // element
    int32_t rows, cols, M, N, Np;
    bool left;           // M rows: the matrix lies across X
    // element (n, m) of X and the way from it to (n, m + 1)
    __device__ __forceinline__ int64_t at(int32_t n, int32_t m) const { return first + (left ? (int64_t)m * cols + n : (int64_t)n * cols + m); }
    __device__ __forceinline__ int32_t stride() const { return left ? cols : 1; }
};
// m = momentum m + g of the whole matrix and the sum of u's squares, four eights a thread at a time
template <typename GT, typename MT, bool VECTORS> __device__ __forceinline__ double momentum_of(const GT *g, MT *p, int32_t each, const MuonPasses &k, float grad_scale) {
    double sum = 0.0;
    for (int32_t i = threadIdx.x * EACH; i < each; i += 4 * THREADS * EACH) {
        float gv[4][EACH], mv[4][EACH];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t at = i + q * THREADS * EACH;
            if (at < each) {
                load8<GT, VECTORS>(g, at, each - at, gv[q]);
                load8<MT, VECTORS>(p, at, each - at, mv[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t at = i + q * THREADS * EACH;
            if (at >= each) continue;
            float u[EACH], s = 0.0f;
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const float gj = gv[q][j] * grad_scale;
                mv[q][j] = held<MT>(fmaf(k.momentum, mv[q][j], gj));
                u[j] = k.nesterov ? fmaf(k.momentum, mv[q][j], gj) : mv[q][j];
                s = fmaf(u[j], u[j], s);
            }
            store8<MT, VECTORS>(p, at, each - at, mv[q]);
            sum += squares(s, u);
        }
    }
    return sum;
}
// X, eight columns of a row a thread, two of them at a time; neighbours have neighbouring elements of memory. What lies behind rows and columns is zero already
template <typename GT, typename MT> __device__ __forceinline__ void make_x(const Matrix &a, const GT *g, const MT *p, const MuonPasses &k, float grad_scale, const Factor &by, uint8_t *x) {
    const int32_t stride = a.stride(), eights = (a.M + 7) / 8, all = a.N * eights, inner = a.left ? a.N : eights;
    const float by_inner = 1.0f / (float)inner;
    for (int32_t i = threadIdx.x; i < all; i += 2 * THREADS) {
        float gv[2][8], mv[2][8];
        int32_t n[2], m[2], live[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int32_t at = i + q * THREADS;
            int32_t outer = (int32_t)((float)at * by_inner), rest = at - outer * inner;  // (at is below 2^14: off by one at most)
            if (rest < 0) { --outer; rest += inner; }
            if (rest >= inner) { ++outer; rest -= inner; }
            n[q] = a.left ? rest : outer;
            m[q] = (a.left ? outer : rest) * 8;
            live[q] = at < all ? a.M - m[q] : 0;
            const int64_t first = live[q] > 0 ? a.at(n[q], m[q]) : a.first;
            const GT *gp = g + first;
            const MT *mp = p + first;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                gv[q][j] = mv[q][j] = 0.0f;
                if (j < live[q]) {
                    mv[q][j] = to_f32(mp[j * stride]);
                    if (k.nesterov) gv[q][j] = to_f32(gp[j * stride]) * grad_scale;
                }
            }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (live[q] <= 0) continue;
            float2 v[4];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float u = by(k.nesterov ? fmaf(k.momentum, mv[q][j], gv[q][j]) : mv[q][j]);
                (j & 1 ? v[j / 2].y : v[j / 2].x) = j < live[q] ? u : 0.0f;  // (a NaN factor leaves the zeros behind the columns alone)
            }
            *reinterpret_cast<uint4 *>(x + (m[q] >> 6) * (a.Np * 128) + n[q] * 128 + ((((m[q] & 63) >> 3) ^ (n[q] & 7)) << 4)) = pack8(v);
        }
    }
}
// The weights, or masters, of X's columns m .. m + live - 1 in row n: all on their way together
template <typename T> __device__ __forceinline__ void load_weights32(const T *p, int32_t stride, int32_t live, float (&w)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = i < live ? to_f32(p[i * stride]) : 0.0f;
}
template <typename T> __device__ __forceinline__ void store_weights32(T *p, int32_t stride, int32_t live, const float (&w)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < live) p[i * stride] = from_f32<T>(w[i]);
}

__global__ void __launch_bounds__(THREADS) muon_small_kernel(const __grid_constant__ MuonBatch b, const MuonPasses k, float lr_given, int32_t steps, int32_t x_rows, uint32_t tmem_cols) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) float d_of[128], r_of[128];
    __shared__ double sh[WARPS];
    __shared__ __align__(8) uint64_t bar_at[MAX_TILES];
    __shared__ uint32_t tmem_at;
    __shared__ int abort_at;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *x = smem_raw + (base - smem_u32(smem_raw)), *ab = x + (int64_t)x_rows * 256;
    const uint32_t x_addr = base, ab_addr = base + (uint32_t)x_rows * 256, bar = smem_u32(bar_at);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3;
    if (threadIdx.x == 0) {
        for (int i = 0; i < MAX_TILES; ++i) mbar_init(bar + 8u * i, 1);
        abort_at = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    volatile int *abort_flag = &abort_at;
    wait_previous_kernel();
    const int32_t matrix = blockIdx.x;
    int q = 0;
    while (q + 1 < b.shapes && matrix >= b.s[q + 1].first) ++q;
    const MuonShape &s = b.s[q];
    const int32_t entry = b.entry_of(matrix);
    const int64_t each = (int64_t)s.rows * s.cols;
    const bool left = s.rows <= s.cols;
    const Matrix a = {(int64_t)(matrix - b.before[entry]) * each, s.rows, s.cols, min(s.rows, s.cols), max(s.rows, s.cols), (max(s.rows, s.cols) + 127) / 128 * 128, left};
    const MuonEntry &t = b.t[entry];
    const float grad_scale = k.rates ? k.rates->grad_scale : k.grad_scale, lr = k.rates ? k.rates->lr : lr_given;
    int32_t *status = k.status;
    if (matrix == 0 && threadIdx.x == 0 && k.clear_status) *status = 0;

    // ------------------------------------------------------------------ momentum and norm
    auto typed = [&](auto f) {  // by the types of gradient and momentum
        switch (t.kind & 6) {
            case 0: f(static_cast<const float *>(t.g), static_cast<float *>(t.m)); break;
            case 2: f(static_cast<const bf16 *>(t.g), static_cast<float *>(t.m)); break;
            case 4: f(static_cast<const float *>(t.g), static_cast<bf16 *>(t.m)); break;
            default: f(static_cast<const bf16 *>(t.g), static_cast<bf16 *>(t.m)); break;
        }
    };
    double sum = 0.0;
    typed([&](auto *g, auto *m) {
        using GT = std::decay_t<decltype(*g)>;
        using MT = std::decay_t<decltype(*m)>;
        sum = each % EACH == 0 ? momentum_of<GT, MT, true>(g + a.first, m + a.first, (int32_t)each, k, grad_scale) : momentum_of<GT, MT, false>(g + a.first, m + a.first, (int32_t)each, k, grad_scale);
    });
    for (int32_t i = threadIdx.x; i < a.Np * 16; i += THREADS) reinterpret_cast<uint4 *>(x)[i] = make_uint4(0u, 0u, 0u, 0u);
    sum = sqrt(block_sum(sum, sh)) + (double)k.eps;  // (whose barrier is behind the block's last store of a momentum, and of a zero)
    const Factor by(sum);
    typed([&](auto *g, auto *m) {
        using GT = std::decay_t<decltype(*g)>;
        using MT = std::decay_t<decltype(*m)>;
        make_x<GT, MT>(a, g, m, k, grad_scale, by, x);
    });
    const int32_t piece_bytes = a.Np * 128;  // of 64 columns

    // ------------------------------------------------------------------ products
    const int32_t tiles = a.Np / 128, n16 = (a.M + 15) & ~15, k_steps = n16 / 16, x_steps = (a.N + 15) / 16;
    const int32_t tile_columns = (a.M + 31) & ~31, at_once = min(tiles, (int32_t)tmem_cols / tile_columns);  // of X's accumulators in tensor memory
    const int32_t columns = (warp >> 2) * 32;  // of this warp, in A, B and a tile of X
    const uint32_t row_tmem = (uint32_t)(quarter * 32) << 16;
    const int32_t m1 = quarter * 32 + lane;  // this lane's row of A and B
    if (threadIdx.x < 128) d_of[threadIdx.x] = r_of[threadIdx.x] = 0.0f;
    uint32_t phase = 0;  // a bit for every barrier
    bool ok = true;
    auto ready = [&]() {  // what has been written to shared memory is there for the tensor cores, and what they wrote has been read
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncthreads();
    };
    auto arrived = [&](int i) {  // the products that barrier i was given
        const bool there = short_wait(bar + 8u * i, phase >> i & 1u, abort_flag, status);
        phase ^= 1u << i;
        tc_fence_after();
        return there;
    };
    auto done = [&]() { ok = __syncthreads_and(arrived(0)) != 0; };
    auto place = [&](uint8_t *from, int32_t bytes, int32_t row, int32_t c) {  // the c-th eight of the warp's columns in a row
        return reinterpret_cast<uint4 *>(from + (columns >> 6) * bytes + row * 128 + ((((columns & 63) / 8 + c) ^ (row & 7)) << 4));
    };
    for (int32_t step = 0; step < steps && ok; ++step) {
        // A
        ready();
        if (warp == 0) {
            tc_fence_after();
            uint64_t xd = desc_columns(x_addr, piece_bytes);
#pragma unroll 4
            for (int32_t i = 0; i < x_steps; ++i, xd += 16 * 128 >> 4) warp_mma(tmem, xd, xd, idesc_small(true, n16), i > 0);
            warp_commit(bar);
        }
        done();
        if (!ok) break;
        if (columns < n16) {
            {
                uint32_t raw[32];
                tc_ld_32x32(tmem + row_tmem + columns, raw);
                tc_ld_wait();
                if (columns == quarter * 32) {
                    float own = 0.0f;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i == lane) { own = __uint_as_float(raw[i]); raw[i] = 0u; }
                    d_of[m1] = m1 < a.M ? own * (1.0f / (MUON_UNIT * MUON_UNIT)) : 0.0f;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float2 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = mul2(make_float2(__uint_as_float(raw[8 * c + 2 * i]), __uint_as_float(raw[8 * c + 2 * i + 1])), both(1.0f / MUON_UNIT));
                    if (columns + 8 * c >= n16)  // no part of the accumulator
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = both(0.0f);
                    *place(ab, 128 * 128, m1, c) = pack8(v);
                }
            }
        }
        // B, in A's place
        ready();
        if (warp == 0) {
            tc_fence_after();
            const uint64_t ad = desc_kmajor(ab_addr);
#pragma unroll
            for (int32_t i = 0; i < 8; ++i)
                if (i < k_steps) warp_mma(tmem, ad + (i >> 2) * (128 * 128 >> 4) + (i & 3) * 2, ad + (i >> 2) * (128 * 128 >> 4) + (i & 3) * 2, idesc_small(false, n16), i > 0);
            warp_commit(bar);
        }
        done();
        if (!ok) break;
        if (columns < n16) {
            const float of_row = d_of[m1];
            {
                uint32_t raw[32];
                tc_ld_32x32(tmem + row_tmem + columns, raw);
                tc_ld_wait();
                if (columns == quarter * 32) {
                    float own = 0.0f;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i == lane) { own = __uint_as_float(raw[i]); raw[i] = 0u; }
                    own *= 1.0f / (MUON_UNIT * MUON_UNIT);
                    r_of[m1] = fmaf(NS_C, fmaf(of_row, of_row, own), fmaf(NS_B, of_row, NS_A));
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int32_t m2 = columns + 8 * c;
                    uint4 *at = place(ab, 128 * 128, m1, c);
                    float2 v[4];
                    unpack8(*at, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = make_float2(fmaf(NS_C, of_row + d_of[m2 + 2 * i], NS_B), fmaf(NS_C, of_row + d_of[m2 + 2 * i + 1], NS_B));
                        v[i] = fma2(make_float2(__uint_as_float(raw[8 * c + 2 * i]), __uint_as_float(raw[8 * c + 2 * i + 1])), both(NS_C / MUON_UNIT), mul2(v[i], f));
                    }
                    if (m2 >= n16)
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = both(0.0f);
                    *at = pack8(v);
                }
            }
        }
        // X, or the weights
        const bool last = step + 1 == steps;
        if (last) {  // into L2 while the products run
            const int32_t size = t.kind & 8 || !(t.kind & 1) ? 4 : 2;
            const char *from = (t.kind & 8 ? reinterpret_cast<const char *>(t.master) : static_cast<const char *>(t.w)) + a.first * size;
            for (int64_t i = (int64_t)threadIdx.x * 128; i < each * size; i += THREADS * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + i));
        }
        for (int32_t first = 0; first < tiles && ok; first += at_once) {
            const int32_t here = min(at_once, tiles - first);
            ready();
            if (warp < here) {  // a tile a warp: a product and a commit take the issuing warp longer than the tensor core
                tc_fence_after();
                const uint64_t xd = desc_kmajor(x_addr + (first + warp) * (128 * 128)), bd = desc_kmajor(ab_addr), piece = piece_bytes >> 4;
#pragma unroll
                for (int32_t i = 0; i < 8; ++i)
                    if (i < k_steps) warp_mma(tmem + warp * tile_columns, xd + (i >> 2) * piece + (i & 3) * 2, bd + (i >> 2) * (128 * 128 >> 4) + (i & 3) * 2, idesc_small(false, n16), i > 0);
                warp_commit(bar + 8u * warp);
            }
            float2 r[16];  // of the warp's columns
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = *reinterpret_cast<const float2 *>(r_of + columns + 2 * i);
            uint8_t *row_of_x = x + (columns >> 6) * piece_bytes + (first * 128 + quarter * 32 + lane) * 128;
            for (int32_t tile = 0; tile < here; ++tile, row_of_x += 128 * 128) {  // a tile is worked on while the next ones' products run
                const int32_t n = (first + tile) * 128 + quarter * 32 + lane, live = last && n < a.N ? min(32, a.M - columns) : 0;
                float w[32];
                const int64_t at_w = a.at(n, columns);
                if (live > 0) {
                    if (t.kind & 8) load_weights32(t.master + at_w, a.stride(), live, w);
                    else if (t.kind & 1) load_weights32(static_cast<const bf16 *>(t.w) + at_w, a.stride(), live, w);
                    else load_weights32(static_cast<const float *>(t.w) + at_w, a.stride(), live, w);
                }
                const bool there = arrived(tile);
                if (!__all_sync(0xffffffffu, there)) { ok = false; break; }
                if (columns >= n16) continue;
                uint32_t raw[32];
                tc_ld_32x32(tmem + row_tmem + tile * tile_columns + columns, raw);
                tc_ld_wait();
                if (columns + 32 > n16)  // what lies behind is no part of the accumulator
#pragma unroll
                    for (int i = 16; i < 32; ++i)
                        if (columns + i >= n16) raw[i] = 0u;
                float2 v[4][4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    unpack8(*reinterpret_cast<const uint4 *>(row_of_x + ((((columns & 63) / 8 + c) ^ (lane & 7)) << 4)), v[c]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[c][i] = fma2(make_float2(__uint_as_float(raw[8 * c + 2 * i]), __uint_as_float(raw[8 * c + 2 * i + 1])), both(1.0f / MUON_UNIT), mul2(v[c][i], r[4 * c + i]));
                }
                if (!last) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(row_of_x + ((((columns & 63) / 8 + c) ^ (lane & 7)) << 4)) = pack8(v[c]);
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] -= lr * fmaf(i & 1 ? v[i / 8][i / 2 % 4].y : v[i / 8][i / 2 % 4].x, t.scale * (1.0f / MUON_UNIT), t.decay * w[i]);
                if (live > 0) {
                    if (t.kind & 8) store_weights32(t.master + at_w, a.stride(), live, w);
                    if (t.kind & 1) store_weights32(static_cast<bf16 *>(t.w) + at_w, a.stride(), live, w);
                    else store_weights32(static_cast<float *>(t.w) + at_w, a.stride(), live, w);
                }
            }
            ok = __syncthreads_and(ok) != 0;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
    }
}

}  // namespace

// By one block: what its shared memory holds, and no more elements than it has done while tiles of several SMs have (newton_schulz.cu; matrices and their transposes: 16 of 128 x 128 31 us by blocks, 98
// by tiles, 500 of them 148 and 228; of 128 x 256 95 and 117, 298 and 341; of 96 x 512 119 and 117, 384 and 415; of 64 x 768 138 and 106, 449 and 440; of 128 x 768 259 and 125, 200 of them 398 and 266)
constexpr int64_t MOST_ELEMENTS = 49152;
bool muon_is_small(int32_t rows, int32_t cols) { return imin(rows, cols) <= 128 && imax(rows, cols) <= MAX_N && (int64_t)rows * cols <= MOST_ELEMENTS; }

int32_t muon_small_ready() {
    static PerDevice allowed;
    return allow_shared(allowed, muon_small_kernel, MAX_N * 256 + 128 * 256 + 1024) ? MOE_OK : MOE_ERR_CUDA;
}

int32_t launch_muon_small(const MuonBatch &b, const MuonPasses &k, float lr, int32_t steps, cudaStream_t st) {
    int64_t longest = 0;
    for (int q = 0; q < b.shapes; ++q) longest = imax(longest, imax(b.s[q].rows, b.s[q].cols));
    const int64_t x_rows = cdiv(longest, 128) * 128, tiles = x_rows / 128;
    const uint32_t tmem_cols = tiles <= 1 ? 128 : tiles == 2 ? 256 : 512;  // (an SM holds three blocks of one tile, two of two, one of more)
    const int bytes = (int)(x_rows * 256 + 128 * 256 + 1024);
    launch_kernel(muon_small_kernel, dim3((unsigned)b.matrices()), dim3(THREADS), (size_t)bytes, st, b, k, lr, steps, (int32_t)x_rows, tmem_cols);
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace moe
