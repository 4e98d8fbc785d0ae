// The whole layer for a few tokens (serving): two launches. The experts' weights are read once, by tensor copies that run ahead of everything else, and that is
// what bounds it: a matrix of 512 x 1024 in bf16 is 1 MB for two or three rows.
//
//   few_logits_kernel   the logits of every token by the fixed chain of multiply-adds of moe_gate, and the second launch's counters set to 0
//   few_experts_kernel  one block per SM. Every block picks the experts itself (top k, softmax): the logits are a few KB. The products then are
//                       tasks that running blocks draw in order from a counter: 64 columns (32 in float) of hid of one expert, for all of its rows; then
//                       64 columns of its part of y, over a piece of h. A task of the second kind waits until its expert's hid is complete. Tasks of the
//                       first kind wait for nothing and stand before all others, so that whoever waits, waits for blocks that are running: no
//                       block has to be resident for another to finish. Who delivers the last part of 64 columns of a token adds the parts in
//                       order: results do not depend on who does what.
//
// In a block one thread draws tasks and copies 64 x 128-byte tiles of weights into a ring, across the borders of tasks and kinds, the copies
// of a waiting task among them; eight warps multiply, every eighth tile each. Weights are the larger operand and the matrix instruction's rows; the tokens are its
// columns, 8 at a time. Rows this few would leave 120 of the 128 rows of a tcgen05 tile empty, and its accumulators would have to come back from
// tensor memory after every 64 KB; mma.sync from shared memory keeps up with the copies up to 64 rows an expert.
#include <float.h>
#include <math_constants.h>

#include "async_copy.cuh"
#include "block.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32 + 32;
constexpr int TILE_K = 64, TILE_BYTES = TILE_K * 128, RING = 16, TASKS = 4;
constexpr int MAX_ROWS = MOE_FEW_MAX_TOKENS * MOE_MAX_K;
constexpr int RED_TOKENS = 8, RED_COLS = 64, RED_STRIDE = RED_COLS + 4;

struct Few {
    const void *x, *b1, *b2;
    void *hid, *y;
    const float *logits;
    float *parts;                // [R][splits][d]
    int32_t *topk_idx;           // what the caller wants of the routing, or nullptr
    float *gates;
    int32_t *ticket, *ready, *done;  // tasks drawn; tiles of hid that an expert has; parts of y by token and tile of columns
    int32_t *status;
    int32_t T, d, h, n, k;
    int32_t tiles_h, tiles_d, splits, split_tiles;  // tiles of columns; pieces of h, of so many tiles of 64
};

// ------------------------------------------------------------------------------------------ logits
constexpr int LOGIT_STEP = 64, LOGIT_STAGES = 8, LOGIT_TOKENS = 8;
// 32 columns of the gate by LOGIT_TOKENS tokens, a warp each: one chain over ascending features per thread. Bound by the chain's latency, four cycles
// a feature, with the weights' way into shared memory beside it.
template <typename T, bool FOURS>
__global__ void __launch_bounds__(256) few_logits_kernel(const T *__restrict__ x, const float *__restrict__ Wg, int32_t tokens, int32_t d, int32_t n,
                                                         float *__restrict__ logits, int32_t *clear, int32_t clear_count, int32_t *status) {
    wait_previous_kernel();
    extern __shared__ __align__(16) char few_shared[];
    float *w = reinterpret_cast<float *>(few_shared);                           // [stage][LOGIT_STEP][32]
    T *xs = reinterpret_cast<T *>(w + LOGIT_STAGES * LOGIT_STEP * 32);          // [stage][LOGIT_TOKENS][LOGIT_STEP]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t col0 = blockIdx.x * 32, tok0 = blockIdx.y * LOGIT_TOKENS;
    const int32_t block = blockIdx.y * gridDim.x + blockIdx.x, blocks = gridDim.x * gridDim.y;
    for (int32_t i = block * 256 + threadIdx.x; i < clear_count; i += blocks * 256) clear[i] = 0;
    if (block == 0 && threadIdx.x == 0) *status = 0;
    const int32_t steps = (d + LOGIT_STEP - 1) / LOGIT_STEP;
    constexpr int XV = 16 / sizeof(T), XP = LOGIT_STEP / XV;  // a token's pieces of 16 bytes
    auto fetch = [&](int32_t s) {
        if (s < steps) {
            const int32_t k0 = s * LOGIT_STEP, at = s % LOGIT_STAGES;
            float *ws = w + at * LOGIT_STEP * 32;
            if constexpr (FOURS) {  // n is a multiple of four
                for (int32_t i = threadIdx.x; i < LOGIT_STEP * 8; i += 256) {
                    const int32_t r = i >> 3, c = (i & 7) * 4;
                    if (k0 + r < d && col0 + c < n) copy16(ws + r * 32 + c, Wg + (int64_t)(k0 + r) * n + col0 + c);
                }
            } else {
                for (int32_t i = threadIdx.x; i < LOGIT_STEP * 32; i += 256) {
                    const int32_t r = i >> 5, c = i & 31;
                    if (k0 + r < d && col0 + c < n) copy4(ws + r * 32 + c, Wg + (int64_t)(k0 + r) * n + col0 + c);
                }
            }
            T *xd = xs + at * LOGIT_TOKENS * LOGIT_STEP;
            for (int32_t i = threadIdx.x; i < LOGIT_TOKENS * XP; i += 256) {
                const int32_t t = i / XP, c = (i % XP) * XV;
                if (tok0 + t < tokens && k0 + c < d) copy16(xd + t * LOGIT_STEP + c, x + (int64_t)(tok0 + t) * d + k0 + c);
            }
        }
        copies_commit();
    };
    for (int32_t s = 0; s < LOGIT_STAGES - 1; ++s) fetch(s);
    const bool live = tok0 + warp < tokens;
    float acc = 0.0f;
    for (int32_t s = 0; s < steps; ++s) {
        copies_wait<LOGIT_STAGES - 2>();
        __syncthreads();
        fetch(s + LOGIT_STAGES - 1);  // where step s - 1 was
        if (!live) continue;
        const float *ws = w + (s % LOGIT_STAGES) * LOGIT_STEP * 32 + lane;
        const T *xt = xs + (s % LOGIT_STAGES) * LOGIT_TOKENS * LOGIT_STEP + warp * LOGIT_STEP;
        const int32_t left = min(LOGIT_STEP, d - s * LOGIT_STEP);
        if (left == LOGIT_STEP) {
#pragma unroll 16
            for (int i = 0; i < LOGIT_STEP; ++i) acc = fmaf(to_f32(xt[i]), ws[i * 32], acc);
        } else {
            for (int i = 0; i < left; ++i) acc = fmaf(to_f32(xt[i]), ws[i * 32], acc);
        }
    }
    if (live && col0 + lane < n) logits[(int64_t)(tok0 + warp) * n + col0 + lane] = acc;
}

// ------------------------------------------------------------------------------------------ experts
struct FewShared {
    uint64_t full[RING], empty[RING], task_full[TASKS], task_empty[TASKS];
    int32_t task[TASKS];
    int32_t abort, used_count;
    uint32_t used_bits[MOE_MAX_EXPERTS / 32];
    int16_t used[MAX_ROWS];
    int16_t idx[MAX_ROWS];
    float gate[MAX_ROWS];
    int16_t rows[FEW_WARPS][MOE_FEW_MAX_TOKENS];
    int32_t last[MOE_FEW_MAX_TOKENS];
    float red[2][FEW_WARPS][RED_TOKENS][RED_STRIDE];
};
constexpr int FEW_SMEM = RING * TILE_BYTES + 1024 + (int)sizeof(FewShared);

__device__ __forceinline__ void workers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool workers_any(bool p) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, 1, 256, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)p) : "memory");
    return r != 0;
}
__device__ __forceinline__ int32_t load_acquire(const int32_t *p) {
    int32_t v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int32_t add_acq_rel(int32_t *p, int32_t by) {
    int32_t v;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(v) : "l"(p), "r"(by) : "memory");
    return v;
}
__device__ __forceinline__ void add_release(int32_t *p, int32_t by) {
    asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(by) : "memory");
}

// The k largest logits of a token in descending order, equal ones by index, NaN below every number; softmax over them (the arithmetic of moe_gate without
// noise). A warp takes a token.
template <int KL>
__device__ void select_token(const Few &a, FewShared &S, int32_t t, int lane) {
    const float *row = a.logits + (int64_t)t * a.n;
    float lv[KL];
    int32_t li[KL];
#pragma unroll
    for (int s = 0; s < KL; ++s) { lv[s] = -CUDART_INF_F; li[s] = INT32_MAX; }
    for (int32_t q = lane; q < a.n; q += 32) {
        float v = row[q];
        v = v == v ? v : -CUDART_INF_F;
        int32_t id = q;
        bool shifting = false;
#pragma unroll
        for (int s = 0; s < KL; ++s) {
            if (shifting || v > lv[s] || li[s] == INT32_MAX) {
                const float tv = lv[s];
                const int32_t ti = li[s];
                lv[s] = v; li[s] = id; v = tv; id = ti;
                shifting = true;
            }
        }
    }
    float myv = -CUDART_INF_F;
    int32_t myi = 0;
    for (int s = 0; s < a.k; ++s) {
        float hv = lv[0];
        int32_t hi = li[0];
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const float ov = __shfl_xor_sync(0xffffffffu, hv, off);
            const int32_t oi = __shfl_xor_sync(0xffffffffu, hi, off);
            if (ov > hv || (ov == hv && oi < hi)) { hv = ov; hi = oi; }
        }
        if (li[0] == hi) {
#pragma unroll
            for (int q = 0; q < KL - 1; ++q) { lv[q] = lv[q + 1]; li[q] = li[q + 1]; }
            lv[KL - 1] = -CUDART_INF_F;
            li[KL - 1] = INT32_MAX;
        }
        if (lane == s) { myv = hv; myi = hi; }
    }
    const float m = __shfl_sync(0xffffffffu, myv, 0);
    const float ex = lane < a.k ? expf(myv - m) : 0.0f;
    float den = 0.0f;
    for (int s = 0; s < a.k; ++s) den += __shfl_sync(0xffffffffu, ex, s);
    if (lane < a.k) {
        const float g = ex / den;
        S.idx[t * a.k + lane] = (int16_t)myi;
        S.gate[t * a.k + lane] = g;
        if (blockIdx.x == 0) {
            if (a.topk_idx) a.topk_idx[t * a.k + lane] = myi;
            if (a.gates) a.gates[t * a.k + lane] = g;
        }
    }
}

struct Task { int32_t expert, rank, col, k0, k1; bool second; };  // rank: among the experts that are used
__device__ __forceinline__ Task task_of(const Few &a, const FewShared &S, int32_t number) {
    Task t;
    const int32_t first = S.used_count * a.tiles_h;
    t.second = number >= first;
    if (!t.second) {
        t.rank = number / a.tiles_h;
        t.col = number % a.tiles_h;
        t.k0 = 0;
        t.k1 = a.d;
    } else {
        const int32_t q = number - first, per = a.tiles_d * a.splits;
        t.rank = q / per;
        t.col = q % per / a.splits;
        t.k0 = q % a.splits * a.split_tiles * TILE_K;
        t.k1 = min(a.h, t.k0 + a.split_tiles * TILE_K);
    }
    t.expert = S.used[t.rank];
    return t;
}
__device__ __forceinline__ int32_t all_tasks(const Few &a, const FewShared &S) { return S.used_count * (a.tiles_h + a.tiles_d * a.splits); }

__device__ __forceinline__ void ldmatrix_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Half a tile, 32 k by 64 columns, bf16. A lane holds eight consecutive k of a row in four registers and gives them to the matrix instruction two at a
// time; any order of k does as long as the weights follow it. Lane c of a row begins with its c-th pair: the eight k of an 8 x 8 matrix then differ modulo 8,
// and their rows in the swizzled tile lie in eight different banks.
template <int NT>
__device__ __forceinline__ void multiply_half(float (&acc)[4][NT][4], uint32_t tile, int j, const uint4 (&xv)[NT], int lane) {
    const int r = lane & 7, m = lane >> 3, c = lane & 3;
    uint32_t b[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        uint32_t v0 = xv[t].x, v1 = xv[t].y, v2 = xv[t].z, v3 = xv[t].w;
        if (c & 1) { const uint32_t s = v0; v0 = v1; v1 = v2; v2 = v3; v3 = s; }
        if (c & 2) { uint32_t s = v0; v0 = v2; v2 = s; s = v1; v1 = v3; v3 = s; }
        b[t][0] = v0; b[t][1] = v1; b[t][2] = v2; b[t][3] = v3;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        // row r of matrix m: lane r / 2's pair 2 s + m / 2, element r % 2
        const int lc = r >> 1, k = 32 * j + 8 * lc + 2 * ((2 * s + (m >> 1) + lc) & 3) + (r & 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t w[4];
            ldmatrix_t(w, tile + k * 128 + (((2 * q + (m & 1)) ^ (k & 7)) << 4));
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_16x8x16(acc[q][t], w, b[t][2 * s], b[t][2 * s + 1]);
        }
    }
}

template <typename T> __device__ __forceinline__ uint4 load_rows(const void *base, int64_t at, bool second) {
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const T *>(base) + at);
    return second ? __ldcg(p) : __ldg(p);  // hid is written by other blocks of this launch: from L2
}

// What a task leaves: a sum already added over the warps
template <typename T> __device__ __forceinline__ void put_sum(const Few &a, const Task &t, int32_t p, int32_t col, float v) {
    if (!t.second) {
        if (col >= a.h) return;
        v += to_f32(static_cast<const T *>(a.b1)[(int64_t)t.expert * a.h + col]);
        v = v < 0.0f ? 0.0f : v;  // a NaN stays
        static_cast<T *>(a.hid)[(int64_t)p * a.h + col] = from_f32<T>(v);
    } else {
        if (col >= a.d) return;
        a.parts[((int64_t)p * a.splits + t.k0 / (a.split_tiles * TILE_K)) * a.d + col] = v;
    }
}

template <typename T, int NT>
__device__ void run_task(const Few &a, FewShared &S, const Task &t, int32_t m, uint32_t ring, int32_t tile0, int warp, int lane) {
    constexpr int COLS = 128 / (int)sizeof(T);
    constexpr bool BF16 = sizeof(T) == 2;
    const int16_t *rows = S.rows[warp];
    const int32_t tiles = (t.k1 - t.k0 + TILE_K - 1) / TILE_K, g = lane >> 2, c = lane & 3;
    const void *base = t.second ? a.hid : a.x;
    const int64_t width = t.second ? a.h : a.d;
    float acc[BF16 ? 4 : 1][NT][BF16 ? 4 : 8];
#pragma unroll
    for (int q = 0; q < (BF16 ? 4 : 1); ++q)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < (BF16 ? 4 : 8); ++i) acc[q][u][i] = 0.0f;
    for (int32_t i = warp; i < tiles; i += FEW_WARPS) {
        const int32_t number = tile0 + i, slot = number % RING, k0 = t.k0 + i * TILE_K;
        const uint32_t tile = ring + slot * TILE_BYTES, full = smem_u32(&S.full[slot]);
        if constexpr (BF16) {
            auto fetch = [&](int j, uint4 (&xv)[NT]) {
                const int32_t k = k0 + 32 * j + 8 * c;
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    const int32_t q = u * 8 + g;
                    const int64_t row = q < m ? (t.second ? rows[q] : rows[q] / a.k) : 0;
                    xv[u] = q < m && k < t.k1 ? load_rows<T>(base, row * width + k, t.second) : make_uint4(0u, 0u, 0u, 0u);
                }
            };
            if constexpr (NT <= 4) {
                uint4 x0[NT], x1[NT];
                fetch(0, x0);
                fetch(1, x1);
                mbar_wait(full, (number / RING) & 1, &S.abort, a.status);
                multiply_half<NT>(acc, tile, 0, x0, lane);
                multiply_half<NT>(acc, tile, 1, x1, lane);
            } else {  // registers for half of it
                mbar_wait(full, (number / RING) & 1, &S.abort, a.status);
#pragma unroll 1
                for (int j = 0; j < 2; ++j) {
                    uint4 xv[NT];
                    fetch(j, xv);
                    multiply_half<NT>(acc, tile, j, xv, lane);
                }
            }
        } else {
            mbar_wait(full, (number / RING) & 1, &S.abort, a.status);
            const char *at = reinterpret_cast<const char *>(__cvta_shared_to_generic(tile));
            for (int32_t kk = 0; kk < TILE_K && k0 + kk < t.k1; kk += 4) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = kk + e;
                    w[e] = *reinterpret_cast<const float *>(at + k * 128 + (((lane >> 2) ^ (k & 7)) << 4) + (lane & 3) * 4);
                }
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        if (u * 8 + q >= m) break;
                        const int64_t row = t.second ? rows[u * 8 + q] : rows[u * 8 + q] / a.k;
                        const uint4 v = load_rows<T>(base, row * width + k0 + kk, t.second);
                        float s = acc[0][u][q];
                        s = fmaf(__uint_as_float(v.x), w[0], s);
                        s = fmaf(__uint_as_float(v.y), w[1], s);
                        s = fmaf(__uint_as_float(v.z), w[2], s);
                        acc[0][u][q] = fmaf(__uint_as_float(v.w), w[3], s);
                    }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.empty[slot]));
    }
    // over the warps that had tiles, in their order
    const int32_t parts = min(tiles, FEW_WARPS);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        if (u * 8 >= m) break;
        float(*red)[RED_TOKENS][RED_STRIDE] = S.red[u & 1];
        if (warp < parts) {
            if constexpr (BF16) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) red[warp][2 * c + (i & 1)][16 * q + g + 8 * (i >> 1)] = acc[q][u][i];
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) red[warp][q][lane] = acc[0][u][q];
            }
        }
        workers_sync();
        for (int32_t i = threadIdx.x; i < RED_TOKENS * COLS; i += FEW_WARPS * 32) {
            const int32_t q = i / COLS, col = i % COLS;
            if (u * 8 + q >= m) continue;
            float v = 0.0f;
            for (int32_t p = 0; p < parts; ++p) v += red[p][q][col];
            put_sum<T>(a, t, rows[u * 8 + q], t.col * COLS + col, v);
        }
    }
    workers_sync();
    if (!t.second) {
        if (threadIdx.x == 0) {
            __threadfence();
            add_release(a.ready + t.rank, 1);
        }
        return;
    }
    // the last part of a token's columns adds up: y = sum over the slots of gate * (b2 + the pieces of h)
    if ((int32_t)threadIdx.x < m) {
        __threadfence();
        const int32_t token = rows[threadIdx.x] / a.k;
        S.last[threadIdx.x] = add_acq_rel(a.done + token * a.tiles_d + t.col, 1) == a.k * a.splits - 1;
    }
    workers_sync();
    for (int32_t i = threadIdx.x; i < m * COLS; i += FEW_WARPS * 32) {
        const int32_t q = i / COLS, col = t.col * COLS + i % COLS;
        if (!S.last[q] || col >= a.d) continue;
        const int32_t token = rows[q] / a.k;
        float y = 0.0f;
        for (int32_t s = 0; s < a.k; ++s) {
            const int32_t p = token * a.k + s;
            float v = 0.0f;
            for (int32_t z = 0; z < a.splits; ++z) v += __ldcg(a.parts + ((int64_t)p * a.splits + z) * a.d + col);
            v += to_f32(static_cast<const T *>(a.b2)[(int64_t)S.idx[p] * a.d + col]);
            y = fmaf(S.gate[p], v, y);
        }
        static_cast<T *>(a.y)[(int64_t)token * a.d + col] = from_f32<T>(y);
    }
}

template <typename T>
__global__ void __launch_bounds__(FEW_THREADS, 1) few_experts_kernel(const __grid_constant__ CUtensorMap w1, const __grid_constant__ CUtensorMap w2, const Few a) {
    extern __shared__ char few_raw[];
    char *base = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(few_raw) + 1023) & ~uintptr_t(1023));
    FewShared &S = *reinterpret_cast<FewShared *>(base + RING * TILE_BYTES);
    const uint32_t ring = smem_u32(base);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) { mbar_init(smem_u32(&S.full[i]), 1); mbar_init(smem_u32(&S.empty[i]), 1); }
        for (int i = 0; i < TASKS; ++i) { mbar_init(smem_u32(&S.task_full[i]), 1); mbar_init(smem_u32(&S.task_empty[i]), FEW_WARPS); }
        S.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = threadIdx.x; i < MOE_MAX_EXPERTS / 32; i += FEW_THREADS) S.used_bits[i] = 0;
    wait_previous_kernel();
    if (warp < FEW_WARPS)
        for (int32_t t = warp; t < a.T; t += FEW_WARPS) {
            if (a.k <= 2) select_token<2>(a, S, t, lane);
            else if (a.k <= 4) select_token<4>(a, S, t, lane);
            else select_token<8>(a, S, t, lane);
        }
    __syncthreads();
    const int32_t R = a.T * a.k;
    for (int32_t p = threadIdx.x; p < R; p += FEW_THREADS) atomicOr(&S.used_bits[S.idx[p] >> 5], 1u << (S.idx[p] & 31));
    __syncthreads();
    if (warp == 0) {  // the experts in use, ascending: eight words a lane at most
        const int32_t words = (a.n + 31) / 32, each = (words + 31) / 32;
        int32_t mine = 0;
        for (int32_t i = 0; i < each; ++i)
            if (lane * each + i < words) mine += __popc(S.used_bits[lane * each + i]);
        int32_t before = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int32_t o = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += o;
        }
        if (lane == 31) S.used_count = before;
        before -= mine;
        for (int32_t i = 0; i < each; ++i) {
            if (lane * each + i >= words) break;
            for (uint32_t b = S.used_bits[lane * each + i]; b; b &= b - 1) S.used[before++] = (int16_t)((lane * each + i) * 32 + __ffs(b) - 1);
        }
    }
    __syncthreads();
    const int32_t total = all_tasks(a, S);

    if (warp == FEW_WARPS) {  // draws tasks and copies their weights
        if (lane == 0) {
            int32_t tile = 0;
            int32_t next = atomicAdd(a.ticket, 1);
            for (int32_t task = 0;; ++task) {
                const int32_t number = next, slot = task % TASKS;
                if (!mbar_wait(smem_u32(&S.task_empty[slot]), ((task / TASKS) & 1) ^ 1, &S.abort, a.status)) break;
                S.task[slot] = number < total ? number : -1;
                mbar_arrive(smem_u32(&S.task_full[slot]));
                if (number >= total) break;
                next = atomicAdd(a.ticket, 1);  // on its way while the tiles are asked for
                const Task t = task_of(a, S, number);
                const CUtensorMap *map = t.second ? &w2 : &w1;
                bool ok = true;
                for (int32_t k = t.k0; k < t.k1; k += TILE_K, ++tile) {
                    const int32_t s = tile % RING;
                    ok = mbar_wait(smem_u32(&S.empty[s]), ((tile / RING) & 1) ^ 1, &S.abort, a.status);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&S.full[s]);
                    mbar_expect_tx(bar, TILE_BYTES);
                    tma_load_3d(ring + s * TILE_BYTES, map, bar, t.col * 64, k, t.expert);
                }
                if (!ok) break;
            }
            // given up: nothing may be on its way into shared memory that is given back
            if (*(volatile int32_t *)&S.abort)
                for (int32_t i = max(0, tile - RING); i < tile; ++i) {
                    const unsigned long long t0 = global_ns();
                    while (!mbar_try_wait(smem_u32(&S.full[i % RING]), (i / RING) & 1) && global_ns() - t0 < WAIT_LIMIT_NS) {}
                }
        }
        return;
    }

    int32_t tile = 0;
    for (int32_t task = 0;; ++task) {
        const int32_t slot = task % TASKS;
        const bool ok = mbar_wait(smem_u32(&S.task_full[slot]), (task / TASKS) & 1, &S.abort, a.status);
        const int32_t number = ok ? S.task[slot] : -1;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&S.task_empty[slot]));
        // all warps go on or none does: a barrier that decides the same for every one of them. It also keeps the rows and sums of the task before
        // until every warp has read them
        if (workers_any(number < 0 || *(volatile int32_t *)&S.abort)) break;
        const Task t = task_of(a, S, number);
        // the expert's rows, slots in ascending order
        int32_t m = 0;
        for (int32_t p0 = 0; p0 < R; p0 += 32) {
            const bool here = p0 + lane < R && S.idx[p0 + lane] == t.expert;
            const uint32_t who = __ballot_sync(0xffffffffu, here);
            if (here) S.rows[warp][m + __popc(who & ((1u << lane) - 1))] = (int16_t)(p0 + lane);
            m += __popc(who);
        }
        __syncwarp();
        if (t.second) {  // its hid complete
            if (lane == 0) {
                const int32_t *ready = a.ready + t.rank;
                unsigned long long t0 = 0;
                while (load_acquire(ready) < a.tiles_h && !*(volatile int32_t *)&S.abort) {
                    const unsigned long long now = global_ns();
                    if (t0 == 0) t0 = now;
                    if (now - t0 > WAIT_LIMIT_NS) {
                        *(volatile int32_t *)&S.abort = 1;
                        atomicExch(a.status, (int32_t)MOE_ERR_TIMEOUT);
                    }
                }
            }
            __syncwarp();
        }
        if (m <= 8) run_task<T, 1>(a, S, t, m, ring, tile, warp, lane);
        else if (m <= 16) run_task<T, 2>(a, S, t, m, ring, tile, warp, lane);
        else if (m <= 32) run_task<T, 4>(a, S, t, m, ring, tile, warp, lane);
        else run_task<T, 8>(a, S, t, m, ring, tile, warp, lane);
        tile += (t.k1 - t.k0 + TILE_K - 1) / TILE_K;
    }
}

struct FewPlan {
    int32_t tiles_h, tiles_d, splits, split_tiles, counters;
};
FewPlan plan_of(const moe_config &c) {
    FewPlan p;
    const int64_t cols = 128 / (int64_t)act_bytes(c.act), R = (int64_t)c.T * c.k, used = imin(c.n, R);
    p.tiles_h = (int32_t)cdiv(c.h, cols);
    p.tiles_d = (int32_t)cdiv(c.d, cols);
    // pieces of h, until every SM has about four tasks, of two tiles or more each
    const int64_t tiles = cdiv(c.h, TILE_K), wanted = cdiv(4 * 148, imax(1, used * p.tiles_d));
    p.split_tiles = (int32_t)imax(imin(2, tiles), cdiv(tiles, wanted));
    p.splits = (int32_t)cdiv(tiles, p.split_tiles);
    p.counters = (int32_t)(64 + MAX_ROWS + (int64_t)c.T * p.tiles_d);
    return p;
}

struct FewWs {
    int32_t *status, *counters;
    float *logits, *parts;
    void *hid;
    size_t bytes;
    FewWs(void *ws, const moe_config &c, const FewPlan &p) {
        Carver cv(ws);
        status = static_cast<int32_t *>(cv.take_bytes(kWsHeader));
        const int64_t R = (int64_t)c.T * c.k;
        counters = cv.take<int32_t>(p.counters);
        logits = cv.take<float>((int64_t)c.T * c.n);
        hid = cv.take_bytes(R * c.h * (int64_t)act_bytes(c.act));
        parts = cv.take<float>(R * p.splits * c.d);
        bytes = cv.off;
    }
};

// [n, K, N] as 16-bit elements: boxes of 64 k by 128 bytes of columns
int32_t weight_map(CUtensorMap *map, const void *w, int64_t n, int64_t K, int64_t N, int32_t act) {
    const uint64_t row = (uint64_t)N * act_bytes(act), dims[3] = {row / 2, (uint64_t)K, (uint64_t)n}, strides[2] = {row, row * (uint64_t)K};
    const uint32_t box[3] = {64, TILE_K, 1};
    return tc_make_map(map, w, 3, dims, strides, box);
}

template <typename T, bool FOURS> int32_t launch_logits(const moe_config &c, const void *x, const float *Wg, const FewWs &w, const FewPlan &p, cudaStream_t st) {
    constexpr int bytes = LOGIT_STAGES * (LOGIT_STEP * 32 * 4 + LOGIT_TOKENS * LOGIT_STEP * (int)sizeof(T));
    static PerDevice allowed;
    if (!allow_shared(allowed, few_logits_kernel<T, FOURS>, bytes)) return MOE_ERR_CUDA;
    launch_kernel(few_logits_kernel<T, FOURS>, dim3((unsigned)cdiv(c.n, 32), (unsigned)cdiv(c.T, LOGIT_TOKENS)), dim3(256), (size_t)bytes, st,
                  static_cast<const T *>(x), Wg, c.T, c.d, c.n, w.logits, w.counters, p.counters, w.status);
    MOE_LAUNCHED();
    return MOE_OK;
}

template <typename T> int32_t launch_experts(const CUtensorMap &w1, const CUtensorMap &w2, const Few &a, cudaStream_t st) {
    static PerDevice allowed;
    if (!allow_shared(allowed, few_experts_kernel<T>, FEW_SMEM)) return MOE_ERR_CUDA;
    launch_kernel(few_experts_kernel<T>, dim3((unsigned)tc_sm_count()), dim3(FEW_THREADS), (size_t)FEW_SMEM, st, w1, w2, a);
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace

int64_t few_tokens_bytes(const moe_config &c) { return (int64_t)FewWs(nullptr, c, plan_of(c)).bytes; }

int32_t launch_few_tokens(const moe_config &c, const void *x, const float *Wg, const void *W1, const void *b1, const void *W2, const void *b2, void *y,
                          int32_t *topk_idx, float *gates, void *ws, cudaStream_t st) {
    if (c.T == 0) {
        MOE_CUDA(cudaMemsetAsync(ws, 0, kWsHeader, st));
        return MOE_OK;
    }
    const FewPlan p = plan_of(c);
    const FewWs w(ws, c, p);
    CUtensorMap m1, m2;
    MOE_TRY(weight_map(&m1, W1, c.n, c.d, c.h, c.act));
    MOE_TRY(weight_map(&m2, W2, c.n, c.h, c.d, c.act));
    Few a = {};
    a.x = x; a.b1 = b1; a.b2 = b2; a.hid = w.hid; a.y = y; a.logits = w.logits; a.parts = w.parts; a.topk_idx = topk_idx; a.gates = gates;
    a.ticket = w.counters; a.ready = w.counters + 64; a.done = a.ready + MAX_ROWS; a.status = w.status;
    a.T = c.T; a.d = c.d; a.h = c.h; a.n = c.n; a.k = c.k;
    a.tiles_h = p.tiles_h; a.tiles_d = p.tiles_d; a.splits = p.splits; a.split_tiles = p.split_tiles;
    if (c.act == MOE_BF16) {
        MOE_TRY(c.n % 4 == 0 ? (launch_logits<bf16, true>(c, x, Wg, w, p, st)) : (launch_logits<bf16, false>(c, x, Wg, w, p, st)));
        return launch_experts<bf16>(m1, m2, a, st);
    }
    MOE_TRY(c.n % 4 == 0 ? (launch_logits<float, true>(c, x, Wg, w, p, st)) : (launch_logits<float, false>(c, x, Wg, w, p, st)));
    return launch_experts<float>(m1, m2, a, st);
}

}  // namespace moe
