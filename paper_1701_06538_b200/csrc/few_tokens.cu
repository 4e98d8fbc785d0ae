// The whole layer for a few tokens (serving): two launches, three with more than 256 experts. The experts' weights are read once, by tensor copies that run ahead
// of everything else, and that is what bounds it: a matrix of 512 x 1024 in bf16 is 1 MB for two or three rows.
//
//   few_logits_kernel   the logits of every token by the fixed chain of multiply-adds of moe_gate, and the second launch's counters set to 0. The blocks of four tokens are a
//                       cluster, whose first block gets all their logits and picks the experts (top k, softmax)
//   few_select_kernel   picks them from logits in memory, where a cluster does not hold the gate (more than 256 experts)
//   few_experts_kernel  one block per SM. Every block sorts the slots by expert. The products then are
//                       tasks that warps draw in order from a counter: 64 columns (32 in float) of a piece of the contraction for hid of one expert's
//                       rows, then the same for y. Pieces leave float sums; whoever delivers the last one of its columns adds them up in order, so that results do not
//                       depend on who does what. A task for y waits until its rows' hid is complete. Tasks for hid wait for nothing and are drawn
//                       before all others, so that whoever waits, waits for warps that are running: no block has to be resident for another to finish.
//
// A warp works by itself: it draws its next tasks and copies their 64 x 128-byte tiles of weights into its own ring while it multiplies. (With one ring for
// a block, a warp that copies and eight that share a task, whatever a task waits for, rows of x, sums, counters, is waited for by the whole SM: 177 us for 64 tokens
// of 256 experts of 512 x 1024.) Weights are the larger operand and the matrix instruction's rows, the tokens its columns, 8 at a time. Rows this few would leave
// most of a tcgen05 tile empty, and its accumulators would have to come back from tensor memory every few KB; mma.sync from shared memory keeps up with the copies.
#include <float.h>
#include <math.h>
#include <math_constants.h>

#include "async_copy.cuh"
#include "block.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32;
constexpr int TILE_K = 64, TILE_BYTES = TILE_K * 128;
constexpr int WARP_BYTES = 3 * TILE_BYTES;  // shared memory of a warp: bf16 a ring of three tiles, float of two and two tiles of its rows
constexpr int MAX_ROWS = MOE_FEW_MAX_TOKENS * MOE_MAX_K;
constexpr int READY_STEP = 32;  // a line for a segment's count, so that those who wait for one do not hold up another's
constexpr int SEG_ROWS = 16, NT = SEG_ROWS / 8;  // rows of a task: an expert with more is several segments, whose weights are read again, from L2. (32: the few experts with that many kept a call waiting)

// bf16 rows that the matrix instruction takes (x, hid) stand in the workspace as it wants them (turned()), widths rounded up to tiles, zeros behind the last column. hid is kept
// in two bf16 terms (float layers: float): in one its rounding would cost as much accuracy as that of y.
struct Few {
    const void *x, *b1, *b2;     // x: [T][d], of bf16 layers the turned copy [T][dw]
    void *y;
    float *hid;                  // [R][h], or
    bf16 *hid_hi;                // [R][hw], and hid_lo_at elements further on the second terms
    int64_t hid_lo_at;
    const int32_t *idx;          // [T][k], and the gates
    const float *gates;
    float *parts1, *parts2;      // [R][pieces][columns]
    int32_t *ticket, *ready, *done1, *done2;  // tasks drawn; columns of hid that a segment has; pieces by segment and columns of hid; by token and columns of y
    int32_t *status;
    int32_t T, d, h, n, k, dw, hw;
    // tiles of columns; pieces of the contraction, of so many tiles of 64
    int32_t cols1, pieces1, piece_tiles1, cols2, pieces2, piece_tiles2;
    Divisor by_k, by_task1, by_task2, by_pieces1, by_pieces2;  // by_task: columns and pieces of a segment
};
constexpr int ROW_SLACK = 128;  // elements behind the last row, which are fetched but not used

// Where column k of a bf16 row stands. A lane of the matrix instruction holds eight consecutive k of a row in four registers and gives them to it two at a
// time; any order of k does as long as the weights follow it. Lane c = (k / 8) % 4 begins with its c-th pair: the eight k of an 8 x 8 matrix of weights then differ
// modulo 8, and their rows in the swizzled tile lie in eight different banks.
__device__ __forceinline__ int32_t turned(int32_t k) {
    const int32_t c = (k >> 3) & 3, pair = (k >> 1) & 3;
    return (k & ~7) + ((pair - c) & 3) * 2 + (k & 1);
}

// ------------------------------------------------------------------------------------------ routing
// Floats as integers of the same order, NaN as the smallest number, -0 as 0. 0 is below all of them.
__device__ __forceinline__ uint32_t ordered(float v) {
    v = v == v ? v + 0.0f : -CUDART_INF_F;
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_ordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// The k largest keys of a warp in descending order, equal ones by index: lane s gets the s-th. A round takes the largest key and the lowest index that has it, by two
// reductions of integers, 250 cycles. The lane's keys: V of them, index of the i-th first + 32 i + lane, and one with an index of its own.
template <int V> __device__ __forceinline__ void take_best(int32_t k, uint32_t (&key)[V], int32_t first, uint32_t own, int32_t own_i, int lane, uint32_t &best, int32_t &best_i) {
    best = 0;
    best_i = 0;
#pragma unroll 1
    for (int s = 0; s < k; ++s) {
        uint32_t m = own;
#pragma unroll
        for (int i = 0; i < V; ++i) m = max(m, key[i]);
        m = __reduce_max_sync(0xffffffffu, m);
        uint32_t at = own == m ? (uint32_t)own_i : 0xffffffffu;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (key[i] == m) at = min(at, (uint32_t)(first + 32 * i + lane));
        at = __reduce_min_sync(0xffffffffu, at);
        if ((uint32_t)own_i == at) own = 0;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if ((uint32_t)(first + 32 * i + lane) == at) key[i] = 0;
        if (lane == s) { best = m; best_i = (int32_t)at; }
    }
}

struct Routing { int32_t *idx, *user_idx; float *gates, *user_gates; };  // [T][k]; user's: nullptr where not wanted
// Softmax over a token's kept logits, lane s the s-th; the sum in the order of moe_gate's
__device__ __forceinline__ void put_routing(const Routing &r, int32_t t, int32_t k, int lane, uint32_t best, int32_t best_i) {
    const float v = of_ordered(best), top = __shfl_sync(0xffffffffu, v, 0);
    const float ex = lane < k ? expf(v - top) : 0.0f;
    float den = 0.0f;
    for (int s = 0; s < k; ++s) den += __shfl_sync(0xffffffffu, ex, s);
    if (lane >= k) return;
    const float g = ex / den;
    r.idx[t * k + lane] = best_i;
    r.gates[t * k + lane] = g;
    if (r.user_idx) r.user_idx[t * k + lane] = best_i;
    if (r.user_gates) r.user_gates[t * k + lane] = g;
}

// A block per token: a warp takes an eighth of the columns, 256 at a time beside the best of those before, then one warp the eight warps' best
__global__ void __launch_bounds__(256) few_select_kernel(const float *__restrict__ logits, int32_t n, int32_t k, const Routing r) {
    wait_previous_kernel();
    constexpr int V = 8;
    __shared__ uint32_t sh_key[64];
    __shared__ int32_t sh_i[64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float *row = logits + (int64_t)blockIdx.x * n;
    const int32_t each = (n + 7) / 8, lo = warp * each, hi = min(n, lo + each);
    uint32_t best = 0;
    int32_t best_i = INT32_MAX;
    for (int32_t c0 = lo; c0 < hi; c0 += 32 * V) {
        uint32_t key[V];
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = c0 + 32 * i + lane < hi ? ordered(row[c0 + 32 * i + lane]) : 0;
        take_best(k, key, c0, best, best_i, lane, best, best_i);
    }
    if (threadIdx.x < 64) sh_key[threadIdx.x] = 0;
    __syncthreads();
    if (lane < k) { sh_key[warp * k + lane] = best; sh_i[warp * k + lane] = best_i; }
    __syncthreads();
    if (warp > 0) return;
    // up to 64 candidates, each with an index of its own: the rounds of take_best on pairs
    uint32_t a = sh_key[lane], b = sh_key[32 + lane];
    const int32_t ai = a ? sh_i[lane] : INT32_MAX, bi = b ? sh_i[32 + lane] : INT32_MAX;
    best = 0;
    best_i = 0;
    for (int s = 0; s < k; ++s) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, max(a, b));
        const uint32_t at = __reduce_min_sync(0xffffffffu, min(a == m ? (uint32_t)ai : 0xffffffffu, b == m ? (uint32_t)bi : 0xffffffffu));
        if ((uint32_t)ai == at) a = 0;
        if ((uint32_t)bi == at) b = 0;
        if (lane == s) { best = m; best_i = (int32_t)at; }
    }
    put_routing(r, blockIdx.x, k, lane, best, best_i);
}

// ------------------------------------------------------------------------------------------ logits
constexpr int LOGIT_STEP = 128, LOGIT_STAGES = 6, LOGIT_TOKENS = 4, LOGIT_RUN = 16, LOGIT_BLOCKS = 8;
// The chain over a step: while a feature's multiply-add waits for the one before it (four cycles), the values of LOGIT_RUN features later are loaded. Written out with volatile
// instructions: left to itself the compiler loads next to the use, 13 cycles a feature.
struct LogitRun {
    float w[LOGIT_RUN], x[LOGIT_RUN];
    __device__ __forceinline__ void load(int i, uint32_t ws, uint32_t xt) {  // of feature i
        if (i % 4 == 0) asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[i]), "=f"(x[i + 1]), "=f"(x[i + 2]), "=f"(x[i + 3]) : "r"(xt + i * 4));
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w[i]) : "r"(ws + i * 128));
    }
    __device__ __forceinline__ void multiply(int i, float &acc) const { asm volatile("fma.rn.f32 %0, %1, %2, %0;" : "+f"(acc) : "f"(x[i]), "f"(w[i])); }
};
__device__ __forceinline__ float logit_step(float acc, uint32_t ws, uint32_t xt) {
    LogitRun even, odd;
#pragma unroll
    for (int i = 0; i < LOGIT_RUN; ++i) even.load(i, ws, xt);
#pragma unroll 1
    for (int r = 0; r < LOGIT_STEP; r += 2 * LOGIT_RUN) {  // few instructions: a launch meets them in no cache
        const uint32_t w1 = ws + LOGIT_RUN * 128, x1 = xt + LOGIT_RUN * 4;
#pragma unroll
        for (int i = 0; i < LOGIT_RUN; ++i) { even.multiply(i, acc); odd.load(i, w1, x1); }
        const bool more = r + 2 * LOGIT_RUN < LOGIT_STEP;  // the last time round: the first run again, which nobody uses
        ws = more ? w1 + LOGIT_RUN * 128 : ws;
        xt = more ? x1 + LOGIT_RUN * 4 : xt;
#pragma unroll
        for (int i = 0; i < LOGIT_RUN; ++i) { odd.multiply(i, acc); even.load(i, ws, xt); }
    }
    return acc;
}
// 32 columns of the gate by LOGIT_TOKENS tokens, one warp for each: one chain over ascending features per thread, one warp per scheduler. Bound by the chain's latency, four
// cycles a feature; the block's other warps make the rows of the next step floats and leave the turned copy that the products take.
// ROUTE: the blocks of a token group are a cluster, of up to LOGIT_BLOCKS; their logits meet in the first one's shared memory, where a warp picks a token's experts.
template <typename T, bool FOURS, bool ROUTE>
__global__ void __launch_bounds__(256) few_logits_kernel(const T *__restrict__ x, const float *__restrict__ Wg, int32_t tokens, int32_t d, int32_t n, int32_t k,
                                                         float *__restrict__ logits, const Routing r, bf16 *copy, int32_t dw, int32_t *clear, int32_t clear_count, int32_t *status) {
    // The experts' blocks may come as soon as there is room for them: they set up barriers and tables meanwhile and wait for this launch's end before they read of it.
    // 29.7 -> 27.8 us (1 token, 1024 x 4096), 36.6 -> 34.4 (24 tokens, 32 experts of 512 x 1024). L2 asked for the weights from there as well cost 2 to 3 us again.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    wait_previous_kernel();
    __shared__ float all[ROUTE ? LOGIT_TOKENS : 1][ROUTE ? LOGIT_BLOCKS * 32 : 1];
    __shared__ __align__(16) float xf[2][LOGIT_TOKENS][LOGIT_STEP];
    extern __shared__ __align__(16) char few_shared[];
    float *w = reinterpret_cast<float *>(few_shared);                           // [stage][LOGIT_STEP][32]
    T *xs = reinterpret_cast<T *>(w + LOGIT_STAGES * LOGIT_STEP * 32);          // [stage][LOGIT_TOKENS][LOGIT_STEP]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t col0 = blockIdx.x * 32, tok0 = blockIdx.y * LOGIT_TOKENS;
    const int32_t steps = (d + LOGIT_STEP - 1) / LOGIT_STEP;
    constexpr int XV = 16 / sizeof(T), XP = LOGIT_STEP / XV;  // a token's pieces of 16 bytes
    auto fetch = [&](int32_t s) {
        if (s < steps) {
            const int32_t k0 = s * LOGIT_STEP, at = s % LOGIT_STAGES;
            T *xd = xs + at * LOGIT_TOKENS * LOGIT_STEP;
            if (threadIdx.x < LOGIT_TOKENS * XP) {
                const int32_t t = threadIdx.x / XP, c = (threadIdx.x % XP) * XV;
                if (tok0 + t < tokens && k0 + c < d) copy16(xd + t * LOGIT_STEP + c, x + (int64_t)(tok0 + t) * d + k0 + c);
            }
            float *ws = w + at * LOGIT_STEP * 32;
            if constexpr (FOURS) {  // n is a multiple of four
                const int32_t c = (threadIdx.x & 7) * 4;
                if (col0 + c < n)
#pragma unroll
                    for (int32_t q = threadIdx.x >> 3; q < LOGIT_STEP; q += 32)
                        if (k0 + q < d) copy16(ws + q * 32 + c, Wg + (int64_t)(k0 + q) * n + col0 + c);
            } else {
                if (col0 + lane < n)
#pragma unroll 4
                    for (int32_t q = warp; q < LOGIT_STEP; q += 8)
                        if (k0 + q < d) copy4(ws + q * 32 + lane, Wg + (int64_t)(k0 + q) * n + col0 + lane);
            }
        }
        copies_commit();
    };
    // a step's rows as floats, and turned (by one block)
    auto convert = [&](int32_t s, int32_t from, int32_t threads) {
        const T *xd = xs + (s % LOGIT_STAGES) * LOGIT_TOKENS * LOGIT_STEP;
#pragma unroll 2
        for (int32_t i = threadIdx.x - from; i < LOGIT_TOKENS * LOGIT_STEP / 2; i += threads) {
            const int32_t t = i / (LOGIT_STEP / 2), c = i % (LOGIT_STEP / 2) * 2, at = s * LOGIT_STEP + c;
            const bool live = tok0 + t < tokens && at < d;  // d is even
            xf[s & 1][t][c] = live ? to_f32(xd[t * LOGIT_STEP + c]) : 0.0f;
            xf[s & 1][t][c + 1] = live ? to_f32(xd[t * LOGIT_STEP + c + 1]) : 0.0f;
            if (sizeof(T) == 2 && blockIdx.x == gridDim.x - 1 && tok0 + t < tokens && at < dw)
                *reinterpret_cast<uint32_t *>(copy + (int64_t)(tok0 + t) * dw + turned(at)) = live ? *reinterpret_cast<const uint32_t *>(xd + t * LOGIT_STEP + c) : 0u;
        }
    };
#pragma unroll 1
    for (int32_t s = 0; s < LOGIT_STAGES - 1; ++s) fetch(s);
    const int32_t block = blockIdx.y * gridDim.x + blockIdx.x, blocks = gridDim.x * gridDim.y;
    for (int32_t i = block * 256 + threadIdx.x; i < clear_count; i += blocks * 256) clear[i] = 0;
    if (block == 0 && threadIdx.x == 0) *status = 0;
    const bool live = warp < LOGIT_TOKENS && tok0 + warp < tokens;
    copies_wait<LOGIT_STAGES - 2>();
    __syncthreads();
    convert(0, 0, 256);
    float acc = 0.0f;
#pragma unroll 1
    for (int32_t s = 0; s < steps; ++s) {
        copies_wait<LOGIT_STAGES - 3>();  // the step after this one too
        __syncthreads();
        fetch(s + LOGIT_STAGES - 1);  // where step s - 1 was
        if (warp >= 4) {
            if (s + 1 < steps) convert(s + 1, 128, 128);
        } else if (live) {
            const float *ws = w + (s % LOGIT_STAGES) * LOGIT_STEP * 32 + lane, *xt = xf[s & 1][warp];
            const int32_t left = min(LOGIT_STEP, d - s * LOGIT_STEP);
            if (left == LOGIT_STEP) {
                acc = logit_step(acc, smem_u32(ws), smem_u32(xt));
            } else {
#pragma unroll 4
                for (int i = 0; i < left; ++i) acc = fmaf(xt[i], ws[i * 32], acc);
            }
        }
    }
    if constexpr (ROUTE) {
        if (warp < LOGIT_TOKENS) {
            const uint32_t to = peer_smem_addr(smem_u32(&all[warp][col0 + lane]), 0);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(acc) : "memory");
        }
        cluster_sync_all();
        if (blockIdx.x > 0 || !live) return;
        uint32_t key[LOGIT_BLOCKS], best;
        int32_t best_i;
#pragma unroll
        for (int i = 0; i < LOGIT_BLOCKS; ++i) key[i] = 32 * i + lane < n ? ordered(all[warp][32 * i + lane]) : 0;
        take_best(k, key, 0, 0u, INT32_MAX, lane, best, best_i);
        put_routing(r, tok0 + warp, k, lane, best, best_i);
    } else if (live && col0 + lane < n) {
        logits[(int64_t)(tok0 + warp) * n + col0 + lane] = acc;
    }
}

// ------------------------------------------------------------------------------------------ experts
struct FewShared {
    uint64_t full[FEW_WARPS][3];
    int32_t abort, segments, scan[FEW_WARPS];
    float gate[MAX_ROWS];                                   // of a slot
    int16_t rows[MAX_ROWS];                                 // slots by expert
    int16_t seg_expert[MAX_ROWS], seg_first[MAX_ROWS], seg_count[MAX_ROWS];
    int32_t known_ready[MAX_ROWS];                          // a warp of this block has seen a segment's hid complete
    int32_t queue[FEW_WARPS][8];                            // a warp's tasks from the one at hand to the one whose tiles are being asked for
};
// Tables by expert, in the place of the rings before the first copy: the tokens that have picked it, a bit each; where its rows begin
struct FewTables {
    uint2 tokens[MOE_MAX_EXPERTS];
    int16_t start[MOE_MAX_EXPERTS];
};
static_assert(sizeof(FewTables) <= FEW_WARPS * WARP_BYTES, "they fit");
static_assert(WARP_BYTES / TILE_BYTES + 2 <= 8, "tasks between the two");
static_assert(MOE_FEW_MAX_TOKENS <= 64, "a bit for a token");
constexpr int FEW_SMEM = FEW_WARPS * WARP_BYTES + 1024 + (int)sizeof(FewShared);

__device__ __forceinline__ int32_t load_relaxed(const int32_t *p) {
    int32_t v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
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

// The segments: the experts in use by their first slots, an expert's slots in ascending order, 16 of them at most in a segment. The same in every block. By the whole block.
__device__ __forceinline__ void make_segments(const Few &a, FewShared &S, FewTables &tab, int warp, int lane) {
    const int32_t R = a.T * a.k, tid = threadIdx.x;
    // two slots a thread
    int32_t e[2], token[2], none;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int32_t p = 2 * tid + i;
        token[i] = a.by_k(p, none);
        e[i] = -1;
        if (p >= R) continue;
        e[i] = __ldg(a.idx + p);
        const float g = __ldg(a.gates + p);
        const bool known = (uint32_t)e[i] < (uint32_t)a.n;  // always, but for a gate of a launch that gave up
        MOE_BOUNDS_NOTE(known);
        e[i] = known ? e[i] : 0;
        S.gate[p] = g;
        atomicOr(token[i] < 32 ? &tab.tokens[e[i]].x : &tab.tokens[e[i]].y, 1u << (token[i] & 31));
    }
    __syncthreads();
    int32_t size[2], pos[2];  // rows (low half) and segments, each expert's at its first slot
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        size[i] = pos[i] = 0;
        if (e[i] < 0) continue;
        const uint2 who = tab.tokens[e[i]];
        const uint32_t below = (1u << (token[i] & 31)) - 1;
        pos[i] = token[i] < 32 ? __popc(who.x & below) : __popc(who.x) + __popc(who.y & below);
        const int32_t count = __popc(who.x) + __popc(who.y);
        if (pos[i] == 0) size[i] = count + (((count + SEG_ROWS - 1) / SEG_ROWS) << 16);
    }
    const int32_t sum = size[0] + size[1];
    int32_t before = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int32_t o = __shfl_up_sync(0xffffffffu, before, off);
        if (lane >= off) before += o;
    }
    if (lane == 31) S.scan[warp] = before;
    __syncthreads();
    before -= sum;
#pragma unroll
    for (int w = 0; w < FEW_WARPS; ++w) before += w < warp ? S.scan[w] : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int32_t count = size[i] & 0xffff, first = before & 0xffff;
        if (size[i]) {
            tab.start[e[i]] = (int16_t)first;
#pragma unroll 1
            for (int32_t q = 0, g = before >> 16; q < count; q += SEG_ROWS, ++g) {
                S.seg_expert[g] = (int16_t)e[i];
                S.seg_first[g] = (int16_t)(first + q);
                S.seg_count[g] = (int16_t)min(SEG_ROWS, count - q);
            }
        }
        before += size[i];
    }
    if (tid == FEW_THREADS - 1) S.segments = before >> 16;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (e[i] >= 0) S.rows[tab.start[e[i]] + pos[i]] = (int16_t)(2 * tid + i);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tables' place belongs to the copies from here on
    __syncthreads();
}

struct Task {
    int32_t segment, col, piece, k0, tiles;
    bool second;
};
__device__ __forceinline__ Task task_of(const Few &a, int32_t segments, int32_t number) {
    Task t;
    int32_t rest;
    const int32_t first = segments * (int32_t)a.by_task1.d;
    t.second = number >= first;
    t.segment = t.second ? a.by_task2(number - first, rest) : a.by_task1(number, rest);
    t.col = t.second ? a.by_pieces2(rest, t.piece) : a.by_pieces1(rest, t.piece);
    const int32_t tiles = t.second ? a.piece_tiles2 : a.piece_tiles1;
    t.k0 = t.piece * tiles * TILE_K;
    t.tiles = min(tiles, ((t.second ? a.h : a.d) - t.k0 + TILE_K - 1) / TILE_K);
    return t;
}

__device__ __forceinline__ void ldmatrix_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 two = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&two);
}
// what two floats are more than their bf16 terms; 0, not the NaN of a difference, beside an infinity
__device__ __forceinline__ uint32_t rest(uint32_t hi, float a, float b) {
    const float h0 = __uint_as_float(hi << 16), h1 = __uint_as_float(hi & 0xffff0000u);
    return pack(fabsf(h0) <= FLT_MAX ? a - h0 : 0.0f, fabsf(h1) <= FLT_MAX ? b - h1 : 0.0f);
}

// A warp's ring
struct Stream {
    uint32_t ring, bars;          // shared memory addresses
    int32_t flying, ask_slot, use_slot, phase;
    int32_t number, next;         // the task whose tiles are being asked for; the one behind it (lane 0: drawn, maybe still on its way), or
    bool drawn;                   // not drawn yet: a warp draws when it begins to multiply, so that one that waits holds no task that another could do
    int32_t left, tasks;          // tiles of that task that have not been asked for; tasks so far
    int32_t x, k, expert;         // where its next tile is
    bool second;
};

template <typename T> struct Worker {
    static constexpr int COLS = 128 / (int)sizeof(T);
    static constexpr bool BF16 = sizeof(T) == 2;
    static constexpr int RING = BF16 ? 3 : 2;
    static_assert(SEG_ROWS * TILE_K * 4 * 2 == TILE_BYTES, "two tiles of rows in the place of one of weights");
    const Few &a;
    FewShared &S;
    const CUtensorMap *w1, *w2;
    const int warp, lane;
    const int32_t segments, total;
    Stream s;

    __device__ __forceinline__ Worker(const Few &a_, FewShared &S_, const CUtensorMap *w1_, const CUtensorMap *w2_, uint32_t ring, int32_t first, int warp_, int lane_)
        : a(a_), S(S_), w1(w1_), w2(w2_), warp(warp_), lane(lane_), segments(S_.segments), total(S_.segments * (a_.cols1 * a_.pieces1 + a_.cols2 * a_.pieces2)) {
        s.ring = ring + warp * WARP_BYTES;
        s.bars = smem_u32(&S.full[warp][0]);
        s.flying = s.ask_slot = s.use_slot = s.phase = s.tasks = s.left = 0;
        s.number = 0;
        s.next = first;
        s.drawn = true;
#pragma unroll 1
        do ask();
        while (s.flying < RING && s.left > 0);
    }
    __device__ __forceinline__ void draw() {
        if (s.drawn || s.number >= total) return;
        s.next = lane == 0 ? atomicAdd(a.ticket, 1) : 0;
        s.drawn = true;
    }
    __device__ __forceinline__ int32_t token_of(int32_t p) const {
        int32_t none;
        return a.by_k(p, none);
    }
    // asks for one more tile, if there is one
    __device__ __forceinline__ void ask() {
        if (s.left == 0) {
            if (!s.drawn) return;
            s.drawn = false;
            s.number = __shfl_sync(0xffffffffu, s.next, 0);
            if (lane == 0) S.queue[warp][s.tasks % 8] = s.number;
            __syncwarp();
            ++s.tasks;
            if (s.number >= total) return;
            const Task t = task_of(a, segments, s.number);
            s.left = t.tiles;
            s.x = t.col * 64;
            s.k = t.k0;
            s.expert = S.seg_expert[t.segment];
            s.second = t.second;
        }
        if (lane == 0) {
            const uint32_t bar = s.bars + s.ask_slot * 8;
            mbar_expect_tx(bar, TILE_BYTES);
            tma_load_3d(s.ring + s.ask_slot * TILE_BYTES, s.second ? w2 : w1, bar, s.x, s.k, s.expert);
        }
        --s.left;
        s.k += TILE_K;
        s.ask_slot = s.ask_slot + 1 == RING ? 0 : s.ask_slot + 1;
        ++s.flying;
    }
    __device__ __forceinline__ bool arrived() {
        const bool ok = mbar_wait(s.bars + s.use_slot * 8, s.phase, &S.abort, a.status);
        return __all_sync(0xffffffffu, ok);
    }
    __device__ __forceinline__ uint32_t tile() const { return s.ring + s.use_slot * TILE_BYTES; }
    __device__ __forceinline__ void use_next() {
        --s.flying;
        s.phase ^= s.use_slot + 1 == RING;
        s.use_slot = s.use_slot + 1 == RING ? 0 : s.use_slot + 1;
    }
    __device__ __forceinline__ void release() {  // the tile at hand has been read
        __syncwarp();
        use_next();
#pragma unroll 1
        do ask();
        while (s.flying < RING && s.left > 0);
    }
    // nothing may be on its way into shared memory that is given back
    __device__ void give_up() {
#pragma unroll 1
        for (; s.flying > 0; use_next()) {
            const unsigned long long t0 = global_ns();
            while (!mbar_try_wait(s.bars + s.use_slot * 8, s.phase) && global_ns() - t0 < WAIT_LIMIT_NS) {}
        }
        copies_wait<0>();
    }
    __device__ bool wait_ready(int32_t segment) {
        bool ok = true;
        int32_t known;  // what the other warp has acquired reaches this one through the block's memory
        asm volatile("ld.acquire.cta.shared.s32 %0, [%1];" : "=r"(known) : "r"(smem_u32(&S.known_ready[segment])) : "memory");
        if (__all_sync(0xffffffffu, known)) return true;
        if (lane == 0) {
            unsigned long long t0 = 0;
            while (load_relaxed(a.ready + segment * READY_STEP) < a.cols1) {
                __nanosleep(100);  // a thousand warps that look at one place hold up those who count there
                const unsigned long long now = global_ns();
                if (t0 == 0) t0 = now;
                if (*(volatile int32_t *)&S.abort) { ok = false; break; }
                if (now - t0 > WAIT_LIMIT_NS) {
                    *(volatile int32_t *)&S.abort = 1;
                    atomicExch(a.status, (int32_t)MOE_ERR_TIMEOUT);
                    ok = false;
                    break;
                }
            }
        }
        __threadfence();
        ok = __all_sync(0xffffffffu, ok);
        if (ok && lane == 0) asm volatile("st.release.cta.shared.s32 [%0], %1;" ::"r"(smem_u32(&S.known_ready[segment])), "r"(1) : "memory");
        return ok;
    }

    // hid of one row, four columns of it, from its sums
    __device__ __forceinline__ void put_hid(int32_t expert, int32_t p, int32_t col, float4 f) {
        float v[4] = {f.x, f.y, f.z, f.w};
        const T *b = static_cast<const T *>(a.b1) + (int64_t)expert * a.h + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // h is a multiple of four
            v[i] += col < a.h ? to_f32(b[i]) : 0.0f;
            v[i] = v[i] < 0.0f || col >= a.h ? 0.0f : v[i];  // a NaN stays
        }
        if constexpr (BF16) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                bf16 *at = a.hid_hi + (int64_t)p * a.hw + turned(col + i);
                const uint32_t hi = pack(v[i], v[i + 1]);
                *reinterpret_cast<uint32_t *>(at) = hi;
                *reinterpret_cast<uint32_t *>(at + a.hid_lo_at) = rest(hi, v[i], v[i + 1]);
            }
        } else if (col < a.h) {
            *reinterpret_cast<float4 *>(a.hid + (int64_t)p * a.h + col) = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
    // What comes behind a task's sums, which are in parts1 / parts2 (or, a hid of one piece, in hid). Sums of pieces are bound by the latency of their loads: a lane
    // has eight or more in flight.
    __device__ __forceinline__ void finish(const Task &t, const int16_t *rows, int32_t m, int32_t expert) {
        __syncwarp();
        constexpr int PER = COLS / 4, SIDES = 32 / PER;  // lanes for a row's columns, four each; rows (hid) or pieces (y) side by side
        const int32_t col = t.col * COLS + lane % PER * 4, side = lane / PER;
        const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        constexpr int B = 8;
        if (!t.second) {
            if (a.pieces1 > 1) {
                int32_t last = 0;
                if (lane == 0) last = add_acq_rel(a.done1 + t.segment * a.cols1 + t.col, 1) == a.pieces1 - 1;
                if (!__shfl_sync(0xffffffffu, last, 0)) return;
#pragma unroll 1
                for (int32_t q = side; q < m; q += SIDES) {
                    const int32_t hid_cols = a.h;
                    const float *from = a.parts1 + (int64_t)rows[q] * a.pieces1 * a.h + col;
                    float4 v = zero;
#pragma unroll 1
                    for (int32_t z = 0; z < a.pieces1; z += B) {
                        float4 f[B];
#pragma unroll
                        for (int i = 0; i < B; ++i) f[i] = col < hid_cols && z + i < a.pieces1 ? __ldcg(reinterpret_cast<const float4 *>(from + (int64_t)(z + i) * a.h)) : zero;
#pragma unroll
                        for (int i = 0; i < B; ++i) { v.x += f[i].x; v.y += f[i].y; v.z += f[i].z; v.w += f[i].w; }
                    }
                    put_hid(expert, rows[q], col, v);
                }
                __syncwarp();
            }
            if (lane == 0) add_release(a.ready + t.segment * READY_STEP, 1);
            return;
        }
        // y = sum over a token's slots and pieces of gate * part, by whoever delivers the last piece of its columns: two tokens at a time, a side of the warp every SIDES-th part
        bool last = false;
        if (lane < m) last = add_acq_rel(a.done2 + token_of(rows[lane]) * a.cols2 + t.col, 1) == a.k * a.pieces2 - 1;
        uint32_t todo = __ballot_sync(0xffffffffu, last);
        const int32_t parts = a.k * a.pieces2;
        const int64_t stride = (int64_t)parts * a.d;  // a token's slots and their pieces stand one behind the other
#pragma unroll 1
        while (todo) {
            int32_t token[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                token[i] = todo ? token_of(rows[__ffs(todo) - 1]) : -1;
                todo &= todo - 1;
            }
            float y[2][4];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i / 4][i % 4] = 0.0f;
#pragma unroll 1
            for (int32_t j0 = side; j0 < parts; j0 += SIDES * B) {
                float4 f[2][B];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < B; ++e)
                        f[i][e] = token[i] >= 0 && col < a.d && j0 + e * SIDES < parts
                                      ? __ldcg(reinterpret_cast<const float4 *>(a.parts2 + token[i] * stride + (int64_t)(j0 + e * SIDES) * a.d + col)) : zero;
#pragma unroll
                for (int e = 0; e < B; ++e) {
                    int32_t none;
                    const int32_t slot = a.by_pieces2(min(j0 + e * SIDES, parts - 1), none);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (token[i] < 0 || j0 + e * SIDES >= parts) continue;
                        const float gate = S.gate[token[i] * a.k + slot];
                        y[i][0] = fmaf(gate, f[i][e].x, y[i][0]);
                        y[i][1] = fmaf(gate, f[i][e].y, y[i][1]);
                        y[i][2] = fmaf(gate, f[i][e].z, y[i][2]);
                        y[i][3] = fmaf(gate, f[i][e].w, y[i][3]);
                    }
                }
            }
            __syncwarp();
#pragma unroll
            for (int off = PER; off < 32; off <<= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i / 4][i % 4] += __shfl_xor_sync(0xffffffffu, y[i / 4][i % 4], off);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (token[i] < 0 || side > 0 || col >= a.d) continue;
                T *to = static_cast<T *>(a.y) + (int64_t)token[i] * a.d + col;  // widths are multiples of four
                if constexpr (BF16) *reinterpret_cast<uint2 *>(to) = make_uint2(pack(y[i][0], y[i][1]), pack(y[i][2], y[i][3]));
                else *reinterpret_cast<float4 *>(to) = make_float4(y[i][0], y[i][1], y[i][2], y[i][3]);
            }
        }
    }
    // where a row's sums of this task go
    __device__ __forceinline__ float *part_of(const Task &t, int32_t p) const {
        return t.second ? a.parts2 + ((int64_t)p * a.pieces2 + t.piece) * a.d : a.parts1 + ((int64_t)p * a.pieces1 + t.piece) * a.h;
    }

    // bf16: half a tile at a time, 32 k by 64 columns, by up to NT x 8 rows. Short code for both kinds of task: what a launch executes it has to fetch first, and fetching
    // unrolled tiles was a third of a call of 24 tokens.
    __device__ __forceinline__ bool run_bf16(const Task &t, const int16_t *rows, int32_t m, int32_t expert) {
        const int g = lane >> 2, c = lane & 3;
        const int32_t out = t.second ? a.d : a.h;
        const bool whole = !t.second && a.pieces1 == 1, more = m > 8;
        const bf16 *row[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int32_t p = rows[min(u * 8 + g, m - 1)];  // lanes without a row: copies whose results are dropped
            row[u] = (t.second ? a.hid_hi + (int64_t)p * a.hw : static_cast<const bf16 *>(a.x) + (int64_t)token_of(p) * a.dw) + t.k0 + 8 * c;
        }
        float bias[8];  // of the lane's columns, on its way during the products; b2 goes with the first piece
        {
            const T *b = (t.second ? static_cast<const T *>(a.b2) + (int64_t)expert * a.d : static_cast<const T *>(a.b1) + (int64_t)expert * a.h) + t.col * 64 + g;
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = (whole || (t.second && t.piece == 0)) && t.col * 64 + g + e * 8 < out ? to_f32(b[e * 8]) : 0.0f;
        }
        // a lane's rows of the weights: row r of matrix mat holds lane r / 2's pair 2 s + mat / 2, element r % 2
        uint32_t at[2][4];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int r = lane & 7, mat = lane >> 3, lc = r >> 1, k = 8 * lc + 2 * ((2 * s + (mat >> 1) + lc) & 3) + (r & 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) at[s][q] = k * 128 + (((2 * q + (mat & 1)) ^ (k & 7)) << 4);
        }
        float acc[4][NT][4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[q][u][i] = 0.0f;
        struct Half { uint4 hi[NT], lo[NT]; };
        auto fetch = [&](Half &h) {  // from L2: hid is written by other blocks of this launch
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                if (u > 0 && !more) break;
                h.hi[u] = __ldcg(reinterpret_cast<const uint4 *>(row[u]));
                if (t.second) h.lo[u] = __ldcg(reinterpret_cast<const uint4 *>(row[u] + a.hid_lo_at));
                row[u] += 32;
            }
        };
        Half now, next;
        fetch(now);
        fetch(next);
#pragma unroll 1
        for (int32_t half = 0; half < 2 * t.tiles; ++half) {
            if (half % 2 == 0 && !arrived()) return false;
            const Half h = now;
            now = next;
            fetch(next);  // two halves ahead
            // all of the weights first, then products that do not need each other: one behind the other each waits for the one before, 1.2 us a tile
            uint32_t w[2][4][4];
            const uint32_t base = tile() + half % 2 * (32 * 128);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int q = 0; q < 4; ++q) ldmatrix_t(w[s][q], base + at[s][q]);
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                if (u > 0 && !more) break;
                const uint32_t hi[4] = {h.hi[u].x, h.hi[u].y, h.hi[u].z, h.hi[u].w}, lo[4] = {h.lo[u].x, h.lo[u].y, h.lo[u].z, h.lo[u].w};
                if (t.second)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int q = 0; q < 4; ++q) mma_16x8x16(acc[q][u], w[s][q], lo[2 * s], lo[2 * s + 1]);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma_16x8x16(acc[q][u], w[s][q], hi[2 * s], hi[2 * s + 1]);
            }
            if (half % 2) release();
        }
        // columns t.col * 64 + 8 e + g of rows 8 u + 2 c + i
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (u > 0 && !more) break;
                const int32_t q = u * 8 + 2 * c + i, p = rows[min(q, m - 1)];
                if (whole) {  // neighbours of a pair of columns: the even one stores the first terms, the odd one the second
                    bf16 *to = a.hid_hi + (int64_t)p * a.hw + t.col * 64 + (g & 1 ? a.hid_lo_at : 0);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float v = acc[e >> 1][u][2 * (e & 1) + i] + bias[e];
                        v = v < 0.0f || t.col * 64 + e * 8 + g >= out ? 0.0f : v;  // a NaN stays
                        const float other = __shfl_xor_sync(0xffffffffu, v, 4), v0 = g & 1 ? other : v, v1 = g & 1 ? v : other;
                        const uint32_t hi = pack(v0, v1), word = g & 1 ? rest(hi, v0, v1) : hi;
                        if (q < m) *reinterpret_cast<uint32_t *>(to + turned(e * 8 + (g & 6))) = word;
                    }
                } else if (q < m) {
                    float *part = part_of(t, p) + t.col * 64 + g;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (t.col * 64 + e * 8 + g < out) part[e * 8] = acc[e >> 1][u][2 * (e & 1) + i] + bias[e];
                }
            }
        return true;
    }

    // Float: a lane has four columns and every fourth run of four k. The rows' values are copied a tile ahead (loaded where they are used, each load was waited for: 117 us for
    // 15 tokens of 13 experts of 1288 x 1696, of k = 4)
    __device__ __forceinline__ bool run_f32(const Task &t, const int16_t *rows, int32_t m, int32_t expert) {
        const int cg = lane & 7, ph = lane >> 3;
        const int32_t width = t.second ? a.h : a.d;
        const float *x = t.second ? a.hid : static_cast<const float *>(a.x);
        char *const mine = static_cast<char *>(__cvta_shared_to_generic(s.ring));
        float *const xs = reinterpret_cast<float *>(mine + RING * TILE_BYTES);  // [2][SEG_ROWS][TILE_K]
        auto copy = [&](int32_t i) {
            if (i < t.tiles) {
                const int32_t k = t.k0 + i * TILE_K + (lane & 15) * 4;
#pragma unroll 1
                for (int q = lane >> 4; q < m; q += 2) {
                    const int32_t p = rows[q], row = t.second ? p : token_of(p);
                    copy16(xs + (i % 2 * SEG_ROWS + q) * TILE_K + (lane & 15) * 4, x + (k < width ? (int64_t)row * width + k : 0), k < width);
                }
            }
            copies_commit();
        };
        float acc[NT * 8][4];
#pragma unroll
        for (int q = 0; q < NT * 8; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[q][i] = 0.0f;
        copy(0);
        for (int32_t i = 0; i < t.tiles; ++i) {
            copy(i + 1);
            copies_wait<1>();
            if (!arrived()) return false;  // and all lanes' copies
            const char *at = mine + s.use_slot * TILE_BYTES;
#pragma unroll 1
            for (int j = 0; j < TILE_K / 16; ++j) {
                const int kk = 16 * j + 4 * ph;
                const float *from = xs + i % 2 * (SEG_ROWS * TILE_K) + kk;
                float4 w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = *reinterpret_cast<const float4 *>(at + (kk + e) * 128 + ((cg ^ ((kk + e) & 7)) << 4));
#pragma unroll
                for (int q = 0; q < NT * 8; ++q) {
                    if (q >= m) break;
                    const float4 v = *reinterpret_cast<const float4 *>(from + q * TILE_K);
                    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        fma_two(acc[q][0], acc[q][1], f[c], w[c].x, w[c].y);
                        fma_two(acc[q][2], acc[q][3], f[c], w[c].z, w[c].w);
                    }
                }
            }
            release();
        }
        const int32_t col = t.col * COLS + 4 * cg;
        const bool whole = !t.second && a.pieces1 == 1;
#pragma unroll
        for (int q = 0; q < NT * 8; ++q) {
            if (q >= m) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[q][i] += __shfl_xor_sync(0xffffffffu, acc[q][i], 8);
                acc[q][i] += __shfl_xor_sync(0xffffffffu, acc[q][i], 16);
            }
            if (q % 4 != ph || col >= (t.second ? a.d : a.h)) continue;  // widths are multiples of four
            const int32_t p = rows[q];
            float4 v = make_float4(acc[q][0], acc[q][1], acc[q][2], acc[q][3]);
            if (whole) {
                put_hid(expert, p, col, v);
                continue;
            }
            if (t.second && t.piece == 0) {  // b2 goes with the first piece
                const float *b = static_cast<const float *>(a.b2) + (int64_t)expert * a.d + col;
                v.x += b[0]; v.y += b[1]; v.z += b[2]; v.w += b[3];
            }
            *reinterpret_cast<float4 *>(part_of(t, p) + col) = v;
        }
        return true;
    }

    __device__ __forceinline__ bool run(int32_t number) {
        const Task t = task_of(a, segments, number);
        const int16_t *rows = S.rows + S.seg_first[t.segment];
        const int32_t m = S.seg_count[t.segment], expert = S.seg_expert[t.segment];
        if (t.second && !wait_ready(t.segment)) return false;
        draw();
        bool ok;
        if constexpr (BF16) ok = run_bf16(t, rows, m, expert);
        else ok = run_f32(t, rows, m, expert);
        if (ok) finish(t, rows, m, expert);
        return ok;
    }
};

template <typename T>
__global__ void __launch_bounds__(FEW_THREADS, 1) few_experts_kernel(const __grid_constant__ CUtensorMap w1, const __grid_constant__ CUtensorMap w2, const Few a) {
    extern __shared__ char few_raw[];
    char *base = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(few_raw) + 1023) & ~uintptr_t(1023));
    FewShared &S = *reinterpret_cast<FewShared *>(base + FEW_WARPS * WARP_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < FEW_WARPS * 3; ++i) mbar_init(smem_u32(&S.full[0][i]), 1);
        S.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    FewTables &tab = *reinterpret_cast<FewTables *>(base);
    for (int32_t i = threadIdx.x; i < a.n; i += FEW_THREADS) tab.tokens[i] = make_uint2(0u, 0u);
    for (int32_t i = threadIdx.x; i < MAX_ROWS; i += FEW_THREADS) S.known_ready[i] = 0;
    if (threadIdx.x < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(threadIdx.x ? &w2 : &w1) : "memory");
    wait_previous_kernel();
    const int32_t first = lane == 0 ? atomicAdd(a.ticket, 1) : 0;  // on its way meanwhile
    make_segments(a, S, tab, warp, lane);

    // From here on a warp is by itself. It takes the tasks in the order in which it has drawn them; tiles of the next ones are asked for as places in the ring get free.
    Worker<T> work(a, S, &w1, &w2, smem_u32(base), first, warp, lane);
    for (int32_t i = 0;; ++i) {
        if (i == work.s.tasks) work.ask();  // a task of so few tiles that the next was not asked for
        const int32_t number = S.queue[warp][i % 8];
        if (number >= work.total) break;
        if (!work.run(number)) {
            work.give_up();
            break;
        }
    }
}

struct FewPlan {
    int32_t cols1, pieces1, piece_tiles1, cols2, pieces2, piece_tiles2;
    int64_t done1, done2, counters;
};
// Pieces of a contraction of `tiles` tiles for `cols` tiles of columns of `segments` experts: at most six tasks for every SM, whose rings together keep memory busy, and none of
// more than `most` tiles. Among these the number for which a task's tiles and the sum of the pieces behind the last of them take least: `each` pieces of the sum are read at a time, by
// turns of TURN tiles' time.
#ifndef TURN
#define TURN 1.0
#endif
void pieces_of(int64_t segments, int64_t cols, int64_t tiles, int64_t most, int64_t turns, int64_t each, int64_t sums, int32_t *pieces, int32_t *piece_tiles) {
    const int64_t least = cdiv(tiles, most), highest = imax(least, imin(tiles, cdiv(6 * 148, segments * cols)));
    int64_t best = 0;
    for (int64_t n = highest; n >= least; --n) {
        const int64_t of = cdiv(tiles, n), now = cdiv(tiles, of);
        const int64_t cost = of + turns * cdiv(sums * now, each);
        if (n < highest && cost >= best) continue;
        best = cost;
        *piece_tiles = (int32_t)of;
        *pieces = (int32_t)now;
    }
}
FewPlan plan_of(const moe_config &c) {
    FewPlan p;
    const int64_t width = 128 / (int64_t)act_bytes(c.act), R = (int64_t)c.T * c.k;
    // experts that some token picks, if it picks any k of them alike
    const double used = c.n * (1.0 - pow(1.0 - (double)c.k / c.n, c.T));
    const int64_t segments = imax(1, imin(R, (int64_t)(used + 0.5)));
    p.cols1 = (int32_t)cdiv(c.h, width);
    p.cols2 = (int32_t)cdiv(c.d, width);
    const int64_t turns = cdiv(imin(SEG_ROWS, cdiv(R, segments)), 2);  // of a segment's rows, two at a time
    pieces_of(segments, p.cols1, cdiv(c.d, TILE_K), 16, turns, 8, 1, &p.pieces1, &p.piece_tiles1);
    pieces_of(segments, p.cols2, cdiv(c.h, TILE_K), 8, turns, 16, c.k, &p.pieces2, &p.piece_tiles2);
    p.done1 = 64 + R * READY_STEP;  // behind the ticket and the segments' columns
    p.done2 = p.done1 + (p.pieces1 > 1 ? R * p.cols1 : 0);
    p.counters = p.done2 + (int64_t)c.T * p.cols2;
    return p;
}

struct FewWs {
    int32_t *status, *counters;
    float *logits, *hid, *parts1, *parts2, *gates;
    bf16 *copy, *hid_hi;
    int64_t dw, hw, hid_lo_at;
    int32_t *idx;
    size_t bytes;
    FewWs(void *ws, const moe_config &c, const FewPlan &p) {
        Carver cv(ws);
        status = static_cast<int32_t *>(cv.take_bytes(kWsHeader));
        const int64_t R = (int64_t)c.T * c.k;
        counters = cv.take<int32_t>(p.counters);
        idx = cv.take<int32_t>(R);
        gates = cv.take<float>(R);
        logits = cv.take<float>(c.n > LOGIT_BLOCKS * 32 ? (int64_t)c.T * c.n : 0);
        dw = cdiv(c.d, TILE_K) * TILE_K;
        hw = cdiv(c.h, TILE_K) * TILE_K;
        hid_lo_at = R * hw;
        const bool two = c.act == MOE_BF16;
        copy = cv.take<bf16>(two ? (int64_t)c.T * dw + ROW_SLACK : 0);
        hid_hi = cv.take<bf16>(two ? 2 * R * hw + ROW_SLACK : 0);
        hid = cv.take<float>(two ? 0 : R * c.h);
        parts1 = cv.take<float>(p.pieces1 > 1 ? R * p.pieces1 * c.h : 0);
        parts2 = cv.take<float>(R * p.pieces2 * c.d);
        bytes = cv.off;
    }
};

// [n, K, N] as 16-bit elements: boxes of 64 k by 128 bytes of columns
int32_t weight_map(CUtensorMap *map, const void *w, int64_t n, int64_t K, int64_t N, int32_t act) {
    const uint64_t row = (uint64_t)N * act_bytes(act), dims[3] = {row / 2, (uint64_t)K, (uint64_t)n}, strides[2] = {row, row * (uint64_t)K};
    const uint32_t box[3] = {64, TILE_K, 1};
    return tc_make_map(map, w, 3, dims, strides, box);
}

template <typename T, bool FOURS, bool ROUTE>
int32_t launch_logits(const moe_config &c, const void *x, const float *Wg, const FewWs &w, const FewPlan &p, const Routing &r, cudaStream_t st) {
    constexpr int bytes = LOGIT_STAGES * (LOGIT_STEP * 32 * 4 + LOGIT_TOKENS * LOGIT_STEP * (int)sizeof(T));
    static PerDevice allowed;
    if (!allow_shared(allowed, few_logits_kernel<T, FOURS, ROUTE>, bytes)) return MOE_ERR_CUDA;
    const unsigned blocks = (unsigned)cdiv(c.n, 32);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ROUTE ? blocks : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, (unsigned)cdiv(c.T, LOGIT_TOKENS));
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaLaunchKernelEx(&cfg, few_logits_kernel<T, FOURS, ROUTE>, static_cast<const T *>(x), Wg, c.T, c.d, c.n, c.k, w.logits, r, w.copy, (int32_t)w.dw, w.counters, (int32_t)p.counters, w.status);
    MOE_LAUNCHED();
    return MOE_OK;
}
template <typename T> int32_t launch_routing(const moe_config &c, const void *x, const float *Wg, const FewWs &w, const FewPlan &p, const Routing &r, cudaStream_t st) {
    if (c.n <= LOGIT_BLOCKS * 32)
        return c.n % 4 == 0 ? launch_logits<T, true, true>(c, x, Wg, w, p, r, st) : launch_logits<T, false, true>(c, x, Wg, w, p, r, st);
    MOE_TRY(c.n % 4 == 0 ? (launch_logits<T, true, false>(c, x, Wg, w, p, r, st)) : (launch_logits<T, false, false>(c, x, Wg, w, p, r, st)));
    launch_kernel(few_select_kernel, dim3((unsigned)c.T), dim3(256), 0, st, (const float *)w.logits, c.n, c.k, r);
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

MOE_BOUNDS_READER(bounds_violations_few_tokens)

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
    a.x = c.act == MOE_BF16 ? (const void *)w.copy : x; a.b1 = b1; a.b2 = b2; a.hid = w.hid; a.hid_hi = w.hid_hi; a.hid_lo_at = w.hid_lo_at; a.dw = (int32_t)w.dw; a.hw = (int32_t)w.hw; a.y = y; a.idx = w.idx; a.gates = w.gates; a.parts1 = w.parts1; a.parts2 = w.parts2;
    a.ticket = w.counters; a.ready = w.counters + 64; a.done1 = w.counters + p.done1; a.done2 = w.counters + p.done2; a.status = w.status;
    a.T = c.T; a.d = c.d; a.h = c.h; a.n = c.n; a.k = c.k;
    a.cols1 = p.cols1; a.pieces1 = p.pieces1; a.piece_tiles1 = p.piece_tiles1; a.cols2 = p.cols2; a.pieces2 = p.pieces2; a.piece_tiles2 = p.piece_tiles2;
    a.by_k = Divisor::of(c.k); a.by_task1 = Divisor::of((int64_t)p.cols1 * p.pieces1); a.by_task2 = Divisor::of((int64_t)p.cols2 * p.pieces2);
    a.by_pieces1 = Divisor::of(p.pieces1); a.by_pieces2 = Divisor::of(p.pieces2);
    const Routing r = {w.idx, topk_idx, w.gates, gates};
    if (c.act == MOE_BF16) {
        MOE_TRY(launch_routing<bf16>(c, x, Wg, w, p, r, st));
        return launch_experts<bf16>(m1, m2, a, st);
    }
    MOE_TRY(launch_routing<float>(c, x, Wg, w, p, r, st));
    return launch_experts<float>(m1, m2, a, st);
}

}  // namespace moe
