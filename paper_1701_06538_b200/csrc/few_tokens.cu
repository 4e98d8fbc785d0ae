// The whole layer for a few tokens (serving): two launches, three with more than 256 experts. The experts' weights are read once, by tensor copies that run ahead
// of everything else, and that is what bounds it: a matrix of 512 x 1024 in bf16 is 1 MB for two or three rows.
//
//   few_logits_kernel   the logits of every token by the fixed chain of multiply-adds of moe_gate, and the second launch's counters set to 0. The blocks of four tokens are a
//                       cluster, whose first block gets all their logits and picks the experts (top k, softmax)
//   few_select_kernel   picks them from logits in memory, where a cluster does not hold the gate (more than 256 experts)
//   few_experts_kernel  one block per SM. Every block sorts the slots by expert; then its teams of warps draw tasks from a counter: an expert's rows (16 at most) and 64 hidden
//                       units. The team makes hid of those units, which nobody else needs, and its part of y from them. (Tasks for hid and tasks for y, hid handed over through
//                       memory: 27.8 us, not 21.3, for 1 token of 1024 x 4096, 35.4, not 24.4, for 24 tokens of 32 experts of 512 x 1024, of which a warp waited 3 to 7 us for hid
//                       and whoever came last summed up a token's y alone, for up to 7.) When all tasks are drawn, warps draw 16 columns of a token's y each, wait until its parts
//                       are there and add them up in order: results do not depend on who does what, and whoever waits, waits for blocks that are running.
//
// Every warp copies the 64 x 128-byte tiles that it will multiply into its own ring, on into the team's next task. Weights are the larger operand and the matrix instruction's rows,
// the tokens its columns, 8 at a time. Rows this few would leave most of a tcgen05 tile empty, and its accumulators would have to come back from tensor memory every few KB;
// mma.sync from shared memory keeps up with the copies. Code is kept short: what a launch executes it has to fetch first.
#include <float.h>
#include <stddef.h>
#include <math.h>
#include <math_constants.h>

#include "async_copy.cuh"
#include "block.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32;
constexpr int TILE_K = 64, TILE_BYTES = TILE_K * 128, RING = 2, SLICE = 64;  // SLICE: hidden units of a task's step
constexpr int WARP_BYTES = (RING + 1) * TILE_BYTES;                           // shared memory of a warp: its ring, and its sums of a slice or (float) two tiles of rows
constexpr int MAX_TEAMS = FEW_WARPS / 2;
constexpr int MAX_ROWS = MOE_FEW_MAX_TOKENS * MOE_MAX_K;
constexpr int SEG_ROWS = 16, NT = SEG_ROWS / 8;  // rows of a task: an expert with more is several segments, whose weights are read again, from L2

// bf16 rows that the matrix instruction takes (x, hid) stand as it wants them (turned()), x in a copy whose width is rounded up to tiles with zeros behind the last column.
// hid is kept in two bf16 terms (float layers: float): in one its rounding would cost as much accuracy as that of y.
// Read by ordinary loads throughout: this launch begins before the one that writes x, idx and gates has ended (and before what wrote the weights has), so nothing of it is read-only for
// as long as the launch runs, which is what non-coherent loads are for.
struct Few {
    const void *x, *b1, *b2;     // x: [T][d], of bf16 layers the turned copy [T][dw]
    void *y;
    const int32_t *idx;          // [T][k], and the gates
    const float *gates;
    float *parts;                // [R][units][d]
    int32_t *ticket, *final_ticket, *done;  // tasks drawn, pieces of y drawn; units that a token has
    int32_t *status;
    int32_t T, d, h, n, k, dw;
    int32_t team_warps;               // 2, 4 or 8
    int32_t slices, per_unit, units;  // of 64 hidden units an expert; slices of a task (a unit), units of an expert
    int32_t tiles1, tiles2, finals;   // tiles of a slice of W1 and W2; pieces of y of a token
    Divisor by_k, by_units, by_finals;
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
__global__ void __launch_bounds__(256) few_select_kernel(const float *logits, int32_t n, int32_t k, const Routing r) {
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
constexpr int LOGIT_STEP = 128, LOGIT_STAGES = 5, LOGIT_TOKENS = 4, LOGIT_RUN = 16, LOGIT_BLOCKS = 8;
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
__device__ __forceinline__ float logit_step(float acc, uint32_t ws, uint32_t xt, int32_t features) {  // a multiple of two runs
    LogitRun even, odd;
#pragma unroll
    for (int i = 0; i < LOGIT_RUN; ++i) even.load(i, ws, xt);
#pragma unroll 1
    for (int r = 0; r < features; r += 2 * LOGIT_RUN) {  // few instructions: a launch meets them in no cache
        const uint32_t w1 = ws + LOGIT_RUN * 128, x1 = xt + LOGIT_RUN * 4;
#pragma unroll
        for (int i = 0; i < LOGIT_RUN; ++i) { even.multiply(i, acc); odd.load(i, w1, x1); }
        const bool more = r + 2 * LOGIT_RUN < features;  // the last time round: the first run again, which nobody uses
        ws = more ? w1 + LOGIT_RUN * 128 : ws;
        xt = more ? x1 + LOGIT_RUN * 4 : xt;
#pragma unroll
        for (int i = 0; i < LOGIT_RUN; ++i) { odd.multiply(i, acc); even.load(i, ws, xt); }
    }
    return acc;
}
// 32 columns of the gate by LOGIT_TOKENS tokens, one warp for each: one chain over ascending features per thread, one warp per scheduler. Bound by the chain's latency, four
// cycles a feature; the block's other warps ask for later steps, make the rows of the next one floats and leave the turned copy that the products take.
// ROUTE: the blocks of a token group are a cluster, of up to LOGIT_BLOCKS; their logits meet in the first one's shared memory, where a warp picks a token's experts.
template <typename T, bool FOURS, bool ROUTE>
__global__ void __launch_bounds__(256) few_logits_kernel(const T *__restrict__ x, const float *__restrict__ Wg, int32_t tokens, int32_t d, int32_t n, int32_t k,
                                                         float *__restrict__ logits, const Routing r, bf16 *copy, int32_t dw, int32_t *clear, int32_t clear_count, int32_t *status) {
    // The experts' blocks may come as soon as there is room for them: they set up barriers and tables meanwhile and wait for this launch's end before they read of it
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    wait_previous_kernel();
    // The first block's shared memory may be written once it is known to run: all blocks say here that they do, and wait for the others behind the chain, where nobody waits any more
    if constexpr (ROUTE) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    __shared__ float all[ROUTE ? LOGIT_TOKENS : 1][ROUTE ? LOGIT_BLOCKS * 32 : 1];
    __shared__ __align__(16) float xf[2][LOGIT_TOKENS][LOGIT_STEP];
    extern __shared__ __align__(16) char few_shared[];
    float *w = reinterpret_cast<float *>(few_shared);                           // [stage][LOGIT_STEP][32]
    T *xs = reinterpret_cast<T *>(w + LOGIT_STAGES * LOGIT_STEP * 32);          // [stage][LOGIT_TOKENS][LOGIT_STEP]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t col0 = blockIdx.x * 32, tok0 = blockIdx.y * LOGIT_TOKENS;
    const int32_t steps = (d + LOGIT_STEP - 1) / LOGIT_STEP;
    constexpr int XV = 16 / sizeof(T), XP = LOGIT_STEP / XV;  // a token's pieces of 16 bytes
    auto fetch = [&](int32_t s, int32_t tid, int32_t threads) {
        if (s < steps && tid >= 0) {
            const int32_t k0 = s * LOGIT_STEP, at = s % LOGIT_STAGES;
            T *xd = xs + at * LOGIT_TOKENS * LOGIT_STEP;
            if (tid < LOGIT_TOKENS * XP) {
                const int32_t t = tid / XP, c = (tid % XP) * XV;
                if (tok0 + t < tokens && k0 + c < d) copy16(xd + t * LOGIT_STEP + c, x + (int64_t)(tok0 + t) * d + k0 + c);
            }
            float *ws = w + at * LOGIT_STEP * 32;
            if constexpr (FOURS) {  // n is a multiple of four
                const int32_t c = (tid & 7) * 4;
                if (col0 + c < n)
#pragma unroll 4
                    for (int32_t q = tid >> 3; q < LOGIT_STEP; q += threads >> 3)
                        if (k0 + q < d) copy16(ws + q * 32 + c, Wg + (int64_t)(k0 + q) * n + col0 + c);
            } else {
                if (col0 + lane < n)
#pragma unroll 4
                    for (int32_t q = tid >> 5; q < LOGIT_STEP; q += threads >> 5)
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
    for (int32_t s = 0; s < LOGIT_STAGES - 1; ++s) fetch(s, threadIdx.x, 256);
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
        fetch(s + LOGIT_STAGES - 1, threadIdx.x - 128, 128);  // where step s - 1 was, by the warps without a chain
        if (warp >= 4) {
            if (s + 1 < steps) convert(s + 1, 128, 128);
        } else if (live) {
            const float *ws = w + (s % LOGIT_STAGES) * LOGIT_STEP * 32 + lane, *xt = xf[s & 1][warp];
            const int32_t left = min(LOGIT_STEP, d - s * LOGIT_STEP);
            const int32_t runs = left & ~(2 * LOGIT_RUN - 1);
            if (runs) acc = logit_step(acc, smem_u32(ws), smem_u32(xt), runs);
#pragma unroll 4
            for (int32_t i = runs; i < left; ++i) acc = fmaf(xt[i], ws[i * 32], acc);
        }
    }
    if constexpr (ROUTE) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
constexpr int RED_STRIDE = 68, HID_STRIDE = 72;
struct FewShared {
    uint64_t full[FEW_WARPS][RING];
    int32_t next[MAX_TEAMS];                                // a team's next task
    int32_t abort, segments, scan[FEW_WARPS];
    float gate[MAX_ROWS];                                   // of a slot
    int16_t rows[MAX_ROWS];                                 // slots by expert
    int16_t seg_expert[MAX_ROWS], seg_first[MAX_ROWS], seg_count[MAX_ROWS];
    alignas(16) union {
        bf16 two[2][SEG_ROWS][HID_STRIDE];                  // hid of a slice, turned, in two terms
        float one[SEG_ROWS][RED_STRIDE];                    // float layers
    } hid[MAX_TEAMS];
};
static_assert(offsetof(FewShared, hid) % 16 == 0 && sizeof(((FewShared *)0)->hid[0]) % 16 == 0 && RED_STRIDE * 4 % 16 == 0 && HID_STRIDE * 2 % 16 == 0, "read 16 bytes at a time");
static_assert(SEG_ROWS * RED_STRIDE * 4 <= TILE_BYTES && SEG_ROWS * TILE_K * 4 * 2 == TILE_BYTES, "sums of a warp, or two tiles of rows, in the place of one of weights");
// Tables by expert, in the place of the rings before the first copy: the tokens that have picked it, a bit each; where its rows begin
struct FewTables {
    uint2 tokens[MOE_MAX_EXPERTS];
    int16_t start[MOE_MAX_EXPERTS];
};
static_assert(sizeof(FewTables) <= FEW_WARPS * WARP_BYTES, "they fit");
static_assert(MOE_FEW_MAX_TOKENS <= 64, "a bit for a token");
constexpr int FEW_SMEM = FEW_WARPS * WARP_BYTES + 1024 + (int)sizeof(FewShared);

__device__ __forceinline__ int32_t load_relaxed(const int32_t *p) {
    int32_t v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void add_release(int32_t *p, int32_t by) {
    asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(by) : "memory");
}
// barrier of a team's warps; whether any of them has p
__device__ __forceinline__ bool team_any(int team, int threads, bool p) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, %3, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)p), "r"(team + 1), "r"(threads) : "memory");
    return r != 0;
}
__device__ __forceinline__ void team_sync(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }

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
        e[i] = a.idx[p];
        const float g = a.gates[p];
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

struct Task { int32_t segment, expert, unit, slice, end; };
__device__ __forceinline__ Task task_of(const Few &a, const FewShared &S, int32_t number) {
    Task t;
    t.segment = a.by_units(number, t.unit);
    t.expert = S.seg_expert[t.segment];
    t.slice = t.unit * a.per_unit;
    t.end = min(a.slices, t.slice + a.per_unit);
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

// A warp of a team. Its tiles of a slice are every team_warps-th of W1's and then of W2's; it asks for them itself, ahead of the products, from slice to slice and on into the team's next
// task once that is known.
template <typename T> struct Worker {
    static constexpr int COLS = 128 / (int)sizeof(T);
    static constexpr int HALVES = SLICE / COLS;  // tiles side by side in a slice of W1
    static constexpr bool BF16 = sizeof(T) == 2;
    const Few &a;
    FewShared &S;
    const CUtensorMap *w1, *w2;
    const int warp, lane, team, w, W;  // w: number in its team of W warps
    const uint32_t place, bars;        // shared memory: the warp's, and its tiles' barriers
    int32_t flying, ask_slot, use_slot, phase;  // tiles on their way or not yet used
    int32_t total, next;               // tasks; the task that the tiles asked for will go on with, -1: not known
    int32_t slice, end, tile, expert;  // the next tile to ask for
    bool live, second;
    uint32_t at[2][4];  // a lane's rows of the weights in half a tile: row r of matrix mat holds lane r / 2's pair 2 s + mat / 2, element r % 2

    __device__ __forceinline__ Worker(const Few &a_, FewShared &S_, const CUtensorMap *w1_, const CUtensorMap *w2_, uint32_t shared, int warp_, int lane_)
        : a(a_), S(S_), w1(w1_), w2(w2_), warp(warp_), lane(lane_), team(warp_ / a_.team_warps), w(warp_ % a_.team_warps), W(a_.team_warps), place(shared + warp_ * WARP_BYTES),
          bars(smem_u32(&S_.full[warp_][0])), flying(0), ask_slot(0), use_slot(0), phase(0), total(S_.segments * a_.units), next(-1), slice(0), end(0), tile(0), expert(0), live(false), second(false) {
        const int r = lane & 7, mat = lane >> 3, lc = r >> 1;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = 8 * lc + 2 * ((2 * s + (mat >> 1) + lc) & 3) + (r & 1);
#pragma unroll
            for (int q = 0; q < 4; ++q) at[s][q] = k * 128 + (((2 * q + (mat & 1)) ^ (k & 7)) << 4);
        }
    }
    // asks for tiles while the ring has room and it is known for which
    __device__ __forceinline__ void fill() {
#pragma unroll 1
        while (flying < RING) {
            if (!live) {
                if (next < 0 || next >= total) return;
                const Task t = task_of(a, S, next);
                next = -1;
                slice = t.slice;
                end = t.end;
                expert = t.expert;
                live = true;
                second = false;
                tile = w;
            }
            if (!second && tile >= a.tiles1) {
                second = true;
                tile = w;
            }
            if (second && tile >= a.tiles2) {
                second = false;
                tile = w;
                live = ++slice < end;
                continue;
            }
            if (lane == 0) {
                const uint32_t bar = bars + ask_slot * 8, to = place + ask_slot * TILE_BYTES;
                mbar_expect_tx(bar, TILE_BYTES);
                if (second) tma_load_3d(to, w2, bar, tile * 64, slice * SLICE, expert);
                else tma_load_3d(to, w1, bar, (slice * HALVES + tile % HALVES) * 64, tile / HALVES * TILE_K, expert);
            }
            tile += W;
            ask_slot ^= 1;
            ++flying;
        }
    }
    __device__ __forceinline__ bool arrived() {
        const bool ok = mbar_wait(bars + use_slot * 8, phase, &S.abort, a.status);
        return __all_sync(0xffffffffu, ok);
    }
    __device__ __forceinline__ uint32_t at_hand() const { return place + use_slot * TILE_BYTES; }
    __device__ __forceinline__ void use_next() {
        --flying;
        use_slot ^= 1;
        phase ^= use_slot == 0;
    }
    __device__ __forceinline__ void release() {  // the tile at hand has been read
        __syncwarp();
        use_next();
        fill();
    }
    // nothing may be on its way into shared memory that is given back
    __device__ void give_up() {
#pragma unroll 1
        for (; flying > 0; use_next()) {
            const unsigned long long t0 = global_ns();
            while (!mbar_try_wait(bars + use_slot * 8, phase) && global_ns() - t0 < WAIT_LIMIT_NS) {}
        }
        copies_wait<0>();
    }
    __device__ __forceinline__ float *red_of(int other) const {  // a warp's sums of a slice
        return reinterpret_cast<float *>(static_cast<char *>(__cvta_shared_to_generic(place)) + (other - warp) * WARP_BYTES + RING * TILE_BYTES);
    }
    __device__ __forceinline__ int32_t token_of(int32_t p) const {
        int32_t none;
        return a.by_k(p, none);
    }
    // 32 k by 64 columns times rows in TERMS bf16 terms. All of the weights first, then products that do not need each other
    template <int TERMS> __device__ __forceinline__ void multiply(float (&acc)[4][NT][4], uint32_t tile, const uint4 (&x)[TERMS][NT], bool more) const {
        uint32_t w[2][4][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int q = 0; q < 4; ++q) ldmatrix_t(w[s][q], tile + at[s][q]);
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            if (u > 0 && !more) break;
#pragma unroll
            for (int e = TERMS - 1; e >= 0; --e) {
                const uint32_t b[4] = {x[e][u].x, x[e][u].y, x[e][u].z, x[e][u].w};
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int q = 0; q < 4; ++q) mma_16x8x16(acc[q][u], w[s][q], b[2 * s], b[2 * s + 1]);
            }
        }
    }

    // hid of the slice: every warp its tiles' part of the sums, in shared memory
    __device__ __forceinline__ void first_bf16(const int16_t *rows, int32_t m) {
        const int g = lane >> 2, c = lane & 3;
        const bool more = m > 8;
        const bf16 *row[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) row[u] = static_cast<const bf16 *>(a.x) + (int64_t)token_of(rows[min(u * 8 + g, m - 1)]) * a.dw + 8 * c;  // lanes without a row: copies
        float acc[4][NT][4];
        clear(acc);
        uint4 next[2][1][NT];
        auto fetch = [&](int32_t i) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int u = 0; u < NT; ++u)
                    if (i < a.tiles1 && (u == 0 || more)) next[j][0][u] = *reinterpret_cast<const uint4 *>(row[u] + i * TILE_K + 32 * j);
        };
        fetch(w);
#pragma unroll 1
        for (int32_t i = w; i < a.tiles1; i += W) {
            uint4 x[2][1][NT];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int u = 0; u < NT; ++u) x[j][0][u] = next[j][0][u];
            fetch(i + W);  // on its way during the products
            if (!arrived()) return;  // and all learn it at the next barrier
#pragma unroll
            for (int j = 0; j < 2; ++j) multiply<1>(acc, at_hand() + j * (32 * 128), x[j], more);
            release();
        }
        float *red = red_of(warp);
        if (w < a.tiles1)
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) red[(u * 8 + 2 * c + (i & 1)) * RED_STRIDE + 16 * q + g + 8 * (i >> 1)] = acc[q][u][i];
    }
    // the part of y that the slice gives, 64 columns at a time
    __device__ __forceinline__ void second_bf16(const Task &t, int32_t slice, const int16_t *rows, int32_t m) {
        const int g = lane >> 2, c = lane & 3;
        const bool more = m > 8;
        uint4 x[2][2][NT];  // half, term
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int u = 0; u < NT; ++u) x[j][e][u] = *reinterpret_cast<const uint4 *>(&S.hid[team].two[e][u * 8 + g][32 * j + 8 * c]);
#pragma unroll 1
        for (int32_t i = w; i < a.tiles2; i += W) {
            const int32_t col = i * 64 + g;
            float bias[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) bias[e] = slice == 0 && col + e * 8 < a.d ? to_f32(static_cast<const T *>(a.b2)[(int64_t)t.expert * a.d + col + e * 8]) : 0.0f;
            float acc[4][NT][4];
            clear(acc);
            if (!arrived()) return;
#pragma unroll
            for (int j = 0; j < 2; ++j) multiply<2>(acc, at_hand() + j * (32 * 128), x[j], more);
            // hid's second term has either sign, or is 0: it makes a NaN of the infinity that the first gives beside an infinite weight or beyond float's range. What is no finite number is
            // therefore the first term's alone, as if hid were one bf16 number. Rare, and found by a sum of zero times every element that is used, and a vote: no time by the clock (24 tokens 28.3 us a
            // call with it, 28.7 without)
            float odd = 0.0f;
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    if (u * 8 + 2 * c + r < m)
#pragma unroll
                        for (int e = 0; e < 8; ++e) odd = fmaf(acc[e >> 1][u][2 * (e & 1) + r], 0.0f, odd);
            if (__any_sync(0xffffffffu, odd != 0.0f)) {
                float first[4][NT][4];
                clear(first);
#pragma unroll
                for (int j = 0; j < 2; ++j) multiply<1>(first, at_hand() + j * (32 * 128), reinterpret_cast<const uint4 (&)[1][NT]>(x[j][0]), more);
#pragma unroll
                for (int i = 0; i < 16 * NT; ++i) {
                    float &v = acc[i / (4 * NT)][i / 4 % NT][i % 4];
                    v = fabsf(v) <= FLT_MAX ? v : first[i / (4 * NT)][i / 4 % NT][i % 4];
                }
            }
            release();
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int32_t q = u * 8 + 2 * c + r;
                    if (q >= m) continue;
                    float *part = a.parts + ((int64_t)rows[q] * a.units + t.unit) * a.d + col;
                    if (slice > t.slice) {  // a unit of several slices: they add up where they end
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (col + e * 8 < a.d) part[e * 8] += acc[e >> 1][u][2 * (e & 1) + r];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (col + e * 8 < a.d) part[e * 8] = acc[e >> 1][u][2 * (e & 1) + r] + bias[e];
                    }
                }
        }
    }
    __device__ __forceinline__ static void clear(float (&acc)[4][NT][4]) {
#pragma unroll
        for (int i = 0; i < 16 * NT; ++i) acc[i / (4 * NT)][i / 4 % NT][i % 4] = 0.0f;
    }

    // Float: 64 k by 32 columns; a lane has four columns and every fourth run of four k. x(row, k) gives four values
    template <typename X> __device__ __forceinline__ void multiply_f32(float (&acc)[SEG_ROWS][4], uint32_t tile, int32_t m, X x) const {
        const int cg = lane & 7, ph = lane >> 3;
        const char *from = static_cast<const char *>(__cvta_shared_to_generic(tile));
#pragma unroll 1
        for (int j = 0; j < TILE_K / 16; ++j) {
            const int kk = 16 * j + 4 * ph;
            float4 w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = *reinterpret_cast<const float4 *>(from + (kk + e) * 128 + ((cg ^ ((kk + e) & 7)) << 4));
#pragma unroll
            for (int q = 0; q < SEG_ROWS; ++q) {
                if (q >= m) break;
                const float4 v = x(q, kk);
                const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    fma_two(acc[q][0], acc[q][1], f[e], w[e].x, w[e].y);
                    fma_two(acc[q][2], acc[q][3], f[e], w[e].z, w[e].w);
                }
            }
        }
    }
    // the lanes' sums added up; put(row, first column of four, sums) by one lane each
    template <typename Put> __device__ __forceinline__ void give_f32(float (&acc)[SEG_ROWS][4], int32_t m, Put put) const {
        const int cg = lane & 7, ph = lane >> 3;
#pragma unroll
        for (int q = 0; q < SEG_ROWS; ++q) {
            if (q >= m) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[q][i] += __shfl_xor_sync(0xffffffffu, acc[q][i], 8);
                acc[q][i] += __shfl_xor_sync(0xffffffffu, acc[q][i], 16);
            }
            if (q % 4 == ph) put(q, 4 * cg, make_float4(acc[q][0], acc[q][1], acc[q][2], acc[q][3]));
        }
    }
    __device__ __forceinline__ static void clear(float (&acc)[SEG_ROWS][4]) {
#pragma unroll
        for (int i = 0; i < SEG_ROWS * 4; ++i) acc[i / 4][i % 4] = 0.0f;
    }
    // Tiles of the slice's two halves of columns in turn: a warp has one of them. Rows are copied a tile ahead: loaded where they are used, each load is waited for
    __device__ __forceinline__ void first_f32(const int16_t *rows, int32_t m) {
        float *const xs = red_of(warp);  // [2][SEG_ROWS][TILE_K], and the sums behind it
        auto copy = [&](int32_t i, int side) {
            if (i < a.tiles1) {
                const int32_t k = i / HALVES * TILE_K + (lane & 15) * 4;
#pragma unroll 1
                for (int q = lane >> 4; q < m; q += 2)
                    copy16(xs + (side * SEG_ROWS + q) * TILE_K + (lane & 15) * 4, static_cast<const float *>(a.x) + (k < a.d ? (int64_t)token_of(rows[q]) * a.d + k : 0), k < a.d);
            }
            copies_commit();
        };
        float acc[SEG_ROWS][4];
        clear(acc);
        int side = 0;
        copy(w, 0);
#pragma unroll 1
        for (int32_t i = w; i < a.tiles1; i += W, side ^= 1) {
            copy(i + W, side ^ 1);
            copies_wait<1>();
            __syncwarp();
            if (!arrived()) return;
            const float *from = xs + side * (SEG_ROWS * TILE_K);
            multiply_f32(acc, at_hand(), m, [&](int q, int kk) { return *reinterpret_cast<const float4 *>(from + q * TILE_K + kk); });
            release();
        }
        copies_wait<0>();
        __syncwarp();
        if (w < a.tiles1) give_f32(acc, m, [&](int q, int col, float4 v) { *reinterpret_cast<float4 *>(xs + q * RED_STRIDE + col) = v; });
    }
    __device__ __forceinline__ void second_f32(const Task &t, int32_t slice, const int16_t *rows, int32_t m) {
#pragma unroll 1
        for (int32_t i = w; i < a.tiles2; i += W) {
            float acc[SEG_ROWS][4];
            clear(acc);
            if (!arrived()) return;
            multiply_f32(acc, at_hand(), m, [&](int q, int kk) { return *reinterpret_cast<const float4 *>(&S.hid[team].one[q][kk]); });
            release();
            give_f32(acc, m, [&](int q, int c, float4 v) {
                const int32_t col = i * COLS + c;
                if (col >= a.d) return;  // widths are multiples of four
                float4 *part = reinterpret_cast<float4 *>(a.parts + ((int64_t)rows[q] * a.units + t.unit) * a.d + col);
                float4 old = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (slice > t.slice) old = *part;
                else if (slice == 0) old = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.b2) + (int64_t)t.expert * a.d + col);
                *part = make_float4(old.x + v.x, old.y + v.y, old.z + v.z, old.w + v.w);
            });
        }
    }
    // hid = relu(the warps' sums + b1), by the team
    __device__ __forceinline__ void make_hid(int32_t slice_, int32_t m, float bias) {
        const int tid = w * 32 + lane, col = tid % SLICE, givers = min(a.tiles1, W);
#pragma unroll 1
        for (int q = tid / SLICE; q < m; q += W * 32 / SLICE) {  // places behind the last row keep what they had: products of theirs are dropped
            float v = bias;
            for (int o = col / COLS; o < givers; o += HALVES) v += red_of(team * W + o)[q * RED_STRIDE + col % COLS];  // float: a warp has sums of one half of the columns
            v = v < 0.0f || slice_ * SLICE + col >= a.h ? 0.0f : v;  // a NaN stays
            if constexpr (BF16) {
                const bf16 hi = __float2bfloat16_rn(v);
                const float f = __bfloat162float(hi);
                S.hid[team].two[0][q][turned(col)] = hi;
                S.hid[team].two[1][q][turned(col)] = __float2bfloat16_rn(fabsf(f) <= FLT_MAX ? v - f : 0.0f);  // beside an infinity 0, not the NaN of a difference
            } else {
                S.hid[team].one[q][col] = v;
            }
        }
    }
    // 16 columns of a token's y: sum over its slots and units of gate * part, in order; eight groups of lanes take every eighth part
    __device__ __forceinline__ void final_piece(int32_t number) {
        int32_t piece, none;
        const int32_t token = a.by_finals(number, piece), col = piece * 16 + (lane & 3) * 4, parts = a.k * a.units;
        const float *from = a.parts + (int64_t)token * parts * a.d + col;
        float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int B = 8;  // loads in flight (4, 16: 0.5 to 1 us more)
#pragma unroll 1
        for (int32_t j0 = lane >> 2; j0 < parts; j0 += 8 * B) {
            float4 f[B];
#pragma unroll
            for (int i = 0; i < B; ++i) f[i] = col < a.d && j0 + 8 * i < parts ? __ldcg(reinterpret_cast<const float4 *>(from + (int64_t)(j0 + 8 * i) * a.d)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < B; ++i) {
                if (j0 + 8 * i >= parts) break;
                const float g = S.gate[token * a.k + a.by_units(j0 + 8 * i, none)];
                y[0] = fmaf(g, f[i].x, y[0]);
                y[1] = fmaf(g, f[i].y, y[1]);
                y[2] = fmaf(g, f[i].z, y[2]);
                y[3] = fmaf(g, f[i].w, y[3]);
            }
        }
        __syncwarp();
#pragma unroll
        for (int off = 4; off < 32; off <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += __shfl_xor_sync(0xffffffffu, y[i], off);
        if (lane >= 4 || col >= a.d) return;
        T *to = static_cast<T *>(a.y) + (int64_t)token * a.d + col;  // widths are multiples of four
        if constexpr (BF16) *reinterpret_cast<uint2 *>(to) = make_uint2(pack(y[0], y[1]), pack(y[2], y[3]));
        else *reinterpret_cast<float4 *>(to) = make_float4(y[0], y[1], y[2], y[3]);
    }
    // until all units of a token are there
    __device__ __forceinline__ bool complete(int32_t token) {
        bool ok = true;
        if (lane == 0) {
            unsigned long long t0 = 0;
            while (load_relaxed(a.done + token) < a.k * a.units) {
                __nanosleep(50);
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
        __syncwarp();  // the other lanes' loads come behind lane 0's look at the counter: a vote orders no memory
        return __all_sync(0xffffffffu, ok);
    }
};

template <typename T>
__global__ void __launch_bounds__(FEW_THREADS, 1) few_experts_kernel(const __grid_constant__ CUtensorMap w1, const __grid_constant__ CUtensorMap w2, const Few a) {
    extern __shared__ char few_raw[];
    char *base = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(few_raw) + 1023) & ~uintptr_t(1023));
    FewShared &S = *reinterpret_cast<FewShared *>(base + FEW_WARPS * WARP_BYTES);
    FewTables &tab = *reinterpret_cast<FewTables *>(base);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < FEW_WARPS * RING; ++i) mbar_init(smem_u32(&S.full[0][i]), 1);
        S.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int32_t i = threadIdx.x; i < a.n; i += FEW_THREADS) tab.tokens[i] = make_uint2(0u, 0u);
    if (threadIdx.x < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(threadIdx.x ? &w2 : &w1) : "memory");
    __syncthreads();  // the tables are clear
    wait_previous_kernel();
    // All tasks are drawn, the first ones too: who waits for a task's results waits for blocks that are running, whatever else the GPU runs
    const bool draws = lane == 0 && warp % a.team_warps == 0;
    const int32_t first = draws ? atomicAdd(a.ticket, 1) : 0;  // on its way meanwhile
    make_segments(a, S, tab, warp, lane);

    Worker<T> work(a, S, &w1, &w2, smem_u32(base), warp, lane);
    const int team = work.team, threads = work.W * 32, tid = work.w * 32 + lane;
    if (draws) S.next[team] = first;
    team_sync(team, threads);
    int32_t number = work.next = S.next[team];
    work.fill();
    bool ended = false;
#pragma unroll 1
    while (number < work.total) {
        const int32_t drawn = tid == 0 ? atomicAdd(a.ticket, 1) : 0;  // on its way during the first product
        const Task t = task_of(a, S, number);
        const int16_t *rows = S.rows + S.seg_first[t.segment];
        const int32_t m = S.seg_count[t.segment];
#pragma unroll 1
        for (int32_t slice = t.slice; slice < t.end; ++slice) {
            const int32_t col = slice * SLICE + tid % SLICE;
            const float bias = col < a.h ? to_f32(static_cast<const T *>(a.b1)[(int64_t)t.expert * a.h + col]) : 0.0f;  // on its way during the products
            if constexpr (Worker<T>::BF16) work.first_bf16(rows, m);
            else work.first_f32(rows, m);
            if (tid == 0 && slice == t.slice) S.next[team] = drawn;
            ended = team_any(team, threads, *(volatile int32_t *)&S.abort);
            if (ended) break;
            if (slice == t.slice) {
                number = work.next = S.next[team];
                work.fill();
            }
            work.make_hid(slice, m, bias);
            team_sync(team, threads);
            if constexpr (Worker<T>::BF16) work.second_bf16(t, slice, rows, m);
            else work.second_f32(t, slice, rows, m);
        }
        if (!ended) ended = team_any(team, threads, *(volatile int32_t *)&S.abort);  // else the unit's parts are all written
        if (ended) break;
        if (tid < m) add_release(a.done + work.token_of(rows[tid]), 1);
    }
    if (ended) {
        work.give_up();
        return;
    }

    // y, by warps on their own
    const int32_t finals = a.T * a.finals;
#pragma unroll 1
    while (true) {
        int32_t piece = lane == 0 ? atomicAdd(a.final_ticket, 1) : 0, none;
        piece = __shfl_sync(0xffffffffu, piece, 0);
        if (piece >= finals || !work.complete(a.by_finals(piece, none))) return;
        work.final_piece(piece);
    }
}

struct FewPlan {
    int32_t slices, per_unit, units, tiles1, tiles2, finals;
    int64_t counters;
};
FewPlan plan_of(const moe_config &c) {
    FewPlan p;
    const int64_t cols = 128 / (int64_t)act_bytes(c.act), R = (int64_t)c.T * c.k;
    p.slices = (int32_t)cdiv(c.h, SLICE);
    // a slice a task, but for parts of y beyond 64 MiB
    p.per_unit = (int32_t)imax(1, cdiv(R * p.slices * c.d * 4, 64 << 20));
    p.units = (int32_t)cdiv(p.slices, p.per_unit);
    p.tiles1 = (int32_t)(cdiv(c.d, TILE_K) * (SLICE / cols));
    p.tiles2 = (int32_t)cdiv(c.d, cols);
    p.finals = (int32_t)cdiv(c.d, 16);
    p.counters = 64 + c.T;
    return p;
}

// Warps of a team: a task takes a step for the hand-over and one for every tile of a warp, so often as teams have one. bf16, 8 / 4 / 2 warps: 1 token of 1024 x 4096 22.0 / 25.8 /
// 35.0 us, 24 of 32 experts of 512 x 1024 28.3 / 26.5 / 26.0, 64 of 256 of them 92.9 / 78.1 / 79.0, 55 of 114 experts of 128 x 2752 122 / 76 / 57
int32_t team_warps_of(const moe_config &c, const FewPlan &p) {
    const double used = c.n * (1.0 - pow(1.0 - (double)c.k / c.n, c.T));  // experts that some token picks, if it picks any k of them alike
    const int64_t tasks = imax(1, imin((int64_t)c.T * c.k, (int64_t)(used + 0.5))) * p.units;
    int64_t best = 0;
    int32_t of = 0;
    for (int32_t warps : {4, 8, 2}) {
        const int64_t cost = cdiv(tasks, tc_sm_count() * (FEW_WARPS / warps)) * p.per_unit * (1 + cdiv(p.tiles1, warps) + cdiv(p.tiles2, warps));
        if (of > 0 && cost >= best) continue;
        best = cost;
        of = warps;
    }
    return of;
}

struct FewWs {
    int32_t *status, *counters, *idx;
    float *logits, *parts, *gates;
    bf16 *copy;
    int64_t dw;
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
        copy = cv.take<bf16>(c.act == MOE_BF16 ? (int64_t)c.T * dw + ROW_SLACK : 0);
        parts = cv.take<float>(R * p.units * c.d);
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
    a.x = c.act == MOE_BF16 ? (const void *)w.copy : x; a.b1 = b1; a.b2 = b2; a.y = y; a.idx = w.idx; a.gates = w.gates; a.parts = w.parts;
    a.ticket = w.counters; a.final_ticket = w.counters + 32; a.done = w.counters + 64; a.status = w.status;
    a.T = c.T; a.d = c.d; a.h = c.h; a.n = c.n; a.k = c.k; a.dw = (int32_t)w.dw;
    a.slices = p.slices; a.per_unit = p.per_unit; a.units = p.units; a.tiles1 = p.tiles1; a.tiles2 = p.tiles2; a.finals = p.finals; a.team_warps = team_warps_of(c, p);
    a.by_k = Divisor::of(c.k); a.by_units = Divisor::of(p.units); a.by_finals = Divisor::of(p.finals);
    const Routing r = {w.idx, topk_idx, w.gates, gates};
    if (c.act == MOE_BF16) {
        MOE_TRY(launch_routing<bf16>(c, x, Wg, w, p, r, st));
        return launch_experts<bf16>(m1, m2, a, st);
    }
    MOE_TRY(launch_routing<float>(c, x, Wg, w, p, r, st));
    return launch_experts<float>(m1, m2, a, st);
}

}  // namespace moe
