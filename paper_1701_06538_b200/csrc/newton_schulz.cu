// Newton-Schulz products of the Muon step (Jordan et al., 2024) on the 5th-generation tensor cores, for a batch of matrices X [rows, cols]. `steps` times
//   A = X X'  (of the shorter side: X' X where there are more rows than columns),   P = a I + b A + c A A,   X <- P X  (X P)
// and the last X goes straight from the accumulators into the weights: w = w - lr (scale X + decay w). M is the shorter side, N the longer one.
//
// P is a polynomial of A, so that all of them commute and a step's A follows from the one before: (P X)(P X)' = P A P. A segment of up to three steps stays with the M x M matrices
// (T = P A, A <- P T, Q <- P Q) and touches X twice, for the first A and for X <- Q X. What that costs in 64-deep blocks of products decides (together_of): a step is M^2 N / 2 + M^3 / 2 +
// M^2 N operations by itself and three together are M^2 N / 2 + 9/2 M^3 + M^2 N: an eighth fewer from N = 1.7 M or so on. 32 of 1024 x 4096: 5727 -> 3750 us, 16 of 1024 x 2048: 1416 -> 1250,
// 256 of 512 x 1024: 4196 -> 4060. A shorter segment goes first: small singular values, which rounding of A hurts most, have grown when A is made of X anew. (Five steps, errors of X by their
// simulation, one by one / 3 and 2 / 2 and 3: 7.5e-4, 1.4e-3, 5.7e-4 for momentum with gradients of 20 to 90 rows; 7e-4, 7e-4, 5e-4 for normal numbers; 3.6e-3, 2.7e-3, 9.9e-3 for singular
// values spread evenly over two powers of ten.) Four or five steps in one segment would leave fp16's range: Q reaches 3.4445^n.
//
// Bound by results (a pair's tile of 512 x 1024: 7500 cycles, products 4500) and in long lists by the power limit too (990 W; 1965 MHz become 1300 to 1500): 593 TFLOP/s of the operations that are needed for
// 512 of 512 x 1024, 1007 for 64 of 1024 x 4096, where a plain product holds 1402. Every M x M matrix goes through L2 as a result, as an operand and as what is added. All M x M matrices are symmetric: the lower half is made, by tiles, and what
// reads a tile of the upper half reads the stored one in its place, transposed by the operand's major-ness, which an instruction has of its own.
//
// Operands are fp16, not bf16: a step multiplies small singular values by 3.4 and what rounding has put beside them too. X over its Frobenius norm and everything made of it stay
// below 8 whatever the input (Q of three steps below 41), so that the range is known and fp16's three bits more are free: held times 2^10, elements down to 2^-24 are normal numbers.
// (With bf16 the power limit allows 2 to 3 % more.) The diagonals of the M x M matrices are not among the operands: they are kept in float and enter the products' results beside the accumulators,
//   U V = U' V' + U' v_j + u_i V' + u_i v_i [i = j],   P X = P' X + p_i X      (U', V', P' without their diagonals u, v, p)
// An element's rounding error off the diagonal is one of many in a singular value and averages out; on the diagonal it scales a whole row, and near the singular value 1.2 a step
// multiplies such an error by 5 (a gate of 512 x 32, whose A is nearly diagonal, was off by 3e-3 with rounded diagonals). Accumulators are float, and the last X is not rounded at all.
//
// All products of all matrices, of several shapes, are one launch: tiles are drawn one after the other in an order in which what a tile reads is always drawn before it (group of
// matrices, phase, shape, matrix, tile: muon_order.cuh), and a count of stored tiles for every matrix tells when it is there. With a group that fills the SMs more than once, what a tile waits
// for was stored long ago, and the chain of a lone matrix' products (a gate's) runs beside the others'. (A launch for every product leaves its last wave of tiles half empty: 3 tiles of A and P
// and 8 of X for each of 512 x 1024.) Whoever waits does so for tiles of blocks that run already, so that no number of resident blocks is presumed.
//
// PAIR: two CTAs (an SM pair) have a tile of 256 x 256 by cta_group::2, each stages 128 rows of A's operand and half of B's columns. Otherwise, for M up to 128, a CTA has 128 x 128.
// Warp 0 copies operands, warp 1 issues the products, warps 2 to 9 make results of accumulators, warp 10 draws tiles, warp 11 stores results and counts them. Every wait is bounded
// (2 s); on expiry the CTA records MOE_ERR_TIMEOUT in the workspace's status word and drains.
#include <string.h>

#include <type_traits>

#include "muon.cuh"
#include "pairs.cuh"
#include "short_wait.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr int RING = 3;                       // tiles drawn ahead (256 of 512 x 1024: 4451 us; with 2 and groups of 111 tiles 4579)
constexpr int NS_THREADS = 384;
constexpr int NS_STAGES = 5;
constexpr uint32_t BOX = 4096;                // a warp's 32 rows of 64 columns
constexpr int NS_DATA = NS_STAGES * STAGE2_BYTES + 2 * 8 * BOX, NS_SMEM = NS_DATA + 1024 /*alignment*/ + 512 /*barriers, ring*/ + 8 * 128 /*factors*/;

struct NsTile { int32_t matrix, shape, segment, kind, a, b, out, row, col, slot; };

template <bool PAIR> constexpr int tile_side() { return PAIR ? 256 : 128; }
template <bool PAIR> constexpr int arrivals() { return PAIR ? 2 : 1; }  // of a stored tile: CTAs

__device__ __forceinline__ int32_t load_acquire(const int32_t *p) {
    int32_t v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ bool wait_count(const int32_t *count, int32_t at_least, volatile int *abort_flag, int32_t *status) {
    for (int i = 0; i < 64; ++i)
        if (load_acquire(count) >= at_least) return true;
    const unsigned long long t0 = global_ns();
    while (load_acquire(count) < at_least) {
        if (*abort_flag) return false;
        if (global_ns() - t0 > WAIT_LIMIT_NS) {
            *abort_flag = 1;
            atomicExch(status, (int32_t)MOE_ERR_TIMEOUT);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async;" ::: "memory"); }

__device__ __forceinline__ void store_box_3d(const CUtensorMap *tm, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(tm), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// As make_idesc, of fp16 operands
__device__ __forceinline__ uint32_t idesc_of(bool pair, bool a_mn, bool b_mn, int n) {
    return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)((pair ? 256 : 128) >> 4) << 24);
}

// Records of drawn tiles, read by every role. The reader's copy is in its registers before its report leaves: see the loads
template <bool PAIR> struct NsRing {
    const NsArgs &p;
    const uint32_t ring, full0, empty0;
    volatile int *abort_flag;
    const bool warp_wide, arrives;
    int i;
    __device__ __forceinline__ bool next(NsTile &t) {
        const uint32_t slot = (uint32_t)i % RING, par = ((uint32_t)i / RING) & 1u, full = full0 + 8u * slot;
        bool ok = short_wait(full, par, abort_flag, p.status);
        if (warp_wide) ok = __all_sync(0xffffffffu, ok);
        if (!ok) return false;
        if (PAIR) mbar_try_wait_cluster(full, par);  // acquire at cluster scope: the record came from the other CTA's thread
        int4 a;
        asm volatile("ld.volatile.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w) : "r"(ring + 16u * slot) : "memory");
        uint32_t seen = (uint32_t)a.w;  // (its sign bit is always 0: the report's address depends on the load)
        if (warp_wide) seen = __reduce_or_sync(0xffffffffu, seen);
        if (arrives) {
            const uint32_t empty = empty0 + 8u * slot + ((seen >> 31) << 3);
            if (PAIR) mbar_arrive_leader_relaxed(empty);
            else mbar_arrive(empty);
        }
        ++i;
        t.matrix = a.x; t.shape = a.y >> 16; t.segment = a.y >> 11 & 31; t.kind = a.y >> 9 & 3; t.a = a.y >> 6 & 7; t.b = a.y >> 3 & 7; t.out = a.y & 7;
        t.row = (a.z >> 16) * tile_side<PAIR>(); t.col = (a.z & 0xffff) * tile_side<PAIR>(); t.slot = a.w;
        return a.x >= 0;
    }
};

// 32 rows of 32 columns of the last X, which lie in `box` as floats, onto the weights: eight lanes a row, so that a row's 32 columns are read and written together
template <bool BF16, bool MASTER, bool VECTORS>
__device__ __forceinline__ void step_box(int32_t cols, const MuonEntry &e, int64_t first, int32_t rows_left, int32_t cols_left, const float *box, int lane, float lr) {
    const int32_t c = (lane & 7) * 4;
    float4 w[8];
    auto at = [&](int i) { return first + (int64_t)(4 * i + (lane >> 3)) * cols + c; };
    auto in = [&](int i) { return 4 * i + (lane >> 3) < rows_left && c < cols_left; };
    const float *floats = MASTER ? e.master : static_cast<const float *>(e.w);
    bf16 *halves = static_cast<bf16 *>(e.w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (!in(i)) continue;
        if constexpr (VECTORS) {
            if constexpr (!BF16 || MASTER) w[i] = *reinterpret_cast<const float4 *>(floats + at(i));
            else {
                const uint2 u = *reinterpret_cast<const uint2 *>(halves + at(i));
                w[i] = make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
            }
        } else {
            float *to = reinterpret_cast<float *>(&w[i]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c + q < cols_left) to[q] = !BF16 || MASTER ? floats[at(i) + q] : to_f32(halves[at(i) + q]);
        }
    }
    const float by = e.scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int32_t r = 4 * i + (lane >> 3);
        const float4 x = *reinterpret_cast<const float4 *>(box + r * 32 + (((lane & 7) ^ (r & 7)) << 2));
        w[i].x -= lr * fmaf(x.x, by, e.decay * w[i].x);
        w[i].y -= lr * fmaf(x.y, by, e.decay * w[i].y);
        w[i].z -= lr * fmaf(x.z, by, e.decay * w[i].z);
        w[i].w -= lr * fmaf(x.w, by, e.decay * w[i].w);
        if (!in(i)) continue;
        float *to = MASTER ? e.master : static_cast<float *>(e.w);
        if constexpr (VECTORS) {
            if constexpr (!BF16 || MASTER) *reinterpret_cast<float4 *>(to + at(i)) = w[i];
            if constexpr (BF16) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(w[i].x, w[i].y), b = __floats2bfloat162_rn(w[i].z, w[i].w);
                *reinterpret_cast<uint2 *>(halves + at(i)) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
            }
        } else {
            const float *v = reinterpret_cast<const float *>(&w[i]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (c + q >= cols_left) break;
                if constexpr (!BF16 || MASTER) to[at(i) + q] = v[q];
                if constexpr (BF16) halves[at(i) + q] = __float2bfloat16_rn(v[q]);
            }
        }
    }
}

// What a result is, besides the accumulator
enum Result { K_FIRST, K_SECOND, K_MULT, K_THIRD, K_LAST };
// 32 columns of 32 rows, a row a lane. old: 32 halves of the operand that is added, times what the diagonals make of it: `of_row`, and of the columns `cols` (shared memory). See factor_of
template <int KIND, bool COLS>
__device__ __forceinline__ void finish(float2 (&v)[16], const uint32_t *old, float of_row, const float *cols) {
    constexpr float UNIT = 1.0f / MUON_UNIT;
    constexpr float by = KIND == K_SECOND ? NS_C * UNIT : KIND == K_LAST ? UNIT * UNIT : UNIT;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float4 c = make_float4(of_row, of_row, of_row, of_row);
        if constexpr (COLS) c = *reinterpret_cast<const float4 *>(cols + 4 * q);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float2 &y = v[2 * q + j];
            if constexpr (KIND == K_FIRST) {
                y = mul2(y, both(by));
            } else {
                float2 f = j ? make_float2(c.z, c.w) : make_float2(c.x, c.y);
                if constexpr (KIND == K_SECOND) f = fma2(f, both(1.0f), both(of_row));
                const float2 o = __half22float2(*reinterpret_cast<const __half2 *>(old + 2 * q + j));
                float2 more = mul2(o, f);
                if constexpr (KIND == K_MULT) more = fma2(__half22float2(*reinterpret_cast<const __half2 *>(old + 16 + 2 * q + j)), both(of_row), more);
                y = fma2(y, both(by), more);
            }
        }
    }
}
// c (d_i + d_j) + b of A' for P; in a product of two the columns' go with the first and the row's with the second; of X; the last X is wanted without MUON_UNIT
template <int KIND> __device__ __forceinline__ float factor_of(float diagonal, bool column) {
    return KIND == K_SECOND ? fmaf(NS_C, diagonal, column ? NS_B : 0.0f) : KIND == K_LAST ? diagonal * (1.0f / MUON_UNIT) : diagonal;
}
// 32 bytes at a time (a whole sector), of what another SM may have written in the meantime
__device__ __forceinline__ void load_32B(const void *from, uint32_t *r) {
    asm volatile("ld.relaxed.gpu.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(from) : "memory");
}
__device__ __forceinline__ void store_32B(void *to, const uint32_t *r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// A row's 32 weights, a row a lane, where rows begin at 32 bytes (columns and tensors: slices of a model's layers may begin at 16): read while the products run
struct RowOfWeights {
    float *floats;   // what the step is taken on: float weights or masters, or nullptr
    bf16 *halves;    // bf16 weights, or nullptr
    float scale, decay;
    uint32_t raw[32];
    __device__ __forceinline__ void load(int32_t at, bool in) {
        if (!in) return;
        if (floats)
#pragma unroll
            for (int q = 0; q < 4; ++q) load_32B(floats + at + 8 * q, raw + 8 * q);
        else
#pragma unroll
            for (int q = 0; q < 2; ++q) load_32B(halves + at + 16 * q, raw + 8 * q);
    }
    __device__ __forceinline__ void step(float2 (&x)[16], float lr) const {  // x: the new weights
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 w = floats ? make_float2(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1])) : make_float2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
            x[i] = fma2(both(-lr), fma2(x[i], both(scale), mul2(w, both(decay))), w);
        }
    }
    __device__ __forceinline__ void store(int32_t at, const float2 (&x)[16]) const {
        if (floats)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t u[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) { u[2 * i] = __float_as_uint(x[4 * q + i].x); u[2 * i + 1] = __float_as_uint(x[4 * q + i].y); }
                store_32B(floats + at + 8 * q, u);
            }
        if (halves)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const __nv_bfloat162 two = __floats2bfloat162_rn(x[8 * q + i].x, x[8 * q + i].y);
                    u[i] = *reinterpret_cast<const uint32_t *>(&two);
                }
                store_32B(halves + at + 16 * q, u);
            }
    }
};

// A warp's part of a tile, box by box (at most two): accumulators -> results -> shared memory, or the weights. What is added comes from `from` (this lane's row from the tile's first column
// of the warp on), a box ahead; of_cols: the diagonal's elements of the columns. Each kind has its own code: with all of them in one loop instructions were fetched again and again.
struct BoxWork {
    uint32_t accumulator;   // in tensor memory
    uint8_t *boxes;
    float *factors;
    const __half *from, *from_b;  // (from_b: K_MULT)
    const float *of_cols;
    float *diagonal;        // of the result
    float of_row, of_row_b;       // (of_row_b: K_MULT)
    int32_t row0, first, boxes_n, M;
    bool in;                // this lane's row exists
    uint32_t box_empty0, box_ready0, box_parity;
    volatile int *abort_flag;
    int32_t *status;
};
// The operand's 32 halves of this lane's row, and the diagonal's element of a column a lane, from a box' first column on
template <int KIND> constexpr int old_words() { return KIND == K_MULT ? 32 : 16; }  // (of two operands)
template <int KIND, bool COLS> __device__ __forceinline__ void fetch_half(const BoxWork &b, int32_t at, int lane, uint32_t (&old)[old_words<KIND>()], float &of_col) {
    if constexpr (KIND != K_FIRST)
        if (b.in) {
            load_32B(b.from + at, old);
            load_32B(b.from + at + 16, old + 8);
            if constexpr (KIND == K_MULT) {
                load_32B(b.from_b + at, old + 16);
                load_32B(b.from_b + at + 16, old + 24);
            }
        }
    if constexpr (COLS)
        if (b.first + at + lane < b.M) of_col = __ldcg(b.of_cols + b.first + at + lane);
}
// Half a box, 32 columns. The next box' half of the operand (of two operands: the next half) is asked for as soon as this one's is used up
template <int KIND, bool COLS, bool ROWS, int J, typename Last>
__device__ __forceinline__ void make_half(const BoxWork &b, int u, int lane, float lr, const uint32_t (&raw)[32], uint32_t (&old)[old_words<KIND>()], float &of_col, RowOfWeights &weights, int32_t weights_end,
                                          Last onto_weights) {
    const int32_t col = b.first + 64 * u + 32 * J;
    uint8_t *box = b.boxes + u * 4 * BOX;
    if constexpr (COLS) {
        __syncwarp();
        b.factors[lane] = factor_of<KIND>(of_col, true);
        __syncwarp();
    }
    float2 v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = make_float2(__uint_as_float(raw[2 * i]), __uint_as_float(raw[2 * i + 1]));
    if (KIND <= K_MULT && col == b.row0) {  // the diagonal: kept in float; no part of the operand (and A' has a zero here)
        float own = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float &e = i & 1 ? v[i / 2].y : v[i / 2].x;
            if (i == lane) { own = e; e = 0.0f; }
        }
        own *= 1.0f / (MUON_UNIT * MUON_UNIT);
        if (b.row0 + lane < b.M) b.diagonal[b.row0 + lane] = KIND == K_FIRST ? own : KIND == K_MULT ? fmaf(b.of_row, b.of_row_b, own) : fmaf(NS_C, fmaf(b.of_row, b.of_row, own), fmaf(NS_B, b.of_row, NS_A));
    }
    finish<KIND, COLS>(v, old, factor_of<KIND>(b.of_row, false), b.factors);
    if constexpr (KIND == K_MULT) {
        if (J == 0 || u + 1 < b.boxes_n) fetch_half<KIND, COLS>(b, 64 * u + 32 * J + 32, lane, old, of_col);
    } else if (u + 1 < b.boxes_n) fetch_half<KIND, COLS>(b, 64 + 32 * J, lane, old, of_col);
    if constexpr (KIND != K_LAST) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t packed[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half2 two = __floats2half2_rn(v[4 * q + i].x, v[4 * q + i].y);
                packed[i] = *reinterpret_cast<const uint32_t *>(&two);
            }
            *reinterpret_cast<uint4 *>(box + lane * 128 + (((4 * J + q) ^ (lane & 7)) << 4)) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
        }
    } else if constexpr (ROWS) {
        const bool live = b.in && col < weights_end;
        if (live) weights.step(v, lr);
        weights.load(col + 32, (J == 0 || u + 1 < b.boxes_n) && b.in && col + 32 < weights_end);
        if (live) weights.store(col, v);
    } else {
        __syncwarp();
        float *floats = reinterpret_cast<float *>(box);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            *reinterpret_cast<float4 *>(floats + lane * 32 + ((q ^ (lane & 7)) << 2)) = make_float4(v[2 * q].x, v[2 * q].y, v[2 * q + 1].x, v[2 * q + 1].y);
        __syncwarp();
        onto_weights(col, floats);
    }
}
// ROWS: the weights row by row (K_LAST), else by `onto_weights` through shared memory
template <int KIND, bool COLS, bool ROWS, typename Wait, typename Release, typename Last>
__device__ __forceinline__ bool make_boxes(const BoxWork &b, int lane, float lr, RowOfWeights &weights, int32_t weights_end, Wait wait_accumulator, Release release, Last onto_weights) {
    constexpr int OLD = old_words<KIND>();
    constexpr bool HALVES = KIND == K_LAST || KIND == K_MULT;  // no registers for both halves of a box' accumulators: beside the weights, beside two operands
    uint32_t old0[OLD], old1[OLD];
    float of_col0 = 0.0f, of_col1 = 0.0f;
#pragma unroll
    for (int i = 0; i < OLD; ++i) old0[i] = old1[i] = 0u;
    if (b.boxes_n > 0) {  // (on their way while the products run)
        fetch_half<KIND, COLS>(b, 0, lane, old0, of_col0);
        if constexpr (KIND != K_MULT) fetch_half<KIND, COLS>(b, 32, lane, old1, of_col1);
        if constexpr (ROWS) weights.load(b.first, b.in && b.first < weights_end);
    }
    bool ok = wait_accumulator();
    if (ok && b.boxes_n == 0) release();
#pragma unroll 1
    for (int u = 0; u < 2; ++u) {
        // The last tile's box has been stored: what a warp without one waits for too, whose report below would else count for that tile's
        ok = ok && __all_sync(0xffffffffu, short_wait(b.box_empty0 + 8u * u, b.box_parity, b.abort_flag, b.status));
        if (ok && u < b.boxes_n) {
            uint32_t raw0[32], raw1[32];
            tc_ld_32x32(b.accumulator + 64 * u, raw0);
            if constexpr (!HALVES) tc_ld_32x32(b.accumulator + 64 * u + 32, raw1);
            tc_ld_wait();
            if (!HALVES && u + 1 == b.boxes_n) release();
            make_half<KIND, COLS, ROWS, 0>(b, u, lane, lr, raw0, old0, of_col0, weights, weights_end, onto_weights);
            if constexpr (HALVES) {
                tc_ld_32x32(b.accumulator + 64 * u + 32, raw1);
                tc_ld_wait();
                if (u + 1 == b.boxes_n) release();
            }
            if constexpr (KIND == K_MULT) make_half<KIND, COLS, ROWS, 1>(b, u, lane, lr, raw1, old0, of_col0, weights, weights_end, onto_weights);
            else make_half<KIND, COLS, ROWS, 1>(b, u, lane, lr, raw1, old1, of_col1, weights, weights_end, onto_weights);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b.box_ready0 + 8u * u);
    }
    return ok;
}

template <bool PAIR>
__global__ void __launch_bounds__(NS_THREADS, 1) newton_schulz_kernel(const __grid_constant__ NsAllMaps all_maps, const __grid_constant__ NsArgs p, const __grid_constant__ MuonBatch batch) {
    constexpr int SIDE = tile_side<PAIR>(), NST = NS_STAGES, STAGE = STAGE2_BYTES, ACC = SIDE;  // ACC: columns of an accumulator
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bars = base + NS_DATA;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (NST + s); };
    auto tfull_bar = [&](int a) { return bars + 8u * (2 * NST + a); };
    auto tempty_bar = [&](int a) { return bars + 8u * (2 * NST + 2 + a); };
    const uint32_t ring_full0 = bars + 128, ring_empty0 = bars + 160, box_ready0 = bars + 208, box_empty0 = bars + 224, ring = bars + 256;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + NS_DATA + 192);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + NS_DATA + 200);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;

    if (threadIdx.x == 0) {
        for (int s = 0; s < NST; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), PAIR ? 16 : 8); }
        // readers of a record: producer, 8 epilogue warps and storer in each CTA, the MMA warp of the even one
        for (int q = 0; q < RING; ++q) { mbar_init(ring_full0 + 8u * q, 1); mbar_init(ring_empty0 + 8u * q, PAIR ? 21 : 11); }
        for (int u = 0; u < 2; ++u) { mbar_init(box_ready0 + 8u * u, 8); mbar_init(box_empty0 + 8u * u, 1); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)), "r"((uint32_t)TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)), "r"((uint32_t)TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();  // both CTAs' barriers exist before anything is signalled across the pair
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    wait_previous_kernel();

    auto kblocks_of = [&](const NsShape &s, const NsTile &t) { return ((t.kind == GRAM ? (s.left ? s.cols : s.rows) : s.M) + BK - 1) / BK; };
    // columns that exist of a tile's output, and of the product (both CTAs' halves of B's operand begin at multiples of 64)
    auto cols_out = [&](const NsShape &s, const NsTile &t) { return t.kind == APPLY ? s.ld : s.Mld; };
    auto rows_out = [&](const NsShape &s, const NsTile &t) { return t.kind == APPLY ? s.rows : s.M; };
    auto width_of = [&](const NsShape &s, const NsTile &t) { return PAIR && cols_out(s, t) - t.col > 128 ? 256 : 128; };
    auto is_last = [&](const NsShape &s, const NsTile &t) { return t.kind == APPLY && (t.segment + 1) * s.together >= p.steps; };
    // Where an operand lies in a product whose contraction runs along the shorter side: block kb of it is in the lower half for rows from `at` on, or has to be transposed
    auto upper = [&](int kb, int32_t at) { return kb * BK / SIDE > at / SIDE; };
    auto a_is_mn = [&](const NsShape &s, const NsTile &t, int kb) { return t.kind == GRAM ? !s.left : t.kind == APPLY && !s.left ? false : upper(kb, t.row); };
    auto b_is_mn = [&](const NsShape &s, const NsTile &t, int kb) { return t.kind == GRAM ? !s.left : t.kind == APPLY && s.left ? true : upper(kb, t.col); };
    // A square on the diagonal of X X' or A A: what a CTA stages of the first operand is what it would stage of the second. Not loaded twice (13 % of what 512 x 1024 loads)
    auto one_operand = [&](const NsShape &s, const NsTile &t) { return t.kind != APPLY && t.a == t.b && t.row == t.col && width_of(s, t) == SIDE; };
    // a warp's boxes of a tile: the rows, the first column and how many there are
    auto boxes_of = [&](const NsShape &s, const NsTile &t, int w, int32_t &row0, int32_t &first) {
        const int32_t width = width_of(s, t);
        row0 = t.row + 128 * (int)rank + 32 * ((w + 2) & 3);  // (epilogue warps are warps 2 to 9, and their quarter of the accumulator's rows is warp % 4)
        first = t.col + (w >> 2) * (width / 2);
        return row0 < rows_out(s, t) ? max(0, min(width / 128, (cols_out(s, t) - first) / 64)) : 0;
    };
    auto gave_up = [&]() {  // copies in flight have landed long before a millisecond is over, and only then may the CTA exit
        for (const unsigned long long t0 = global_ns(); global_ns() - t0 < 1000000ull;) {}
    };

    if (warp == 0) {
        // ------------------------------------------------------------------ bulk tensor copies (both CTAs)
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            NsRing<PAIR> tiles{p, ring, ring_full0, ring_empty0, abort_flag, false, true, 0};
            NsTile t;
            while (ok && tiles.next(t)) {
                const NsShape &h = p.s[t.shape];
                const NsMaps &maps = all_maps.m[t.shape];
                const int slot = t.slot, x = t.segment & 1, xm = x ? slot : t.matrix;
                const bool a_x = t.kind == GRAM || (t.kind == APPLY && !h.left), b_x = t.kind == GRAM || (t.kind == APPLY && h.left);
                const int sb = t.kind == APPLY ? t.a : t.b;  // (X B: the symmetric one is the second)
                const CUtensorMap *ak = a_x ? &maps.x_k[x] : &maps.s_k[t.a], *an = a_x ? &maps.x_mn[x] : &maps.s_mn[t.a], *bk = b_x ? &maps.x_k[x] : &maps.s_k[sb], *bn = b_x ? &maps.x_mn[x] : &maps.s_mn[sb];
                const int am = a_x ? xm : slot, bm = b_x ? xm : slot;
                const int a0 = t.row + 128 * (int)rank, b0 = t.col + (PAIR ? width_of(h, t) / 2 * (int)rank : 0);
                const int kblocks = kblocks_of(h, t);
                const bool once = one_operand(h, t);
                const uint32_t bytes = (PAIR ? 2 : 1) * (once ? A2_BYTES : STAGE);
                for (int kb = 0; kb < kblocks; ++kb) {
                    ok = short_wait(empty_bar(s), ph ^ 1u, abort_flag, p.status);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(full_bar(s), bytes);
                    auto load = [&](uint32_t dst, bool mn, const CUtensorMap *k_map, const CUtensorMap *mn_map, int at, int matrix) {
                        if (mn) {
                            if (PAIR) tma2_load_4d(dst, mn_map, full_bar(s), 0, kb * BK, at / 64, matrix);
                            else tma_load_4d(dst, mn_map, full_bar(s), 0, kb * BK, at / 64, matrix);
                        } else {
                            if (PAIR) tma2_load_3d(dst, k_map, full_bar(s), kb * BK, at, matrix);
                            else tma_load_3d(dst, k_map, full_bar(s), kb * BK, at, matrix);
                        }
                    };
                    load(base + s * STAGE, a_is_mn(h, t, kb), ak, an, a0, am);
                    if (!once) load(base + s * STAGE + A2_BYTES, b_is_mn(h, t, kb), bk, bn, b0, bm);
                    if (++s == NST) { s = 0; ph ^= 1u; }
                }
            }
            if (!ok) gave_up();
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (even CTA only; the warp stays together)
        if (rank == 0) {
            int s = 0, acc = 0;
            uint32_t ph = 0, acc_ph = 0;
            bool ok = true;
            NsRing<PAIR> tiles{p, ring, ring_full0, ring_empty0, abort_flag, true, lane == 0, 0};
            NsTile t;
            while (ok && tiles.next(t)) {
                const NsShape &h = p.s[t.shape];
                ok = __all_sync(0xffffffffu, short_wait(tempty_bar(acc), acc_ph ^ 1u, abort_flag, p.status));
                if (!ok) break;
                tc_fence_after();
                const uint32_t d_tmem = tmem_base + acc * ACC;
                const int kblocks = kblocks_of(h, t), width = width_of(h, t);
                const uint32_t b_offset = one_operand(h, t) ? 0u : (uint32_t)A2_BYTES;
                for (int kb = 0; kb < kblocks; ++kb) {
                    const bool a_mn = a_is_mn(h, t, kb), b_mn = b_is_mn(h, t, kb);
                    ok = __all_sync(0xffffffffu, short_wait(full_bar(s), ph, abort_flag, p.status));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a_src = base + s * STAGE, b_src = a_src + b_offset, idesc = idesc_of(PAIR, a_mn, b_mn, width);
                    const uint64_t ad = a_mn ? desc_mnmajor(a_src) : desc_kmajor(a_src), bd = b_mn ? desc_mnmajor(b_src) : desc_kmajor(b_src);
                    const uint32_t a_step = a_mn ? (16 * 128) >> 4 : 32 >> 4, b_step = b_mn ? (16 * 128) >> 4 : 32 >> 4;
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) {
                        if (PAIR) warp_mma2(d_tmem, ad + k * a_step, bd + k * b_step, idesc, (kb > 0 || k > 0) ? 1u : 0u);
                        else warp_mma(d_tmem, ad + k * a_step, bd + k * b_step, idesc, (kb > 0 || k > 0) ? 1u : 0u);
                    }
                    if (PAIR) warp_commit2(empty_bar(s));
                    else warp_commit(empty_bar(s));
                    if (++s == NST) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (PAIR) warp_commit2(tfull_bar(acc));
                else warp_commit(tfull_bar(acc));
                if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
            }
        }
    } else if (warp == 10) {
        // ------------------------------------------------------------------ drawing tiles (even CTA, one thread)
        if (rank == 0 && lane == 0) {
            const uint32_t peer_ring = PAIR ? peer_smem_addr(ring, 1) : 0u, peer_full0 = PAIR ? peer_smem_addr(ring_full0, 1) : 0u;
            NsOrder order(p);
            for (int i = 0;; ++i) {
                const uint32_t slot = (uint32_t)i % RING;
                if (i >= RING) {  // every reader of the record this slot held has its copy
                    const uint32_t par = ((uint32_t)i / RING - 1) & 1u;
                    if (!short_wait(ring_empty0 + 8u * slot, par, abort_flag, p.status)) break;
                    if (PAIR) mbar_try_wait_cluster(ring_empty0 + 8u * slot, par);
                }
                const NsTileRecord drawn = order.find(atomicAdd(p.next, 1));
                const int4 a = make_int4(drawn.matrix, drawn.what, drawn.place, drawn.slot);
                if (a.x >= 0) {  // handed out when what it reads is there: then nobody else has to look
                    const NsShape &h = p.s[a.y >> 16];
                    const int32_t *count = p.done + h.first + a.x;
                    bool ok = wait_count(count, arrivals<PAIR>() * order.tiles_before, abort_flag, p.status);
                    if (ok && order.tiles_before == 0 && a.x >= h.slots)  // and the slot's last user has read what is overwritten now
                        ok = wait_count(count - h.slots, arrivals<PAIR>() * tiles_of_matrix(h, p.steps), abort_flag, p.status);
                    if (!ok) break;
                    fence_async();  // what other SMs' copies have stored, before copies read it
                }
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(ring + 16u * slot), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w) : "memory");
                if (PAIR) st_cluster_v4(peer_ring + 16u * slot, a);
                mbar_arrive(ring_full0 + 8u * slot);
                if (PAIR) mbar_arrive_cluster_addr(peer_full0 + 8u * slot);
                if (a.x < 0) break;
            }
        }
    } else if (warp == 11) {
        // ------------------------------------------------------------------ storing results (both CTAs, one thread)
        if (lane == 0) {
            uint32_t ph = 0;
            bool ok = true;
            NsRing<PAIR> tiles{p, ring, ring_full0, ring_empty0, abort_flag, false, true, 0};
            NsTile t;
            while (ok && tiles.next(t)) {
                const NsShape &h = p.s[t.shape];
                const NsMaps &maps = all_maps.m[t.shape];
                const bool last = is_last(h, t);
                const int to = (t.segment & 1) ^ 1;  // of X
                const CUtensorMap *out = t.kind == APPLY ? &maps.x_k[to] : &maps.s_k[t.out];
                const int matrix = t.kind == APPLY && !to ? t.matrix : t.slot;
                const int32_t row0 = t.row + 128 * (int)rank, cols = cols_out(h, t), width = width_of(h, t);
                const bool here = row0 < rows_out(h, t);
                for (int u = 0; u < 2 && ok; ++u) {
                    ok = short_wait(box_ready0 + 8u * u, ph, abort_flag, p.status);
                    if (!ok) break;
                    if (!last) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // what the workers have written, before this thread's copies read it
                        if (here)
                            for (int half = 0; half < 2; ++half) {
                                const int32_t col = t.col + half * (width / 2) + 64 * u;
                                if (64 * u < width / 2 && col < cols) store_box_3d(out, base + NST * STAGE + (half * 2 + u) * 4 * BOX, col, row0, matrix);
                            }
                        tma_store_commit();
                        tma_store_wait_read();
                    }
                    mbar_arrive(box_empty0 + 8u * u);
                }
                if (!ok) break;
                ph ^= 1u;
                tma_store_wait_all();
                fence_async();
                asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p.done + h.first + t.matrix) : "memory");
            }
            tma_store_wait_all();  // no bulk store may outlive the CTA's shared memory
        }
    } else {
        // ------------------------------------------------------------------ results (warps 2..9, both CTAs)
        // Two warps share each quarter of the accumulator's rows and take half of its columns each, in boxes of 64.
        const int w = warp - 2, quarter = warp & 3, half = w >> 2;
        uint8_t *boxes_at = smem + NST * STAGE + (half * 8 + quarter) * BOX;  // of the first box; the second one's are 4 boxes on: the four quarters' rows lie together
        float *factors = reinterpret_cast<float *>(smem + NS_DATA + 512 + w * 128);
        const float lr = p.rates ? p.rates->lr : p.lr;
        int acc = 0;
        uint32_t acc_ph = 0, box_ph = 0;
        NsRing<PAIR> tiles{p, ring, ring_full0, ring_empty0, abort_flag, true, lane == 0, 0};
        NsTile t;
        bool ok = true;
        while (ok && tiles.next(t)) {
            const NsShape &h = p.s[t.shape];
            BoxWork b;
            b.boxes_n = boxes_of(h, t, w, b.row0, b.first);
            const int32_t row = b.row0 + lane;
            const int slot = t.slot, x = t.segment & 1;
            const bool last = is_last(h, t);
            auto diagonal_of = [&](int s) { return h.d + ((int64_t)s * h.slots + slot) * h.M; };
            auto symmetric_at = [&](int s) { return h.s[s] + ((int64_t)slot * h.M + row) * h.Mld + b.first; };
            b.boxes = boxes_at; b.factors = factors; b.M = h.M;
            b.box_empty0 = box_empty0; b.box_ready0 = box_ready0; b.box_parity = box_ph ^ 1u;
            b.abort_flag = abort_flag; b.status = p.status;
            b.diagonal = diagonal_of(t.out);
            // What the result is added to: the operands or X as it was, and the diagonals' elements of this lane's row and of its columns
            b.from = t.kind == APPLY ? h.x[x] + ((int64_t)(x ? slot : t.matrix) * h.rows + row) * h.ld + b.first : symmetric_at(t.a);
            b.from_b = symmetric_at(t.b);
            b.in = row < rows_out(h, t);
            b.of_cols = diagonal_of(t.kind == MULT ? t.b : t.a);
            b.of_row = t.kind != GRAM && row < h.M && (t.kind != APPLY || h.left) ? __ldcg(diagonal_of(t.a) + row) : 0.0f;
            b.of_row_b = t.kind == MULT && row < h.M ? __ldcg(diagonal_of(t.b) + row) : 0.0f;
            auto wait_accumulator = [&]() {
                const bool full = __all_sync(0xffffffffu, short_wait(tfull_bar(acc), acc_ph, abort_flag, p.status));
                tc_fence_after();
                return full;
            };
            b.accumulator = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * ACC + half * (width_of(h, t) / 2);
            auto release = [&]() {  // the warp's part of the accumulator is in registers: the buffer goes back
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_leader_relaxed(tempty_bar(acc));
                    else mbar_arrive(tempty_bar(acc));
                }
            };
            const int32_t entry = last ? batch.entry_of(h.first + t.matrix) : 0;
            const MuonEntry &e = batch.t[entry];
            const int64_t weights_at = ((int64_t)(h.first + t.matrix - batch.before[entry]) * h.rows + b.row0) * h.cols;
            RowOfWeights weights;
            weights.floats = nullptr;
            weights.halves = nullptr;
            if (last) {
                const int64_t at = weights_at + (int64_t)lane * h.cols;
                weights.floats = e.kind & 8 ? e.master + at : e.kind & 1 ? nullptr : static_cast<float *>(e.w) + at;
                weights.halves = e.kind & 1 ? static_cast<bf16 *>(e.w) + at : nullptr;
                weights.scale = e.scale; weights.decay = e.decay;
            }
            auto onto_weights = [&](int32_t col, const float *floats) {
                if (col >= h.cols) return;
                const int64_t at = weights_at + col;
                const int32_t rl = h.rows - b.row0, cl = h.cols - col;
                const bool vectors = h.cols % 4 == 0;
                if (e.kind & 8) vectors ? step_box<true, true, true>(h.cols, e, at, rl, cl, floats, lane, lr) : step_box<true, true, false>(h.cols, e, at, rl, cl, floats, lane, lr);
                else if (e.kind & 1) vectors ? step_box<true, false, true>(h.cols, e, at, rl, cl, floats, lane, lr) : step_box<true, false, false>(h.cols, e, at, rl, cl, floats, lane, lr);
                else vectors ? step_box<false, false, true>(h.cols, e, at, rl, cl, floats, lane, lr) : step_box<false, false, false>(h.cols, e, at, rl, cl, floats, lane, lr);
            };
            auto make = [&](auto kind, auto cols, auto rows) {
                return make_boxes<decltype(kind)::value, decltype(cols)::value, decltype(rows)::value>(b, lane, lr, weights, h.cols, wait_accumulator, release, onto_weights);
            };
            using Yes = std::true_type;
            using No = std::false_type;
            if (t.kind == GRAM) ok = make(std::integral_constant<int, K_FIRST>(), No(), No());
            else if (t.kind == POLY) ok = make(std::integral_constant<int, K_SECOND>(), Yes(), No());
            else if (t.kind == MULT) ok = make(std::integral_constant<int, K_MULT>(), Yes(), No());
            else if (!last) ok = h.left ? make(std::integral_constant<int, K_THIRD>(), No(), No()) : make(std::integral_constant<int, K_THIRD>(), Yes(), No());
            else if (h.cols % 32 == 0 && (e.kind & 16)) ok = h.left ? make(std::integral_constant<int, K_LAST>(), No(), Yes()) : make(std::integral_constant<int, K_LAST>(), Yes(), Yes());
            else ok = h.left ? make(std::integral_constant<int, K_LAST>(), No(), No()) : make(std::integral_constant<int, K_LAST>(), Yes(), No());
            box_ph ^= 1u;
            if (++acc == 2) { acc = 0; acc_ph ^= 1u; }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();  // the pair's MMAs read both CTAs' shared memory: leave together
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
    }
}

// ------------------------------------------------------------------------------------------ host
// Tiles of A in a group, on SM pairs (74): two for each, twice as many on single SMs. A pair with one has to wait for others' tiles (256 of 512 x 1024, graph replay: 4911 us with 74, 4455 with
// 111, 4335 with 148), more only take workspace (4287 with 222, 4377 with 296; 32 of 1024 x 4096: 4312, 4122, 3954, 4050, 4019).
constexpr int64_t GROUP_TILES = 148;
void tiles_of(int32_t rows, int32_t cols, bool pair, NsShape *s) {
    const int side = pair ? 256 : 128;
    const int64_t edge = cdiv(imin(rows, cols), side);
    s->square = (int32_t)(edge * (edge + 1) / 2);
    s->cols3 = (int32_t)cdiv(cols, side);
    s->tiles3 = (int32_t)cdiv(rows, side) * s->cols3;
}
int64_t groups_of(const MuonBatch &b, bool pair) {
    int64_t square = 0;
    for (int i = 0; i < b.shapes; ++i) {
        NsShape s;
        tiles_of(b.s[i].rows, b.s[i].cols, pair, &s);
        square += (int64_t)s.square * b.s[i].matrices;
    }
    return imax(1, square / (pair ? GROUP_TILES : 2 * GROUP_TILES));
}
// How many steps a segment has at most: what makes the fewest 64-deep blocks of products a step, one where that saves less than an eighth (near-square matrices have small singular values,
// see above: X of 512 x 576 normal numbers is off by 1.5e-3 in segments and by 8e-4 without). By the shape alone, whatever else is in the list and wherever its tiles are made
int32_t together_of(int32_t rows, int32_t cols) {
    int32_t best = 1;
    int64_t least = 0, alone = 0;  // blocks of six steps
    NsShape s;
    tiles_of(rows, cols, ns_pairs(rows, cols), &s);
    const int64_t M = cdiv(imin(rows, cols), BK), N = cdiv(imax(rows, cols), BK);
    for (int32_t n = 1; n <= MOST_TOGETHER; ++n) {
        const int64_t work = (s.square * (N + (programs_host[n].squares - 1) * M) + s.tiles3 * M) * (6 / n);
        if (n == 1) least = alone = work;
        else if (work < least && 8 * work <= 7 * alone) { best = n; least = work; }
    }
    return best;
}
struct NsScratch { __half *x, *s[SYMMETRIC]; };
// Everything about a shape but its place in memory, and with scratch that too
NsShape shape_of(const MuonShape &m, bool pair, int64_t groups, int32_t steps, Carver &cv, NsScratch *at) {
    NsShape s = {};
    s.together = (int32_t)imin(steps, together_of(m.rows, m.cols));
    s.turns = turns_of(steps, s.together);
    tiles_of(m.rows, m.cols, pair, &s);
    s.rows = m.rows; s.cols = m.cols; s.ld = m.ld;
    s.M = (int32_t)imin(m.rows, m.cols);
    s.Mld = (int32_t)muon_ld(s.M);
    s.first = m.first; s.matrices = m.matrices; s.left = m.rows <= m.cols;
    s.group = (int32_t)cdiv(m.matrices, groups);
    s.slots = (int32_t)imin(m.matrices, 2 * (int64_t)s.group);  // a group's begin while the last one's end
    at->x = cv.take<__half>((int64_t)s.slots * s.rows * s.ld);
    for (int i = 0; i < symmetric_of(s.together); ++i) s.s[i] = at->s[i] = cv.take<__half>((int64_t)s.slots * s.M * s.Mld);
    s.d = cv.take<float>((int64_t)symmetric_of(s.together) * s.slots * s.M);
    s.x[0] = m.x; s.x[1] = at->x;
    return s;
}
// [count][rows][ld] halves: boxes of 64 columns x 128 rows (of stores too), and of 64 rows x two pieces of 64 columns
int32_t maps_of(const __half *at, int64_t count, int64_t rows, int64_t ld, CUtensorMap *k, CUtensorMap *mn) {
    const uint64_t dims[3] = {(uint64_t)ld, (uint64_t)rows, (uint64_t)count}, str[2] = {(uint64_t)ld * 2, (uint64_t)(rows * ld) * 2};
    const uint32_t box[3] = {64, 128, 1};
    MOE_TRY(tc_make_map(k, at, 3, dims, str, box));
    const uint64_t dims4[4] = {64, (uint64_t)rows, (uint64_t)(ld / 64), (uint64_t)count}, str4[3] = {(uint64_t)ld * 2, 128, (uint64_t)(rows * ld) * 2};
    const uint32_t box4[4] = {64, BK, 2, 1};
    return tc_make_map(mn, at, 4, dims4, str4, box4);
}

// By as many CTAs, or pairs of them, as the device runs at once. l == nullptr: only whether it runs any
template <bool PAIR> int32_t launch_ns(const NsLaunch *l, const MuonBatch *batch, cudaStream_t st) {
    static PerDevice most;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // as launch_kernel
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = 2; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
    cfg.blockDim = dim3(NS_THREADS); cfg.dynamicSmemBytes = NS_SMEM; cfg.stream = st;
    cfg.attrs = attrs; cfg.numAttrs = PAIR ? 2 : 1;
    const auto kernel = newton_schulz_kernel<PAIR>;
    const int workers = most.get([&]() {
        if (cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM) != cudaSuccess) return 0;
        if (!PAIR) return tc_sm_count();
        int n = 0;
        cfg.gridDim = dim3(2 * (tc_sm_count() / 2));
        return cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess ? n : 0;
    });
    if (workers <= 0) return MOE_ERR_CUDA;
    if (!l) return MOE_OK;
    cfg.gridDim = dim3((PAIR ? 2 : 1) * (unsigned)imin(l->tiles, workers));
    MOE_CUDA(cudaLaunchKernelEx(&cfg, kernel, l->maps, l->args, *batch));
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace

int64_t ns_tiles(int32_t rows, int32_t cols, bool pair) {
    NsShape s;
    tiles_of(rows, cols, pair, &s);
    return 2 * (int64_t)s.square + s.tiles3;
}

int64_t ns_scratch_bytes(const MuonBatch &batch, bool pair) {
    Carver cv(nullptr);
    const int64_t groups = groups_of(batch, pair);
    NsScratch at;
    for (int i = 0; i < batch.shapes; ++i) shape_of(batch.s[i], pair, groups, MOE_MUON_MAX_STEPS, cv, &at);  // (enough for any number of steps)
    return (int64_t)cv.off;
}

int32_t prepare_newton_schulz(const NsWork &w, NsLaunch *to) {
    const MuonBatch &b = *w.batch;
    Carver cv(w.scratch);
    const int64_t groups = groups_of(b, w.pair);
    NsArgs &p = to->args;
    p = {};
    to->pair = w.pair;
    to->tiles = 0;
    p.shapes = b.shapes; p.steps = w.steps;
    for (int i = 0; i < b.shapes; ++i) {
        NsScratch at;
        NsShape &s = p.s[i];
        NsMaps &m = to->maps.m[i];
        s = shape_of(b.s[i], w.pair, groups, w.steps, cv, &at);
        MOE_TRY(maps_of(b.s[i].x, s.matrices, s.rows, s.ld, &m.x_k[0], &m.x_mn[0]));
        MOE_TRY(maps_of(at.x, s.slots, s.rows, s.ld, &m.x_k[1], &m.x_mn[1]));
        for (int j = 0; j < symmetric_of(s.together); ++j) MOE_TRY(maps_of(at.s[j], s.slots, s.M, s.Mld, &m.s_k[j], &m.s_mn[j]));
        to->tiles += (int64_t)s.matrices * tiles_of_matrix(s, w.steps);
        p.turns = (int32_t)imax(p.turns, s.turns);
        p.groups = (int32_t)imax(p.groups, cdiv(s.matrices, s.group));
    }
    if (to->tiles > (int64_t)1 << 30) return MOE_ERR_UNSUPPORTED;
    p.done = w.done; p.next = w.next; p.status = w.status; p.lr = w.lr; p.rates = w.rates;
    return w.pair ? launch_ns<true>(nullptr, nullptr, nullptr) : launch_ns<false>(nullptr, nullptr, nullptr);
}

int32_t launch_newton_schulz(const NsLaunch &l, const MuonBatch &batch, cudaStream_t st) { return l.pair ? launch_ns<true>(&l, &batch, st) : launch_ns<false>(&l, &batch, st); }

}  // namespace moe
