// AdamW (Loshchilov and Hutter, 2019) over a list of tensors, moments in float or in 8 bits. One pass over memory: every element's
// weight, gradient and moments are read once and what changes is written once; nothing else bounds it but, with 8-bit moments, the
// arithmetic of the codes.
//
// 8-bit moments: a block of MOE_ADAMW_BLOCK consecutive elements shares a float scale, the largest magnitude over 448, and holds e4m3
// codes of m / scale and of sqrt(v) / scale. The square root halves v's range in powers of two, so that the 17 binades of e4m3 are 34
// of v, and the update needs it anyway. A second moment changes by (1 - beta2) of itself a step, 1e-3, and a code's neighbour is
// 6 to 12 % away: rounded to nearest it would never move. Codes are therefore rounded up or down at random, the chance being the distance to the
// neighbours, with bits that are a hash of the caller's seed and the element's number: the same call gives the same codes.
#include <float.h>
#include <math.h>

#include <type_traits>

#include <cuda_fp8.h>

#include "block.cuh"
#include "pairs.cuh"
#include "tc.cuh"

namespace moe {

namespace {

constexpr int THREADS = 256, EACH = 8;            // elements a thread holds at a time
constexpr int STEP = THREADS * EACH;              // elements a block holds at a time: 16 blocks of codes, 16 lanes each
constexpr int FLOAT_STEPS = 4, MOST_STEPS = 16;   // steps of a block of the grid: with float moments (16 of them: 163 us for 33 million elements, not 144); with 8-bit ones at most,
                                                  // which have more to do before the first (268 million elements: 4, 8, 16 and 32 steps 635, 612, 605 and 609 us)
constexpr int EIGHT_BLOCKS = 3;                   // blocks of an SM with 8-bit moments (4, whose 64 registers are too few: 642 us with 4 steps; 2: 763)
constexpr int MAX_LIST = 96;                      // tensors of a launch (a launch's parameters hold them: 9 KiB)

struct Entry {
    void *w;
    const void *g;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t count, first;
    float decay;
    int32_t kind;  // bit 0: bf16 weights, 1: bf16 gradients, 2: float masters
};
struct Batch {
    Entry t[MAX_LIST];
    int32_t chunks_before[MAX_LIST + 1];
    int32_t n, steps;
};
struct Constants { float beta1, one_beta1, beta2, one_beta2, eps, one; };

// The low-bias hash of 32 bits of C. Wellons ("Prospecting for Hash Functions", 2018): two multiplications between three shifts. mix_inner: without the first shift, which is the same for
// numbers that differ in their lower half alone, and the last, which changes the lower half alone
__device__ __forceinline__ uint32_t mix_inner(uint32_t x) {
    x *= 0x7feb352du;
    return (x ^ (x >> 15)) * 0x846ca68bu;
}
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = mix_inner(x ^ (x >> 16));
    return x ^ (x >> 16);
}

// The hardware's root and reciprocal, within two units of the last place: of the divisor of a step
__device__ __forceinline__ float root_of(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Minus the roots of two second moments, which are given as minus v: the hardware's reciprocal root y, s = v y and a Newton step s + (v - s s) y / 2, whose rounding is that of
// the root itself but for one in a million or so. What goes into a code has to be exact: a unit of the last place turns a code over in one element of 600,000, and a code is 6 to 12 %.
// Of v below float's smallest normal number it is off, but still between 0 and that number's root; of an infinite v it is a NaN, which it is held as too.
__device__ __forceinline__ float2 minus_roots(float2 minus_v) {
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(-minus_v.x, FLT_MIN)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(-minus_v.y, FLT_MIN)));
    const float2 s = mul2(minus_v, y);
    return fma2(fma2(s, s, minus_v), mul2(y, both(0.5f)), s);
}
__device__ __forceinline__ float reciprocal(float v) {  // of normal numbers; 0 beyond 2^126
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float is_below(float a, float b) {  // 1 or 0
    float r;
    asm("set.lt.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_of_block(float v) {  // over the half of a warp that holds a block of codes; a NaN stays. (One redux.sync for the four steps: 687 us, not 647.)
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, v, off);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(o));
    }
    return v;
}
__device__ __forceinline__ float max_size(float a, float b, float c) {  // of three magnitudes
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Eight elements as they stand in memory
template <typename T> struct Raw8 {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void floats(float (&v)[EACH]) const {
        const uint32_t *u = reinterpret_cast<const uint32_t *>(q);
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] = sizeof(T) == 4 ? __uint_as_float(u[i * sizeof(T) / 4]) : __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};
template <typename T> __device__ __forceinline__ void load8(const T *p, int64_t at, int64_t live, float (&v)[EACH]) {
    if (live >= EACH) {
        Raw8<T> raw;
        raw.load(p + at);
        raw.floats(v);
        return;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) v[i] = i < live ? to_f32(p[at + i]) : 0.0f;
}
template <typename T> __device__ __forceinline__ void store8(T *p, int64_t at, int64_t live, const float (&v)[EACH]) {
    if (live >= EACH) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(p + at) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(p + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                u[i] = *reinterpret_cast<const uint32_t *>(&two);
            }
            *reinterpret_cast<uint4 *>(p + at) = make_uint4(u[0], u[1], u[2], u[3]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (i < live) p[at + i] = from_f32<T>(v[i]);
}
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int64_t at, int64_t live) {
    if (live >= EACH) return *reinterpret_cast<const uint2 *>(p + at);
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (i < live) c[i / 4] |= (uint32_t)p[at + i] << (8 * (i % 4));
    return make_uint2(c[0], c[1]);
}
__device__ __forceinline__ void decode(const uint2 &two, float (&v)[EACH]) {
    const uint32_t c[2] = {two.x, two.y};
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[i / 4] >> (8 * (i % 4))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[i] = f.x;
        v[i + 1] = f.y;
    }
}
// The codes of a block and its scale; an element that is no finite number is held as a NaN and has no part in the scale. ROOT: minus values of 0 and more, whose codes stay above 0 (they
// divide). bits: the hash without its last shift; its upper half is that of the hash, the lower half changes
template <bool ROOT, bool FULL>
__device__ __forceinline__ void store_codes(uint8_t *p, float *scale_at, int64_t live, const float (&v)[EACH], const uint32_t (&bits)[EACH]) {
    static_assert(EACH == 8, "its magnitudes, two at a time behind the first");
    float largest = max_size(max_size(max_size(max_size(v[0], v[1], v[2]), v[3], v[4]), v[5], v[6]), v[7], 0.0f);
    largest = max_of_block(largest);
    const bool odd = __any_sync(0xffffffffu, !(largest <= FLT_MAX));  // rare: the largest of the others
    if (odd) {
        largest = 0.0f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) largest = fabsf(v[i]) <= FLT_MAX ? fmaxf(largest, fabsf(v[i])) : largest;
        largest = max_of_block(largest);
    }
    const float scale = largest > 0.0f ? fmaxf(largest * (1.0f / 448.0f), FLT_MIN) : 0.0f, guess = reciprocal(scale);
    // Values over the scale, rounded as a division rounds: a product with the reciprocal, its remainder, and the product corrected by it (Markstein, 1990)
    const float by = largest > 0.0f ? fmaf(fmaf(-scale, guess, 1.0f), guess, guess) : 0.0f;
    uint32_t c[2] = {0u, 0u};
    // Up or down to a multiple of the code's unit: the 20 bits below e4m3's three are added a dither (16 random bits in bits 4 to 19, and 8) and cut off, whatever the sign. Below 2^-6
    // the unit stays 2^-9, which is that of the numbers from 2^-6 to 2^-5. (Up from 448 gives 480, which the conversion takes for 448.)
    const float near = ROOT ? -by : by, off_by = ROOT ? scale : -scale;
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
        const float2 of = make_float2(v[i], v[i + 1]), first = mul2(of, both(near)), q = fma2(fma2(first, both(off_by), of), both(near), first);
        float2 small = make_float2(is_below(fabsf(q.x), 0.015625f), is_below(fabsf(q.y), 0.015625f));
        if (!ROOT) small = make_float2(copysignf(small.x, q.x), copysignf(small.y, q.y));
        const float2 up = fma2(small, both(0.015625f), q);
        auto cut = [&](float u, uint32_t x) {
            const uint32_t dither = ROOT ? (x & 0xffff0000u) | 0x8000u : (x * 0x10000u + 0x8000u) ^ (x & 0xffff0000u);  // 12 bits up: the hash's upper half, or its lower half
            return __uint_as_float((__float_as_uint(u) + (dither >> 12)) & ~0xfffffu);
        };
        const float2 z = fma2(small, both(-0.015625f), make_float2(cut(up.x, bits[i]), cut(up.y, bits[i + 1])));
        const __nv_fp8x2_storage_t two = __nv_cvt_float2_to_fp8x2(z, __NV_SATFINITE, __NV_E4M3);
        c[i / 4] |= (uint32_t)two << (8 * (i % 4));
    }
    // the smallest code at least for a root that is not 0. Few codes are 0: one test for four of them
    if (ROOT)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if ((c[j] - 0x01010101u) & ~c[j] & 0x80808080u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((c[j] >> (8 * i) & 0xffu) == 0 && v[4 * j + i] != 0.0f) c[j] |= 1u << (8 * i);
    if (odd)
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (!(fabsf(v[i]) <= FLT_MAX)) c[i / 4] |= 0x7fu << (8 * (i % 4));
    if (FULL || live >= EACH) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(c[0], c[1]);
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < live) p[i] = (uint8_t)(c[i / 4] >> (8 * (i % 4)));
    }
    if (threadIdx.x % (MOE_ADAMW_BLOCK / EACH) == 0 && (FULL || live > 0)) *scale_at = scale;
}

template <typename WT, typename GT, bool MASTER>
__device__ __forceinline__ void update(const Entry &t, int64_t chunk, const Constants &k, const moe_adamw_rates &r) {
    const float step = r.lr / r.bias1, root_by = 1.0f / sqrtf(r.bias2), keep = r.lr * t.decay;
    constexpr int CHUNK = FLOAT_STEPS * STEP;
    const int64_t end = min(t.count, (chunk + 1) * CHUNK);
    for (int64_t base = chunk * CHUNK; base < end; base += STEP) {
        const int64_t at = base + threadIdx.x * EACH, live = end - at;  // at most 0 behind the end
        float w[EACH], g[EACH], m[EACH], v[EACH];
        if constexpr (MASTER) load8(t.master, at, live, w);
        else load8(static_cast<const WT *>(t.w), at, live, w);
        load8(static_cast<const GT *>(t.g), at, live, g);
        load8(static_cast<const float *>(t.m), at, live, m);
        load8(static_cast<const float *>(t.v), at, live, v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float gi = g[i] * r.grad_scale;
            m[i] = k.beta1 * m[i] + k.one_beta1 * gi;
            v[i] = k.beta2 * v[i] + k.one_beta2 * (gi * gi);
            w[i] = w[i] - (step * __fdividef(m[i], fmaf(root_of(v[i]), root_by, k.eps)) + keep * w[i]);
        }
        if constexpr (MASTER) store8(t.master, at, live, w);
        store8(static_cast<WT *>(t.w), at, live, w);
        store8(static_cast<float *>(t.m), at, live, m);
        store8(static_cast<float *>(t.v), at, live, v);
    }
}

// With 8-bit moments the arithmetic is more than the memory: 59 instructions an element (93 as it was written first: 1218 us), 576 us for 268
// million elements, whose bytes take 415. begin: the block's first element; FULL: none of its steps meets the tensor's end
template <typename WT, typename GT, bool MASTER, bool FULL>
__device__ __forceinline__ void update_eight(const Entry &t, int64_t begin, int32_t steps, const Constants &k, const moe_adamw_rates &r) {
    using MT = typename std::conditional<MASTER, float, WT>::type;  // of what the step is taken on
    const float down = -r.lr / r.bias1, root_by = 1.0f / sqrtf(r.bias2), decay = t.decay * r.bias1;
    const float by_g = k.one_beta1 * r.grad_scale, minus_by_gg = -k.one_beta2 * r.grad_scale * r.grad_scale;
    const int64_t at = begin + threadIdx.x * EACH;
    WT *w_at = static_cast<WT *>(t.w) + at;
    MT *from = MASTER ? reinterpret_cast<MT *>(t.master) + at : reinterpret_cast<MT *>(w_at);
    const GT *g_at = static_cast<const GT *>(t.g) + at;
    uint8_t *m_at = static_cast<uint8_t *>(t.m) + at, *v_at = static_cast<uint8_t *>(t.v) + at;
    float *ms_at = t.m_scale + at / MOE_ADAMW_BLOCK, *vs_at = t.v_scale + at / MOE_ADAMW_BLOCK;
    int64_t live = FULL ? EACH : t.count - at;  // at most 0 behind the end
    uint64_t number = (uint64_t)(t.first + at);  // a multiple of EACH: adding is setting bits
    const uint32_t seed = r.seed;
    struct Held {
        Raw8<MT> w;
        Raw8<GT> g;
        uint2 m, v;
        float ms, vs;
    } held;
    auto fetch = [&](int i) {
        held.w.load(from + i * STEP);
        held.g.load(g_at + i * STEP);
        held.m = *reinterpret_cast<const uint2 *>(m_at + i * STEP);
        held.v = *reinterpret_cast<const uint2 *>(v_at + i * STEP);
        held.ms = ms_at[i * (STEP / MOE_ADAMW_BLOCK)];
        held.vs = vs_at[i * (STEP / MOE_ADAMW_BLOCK)];
    };
    if constexpr (FULL) fetch(0);
#pragma unroll 1
    for (int32_t i = 0; i < steps; ++i) {
        if (!FULL && begin + i * STEP >= t.count) break;  // the whole block
        float g[EACH], m[EACH], root[EACH], w[EACH];
        uint2 m_codes, v_codes;
        float ms, vs;
        if constexpr (FULL) {
            held.w.floats(w);
            held.g.floats(g);
            m_codes = held.m; v_codes = held.v; ms = held.ms; vs = held.vs;
            if (i + 1 < steps) fetch(1);
        } else {
            load8(from, 0, live, w);
            load8(g_at, 0, live, g);
            m_codes = load_codes(m_at, 0, live);
            v_codes = load_codes(v_at, 0, live);
            ms = live > 0 ? *ms_at : 0.0f;
            vs = live > 0 ? *vs_at : 0.0f;
        }
        uint32_t key = mix(seed + (uint32_t)(number >> 32) * 0x9e3779b9u) ^ (uint32_t)number;
        key ^= key >> 16;
        uint32_t bits[EACH];
        decode(m_codes, m);
        decode(v_codes, root);
#pragma unroll
        for (int e = 0; e < EACH; e += 2) {
            bits[e] = mix_inner(key ^ e);
            bits[e + 1] = mix_inner(key ^ (e + 1));
            const float2 gg = make_float2(g[e], g[e + 1]);
            // Every product and sum rounded by itself, as the formulas have them: other roundings are as good, but turn codes over (minus_roots()). A sum is a
            // multiply-add by a 1 that the compiler does not know: of a packed product and a packed sum the assembler makes one multiply-add
            const float2 mm = fma2(both(k.one), mul2(both(k.beta1), mul2(make_float2(m[e], m[e + 1]), both(ms))), mul2(both(by_g), gg));
            const float2 old = mul2(make_float2(root[e], root[e + 1]), both(vs));
            const float2 rt = minus_roots(fma2(both(k.one), mul2(both(-k.beta2), mul2(old, old)), mul2(both(minus_by_gg), mul2(gg, gg)))), den = fma2(rt, both(-root_by), both(k.eps));
            // w - lr / bias1 (m / den + weight_decay bias1 w): the step is one number before it meets the weight. (1 - lr weight_decay as a factor of the weight is rounded to 2^-24, which is
            // all of a small rate)
            const float2 old_w = make_float2(w[e], w[e + 1]), part = mul2(mm, make_float2(reciprocal(den.x), reciprocal(den.y)));
            const float2 ww = fma2(fma2(old_w, both(decay), part), both(down), old_w);
            m[e] = mm.x; m[e + 1] = mm.y;
            root[e] = rt.x; root[e + 1] = rt.y;
            w[e] = ww.x; w[e + 1] = ww.y;
        }
        if constexpr (MASTER) store8(from, 0, live, w);
        store8(w_at, 0, live, w);
        __syncwarp();  // a block's scales have been read by all of its lanes
        store_codes<false, FULL>(m_at, ms_at, live, m, bits);
        store_codes<true, FULL>(v_at, vs_at, live, root, bits);
        w_at += STEP; from += STEP; g_at += STEP; m_at += STEP; v_at += STEP; ms_at += STEP / MOE_ADAMW_BLOCK; vs_at += STEP / MOE_ADAMW_BLOCK;
        number += STEP;
        if (!FULL) live -= STEP;
    }
}
template <typename WT, typename GT, bool MASTER>
__device__ __forceinline__ void update_eight(const Entry &t, int64_t begin, int32_t steps, const Constants &k, const moe_adamw_rates &r) {
    if (begin + steps * STEP <= t.count) update_eight<WT, GT, MASTER, true>(t, begin, steps, k, r);
    else update_eight<WT, GT, MASTER, false>(t, begin, steps, k, r);
}

// A block finds its tensor in the list and takes b.steps steps of it. Tensors with 8-bit moments are launched apart from those with float ones, whose kernel needs fewer registers.
template <bool EIGHT>
__global__ void __launch_bounds__(THREADS, EIGHT ? EIGHT_BLOCKS : 3) adamw_kernel(const __grid_constant__ Batch b, Constants k, moe_adamw_rates given, const moe_adamw_rates *read) {
    wait_previous_kernel();
    const moe_adamw_rates r = read ? *read : given;
    int32_t lo = 0, hi = b.n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (b.chunks_before[mid] <= (int32_t)blockIdx.x) lo = mid; else hi = mid;
    }
    const Entry &t = b.t[lo];
    const int64_t chunk = (int32_t)blockIdx.x - b.chunks_before[lo];
    if constexpr (EIGHT) {
        const int64_t begin = chunk * b.steps * STEP;
        switch (t.kind) {
            case 0: update_eight<float, float, false>(t, begin, b.steps, k, r); break;
            case 1: update_eight<bf16, float, false>(t, begin, b.steps, k, r); break;
            case 2: update_eight<float, bf16, false>(t, begin, b.steps, k, r); break;
            case 3: update_eight<bf16, bf16, false>(t, begin, b.steps, k, r); break;
            case 5: update_eight<bf16, float, true>(t, begin, b.steps, k, r); break;
            case 7: update_eight<bf16, bf16, true>(t, begin, b.steps, k, r); break;
        }
    } else {
        switch (t.kind) {
            case 0: update<float, float, false>(t, chunk, k, r); break;
            case 1: update<bf16, float, false>(t, chunk, k, r); break;
            case 2: update<float, bf16, false>(t, chunk, k, r); break;
            case 3: update<bf16, bf16, false>(t, chunk, k, r); break;
            case 5: update<bf16, float, true>(t, chunk, k, r); break;
            case 7: update<bf16, bf16, true>(t, chunk, k, r); break;
        }
    }
}

int32_t check_tensor(const moe_adamw_tensor &t) {
    if (t.count < 0 || t.count > (int64_t)1 << 40) return MOE_ERR_INVALID_ARG;
    if ((t.w_type != MOE_F32 && t.w_type != MOE_BF16) || (t.g_type != MOE_F32 && t.g_type != MOE_BF16)) return MOE_ERR_INVALID_ARG;
    if (t.moment_bits != 32 && t.moment_bits != 8) return MOE_ERR_INVALID_ARG;
    if (!(t.weight_decay >= 0.0f) || !(t.weight_decay <= FLT_MAX)) return MOE_ERR_INVALID_ARG;
    if (t.first < 0 || t.first % MOE_ADAMW_BLOCK != 0) return MOE_ERR_INVALID_ARG;
    if (t.count == 0) return MOE_OK;
    const void *all[] = {t.w, t.g, t.m, t.v};
    for (const void *p : all)
        if (!p || !aligned16(p)) return MOE_ERR_INVALID_ARG;
    if (t.master && (t.w_type != MOE_BF16 || !aligned16(t.master))) return MOE_ERR_INVALID_ARG;
    if (t.moment_bits == 8 && (!t.m_scale || !t.v_scale || ((uintptr_t)t.m_scale & 3) || ((uintptr_t)t.v_scale & 3))) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

}  // namespace

int32_t launch_adamw(const moe_adamw_tensor *tensors, int32_t count, const moe_adamw_params &p, const moe_adamw_rates *rates, cudaStream_t st) {
    for (int32_t i = 0; i < count; ++i) MOE_TRY(check_tensor(tensors[i]));
    const Constants k = {(float)p.beta1, (float)(1.0 - p.beta1), (float)p.beta2, (float)(1.0 - p.beta2), (float)p.eps, 1.0f};
    moe_adamw_rates given = {};
    if (!rates) given = {(float)p.lr, (float)(1.0 - pow(p.beta1, p.step)), (float)(1.0 - pow(p.beta2, p.step)), (float)p.grad_scale, p.seed};
    Batch lists[2];  // of float moments, of 8-bit ones
    auto flush = [&](int eight) -> int32_t {
        Batch &b = lists[eight];
        if (b.n == 0) return MOE_OK;
        launch_kernel(eight ? adamw_kernel<true> : adamw_kernel<false>, dim3((unsigned)b.chunks_before[b.n]), dim3(THREADS), 0, st, b, k, given, rates);
        MOE_LAUNCHED();
        b.n = 0;
        return MOE_OK;
    };
    int64_t all = 0;  // elements with 8-bit moments
    for (int32_t i = 0; i < count; ++i) all = imin(all + (tensors[i].moment_bits == 8 ? tensors[i].count : 0), (int64_t)1 << 41);
    for (Batch &b : lists) b.n = b.chunks_before[0] = 0;
    lists[0].steps = FLOAT_STEPS;
    lists[1].steps = (int32_t)imax(1, imin(MOST_STEPS, all / ((int64_t)4 * EIGHT_BLOCKS * tc_sm_count() * STEP)));  // four blocks for each that an SM holds, if there are as many
    for (int32_t i = 0; i < count; ++i) {
        const moe_adamw_tensor &t = tensors[i];
        if (t.count == 0) continue;
        const int eight = t.moment_bits == 8;
        Batch &b = lists[eight];
        const int64_t chunks = cdiv(t.count, b.steps * STEP);  // at most 2^27
        if (b.n == MAX_LIST || (b.n > 0 && b.chunks_before[b.n] + chunks > (1 << 30))) MOE_TRY(flush(eight));
        b.t[b.n] = {t.w, t.g, t.master, t.m, t.v, t.m_scale, t.v_scale, t.count, t.first, t.weight_decay,
                    (t.w_type == MOE_BF16 ? 1 : 0) | (t.g_type == MOE_BF16 ? 2 : 0) | (t.master ? 4 : 0)};
        b.chunks_before[b.n + 1] = b.chunks_before[b.n] + (int32_t)chunks;
        ++b.n;
    }
    MOE_TRY(flush(0));
    return flush(1);
}

}  // namespace moe
