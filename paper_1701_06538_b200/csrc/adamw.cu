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

#include <cuda_fp8.h>

#include "block.cuh"

namespace moe {

namespace {

constexpr int THREADS = 256, EACH = 8;            // elements a thread holds at a time
constexpr int STEP = THREADS * EACH;              // elements a block holds at a time: 16 blocks of codes, 16 lanes each
constexpr int CHUNK = 4 * STEP;                   // elements of a block of the grid
constexpr int MAX_LIST = 96;                      // tensors of a launch (a launch's parameters hold them: 9 KiB)

struct Entry {
    void *w;
    const void *g;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t count, first;
    float decay;
    int32_t kind;  // bit 0: bf16 weights, 1: bf16 gradients, 2: float masters, 3: 8-bit moments
};
struct Batch {
    Entry t[MAX_LIST];
    int32_t chunks_before[MAX_LIST + 1];
    int32_t n;
};
struct Constants { float beta1, one_beta1, beta2, one_beta2, eps; };

// The low-bias hash of 32 bits of C. Wellons ("Prospecting for Hash Functions", 2018): two multiplications between three shifts
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7feb352du;
    x = (x ^ (x >> 15)) * 0x846ca68bu;
    return x ^ (x >> 16);
}

// |q| <= 448 up or down to a multiple of its code's unit: the 20 bits below e4m3's three are added a dither (at most 2^20 - 8) and cut off. Below 2^-6
// the unit stays 2^-9, which is that of the numbers from 2^-6 to 2^-5.
__device__ __forceinline__ float dithered(float q, uint32_t bits16) {
    const float size = fabsf(q);
    const bool small = size < 0.015625f;
    const float up = small ? size + 0.015625f : size;
    float z = __uint_as_float((__float_as_uint(up) + bits16 * 16u + 8u) & ~0xfffffu);
    z = small ? z - 0.015625f : z;
    return fminf(z, 448.0f);
}

template <typename T> __device__ __forceinline__ void load8(const T *p, int64_t at, int64_t live, float (&v)[EACH]) {
    if (live >= EACH) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4 *>(p + at), b = *reinterpret_cast<const float4 *>(p + at + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(p + at);
            const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
        }
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
__device__ __forceinline__ void load_codes(const uint8_t *p, int64_t at, int64_t live, float scale, float (&v)[EACH]) {
    uint32_t c[2] = {0u, 0u};
    if (live >= EACH) {
        const uint2 two = *reinterpret_cast<const uint2 *>(p + at);
        c[0] = two.x; c[1] = two.y;
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < live) c[i / 4] |= (uint32_t)p[at + i] << (8 * (i % 4));
    }
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[i / 4] >> (8 * (i % 4))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[i] = f.x * scale;
        v[i + 1] = f.y * scale;
    }
}
// The codes of a block and its scale; an element that is no finite number is held as a NaN and has no part in the scale
template <bool ROOT>
__device__ __forceinline__ void store_codes(uint8_t *p, float *scales, int64_t at, int64_t live, const float (&v)[EACH], const uint32_t (&bits)[EACH]) {
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const float a = fabsf(v[i]);
        largest = a <= FLT_MAX ? fmaxf(largest, a) : largest;
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, off));
    const float scale = largest > 0.0f ? fmaxf(largest * (1.0f / 448.0f), FLT_MIN) : 0.0f, by = scale > 0.0f ? scale : 1.0f;
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < EACH; i += 2) {
        float z[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float q = v[i + j] / by;
            float t = dithered(q, ROOT ? bits[i + j] >> 16 : bits[i + j] & 0xffffu);
            if (ROOT) t = q > 0.0f ? fmaxf(t, 0.001953125f) : t;  // a second moment that is not 0 stays above 0: it divides
            t = fabsf(v[i + j]) <= FLT_MAX ? t : __int_as_float(0x7fffffff);
            z[j] = copysignf(t, q);
        }
        const __nv_fp8x2_storage_t two = __nv_cvt_float2_to_fp8x2(make_float2(z[0], z[1]), __NV_SATFINITE, __NV_E4M3);
        c[i / 4] |= (uint32_t)two << (8 * (i % 4));
    }
    if (live >= EACH) {
        *reinterpret_cast<uint2 *>(p + at) = make_uint2(c[0], c[1]);
    } else {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i < live) p[at + i] = (uint8_t)(c[i / 4] >> (8 * (i % 4)));
    }
    if (at % MOE_ADAMW_BLOCK == 0 && live > 0) scales[at / MOE_ADAMW_BLOCK] = scale;
}

template <typename WT, typename GT, bool MASTER, bool EIGHT>
__device__ __forceinline__ void update(const Entry &t, int64_t chunk, const Constants &k, const moe_adamw_rates &r) {
    const float step = r.lr / r.bias1, root_by = 1.0f / sqrtf(r.bias2), keep = r.lr * t.decay;
    const int64_t end = min(t.count, (chunk + 1) * CHUNK);
    for (int64_t base = chunk * CHUNK; base < end; base += STEP) {
        const int64_t at = base + threadIdx.x * EACH, live = end - at;  // at most 0 behind the end
        float w[EACH], g[EACH], m[EACH], v[EACH];
        if constexpr (MASTER) load8(t.master, at, live, w);
        else load8(static_cast<const WT *>(t.w), at, live, w);
        load8(static_cast<const GT *>(t.g), at, live, g);
        uint32_t bits[EACH];
        if constexpr (EIGHT) {
            const int64_t number = t.first + at;
            const uint32_t key = mix(r.seed + (uint32_t)(number >> 32) * 0x9e3779b9u);  // a multiple of EACH: the upper half is that of all eight
            const float ms = live > 0 ? t.m_scale[at / MOE_ADAMW_BLOCK] : 0.0f, vs = live > 0 ? t.v_scale[at / MOE_ADAMW_BLOCK] : 0.0f;
            load_codes(static_cast<const uint8_t *>(t.m), at, live, ms, m);
            load_codes(static_cast<const uint8_t *>(t.v), at, live, vs, v);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                bits[i] = mix(((uint32_t)number + i) ^ key);
                v[i] *= v[i];
            }
        } else {
            load8(static_cast<const float *>(t.m), at, live, m);
            load8(static_cast<const float *>(t.v), at, live, v);
        }
        float root[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float gi = g[i] * r.grad_scale;
            m[i] = k.beta1 * m[i] + k.one_beta1 * gi;
            v[i] = k.beta2 * v[i] + k.one_beta2 * (gi * gi);
            root[i] = sqrtf(v[i]);
            w[i] = w[i] - (step * (m[i] / (root[i] * root_by + k.eps)) + keep * w[i]);
        }
        if constexpr (MASTER) store8(t.master, at, live, w);
        store8(static_cast<WT *>(t.w), at, live, w);
        if constexpr (EIGHT) {
            __syncwarp();  // a block's scales have been read by all of its lanes
            store_codes<false>(static_cast<uint8_t *>(t.m), t.m_scale, at, live, m, bits);
            store_codes<true>(static_cast<uint8_t *>(t.v), t.v_scale, at, live, root, bits);
        } else {
            store8(static_cast<float *>(t.m), at, live, m);
            store8(static_cast<float *>(t.v), at, live, v);
        }
    }
}

// A block finds its tensor in the list and takes CHUNK elements of it.
__global__ void __launch_bounds__(THREADS) adamw_kernel(const __grid_constant__ Batch b, Constants k, moe_adamw_rates given, const moe_adamw_rates *read) {
    wait_previous_kernel();
    const moe_adamw_rates r = read ? *read : given;
    int32_t lo = 0, hi = b.n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (b.chunks_before[mid] <= (int32_t)blockIdx.x) lo = mid; else hi = mid;
    }
    const Entry &t = b.t[lo];
    const int64_t chunk = (int32_t)blockIdx.x - b.chunks_before[lo];
    switch (t.kind) {
        case 0: update<float, float, false, false>(t, chunk, k, r); break;
        case 1: update<bf16, float, false, false>(t, chunk, k, r); break;
        case 2: update<float, bf16, false, false>(t, chunk, k, r); break;
        case 3: update<bf16, bf16, false, false>(t, chunk, k, r); break;
        case 5: update<bf16, float, true, false>(t, chunk, k, r); break;
        case 7: update<bf16, bf16, true, false>(t, chunk, k, r); break;
        case 8: update<float, float, false, true>(t, chunk, k, r); break;
        case 9: update<bf16, float, false, true>(t, chunk, k, r); break;
        case 10: update<float, bf16, false, true>(t, chunk, k, r); break;
        case 11: update<bf16, bf16, false, true>(t, chunk, k, r); break;
        case 13: update<bf16, float, true, true>(t, chunk, k, r); break;
        case 15: update<bf16, bf16, true, true>(t, chunk, k, r); break;
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
    const Constants k = {(float)p.beta1, (float)(1.0 - p.beta1), (float)p.beta2, (float)(1.0 - p.beta2), (float)p.eps};
    moe_adamw_rates given = {};
    if (!rates) given = {(float)p.lr, (float)(1.0 - pow(p.beta1, p.step)), (float)(1.0 - pow(p.beta2, p.step)), (float)p.grad_scale, p.seed};
    Batch b;
    b.n = 0;
    b.chunks_before[0] = 0;
    auto flush = [&]() -> int32_t {
        if (b.n == 0) return MOE_OK;
        launch_kernel(adamw_kernel, dim3((unsigned)b.chunks_before[b.n]), dim3(THREADS), 0, st, b, k, given, rates);
        MOE_LAUNCHED();
        b.n = 0;
        return MOE_OK;
    };
    for (int32_t i = 0; i < count; ++i) {
        const moe_adamw_tensor &t = tensors[i];
        if (t.count == 0) continue;
        const int64_t chunks = cdiv(t.count, CHUNK);  // at most 2^27
        if (b.n == MAX_LIST || (b.n > 0 && b.chunks_before[b.n] + chunks > (1 << 30))) MOE_TRY(flush());
        b.t[b.n] = {t.w, t.g, t.master, t.m, t.v, t.m_scale, t.v_scale, t.count, t.first, t.weight_decay,
                    (t.w_type == MOE_BF16 ? 1 : 0) | (t.g_type == MOE_BF16 ? 2 : 0) | (t.master ? 4 : 0) | (t.moment_bits == 8 ? 8 : 0)};
        b.chunks_before[b.n + 1] = b.chunks_before[b.n] + (int32_t)chunks;
        ++b.n;
    }
    return flush();
}

}  // namespace moe
