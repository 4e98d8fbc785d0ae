// The first pass of the Muon step over a block's elements, 256 threads a chunk (muon.cu, muon_small.cu): m = momentum m + g and the squares of u
#pragma once

#include <float.h>
#include <math_constants.h>

#include "muon.cuh"
#include "vectors.cuh"

namespace moe {

namespace {

constexpr int PASS_THREADS = 256, EACH = 8, TURNS = 4, PASS_TURNS = 8;
constexpr int PASS_CHUNK = PASS_THREADS * EACH * PASS_TURNS;  // elements of a block of the first pass

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

// The sum of eight squares, s as it came out in float. Squares of elements below 2^-63 or so are no normal numbers, below 2^-75 they are 0: where s is small (below 2^-100, of which what s lost is 2^-46), of
// 2^100 times the elements, none of which is then above 2^50 or, but for zeros, below 2^-49
__device__ __forceinline__ double squares(float s, const float (&u)[EACH]) {
    if (s >= 0x1p-100f) return (double)s;
    float t = 0.0f;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const float v = u[j] * 0x1p100f;
        t = fmaf(v, v, t);
    }
    return (double)t * 0x1p-200;
}
// What u is multiplied by to make X of it, held as MUON_UNIT: `lift` first and `by` then, since MUON_UNIT over the least norm (eps) is beyond float's range and u times `lift` is not. A matrix whose norm is
// no finite number becomes NaN as a whole
struct Factor {
    float lift, by;
    __device__ __forceinline__ explicit Factor(double norm) {
        lift = norm < 0x1p-64 ? 0x1p64f : 1.0f;
        by = norm <= (double)FLT_MAX ? (float)((double)MUON_UNIT / (norm * (double)lift)) : CUDART_NAN_F;
    }
    __device__ __forceinline__ float operator()(float u) const { return u * lift * by; }
};

// Eight elements as they are loaded
template <typename T, bool VECTORS> struct Eight {
    static constexpr int N = VECTORS ? Vec<T>::N : EACH;
    Vec<T> raw[VECTORS ? EACH / N : 1];
    float v[VECTORS ? 1 : EACH];
    __device__ __forceinline__ void load(const T *p, int64_t at, int64_t live) {
        if constexpr (VECTORS) {
#pragma unroll
            for (int i = 0; i < EACH / N; ++i) raw[i].raw = *reinterpret_cast<const uint4 *>(p + at + i * N);
        } else {
            load8<T, false>(p, at, live, v);
        }
    }
    __device__ __forceinline__ void get(float (&to)[EACH]) const {
#pragma unroll
        for (int j = 0; j < EACH; j += 2) {
            if constexpr (VECTORS) {
                const float2 f = raw[j / N].get(j % N);
                to[j] = f.x;
                to[j + 1] = f.y;
            } else {
                to[j] = v[j];
                to[j + 1] = v[j + 1];
            }
        }
    }
};
// Squares are added up in float over eight elements, then in double. All loads of a round before its first store: as many as there are registers for. (bf16 gradients
// and momentum, 512 of 512 x 1024 with all else, graph replay: by eights in one round of eight 4019 us, in one of four kept as floats 4144; the
// pass by itself 231 and 413 us, 7.0 TB/s; float momentum 381 and 431, 7.1 TB/s)
template <typename GT, typename MT, bool VECTORS>
__device__ __forceinline__ double momentum_chunk(const GT *g, MT *m, int64_t at, int64_t end, float grad_scale, const MuonPasses &k) {
    constexpr int ROUND = VECTORS && sizeof(GT) + sizeof(MT) == 4 ? PASS_TURNS : TURNS;
    double sum = 0.0;
    const int64_t first = at + (int64_t)(threadIdx.x % PASS_THREADS) * EACH;
#pragma unroll 1
    for (int round = 0; round < PASS_TURNS; round += ROUND) {
        Eight<GT, VECTORS> gq[ROUND];
        Eight<MT, VECTORS> mq[ROUND];
#pragma unroll
        for (int i = 0; i < ROUND; ++i) {
            const int64_t here = first + (int64_t)(round + i) * (PASS_THREADS * EACH), live = end - here;
            if (live > 0) {
                gq[i].load(g, here, live);
                mq[i].load(m, here, live);
            }
        }
#pragma unroll
        for (int i = 0; i < ROUND; ++i) {
            const int64_t here = first + (int64_t)(round + i) * (PASS_THREADS * EACH), live = end - here;
            if (live <= 0) continue;
            float gv[EACH], mv[EACH], u[EACH], s = 0.0f;
            gq[i].get(gv);
            mq[i].get(mv);
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
                const float gj = gv[j] * grad_scale;
                mv[j] = held<MT>(fmaf(k.momentum, mv[j], gj));
                u[j] = k.nesterov ? fmaf(k.momentum, mv[j], gj) : mv[j];
                s = fmaf(u[j], u[j], s);
            }
            store8<MT, VECTORS>(m, here, live, mv);
            sum += squares(s, u);
        }
    }
    return sum;
}
template <bool VECTORS>
__device__ __forceinline__ double momentum_block(const MuonEntry &t, int64_t at, int64_t end, float grad_scale, const MuonPasses &k) {
    switch (t.kind & 6) {
        case 0: return momentum_chunk<float, float, VECTORS>(static_cast<const float *>(t.g), static_cast<float *>(t.m), at, end, grad_scale, k);
        case 2: return momentum_chunk<bf16, float, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<float *>(t.m), at, end, grad_scale, k);
        case 4: return momentum_chunk<float, bf16, VECTORS>(static_cast<const float *>(t.g), static_cast<bf16 *>(t.m), at, end, grad_scale, k);
        default: return momentum_chunk<bf16, bf16, VECTORS>(static_cast<const bf16 *>(t.g), static_cast<bf16 *>(t.m), at, end, grad_scale, k);
    }
}

}  // namespace

}  // namespace moe
