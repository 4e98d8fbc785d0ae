// Rows of floats or bf16 in vectors of 16 bytes
#pragma once

#include "moe_internal.cuh"

namespace moe {

// 16 bytes of a row, as pairs of floats
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ float2 get(int i) const {  // elements i, i + 1
        const uint32_t *u = reinterpret_cast<const uint32_t *>(&raw);
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(u[i]), __uint_as_float(u[i + 1]));
        else return make_float2(__uint_as_float(u[i / 2] << 16), __uint_as_float(u[i / 2] & 0xffff0000u));
    }
    __device__ __forceinline__ void set(int i, float2 v) {
        uint32_t *u = reinterpret_cast<uint32_t *>(&raw);
        if constexpr (sizeof(T) == 4) {
            u[i] = __float_as_uint(v.x);
            u[i + 1] = __float_as_uint(v.y);
        } else {
            const __nv_bfloat162 two = __floats2bfloat162_rn(v.x, v.y);
            u[i / 2] = *reinterpret_cast<const uint32_t *>(&two);
        }
    }
};
template <typename T> __device__ __forceinline__ Vec<T> load_vec(const void *base, int64_t row, int32_t d, int32_t q) {
    Vec<T> v;
    v.raw = *reinterpret_cast<const uint4 *>(static_cast<const T *>(base) + row * d + (int64_t)q * Vec<T>::N);
    return v;
}
template <typename T> __device__ __forceinline__ void store_vec(void *base, int64_t row, int32_t d, int32_t q, const Vec<T> &v) {
    *reinterpret_cast<uint4 *>(static_cast<T *>(base) + row * d + (int64_t)q * Vec<T>::N) = v.raw;
}
template <int N> __device__ __forceinline__ void load_floats(const float *p, float2 (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float4 a = *reinterpret_cast<const float4 *>(p + 2 * i);
        v[i] = make_float2(a.x, a.y);
        v[i + 1] = make_float2(a.z, a.w);
    }
}

}  // namespace moe
