// Values of the three floating types as the norm, clipping and embedding kernels read and write them: V consecutive values a
// lane, held as fp32 in between.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mqgrad.h"

namespace mqg {
namespace values {

constexpr int kF32 = MQG_FLOAT32, kF16 = MQG_FLOAT16, kBF16 = MQG_BFLOAT16;
constexpr uint32_t bytes_of(int dtype) { return dtype == kF32 ? 4u : 2u; }

// one value
template <int DTYPE>
__device__ __forceinline__ float load_one(const void* p, uint64_t i) {
    if constexpr (DTYPE == kF32) return reinterpret_cast<const float*>(p)[i];
    else if constexpr (DTYPE == kF16) return (float)reinterpret_cast<const _Float16*>(p)[i];
    else return __builtin_bit_cast(float, (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
}
template <int DTYPE>
__device__ __forceinline__ void store_one(void* p, uint64_t i, float x) {
    if constexpr (DTYPE == kF32) reinterpret_cast<float*>(p)[i] = x;
    else if constexpr (DTYPE == kF16) reinterpret_cast<_Float16*>(p)[i] = (_Float16)x;
    else reinterpret_cast<__bf16*>(p)[i] = (__bf16)x;
}
template <int BYTES>
struct Words;
template <>
struct Words<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2)));
};
template <>
struct Words<16> {
    typedef uint32_t type __attribute__((ext_vector_type(4)));
};

// Global memory takes accesses of 8 and 16 bytes at any address: a tensor need only be aligned to its values.
template <int DTYPE, int V>
struct Pack {
    static constexpr int kBytes = V * (int)bytes_of(DTYPE), kPart = kBytes > 16 ? 16 : kBytes, kParts = kBytes / kPart;
    typedef typename Words<kPart>::type Part;
    typedef Part AnyPart __attribute__((aligned(2)));
    Part part[kParts];

    __device__ __forceinline__ void load(const void* p) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) part[i] = reinterpret_cast<const AnyPart*>(p)[i];
    }
    __device__ __forceinline__ void load_once(const void* p) {   // streaming
#pragma unroll
        for (int i = 0; i < kParts; ++i) part[i] = __builtin_nontemporal_load(reinterpret_cast<const AnyPart*>(p) + i);
    }
    __device__ __forceinline__ void store(void* p) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) reinterpret_cast<AnyPart*>(p)[i] = part[i];
    }
    __device__ __forceinline__ void store_once(void* p) const {   // streaming
#pragma unroll
        for (int i = 0; i < kParts; ++i) __builtin_nontemporal_store(part[i], reinterpret_cast<AnyPart*>(p) + i);
    }
    __device__ __forceinline__ void get(float (&x)[V]) const {
        uint32_t w[kBytes / 4];
        __builtin_memcpy(w, part, sizeof w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (DTYPE == kF32) {
                x[i] = __builtin_bit_cast(float, w[i]);
            } else {
                const uint16_t h = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                if constexpr (DTYPE == kF16) x[i] = (float)__builtin_bit_cast(_Float16, h);
                else x[i] = __builtin_bit_cast(float, (uint32_t)h << 16);
            }
        }
    }
    // the first `count` of V values, the others 0
    __device__ __forceinline__ void load_some(const void* p, uint32_t count) {
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (uint32_t)i < count ? load_one<DTYPE>(p, i) : 0.0f;
        set(x);
    }
    // rounded once, to the nearest value, ties to even
    __device__ __forceinline__ void set(const float (&x)[V]) {
        uint32_t w[kBytes / 4];
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) {
            if constexpr (DTYPE == kF32) {
                w[i] = __builtin_bit_cast(uint32_t, x[i]);
            } else if constexpr (DTYPE == kF16) {
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * i + 1]) << 16;
            } else {
                w[i] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * i + 1]) << 16;
            }
        }
        __builtin_memcpy(part, w, sizeof w);
    }
};

template <int DTYPE>
__device__ __forceinline__ const void* at(const void* p, uint64_t i) { return static_cast<const char*>(p) + i * bytes_of(DTYPE); }
template <int DTYPE>
__device__ __forceinline__ void* at(void* p, uint64_t i) { return static_cast<char*>(p) + i * bytes_of(DTYPE); }

// f(integral_constant<int, dtype>)
template <class F>
__host__ __device__ __forceinline__ auto with_dtype(int dtype, F f) {
    if (dtype == kF32) return f(std::integral_constant<int, kF32>{});
    if (dtype == kF16) return f(std::integral_constant<int, kF16>{});
    return f(std::integral_constant<int, kBF16>{});
}

}  // namespace values
}  // namespace mqg
