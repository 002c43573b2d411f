// Eight consecutive elements of fp32 or bf16 at any address, as 16-byte accesses where all eight are there.
#ifndef SPION_CHUNKS_H_
#define SPION_CHUNKS_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spion {

template <typename T>
struct Eight {
    T v[8];
};
struct __attribute__((packed, aligned(2))) Words {   // 16 bytes at any address
    unsigned w[4];
};

template <typename T, bool WHOLE>
__device__ __forceinline__ void load8(float (&v)[8], const T* p, int n) {
    if constexpr (WHOLE) {
        Eight<T> e;
        constexpr int words = sizeof(e) / 16;
#pragma unroll
        for (int i = 0; i < words; ++i) reinterpret_cast<Words*>(&e)[i] = reinterpret_cast<const Words*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)e.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.f;
    }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store8(T* p, const float (&v)[8], int n) {
    if constexpr (WHOLE) {
        Eight<T> e;
        constexpr int words = sizeof(e) / 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) e.v[i] = (T)v[i];
#pragma unroll
        for (int i = 0; i < words; ++i) reinterpret_cast<Words*>(p)[i] = reinterpret_cast<const Words*>(&e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

}  // namespace spion
#endif
