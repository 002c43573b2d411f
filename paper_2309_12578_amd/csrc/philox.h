// Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011, Section
// 4.3 and table 2: the fewest rounds that pass BigCrush), keyed by a seed and an offset that lie in device memory.
#ifndef SPION_PHILOX_H_
#define SPION_PHILOX_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spion {

// a ^ b ^ c in one instruction
__device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) { return (unsigned)__builtin_amdgcn_bitop3_b32((int)a, (int)b, (int)c, 0x96); }

struct PhiloxKey {
    unsigned k0, k1, c2, c3;   // the same for a whole launch: kept in scalar registers
    __device__ __forceinline__ PhiloxKey() : k0(0), k1(0), c2(0), c3(0) {}
    __device__ __forceinline__ PhiloxKey(const long long* __restrict__ rng, unsigned stream)
        : k0(uniform((unsigned)rng[0])), k1(uniform((unsigned)((unsigned long long)rng[0] >> 32))), c2(uniform((unsigned)rng[1])), c3(stream) {}
    static __device__ __forceinline__ unsigned uniform(unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); }
    __device__ __forceinline__ uint4 words(unsigned c0, unsigned c1) const {
        unsigned a = c0, b = c1, c = c2, d = c3, x = k0, y = k1;
        // what is uniform is made again for each call, by scalar instructions beside the vector work: kept, it takes 20 registers
        asm volatile("" : "+s"(x), "+s"(y), "+s"(c));
#pragma unroll
        for (int r = 0; r < 7; ++r) {
            const unsigned long long p = (unsigned long long)a * 0xD2511F53u, q = (unsigned long long)c * 0xCD9E8D57u;
            a = xor3((unsigned)(q >> 32), b, x);
            b = (unsigned)q;
            c = xor3((unsigned)(p >> 32), d, y);
            d = (unsigned)p;
            x += 0x9E3779B9u;
            y += 0xBB67AE85u;
        }
        return make_uint4(a, b, c, d);
    }
};

}  // namespace spion
#endif
