// The end of a bias table's gradient: sums by bucket, of every thread's own copy, of a workgroup's threads, of a head's workgroups.
#ifndef SPION_TABLE_GRAD_H_
#define SPION_TABLE_GRAD_H_

#include <hip/hip_runtime.h>

#include "attn_bf16_tiles.h"

namespace spion {

// Threads of a workgroup: at most 64 KB of copies in LDS.
inline int table_grad_threads(int n_buckets) { return n_buckets <= 64 ? 256 : 64; }

// hist [n_buckets][threads] in LDS.  Workgroup `part` of `parts` (fewer than 2^kArriveBits) of head h leaves its sums in
// partial[h][part][n_buckets]; the last of them to arrive adds the parts up in their order and writes column h of dtable
// [n_buckets, H].  All threads of the workgroup; every order is fixed.
__device__ __forceinline__ void finish_table_grad(float* hist, int n_buckets, int part, int parts, int h, int H, float* __restrict__ partial,
                                                  unsigned long long* __restrict__ counters, unsigned long long tag, void* __restrict__ dtable,
                                                  bool is_bf16) {
    const int tid = threadIdx.x, threads = blockDim.x;
    __syncthreads();
    // a wave takes every (threads / 64)th bucket: its copies, 64 at a time, then over the lanes
    const int lane = tid & 63, wave = tid >> 6, waves = threads >> 6;
    for (int b = wave; b < n_buckets; b += waves) {
        float v = 0.f;
        for (int i = lane; i < threads; i += 64) v += hist[b * threads + i];
        for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
        if (lane == 0)
            __hip_atomic_store(&partial[((size_t)h * parts + part) * n_buckets + b], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // (the flag's place: every wave is done with the copies behind the first barrier of this call)
    if (!last_to_arrive(counters + h, tag, parts, reinterpret_cast<int*>(hist))) return;
    for (int b = tid; b < n_buckets; b += threads) {
        float v = 0.f;
        for (int p = 0; p < parts; ++p)
            v += __hip_atomic_load(&partial[((size_t)h * parts + p) * n_buckets + b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const size_t at = (size_t)b * H + h;
        if (is_bf16) static_cast<bf16_t*>(dtable)[at] = (bf16_t)v;
        else static_cast<float*>(dtable)[at] = v;
    }
}

}  // namespace spion
#endif
