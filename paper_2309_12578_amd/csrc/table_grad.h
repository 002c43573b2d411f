// The end of a bias table's gradient: sums by bucket, of every thread's own copy, then of a head's workgroups.  Every order is fixed.
#ifndef SPION_TABLE_GRAD_H_
#define SPION_TABLE_GRAD_H_

#include <hip/hip_runtime.h>

#include "attn_common.h"

namespace spion {

// Threads of a workgroup: at most 64 KB of copies in LDS.
inline int table_grad_threads(int n_buckets) { return n_buckets <= 64 ? 256 : 64; }

// Four sums whose diagonals lie beside each other, into this thread's own copy; far diagonals share their bucket mostly, and then it is one
// addition.  Plain reads and writes, as nothing else touches the copy: additions by the LDS unit took twice the time of the whole kernel.
__device__ __forceinline__ void add_four(float* copy, int threads, const float* v, unsigned buckets, int n_buckets) {
    float sum = v[0];
    int in = min((int)(buckets & 255u), n_buckets - 1);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        const int next = min((int)(buckets >> (8 * i) & 255u), n_buckets - 1);
        if (next != in) {
            copy[in * threads] += sum;
            sum = 0.f;
            in = next;
        }
        sum += v[i];
    }
    copy[in * threads] += sum;
}

struct __attribute__((packed)) FourBuckets { unsigned u; };   // at any address

// result(b, sum of value(b, 0 .. count - 1)) for every bucket b: `team` neighbouring lanes add up a bucket together, a fixed
// share each, then by exchanges between lanes.  All threads of the workgroup.
template <typename Value, typename Result>
__device__ __forceinline__ void sums_by_bucket(int n_buckets, int count, Value value, Result result) {
    const int tid = threadIdx.x, threads = blockDim.x;
    int team = 64;
    while (team > 1 && team * n_buckets > threads) team >>= 1;
    for (int b0 = 0; b0 < n_buckets; b0 += threads / team) {
        const int b = b0 + tid / team, i0 = tid % team;
        float v = 0.f;
        if (b < n_buckets)
#pragma unroll 8
            for (int i = i0; i < count; i += team) v += value(b, i, team);
        for (int o = team >> 1; o; o >>= 1) v += __shfl_xor(v, o);
        if (b < n_buckets && i0 == 0) result(b, v);
    }
}

// Column h of dtable [n_buckets, H] from partial[h][parts][n_buckets], in the order of the parts.
__device__ __forceinline__ void write_table_column(const float* partial, int n_buckets, int parts, int h, int H, void* __restrict__ dtable, bool is_bf16) {
    sums_by_bucket(n_buckets, parts, [&](int b, int p, int) {
        return __hip_atomic_load(&partial[((size_t)h * parts + p) * n_buckets + b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }, [&](int b, float v) {
        const size_t at = (size_t)b * H + h;
        if (is_bf16) static_cast<bf16_t*>(dtable)[at] = (bf16_t)v;
        else static_cast<float*>(dtable)[at] = v;
    });
}

// Sums of the copies hist [n_buckets][threads] in LDS to partial[h][part][n_buckets].
__device__ __forceinline__ void leave_partial(const float* hist, int n_buckets, int part, int parts, int h, float* partial) {
    __syncthreads();
    const int threads = blockDim.x;
    // (copy i + b team: neighbouring teams start in different banks)
    sums_by_bucket(n_buckets, threads, [&](int b, int i, int team) { return hist[b * threads + ((i + b * team) & (threads - 1))]; },
                   [&](int b, float v) {
                       __hip_atomic_store(&partial[((size_t)h * parts + part) * n_buckets + b], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                   });
}

// Leaves the sums of the copies and, in the last of the head's `parts` workgroups to arrive, writes its column of dtable.  *counter is 0
// before the first of them starts, and all of them count in one addition each (by compare and swap, as where a few pieces of a row
// meet, hundreds of workgroups took 500 to 1500 us).
__device__ __forceinline__ void finish_table_grad(float* hist, int n_buckets, int part, int parts, int h, int H, float* partial,
                                                  unsigned long long* counter, void* __restrict__ dtable, bool is_bf16) {
    leave_partial(hist, n_buckets, part, parts, h, partial);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's stores are done, at device scope
    __syncthreads();                                   // and those of the others, and every wave is done with the copies
    int* const flag = reinterpret_cast<int*>(hist);
    if (threadIdx.x == 0) {
        const unsigned long long before = __hip_atomic_fetch_add(counter, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = before == (unsigned long long)parts - 1ull;
    }
    __syncthreads();
    asm volatile("" ::: "memory");   // nothing of the others' is read before
    if (*flag) write_table_column(partial, n_buckets, parts, h, H, dtable, is_bf16);
}

}  // namespace spion
#endif
