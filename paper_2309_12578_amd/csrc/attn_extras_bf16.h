// Shared by the bf16 attention kernels with a relative position bias, dropout and lengths (block size 32 or 64).
#ifndef SPION_ATTN_EXTRAS_BF16_H_
#define SPION_ATTN_EXTRAS_BF16_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "attn_extras.h"
#include "spion_internal.h"

namespace spion {

namespace {

// Own loads landed (all, or all but the four youngest), previous LDS accesses done, then meet the other waves.
__device__ __forceinline__ void meet(bool four_younger_in_flight) {
    if (four_younger_in_flight) __builtin_amdgcn_s_waitcnt(kWaitVm4);
    else __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void lds_meet() {
    __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The lane's number where addresses are made from it that are used there alone: the compiler makes them there, and does not keep them
// in registers over the loop.
__device__ __forceinline__ int once(int lane) {
    asm volatile("" : "+v"(lane));
    return lane;
}

// Entries of an ascending list whose block starts below `length`, of the n from list on.
template <int BS>
__device__ __forceinline__ int blocks_below(const int* list, int n, int length, int L, int lane) {
    if (length >= L) return n;
    int count = 0;
    for (int base = 0; base < n; base += 64) {
        const int at = base + lane;
        const int here = __popcll(__ballot(at < n && list[at < n ? at : n - 1] * BS < length));
        count += here;
        if (here < 64) break;
    }
    return count;
}

// The biases of a block's distances.  The first BS / 32 waves bring them, a distance a lane: the map's byte is
// requested a step before it is looked up.
template <int BS, bool BIAS>
struct BlockBias {
    const uint8_t* map;
    const float* tab;
    int last, first;   // map entry of the smallest distance in a block on the diagonal
    bool mine;
    __device__ __forceinline__ BlockBias(const Extras& x, const float* tab_, int L, int wave)
        : map(x.bucket_of), tab(tab_), last(x.n_buckets - 1), first(L - BS), mine(BIAS && wave < BS / 32) {}
    // Key block - query block.  (The last lane has no distance.)
    __device__ __forceinline__ unsigned request(int blocks_off, int tid) const {
        return mine ? map[(unsigned)(first + blocks_off * BS + min(once(tid), 2 * BS - 2))] : 0u;
    }
    // Behind the biases, for either half of the distances: the bucket they are all of, or -1, and its bias.
    __device__ __forceinline__ void put(float* slice, unsigned bucket, int tid) const {
        if (mine) {
            tid = once(tid);
            const int b = min((int)bucket, last);
            const float v = tab[b];
            slice[tid] = v;
            const bool alike = __all(b == __builtin_amdgcn_readfirstlane(b));
            const float2 all = make_float2(__builtin_bit_cast(float, alike ? b : -1), v);
            if ((tid & 63) == 0) {
                *reinterpret_cast<float2*>(slice + 2 * BS + (tid >> 6) * 2) = all;
                if (BS == 32) *reinterpret_cast<float2*>(slice + 2 * BS + 2) = all;
            }
        }
    }
};
template <int BS>
constexpr int kSlice = 2 * BS + 4;   // floats

// Whether all distances of a block are of one bucket (it is far off the diagonal, as most are), and its bias: then no lane needs to
// look up its own.
template <int BS>
__device__ __forceinline__ bool one_bucket(const float* slice, float& bias) {
    const float4 all = *reinterpret_cast<const float4*>(slice + 2 * BS);
    const int first = __builtin_amdgcn_readfirstlane(__float_as_int(all.x));
    bias = all.y;
    return first >= 0 && first == __builtin_amdgcn_readfirstlane(__float_as_int(all.z));
}

// The head's column of the bias table in registers (requested before anything else is), then in LDS.
template <int BS, bool BIAS>
struct TableColumn {
    static constexpr int N = Extras::kMaxBuckets / (BS * 4);
    float v[N];
    __device__ __forceinline__ TableColumn(const Extras& x, int h, int tid) {
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int b = tid + i * BS * 4;
                v[i] = 0.f;
                if (b < x.n_buckets) {
                    const size_t at = (size_t)b * x.H + h;
                    v[i] = x.table_bf16 ? (float)static_cast<const bf16_t*>(x.table)[at] : static_cast<const float*>(x.table)[at];
                }
            }
        }
    }
    __device__ __forceinline__ void put(float* tab, const Extras& x, int tid) const {
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i < N; ++i) tab[tid + i * BS * 4] = v[i] <= kMaskedBias ? -INFINITY : v[i] * x.inv_scale;
        }
    }
};

// What the end of a row's piece needs of its cut, in one register: at most RowCut::kSlots each.
struct CutRow {
    int count, slot, piece;
};
static_assert(RowCut::kSlots < 1024, "ten bits each");
__device__ __forceinline__ int pack_cut(const RowPieces& cuts, int piece) { return cuts.count | cuts.slot << 10 | piece << 20; }
__device__ __forceinline__ CutRow unpack_cut(int packed) { return {packed & 1023, packed >> 10 & 1023, packed >> 20}; }

// Bytes of a tile that starts at row `row0` up to the sequence's end.
template <int BS>
__device__ __forceinline__ unsigned tile_range(int row0, int length, int row_len) {
    const int rows = length - row0;
    return rows >= BS ? 0xffffffffu : rows <= 0 ? 0u : (unsigned)rows * (unsigned)row_len * (unsigned)sizeof(bf16_t);
}

}  // namespace

}  // namespace spion
#endif
