// Dropout and the dense relative position bias: what the sub-layer has besides its attention, elementwise and bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_common.h"
#include "chunks.h"
#include "philox.h"
#include "spion_internal.h"
#include "table_grad.h"

namespace spion {

namespace {

// Elements 8 c .. 8 c + 7: the eight halves of the call with counter c.
template <typename T, bool WHOLE>
__device__ __forceinline__ void dropout8(const PhiloxKey& key, const T* x, const T* residual, T* y, long long c, int n, unsigned threshold,
                                         float keep_scale) {
    float v[8], res[8];
    load8<T, WHOLE>(v, x + 8 * c, n);
    if (residual) load8<T, WHOLE>(res, residual + 8 * c, n);
    const uint4 w = key.words((unsigned)c, (unsigned)(c >> 32));
    const unsigned words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned draw = i & 1 ? words[i / 2] >> 16 : words[i / 2] & 0xffffu;
        const float d = draw < threshold ? 0.f : v[i];
        v[i] = residual ? fmaf(d, keep_scale, res[i]) : d * keep_scale;
    }
    store8<T, WHOLE>(y + 8 * c, v, n);
}

}  // namespace

// Bound by memory: a call of the generator for 16 bytes of bf16, 32 of fp32.  2^27 bf16 elements with a residual 154 us, 5.2 TB/s; without one
// (the gradient) 96 us, 5.6 TB/s; from odd addresses the same.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* __restrict__ x, const T* __restrict__ residual, T* __restrict__ y,
                                                      long long n, const long long* __restrict__ rng, long long* __restrict__ rng_used,
                                                      unsigned stream, unsigned threshold, float keep_scale) {
    if (blockIdx.x == 0 && threadIdx.x < 2 && rng_used) rng_used[threadIdx.x] = rng[threadIdx.x];
    const PhiloxKey key(rng, stream);
    const long long whole = n / 8, calls = (n + 7) / 8, step = (long long)gridDim.x * 256;
    long long c = (long long)blockIdx.x * 256 + threadIdx.x;
    for (; c < whole; c += step) dropout8<T, true>(key, x, residual, y, c, 8, threshold, keep_scale);
    for (; c < calls; c += step) dropout8<T, false>(key, x, residual, y, c, (int)min(8ll, n - 8 * c), threshold, keep_scale);
}

hipError_t launch_dropout(const void* x, const void* residual, void* y, long long n, const long long* rng, long long* rng_used, unsigned stream,
                          unsigned threshold, float keep_scale, bool is_bf16, hipStream_t st) {
    const long long groups = ((n + 7) / 8 + 255) / 256;
    const unsigned grid = (unsigned)std::min<long long>(groups, 256 * 32);
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3(grid), dim3(256), 0, st>>>(static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(y), n, rng, rng_used,
                                                 stream, threshold, keep_scale);
    };
    if (is_bf16) launch(dropout_kernel<bf16_t>, bf16_t{});
    else launch(dropout_kernel<float>, float{});
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// bias[h][i][j] = table[bucket_of[j - i - q_start + reach - 1]][h]: bound by its stores.  A row is a window of one vector of values
// by distance, which each row has one place further on.  A workgroup has `rows` rows of up to 256 chunks of 16 bytes; it brings the values of
// its distances into LDS once, as many copies of them as a chunk has elements, each one element further on than the last, so that whatever
// the place of a chunk is, one of the copies has it aligned: a 16-byte read and a 16-byte store a chunk.  Chunks are aligned in memory
// whatever k_len is; those at a row's ends are stored by elements.  8 heads x 4096 x 4096, bf16: 45 us, 6.0 TB/s (element by element 86).
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void relative_bias_kernel(const T* __restrict__ table, const uint8_t* __restrict__ bucket_of, T* __restrict__ bias,
                                                            int reach, int n_buckets, int H, int q_len, int k_len, int q_start, int rows, int wide,
                                                            int col_tiles, int row_tiles, int copy_len) {
    constexpr int VEC = 16 / sizeof(T);
    extern __shared__ __attribute__((aligned(16))) char bias_lds[];
    T* const copies = reinterpret_cast<T*>(bias_lds);   // [VEC][copy_len]
    const int tid = threadIdx.x;
    const unsigned col_tile = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles;
    const int i0 = (int)(rest % row_tiles) * rows, h = rest / row_tiles, c0 = (int)col_tile * wide;
    // place p of the values is distance first + p; a copy s has place p at p - s
    const int first = c0 * VEC - (VEC - 1) - (i0 + rows - 1) - q_start;
    for (int p = tid; p < copy_len + VEC - 1; p += 256) {
        const int at = max(0, min(first + p + reach - 1, 2 * reach - 2));   // (distances outside belong to no element)
        const T v = table[(size_t)min((int)bucket_of[at], n_buckets - 1) * H + h];
#pragma unroll
        for (int s = 0; s < VEC; ++s)
            if (p >= s && p - s < copy_len) copies[s * copy_len + p - s] = v;
    }
    __syncthreads();
    int x = tid % wide, i = i0 + tid / wide;
    const int step_x = 256 % wide, step_i = 256 / wide;
    auto next = [&] {
        x += step_x;
        i += step_i;
        if (x >= wide) {
            x -= wide;
            ++i;
        }
    };
    for (; i < min(i0 + rows, q_len); next()) {
        const size_t start = ((size_t)h * q_len + i) * k_len;
        const int off = (int)(((size_t)bias / sizeof(T) + start) % VEC), j = (c0 + x) * VEC - off;
        if (j >= k_len) continue;
        const int p = x * VEC - off + (VEC - 1) + (i0 + rows - 1 - i), s = p % VEC;
        const uint4 v = *reinterpret_cast<const uint4*>(copies + s * copy_len + (p - s));
        T* const out = bias + start + j;
        if (j >= 0 && j + VEC <= k_len) {
            *reinterpret_cast<uint4*>(out) = v;
        } else {
            const T* const e = copies + s * copy_len + (p - s);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (j + k >= 0 && j + k < k_len) out[k] = e[k];
        }
    }
}

hipError_t launch_relative_bias(const void* table, const uint8_t* bucket_of, void* bias, int reach, int n_buckets, int H, int q_len, int k_len,
                                int q_start, bool is_bf16, hipStream_t st) {
    const int vec = is_bf16 ? 8 : 4;
    const bool aligned = k_len % vec == 0 && (uintptr_t)bias % 16 == 0;   // otherwise a row's chunks may begin before it
    const int chunks = aligned ? k_len / vec : (k_len + 2 * vec - 2) / vec;
    // Up to 256 chunks of a row each.  A few rows are cut into more pieces, whose values are there after one load of each thread:
    // one row of 4097, 8 heads, 5.9 -> 3.1 us.
    int col_tiles = (chunks + 255) / 256;
    const int most = (chunks + 31) / 32;
    if ((long long)H * q_len * col_tiles < 512) col_tiles = (int)std::min<long long>(most, 512 / ((long long)H * q_len) + 1);
    const int wide = (chunks + col_tiles - 1) / col_tiles, at_once = 256 / wide;
    // About four workgroups a compute unit, up to 128 rows each: bringing the values takes as long as some 70 chunks a thread.
    const long long all = (long long)H * q_len * col_tiles;
    int rows = (int)std::min<long long>(128, std::max<long long>(all / 1024, 1));
    rows = std::max(rows, std::min(at_once, q_len));
    const int row_tiles = (q_len + rows - 1) / rows;
    const int copy_len = (wide * vec + rows + vec + vec - 1) / vec * vec;
    const long long grid = (long long)H * row_tiles * col_tiles;
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)grid), dim3(256), (size_t)vec * copy_len * sizeof(T), st>>>(
            static_cast<const T*>(table), bucket_of, static_cast<T*>(bias), reach, n_buckets, H, q_len, k_len, q_start, rows, wide, col_tiles,
            row_tiles, copy_len);
    };
    if (is_bf16) launch(relative_bias_kernel<bf16_t>, bf16_t{});
    else launch(relative_bias_kernel<float>, float{});
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// dtable[b][h] = sum of dbias[h][i][j] over bucket_of[j - i - q_start + reach - 1] == b: bound by its loads.  First the sums over diagonals within
// bands of rows: a thread walks down the 16 bytes' worth of diagonals beside each other, whose elements a row has together (at any
// address: the loads need not be aligned).  Then those sums by bucket.  8 heads x 4096 x 4096, bf16: 57 us, 4.7 TB/s, and 9 us (element by
// element 328); right behind as many bytes of stores, which still drain, 92 and 9.
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void diagonal_sums_kernel(const T* __restrict__ dbias, float* __restrict__ sums, int q_len, int k_len, int H, int band,
                                                            int bands, int chunks, int groups, unsigned long long* __restrict__ counters) {
    constexpr int VEC = 16 / sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) Chunk { unsigned w[4]; };
    if (blockIdx.x == 0)
        for (int k = threadIdx.x; k < H; k += 256) counters[k * Extras::kCounterStride] = 0ull;
    const int h = blockIdx.x / groups;
    const unsigned thread = (blockIdx.x % groups) * 256u + threadIdx.x;   // of the head's bands * chunks
    if (thread >= (unsigned)bands * chunks) return;
    const int t = (int)(thread % chunks) * VEC, i0 = (int)(thread / chunks) * band, end = min(i0 + band, q_len);
    const int d = t - (i0 + band - 1);   // j - i of the first
    const T* const g = dbias + (size_t)h * q_len * k_len;
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    // rows that have some of the diagonals, and those in the middle that have them all
    const int some = min(max(i0, -(d + VEC - 1)), end), some_end = max(min(end, k_len - d), some);
    const int from = min(max(-d, some), some_end), to = max(min(end, k_len - (d + VEC - 1)), from);
    constexpr int kInFlight = 8;
    const size_t step = (size_t)k_len + 1;
    auto add_masked = [&](int a, int b) {   // chunks that reach over a row's ends, or over the tensor's
        const long long at_h = (long long)h * q_len * k_len, total = (long long)H * q_len * k_len;
        for (int r = a; r < b; r += kInFlight) {
            Chunk c[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const int i = min(r + u, b - 1);
                const long long at = at_h + (long long)i * k_len + (i + d);
                if (at >= 0 && at + VEC <= total) {
                    c[u] = *reinterpret_cast<const Chunk*>(dbias + at);
                } else {
                    T* const v = reinterpret_cast<T*>(&c[u]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[e] = at + e >= 0 && at + e < total ? dbias[at + e] : (T)0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const T* const v = reinterpret_cast<const T*>(&c[u]);
                const int j = r + u + d;
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += r + u < b && j + e >= 0 && j + e < k_len ? (float)v[e] : 0.f;
            }
        }
    };
    add_masked(some, from);
    add_masked(to, some_end);
    const T* p = g + (size_t)from * k_len + (from + d);
    auto add = [&](const Chunk& c) {
        const T* const v = reinterpret_cast<const T*>(&c);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += (float)v[e];
    };
    int i = from;
    for (; i + kInFlight <= to; i += kInFlight, p += kInFlight * step) {
        Chunk c[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) c[u] = *reinterpret_cast<const Chunk*>(p + u * step);
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) add(c[u]);
    }
    for (; i < to; ++i, p += step) add(*reinterpret_cast<const Chunk*>(p));
    // (of the last chunk, diagonals past the band's have no element: 0)
    float4* const out = reinterpret_cast<float4*>(sums + (((size_t)h * bands + (unsigned)(i0 / band)) * chunks * VEC + t));
#pragma unroll
    for (int e = 0; e < VEC; e += 4) out[e / 4] = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
}

// sums [H][bands][fours][4]; the first diagonal of the first band has bucket_of[first], that of each further band `band` before it
__global__ __launch_bounds__(256) void buckets_of_sums_kernel(const float* __restrict__ sums, const uint8_t* __restrict__ bucket_of, int n_distances, int first,
                                                              int band, unsigned n, unsigned fours, int n_buckets, int H, int parts, float* partial,
                                                              unsigned long long* __restrict__ counters, void* __restrict__ dtable, int is_bf16) {
    extern __shared__ float hist[];   // [n_buckets][threads]
    const int h = blockIdx.x % H, part = blockIdx.x / H, tid = threadIdx.x, threads = blockDim.x;
    for (int b = 0; b < n_buckets; ++b) hist[b * threads + tid] = 0.f;
    const unsigned begin = (unsigned)((unsigned long long)part * n / parts), end = (unsigned)((unsigned long long)(part + 1) * n / parts);
    const float4* const mine = reinterpret_cast<const float4*>(sums) + (size_t)h * n;
    constexpr int kInFlight = 2;
    for (unsigned k0 = begin + tid; k0 < end; k0 += kInFlight * threads) {
        float4 v[kInFlight];
        unsigned buckets[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const unsigned k = min(k0 + u * threads, end - 1);
            v[u] = mine[k];
            const int at = first + (int)(k % fours) * 4 - (int)(k / fours) * band;
            if (at >= 0 && at + 4 <= n_distances) {
                buckets[u] = reinterpret_cast<const FourBuckets*>(bucket_of + at)->u;
            } else {   // (some of them are past the last row's or column's, and 0)
                buckets[u] = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) buckets[u] |= (unsigned)bucket_of[max(0, min(at + i, n_distances - 1))] << (8 * i);
            }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const float four[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
            if (k0 + u * threads < end) add_four(hist + tid, threads, four, buckets[u], n_buckets);
        }
    }
    finish_table_grad(hist, n_buckets, part, parts, h, H, partial, counters + h * Extras::kCounterStride, dtable, is_bf16 != 0);
}

namespace {
struct BiasGradPlan {
    int band, bands, chunks, groups, parts;   // rows of a band; 16 bytes' worth of its diagonals; workgroups of a head, first and second kernel
    long long sums;                           // of a head
    size_t partial, counters, total;          // behind the sums
    BiasGradPlan(int H, int q_len, int k_len, int n_buckets, bool is_bf16) {
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        const int vec = is_bf16 ? 8 : 4;
        // four waves a SIMD, of 16 to 256 rows
        const long long rows = (long long)H * q_len * ((k_len + vec - 1) / vec) / 262144;
        band = (int)std::min<long long>(256, std::max<long long>(16, rows));
        bands = (q_len + band - 1) / band;
        chunks = (k_len + band - 1 + vec - 1) / vec;
        sums = (long long)bands * chunks * vec;
        groups = (int)(((long long)bands * chunks + 255) / 256);
        parts = (int)std::max<long long>(1, std::min<long long>(sums / (table_grad_threads(n_buckets) * 8), 1024 / H));
        partial = up((size_t)H * sums * sizeof(float));
        counters = up(partial + (size_t)H * parts * n_buckets * sizeof(float));
        total = up(counters + (size_t)H * Extras::kCounterStride * 8);
    }
};
}  // namespace

size_t relative_bias_grad_workspace_bytes(int H, int q_len, int k_len, int n_buckets) {
    const BiasGradPlan a(H, q_len, k_len, n_buckets, true), b(H, q_len, k_len, n_buckets, false);
    return std::max(a.total, b.total);
}

hipError_t launch_relative_bias_grad(const void* dbias, const uint8_t* bucket_of, void* dtable, int reach, int n_buckets, int H, int q_len, int k_len,
                                     int q_start, bool is_bf16, void* workspace, hipStream_t st) {
    const BiasGradPlan plan(H, q_len, k_len, n_buckets, is_bf16);
    const long long grid = (long long)H * plan.groups;
    if (grid > 0x7fffffffll || plan.sums > 0x3fffffffll) return hipErrorInvalidValue;
    float* const sums = static_cast<float*>(workspace);
    auto* const counters = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + plan.counters);
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)grid), dim3(256), 0, st>>>(static_cast<const T*>(dbias), sums, q_len, k_len, H, plan.band, plan.bands, plan.chunks,
                                                           plan.groups, counters);
    };
    if (is_bf16) launch(diagonal_sums_kernel<bf16_t>, bf16_t{});
    else launch(diagonal_sums_kernel<float>, float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int threads = table_grad_threads(n_buckets);
    buckets_of_sums_kernel<<<dim3((unsigned)(H * plan.parts)), dim3(threads), (size_t)n_buckets * threads * sizeof(float), st>>>(
        sums, bucket_of, 2 * reach - 1, reach - 1 - q_start - (plan.band - 1), plan.band, (unsigned)(plan.sums / 4),
        (unsigned)(plan.chunks * (is_bf16 ? 2 : 1)), n_buckets, H, plan.parts,
        reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.partial), counters, dtable, is_bf16);
    return hipGetLastError();
}

}  // namespace spion
