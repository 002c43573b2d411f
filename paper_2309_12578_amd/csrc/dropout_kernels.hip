// Dropout and the dense relative position bias: what the sub-layer has besides its attention, elementwise and bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_common.h"
#include "philox.h"
#include "spion_internal.h"
#include "table_grad.h"

namespace spion {

namespace {

template <typename T>
struct Eight {
    T v[8];
};

template <typename T, bool WHOLE>
__device__ __forceinline__ void load8(float (&v)[8], const T* p, int n) {
    if constexpr (WHOLE) {
        Eight<T> e;
        constexpr int words = sizeof(e) / 16;
#pragma unroll
        for (int i = 0; i < words; ++i) reinterpret_cast<uint4*>(&e)[i] = reinterpret_cast<const uint4*>(p)[i];
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
        for (int i = 0; i < words; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(&e)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

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

template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void dropout_kernel(const T* __restrict__ x, const T* __restrict__ residual, T* __restrict__ y,
                                                      long long n, const long long* __restrict__ rng, long long* __restrict__ rng_used,
                                                      unsigned stream, unsigned threshold, float keep_scale) {
    if (blockIdx.x == 0 && threadIdx.x < 2 && rng_used) rng_used[threadIdx.x] = rng[threadIdx.x];
    const PhiloxKey key(rng, stream);
    const long long whole = ALIGNED ? n / 8 : 0, calls = (n + 7) / 8, step = (long long)gridDim.x * 256;
    long long c = (long long)blockIdx.x * 256 + threadIdx.x;
    for (; c < whole; c += step) dropout8<T, true>(key, x, residual, y, c, 8, threshold, keep_scale);
    for (; c < calls; c += step) dropout8<T, false>(key, x, residual, y, c, (int)min(8ll, n - 8 * c), threshold, keep_scale);
}

hipError_t launch_dropout(const void* x, const void* residual, void* y, long long n, const long long* rng, long long* rng_used, unsigned stream,
                          unsigned threshold, float keep_scale, bool is_bf16, hipStream_t st) {
    const long long groups = ((n + 7) / 8 + 255) / 256;
    const unsigned grid = (unsigned)std::min<long long>(groups, 256 * 32);
    const bool aligned = ((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) % 16 == 0;
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3(grid), dim3(256), 0, st>>>(static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(y), n, rng, rng_used,
                                                 stream, threshold, keep_scale);
    };
    if (is_bf16) {
        if (aligned) launch(dropout_kernel<bf16_t, true>, bf16_t{});
        else launch(dropout_kernel<bf16_t, false>, bf16_t{});
    } else {
        if (aligned) launch(dropout_kernel<float, true>, float{});
        else launch(dropout_kernel<float, false>, float{});
    }
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// bias[h][i][j] = table[bucket_of[j - i - q_start + reach - 1]][h]
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void relative_bias_kernel(const T* __restrict__ table, const uint8_t* __restrict__ bucket_of, T* __restrict__ bias,
                                                            int reach, int n_buckets, int H, int q_len, int k_len, int q_start, int rows) {
    const int h = blockIdx.z, j = blockIdx.x * 256 + threadIdx.x, i0 = blockIdx.y * rows;
    if (j >= k_len) return;
    for (int i = i0; i < min(i0 + rows, q_len); ++i) {
        const unsigned b = bucket_of[j - i - q_start + reach - 1];
        bias[((size_t)h * q_len + i) * k_len + j] = table[(size_t)min(b, (unsigned)n_buckets - 1u) * H + h];
    }
}

hipError_t launch_relative_bias(const void* table, const uint8_t* bucket_of, void* bias, int reach, int n_buckets, int H, int q_len, int k_len,
                                int q_start, bool is_bf16, hipStream_t st) {
    const int rows = 16;
    const dim3 grid((k_len + 255) / 256, (q_len + rows - 1) / rows, H);
    if (is_bf16)
        relative_bias_kernel<bf16_t><<<grid, dim3(256), 0, st>>>(static_cast<const bf16_t*>(table), bucket_of, static_cast<bf16_t*>(bias), reach,
                                                                n_buckets, H, q_len, k_len, q_start, rows);
    else
        relative_bias_kernel<float><<<grid, dim3(256), 0, st>>>(static_cast<const float*>(table), bucket_of, static_cast<float*>(bias), reach,
                                                               n_buckets, H, q_len, k_len, q_start, rows);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// dtable[b][h] = sum of dbias[h][i][j] over bucket_of[j - i - q_start + reach - 1] == b.  A thread walks down its diagonals
// (neighbours in a wave read neighbours in memory), then adds each sum into its own copy of the buckets.
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void relative_bias_grad_kernel(const T* __restrict__ dbias, const uint8_t* __restrict__ bucket_of,
                                                                 int reach, int n_buckets, int H, int q_len, int k_len, int q_start, int parts, int band, float* partial) {
    extern __shared__ float hist[];   // [n_buckets][threads]
    const int h = blockIdx.x % H, part = blockIdx.x / H, tid = threadIdx.x, threads = blockDim.x;
    for (int b = 0; b < n_buckets; ++b) hist[b * threads + tid] = 0.f;
    const T* const g = dbias + (size_t)h * q_len * k_len;
    const int diagonals = q_len + k_len - 1, tiles_d = (diagonals + threads - 1) / threads, bands = (q_len + band - 1) / band;
    for (long long tile = part; tile < (long long)tiles_d * bands; tile += parts) {
        const int t = (int)(tile % tiles_d) * threads + tid, i0 = (int)(tile / tiles_d) * band;
        if (t >= diagonals) continue;
        const int d = t - (q_len - 1);   // j - i
        const int from = max(i0, -d), to = min(min(i0 + band, q_len), k_len - d);
        if (from >= to) continue;
        float sum = 0.f;
        const T* p = g + (size_t)from * k_len + from + d;
        for (int i = from; i < to; ++i, p += k_len + 1) sum += (float)*p;
        const unsigned b = bucket_of[d - q_start + reach - 1];
        hist[min(b, (unsigned)n_buckets - 1u) * threads + tid] += sum;
    }
    leave_partial(hist, n_buckets, part, parts, h, partial);
}

__global__ __launch_bounds__(256) void relative_bias_sum_kernel(const float* partial, void* __restrict__ dtable, int n_buckets, int H, int parts, int is_bf16) {
    write_table_column(partial, n_buckets, parts, blockIdx.x, H, dtable, is_bf16 != 0);
}

namespace {
struct BiasGradPlan {
    int band = 256, parts;
    size_t total;
    BiasGradPlan(int H, int q_len, int k_len, int n_buckets) {
        const long long tiles = (long long)((q_len + k_len) / table_grad_threads(n_buckets) + 1) * ((q_len + band - 1) / band);
        parts = (int)std::min<long long>(tiles, std::max(1, 2048 / H));
        total = ((size_t)H * parts * n_buckets * sizeof(float) + 255) / 256 * 256;
    }
};
}  // namespace

size_t relative_bias_grad_workspace_bytes(int H, int q_len, int k_len, int n_buckets) { return BiasGradPlan(H, q_len, k_len, n_buckets).total; }

hipError_t launch_relative_bias_grad(const void* dbias, const uint8_t* bucket_of, void* dtable, int reach, int n_buckets, int H, int q_len, int k_len,
                                     int q_start, bool is_bf16, void* workspace, hipStream_t st) {
    const BiasGradPlan plan(H, q_len, k_len, n_buckets);
    const int threads = table_grad_threads(n_buckets);
    float* const partial = static_cast<float*>(workspace);
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)(H * plan.parts)), dim3(threads), (size_t)n_buckets * threads * sizeof(float), st>>>(
            static_cast<const T*>(dbias), bucket_of, reach, n_buckets, H, q_len, k_len, q_start, plan.parts, plan.band, partial);
    };
    if (is_bf16) launch(relative_bias_grad_kernel<bf16_t>, bf16_t{});
    else launch(relative_bias_grad_kernel<float>, float{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    relative_bias_sum_kernel<<<dim3((unsigned)H), dim3(256), 0, st>>>(partial, dtable, n_buckets, H, plan.parts, is_bf16);
    return hipGetLastError();
}

}  // namespace spion
