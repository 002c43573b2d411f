// Root-mean-square norm with the residual's addition, its gradient, and rows in 8 bits (eight_bit.h).
//
//   s = x + residual, rstd = 1 / sqrt(mean s^2 + eps), z = s rstd, y = z w
//   dx = ds + rstd (w dy - z mean(w dy z)), dw = sum over rows of dy z
//
// Bound by HBM.  LANES lanes have a row, 8 consecutive elements each, every 8 LANES, in registers: one pass over the data.  The sum of squares is in
// 64 bits, and so is all that decides a code: with a row's sum in another order, or in 32 bits, one in 10^5 codes would be its neighbour.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "attn_common.h"
#include "chunks.h"
#include "eight_bit.h"
#include "spion_internal.h"

namespace spion {

namespace {

constexpr int kNormGroups = 1024;   // workgroups of the backward, at most: partial rows that the second launch adds

template <int LANES>
struct RowThreads {
    static constexpr int threads = LANES > 256 ? LANES : 256, rows = threads / LANES;
};

// Sum over the LANES lanes of a row; every lane of the workgroup takes part.
template <int LANES, typename S>
__device__ __forceinline__ S row_sum(S v, S* shared) {
#pragma unroll
    for (int off = 1; off < LANES && off < 64; off <<= 1) v += __shfl_xor(v, off);
    if constexpr (LANES > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();   // what was there has been read
        if ((threadIdx.x & 63) == 0) shared[wave] = v;
        __syncthreads();
        v = shared[0];
#pragma unroll
        for (int k = 1; k < LANES / 64; ++k) v += shared[k];
    }
    return v;
}

template <typename T>
__device__ __forceinline__ void load_chunk(float (&v)[8], const T* row, int c, int D) {
    if (c + 8 <= D) load8<T, true>(v, row + c, 8);
    else load8<T, false>(v, row + c, D - c);
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int c, int D, const float (&v)[8]) {
    if (c + 8 <= D) store8<T, true>(row + c, v, 8);
    else store8<T, false>(row + c, v, D - c);
}

// Which codes are written: none, of z (what the backward passes take) or of y.
enum { kNoCodes = 0, kCodesOfZ = 1, kCodesOfY = 2 };

template <typename T, int LANES, int K, int CODES>
__global__ __launch_bounds__(RowThreads<LANES>::threads) void rms_norm_kernel(const T* __restrict__ x, const T* __restrict__ residual,
                                                                              const T* __restrict__ w, T* __restrict__ y, T* __restrict__ h,
                                                                              float* __restrict__ rstd, signed char* __restrict__ codes,
                                                                              uint8_t* __restrict__ exponents, long long rows, int D, double eps) {
    typedef std::conditional_t<(CODES != kNoCodes && sizeof(T) == 4), double, float> S;   // (a sum of two bf16 numbers is exact in fp32, or off by 2^-24)
    __shared__ double shared[LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int pitch = (int)eight_pitch(D);
    float wv[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) load_chunk(wv[k], w, min(8 * (lane + k * LANES), D), D);
    for (long long first = (long long)blockIdx.x * RowThreads<LANES>::rows; first < rows; first += (long long)gridDim.x * RowThreads<LANES>::rows) {
        const bool has = first + slot < rows;
        const long long row = has ? first + slot : rows - 1;
        S s[K][8];
        double squares = 0.0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = min(8 * (lane + k * LANES), D);
            float a[8], r[8];
            load_chunk(a, x + row * D, c, D);
            if (residual) load_chunk(r, residual + row * D, c, D);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[k][i] = residual ? (S)a[i] + (S)r[i] : (S)a[i];
                squares += (double)s[k][i] * (double)s[k][i];
            }
        }
        const double inverse = 1.0 / sqrt(row_sum<LANES>(squares, shared) / D + eps);
        if (lane == 0 && has && rstd) rstd[row] = (float)inverse;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES);
            float v[8];
            if (h) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)s[k][i];
                if (has && c < D) store_chunk(h + row * D, c, D, v);
            }
            if constexpr (CODES == kNoCodes) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = s[k][i] * (float)inverse * wv[k][i];
            } else {
                double z[8], most = 0.0;
                bool finite = true;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[i] = (double)s[k][i] * inverse;
                    v[i] = (float)z[i] * wv[k][i];
                    if constexpr (CODES == kCodesOfY) z[i] *= (double)wv[k][i];
                    most = fmax(most, fabs(z[i]));
                    finite = finite && z[i] == z[i];
                }
                const int exponent = group_exponent(finite ? exponent_byte(most) : kNotFinite);
                if (has && c < pitch) {
                    *reinterpret_cast<Codes8*>(codes + row * pitch + c) = codes_of(z, exponent);
                    if (c % kGroup == 0) exponents[row * (pitch / kGroup) + c / kGroup] = (uint8_t)exponent;
                }
            }
            if (y && has && c < D) store_chunk(y + row * D, c, D, v);
        }
    }
}

// z from codes, or from s = h in the row's type.
template <typename T, int LANES, int K, bool CODES>
__global__ __launch_bounds__(RowThreads<LANES>::threads) void rms_norm_grad_kernel(const T* __restrict__ dy, const T* __restrict__ dh,
                                                                                   const T* __restrict__ h, const signed char* __restrict__ codes,
                                                                                   const uint8_t* __restrict__ exponents, const T* __restrict__ w,
                                                                                   const float* __restrict__ rstd, T* __restrict__ dx,
                                                                                   float* __restrict__ partial, long long rows, int D) {
    constexpr int ROWS = RowThreads<LANES>::rows;
    __shared__ float shared[LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int pitch = (int)eight_pitch(D);
    float wv[K][8], dw[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_chunk(wv[k], w, min(8 * (lane + k * LANES), D), D);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    }
    for (long long first = (long long)blockIdx.x * ROWS; first < rows; first += (long long)gridDim.x * ROWS) {
        const bool has = first + slot < rows;
        const long long row = has ? first + slot : rows - 1;
        const float rs = rstd[row];
        float z[K][8], g[K][8], sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES);
            load_chunk(g[k], dy + row * D, min(c, D), D);
            if constexpr (CODES) {
                Codes8 q = {0u, 0u};
                int exponent = 1;
                if (c < pitch) {
                    q = *reinterpret_cast<const Codes8*>(codes + row * pitch + c);
                    exponent = exponents[row * (pitch / kGroup) + c / kGroup];
                }
                values_of(z[k], q, eight_scale(exponent));
            } else {
                load_chunk(z[k], h + row * D, min(c, D), D);
#pragma unroll
                for (int i = 0; i < 8; ++i) z[k][i] *= rs;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c + i >= D) z[k][i] = 0.f;   // (a last group that is not finite)
                if (has) dw[k][i] += g[k][i] * z[k][i];
                g[k][i] *= wv[k][i];
                sum += g[k][i] * z[k][i];
            }
        }
        const float mean = row_sum<LANES>(sum, shared) / (float)D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES);
            if (!has || c >= D) continue;
            float r[8];
            if (dh) load_chunk(r, dh + row * D, c, D);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[k][i] = rs * (g[k][i] - z[k][i] * mean);
                if (dh) g[k][i] += r[i];
            }
            store_chunk(dx + row * D, c, D, g[k]);
        }
    }
    if (!partial) return;
    // the workgroup's rows of dw, added in their order
    if constexpr (ROWS > 1) {
        __shared__ float parts[ROWS][LANES * K * 8];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) parts[slot][8 * (lane + k * LANES) + i] = dw[k][i];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += RowThreads<LANES>::threads) {
            float v = parts[0][c];
#pragma unroll
            for (int r = 1; r < ROWS; ++r) v += parts[r][c];
            partial[(size_t)blockIdx.x * D + c] = v;
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (8 * (lane + k * LANES) < D) store_chunk(partial + (size_t)blockIdx.x * D, 8 * (lane + k * LANES), D, dw[k]);
    }
}

// 64 columns a workgroup, a wave every 16th partial row.
template <typename T>
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ partial, int groups, int D, T* __restrict__ out) {
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (col < D) {
#pragma unroll 8
        for (int g = wave; g < groups; g += 16) s += partial[(size_t)g * D + col];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= D) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += part[k][lane];
    out[col] = (T)s;
}

// A thread has 8 elements of the padded row.
template <typename T>
__global__ __launch_bounds__(256) void pack_eight_kernel(const T* __restrict__ x, signed char* __restrict__ codes, uint8_t* __restrict__ exponents,
                                                         long long rows, int D) {
    const int chunks = (int)eight_pitch(D) / 8;
    const long long n = rows * chunks, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {   // (n and step are multiples of 8: a group's lanes leave together)
        const long long row = i / chunks;
        const int c = (int)(i - row * chunks) * 8;
        float v[8], most = 0.f;
        load_chunk(v, x + row * D, min(c, D), D);
        bool finite = true;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            most = fmaxf(most, fabsf(v[k]));
            finite = finite && v[k] == v[k];
        }
        const int exponent = group_exponent(finite ? exponent_byte(most) : kNotFinite);
        *reinterpret_cast<Codes8*>(codes + 8 * i) = codes_of(v, exponent);
        if (i % 8 == 0) exponents[i / 8] = (uint8_t)exponent;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_eight_kernel(const signed char* __restrict__ codes, const uint8_t* __restrict__ exponents,
                                                           const void* __restrict__ weight, int weight_bf16, T* __restrict__ y, long long rows, int D) {
    const int chunks = (D + 7) / 8, pitch = (int)eight_pitch(D);
    const long long n = rows * chunks, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const long long row = i / chunks;
        const int c = (int)(i - row * chunks) * 8;
        float v[8];
        values_of(v, *reinterpret_cast<const Codes8*>(codes + row * pitch + c), eight_scale(exponents[row * (pitch / kGroup) + c / kGroup]));
        if (weight) {
            float wv[8];
            if (weight_bf16) load_chunk(wv, static_cast<const bf16_t*>(weight), c, D);
            else load_chunk(wv, static_cast<const float*>(weight), c, D);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= wv[k];
        }
        store_chunk(y + row * D, c, D, v);
    }
}

// Lanes that have a row of D elements, and chunks a lane.
template <class F>
hipError_t by_width(int D, F&& f) {
    if (D <= 64) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (D <= 128) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (D <= 256) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (D <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (D <= 1024) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (D <= 2048) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (D <= 4096) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (D <= 8192) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
    return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
int rows_at_once(int D) { return D <= 64 ? 32 : D <= 128 ? 16 : D <= 256 ? 8 : D <= 1024 ? 4 : 1; }
int grad_groups(long long rows, int D) {
    const long long at_once = rows_at_once(D), groups = (rows + at_once - 1) / at_once;
    return (int)std::min<long long>(groups, kNormGroups);
}

template <typename T>
hipError_t forward_t(const RmsNorm& a, hipStream_t st) {
    return by_width(a.D, [&](auto lanes, auto k) {
        constexpr int LANES = decltype(lanes)::value, K = decltype(k)::value;
        const long long at_once = RowThreads<LANES>::rows;
        const unsigned grid = (unsigned)std::min<long long>((a.rows + at_once - 1) / at_once, 16384);
        auto launch = [&](auto kernel) {
            kernel<<<dim3(grid), dim3(RowThreads<LANES>::threads), 0, st>>>(
                static_cast<const T*>(a.x), static_cast<const T*>(a.residual), static_cast<const T*>(a.w), static_cast<T*>(a.y), static_cast<T*>(a.h), a.rstd,
                a.codes, a.exponents, a.rows, a.D, a.eps);
        };
        if (!a.codes) launch(rms_norm_kernel<T, LANES, K, kNoCodes>);
        else if (a.codes_of_y) launch(rms_norm_kernel<T, LANES, K, kCodesOfY>);
        else launch(rms_norm_kernel<T, LANES, K, kCodesOfZ>);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward_t(const RmsNormGrad& a, hipStream_t st) {
    const int groups = grad_groups(a.rows, a.D);
    const hipError_t e = by_width(a.D, [&](auto lanes, auto k) {
        constexpr int LANES = decltype(lanes)::value, K = decltype(k)::value;
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)groups), dim3(RowThreads<LANES>::threads), 0, st>>>(
                static_cast<const T*>(a.dy), static_cast<const T*>(a.dh), static_cast<const T*>(a.h), a.codes, a.exponents, static_cast<const T*>(a.w), a.rstd,
                static_cast<T*>(a.dx), a.dw ? a.partial : nullptr, a.rows, a.D);
        };
        if (a.codes) launch(rms_norm_grad_kernel<T, LANES, K, true>);
        else launch(rms_norm_grad_kernel<T, LANES, K, false>);
        return hipGetLastError();
    });
    if (e != hipSuccess || !a.dw) return e;
    column_sum_kernel<T><<<dim3((unsigned)((a.D + 63) / 64)), dim3(1024), 0, st>>>(a.partial, groups, a.D, static_cast<T*>(a.dw));
    return hipGetLastError();
}

unsigned chunk_grid(long long chunks) { return (unsigned)std::min<long long>((chunks + 255) / 256, 256 * 32); }

}  // namespace

size_t rms_norm_workspace_bytes(long long rows, int D) { return (size_t)grad_groups(rows, D) * D * sizeof(float); }

hipError_t launch_rms_norm(const RmsNorm& a, bool is_bf16, hipStream_t st) { return is_bf16 ? forward_t<bf16_t>(a, st) : forward_t<float>(a, st); }
hipError_t launch_rms_norm_grad(const RmsNormGrad& a, bool is_bf16, hipStream_t st) { return is_bf16 ? backward_t<bf16_t>(a, st) : backward_t<float>(a, st); }

hipError_t launch_pack_eight(const void* x, signed char* codes, uint8_t* exponents, long long rows, int D, bool is_bf16, hipStream_t st) {
    const dim3 grid(chunk_grid(rows * (eight_pitch(D) / 8)));
    if (is_bf16) pack_eight_kernel<<<grid, dim3(256), 0, st>>>(static_cast<const bf16_t*>(x), codes, exponents, rows, D);
    else pack_eight_kernel<<<grid, dim3(256), 0, st>>>(static_cast<const float*>(x), codes, exponents, rows, D);
    return hipGetLastError();
}
hipError_t launch_unpack_eight(const signed char* codes, const uint8_t* exponents, const void* weight, bool weight_bf16, void* y, long long rows, int D,
                               bool is_bf16, hipStream_t st) {
    const dim3 grid(chunk_grid(rows * ((D + 7) / 8)));
    if (is_bf16) unpack_eight_kernel<<<grid, dim3(256), 0, st>>>(codes, exponents, weight, weight_bf16, static_cast<bf16_t*>(y), rows, D);
    else unpack_eight_kernel<<<grid, dim3(256), 0, st>>>(codes, exponents, weight, weight_bf16, static_cast<float*>(y), rows, D);
    return hipGetLastError();
}

}  // namespace spion
