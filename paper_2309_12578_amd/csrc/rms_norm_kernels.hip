// Root-mean-square norm with the residual's addition, its gradient, and rows in 8 bits (eight_bit.h).
//
//   s = x + residual, rstd = 1 / sqrt(mean s^2 + eps), z = s rstd, y = z w
//   dx = ds + rstd (w dy - z mean(w dy z)), dw = sum over rows of dy z
//
// Bound by HBM.  LANES lanes have a row in registers, K times 8 consecutive elements each: one pass over the data.  What a row costs beside its elements
// (the sum over its lanes, the root) is shared by K times as many.  The sum of squares is in 64 bits, and so is all that decides a code: with a row's sum in
// another order, or in 32 bits, one in 10^5 codes would be its neighbour.
//
// 65536 x 4096, bf16, with residual: forward with codes 440 - 465 us, 5.2 - 5.4 TB/s, without 406, 5.3; y in 8 bits only 349; backward from the codes 355 - 430, 4.4 - 5.3, from h 400,
// 5.4 (copies here reach 5.0 - 5.6).  fp32, 16384 x 4096: 210, 195, 156; 160, 197.  bf16, 16384 x 256, with codes: 10.4 and 8.3 us, and 3.8 for the weight's sums.  With
// all of a code's arithmetic in 64 bits the forward pass took 523 us: 64 bits only where 32 cannot tell.
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

// Workgroups at most.  Forward: few rows each, so that they end together (65536 x 4096, bf16, with codes, 4096 and 8192 of them 474 and 459 us, 65536 x 512 59.5 and 58.4).
// Backward: as many as run at once, and leave partial rows that the second launch adds: of 256 threads three a compute unit, of more two (65536 x 512, 512, 768, 1024 and
// 1536 of them 55.8, 49.2, 52.0 and 53.9; 65536 x 4096 363, 422, 389 and 392).
constexpr int kForwardGroups = 8192;
constexpr int grad_groups_most(int threads) { return threads <= 256 ? 768 : 512; }

template <int LANES>
struct RowThreads {
    static constexpr int threads = LANES > 256 ? LANES : 256, rows = threads / LANES;
};

// Sum over the LANES lanes of a row; every lane of the workgroup takes part.  `shared` has two sets of places, used in turn: one barrier a call.
template <int LANES, typename S>
__device__ __forceinline__ S row_sum(S v, S (*shared)[LANES > 64 ? LANES / 64 : 1], int turn) {
#pragma unroll
    for (int off = 1; off < LANES && off < 64; off <<= 1) v += __shfl_xor(v, off);
    if constexpr (LANES > 64) {
        const int wave = (threadIdx.x % LANES) >> 6, row = threadIdx.x / LANES;
        static_assert(RowThreads<LANES>::rows <= 2, "rows of several waves beside each other");
        S* const place = shared[2 * turn + row];
        if ((threadIdx.x & 63) == 0) place[wave] = v;
        __syncthreads();
        v = place[0];
#pragma unroll
        for (int k = 1; k < LANES / 64; ++k) v += place[k];
    }
    return v;
}

// Elements c .. c + 7 of a row as they are in memory, beyond its D elements zeros.  In words: as elements each would take a register.
template <typename T>
struct Chunk {
    static constexpr int kWords = 2 * sizeof(T);
    unsigned w[kWords];
    __device__ __forceinline__ float at(int i) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        else return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    // as numbers that the compiler has not met
    __device__ __forceinline__ void opaque() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
};
// WHOLE: D is a multiple of 8.
template <bool WHOLE, typename T>
__device__ __forceinline__ void request(Chunk<T>& e, const T* row, int c, int D) {
    if (c + 8 <= D) {
#pragma unroll
        for (int i = 0; i < Chunk<T>::kWords / 4; ++i) *reinterpret_cast<Words*>(e.w + 4 * i) = reinterpret_cast<const Words*>(row + c)[i];
    } else {
#pragma unroll
        for (int i = 0; i < Chunk<T>::kWords; ++i) e.w[i] = 0u;
        if constexpr (!WHOLE) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < D) {
                    if constexpr (sizeof(T) == 4) e.w[i] = __builtin_bit_cast(unsigned, row[c + i]);
                    else e.w[i / 2] |= (unsigned)__builtin_bit_cast(unsigned short, row[c + i]) << (16 * (i & 1));
                }
        }
    }
}
template <typename T>
__device__ __forceinline__ void load_chunk(float (&v)[8], const T* row, int c, int D) {
    if (c + 8 <= D) load8<T, true>(v, row + c, 8);
    else load8<T, false>(v, row + c, D - c);
}
template <bool WHOLE = false, typename T>
__device__ __forceinline__ void store_chunk(T* row, int c, int D, const float (&v)[8]) {
    if (c + 8 <= D) store8<T, true>(row + c, v, 8);
    else if constexpr (!WHOLE) store8<T, false>(row + c, v, D - c);
}
// 1 / sqrt(v): the estimate's 2^-23 or better squared twice
__device__ __forceinline__ double inverse_root(double v) {
    double y = __builtin_amdgcn_rsq(v);
    if (!(v > 0.0 && y > 0.0)) return y;   // of 0, infinity and NaN: infinity, 0, NaN
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y * 0.5, fma(-v * y, y, 1.0), y);
    return y;
}

// Which codes are written: none, of z (what the backward passes take) or of y.
enum { kNoCodes = 0, kCodesOfZ = 1, kCodesOfY = 2 };

template <typename T, int LANES, int K, int CODES, bool WHOLE>
__global__ __launch_bounds__(RowThreads<LANES>::threads) void rms_norm_kernel(const T* __restrict__ x, const T* __restrict__ residual,
                                                                              const T* __restrict__ w, T* __restrict__ y, T* __restrict__ h,
                                                                              float* __restrict__ rstd, signed char* __restrict__ codes,
                                                                              uint8_t* __restrict__ exponents, long long rows, int D, double eps) {
    typedef std::conditional_t<(CODES != kNoCodes && sizeof(T) == 4), double, float> S;
    // Of two bf16 numbers a sum is exact in fp32 unless they are some 17 binary orders apart (of normal data one element in 10^5).  Where codes are decided, a wave
    // that has such an element takes its squares again, and that element's chunk its codes, from sums in 64 bits (16384 x 256 8.5 us, without that 7.6; 65536 x 4096 the
    // same).
    constexpr bool SUMS = CODES != kNoCodes && sizeof(T) == 2;
    constexpr int ROWS = RowThreads<LANES>::rows;
    __shared__ double shared[4][LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int pitch = (int)eight_pitch(D);
    const long long step = (long long)gridDim.x * ROWS;
    Chunk<T> wv[K], a[K], r[K];
#pragma unroll
    for (int k = 0; k < K; ++k) request<WHOLE>(wv[k], w, 8 * (lane + k * LANES), D);
    auto fetch = [&](long long row) {
        row = min(row, rows - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            request<WHOLE>(a[k], x + row * D, 8 * (lane + k * LANES), D);
            if (residual) request<WHOLE>(r[k], residual + row * D, 8 * (lane + k * LANES), D);
        }
    };
    long long row = (long long)blockIdx.x * ROWS + slot;
    fetch(row);
    int turn = 0;
    for (long long first = (long long)blockIdx.x * ROWS; first < rows; first += step, row += step, turn ^= 1) {
        const bool has = row < rows;
#pragma unroll
        for (int k = 0; k < K; ++k) wv[k].opaque();   // else the weights are kept in fp32
        S s[K][8];
        double squares = 0.0;
        unsigned rounded = 0;   // (of the wave) chunks with sums that fp32 does not hold
#pragma unroll
        for (int k = 0; k < K; ++k) {
            unsigned lost = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[k][i] = residual ? (S)a[k].at(i) + (S)r[k].at(i) : (S)a[k].at(i);
                if constexpr (SUMS)
                    if (residual)
                        lost |= __builtin_bit_cast(unsigned, (s[k][i] - a[k].at(i)) - r[k].at(i)) | __builtin_bit_cast(unsigned, (s[k][i] - r[k].at(i)) - a[k].at(i));
                squares = fma((double)s[k][i], (double)s[k][i], squares);
            }
            if (SUMS && __any(lost != 0)) rounded |= 1u << k;
        }
        if (SUMS && rounded) {
            squares = 0.0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                a[k].opaque();   // (else their numbers are kept in fp32)
                r[k].opaque();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double sum = (double)a[k].at(i) + (double)r[k].at(i);
                    squares = fma(sum, sum, squares);
                }
            }
        }
        if (first + step < rows) fetch(row + step);   // uniform
        const double inverse = inverse_root(row_sum<LANES>(squares, shared, turn) / D + eps);
        // else fp32 holds it with fewer bits, or (a row that is not finite, or 0) not at all
        const bool held = inverse >= 0x1p-126 && inverse <= (double)kMost;
        if (lane == 0 && has && rstd) rstd[row] = (float)inverse;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES);
            float v[8];
            if (h) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)s[k][i];
                if (has && c < D) store_chunk<WHOLE>(h + row * D, c, D, v);
            }
            // In 32 bits z is off by 3 roundings (4 with the weight): that decides a code unless it lies that near a border, or its group's largest element does.
            float z[8], most = 0.f;
            bool unsure = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = (float)s[k][i] * (float)inverse;
            if (__any(!held)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    S again = s[k][i];
                    asm volatile("" : "+v"(again));   // else what the squares were made of is kept in 64 bits
                    z[i] = held ? z[i] : (float)((double)again * inverse);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = z[i] * wv[k].at(i);
                if constexpr (CODES == kCodesOfY) {
                    z[i] = v[i];
                    unsure = unsure || !(fabsf(z[i]) < kMost * (1.f - 0x1p-20f));   // (next to infinity as well)
                }
                most = fmaxf(most, fabsf(z[i]));
            }
            if constexpr (CODES != kNoCodes) {
                unsure = unsure || !held || near_border(most);
                int exponent = group_exponent(exponent_byte(most));
                Codes8 q;
                unsure = !codes_of(q, z, exponent) || unsure;
                if (__any(unsure) || rounded >> k & 1) {   // some 3 waves in 100
                    double exact[8], largest = 0.0;
                    bool finite = true;
                    Chunk<T> again_a, again_r;
                    if (SUMS && residual) {   // (by now a and r are another row's)
                        request<WHOLE>(again_a, x + min(row, rows - 1) * D, c, D);
                        request<WHOLE>(again_r, residual + min(row, rows - 1) * D, c, D);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (SUMS && residual) {
                            exact[i] = ((double)again_a.at(i) + (double)again_r.at(i)) * inverse;
                        } else {
                            S again = s[k][i];
                            asm volatile("" : "+v"(again));   // (as above)
                            exact[i] = (double)again * inverse;
                        }
                        if constexpr (CODES == kCodesOfY) exact[i] *= (double)wv[k].at(i);
                        largest = fmax(largest, fabs(exact[i]));
                        finite = finite && exact[i] == exact[i];
                    }
                    exponent = group_exponent(finite ? exponent_byte(largest) : kNotFinite);
                    q = codes_of(exact, exponent);
                }
                if (has && c < pitch) {
                    *reinterpret_cast<Codes8*>(codes + row * pitch + c) = q;
                    if (c % kGroup == 0) exponents[row * (pitch / kGroup) + c / kGroup] = (uint8_t)exponent;
                }
            }
            if (y && has && c < D) store_chunk<WHOLE>(y + row * D, c, D, v);
            __builtin_amdgcn_sched_barrier(0);   // a chunk after the other: side by side they take twice the registers
        }
    }
}

// z from codes, or from s = h in the row's type.
template <typename T, int LANES, int K, bool CODES, bool WHOLE>
__global__ __launch_bounds__(RowThreads<LANES>::threads) void rms_norm_grad_kernel(const T* __restrict__ dy, const T* __restrict__ dh,
                                                                                   const T* __restrict__ h, const signed char* __restrict__ codes,
                                                                                   const uint8_t* __restrict__ exponents, const T* __restrict__ w,
                                                                                   const float* __restrict__ rstd, T* __restrict__ dx,
                                                                                   float* __restrict__ partial, long long rows, int D) {
    constexpr int ROWS = RowThreads<LANES>::rows;
    __shared__ float shared[4][LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int pitch = (int)eight_pitch(D);
    const long long step = (long long)gridDim.x * ROWS;
    Chunk<T> wv[K];
    float dw[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        request<WHOLE>(wv[k], w, 8 * (lane + k * LANES), D);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
    }
    // A row as it is in memory; what it stands for is made twice.
    struct Row {
        Chunk<T> dy[K], dh[K], h[K];
        Codes8 q[K];
        int exponent[K];
        float rstd;
    };
    auto fetch = [&](Row& e, long long row) {
        row = min(row, rows - 1);
        e.rstd = rstd[row];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES), p = min(c, pitch - 8);   // (beyond a row: as its last chunk, and not counted)
            request<WHOLE>(e.dy[k], dy + row * D, c, D);
            if (dh) request<WHOLE>(e.dh[k], dh + row * D, c, D);
            if constexpr (CODES) {
                e.q[k] = *reinterpret_cast<const Codes8*>(codes + row * pitch + p);
                e.exponent[k] = exponents[row * (pitch / kGroup) + p / kGroup];
            } else {
                request<WHOLE>(e.h[k], h + row * D, c, D);
            }
        }
    };
    auto z_of = [&](float (&z)[8], const Row& e, int k) {
        if constexpr (CODES) {
            values_of(z, e.q[k], eight_scale(e.exponent[k]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = e.h[k].at(i) * e.rstd;
        }
        if (WHOLE) {
            if (8 * (lane + k * LANES) >= D) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = 0.f;   // (a last group that is not finite)
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (8 * (lane + k * LANES) + i >= D) z[i] = 0.f;
        }
    };
    Row e;
    long long row = (long long)blockIdx.x * ROWS + slot;
    fetch(e, row);
    int turn = 0;
    for (long long first = (long long)blockIdx.x * ROWS; first < rows; first += step, row += step, turn ^= 1) {
        const bool has = row < rows;
#pragma unroll
        for (int k = 0; k < K; ++k) wv[k].opaque();   // else the weights are kept in fp32
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float z[8];
            z_of(z, e, k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = e.dy[k].at(i);
                if (has) dw[k][i] += g * z[i];
                sum += g * wv[k].at(i) * z[i];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {   // (as numbers that the compiler has not met: it would keep the row in fp32)
            e.dy[k].opaque();
            if constexpr (CODES) asm volatile("" : "+v"(e.q[k]), "+v"(e.exponent[k]));
            else e.h[k].opaque();
        }
        const float mean = row_sum<LANES>(sum, shared, turn) / (float)D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = 8 * (lane + k * LANES);
            float z[8], v[8];
            z_of(z, e, k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = e.rstd * (e.dy[k].at(i) * wv[k].at(i) - z[i] * mean);
                if (dh) v[i] += e.dh[k].at(i);
            }
            if (has && c < D) store_chunk<WHOLE>(dx + row * D, c, D, v);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (first + step < rows) fetch(e, row + step);   // uniform
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
            if (8 * (lane + k * LANES) < D) store_chunk<WHOLE>(partial + (size_t)blockIdx.x * D, 8 * (lane + k * LANES), D, dw[k]);
    }
}

// 16 columns a workgroup, 64 runs of partial rows, each every 64th; sums in one order.
template <typename T>
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ partial, int groups, int D, T* __restrict__ out) {
    constexpr int kColumns = 16, kRuns = 64, kInFlight = 8;
    __shared__ float part[16][kColumns];
    const int column = threadIdx.x % kColumns, run = threadIdx.x / kColumns, col = blockIdx.x * kColumns + column;
    float s = 0.f;
    for (int g = run; g < groups; g += kRuns * kInFlight) {
        float v[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) v[u] = partial[(size_t)min(g + u * kRuns, groups - 1) * D + min(col, D - 1)];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) s += g + u * kRuns < groups ? v[u] : 0.f;
    }
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if ((threadIdx.x & 63) < kColumns) part[threadIdx.x >> 6][column] = s;
    __syncthreads();
    if (threadIdx.x >= kColumns || col >= D) return;
#pragma unroll
    for (int k = 1; k < 16; ++k) s += part[k][column];
    out[col] = (T)s;
}

// i / chunks for i < n: a 64-bit division takes longer than all else here
__device__ __forceinline__ long long divided(long long i, int chunks, long long n) {
    return n <= 0x7fffffff ? (long long)((unsigned)i / (unsigned)chunks) : i / chunks;
}

// A thread has 8 elements of the padded row.  65536 x 2048, bf16, 73 us, 5.5 TB/s.  WHOLE: D is a multiple of 64, so that chunks lie in both as they are counted.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void pack_eight_kernel(const T* __restrict__ x, signed char* __restrict__ codes, uint8_t* __restrict__ exponents,
                                                         long long rows, int D) {
    const int chunks = (int)eight_pitch(D) / 8;
    const long long n = rows * chunks, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {   // (n and step are multiples of 8: a group's lanes leave together)
        float v[8], most = 0.f;
        if constexpr (WHOLE) {
            load8<T, true>(v, x + 8 * i, 8);
        } else {
            const long long row = divided(i, chunks, n);
            load_chunk(v, x + row * D, min((int)(i - row * chunks) * 8, D), D);
        }
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

// A thread has 8 elements.  WHOLE: D is a multiple of 64, and there is no weight.  65536 x 4096 to bf16 136 us, 6.0 TB/s (as rows and columns 168); 65536 x 1000 46 us, 4.3 TB/s.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void unpack_eight_kernel(const signed char* __restrict__ codes, const uint8_t* __restrict__ exponents,
                                                           const void* __restrict__ weight, int weight_bf16, T* __restrict__ y, long long rows, int D) {
    const int chunks = (D + 7) / 8, pitch = (int)eight_pitch(D);
    const long long n = rows * chunks, step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        float v[8];
        if constexpr (WHOLE) {
            values_of(v, *reinterpret_cast<const Codes8*>(codes + 8 * i), eight_scale(exponents[i / 8]));
            store8<T, true>(y + 8 * i, v, 8);
        } else {
            const long long row = divided(i, chunks, n);
            const int c = (int)(i - row * chunks) * 8;
            values_of(v, *reinterpret_cast<const Codes8*>(codes + row * pitch + c), eight_scale(exponents[row * (pitch / kGroup) + c / kGroup]));
            if (weight) {
                float wv[8];
                if (weight_bf16) load_chunk(wv, static_cast<const bf16_t*>(weight), c, D);
                else load_chunk(wv, static_cast<const float*>(weight), c, D);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= wv[e];
            }
            store_chunk(y + row * D, c, D, v);
        }
    }
}

// Lanes that have a row of D elements, and chunks a lane.
template <int LANES_, int K_>
struct Width {
    static constexpr int LANES = LANES_, K = K_, threads = RowThreads<LANES_>::threads, rows = RowThreads<LANES_>::rows;
};
// K: at most so many chunks a lane (1, 2 or 4)
template <int K, class F>
auto by_width(int D, F&& f) {
    if (D <= 64) return f(Width<8, 1>{});
    if (D <= 128) return f(Width<16 / std::min(K, 2), std::min(K, 2)>{});
    if (D <= 256) return f(Width<32 / K, K>{});
    if (D <= 512) return f(Width<64 / K, K>{});
    if (D <= 1024) return f(Width<128 / K, K>{});
    if (D <= 2048) return f(Width<256 / K, K>{});
    if (D <= 4096) return f(Width<512 / K, K>{});
    if (D <= 8192) return f(Width<1024 / K, K>{});
    return f(Width<512, 4>{});   // (1024 lanes with two chunks have too few registers)
}
// Forward, with codes, two and four chunks a lane: bf16, 65536 x 256 30.9 and 33.3 us, 16384 x 1024 30.6 and 32.9, 32768 x 2048 112.9 and 109.1, 65536 x 4096 494 and 459,
// 32768 x 8192 446 and 449; fp32, 65536 x 256 56 and 62, 16384 x 4096 210 and 217.  Backward, one and two: 65536 x 512 49 and 50, 65536 x 4096 363 and 354,
// 32768 x 8192 351 and 379.
template <typename T, class F>
auto by_forward_width(int D, F&& f) {
    if constexpr (sizeof(T) == 2)
        if (D > 1024) return by_width<4>(D, f);
    return by_width<2>(D, f);
}
int grad_groups(long long rows, int D) {
    return by_width<1>(D, [&](auto w) {
        typedef decltype(w) W;
        return (int)std::min<long long>((rows + W::rows - 1) / W::rows, grad_groups_most(W::threads));
    });
}

template <typename T>
hipError_t forward_t(const RmsNorm& a, hipStream_t st) {
    return by_forward_width<T>(a.D, [&](auto width) {
        typedef decltype(width) W;
        const unsigned grid = (unsigned)std::min<long long>((a.rows + W::rows - 1) / W::rows, kForwardGroups);
        auto launch = [&](auto kernel) {
            kernel<<<dim3(grid), dim3(W::threads), 0, st>>>(
                static_cast<const T*>(a.x), static_cast<const T*>(a.residual), static_cast<const T*>(a.w), static_cast<T*>(a.y), static_cast<T*>(a.h), a.rstd,
                a.codes, a.exponents, a.rows, a.D, a.eps);
        };
        auto codes = [&](auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            if (!a.codes) launch(rms_norm_kernel<T, W::LANES, W::K, kNoCodes, WHOLE>);
            else if (a.codes_of_y) launch(rms_norm_kernel<T, W::LANES, W::K, kCodesOfY, WHOLE>);
            else launch(rms_norm_kernel<T, W::LANES, W::K, kCodesOfZ, WHOLE>);
        };
        if (a.D % 8 == 0) codes(std::true_type{});
        else codes(std::false_type{});
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward_t(const RmsNormGrad& a, hipStream_t st) {
    const int groups = grad_groups(a.rows, a.D);
    const hipError_t e = by_width<1>(a.D, [&](auto width) {
        typedef decltype(width) W;
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)groups), dim3(W::threads), 0, st>>>(
                static_cast<const T*>(a.dy), static_cast<const T*>(a.dh), static_cast<const T*>(a.h), a.codes, a.exponents, static_cast<const T*>(a.w), a.rstd,
                static_cast<T*>(a.dx), a.dw ? a.partial : nullptr, a.rows, a.D);
        };
        auto codes = [&](auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            if (a.codes) launch(rms_norm_grad_kernel<T, W::LANES, W::K, true, WHOLE>);
            else launch(rms_norm_grad_kernel<T, W::LANES, W::K, false, WHOLE>);
        };
        if (a.D % 8 == 0) codes(std::true_type{});
        else codes(std::false_type{});
        return hipGetLastError();
    });
    if (e != hipSuccess || !a.dw) return e;
    column_sum_kernel<T><<<dim3((unsigned)((a.D + 15) / 16)), dim3(1024), 0, st>>>(a.partial, groups, a.D, static_cast<T*>(a.dw));
    return hipGetLastError();
}

// A chunk a thread, so that memory is met in order (65536 x 4096 to bf16, 8192 workgroups that go round, a chunk a thread at once 153 us, four 214; 65536 x 2048 from fp32
// 129, so 115), up to the threads that a launch can have, 2^32 - 1.
unsigned chunk_grid(long long chunks) { return (unsigned)std::min<long long>((chunks + 255) / 256, (1 << 24) - 1); }

}  // namespace

size_t rms_norm_workspace_bytes(long long rows, int D) { return (size_t)grad_groups(rows, D) * D * sizeof(float); }

hipError_t launch_rms_norm(const RmsNorm& a, bool is_bf16, hipStream_t st) { return is_bf16 ? forward_t<bf16_t>(a, st) : forward_t<float>(a, st); }
hipError_t launch_rms_norm_grad(const RmsNormGrad& a, bool is_bf16, hipStream_t st) { return is_bf16 ? backward_t<bf16_t>(a, st) : backward_t<float>(a, st); }

hipError_t launch_pack_eight(const void* x, signed char* codes, uint8_t* exponents, long long rows, int D, bool is_bf16, hipStream_t st) {
    const dim3 grid(chunk_grid(rows * (eight_pitch(D) / 8)));
    auto launch = [&](auto kernel, auto type) { kernel<<<grid, dim3(256), 0, st>>>(static_cast<const decltype(type)*>(x), codes, exponents, rows, D); };
    if (is_bf16) D % kGroup == 0 ? launch(pack_eight_kernel<bf16_t, true>, bf16_t{}) : launch(pack_eight_kernel<bf16_t, false>, bf16_t{});
    else D % kGroup == 0 ? launch(pack_eight_kernel<float, true>, float{}) : launch(pack_eight_kernel<float, false>, float{});
    return hipGetLastError();
}
hipError_t launch_unpack_eight(const signed char* codes, const uint8_t* exponents, const void* weight, bool weight_bf16, void* y, long long rows, int D,
                               bool is_bf16, hipStream_t st) {
    const dim3 grid(chunk_grid(rows * ((D + 7) / 8)));
    const bool whole = D % kGroup == 0 && !weight;
    auto launch = [&](auto kernel, auto type) { kernel<<<grid, dim3(256), 0, st>>>(codes, exponents, weight, weight_bf16, static_cast<decltype(type)*>(y), rows, D); };
    if (is_bf16) whole ? launch(unpack_eight_kernel<bf16_t, true>, bf16_t{}) : launch(unpack_eight_kernel<bf16_t, false>, bf16_t{});
    else whole ? launch(unpack_eight_kernel<float, true>, float{}) : launch(unpack_eight_kernel<float, false>, float{});
    return hipGetLastError();
}

}  // namespace spion
