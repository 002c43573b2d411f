// The weight's gradient of a projection whose input was kept in 8 bits (eight_bit.h): dW[n][m] = w[m] * sum over rows of dY[row][n] * code * 2^k,
// and beside it the bias' gradient, the column sums of dY.
//
// code * 2^k is exact in bf16, so X enters the product as it was kept, without a rounding.  An fp32 dY enters as the sum of three bf16 numbers, its
// significand's 24 bits by eights: three bf16 products, exact but for the sums, at 8 times the rate of the fp32 matrix instruction each.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "eight_bit.h"
#include "spion_internal.h"

namespace spion {

namespace {

constexpr int kGradGroups = 384;
constexpr int kGradMinRows = 128;
constexpr int kTile = 128;       // outputs of a workgroup in each direction; a wave has 64 x 64 of them
constexpr int kStepRows = 32;    // rows of a step: one bf16 MFMA contracts over 32
constexpr int kLd = kTile + 16;  // elements between rows in LDS

template <typename T>
struct Planes {
    static constexpr int n = sizeof(T) == 4 ? 3 : 1;
};

// v as a sum of three numbers of 8 significant bits; what is not finite stays in the first.
__device__ __forceinline__ void three_parts(float v, bf16_t& a, bf16_t& b, bf16_t& c) {
    auto top = [](float f) { return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, f) & 0xffff0000u); };
    auto half = [](float f) { return __builtin_bit_cast(bf16_t, (unsigned short)(__builtin_bit_cast(unsigned, f) >> 16)); };
    const bool finite = fabsf(v) <= 3.4028234663852886e38f;
    const float first = v != v ? __builtin_nanf("") : top(v);
    const float rest = finite ? v - first : 0.f;
    a = half(first);
    b = half(rest);
    c = half(rest - top(rest));
}

template <typename T, bool WHOLE>   // WHOLE: 16-byte loads of dY, whose rows are then aligned
__global__ __launch_bounds__(256) void weight_grad_eight_kernel(const T* __restrict__ dY, const signed char* __restrict__ codes,
                                                                const uint8_t* __restrict__ exponents, float* __restrict__ partial,
                                                                float* __restrict__ bias_partial, int rows, int N, int M, int slices, int slice_rows,
                                                                int tiles_n, int tiles_m) {
    constexpr int PLANES = Planes<T>::n;
    __shared__ __attribute__((aligned(16))) bf16_t ys[2][PLANES][kStepRows * kLd], xs[2][kStepRows * kLd];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pitch = (int)eight_pitch(M);
    // the tiles of a slice on one XCD: they read the same rows
    const int tiles = tiles_n * tiles_m, l = blockIdx.x >> 3;
    const int slice = l / tiles * 8 + (blockIdx.x & 7), tile = l % tiles;
    if (slice >= slices) return;
    const int n0 = tile / tiles_m * kTile, m0 = tile % tiles_m * kTile;
    const int first = slice * slice_rows, end = min(rows, first + slice_rows);
    const bool sums_bias = bias_partial && m0 == 0;

    // a thread brings 8 columns of rows row, row + 16 of dY, 16 columns of row x_row of the codes
    const int row = tid >> 4, col = (tid & 15) * 8, x_row = tid >> 3, x_col = (tid & 7) * 16;
    const bool has_n = n0 + col < N, has_m = m0 + x_col < pitch;
    struct Rows {
        float y[2][8];
        uint4 x;
        int exponent;
    };
    auto request = [&](Rows& v, int at) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const T* const p = dY + (size_t)min(at + row + 16 * k, end - 1) * N + n0 + (has_n ? col : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) v.y[k][i] = WHOLE || n0 + col + i < N ? (float)p[i] : 0.f;
        }
        const size_t i = (size_t)min(at + x_row, end - 1);
        const int c = m0 + (has_m ? x_col : 0);
        v.x = *reinterpret_cast<const uint4*>(codes + i * pitch + c);
        v.exponent = exponents[i * (pitch / kGroup) + c / kGroup];
    };
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto put = [&](const Rows& v, int at, int b) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            bf16x8 part[3];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = at + row + 16 * k < end ? v.y[k][i] : 0.f;
                bias[i] += y;
                if constexpr (PLANES == 3) {
                    bf16_t p, q, s;
                    three_parts(y, p, q, s);
                    part[0][i] = p, part[1][i] = q, part[2][i] = s;
                } else {
                    part[0][i] = (bf16_t)y;
                }
            }
#pragma unroll
            for (int p = 0; p < PLANES; ++p) *reinterpret_cast<bf16x8*>(&ys[b][p][(row + 16 * k) * kLd + col]) = part[p];
        }
        const bool has = at + x_row < end;
        const float scale = eight_scale(v.exponent);
        const unsigned words[4] = {v.x.x, v.x.y, v.x.z, v.x.w};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float x[8];
            values_of(x, Codes8{words[2 * k], words[2 * k + 1]}, scale);
            bf16x8 q;
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = has ? (bf16_t)x[i] : (bf16_t)0.f;
            *reinterpret_cast<bf16x8*>(&xs[b][x_row * kLd + x_col + 8 * k]) = q;
        }
    };
    const int wn = (wave >> 1) * 64, wm = (wave & 1) * 64;
    const int tr = (4 * g + (r >> 2)) * kLd + 4 * (r & 3);   // transpose read: lane r receives column r of rows 4 g ..
    f32x4 acc[4][4];   // [n tile][m tile]
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](int b) {
        bf16x8 fx[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const bf16_t* const x = &xs[b][tr + wm + 16 * t];
            fx[t] = join(lds_read_tr(x), lds_read_tr(x + 16 * kLd));
        }
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            bf16x8 fy[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const bf16_t* const y = &ys[b][p][tr + wn + 16 * t];
                fy[t] = join(lds_read_tr(y), lds_read_tr(y + 16 * kLd));
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[a][c] = mma_d(acc[a][c], fx[c], fy[a]);   // [m][n]
        }
    };
    const int steps = (end - first + kStepRows - 1) / kStepRows;
    Rows v;
    request(v, first);
    for (int s = 0, at = first; s < steps; ++s, at += kStepRows) {
        put(v, at, s & 1);
        request(v, at + kStepRows);
        __syncthreads();   // (the stage written two steps on has been read by then)
        multiply(s & 1);
    }
    float* const out = partial + (size_t)slice * N * pitch;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int n = n0 + wn + 16 * a + r;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int m = m0 + wm + 16 * c + 4 * g;
            if (n < N && m < pitch) *reinterpret_cast<f32x4*>(out + (size_t)n * pitch + m) = acc[a][c];
        }
    }
    if (!sums_bias) return;
    float(*const part)[kTile] = reinterpret_cast<float(*)[kTile]>(&xs[0][0]);   // [16][kTile]
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) part[row][col + i] = bias[i];
    __syncthreads();
    if (tid < kTile && n0 + tid < N) {
        float s = part[0][tid];
#pragma unroll
        for (int k = 1; k < 16; ++k) s += part[k][tid];
        bias_partial[(size_t)slice * N + n0 + tid] = s;
    }
}

// A workgroup has 64 vectors of 4 outputs of dW (the last workgroups: of db), a wave a quarter of their slices; the quarters are added in order.
template <typename T>
__global__ __launch_bounds__(256) void weight_grad_eight_sum_kernel(const float* __restrict__ partial, const float* __restrict__ bias_partial, int slices,
                                                                    int N, int M, const T* __restrict__ weight, T* __restrict__ dW, T* __restrict__ db,
                                                                    unsigned groups) {
    __shared__ float part[4][64][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pitch = (int)eight_pitch(M);
    const bool bias = blockIdx.x >= groups;
    const size_t n4 = (size_t)N * (pitch / 4), i = (size_t)(bias ? blockIdx.x - groups : blockIdx.x) * 64 + lane;
    const int begin = wave * slices / 4, end = (wave + 1) * slices / 4;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = begin; s < end; ++s) {
        if (bias) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (4 * i + k < (size_t)N) acc[k] += bias_partial[(size_t)s * N + 4 * i + k];
        } else if (i < n4) {
            const f32x4 v = reinterpret_cast<const f32x4*>(partial)[s * n4 + i];
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] += v[k];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][lane][k] = acc[k];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float v = ((part[0][lane][k] + part[1][lane][k]) + part[2][lane][k]) + part[3][lane][k];
        if (bias) {
            if (4 * i + k < (size_t)N) db[4 * i + k] = (T)v;
        } else if (i < n4) {
            const size_t n = i / (pitch / 4);
            const int m = (int)(i - n * (pitch / 4)) * 4 + k;
            if (m < M) dW[n * M + m] = (T)(weight ? v * (float)weight[m] : v);
        }
    }
}

struct Plan {
    int tiles_n, tiles_m, slices, slice_rows;
    size_t bias_at, total;   // bytes
    Plan(int rows, int N, int M) {
        tiles_n = (N + kTile - 1) / kTile;
        tiles_m = (int)((eight_pitch(M) + kTile - 1) / kTile);
        const long long most = ((long long)rows + kGradMinRows - 1) / kGradMinRows, want = kGradGroups / ((long long)tiles_n * tiles_m);
        slices = (int)std::max<long long>(1, std::min(want, most));
        slice_rows = (int)((((long long)rows + slices - 1) / slices + kStepRows - 1) / kStepRows * kStepRows);
        slices = (int)(((long long)rows + slice_rows - 1) / slice_rows);
        bias_at = (size_t)slices * N * eight_pitch(M) * sizeof(float);
        total = bias_at + (size_t)slices * N * sizeof(float);
    }
};

}  // namespace

size_t weight_grad_eight_workspace_bytes(int rows, int N, int M) { return Plan(rows, N, M).total; }

template <typename T>
static hipError_t launch_t(const WeightGradEight& a, hipStream_t st) {
    const Plan p(a.rows, a.N, a.M);
    float *const partial = static_cast<float*>(a.workspace),
                 *const bias_partial = a.db ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + p.bias_at) : nullptr;
    const unsigned groups = (unsigned)((p.slices + 7) / 8 * 8) * (unsigned)(p.tiles_n * p.tiles_m);
    auto launch = [&](auto kernel) {
        kernel<<<dim3(groups), dim3(256), 0, st>>>(static_cast<const T*>(a.dY), a.codes, a.exponents, partial, bias_partial, a.rows, a.N, a.M, p.slices,
                                                   p.slice_rows, p.tiles_n, p.tiles_m);
    };
    const bool whole = a.N % 8 == 0 && (uintptr_t)a.dY % 16 == 0;
    whole ? launch(weight_grad_eight_kernel<T, true>) : launch(weight_grad_eight_kernel<T, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const unsigned sums = (unsigned)(((size_t)a.N * (eight_pitch(a.M) / 4) + 63) / 64), more = a.db ? (unsigned)((a.N + 255) / 256) : 0u;
    weight_grad_eight_sum_kernel<T><<<dim3(sums + more), dim3(256), 0, st>>>(partial, bias_partial, p.slices, a.N, a.M, static_cast<const T*>(a.weight),
                                                                             static_cast<T*>(a.dW), static_cast<T*>(a.db), sums);
    return hipGetLastError();
}
hipError_t launch_weight_grad_eight(const WeightGradEight& a, bool is_bf16, hipStream_t st) { return is_bf16 ? launch_t<bf16_t>(a, st) : launch_t<float>(a, st); }

}  // namespace spion
