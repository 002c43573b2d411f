// Positions as rotations of pairs of a head's elements, with several axes.
//
// Pair i of token t turns by position[axis(i)][t] * frequency(i).  The frequency is held as turns in 2^-64, so that the product with a position,
// modulo 2^64, is the angle's fraction of a turn to position * 2^-65 turns, however far the position: no reduction loses bits.  A workgroup makes
// the sines of its tokens once, for all heads, and then moves 2 x 8 elements a thread.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_common.h"
#include "chunks.h"
#include "spion_internal.h"

namespace spion {

namespace {

constexpr int kRotaryTable = 2048;   // pairs of cosine and sine a workgroup holds

template <typename T, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(const T* __restrict__ x, T* __restrict__ y, const RotaryShape s, const long long* __restrict__ turns,
                                                     const uint8_t* __restrict__ axis, const void* __restrict__ positions, int tokens) {
    __shared__ float2 table[kRotaryTable];
    const int pairs = s.d / 2, tid = threadIdx.x;
    const long long first = (long long)blockIdx.x * tokens, total = (long long)s.B * s.L;
    const int here = (int)min((long long)tokens, total - first);
    for (int i = tid; i < here * pairs; i += 256) {
        const int t = i / pairs, p = i - t * pairs;
        const long long token = first + t, b = token / s.L, l = token - b * s.L;
        const long long at = min((int)axis[p], s.axes - 1) * s.pos_axis + b * s.pos_batch + l * s.pos_token;
        const long long pos = s.pos_bytes == 8 ? static_cast<const long long*>(positions)[at] : (long long)static_cast<const int*>(positions)[at];
        const unsigned long long angle = (unsigned long long)pos * (unsigned long long)turns[p];
        const unsigned long long quarter = (angle + (1ull << 61)) >> 62;
        // in half turns, -1/4 .. 1/4
        const float rest = (float)(long long)(angle - (quarter << 62)) * 1.0842021724855044e-19f;
        float sine, cosine;
        sincospif(rest, &sine, &cosine);
        float c = quarter & 1 ? sine : cosine, n = quarter & 1 ? cosine : sine;
        if ((quarter + 1) & 2) c = -c;
        if (quarter & 2) n = -n;
        table[i] = make_float2(c, s.back ? -n : n);
    }
    __syncthreads();
    const int chunks = s.d / 16;   // of 8 elements, and as many half a head further on
    const int items = here * s.N * chunks;
    for (int i = tid; i < items; i += 256) {
        const int c = i % chunks, rest = i / chunks;
        const int n = s.tokens_first ? rest % s.N : rest / here, t = s.tokens_first ? rest / s.N : rest % here;
        const long long token = first + t, b = token / s.L, l = token - b * s.L;
        const T* const from = x + (b * s.x_stride[0] + n * s.x_stride[1] + l * s.x_stride[2]) + 8 * c;
        T* const to = y + (b * s.y_stride[0] + n * s.y_stride[1] + l * s.y_stride[2]) + 8 * c;
        float lo[8], hi[8];
        load8<T, true>(lo, from, 8);
        load8<T, true>(hi, from + pairs, 8);
        if (n < s.rotated) {
            const float2* const cs = table + t * pairs;
            if constexpr (NEIGHBOURS) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 u = cs[4 * c + k], v = cs[pairs / 2 + 4 * c + k];
                    const float a = lo[2 * k], e = hi[2 * k];
                    lo[2 * k] = a * u.x - lo[2 * k + 1] * u.y;
                    lo[2 * k + 1] = lo[2 * k + 1] * u.x + a * u.y;
                    hi[2 * k] = e * v.x - hi[2 * k + 1] * v.y;
                    hi[2 * k + 1] = hi[2 * k + 1] * v.x + e * v.y;
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 u = cs[8 * c + k];
                    const float a = lo[k];
                    lo[k] = a * u.x - hi[k] * u.y;
                    hi[k] = hi[k] * u.x + a * u.y;
                }
            }
        }
        store8<T, true>(to, lo, 8);
        store8<T, true>(to + pairs, hi, 8);
    }
}

}  // namespace

hipError_t launch_rotary(const void* x, void* y, const RotaryShape& s, const long long* turns, const uint8_t* axis, const void* positions, bool is_bf16,
                         hipStream_t st) {
    const long long total = (long long)s.B * s.L;
    int tokens = std::max(1, kRotaryTable / (s.d / 2));
    while (tokens > 1 && (total / tokens < 1024 || (long long)tokens * s.N * (s.d / 16) > 2048)) tokens /= 2;
    const long long grid = (total + tokens - 1) / tokens;
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)grid), dim3(256), 0, st>>>(static_cast<const T*>(x), static_cast<T*>(y), s, turns, axis, positions, tokens);
    };
    if (is_bf16) s.neighbours ? launch(rotary_kernel<bf16_t, true>, bf16_t{}) : launch(rotary_kernel<bf16_t, false>, bf16_t{});
    else s.neighbours ? launch(rotary_kernel<float, true>, float{}) : launch(rotary_kernel<float, false>, float{});
    return hipGetLastError();
}

}  // namespace spion
