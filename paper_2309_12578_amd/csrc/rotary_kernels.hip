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

constexpr int kRotaryTable = 2048, kRotaryTokens = 128;   // pairs of cosine and sine, and tokens, that a workgroup has room for

// Of an eighth of a turn at most, either way, given in 2^-64 turns: the series, whose next terms are below 2^-28.5 of the results there.
__device__ __forceinline__ void sine_cosine(float turns, float& sine, float& cosine) {
    const float t = turns * 3.4061215800098876e-19f;   // 2 pi / 2^64
    const float q = t * t;
    sine = fmaf(t * q, fmaf(q, fmaf(q, fmaf(q, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), t);
    cosine = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
}

// (a, b) by the turn with cosine u.x and sine u.y.  A sine of 0 adds nothing: a pair that does not turn stays as it is beside an infinity or NaN, too.
__device__ __forceinline__ void turn_pair(float& a, float& b, float2 u) {
    const float of_a = u.y == 0.f ? 0.f : a * u.y, of_b = u.y == 0.f ? 0.f : b * u.y;
    a = fmaf(a, u.x, -of_b);
    b = fmaf(b, u.x, of_a);
}

template <typename T, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(const T* __restrict__ x, T* __restrict__ y, const RotaryShape s, const long long* __restrict__ turns,
                                                     const uint8_t* __restrict__ axis, const void* __restrict__ positions, int tokens, unsigned begin) {
    __shared__ float2 table[kRotaryTable];
    __shared__ long long place[kRotaryTokens][2];   // of the tokens in x and y
    const int pairs = s.d / 2, tid = threadIdx.x;
    const unsigned first = begin + blockIdx.x * (unsigned)tokens, total = (unsigned)s.B * (unsigned)s.L;   // (below 2^31)
    const int here = (int)min((unsigned)tokens, total - first);
    // A thread has every 256th of what follows, by numbers that are carried: no divisions.
    {
        const int p_step = 256 % pairs, t_step = 256 / pairs;
        int p = tid % pairs, t = tid / pairs, known = -1;
        unsigned b = (first + t) / (unsigned)s.L, l = first + t - b * s.L;
        unsigned long long frequency = 0;
        long long of_axis = 0;
        while (t < here) {
            if (p != known) {   // the same each time where the pairs divide the threads
                known = p;
                of_axis = min((int)axis[p], s.axes - 1) * s.pos_axis;
                frequency = (unsigned long long)turns[p];
            }
            const long long at = of_axis + b * s.pos_batch + l * s.pos_token;
            const long long pos = s.pos_bytes == 8 ? static_cast<const long long*>(positions)[at] : (long long)static_cast<const int*>(positions)[at];
            const unsigned long long angle = (unsigned long long)pos * frequency;
            const unsigned long long quarter = (angle + (1ull << 61)) >> 62;
            float sine, cosine;
            sine_cosine((float)(long long)(angle - (quarter << 62)), sine, cosine);
            float c = quarter & 1 ? sine : cosine, n = quarter & 1 ? cosine : sine;
            if ((quarter + 1) & 2) c = -c;
            if (quarter & 2) n = -n;
            table[t * pairs + p] = make_float2(c, s.back ? -n : n);
            if (p == 0) {
                place[t][0] = b * s.x_stride[0] + l * s.x_stride[2];
                place[t][1] = b * s.y_stride[0] + l * s.y_stride[2];
            }
            const int was = t;
            p += p_step;
            t += t_step;
            if (p >= pairs) {
                p -= pairs;
                ++t;
            }
            l += t - was;
            if (l >= (unsigned)s.L) {
                b = (first + t) / (unsigned)s.L;
                l = first + t - b * s.L;
            }
        }
    }
    __syncthreads();
    // Items (token, head, 8 elements and as many half a head further on), in the order of memory: the elements, then heads and tokens, or tokens and heads.
    const int chunks = s.d / 16, inner_size = s.tokens_first ? s.N : here, outer_size = s.tokens_first ? here : s.N;
    const int c_step = 256 % chunks, inner_step = 256 / chunks % inner_size, outer_step = 256 / chunks / inner_size;
    int c = tid % chunks, inner = tid / chunks % inner_size, outer = tid / chunks / inner_size;
    while (outer < outer_size) {
        const int n = s.tokens_first ? inner : outer, t = s.tokens_first ? outer : inner;
        const T* const from = x + (place[t][0] + n * s.x_stride[1]) + 8 * c;
        T* const to = y + (place[t][1] + n * s.y_stride[1]) + 8 * c;
        float lo[8], hi[8];
        load8<T, true>(lo, from, 8);
        load8<T, true>(hi, from + pairs, 8);
        if (n < s.rotated) {
            const float2* const cs = table + t * pairs;
            if constexpr (NEIGHBOURS) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    turn_pair(lo[2 * k], lo[2 * k + 1], cs[4 * c + k]);
                    turn_pair(hi[2 * k], hi[2 * k + 1], cs[pairs / 2 + 4 * c + k]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) turn_pair(lo[k], hi[k], cs[8 * c + k]);
            }
        }
        store8<T, true>(to, lo, 8);
        store8<T, true>(to + pairs, hi, 8);
        c += c_step;
        inner += inner_step;
        outer += outer_step;
        if (c >= chunks) {
            c -= chunks;
            ++inner;
        }
        if (inner >= inner_size) {
            inner -= inner_size;
            ++outer;
        }
    }
}

}  // namespace

hipError_t launch_rotary(const void* x, void* y, const RotaryShape& s, const long long* turns, const uint8_t* axis, const void* positions, bool is_bf16,
                         hipStream_t st) {
    const long long total = (long long)s.B * s.L;
    // Tokens of a workgroup: two items a thread where the heads of a token lie together, eight where a head's tokens do, whose lines then are longer (4 x 24 x 16384 x 64,
    // bf16, 512, 1024, 2048 and 4096 items: 75, 79, 83 and 88 us, 91, 85, 82 and 83), but 1024 workgroups first.
    const long long most = s.tokens_first ? 512 : 2048;
    int tokens = std::min(kRotaryTokens, kRotaryTable / (s.d / 2));
    while (tokens > 1 && (total / tokens < 1024 || (long long)tokens * s.N * (s.d / 16) > most)) tokens /= 2;
    const long long grid = (total + tokens - 1) / tokens;
    constexpr long long kMostGroups = 1 << 23;   // of a launch, which can have 2^32 - 1 threads
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        for (long long g = 0; g < grid; g += kMostGroups)
            kernel<<<dim3((unsigned)std::min(grid - g, kMostGroups)), dim3(256), 0, st>>>(static_cast<const T*>(x), static_cast<T*>(y), s, turns, axis, positions, tokens,
                                                                                         (unsigned)(g * tokens));
    };
    if (is_bf16) s.neighbours ? launch(rotary_kernel<bf16_t, true>, bf16_t{}) : launch(rotary_kernel<bf16_t, false>, bf16_t{});
    else s.neighbours ? launch(rotary_kernel<float, true>, float{}) : launch(rotary_kernel<float, false>, float{});
    return hipGetLastError();
}

}  // namespace spion
