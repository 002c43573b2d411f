// Gradients of a projection whose input was kept in 8 bits (eight_bit.h).  The input's, where it is small: input_grad_kernel.  The weight's: dW[n][m] = w[m] * sum over rows of dY[row][n] * code * 2^k,
// and beside it the bias' gradient, the column sums of dY.
//
// code * 2^k is exact in bf16, so X enters the product as it was kept, without a rounding.  An fp32 dY enters as the sum of three bf16 numbers, its
// significand's 24 bits by eights (but for bits below 2^-133, which bf16 does not have: of numbers below 2^-110): three bf16 products, exact but for the sums, at 8 times
// the rate of the fp32 matrix instruction each.
//
// Bound by the matrix units where N and M are large (65536 x 2048 x 2048 bf16 540 - 630 us, 0.87 - 1.0 PFLOP/s, the sums of its slices 16 us; fp32 8192 x 1536 x 512 59 us and 7), by the
// start and the end of a slice where they are small (16384 x 768 x 256 bf16 21 us and 5).  Tiles as large as the registers hold, so that LDS feeds them; bf16 as two workgroups
// a compute unit, one of which multiplies while the other waits (one of 256 x 256: 685 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "eight_bit.h"
#include "spion_internal.h"

namespace spion {

namespace {

constexpr int kStepRows = 32;   // rows of a step
constexpr int kWaitVm6 = 0x0F76;
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Outputs of a workgroup, [TN][TM], and how its waves share them.
template <int TN_, int TM_, int WN_, int WM_>
struct Tile {
    static constexpr int TN = TN_, TM = TM_, WN = WN_, WM = WM_, threads = 64 * WN_ * WM_;
    static constexpr int FN = TN / WN / 32, FM = TM / WM / 32;   // 32 x 32 outputs of a wave
};
typedef Tile<128, 128, 2, 2> Small;
typedef Tile<256, 128, 2, 2> Wide;    // bf16: two workgroups a compute unit
typedef Tile<256, 256, 4, 2> Large;   // fp32: one

template <typename T>
struct Planes {
    static constexpr int n = sizeof(T) == 4 ? 3 : 1;
};

// v as a sum of three numbers of 8 significant bits.  An infinity stays in the first; of a NaN at least one part is NaN.
__device__ __forceinline__ void three_parts(float v, bf16_t& a, bf16_t& b, bf16_t& c) {
    auto top = [](float f) { return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, f) & 0xffff0000u); };
    auto half = [](float f) { return __builtin_bit_cast(bf16_t, (unsigned short)(__builtin_bit_cast(unsigned, f) >> 16)); };
    const float first = top(v), rest = first == v ? 0.f : v - first;
    a = half(first);
    b = half(rest);
    c = half(rest - top(rest));
}

// Rows in LDS are 2 TN or 2 TM bytes long without padding; the 16-byte slots of a row are permuted by its number, so that the four rows of 64 bytes that half a
// wave fetches with a transposing read are on different banks.
__device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((row & 3) << 2); }

// Where a lane's part of a transposing read is: rows 8 j + 4 (lane / 32) + .., columns 32 q + 16 (lane / 16 % 2) + .. of a matrix of W columns; lane l receives column
// 32 q + l % 32 of four rows.
template <int W>
__device__ __forceinline__ int read_offset(int lane, int q) {
    const int r = lane & 15, row = 4 * (lane >> 5) + (r >> 2);
    return row * W + slot_of(row, 4 * q + 2 * ((lane >> 4) & 1) + ((r & 3) >> 1)) * 8 + 4 * (r & 1);
}

// Rows `first` to `end` of a matrix with rows of `row` bytes, fewer than 2^31 bytes; what a load asks for beyond them comes as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_between(const void* p, int first, int end, size_t row) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p)) + (size_t)first * row, (short)0, (int)((end - first) * row), 0x00027000);
}
typedef unsigned Four __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Four fetch_four(__amdgpu_buffer_rsrc_t from, unsigned off) { return __builtin_amdgcn_raw_buffer_load_b128(from, off, 0, 0); }
__device__ __forceinline__ unsigned fetch_byte(__amdgpu_buffer_rsrc_t from, unsigned off) { return __builtin_amdgcn_raw_buffer_load_b8(from, off, 0, 0); }
// Into consecutive LDS: 16 bytes a lane from byte `off` on, or one byte, which becomes a word.
__device__ __forceinline__ void load_rows(__amdgpu_buffer_rsrc_t from, unsigned off, void* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void_ptr)to, 16, off, 0, 0, 0);
}
__device__ __forceinline__ void load_bytes(__amdgpu_buffer_rsrc_t from, unsigned off, void* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void_ptr)to, 1, off, 0, 0, 0);
}

// fp32 sums of products.  A step brings 32 rows of dY and of the codes, and has one barrier.  Codes become bf16 in LDS a step before they are multiplied.
// bf16 and WHOLE (rows of dY aligned to 16 bytes): dY goes from memory straight into LDS, two steps ahead; codes and exponents too, three steps ahead, each lane's
// to where it takes them from again.  (All by the same instruction, so that the counts that are waited for do not depend on how the compiler orders loads.)  Rows
// behind the last come as zeros, codes and scales as well, by the range of the loads.
// Else through registers, requested two steps ahead; where rows of dY are not aligned, by elements (bf16, with the sums, 16384 x 1000 x 768 46 us, x 1001 119).
template <typename T, typename S, bool WHOLE>
__global__ __launch_bounds__(S::threads, 2) void weight_grad_eight_kernel(
    const T* __restrict__ dY, const signed char* __restrict__ codes, const uint8_t* __restrict__ exponents, const T* __restrict__ weight, T* __restrict__ dW,
    float* __restrict__ partial, float* __restrict__ bias_partial, int rows, int N, int M, int slices, int slice_rows, int span_rows, int tiles_n,
    int tiles_m) {
    constexpr int PLANES = Planes<T>::n, TN = S::TN, TM = S::TM, FN = S::FN, FM = S::FM, WAVES = S::threads / 64;
    constexpr bool ASYNC = WHOLE && PLANES == 1;
    struct Y {
        bf16_t v[PLANES][kStepRows * TN];
    };
    struct X {
        bf16_t v[kStepRows * TM];
    };
    struct Raw {
        uint4 codes[S::threads];
        int exponents[S::threads];
    };
    // objects of their own, so that the compiler can tell a read of one stage from a load in flight into another
    __shared__ __attribute__((aligned(1024))) Y ys0, ys1;
    __shared__ __attribute__((aligned(1024))) X xs0, xs1;
    __shared__ __attribute__((aligned(1024))) std::conditional_t<ASYNC, Y, char> ys2;
    __shared__ __attribute__((aligned(1024))) std::conditional_t<ASYNC, Raw, char> raw0, raw1, raw2;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pitch = (int)eight_pitch(M);
    // an XCD has slices, or a part of one, whose tiles read the same rows
    const int tiles = tiles_n * tiles_m, item = xcd_deal(blockIdx.x, 0, gridDim.x);
    const int slice = item / tiles, tile = item % tiles, tile_n = tile / tiles_m, tile_m = tile % tiles_m;
    const int n0 = tile_n * TN, m0 = tile_m * TM;
    // the rows of a slice, in spans whose bytes have offsets of 31 bits
    int first = slice * slice_rows;
    const int slice_end = first + min(rows - first, slice_rows);   // (first + slice_rows may be 2^31)
    int end = first + min(slice_end - first, span_rows);
    const int wave_n = wave / S::WM, wave_m = wave % S::WM;

    // dY into LDS in pieces of 1 KB
    constexpr int Y_SLOTS = TN / 8, Y_PIECE = 64 / Y_SLOTS, Y_PIECES = kStepRows / Y_PIECE / WAVES;   // rows of a piece, pieces of a wave
    unsigned y_off[Y_PIECES];
    // the next 32 rows, each time
    auto y_rows = rows_between(dY, first, end, (size_t)N * sizeof(T)), x_rows = rows_between(codes, first, end, (size_t)pitch),
         e_rows = rows_between(exponents, first, end, (size_t)(pitch / kGroup));
    auto own = [&]() {   // the wave's number; computed from it anew each time: kept for every stage, the addresses would not fit the scalar registers
        int w = wave;
        asm volatile("" : "+s"(w));
        return w;
    };
    auto request_y = [&](auto& to) {
        bf16_t* const p = to.v[0] + own() * (Y_PIECES * 512);
#pragma unroll
        for (int k = 0; k < Y_PIECES; ++k) {
            load_rows(y_rows, y_off[k], p + k * 512);
            y_off[k] += (unsigned)(kStepRows * N) * (unsigned)sizeof(T);
        }
    };
    // through registers: 8 columns of every Y_ROWS-th row from y_row on; 16 columns of row x_row of the codes
    constexpr int Y_ROWS = S::threads / Y_SLOTS, Y_TIMES = kStepRows / Y_ROWS;
    const int y_row = tid / Y_SLOTS, y_chunk = tid % Y_SLOTS, x_row = tid / (TM / 16), x_chunk = tid % (TM / 16);
    static_assert(Y_ROWS * Y_TIMES == kStepRows && S::threads / (TM / 16) == kStepRows && WAVES * Y_PIECES * Y_PIECE == kStepRows, "a step's pieces");
    const bool has_m = m0 + 16 * x_chunk < pitch;
    unsigned x_off, v_off;
    auto to_first = [&]() {
        int t = tid;
        asm volatile("" : "+v"(t));   // anew for each span: kept for the next one they would take registers throughout
#pragma unroll
        for (int k = 0; k < Y_PIECES; ++k) {
            const int row = (Y_PIECES * wave + k) * Y_PIECE + (t & 63) / Y_SLOTS;
            y_off[k] = (unsigned)(row * N + n0 + slot_of(row, (t & 63) % Y_SLOTS) * 8) * (unsigned)sizeof(bf16_t);
        }
        x_off = (unsigned)(t / (TM / 16) * pitch + m0 + 16 * (t % (TM / 16)));
        v_off = (unsigned)(t / Y_SLOTS * N + n0 + 8 * (t % Y_SLOTS)) * (unsigned)sizeof(T);
    };
    auto request_raw = [&](auto& to) {
        const int w = own();
        load_rows(x_rows, x_off, to.codes + 64 * w);
        load_bytes(e_rows, x_off / kGroup, to.exponents + 64 * w);
        x_off += (unsigned)(kStepRows * pitch);
    };
    // Codes 2 i and 2 i + 1 of 16 as bf16: products that are exact, or 2^128.
    auto convert = [&](uint4 q, float scale, int i) {
        const unsigned words[4] = {q.x, q.y, q.z, q.w};
        const unsigned w = words[i / 2] >> (16 * (i & 1));
        const float a = (float)(signed char)w * scale, b = (float)(signed char)(w >> 8) * scale;
        return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
    };
    auto put_x = [&](const unsigned (&v)[8], X& to) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            *reinterpret_cast<uint4*>(&to.v[x_row * TM + slot_of(x_row, 2 * x_chunk + k) * 8]) = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    };
    struct Rows {
        T y[Y_TIMES][8];
        uint4 x;
        int exponent;
    };
    constexpr bool RANGED = WHOLE && !ASYNC;
    auto request = [&](Rows& v, int at) {
        if constexpr (RANGED) {   // (fp32) the next 32 rows each time, by their range as above
#pragma unroll
            for (int k = 0; k < Y_TIMES; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const Four f = fetch_four(y_rows, v_off + (unsigned)(Y_ROWS * k * N) * 4u + 16u * i);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const unsigned word = f[u];   // (a cast of the vector's element itself takes the first one)
                        v.y[k][4 * i + u] = __builtin_bit_cast(float, word);
                    }
                }
            const Four q = fetch_four(x_rows, x_off);
            v.x = make_uint4(q[0], q[1], q[2], q[3]);
            v.exponent = (int)fetch_byte(e_rows, x_off / kGroup);
            v_off += (unsigned)(kStepRows * N) * 4u;
            x_off += (unsigned)(kStepRows * pitch);
            return;
        }
        const int n = n0 + 8 * y_chunk;
#pragma unroll
        for (int k = 0; k < Y_TIMES; ++k) {
            const T* const p = dY + (size_t)min(at + y_row + Y_ROWS * k, end - 1) * N + (n < N ? n : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) v.y[k][i] = WHOLE || n + i < N ? p[i] : (T)0.f;
        }
        const size_t i = (size_t)min(at + x_row, end - 1);
        const int c = has_m ? m0 + 16 * x_chunk : 0;
        v.x = *reinterpret_cast<const uint4*>(codes + i * pitch + c);
        v.exponent = exponents[i * (pitch / kGroup) + c / kGroup];
    };
    auto put = [&](Rows& v, int at, Y& to_y, X& to_x) {
        if (!RANGED && at + kStepRows > end) {   // uniform
#pragma unroll
            for (int k = 0; k < Y_TIMES; ++k)
                if (at + y_row + Y_ROWS * k >= end) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v.y[k][i] = (T)0.f;
                }
            if (at + x_row >= end) v.exponent = 0;   // the scale 0
        }
#pragma unroll
        for (int k = 0; k < Y_TIMES; ++k) {
            const int row = y_row + Y_ROWS * k;
            bf16x8 part[3];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (PLANES == 3) {
                    bf16_t p, q, s;
                    three_parts(v.y[k][i], p, q, s);
                    part[0][i] = p, part[1][i] = q, part[2][i] = s;
                } else {
                    part[0][i] = v.y[k][i];
                }
            }
#pragma unroll
            for (int p = 0; p < PLANES; ++p) *reinterpret_cast<bf16x8*>(&to_y.v[p][row * TN + slot_of(row, y_chunk) * 8]) = part[p];
        }
        const float scale = eight_scale(v.exponent);
        unsigned x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = convert(v.x, scale, i);
        put_x(x, to_x);
    };

    int fy_off[FN], fx_off[FM];
#pragma unroll
    for (int f = 0; f < FN; ++f) fy_off[f] = read_offset<TN>(lane, wave_n * FN + f);
#pragma unroll
    for (int f = 0; f < FM; ++f) fx_off[f] = read_offset<TM>(lane, wave_m * FM + f);
    f32x16 acc[FN][FM];
    float bias[FN];
#pragma unroll
    for (int a = 0; a < FN; ++a) {
        bias[a] = 0.f;
#pragma unroll
        for (int b = 0; b < FM; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
    }
    // operands of 16 rows
    struct Operands {
        bf16x8 y[FN], x[FM];
    };
    auto read_y = [&](Operands& o, const Y& y, int p, int k, int f) {
        o.y[f] = join(lds_read_tr(y.v[p] + fy_off[f] + 16 * k * TN), lds_read_tr(y.v[p] + fy_off[f] + (16 * k + 8) * TN));
    };
    auto read_x = [&](Operands& o, const X& x, int k, int f) {
        o.x[f] = join(lds_read_tr(x.v + fx_off[f] + 16 * k * TM), lds_read_tr(x.v + fx_off[f] + (16 * k + 8) * TM));
    };
    auto multiply = [&](const Operands& o, int i) {
        const int a = i / FM, b = i % FM;
        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(o.y[a], o.x[b], acc[a][b], 0, 0, 0);
    };
    auto add_bias = [&](const Operands& o) {
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
            for (int i = 0; i < 8; ++i) bias[f] += (float)o.y[f][i];
    };
    // the steps' column sums of dY are shared by the workgroups and waves that have the same columns
    const int shares = tiles_m * S::WM, share = tile_m * S::WM + wave_m;
    const bool wants_bias = bias_partial != nullptr;
    int turn = 0;
    auto meet = [&]() {
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    for (;;) {
        to_first();
        const int steps = (end - first + kStepRows - 1) / kStepRows;
        if constexpr (ASYNC) {
            // Step s reads ys[s % 3] and xs[s % 2], makes xs[(s + 1) % 2] from raw[(s + 1) % 3], and requests what two and three steps on takes into the stages
            // that step s - 1 has read.  Of what is in flight at its start, the loads of step s - 1 may stay there: codes and exponents of s + 2, rows of s + 1.
            static_assert(Y_PIECES == 2 || Y_PIECES == 4, "loads of a step");
            auto step = [&](Y& y, Y& y_free, X& x, X& x_free, Raw& raw, Raw& raw_free) {
                __builtin_amdgcn_s_waitcnt(Y_PIECES == 2 ? kWaitVm4 : kWaitVm6);
                meet();
                Operands o[2];
                const uint4 q = raw.codes[tid];
                const int e = raw.exponents[tid];
#pragma unroll
                for (int f = 0; f < FM; ++f) read_x(o[0], x, 0, f);
#pragma unroll
                for (int f = 0; f < FN; ++f) read_y(o[0], y, 0, 0, f);
                request_raw(raw_free);
                request_y(y_free);
                const float scale = eight_scale(e);
                unsigned next[8];
                __builtin_amdgcn_sched_barrier(0);
                // each of the first products with some of the second's operands and of the next step's codes beside it
#pragma unroll
                for (int i = 0; i < FN * FM; ++i) {
                    multiply(o[0], i);
                    if (i < FM) read_x(o[1], x, 1, i);
                    else if (i < FM + FN) read_y(o[1], y, 0, 1, i - FM);
#pragma unroll
                    for (int k = 0; k < 8 / (FN * FM); ++k) next[i * (8 / (FN * FM)) + k] = convert(q, scale, i * (8 / (FN * FM)) + k);
                    __builtin_amdgcn_sched_barrier(0);
                }
                put_x(next, x_free);
#pragma unroll
                for (int i = 0; i < FN * FM; ++i) multiply(o[1], i);
                if (wants_bias && turn == share) {
                    add_bias(o[0]);
                    add_bias(o[1]);
                }
                turn = turn + 1 == shares ? 0 : turn + 1;
            };
            request_raw(raw0);
            request_raw(raw1);
            request_y(ys0);
            request_raw(raw2);
            request_y(ys1);
            __builtin_amdgcn_s_waitcnt(kWaitVm0);
            unsigned x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = convert(raw0.codes[tid], eight_scale(raw0.exponents[tid]), i);
            put_x(x, xs0);
            for (int s = 0; s < steps; s += 6) {
                step(ys0, ys2, xs0, xs1, raw1, raw0);
                if (s + 1 >= steps) break;
                step(ys1, ys0, xs1, xs0, raw2, raw1);
                if (s + 2 >= steps) break;
                step(ys2, ys1, xs0, xs1, raw0, raw2);
                if (s + 3 >= steps) break;
                step(ys0, ys2, xs1, xs0, raw1, raw0);
                if (s + 4 >= steps) break;
                step(ys1, ys0, xs0, xs1, raw2, raw1);
                if (s + 5 >= steps) break;
                step(ys2, ys1, xs1, xs0, raw0, raw2);
            }
            __builtin_amdgcn_s_waitcnt(kWaitVm0);   // what was requested for steps that are not there
        } else {
            // rows are requested two steps before they are written to LDS, and three before they are multiplied
            Rows va, vb;
            auto step = [&](int s, Rows& v, Y& y, Y& y_free, X& x, X& x_free) {
                const int at = first + s * kStepRows;
                meet();
                put(v, at + kStepRows, y_free, x_free);
                request(v, at + 3 * kStepRows);
                const bool sums = wants_bias && turn == share;
#pragma unroll
                for (int k = 0; k < kStepRows / 16; ++k) {
                    Operands o;
#pragma unroll
                    for (int f = 0; f < FM; ++f) read_x(o, x, k, f);
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                        for (int f = 0; f < FN; ++f) read_y(o, y, p, k, f);
#pragma unroll
                        for (int i = 0; i < FN * FM; ++i) multiply(o, i);
                        if (sums) add_bias(o);
                    }
                }
                turn = turn + 1 == shares ? 0 : turn + 1;
            };
            request(va, first);
            request(vb, first + kStepRows);
            put(va, first, ys0, xs0);
            request(va, first + 2 * kStepRows);
            for (int s = 0; s < steps; s += 2) {
                step(s, vb, ys0, ys1, xs0, xs1);
                if (s + 1 >= steps) break;
                step(s + 1, va, ys1, ys0, xs1, xs0);
            }
        }
        if (end == slice_end) break;
        // the next span: the pipeline starts anew, the sums go on
        first = end;
        end = first + min(slice_end - first, span_rows);
        y_rows = rows_between(dY, first, end, (size_t)N * sizeof(T));
        x_rows = rows_between(codes, first, end, (size_t)pitch);
        e_rows = rows_between(exponents, first, end, (size_t)(pitch / kGroup));
        meet();   // what the span before has in LDS is read
    }

    // lane l has m = .. + l % 32 of rows n = .. + 8 (i / 4) + 4 (l / 32) + i % 4: whole lines
#pragma unroll
    for (int b = 0; b < FM; ++b) {
        const int m = m0 + (wave_m * FM + b) * 32 + (lane & 31);
        const float column = weight && m < M ? (float)weight[m] : 1.f;
#pragma unroll
        for (int a = 0; a < FN; ++a)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = n0 + (wave_n * FN + a) * 32 + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
                if (n >= N) continue;
                if (partial) {
                    if (m < pitch) partial[((size_t)slice * N + n) * pitch + m] = acc[a][b][i];
                } else if (m < M) {
                    dW[(size_t)n * M + m] = (T)(acc[a][b][i] * column);
                }
            }
    }
    if (!wants_bias) return;
#pragma unroll
    for (int a = 0; a < FN; ++a) {
        const float v = bias[a] + __shfl_xor(bias[a], 32);
        const int n = n0 + (wave_n * FN + a) * 32 + (lane & 31);
        if (lane < 32 && n < N) bias_partial[((size_t)slice * shares + share) * N + n] = v;
    }
}

// COLUMNS vectors of 4 outputs of dW a workgroup, each by 256 / COLUMNS threads that have a run of slices; their sums are added in order.
// The last workgroups have 16 outputs of db each.
template <typename T, int COLUMNS>
__global__ __launch_bounds__(256) void weight_grad_eight_sum_kernel(const float* __restrict__ partial, const float* __restrict__ bias_partial, int slices,
                                                                    int bias_slices, int N, int M, const T* __restrict__ weight, T* __restrict__ dW,
                                                                    T* __restrict__ db, unsigned groups) {
    constexpr int RUNS = 256 / COLUMNS, BIAS_COLUMNS = 16, BIAS_RUNS = 256 / BIAS_COLUMNS, kInFlight = 8;
    __shared__ union {
        f32x4 part[RUNS][COLUMNS];
        float bias[BIAS_RUNS][BIAS_COLUMNS];
    } shared;
    if (blockIdx.x >= groups) {
        const int column = threadIdx.x % BIAS_COLUMNS, run = threadIdx.x / BIAS_COLUMNS, n = (int)(blockIdx.x - groups) * BIAS_COLUMNS + column;
        const int begin = (int)((long long)run * bias_slices / BIAS_RUNS), end = (int)((long long)(run + 1) * bias_slices / BIAS_RUNS);
        float sum = 0.f;
        for (int s = begin; s < end; s += kInFlight) {
            float v[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) v[u] = bias_partial[(size_t)min(s + u, end - 1) * N + min(n, N - 1)];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) sum += s + u < end ? v[u] : 0.f;
        }
        shared.bias[run][column] = sum;
        __syncthreads();
        if (run != 0 || n >= N) return;
#pragma unroll
        for (int k = 1; k < BIAS_RUNS; ++k) sum += shared.bias[k][column];
        db[n] = (T)sum;
        return;
    }
    const int column = threadIdx.x % COLUMNS, run = threadIdx.x / COLUMNS, pitch = (int)eight_pitch(M);
    const size_t n4 = (size_t)N * (pitch / 4), i = (size_t)blockIdx.x * COLUMNS + column;
    const int begin = (int)((long long)run * slices / RUNS), end = (int)((long long)(run + 1) * slices / RUNS);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const f32x4* const p = reinterpret_cast<const f32x4*>(partial) + (i < n4 ? i : n4 - 1);
    for (int s = begin; s < end; s += kInFlight) {
        f32x4 v[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) v[u] = p[(size_t)min(s + u, end - 1) * n4];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u)
            if (s + u < end) acc += v[u];
    }
    if constexpr (RUNS > 1) {
        shared.part[run][column] = acc;
        __syncthreads();
        if (run != 0) return;
#pragma unroll
        for (int k = 1; k < RUNS; ++k) acc += shared.part[k][column];
    }
    if (i >= n4) return;
    const size_t n = i / (pitch / 4);
    const int m = (int)(i - n * (pitch / 4)) * 4;
    if (weight) {
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] *= (float)weight[min(m + k, M - 1)];
    }
    T* const out = dW + n * M + m;
    if (m + 4 <= M && M % 4 == 0 && (uintptr_t)dW % (4 * sizeof(T)) == 0) {
        store_quad<T>(out, acc);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (m + k < M) out[k] = (T)acc[k];
    }
}

// The input's gradient where it is small: dX [rows, M] = dY [rows, N] W [N, M], fp32 sums.  A workgroup has 32 x 32 outputs, its waves an eighth of the sum each, operands
// straight from the L2s, a run of summands requested while the one before is multiplied.  The waves then add the eighths, in order, of two rows a half each.
//
// Where: a tile a compute unit at most, and sums of up to 2048.  The library's product then has 5 - 10 us on the GPU (fp32 and bf16, 255 x 512 x 512 6.7 and 6.9, 1024 x 768 x 256 7.7
// and 6.9; at some sizes far more, 255 x 576 x 192 104 and 20, 130 x 640 x 128 49 and 11) and 18 on the host, this kernel 7 - 16 in fp32 and 5 - 10 in bf16 (7.4 and 5.2, 11.6
// and 6.8; 10.4 and 6.7, 10.8 and 7.5) and 3 on the host, which sets the pace of such steps.  Beyond, the library's tiles win: 2000 x 1536 x 512 28 and 11, here 61 and 32.
constexpr int kInputTile = 32, kInputWaves = 8, kInputTiles = 256, kInputSummands = 2048;

template <typename T>
__global__ __launch_bounds__(64 * kInputWaves) void input_grad_kernel(const T* __restrict__ dY, const T* __restrict__ W, T* __restrict__ dX, int rows, int N, int M,
                                                                      int tiles_m) {
    constexpr int EACH = sizeof(T) == 2 ? 8 : 4, PIECE = 2 * EACH, PIECES = 32 / PIECE;   // summands of a lane, of a piece; pieces of a run of 32
    __shared__ float part[kInputWaves][16][64];
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = (int)(blockIdx.x / tiles_m) * kInputTile, col0 = (int)(blockIdx.x % tiles_m) * kInputTile, col = min(col0 + (lane & 31), M - 1);
    const int pieces = (N + PIECE - 1) / PIECE, begin = wave * pieces / kInputWaves * PIECE, end = min(N, (wave + 1) * pieces / kInputWaves * PIECE);
    const T *const a_row = dY + (size_t)min(row0 + (lane & 31), rows - 1) * N, *const b_column = W + col;
    struct __attribute__((packed)) Each {
        T v[EACH];
    };
    // A lane has EACH summands in a row of a piece, the other half of the wave the next: as both operands have them so, which ones an instruction takes does not matter.
    struct Run {
        T a[PIECES][EACH], b[PIECES][EACH];
    };
    auto fetch = [&](Run& r, int at) {
        if (at + 32 <= end) {   // uniform
#pragma unroll
            for (int u = 0; u < PIECES; ++u) {
                const int k = at + PIECE * u + EACH * half;
                const Each q = *reinterpret_cast<const Each*>(a_row + k);
#pragma unroll
                for (int j = 0; j < EACH; ++j) r.a[u][j] = q.v[j];
#pragma unroll
                for (int j = 0; j < EACH; ++j) r.b[u][j] = b_column[(size_t)(k + j) * M];
            }
        } else {
#pragma unroll
            for (int u = 0; u < PIECES; ++u)
#pragma unroll
                for (int j = 0; j < EACH; ++j) {
                    const int k = at + PIECE * u + EACH * half + j;
                    r.a[u][j] = k < end ? a_row[k] : (T)0.f;
                    r.b[u][j] = k < end ? b_column[(size_t)k * M] : (T)0.f;
                }
        }
    };
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    auto multiply = [&](const Run& r) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            if constexpr (sizeof(T) == 2) {
                bf16x8 a, b;
#pragma unroll
                for (int j = 0; j < EACH; ++j) a[j] = r.a[u][j], b[j] = r.b[u][j];
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < EACH; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(r.a[u][j], r.b[u][j], acc, 0, 0, 0);
            }
        }
    };
    Run x, y;
    fetch(x, begin);
    for (int at = begin; at < end; at += 64) {
        fetch(y, at + 32);
        multiply(x);
        fetch(x, at + 64);
        multiply(y);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 16 / kInputWaves; ++n) {
        const int i = 16 / kInputWaves * wave + n, row = row0 + 8 * (i / 4) + 4 * half + i % 4;
        float v = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < kInputWaves; ++w) v += part[w][i][lane];
        if (row < rows && col0 + (lane & 31) < M) dX[(size_t)row * M + col] = (T)v;
    }
}

// Slices of at least so many rows, and workgroups to aim at: two on a compute unit, or one where bf16 slices would have fewer than 512 rows, whose partial sums take
// longer than what more of them save (256 and 512: 4096 x 512 x 512 22.3 and 25.5 us, 65536 x 128 x 128 20 and 24, 65536 x 512 x 512 68 and 61; fp32, 8192 x 1536 x 512,
// 74 and 60).
constexpr int kMinRows = 128, kGroups = 512, kFewRows = 512;
// Outputs from which tiles are 256 wide (at 2^18 and 2^20: 16384 x 768 x 768 47.5 and 42.5 us, 65536 x 512 x 512 72 and 61, 32768 x 1536 x 512 89 and 100; fp32 4096 x 1024 x 512
// 38 and 33, 16384 x 768 x 768 74 and 77).
constexpr long long kBigOutputs = 1 << 20;
constexpr int kBigRows = 2048;

struct Plan {
    int side_n = 128, side_m = 128;   // of a tile
    int tiles_n, tiles_m, slices, slice_rows, span_rows, shares;
    size_t bias_at, total;   // bytes
    Plan(int rows, int N, int M, bool is_bf16, bool whole) {
        const long long pitch = eight_pitch(M);
        const long long outputs = (long long)N * pitch;
        if (outputs >= kBigOutputs && rows >= kBigRows && (whole || !is_bf16)) {
            side_n = 256;
            side_m = is_bf16 ? 128 : 256;
        }
        tiles_n = (N + side_n - 1) / side_n;
        tiles_m = (int)((pitch + side_m - 1) / side_m);
        const long long tiles = (long long)tiles_n * tiles_m, most = ((long long)rows + kMinRows - 1) / kMinRows;
        long long groups = side_m == 256 ? kGroups / 2 : kGroups;
        if (is_bf16 && side_n == 128 && rows * tiles < (long long)kFewRows * kGroups) groups = kGroups / 2;
        slices = (int)std::max<long long>(1, std::min(groups / tiles, most));
        slice_rows = (int)((((long long)rows + slices - 1) / slices + kStepRows - 1) / kStepRows * kStepRows);
        // 31 bits of offset, three steps beyond the last one's too
        span_rows = (int)std::min<long long>(slice_rows, (0x7fffffffll / std::max<long long>((is_bf16 ? 2ll : 4ll) * N, pitch) - 4 * kStepRows) / kStepRows * kStepRows);
        slices = (int)(((long long)rows + slice_rows - 1) / slice_rows);
        shares = tiles_m * 2;
        bias_at = slices > 1 ? (size_t)slices * outputs * sizeof(float) : 0;
        total = bias_at + (size_t)slices * shares * N * sizeof(float);
    }
};

}  // namespace

size_t weight_grad_eight_workspace_bytes(int rows, int N, int M) {
    return std::max({Plan(rows, N, M, false, true).total, Plan(rows, N, M, true, true).total, Plan(rows, N, M, true, false).total});
}

template <typename T>
static hipError_t launch_t(const WeightGradEight& a, hipStream_t st) {
    constexpr bool is_bf16 = sizeof(T) == 2;
    const bool whole = a.N % 8 == 0 && (uintptr_t)a.dY % 16 == 0;
    const Plan p(a.rows, a.N, a.M, is_bf16, whole);
    if ((long long)p.slices * p.tiles_n * p.tiles_m > 0x7fffffffll) return hipErrorInvalidValue;
    float *const partial = p.slices > 1 ? static_cast<float*>(a.workspace) : nullptr,
                 *const bias_partial = a.db ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + p.bias_at) : nullptr;
    T *const dW = static_cast<T*>(a.dW), *const db = static_cast<T*>(a.db);
    const T* const weight = static_cast<const T*>(a.weight);
    const unsigned groups = (unsigned)p.slices * (unsigned)p.tiles_n * (unsigned)p.tiles_m;
    auto launch = [&](auto kernel, int threads) {
        kernel<<<dim3(groups), dim3(threads), 0, st>>>(static_cast<const T*>(a.dY), a.codes, a.exponents, weight, dW, partial, bias_partial, a.rows, a.N,
                                                       a.M, p.slices, p.slice_rows, p.span_rows, p.tiles_n, p.tiles_m);
    };
    typedef std::conditional_t<is_bf16, Wide, Large> Big;
    if (p.side_n == 256 && whole) launch(weight_grad_eight_kernel<T, Big, true>, Big::threads);
    else if (p.side_n == 256) launch(weight_grad_eight_kernel<T, std::conditional_t<is_bf16, Small, Big>, false>, Big::threads);   // (fp32 only)
    else whole ? launch(weight_grad_eight_kernel<T, Small, true>, Small::threads) : launch(weight_grad_eight_kernel<T, Small, false>, Small::threads);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!partial && !a.db)) return e;
    const size_t quads = partial ? (size_t)a.N * (eight_pitch(a.M) / 4) : 0;
    auto sum = [&](auto columns) {
        constexpr int C = decltype(columns)::value;
        const unsigned sums = (unsigned)((quads + C - 1) / C), more = a.db ? (unsigned)((a.N + 15) / 16) : 0u;
        weight_grad_eight_sum_kernel<T, C><<<dim3(sums + more), dim3(256), 0, st>>>(partial, bias_partial, p.slices, p.slices * p.shares, a.N, a.M, weight, dW, db,
                                                                                    sums);
    };
    if (p.slices >= 64) sum(std::integral_constant<int, 8>{});
    else if (p.slices >= 16) sum(std::integral_constant<int, 32>{});
    else sum(std::integral_constant<int, 128>{});
    return hipGetLastError();
}
hipError_t launch_weight_grad_eight(const WeightGradEight& a, bool is_bf16, hipStream_t st) { return is_bf16 ? launch_t<bf16_t>(a, st) : launch_t<float>(a, st); }

static long long input_tiles(int n) { return (n + (long long)kInputTile - 1) / kInputTile; }
bool input_grad_suits(int rows, int N, int M) { return rows >= 1 && N <= kInputSummands && input_tiles(rows) * input_tiles(M) <= kInputTiles; }

hipError_t launch_input_grad(const void* dY, const void* W, void* dX, int rows, int N, int M, bool is_bf16, hipStream_t st) {
    const long long tiles_m = input_tiles(M), tiles = input_tiles(rows) * tiles_m;
    if (tiles > 0x7fffffffll) return hipErrorInvalidValue;
    auto launch = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)tiles), dim3(64 * kInputWaves), 0, st>>>(static_cast<const T*>(dY), static_cast<const T*>(W), static_cast<T*>(dX), rows, N, M, (int)tiles_m);
    };
    if (is_bf16) launch(input_grad_kernel<bf16_t>, bf16_t{});
    else launch(input_grad_kernel<float>, float{});
    return hipGetLastError();
}

}  // namespace spion
