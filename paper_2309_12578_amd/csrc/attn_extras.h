// What the attention kernels with a relative position bias, dropout and sequence lengths have in common.
//
// Bias: score(q, k) += T[bucket_of[k - q + L - 1]][head].  The kernels add it as the value an MFMA accumulator starts from,
// divided by the score scale, so that it costs no instruction beside its reading.
//
// Dropout: Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011: the
// fewest that pass BigCrush).  Query q and key k of head bh have half q % 2 of word k % 4 of the call with counter
// ((q / 2) 2^14 + k / 4, bh + 2^31, offset, stream) and key seed: 16 bits, so that p is taken in steps of 2^-16.  The
// mask depends on the element's place alone, not on which kernel, side or block size computes it, and is never stored.
// A call serves two queries by four keys: the lanes of a query-side tile (one query, four keys each) share it in pairs, those
// of a key-side tile (one key, four queries each) in fours.
#ifndef SPION_ATTN_EXTRAS_H_
#define SPION_ATTN_EXTRAS_H_

#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "attn_common.h"
#include "philox.h"
#include "spion_internal.h"

namespace spion {

constexpr int kNoSlice = INT_MIN;       // in place of a slice's distance: nothing was computed
constexpr float kMaskedBias = -1e30f;   // a bias from here down masks, as -infinity does

__device__ __forceinline__ int length_of(const Extras& x, int bh, int L) {
    if (!x.lengths) return L;
    const int n = x.lengths[bh / x.H];
    return n < 0 ? 0 : n > L ? L : n;
}

// Where rows of head bh are, see HeadRows.
struct Rows {
    int H, beside;
    __device__ __forceinline__ int in_row() const { return beside ? 3 * H * kD : kD; }
    __device__ __forceinline__ int out_row() const { return beside ? H * kD : kD; }
    __device__ __forceinline__ size_t in_head(int bh, int L) const {
        return beside ? ((size_t)(bh / H) * L * 3 * H + bh % H) * kD : (size_t)bh * L * kD;
    }
    __device__ __forceinline__ size_t out_head(int bh, int L) const {
        return beside ? ((size_t)(bh / H) * L * H + bh % H) * kD : (size_t)bh * L * kD;
    }
};

// What is lost of v when it is stored as T.
template <typename T>
__device__ __forceinline__ float rounded_off(float v) { return v - (float)(T)v; }

// The head's column of the table into LDS, as what the accumulators start from; all threads of the workgroup, which has to
// meet before it is read.  Entries of the map beyond the table read its last bucket (the table is never read past its end).
__device__ __forceinline__ void load_bias_table(float* tab, const Extras& x, int h, int tid, int threads) {
    for (int b = tid; b < x.n_buckets; b += threads) {
        const size_t at = (size_t)b * x.H + h;
        const float v = x.table_bf16 ? (float)static_cast<const bf16_t*>(x.table)[at] : static_cast<const float*>(x.table)[at];
        tab[b] = v <= kMaskedBias ? -INFINITY : v * x.inv_scale;
    }
}
__device__ __forceinline__ int bucket_index(const Extras& x, unsigned b) { return (int)min(b, (unsigned)x.n_buckets - 1u); }

struct ScoreDraws {
    PhiloxKey key;
    unsigned bh;
    // `any`: whether there is dropout; without it rng may be a null pointer
    __device__ __forceinline__ ScoreDraws(bool any, const long long* rng, unsigned stream, int bh_)
        : key(any ? PhiloxKey(rng, stream) : PhiloxKey()), bh((unsigned)bh_ | 0x80000000u) {}
    // queries q, q ^ 1 and keys k .. k + 3 (k a multiple of 4)
    __device__ __forceinline__ uint4 call(int q, int k) const { return key.words((unsigned)(q >> 1) << 14 | (unsigned)k >> 2, bh); }
};

// Draws of query q and the keys k .. k + 3, one call a lane.
__device__ __forceinline__ void query_draws(const ScoreDraws& d, int q, int k, unsigned (&u)[4]) {
    const uint4 w = d.call(q, k);
    const int s = (q & 1) * 16;
    u[0] = w.x >> s & 0xffffu;
    u[1] = w.y >> s & 0xffffu;
    u[2] = w.z >> s & 0xffffu;
    u[3] = w.w >> s & 0xffffu;
}
// Draws of the queries q .. q + 3 (q a multiple of 4) and key k.
__device__ __forceinline__ void key_draws(const ScoreDraws& d, int q, int k, unsigned (&u)[4]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint4 w = d.call(q + 2 * e, k & ~3);
        const unsigned lo = (k & 1) ? w.y : w.x, hi = (k & 1) ? w.w : w.z, v = (k & 2) ? hi : lo;
        u[2 * e] = v & 0xffffu;
        u[2 * e + 1] = v >> 16;
    }
}

// Lane l's word of lane l ^ 1, and of l ^ 2.
__device__ __forceinline__ unsigned from_pair(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true); }
__device__ __forceinline__ unsigned from_other_pair(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true); }

// Factors 0 (dropped) and 1 of two draws; `below` = threshold - 1 in both halves (the threshold is not 0): min(draw - below,
// 1), the difference cut off at 0.  (Written with vector types, these become comparisons and selections of single halves, five
// instructions for what takes three here.)
__device__ __forceinline__ unsigned kept(unsigned draws, unsigned below) {
    unsigned f;
    asm("v_pk_sub_u16 %0, %1, %2 clamp" : "=v"(f) : "v"(draws), "s"(below));
    asm("v_pk_min_u16 %0, %1, 1 op_sel_hi:[1,0]" : "=v"(f) : "v"(f));
    return f;
}
__device__ __forceinline__ unsigned both_halves(unsigned v) { return v << 16 | (v & 0xffffu); }

// Probabilities with the dropped ones 0: their bit patterns times the factors, so that nothing is rounded.
__device__ __forceinline__ bf16x4 drop(bf16x4 p, const unsigned (&f)[2]) {
    typedef unsigned Words __attribute__((ext_vector_type(2)));
    const Words w = __builtin_bit_cast(Words, p);
    unsigned lo = w[0], hi = w[1];
    asm("v_pk_mul_lo_u16 %0, %1, %2" : "=v"(lo) : "v"(lo), "v"(f[0]));
    asm("v_pk_mul_lo_u16 %0, %1, %2" : "=v"(hi) : "v"(hi), "v"(f[1]));
    return __builtin_bit_cast(bf16x4, (Words){lo, hi});
}

// Query side: factors of this lane's query q = 16-row tile + r and the keys k0 + 16 kt + 4 g + i, two to a word, NKT even.  A call
// has two queries' draws: lane r makes those of tile kt = 2 j + r % 2 for itself and its neighbour r ^ 1, which makes the other tile's.
template <int NKT>
__device__ __forceinline__ void query_factors(const ScoreDraws& d, int q, int k0, int g, unsigned below, unsigned (&f)[NKT][2]) {
    const bool odd = q & 1;
    const unsigned mine = odd ? 0x07060302u : 0x05040100u, other = odd ? 0x05040100u : 0x07060302u;   // high or low halves of two words
#pragma unroll
    for (int j = 0; j < NKT / 2; ++j) {
        const uint4 w = d.call(q, k0 + 16 * (2 * j + (q & 1)) + 4 * g);
        const unsigned a0 = __builtin_amdgcn_perm(w.y, w.x, mine), a1 = __builtin_amdgcn_perm(w.w, w.z, mine);
        const unsigned b0 = from_pair(__builtin_amdgcn_perm(w.y, w.x, other)), b1 = from_pair(__builtin_amdgcn_perm(w.w, w.z, other));
        f[2 * j][0] = kept(odd ? b0 : a0, below);
        f[2 * j][1] = kept(odd ? b1 : a1, below);
        f[2 * j + 1][0] = kept(odd ? a0 : b0, below);
        f[2 * j + 1][1] = kept(odd ? a1 : b1, below);
    }
}

// Key side: draws of this lane's key k = 16-row tile + r and the queries q0 + 16 h + 4 g + i, h < 2: words [2 h] have i = 0, 1,
// [2 h + 1] i = 2, 3.  Four calls serve the four keys of lanes 4 a .. 4 a + 3: lane r makes number r % 4 and gets word r % 4 of
// each of the four (a 4 x 4 transpose in two steps).
__device__ __forceinline__ void key_words(const ScoreDraws& d, int q0, int k, int g, unsigned (&u)[4]) {
    const int c = k & 3;
    const uint4 w = d.call(q0 + 16 * (c >> 1) + 4 * g + 2 * (c & 1), k & ~3);
    const bool b0 = c & 1, b1 = c & 2;
    // every lane takes part in every exchange, whichever of the two it then keeps
    const unsigned px = from_pair(w.x), py = from_pair(w.y), pz = from_pair(w.z), pw = from_pair(w.w);
    const unsigned x0 = b0 ? py : w.x, x1 = b0 ? w.y : px, x2 = b0 ? pw : w.z, x3 = b0 ? w.w : pz;
    const unsigned o0 = from_other_pair(x0), o1 = from_other_pair(x1), o2 = from_other_pair(x2), o3 = from_other_pair(x3);
    u[0] = b1 ? o2 : x0;
    u[2] = b1 ? x2 : o0;
    u[1] = b1 ? o3 : x1;
    u[3] = b1 ? x3 : o1;
}

// ------------------------------------------------------------------------------------------------
// Sums over the diagonals (equal key - query) of dS tiles.  Lane (r, g) holds dS of query r and keys 16 kt + 4 g + i, i.e. of
// distance d = 16 kt + 4 g + i - r.  Element i moved i lanes down the row of 16 lies in the lane p = r - i of distance 16 kt + 4 g - p
// whatever i; those that leave the row at its lower end come in again at its upper one, one tile of 16 keys further on.
// Six additions with a lane shift for each tile of 16 keys leave u[0 .. NKT], of distance 16 kt + 4 g - p.
// ------------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float row_moved(float v) {   // 0 from beyond the row of 16 lanes
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int NKT>
__device__ __forceinline__ void diagonal_sums(const f32x4 (&ds)[NKT], float (&u)[NKT + 1]) {
    float carry = 0.f;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
        const f32x4 x = ds[kt];
        u[kt] = carry + (x[0] + row_moved<0x101>(x[1]) + row_moved<0x102>(x[2]) + row_moved<0x103>(x[3]));   // row_shl:1, 2, 3
        carry = row_moved<0x11f>(x[1]) + row_moved<0x11e>(x[2]) + row_moved<0x11d>(x[3]);                    // row_shr:15, 14, 13
    }
    u[NKT] = carry;
}

// The kernel's arguments once more, from memory: what is used at its end only would otherwise sit in scalar registers over the
// loop, of which there are too few (7 to 61 of them were spilled).
template <typename Args>
__device__ __forceinline__ const __attribute__((address_space(4))) Args& args_again() {
    auto p = reinterpret_cast<const __attribute__((address_space(4))) Args*>(reinterpret_cast<uintptr_t>(__builtin_amdgcn_kernarg_segment_ptr()));
    asm volatile("" : "+s"(p));
    return *p;
}

}  // namespace spion
#endif
