// Tiles straight from global memory into registers and what is done with them: shared by the kernels whose waves walk 16-row
// tiles on their own (fp32 with every block size, bf16 with block size 16).
#ifndef SPION_ATTN_REGISTER_TILES_H_
#define SPION_ATTN_REGISTER_TILES_H_

#include <hip/hip_runtime.h>

#include "attn_bf16_tiles.h"
#include "attn_common.h"

namespace spion {

namespace {

constexpr int kPatchLd = kD + 4;   // floats per row of the merge area: b128 accesses of 16 rows hit all banks evenly

// lane (r, g): elements g EPL .. of each d chunk of row r
template <typename T>
__device__ __forceinline__ void load_rows(typename Elem<T>::Frag (&f)[kD / Elem<T>::KC], const T* tile, int r, int g) {
#pragma unroll
    for (int c = 0; c < kD / Elem<T>::KC; ++c)
        f[c] = *reinterpret_cast<const typename Elem<T>::Frag*>(tile + r * kD + g * Elem<T>::EPL + c * Elem<T>::KC);
}
// lane (r, g): columns 4 r .. 4 r + 3 of rows 4 g + i
template <typename T>
__device__ __forceinline__ void load_cols(typename Elem<T>::Quad (&v)[4], const T* tile, int r, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = *reinterpret_cast<const typename Elem<T>::Quad*>(tile + 4 * g * kD + 4 * r + i * kD);
}
template <typename V, int N>
__device__ __forceinline__ void clear(V (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = V{};
}

// acc[e][M = m] += sum over the tiles' rows of tile[row][4 m + e] * x[row][owned]
template <int NQ, int KT>
__device__ __forceinline__ void mma_cols(f32x4 (&acc)[NQ][4], const f32x4 (&v)[KT][4], const f32x4 (&x)[NQ][KT]) {
#pragma unroll
    for (int j = 0; j < 4 * KT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < NQ; ++h)
                acc[h][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j / 4][j % 4][e], x[h][j / 4][j % 4], acc[h][e], 0, 0, 0);
}
template <int NQ>
__device__ __forceinline__ void mma_cols(f32x4 (&acc)[NQ][4], const bf16x4 (&v)[2][4], const bf16x4 (&x)[NQ][2]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bf16x8 a = {v[0][0][e], v[0][1][e], v[0][2][e], v[0][3][e], v[1][0][e], v[1][1][e], v[1][2][e], v[1][3][e]};
#pragma unroll
        for (int h = 0; h < NQ; ++h) acc[h][e] = mma_d(acc[h][e], a, join(x[h][0], x[h][1]));
    }
}

template <int NQ>
__device__ __forceinline__ void clear_acc(f32x4 (&acc)[NQ][4]) {
#pragma unroll
    for (int h = 0; h < NQ; ++h) clear(acc[h]);
}

// A wave's accumulators into its part of the merge area (row-major, fp32).
template <int NQ>
__device__ __forceinline__ void put_patch(float* patch, const f32x4 (&acc)[NQ][4], int r, int g) {
#pragma unroll
    for (int h = 0; h < NQ; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<f32x4*>(patch + (h * 16 + r) * kPatchLd + 16 * g + 4 * i) =
                f32x4{acc[h][0][i], acc[h][1][i], acc[h][2][i], acc[h][3][i]};
}

// The same values as rows of the output, when no other wave holds a share of them.
template <typename T>
__device__ __forceinline__ void store_acc(T* row, const f32x4 (&acc)[4], float f, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) store_quad<T>(row + 16 * g + 4 * i, f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]} * f);
}

// Block j of the list, lists of up to 64 blocks from the lanes of `head64` (no scalar load in the loop).
__device__ __forceinline__ int list_at(const int* list, int head64, int j) {
    return j < 64 ? __builtin_amdgcn_readlane(head64, j) : list[j];
}

// Work of a group of n items, dealt to the XCDs in contiguous eighths: items of one head share an L2.  The
// group takes 8 * ceil(n / 8) workgroups from a multiple of 8 on; -1: a workgroup past the end.
__device__ __forceinline__ int item_of_group(int id, int n) {
    const int item = (id & 7) * ((n + 7) >> 3) + (id >> 3);
    return item < n ? item : -1;
}
inline long long group_grid(long long n) { return (n + 7) / 8 * 8; }

// The block row that workgroup number l (all of a row's beside each other) takes when there are more than run at once.
// Heads that do not divide over the XCDs: the rows with more than twice the mean number of kept blocks first, of all the heads (a
// row of 80 blocks that starts last runs alone for as long as everything before it took), then head by
// head the others, so that neighbours in time share K and V in an L2; each of the two lists is shared out over the XCDs head by head.
// Patterns without a long row skip the second search, and the counts are loaded four groups at a time.  By length, on the XCDs
// as deal_heads() has them, which the bf16 kernels gain by, took as long: 96 shapes, forward 0.95 to 1.04 of the time, backward 0.95 to 1.11.
// All lanes of the calling wave must be active.
__device__ __forceinline__ ItemOfHead long_rows_first(const int* __restrict__ row_ptr, int nb, int heads, int l, int lane) {
    const int limit = 2 * row_ptr[nb] / nb;
    int n_long = 0, cnt_first = 0;   // rows 0 .. 63 are kept for the second search
    int base0 = 0;
    for (; base0 + 256 <= nb; base0 += 256) {   // four groups whose loads are in flight together
        int from[4], to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            from[k] = row_ptr[base0 + 64 * k + lane];
            to[k] = row_ptr[base0 + 64 * k + lane + 1];
        }
        if (base0 == 0) cnt_first = to[0] - from[0];
#pragma unroll
        for (int k = 0; k < 4; ++k) n_long += __popcll(__ballot(to[k] - from[k] > limit));
    }
    for (int base = base0; base < nb; base += 64) {
        const int r = base + lane;
        const int cnt = r < nb ? row_ptr[r + 1] - row_ptr[r] : 0;
        if (base == 0) cnt_first = cnt;
        n_long += __popcll(__ballot(r < nb && cnt > limit));
    }
    const int longs = heads * n_long;
    const bool want_long = l < longs;
    int head, rank;
    if (want_long) {
        l = xcd_deal(l, 0, longs);
        head = l / n_long;
        rank = l % n_long;
    } else {
        l = xcd_deal(l, longs, heads * nb);
        head = l / (nb - n_long);
        rank = l % (nb - n_long);
    }
    if (n_long == 0) return {head, rank};
    for (int base = 0; base < nb; base += 64) {   // the counts are in the cache by now
        const int r = base + lane;
        int cnt = cnt_first;
        if (base != 0) cnt = r < nb ? row_ptr[r + 1] - row_ptr[r] : 0;
        const unsigned long long mine = __ballot(r < nb && (cnt > limit) == want_long);
        const int members = __popcll(mine);
        if (rank < members) {
            const unsigned long long hit = __ballot(((mine >> lane) & 1ull) && lanes_below(mine) == rank);
            return {head, base + __ffsll((long long)hit) - 1};
        }
        rank -= members;
    }
    return {head, 0};
}

// By length, all heads of an XCD together, where each XCD has whole heads: what starts last is short then.  Forward, long rows
// first and so: fp32, block 16, 16 x 2048 23.5 -> 22.5.
__device__ __forceinline__ ItemOfHead rows_in_order(const int* __restrict__ row_ptr, int nb, int heads, int l, int lane) {
    if (heads & 7) return long_rows_first(row_ptr, nb, heads, l, lane);
    const ItemOfHead mine = deal_heads(l, heads, false);
    return {mine.head, row_by_length(row_ptr, nb, mine.item, lane)};
}

}  // namespace

}  // namespace spion
#endif
