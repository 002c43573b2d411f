// Block-sparse attention (Eq. 5 on the kept blocks) with what a Transformer adds inside the softmax: a learned relative
// position bias by buckets, dropout of the probabilities, sequences shorter than the batch's length.
//   S_qk = scale Q_q K_k + T[bucket(k - q)][head], P = softmax over the kept k < length, O = (c M . P) V, c = 1 / (1 - p)
//   delta = rowsum(dO . O), dP = c M . (dO V^T), dS = P . (dP - delta)
//   dV = (c M . P)^T dO, dQ = scale dS K, dK = scale dS^T Q, dT[b][head] = sum of dS over the elements of bucket b
// Queries and keys from the length on: O = 0, LSE = -inf, gradients 0; nothing of theirs is added up.
//
// The kernels of this file are for fp32 and block 16: a workgroup of four waves has 16 or 32 rows, whose 16-row tiles of the other
// side the waves take in turn, straight from memory into registers (layouts, order and pieces as in attn_kernels.hip).  Bound, as there, by the
// latency of those loads, and in fp32 by its MFMA rate.  Kernel time, us, of the plain ones, with lengths, bias, dropout, bias and dropout, forward and
// backward (row_terms_kernel takes 4.7, 6.5, 5.2 and 9.3 besides): fp32, 8 heads x 2048, block 32, 10 %, 20.2 / 21 / 22.3 / 22.5 / 23.8, 54 / 52.4 / 55.7 / 56.6 / 60.5; 16 x
// 4096, block 64, 10 %, 79 / 80 / 83 / 87 / 91, 280 / 265 / 280 / 282 / 298; bf16, block 16, 9 x 1936, 8 %, 12.7 / 15.2 / 16.3 / 15.9 / 17, 27 / 26.7 / 29 / 27.7 / 30.5; 32 x 4096
// 78 / 80 / 89 / 86 / 95, 296 / 261 / 278 / 271 / 290.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <climits>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "attn_extras.h"
#include "attn_key_items.h"
#include "attn_register_tiles.h"
#include "spion_internal.h"
#include "table_grad.h"

namespace spion {

namespace {

typedef unsigned u32_any __attribute__((aligned(1)));

// Entries of an ascending list whose block starts below `length`.
template <int BS>
__device__ __forceinline__ int blocks_below(const int* list, int n, int length, int lane) {
    int count = 0;
    for (int base = 0; base < n; base += 64) {
        const int here = __popcll(__ballot(base + lane < n && list[base + lane < n ? base + lane : n - 1] * BS < length));
        count += here;
        if (here < 64) break;
    }
    return count;
}

template <typename T>
__device__ __forceinline__ void zero_rows_from(typename Elem<T>::Frag (&f)[kD / Elem<T>::KC], bool zero) {
    if (zero) clear(f);
}
template <typename T>
__device__ __forceinline__ void zero_cols_from(typename Elem<T>::Quad (&v)[4], int row0, int length) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (row0 + i >= length) v[i] = typename Elem<T>::Quad{};
}

// A workgroup's 16 NQ rows, whose tiles its four waves share.
template <typename T, int BS, int NQ>
struct Tiles {
    static constexpr int KT = sizeof(T) == 2 ? 2 : 1;   // tiles per step: a bf16 MFMA contracts over 32 rows
    static constexpr int NDC = kD / Elem<T>::KC, TPB = BS / 16, OWN = 16 * NQ, PARTS = BS / OWN;
};

constexpr int kWaves = 4;

// The buckets of query q and the keys k .. k + 3 (or, KEYS, of key k and the queries q .. q + 3), and their biases / scale
template <bool KEYS>
__device__ __forceinline__ unsigned buckets_of(const Extras& x, int q, int k, int L) {
    return x.table ? (unsigned)*reinterpret_cast<const u32_any*>(x.bucket_of + (k - q - (KEYS ? 3 : 0) + L - 1)) : 0u;
}
template <bool KEYS>
__device__ __forceinline__ f32x4 bias_of(const Extras& x, const float* tab, unsigned b) {
    if (!x.table) return f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = tab[bucket_index(x, b >> (KEYS ? 24 - 8 * i : 8 * i) & 255u)];
    return v;
}

// The rows that a workgroup of the forward or of the query side has: of helpers (cut.groups, which come first) a piece of a long row, of the others a
// row's first piece or all of it, by length where sort_rows.  false: none.
template <int PARTS>
__device__ __forceinline__ bool row_of_group(const int* __restrict__ row_ptr, int nb, int BH, const RowCut& cut, int sort_rows, int id, int lane, int& bh,
                                             int& I, int& part, RowPieces& cuts, int& piece) {
    cuts = {0, 1, 0, 0};
    piece = 0;
    const int at = (id >> 3) / PARTS * 8 + (id & 7);   // a row's workgroups on one XCD
    part = (id >> 3) % PARTS;
    if (id < cut.groups) {
        const int want = at / BH;
        if (want >= cut.helpers) return false;
        cuts = row_pieces<false>(row_ptr, nb, cut, want, lane);
        if (cuts.row < 0) return false;
        bh = at % BH;
        I = cuts.row;
        piece = want - cuts.first + 1;
        return true;
    }
    if (sort_rows) {
        const int row = at - cut.groups / PARTS;   // (a multiple of 8)
        if (row >= BH * nb) return false;
        const ItemOfHead mine = rows_in_order(row_ptr, nb, BH, row, lane);
        bh = mine.head;
        I = mine.item;
        return true;
    }
    const int item = item_of_group(id - cut.groups, BH * nb * PARTS);
    if (item < 0) return false;
    bh = item / (nb * PARTS);
    I = item % (nb * PARTS) / PARTS;
    part = item % PARTS;
    return true;
}
// The piece of a row of more than cut.longest blocks from jb on: which blocks it has.
__device__ __forceinline__ void piece_of_row(const int* __restrict__ row_ptr, int nb, const RowCut& cut, int I, int lane, RowPieces& cuts, int piece, int& jb,
                                             int& n) {
    if (piece == 0) cuts = row_pieces<true>(row_ptr, nb, cut, I, lane);
    const int from = piece * n / cuts.count;
    n = (piece + 1) * n / cuts.count - from;
    jb += from;
}

}  // namespace

// ------------------------------------------------------------------------------------------------
// forward: workgroup = (head, Tiles::OWN query rows)
// ------------------------------------------------------------------------------------------------
template <typename T, int BS, int NQ, bool DROP>
__global__ __launch_bounds__(kWaves * 64, 2) void attn_fwd_with_kernel(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O, float* __restrict__ LSE,
    const int* __restrict__ row_ptr, const int* __restrict__ col_idx, Extras x, RowCut cut, int BH, int L, int nb, int sort_rows, float scale_log2) {
    typedef typename Elem<T>::Frag Frag;
    typedef typename Elem<T>::Quad Quad;
    typedef Tiles<T, BS, NQ> S;
    constexpr int KT = S::KT, NDC = S::NDC, STRIDE = kWaves * KT;
    __shared__ int flag;
    __shared__ __attribute__((aligned(16))) float o_s[kWaves][S::OWN * kPatchLd];
    __shared__ float m_s[kWaves][S::OWN], l_s[kWaves][S::OWN], tab[Extras::kMaxBuckets];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (DROP && blockIdx.x == 0 && tid < 2 && x.rng_used) x.rng_used[tid] = x.rng[tid];
    int bh, I, part, piece, id = blockIdx.x;
    RowPieces cuts;
    if (!row_of_group<S::PARTS>(row_ptr, nb, BH, cut, sort_rows, id, lane, bh, I, part, cuts, piece)) return;
    const int row0 = I * BS + part * S::OWN;
    const size_t head = (size_t)bh * L * kD;
    const int length = length_of(x, bh, L);
    if (x.table) load_bias_table(tab, x, bh % x.H, tid, kWaves * 64);
    __syncthreads();

    int jb = row_ptr[I], n = row_ptr[I + 1] - jb;
    if (n > cut.longest) piece_of_row(row_ptr, nb, cut, I, lane, cuts, piece, jb, n);
    const int* cols = col_idx + jb;
    n = row0 < length ? blocks_below<BS>(cols, n, length, lane) : 0;
    const int nt = n * S::TPB;
    const int cols64 = n > 0 ? cols[lane < n ? lane : n - 1] : 0;
    auto key0 = [&](int t) { return list_at(cols, cols64, t / S::TPB) * BS + t % S::TPB * 16; };
    Frag qf[NQ][NDC];
#pragma unroll
    for (int h = 0; h < NQ; ++h) {
        if (row0 + 16 * h + r < length) load_rows<T>(qf[h], Q + head + (size_t)(row0 + 16 * h) * kD, r, g);
        else clear(qf[h]);
    }
    [[maybe_unused]] ScoreDraws draws(DROP, x.rng, x.stream, bh);
    // K of tiles t, t + 1, .. and the buckets (past the end: tile t once more, which counts nothing)
    auto load_k = [&](Frag (&k)[KT][NDC], unsigned (&buckets)[NQ][KT], int t) {
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const int k0 = key0(t + u < nt ? t + u : t);
            load_rows<T>(k[u], K + head + (size_t)k0 * kD, r, g);
#pragma unroll
            for (int h = 0; h < NQ; ++h) buckets[h][u] = buckets_of<false>(x, row0 + 16 * h + r, k0 + 4 * g, L);
        }
    };

    float m[NQ], limit[NQ], lsum[NQ];
    f32x4 oacc[NQ][4];
    clear_acc<NQ>(oacc);
#pragma unroll
    for (int h = 0; h < NQ; ++h) {
        m[h] = kLowest;
        limit[h] = -INFINITY;
        lsum[h] = 0.f;
    }
    auto step = [&](Frag (&kf)[KT][NDC], const unsigned (&buckets)[NQ][KT], Frag (&knext)[KT][NDC], unsigned (&bnext)[NQ][KT], int t) {
        Quad vc[KT][4];
        f32x4 s[NQ][KT];
        int k0[KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            k0[u] = key0(t + u < nt ? t + u : t);
            load_cols<T>(vc[u], V + head + (size_t)k0[u] * kD, r, g);
        }
        if (t + STRIDE < nt) load_k(knext, bnext, t + STRIDE);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (k0[u] + 16 > length) {
                zero_rows_from<T>(kf[u], k0[u] + r >= length);
                zero_cols_from<T>(vc[u], k0[u] + 4 * g, length);
            }
            if (u > 0 && t + u >= nt) clear(vc[u]);
        }
        float mx[NQ];
        bool above = false;
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
            mx[h] = -INFINITY;
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                s[h][u] = bias_of<false>(x, tab, buckets[h][u]);
#pragma unroll
                for (int c = 0; c < NDC; ++c) s[h][u] = mma_d(s[h][u], kf[u][c], qf[h][c]);   // S^T: [key 4 g + i][query r]
                const bool there = u == 0 || t + u < nt;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!there || k0[u] + 4 * g + i >= length) s[h][u][i] = -INFINITY;
                    mx[h] = fmaxf(mx[h], s[h][u][i]);
                }
            }
            above |= mx[h] * scale_log2 > limit[h];
        }
        if (__any(above)) {
#pragma unroll
            for (int h = 0; h < NQ; ++h) {
                const float m_new = fmaxf(m[h], group_max(mx[h]) * scale_log2);
                const float alpha = exp2f(m[h] - m_new);
                m[h] = m_new;
                limit[h] = m_new + kRescaleSlack;
                lsum[h] *= alpha;
#pragma unroll
                for (int e = 0; e < 4; ++e) oacc[h][e] *= alpha;
            }
        }
        Quad pq[NQ][KT];
        [[maybe_unused]] Quad rest[NQ][KT];   // of bf16: what the rounding leaves, see attn_extras_bf16_kernels.hip
#pragma unroll
        for (int h = 0; h < NQ; ++h)
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                f32x4 p;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = exp2f(fmaf(s[h][u][i], scale_log2, -m[h]));
                    lsum[h] += p[i];
                }
                if constexpr (DROP) {
                    unsigned d[4];
                    query_draws(draws, row0 + 16 * h + r, k0[u] + 4 * g, d);
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = d[i] < x.threshold ? 0.f : p[i];
                }
                pq[h][u] = to_quad<T>(p);
                if constexpr (sizeof(T) == 2) rest[h][u] = to_quad<T>(f32x4{rounded_off<T>(p[0]), rounded_off<T>(p[1]), rounded_off<T>(p[2]), rounded_off<T>(p[3])});
            }
        mma_cols(oacc, vc, pq);   // O^T += V^T P^T
        if constexpr (sizeof(T) == 2) {
            if (x.table && x.rest) mma_cols(oacc, vc, rest);
        }
    };
    {
        Frag ka[KT][NDC], kb[KT][NDC];
        unsigned ba[NQ][KT], bb[NQ][KT];
        int t = wave * KT;
        if (t < nt) load_k(ka, ba, t);
        for (; t < nt; t += 2 * STRIDE) {
            step(ka, ba, kb, bb, t);
            if (t + STRIDE < nt) step(kb, bb, ka, ba, t + STRIDE);
        }
    }

    // the waves' shares of each row: rescaled to the row's largest m and added up in wave order
    put_patch<NQ>(&o_s[wave][0], oacc, r, g);
#pragma unroll
    for (int h = 0; h < NQ; ++h) {
        const float l = group_sum(lsum[h]);
        if (g == 0) {
            m_s[wave][16 * h + r] = m[h];
            l_s[wave][16 * h + r] = l;
        }
    }
    __syncthreads();
    auto merged = [&](int q, int d, float& mm, float& l) {
        mm = m_s[0][q];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, m_s[w][q]);
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float a = exp2f(m_s[w][q] - mm);
            l += l_s[w][q] * a;
            o += *reinterpret_cast<const f32x4*>(&o_s[w][q * kPatchLd + d]) * a;
        }
        return o;
    };
    // [head][slot][part]: the rows' numbers, then their references and sums
    constexpr int kPart = S::OWN * (kD + 2);
    const float* parts = nullptr;
    if (cuts.count > 1) {   // a long row in pieces, as in the plain kernel
        const size_t slot = ((size_t)bh * cut.slots + cuts.slot) * S::PARTS + part;
        float* const mine = cut.parts + slot * kPart + (size_t)piece * (S::PARTS * kPart);
        parts = cut.parts + slot * kPart;
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
            const int q = 16 * h + (tid >> 4), d = (tid & 15) * 4;
            float mm, l;
            const f32x4 o = merged(q, d, mm, l);
            put_shared(mine + q * kD + d, o[0], o[1]);
            put_shared(mine + q * kD + d + 2, o[2], o[3]);
            if (d == 0) put_shared(mine + S::OWN * kD + 2 * q, mm, l);
        }
        if (!last_to_arrive(cut.counters + slot, cut.tag, cuts.count, &flag)) return;
    }
#pragma unroll
    for (int h = 0; h < NQ; ++h) {
        const int q = 16 * h + (tid >> 4), d = (tid & 15) * 4;
        float mm, l;
        f32x4 o;
        if (parts) {   // (a reference is kLowest at least)
            mm = -INFINITY;
            l = 0.f;
            o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int c = 0; c < cuts.count; ++c) {
                const float* const p = parts + (size_t)c * (S::PARTS * kPart);
                const float2 lo = get_shared(p + q * kD + d), hi = get_shared(p + q * kD + d + 2);
                const float2 ml = get_shared(p + S::OWN * kD + 2 * q);
                const float m_new = fmaxf(mm, ml.x), a = exp2f(mm - m_new), b = exp2f(ml.x - m_new);
                mm = m_new;
                l = l * a + ml.y * b;
                o = o * a + f32x4{lo.x, lo.y, hi.x, hi.y} * b;
            }
        } else {
            o = merged(q, d, mm, l);
        }
        const bool empty = (!(l > 0.f) && l == l) || row0 + q >= length;
        o = empty ? f32x4{0.f, 0.f, 0.f, 0.f} : o * ((DROP ? x.keep_scale : 1.f) / l);
        store_quad<T>(O + head + (size_t)(row0 + q) * kD + d, o);
        if constexpr (sizeof(T) == 2) {
            if (x.rest)
                store_quad<T>(static_cast<T*>(x.rest) + head + (size_t)(row0 + q) * kD + d,
                              f32x4{rounded_off<T>(o[0]), rounded_off<T>(o[1]), rounded_off<T>(o[2]), rounded_off<T>(o[3])});
        }
        if (d == 0) LSE[(size_t)bh * L + row0 + q] = empty ? -INFINITY : (mm + log2f(l)) * kLn2;
    }
}

// The key side's work items, see attn_key_items.h.
struct ColumnCut {
    int chunk, n_first, n_items, n_slots, by_length;   // items per head that come before the rows, and all
    unsigned long long tag;
    unsigned long long* counters;   // one per slot and 16 rows
    float* parts;
};

// ------------------------------------------------------------------------------------------------
// Before the backward: the two numbers of a row that both of its sides need.  Exponentials are taken against log2(e) LSE - log2(c), so that they are
// c P, and delta = rowsum(dO . O) is left as -delta / c; a row that keeps nothing, or past the sequence's end, has no probabilities.  O is
// what the forward stored plus what its rounding left (x.rest): with bf16's rounding alone dQ and dK are off by a twentieth more and the table's
// gradient, over whose far buckets a row's error adds up, by 2.0e-3 to 3.9e-3 in place of 3e-6 to 5e-6 where two buckets have all but one key of a row (with P's
// rounding; 16 heads x 1024).  Bound by memory, 8 lanes a row.
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void row_terms_kernel(const T* __restrict__ O, const T* __restrict__ dO, const float* __restrict__ LSE, Extras x, int beside,
                                                        int L, long long rows, float delta_scale) {
    constexpr int VEC = 16 / sizeof(T), LANES = 8, PER = kD / LANES;
    typedef T Vec __attribute__((ext_vector_type(VEC)));
    if (blockIdx.x == 0 && x.counters)
        for (int h = threadIdx.x; h < x.H; h += 256) x.counters[h * Extras::kCounterStride] = 0ull;
    const long long row = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= rows) return;   // (all lanes of a row together)
    const int bh = (int)(row / L), i = (int)(row % L), part = threadIdx.x % LANES;
    const Rows at = {x.H, beside};
    float delta = 0.f, lse = -INFINITY;
    if (i < length_of(x, bh, L)) {
        const size_t from = at.out_head(bh, L) + (size_t)i * at.out_row() + part * PER;
        lse = LSE[row];
#pragma unroll
        for (int c = 0; c < PER; c += VEC) {
            const Vec o = *reinterpret_cast<const Vec*>(O + from + c), g = *reinterpret_cast<const Vec*>(dO + from + c);
            Vec rest = {};
            if (sizeof(T) == 2 && x.rest) rest = *reinterpret_cast<const Vec*>(static_cast<const T*>(x.rest) + from + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) delta = fmaf((float)g[e], (float)o[e] + (float)rest[e], delta);
        }
    }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) delta += __shfl_xor(delta, o);
    if (part == 0) {
        x.row_lse[row] = lse == -INFINITY ? INFINITY : fmaf(lse, kLog2e, -log2f(x.keep_scale));
        x.row_delta[row] = lse == -INFINITY ? 0.f : delta * delta_scale;
    }
}

// ------------------------------------------------------------------------------------------------
// backward: workgroup = (head, Tiles::OWN rows of a block row) on the query side, (head, as many keys of a block column) on the key side.
// The exponentials are c P, delta is divided by c to match (see row_terms_kernel).  The sides share no data; all sums in fixed order.  The query side leaves, for the table's gradient, the sums over the 31 diagonals of each
// 16 x 16 tile of dS in slices[head][kept block][query tile][key tile][32].
// ------------------------------------------------------------------------------------------------
template <typename T>
struct BwdOfRows {
    const T *Q, *K, *V, *dO;
    T *dQ, *dK, *dV;
    const int *row_ptr, *col_idx, *col_ptr, *row_idx;
    Extras x;
    RowCut cut;
    ColumnCut columns;
    int BH, L, nb, nnzb, sort_rows;
    float scale, scale_log2;
};

template <typename T, int BS, int NQ, int W, bool DROP>
__global__ __launch_bounds__(W * 64, 2) void attn_bwd_with_kernel(const BwdOfRows<T> a) {
    const T *__restrict__ const Q = a.Q, *__restrict__ const K = a.K, *__restrict__ const V = a.V, *__restrict__ const dO = a.dO;
    const Extras& x = a.x;
    const int L = a.L;
    const float scale_log2 = a.scale_log2;
    typedef typename Elem<T>::Frag Frag;
    typedef typename Elem<T>::Quad Quad;
    typedef Tiles<T, BS, NQ> S;
    constexpr int KT = S::KT, NDC = S::NDC, TPB = S::TPB, STRIDE = W * KT;
    constexpr int kDiag = 48;   // floats per lane group and wave: places of distance 16 kt + 4 g - p, behind each other
    __shared__ __attribute__((aligned(16))) float acc_s[W][S::OWN * kPatchLd];
    __shared__ float tab[Extras::kMaxBuckets], diag_s[W][4][kDiag];
    __shared__ int flag;

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowCut& cut = a.cut;
    const ColumnCut& columns = a.columns;
    const int BH = a.BH, nb = a.nb, sort_rows = a.sort_rows;
    const int *__restrict__ const row_ptr = a.row_ptr, *__restrict__ const col_ptr = a.col_ptr;
    // helpers, chunks of columns and long columns, rows, the other columns
    const int first = BH * columns.n_first * S::PARTS, first_groups = (first + 7) & ~7;
    const int row_groups = sort_rows ? S::PARTS * ((BH * nb + 7) & ~7) : (BH * nb * S::PARTS + 7) & ~7;
    int id = (int)blockIdx.x, bh, block, part, piece = 0;
    RowPieces cuts = {0, 1, 0, 0};
    KeyItem it = {0, 0, 0, -1, 0, 1};
    const bool key_side = id >= cut.groups && (id < cut.groups + first_groups || id >= cut.groups + first_groups + row_groups);
    if (key_side) {   // the items of all heads together, longest first; heads keep to an XCD where that shares them out evenly
        id -= cut.groups;
        int from = 0;
        if (id >= first_groups) {
            id -= first_groups + row_groups;
            from = columns.n_first;
        }
        int xcd = 0, heads = BH;
        if ((BH & 7) == 0) {
            xcd = id & 7;
            heads = BH >> 3;
            id >>= 3;
        }
        bh = xcd * heads + id % heads;
        part = id / heads % S::PARTS;
        const int idx = from + id / heads / S::PARTS;
        if (idx >= (from ? columns.n_items : columns.n_first)) return;
        it = key_item_lookup(col_ptr, nb, columns.chunk, columns.by_length, idx, lane);
        if (it.J < 0) return;
        block = it.J;
    } else {
        if (id >= cut.groups) id -= first_groups;
        if (!row_of_group<S::PARTS>(row_ptr, nb, BH, cut, sort_rows, id, lane, bh, block, part, cuts, piece)) return;
    }
    const int sub = part * NQ, row0 = block * BS + sub * 16;
    const size_t head = (size_t)bh * L * kD, vec = (size_t)bh * L;
    const int length = length_of(x, bh, L);
    if (x.table) load_bias_table(tab, x, bh % x.H, tid, W * 64);
    if (!key_side && x.slices)
        for (int i = tid; i < W * 4 * kDiag; i += W * 64) (&diag_s[0][0][0])[i] = 0.f;
    __syncthreads();
    [[maybe_unused]] ScoreDraws draws(DROP, x.rng, x.stream, bh);

    constexpr int kAtOnce = 4 * W;   // rows that all threads have together, 4 columns each
    auto merged = [&](int p) {       // rows p + tid / 16
        const int q = p + (tid >> 4), o = q * kPatchLd + (tid & 15) * 4;
        f32x4 v = *reinterpret_cast<const f32x4*>(&acc_s[0][o]);
#pragma unroll
        for (int w = 1; w < W; ++w) v += *reinterpret_cast<const f32x4*>(&acc_s[w][o]);
        return row0 + q < length ? v : f32x4{0.f, 0.f, 0.f, 0.f};
    };
    const int out = (sub * 16 + (tid >> 4)) * kD + (tid & 15) * 4;   // in the block
    int entry0 = key_side ? it.kb : row_ptr[block], n_list = key_side ? it.ke - it.kb : row_ptr[block + 1] - entry0;
    if (!key_side && n_list > cut.longest) piece_of_row(row_ptr, nb, cut, block, lane, cuts, piece, entry0, n_list);
    const int* list = (key_side ? a.row_idx : a.col_idx) + entry0;
    const int n = row0 < length ? blocks_below<BS>(list, n_list, length, lane) : 0;
    const int nt = n * TPB;
    const int list64 = n > 0 ? list[lane < n ? lane : n - 1] : 0;
    auto tile0 = [&](int t) { return list_at(list, list64, t / TPB) * BS + t % TPB * 16; };

    if (!key_side) {
        Frag qf[NQ][NDC], dof[NQ][NDC];
        float ndelta[NQ], lse2[NQ];
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
            const int row = row0 + 16 * h + r;
            const size_t at = head + (size_t)(row0 + 16 * h) * kD;
            if (row < length) {
                load_rows<T>(qf[h], Q + at, r, g);
                load_rows<T>(dof[h], dO + at, r, g);
            } else {
                clear(qf[h]);
                clear(dof[h]);
            }
            lse2[h] = x.row_lse[vec + row];
            ndelta[h] = x.row_delta[vec + row];
        }
        auto slice = [&](int entry, int h, int key_tile) {
            return a.x.slices + ((((size_t)bh * a.nnzb + entry0 + entry) * TPB + sub + h) * TPB + key_tile) * 32;
        };
        if (x.slices)   // what is not computed
            for (int e = n * TPB + tid; e < n_list * TPB; e += W * 64)
#pragma unroll
                for (int h = 0; h < NQ; ++h) slice(e / TPB, h, e % TPB)[31] = __builtin_bit_cast(float, kNoSlice);
        f32x4 dq[NQ][4];
        clear_acc<NQ>(dq);
        for (int t = wave * KT; t < nt; t += STRIDE) {
            Quad kc[KT][4], dsq[NQ][KT];
            Frag kf[KT][NDC], vf[KT][NDC];
            unsigned buckets[NQ][KT];
            int k0[KT];
#pragma unroll
            for (int u = 0; u < KT; ++u) {   // past the end: tile t once more, which counts nothing
                k0[u] = tile0(u == 0 || t + u < nt ? t + u : t);
                const size_t at = head + (size_t)k0[u] * kD;
                load_rows<T>(kf[u], K + at, r, g);
                load_rows<T>(vf[u], V + at, r, g);
                load_cols<T>(kc[u], K + at, r, g);
#pragma unroll
                for (int h = 0; h < NQ; ++h) buckets[h][u] = buckets_of<false>(x, row0 + 16 * h + r, k0[u] + 4 * g, L);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                const bool there = u == 0 || t + u < nt;
                if (k0[u] + 16 > length) {
                    zero_rows_from<T>(kf[u], k0[u] + r >= length);
                    zero_rows_from<T>(vf[u], k0[u] + r >= length);
                    zero_cols_from<T>(kc[u], k0[u] + 4 * g, length);
                }
                if (!there) clear(kc[u]);
#pragma unroll
                for (int h = 0; h < NQ; ++h) {
                    f32x4 s = bias_of<false>(x, tab, buckets[h][u]), dp = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < NDC; ++c) {
                        s = mma_d(s, kf[u][c], qf[h][c]);      // S^T = K Q^T
                        dp = mma_d(dp, vf[u][c], dof[h][c]);   // dP^T = V dO^T
                    }
                    unsigned d[4] = {};
                    if constexpr (DROP) query_draws(draws, row0 + 16 * h + r, k0[u] + 4 * g, d);
                    f32x4 ds;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool masked = !there || k0[u] + 4 * g + i >= length;
                        const float p = masked ? 0.f : exp2f(fmaf(s[i], scale_log2, -lse2[h]));
                        ds[i] = p * ((DROP && d[i] < x.threshold ? 0.f : dp[i]) + ndelta[h]);
                    }
                    dsq[h][u] = to_quad<T>(ds);
                    if (x.slices && there) {
                        const f32x4 one[1] = {ds};
                        float du[2];
                        diagonal_sums<1>(one, du);
                        diag_s[wave][g][4 * g - r + 15] = du[0];
                        diag_s[wave][g][4 * g - r + 31] = du[1];
                        __builtin_amdgcn_wave_barrier();
                        if (lane < 32) {
                            const float v = diag_s[wave][0][lane] + diag_s[wave][1][lane] + diag_s[wave][2][lane] + diag_s[wave][3][lane];
                            slice((t + u) / TPB, h, (t + u) % TPB)[lane] = lane < 31 ? v : __builtin_bit_cast(float, k0[u] - row0 - 16 * h);
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
                }
            }
            mma_cols(dq, kc, dsq);   // dQ^T += K^T dS^T
        }
        put_patch<NQ>(&acc_s[wave][0], dq, r, g);
        __syncthreads();
        const auto& z = args_again<BwdOfRows<T>>();
        const float scale = z.scale;
        T* const rows = z.dQ + head + (size_t)block * BS * kD + out;
        if (cuts.count > 1) {   // a long row in pieces
            const size_t slot = ((size_t)bh * z.cut.slots + cuts.slot) * S::PARTS + part;
            float* const parts = z.cut.parts + slot * (S::OWN * kD) + tid * 4;
            constexpr int kPiece = S::PARTS * S::OWN * kD;
#pragma unroll
            for (int p = 0; p < S::OWN; p += kAtOnce) {
                const f32x4 v = merged(p);
                float* const mine = parts + (size_t)piece * kPiece + p * kD;
                put_shared(mine, v[0], v[1]);
                put_shared(mine + 2, v[2], v[3]);
            }
            if (!last_to_arrive(z.cut.counters + slot, z.cut.tag, cuts.count, &flag)) return;
#pragma unroll
            for (int p = 0; p < S::OWN; p += kAtOnce) {
                f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                for (int c = 0; c < cuts.count; ++c) {
                    const float* const from = parts + (size_t)c * kPiece + p * kD;
                    const float2 lo = get_shared(from), hi = get_shared(from + 2);
                    v += f32x4{lo.x, lo.y, hi.x, hi.y};
                }
                store_quad<T>(rows + p * kD, v * scale);
            }
            return;
        }
#pragma unroll
        for (int p = 0; p < S::OWN; p += kAtOnce) store_quad<T>(rows + p * kD, merged(p) * scale);
        return;
    }

    Frag kf[NQ][NDC], vf[NQ][NDC];
#pragma unroll
    for (int h = 0; h < NQ; ++h) {
        if (row0 + 16 * h + r < length) {
            load_rows<T>(kf[h], K + head + (size_t)(row0 + 16 * h) * kD, r, g);
            load_rows<T>(vf[h], V + head + (size_t)(row0 + 16 * h) * kD, r, g);
        } else {
            clear(kf[h]);
            clear(vf[h]);
        }
    }
    f32x4 dk[NQ][4], dv[NQ][4];
    clear_acc<NQ>(dk);
    clear_acc<NQ>(dv);
    for (int t = wave * KT; t < nt; t += STRIDE) {
        Quad qc[KT][4], dc[KT][4], pq[NQ][KT], dsq[NQ][KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if (u > 0 && t + u >= nt) {
                clear(dc[u]);
                clear(qc[u]);
#pragma unroll
                for (int h = 0; h < NQ; ++h) pq[h][u] = dsq[h][u] = Quad{};
                continue;
            }
            const int q0 = tile0(t + u);
            const size_t at = head + (size_t)q0 * kD;
            Frag qf[NDC], df[NDC];
            unsigned buckets[NQ];
            load_rows<T>(df, dO + at, r, g);
            load_rows<T>(qf, Q + at, r, g);
            const f32x4 lse2 = *reinterpret_cast<const f32x4*>(x.row_lse + vec + q0 + 4 * g);
            const f32x4 ndelta = *reinterpret_cast<const f32x4*>(x.row_delta + vec + q0 + 4 * g);
            load_cols<T>(dc[u], dO + at, r, g);
            load_cols<T>(qc[u], Q + at, r, g);
#pragma unroll
            for (int h = 0; h < NQ; ++h) buckets[h] = buckets_of<true>(x, q0 + 4 * g, row0 + 16 * h + r, L);
            __builtin_amdgcn_sched_barrier(0);
            if (q0 + 16 > length) {
                zero_rows_from<T>(df, q0 + r >= length);
                zero_rows_from<T>(qf, q0 + r >= length);
                zero_cols_from<T>(dc[u], q0 + 4 * g, length);
                zero_cols_from<T>(qc[u], q0 + 4 * g, length);
            }
#pragma unroll
            for (int h = 0; h < NQ; ++h) {
                f32x4 s = bias_of<true>(x, tab, buckets[h]), dp = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NDC; ++c) {
                    s = mma_d(s, qf[c], kf[h][c]);     // S = Q K^T
                    dp = mma_d(dp, df[c], vf[h][c]);   // dP = dO V^T
                }
                unsigned d[4] = {};
                if constexpr (DROP) key_draws(draws, q0 + 4 * g, row0 + 16 * h + r, d);
                f32x4 p, ds;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float pi = exp2f(fmaf(s[i], scale_log2, -lse2[i]));
                    const bool drop = DROP && d[i] < x.threshold;
                    p[i] = drop ? 0.f : pi;
                    ds[i] = pi * ((drop ? 0.f : dp[i]) + ndelta[i]);
                }
                pq[h][u] = to_quad<T>(p);
                dsq[h][u] = to_quad<T>(ds);
            }
        }
        mma_cols(dv, dc, pq);    // dV^T += dO^T P
        mma_cols(dk, qc, dsq);   // dK^T += Q^T dS
    }
    const auto& z = args_again<BwdOfRows<T>>();
    const float scale = z.scale;
    // The rows, or a chunk's sums, unscaled: [head][slot][dK | dV][block][64], which the last of a column's chunks with these rows adds up in their order.
    constexpr int kPart = 2 * BS * kD;
    float* const parts = z.columns.parts + ((size_t)bh * z.columns.n_slots + it.first) * kPart + out;
    float* const mine = parts + (size_t)(it.slot - it.first) * kPart;   // where slot >= 0
    const size_t column = head + (size_t)block * BS * kD + out;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which) __syncthreads();
        put_patch<NQ>(&acc_s[wave][0], which ? dv : dk, r, g);
        __syncthreads();
#pragma unroll
        for (int p = 0; p < S::OWN; p += kAtOnce) {
            const f32x4 v = merged(p);
            if (it.slot >= 0) {
                float* const to = mine + which * BS * kD + p * kD;
                put_shared(to, v[0], v[1]);
                put_shared(to + 2, v[2], v[3]);
            } else {
                store_quad<T>((which ? z.dV : z.dK) + column + p * kD, which ? v : v * scale);
            }
        }
    }
    if (it.slot < 0) return;
    if (!last_to_arrive(z.columns.counters + ((size_t)bh * z.columns.n_slots + it.first) * TPB + part, z.columns.tag, it.count, &flag)) return;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int p = 0; p < S::OWN; p += kAtOnce) {
            f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (int c = 0; c < it.count; ++c) {
                const float* const from = parts + (size_t)c * kPart + which * BS * kD + p * kD;
                const float2 lo = get_shared(from), hi = get_shared(from + 2);
                v += f32x4{lo.x, lo.y, hi.x, hi.y};
            }
            store_quad<T>((which ? z.dV : z.dK) + column + p * kD, which ? v : v * scale);
        }
}

// ------------------------------------------------------------------------------------------------
// The table's gradient from the slices, 2 TS numbers each: number t < 2 TS - 1 is the sum of dS over distance base + t - (TS - 1) of
// a TS x TS tile whose first key is `base` from its first query; the last has `base` as an integer, or kNoSlice where nothing was
// computed.  Every thread adds into its own copy of the buckets in LDS, the copies are added up in a fixed order, and so
// are the parts of a head, by the last of its workgroups to arrive; the counters of arrivals, a line each, are 0 from the backward kernel on.
// kInFlight tiles a wave and share of it at a time, whose numbers are requested together, then their buckets: 4 x 8 heads x 4096, 851 blocks
// of 64, 11.3 us; 2 x 8 heads x 16320, 13.5; 16 x 4 heads x 1024, 157 blocks of 32, 8.3.
// ------------------------------------------------------------------------------------------------
constexpr int kTilesInFlight = 4;   // of a share of a wave
template <int TS>
__global__ __launch_bounds__(256) void table_grad_kernel(const float* __restrict__ slices, Extras x, int L, unsigned tiles_of_head,
                                                         unsigned tiles_a_sequence, int parts, float* partial, unsigned long long* __restrict__ counters,
                                                         void* __restrict__ dtable) {
    extern __shared__ float hist[];   // [n_buckets][threads]
    constexpr int F = 2 * TS, LANES = F / 4, GROUP = 64 / LANES, kInFlight = kTilesInFlight;   // lanes of a tile, four numbers each; tiles of a wave
    const int h = blockIdx.x % x.H, part = blockIdx.x / x.H, tid = threadIdx.x, threads = blockDim.x, lane = tid & 63;
    for (int b = 0; b < x.n_buckets; ++b) hist[b * threads + tid] = 0.f;
    const int t = lane % LANES * 4;
    const unsigned first = (unsigned)((unsigned long long)part * tiles_of_head / parts);
    const unsigned end = (unsigned)((unsigned long long)(part + 1) * tiles_of_head / parts);
    const unsigned at_once = (threads >> 6) * GROUP, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (unsigned c0 = first + wave * GROUP; c0 < end; c0 += kInFlight * at_once) {
        float4 v[kInFlight];
        int base[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const unsigned tile = c0 + u * at_once + lane / LANES, at = tile < end ? tile : end - 1;
            const unsigned b = at / tiles_a_sequence, e = at % tiles_a_sequence;
            v[u] = *reinterpret_cast<const float4*>(slices + ((size_t)(b * x.H + h) * tiles_a_sequence + e) * F + t);
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const float place = v[u].w;
            const int from = __shfl(__builtin_bit_cast(int, place), lane | (LANES - 1));
            base[u] = c0 + u * at_once + lane / LANES < end ? from : kNoSlice;
        }
        unsigned buckets[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {   // (no place leads past the map's 2 L - 1; the last number of a tile belongs to no distance)
            const unsigned at = (unsigned)(base[u] + L - TS + t), from = min(at, 2u * L - 5u);
            buckets[u] = reinterpret_cast<const FourBuckets*>(x.bucket_of + from)->u >> (at == from ? 0 : 8);
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u)
            if (base[u] != kNoSlice) {
                const float four[4] = {v[u].x, v[u].y, v[u].z, t + 3 == F - 1 ? 0.f : v[u].w};
                add_four(hist + tid, threads, four, buckets[u], x.n_buckets);
            }
    }
    finish_table_grad(hist, x.n_buckets, part, parts, h, x.H, partial, counters + h * Extras::kCounterStride, dtable, x.table_bf16 != 0);
}

// ------------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------------
namespace {

// The backward plan of fp32 and block 16: rows and waves of a workgroup, pieces of rows and columns as in the plain kernel.
struct GenericBwd {
    bool wide;          // 32 rows
    int waves, parts;   // workgroups a block row
    long long resident;
    RowCut cut;
    BwdWorkspace ws;
    GenericBwd(const AttnShape& s, int nnzb)
        : wide(s.bs > 16), waves(s.bs == 16 && generic_bwd_many_short_rows(s, nnzb) ? 2 : 4), parts(s.bs / (wide ? 32 : 16)),
          resident(generic_bwd_resident(s.is_bf16, waves)), cut(decide(s, nnzb, parts, resident)), ws(s.BH, s.bs, s.nb, nnzb, kChunk, 0, cut.slots) {}
    static RowCut decide(const AttnShape& s, int nnzb, int parts, long long resident) {
        RowCut cut;
        generic_bwd_decide(cut, s, nnzb, parts, resident);
        if (cut.slots == 0) {
            cut = RowCut{};
            cut.longest = INT_MAX;
            return cut;
        }
        cut.helpers = cut.slots - 1;
        cut.groups = parts * ((s.BH * cut.helpers + 7) & ~7);
        return cut;
    }
};

// The backward's: of pieces of rows and columns first, then the rows' numbers and what the table's gradient takes.
struct WithWorkspace {
    int tile, parts;                                 // rows of a tile that has its own slice; workgroups per head
    size_t rows, slices, partial, counters, total;   // offsets, and the end
    WithWorkspace(const AttnShape& s, int n_buckets, int H, int nnzb) {   // n_buckets 0: no table
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        const bool tiled = s.is_bf16 && s.bs > 16;
        tile = tiled ? s.bs : 16;
        rows = up(tiled ? attn_bwd_workspace(s, nnzb).with_rows : GenericBwd(s, nnzb).ws.with_rows);
        slices = up(rows + 2 * (size_t)s.BH * s.L * sizeof(float));
        if (n_buckets == 0) {
            total = slices;
            return;
        }
        // as many slices as a workgroup requests together, or more, and up to four workgroups a compute unit
        const long long together = (long long)table_grad_threads(n_buckets) / (tile / 2) * kTilesInFlight;
        const long long tiles = (long long)s.BH / H * nnzb * (s.bs / tile) * (s.bs / tile);
        parts = (int)std::max<long long>(1, std::min<long long>((tiles + together - 1) / together, 1024 / H));
        partial = up(slices + (size_t)s.BH * nnzb * (s.bs / tile) * (s.bs / tile) * 2 * tile * sizeof(float));
        counters = up(partial + (size_t)H * parts * n_buckets * sizeof(float));
        total = up(counters + (size_t)H * Extras::kCounterStride * 8);
    }
};

template <typename T, int BS>
hipError_t fwd_with(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, void* O, float* LSE,
                    const int* row_ptr, const int* col_idx, int nnzb, hipStream_t st) {
    if constexpr (sizeof(T) == 2 && BS > 16) {
        return fwd_with_bf16<BS>(s, x, Q, K, V, O, LSE, row_ptr, col_idx, nnzb, st);
    } else {
        const int rows = generic_fwd_rows(s, nnzb) == 32 ? 32 : 16, parts = BS / rows;
        const long long all = (long long)s.BH * s.nb;
        // (rows of fewer than 6 tiles gain nothing by their order and pay the search; see launch_fwd)
        const int sort_rows = s.nb > 32 && (long long)nnzb * (BS / 16) >= 6ll * s.nb && 2 * all * parts > 3 * 256 * (rows == 16 ? 4 : 3);
        RowCut cut;
        if (s.fwd_room) cut = RowCut(s, nnzb);
        if (cut.slots == 0) {
            cut = RowCut{};
            cut.longest = INT_MAX;
        }
        const long long grid = cut.groups + (sort_rows ? parts * group_grid(all) : group_grid(all * parts));
        if (grid > 0x7fffffffll) return hipErrorInvalidValue;
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)grid), dim3(kWaves * 64), 0, st>>>(
                static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V), static_cast<T*>(O), LSE, row_ptr, col_idx, x,
                cut, s.BH, s.L, s.nb, sort_rows, s.scale * kLog2e);
        };
        if constexpr (BS > 16) {
            if (rows == 32) {
                if (x.threshold) launch(attn_fwd_with_kernel<T, BS, 2, true>);
                else launch(attn_fwd_with_kernel<T, BS, 2, false>);
                return hipGetLastError();
            }
        }
        if (x.threshold) launch(attn_fwd_with_kernel<T, BS, 1, true>);
        else launch(attn_fwd_with_kernel<T, BS, 1, false>);
        return hipGetLastError();
    }
}

template <typename T, int BS>
hipError_t bwd_with(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, const void* dO, void* dQ, void* dK, void* dV,
                    const int* row_ptr, const int* col_idx, const int* col_ptr, const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    if constexpr (sizeof(T) == 2 && BS > 16) {
        return bwd_with_bf16<BS>(s, x, Q, K, V, dO, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
    } else {
        GenericBwd plan(s, nnzb);
        const long long all = (long long)s.BH * s.nb, items = (long long)s.BH * plan.parts * (plan.ws.w_max + s.nb);
        const int sort_rows = (long long)nnzb * (BS / 16) >= 6ll * s.nb && s.nb >= 32 && 4 * items > 5 * plan.resident;   // see launch_bwd
        plan.cut.counters = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + plan.ws.total);
        plan.cut.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.ws.row_parts);
        const ColumnCut columns = {plan.ws.chunk, plan.ws.w_first, plan.ws.w_max, plan.ws.n_slots, 2 * items > 3 * plan.resident, s.tag,
                                   static_cast<unsigned long long*>(workspace),
                                   reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.ws.counter_bytes)};
        const long long grid = plan.cut.groups + group_grid((long long)s.BH * plan.parts * columns.n_first) + (sort_rows ? plan.parts * group_grid(all) : group_grid(all * plan.parts)) +
                               group_grid((long long)s.BH * plan.parts * (columns.n_items - columns.n_first));
        if (grid > 0x7fffffffll) return hipErrorInvalidValue;
        const BwdOfRows<T> args = {static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V),
                                   static_cast<const T*>(dO), static_cast<T*>(dQ), static_cast<T*>(dK), static_cast<T*>(dV), row_ptr, col_idx,
                                   col_ptr, row_idx, x, plan.cut, columns, s.BH, s.L, s.nb, nnzb, sort_rows, s.scale, s.scale * kLog2e};
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)grid), dim3(plan.waves * 64), 0, st>>>(args);
        };
        if constexpr (BS > 16) {
            if (x.threshold) launch(attn_bwd_with_kernel<T, BS, 2, 4, true>);
            else launch(attn_bwd_with_kernel<T, BS, 2, 4, false>);
        } else if (plan.waves == 2) {
            if (x.threshold) launch(attn_bwd_with_kernel<T, BS, 1, 2, true>);
            else launch(attn_bwd_with_kernel<T, BS, 1, 2, false>);
        } else {
            if (x.threshold) launch(attn_bwd_with_kernel<T, BS, 1, 4, true>);
            else launch(attn_bwd_with_kernel<T, BS, 1, 4, false>);
        }
        return hipGetLastError();
    }
}

}  // namespace

size_t attn_with_workspace_bytes(const AttnShape& s, int n_buckets, int H, int nnzb, bool is_bwd) {
    if (!is_bwd) return RowCut(s, nnzb).room_bytes(s.BH, s.bs);
    return WithWorkspace(s, n_buckets, H, nnzb).total;
}

#define SPION_DISPATCH(FN, ...)                                                   \
    do {                                                                          \
        if (s.is_bf16) {                                                          \
            if (s.bs == 16) return FN<bf16_t, 16>(__VA_ARGS__);                   \
            if (s.bs == 32) return FN<bf16_t, 32>(__VA_ARGS__);                   \
            return FN<bf16_t, 64>(__VA_ARGS__);                                   \
        }                                                                         \
        if (s.bs == 16) return FN<float, 16>(__VA_ARGS__);                        \
        if (s.bs == 32) return FN<float, 32>(__VA_ARGS__);                        \
        return FN<float, 64>(__VA_ARGS__);                                        \
    } while (0)

hipError_t launch_attn_fwd_with(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, void* O, float* LSE,
                                const int* row_ptr, const int* col_idx, int nnzb, hipStream_t st) {
    SPION_DISPATCH(fwd_with, s, x, Q, K, V, O, LSE, row_ptr, col_idx, nnzb, st);
}

static hipError_t launch_bwd(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, const void* dO, void* dQ, void* dK,
                             void* dV, const int* row_ptr, const int* col_idx, const int* col_ptr, const int* row_idx, int nnzb, void* workspace,
                             hipStream_t st) {
    SPION_DISPATCH(bwd_with, s, x, Q, K, V, dO, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
}

hipError_t launch_attn_bwd_with(const AttnShape& s, const Extras& extras, const void* Q, const void* K, const void* V, const void* O,
                                const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* dtable, const int* row_ptr,
                                const int* col_idx, const int* col_ptr, const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    Extras x = extras;
    const WithWorkspace ws(s, x.n_buckets, x.H, nnzb);
    char* const base = static_cast<char*>(workspace);
    x.slices = x.table ? reinterpret_cast<float*>(base + ws.slices) : nullptr;
    x.counters = x.table ? reinterpret_cast<unsigned long long*>(base + ws.counters) : nullptr;
    const long long rows = (long long)s.BH * s.L;
    x.row_lse = reinterpret_cast<float*>(base + ws.rows);
    x.row_delta = x.row_lse + rows;
    // the kernels of bf16 and block 32 and 64 take it times 2^-24 with dropout
    const float delta_scale = (x.threshold && s.is_bf16 && s.bs > 16 ? -1.f / 16777216.f : -1.f) / x.keep_scale;
    auto row_terms = [&](auto kernel, auto type) {
        typedef decltype(type) T;
        kernel<<<dim3((unsigned)((rows + 31) / 32)), dim3(256), 0, st>>>(static_cast<const T*>(O), static_cast<const T*>(dO), LSE, x, s.heads_beside != 0, s.L, rows,
                                                                           delta_scale);
    };
    if ((rows + 31) / 32 > 0x7fffffffll) return hipErrorInvalidValue;
    if (s.is_bf16) row_terms(row_terms_kernel<bf16_t>, bf16_t{});
    else row_terms(row_terms_kernel<float>, float{});
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = launch_bwd(s, x, Q, K, V, dO, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
    if (e != hipSuccess || !dtable) return e;
    const long long tiles = (long long)nnzb * (s.bs / ws.tile) * (s.bs / ws.tile);
    if (s.BH / x.H * tiles > 0x7fffffffll) return hipErrorInvalidValue;   // (256 GB of slices and more)
    const int threads = table_grad_threads(x.n_buckets);
    auto launch = [&](auto kernel) {
        kernel<<<dim3((unsigned)(x.H * ws.parts)), dim3(threads), (size_t)x.n_buckets * threads * sizeof(float), st>>>(
            x.slices, x, s.L, (unsigned)(s.BH / x.H * tiles), (unsigned)tiles, ws.parts, reinterpret_cast<float*>(base + ws.partial), x.counters, dtable);
    };
    if (ws.tile == 16) launch(table_grad_kernel<16>);
    else if (ws.tile == 32) launch(table_grad_kernel<32>);
    else launch(table_grad_kernel<64>);
    return hipGetLastError();
}

}  // namespace spion
