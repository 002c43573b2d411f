// Block-sparse attention (Eq. 5 on the kept blocks) with what a Transformer adds inside the softmax: a learned relative
// position bias by buckets, dropout of the probabilities, sequences shorter than the batch's length.
//   S_qk = scale Q_q K_k + T[bucket(k - q)][head], P = softmax over the kept k < length, O = (c M . P) V, c = 1 / (1 - p)
//   delta = rowsum(dO . O), dP = c M . (dO V^T), dS = P . (dP - delta)
//   dV = (c M . P)^T dO, dQ = scale dS K, dK = scale dS^T Q, dT[b][head] = sum of dS over the elements of bucket b
// Queries and keys from the length on: O = 0, LSE = -inf, gradients 0; nothing of theirs is added up.
//
// The kernels of this file take every type and block size: a workgroup of four waves has 16 rows, whose 16-row tiles of the other
// side the waves take in turn, straight from memory into registers (layouts as in attn_kernels.hip).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "attn_extras.h"
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

template <typename T>
struct Tiles {
    static constexpr int KT = sizeof(T) == 2 ? 2 : 1;   // tiles per step: a bf16 MFMA contracts over 32 rows
    static constexpr int NDC = kD / Elem<T>::KC;
};

constexpr int kWaves = 4;

// bias / scale of query q and the keys k .. k + 3 (or, KEYS, of key k and the queries q .. q + 3)
template <bool KEYS>
__device__ __forceinline__ f32x4 bias_of(const Extras& x, const float* tab, int q, int k, int L) {
    if (!x.table) return f32x4{0.f, 0.f, 0.f, 0.f};
    const unsigned b = *reinterpret_cast<const u32_any*>(x.bucket_of + (k - q - (KEYS ? 3 : 0) + L - 1));
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = tab[bucket_index(x, b >> (KEYS ? 24 - 8 * i : 8 * i) & 255u)];
    return v;
}

}  // namespace

// ------------------------------------------------------------------------------------------------
// forward: workgroup = (head, 16 query rows)
// ------------------------------------------------------------------------------------------------
template <typename T, int BS, bool DROP>
__global__ __launch_bounds__(kWaves * 64, 2) void attn_fwd_with_kernel(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O, float* __restrict__ LSE,
    const int* __restrict__ row_ptr, const int* __restrict__ col_idx, Extras x, int L, int nb, int total, float scale_log2) {
    typedef typename Elem<T>::Frag Frag;
    typedef typename Elem<T>::Quad Quad;
    constexpr int KT = Tiles<T>::KT, NDC = Tiles<T>::NDC, TPB = BS / 16, STRIDE = kWaves * KT;
    __shared__ __attribute__((aligned(16))) float o_s[kWaves][16 * kPatchLd];
    __shared__ float m_s[kWaves][16], l_s[kWaves][16], tab[Extras::kMaxBuckets];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (DROP && blockIdx.x == 0 && tid < 2 && x.rng_used) x.rng_used[tid] = x.rng[tid];
    const int item = item_of_group(blockIdx.x, total);
    if (item < 0) return;
    const int bh = item / (nb * TPB), I = item % (nb * TPB) / TPB, row0 = I * BS + item % TPB * 16;
    const size_t head = (size_t)bh * L * kD;
    const int length = length_of(x, bh, L);
    if (x.table) load_bias_table(tab, x, bh % x.H, tid, kWaves * 64);
    __syncthreads();

    const int* cols = col_idx + row_ptr[I];
    const int n = row0 < length ? blocks_below<BS>(cols, row_ptr[I + 1] - row_ptr[I], length, lane) : 0;
    const int nt = n * TPB;
    const int cols64 = n > 0 ? cols[lane < n ? lane : n - 1] : 0;
    auto key0 = [&](int t) { return list_at(cols, cols64, t / TPB) * BS + t % TPB * 16; };
    Frag qf[NDC];
    const int query = row0 + r;
    if (query < length) load_rows<T>(qf, Q + head + (size_t)row0 * kD, r, g);
    else clear(qf);
    [[maybe_unused]] ScoreDraws draws(x.rng, x.stream, bh);

    float m = kLowest, limit = -INFINITY, lsum = 0.f;
    f32x4 oacc[1][4];
    clear_acc<1>(oacc);
    for (int t = wave * KT; t < nt; t += STRIDE) {
        Frag kf[KT][NDC];
        Quad vc[KT][4];
        f32x4 s[KT];
        int k0[KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            k0[u] = key0(t + u < nt ? t + u : t);
            const size_t at = head + (size_t)k0[u] * kD;
            load_rows<T>(kf[u], K + at, r, g);
            load_cols<T>(vc[u], V + at, r, g);
            s[u] = bias_of<false>(x, tab, query, k0[u] + 4 * g, L);
            if (k0[u] + 16 > length) {
                zero_rows_from<T>(kf[u], k0[u] + r >= length);
                zero_cols_from<T>(vc[u], k0[u] + 4 * g, length);
            }
            if (u > 0 && t + u >= nt) clear(vc[u]);
        }
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < KT; ++u) {
#pragma unroll
            for (int c = 0; c < NDC; ++c) s[u] = mma_d(s[u], kf[u][c], qf[c]);   // S^T: [key 4 g + i][query r]
            const bool there = u == 0 || t + u < nt;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!there || k0[u] + 4 * g + i >= length) s[u][i] = -INFINITY;
                mx = fmaxf(mx, s[u][i]);
            }
        }
        if (__any(mx * scale_log2 > limit)) {
            const float m_new = fmaxf(m, group_max(mx) * scale_log2);
            const float alpha = exp2f(m - m_new);
            m = m_new;
            limit = m_new + kRescaleSlack;
            lsum *= alpha;
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[0][e] *= alpha;
        }
        Quad pq[1][KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            f32x4 p;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = exp2f(fmaf(s[u][i], scale_log2, -m));
                lsum += p[i];
            }
            if constexpr (DROP) {
                unsigned d[4];
                query_draws(draws, query, k0[u] + 4 * g, d);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = d[i] < x.threshold ? 0.f : p[i];
            }
            pq[0][u] = to_quad<T>(p);
        }
        mma_cols(oacc, vc, pq);   // O^T += V^T P^T
    }

    // the waves' shares of each row: rescaled to the row's largest m and added up in wave order
    put_patch<1>(&o_s[wave][0], oacc, r, g);
    const float l = group_sum(lsum);
    if (g == 0) {
        m_s[wave][r] = m;
        l_s[wave][r] = l;
    }
    __syncthreads();
    const int q = tid >> 4, d = (tid & 15) * 4;
    float mm = m_s[0][q], ll = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, m_s[w][q]);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const float a = exp2f(m_s[w][q] - mm);
        ll += l_s[w][q] * a;
        o += *reinterpret_cast<const f32x4*>(&o_s[w][q * kPatchLd + d]) * a;
    }
    const bool empty = !(ll > 0.f) && ll == ll;
    o = empty || row0 + q >= length ? f32x4{0.f, 0.f, 0.f, 0.f} : o * ((DROP ? x.keep_scale : 1.f) / ll);
    store_quad<T>(O + head + (size_t)(row0 + q) * kD + d, o);
    if (d == 0) LSE[(size_t)bh * L + row0 + q] = empty || row0 + q >= length ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

// ------------------------------------------------------------------------------------------------
// backward: workgroup = (head, 16 rows of a block row) on the query side, (head, 16 keys of a block column) on the key side.
// The sides share no data; all sums in fixed order.  The query side leaves, for the table's gradient, the sums over the 31 diagonals of each
// 16 x 16 tile of dS in slices[head][kept block][query tile][key tile][32].
// ------------------------------------------------------------------------------------------------
template <typename T, int BS, bool DROP>
__global__ __launch_bounds__(kWaves * 64, 2) void attn_bwd_with_kernel(
    const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O, const T* __restrict__ dO,
    const float* __restrict__ LSE, T* __restrict__ dQ, T* __restrict__ dK, T* __restrict__ dV, const int* __restrict__ row_ptr,
    const int* __restrict__ col_idx, const int* __restrict__ col_ptr, const int* __restrict__ row_idx, Extras x, int L, int nb, int nnzb,
    int total, float scale, float scale_log2) {
    typedef typename Elem<T>::Frag Frag;
    typedef typename Elem<T>::Quad Quad;
    typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int KT = Tiles<T>::KT, NDC = Tiles<T>::NDC, TPB = BS / 16, STRIDE = kWaves * KT;
    constexpr int kDiag = 48;   // floats per lane group and wave: places of distance 16 kt + 4 g - p, behind each other
    __shared__ __attribute__((aligned(16))) float acc_s[kWaves][16 * kPatchLd];
    __shared__ float tab[Extras::kMaxBuckets], diag_s[kWaves][4][kDiag];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x == 0 && x.counters)
        for (int h = tid; h < x.H; h += kWaves * 64) x.counters[h * Extras::kCounterStride] = 0u;
    const int half = (total + 7) / 8 * 8;   // workgroups of a side
    const bool key_side = (int)blockIdx.x >= half;
    const int item = item_of_group(key_side ? blockIdx.x - half : blockIdx.x, total);
    if (item < 0) return;
    const int bh = item / (nb * TPB), block = item % (nb * TPB) / TPB, sub = item % TPB, row0 = block * BS + sub * 16;
    const size_t head = (size_t)bh * L * kD, vec = (size_t)bh * L;
    const int length = length_of(x, bh, L);
    if (x.table) load_bias_table(tab, x, bh % x.H, tid, kWaves * 64);
    if (!key_side && x.slices)
        for (int i = tid; i < kWaves * 4 * kDiag; i += kWaves * 64) (&diag_s[0][0][0])[i] = 0.f;
    __syncthreads();
    [[maybe_unused]] ScoreDraws draws(x.rng, x.stream, bh);
    const float keep = DROP ? x.keep_scale : 1.f;
    const int own = row0 + r;

    auto merged = [&]() {
        const int o = (tid >> 4) * kPatchLd + (tid & 15) * 4;
        f32x4 v = *reinterpret_cast<const f32x4*>(&acc_s[0][o]);
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(&acc_s[w][o]);
        return row0 + (tid >> 4) < length ? v : f32x4{0.f, 0.f, 0.f, 0.f};
    };
    const size_t out = head + (size_t)(row0 + (tid >> 4)) * kD + (tid & 15) * 4;
    const int* list = (key_side ? row_idx : col_idx) + (key_side ? col_ptr : row_ptr)[block];
    const int n_list = (key_side ? col_ptr : row_ptr)[block + 1] - (key_side ? col_ptr : row_ptr)[block];
    const int n = row0 < length ? blocks_below<BS>(list, n_list, length, lane) : 0;
    const int nt = n * TPB;
    const int list64 = n > 0 ? list[lane < n ? lane : n - 1] : 0;
    auto tile0 = [&](int t) { return list_at(list, list64, t / TPB) * BS + t % TPB * 16; };

    if (!key_side) {
        Frag qf[NDC], dof[NDC];
        float delta = 0.f, lse2 = INFINITY;
        if (own < length) {
            Frag of[NDC];
            const size_t at = head + (size_t)row0 * kD;
            load_rows<T>(qf, Q + at, r, g);
            load_rows<T>(dof, dO + at, r, g);
            load_rows<T>(of, O + at, r, g);
            lse2 = LSE[vec + own] * kLog2e;
            if (lse2 == -INFINITY) lse2 = INFINITY;   // a row that keeps nothing
#pragma unroll
            for (int c = 0; c < NDC; ++c)
#pragma unroll
                for (int e = 0; e < Elem<T>::EPL; ++e) delta = fmaf((float)dof[c][e], (float)of[c][e], delta);
        } else {
            clear(qf);
            clear(dof);
        }
        delta = group_sum(delta);
        if (x.slices)   // what is not computed
            for (int e = n * TPB + tid; e < n_list * TPB; e += kWaves * 64)
                x.slices[((((size_t)bh * nnzb + row_ptr[block] + e / TPB) * TPB + sub) * TPB + e % TPB) * 32 + 31] = __builtin_bit_cast(float, kNoSlice);
        f32x4 dq[1][4];
        clear_acc<1>(dq);
        for (int t = wave * KT; t < nt; t += STRIDE) {
            Quad kc[KT][4], dsq[1][KT];
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                const bool there = u == 0 || t + u < nt;
                const int k0 = tile0(there ? t + u : t);
                const size_t at = head + (size_t)k0 * kD;
                Frag kf[NDC], vf[NDC];
                load_rows<T>(kf, K + at, r, g);
                load_rows<T>(vf, V + at, r, g);
                load_cols<T>(kc[u], K + at, r, g);
                f32x4 s = bias_of<false>(x, tab, own, k0 + 4 * g, L), dp = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k0 + 16 > length) {
                    zero_rows_from<T>(kf, k0 + r >= length);
                    zero_rows_from<T>(vf, k0 + r >= length);
                    zero_cols_from<T>(kc[u], k0 + 4 * g, length);
                }
                if (!there) clear(kc[u]);
#pragma unroll
                for (int c = 0; c < NDC; ++c) {
                    s = mma_d(s, kf[c], qf[c]);      // S^T = K Q^T
                    dp = mma_d(dp, vf[c], dof[c]);   // dP^T = V dO^T
                }
                unsigned d[4] = {};
                if constexpr (DROP) query_draws(draws, own, k0 + 4 * g, d);
                f32x4 ds;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool masked = !there || k0 + 4 * g + i >= length;
                    const float p = masked ? 0.f : exp2f(fmaf(s[i], scale_log2, -lse2));
                    const float dpi = DROP && d[i] < x.threshold ? 0.f : dp[i] * keep;
                    ds[i] = p * (dpi - delta);
                }
                dsq[0][u] = to_quad<T>(ds);
                if (x.slices && there) {
                    const f32x4 one[1] = {ds};
                    float du[2];
                    diagonal_sums<1>(one, du);
                    diag_s[wave][g][4 * g - r + 15] = du[0];
                    diag_s[wave][g][4 * g - r + 31] = du[1];
                    __builtin_amdgcn_wave_barrier();
                    if (lane < 32) {
                        const float v = diag_s[wave][0][lane] + diag_s[wave][1][lane] + diag_s[wave][2][lane] + diag_s[wave][3][lane];
                        const size_t entry = (size_t)bh * nnzb + row_ptr[block] + (t + u) / TPB;
                        x.slices[((entry * TPB + sub) * TPB + (t + u) % TPB) * 32 + lane] = lane < 31 ? v : __builtin_bit_cast(float, k0 - row0);
                    }
                    __builtin_amdgcn_wave_barrier();
                }
            }
            mma_cols(dq, kc, dsq);   // dQ^T += K^T dS^T
        }
        put_patch<1>(&acc_s[wave][0], dq, r, g);
        __syncthreads();
        store_quad<T>(dQ + out, merged() * scale);
        return;
    }

    Frag kf[NDC], vf[NDC];
    if (own < length) {
        load_rows<T>(kf, K + head + (size_t)row0 * kD, r, g);
        load_rows<T>(vf, V + head + (size_t)row0 * kD, r, g);
    } else {
        clear(kf);
        clear(vf);
    }
    f32x4 dk[1][4], dv[1][4];
    clear_acc<1>(dk);
    clear_acc<1>(dv);
    for (int t = wave * KT; t < nt; t += STRIDE) {
        Quad qc[KT][4], dc[KT][4], pq[1][KT], dsq[1][KT];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const bool there = u == 0 || t + u < nt;
            const int q0 = tile0(there ? t + u : t);
            const size_t at = head + (size_t)q0 * kD;
            Frag qf[NDC], df[NDC], of[NDC];
            load_rows<T>(df, dO + at, r, g);
            load_rows<T>(of, O + at, r, g);
            load_rows<T>(qf, Q + at, r, g);
            const f32x4_any lse = *reinterpret_cast<const f32x4_any*>(LSE + vec + q0 + 4 * g);
            load_cols<T>(dc[u], dO + at, r, g);
            load_cols<T>(qc[u], Q + at, r, g);
            if (q0 + 16 > length) {
                zero_rows_from<T>(df, q0 + r >= length);
                zero_rows_from<T>(of, q0 + r >= length);
                zero_rows_from<T>(qf, q0 + r >= length);
                zero_cols_from<T>(dc[u], q0 + 4 * g, length);
                zero_cols_from<T>(qc[u], q0 + 4 * g, length);
            }
            if (!there) {
                clear(dc[u]);
                clear(qc[u]);
            }
            float part = 0.f;
#pragma unroll
            for (int c = 0; c < NDC; ++c)
#pragma unroll
                for (int e = 0; e < Elem<T>::EPL; ++e) part = fmaf((float)df[c][e], (float)of[c][e], part);
            // delta of rows 4 g + i in every lane: the lanes' shares of row r times a tile of ones
            const f32x4 delta = __builtin_amdgcn_mfma_f32_16x16x4f32(part, 1.f, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            f32x4 s = bias_of<true>(x, tab, q0 + 4 * g, own, L), dp = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NDC; ++c) {
                s = mma_d(s, qf[c], kf[c]);     // S = Q K^T
                dp = mma_d(dp, df[c], vf[c]);   // dP = dO V^T
            }
            unsigned d[4] = {};
            if constexpr (DROP) key_draws(draws, q0 + 4 * g, own, d);
            f32x4 p, ds;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lse2 = lse[i] == -INFINITY || q0 + 4 * g + i >= length ? INFINITY : lse[i] * kLog2e;
                const float pi = there ? exp2f(fmaf(s[i], scale_log2, -lse2)) : 0.f;
                const bool drop = DROP && d[i] < x.threshold;
                p[i] = drop ? 0.f : pi * keep;
                ds[i] = there ? pi * ((drop ? 0.f : dp[i] * keep) - delta[i]) : 0.f;
            }
            pq[0][u] = to_quad<T>(p);
            dsq[0][u] = to_quad<T>(ds);
        }
        mma_cols(dv, dc, pq);    // dV^T += dO^T P
        mma_cols(dk, qc, dsq);   // dK^T += Q^T dS
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (which) __syncthreads();
        put_patch<1>(&acc_s[wave][0], which ? dv : dk, r, g);
        __syncthreads();
        const f32x4 v = merged();
        store_quad<T>((which ? dV : dK) + out, which ? v : v * scale);
    }
}

// ------------------------------------------------------------------------------------------------
// The table's gradient from the slices, 2 TS numbers each: number t < 2 TS - 1 is the sum of dS over distance base + t - (TS - 1) of
// a TS x TS tile whose first key is `base` from its first query; the last has `base` as an integer, or kNoSlice where nothing was
// computed.  Every thread adds into its own copy of the buckets in LDS, the copies are added up in a fixed order, and so
// are the parts of a head, by the last of its workgroups to arrive; the counters of arrivals, a line each, are 0 from the backward kernel on.
// kInFlight tiles a wave and share of it at a time, whose numbers are requested together, then their buckets: 4 x 8 heads x 4096, 851 blocks
// of 64, 10.5 us; 2 x 8 heads x 16320, 13.5 us.
// ------------------------------------------------------------------------------------------------
template <int TS>
__global__ __launch_bounds__(256) void table_grad_kernel(const float* __restrict__ slices, Extras x, int L, unsigned tiles_of_head,
                                                         unsigned tiles_a_sequence, int parts, float* partial, unsigned long long* __restrict__ counters,
                                                         void* __restrict__ dtable) {
    extern __shared__ float hist[];   // [n_buckets][threads]
    constexpr int F = 2 * TS, LANES = F / 4, GROUP = 64 / LANES, kInFlight = 4;   // lanes of a tile, four numbers each; tiles of a wave
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

// The backward's: of the bf16 kernels of block 32 and 64 first, then what the table's gradient takes.
struct WithWorkspace {
    int tile, parts;                           // rows of a tile that has its own slice; workgroups per head
    size_t slices, partial, counters, total;   // offsets, and the end
    WithWorkspace(const AttnShape& s, int n_buckets, int H, int nnzb) {   // n_buckets 0: no table
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        const bool tiled = s.is_bf16 && s.bs > 16;
        tile = tiled ? s.bs : 16;
        slices = tiled ? up(attn_bwd_workspace(s, nnzb).with_rows) : 0;
        if (n_buckets == 0) {
            total = slices;
            return;
        }
        // sixteen slices a workgroup or more, and about two workgroups a compute unit
        const long long tiles = (long long)s.BH / H * nnzb * (s.bs / tile) * (s.bs / tile);
        parts = (int)std::max<long long>(1, std::min<long long>(tiles / 16, 1024 / H));
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
        const long long total = (long long)s.BH * s.nb * (BS / 16), grid = group_grid(total);
        if (grid > 0x7fffffffll) return hipErrorInvalidValue;
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)grid), dim3(kWaves * 64), 0, st>>>(
                static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V), static_cast<T*>(O), LSE, row_ptr, col_idx, x,
                s.L, s.nb, (int)total, s.scale * kLog2e);
        };
        if (x.threshold) launch(attn_fwd_with_kernel<T, BS, true>);
        else launch(attn_fwd_with_kernel<T, BS, false>);
        return hipGetLastError();
    }
}

template <typename T, int BS>
hipError_t bwd_with(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, const void* O, const void* dO,
                    const float* LSE, void* dQ, void* dK, void* dV, const int* row_ptr, const int* col_idx, const int* col_ptr,
                    const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    if constexpr (sizeof(T) == 2 && BS > 16) {
        return bwd_with_bf16<BS>(s, x, Q, K, V, O, dO, LSE, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
    } else {
        const long long total = (long long)s.BH * s.nb * (BS / 16), grid = 2 * group_grid(total);
        if (grid > 0x7fffffffll) return hipErrorInvalidValue;
        auto launch = [&](auto kernel) {
            kernel<<<dim3((unsigned)grid), dim3(kWaves * 64), 0, st>>>(
                static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V), static_cast<const T*>(O),
                static_cast<const T*>(dO), LSE, static_cast<T*>(dQ), static_cast<T*>(dK), static_cast<T*>(dV), row_ptr, col_idx, col_ptr,
                row_idx, x, s.L, s.nb, nnzb, (int)total, s.scale, s.scale * kLog2e);
        };
        if (x.threshold) launch(attn_bwd_with_kernel<T, BS, true>);
        else launch(attn_bwd_with_kernel<T, BS, false>);
        return hipGetLastError();
    }
}

}  // namespace

size_t attn_with_workspace_bytes(const AttnShape& s, int n_buckets, int H, int nnzb, bool is_bwd) {
    if (!is_bwd) return s.is_bf16 && s.bs > 16 ? RowCut(s, nnzb).room_bytes(s.BH, s.bs) : 0;
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

static hipError_t launch_bwd(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, const void* O,
                             const void* dO, const float* LSE, void* dQ, void* dK, void* dV, const int* row_ptr, const int* col_idx,
                             const int* col_ptr, const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    SPION_DISPATCH(bwd_with, s, x, Q, K, V, O, dO, LSE, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
}

hipError_t launch_attn_bwd_with(const AttnShape& s, const Extras& extras, const void* Q, const void* K, const void* V, const void* O,
                                const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* dtable, const int* row_ptr,
                                const int* col_idx, const int* col_ptr, const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    Extras x = extras;
    const WithWorkspace ws(s, x.n_buckets, x.H, nnzb);
    char* const base = static_cast<char*>(workspace);
    x.slices = x.table ? reinterpret_cast<float*>(base + ws.slices) : nullptr;
    x.counters = x.table ? reinterpret_cast<unsigned long long*>(base + ws.counters) : nullptr;
    hipError_t e = launch_bwd(s, x, Q, K, V, O, dO, LSE, dQ, dK, dV, row_ptr, col_idx, col_ptr, row_idx, nnzb, workspace, st);
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
