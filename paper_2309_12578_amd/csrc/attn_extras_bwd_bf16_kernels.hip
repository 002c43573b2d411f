// Backward pass of the attention with a relative position bias, dropout and lengths for bf16 and block size 32 or 64: one launch with the
// grid, the work items and the cuts of the plain bf16 kernel (attn_bwd_bf16_kernels.hip).
//
// With c = 1 / (1 - p) the exponentials are taken against LSE - log c, so that they are c P; delta is divided by c to match:
// dS = c P (M dP - delta / c), dV = (M c P)^T dO.  Both sides make the factors M anew.  Both numbers of every row come from a
// kernel before this one (row_terms_kernel): made by the key side from its tiles of O, each step had a third tile, a product and a
// barrier more.
//
// The table's gradient needs dS by distance.  The query side adds up its diagonals: within a wave's 16 queries by lane
// shifts (diagonal_sums) and through LDS, over the waves of the workgroup one step later, behind the barrier that is there anyway.  What leaves
// is one number for each distance of a block, slices[head][kept block][2 BS], 1/32 of what the block's tiles bring in.
//
// Three waves a SIMD at up to 168 registers (block 32: four at 128; with a bias LDS has room for seven workgroups of two, 3.5), which the arguments read again where they are used (args_again) and addresses made
// anew for each block (once) leave room for; at two the backward with bias and dropout took 253 instead of 220 us (4 x 8 heads x 4096, 20.8 %).  Neither
// the matrix nor the vector pipes are busy half of the time: a step is one chain of products, exponentials and products, longer than the plain one by
// the draws and the biases.  Kernel time, us, of the plain one, with lengths, bias, dropout, bias and dropout (row_terms_kernel not counted): 4 x 4 heads x 4096,
// block 64, 8 %, 45.5 / 48.5 / 62 / 64 / 80; 4 x 8 heads, 20.8 %, 151 / 145 / 160 / 186 / 204; 2 x 8 x 16320, 5 %, 303 / 263 / 306 / 335 / 364; 16 x 4 x 1024, block 32,
// 15 %, 28.5 / 28.7 / 38.6 / 36.6 / 48.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "attn_extras.h"
#include "attn_extras_bf16.h"
#include "attn_key_items.h"
#include "spion_internal.h"

namespace spion {

struct BwdWith {
    const bf16_t *Q, *K, *V, *dO;
    bf16_t *dQ, *dK, *dV;
    const int *row_ptr, *col_idx, *col_ptr, *row_idx;
    float* partial;
    unsigned long long *counters, tag;
    Rows at;
    Extras x;
    RowCut cut;
    int n_slots, BH, L, nb, nnzb, n_key_a, n_key_c, w_first, chunk, sort_rows, finest, few;
    float scale, scale_log2;
};

namespace {

// With dropout, 2^-24 (M dP - delta / c) in one instruction: the factor, 0 or 1 in 16 bits, is 0 or 2^-24 as a half, what is added comes times
// 2^-24, and the exponentials (query side) or the result (key side) are taken times 2^24.
constexpr float kHalfOne = 1.f / 16777216.f;
__device__ __forceinline__ float where_kept_plus(float v, const unsigned (&f)[2], int i, float add) {   // element i of four whose factors are f
    float d;
    if (i & 1) asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel:[0,1,0] op_sel_hi:[0,1,0]" : "=v"(d) : "v"(v), "v"(f[i >> 1]), "v"(add));
    else asm("v_fma_mix_f32 %0, %1, %2, %3 op_sel_hi:[0,1,0]" : "=v"(d) : "v"(v), "v"(f[i >> 1]), "v"(add));
    return d;
}

}  // namespace

template <int BS, bool BIAS, bool DROP>
__global__ __launch_bounds__(BS * 4, BS == 32 ? 4 : 3) void attn_bwd_with_bf16_kernel(BwdWith a) {
    constexpr int NT = BS / 16;   // 16-row tiles per block = waves per workgroup
    // {ta, tb} hold {K, V} of a block (query side) or {Q, dO} of a block row (key side), two stages
    __shared__ __attribute__((aligned(16))) bf16_t ta0[BS * kD], tb0[BS * kD], ta1[BS * kD], tb1[BS * kD];
    // Diagonals (query side): each wave's places (lane group, distance), of which those it never writes stay 0, and for two steps each
    // wave's sums of every distance of the block.
    constexpr int kPlaces = 16 * NT + 32;
    __shared__ float all_places[BIAS ? NT * 4 * kPlaces : 1], sums[BIAS ? 2 * NT * 2 * BS : 1];   // sums [step % 2][wave][2 BS]
    __shared__ __attribute__((aligned(16))) float lse0[BS], del0[BS], lse1[BS], del1[BS];
    __shared__ __attribute__((aligned(16))) float bias0[kSlice<BS>], bias1[kSlice<BS>];
    __shared__ float tab[BIAS ? Extras::kMaxBuckets : 1];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int L = a.L, nb = a.nb;

    // which workgroup am I
    const ItemOfHead dealt_to = deal_heads(blockIdx.x, a.BH, a.few != 0);
    int bh = dealt_to.head, idx = dealt_to.item;   // work item (key side) or block row (query side)
    RowPieces cuts = {0, 1, 0, 0};
    int piece = 0;
    bool key_side = false;
    const bool helper = idx < a.cut.helpers;
    if (helper) {
        cuts = row_pieces<false>(a.row_ptr, nb, a.cut, idx, lane);
        if (cuts.row < 0) return;
        piece = idx - cuts.first + 1;
        idx = cuts.row;
    } else {
        idx -= a.cut.helpers;
        if (idx < a.n_key_a) {
            key_side = true;
        } else if (idx < a.n_key_a + nb) {
            idx -= a.n_key_a;
            if (a.sort_rows) {
                idx = row_by_length(a.row_ptr, nb, idx, lane);
            } else if ((a.BH & 7) == 0) {   // whole heads: one after the other
                const int hpx = a.BH >> 3, first = (blockIdx.x & 7) * hpx, l = idx * hpx + bh - first;
                bh = first + l / nb;
                idx = l % nb;
            }
        } else {
            idx -= a.n_key_a + nb;
            if (idx >= a.n_key_c) return;
            key_side = true;
            idx += a.w_first;
        }
    }
    const TableColumn<BS, BIAS> column(a.x, bh % a.x.H, tid);
    const BlockBias<BS, BIAS> biases(a.x, tab, L, wave);
    const SwzLane sl(r, g);
    const int length = length_of(a.x, bh, L);

    if (!key_side) {
        // ========================================================================================
        // query side: block row I
        // ========================================================================================
        const auto& b = args_again<BwdWith>();   // this side's
        const Rows at = {b.at.H, b.at.beside};
        const int in_row = at.in_row(), out_row = at.out_row();   // elements between rows of Q, K, V and of O, dO
        const size_t head = at.in_head(bh, L), out_head = at.out_head(bh, L), vec = (size_t)bh * L;
        [[maybe_unused]] const ScoreDraws draws(DROP, b.x.rng, b.x.stream, bh);
        [[maybe_unused]] const unsigned below = both_halves(b.x.threshold - 1u);
        const float scale_log2 = b.scale_log2;
        const int I = idx;
        const int qrow = I * BS + wave * 16 + r;
        unsigned bucket = biases.request(0, tid);
        const bf16_t *const Kh = b.K + head, *const Vh = b.V + head;
        const TileLoadLane tl(wave, lane, in_row);
        auto issue = [&](bf16_t* kt, bf16_t* vt, int J) {
            const unsigned range = tile_range<BS>(J * BS, length, in_row);
            tile_load_async(Kh + (size_t)J * BS * in_row, kt, wave, tl, range);
            tile_load_async(Vh + (size_t)J * BS * in_row, vt, wave, tl, range);
        };
        if (!helper) issue(ta0, tb0, I);   // the diagonal block, before any index is known
        bf16x8 qf[2], dof[2];
        const float lse2 = b.x.row_lse[vec + qrow] - (DROP ? 24.f : 0.f), ndelta = b.x.row_delta[vec + qrow];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            qf[c] = *reinterpret_cast<const bf16x8*>(b.Q + head + (size_t)qrow * in_row + c * 32 + g * 8);
            dof[c] = *reinterpret_cast<const bf16x8*>(b.dO + out_head + (size_t)qrow * out_row + c * 32 + g * 8);
            if (qrow >= length) qf[c] = dof[c] = bf16x8{};
        }
        int jb = b.row_ptr[I], n = b.row_ptr[I + 1] - jb;
        if (n > a.cut.longest) {
            if (!helper) cuts = row_pieces<true>(a.row_ptr, nb, a.cut, I, lane);
            const int from = piece * n / cuts.count;
            n = (piece + 1) * n / cuts.count - from;
            jb += from;
        }
        const int* cols = b.col_idx + jb;
        const int n_all = n;
        n = I * BS < length ? blocks_below<BS>(cols, n, length, L, lane) : 0;
        const int last = n > 0 ? n - 1 : 0;
        int first[8];
        int pd = n > 0 ? find_in_row(cols, n, I, first) : -1;
        if (helper) pd = -1;   // in index order, the diagonal block where it comes
        // block visited at step t (clamped reads stay inside this row's entries; an empty row reads nothing)
        auto col_at = [&](int t) {
            const int j = walk_index(t < last ? t : last, pd);
            return j < 8 ? pick8(first, j) : cols[j];
        };
        int walk_v = 0;   // 64 blocks of the walk, one per lane
        if (n > 2) walk_v = cols[walk_index(lane < last ? lane : last, pd)];
        int pd_v = pd, jb_v = jb;   // (scalar registers are short)
        asm volatile("" : "+v"(pd_v), "+v"(jb_v));
        auto later_col = [&](int t) {   // t >= 2, one after the other
            const int u = t < last ? t : last;
            if (u >= 64 && (u & 63) == 0) walk_v = args_again<BwdWith>().col_idx[jb_v + walk_index(u + lane < last ? u + lane : last, pd_v)];
            return __builtin_amdgcn_readlane(walk_v, u & 63);
        };
        int jcur = __builtin_amdgcn_readfirstlane(n > 0 ? col_at(0) : I), jnext = __builtin_amdgcn_readfirstlane(n > 0 ? col_at(1) : I);
        column.put(tab, a.x, tid);
        if (pd < 0 && n > 0) {
            // no diagonal block in this row (piece): once everyone's early load has landed, load block 0 over it
            if (BIAS) bucket = biases.request(jcur - I, tid);
            if (!helper) {
                __builtin_amdgcn_s_waitcnt(kWaitVm0);
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
            issue(ta0, tb0, jcur);
        }
        float* const places = all_places + wave * (4 * kPlaces);
        float* const my_slices = BIAS ? b.x.slices + ((size_t)bh * b.nnzb + jb) * (2 * BS) + tid : nullptr;   // of this row (piece)
        if constexpr (BIAS) {
            for (int i = tid; i < NT * 4 * kPlaces; i += BS * 4) all_places[i] = 0.f;
            for (int e = n + tid; e < n_all; e += BS * 4)   // what is not computed
                (my_slices - tid)[(size_t)e * (2 * BS) + 2 * BS - 1] = __builtin_bit_cast(float, kNoSlice);
        }
        const int packed = pack_cut(cuts, piece);   // one register over the loop
        if (n > 0) {
            const unsigned first = bucket;
            bucket = biases.request(jnext - I, tid);
            issue(ta1, tb1, jnext);   // the youngest load at step 0 (a one-block row loads its block twice)
            if constexpr (BIAS) {
                lds_meet();   // the table is there, the places are clear
                biases.put(bias0, first, tid);
            }
        }
        f32x4 dq[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) dq[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int slice_at = 4 * g - wave * 16 - r + BS - 1;   // of key 4 g of the block
        // the distances of the block of step t, from the waves' sums; the first wave's last number is where the block lies
        auto write_slice = [&](int t) {
            if (tid < 2 * BS) {
                const float* const from = sums + (t & 1) * (NT * 2 * BS) + tid;
                float v = from[0];
#pragma unroll
                for (int w = 1; w < NT; ++w) v += from[w * (2 * BS)];
                if (tid == 2 * BS - 1) v = from[0];
                my_slices[(size_t)(walk_index(t, pd_v) * (2 * BS))] = v;
            }
        };

        auto step = [&](const bf16_t* kt, const bf16_t* vt, bf16_t* tk, bf16_t* tv, const float* bias_c, float* bias_n, int it) {
            meet(it == 0);
            if (BIAS && it > 0) write_slice(it - 1);
            if constexpr (BIAS) biases.put(bias_n, bucket, tid);
            if (it > 0 && it + 1 < n) issue(tk, tv, jnext);
            const int jafter = later_col(it + 2);
            if constexpr (BIAS) bucket = biases.request(jafter - I, tid);
            f32x4 s[NT];
            float bias = 0.f;
            const bool one = !BIAS || one_bucket<BS>(bias_c, bias);
#pragma unroll
            for (int kt16 = 0; kt16 < NT; ++kt16) s[kt16] = f32x4{bias, bias, bias, bias};
            if (BIAS && !one) {
#pragma unroll
                for (int kt16 = 0; kt16 < NT; ++kt16)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[kt16][i] = bias_c[slice_at + 16 * kt16 + i];
            }
            bf16x8 kfr[NT][2], vfr[NT][2];
#pragma unroll
            for (int kt16 = 0; kt16 < NT; ++kt16)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    kfr[kt16][c] = *reinterpret_cast<const bf16x8*>(kt + kt16 * 16 * kD + sl.frag[c]);
                    vfr[kt16][c] = *reinterpret_cast<const bf16x8*>(vt + kt16 * 16 * kD + sl.frag[c]);
                }
            f32x4 dp[NT];
#pragma unroll
            for (int kt16 = 0; kt16 < NT; ++kt16) {
                // without dropout dP - delta comes out of the MFMA: the accumulator starts at -delta
                dp[kt16] = DROP ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{ndelta, ndelta, ndelta, ndelta};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    s[kt16] = mma_d(s[kt16], kfr[kt16][c], qf[c]);      // S^T = K Q^T
                    dp[kt16] = mma_d(dp[kt16], vfr[kt16][c], dof[c]);   // dP^T = V dO^T
                }
            }
            if (jcur * BS + BS > length) {   // the block that the sequence ends in
                const int left = length - jcur * BS - 4 * (once(lane) >> 4);
#pragma unroll
                for (int kt16 = 0; kt16 < NT; ++kt16)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (kt16 * 16 + i >= left) s[kt16][i] = -INFINITY;
            }
            // the generator's turn: the matrix cores have the scores to do
            [[maybe_unused]] unsigned factors[NT][2];
            if constexpr (DROP) {
                __builtin_amdgcn_sched_barrier(0);
                query_factors<NT>(draws, qrow, jcur * BS, g, below, factors);
                __builtin_amdgcn_sched_barrier(0);
            }
            // the transposed K operands of dQ^T += K^T dS^T for 32 keys: they land while the exponentials are computed
            bf16x8 kop[4];
            auto request_k = [&](int pc) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int o = sl.tr(j) + pc * 32 * kD;
                    kop[j] = join(lds_read_tr(kt + o), lds_read_tr(kt + 16 * kD + o));
                }
            };
            request_k(0);
            __builtin_amdgcn_sched_barrier(0);
            bf16x4 dsq[NT];
#pragma unroll
            for (int kt16 = 0; kt16 < NT; ++kt16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = fast_exp2(fmaf(s[kt16][i], scale_log2, -lse2));
                    s[kt16][i] = p * (DROP ? where_kept_plus(dp[kt16][i], factors[kt16], i, ndelta) : dp[kt16][i]);
                }
                dsq[kt16] = to_quad<bf16_t>(s[kt16]);
            }
#pragma unroll
            for (int pc = 0; pc < BS / 32; ++pc) {
                const bf16x8 ds = join(dsq[2 * pc], dsq[2 * pc + 1]);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) dq[dt] = mma_d(dq[dt], kop[dt], ds);   // dQ^T[d][query] += K^T dS^T
                if (pc + 1 < BS / 32) request_k(pc + 1);
            }
            if constexpr (BIAS) {
                const int l = once(lane);
                float* const mine = sums + ((it & 1) * NT + wave) * (2 * BS) + l;   // numbers l, l + 64, .. of the block's 2 BS
                const float place = l == 63 ? __int_as_float((jcur - I) * BS) : 0.f;   // for the last number
                if (one) {   // of one bucket: it does not matter which distance has what
                    f32x4 v = s[0];
#pragma unroll
                    for (int kt16 = 1; kt16 < NT; ++kt16) v += s[kt16];
                    float sum = (v[0] + v[1]) + (v[2] + v[3]);
                    if (BS == 64) {
                        mine[0] = sum;
                        mine[64] = place;
                    } else {
                        float lower, upper;
                        swap_halves32(sum, lower, upper);
                        mine[0] = l < 32 ? lower + upper : place;
                    }
                } else {
                    float u[NT + 1];
                    diagonal_sums<NT>(s, u);
                    float* const of_lane = places + (l >> 4) * (kPlaces + 4) - (l & 15) + 15;   // of lane group g, distance 4 g - r
#pragma unroll
                    for (int kt16 = 0; kt16 <= NT; ++kt16) of_lane[16 * kt16] = u[kt16];
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int t = 0; t < 2 * BS; t += 64) {
                        const int e = t + l - (BS - 16 - 16 * wave);   // place of this distance; a wave has those of its queries
                        float v = t + 64 == 2 * BS ? place : 0.f;
                        if (e >= 0 && e < 16 * NT + 15) {
                            v = places[e];
#pragma unroll
                            for (int gg = 1; gg < 4; ++gg) v += places[gg * kPlaces + e];
                        }
                        mine[t] = v;
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
            jcur = jnext;
            jnext = jafter;
        };

        for (int it = 0; it < n; it += 2) {
            step(ta0, tb0, ta1, tb1, bias0, bias1, it);
            if (it + 1 < n) step(ta1, tb1, ta0, tb0, bias1, bias0, it + 1);
        }
        // an empty row never waited for its early load: it must land before this workgroup's LDS is freed
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        if (BIAS && n > 0) {
            lds_meet();
            write_slice(n - 1);
        }
        const auto& z = args_again<BwdWith>();
        const int l = once(lane);
        const CutRow mine_of = unpack_cut(packed);
        if (mine_of.count > 1) {   // a long row in pieces: see attn_bf16_tiles.h
            constexpr int kPart = 8 * 128;   // eight pairs a lane
            const size_t first_slot = (size_t)bh * z.cut.slots + mine_of.slot;
            float* const parts = z.cut.parts + (first_slot * NT + wave) * kPart + l * 2;
            float* const mine = parts + (size_t)mine_of.piece * NT * kPart;
#pragma unroll
            for (int i = 0; i < 8; ++i) put_shared(mine + i * 128, dq[i / 2][i % 2 * 2], dq[i / 2][i % 2 * 2 + 1]);
            if (!last_to_arrive(z.cut.counters + first_slot, z.cut.tag, mine_of.count, reinterpret_cast<int*>(lse0))) return;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) dq[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int c = 0; c < mine_of.count; ++c) {
                float2 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = get_shared(parts + (size_t)c * NT * kPart + i * 128);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dq[i / 2][i % 2 * 2] += v[i].x;
                    dq[i / 2][i % 2 * 2 + 1] += v[i].y;
                }
            }
        }
        // Through the K tile of the stage that the last block did not use: every wave is past the barrier of the last step,
        // and the wave's own 2 KB of it were only ever written by the wave's own loads, which have all landed.
        bf16_t* patch = ((n & 1) ? ta1 : ta0) + wave * (16 * kD);
        const Rows out = {z.at.H, z.at.beside};
        store_rows_coalesced(patch, z.dQ + out.in_head(bh, z.L) + (size_t)(I * BS + wave * 16) * out.in_row(), out.in_row(), dq, z.scale, l);
        return;
    }

    // ============================================================================================
    // key side: work item idx of head bh.  {Q, dO} tiles and the rows' numbers of a block row in two stages.
    // ============================================================================================
    const auto& b = args_again<BwdWith>();   // this side's
    const Rows at = {b.at.H, b.at.beside};
    const int in_row = at.in_row(), out_row = at.out_row();   // elements between rows of Q, K, V and of O, dO
    const size_t head = at.in_head(bh, L), out_head = at.out_head(bh, L), vec = (size_t)bh * L;
    [[maybe_unused]] const ScoreDraws draws(DROP, b.x.rng, b.x.stream, bh);
    [[maybe_unused]] const unsigned below = both_halves(b.x.threshold - 1u);
    const float scale_log2 = b.scale_log2;
    const KeyItem item = key_item_lookup(b.col_ptr, nb, b.chunk, b.finest, idx, lane);
    if (item.J < 0) return;
    const int J = item.J, slot = item.slot;
    const int krow = J * BS + wave * 16 + r;
    // the item's block rows, one per lane (an item has at most 64 of them)
    static_assert(kChunkMax <= 64, "a key-side work item must fit one wave's lanes");
    int n = item.ke - item.kb;
    const int rows_v = n > 0 ? b.row_idx[item.kb + (lane < n ? lane : n - 1)] : 0;
    if (length < L) n = J * BS < length ? __popcll(__ballot(lane < n && rows_v * BS < length)) : 0;   // ascending
    const int last = n > 0 ? n - 1 : 0;
    auto row_at = [&](int t) { return __builtin_amdgcn_readlane(rows_v, t < last ? t : last); };

    const bf16_t *const Qh = b.Q + head, *const dOh = b.dO + out_head;
    const float *const lse_h = b.x.row_lse + vec, *const delta_h = b.x.row_delta + vec;
    // four tile loads per wave, plus one 4-byte-per-lane load in waves 0 and 1
    auto load_q = [&](bf16_t* qt, int I) {   // (offsets of the lane made here each time: registers are short)
        const TileLoadLane tli(wave, once(lane), in_row);
        tile_load_async(Qh + (size_t)I * BS * in_row, qt, wave, tli, tile_range<BS>(I * BS, length, in_row));
    };
    auto load_do = [&](bf16_t* dt_, int I) {
        const TileLoadLane tlo(wave, once(lane), out_row);
        tile_load_async(dOh + (size_t)I * BS * out_row, dt_, wave, tlo, tile_range<BS>(I * BS, length, out_row));
    };
    auto load_rows = [&](float* lse_s, float* del_s, int I) {
        if (wave < 2 && lane < BS)
            __builtin_amdgcn_global_load_lds((wave ? delta_h : lse_h) + (size_t)I * BS + once(lane), (lds_void_ptr)(wave ? del_s : lse_s), 4, 0, 0);
    };
    unsigned bucket = 0;
    int icur = 0, inext = 0;   // block row of steps it, it + 1
    column.put(tab, a.x, tid);
    if (n > 0) {
        icur = row_at(0);
        inext = row_at(1);
        const unsigned first = biases.request(J - icur, tid);
        bucket = biases.request(J - inext, tid);
        load_q(ta0, icur);
        load_do(tb0, icur);
        load_rows(lse0, del0, icur);
        if constexpr (BIAS) {
            lds_meet();   // the table is there
            biases.put(bias0, first, tid);
        }
    }
    // owned K / V fragments (step 0 waits for everything issued up to here)
    bf16x8 kf[2], vf[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const size_t off = head + (size_t)krow * in_row + c * 32 + g * 8;
        kf[c] = *reinterpret_cast<const bf16x8*>(b.K + off);
        vf[c] = *reinterpret_cast<const bf16x8*>(b.V + off);
    }
    f32x4 dk[4], dv[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
        dk[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int slice_at = wave * 16 + r - 4 * g + BS - 1;   // of query 4 g of the block

    auto step = [&](const bf16_t* qt, const bf16_t* dt_, const float* lse_s, const float* del_s, const float* bias_c, bf16_t* nq, bf16_t* nd,
                    float* nlse, float* ndel, float* bias_n, int it) {
        // everyone's part of block `it` has landed and the other stage is no longer read
        meet(false);
        constexpr bool kSpread = BS == 64;   // the next tiles are requested in two places, see the plain kernel
        const bool more = it + 1 < n;
        if (more) {
            if constexpr (BIAS) biases.put(bias_n, bucket, tid);
            load_q(nq, inext);
            load_rows(nlse, ndel, inext);
            if (!kSpread) load_do(nd, inext);
        }
        if constexpr (BIAS) bucket = biases.request(J - row_at(it + 2), tid);
        // 32 query rows at a time: S and dP of two 16-row tiles, then their share of dV and dK
        bf16x8 fq[2], fd[2];
        auto frags = [&](int qt16) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                fq[c] = *reinterpret_cast<const bf16x8*>(qt + qt16 * 16 * kD + sl.frag[c]);
                fd[c] = *reinterpret_cast<const bf16x8*>(dt_ + qt16 * 16 * kD + sl.frag[c]);
            }
        };
        auto opnd = [&](int pc, int j) {   // transposed operand of MFMA j of this 32-row group
            const bf16_t* tile = (j & 1) ? qt : dt_;
            const int o = sl.tr(j >> 1) + pc * 32 * kD;
            return join(lds_read_tr(tile + o), lds_read_tr(tile + 16 * kD + o));
        };
        float bias = 0.f;
        const bool one = !BIAS || one_bucket<BS>(bias_c, bias);
        frags(0);
#pragma unroll
        for (int pc = 0; pc < NT / 2; ++pc) {
            [[maybe_unused]] unsigned factors[2][2];
            if constexpr (DROP) {
                __builtin_amdgcn_sched_barrier(0);
                unsigned u[4];
                key_words(draws, icur * BS + 32 * pc, krow, g, u);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    factors[h][0] = kept(u[2 * h], below);
                    factors[h][1] = kept(u[2 * h + 1], below);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            bf16x4 pq[2], dsq[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int qt16 = 2 * pc + h;
                const f32x4 ndelta = *reinterpret_cast<const f32x4*>(&del_s[qt16 * 16 + 4 * g]);
                const f32x4 lse4 = *reinterpret_cast<const f32x4*>(&lse_s[qt16 * 16 + 4 * g]);   // log2 units
                f32x4 s = f32x4{bias, bias, bias, bias}, dp = DROP ? f32x4{0.f, 0.f, 0.f, 0.f} : ndelta;   // the MFMA returns dP - delta
                if (BIAS && !one) {
                    const float* const from = bias_c + slice_at - 16 * qt16;
                    s = f32x4{from[0], from[-1], from[-2], from[-3]};
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    s = mma_d(s, fq[c], kf[c]);     // S = Q K^T
                    dp = mma_d(dp, fd[c], vf[c]);   // dP = dO V^T
                }
                __builtin_amdgcn_sched_barrier(0);
                if (qt16 + 1 < NT) frags(qt16 + 1);   // lands while the exponentials below run
                __builtin_amdgcn_sched_barrier(0);
                f32x4 p, ds;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = fast_exp2(fmaf(s[i], scale_log2, -lse4[i]));
                    ds[i] = p[i] * (DROP ? where_kept_plus(dp[i], factors[h], i, ndelta[i]) : dp[i]);
                }
                pq[h] = to_quad<bf16_t>(p);
                if constexpr (DROP) pq[h] = drop(pq[h], factors[h]);
                dsq[h] = to_quad<bf16_t>(ds);
            }
            if (kSpread && pc == 0 && more) load_do(nd, inext);
            // dV^T[d][key] += dO^T P and dK^T[d][key] += Q^T dS for these 32 rows, interleaved
            const bf16x8 pf = join(pq[0], pq[1]), dsf = join(dsq[0], dsq[1]);
            bf16x8 ring[2];
            ring[0] = opnd(pc, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j + 1 < 8) ring[(j + 1) & 1] = opnd(pc, j + 1);
                __builtin_amdgcn_sched_barrier(0);
                if (j & 1) dk[j >> 1] = mma_d(dk[j >> 1], ring[j & 1], dsf);
                else dv[j >> 1] = mma_d(dv[j >> 1], ring[j & 1], pf);
            }
        }
        icur = inext;
        inext = row_at(it + 2);
    };

    for (int it = 0; it < n; it += 2) {
        step(ta0, tb0, lse0, del0, bias0, ta1, tb1, lse1, del1, bias1, it);
        if (it + 1 < n) step(ta1, tb1, lse1, del1, bias1, ta0, tb0, lse0, del0, bias0, it + 1);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVm0);   // the owned fragments of a column without kept rows

    const auto& z = args_again<BwdWith>();
    const int l = once(lane);
    if (slot >= 0) {
        // a chunk of a column: the last of them to arrive adds all of them up, in their order
        constexpr int kPart = 16 * 128;
        float* const parts = z.partial + (((size_t)bh * z.n_slots + item.first) * NT + wave) * kPart + l * 2;
        float* const mine = parts + (size_t)(slot - item.first) * NT * kPart;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            put_shared(mine + i * 128, dk[i / 2][i % 2 * 2], dk[i / 2][i % 2 * 2 + 1]);
            put_shared(mine + (8 + i) * 128, dv[i / 2][i % 2 * 2], dv[i / 2][i % 2 * 2 + 1]);
        }
        if (!last_to_arrive(z.counters + (size_t)bh * z.n_slots + item.first, z.tag, item.count, reinterpret_cast<int*>(lse0))) return;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
            dk[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
            dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        for (int c = 0; c < item.count; ++c) {
            float2 v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = get_shared(parts + (size_t)c * NT * kPart + i * 128);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dk[i / 2][i % 2 * 2] += v[i].x;
                dk[i / 2][i % 2 * 2 + 1] += v[i].y;
                dv[i / 2][i % 2 * 2] += v[8 + i].x;
                dv[i / 2][i % 2 * 2 + 1] += v[8 + i].y;
            }
        }
    }
    if (J * BS + wave * 16 + (l & 15) >= length)   // what memory holds there has gone into this key's sums alone
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) dk[dt] = dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    // through the stage the last block did not use, see the plain kernel
    const bool odd = (n & 1) != 0;   // last block in stage 0 -> stage 1 is free
    bf16_t* pa = (odd ? ta1 : ta0) + wave * (16 * kD);
    bf16_t* pb = (odd ? tb1 : tb0) + wave * (16 * kD);
    const Rows out = {z.at.H, z.at.beside};
    const size_t row0 = out.in_head(bh, z.L) + (size_t)(J * BS + wave * 16) * out.in_row();
    store_rows_coalesced(pa, z.dK + row0, out.in_row(), dk, DROP ? z.scale / kHalfOne : z.scale, l);
    store_rows_coalesced(pb, z.dV + row0, out.in_row(), dv, 1.f, l);
}

// Most kept rows of a work item, as in the plain kernel but 24 at least where the launch has enough to do beside the longest chain: a step does more here, and
// the partial tiles of a cut are as many.  16 / 24 / 32 rows, with bias and dropout, us: 15.9 steps a slot (16 heads x 4096, block 64, columns of up
// to 60 rows) 53.1 / 52.3 / 63, without tall columns 86 / 83.6 / 81; 15.4 (64 x 1024, block 32) 36.4 / 36.1 / 42, 53.4 / 51.8 / 50.7; 11.9 (12 x 4096) 41.6 /
// 46.6; 7.7 (32 x 1024) 26.4 / 28.0.
static int key_chunk_with(int BH, int bs, int nb, int nnzb) {
    const int c = key_chunk(BH, bs, nb, nnzb);
    return c < 24 && bwd_steps_per_slot(BH, bs, nb, nnzb) >= 15 ? 24 : c;
}

// The plan of the plain kernel: cuts, order and lengths of work items as there.
template <int BS>
hipError_t bwd_with_bf16(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, const void* dO, void* dQ, void* dK, void* dV, const int* row_ptr, const int* col_idx, const int* col_ptr,
                         const int* row_idx, int nnzb, void* workspace, hipStream_t st) {
    const BwdWorkspace ws(s.BH, s.bs, s.nb, nnzb, key_chunk_with(s.BH, BS, s.nb, nnzb), s.nb / 4, bwd_bf16_row_slots(s, nnzb));
    const int n_key_a = ws.w_first, n_key_c = ws.w_max - ws.w_first;
    RowCut cut;
    bwd_bf16_decide_row_cut(cut, s, nnzb);
    if (cut.slots && (long long)s.BH * (cut.slots + s.nb + ws.w_max) <= 0x7fffffffll) {
        cut.helpers = cut.slots - 1;
        cut.counters = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + ws.total);
        cut.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.row_parts);
    } else {
        cut = RowCut{};
        cut.longest = INT_MAX;
    }
    const long long items = cut.helpers + n_key_a + s.nb + n_key_c, total = s.BH * items;
    const int few = total <= 512;   // deal_heads()
    const long long grid = dealt(s.BH, items, few != 0);
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    const int sort_rows = total > bwd_resident(BS) && (nnzb >= 6 * s.nb || s.nb >= 8 * bwd_steps_per_slot(s.BH, BS, s.nb, nnzb));
    const long long at_once = bwd_resident(BS);
    const int finest = 3 * total <= at_once ? 0 : total <= at_once ? 1 : total <= 4 * at_once ? 2 : 4;
    const BwdWith args = {static_cast<const bf16_t*>(Q), static_cast<const bf16_t*>(K), static_cast<const bf16_t*>(V),
                          static_cast<const bf16_t*>(dO), static_cast<bf16_t*>(dQ), static_cast<bf16_t*>(dK), static_cast<bf16_t*>(dV),
                          row_ptr, col_idx, col_ptr, row_idx, reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.counter_bytes),
                          static_cast<unsigned long long*>(workspace), s.tag, Rows{x.H, s.heads_beside != 0}, x, cut, ws.n_slots, s.BH, s.L, s.nb,
                          nnzb, n_key_a, n_key_c, ws.w_first, ws.chunk, sort_rows, finest, few, s.scale, s.scale * kLog2e};
    auto launch = [&](auto kernel) { kernel<<<dim3((unsigned)grid), dim3(BS * 4), 0, st>>>(args); };
    if (x.table) {
        if (x.threshold) launch(attn_bwd_with_bf16_kernel<BS, true, true>);
        else launch(attn_bwd_with_bf16_kernel<BS, true, false>);
    } else {
        if (x.threshold) launch(attn_bwd_with_bf16_kernel<BS, false, true>);
        else launch(attn_bwd_with_bf16_kernel<BS, false, false>);
    }
    return hipGetLastError();
}
template hipError_t bwd_with_bf16<32>(const AttnShape&, const Extras&, const void*, const void*, const void*, const void*,
                                      void*, void*, void*, const int*, const int*, const int*, const int*, int, void*, hipStream_t);
template hipError_t bwd_with_bf16<64>(const AttnShape&, const Extras&, const void*, const void*, const void*, const void*,
                                      void*, void*, void*, const int*, const int*, const int*, const int*, int, void*, hipStream_t);

}  // namespace spion
