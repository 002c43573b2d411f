// The attention of attn_extras_kernels.hip (relative position bias, dropout, lengths) for bf16 and block size 32 or 64: the tile
// movement, work order and cuts of the plain bf16 kernels, with
//   - the biases of a block, one for each of its 2 BS - 1 distances, in LDS: two stages, as the tiles; what an accumulator of
//     S^T starts from is read from there (neighbouring lanes read neighbouring words);
//   - dropout factors made while the tiles are on their way;
//   - tiles whose rows from the sequence's length on come as zeros, whatever memory holds there: the loads' range ends with the sequence.
// WHOLE, where the backward pass may have a table's gradient to make (there is a table and o_rest; the call does not say whether the table is learned): the probabilities' rounding to bf16 goes through the product with V (and the sums) as
// well.  A row's delta comes from O, and its error is the same for all of the row's dS: over the far buckets, which have many keys of a row, it added
// up to 0.9e-3 of the table's gradient in the mean (bf16's own rounding of it is 1.7e-3).
//
// What it adds is vector work beside the products (seven rounds of Philox for eight draws, a sixteenth of a 64 x 64 block's a wave; 16
// biases a lane) and, where rows are short, the table's way into LDS before the first scores.  Kernel time, us, of the plain one, with lengths,
// bias, dropout, bias and dropout, and the last as WHOLE: 4 x 4 heads x 4096, block 64, 8 %, 16.9 / 18.9 / 21.5 / 24.5 / 26.5 / 30; 4 x 8 heads, 20.8 %,
// 47 / 50 / 58 / 72 / 76 / 92; 2 x 8 x 16320, 5 %, 92 / 107 / 121 / 150 / 157 / 186; 16 x 4 x 1024, block 32, 15 %, 13.0 / 15.8 / 20.4 / 20.1 / 25.0 / 28.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "attn_bf16_tiles.h"
#include "attn_common.h"
#include "attn_extras.h"
#include "attn_extras_bf16.h"
#include "spion_internal.h"

namespace spion {

namespace {

// p - q, exact where q is p rounded: a product of two pairs each takes one of q's halves off, in place of two instructions that widen and subtract.
__device__ __forceinline__ f32x4 without(f32x4 p, bf16x4 q) {
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    typedef unsigned Words __attribute__((ext_vector_type(2)));
    const Words w = __builtin_bit_cast(Words, q);
    unsigned first = 0x0000bf80u, second = 0xbf800000u;   // {-1, 0} and {0, -1}, in registers: as a constant the first comes out as -1.0 in 32 bits
    asm("" : "+s"(first), "+s"(second));
    const Pair even = __builtin_bit_cast(Pair, first), odd = __builtin_bit_cast(Pair, second);
    const unsigned w0 = w[0], w1 = w[1];
    const Pair lo = __builtin_bit_cast(Pair, w0), hi = __builtin_bit_cast(Pair, w1);
    return f32x4{__builtin_amdgcn_fdot2_f32_bf16(lo, even, p[0], false), __builtin_amdgcn_fdot2_f32_bf16(lo, odd, p[1], false),
                 __builtin_amdgcn_fdot2_f32_bf16(hi, even, p[2], false), __builtin_amdgcn_fdot2_f32_bf16(hi, odd, p[3], false)};
}

template <int BS>
struct KvTiles {
    bf16_t k[BS * kD];
    bf16_t v[BS * kD];
};

}  // namespace

// ------------------------------------------------------------------------------------------------
// forward
// ------------------------------------------------------------------------------------------------
struct FwdWith {
    const bf16_t *Q, *K, *V;
    bf16_t* O;
    float* LSE;
    const int *row_ptr, *col_idx;
    Rows at;
    Extras x;
    RowCut cut;
    int L, nb, heads, order;
    float scale_log2;
};

// In which order block rows start, see the launcher.
enum WithOrder { kInOrder, kDealtHeads, kLongestFirst };

template <int BS, bool BIAS, bool DROP, bool WHOLE>
__global__ __launch_bounds__(BS * 4, BS == 32 && DROP && !WHOLE ? 5 : 4) void attn_fwd_with_bf16_kernel(FwdWith a) {
    constexpr int NKT = BS / 16;
    __shared__ __attribute__((aligned(16))) KvTiles<BS> sm0, sm1;
    __shared__ __attribute__((aligned(16))) float bias0[kSlice<BS>], bias1[kSlice<BS>];
    __shared__ float tab[BIAS ? Extras::kMaxBuckets : 1];

    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int L = a.L;
    if (DROP && blockIdx.x == 0 && tid < 2 && a.x.rng_used) a.x.rng_used[tid] = a.x.rng[tid];

    // which block row, or piece of a long one
    int id = blockIdx.x;
    const bool helper = id < a.cut.groups;
    RowPieces cuts = {0, 1, 0, 0};
    int bh, I, piece = 0;
    if (helper) {
        const int all = a.heads * a.cut.helpers;
        if (id >= all) return;
        const int l = xcd_deal(id, 0, all), p = l % a.cut.helpers;
        cuts = row_pieces<false>(a.row_ptr, a.nb, a.cut, p, lane);
        if (cuts.row < 0) return;
        bh = l / a.cut.helpers;
        I = cuts.row;
        piece = p - cuts.first + 1;
    } else {
        id -= a.cut.groups;
        ItemOfHead mine;
        if (a.order == kInOrder) {
            const int vid = xcd_deal(id, 0, a.heads * a.nb);
            mine = {vid / a.nb, vid % a.nb};
        } else {
            mine = deal_heads(id, a.heads, false);
            if (mine.item >= a.nb) return;
            if (a.order == kLongestFirst) mine.item = row_by_length(a.row_ptr, a.nb, mine.item, lane);
        }
        bh = mine.head;
        I = mine.item;
    }

    const TableColumn<BS, BIAS> column(a.x, bh % a.x.H, tid);
    const BlockBias<BS, BIAS> biases(a.x, tab, L, wave);
    unsigned bucket = biases.request(0, tid);
    const size_t head = a.at.in_head(bh, L);
    const int row_len = a.at.in_row(), length = length_of(a.x, bh, L);
    const int qrow = I * BS + wave * 16 + r;
    const SwzLane sl(r, g);
    const TileLoadLane tl(wave, lane, row_len);
    const bf16_t *const Kh = a.K + head, *const Vh = a.V + head;
    auto issue = [&](KvTiles<BS>& st, int J) {
        const unsigned range = tile_range<BS>(J * BS, length, row_len);
        tile_load_async(Kh + (size_t)J * BS * row_len, st.k, wave, tl, range);
        tile_load_async(Vh + (size_t)J * BS * row_len, st.v, wave, tl, range);
    };
    if (!helper) issue(sm0, I);   // the diagonal block, before any index is known
    bf16x8 qf[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        qf[c] = *reinterpret_cast<const bf16x8*>(a.Q + head + (size_t)qrow * row_len + c * 32 + g * 8);
        if (qrow >= length) qf[c] = bf16x8{};
    }
    int jb = a.row_ptr[I], n = a.row_ptr[I + 1] - jb;   // blocks of this workgroup
    if (n > a.cut.longest) {
        if (!helper) cuts = row_pieces<true>(a.row_ptr, a.nb, a.cut, I, lane);
        const int from = piece * n / cuts.count;
        n = (piece + 1) * n / cuts.count - from;
        jb += from;
    }
    const int* cols = a.col_idx + jb;
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
    auto later_col = [&](int t) {   // t >= 2, one after the other
        const int u = t < last ? t : last;
        if (u >= 64 && (u & 63) == 0) walk_v = args_again<FwdWith>().col_idx[jb + walk_index(u + lane < last ? u + lane : last, pd)];
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
        issue(sm0, jcur);
    }
    // the second block goes out as soon as its index is known; it is the youngest load from here on
    const int packed = pack_cut(cuts, piece);   // one register over the loop
    if (n > 0) {
        const unsigned first = bucket;
        bucket = biases.request(jnext - I, tid);
        issue(sm1, jnext);   // (a one-block row loads its block twice: keeps the wait below uniform)
        if constexpr (BIAS) {
            lds_meet();   // the table is there
            biases.put(bias0, first, tid);
        }
    }
    [[maybe_unused]] const ScoreDraws draws(DROP, a.x.rng, a.x.stream, bh);
    [[maybe_unused]] const unsigned below = both_halves(a.x.threshold - 1u);
    const float scale_log2 = a.scale_log2;

    float m = kLowest;   // what the row's exponentials are taken against, log2 units
    f32x4 lacc = f32x4{0.f, 0.f, 0.f, 0.f};   // running row sum, replicated in its 4 elements
    f32x4 oacc[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)1.0f;
    const int slice_at = 4 * g - wave * 16 - r + BS - 1;   // of key 4 g of the block

    auto step = [&](const KvTiles<BS>& cur, KvTiles<BS>& tgt, const float* bias_c, float* bias_n, int it) {
        meet(it == 0);
        if constexpr (BIAS) biases.put(bias_n, bucket, tid);
        if (it > 0 && it + 1 < n) issue(tgt, jnext);
        const int jafter = later_col(it + 2);
        if constexpr (BIAS) bucket = biases.request(jafter - I, tid);
        // S^T tile kt: [key 16 kt + 4 g + i][query r]; all K fragments are requested up front
        bf16x8 kfr[NKT][2];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                kfr[kt][c] = *reinterpret_cast<const bf16x8*>(cur.k + kt * 16 * kD + sl.frag[c]);
        f32x4 s[NKT];
        float bias = 0.f;
        const bool one = !BIAS || one_bucket<BS>(bias_c, bias);
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) s[kt] = f32x4{bias, bias, bias, bias};
        if (BIAS && !one) {
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[kt][i] = bias_c[slice_at + 16 * kt + i];
        }
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int c = 0; c < 2; ++c) s[kt] = mma_d(s[kt], kfr[kt][c], qf[c]);
        if (jcur * BS + BS > length) {   // the block that the sequence ends in
            const int left = length - jcur * BS - 4 * (once(lane) >> 4);
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (kt * 16 + i >= left) s[kt][i] = -INFINITY;
        }
        // the generator's turn: the matrix cores have the scores to do
        [[maybe_unused]] unsigned factors[NKT][2];
        auto make_factors = [&]() {
            __builtin_amdgcn_sched_barrier(0);
            query_factors<NKT>(draws, qrow, jcur * BS, g, below, factors);
            __builtin_amdgcn_sched_barrier(0);
        };
        if constexpr (DROP && !WHOLE) make_factors();   // (else there is no room for them yet)
        // the transposed V operands of O^T += V^T P^T for 32 keys: requested here, they land while the exponentials are computed
        bf16x8 vop[4];
        auto request_v = [&](int pc) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int o = sl.tr(j) + pc * 32 * kD;
                vop[j] = join(lds_read_tr(cur.v + o), lds_read_tr(cur.v + 16 * kD + o));
            }
        };
        request_v(0);
        __builtin_amdgcn_sched_barrier(0);
        bf16x4 pq[NKT];
        [[maybe_unused]] bf16x4 rest[NKT];
        f32x4 sums;
        auto probabilities = [&]() {   // and their sums, see the plain kernel
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) {
                f32x4 p;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = fast_exp2(fmaf(s[kt][i], scale_log2, -m));
                pq[kt] = to_quad<bf16_t>(p);
                if constexpr (WHOLE) rest[kt] = to_quad<bf16_t>(without(p, pq[kt]));
            }
            sums = lacc;
#pragma unroll
            for (int pc = 0; pc < BS / 32; ++pc) {
                sums = mma_d(sums, ones, join(pq[2 * pc], pq[2 * pc + 1]));
                if constexpr (WHOLE) sums = mma_d(sums, ones, join(rest[2 * pc], rest[2 * pc + 1]));
            }
        };
        if (it > 0) probabilities();
        if (it == 0 || __any(!(sums[0] <= kSumLimit))) {
            float mx = s[0][0];
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[kt][i]);
            float m_new = fmaxf(m, group_max(mx) * scale_log2);
            if (lacc[0] > 1.f) m_new = fmaxf(m_new, m + log2f(lacc[0]));   // a sum that many blocks have added up to
            const float alpha = fast_exp2(m - m_new);
            m = m_new;
            lacc *= alpha;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) oacc[dt] *= alpha;
            probabilities();
        }
        lacc = sums;
        if constexpr (DROP && WHOLE) make_factors();
        if constexpr (DROP) {   // behind the sums: the softmax is over all of them
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) {
                pq[kt] = drop(pq[kt], factors[kt]);
                if constexpr (WHOLE) rest[kt] = drop(rest[kt], factors[kt]);
            }
        }
#pragma unroll
        for (int pc = 0; pc < BS / 32; ++pc) {
            const bf16x8 p = join(pq[2 * pc], pq[2 * pc + 1]);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) oacc[dt] = mma_d(oacc[dt], vop[dt], p);   // O^T[d][query] += V^T P^T
            if constexpr (WHOLE) {
                const bf16x8 q = join(rest[2 * pc], rest[2 * pc + 1]);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) oacc[dt] = mma_d(oacc[dt], vop[dt], q);
            }
            if (pc + 1 < BS / 32) request_v(pc + 1);
        }
        jcur = jnext;
        jnext = jafter;
    };

    for (int it = 0; it < n; it += 2) {
        step(sm0, sm1, bias0, bias1, it);
        if (it + 1 < n) step(sm1, sm0, bias1, bias0, it + 1);
    }

    // an empty row never waited for its early load: it must land before this workgroup's LDS is freed
    __builtin_amdgcn_s_waitcnt(kWaitVm0);

    const auto& z = args_again<FwdWith>();
    const int l = once(lane), qrow_l = I * BS + wave * 16 + (l & 15);
    const CutRow mine_of = unpack_cut(packed);
    if (mine_of.count > 1) {   // a long row in pieces: see attn_bf16_tiles.h
        constexpr int kPart = 64 * 18;   // floats of a wave: nine pairs a lane, its accumulators, then reference and sum
        const size_t slot = (size_t)bh * z.cut.slots + mine_of.slot;
        float* const parts = z.cut.parts + (slot * (BS / 16) + wave) * kPart + l * 2;
        float* const mine = parts + (size_t)mine_of.piece * (BS / 16) * kPart;
#pragma unroll
        for (int i = 0; i < 8; ++i) put_shared(mine + i * 128, oacc[i / 2][i % 2 * 2], oacc[i / 2][i % 2 * 2 + 1]);
        put_shared(mine + 1024, m, lacc[0]);
        if (!last_to_arrive(z.cut.counters + slot, z.cut.tag, mine_of.count, reinterpret_cast<int*>(sm0.v))) return;
        m = -INFINITY;
        lacc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int c = 0; c < mine_of.count; ++c) {
            const float* const part = parts + (size_t)c * (BS / 16) * kPart;
            float2 v[9];
#pragma unroll
            for (int i = 0; i < 9; ++i) v[i] = get_shared(part + i * 128);
            const float m_new = fmaxf(m, v[8].x), down = fast_exp2(m - m_new), up = fast_exp2(v[8].x - m_new);
            m = m_new;
            lacc = lacc * down + v[8].y * up;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = i % 2 * 2;
                oacc[i / 2][e] = oacc[i / 2][e] * down + v[i].x * up;
                oacc[i / 2][e + 1] = oacc[i / 2][e + 1] * down + v[i].y * up;
            }
        }
    }
    const float lsum = lacc[0];
    const bool none = lsum == 0.f || qrow_l >= length;
    const float inv = none ? 0.f : (DROP ? z.x.keep_scale : 1.f) / lsum;
    // the stage that the last block did not use is free, see the plain kernel
    bf16_t* patch = ((n & 1) ? sm1.k : sm0.k) + wave * (16 * kD);
    const Rows at = {z.at.H, z.at.beside};
    const size_t row0 = at.out_head(bh, z.L) + (size_t)(I * BS + wave * 16) * at.out_row();
    store_rows_coalesced(patch, z.O + row0, at.out_row(), oacc, inv, l);
    if (z.x.rest) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) oacc[dt][i] = rounded_off<bf16_t>(oacc[dt][i] * inv);
        store_rows_coalesced(patch, static_cast<bf16_t*>(z.x.rest) + row0, at.out_row(), oacc, 1.f, l);
    }
    if (l < 16) z.LSE[(size_t)bh * z.L + qrow_l] = none ? -INFINITY : (m + log2f(lsum)) * kLn2;
}

static int resident(int bs) { return 256 * (bs == 64 ? 4 : 8); }

// Order of the rows and their cuts: the plain kernel's rules.
template <int BS>
hipError_t fwd_with_bf16(const AttnShape& s, const Extras& x, const void* Q, const void* K, const void* V, void* O, float* LSE,
                         const int* row_ptr, const int* col_idx, int nnzb, hipStream_t st) {
    const int total = s.nb * s.BH;
    RowCut cut;
    if (s.fwd_room) cut = RowCut(s, nnzb);
    if (cut.slots) {   // a helper for each piece
        cut.helpers = cut.slots - 1;
        cut.groups = (s.BH * cut.helpers + 7) & ~7;
    } else {
        cut = RowCut{};
        cut.longest = INT_MAX;
    }
    const bool short_rows = BS == 32 ? nnzb < 6 * s.nb && 4 * total >= 5 * resident(BS) : nnzb < 4 * s.nb && total >= 2 * resident(BS);
    const WithOrder order = !short_rows && (total > resident(BS) || (total > 256 && nnzb >= 6 * s.nb)) ? kLongestFirst
                            : !short_rows && total > (BS == 64 ? 512 : 768) && 2 * nnzb >= 3 * s.nb   ? kDealtHeads
                                                                                                        : kInOrder;
    const long long grid = cut.groups + (order == kInOrder ? total : dealt(s.BH, s.nb, false));
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    const FwdWith args = {static_cast<const bf16_t*>(Q), static_cast<const bf16_t*>(K), static_cast<const bf16_t*>(V), static_cast<bf16_t*>(O), LSE,
                          row_ptr, col_idx, Rows{x.H, s.heads_beside != 0}, x, cut, s.L, s.nb, s.BH, order, s.scale * kLog2e};
    auto launch = [&](auto kernel) { kernel<<<dim3((unsigned)grid), dim3(BS * 4), 0, st>>>(args); };
    if (x.table && x.rest) {   // a gradient of the table may follow
        if (x.threshold) launch(attn_fwd_with_bf16_kernel<BS, true, true, true>);
        else launch(attn_fwd_with_bf16_kernel<BS, true, false, true>);
    } else if (x.table) {
        if (x.threshold) launch(attn_fwd_with_bf16_kernel<BS, true, true, false>);
        else launch(attn_fwd_with_bf16_kernel<BS, true, false, false>);
    } else {
        if (x.threshold) launch(attn_fwd_with_bf16_kernel<BS, false, true, false>);
        else launch(attn_fwd_with_bf16_kernel<BS, false, false, false>);
    }
    return hipGetLastError();
}
template hipError_t fwd_with_bf16<32>(const AttnShape&, const Extras&, const void*, const void*, const void*, void*, float*, const int*, const int*,
                                      int, hipStream_t);
template hipError_t fwd_with_bf16<64>(const AttnShape&, const Extras&, const void*, const void*, const void*, void*, float*, const int*, const int*,
                                      int, hipStream_t);

}  // namespace spion
