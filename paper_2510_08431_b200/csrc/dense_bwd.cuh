// Gradients of dense attention, with a causal mask, key lengths and key heads that several query heads share.  For a query i and a
// key j that it sees,
//     P = exp(s q.k - LSE_i),  dP = dO_i . v_j,  delta_i = dO_i . O_i,  dS = P (dP - delta_i)
//     dQ_i = s sum_j dS k_j,   dK_j = s sum_i dS q_i,   dV_j = sum_i P dO_i,     dK, dV summed over the heads that share theirs
// The formulas and the two passes are those of sparse_bwd.cuh: kDkv keeps K, V of a key block and streams the query blocks by (of one sharing head
// after the other, into the same accumulators), kDq keeps Q, dO of a query block and streams the key blocks; no atomics, so a gradient is the same from run to run.
//
// Score buffers in tensor memory (512 columns: kDkv has two accumulators of D columns, kDq one): three where they fit -- matrix 2 T is S_T, 2 T + 1 is dP_T,
// matrix m is in buffer m % 3 -- and two in kDkv at D = 128.  P^T overwrites S and dS^T (kDq: dS) overwrites dP as bf16 operands, and the next matrix goes into a
// buffer behind the product that reads it:
//     kDkv, three:  dV += P_j dO_j, dP_(j+1) = V dO_(j+1)^T   |   dK += dS_j Q_j, S_(j+2) = K Q_(j+2)^T
//     kDkv, two:    dV += P_j dO_j, S_(j+1)                   |   dK += dS_j Q_j, dP_(j+1)
//     kDq:          dP_(j+1) as soon as S_j has been read     |   dQ += dS_j K_j, S_(j+2)
// All score warps share a tile, some columns each, so that what the next tile needs is handed over early and the MMAs run a tile ahead of them.  kDq takes S and
// dP together, kDkv hands P over before it looks at dP.
//
// CTAs are persistent, one per SM, and draw their items (stationary blocks, or parts of their tiles where there are few) from a counter; tiles are
// numbered T = 0, 1, ... over all items and run on without a break.
//
// What bounds it.  Of the 14 D operations per pair of a training pass the gradients count 10 D, as five products; they take seven, since dQ runs over keys and
// dK, dV over queries, so that both passes form S and dP, and adding dQ up by atomics would make it differ from run to run.  At D = 128 a product of a tile is 512 cycles of
// the tensor pipe: a tile of kDkv takes 3100 to 3300 for its four, with P and dS handed over in two buffers, of kDq 2000 to 2300 for its three; in long runs the
// power limit takes the rest: 12 heads of 32760 tokens 18.0 ms, 916 TF of what counts, 1280 with what is done twice.  At D = 64 (256 cycles a product) the scores
// set the pace, an exponential, a difference, a product and two roundings per pair: 2350 and 1980 cycles a tile; 2 x 24 / 6 causal heads of 4001 tokens, keys 4001 and 3277: 410 us.
#pragma once

#include "attn_jvp_kernel.cuh"
#include "sparse_bwd.cuh"

namespace attn_jvp {

constexpr int kDenseBlock = 128;
// Warps 0..3: MMA issue and loads; then the score warps, and four epilogue warps.  At D = 64, where the scores set the pace, four score warps to a scheduler, 32 columns
// of a tile each; at D = 128, where they take issue slots from the warp that feeds the tensor pipe, two, 64 columns each (D = 64, the causal case above when this
// was taken: 413 us with four, 453 with two; 12 heads of 32760 at D = 128: 18.3 ms with two, 19.1 with four, though four are 4 % faster on items of four tiles).
// Registers per thread: those of the launch, which setmaxnreg shares out anew.
template <int D>
struct DenseRoles {
    static constexpr int kScoreWarps = D == 64 ? 16 : 8, kEpilogueWarps = 4;
    static constexpr int kThreads = 32 * (4 + kScoreWarps + kEpilogueWarps);
    static constexpr int kCols = 512 / kScoreWarps;              // of a tile, per score warp
    static constexpr int kRegsLaunch = D == 64 ? 80 : 128;
    static constexpr int kRegsLight = 64, kRegsScore = D == 64 ? 88 : 200, kRegsEpilogue = D == 64 ? 64 : 48;
    static_assert(128 * kRegsLight + 32 * kScoreWarps * kRegsScore + 32 * kEpilogueWarps * kRegsEpilogue <= kThreads * kRegsLaunch, "registers");
};
struct DenseBwdArgs {
    // kDkv: X1, X2 = K, V of the block, Y1, Y2 = Q, dO.  kDq: X1, X2 = Q, dO; Y1, Y2 = K, V.  S = X1 Y1^T, dP = X2 Y2^T (rows: the stationary side); dV += P Y2,
    // dK += dS Y1, dQ += dS Y1.  tail1, tail2: kDq, K and V of the block in which a batch's keys end, [B][128][heads][D], zeros behind the end.
    alignas(64) CUtensorMap x1, x2, y1, y2, tail1, tail2;
    const float* rows;          // [B][heads of Q][n_q][2][128]: per block of queries -LSE log2 e (-inf: no probability), then -delta
    __nv_bfloat16* out1;        // kDkv: dV, kDq: dQ        [B][L][heads][D]
    __nv_bfloat16* out2;        // kDkv: dK
    float* part;                // splits > 1: [splits][n_items][rows of an item][kDkv: dV, dK; kDq: dQ] in fp32, which dense_join_kernel adds
    int* host_status;
    int* counter;               // items handed out beyond the first one of every CTA; starts at 0
    KeyMask mask;               // window: in items
    int H;                      // heads of the stationary side
    int n_items, n_items_per_head;
    int splits;                 // parts that an item's tiles are cut into
    int L_own, Lq, Lk, n_q;
    int wide_out;               // out1, out2 are 32-byte aligned
    float scale, scale_log2;
};
// The tiles of an item.  kDkv: count query blocks from `first` on, for each of the heads that share the key head in turn, n = group count.  kDq:
// key blocks 0 .. n - 1.  len: the keys of the batch.
struct DenseSpan { int n, len, first, count; };
template <bool kDkv>
__device__ __forceinline__ DenseSpan dense_span(const DenseBwdArgs& a, int item) {
    const int bh = item / a.n_items_per_head, x0 = (item - bh * a.n_items_per_head) * kDenseBlock;
    DenseSpan s;
    s.len = a.mask.lengths == nullptr ? a.Lk : min(max(__ldg(a.mask.lengths + bh / a.H), 0), a.Lk);
    s.first = 0;
    if (kDkv) {
        if (a.mask.causal) s.first = max(0, x0 - a.mask.offset) / kDenseBlock;       // the first query that sees key x0
        s.count = x0 < s.len ? max(0, a.n_q - s.first) : 0;
        s.n = s.count * a.mask.group;
    } else {
        const int seen = a.mask.causal ? min(s.len, max(0, min(x0 + kDenseBlock, a.Lq) + a.mask.offset)) : s.len;
        s.n = s.count = (seen + kDenseBlock - 1) / kDenseBlock;
    }
    return s;
}
// the first tile of part i (n at most 10^7, splits 16)
__device__ __forceinline__ int part_begin(int n, int i, int splits) { return n * i / splits; }

// Shared memory: the stationary operands, rings of the streaming ones, LSE and delta of kRowSets tiles (kDkv).
template <int D, bool kDkv>
struct DenseBwdPlan {
    static constexpr int kTile = 128 * D * 2;                    // a 128 x D operand
    static constexpr int kY1 = D == 128 ? 3 : (kDkv ? 5 : 4), kY2 = D == 128 ? 2 : (kDkv ? 5 : 4);
    static constexpr int kRowSets = D == 128 ? 2 : 4;
    static constexpr int kY1Off = 2 * kTile;
    static constexpr int kY2Off = kY1Off + kY1 * kTile;
    static constexpr int kRowsOff = kY2Off + kY2 * kTile;
    static constexpr int kRowsBytes = kDenseBlock * 8;
    static constexpr int kDynBytes = kRowsOff + (kDkv ? kRowSets * kRowsBytes : 0);      // 226 KB in kDkv at D = 128
};

// ---------------------------------------------------------------------------------------------
// Before and after the passes
// ---------------------------------------------------------------------------------------------
// The passes are launched as programmatic dependents.  kDkv is set up beside the preparation and waits for its end.  kDq depends on the
// preparation alone, which is over once every CTA of kDkv has got past that wait and said so: its CTAs start on the SMs that kDkv leaves (or never
// took), and wait for kDkv's end only before they leave, so that what comes after them in the stream comes after both.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Blocks below `row_blocks`: -LSE log2 e and -delta per query row, padded to whole blocks; rows behind the last query and rows without any key get
// -inf, which makes their P exactly 0; a group of D / 8 threads per row reads dO and O once. Then (lengths given) a block per batch and key head, which
// copies the keys and values of the block in which the batch ends with zeros behind the end: the products of kDq would otherwise take up what lies there.
// Both passes' counters start at 0.  (delta of rows that see few keys: below.)
struct DenseBwdPrep {
    const uint4 *o, *d_o;
    const float* lse;
    float* rows;
    const __nv_bfloat16 *k, *v;
    long long k_b, k_l, k_h, v_b, v_l, v_h;      // strides
    __nv_bfloat16 *tail_k, *tail_v;
    int* counters;
    const __nv_bfloat16* q;
    long long q_b, q_l, q_h;
    const int* lengths;
    int B, H, Hk, Lq, Lk, n_q, row_blocks;
    int causal, offset;
    float scale_log2;
};
// O comes in bf16, and its products took the exponentials in bf16: delta is off by some 2^-9 of the root of sum (dO O)^2, which moves dS = P (dP - delta) by P times that.  How much it shows hangs on
// the size of O beside that of the values, so on how few keys hold a row's probability, not on how many it sees.  Errors of dQ in the 2-norm over unit-normal keys and
// values (dK alike, dV 0.0024 throughout; with an exact delta 0.0024 throughout, which are the roundings of dS and of the result), D = 64:
//     queries of      1      2      4      8    times unit size            (mean largest probability over 512 keys: 0.03, 0.14, 0.45, 0.72)
//       13 keys    0.0026 0.0032 0.0044 0.0057
//       64         0.0025 0.0028 0.0038 0.0050
//      512         0.0024 0.0028 0.0037 0.0055
//     4096         0.0024 0.0026 0.0035 0.0052
// An exact delta for every row would take S and dP of all its keys before the passes: two more products beside the seven.  An O that is not rounded would not do: the
// exponentials in bf16 alone leave up to 0.005 at 512 keys and 8 times unit size (modelled, with the forward's reference up to 5 below a row's maximum).
// Rows that see at most kExactKeys keys always have a large O (of two keys 0.0036, with unit-normal queries) and are cheap to form anew, from fp32 scores:
// delta = sum_j P_j (dO . v_j).  Blocks walk over the query blocks that can have such rows (a causal mask: the first of a head; lengths: any), in a kernel of its
// own beside the preparation, whose registers it would double.  Costs 1 % where a mask leaves few such rows or none (gradients of the causal case
// 407 -> 410 us; 3 x 16 heads of 8190 queries, keys 77 / 0 / 512, 218 -> 221), more than the rest where all rows are (2 x 16 heads of 8190 queries and 12 keys: 138 -> 340,
// for errors that go from 0.0025 to 0.0024).
constexpr int kExactKeys = 12;
// the keys that query l sees of a batch's `len` where they are few, else 0
__device__ __forceinline__ int few_keys(const DenseBwdPrep& p, int len, int l) {
    const int seen = p.causal ? min(len, l + 1 + p.offset) : len;
    return seen > 0 && seen <= kExactKeys ? seen : 0;
}
template <int D>
__global__ void __launch_bounds__(256)
dense_bwd_few_kernel(const __grid_constant__ DenseBwdPrep p, int blocks) {
    constexpr int kLanes = D / 8;
    grid_launch_dependents();
    const int sub = threadIdx.x % kLanes;
    for (int i = blockIdx.x; i < p.B * p.H * blocks; i += gridDim.x) {
        const int bh = i / blocks, b = bh / p.H, h = bh - b * p.H, hk = h / (p.H / p.Hk);
        const int len = p.lengths == nullptr ? p.Lk : min(__ldg(p.lengths + b), p.Lk);
        if (len <= 0 || (!p.causal && len > kExactKeys)) continue;
        const int l0 = (i - bh * blocks) * kDenseBlock + threadIdx.x / kLanes;
#pragma unroll 1
        for (int l = l0; l < l0 + kDenseBlock; l += 256 / kLanes) {
            const int seen = l < p.Lq ? few_keys(p, len, l) : 0;
            const int most = __reduce_max_sync(0xffffffffu, seen);   // (the shuffles need whole warps)
            if (most <= 0) continue;
            uint4 qv = make_uint4(0u, 0u, 0u, 0u), gv = qv;
            float ls = -INFINITY;
            if (seen > 0) {
                qv = __ldg(reinterpret_cast<const uint4*>(p.q + b * p.q_b + l * p.q_l + h * p.q_h + sub * 8));
                gv = __ldg(p.d_o + ((static_cast<long long>(b) * p.Lq + l) * p.H + h) * kLanes + sub);
                ls = __ldg(p.lse + static_cast<long long>(bh) * p.Lq + l) * -1.4426950408889634f;
                if (ls == INFINITY) ls = -INFINITY;
            }
            auto dot = [](const uint4& x, const uint4& y) {
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), v);
                    v = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), v);
                }
#pragma unroll
                for (int m = kLanes / 2; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
                return v;
            };
            float delta = 0.0f;
            for (int j0 = 0; j0 < most; j0 += 4) {                   // (loads of four keys in flight)
                uint4 k[4], v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (j0 + i < seen) {
                        k[i] = __ldg(reinterpret_cast<const uint4*>(p.k + b * p.k_b + (j0 + i) * p.k_l + hk * p.k_h + sub * 8));
                        v[i] = __ldg(reinterpret_cast<const uint4*>(p.v + b * p.v_b + (j0 + i) * p.v_l + hk * p.v_h + sub * 8));
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float score = dot(qv, k[i]), dp = dot(gv, v[i]);
                    if (j0 + i < seen) delta = fmaf(ex2f(fmaf(score, p.scale_log2, ls)), dp, delta);
                }
            }
            if (sub == 0 && seen > 0) p.rows[(static_cast<long long>(bh) * p.n_q + l / kDenseBlock) * (2 * kDenseBlock) + kDenseBlock + l % kDenseBlock] = -delta;
        }
    }
}
// (40 heads of 32760 queries: 108 us = 6.2 TB/s; with blocks of one turn and four heads per thread 136)
constexpr int kPrepTurns = 8;
template <int D>
constexpr int kPrepHeads = 256 / (D / 8) / 8;
template <int D>
__global__ void __launch_bounds__(256)
dense_bwd_prep_kernel(const __grid_constant__ DenseBwdPrep p) {
    constexpr int kLanes = D / 8;
    grid_launch_dependents();
    if (static_cast<int>(blockIdx.x) >= p.row_blocks) {
        const int Hk = p.Hk, bh = blockIdx.x - p.row_blocks, b = bh / Hk, h = bh - b * Hk;
        const int len = min(max(__ldg(p.lengths + b), 0), p.Lk), r0 = len / kDenseBlock * kDenseBlock;
        for (int e = threadIdx.x; len != r0 && len != p.Lk && e < kDenseBlock * kLanes; e += 256) {
            const int r = e / kLanes, c = e % kLanes * 8;
            uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
            if (r0 + r < len) {
                k = __ldg(reinterpret_cast<const uint4*>(p.k + b * p.k_b + (r0 + r) * p.k_l + h * p.k_h + c));
                v = __ldg(reinterpret_cast<const uint4*>(p.v + b * p.v_b + (r0 + r) * p.v_l + h * p.v_h + c));
            }
            const long long at = ((static_cast<long long>(b) * kDenseBlock + r) * Hk + h) * D + c;
            *reinterpret_cast<uint4*>(p.tail_k + at) = k;
            *reinterpret_cast<uint4*>(p.tail_v + at) = v;
        }
        grid_dependency_wait();
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) p.counters[threadIdx.x] = 0;
    // A CTA takes kPrepTurns times eight queries of kPrepHeads heads (what eight queries write fills sectors of `rows`), each turn's loads beside the sums of the one before.
    const unsigned head_groups = (p.H + kPrepHeads<D> - 1) / kPrepHeads<D>, groups = p.n_q * (kDenseBlock / 8 / kPrepTurns);
    const unsigned bl = blockIdx.x / head_groups, b = bl / groups;
    const int len = p.lengths == nullptr ? p.Lk : min(__ldg(p.lengths + b), p.Lk);
    if (len <= 0) {                                              // (no pass looks at a batch without keys)
        grid_dependency_wait();
        return;
    }
    const unsigned group = threadIdx.x / kLanes, sub = threadIdx.x % kLanes;
    const unsigned l0 = (bl - b * groups) * (8 * kPrepTurns) + group % 8, h = (blockIdx.x - bl * head_groups) * kPrepHeads<D> + group / 8;
    const bool mine = h < static_cast<unsigned>(p.H);
    const long long bh = static_cast<long long>(b) * p.H + h;
    uint4 x[2], y[2];
    auto fetch = [&](unsigned l, uint4& xs, uint4& ys) {
        xs = ys = make_uint4(0u, 0u, 0u, 0u);
        if (mine && l < static_cast<unsigned>(p.Lq)) {
            const long long at = ((static_cast<long long>(b) * p.Lq + l) * p.H + h) * kLanes + sub;
            xs = __ldg(p.o + at);
            ys = __ldg(p.d_o + at);
        }
    };
    fetch(l0, x[0], y[0]);
#pragma unroll
    for (int turn = 0; turn < kPrepTurns; ++turn) {
        const unsigned l = l0 + 8 * turn;
        if (turn + 1 < kPrepTurns) fetch(l + 8, x[(turn + 1) & 1], y[(turn + 1) & 1]);
        const uint4 xv = x[turn & 1], yv = y[turn & 1];
        const uint32_t xs[4] = {xv.x, xv.y, xv.z, xv.w}, ys[4] = {yv.x, yv.y, yv.z, yv.w};
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), sum);
            sum = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), sum);
        }
#pragma unroll
        for (int m = kLanes / 2; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if (sub == 0 && mine) {
            float ls = -INFINITY;
            if (l < static_cast<unsigned>(p.Lq)) {
                ls = p.lse[bh * p.Lq + l] * -1.4426950408889634f;
                if (ls == INFINITY) ls = -INFINITY;
            }
            float* out = p.rows + (bh * p.n_q + l / kDenseBlock) * (2 * kDenseBlock) + l % kDenseBlock;
            out[0] = ls;
            if (few_keys(p, len, l) == 0 || l >= static_cast<unsigned>(p.Lq)) out[kDenseBlock] = -sum;
        }
    }
    grid_dependency_wait();                                      // (for dense_bwd_few_kernel, if it was launched: the end of this grid is then the end of both)
}

// Adds the parts of split items in a fixed order: eight columns per thread.
template <int D, bool kDkv>
__global__ void __launch_bounds__(256)
dense_join_kernel(const __grid_constant__ DenseBwdArgs a) {
    constexpr int kCols = kDkv ? 2 * D : D, kPerRow = kCols / 8, kRows = kDenseBlock, kBlocks = kRows * kPerRow / 256;
    const int item = blockIdx.x / kBlocks;
    const int e = (blockIdx.x % kBlocks) * 256 + threadIdx.x, row = e / kPerRow, c = e % kPerRow * 8;
    const DenseSpan span = dense_span<kDkv>(a, item);
    const int bh = item / a.n_items_per_head, b = bh / a.H, h = bh - b * a.H, r = (item - bh * a.n_items_per_head) * kRows + row;
    if (r >= a.L_own) return;
    float sum[8] = {};
    if (span.n > 0 && (!kDkv || r < span.len)) {
#pragma unroll 4
        for (int i = 0; i < a.splits; ++i) {
            const bool there = part_begin(span.n, i, a.splits) < part_begin(span.n, i + 1, a.splits);      // (a part without tiles was never written)
            const float4* at = reinterpret_cast<const float4*>(a.part + ((static_cast<long long>(i) * a.n_items + item) * kRows + row) * kCols + c);
            const float4 none = make_float4(0.0f, 0.0f, 0.0f, 0.0f), x = there ? __ldg(at) : none, y = there ? __ldg(at + 1) : none;
            sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
            sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
        }
    }
    const bool second = kDkv && c >= D;
    const float factor = (kDkv && !second) ? 1.0f : a.scale;
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16(sum[2 * i] * factor, sum[2 * i + 1] * factor);
    const long long at = ((static_cast<long long>(b) * a.L_own + r) * a.H + h) * D + (second ? c - D : c);
    *reinterpret_cast<uint4*>((second ? a.out2 : a.out1) + at) = make_uint4(v[0], v[1], v[2], v[3]);
}

// ---------------------------------------------------------------------------------------------
// The passes.  Warp 0 (kDq: and warp 2) issues the MMAs, warp 1 the TMA loads, warp 3 writes the zero gradients of items that see nothing or that nothing
// sees (beside the MMAs: as blocks of the preparation, before them, 3 x 16 heads of 8190 queries with keys 77 / 0 / 512 235 us against 226); the score and epilogue warps are those of DenseRoles.
// ---------------------------------------------------------------------------------------------
template <int D, bool kDkv>
__global__ void __launch_bounds__(DenseRoles<D>::kThreads, 1)
dense_bwd_kernel(const __grid_constant__ DenseBwdArgs args) {
    using Plan = DenseBwdPlan<D, kDkv>;
    using Roles = DenseRoles<D>;
    constexpr int kScoreWarps = Roles::kScoreWarps, kEpilogueWarps = Roles::kEpilogueWarps;
    constexpr bool kThree = !kDkv || D == 64;
    constexpr int kY1 = Plan::kY1, kY2 = Plan::kY2, kRowSets = Plan::kRowSets;
    constexpr int kHalf = kDenseBlock * 128;                     // 128 rows x 64 columns
    constexpr int kAcc2 = D;                                     // kDkv: first column of dK
    constexpr int kScore0 = kDkv ? 2 * D : D;                    // first column of score buffer 0
    static_assert(kScore0 + (kThree ? 3 : 2) * 128 <= kTmemCols, "tensor memory");
    static_assert(kThree || Roles::kCols == 64, "P in two halves");
    static_assert(Plan::kDynBytes <= 227 * 1024 - 1024, "shared memory");

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_x1_full, bar_x2_full;   // the item's stationary tiles are there, phase it & 1
    __shared__ __align__(8) uint64_t bar_x1_free, bar_x2_free;   // ... and its last S / dP is complete: they may be replaced
    __shared__ __align__(8) uint64_t bar_y1_full[kY1], bar_y1_empty[kY1], bar_y2_full[kY2], bar_y2_empty[kY2];
    __shared__ __align__(8) uint64_t bar_rows_full[kRowSets];        // kDkv: LSE and delta of the tile
    // per tile, two barriers in turn (tile T: [T & 1], phase (T >> 1) & 1): the MMAs run up to two tiles ahead of the warps that wait for
    // them, which a single barrier's parity could not tell apart
    __shared__ __align__(8) uint64_t bar_s_full[2], bar_dp_full[2];      // S_T / dP_T complete
    __shared__ __align__(8) uint64_t bar_p_ready[2];             // kDkv: P_T is in tensor memory, all of it; kDq: S_T has been read
    __shared__ __align__(8) uint64_t bar_p_half[2];              // kDkv, two buffers: the first 32 columns of every score warp's part of P_T are
    __shared__ __align__(8) uint64_t bar_ds_ready[2];            // dS_T is in tensor memory
    __shared__ __align__(8) uint64_t bar_done;                   // the item's accumulators are complete, phase it & 1 ...
    __shared__ __align__(8) uint64_t bar_acc_free;               // ... and have been read: the next item may overwrite them
    __shared__ __align__(8) uint64_t bar_item_full[kItemRing], bar_item_empty[kItemRing];
    __shared__ __align__(8) uint64_t bar_drain, bar_drain2;
    __shared__ int4 items[kItemRing];                            // {item (-1: no more), tiles, the first of them, part}
    __shared__ int4 spans[kItemRing];                            // {keys of the batch, first streaming block, blocks per head, -}
    __shared__ uint32_t tmem_base_smem;
    __shared__ int cta_abort;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (threadIdx.x == 0) cta_abort = *reinterpret_cast<volatile int*>(&g_abort_flag);
    const uint32_t smem = smem_u32(smem_raw);
    AbortState abort_state{&cta_abort, args.host_status};
    {
        uint32_t dyn_size;
        asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(dyn_size));
        if ((smem & 1023u) != 0u || static_cast<uint32_t>(Plan::kDynBytes) > dyn_size) {
            if (threadIdx.x == 0) report_device_error(abort_state, 11);   // ATTN_JVP_ERR_DEVICE_LAYOUT
            grid_dependency_wait();
            return;
        }
    }
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bar_x1_full), 1);
        mbar_init(smem_u32(&bar_x2_full), 1);
        mbar_init(smem_u32(&bar_x1_free), 1);
        mbar_init(smem_u32(&bar_x2_free), 1);
        for (int i = 0; i < kY1; ++i) { mbar_init(smem_u32(&bar_y1_full[i]), 1); mbar_init(smem_u32(&bar_y1_empty[i]), 1); }
        for (int i = 0; i < kY2; ++i) { mbar_init(smem_u32(&bar_y2_full[i]), 1); mbar_init(smem_u32(&bar_y2_empty[i]), 1); }
        for (int i = 0; i < kRowSets; ++i) mbar_init(smem_u32(&bar_rows_full[i]), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bar_s_full[i]), 1);
            mbar_init(smem_u32(&bar_dp_full[i]), 1);
            mbar_init(smem_u32(&bar_p_ready[i]), kScoreWarps);
            mbar_init(smem_u32(&bar_p_half[i]), kScoreWarps);
            mbar_init(smem_u32(&bar_ds_ready[i]), kScoreWarps);
        }
        for (int i = 0; i < kItemRing; ++i) {
            mbar_init(smem_u32(&bar_item_full[i]), 1);
            mbar_init(smem_u32(&bar_item_empty[i]), (kDkv ? 1 : 2) + kScoreWarps + kEpilogueWarps);
        }
        mbar_init(smem_u32(&bar_done), 1);
        mbar_init(smem_u32(&bar_acc_free), kEpilogueWarps);
        mbar_init(smem_u32(&bar_drain), 1);
        mbar_init(smem_u32(&bar_drain2), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (*reinterpret_cast<volatile int*>(&cta_abort) != 0) {
        grid_dependency_wait();
        return;
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&tmem_base_smem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_base_smem);
    if (kDkv) {
        grid_dependency_wait();
        grid_launch_dependents();
    }

    // entry `it` of the CTA's sequence of items (it = 0, 1, ...); whole warp
    auto item_at = [&](int it, int4& entry) -> bool {
        if (!mbar_wait_warp(smem_u32(&bar_item_full[it % kItemRing]), static_cast<uint32_t>(it / kItemRing) & 1u, abort_state)) return false;
        entry = *const_cast<const int4*>(&items[it % kItemRing]);
        return true;
    };
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Roles::kRegsLight));
        if (warp == kProducerWarp && lane == 0) {
            // ---- TMA producer and scheduler ----
            prefetch_tensormap(&args.x1);
            prefetch_tensormap(&args.x2);
            prefetch_tensormap(&args.y1);
            prefetch_tensormap(&args.y2);
            bool ok = true;
            int T = 0;
            // a ring's next slot, and the parity of its current lap
            struct Ring { int slot; uint32_t parity; };
            Ring r1{0, 0}, r2{0, 0};
            // The item (or part of one) at a place of the order, and its tiles; item -1: no more.
            struct Work { int item, part, tile0, n; DenseSpan span; };
            auto work_from = [&](int at) -> Work {
                for (;; at = static_cast<int>(gridDim.x) + atomicAdd(args.counter, 1)) {
                    Work w{-1, 0, 0, 0, {}};
                    if (static_cast<unsigned>(at) >= static_cast<unsigned>(args.n_items * args.splits)) return w;
                    w.item = at / args.splits;
                    w.part = at - w.item * args.splits;
                    if (args.mask.causal) {                      // long items first: early key blocks, late query blocks
                        const int per = args.n_items_per_head;
                        const CausalItem c = causal_item(w.item, per, args.n_items / per, args.mask.window);
                        w.item = c.bh * per + (kDkv ? c.rank : per - 1 - c.rank);
                    }
                    w.span = dense_span<kDkv>(args, w.item);
                    w.tile0 = part_begin(w.span.n, w.part, args.splits);
                    w.n = part_begin(w.span.n, w.part + 1, args.splits) - w.tile0;
                    if (w.n > 0) return w;
                }
            };
            Work w = work_from(blockIdx.x);
            for (int it = 0; ok; ++it) {
                const int e = it % kItemRing;
                if (it >= kItemRing) ok = mbar_wait(smem_u32(&bar_item_empty[e]), (static_cast<uint32_t>(it / kItemRing) & 1u) ^ 1u, abort_state);
                if (!ok) break;
                items[e] = make_int4(w.item, w.n, w.tile0, w.part);
                spans[e] = make_int4(w.span.len, w.span.first, w.span.count, 0);
                mbar_arrive(smem_u32(&bar_item_full[e]));
                if (w.item < 0) break;
                const int bh = w.item / args.n_items_per_head, b = bh / args.H, h = bh - b * args.H;
                const int own0 = (w.item - bh * args.n_items_per_head) * kDenseBlock;
                auto load_tile = [&](uint32_t dst, const CUtensorMap* map, uint64_t& full, int head, int row0) {
                    mbar_arrive_expect_tx(smem_u32(&full), Plan::kTile);
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) tma_load_4d(dst + c * kHalf, map, smem_u32(&full), c * 64, head, row0, b);
                };
                // the streaming head (kDkv: of those that share the item's, one after the other) and block
                int head = kDkv ? h * args.mask.group + w.tile0 / w.span.count : h / args.mask.group;
                int streaming = kDkv ? w.tile0 % w.span.count : w.tile0;
                Work next{-1, 0, 0, 0, {}};
                for (int j = 0; j < w.n; ++j, ++T) {
                    if (kDkv && streaming == w.span.count) { streaming = 0; ++head; }
                    const int block = w.span.first + streaming++;
                    int row0 = block * kDenseBlock;
                    const bool tail = !kDkv && w.span.len < args.Lk && w.span.len - row0 < kDenseBlock;
                    if (tail) row0 = 0;
                    if (j == 0) {
                        if (it > 0) ok = mbar_wait(smem_u32(&bar_x1_free), (it - 1) & 1, abort_state);
                        if (!ok) break;
                        load_tile(smem, &args.x1, bar_x1_full, h, own0);
                    }
                    if (T >= kY1) ok = mbar_wait(smem_u32(&bar_y1_empty[r1.slot]), r1.parity ^ 1u, abort_state);
                    if (!ok) break;
                    load_tile(smem + Plan::kY1Off + r1.slot * Plan::kTile, tail ? &args.tail1 : &args.y1, bar_y1_full[r1.slot], head, row0);
                    if (j == 0) {
                        if (it > 0) ok = mbar_wait(smem_u32(&bar_x2_free), (it - 1) & 1, abort_state);
                        if (!ok) break;
                        load_tile(smem + Plan::kTile, &args.x2, bar_x2_full, h, own0);
                    }
                    if (T >= kY2) ok = mbar_wait(smem_u32(&bar_y2_empty[r2.slot]), r2.parity ^ 1u, abort_state);
                    if (!ok) break;
                    load_tile(smem + Plan::kY2Off + r2.slot * Plan::kTile, tail ? &args.tail2 : &args.y2, bar_y2_full[r2.slot], head, row0);
                    if (kDkv) {
                        // Row constants: the set of tile T - kRowSets is free once that tile's dS has been formed, which the release of
                        // its Q tile (after dK += dS Q) says
                        if (T >= kRowSets) {
                            const int t = T - kRowSets;
                            ok = mbar_wait(smem_u32(&bar_y1_empty[t % kY1]), static_cast<uint32_t>(t / kY1) & 1u, abort_state);
                            if (!ok) break;
                        }
                        const uint32_t rb = smem_u32(&bar_rows_full[T % kRowSets]);
                        mbar_arrive_expect_tx(rb, Plan::kRowsBytes);
                        const float* rows = args.rows + ((static_cast<long long>(b) * args.H * args.mask.group + head) * args.n_q + block) * (2 * kDenseBlock);
                        bulk_load(smem + Plan::kRowsOff + (T % kRowSets) * Plan::kRowsBytes, rows, Plan::kRowsBytes, rb);
                    }
                    if (++r1.slot == kY1) { r1.slot = 0; r1.parity ^= 1u; }
                    if (++r2.slot == kY2) { r2.slot = 0; r2.parity ^= 1u; }
                    if (j == min(w.n - 1, 2)) next = work_from(static_cast<int>(gridDim.x) + atomicAdd(args.counter, 1));
                }
                w = next;
            }
            if (!ok) {
                // give up: let the copies in flight land (bounded) before the CTA exits
                const unsigned long long t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < 100000000ull) {}
            }
        } else if (warp == kMmaWarp || (!kDkv && warp == kMmaWarp2)) {
            // ---- MMA issuers (each warp in lock step, one elected lane's instructions take effect).  kDq: the second warp issues dP. ----
            constexpr uint32_t kIdescS = make_idesc(kDenseBlock, false);
            constexpr uint32_t kIdescV = make_idesc(D, true);
            const uint32_t pred = elect_one() ? 1u : 0u;
            const uint32_t x1_lo = make_desc_lo(smem, 16), x2_lo = make_desc_lo(smem + Plan::kTile, 16);
            // scores: rows x 128 over D
            auto scores = [&](uint32_t d, uint32_t x_lo, uint32_t y) {
                const uint32_t y_lo = make_desc_lo(y, 16);
                auto koff = [](int k) -> uint32_t { return ((k / 4) * kHalf + (k % 4) * 32) >> 4; };
                mma_ss_if<false, false>(pred, d, make_desc(x_lo), make_desc(y_lo), kIdescS);
#pragma unroll
                for (int k = 1; k < D / 16; ++k) mma_ss_if<true, false>(pred, d, make_desc(x_lo + koff(k)), make_desc(y_lo + koff(k)), kIdescS);
            };
            // accumulator += (bf16 rows x 128 in a score buffer) y; a score warp's columns of it are at the start of the fp32 columns that they come from
            // (`part`: 0 = all of it, 1 / 2 = the first / second 32 columns of each 64)
            auto values = [&](uint32_t d, uint32_t a, uint32_t y, bool first, int part) {
                const uint32_t y_lo = make_desc_lo(y, kHalf);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (part == 0 || (k % 4) / 2 == part - 1) mma_ts_if<false>(pred, d, a + k * 16 / Roles::kCols * Roles::kCols + k * 16 % Roles::kCols / 2, make_desc(y_lo + k * (2048 >> 4)), kIdescV, (first && k == 0) ? 0u : 1u);
            };
            auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait_warp(smem_u32(&bar), parity & 1u, abort_state); };
            auto commit = [&](uint64_t& bar) { tc_commit_if<false>(pred, smem_u32(&bar)); };
            auto buf = [&](int m) { return tmem + kScore0 + (m % 3) * 128; };
            auto buf_s = [&](int T) { return kThree ? buf(2 * T) : tmem + kScore0; };
            auto buf_dp = [&](int T) { return kThree ? buf(2 * T + 1) : tmem + kScore0 + 128; };
            // A place in the stream of tiles: tile T is number j of the n of item `it`; n = 0: the stream has ended.
            struct Place { int it, n, j, T; };
            bool ok = true;
            auto next_place = [&](Place& c) {
                ++c.T;
                if (++c.j < c.n) return;
                int4 entry;
                ok = item_at(++c.it, entry);
                // (through a reduction, whose result lies in a uniform register: with it everything that the loop below derives
                // from it does, addresses and descriptors among them, and that is where the MMAs take them from)
                c.n = static_cast<int>(__reduce_max_sync(0xffffffffu, ok && entry.x >= 0 ? entry.y : 0));
                c.j = 0;
            };
            // S / dP of the tile at a place, and on to the next
            auto issue_s = [&](Place& c) {
                if (!ok || c.n == 0) return;
                if (c.j == 0) ok = wait(bar_x1_full, c.it);
                if (ok) ok = wait(bar_y1_full[c.T % kY1], c.T / kY1);
                if (!ok) return;
                scores(buf_s(c.T), x1_lo, smem + Plan::kY1Off + (c.T % kY1) * Plan::kTile);
                commit(bar_s_full[c.T & 1]);
                if (c.j + 1 == c.n) commit(bar_x1_free);
                next_place(c);
            };
            auto issue_dp = [&](Place& c) {
                if (!ok || c.n == 0) return;
                if (c.j == 0) ok = wait(bar_x2_full, c.it);
                if (ok) ok = wait(bar_y2_full[c.T % kY2], c.T / kY2);
                if (ok && !kDkv && c.T > 0) {
                    // goes where S of the tile before was, once that has been read
                    ok = wait(bar_p_ready[(c.T - 1) & 1], (c.T - 1) >> 1);
                    tc_fence_after();
                }
                if (!ok) return;
                scores(buf_dp(c.T), x2_lo, smem + Plan::kY2Off + (c.T % kY2) * Plan::kTile);
                commit(bar_dp_full[c.T & 1]);
                if (!kDkv) commit(bar_y2_empty[c.T % kY2]);
                if (c.j + 1 == c.n) commit(bar_x2_free);
                next_place(c);
            };
            Place s{-1, 0, 0, -1};
            next_place(s);
            Place dp = s, v = s;
            if (!kDkv && warp == kMmaWarp2) {
                while (ok && dp.n > 0) {
                    const int it = dp.it;
                    issue_dp(dp);
                    if (dp.it != it && lane == 0) mbar_arrive(smem_u32(&bar_item_empty[it % kItemRing]));
                }
                v.n = 0;
            } else {
                issue_s(s);
                if (kDkv) issue_dp(dp);
                if (kThree) issue_s(s);
            }
            auto y1_at = [&](int T) { return smem + Plan::kY1Off + (T % kY1) * Plan::kTile; };
            auto y2_at = [&](int T) { return smem + Plan::kY2Off + (T % kY2) * Plan::kTile; };
            while (ok && v.n > 0) {
                const bool first = v.j == 0, last = v.j + 1 == v.n;
                // the first values of an item overwrite the accumulators: the epilogue of the one before must have read them
                auto values_ready = [&](uint64_t& bar) {
                    ok = wait(bar, v.T >> 1);
                    if (ok && first && v.it > 0) ok = wait(bar_acc_free, v.it - 1);
                    if (ok) tc_fence_after();
                    return ok;
                };
                if (kDkv) {
                    if (kThree) {
                        if (!values_ready(bar_p_ready[v.T & 1])) break;
                        values(tmem, buf_s(v.T), y2_at(v.T), first, 0);
                    } else {
                        // (what the next tile's S waits for is the second half alone)
                        if (!values_ready(bar_p_half[v.T & 1])) break;
                        values(tmem, buf_s(v.T), y2_at(v.T), first, 1);
                        ok = wait(bar_p_ready[v.T & 1], v.T >> 1);
                        if (!ok) break;
                        tc_fence_after();
                        values(tmem, buf_s(v.T), y2_at(v.T), false, 2);
                    }
                    commit(bar_y2_empty[v.T % kY2]);
                    // (into the buffer that P has just been read from)
                    if (kThree) issue_dp(dp);
                    else issue_s(s);
                    if (ok) ok = wait(bar_ds_ready[v.T & 1], v.T >> 1);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem + kAcc2, buf_dp(v.T), y1_at(v.T), first, 0);
                    commit(bar_y1_empty[v.T % kY1]);
                    if (last) commit(bar_done);
                    if (kThree) issue_s(s);                      // (into the buffer that dS has just been read from)
                    else issue_dp(dp);
                } else {
                    if (!values_ready(bar_ds_ready[v.T & 1])) break;
                    values(tmem, buf_dp(v.T), y1_at(v.T), first, 0);
                    commit(bar_y1_empty[v.T % kY1]);
                    if (last) commit(bar_done);
                    issue_s(s);                                  // (into the buffer that dS has just been read from)
                }
                if (!ok) break;
                if (last && lane == 0) mbar_arrive(smem_u32(&bar_item_empty[v.it % kItemRing]));
                next_place(v);
            }
            if (!ok) {
                // give up: wait (bounded) until the tensor core has drained what was issued
                uint64_t& drain = warp == kMmaWarp ? bar_drain : bar_drain2;
                commit(drain);
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(smem_u32(&drain), 0) && globaltimer_ns() - t0 < 100000000ull) {}
            }
            __syncwarp();
        } else if (warp == 3 && args.splits == 1 && (args.mask.lengths != nullptr || args.mask.causal)) {
            // ---- items without tiles (split ones: dense_join_kernel writes all of them; without a mask every item has tiles) ----
            for (int item = blockIdx.x; item < args.n_items; item += gridDim.x) {
                if (dense_span<kDkv>(args, item).n > 0) continue;
                const int bh = item / args.n_items_per_head, b = bh / args.H, h = bh - b * args.H, r0 = (item - bh * args.n_items_per_head) * kDenseBlock;
                const int cells = min(kDenseBlock, args.L_own - r0) * (D / 8);
                for (int e = lane; e < cells; e += 32) {
                    const long long at = ((static_cast<long long>(b) * args.L_own + r0 + e / (D / 8)) * args.H + h) * D + e % (D / 8) * 8;
                    *reinterpret_cast<uint4*>(args.out1 + at) = make_uint4(0u, 0u, 0u, 0u);
                    if (kDkv) *reinterpret_cast<uint4*>(args.out2 + at) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        }
    } else if (warp < 4 + kScoreWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Roles::kRegsScore));
        // ---- scores.  Warp w owns rows 32 (w % 4) + lane (its lanes of tensor memory) and kCols columns of every tile. ----
        constexpr int kCols = Roles::kCols;
        const int quarter = warp & 3, col0 = kCols * ((warp - 4) >> 2);
        const int row = quarter * 32 + lane;
        const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
        const float c1 = args.scale_log2;
        const uint64_t c1c1 = pack_f32x2(c1, c1);
        float own_lse = 0.0f, own_delta = 0.0f;                  // kDq: of the row, negative as they come
        auto read_own = [&](int item) {                          // (rows of a query block: [LSE 128][delta 128])
            if (kDkv || item < 0) return;
            const float* own = args.rows + static_cast<long long>(item) * (2 * kDenseBlock) + row;
            own_lse = __ldg(own);
            own_delta = __ldg(own + kDenseBlock);
        };
        // P = 2^(S c1 - LSE log2 e) of 32 columns, in fp32; part of the exponentials on the FMA pipe
        auto exps = [&](const uint32_t* sv, float* p, const float4* lse) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                const float4 l = kDkv ? lse[c / 4] : make_float4(own_lse, own_lse, own_lse, own_lse);
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    const uint64_t x = fma_f32x2(pack_f32x2(__uint_as_float(sv[c + u]), __uint_as_float(sv[c + u + 1])), c1c1,
                                                 u == 0 ? pack_f32x2(l.x, l.y) : pack_f32x2(l.z, l.w));
                    if (((c + u) >> 1) % 8 < kBwdPoly) {
                        exp2_poly_pair(x, p[c + u], p[c + u + 1]);
                    } else {
                        float x0, x1;
                        unpack_f32x2(x, x0, x1);
                        p[c + u] = ex2f(x0);
                        p[c + u + 1] = ex2f(x1);
                    }
                }
            }
        };
        // dS = P (dP - delta) of 32 columns, rounded to bf16
        auto ds_of = [&](const uint32_t* dp, const float* p, const float4* delta, uint32_t* ds) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                const float4 d = kDkv ? delta[c / 4] : make_float4(own_delta, own_delta, own_delta, own_delta);
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    const uint64_t v = add_f32x2(pack_f32x2(__uint_as_float(dp[c + u]), __uint_as_float(dp[c + u + 1])),
                                                 u == 0 ? pack_f32x2(d.x, d.y) : pack_f32x2(d.z, d.w));
                    float v0, v1;
                    unpack_f32x2(mul_f32x2(v, pack_f32x2(p[c + u], p[c + u + 1])), v0, v1);
                    ds[(c + u) >> 1] = pack_bf16(v0, v1);
                }
            }
        };
        int T = 0;
        int s_buf = 0;                                           // three buffers: that of S_T, 2 T mod 3; dP_T is in the next one
        int4 cur;
        bool ok = item_at(0, cur);
        if (ok) read_own(cur.x);
        for (int it = 0; ok && cur.x >= 0; ++it) {
            const int n = cur.y;
            // kDq: how many keys the row sees, from the first key of the tile on.  kDkv: the first query that sees the row's key, from the first query of
            // the tile on; and the tile's block of those of a head
            const int4 span = *const_cast<const int4*>(&spans[it % kItemRing]);
            const int own = (cur.x % args.n_items_per_head) * kDenseBlock + row;
            int streaming = kDkv ? cur.z % span.z : cur.z;
            int sees;
            if (kDkv) sees = args.mask.causal ? own - args.mask.offset - (span.y + streaming) * kDenseBlock : -(1 << 30);
            else sees = (args.mask.causal ? min(span.x, own + 1 + args.mask.offset) : span.x) - streaming * kDenseBlock;
            for (int j = 0; j < n; ++j, ++T) {
                const uint32_t buf_s = tmem + lane_base + kScore0 + (kThree ? s_buf * 128 : 0) + col0;
                const uint32_t buf_dp = tmem + lane_base + kScore0 + (kThree ? (s_buf == 2 ? 0 : s_buf + 1) * 128 : 128) + col0;
                const int set = T % kRowSets;
                const float4* lse = reinterpret_cast<const float4*>(smem_raw + Plan::kRowsOff + set * Plan::kRowsBytes) + col0 / 4;
                const float4* delta = lse + kDenseBlock / 4;
                const uint32_t phase = static_cast<uint32_t>(T >> 1) & 1u;
                if (kDkv) ok = mbar_wait_patient(smem_u32(&bar_rows_full[set]), static_cast<uint32_t>(T / kRowSets) & 1u, abort_state);
                if (ok) ok = mbar_wait_patient(smem_u32(&bar_s_full[T & 1]), phase, abort_state);
                if (ok && !kDkv) ok = mbar_wait_patient(smem_u32(&bar_dp_full[T & 1]), phase, abort_state);
                if (!ok) break;
                tc_fence_after();
                uint32_t sv[kCols], dp[kCols];
                float p[kCols];
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += 32) TMEM_LD32(buf_s + c0, sv, c0);
                if (!kDkv) {
                    // (all of S first: loads that go to and fro between the buffers cost kDq 15 % at D = 128)
#pragma unroll
                    for (int c0 = 0; c0 < kCols; c0 += 32) TMEM_LD32(buf_dp + c0, dp, c0);
                }
                tc_wait_ld();
                if (!kDkv) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_p_ready[T & 1]));
                }
                // (P^T in bf16 over the S that it came from, dS over dP: in the first half of the warp's columns)
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += 32) {
                    uint32_t packed[16];
                    exps(sv + c0, p + c0, lse + c0 / 4);
                    // what does not see each other: replaced (a product with 0 would keep an infinity or a NaN)
                    if (kDkv ? sees > col0 + c0 : sees < col0 + c0 + 32) {
#pragma unroll
                        for (int c = 0; c < 32; ++c) if (kDkv ? col0 + c0 + c < sees : col0 + c0 + c >= sees) p[c0 + c] = 0.0f;
                    }
                    if (kDkv) {
#pragma unroll
                        for (int c = 0; c < 16; ++c) packed[c] = pack_bf16(p[c0 + 2 * c], p[c0 + 2 * c + 1]);
                        TMEM_ST16(buf_s + c0 / 2, packed, 0);
                        if (kThree && c0 + 32 < kCols) continue;
                        tc_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(c0 + 32 < kCols ? &bar_p_half[T & 1] : &bar_p_ready[T & 1]));
                    } else {
                        ds_of(dp + c0, p + c0, delta, packed);
                        TMEM_ST16(buf_dp + c0 / 2, packed, 0);
                    }
                }
                if (kDkv) {
                    ok = mbar_wait_patient(smem_u32(&bar_dp_full[T & 1]), phase, abort_state);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int c0 = 0; c0 < kCols; c0 += 32) TMEM_LD32(buf_dp + c0, dp, c0);
                    tc_wait_ld();
#pragma unroll
                    for (int c0 = 0; c0 < kCols; c0 += 32) {
                        uint32_t packed[16];
                        ds_of(dp + c0, p + c0, delta + c0 / 4, packed);
                        TMEM_ST16(buf_dp + c0 / 2, packed, 0);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_ds_ready[T & 1]));
                // to the next tile: the next block, or the first one of the next head
                s_buf = s_buf >= 1 ? s_buf - 1 : s_buf + 2;
                sees -= kDenseBlock;
                if (kDkv && ++streaming == span.z) {
                    streaming = 0;
                    sees += span.z * kDenseBlock;
                }
            }
            if (!ok) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_item_empty[it % kItemRing]));
            ok = item_at(it + 1, cur);
            if (ok) read_own(cur.x);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Roles::kRegsEpilogue));
        // ---- accumulators out: thread (warp, lane) owns row 32 (warp % 4) + lane of both ----
        const int row = (warp & 3) * 32 + lane;
        const uint32_t acc = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        int4 cur;
        bool ok = item_at(0, cur);
        for (int it = 0; ok && cur.x >= 0; ++it) {
            const int item = cur.x;
            const int len = spans[it % kItemRing].x;             // (keys behind it: gradients of 0, whatever their rows hold)
            const int bh = item / args.n_items_per_head, b = bh / args.H, h = bh - b * args.H;
            const int r = (item - bh * args.n_items_per_head) * kDenseBlock + row;
            const long long at = ((static_cast<long long>(b) * args.L_own + r) * args.H + h) * D;
            ok = mbar_wait_patient(smem_u32(&bar_done), it & 1, abort_state);
            if (!ok) break;
            tc_fence_after();
            constexpr int kCols = kDkv ? 2 * D : D;
#pragma unroll 1
            for (int c0 = 0; c0 < kCols; c0 += 32) {
                uint32_t v[32];
                TMEM_LD32(acc + c0, v, 0);
                tc_wait_ld();
                if (c0 + 32 == kCols) {
                    // all in registers or stored: the next item's first values may overwrite them
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&bar_acc_free));
                        mbar_arrive(smem_u32(&bar_item_empty[it % kItemRing]));
                    }
                }
                if (args.splits > 1) {
                    float* out = args.part + ((static_cast<long long>(cur.w) * args.n_items + item) * kDenseBlock + row) * kCols + c0;
#pragma unroll
                    for (int c = 0; c < 32; c += 8)
                        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + c), "r"(v[c]), "r"(v[c + 1]),
                                     "r"(v[c + 2]), "r"(v[c + 3]), "r"(v[c + 4]), "r"(v[c + 5]), "r"(v[c + 6]), "r"(v[c + 7]) : "memory");
                    continue;
                }
                if (kDkv && r >= len) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0u;
                }
                const bool second = kDkv && c0 >= D;
                const float factor = (kDkv && !second) ? 1.0f : args.scale;
#pragma unroll
                for (int c = 0; c < 16; ++c) v[c] = pack_bf16(__uint_as_float(v[2 * c]) * factor, __uint_as_float(v[2 * c + 1]) * factor);
                if (r < args.L_own) {
                    __nv_bfloat16* out = (second ? args.out2 + (c0 - D) : args.out1 + c0) + at;
                    if (args.wide_out) {                         // whole 32-byte sectors
#pragma unroll
                        for (int c = 0; c < 16; c += 8)
                            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + 2 * c), "r"(v[c]), "r"(v[c + 1]),
                                         "r"(v[c + 2]), "r"(v[c + 3]), "r"(v[c + 4]), "r"(v[c + 5]), "r"(v[c + 6]), "r"(v[c + 7]) : "memory");
                    } else {
#pragma unroll
                        for (int c = 0; c < 16; c += 4) *reinterpret_cast<uint4*>(out + 2 * c) = make_uint4(v[c], v[c + 1], v[c + 2], v[c + 3]);
                    }
                }
            }
            ok = item_at(it + 1, cur);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
    if (!kDkv) grid_dependency_wait();
}

}  // namespace attn_jvp
