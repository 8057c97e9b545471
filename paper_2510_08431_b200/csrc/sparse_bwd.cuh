// Gradients of attention over selected key blocks (block_select.cuh), for a query row i and a kept key j:
//     P = exp(s q.k - LSE_i),  dP = dO_i . v_j,  delta_i = dO_i . O_i,  dS = P (dP - delta_i)
//     dQ_i = s sum_j dS k_j,   dK_j = s sum_i dS q_i,   dV_j = sum_i P dO_i
// The selection is a constant.  Two passes, neither with atomics, so a gradient is the same from run to run:
//   kDkv   one CTA per key block: K, V stay in shared memory, the query blocks that kept it stream by.  Scores are formed
//          transposed (keys = rows of the MMA = lanes of tensor memory), so that P^T and dS^T lie where the A operand of
//          dV += P^T dO and dK += dS^T Q is read from: they never leave tensor memory.
//   kDq    one CTA per query block: Q, dO stay, the kept K, V blocks stream by; dQ += dS K.
// That is seven products per pair of blocks where a single pass with atomics on dQ needs five; with 128 x 128 blocks the
// two passes take 7 x 512 tensor cycles per pair at D = 128.
//
// 512 threads: warp 0 (kDq: and warp 2) issues the MMAs, warp 1 the TMA loads, warps 4..11 work on the scores, warps 12..15 write finished
// accumulators out (a thread's row is 32 separate sectors away from its neighbour's: the stores keep the load/store unit
// busy for some 2000 cycles, during which the others are in the next item).
//
// Order of work, kDkv (tensor memory: dV, dK, one buffer for S, one for dP, 512 columns at D = 128): P^T overwrites S and
// dS^T overwrites dP, and the MMAs of tile j + 1 are queued behind those that read them,
//     dV += P_j dO_j, S_(j+1) = K Q_(j+1)^T   |   dK += dS_j Q_j, dP_(j+1) = V dO_(j+1)^T
// so the exponentials of tile j + 1 run beside dK_j and dP_(j+1), and its dS beside dV_(j+1) and S_(j+2).
// kDq has no P operand and one accumulator: three score buffers in turn (matrix 2 T is S_T, 2 T + 1 is dP_T, matrix m is in
// buffer m % 3) let S run two tiles ahead.
// CTAs are persistent, one per SM, and draw their items (stationary blocks) from a counter: lists differ in length.  Tiles
// are numbered T = 0, 1, ... over all items of a CTA and run on without a break: the first score MMAs of an item go out
// with the last value MMAs of the one before, and all that an item boundary costs is the hand-over of the accumulators
// (with one CTA per item a boundary cost about 15 thousand cycles at D = 128, as much as six tiles).
// Bound by the tensor pipe (active 76 % in kDkv, 70 % in kDq) in short runs and by power in long ones.  12 heads of 32760 tokens at
// D = 128, 32 of 256 blocks kept: preparation 46, kDkv 1156, kDq 903 us in a short run; D = 64, 12 heads of 4000, lists of
// eight blocks: 6, 40, 32 us.
#pragma once

#include "attn_jvp_kernel.cuh"
#include "block_select.cuh"

namespace attn_jvp {

constexpr int kBwdBlock = 128;
constexpr int kBwdThreads = 512;
constexpr int kBwdComputeWarps = 8, kBwdEpilogueWarps = 4;
constexpr int kBwdRegsLight = 64, kBwdRegsCompute = 200, kBwdRegsEpilogue = 48;      // 128 (64 + 200 + 200 + 48) = 65536
constexpr int kItemRing = 4;                 // items known ahead: the score MMAs are at most two items ahead of the values
constexpr int kMmaWarp2 = 2;
constexpr int kBwdY1 = 3, kBwdY2 = 2;        // shared-memory buffers of the two streaming tensors
constexpr int kBwdPoly = 2;                  // of 8 pairs of exponentials, how many take the FMA pipe (0: 1 to 3 % slower, 4: 4 %)

struct SparseBwdArgs {
    const int* list;            // kDkv: [B][H][n_k][n_q] query blocks of a key block; kDq: [B][H][n_q][n_k]
    const int* tiles;           // their lengths in 64-token tiles
    const int* order;           // the order in which they are handed out (block_order()); null: as they lie
    const float* rows;          // [B][H][n_q][2][128]: per block of queries LSE log2 e (+inf: no probability), then delta
    __nv_bfloat16* out1;        // kDkv: dV, kDq: dQ        [B][L][H][D]
    __nv_bfloat16* out2;        // kDkv: dK
    int* host_status;
    int* counter;               // items handed out beyond the first one of every CTA; starts at 0
    int H, n_items, n_items_per_head, list_stride;
    int L_own, L_other;         // tokens on the stationary / streaming side
    int n_q;                    // query blocks
    int wide_out;               // out1, out2 are 32-byte aligned
    float scale, scale_log2;
};

template <int D>
struct SparseBwdPlan {
    static constexpr int kHalf = kBwdBlock * 128;                // 128 rows x 64 bf16
    static constexpr int kTile = (D / 64) * kHalf;               // a 128 x D operand
    static constexpr int kX = 0;
    static constexpr int kY1Off = 2 * kTile;
    static constexpr int kY2Off = kY1Off + kBwdY1 * kTile;
    static constexpr int kRowsOff = kY2Off + kBwdY2 * kTile;     // kDkv: LSE and delta of two streaming tiles
    static constexpr int kRowsBytes = kBwdBlock * 8;
    static constexpr int kDynBytes = kRowsOff + 2 * kRowsBytes;  // 226 KB at D = 128
};

// What the two passes need beforehand.  Blocks below `row_blocks`: LSE log2 e and delta per query row, padded to whole
// blocks; rows behind the last query and rows without any key get LSE = +inf, which makes their P exactly 0; a group of
// D / 8 threads per row reads dO and O once.  The blocks after them: a warp per stationary block of either pass, which
// writes zero gradients where its list is empty (the passes never see those).  The last blocks sort the transposed lists,
// which differ in length whatever selection there was.  Both passes' counters start at 0.
struct SparseBwdPrep {
    const uint4 *o, *d_o;
    const float* lse;
    float* rows;
    const int *q_tiles, *k_tiles;
    int* k_order;
    __nv_bfloat16 *dq, *dk, *dv;
    int* counters;
    int B, H, Lq, Lk, n_q, n_k, row_blocks, zero_blocks;
};
constexpr int kPrepEach = 2;                 // rows per thread, their loads in flight together
template <int D>
constexpr unsigned kPrepRows = kPrepEach * 256 / (D / 8);        // ... per CTA
template <int D>
__global__ void __launch_bounds__(256)
sparse_bwd_prep_kernel(const SparseBwdPrep p) {
    constexpr int kLanes = D / 8;
    if (static_cast<int>(blockIdx.x) >= p.row_blocks + p.zero_blocks) {
        __shared__ uint4 swap[kOrderThreads];
        static_assert(kOrderThreads == 256, "the sort's CTA");
        block_order(p.k_tiles, p.k_order, p.B * p.H * p.n_k, blockIdx.x - p.row_blocks - p.zero_blocks, swap);
        return;
    }
    if (static_cast<int>(blockIdx.x) >= p.row_blocks) {
        const int lane = threadIdx.x & 31;
        int item = (blockIdx.x - p.row_blocks) * 8 + (threadIdx.x >> 5);
        const int q_items = p.B * p.H * p.n_q;
        const bool keys = item >= q_items;
        if (keys) item -= q_items;
        const int per_head = keys ? p.n_k : p.n_q, L = keys ? p.Lk : p.Lq;
        if (item >= p.B * p.H * per_head || (keys ? p.k_tiles : p.q_tiles)[item] > 0) return;
        const int bh = item / per_head, blk = item - bh * per_head, b = bh / p.H, h = bh - b * p.H;
        for (int e = lane; e < kBwdBlock * kLanes; e += 32) {
            const int r = blk * kBwdBlock + e / kLanes;
            if (r >= L) break;
            const long long at = ((static_cast<long long>(b) * L + r) * p.H + h) * D + (e % kLanes) * 8;
            *reinterpret_cast<uint4*>((keys ? p.dk : p.dq) + at) = make_uint4(0u, 0u, 0u, 0u);
            if (keys) *reinterpret_cast<uint4*>(p.dv + at) = make_uint4(0u, 0u, 0u, 0u);
        }
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) p.counters[threadIdx.x] = 0;
    // (row order [B][padded][H], that of the tensors; their number fits 32 bits)
    const unsigned padded = p.n_q * kBwdBlock, n = static_cast<unsigned>(p.B) * padded * p.H;
    const unsigned r0 = blockIdx.x * kPrepRows<D> + threadIdx.x / kLanes, sub = threadIdx.x % kLanes;
    constexpr unsigned kStep = 256 / kLanes;
    uint4 x[kPrepEach], y[kPrepEach];
    unsigned b[kPrepEach], l[kPrepEach], h[kPrepEach];
#pragma unroll
    for (int u = 0; u < kPrepEach; ++u) {
        const unsigned r = min(r0 + u * kStep, n - 1), bl = r / p.H;
        h[u] = r - bl * p.H;
        b[u] = bl / padded;
        l[u] = bl - b[u] * padded;
        x[u] = y[u] = make_uint4(0u, 0u, 0u, 0u);
        if (l[u] < static_cast<unsigned>(p.Lq)) {
            const long long at = ((static_cast<long long>(b[u]) * p.Lq + l[u]) * p.H + h[u]) * kLanes + sub;
            x[u] = __ldg(p.o + at);
            y[u] = __ldg(p.d_o + at);
        }
    }
#pragma unroll
    for (int u = 0; u < kPrepEach; ++u) {
        const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w}, ys[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), sum);
            sum = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), sum);
        }
#pragma unroll
        for (int m = kLanes / 2; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if (sub == 0 && r0 + u * kStep < n) {
            const long long bh = static_cast<long long>(b[u]) * p.H + h[u];
            float ls = INFINITY;
            if (l[u] < static_cast<unsigned>(p.Lq)) {
                ls = p.lse[bh * p.Lq + l[u]] * 1.4426950408889634f;
                if (ls == -INFINITY) ls = INFINITY;
            }
            float* out = p.rows + 2 * bh * padded + (l[u] / kBwdBlock) * (2 * kBwdBlock) + l[u] % kBwdBlock;
            out[0] = ls;
            out[kBwdBlock] = sum;
        }
    }
}

// 2^x of two values on the FMA pipe, for kernels whose pace the special-function unit sets (8 cycles per warp instruction):
// x = n + f with n the nearest integer (added and taken off again as 1.5 * 2^23 + n), 2^f by a polynomial on [-1/2, 1/2]
// whose coefficients minimise the largest relative error with p(0) = 1 (2.9e-6 in fp32; P is rounded to bf16 for the value
// products, an error of 3.9e-3, and sums of P take the error on average), times 2^n.  x below -127 is taken as -127, where the
// factor is exactly +0; a NaN stays one (hence a maximum that hands NaN on, and a product instead of an addition to the exponent
// field, which would make a number of it); x must not exceed 127.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void exp2_poly_pair(uint64_t x, float& p0, float& p1) {
    float x0, x1;
    unpack_f32x2(x, x0, x1);
    x = pack_f32x2(max_nan(x0, -127.0f), max_nan(x1, -127.0f));
    const uint64_t t = add_f32x2(x, pack_f32x2(12582912.0f, 12582912.0f));
    const uint64_t f = add_f32x2(x, fma_f32x2(t, pack_f32x2(-1.0f, -1.0f), pack_f32x2(12582912.0f, 12582912.0f)));
    uint64_t y = fma_f32x2(f, pack_f32x2(0x1.3a02ccp-7f, 0x1.3a02ccp-7f), pack_f32x2(0x1.c9fc46p-5f, 0x1.c9fc46p-5f));
    y = fma_f32x2(f, y, pack_f32x2(0x1.ec037ap-3f, 0x1.ec037ap-3f));
    y = fma_f32x2(f, y, pack_f32x2(0x1.62e12cp-1f, 0x1.62e12cp-1f));
    y = fma_f32x2(f, y, pack_f32x2(1.0f, 1.0f));
    float t0, t1;
    unpack_f32x2(t, t0, t1);
    const uint64_t two_n = pack_f32x2(__int_as_float((__float_as_int(t0) << 23) + 0x3F800000), __int_as_float((__float_as_int(t1) << 23) + 0x3F800000));
    unpack_f32x2(mul_f32x2(y, two_n), p0, p1);
}
// A number read from a list as an index below n.  The lists, the order and the counter lie in memory that a caller can have
// shared between two calls at once by mistake: results are then undefined, addresses formed from them are not.  (Coordinates of
// tensor maps need no such care: the copy fills in zeros outside the tensor.)
__host__ __device__ constexpr int index_below(int v, int n) { return static_cast<unsigned>(v) < static_cast<unsigned>(n) ? v : n - 1; }
static_assert(index_below(-1, 3) == 2 && index_below(2, 3) == 2 && index_below(3, 3) == 2 && index_below(0x7fffffff, 1) == 0, "inside");
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

// mbar_wait_warp() of a warp that has time: it looks again every 64 ns or so.  A dozen warps that look all the time take issue
// slots (and shared memory cycles, which the MMAs use in full) from the warp that feeds the tensor pipe: with a tight loop
// here kDkv took 289 us where it takes 235.
__device__ __forceinline__ bool mbar_wait_patient(uint32_t bar, uint32_t parity, const AbortState& st) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    const unsigned long long t0 = globaltimer_ns();
    for (uint32_t it = 1;; ++it) {
        __nanosleep(64);
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if ((it & 255u) == 0u) {
            if (__any_sync(0xffffffffu, *st.cta_flag != 0)) return false;
            if (__any_sync(0xffffffffu, globaltimer_ns() - t0 > kWaitLimitNs)) {
                report_device_error(st, 10);                     // ATTN_JVP_ERR_DEVICE_TIMEOUT
                return false;
            }
        }
    }
}

template <int D, bool kDkv>
__global__ void __launch_bounds__(kBwdThreads, 1)
sparse_bwd_kernel(const __grid_constant__ CUtensorMap tm_x1, const __grid_constant__ CUtensorMap tm_x2,
                  const __grid_constant__ CUtensorMap tm_y1, const __grid_constant__ CUtensorMap tm_y2, const SparseBwdArgs args) {
    // kDkv: X1, X2 = K, V of the key block, Y1, Y2 = Q, dO of a query block.  kDq: X1, X2 = Q, dO; Y1, Y2 = K, V.
    // S = X1 Y1^T, dP = X2 Y2^T (rows: the stationary side)
    using Plan = SparseBwdPlan<D>;
    constexpr int kHalves = D / 64;
    constexpr int kAcc2 = D;                                     // kDkv: first column of dK
    constexpr int kScore0 = kDkv ? 2 * D : D;                    // first column of score buffer 0
    constexpr int kBufs = kDkv ? 2 : 3;
    constexpr int kTileWarps = kDkv ? kBwdComputeWarps : kBwdComputeWarps / 2;      // warps that work on one tile
    static_assert(kScore0 + kBufs * 128 <= kTmemCols, "tensor memory");

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_x1_full, bar_x2_full;   // the item's stationary tiles are there, phase it & 1
    __shared__ __align__(8) uint64_t bar_x1_free, bar_x2_free;   // ... and its last S / dP is complete: they may be replaced
    __shared__ __align__(8) uint64_t bar_y1_full[kBwdY1], bar_y1_empty[kBwdY1], bar_y2_full[kBwdY2], bar_y2_empty[kBwdY2];
    __shared__ __align__(8) uint64_t bar_rows_full[2];           // kDkv: LSE and delta of the tile
    // per tile, two barriers in turn (tile T: [T & 1], phase (T >> 1) & 1): kDq's S and dP run up to two tiles ahead of the
    // warps that wait for them, which a single barrier's parity could not tell apart
    __shared__ __align__(8) uint64_t bar_s_full[2], bar_dp_full[2];      // S_T / dP_T complete
    __shared__ __align__(8) uint64_t bar_p_ready[2];             // kDkv: P_T is in tensor memory, all of it; kDq: S_T has been read
    __shared__ __align__(8) uint64_t bar_p_half[2];              // kDkv: the first half of every thread's part of P_T is
    __shared__ __align__(8) uint64_t bar_ds_ready[2];            // dS_T is in tensor memory
    __shared__ __align__(8) uint64_t bar_done;                   // the item's accumulators are complete, phase it & 1 ...
    __shared__ __align__(8) uint64_t bar_acc_free;               // ... and have been read: the next item may overwrite them
    __shared__ __align__(8) uint64_t bar_item_full[kItemRing], bar_item_empty[kItemRing];
    __shared__ __align__(8) uint64_t bar_drain, bar_drain2;
    __shared__ int4 items[kItemRing];                            // {item (-1: no more), streaming blocks, the last of them, -}
    __shared__ uint32_t tmem_base_smem;
    __shared__ int cta_abort;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;

    if (threadIdx.x == 0) cta_abort = *reinterpret_cast<volatile int*>(&g_abort_flag);
    __syncthreads();
    if (cta_abort != 0) return;
    const uint32_t smem = smem_u32(smem_raw);
    AbortState abort_state{&cta_abort, args.host_status};
    {
        uint32_t dyn_size;
        asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(dyn_size));
        if ((smem & 1023u) != 0u || static_cast<uint32_t>(Plan::kDynBytes) > dyn_size) {
            if (threadIdx.x == 0) report_device_error(abort_state, 11);   // ATTN_JVP_ERR_DEVICE_LAYOUT
            return;
        }
    }
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&bar_x1_full), 1);
        mbar_init(smem_u32(&bar_x2_full), 1);
        mbar_init(smem_u32(&bar_x1_free), 1);
        mbar_init(smem_u32(&bar_x2_free), 1);
        for (int i = 0; i < kBwdY1; ++i) { mbar_init(smem_u32(&bar_y1_full[i]), 1); mbar_init(smem_u32(&bar_y1_empty[i]), 1); }
        for (int i = 0; i < kBwdY2; ++i) { mbar_init(smem_u32(&bar_y2_full[i]), 1); mbar_init(smem_u32(&bar_y2_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bar_rows_full[i]), 1);
            mbar_init(smem_u32(&bar_s_full[i]), 1);
            mbar_init(smem_u32(&bar_dp_full[i]), 1);
            mbar_init(smem_u32(&bar_p_ready[i]), kTileWarps);
            mbar_init(smem_u32(&bar_p_half[i]), kTileWarps);
            mbar_init(smem_u32(&bar_ds_ready[i]), kTileWarps);
        }
        for (int i = 0; i < kItemRing; ++i) {
            mbar_init(smem_u32(&bar_item_full[i]), 1);
            mbar_init(smem_u32(&bar_item_empty[i]), (kDkv ? 1 : 2) + kBwdComputeWarps + kBwdEpilogueWarps);
        }
        mbar_init(smem_u32(&bar_done), 1);
        mbar_init(smem_u32(&bar_acc_free), kBwdEpilogueWarps);
        mbar_init(smem_u32(&bar_drain), 1);
        mbar_init(smem_u32(&bar_drain2), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
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

    // entry `it` of the CTA's sequence of items (it = 0, 1, ...); whole warp
    auto item_at = [&](int it, int4& entry) -> bool {
        if (!mbar_wait_warp(smem_u32(&bar_item_full[it % kItemRing]), static_cast<uint32_t>(it / kItemRing) & 1u, abort_state)) return false;
        entry = *const_cast<const int4*>(&items[it % kItemRing]);
        return true;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBwdRegsLight));
        if (warp == kProducerWarp && lane == 0) {
            // ---- TMA producer and scheduler: per item X1, Y1, X2, Y2 in the order the MMAs take them, then Y1_1, Y2_1, ... ----
            prefetch_tensormap(&tm_x1);
            prefetch_tensormap(&tm_x2);
            prefetch_tensormap(&tm_y1);
            prefetch_tensormap(&tm_y2);
            bool ok = true;
            int T = 0, s1 = 0, s2 = 0;
            uint32_t ph1 = 0, ph2 = 0;                           // parity of the Y buffers' current lap
            // the next item that keeps anything, from place `at` of the order on; -1: none.  n: its streaming blocks
            auto next_item = [&](int at, int& n) -> int {
                for (;; at = static_cast<int>(gridDim.x) + atomicAdd(args.counter, 1)) {
                    if (static_cast<unsigned>(at) >= static_cast<unsigned>(args.n_items)) return -1;
                    const int item = args.order == nullptr ? at : index_below(__ldg(args.order + at), args.n_items);
                    n = min((__ldg(args.tiles + item) + 1) >> 1, args.list_stride);
                    if (n > 0) return item;
                }
            };
            int n = 0, n_next = 0;
            int item = next_item(blockIdx.x, n);
            for (int it = 0; ok; ++it) {
                const int e = it % kItemRing;
                if (it >= kItemRing) ok = mbar_wait(smem_u32(&bar_item_empty[e]), (static_cast<uint32_t>(it / kItemRing) & 1u) ^ 1u, abort_state);
                if (!ok) break;
                const int* list = args.list + static_cast<long long>(max(item, 0)) * args.list_stride;
                items[e] = make_int4(item, n, item >= 0 ? __ldg(list + n - 1) : 0, 0);
                mbar_arrive(smem_u32(&bar_item_full[e]));
                if (item < 0) break;
                const int bh = item / args.n_items_per_head, own0 = (item - bh * args.n_items_per_head) * kBwdBlock;
                const int b = bh / args.H, h = bh - b * args.H;
                auto load_tile = [&](uint32_t dst, const CUtensorMap* map, uint32_t bar, int row0) {
                    mbar_arrive_expect_tx(bar, Plan::kTile);
#pragma unroll
                    for (int hf = 0; hf < kHalves; ++hf) tma_load_4d(dst + hf * Plan::kHalf, map, bar, hf * 64, h, row0, b);
                };
                const float* rows = args.rows + static_cast<long long>(bh) * args.n_q * (2 * kBwdBlock);
                int next = -1;
                for (int j = 0; j < n; ++j, ++T) {
                    const int block = __ldg(list + j), row0 = block * kBwdBlock;
                    if (j == 0) {
                        if (it > 0) ok = mbar_wait(smem_u32(&bar_x1_free), (it - 1) & 1, abort_state);
                        if (!ok) break;
                        load_tile(smem + Plan::kX, &tm_x1, smem_u32(&bar_x1_full), own0);
                    }
                    if (T >= kBwdY1) ok = mbar_wait(smem_u32(&bar_y1_empty[s1]), ph1 ^ 1u, abort_state);
                    if (!ok) break;
                    load_tile(smem + Plan::kY1Off + s1 * Plan::kTile, &tm_y1, smem_u32(&bar_y1_full[s1]), row0);
                    if (j == 0) {
                        if (it > 0) ok = mbar_wait(smem_u32(&bar_x2_free), (it - 1) & 1, abort_state);
                        if (!ok) break;
                        load_tile(smem + Plan::kX + Plan::kTile, &tm_x2, smem_u32(&bar_x2_full), own0);
                    }
                    if (T >= kBwdY2) ok = mbar_wait(smem_u32(&bar_y2_empty[s2]), ph2 ^ 1u, abort_state);
                    if (!ok) break;
                    load_tile(smem + Plan::kY2Off + s2 * Plan::kTile, &tm_y2, smem_u32(&bar_y2_full[s2]), row0);
                    if (kDkv) {
                        // Two sets of row constants: the one of tile T - 2 is free once that tile's dS has been formed, which
                        // the release of its Q tile (after dK += dS Q) says
                        if (T >= 2) {
                            const int t = T - 2;
                            ok = mbar_wait(smem_u32(&bar_y1_empty[t % kBwdY1]), static_cast<uint32_t>(t / kBwdY1) & 1u, abort_state);
                            if (!ok) break;
                        }
                        const uint32_t rb = smem_u32(&bar_rows_full[T & 1]);
                        mbar_arrive_expect_tx(rb, Plan::kRowsBytes);
                        bulk_load(smem + Plan::kRowsOff + (T & 1) * Plan::kRowsBytes, rows + index_below(block, args.n_q) * (2 * kBwdBlock), Plan::kRowsBytes, rb);
                    }
                    if (++s1 == kBwdY1) { s1 = 0; ph1 ^= 1u; }
                    if (++s2 == kBwdY2) { s2 = 0; ph2 ^= 1u; }
                    if (j == min(n - 1, 2)) next = next_item(static_cast<int>(gridDim.x) + atomicAdd(args.counter, 1), n_next);
                }
                item = next;
                n = n_next;
            }
            if (!ok) {
                // give up: let the copies in flight land (bounded) before the CTA exits
                const unsigned long long t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < 100000000ull) {}
            }
        } else if (warp == kMmaWarp || (!kDkv && warp == kMmaWarp2)) {
            // ---- MMA issuers (each warp in lock step, one elected lane's instructions take effect).  kDkv: one warp, so that
            // dK and dP stand behind dV and S, for which the exponentials of the next tile wait (two warps, one for each half of
            // the line above: 465 thousand cycles instead of 364 for 128 tiles).  kDq: the second warp issues dP (one warp:
            // 10 % slower; it cannot issue fast enough beside the warps that work on scores). ----
            constexpr uint32_t kIdescS = make_idesc(kBwdBlock, false);
            constexpr uint32_t kIdescV = make_idesc(D, true);
            const uint32_t pred = elect_one() ? 1u : 0u;
            const uint32_t x1_lo = make_desc_lo(smem + Plan::kX, 16), x2_lo = make_desc_lo(smem + Plan::kX + Plan::kTile, 16);
            auto koff = [](int k) -> uint32_t { return ((k / 4) * Plan::kHalf + (k % 4) * 32) >> 4; };
            // scores: 128 x 128 over D
            auto scores = [&](uint32_t d, uint32_t x_lo, uint32_t y) {
                const uint32_t y_lo = make_desc_lo(y, 16);
                mma_ss_if<false, false>(pred, d, make_desc(x_lo), make_desc(y_lo), kIdescS);
#pragma unroll
                for (int k = 1; k < D / 16; ++k)
                    mma_ss_if<true, false>(pred, d, make_desc(x_lo + koff(k)), make_desc(y_lo + koff(k)), kIdescS);
            };
            // accumulator += (bf16 128 x 128 in a score buffer) y; columns 0..63 of it are at its start, 64..127 64 columns on
            // (`part`: 0 = all of it, 1 / 2 = the first / second 32 columns of each 64)
            auto values = [&](uint32_t d, uint32_t a, uint32_t y, bool first, int part) {
                const uint32_t y_lo = make_desc_lo(y, Plan::kHalf);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (part != 0 && (k % 4) / 2 != part - 1) continue;
                    mma_ts_if<false>(pred, d, a + (k / 4) * 64 + (k % 4) * 8, make_desc(y_lo + k * (2048 >> 4)), kIdescV,
                                     (first && k == 0) ? 0u : 1u);
                }
            };
            auto y1 = [&](int T) { return smem + Plan::kY1Off + (T % kBwdY1) * Plan::kTile; };
            auto y2 = [&](int T) { return smem + Plan::kY2Off + (T % kBwdY2) * Plan::kTile; };
            auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait_warp(smem_u32(&bar), parity & 1u, abort_state); };
            auto commit = [&](uint64_t& bar) { tc_commit_if<false>(pred, smem_u32(&bar)); };
            auto buf = [&](int m) { return tmem + kScore0 + (m % kBufs) * 128; };
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
                if (ok) ok = wait(bar_y1_full[c.T % kBwdY1], c.T / kBwdY1);
                if (!ok) return;
                scores(buf(kDkv ? 0 : 2 * c.T), x1_lo, y1(c.T));
                commit(bar_s_full[c.T & 1]);
                if (c.j + 1 == c.n) commit(bar_x1_free);
                next_place(c);
            };
            auto issue_dp = [&](Place& c) {
                if (!ok || c.n == 0) return;
                if (c.j == 0) ok = wait(bar_x2_full, c.it);
                if (ok) ok = wait(bar_y2_full[c.T % kBwdY2], c.T / kBwdY2);
                if (ok && !kDkv && c.T > 0) {
                    // goes where S of the tile before was, once that has been read
                    ok = wait(bar_p_ready[(c.T - 1) & 1], (c.T - 1) >> 1);
                    tc_fence_after();
                }
                if (!ok) return;
                scores(buf(kDkv ? 1 : 2 * c.T + 1), x2_lo, y2(c.T));
                commit(bar_dp_full[c.T & 1]);
                if (!kDkv) commit(bar_y2_empty[c.T % kBwdY2]);
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
                else issue_s(s);
            }
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
                    if (!values_ready(bar_p_half[v.T & 1])) break;
                    values(tmem, buf(0), y2(v.T), first, 1);
                    ok = wait(bar_p_ready[v.T & 1], v.T >> 1);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem, buf(0), y2(v.T), false, 2);
                    commit(bar_y2_empty[v.T % kBwdY2]);
                    issue_s(s);                                  // (into the buffer that P has just been read from)
                    if (!ok) break;
                    ok = wait(bar_ds_ready[v.T & 1], v.T >> 1);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem + kAcc2, buf(1), y1(v.T), first, 0);
                    commit(bar_y1_empty[v.T % kBwdY1]);
                    if (last) commit(bar_done);
                    issue_dp(dp);
                } else {
                    if (!values_ready(bar_ds_ready[v.T & 1])) break;
                    values(tmem, buf(2 * v.T + 1), y1(v.T), first, 0);
                    commit(bar_y1_empty[v.T % kBwdY1]);
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
        }
    } else if (warp < 4 + kBwdComputeWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kBwdRegsCompute));
        // ---- scores.  Warp w owns rows 32 (w % 4) + lane (its lanes of tensor memory).  kDkv: both groups of four warps take
        // every tile, 64 columns each (the exponentials of a tile stand between its S and everything after).  kDq: the groups
        // take alternate tiles, all columns, so that one group's waits are covered by the other's exponentials. ----
        const int quarter = warp & 3, group = (warp - 4) >> 2;
        const int row = quarter * 32 + lane;
        const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
        const float c1 = args.scale_log2;
        const uint64_t c1c1 = pack_f32x2(c1, c1);
        float own_lse = 0.0f, own_delta = 0.0f;                  // kDq: of the row
        auto read_own = [&](int item) {                          // (rows of a query block: [LSE 128][delta 128])
            if (kDkv || item < 0) return;
            const float* own = args.rows + static_cast<long long>(item) * (2 * kBwdBlock) + row;
            own_lse = __ldg(own);
            own_delta = __ldg(own + kBwdBlock);
        };
        // P = 2^(S c1 - LSE log2 e) of 32 columns, kept in fp32 for dS; part of the exponentials on the FMA pipe
        auto exps = [&](const uint32_t* sv, float* p, uint32_t lse_smem) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                float4 l = make_float4(own_lse, own_lse, own_lse, own_lse);
                if (kDkv) l = ld_shared_f4(lse_smem + c * 4);
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    const uint64_t x = fma_f32x2(pack_f32x2(__uint_as_float(sv[c + u]), __uint_as_float(sv[c + u + 1])), c1c1,
                                                 u == 0 ? pack_f32x2(-l.x, -l.y) : pack_f32x2(-l.z, -l.w));
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
        auto ds_of = [&](const uint32_t* dp, const float* p, uint32_t delta_smem, uint32_t* ds) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
                float4 d = make_float4(own_delta, own_delta, own_delta, own_delta);
                if (kDkv) d = ld_shared_f4(delta_smem + c * 4);
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    const uint64_t v = add_f32x2(pack_f32x2(__uint_as_float(dp[c + u]), __uint_as_float(dp[c + u + 1])),
                                                 u == 0 ? pack_f32x2(-d.x, -d.y) : pack_f32x2(-d.z, -d.w));
                    float v0, v1;
                    unpack_f32x2(mul_f32x2(v, pack_f32x2(p[c + u], p[c + u + 1])), v0, v1);
                    ds[(c + u) >> 1] = pack_bf16(v0, v1);
                }
            }
        };
        int T = 0;
        int s_buf = 0;                                           // kDq: the score buffer of S_T, 2 T mod 3; dP_T is in the next one
        int4 cur;
        bool ok = item_at(0, cur);
        if (ok) read_own(cur.x);
        for (int it = 0; ok && cur.x >= 0; ++it) {
            const int n = cur.y;
            const int last_valid = kDkv ? kBwdBlock : args.L_other - cur.z * kBwdBlock;      // kDq: keys of the last block
            for (int j = 0; j < n; ++j, ++T, s_buf = s_buf >= 1 ? s_buf - 1 : s_buf + 2) {
                if (!kDkv && (T & 1) != group) continue;
                const uint32_t buf_s = tmem + lane_base + kScore0 + (kDkv ? 0 : s_buf * 128);
                const uint32_t buf_dp = tmem + lane_base + kScore0 + (kDkv ? 128 : (s_buf == 2 ? 0 : s_buf + 1) * 128);
                const uint32_t rows_smem = smem + Plan::kRowsOff + (T & 1) * Plan::kRowsBytes;
                const uint32_t phase = static_cast<uint32_t>(T >> 1) & 1u;
                if (kDkv) ok = mbar_wait_patient(smem_u32(&bar_rows_full[T & 1]), phase, abort_state);
                if (ok) ok = mbar_wait_patient(smem_u32(&bar_s_full[T & 1]), phase, abort_state);
                if (!ok) break;
                tc_fence_after();
#pragma unroll 1
                for (int half = 0; half < (kDkv ? 1 : 2); ++half) {
                    const int col0 = 64 * (kDkv ? group : half);
                    uint32_t sv[64];
                    float p[64];
                    TMEM_LD32(buf_s + col0, sv, 0);
                    TMEM_LD32(buf_s + col0 + 32, sv, 32);
                    tc_wait_ld();
                    if (!kDkv && half == 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bar_p_ready[T & 1]));
                    }
#pragma unroll
                    for (int c0 = 0; c0 < 64; c0 += 32) {
                        exps(sv + c0, p + c0, rows_smem + (col0 + c0) * 4);
                        if (kDkv) {
                            // P^T in bf16 over the S that it came from; the MMAs take it in two halves
                            uint32_t pk[16];
#pragma unroll
                            for (int c = 0; c < 16; ++c) pk[c] = pack_bf16(p[c0 + 2 * c], p[c0 + 2 * c + 1]);
                            TMEM_ST16(buf_s + col0 + c0 / 2, pk, 0);
                            tc_wait_st();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(smem_u32(c0 == 0 ? &bar_p_half[T & 1] : &bar_p_ready[T & 1]));
                        }
                    }
                    if (!kDkv && j + 1 == n && last_valid < kBwdBlock) {
                        // keys behind the last one: their zero rows of K make any finite dS harmless, but 2^(-LSE) need not be finite
#pragma unroll
                        for (int c = 0; c < 64; ++c) if (col0 + c >= last_valid) p[c] = 0.0f;
                    }
                    if (half == 0) {
                        ok = mbar_wait_patient(smem_u32(&bar_dp_full[T & 1]), phase, abort_state);
                        if (!ok) break;
                        tc_fence_after();
                    }
                    uint32_t ds[32];
#pragma unroll
                    for (int c0 = 0; c0 < 64; c0 += 32) {
                        uint32_t dp[32];
                        TMEM_LD32(buf_dp + col0 + c0, dp, 0);
                        tc_wait_ld();
                        ds_of(dp, p + c0, rows_smem + (kBwdBlock + col0 + c0) * 4, ds + c0 / 2);
                    }
                    TMEM_ST32(buf_dp + col0, ds, 0);
                }
                if (!ok) break;
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_ds_ready[T & 1]));
            }
            if (!ok) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_item_empty[it % kItemRing]));
            ok = item_at(it + 1, cur);
            if (ok) read_own(cur.x);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBwdRegsEpilogue));
        // ---- accumulators out: thread (warp, lane) owns row 32 (warp % 4) + lane of both ----
        const int row = (warp & 3) * 32 + lane;
        const uint32_t acc = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        int4 cur;
        bool ok = item_at(0, cur);
        for (int it = 0; ok && cur.x >= 0; ++it) {
            const int item = cur.x;
            const int bh = item / args.n_items_per_head, b = bh / args.H, h = bh - b * args.H;
            const int r = (item - bh * args.n_items_per_head) * kBwdBlock + row;
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
}

}  // namespace attn_jvp
