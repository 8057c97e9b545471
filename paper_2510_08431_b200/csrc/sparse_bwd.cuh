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
// 384 threads: warp 0 issues the MMAs, warp 1 the TMA loads, warps 4..11 work on the scores: warp w owns the rows (lanes)
// 32 (w % 4) .. + 31 and the columns 64 ((w - 4) / 4) .. + 63 of every 128 x 128 score tile.
//
// Order of work, kDkv (tensor memory: dV, dK, one buffer for S, one for dP, 512 columns at D = 128): P^T overwrites S and
// dS^T overwrites dP, and the MMAs of tile j + 1 are queued behind those that read them,
//     dV += P_j dO_j, S_(j+1) = K Q_(j+1)^T   |   dK += dS_j Q_j, dP_(j+1) = V dO_(j+1)^T
// so the exponentials of tile j + 1 run beside dK_j and dP_(j+1), and its dS beside dV_(j+1) and S_(j+2).
// kDq has no P operand and one accumulator: three score buffers in turn (matrix 2 j is S_j, 2 j + 1 is dP_j, matrix m is in
// buffer m % 3) let S run two tiles ahead.
#pragma once

#include "attn_jvp_kernel.cuh"

namespace attn_jvp {

constexpr int kBwdBlock = 128;
constexpr int kBwdThreads = 384;
constexpr int kBwdComputeWarps = 8;
constexpr int kBwdY1 = 3, kBwdY2 = 2;        // shared-memory buffers of the two streaming tensors

struct SparseBwdArgs {
    const int* list;            // kDkv: [B][H][n_k][n_q] query blocks of a key block; kDq: [B][H][n_q][n_k]
    const int* tiles;           // their lengths in 64-token tiles
    const float2* rows;         // [B][H][n_q * 128]: {LSE log2 e (+inf: the row has no probability), delta}
    __nv_bfloat16* out1;        // kDkv: dV, kDq: dQ        [B][L][H][D]
    __nv_bfloat16* out2;        // kDkv: dK
    int* host_status;
    int H, n_items_per_head, list_stride;
    int L_own, L_other;         // tokens on the stationary / streaming side
    int n_q;                    // query blocks
    float scale, scale_log2;
};

template <int D>
struct SparseBwdPlan {
    static constexpr int kHalf = kBwdBlock * 128;                // 128 rows x 64 bf16
    static constexpr int kTile = (D / 64) * kHalf;               // a 128 x D operand
    static constexpr int kX = 0;
    static constexpr int kY1Off = 2 * kTile;
    static constexpr int kY2Off = kY1Off + kBwdY1 * kTile;
    static constexpr int kRowsOff = kY2Off + kBwdY2 * kTile;     // kDkv: {LSE, delta} of two streaming tiles
    static constexpr int kRowsBytes = kBwdBlock * 8;
    static constexpr int kDynBytes = kRowsOff + 2 * kRowsBytes;  // 226 KB at D = 128
};

// {LSE log2 e, delta} per query row, padded to whole blocks.  Rows behind the last query and rows without any key get
// LSE = +inf, which makes their P exactly 0.  One group of D / 8 threads per row; reads dO and O once.
template <int D>
__global__ void __launch_bounds__(256)
sparse_bwd_rows_kernel(const uint4* __restrict__ o, const uint4* __restrict__ d_o, const float* __restrict__ lse,
                       float2* __restrict__ rows, int B, int H, int Lq, int padded) {
    constexpr int kLanes = D / 8;
    const long long n = static_cast<long long>(B) * padded * H;
    const long long r = (static_cast<long long>(blockIdx.x) * 256 + threadIdx.x) / kLanes;
    const int sub = threadIdx.x % kLanes;
    // (row order [B][padded][H], that of the tensors)
    const long long bl = min(r, n - 1) / H;
    const int h = static_cast<int>(min(r, n - 1) - bl * H);
    const int b = static_cast<int>(bl / padded), l = static_cast<int>(bl - static_cast<long long>(b) * padded);
    float sum = 0.0f;
    if (l < Lq) {
        const long long at = ((static_cast<long long>(b) * Lq + l) * H + h) * kLanes + sub;
        const uint4 x = __ldg(o + at), y = __ldg(d_o + at);
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), sum);
            sum = fmaf(__uint_as_float(xs[i] & 0xFFFF0000u), __uint_as_float(ys[i] & 0xFFFF0000u), sum);
        }
    }
#pragma unroll
    for (int m = kLanes / 2; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
    if (sub == 0 && r < n) {
        const long long bh = static_cast<long long>(b) * H + h;
        float ls = INFINITY;
        if (l < Lq) {
            ls = lse[bh * Lq + l] * 1.4426950408889634f;
            if (ls == -INFINITY) ls = INFINITY;
        }
        rows[bh * padded + l] = make_float2(ls, sum);
    }
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
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
    static_assert(kScore0 + kBufs * 128 <= kTmemCols, "tensor memory");

    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_x, bar_y1_full[kBwdY1], bar_y1_empty[kBwdY1], bar_y2_full[kBwdY2], bar_y2_empty[kBwdY2];
    __shared__ __align__(8) uint64_t bar_rows_full[2];           // kDkv: {LSE, delta} of the tile
    // per tile, two barriers in turn (tile j: [j & 1], phase (j >> 1) & 1): kDq's S and dP run up to two tiles ahead of the
    // warps that wait for them, which a single barrier's parity could not tell apart
    __shared__ __align__(8) uint64_t bar_s_full[2], bar_dp_full[2];      // S_j / dP_j complete
    __shared__ __align__(8) uint64_t bar_p_ready[2];             // kDkv: P_j is in tensor memory; kDq: S_j has been read
    __shared__ __align__(8) uint64_t bar_ds_ready[2];            // dS_j is in tensor memory
    __shared__ __align__(8) uint64_t bar_done, bar_drain;
    __shared__ uint32_t tmem_base_smem;
    __shared__ int cta_abort;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int lane = threadIdx.x & 31;
    const int item = blockIdx.x;
    const int bh = item / args.n_items_per_head, blk = item - bh * args.n_items_per_head;
    const int b = bh / args.H, h = bh - b * args.H;
    const int own0 = blk * kBwdBlock;
    const int* list = args.list + static_cast<long long>(item) * args.list_stride;
    const int n = min((args.tiles[item] + 1) >> 1, args.list_stride);     // streaming blocks of this item

    if (n <= 0) {
        // nothing was kept: the gradients are zero
        for (int e = threadIdx.x; e < kBwdBlock * (D / 8); e += kBwdThreads) {
            const int r = own0 + e / (D / 8), c = (e % (D / 8)) * 8;
            if (r < args.L_own) {
                const long long at = ((static_cast<long long>(b) * args.L_own + r) * args.H + h) * D + c;
                *reinterpret_cast<uint4*>(args.out1 + at) = make_uint4(0u, 0u, 0u, 0u);
                if (kDkv) *reinterpret_cast<uint4*>(args.out2 + at) = make_uint4(0u, 0u, 0u, 0u);
            }
        }
        return;
    }

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
        mbar_init(smem_u32(&bar_x), 1);
        for (int i = 0; i < kBwdY1; ++i) { mbar_init(smem_u32(&bar_y1_full[i]), 1); mbar_init(smem_u32(&bar_y1_empty[i]), 1); }
        for (int i = 0; i < kBwdY2; ++i) { mbar_init(smem_u32(&bar_y2_full[i]), 1); mbar_init(smem_u32(&bar_y2_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bar_rows_full[i]), 1);
            mbar_init(smem_u32(&bar_s_full[i]), 1);
            mbar_init(smem_u32(&bar_dp_full[i]), 1);
            mbar_init(smem_u32(&bar_p_ready[i]), kBwdComputeWarps);
            mbar_init(smem_u32(&bar_ds_ready[i]), kBwdComputeWarps);
        }
        mbar_init(smem_u32(&bar_done), 1);
        mbar_init(smem_u32(&bar_drain), 1);
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

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLightWarps));
        if (warp == kProducerWarp && lane == 0) {
            // ---- TMA producer: X once, then Y1_0, Y2_0, Y1_1, ... in the order the MMAs take them ----
            prefetch_tensormap(&tm_x1);
            prefetch_tensormap(&tm_x2);
            prefetch_tensormap(&tm_y1);
            prefetch_tensormap(&tm_y2);
            auto load_tile = [&](uint32_t dst, const CUtensorMap* map, uint32_t bar, int row0) {
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) tma_load_4d(dst + hf * Plan::kHalf, map, bar, hf * 64, h, row0, b);
            };
            mbar_arrive_expect_tx(smem_u32(&bar_x), 2 * Plan::kTile);
            load_tile(smem + Plan::kX, &tm_x1, smem_u32(&bar_x), own0);
            load_tile(smem + Plan::kX + Plan::kTile, &tm_x2, smem_u32(&bar_x), own0);
            const float2* rows = args.rows + static_cast<long long>(bh) * args.n_q * kBwdBlock;
            bool ok = true;
            int s1 = 0, s2 = 0;
            uint32_t ph1 = 0, ph2 = 0;                           // parity of the buffers' current lap
            for (int j = 0; j < n; ++j) {
                const int other = __ldg(list + j);
                const int row0 = other * kBwdBlock;
                if (j >= kBwdY1) ok = mbar_wait(smem_u32(&bar_y1_empty[s1]), ph1 ^ 1u, abort_state);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bar_y1_full[s1]), Plan::kTile);
                load_tile(smem + Plan::kY1Off + s1 * Plan::kTile, &tm_y1, smem_u32(&bar_y1_full[s1]), row0);
                if (j >= kBwdY2) ok = mbar_wait(smem_u32(&bar_y2_empty[s2]), ph2 ^ 1u, abort_state);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bar_y2_full[s2]), Plan::kTile);
                load_tile(smem + Plan::kY2Off + s2 * Plan::kTile, &tm_y2, smem_u32(&bar_y2_full[s2]), row0);
                if (kDkv) {
                    // Two sets of row constants: the one of tile j - 2 is free once that tile's dS has been formed, which
                    // the release of its Q tile (after dK += dS Q) says
                    if (j >= 2) {
                        const int t = j - 2;
                        ok = mbar_wait(smem_u32(&bar_y1_empty[t % kBwdY1]), static_cast<uint32_t>(t / kBwdY1) & 1u, abort_state);
                        if (!ok) break;
                    }
                    const uint32_t rb = smem_u32(&bar_rows_full[j & 1]);
                    mbar_arrive_expect_tx(rb, Plan::kRowsBytes);
                    bulk_load(smem + Plan::kRowsOff + (j & 1) * Plan::kRowsBytes, rows + row0, Plan::kRowsBytes, rb);
                }
                if (++s1 == kBwdY1) { s1 = 0; ph1 ^= 1u; }
                if (++s2 == kBwdY2) { s2 = 0; ph2 ^= 1u; }
            }
            if (!ok) {
                // give up: let the copies in flight land (bounded) before the CTA exits
                const unsigned long long t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < 100000000ull) {}
            }
        } else if (warp == kMmaWarp) {
            // ---- MMA issuer (whole warp in lock step, one elected lane's instructions take effect) ----
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
            auto values = [&](uint32_t d, uint32_t a, uint32_t y, bool first) {
                const uint32_t y_lo = make_desc_lo(y, Plan::kHalf);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    mma_ts_if<false>(pred, d, a + (k / 4) * 64 + (k % 4) * 8, make_desc(y_lo + k * (2048 >> 4)), kIdescV,
                                     (first && k == 0) ? 0u : 1u);
            };
            auto y1 = [&](int j) { return smem + Plan::kY1Off + (j % kBwdY1) * Plan::kTile; };
            auto y2 = [&](int j) { return smem + Plan::kY2Off + (j % kBwdY2) * Plan::kTile; };
            auto y1_full = [&](int j) { return mbar_wait_warp(smem_u32(&bar_y1_full[j % kBwdY1]), static_cast<uint32_t>(j / kBwdY1) & 1u, abort_state); };
            auto y2_full = [&](int j) { return mbar_wait_warp(smem_u32(&bar_y2_full[j % kBwdY2]), static_cast<uint32_t>(j / kBwdY2) & 1u, abort_state); };
            auto commit = [&](uint64_t& bar) { tc_commit_if<false>(pred, smem_u32(&bar)); };
            auto buf = [&](int m) { return tmem + kScore0 + (m % kBufs) * 128; };
            bool ok = mbar_wait_warp(smem_u32(&bar_x), 0, abort_state) && y1_full(0);
            if (ok) {
                scores(buf(0), x1_lo, y1(0));
                commit(bar_s_full[0]);
                ok = y2_full(0);
            }
            if (ok) {
                scores(buf(1), x2_lo, y2(0));
                commit(bar_dp_full[0]);
                if (!kDkv) commit(bar_y2_empty[0]);
            }
            if (kDkv) {
                for (int j = 0; ok && j < n; ++j) {
                    ok = mbar_wait_warp(smem_u32(&bar_p_ready[j & 1]), (j >> 1) & 1, abort_state);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem, buf(0), y2(j), j == 0);
                    commit(bar_y2_empty[j % kBwdY2]);
                    if (j + 1 < n) {
                        ok = y1_full(j + 1);
                        if (!ok) break;
                        scores(buf(0), x1_lo, y1(j + 1));
                        commit(bar_s_full[(j + 1) & 1]);
                    }
                    ok = mbar_wait_warp(smem_u32(&bar_ds_ready[j & 1]), (j >> 1) & 1, abort_state);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem + kAcc2, buf(1), y1(j), j == 0);
                    commit(bar_y1_empty[j % kBwdY1]);
                    if (j + 1 < n) {
                        ok = y2_full(j + 1);
                        if (!ok) break;
                        scores(buf(1), x2_lo, y2(j + 1));
                        commit(bar_dp_full[(j + 1) & 1]);
                    }
                }
            } else {
                if (ok && n > 1) {
                    ok = y1_full(1);
                    if (ok) {
                        scores(buf(2), x1_lo, y1(1));
                        commit(bar_s_full[1]);
                    }
                }
                for (int j = 0; ok && j < n; ++j) {
                    if (j + 1 < n) {
                        // dP_(j+1) goes where S_j was, once that has been read
                        ok = y2_full(j + 1) && mbar_wait_warp(smem_u32(&bar_p_ready[j & 1]), (j >> 1) & 1, abort_state);
                        if (!ok) break;
                        tc_fence_after();
                        scores(buf(2 * j + 3), x2_lo, y2(j + 1));
                        commit(bar_dp_full[(j + 1) & 1]);
                        commit(bar_y2_empty[(j + 1) % kBwdY2]);
                    }
                    ok = mbar_wait_warp(smem_u32(&bar_ds_ready[j & 1]), (j >> 1) & 1, abort_state);
                    if (!ok) break;
                    tc_fence_after();
                    values(tmem, buf(2 * j + 1), y1(j), j == 0);
                    commit(bar_y1_empty[j % kBwdY1]);
                    if (j + 2 < n) {
                        ok = y1_full(j + 2);
                        if (!ok) break;
                        scores(buf(2 * j + 4), x1_lo, y1(j + 2));     // (the buffer that dS_j is read from by the MMAs before it)
                        commit(bar_s_full[j & 1]);
                    }
                }
            }
            if (ok) commit(bar_done);
            if (!ok) {
                // give up: wait (bounded) until the tensor core has drained what was issued
                commit(bar_drain);
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(smem_u32(&bar_drain), 0) && globaltimer_ns() - t0 < 100000000ull) {}
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmaxWarps));
        // ---- scores: this thread's row and 64 of its columns ----
        const int quarter = warp & 3, col0 = ((warp - 4) >> 2) * 64;
        const int row = quarter * 32 + lane;
        const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
        const float c1 = args.scale_log2;
        float2 own = make_float2(0.0f, 0.0f);                    // kDq: the row's {LSE, delta}
        if (!kDkv) own = __ldg(args.rows + (static_cast<long long>(bh) * args.n_q + blk) * kBwdBlock + row);
        const int last_valid = args.L_other - (kDkv ? 0 : __ldg(list + n - 1) * kBwdBlock);   // kDq: keys of the last block
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const uint32_t tm_s = tmem + lane_base + kScore0 + (kDkv ? 0 : ((2 * j) % kBufs) * 128) + col0;
            const uint32_t tm_dp = tmem + lane_base + kScore0 + (kDkv ? 128 : ((2 * j + 1) % kBufs) * 128) + col0;
            const uint32_t rows_smem = smem + Plan::kRowsOff + (j & 1) * Plan::kRowsBytes + col0 * 8;
            uint32_t sv[64];
            if (kDkv) ok = mbar_wait_warp(smem_u32(&bar_rows_full[j & 1]), (j >> 1) & 1, abort_state);
            if (ok) ok = mbar_wait_warp(smem_u32(&bar_s_full[j & 1]), (j >> 1) & 1, abort_state);
            if (!ok) break;
            tc_fence_after();
            TMEM_LD32(tm_s, sv, 0);
            TMEM_LD32(tm_s + 32, sv, 32);
            tc_wait_ld();
            if (!kDkv) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p_ready[j & 1]));
            }
            // P = 2^(S c1 - LSE log2 e), kept in fp32 for dS
            float p[64];
            if (kDkv) {
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 64; c += 2) {
                    const float4 r = ld_shared_f4(rows_smem + c * 8);     // LSE, delta of two queries
                    p[c] = ex2f(fmaf(__uint_as_float(sv[c]), c1, -r.x));
                    p[c + 1] = ex2f(fmaf(__uint_as_float(sv[c + 1]), c1, -r.z));
                    pk[c >> 1] = pack_bf16(p[c], p[c + 1]);
                }
                TMEM_ST32(tm_s, pk, 0);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_p_ready[j & 1]));
            } else {
#pragma unroll
                for (int c = 0; c < 64; ++c) p[c] = ex2f(fmaf(__uint_as_float(sv[c]), c1, -own.x));
                if (j + 1 == n && last_valid < kBwdBlock) {
                    // keys behind the last one: their zero rows of K make any finite dS harmless, but 2^(-LSE) need not be finite
#pragma unroll
                    for (int c = 0; c < 64; ++c) if (col0 + c >= last_valid) p[c] = 0.0f;
                }
            }
            ok = mbar_wait_warp(smem_u32(&bar_dp_full[j & 1]), (j >> 1) & 1, abort_state);
            if (!ok) break;
            tc_fence_after();
            uint32_t ds[32];
#pragma unroll
            for (int c0 = 0; c0 < 64; c0 += 32) {
                uint32_t dp[32];
                TMEM_LD32(tm_dp + c0, dp, 0);
                tc_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    float d0 = own.y, d1 = own.y;
                    if (kDkv) {
                        const float4 r = ld_shared_f4(rows_smem + (c0 + c) * 8);
                        d0 = r.y;
                        d1 = r.w;
                    }
                    ds[(c0 + c) >> 1] = pack_bf16(p[c0 + c] * (__uint_as_float(dp[c]) - d0), p[c0 + c + 1] * (__uint_as_float(dp[c + 1]) - d1));
                }
            }
            TMEM_ST32(tm_dp, ds, 0);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_ds_ready[j & 1]));
        }
        // ---- accumulators out: kDkv: the first four warps dV, the others dK; kDq: half of the columns each ----
        if (ok) ok = mbar_wait_warp(smem_u32(&bar_done), 0, abort_state);
        if (ok) {
            tc_fence_after();
            const bool second = col0 != 0;
            constexpr int kCols = kDkv ? D : D / 2;
            const uint32_t acc = tmem + lane_base + (second ? (kDkv ? kAcc2 : D / 2) : 0);
            __nv_bfloat16* out = (kDkv && second) ? args.out2 : args.out1;
            const float factor = (kDkv && !second) ? 1.0f : args.scale;
            const int r = own0 + row;
            const long long at = ((static_cast<long long>(b) * args.L_own + r) * args.H + h) * D + (kDkv ? 0 : (second ? D / 2 : 0));
#pragma unroll
            for (int c0 = 0; c0 < kCols; c0 += 32) {
                uint32_t v[32];
                TMEM_LD32(acc + c0, v, 0);
                tc_wait_ld();
                if (r < args.L_own) {
#pragma unroll
                    for (int c = 0; c < 32; c += 8) {
                        uint32_t u[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            u[i] = pack_bf16(__uint_as_float(v[c + 2 * i]) * factor, __uint_as_float(v[c + 2 * i + 1]) * factor);
                        *reinterpret_cast<uint4*>(out + at + c0 + c) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                }
            }
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
