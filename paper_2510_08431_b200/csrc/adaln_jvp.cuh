// Gate + residual + norm + modulation around the branches of a DiT block, in one pass over HBM: forward, with
// tangents, and backward.  For one token (a row of C channels) of batch b:
//     hn = post(h)                   layer: (h - mean h) rp, rp = (var h + eps)^-1/2;  rms: h rp, rp = (mean h^2 + eps)^-1/2
//     x' = x + gate_b . (wp . hn)
//     n  = norm(x'),   y = n . w (1 + scale_b) + shift_b
// A normalisation's derivative applied to t is r (t - [mean t] - n mean(n t)) (the bracket for layer only).  The matrix
// is symmetric, so the same expression serves the tangent and the gradient:
//     tn = r (tx' - [mean tx'] - n mean(n tx')),   ty = tn . w (1 + scale) + n . w tscale + tshift
//     dx = dx' + r (dn - [mean dn] - n mean(n dn)),   dn = dy . w (1 + scale)
// and per batch and channel dshift = sum_l dy, dscale = w sum_l dy n, dgate = wp sum_l dx hn.
//
// Bound by HBM: a few dozen operations per element against 8 to 24 bytes.  One CTA works on one row at a time (the
// forward on two), thread t owns channels 8 t .. 8 t + 7 (16-byte accesses) and keeps that batch's modulation of its
// channels in registers while the CTA walks down its rows, so HBM sees each row once and the modulation about never.
// Rows come in through cp.async into a slot of shared memory that only the issuing thread reads back: the ring needs
// no barrier, and it keeps several rows per CTA in flight whatever the registers allow.
// All sums a row needs (of x', of x'^2, of t, of x' t) go through ONE block-wide reduction: each warp takes them
// about its own mean and the warps' results are shifted to the row's mean when they are joined, so that a row whose
// mean is large against its deviation loses nothing and no second pass over the block is needed.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace attn_jvp {

constexpr int kAdalnMaxC = 8192;            // 1024 threads of 8 channels
// kinds of a normalisation (ATTN_JVP_NORM_*); kAdalnMeans: row_norms() hands out mean t and mean(x t) alone
constexpr int kAdalnNone = 0, kAdalnLayer = 1, kAdalnRms = 2, kAdalnMeans = 3;

struct AdalnParams {
    const void *x, *tx, *dxn;               // [B][L][C], bf16 or fp32
    const __nv_bfloat16 *h, *th, *dy;       // [B][L][C]
    const float *gate, *scale, *shift, *tgate, *tscale, *tshift;    // [B] rows of C, strides below (elements)
    long long ld_gate, ld_scale, ld_shift, ld_tgate, ld_tscale, ld_tshift;
    const float *w, *wp;                    // [C]
    void *xn, *txn, *dx;                    // outputs, type of x
    __nv_bfloat16 *y, *ty, *dh;
    float* part;                            // backward: [gridDim.x][3][C] column sums of each CTA
    int L, C, norm, post;
    int rows_per_cta, chunks;               // CTAs per batch
    float eps;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void bf16x8_to_f32(const uint4& r, float (&v)[8]) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 f32_to_bf16x8(const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// outputs are not read again by this kernel: streaming stores
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), f32_to_bf16x8(v));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
template <typename T>
__device__ __forceinline__ void load_slot(uint32_t a, float (&v)[8]);
template <>
__device__ __forceinline__ void load_slot<__nv_bfloat16>(uint32_t a, float (&v)[8]) { bf16x8_to_f32(lds128(a), v); }
template <>
__device__ __forceinline__ void load_slot<float>(uint32_t a, float (&v)[8]) {
    // (the two halves of all threads' 32 bytes lie apart so that 16-byte accesses of a warp are contiguous)
    const uint4 lo = lds128(a), hi = lds128(a + blockDim.x * 16);
    const uint32_t u[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
}
template <typename T>
__device__ __forceinline__ void fetch_slot(uint32_t a, const T* src) {
    cp_async16(a, src);
    if (sizeof(T) == 4) cp_async16(a + blockDim.x * 16, src + 4);
}
// 8 values of a modulation row, `none` where there is none
__device__ __forceinline__ void load_mod(const float* p, long long off, float none, float (&v)[8]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    } else {
        p += off;
        if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
            const float4 lo = __ldg(reinterpret_cast<const float4*>(p)), hi = __ldg(reinterpret_cast<const float4*>(p) + 1);
            v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
            v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
        } else {        // (a row of any stride is 4-byte aligned at least)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __ldg(p + i);
        }
    }
}

// What a row's normalisation needs, the same in every thread: n = (x - mean) r, and for a companion row t the two
// constants of r (t - tbar - n q).
struct RowNorm { float mean, r, tbar, q; };

// One block-wide reduction for kRows rows at a time.  `red`: 2 x kRows x 32 float4 of shared memory used in turn
// (`turn` flips per call: one barrier per call suffices, since a buffer is written again only after the next call's
// barrier, which every thread reaches after its reads).
template <int kRows, bool kCompanion>
__device__ __forceinline__ void row_norms(const float (&x)[kRows][8], const float (&t)[kRows][8], bool active, int C, int kind,
                                          float eps, float4* red, int& turn, RowNorm (&out)[kRows]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5;
    const int n_mine = min(256, C - warp * 256);                 // channels of this warp
    float s[kRows], T[kRows], m2[kRows], q[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        s[k] = ((x[k][0] + x[k][1]) + (x[k][2] + x[k][3])) + ((x[k][4] + x[k][5]) + (x[k][6] + x[k][7]));
        T[k] = kCompanion ? ((t[k][0] + t[k][1]) + (t[k][2] + t[k][3])) + ((t[k][4] + t[k][5]) + (t[k][6] + t[k][7])) : 0.0f;
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            s[k] += __shfl_xor_sync(0xffffffffu, s[k], m);
            if (kCompanion) T[k] += __shfl_xor_sync(0xffffffffu, T[k], m);
        }
    const float inv_mine = 1.0f / static_cast<float>(n_mine);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const float mean = s[k] * inv_mine;
        m2[k] = q[k] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = active ? x[k][i] - mean : 0.0f;      // (threads past C hold zeros that are not channels)
            m2[k] = fmaf(d, d, m2[k]);
            if (kCompanion) q[k] = fmaf(d, t[k][i], q[k]);
        }
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            m2[k] += __shfl_xor_sync(0xffffffffu, m2[k], m);
            if (kCompanion) q[k] += __shfl_xor_sync(0xffffffffu, q[k], m);
        }
    const float inv_c = 1.0f / static_cast<float>(C);
    if (n_warps > 1) {
        float4* buf = red + turn * (kRows * 32);
        turn ^= 1;
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < kRows; ++k) buf[k * 32 + warp] = make_float4(s[k], m2[k], T[k], q[k]);
        }
        __syncthreads();
        float4 v[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            v[k] = lane < n_warps ? buf[k * 32 + lane] : make_float4(0.f, 0.f, 0.f, 0.f);
            s[k] = v[k].x;
            T[k] = v[k].z;
        }
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                s[k] += __shfl_xor_sync(0xffffffffu, s[k], m);
                if (kCompanion) T[k] += __shfl_xor_sync(0xffffffffu, T[k], m);
            }
        const float n_theirs = static_cast<float>(max(1, min(256, C - lane * 256)));
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const float d = lane < n_warps ? v[k].x / n_theirs - s[k] * inv_c : 0.0f;
            m2[k] = fmaf(n_theirs * d, d, v[k].y);
            if (kCompanion) q[k] = fmaf(d, v[k].z, v[k].w);
        }
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                m2[k] += __shfl_xor_sync(0xffffffffu, m2[k], m);
                if (kCompanion) q[k] += __shfl_xor_sync(0xffffffffu, q[k], m);
            }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const float mean = s[k] * inv_c;
        const bool layer = kind == kAdalnLayer;
        // rms: sum x^2 = M2 + C mean^2, sum x t = Q + mean sum t
        const float var = layer ? m2[k] * inv_c : fmaf(mean, mean, m2[k] * inv_c);
        out[k].mean = layer ? mean : 0.0f;
        out[k].r = 1.0f / sqrtf(var + eps);
        out[k].tbar = kCompanion && kind != kAdalnRms ? T[k] * inv_c : 0.0f;
        out[k].q = kCompanion ? inv_c * (layer ? q[k] : fmaf(mean, T[k], q[k])) : 0.0f;      // mean(x t), for layer of the centred x
        if (kind != kAdalnMeans) out[k].q *= out[k].r;
    }
}

// Shared memory per thread and ring stage: one 16-byte slot per bf16 operand, two per fp32 operand.
__host__ __device__ constexpr int adaln_slot_bytes(bool x_fp32, bool has_h, int companions) {
    // companions: rows that come beside x and h (forward 0; JVP: tx, th; backward: dx', dy)
    const int xs = x_fp32 ? 32 : 16;
    return (companions ? 2 : 1) * xs + (has_h ? 16 : 0) + (companions == 1 ? (has_h ? 16 : 0) : companions == 2 ? 16 : 0);
}

// kMode: 0 forward, 1 forward with tangents, 2 backward.  kThreads: the most threads a CTA is launched with.
template <typename TX, int kMode, int kRows, int kStages, int kThreads>
__global__ void __launch_bounds__(kThreads) adaln_kernel(const AdalnParams p) {
    extern __shared__ __align__(16) uint8_t adaln_smem[];
    __shared__ float4 red[2 * kRows * 32];
    constexpr bool kJvp = kMode == 1, kBwd = kMode == 2;
    const int t = threadIdx.x, c = 8 * t;
    const bool active = c < p.C;
    const int b = blockIdx.x / p.chunks;                         // a CTA's rows are of one batch
    const int row0 = (blockIdx.x - b * p.chunks) * p.rows_per_cta, row1 = min(p.L, row0 + p.rows_per_cta);
    const long long base = (static_cast<long long>(b) * p.L) * p.C + c;       // channel c of the batch's first token
    const bool has_h = p.h != nullptr, has_norm = p.norm != kAdalnNone, has_dxn = kBwd && p.dxn != nullptr, has_dy = kBwd && p.dy != nullptr;

    float gate[8], mul[8], shift[8], wp[8];
    float tgate[8], tmul[8], tshift[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gate[i] = mul[i] = shift[i] = wp[i] = tgate[i] = tmul[i] = tshift[i] = 0.0f;
    if (active) {
        // u = wp hn enters only as gate u: both factors in one
        load_mod(p.wp, c, 1.0f, wp);
        load_mod(p.gate, b * p.ld_gate + c, 1.0f, gate);
        load_mod(p.scale, b * p.ld_scale + c, 0.0f, mul);
        load_mod(p.shift, b * p.ld_shift + c, 0.0f, shift);
        float w[8];
        load_mod(p.w, c, 1.0f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gate[i] *= wp[i];
            mul[i] = w[i] * (1.0f + mul[i]);
        }
        if (kJvp) {
            load_mod(p.tgate, b * p.ld_tgate + c, 0.0f, tgate);
            load_mod(p.tscale, b * p.ld_tscale + c, 0.0f, tmul);
            load_mod(p.tshift, b * p.ld_tshift + c, 0.0f, tshift);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                tgate[i] *= wp[i];
                tmul[i] *= w[i];
            }
        }
    }

    // ring: stage s holds kRows rows; per row the slots x [, h] [, companion of x] [, companion of h / dy]
    const uint32_t smem = static_cast<uint32_t>(__cvta_generic_to_shared(adaln_smem)) + t * 16;
    const uint32_t plane = blockDim.x * 16;
    constexpr uint32_t kXPlanes = sizeof(TX) / 2;
    const uint32_t off_h = kXPlanes * plane, off_x2 = off_h + (has_h ? plane : 0);
    const uint32_t off_h2 = off_x2 + kXPlanes * plane;
    const uint32_t row_bytes = kMode == 0 ? off_x2 : off_h2 + ((kBwd || has_h) ? plane : 0);
    auto fetch = [&](int i, int stage) {          // kRows rows from row i on
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (active && i + k < row1) {
                const long long at = base + static_cast<long long>(i + k) * p.C;
                const uint32_t s = smem + (stage * kRows + k) * row_bytes;
                fetch_slot(s, static_cast<const TX*>(p.x) + at);
                if (has_h) fetch_slot(s + off_h, p.h + at);
                if (kJvp) {
                    fetch_slot(s + off_x2, static_cast<const TX*>(p.tx) + at);
                    if (has_h) fetch_slot(s + off_h2, p.th + at);
                }
                if (has_dxn) fetch_slot(s + off_x2, static_cast<const TX*>(p.dxn) + at);
                if (has_dy) fetch_slot(s + off_h2, p.dy + at);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(row0 + s * kRows, s);

    float sum_dy[8], sum_dyn[8], sum_dhn[8];
    if (kBwd) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_dy[i] = sum_dyn[i] = sum_dhn[i] = 0.0f;
    }
    int turn = 0, stage = 0;
    for (int row = row0; row < row1; row += kRows) {
        {
            int ahead = stage + kStages - 1;
            if (ahead >= kStages) ahead -= kStages;
            fetch(row + (kStages - 1) * kRows, ahead);       // (the slot read back an iteration ago, by this thread)
        }
        cp_async_wait<kStages - 1>();
        float x[kRows][8], h[kRows][8], x2[kRows][8], h2[kRows][8];     // x2, h2: tangents, or dx' and dy
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[k][i] = h[k][i] = x2[k][i] = h2[k][i] = 0.0f;
            if (active && row + k < row1) {
                const uint32_t s = smem + (stage * kRows + k) * row_bytes;
                load_slot<TX>(s, x[k]);
                if (has_h) load_slot<__nv_bfloat16>(s + off_h, h[k]);
                if (kJvp || has_dxn) load_slot<TX>(s + off_x2, x2[k]);
                if ((kJvp && has_h) || has_dy) load_slot<__nv_bfloat16>(s + off_h2, h2[k]);
            }
        }
        if (++stage == kStages) stage = 0;

        RowNorm hs[kRows], xs[kRows];
        if (has_h) {
            if (p.post != kAdalnNone) {
                row_norms<kRows, kJvp>(h, h2, active, p.C, p.post, p.eps, red, turn, hs);
#pragma unroll
                for (int k = 0; k < kRows; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        h[k][i] = active ? (h[k][i] - hs[k].mean) * hs[k].r : 0.0f;
                        if (kJvp) h2[k][i] = active ? hs[k].r * (h2[k][i] - hs[k].tbar - h[k][i] * hs[k].q) : 0.0f;
                    }
            }
#pragma unroll
            for (int k = 0; k < kRows; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[k][i] = fmaf(gate[i], h[k][i], x[k][i]);
                    if (kJvp) x2[k][i] = fmaf(gate[i], h2[k][i], fmaf(tgate[i], h[k][i], x2[k][i]));
                }
            if (!kBwd) {
#pragma unroll
                for (int k = 0; k < kRows; ++k) {
                    if (active && row + k < row1) {
                        const long long at = base + static_cast<long long>(row + k) * p.C;
                        store8(static_cast<TX*>(p.xn) + at, x[k]);
                        if (kJvp) store8(static_cast<TX*>(p.txn) + at, x2[k]);
                    }
                }
            }
        }
        if (!kBwd) {
            if (has_norm) {
                row_norms<kRows, kJvp>(x, x2, active, p.C, p.norm, p.eps, red, turn, xs);
#pragma unroll
                for (int k = 0; k < kRows; ++k) {
                    float y[8], ty[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float n = (x[k][i] - xs[k].mean) * xs[k].r;
                        y[i] = fmaf(n, mul[i], shift[i]);
                        if (kJvp) ty[i] = fmaf(xs[k].r * (x2[k][i] - xs[k].tbar - n * xs[k].q), mul[i], fmaf(n, tmul[i], tshift[i]));
                    }
                    if (active && row + k < row1) {
                        const long long at = base + static_cast<long long>(row + k) * p.C;
                        store8(p.y + at, y);
                        if (kJvp) store8(p.ty + at, ty);
                    }
                }
            }
        } else {
            float dn[kRows][8];
            if (has_norm) {
#pragma unroll
                for (int k = 0; k < kRows; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) dn[k][i] = h2[k][i] * mul[i];
                row_norms<kRows, true>(x, dn, active, p.C, p.norm, p.eps, red, turn, xs);
#pragma unroll
                for (int k = 0; k < kRows; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float n = active ? (x[k][i] - xs[k].mean) * xs[k].r : 0.0f;
                        sum_dy[i] += h2[k][i];
                        sum_dyn[i] = fmaf(h2[k][i], n, sum_dyn[i]);
                        x2[k][i] += active ? xs[k].r * (dn[k][i] - xs[k].tbar - n * xs[k].q) : 0.0f;
                    }
            }
#pragma unroll
            for (int k = 0; k < kRows; ++k) {       // x2 is the whole gradient of x' now, which is that of x
                if (active && row + k < row1)
                    store8(static_cast<TX*>(p.dx) + base + static_cast<long long>(row + k) * p.C, x2[k]);
            }
            if (has_h) {
#pragma unroll
                for (int k = 0; k < kRows; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sum_dhn[i] = fmaf(x2[k][i], h[k][i], sum_dhn[i]);
                        x2[k][i] *= gate[i];
                    }
                if (p.post != kAdalnNone) {
                    RowNorm es[kRows];       // h holds hn here: tbar = mean e, q = mean(e hn)
                    row_norms<kRows, true>(h, x2, active, p.C, kAdalnMeans, 0.0f, red, turn, es);
#pragma unroll
                    for (int k = 0; k < kRows; ++k)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            x2[k][i] = hs[k].r * (x2[k][i] - (p.post == kAdalnLayer ? es[k].tbar : 0.0f) - h[k][i] * es[k].q);
                }
#pragma unroll
                for (int k = 0; k < kRows; ++k)
                    if (active && row + k < row1) store8(p.dh + base + static_cast<long long>(row + k) * p.C, x2[k]);
            }
        }
    }
    if (kBwd && active) {
        float* out = p.part + static_cast<long long>(blockIdx.x) * 3 * p.C + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            out[i] = sum_dy[i];
            out[p.C + i] = sum_dyn[i];
            out[2 * p.C + i] = sum_dhn[i];
        }
    }
}

// Joins the CTAs' column sums, always in the same order (no atomics: a gradient is the same from run to run):
//     dshift = S0,  dscale = w S1,  dgate = wp S2,  dw = sum_b (1 + scale) S1,  dwp = sum_b gate S2.
// A block owns 32 channels; its 8 warps share the CTAs' rows.
constexpr int kAdalnJoinRows = 8;
struct AdalnJoin {
    const float* part;
    const float *gate, *scale, *w, *wp;
    long long ld_gate, ld_scale;
    float *dgate, *dscale, *dshift, *dw, *dwp;
    int B, C, n_parts;
};
__global__ void __launch_bounds__(32 * kAdalnJoinRows) adaln_join_kernel(const AdalnJoin p) {
    __shared__ float part[3][kAdalnJoinRows][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const bool active = c < p.C;
    float dw = 0.0f, dwp = 0.0f;
    for (int b = 0; b < p.B; ++b) {
        float s[3] = {0.0f, 0.0f, 0.0f};
        if (active) {
            const float* in = p.part + static_cast<long long>(b) * p.n_parts * 3 * p.C + c;
#pragma unroll 4
            for (int i = g; i < p.n_parts; i += kAdalnJoinRows) {
#pragma unroll
                for (int k = 0; k < 3; ++k) s[k] += in[(static_cast<long long>(i) * 3 + k) * p.C];
            }
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) part[k][g][lane] = s[k];
        __syncthreads();
        if (g == 0 && active) {
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                s[k] = 0.0f;
#pragma unroll
                for (int j = 0; j < kAdalnJoinRows; ++j) s[k] += part[k][j][lane];
            }
            const long long at = static_cast<long long>(b) * p.C + c;
            if (p.dshift) p.dshift[at] = s[0];
            if (p.dscale) p.dscale[at] = (p.w ? p.w[c] : 1.0f) * s[1];
            if (p.dgate) p.dgate[at] = (p.wp ? p.wp[c] : 1.0f) * s[2];
            dw = fmaf(1.0f + (p.scale ? p.scale[b * p.ld_scale + c] : 0.0f), s[1], dw);
            dwp = fmaf(p.gate ? p.gate[b * p.ld_gate + c] : 1.0f, s[2], dwp);
        }
        __syncthreads();
    }
    if (g == 0 && active) {
        if (p.dw) p.dw[c] = dw;
        if (p.dwp) p.dwp[c] = dwp;
    }
}

}  // namespace attn_jvp
