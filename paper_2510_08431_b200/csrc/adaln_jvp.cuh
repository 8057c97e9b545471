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
// Bound by HBM, if the instructions and the waits are kept few: a row of 5120 channels has 1700 cycles of an SM's share of
// the bandwidth in the forward pass, 2600 in the backward pass, and a row's sums are a chain of shuffles and a barrier.
// Hence two fp32 values per instruction (packed fp32x2 arithmetic), kRows rows at a time where one row's chain would not
// be covered by other CTAs (their shuffles interleave and share the barrier) or one row's sums beside the row before (kPipe),
// and only what a sum needs is held across it: everything else is read from shared memory again.
// Measured, inputs in HBM, launch after launch on the GPU alone: forward at 32760 x 5120 bf16 212 us (6.3 TB/s, 98 % of a copy's
// rate; a single call behind other work, which leaves L2 full of lines to write back, 229 to 239), forward and gradients 556 us
// (4.8 TB/s; 604 to 633), tangents at 2 x 4096 x 2048 with an fp32 stream 77 us (5.2 TB/s), with a post norm at 3 x 10007 x 1536 bf16
// 147 us (5.0 TB/s).  Widths between 2048 and 5120 and above 5120 channels are slower: see the launch code's comments.
// One CTA works down a range of rows, thread t owns channels 8 t .. 8 t + 7 (16-byte accesses) and keeps that batch's
// modulation of its channels in registers, so HBM sees each row once and the modulation about never.  Rows come in
// through cp.async into a slot of shared memory that only the issuing warp reads back: the ring needs no block-wide
// barrier, and it keeps several rows per CTA in flight whatever the registers allow.
// All sums a row needs (of x', of x'^2, of t, of x' t) go through ONE block-wide reduction of 5 + 5 shuffle levels.  They
// are taken about a pivot instead of zero, so that a row whose mean is large against its deviation loses nothing: a warp's
// pivot is the mean p of 8 of its n <= 256 channels, and since 8 (p - mean)^2 is part of the n var that the sum of squares
// holds, (p - mean)^2 <= 32 var: taking n (p - mean)^2 off again costs 5 bits at the very worst, on one outlier among the
// 8, and usually none.  The warps' results are joined the same way about the first warp's mean.
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
    bool wide;                              // fp32 outputs are 32-byte aligned
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
// Pairs of fp32 values (f32x2) hold two neighbouring channels.
using pair_t = uint64_t;
__device__ __forceinline__ pair_t pair_of(float lo, float hi) {
    pair_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ pair_t twice(float v) { return pair_of(v, v); }
__device__ __forceinline__ void halves(pair_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
    pair_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
    pair_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
    pair_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float sum2(pair_t v) {
    float a, b;
    halves(v, a, b);
    return a + b;
}
// 8 channels to and from memory
__device__ __forceinline__ void store8(__nv_bfloat16* p, const pair_t* v) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        halves(v[i], lo, hi);
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(u[0], u[1], u[2], u[3]));      // (not read again by this kernel)
}
__device__ __forceinline__ void store8(float* p, const pair_t* v) {
    __stcs(reinterpret_cast<ulonglong2*>(p), make_ulonglong2(v[0], v[1]));
    __stcs(reinterpret_cast<ulonglong2*>(p) + 1, make_ulonglong2(v[2], v[3]));
}
// `wide`: p is 32-byte aligned, and a thread's 32 bytes leave in one access (as two of 16, each would fill only half of
// every 32-byte sector it touches)
__device__ __forceinline__ void store8(float* p, const pair_t* v, bool wide) {
    if (wide) asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(v[0]), "l"(v[1]), "l"(v[2]), "l"(v[3]) : "memory");
    else store8(p, v);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const pair_t* v, bool) { store8(p, v); }
// A warp's 256 channels of an operand in the ring.  bf16: lane l's 16 bytes at 16 l.  fp32: 1024 bytes in their order in
// memory; lane l copies pieces l and l + 32 (whole sectors per access) and reads back the 32 bytes at 32 l, which other
// lanes of the warp have copied.
template <typename T>
__device__ __forceinline__ void load_slot(uint32_t a, int lane, pair_t* v) {
    if (sizeof(T) == 2) {
        const uint4 r = lds128(a + lane * 16);
        const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
    } else {
        const uint4 lo = lds128(a + lane * 32), hi = lds128(a + lane * 32 + 16);
        const uint32_t u[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
    }
}
// `src`: channel 0 of the warp in this row; `left`: channels from there to the row's end
template <typename T>
__device__ __forceinline__ void fetch_slot(uint32_t a, int lane, const T* src, int left) {
    constexpr int kPer = 16 / sizeof(T);                         // channels of a 16-byte piece
#pragma unroll
    for (int k = 0; k < 8 / kPer; ++k) {
        const int e = lane + 32 * k;
        if (e * kPer < left) cp_async16(a + e * 16, src + e * kPer);
    }
}
__device__ __forceinline__ void zero4(pair_t* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = 0ull;
}
// 8 values of a modulation row, `none` where there is none
__device__ __forceinline__ void load_mod(const float* p, long long off, float none, pair_t* v) {
    float f[8];
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = none;
    } else {
        p += off;
        if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
            const float4 lo = __ldg(reinterpret_cast<const float4*>(p)), hi = __ldg(reinterpret_cast<const float4*>(p) + 1);
            f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w;
            f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
        } else {        // (a row of any stride is 4-byte aligned at least)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __ldg(p + i);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

// What a row's normalisation needs, the same in every thread: n = (x - mean) r, and for a companion row t the two
// constants of r (t - tbar - n q).
struct RowNorm { float mean, r, tbar, q; };

// What a thread needs of the row's geometry, worked out once.
struct RowShape {
    float inv_c;          // 1 / C
    float inv_mine;       // 1 / channels of this warp
    float n_theirs;       // channels of the warp whose sums this lane joins (0: none)
    int warps2;           // warps of the CTA, rounded up to a power of two: lane reads the sums of warp lane % warps2
    bool active;          // this thread has channels (below C)
};

// Sums of N values over a warp's lanes, N = 2, 4 or 8: while a lane holds more than one value it hands half of them to its
// partner and takes the other half over, so that N values cost N - 1 + log2(32 / N) shuffles instead of 5 N.  Afterwards v[0]
// of lane l is the sum of value l / (32 / N).
template <int N>
__device__ __forceinline__ void join_lanes(float (&v)[N]) {
    const int lane = threadIdx.x & 31;
    int m = 16;
#pragma unroll
    for (int n = N / 2; n >= 1; n /= 2, m /= 2) {
        const bool upper = (lane & m) != 0;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = upper ? v[i] : v[i + n], keep = upper ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, m);
        }
    }
#pragma unroll
    for (; m >= 1; m /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
}

// One block-wide reduction for kRows rows.  `red`: 2 x kRows x 32 float4 of shared memory used in turn (`turn` flips per
// call: one barrier per call suffices, since a buffer is written again only after the next call's barrier, which every
// thread reaches after its reads).  Channels that a thread does not have (behind C) hold zeros.
template <int kRows, bool kCompanion>
__device__ __forceinline__ void row_norms(const pair_t (&x)[kRows][4], const pair_t (&t)[kRows][4], const RowShape& shape, int kind,
                                          float eps, float4* red, int& turn, RowNorm (&out)[kRows]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float s[kRows], m2[kRows], T[kRows], q[kRows], mean[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        // sums about a pivot near the warp's mean: the mean of the first 8 channels it has
        mean[r] = __shfl_sync(0xffffffffu, sum2(add2(add2(x[r][0], x[r][1]), add2(x[r][2], x[r][3]))), 0) * 0.125f;
        const pair_t minus = twice(shape.active ? -mean[r] : 0.0f);
        pair_t d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = add2(x[r][i], minus);
        s[r] = sum2(add2(add2(d[0], d[1]), add2(d[2], d[3])));
        m2[r] = sum2(add2(fma2(d[1], d[1], mul2(d[0], d[0])), fma2(d[3], d[3], mul2(d[2], d[2]))));
        T[r] = kCompanion ? sum2(add2(add2(t[r][0], t[r][1]), add2(t[r][2], t[r][3]))) : 0.0f;
        q[r] = kCompanion ? sum2(add2(fma2(d[1], t[r][1], mul2(d[0], t[r][0])), fma2(d[3], t[r][3], mul2(d[2], t[r][2])))) : 0.0f;
    }
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            s[r] += __shfl_xor_sync(0xffffffffu, s[r], m);
            m2[r] += __shfl_xor_sync(0xffffffffu, m2[r], m);
            if (kCompanion) T[r] += __shfl_xor_sync(0xffffffffu, T[r], m);
            if (kCompanion) q[r] += __shfl_xor_sync(0xffffffffu, q[r], m);
        }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {       // about the warp's mean
        const float d = s[r] * shape.inv_mine;
        mean[r] += d;
        m2[r] = fmaf(-d, s[r], m2[r]);
        if (kCompanion) q[r] = fmaf(-d, T[r], q[r]);
    }
    if (shape.warps2 > 1) {
        float4* buf = red + turn * (kRows * 32);
        turn ^= 1;
        if (lane == 0) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) buf[r * 32 + warp] = make_float4(mean[r], m2[r], T[r], q[r]);
        }
        __syncthreads();
        // the same again with the first warp's mean as the pivot
        // (the entries of warps that do not exist are zero from the start and are never written)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float4 v = buf[r * 32 + (lane & (shape.warps2 - 1))];
            mean[r] = buf[r * 32].x;
            const float d = v.x - mean[r];
            s[r] = shape.n_theirs * d;
            m2[r] = fmaf(s[r], d, v.y);
            T[r] = v.z;
            if (kCompanion) q[r] = fmaf(d, v.z, v.w);
        }
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1)
            if (m < shape.warps2) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    s[r] += __shfl_xor_sync(0xffffffffu, s[r], m);
                    m2[r] += __shfl_xor_sync(0xffffffffu, m2[r], m);
                    if (kCompanion) T[r] += __shfl_xor_sync(0xffffffffu, T[r], m);
                    if (kCompanion) q[r] += __shfl_xor_sync(0xffffffffu, q[r], m);
                }
            }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float d = s[r] * shape.inv_c;
            mean[r] += d;
            m2[r] = fmaf(-d, s[r], m2[r]);
            if (kCompanion) q[r] = fmaf(-d, T[r], q[r]);
        }
    }
    const bool layer = kind == kAdalnLayer;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        m2[r] = fmaxf(m2[r], 0.0f);         // (a row of equal values may leave a rounding below zero)
        // rms: sum x^2 = M2 + C mean^2, sum x t = Q + mean sum t
        const float var = layer ? m2[r] * shape.inv_c : fmaf(mean[r], mean[r], m2[r] * shape.inv_c);
        out[r].mean = layer ? mean[r] : 0.0f;
        out[r].r = rsqrtf(var + eps);
        out[r].tbar = kCompanion && kind != kAdalnRms ? T[r] * shape.inv_c : 0.0f;
        out[r].q = kCompanion ? shape.inv_c * (layer ? q[r] : fmaf(mean[r], T[r], q[r])) : 0.0f;   // mean(x t), layer: of the centred x
        if (kind != kAdalnMeans) out[r].q *= out[r].r;
    }
}

// Shared memory per thread and row of the ring: 16 bytes per bf16 operand, 32 per fp32 operand.
__host__ __device__ constexpr int adaln_slot_bytes(bool x_fp32, bool has_h, int companions) {
    // companions: rows that come beside x and h (forward 0; JVP 1: tx, th; backward 2: dx', dy)
    const int xs = x_fp32 ? 32 : 16;
    return (companions ? 2 : 1) * xs + (has_h ? 16 : 0) + (companions == 1 ? (has_h ? 16 : 0) : companions == 2 ? 16 : 0);
}

// kMode: 0 forward, 1 forward with tangents, 2 backward.  kThreads: the most threads a CTA is launched with; kCtas: how
// many of those an SM should hold.  kPipe: a row's sums are formed while the row before it is finished (for calls with a norm
// and without a post norm): the wait for one row's chain of shuffles is filled with the other row's arithmetic.
template <typename TX, int kMode, int kRows, int kStages, int kThreads, int kCtas, bool kPipe = false>
__global__ void __launch_bounds__(kThreads, kCtas) adaln_kernel(const AdalnParams p) {
    extern __shared__ __align__(16) uint8_t adaln_smem[];
    constexpr int kRed = 2 * kRows * 32 + (kPipe ? 16 : 0);     // (kPipe: pivots behind the sums)
    __shared__ float4 red[kRed];
    constexpr bool kJvp = kMode == 1, kBwd = kMode == 2;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, n_warps = blockDim.x >> 5;
    const int c = 8 * t, left = p.C - 256 * warp;                // first channel of the thread; channels from the warp's first on
    RowShape shape;
    shape.active = c < p.C;
    shape.warps2 = n_warps > 1 ? 1 << (32 - __clz(n_warps - 1)) : 1;
    {
        const int w = lane & (shape.warps2 - 1);
        shape.inv_c = 1.0f / static_cast<float>(p.C);
        shape.inv_mine = 1.0f / static_cast<float>(min(256, left));
        shape.n_theirs = w < n_warps ? static_cast<float>(min(256, p.C - w * 256)) : 0.0f;
        for (int i = t; i < kRed; i += blockDim.x) red[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const bool active = shape.active;
    const int b = blockIdx.x / p.chunks;                         // a CTA's rows are of one batch
    const int row0 = (blockIdx.x - b * p.chunks) * p.rows_per_cta, row1 = min(p.L, row0 + p.rows_per_cta);
    const long long first = (static_cast<long long>(b) * p.L + row0) * p.C;      // element 0 of the CTA's first row
    const bool has_h = p.h != nullptr, has_norm = p.norm != kAdalnNone, has_dxn = kBwd && p.dxn != nullptr, has_dy = kBwd && p.dy != nullptr;

    // ring of kStages x kRows rows: per row the operands x [, h] [, companion of x] [, companion of h / dy], each with
    // the warps' slots one after the other
    const uint32_t plane = blockDim.x * 16;
    constexpr uint32_t kXPlanes = sizeof(TX) / 2;
    const uint32_t smem = static_cast<uint32_t>(__cvta_generic_to_shared(adaln_smem));
    const uint32_t at_x = warp * 512 * kXPlanes, at_h = kXPlanes * plane + warp * 512;
    const uint32_t end_h = kXPlanes * plane + (has_h ? plane : 0);
    const uint32_t at_x2 = end_h + warp * 512 * kXPlanes, at_h2 = end_h + kXPlanes * plane + warp * 512;
    const uint32_t row_bytes = kMode == 0 ? end_h : end_h + kXPlanes * plane + ((kBwd || has_h) ? plane : 0);
    const uint32_t ring_end = smem + kStages * kRows * row_bytes;
    // channels behind C: their slots are read like the others and have to hold zeros
    if (left < 256) {
        for (uint32_t a = smem; a < ring_end; a += row_bytes)
            for (uint32_t o = lane * 16; o < 512 * kXPlanes; o += 512) {
                auto zero = [](uint32_t d) { asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(d), "r"(0) : "memory"); };
                zero(a + at_x + o);
                if (kMode != 0) zero(a + at_x2 + o);
                if (o < 512) {
                    if (has_h) zero(a + at_h + o);
                    if (kBwd || (kJvp && has_h)) zero(a + at_h2 + o);
                }
            }
        __syncwarp();
    }
    long long ahead = first + 256 * warp;                        // the row that is fetched next, at this warp's first channel
    int row_ahead = row0;
    uint32_t slot_ahead = smem;
    auto fetch = [&]() {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (row_ahead + r < row1) {
                const long long e = ahead + static_cast<long long>(r) * p.C;
                const uint32_t s = slot_ahead + r * row_bytes;
                fetch_slot(s + at_x, lane, static_cast<const TX*>(p.x) + e, left);
                if (has_h) fetch_slot(s + at_h, lane, p.h + e, left);
                if (kJvp) {
                    fetch_slot(s + at_x2, lane, static_cast<const TX*>(p.tx) + e, left);
                    if (has_h) fetch_slot(s + at_h2, lane, p.th + e, left);
                }
                if (has_dxn) fetch_slot(s + at_x2, lane, static_cast<const TX*>(p.dxn) + e, left);
                if (has_dy) fetch_slot(s + at_h2, lane, p.dy + e, left);
            }
        }
        cp_async_commit();
        ahead += static_cast<long long>(kRows) * p.C;
        row_ahead += kRows;
        slot_ahead += kRows * row_bytes;
        if (slot_ahead == ring_end) slot_ahead = smem;
    };
#pragma unroll
    for (int s = 0; s < kStages - (kPipe ? 2 : 1); ++s) fetch();

    pair_t gate[4], mul[4], shift[4], tgate[4], tmul[4], tshift[4];
    zero4(gate); zero4(mul); zero4(shift); zero4(tgate); zero4(tmul); zero4(tshift);
    if (active) {
        // u = wp hn enters only as gate u: both factors in one; likewise w (1 + scale)
        pair_t w[4], wp[4];
        load_mod(p.wp, c, 1.0f, wp);
        load_mod(p.gate, b * p.ld_gate + c, 1.0f, gate);
        load_mod(p.scale, b * p.ld_scale + c, 0.0f, mul);
        if (!kBwd) load_mod(p.shift, b * p.ld_shift + c, 0.0f, shift);
        load_mod(p.w, c, 1.0f, w);
        if (kJvp) {
            load_mod(p.tgate, b * p.ld_tgate + c, 0.0f, tgate);
            load_mod(p.tscale, b * p.ld_tscale + c, 0.0f, tmul);
            load_mod(p.tshift, b * p.ld_tshift + c, 0.0f, tshift);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            gate[i] = mul2(gate[i], wp[i]);
            mul[i] = fma2(mul[i], w[i], w[i]);
            if (kJvp) {
                tgate[i] = mul2(tgate[i], wp[i]);
                tmul[i] = mul2(tmul[i], w[i]);
            }
        }
    }

    pair_t sum_dy[4], sum_dyn[4], sum_dhn[4];
    zero4(sum_dy); zero4(sum_dyn); zero4(sum_dhn);
    int turn = 0;
    uint32_t slot = smem;
    long long at = first + c;
    __syncthreads();                                             // (the zeros in `red`)
    if constexpr (kPipe) {
        static_assert(kRows == 1 && (kJvp || kBwd), "one row at a time, two sums and a companion's two");
        // The norm of x' alone (no post norm), of row r + 1 while row r is finished: the sums of r + 1 over this warp and those of
        // r over the warps go through the same five levels of shuffles, and the barrier between them is that of the row.
        float* pivots = reinterpret_cast<float*>(red + 64);
        const float inv_first = 1.0f / static_cast<float>(min(256, p.C));
        const float n_theirs = lane < n_warps ? static_cast<float>(min(256, p.C - lane * 256)) : 0.0f;
        const float inv_theirs = lane < n_warps ? 1.0f / n_theirs : 0.0f;
        // x' and its companion (tx', or dy w (1 + scale)) of a row from the ring
        auto row_of = [&](uint32_t s, pair_t (&x)[4], pair_t (&x2)[4]) {
            load_slot<TX>(s + at_x, lane, x);
            pair_t h[4];
            if (kJvp) load_slot<TX>(s + at_x2, lane, x2);
            if (has_h) {
                load_slot<__nv_bfloat16>(s + at_h, lane, h);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = fma2(gate[i], h[i], x[i]);
                    if (kJvp) x2[i] = fma2(tgate[i], h[i], x2[i]);
                }
                if (kJvp) {
                    load_slot<__nv_bfloat16>(s + at_h2, lane, h);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x2[i] = fma2(gate[i], h[i], x2[i]);
                }
            }
            if (kBwd) {
                if (has_dy) load_slot<__nv_bfloat16>(s + at_h2, lane, x2); else zero4(x2);
            }
        };
        uint32_t before = ring_end - row_bytes;                  // the slot of row r; `slot`: that of row r + 1
        for (int row = row0 - 1; row < row1; ++row) {
            float v[8], mean = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
            if (row + 1 < row1) {
                __syncwarp();                                    // (the slot that is filled now was read by the whole warp)
                fetch();
                cp_async_wait<kStages - 2>();
                __syncwarp();
                pair_t x[4], t2[4], d[4];
                row_of(slot, x, t2);
                if (kBwd) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) t2[i] = mul2(t2[i], mul[i]);
                }
                mean = __shfl_sync(0xffffffffu, sum2(add2(add2(x[0], x[1]), add2(x[2], x[3]))), 0) * 0.125f;
                const pair_t minus = twice(active ? -mean : 0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = add2(x[i], minus);
                v[0] = sum2(add2(add2(d[0], d[1]), add2(d[2], d[3])));
                v[1] = sum2(add2(fma2(d[1], d[1], mul2(d[0], d[0])), fma2(d[3], d[3], mul2(d[2], d[2]))));
                v[2] = sum2(add2(add2(t2[0], t2[1]), add2(t2[2], t2[3])));
                v[3] = sum2(add2(fma2(d[1], t2[1], mul2(d[0], t2[0])), fma2(d[3], t2[3], mul2(d[2], t2[2]))));
            }
            float mean0 = 0.0f;
            if (row >= row0) {
                // lane w: warp w's sums of row r, about that warp's mean and then about the first warp's
                const float4* buf = red + (turn ^ 1) * 32;
                const float* piv = pivots + (turn ^ 1) * 32;
                const float4 e = buf[lane];
                const float d = e.x * inv_theirs;
                mean0 = fmaf(buf[0].x, inv_first, piv[0]);
                const float d2 = piv[lane] + d - mean0;
                v[4] = n_theirs * d2;
                v[5] = fmaf(v[4], d2, fmaf(-d, e.x, e.y));
                v[6] = e.z;
                v[7] = fmaf(d2, e.z, fmaf(-d, e.z, e.w));
            }
            join_lanes(v);
            if ((lane & 3) == 0 && lane < 16) reinterpret_cast<float*>(red + turn * 32 + warp)[lane >> 2] = v[0];
            if (lane == 0) pivots[turn * 32 + warp] = mean;
            turn ^= 1;
            if (row >= row0) {
                const float s = __shfl_sync(0xffffffffu, v[0], 16), sq = __shfl_sync(0xffffffffu, v[0], 20);
                const float T = __shfl_sync(0xffffffffu, v[0], 24), Q = __shfl_sync(0xffffffffu, v[0], 28);
                const bool layer = p.norm == kAdalnLayer;
                const float d = s * shape.inv_c, mu = mean0 + d, m2 = fmaxf(fmaf(-d, s, sq), 0.0f), q = fmaf(-d, T, Q);
                const float r = rsqrtf((layer ? m2 * shape.inv_c : fmaf(mu, mu, m2 * shape.inv_c)) + p.eps);
                const pair_t rr = twice(r), minus_q = twice(-r * shape.inv_c * (layer ? q : fmaf(mu, T, q)));
                const pair_t minus_mean = twice(layer && active ? -mu : 0.0f), minus_tbar = twice(layer && active ? -T * shape.inv_c : 0.0f);
                pair_t x[4], x2[4];
                row_of(before, x, x2);
                if (kJvp) {
                    if (has_h && active) {
                        store8(static_cast<TX*>(p.xn) + at, x, p.wide);
                        store8(static_cast<TX*>(p.txn) + at, x2, p.wide);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const pair_t n = mul2(add2(x[i], minus_mean), rr);
                        const pair_t tn = mul2(rr, fma2(n, minus_q, add2(x2[i], minus_tbar)));
                        x[i] = fma2(n, mul[i], shift[i]);
                        x2[i] = fma2(tn, mul[i], fma2(n, tmul[i], tshift[i]));
                    }
                    if (active) {
                        store8(p.y + at, x);
                        store8(p.ty + at, x2);
                    }
                } else {
                    pair_t g[4], h[4];
                    if (has_dxn) load_slot<TX>(before + at_x2, lane, g); else zero4(g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const pair_t n = mul2(add2(x[i], minus_mean), rr);
                        sum_dy[i] = add2(sum_dy[i], x2[i]);
                        sum_dyn[i] = fma2(x2[i], n, sum_dyn[i]);
                        g[i] = fma2(rr, fma2(n, minus_q, fma2(x2[i], mul[i], minus_tbar)), g[i]);
                    }
                    if (active) store8(static_cast<TX*>(p.dx) + at, g, p.wide);
                    if (has_h) {
                        load_slot<__nv_bfloat16>(before + at_h, lane, h);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            sum_dhn[i] = fma2(g[i], h[i], sum_dhn[i]);
                            g[i] = mul2(g[i], gate[i]);
                        }
                        if (active) store8(p.dh + at, g);
                    }
                }
                at += p.C;
            }
            __syncthreads();
            before = slot;
            slot += row_bytes;
            if (slot == ring_end) slot = smem;
        }
    } else
    for (int row = row0; row < row1; row += kRows, at += static_cast<long long>(kRows) * p.C) {
        __syncwarp();                                            // (the slot that is filled now was read by the whole warp)
        fetch();
        cp_async_wait<kStages - 1>();
        __syncwarp();                                            // (the lanes read what other lanes have copied)
        // the branch's output, normalised if there is a post norm (hn)
        pair_t x[kRows][4], x2[kRows][4];                        // x', and tx' / the gradient of x'
        pair_t h[kRows][4], h2[kRows][4];                        // h, and th / dy
        RowNorm hs[kRows] = {}, xs[kRows] = {};
        // hn of row r again, from the ring
        auto reload_hn = [&](int r) {
            load_slot<__nv_bfloat16>(slot + r * row_bytes + at_h, lane, h[r]);
            if (p.post != kAdalnNone) {
                const pair_t minus_mean = twice(active ? -hs[r].mean : 0.0f), rr = twice(hs[r].r);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[r][i] = mul2(add2(h[r][i], minus_mean), rr);
            }
        };
        if (has_h && p.post != kAdalnNone) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                load_slot<__nv_bfloat16>(slot + r * row_bytes + at_h, lane, h[r]);
                if (kJvp) load_slot<__nv_bfloat16>(slot + r * row_bytes + at_h2, lane, h2[r]);
            }
            row_norms<kRows, kJvp>(h, h2, shape, p.post, p.eps, red, turn, hs);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const uint32_t s = slot + r * row_bytes;
            load_slot<TX>(s + at_x, lane, x[r]);
            if (kJvp) load_slot<TX>(s + at_x2, lane, x2[r]);
            if (has_h) {
                reload_hn(r);
                if (kJvp) {
                    load_slot<__nv_bfloat16>(s + at_h2, lane, h2[r]);
                    if (p.post != kAdalnNone) {
                        // (channels behind C stay zero: sums run over them)
                        const pair_t rr = twice(hs[r].r), minus_q = twice(-hs[r].q), minus_tbar = twice(active ? -hs[r].tbar : 0.0f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) h2[r][i] = mul2(rr, fma2(h[r][i], minus_q, add2(h2[r][i], minus_tbar)));
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[r][i] = fma2(gate[i], h[r][i], x[r][i]);
                    if (kJvp) x2[r][i] = fma2(gate[i], h2[r][i], fma2(tgate[i], h[r][i], x2[r][i]));
                }
                if (!kBwd && active && row + r < row1) {
                    store8(static_cast<TX*>(p.xn) + at + r * p.C, x[r], p.wide);
                    if (kJvp) store8(static_cast<TX*>(p.txn) + at + r * p.C, x2[r], p.wide);
                }
            }
        }
        if (!kBwd) {
            if (has_norm) {
                row_norms<kRows, kJvp>(x, x2, shape, p.norm, p.eps, red, turn, xs);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const pair_t rr = twice(xs[r].r), minus_q = twice(-xs[r].q);
                    const pair_t minus_mean = twice(-xs[r].mean), minus_tbar = twice(-xs[r].tbar);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const pair_t n = mul2(add2(x[r][i], minus_mean), rr);
                        x[r][i] = fma2(n, mul[i], shift[i]);
                        if (kJvp) {
                            const pair_t tn = mul2(rr, fma2(n, minus_q, add2(x2[r][i], minus_tbar)));
                            x2[r][i] = fma2(tn, mul[i], fma2(n, tmul[i], tshift[i]));
                        }
                    }
                    if (active && row + r < row1) {
                        store8(p.y + at + r * p.C, x[r]);
                        if (kJvp) store8(p.ty + at + r * p.C, x2[r]);
                    }
                }
            }
        } else {
            if (has_norm) {
                pair_t dn[kRows][4];
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (has_dy) load_slot<__nv_bfloat16>(slot + r * row_bytes + at_h2, lane, dn[r]); else zero4(dn[r]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dn[r][i] = mul2(dn[r][i], mul[i]);
                }
                row_norms<kRows, true>(x, dn, shape, p.norm, p.eps, red, turn, xs);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (row + r < row1) {                            // (uniform)
                    const uint32_t s = slot + r * row_bytes;
                    if (has_dxn) load_slot<TX>(s + at_x2, lane, x2[r]); else zero4(x2[r]);
                    if (has_norm) {
                        if (has_dy) load_slot<__nv_bfloat16>(s + at_h2, lane, h2[r]); else zero4(h2[r]);
                        const pair_t rr = twice(xs[r].r), minus_q = twice(-xs[r].q);
                        const pair_t minus_mean = twice(active ? -xs[r].mean : 0.0f), minus_tbar = twice(active ? -xs[r].tbar : 0.0f);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const pair_t n = mul2(add2(x[r][i], minus_mean), rr);
                            sum_dy[i] = add2(sum_dy[i], h2[r][i]);
                            sum_dyn[i] = fma2(h2[r][i], n, sum_dyn[i]);
                            x2[r][i] = fma2(rr, fma2(n, minus_q, fma2(h2[r][i], mul[i], minus_tbar)), x2[r][i]);
                        }
                    }
                    // x2 is the whole gradient of x' now, which is that of x
                    if (active) store8(static_cast<TX*>(p.dx) + at + r * p.C, x2[r], p.wide);
                    if (has_h) {
                        reload_hn(r);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            sum_dhn[i] = fma2(x2[r][i], h[r][i], sum_dhn[i]);
                            x2[r][i] = mul2(x2[r][i], gate[i]);
                        }
                        if (p.post == kAdalnNone && active) store8(p.dh + at + r * p.C, x2[r]);
                    }
                } else {
                    zero4(x2[r]);
                    zero4(h[r]);
                }
            }
            if (has_h && p.post != kAdalnNone) {
                RowNorm es[kRows];                               // of hn and e = dx gate wp: tbar = mean e, q = mean(e hn)
                row_norms<kRows, true>(h, x2, shape, kAdalnMeans, 0.0f, red, turn, es);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const pair_t rr = twice(hs[r].r), minus_tbar = twice(p.post == kAdalnLayer ? -es[r].tbar : 0.0f), minus_q = twice(-es[r].q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x2[r][i] = mul2(rr, fma2(h[r][i], minus_q, add2(x2[r][i], minus_tbar)));
                    if (active && row + r < row1) store8(p.dh + at + r * p.C, x2[r]);
                }
            }
        }
        slot += kRows * row_bytes;
        if (slot == ring_end) slot = smem;
    }
    if (kBwd && active) {
        float* out = p.part + static_cast<long long>(blockIdx.x) * 3 * p.C + c;
        store8(out, sum_dy);
        store8(out + p.C, sum_dyn);
        store8(out + 2 * p.C, sum_dhn);
    }
}

// Joins the CTAs' column sums, always in the same order (no atomics: a gradient is the same from run to run):
//     dshift = S0,  dscale = w S1,  dgate = wp S2,  dw = sum_b (1 + scale) S1,  dwp = sum_b gate S2.
// A block owns 32 channels and takes up to kAdalnJoinBatches batches at a time, each with its share of the 32 warps: its time is
// the latency of the loads that one warp makes one after the other (2 batches of 129 CTAs, 1536 channels: 6.1 us, one batch
// after the other 10.4; one batch of 147 CTAs, 5120 channels: 7.4 us, with eight loads ahead and thus one CTA per SM 9.1).
constexpr int kAdalnJoinRows = 32, kAdalnJoinBatches = 4, kAdalnJoinAhead = 4;
struct AdalnJoin {
    const float* part;
    const float *gate, *scale, *w, *wp;
    long long ld_gate, ld_scale;
    float *dgate, *dscale, *dshift, *dw, *dwp;
    int B, C, n_parts;
};
__global__ void __launch_bounds__(32 * kAdalnJoinRows, 2) adaln_join_kernel(const AdalnJoin p) {
    __shared__ float part[3][kAdalnJoinRows][32], fold[2][kAdalnJoinBatches][32];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const bool active = c < p.C;
    const int batches = p.B >= 3 ? 4 : p.B, share = kAdalnJoinRows / batches;      // (1, 2 or 4 at a time)
    const int own = g / share, first = g - own * share;          // this warp's batch of the group, its first CTA
    // (warp 3 b + k < 3 batches joins the warps' sums k of batch b; warps 0 and 1 add up dw and dwp)
    const int jb = g / 3, k = g - 3 * jb;
    float total = 0.0f;
    for (int b0 = 0; b0 < p.B; b0 += batches) {
        float s[3] = {0.0f, 0.0f, 0.0f};
        if (active && b0 + own < p.B) {
            const float* in = p.part + static_cast<long long>(b0 + own) * p.n_parts * 3 * p.C + c;
            for (int i0 = first; i0 < p.n_parts; i0 += kAdalnJoinAhead * share) {
                float v[kAdalnJoinAhead][3];
#pragma unroll
                for (int u = 0; u < kAdalnJoinAhead; ++u) {
                    const int i = i0 + u * share;
#pragma unroll
                    for (int q = 0; q < 3; ++q) v[u][q] = i < p.n_parts ? __ldg(in + (static_cast<long long>(i) * 3 + q) * p.C) : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < kAdalnJoinAhead; ++u)
#pragma unroll
                    for (int q = 0; q < 3; ++q) s[q] += v[u][q];
            }
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) part[q][g][lane] = s[q];
        __syncthreads();
        const int b = b0 + jb;
        if (jb < batches && active) {
            float sum = 0.0f, f = 0.0f;
            if (b < p.B) {
                for (int j = 0; j < share; ++j) sum += part[k][jb * share + j][lane];
                const long long at = static_cast<long long>(b) * p.C + c;
                if (k == 0 && p.dshift) p.dshift[at] = sum;
                if (k == 1 && p.dscale) p.dscale[at] = (p.w ? p.w[c] : 1.0f) * sum;
                if (k == 2 && p.dgate) p.dgate[at] = (p.wp ? p.wp[c] : 1.0f) * sum;
                if (k == 1) f = 1.0f + (p.scale ? p.scale[b * p.ld_scale + c] : 0.0f);
                if (k == 2) f = p.gate ? p.gate[b * p.ld_gate + c] : 1.0f;
            }
            if (k > 0) fold[k - 1][jb][lane] = f * sum;
        }
        __syncthreads();
        if (g < 2) {
            for (int j = 0; j < batches; ++j) total += fold[g][j][lane];
        }
        // (`fold` is written again only behind the next group's first barrier)
    }
    if (g == 0 && active && p.dw) p.dw[c] = total;
    if (g == 1 && active && p.dwp) p.dwp[c] = total;
}

}  // namespace attn_jvp
