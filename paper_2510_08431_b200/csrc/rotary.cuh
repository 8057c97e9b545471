// Rotary positions: the table of angles, and the step between the projections and the attention core that normalises the heads
// of queries and keys and rotates them, with tangents and gradients.
//
// Table, for pair i of axis a (base theta, d_a channels per axis):  angle = position_a . theta_a^(-2 i / d_a), stretched as the
// host asks; an entry is (m cos, m sin).  The angle of a far position has lost its fraction in 32 bits, so it is counted in turns of which whole ones
// drop out: a whole position times the turns per position in 2^-64 of a turn, modulo 2^64 (an integer product), a fractional position in fp64.
// What is left goes on as 2^-32 of a turn: the nearest quarter turn picks and signs the results, the rest is at most pi / 4, where
// sin y = y + y^3 S(y^2) and cos y = 1 - y^2 / 2 + y^4 C(y^2) with polynomials of smallest error (as stored in fp32 4.3e-9 of sin, 5e-10 of cos) are right to fp32 rounding.
// 262144 positions of 64 pairs (134 MB) 35 us; with the fraction in fp64 and sincospif 86.  Bound by the instructions of an entry, mostly integer ones (46 per 32 entries, issue slots 69 % busy, DRAM
// 26 %); short tables by a thread's first reads of its pair's constants, which the constant cache serves one address at a time (32760 positions of three axes 10.6 to 11.8 us).
//
// Heads, for a row x in R^D of one token and head, with the token's table row R (a rotation of the first R channels by pairs):
//     n = (x - mean x) / sqrt(var x + eps)   or   x / sqrt(mean x^2 + eps)   or   x,      u = w . n + b,      y = R u
//     ty = R (w . N tx),     dx = N (w . R^T dy),  dw = sum (R^T dy) . n,  db = sum R^T dy
// where N t = r (t - [mean t] - n mean(n . t)) is the normalisation's derivative, which is symmetric: tangents and gradients share
// it.  Bound by HBM: one read and one write of a row per tensor.  D / 8 lanes own a row, each with both channels of its four
// pairs (layout "half", pairs (i, i + R / 2): four channels from either half, two 8-byte accesses that fill whole lines together;
// "interleaved", pairs (2 i, 2 i + 1): one 16-byte access), so that the rotation needs no exchange; the row's sums are
// shuffles.  A group of lanes takes a token and several of its heads, several rows at a time: the token's table row is read once for them and the rows' loads
// are in flight together.  Queries and keys go into one launch, each on blocks of its own.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_jvp_kernel.cuh"

namespace attn_jvp {

// ---------------------------------------------------------------------------------------------
// The table
// ---------------------------------------------------------------------------------------------
constexpr int kRotaryMaxPairs = 128, kRotaryMaxAxes = 8;
constexpr int kTableThreads = 256;
struct RotaryTableParams {
    unsigned long long steps[kRotaryMaxPairs];   // 2^-64 turns per unit of position (whole turns dropped) ...
    double turns[kRotaryMaxPairs];               // ... and turns, for fractional positions
    unsigned char axis[kRotaryMaxPairs];
    const void* positions;                // [n][axes]
    float2* table;                        // [n][pairs]
    long long n;
    int axes, pairs;
    float size;                           // m
};

// (cos, sin) of u 2^-32 turns
__device__ __forceinline__ float2 cos_sin_turns(unsigned u) {
    const unsigned quarter = (u + 0x20000000u) >> 30;
    const float y = static_cast<float>(static_cast<int>(u - (quarter << 30))) * 0x1.921fb6p-30f;      // 2 pi 2^-32
    const float z = y * y;
    const float s = fmaf(y * z, fmaf(fmaf(-0x1.994eb4p-13f, z, 0x1.11076p-7f), z, -0x1.555546p-3f), y);
    const float c = fmaf(z, fmaf(fmaf(fmaf(0x1.9a025ap-16f, z, -0x1.6c0c8cp-10f), z, 0x1.55554ap-5f), z, -0.5f), 1.0f);
    const float a = quarter & 1u ? s : c, b = quarter & 1u ? c : s;       // (cos, sin), (-sin, cos), (-cos, -sin), (sin, -cos)
    return make_float2((quarter + 1u) & 2u ? -a : a, quarter & 2u ? -b : b);
}

template <typename T>
__global__ void __launch_bounds__(kTableThreads)
rotary_table_kernel(const __grid_constant__ RotaryTableParams p) {
    // a thread keeps its pair; the threads of a block cover whole rows of the table
    const int rows = blockDim.x / p.pairs;
    const int pair = threadIdx.x % p.pairs, sub = threadIdx.x / p.pairs;
    const unsigned long long step = p.steps[pair];
    const double turns = p.turns[pair];
    const long long stride = static_cast<long long>(gridDim.x) * rows;
    long long i = static_cast<long long>(blockIdx.x) * rows + sub;
    const T* pos = static_cast<const T*>(p.positions) + p.axis[pair] + i * p.axes;
    float2* out = p.table + i * p.pairs + pair;
#pragma unroll 4
    for (; i < p.n; i += stride, pos += stride * p.axes, out += stride * p.pairs) {
        unsigned u;
        float size = p.size;
        if constexpr (std::is_floating_point_v<T>) {
            const double t = static_cast<double>(__ldg(pos)) * turns, f = t - rint(t);
            u = static_cast<unsigned>(__double2int_rn(f * 4294967296.0));        // (half a turn saturates: 2^-32 of one off)
            if (f != f) size = NAN;                              // (a position that is none: infinite or NaN)
        } else {
            u = static_cast<unsigned>((static_cast<unsigned long long>(static_cast<long long>(__ldg(pos))) * step + 0x80000000ull) >> 32);
        }
        const float2 cs = cos_sin_turns(u);
        *out = make_float2(size * cs.x, size * cs.y);
    }
}

// ---------------------------------------------------------------------------------------------
// Heads of queries and keys
// ---------------------------------------------------------------------------------------------
constexpr int kRotaryThreads = 256;
enum RotaryMode : int { kRotaryFwd = 0, kRotaryJvp = 1, kRotaryBwd = 2 };
// Rows that a group of lanes works on at a time, blocks that share an SM (what the registers are budgeted for), and whether the next rows are loaded beside these.
// 40 + 40 heads of 32760 tokens: forward 230 us with four rows, 221 with two and the next two ahead; tangents 471 us with two rows at four blocks, 422 with four
// at two, 480 with two and two ahead; gradients 398, 348, 361.
__host__ __device__ constexpr int rotary_rows(int mode) { return mode == kRotaryFwd ? 2 : 4; }
__host__ __device__ constexpr int rotary_ctas(int mode) { return mode == kRotaryFwd ? 4 : 2; }
__host__ __device__ constexpr bool rotary_ahead(int mode) { return mode == kRotaryFwd; }

struct RotaryTensor {
    const __nv_bfloat16* x;
    const __nv_bfloat16* t;               // tangent of x, or gradient of y
    __nv_bfloat16* y;                     // y; backward: dx            [B][L][H][D]
    __nv_bfloat16* ty;                    // tangent of y
    const float* w;
    const float* b;
    long long x_b, x_l, x_h, t_b, t_l, t_h;      // strides in elements
    int H;
    int chunks, heads;                    // a token's heads are cut into `chunks` of `heads`
    unsigned blocks;                      // of this tensor
};
struct RotaryParams {
    RotaryTensor q, k;                    // k.blocks = 0: queries alone
    const float2* table;                  // [rows][R / 2]
    const int* index;                     // table row of a token, or null: its place
    long long table_batch, index_batch;   // rows per batch; 0: the same for all
    long long table_rows;
    long long tokens;
    int L, R, norm;
    float eps;
    float* part;                          // backward: [blocks][2][D], sums of dw and db; null: not wanted
};

template <int kLanes>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
    for (int m = kLanes / 2; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}

template <int D, int MODE, bool kHalf>
__global__ void __launch_bounds__(kRotaryThreads, rotary_ctas(MODE))
qk_rotary_kernel(const __grid_constant__ RotaryParams p) {
    constexpr int kLanes = D / 8, kGroups = kRotaryThreads / kLanes, kRows = rotary_rows(MODE);
    constexpr bool kAhead = rotary_ahead(MODE);
    const bool second = blockIdx.x >= p.q.blocks;
    const RotaryTensor& T = second ? p.k : p.q;
    const unsigned block = second ? blockIdx.x - p.q.blocks : blockIdx.x;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const bool turned = lane < p.R / 8;
    // The lane's channels: o1 .. o1 + 3 and o2 .. o2 + 3.  In registers the four pairs' first channels come first, then the four second ones (half: as they lie;
    // interleaved: from words that hold a pair each), two to a 64-bit register: the packed instructions below then do the same for either layout.
    int o1 = 8 * lane, o2 = o1 + 4;
    if (kHalf && turned) {
        o1 = 4 * lane;
        o2 = p.R / 2 + 4 * lane;
    }
    auto channel = [&](int i) {                                  // of place i in registers
        if (kHalf) return i < 4 ? o1 + i : o2 + i - 4;
        return o1 + 2 * (i % 4) + i / 4;
    };
    using Row = uint64_t[4];
    auto load8 = [&](const __nv_bfloat16* at, uint32_t (&v)[4]) {
        if (kHalf) {
            const uint2 a = __ldg(reinterpret_cast<const uint2*>(at + o1)), c = __ldg(reinterpret_cast<const uint2*>(at + o2));
            v[0] = a.x; v[1] = a.y; v[2] = c.x; v[3] = c.y;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(at + o1));
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        }
    };
    auto unpack8 = [&](const uint32_t (&v)[4], Row& f) {         // (bf16 -> fp32 is a shift)
        auto lo = [&](int i) { return __uint_as_float(v[i] << 16); };
        auto hi = [&](int i) { return __uint_as_float(v[i] & 0xFFFF0000u); };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kHalf) f[i] = pack_f32x2(lo(i), hi(i));
            else f[i] = i < 2 ? pack_f32x2(lo(2 * i), lo(2 * i + 1)) : pack_f32x2(hi(2 * i - 4), hi(2 * i - 3));
        }
    };
    auto store8 = [&](__nv_bfloat16* at, const Row& f) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack_f32x2(f[i], x[2 * i], x[2 * i + 1]);
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = kHalf ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_bf16(x[i], x[i + 4]);
        if (kHalf) {
            *reinterpret_cast<uint2*>(at + o1) = make_uint2(v[0], v[1]);
            *reinterpret_cast<uint2*>(at + o2) = make_uint2(v[2], v[3]);
        } else {
            *reinterpret_cast<uint4*>(at + o1) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    };
    // the four pairs rotated, with sines (forward) or their negatives (back) and the other sign in `neg`
    auto turn = [&](Row& f, const uint64_t (&co)[2], const uint64_t (&si)[2], const uint64_t (&neg)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t x = f[i], y = f[i + 2];
            f[i] = fma_f32x2(y, neg[i], mul_f32x2(x, co[i]));
            f[i + 2] = fma_f32x2(x, si[i], mul_f32x2(y, co[i]));
        }
    };
    auto sum2 = [](uint64_t a, uint64_t b) {
        float x, y;
        unpack_f32x2(add_f32x2(a, b), x, y);
        return x + y;
    };
    auto twice = [](float v) { return pack_f32x2(v, v); };
    Row w, bias;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c0 = channel(2 * i), c1 = channel(2 * i + 1);
        w[i] = T.w ? pack_f32x2(__ldg(T.w + c0), __ldg(T.w + c1)) : twice(1.0f);
        bias[i] = (MODE != kRotaryBwd && T.b) ? pack_f32x2(__ldg(T.b + c0), __ldg(T.b + c1)) : 0ull;
    }
    Row dw = {}, db = {};

    const unsigned units = static_cast<unsigned>(p.tokens) * T.chunks, stride = T.blocks * kGroups;
    // The bounds of both loops are the same for the whole block (the shuffles need whole warps); what lies behind the last unit or
    // head is worked on again, and neither stored nor summed.
    for (unsigned base = block * kGroups; base < units; base += stride) {
        const bool exists = base + group < units;
        const unsigned unit = exists ? base + group : units - 1;
        const unsigned token = unit / T.chunks, chunk = unit - token * T.chunks;
        const unsigned b = token / p.L, l = token - b * p.L;
        uint64_t co[2] = {twice(1.0f), twice(1.0f)}, si[2] = {0ull, 0ull}, neg[2];
        if (turned) {
            long long row = l;
            if (p.index) row = __ldg(p.index + b * p.index_batch + l);
            row = row < 0 ? 0 : row >= p.table_rows ? p.table_rows - 1 : row;          // (an index from anywhere reads inside the table)
            const float4* at = reinterpret_cast<const float4*>(p.table + (b * p.table_batch + row) * (p.R / 2) + 4 * lane);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 c = __ldg(at + i);
                co[i] = pack_f32x2(c.x, c.z);
                si[i] = MODE == kRotaryBwd ? pack_f32x2(-c.y, -c.w) : pack_f32x2(c.y, c.w);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) neg[i] = mul_f32x2(si[i], twice(-1.0f));
        const __nv_bfloat16* x = T.x + b * T.x_b + l * T.x_l;
        const __nv_bfloat16* t = MODE == kRotaryFwd ? nullptr : T.t + b * T.t_b + l * T.t_l;
        const long long out = static_cast<long long>(token) * T.H * D;
        uint32_t xr[kRows][4], tr[kRows][4], x_next[kRows][4], t_next[kRows][4];
        auto load_rows = [&](int first, uint32_t (&xs)[kRows][4], uint32_t (&ts)[kRows][4]) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int h = min(first + r, T.H - 1);
                load8(x + h * T.x_h, xs[r]);
                if (MODE != kRotaryFwd) load8(t + h * T.t_h, ts[r]);
            }
        };
        if (kAhead) load_rows(static_cast<int>(chunk) * T.heads, x_next, t_next);
        for (int h0 = 0; h0 < T.heads; h0 += kRows) {
            const int first = static_cast<int>(chunk) * T.heads + h0;
            if (kAhead) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        xr[r][i] = x_next[r][i];
                        if (MODE != kRotaryFwd) tr[r][i] = t_next[r][i];
                    }
                }
                if (h0 + kRows < T.heads) load_rows(first + kRows, x_next, t_next);
            } else {
                load_rows(first, xr, tr);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int h = first + r;
                const bool real = exists && h0 + r < T.heads && h < T.H;
                Row v, g, du;
                unpack8(xr[r], v);
                if (MODE != kRotaryFwd) unpack8(tr[r], g);
                if (MODE == kRotaryBwd) {
                    turn(g, co, si, neg);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        du[i] = g[i];
                        g[i] = mul_f32x2(g[i], w[i]);
                    }
                }
                if (p.norm != 0) {
                    constexpr float kInv = 1.0f / D;
                    if (p.norm == 1) {                           // layer: centred first
                        const uint64_t mean = twice(sum_lanes<kLanes>(sum2(add_f32x2(v[0], v[1]), add_f32x2(v[2], v[3]))) * -kInv);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = add_f32x2(v[i], mean);
                        if (MODE != kRotaryFwd) {
                            const uint64_t gmean = twice(sum_lanes<kLanes>(sum2(add_f32x2(g[0], g[1]), add_f32x2(g[2], g[3]))) * -kInv);
#pragma unroll
                            for (int i = 0; i < 4; ++i) g[i] = add_f32x2(g[i], gmean);
                        }
                    }
                    const float ss = sum2(fma_f32x2(v[1], v[1], mul_f32x2(v[0], v[0])), fma_f32x2(v[3], v[3], mul_f32x2(v[2], v[2])));
                    const float rn = rsqrtf(fmaf(sum_lanes<kLanes>(ss), kInv, p.eps));
                    const uint64_t rn2 = twice(rn);
                    if (MODE != kRotaryFwd) {
                        const float sg = sum2(fma_f32x2(v[1], g[1], mul_f32x2(v[0], g[0])), fma_f32x2(v[3], g[3], mul_f32x2(v[2], g[2])));
                        const uint64_t m = twice(sum_lanes<kLanes>(sg) * -kInv * rn * rn);       // -mean(n . g) in units of v
#pragma unroll
                        for (int i = 0; i < 4; ++i) g[i] = mul_f32x2(fma_f32x2(v[i], m, g[i]), rn2);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = mul_f32x2(v[i], rn2);
                }
                const long long at = out + static_cast<long long>(h) * D;
                if (MODE == kRotaryBwd) {
                    if (real) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            dw[i] = fma_f32x2(du[i], v[i], dw[i]);
                            db[i] = add_f32x2(db[i], du[i]);
                        }
                        store8(T.y + at, g);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = fma_f32x2(w[i], v[i], bias[i]);
                        if (MODE == kRotaryJvp) g[i] = mul_f32x2(g[i], w[i]);
                    }
                    turn(v, co, si, neg);
                    if (MODE == kRotaryJvp) turn(g, co, si, neg);
                    if (real) {
                        store8(T.y + at, v);
                        if (MODE == kRotaryJvp) store8(T.ty + at, g);
                    }
                }
            }
        }
    }
    if (MODE == kRotaryBwd && p.part) {
        // the block's groups in a fixed order
        __shared__ float sums[kGroups][2][D];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unpack_f32x2(dw[i], sums[group][0][channel(2 * i)], sums[group][0][channel(2 * i + 1)]);
            unpack_f32x2(db[i], sums[group][1][channel(2 * i)], sums[group][1][channel(2 * i + 1)]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * D; c += kRotaryThreads) {
            float s = 0.0f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) s += (&sums[g][0][0])[c];
            p.part[static_cast<size_t>(blockIdx.x) * 2 * D + c] = s;
        }
    }
}

// Joins the blocks' sums of dw and db, in a fixed order: blockIdx.y = 2 tensor + (0: weight, 1: bias), 32 columns per block.
struct RotaryJoin {
    const float* part;
    float* out[4];
    unsigned blocks[2];
    int D;
};
constexpr int kRotaryJoinRows = 32;
__global__ void __launch_bounds__(32 * kRotaryJoinRows)
qk_rotary_join_kernel(const __grid_constant__ RotaryJoin j) {
    __shared__ float sums[kRotaryJoinRows][32];
    float* out = j.out[blockIdx.y];
    if (out == nullptr) return;
    const unsigned tensor = blockIdx.y >> 1, first = tensor ? j.blocks[0] : 0;
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5, column = blockIdx.x * 32 + lane;
    const float* at = j.part + static_cast<size_t>(first) * 2 * j.D + (blockIdx.y & 1) * j.D + column;
    float s = 0.0f;
#pragma unroll 4
    for (unsigned i = row; i < j.blocks[tensor]; i += kRotaryJoinRows) s += at[static_cast<size_t>(i) * 2 * j.D];
    sums[row][lane] = s;
    __syncthreads();
    if (row == 0) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < kRotaryJoinRows; ++i) t += sums[i][lane];
        out[column] = t;
    }
}

}  // namespace attn_jvp
