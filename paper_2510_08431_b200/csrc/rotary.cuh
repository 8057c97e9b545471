// Rotary positions: the table of angles, and the step between the projections and the attention core that normalises the heads
// of queries and keys and rotates them, with tangents and gradients.
//
// Table, for pair i of axis a (base theta, d_a channels per axis):  angle = position_a . theta_a^(-2 i / d_a), stretched as the
// host asks; an entry is (m cos, m sin).  The angle of a far position has lost its fraction in 32 bits, so it is counted in turns of which whole ones
// drop out: a whole position times the turns per position in 2^-64 of a turn, modulo 2^64 (an integer product), a fractional position in fp64.
// What is left goes on as 2^-32 of a turn: the nearest quarter turn picks and signs the results, the rest is at most pi / 4, where
// sin y = y + y^3 S(y^2) and cos y = 1 - y^2 / 2 + y^4 C(y^2) with polynomials of smallest error (4e-9 of sin, 1e-10 of cos) are right to fp32 rounding.
// Bound by the 8 bytes written per pair: 262144 positions of 64 pairs XX us.
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
        if constexpr (std::is_floating_point_v<T>) {
            const double t = static_cast<double>(__ldg(pos)) * turns;
            u = static_cast<unsigned>(__double2int_rn((t - rint(t)) * 4294967296.0));        // (half a turn saturates: 2^-32 of one off)
        } else {
            u = static_cast<unsigned>((static_cast<unsigned long long>(static_cast<long long>(__ldg(pos))) * step + 0x80000000ull) >> 32);
        }
        const float2 cs = cos_sin_turns(u);
        *out = make_float2(p.size * cs.x, p.size * cs.y);
    }
}

// ---------------------------------------------------------------------------------------------
// Heads of queries and keys
// ---------------------------------------------------------------------------------------------
constexpr int kRotaryThreads = 256;
enum RotaryMode : int { kRotaryFwd = 0, kRotaryJvp = 1, kRotaryBwd = 2 };
// rows that a group of lanes has in flight, and blocks that share an SM (what the registers are budgeted for)
__host__ __device__ constexpr int rotary_rows(int mode) { return mode == kRotaryFwd ? 4 : 2; }
__host__ __device__ constexpr int rotary_ctas(int mode) { return mode == kRotaryBwd ? 3 : 4; }

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

__device__ __forceinline__ void unpack8(const uint32_t (&v)[4], float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(v[i] << 16);                  // bf16 -> fp32 is a shift
        f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
}
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
    const bool second = blockIdx.x >= p.q.blocks;
    const RotaryTensor& T = second ? p.k : p.q;
    const unsigned block = second ? blockIdx.x - p.q.blocks : blockIdx.x;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const bool turned = lane < p.R / 8;
    // the lane's channels: o1 .. o1 + 3 and o2 .. o2 + 3; pairs (o1 + i, o2 + i), or (2 i, 2 i + 1) of the eight
    int o1 = 8 * lane, o2 = o1 + 4;
    if (kHalf && turned) {
        o1 = 4 * lane;
        o2 = p.R / 2 + 4 * lane;
    }
    auto channel = [&](int i) { return i < 4 ? o1 + i : o2 + i - 4; };
    auto load8 = [&](const __nv_bfloat16* at, uint32_t (&v)[4]) {
        if (kHalf) {
            const uint2 a = __ldg(reinterpret_cast<const uint2*>(at + o1)), c = __ldg(reinterpret_cast<const uint2*>(at + o2));
            v[0] = a.x; v[1] = a.y; v[2] = c.x; v[3] = c.y;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(at + o1));
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        }
    };
    auto store8 = [&](__nv_bfloat16* at, const float (&f)[8]) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            v[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        if (kHalf) {
            *reinterpret_cast<uint2*>(at + o1) = make_uint2(v[0], v[1]);
            *reinterpret_cast<uint2*>(at + o2) = make_uint2(v[2], v[3]);
        } else {
            *reinterpret_cast<uint4*>(at + o1) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    };
    // a rotation (back = false) or its transpose of the lane's four pairs
    auto turn = [&](float (&f)[8], const float (&cs)[8], bool back) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int a = kHalf ? i : 2 * i, c = kHalf ? i + 4 : 2 * i + 1;
            const float co = cs[2 * i], si = back ? -cs[2 * i + 1] : cs[2 * i + 1];
            const float x = f[a], y = f[c];
            f[a] = x * co - y * si;
            f[c] = y * co + x * si;
        }
    };
    float w[8], bias[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[i] = T.w ? __ldg(T.w + channel(i)) : 1.0f;
        bias[i] = (MODE != kRotaryBwd && T.b) ? __ldg(T.b + channel(i)) : 0.0f;
    }
    float dw[8] = {}, db[8] = {};

    const unsigned units = static_cast<unsigned>(p.tokens) * T.chunks, stride = T.blocks * kGroups;
    // The bounds of both loops are the same for the whole block (the shuffles need whole warps); what lies behind the last unit or
    // head is worked on again, and neither stored nor summed.
    for (unsigned base = block * kGroups; base < units; base += stride) {
        const bool exists = base + group < units;
        const unsigned unit = exists ? base + group : units - 1;
        const unsigned token = unit / T.chunks, chunk = unit - token * T.chunks;
        const unsigned b = token / p.L, l = token - b * p.L;
        float cs[8];
        if (turned) {
            long long row = l;
            if (p.index) row = __ldg(p.index + b * p.index_batch + l);
            row = row < 0 ? 0 : row >= p.table_rows ? p.table_rows - 1 : row;          // (an index from anywhere reads inside the table)
            const float4* at = reinterpret_cast<const float4*>(p.table + (b * p.table_batch + row) * (p.R / 2) + 4 * lane);
            const float4 c0 = __ldg(at), c1 = __ldg(at + 1);
            cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w;
            cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = i & 1 ? 0.0f : 1.0f;
        }
        const __nv_bfloat16* x = T.x + b * T.x_b + l * T.x_l;
        const __nv_bfloat16* t = MODE == kRotaryFwd ? nullptr : T.t + b * T.t_b + l * T.t_l;
        const long long out = static_cast<long long>(token) * T.H * D;
        for (int h0 = 0; h0 < T.heads; h0 += kRows) {
            const int first = static_cast<int>(chunk) * T.heads + h0;
            uint32_t xr[kRows][4], tr[kRows][4];
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int h = min(first + r, T.H - 1);
                load8(x + h * T.x_h, xr[r]);
                if (MODE != kRotaryFwd) load8(t + h * T.t_h, tr[r]);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int h = first + r;
                const bool real = exists && h0 + r < T.heads && h < T.H;
                float v[8], g[8];
                unpack8(xr[r], v);
                if (MODE != kRotaryFwd) unpack8(tr[r], g);
                float du[8];
                if (MODE == kRotaryBwd) {
                    turn(g, cs, true);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        du[i] = g[i];
                        g[i] *= w[i];
                    }
                }
                if (p.norm != 0) {
                    constexpr float kInv = 1.0f / D;
                    float mean = 0.0f, gmean = 0.0f;
                    if (p.norm == 1) {                           // layer: centred first
                        float s = 0.0f, sg = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            s += v[i];
                            if (MODE != kRotaryFwd) sg += g[i];
                        }
                        mean = sum_lanes<kLanes>(s) * kInv;
                        if (MODE != kRotaryFwd) gmean = sum_lanes<kLanes>(sg) * kInv;
                    }
                    float ss = 0.0f, sg = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] -= mean;
                        ss = fmaf(v[i], v[i], ss);
                        if (MODE != kRotaryFwd) {
                            g[i] -= gmean;
                            sg = fmaf(v[i], g[i], sg);
                        }
                    }
                    const float rn = rsqrtf(fmaf(sum_lanes<kLanes>(ss), kInv, p.eps));
                    const float m = MODE == kRotaryFwd ? 0.0f : sum_lanes<kLanes>(sg) * kInv * rn;       // mean(n . g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] *= rn;
                        if (MODE != kRotaryFwd) g[i] = rn * fmaf(-v[i], m, g[i]);
                    }
                }
                const long long at = out + static_cast<long long>(h) * D;
                if (MODE == kRotaryBwd) {
                    if (real) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            dw[i] = fmaf(du[i], v[i], dw[i]);
                            db[i] += du[i];
                        }
                        store8(T.y + at, g);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] = fmaf(w[i], v[i], bias[i]);
                        if (MODE == kRotaryJvp) g[i] *= w[i];
                    }
                    turn(v, cs, false);
                    if (MODE == kRotaryJvp) turn(g, cs, false);
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
        for (int i = 0; i < 8; ++i) {
            sums[group][0][channel(i)] = dw[i];
            sums[group][1][channel(i)] = db[i];
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
