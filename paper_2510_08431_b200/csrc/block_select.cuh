// Which key blocks each query block attends to.  Queries and keys are cut into blocks of 128 tokens (the last one
// ragged); a selection is a truth value per (batch, head, query block, key block), and beside it the lists that the
// attention kernels walk: for every query block its key blocks in ascending order, and the transpose for the gradient
// of the keys.
//
// The score of a pair is the dot product of the blocks' mean query and mean key, and the topk largest are kept, ties
// going to the lower key block.  One wrong comparison exchanges 128 keys of 128 queries, so the order has to be that of
// the scores themselves: means and dot products are formed in 64 bits, where the sum of 128 bf16 values is exact unless
// their exponents lie more than 38 apart.  (In 32 bits neighbours around the topk-th place, about a hundredth of a
// deviation apart, would change places a few times per call of a long video.)  Infinities and NaN go through means and
// scores by the rules of IEEE arithmetic, and a score that is NaN counts as the largest: a block that holds one is kept, and the
// NaN shows in the result, instead of dropping out of it.  The arithmetic is cheap all the same:
// tokens / 128 means per head, 0.17 G multiply-adds for 12 heads of 32760 tokens, while reading q and k once bounds the
// whole selection (201 MB there, 31 us).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace attn_jvp {

constexpr int kSelBlock = 128;       // tokens of a block
constexpr int kPoolRows = 8;         // row groups of a pooling CTA: 8 x 16 tokens
constexpr int kPoolCols = 16;        // 16-byte pieces (8 channels) of a row it takes

// A bf16 value's bits (the upper half of `u`) as the upper word of a double, without a conversion to fp64 (a quarter-rate
// instruction): sign, exponent and mantissa land in place with the exponent field taken as it is, which scales every finite
// value, subnormal ones included, by exactly 2^-896.  (An infinity or NaN comes out as a finite number, see not_finite().)
__device__ __forceinline__ double scaled_bf16(int u) { return __hiloint2double((u >> 3) & 0x8FFFE000, 0); }
// Bit 15 or 31 is set if the lower or upper of two bf16 values is an infinity or NaN (other bits: anything): an exponent
// field of ones carries into the sign's place.
__device__ __forceinline__ uint32_t not_finite(uint32_t two) { return (two & 0x7FFF7FFFu) + 0x00800080u; }

// Block means of q and k in one launch.  q, k: [B][L][H * D] bf16.  qm: [B * H][n_q][D] fp64, kmt: [B * H][D][n_k] fp64 (a
// channel's values of all key blocks side by side, as the scores read them).
// A work item is 128 channels of one block, thread (piece, row group) sums 16 tokens of 8 channels.  CTAs are persistent and a
// thread keeps eight 16-byte loads in flight across its items (for every row it has added it asks for the row eight further on,
// of the next item where this one ends): with a CTA per item the CTAs of an SM load and then add, all at the same time (12
// heads of 32760 tokens, 201 MB, behind a full L2: 54 us, now 43; 40 heads: 143, now 121; 2 x 16 heads of 4096: 22, now 18).
constexpr int kPoolAhead = 8, kPoolCtas = 8;          // loads in flight per thread, CTAs per SM
__global__ void __launch_bounds__(kPoolRows* kPoolCols, kPoolCtas)
block_mean_kernel(const uint4* __restrict__ q, const uint4* __restrict__ k, double* __restrict__ qm, double* __restrict__ kmt, int Lq,
                  int Lk, int H, int D, int n_q, int n_k, int n_items) {
    constexpr int kEach = kSelBlock / kPoolRows;
    __shared__ double part[2][kPoolRows][kPoolCols * 8];
    const int piece = threadIdx.x % kPoolCols, group = threadIdx.x / kPoolCols;
    const int pieces = H * D / 8, cols = (pieces + kPoolCols - 1) / kPoolCols;
    struct Work { const uint4* row; int left, chunk, b, block, rows; bool keys; };      // left: rows of the block from this thread's first on
    auto work = [&](int item) {
        Work w{};
        if (item >= n_items) return w;                           // (no rows)
        const int rest = item / cols;
        w.chunk = item - rest * cols;
        w.b = rest / (n_q + n_k);
        w.block = rest - w.b * (n_q + n_k);
        w.keys = w.block >= n_q;
        if (w.keys) w.block -= n_q;
        const int L = w.keys ? Lk : Lq, col = w.chunk * kPoolCols + piece;
        w.rows = min(kSelBlock, L - w.block * kSelBlock);
        w.left = col < pieces ? w.rows - group : 0;
        w.row = (w.keys ? k : q) + (static_cast<long long>(w.b) * L + w.block * kSelBlock + group) * pieces + col;
        return w;
    };
    auto load = [&](const Work& w, int r) {
        return r * kPoolRows < w.left ? __ldg(w.row + static_cast<long long>(r * kPoolRows) * pieces) : make_uint4(0u, 0u, 0u, 0u);
    };
    uint4 v[kPoolAhead];
    Work w = work(blockIdx.x);
#pragma unroll
    for (int r = 0; r < kPoolAhead; ++r) v[r] = load(w, r);
    int turn = 0;
    for (int item = blockIdx.x; item < n_items; item += gridDim.x, turn ^= 1) {
        const Work next = work(n_items - item > static_cast<int>(gridDim.x) ? item + gridDim.x : n_items);
        double s[8];
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = 0.0;
#pragma unroll
        for (int r = 0; r < kEach; ++r) {
            uint4& at = v[r % kPoolAhead];
            const uint32_t u[4] = {at.x, at.y, at.z, at.w};
            at = r + kPoolAhead < kEach ? load(w, r + kPoolAhead) : load(next, r + kPoolAhead - kEach);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[2 * i] += scaled_bf16(static_cast<int>(u[i] << 16));
                s[2 * i + 1] += scaled_bf16(static_cast<int>(u[i]));
                bad |= not_finite(u[i]);
            }
        }
        if (bad & 0x80008000u) {                                 // (rare: the channel's sum is then taken again below)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = __longlong_as_double(0x7FF8000000000000ll);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) part[turn][group][i * kPoolCols + piece] = s[i];
        __syncthreads();                                         // (the other buffer was read before the last one)
        const int c = threadIdx.x;                               // one of the item's channels, of which it has as many as threads
        static_assert(kPoolRows * kPoolCols == 8 * kPoolCols, "a thread per channel");
        const int channel = w.chunk * kPoolCols * 8 + c;
        if (channel < H * D) {
            const int at = (c & 7) * kPoolCols + (c >> 3);
            double sum = 0.0;
#pragma unroll
            for (int g = 0; g < kPoolRows; ++g) sum += part[turn][g][at];
            // (every term is a multiple of 2^-1029, far above the last place of a subnormal double: nothing is lost down there)
            double mean = sum * 0x1p896 / static_cast<double>(w.rows);
            if (isnan(sum)) {                                    // an infinity or NaN near this channel: unscaled, in IEEE arithmetic
                const long long token = static_cast<long long>(w.b) * (w.keys ? Lk : Lq) + w.block * kSelBlock;
                const unsigned short* x = reinterpret_cast<const unsigned short*>(w.keys ? k : q) + token * H * D + channel;
                mean = 0.0;
#pragma unroll 1
                for (int r = 0; r < w.rows; ++r) mean += static_cast<double>(__uint_as_float(static_cast<uint32_t>(x[static_cast<long long>(r) * H * D]) << 16));
                mean /= static_cast<double>(w.rows);
            }
            const int h = channel / D, d = channel - h * D;
            const long long bh = static_cast<long long>(w.b) * H + h;
            if (w.keys) kmt[(bh * D + d) * n_k + w.block] = mean;
            else qm[(bh * n_q + w.block) * D + d] = mean;
        }
        w = next;
    }
}

// 64-bit keys whose unsigned order is the order of the doubles, with every NaN above the rest.  (NaN is told by its bits: an fp64
// comparison and its branch per score made the top-k 25 % slower, 16.7 -> 21 us for 4 heads of 148 x 148 blocks.)
__device__ __forceinline__ unsigned long long ordered_key(double v) {
    const long long b = __double_as_longlong(v + 0.0);           // (-0 becomes +0: equal scores have equal keys)
    const unsigned long long u = static_cast<unsigned long long>(b), key = b < 0 ? ~u : u | 0x8000000000000000ull;
    return (u & 0x7FFFFFFFFFFFFFFFull) > 0x7FF0000000000000ull ? ~0ull : key;
}

// Writes one row of a selection: mask bytes (optional), the ascending list and its length in 64-token tiles (a last
// block of at most 64 tokens is one tile, every other block two).  Whole warp; `keep(j, inside)` is called by all lanes for
// j = lane, lane + 32, ... in this order, also behind the row's end (inside = false, its result is not used there).
template <typename Keep>
__device__ __forceinline__ void write_row(const Keep& keep, int n, int tokens, unsigned char* mask, int* list, int* tiles) {
    const int lane = threadIdx.x & 31;
    int count = 0;
    bool last_kept = false;
    for (int j0 = 0; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        const bool inside = j < n, k = keep(j, inside) && inside;
        const unsigned votes = __ballot_sync(0xffffffffu, k);
        if (mask != nullptr && inside) mask[j] = k ? 1 : 0;
        if (k) list[count + __popc(votes & ((1u << lane) - 1u))] = j;
        count += __popc(votes);
        if (j0 + 32 >= n) last_kept = (votes >> (n - 1 - j0)) & 1u;
    }
    if (lane == 0) *tiles = 2 * count - ((last_kept && tokens - (n - 1) * kSelBlock <= 64) ? 1 : 0);
}

// The topk-th largest of a row's keys, bit by bit from the first bit in which the keys differ: `count(trial)` says how many
// keys reach a trial value; the search ends when exactly `want` do.  Whole warp; returns the bound and how many reach it.
template <typename Count>
__device__ __forceinline__ unsigned long long find_bound(const Count& count, unsigned long long all_or, unsigned long long all_and,
                                                         int n, int want, int& reached) {
    const unsigned long long differ = all_or ^ all_and;
    reached = n;
    if (differ == 0) return all_and;
    const int top = 63 - __clzll(static_cast<long long>(differ));
    unsigned long long bound = top == 63 ? 0ull : all_and & ~((1ull << (top + 1)) - 1ull);     // the common leading bits
    for (int bit = top; bit >= 0 && reached != want; --bit) {
        const unsigned long long trial = bound | (1ull << bit);
        const int c = __reduce_add_sync(0xffffffffu, count(trial));
        if (c >= want) { bound = trial; reached = c; }
    }
    return bound;
}

// Scores and top-k.  A CTA of 256 threads takes kRows query blocks of one (batch, head).  Thread (slice, j): key block j,
// j + keys, ... and a slice of the channels, with all rows (the means of k are stored channel by channel, so a warp reads
// contiguous bytes, and every value feeds kRows multiply-adds); few key blocks leave several slices per key, whose
// sums are joined in a fixed order, so that equal key blocks have equal scores.  Then a warp per row finds the topk-th
// largest key by counting (find_bound) and keeps the keys above it and, of those equal to it, the first ones.  Up to 256
// key blocks a lane holds its share of the row in registers.
// What bounds it is latency: with 12 heads of 256 x 256 blocks 201 M multiply-adds in fp64 are 12 us of the fp64 pipes.
constexpr int kTopkThreads = 256;
template <int kRows>
__global__ void __launch_bounds__(kTopkThreads)
block_topk_kernel(const double* __restrict__ qm, const double* __restrict__ kmt, unsigned char* __restrict__ mask,
                  int* __restrict__ index, int* __restrict__ tiles, int n_q, int n_k, int D, int Lk, int topk, int slices) {
    // keys [kRows][n_k], the queries' means [D][kRows], and with slices their sums [slices][kRows][256 / slices]
    extern __shared__ unsigned long long sel_keys[];
    double* qs = reinterpret_cast<double*>(sel_keys + static_cast<size_t>(kRows) * n_k);
    double* part = qs + D * kRows;
    const int groups = (n_q + kRows - 1) / kRows;
    const long long bh = blockIdx.x / groups;
    const int i0 = static_cast<int>(blockIdx.x - bh * groups) * kRows;
    for (int e = threadIdx.x; e < kRows * D; e += kTopkThreads) {
        const int r = e / D, d = e - r * D;
        qs[d * kRows + r] = i0 + r < n_q ? qm[(bh * n_q + i0 + r) * D + d] : 0.0;
    }
    __syncthreads();
    const int keys = kTopkThreads / slices, slice = threadIdx.x / keys, j_own = threadIdx.x - slice * keys;
    const int each = D / slices, d0 = slice * each;
    for (int j0 = 0; j0 < n_k; j0 += keys) {                     // (once where there are slices)
        const int j = j0 + j_own;
        double acc[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) acc[r] = 0.0;
        if (j < n_k) {
            const double* kp = kmt + (bh * D + d0) * n_k + j;
#pragma unroll 16
            for (int d = 0; d < each; ++d) {
                const double kv = __ldg(kp + static_cast<long long>(d) * n_k);
#pragma unroll
                for (int r = 0; r < kRows; ++r) acc[r] = fma(qs[(d0 + d) * kRows + r], kv, acc[r]);
            }
        }
        if (slices == 1) {
            if (j < n_k) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) sel_keys[static_cast<size_t>(r) * n_k + j] = ordered_key(acc[r]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRows; ++r) part[(slice * kRows + r) * keys + j_own] = acc[r];
            __syncthreads();
            for (int e = threadIdx.x; e < kRows * keys; e += kTopkThreads) {
                const int r = e / keys, jj = e - r * keys;
                double sum = 0.0;
                for (int s = 0; s < slices; ++s) sum += part[(s * kRows + r) * keys + jj];
                if (jj < n_k) sel_keys[static_cast<size_t>(r) * n_k + jj] = ordered_key(sum);
            }
        }
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r = warp; r < kRows && i0 + r < n_q; r += kTopkThreads / 32) {
        const unsigned long long* row_keys = sel_keys + static_cast<size_t>(r) * n_k;
        const int want = min(topk, n_k);
        unsigned long long all_or = 0, all_and = ~0ull, bound;
        int reached;
        if (n_k <= 256) {
            unsigned long long own[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int j = lane + 32 * u;
                own[u] = j < n_k ? row_keys[j] : 0ull;           // (0 is below every key of a score)
                if (j < n_k) { all_or |= own[u]; all_and &= own[u]; }
            }
            for (int m = 16; m >= 1; m >>= 1) {
                all_or |= __shfl_xor_sync(0xffffffffu, all_or, m);
                all_and &= __shfl_xor_sync(0xffffffffu, all_and, m);
            }
            bound = find_bound([&](unsigned long long trial) {
                int c = 0;
#pragma unroll
                for (int u = 0; u < 8; ++u) c += own[u] >= trial ? 1 : 0;
                return c;
            }, all_or, all_and, n_k, want, reached);
        } else {
            for (int j = lane; j < n_k; j += 32) { all_or |= row_keys[j]; all_and &= row_keys[j]; }
            for (int m = 16; m >= 1; m >>= 1) {
                all_or |= __shfl_xor_sync(0xffffffffu, all_or, m);
                all_and &= __shfl_xor_sync(0xffffffffu, all_and, m);
            }
            bound = find_bound([&](unsigned long long trial) {
                int c = 0;
                for (int j = lane; j < n_k; j += 32) c += row_keys[j] >= trial ? 1 : 0;
                return c;
            }, all_or, all_and, n_k, want, reached);
        }
        // more than `want` keys reach the bound: of those equal to it only the first ones are kept
        const int spare = reached - want;
        int equal = 0;
        if (spare > 0) {
            for (int j = lane; j < n_k; j += 32) equal += row_keys[j] == bound ? 1 : 0;
            equal = __reduce_add_sync(0xffffffffu, equal);
        }
        const int keep_equal = equal - spare;
        int seen = 0;                                            // keys equal to the bound among the columns so far
        auto keep = [&](int j, bool inside) {
            const unsigned long long key = inside ? row_keys[j] : 0ull;
            if (spare == 0) return key >= bound;
            const unsigned ties = __ballot_sync(0xffffffffu, inside && key == bound);
            const int before = seen + __popc(ties & ((1u << lane) - 1u));
            seen += __popc(ties);
            return key > bound || (key == bound && before < keep_equal);
        };
        const long long row = bh * n_q + i0 + r;
        write_row(keep, n_k, Lk, mask + row * n_k, index + row * n_k, tiles + row);
    }
}

// Lists of a given mask: a warp per row.
__global__ void __launch_bounds__(256)
block_lists_kernel(const unsigned char* __restrict__ mask, int* __restrict__ index, int* __restrict__ tiles, long long rows,
                   int n_k, int Lk) {
    const long long row = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const unsigned char* m = mask + row * n_k;
    write_row([&](int j, bool inside) { return inside && m[j] != 0; }, n_k, Lk, nullptr, index + row * n_k, tiles + row);
}

// The order in which lists are worked on: inside every window of consecutive rows the longest first, rows of equal length in
// their order.  Persistent CTAs then end together (24 heads of 33 lists of 0 to 30 of 63 blocks, 148 CTAs: 107 tiles of work
// on the busiest one instead of 136, 98 on average).  A window is six rows per SM: large enough to even out, small enough
// that the CTAs stay with a few heads at a time, whose keys and values the L2 cache then holds (sorted across all heads, no two
// CTAs would read the same ones).  `swap`: kOrderKeys words of shared memory; a CTA of kOrderThreads threads.
// A bitonic network over four keys per thread: the exchanges happen in registers and between lanes, and only six of the 55
// steps, those between warps, go through shared memory (all of them there: 8.4 us for a window instead of 3).
constexpr int kOrderWindow = 6 * 148, kOrderKeys = 1024, kOrderThreads = kOrderKeys / 4;
__device__ __forceinline__ void block_order(const int* tiles, int* order, int n_rows, int window, uint4* swap) {
    const int t = threadIdx.x, base = window * kOrderWindow, count = min(kOrderWindow, n_rows - base);
    uint32_t v[4];                                               // elements 4 t .. 4 t + 3; filling zeros stay behind every row
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * t + i;
        v[i] = e < count ? static_cast<uint32_t>(max(tiles[base + e], 0)) * kOrderKeys + (kOrderKeys - 1 - e) : 0u;
    }
#pragma unroll
    for (int k = 2; k <= kOrderKeys; k *= 2)
#pragma unroll
        for (int j = k / 2; j >= 1; j /= 2) {
            uint32_t other[4];                                   // elements e ^ j
            if (j >= 128) {
                swap[t] = make_uint4(v[0], v[1], v[2], v[3]);
                __syncthreads();
                const uint4 o = swap[t ^ (j / 4)];
                other[0] = o.x; other[1] = o.y; other[2] = o.z; other[3] = o.w;
                __syncthreads();
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) other[i] = j >= 4 ? __shfl_xor_sync(0xffffffffu, v[i], j / 4) : v[i ^ (j & 3)];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 4 * t + i;
                v[i] = ((e & j) == 0) == ((e & k) == 0) ? max(v[i], other[i]) : min(v[i], other[i]);
            }
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * t + i < count) order[base + 4 * t + i] = base + (kOrderKeys - 1 - static_cast<int>(v[i] % kOrderKeys));
}
__global__ void __launch_bounds__(kOrderThreads) block_order_kernel(const int* __restrict__ tiles, int* __restrict__ order, int n_rows) {
    __shared__ uint4 swap[kOrderThreads];
    block_order(tiles, order, n_rows, blockIdx.x, swap);
}

// The transposed lists: for every key block the query blocks that kept it.  A CTA takes 32 key blocks of one (batch,
// head): one word per query block holds their truth values, and a warp then walks the words for each of them.
__global__ void __launch_bounds__(256)
block_transpose_kernel(const unsigned char* __restrict__ mask, int* __restrict__ index, int* __restrict__ tiles, int n_q,
                       int n_k, int Lq) {
    extern __shared__ unsigned sel_words[];                      // [n_q]
    const int groups = (n_k + 31) / 32;
    const long long bh = blockIdx.x / groups;
    const int j0 = static_cast<int>(blockIdx.x - bh * groups) * 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned char* column = mask + bh * n_q * n_k + j0 + lane;
    const bool inside = j0 + lane < n_k;
    for (int i0 = warp * 8; i0 < n_q; i0 += 64) {                // (eight rows' loads in flight per warp)
        unsigned char v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = inside && i0 + u < n_q ? __ldg(column + static_cast<long long>(i0 + u) * n_k) : 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const unsigned votes = __ballot_sync(0xffffffffu, v[u] != 0);
            if (lane == u && i0 + u < n_q) sel_words[i0 + u] = votes;
        }
    }
    __syncthreads();
    for (int c = warp; c < 32 && j0 + c < n_k; c += 8) {
        const long long row = bh * n_k + j0 + c;
        write_row([&](int i, bool inside) { return inside && (sel_words[i] >> c & 1u) != 0; }, n_q, Lq, nullptr, index + row * n_q, tiles + row);
    }
}

}  // namespace attn_jvp
