// Low-rank adapters of many requests beside one linear layer, and their gradients.
//
//   h[m] = A_i x[m] (rank values);  out[m] = base[m] + s_i sum_k h[m,k] B_i[k]     for the tokens m of every run of adapter i
//
// A and B are both stored rank first, [rank, I] and [rank, O]: the gradient of x is then the same operator with A and B
// exchanged (dx = dbase + s (B dy) A), and both weight gradients have one form, G[k,c] = s sum_m f[m,k] z[m,c].
//
// Bound by memory: a token's row of x, base and out and the weights of the adapters in use, 2 rank operations an element.  One
// launch carries a tile of tokens through both products: the CTAs of a cluster share x's columns, their partial h meet through the
// cluster's shared memory, then they share the output's columns.  h never leaves the chip (it is written only where the backward
// pass asks for it).  Three kernels: tiles of 16 tokens (few tokens, short runs), and tiles of 128 on the tensor cores' own memory
// (16-bit rows that begin on 16 bytes: lbt_adapters_tc.cu) or, for fp32 and rows that begin anywhere, on fragments in registers.
// The rule between them stands at the launch, with both sides' times.
//
// Here bf16 and fp16 products run on fragments as they lie in memory, h entering the second one as two 16-bit numbers (fp16: after a
// power of two for each row); fp32 ones as tf32, both operands split into two.  The reduced index may be taken in any order that
// both operands share, so a lane's 32 contiguous bytes of x and A serve four instructions, and a lane ends up with 16 contiguous columns of
// the output.  mma.sync reaches about 1250 multiply-adds a clock and SM here.
#include <algorithm>
#include <atomic>

#include "lbt_adapters.cuh"

namespace lbt {

// Few tokens a run: 16 of them a tile; the weights are what is read.  A cluster of one to eight CTAs and its warps share x's columns, then the
// output's: a warp copies 128 bytes of each row (of x and A, then of base and B) into a buffer of its own, kStride bytes a row (no two
// of the eight lanes of an access meet in a bank).  The second product's first columns are under way while the cluster adds up h.
// kN: blocks of eight ranks.  kWords: rows that begin anywhere.
constexpr int kStride = 144;

template <typename T, int kN, bool kWords>
__global__ void __launch_bounds__(kAdThreads, kN <= 2 ? 4 : kN <= 8 ? 2 : 1) adapter_few_kernel(const __grid_constant__ AdapterArgs g) {
    constexpr bool kF32 = IsF32<T>::value, kHalf = IsHalf<T>::value;
    constexpr int kR = 8 * kN, kRow = kR + 4, kBuffer = (kAdTokens + kR) * kStride;
    constexpr int kStep = 128 / (int)sizeof(T), kCols = kF32 ? 4 : 8;   // columns of a step; instructions along them
    extern __shared__ __align__(16) uint8_t buffers[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t = lane & 3;
    uint8_t* s = buffers + warp * kBuffer;
    float* mine = reinterpret_cast<float*>(buffers + kAdWarps * kBuffer);   // [16][kR], read by the other CTAs
    float* hs = mine + kAdTokens * kR;                                      // [16][kRow]
    float* factor = hs + kAdTokens * kRow;                                  // [16], of fp16 rows
    const int cta = (int)cluster_ctarank(), ctas = g.ctas;
    int row, rows, adapter;
    if (!run_of_tile(g, kAdTokens, blockIdx.x / ctas, row, rows, adapter)) return;   // (all CTAs of the cluster)
    const int groups = (g.O + kStep - 1) / kStep, steps = (g.I + kStep - 1) / kStep;       // this CTA's columns of the output and of x
    const int group_lo = (int)((int64_t)groups * cta / ctas), group_hi = (int)((int64_t)groups * (cta + 1) / ctas);
    const int step_lo = (int)((int64_t)steps * cta / ctas), step_hi = (int)((int64_t)steps * (cta + 1) / ctas);
    const T* base = static_cast<const T*>(g.base) + row * g.ld_base;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {
        copy_rows<T, kWords>(g, base, out, rows, kStep * group_lo, kStep * group_hi, kAdWarps);
        return;
    }
    const T* x = static_cast<const T*>(g.x) + row * g.ld_x;
    const T* a = static_cast<const T*>(g.a) + (int64_t)adapter * g.rank * g.I;
    const T* b = static_cast<const T*>(g.b) + (int64_t)adapter * g.rank * g.O;

    // kStep columns from c0 on of the tile's rows and of the weights, by the warp.  Columns that do not exist are zeros; rows that do not
    // are left as they are (their h is not used, or set to 0).
    auto fetch = [&](const T* left, int64_t ld, const T* right, int width, int c0, const T* left0, const T* right0) {
        const uint32_t to = smem_u32(s);
        if constexpr (kWords) {   // a row at a time
            const int n = min(kStep, width - c0);
            copy_words<T, 1>(to, kStride, left + c0, ld, rows, n, left0);
            copy_words<T, 1>(to + kAdTokens * kStride, kStride, right + c0, width, g.rank, n, right0);
            if constexpr (!kF32) {   // the 33rd word of rows that begin odd
                if (lane < rows && begins_odd(left + lane * ld + c0)) copy_word(to + lane * kStride, left + lane * ld + c0, 32, n, left0);
                for (int r = lane; r < g.rank; r += 32)
                    if (begins_odd(right + (int64_t)r * width + c0)) copy_word(to + (kAdTokens + r) * kStride, right + (int64_t)r * width + c0, 32, n, right0);
            }
        } else {                  // four rows at a time
            const int c = c0 + 16 / (int)sizeof(T) * (lane & 7);
#pragma unroll
            for (int q = 0; q < (kAdTokens + kR) / 4; ++q) {
                const int r = (lane >> 3) + 4 * q, k = r - kAdTokens;
                const T* from = q < kAdTokens / 4 ? left + r * ld + c : right + (int64_t)k * width + c;
                if (q < kAdTokens / 4 ? r < rows : k < g.rank) copy16(to + r * kStride + 16 * (lane & 7), c < width ? from : left0, c < width ? 16 : 0);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto arrived = [&]() {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
    };

    float acc[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    {
        const bool odd0 = begins_odd(x + gq * g.ld_x), odd1 = begins_odd(x + (gq + 8) * g.ld_x), odd_a = begins_odd(a + (int64_t)gq * g.I);   // (8 I is even)
        for (int i = step_lo + warp; i < step_hi; i += kAdWarps) {
            fetch(x, g.ld_x, a, g.I, kStep * i, static_cast<const T*>(g.x), static_cast<const T*>(g.a));
            arrived();
            uint32_t v0[8], v1[8];
            ld_row<T, kWords>(s + gq * kStride + 32 * t, odd0, v0);
            ld_row<T, kWords>(s + (gq + 8) * kStride + 32 * t, odd1, v1);
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                uint32_t w[8];
                ld_row<T, kWords>(s + (kAdTokens + 8 * n + gq) * kStride + 32 * t, odd_a, w);
                mma_step<T>(acc[n], v0, v1, w);
            }
            __syncwarp();
        }
    }
    // The warps' sums, in their buffers' place, then the CTA's.
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        float* p = reinterpret_cast<float*>(s) + gq * kR + 8 * n + 2 * t;
        *reinterpret_cast<float2*>(p) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(p + 8 * kR) = make_float2(acc[n][2], acc[n][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * kR; i += kAdThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kAdWarps; ++w) v += reinterpret_cast<const float*>(buffers + w * kBuffer)[i];
        mine[i] = v;
    }
    __syncthreads();
    int group = group_lo + warp;
    if (g.out != nullptr && group < group_hi) fetch(base, g.ld_base, b, g.O, kStep * group, static_cast<const T*>(g.base), static_cast<const T*>(g.b));
    cluster_sync_all();
    // Eight lanes add up a row of h from all CTAs, in each CTA (handing it round would cost another meeting).
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    if (threadIdx.x < 8 * kAdTokens) {
        const int m = threadIdx.x >> 3, j = threadIdx.x & 7;
        float v[kN];
        uint32_t most = 0;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            v[n] = 0.0f;
            if (m < rows && 8 * n + j < g.rank) {
#pragma unroll
                for (int c = 0; c < kAdCluster; ++c)
                    if (c < ctas) v[n] += ld_cluster(map_to_cta(smem_u32(mine + m * kR + 8 * n + j), c));
                if (g.h != nullptr && cta == 0) g.h[(int64_t)(row + m) * g.rank + 8 * n + j] = v[n];
                v[n] *= scale;
                most = max(most, abs_bits(v[n]));
            }
        }
        float f = 1.0f;
        if (kHalf) {
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            f = row_factor(most);
            if (j == 0) factor[m] = 1.0f / f;
        }
#pragma unroll
        for (int n = 0; n < kN; ++n) hs[m * kRow + 8 * n + j] = v[n] * f;
    }
    cluster_sync_all();   // nobody leaves, and nobody's h is read, before the partial sums have been fetched
    if (g.out == nullptr) return;

    const float back0 = kHalf ? factor[gq] : 1.0f, back1 = kHalf ? factor[gq + 8] : 1.0f;
    const bool odd0 = begins_odd(base + gq * g.ld_base), odd1 = begins_odd(base + (gq + 8) * g.ld_base), odd_b = begins_odd(b), turns = (g.O & 1) != 0;
    const RankRows<T, kN> h(hs + gq * kRow, hs + (gq + 8) * kRow, t);
    for (; group < group_hi; group += kAdWarps) {
        arrived();
        float d[kCols][4];
        rank_product<T, kN, kCols, kWords>(d, h, s + kAdTokens * kStride, g.rank, gq, t, 0, odd_b, turns);
        constexpr int kOld = 2 * kCols * (int)sizeof(T) / 4;
        const int at = 4 * kOld * t, c0 = kStep * group, c = c0 + 2 * kCols * t;
        uint32_t old0[kOld], old1[kOld];
        ld_row<T, kWords>(s + gq * kStride + at, odd0, old0);
        ld_row<T, kWords>(s + (gq + 8) * kStride + at, odd1, old1);
        add_words<T>(old0, d, 0, back0);
        add_words<T>(old1, d, 1, back1);
        if constexpr (!kWords) {
            if (gq < rows) st_row<T>(out + gq * g.ld_out + c, old0, g.O - c, g.wide);
            if (gq + 8 < rows) st_row<T>(out + (gq + 8) * g.ld_out + c, old1, g.O - c, g.wide);
        } else {
            __syncwarp();   // (a lane that begins odd has read a word of its neighbour's)
            put_words(s + gq * kStride + at, old0);
            put_words(s + (gq + 8) * kStride + at, old1);
            __syncwarp();
            store_rows<T, kStep>(out + c0, g.ld_out, s, 0, rows, min(kStep, g.O - c0));
        }
        __syncwarp();
        if (group + kAdWarps < group_hi) fetch(base, g.ld_base, b, g.O, kStep * (group + kAdWarps), static_cast<const T*>(g.base), static_cast<const T*>(g.b));
    }
}

// Long runs: 128 tokens a tile, a warp for each 16 of them, and a cluster of one to eight CTAs that share x's columns and then the
// output's.  Both products walk over 128 bytes of each row at a time, whose 128 rows (of x, then of base) and weights come through a ring
// of stages in shared memory (cp.async; the second product's first stages are under way while the cluster adds up h).  Rows are kStride
// bytes apart in a stage: the eight lanes of an access meet no bank twice.  Each CTA adds up its share of h's rows and hands them to the
// others: all of them everywhere would be 128 rows times the cluster.  (The tensor core's own sums are cut off, not rounded: those of a
// step are added up in fp32.)
// kWords: rows that begin anywhere; their results go through shared memory, so that a warp stores neighbouring elements.
constexpr int kTileTokens = 128;
// above 32 ranks of 16-bit types: two warps for each 16 tokens, which take half of the ranks and then half of the columns each
template <typename T, int kN> constexpr int kTileThreads = kN <= 4 || sizeof(T) == 4 ? 256 : 512;
template <int kN> constexpr int kTileStages = kN <= 2 ? 4 : kN <= 4 ? 3 : kN <= 8 ? 5 : 2;   // what fits two blocks to an SM (to rank 32), or one

template <typename T, int kN, bool kWords>
__global__ void __launch_bounds__(kTileThreads<T, kN>, kN <= 4 ? 2 : 1) adapter_tile_kernel(const __grid_constant__ AdapterArgs g) {
    constexpr bool kF32 = IsF32<T>::value, kHalf = IsHalf<T>::value;
    constexpr int kThreads = kTileThreads<T, kN>, kHalves = kThreads / kAdThreads, kOwn = kN / kHalves;   // kOwn: blocks of ranks of a warp's first product
    constexpr int kR = 8 * kN, kRow = kR + 4, kStage = (kTileTokens + kR) * kStride, kStages = kTileStages<kN>;
    constexpr int kStep = 128 / (int)sizeof(T), kCols = kF32 ? 4 : 8 / kHalves;   // columns of a step; instructions along a warp's columns
    extern __shared__ __align__(16) uint8_t ring[];
    float* mine = reinterpret_cast<float*>(ring + kStages * kStage);   // [128][kR], read by the other CTAs
    float* hs = mine + kTileTokens * kR;                               // [128][kRow]
    float* factor = hs + kTileTokens * kRow;                           // [128], of fp16 rows
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 7, part = threadIdx.x >> 8, gq = lane >> 2, t = lane & 3;
    const int cta = (int)cluster_ctarank(), ctas = g.ctas;
    int row, rows, adapter;
    if (!run_of_tile(g, kTileTokens, blockIdx.x / ctas, row, rows, adapter)) return;   // (all CTAs of the cluster)
    const int groups = (g.O + kStep - 1) / kStep, steps = (g.I + kStep - 1) / kStep;
    const int group_lo = (int)((int64_t)groups * cta / ctas), group_hi = (int)((int64_t)groups * (cta + 1) / ctas);
    const int step_lo = (int)((int64_t)steps * cta / ctas), n1 = (int)((int64_t)steps * (cta + 1) / ctas) - step_lo;
    const T* base = static_cast<const T*>(g.base) + row * g.ld_base;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {
        copy_rows<T, kWords>(g, base, out, rows, kStep * group_lo, kStep * group_hi, kThreads / 32);
        return;
    }
    const T* x = static_cast<const T*>(g.x) + row * g.ld_x;
    const T* a = static_cast<const T*>(g.a) + (int64_t)adapter * g.rank * g.I;
    const T* b = static_cast<const T*>(g.b) + (int64_t)adapter * g.rank * g.O;
    const int n2 = g.out != nullptr ? group_hi - group_lo : 0, all = n1 + n2;

    // The next step's columns.  Columns that do not exist are zeros; rows that do not are left as they are (their h is not used, or set to 0).
    constexpr int kEach = kWords ? 1 : 16 / (int)sizeof(T), kLanes = kThreads / 8;   // aligned rows: eight threads a row, kLanes rows at a time
    constexpr int kLeft = kTileTokens / kLanes, kRight = (kR + kLanes - 1) / kLanes;
    const int own = kWords ? threadIdx.x >> 5 : threadIdx.x >> 3;                    // this thread's first row
    int next = 0, column = kStep * step_lo + (kWords ? 0 : kEach * (threadIdx.x & 7)), width = g.I;
    uint32_t slot = smem_u32(ring) + own * kStride + (kWords ? 0 : 16 * (threadIdx.x & 7));
    const T* left = x + own * g.ld_x + column;
    const T* right = a + (int64_t)own * g.I + column;
    int64_t left_step = (kWords ? kThreads / 32 : kLanes) * g.ld_x;
    const int mine_left = max(0, (rows - own + (kWords ? kThreads / 32 : kLanes) - 1) / (kWords ? kThreads / 32 : kLanes));
    const int mine_right = max(0, (g.rank - own + (kWords ? kThreads / 32 : kLanes) - 1) / (kWords ? kThreads / 32 : kLanes));
    auto fetch = [&]() {
        if (next < all) {
            if (next == n1) {   // on to the second product
                column = kStep * group_lo + (kWords ? 0 : kEach * (threadIdx.x & 7));
                width = g.O;
                left = base + own * g.ld_base + column;
                right = b + (int64_t)own * g.O + column;
                left_step = (kWords ? kThreads / 32 : kLanes) * g.ld_base;
            }
            if constexpr (kWords) {   // a warp a row
                const bool second = next >= n1;
                const int n = min(kStep, width - column);
                const T* left0 = static_cast<const T*>(second ? g.base : g.x);
                const T* right0 = static_cast<const T*>(second ? g.b : g.a);
                copy_words<T, 1>(slot, kThreads / 32 * kStride, left, left_step, mine_left, n, left0);
                copy_words<T, 1>(slot + kTileTokens * kStride, kThreads / 32 * kStride, right, (int64_t)(kThreads / 32) * width, mine_right, n, right0);
                if constexpr (!kF32) {   // the 33rd word of rows that begin odd
                    const T* l = second ? base : x;
                    const T* r0 = second ? b : a;
                    const int64_t ld = second ? g.ld_base : g.ld_x;
                    const uint32_t to = slot - own * kStride;
                    for (int r = threadIdx.x; r < kTileTokens + kR; r += kThreads) {
                        const bool is_left = r < kTileTokens;
                        const T* p = is_left ? l + r * ld + column : r0 + (int64_t)(r - kTileTokens) * width + column;
                        if ((is_left ? r < rows : r - kTileTokens < g.rank) && begins_odd(p)) copy_word(to + r * kStride, p, 32, n, is_left ? left0 : right0);
                    }
                }
            } else {
                const uint32_t bytes = column < width ? 16 : 0;
                const T* from = left;
#pragma unroll
                for (int q = 0; q < kLeft; ++q, from += left_step)
                    if (q < mine_left) copy16(slot + kLanes * q * kStride, bytes ? from : left, bytes);
                from = right;
#pragma unroll
                for (int q = 0; q < kRight; ++q, from += (int64_t)kLanes * width)
                    if (q < mine_right) copy16(slot + (kTileTokens + kLanes * q) * kStride, bytes ? from : right, bytes);
            }
            ++next;
            column += kStep;
            left += kStep;
            right += kStep;
            slot = next % kStages == 0 ? slot - (kStages - 1) * kStage : slot + kStage;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        __syncwarp();   // (lanes copied words of their own number; matrix instructions, a whole warp's, follow)
    };
    // Step i's stage, once it has come for all threads; the one behind the ring's end is then on its way.
    auto stage = [&](int i) -> uint8_t* {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();   // (all warps have left the stage that is filled next)
        fetch();
        return ring + (i % kStages) * kStage;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch();

    const int m0 = 16 * warp + gq, m1 = m0 + 8;
    float acc[kOwn][4];
#pragma unroll
    for (int n = 0; n < kOwn; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    {
        const bool odd0 = begins_odd(x + m0 * g.ld_x), odd1 = begins_odd(x + m1 * g.ld_x), odd_a = begins_odd(a + (int64_t)gq * g.I);   // (8 I is even)
        for (int i = 0; i < n1; ++i) {
            const uint8_t* s = stage(i) + 32 * t;
            uint32_t v0[8], v1[8];
            ld_row<T, kWords>(s + m0 * kStride, odd0, v0);
            ld_row<T, kWords>(s + m1 * kStride, odd1, v1);
#pragma unroll
            for (int n = 0; n < kOwn; ++n) {
                uint32_t w[8];
                ld_row<T, kWords>(s + (kTileTokens + 8 * (kOwn * part + n) + gq) * kStride, odd_a, w);
                mma_step<T>(acc[n], v0, v1, w);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kOwn; ++n) {
        const int k = 8 * (kOwn * part + n) + 2 * t;
        *reinterpret_cast<float2*>(mine + m0 * kR + k) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(mine + m1 * kR + k) = make_float2(acc[n][2], acc[n][3]);
    }
    cluster_sync_all();
    // Eight lanes add up a row of h.
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    const int first = kTileTokens * cta / ctas, last = kTileTokens * (cta + 1) / ctas;
    for (int m = first + (threadIdx.x >> 3); m - (int)(threadIdx.x >> 3) < last; m += kThreads / 8) {   // (whole warps stay together)
        const int j = threadIdx.x & 7;
        float v[kN];
        uint32_t most = 0;
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] = 0.0f;
        if (m < last && m < rows)
            for (int c = 0; c < ctas; ++c) {
                const uint32_t from = map_to_cta(smem_u32(mine + m * kR + j), c);
#pragma unroll
                for (int n = 0; n < kN; ++n) v[n] += ld_cluster(from + 32 * n);
            }
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            if (8 * n + j >= g.rank) v[n] = 0.0f;
            else if (g.h != nullptr && m < last && m < rows) g.h[(int64_t)(row + m) * g.rank + 8 * n + j] = v[n];
            v[n] *= scale;
            most = max(most, abs_bits(v[n]));
        }
        float f = 1.0f;
        if (kHalf) {
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            f = row_factor(most);
        }
        if (m >= last) continue;
        for (int c = 0; c < ctas; ++c) {
            const uint32_t to = map_to_cta(smem_u32(hs + m * kRow + j), c);
#pragma unroll
            for (int n = 0; n < kN; ++n) st_cluster(to + 32 * n, v[n] * f);
            if (kHalf && j == 0) st_cluster(map_to_cta(smem_u32(factor + m), c), 1.0f / f);
        }
    }
    cluster_sync_all();   // nobody leaves before the partial sums have been fetched, nobody goes on before h is there
    if (n2 == 0) return;

    // A warp's columns: those of a step, or half of them where two warps share it.
    const float back0 = kHalf ? factor[m0] : 1.0f, back1 = kHalf ? factor[m1] : 1.0f;
    const bool odd0 = begins_odd(base + m0 * g.ld_base), odd1 = begins_odd(base + m1 * g.ld_base), odd_b = begins_odd(b), turns = (g.O & 1) != 0;
    const RankRows<T, kN> h(hs + m0 * kRow, hs + m1 * kRow, t);
    for (int i = n1; i < all; ++i) {
        uint8_t* s = stage(i);
        float d[kCols][4];
        rank_product<T, kN, kCols, kWords>(d, h, s + kTileTokens * kStride, g.rank, gq, t, 64 * part, odd_b, turns);
        // The lane's 2 kCols neighbouring columns of both rows.
        const int at = 64 * part + 2 * kCols * (int)sizeof(T) * t, c0 = kStep * (group_lo + i - n1) + (kStep / kHalves) * part, c = c0 + 2 * kCols * t;
        constexpr int kOld = 2 * kCols * (int)sizeof(T) / 4;
        uint32_t old0[kOld], old1[kOld];
        ld_row<T, kWords>(s + m0 * kStride + at, odd0, old0);
        ld_row<T, kWords>(s + m1 * kStride + at, odd1, old1);
        add_words<T>(old0, d, 0, back0);
        add_words<T>(old1, d, 1, back1);
        if constexpr (!kWords) {
            if (m0 < rows) st_row<T>(out + m0 * g.ld_out + c, old0, g.O - c, g.wide);
            if (m1 < rows) st_row<T>(out + m1 * g.ld_out + c, old1, g.O - c, g.wide);
        } else {
            // (a lane that begins odd has read a word of its neighbour's, the last one a word of the other warp's)
            if (kHalves > 1) __syncthreads();
            else __syncwarp();
            put_words(s + m0 * kStride + at, old0);
            put_words(s + m1 * kStride + at, old1);
            __syncwarp();
            store_rows<T, kStep / kHalves>(out + 16 * warp * g.ld_out + c0, g.ld_out, s + 16 * warp * kStride, 64 * part, rows - 16 * warp, min(kStep / kHalves, g.O - c0));
        }
    }
}

// ---------------------------------------------------------------------------------------------- launches
// Clusters of `ctas` blocks that are resident at once (a cluster stays within a group of 16 to 20 SMs: where an SM holds one block, 15
// clusters of eight fit), asked once for each size.
template <typename Args>
static int clusters_fit(void (*kernel)(Args), size_t smem, int ctas, int threads, std::atomic<int>* known) {
    int n = known[ctas].load(std::memory_order_relaxed);
    if (n > 0) return n;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(ctas);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &config) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = 1;
    }
    known[ctas].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T, int kN, bool kWords>
static lbt_status adapter_launch(AdapterArgs g, cudaStream_t stream) {
    const int64_t runs = g.offsets == nullptr ? 1 : g.runs;
    constexpr int kR = 8 * kN;
    // 16 tokens a tile where runs are short on average, or where such tiles are few: a tile of 128 takes the time of its steps one after the
    // other, whatever its number.  (Both sides were timed at the widths below alone.)
    // 4096 -> 4096, 16 against 128 tokens a tile on the tensor cores' own memory: rank 16 with 1024 tokens 12 against 14 us, 2048 tokens 17 against 16; rank 32 with 1024 tokens 15 against 15; rank 64 with 128 tokens 13 against 15, 256 tokens 16 against 15;
    // rank 128 with 128 tokens 19 against 20; 2048 tokens in runs of 96: rank 16 17 against 34, rank 64 31 against 36, rank 128 60 against
    // 45, in runs of 192: 17 against 17, 31 against 19, 60 against 24.  On the other kernel, 1023 -> 2047 bf16: rank 13 with 2048 tokens 18 against
    // 21, 8192 tokens 49 against 38, in runs of 64 49 against 68, of 256 49 against 50; rank 64 28 against 36, 91 against 76, 92 against 147, 91 against
    // 145; fp32 1024 -> 2048: rank 13 16 against 22, 49 against 43; rank 64 37 against 51, 120 against 126; rank 128 82 against 86, 312 against 215.
    constexpr bool kTc = !IsF32<T>::value && !kWords;
    constexpr int kFewTiles = kTc ? (kN <= 2 ? 80 : kN <= 4 ? 64 : kN <= 8 ? 12 : 8) : kN == 16 ? 128 : IsF32<T>::value ? 256 : 160;
    constexpr int kShort = !kTc ? (kN <= 4 ? 256 : 512) : kN <= 2 ? 256 : kN <= 4 ? 64 : kN <= 8 ? 48 : 16;
    const int64_t few_tiles = std::min<int64_t>(g.M, (g.M + (kAdTokens - 1) * runs) / kAdTokens);
    if (few_tiles <= kFewTiles || (runs > 1 && g.M < kShort * runs)) {
        constexpr size_t smem = kAdWarps * (kAdTokens + kR) * kStride + sizeof(float) * kAdTokens * (kR + kR + 4 + 1);
        static std::atomic<int> fit[kAdCluster + 1];   // as many CTAs to a cluster as leave all clusters resident at once
        g.ctas = kAdCluster;
        while (g.ctas > 1 && few_tiles > clusters_fit(adapter_few_kernel<T, kN, kWords>, smem, g.ctas, kAdThreads, fit)) --g.ctas;
        return cluster_launch(adapter_few_kernel<T, kN, kWords>, g, dim3((unsigned)(few_tiles * g.ctas)), smem, stream, g.ctas);
    }
    if constexpr (kTc) {
        return adapter_tc(g, IsHalf<T>::value ? LBT_F16 : LBT_BF16, stream);
    } else {
        const int64_t tiles = (g.M + (kTileTokens - 1) * runs) / kTileTokens;   // at most
        constexpr size_t smem = kTileStages<kN> * (kTileTokens + kR) * kStride + sizeof(float) * kTileTokens * (kR + kR + 4 + 1);
        // As many CTAs to a cluster as leave all clusters resident at once, where every other run ends in the middle of a tile's half.
        static std::atomic<int> fit[kAdCluster + 1];
        g.ctas = kAdCluster;
        while (g.ctas > 1 && (g.M + kTileTokens / 2 * runs) / kTileTokens > clusters_fit(adapter_tile_kernel<T, kN, kWords>, smem, g.ctas, kTileThreads<T, kN>, fit)) --g.ctas;
        return cluster_launch(adapter_tile_kernel<T, kN, kWords>, g, dim3((unsigned)(tiles * g.ctas)), smem, stream, g.ctas, kTileThreads<T, kN>);
    }
}

template <typename T, bool kWords>
static lbt_status adapter_run(const AdapterArgs& g, cudaStream_t stream) {
    if (g.rank <= 8) return adapter_launch<T, 1, kWords>(g, stream);
    if (g.rank <= 16) return adapter_launch<T, 2, kWords>(g, stream);
    if (g.rank <= 32) return adapter_launch<T, 4, kWords>(g, stream);
    if (g.rank <= 64) return adapter_launch<T, 8, kWords>(g, stream);
    return adapter_launch<T, 16, kWords>(g, stream);
}

// Rows that begin on eight elements
static bool adapter_aligned(const AdapterArgs& g, int type) {
    auto ok = [&](const void* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * type_size(type) - 1)) == 0; };
    return g.I % 8 == 0 && g.O % 8 == 0 && g.ld_x % 8 == 0 && g.ld_base % 8 == 0 && g.ld_out % 8 == 0 && ok(g.x) && ok(g.a) && ok(g.b) && ok(g.base) && ok(g.out);
}

// One pass through both products; g.M > 0 and something to do.
static lbt_status adapter_pass(AdapterArgs g, int type, cudaStream_t stream) {
    const bool aligned = adapter_aligned(g, type);
    auto wide = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; };
    g.wide = g.I % 16 == 0 && g.O % 16 == 0 && g.ld_x % 16 == 0 && g.ld_base % 16 == 0 && g.ld_out % 16 == 0 && wide(g.x) && wide(g.a) && wide(g.base) && wide(g.out);
    if (type == LBT_F32) return aligned ? adapter_run<float, false>(g, stream) : adapter_run<float, true>(g, stream);
    if (type == LBT_BF16) return aligned ? adapter_run<__nv_bfloat16, false>(g, stream) : adapter_run<__nv_bfloat16, true>(g, stream);
    return aligned ? adapter_run<__half, false>(g, stream) : adapter_run<__half, true>(g, stream);
}

static bool off(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Sizes, types and leading dimensions (0 replaced by the row's length).
static lbt_status adapter_check(const lbt_adapters_desc* desc, lbt_adapters_desc* d) {
    if (desc == nullptr) return LBT_ERR_INVALID_ARG;
    *d = *desc;
    if (d->M < 0 || d->I < 1 || d->O < 1 || d->runs < 0 || d->adapters < 1 || d->rank < 1 || !type_ok(d->type)) return LBT_ERR_INVALID_ARG;
    int64_t* lds[] = {&d->ld_x, &d->ld_dbase, &d->ld_dx, &d->ld_base, &d->ld_out, &d->ld_dy};
    for (int i = 0; i < 6; ++i) {
        const int64_t row = i < 3 ? d->I : d->O;
        if (*lds[i] == 0) *lds[i] = row;
        if (*lds[i] < row) return LBT_ERR_INVALID_ARG;
    }
    if (d->rank > kAdMaxRank || d->I > (1 << 30) || d->O > (1 << 30) || d->M > (1 << 28) || d->runs > (1 << 28) || d->adapters > 65535)
        return LBT_ERR_UNSUPPORTED;
    return LBT_OK;
}

}  // namespace lbt

using namespace lbt;

extern "C" lbt_status lbt_adapters_forward(const lbt_adapters_desc* desc, const void* x, const void* a, const void* b, const float* scale,
                                           const int32_t* offsets, const int32_t* index, const void* base, void* out, float* h,
                                           int32_t* dev_status, void* cuda_stream) {
    lbt_adapters_desc d;
    const lbt_status rc = adapter_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (a == nullptr || b == nullptr || (d.runs > 0 && (offsets == nullptr) != (index == nullptr))) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type);
    if (off(x, e) || off(a, e) || off(b, e) || off(base, e) || off(out, e) || off(scale, 4) || off(offsets, 4) || off(index, 4) || off(h, 4) || off(dev_status, 4))
        return LBT_ERR_ALIGNMENT;
    if (d.M == 0 || (offsets != nullptr && d.runs == 0)) return LBT_OK;
    if (x == nullptr || base == nullptr || out == nullptr) return LBT_ERR_INVALID_ARG;
    const AdapterArgs g{x, a, b, scale, offsets, index, base, out, h, d.M, d.ld_x, d.ld_base, d.ld_out, (int)d.I, (int)d.O, (int)d.runs, d.adapters, d.rank, dev_status};
    return adapter_pass(g, d.type, as_stream(cuda_stream));
}

extern "C" lbt_status lbt_selftest_adapters_timeout(const lbt_adapters_desc* desc, const void* x, const void* a, const void* b, const void* base, void* out,
                                                    int rank, uint32_t limit_us, int32_t* dev_status, void* cuda_stream) {
    if (dev_status == nullptr || rank < 0 || rank >= kAdCluster || limit_us == 0 || limit_us > 1000000u) return LBT_ERR_INVALID_ARG;
    lbt_adapters_desc d;
    const lbt_status rc = adapter_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (x == nullptr || a == nullptr || b == nullptr || base == nullptr || out == nullptr) return LBT_ERR_INVALID_ARG;
    AdapterArgs g{x, a, b, nullptr, nullptr, nullptr, base, out, nullptr, d.M, d.ld_x, d.ld_base, d.ld_out, (int)d.I, (int)d.O, 1, d.adapters, d.rank, dev_status};
    if (d.M == 0 || !adapter_aligned(g, d.type) || d.type == LBT_F32) return LBT_ERR_UNSUPPORTED;
    g.limit_ns = (uint64_t)limit_us * 1000ull;
    g.mute = rank;
    return adapter_tc(g, d.type, as_stream(cuda_stream));
}

extern "C" size_t lbt_adapters_workspace_bytes(const lbt_adapters_desc* desc) {
    lbt_adapters_desc d;
    return adapter_check(desc, &d) == LBT_OK ? sizeof(float) * (size_t)std::max<int64_t>(d.M, 1) * d.rank : 0;
}

extern "C" lbt_status lbt_adapters_backward(const lbt_adapters_desc* desc, const void* dy, const void* x, const float* h, const void* a, const void* b,
                                            const float* scale, const int32_t* offsets, const int32_t* index, const void* dbase, void* dx, void* da,
                                            void* db, int grad_type, int32_t* dev_status, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_adapters_desc d;
    const lbt_status rc = adapter_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (a == nullptr || b == nullptr || (dx == nullptr && da == nullptr && db == nullptr) || (dx != nullptr && dbase == nullptr && d.M > 0) ||
        (d.runs > 0 && (offsets == nullptr) != (index == nullptr)) || (grad_type != LBT_F32 && grad_type != d.type))
        return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type), ge = type_size(grad_type);
    if (off(dy, e) || off(x, e) || off(a, e) || off(b, e) || off(dbase, e) || off(dx, e) || off(da, ge) || off(db, ge) || off(scale, 4) || off(h, 4) ||
        off(offsets, 4) || off(index, 4) || off(ws, 4) || off(dev_status, 4))
        return LBT_ERR_ALIGNMENT;
    const bool any = d.M > 0 && (offsets == nullptr || d.runs > 0);
    if (any && (dy == nullptr || (da != nullptr && x == nullptr) || (db != nullptr && h == nullptr))) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_adapters_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    if (any && dx != nullptr && ((da != nullptr && dx == x) || (db != nullptr && dx == dy))) return LBT_ERR_INVALID_ARG;   // written ahead of what reads it
    const cudaStream_t stream = as_stream(cuda_stream);
    float* dh = static_cast<float*>(ws);
    if (any && (dx != nullptr || da != nullptr)) {   // the same operator with A and B exchanged
        const AdapterArgs g{dy, b, a, scale, offsets, index, dbase, dx, da != nullptr ? dh : nullptr, d.M, d.ld_dy, d.ld_dbase, d.ld_dx, (int)d.O, (int)d.I,
                            (int)d.runs, d.adapters, d.rank, dev_status};
        const lbt_status s = adapter_pass(g, d.type, stream);
        if (s != LBT_OK) return s;
    }
    if (da == nullptr && db == nullptr) return LBT_OK;
    AdapterGradArgs g{};
    g.f[0] = dh; g.z[0] = x; g.out[0] = da; g.ld[0] = d.ld_x; g.cols[0] = (int)d.I; g.wanted[0] = da != nullptr;
    g.f[1] = h; g.z[1] = dy; g.out[1] = db; g.ld[1] = d.ld_dy; g.cols[1] = (int)d.O; g.wanted[1] = db != nullptr;
    g.scale = scale; g.offsets = offsets; g.index = index; g.M = d.M;
    g.runs = offsets == nullptr ? 1 : (int)d.runs;
    g.adapters = d.adapters; g.rank = d.rank;
    auto wide = [&](const void* p) { return !off(p, 8 * e); };
    const bool aligned = (da == nullptr || (d.I % 8 == 0 && d.ld_x % 8 == 0 && wide(x))) && (db == nullptr || (d.O % 8 == 0 && d.ld_dy % 8 == 0 && wide(dy)));
    return adapter_grads(g, d.type, grad_type, aligned, stream);
}
