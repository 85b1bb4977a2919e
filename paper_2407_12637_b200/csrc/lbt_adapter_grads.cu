// Weight gradients of the low-rank adapters: G[k,c] = s sum_m f[m,k] z[m,c] over the tokens m of one adapter's runs (dA: f = B dy, z = x;
// dB: f = A x, z = dy).
//
// Bound by memory: z is read once (2 rank operations an element).  A cluster takes 256 bytes of each row (128 or 64 columns) and up to
// 64 ranks; its CTAs take 64 tokens at a time in turn, z's rows and f's through a ring of stages in shared memory.  The warps of a CTA
// share a stage's tokens and columns.  16-bit z enters the matrix instructions as it is, pairs of its rows joined; f is split into three
// bf16 or two fp16 numbers (24 or 22 bits: the gradients are fp32).  fp32 z and f are split into two tf32 numbers each.  fp16 holds no
// more than 65504: there f enters times a power of two that brings the largest finite value of the CTA's tokens to [512, 1024) (an infinity or
// NaN spoils its own rank's gradient alone).
// (The tensor core's own sums are cut off, not rounded: those of four stages at most are added up in fp32.)
// 8192 tokens, 4096 and 4096 columns, bf16, rank 16: 41 us for both gradients (56 with cold caches; reading x and dy takes 20): issue slots are
// 0.46 busy with joining rows, splitting f and the ring, and the two kernels' data meet in L2 only in part.
#include <algorithm>

#include "lbt_adapters.cuh"

namespace lbt {

constexpr int kAgTokens = 64, kAgStride = 256 + 16;
template <int kR16> constexpr int kAgStages = kR16 <= 2 ? 4 : 3;

// An adapter's tokens, one run after the other, 64 at a time, by a warp: a window of 32 runs lies in its lanes.
struct Tokens {
    int window, before, upto, lo, total, pos;   // the window's first run; this lane's run: tokens ahead of it and up to its end, first token; the window's tokens, where the next is
    int end, shift;                             // the run that the last piece ended in: its tokens lie at place + shift up to place `end`
    __device__ __forceinline__ Tokens() : window(-32), before(0), upto(0), lo(0), total(0), pos(0), end(0), shift(0) {}
    __device__ __forceinline__ bool next_window(const AdapterGradArgs& g, int adapter) {
        window += 32;
        end = 0;
        if (window >= g.runs) { window = g.runs; total = pos = 0; return false; }
        const int lane = threadIdx.x & 31, r = window + lane;
        int hi = 0;
        lo = 0;
        if (r < g.runs) {
            if (g.offsets == nullptr) hi = adapter == 0 ? (int)g.M : 0;
            else if (g.index[r] == adapter) run_range(g.offsets, r, g.M, lo, hi);
        }
        upto = hi - lo;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += v;
        }
        before = upto - (hi - lo);
        total = __shfl_sync(0xFFFFFFFFu, upto, 31);
        return true;
    }
    __device__ __forceinline__ void skip(const AdapterGradArgs& g, int adapter, int count) {
        pos += count;
        while (pos >= total) {
            const int over = pos - total;
            if (!next_window(g, adapter)) return;
            pos = over;
        }
    }
    // The next 64 tokens into ids (-1: there are no more); how many there are.
    __device__ __forceinline__ int take(const AdapterGradArgs& g, int adapter, int* ids) {
        const int lane = threadIdx.x & 31;
        int filled = 0;
        if (pos + kAgTokens <= end) {   // all of them in that run
            ids[lane] = pos + shift + lane;
            ids[lane + 32] = pos + shift + lane + 32;
            pos += kAgTokens;
            return kAgTokens;
        }
        while (filled < kAgTokens) {
            if (pos >= total) {   // (the next window may hold none of this adapter's)
                if (!next_window(g, adapter)) break;
                pos = 0;
            }
            const int n = min(kAgTokens - filled, total - pos);
            for (int j = lane; j - lane < n; j += 32) {
                const int at = pos + min(j, n - 1);
                int own = 0;   // the last run that begins at or ahead of `at` and is not empty there
#pragma unroll
                for (int d = 16; d > 0; d >>= 1)
                    if (__shfl_sync(0xFFFFFFFFu, before, own + d) <= at) own += d;
                const int token = __shfl_sync(0xFFFFFFFFu, lo, own) + at - __shfl_sync(0xFFFFFFFFu, before, own);
                if (j < n) ids[filled + j] = token;
                if (j - lane + 32 >= n) {   // the run of the last token
                    shift = __shfl_sync(0xFFFFFFFFu, token - at, 31);
                    end = __shfl_sync(0xFFFFFFFFu, upto, __shfl_sync(0xFFFFFFFFu, own, 31));
                }
            }
            filled += n;
            pos += n;
        }
        for (int j = filled + lane; j < kAgTokens; j += 32) ids[j] = -1;
        return filled;
    }
};

template <typename T, typename G, int kR16, bool kWords>
__global__ void __launch_bounds__(kAdThreads, 2) adapter_grad_kernel(const __grid_constant__ AdapterGradArgs g) {
    constexpr bool kF32 = IsF32<T>::value, kHalf = IsHalf<T>::value;
    constexpr int kAgCols = 256 / (int)sizeof(T), kTerms = kF32 ? 8 : 16;      // tokens of an instruction
    constexpr int kR = 16 * kR16, kRow = kR + 4, kNt = kR16 <= 2 ? 8 : 4;      // kNt: a warp's instructions along the columns
    constexpr int kAcross = kAgCols / (8 * kNt), kAlong = kAdWarps / kAcross;  // warps along the columns, along the tokens
    constexpr int kStage = kAgTokens * (kAgStride + 4 * kRow), kStages = kAgStages<kR16>;
    constexpr int kEach = kAgTokens / kTerms / kAlong;                          // instructions of a warp along a stage's tokens
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ uint32_t most_of[kAdWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t = lane & 3, across = warp % kAcross, along = warp / kAcross;
    const int cta = (int)cluster_ctarank(), ctas = g.ctas;
    int block = blockIdx.x / ctas;
    const int which = block < g.groups[0] ? 0 : 1;
    if (which == 1) block -= g.groups[0];
    const int col = kAgCols * block, cols = g.cols[which], adapter = blockIdx.y, rank0 = blockIdx.z * kR, ranks = min(kR, g.rank - rank0);
    const float* f = g.f[which] + rank0;
    const T* z = static_cast<const T*>(g.z[which]) + col;
    const int64_t ld = g.ld[which];
    const bool even_ranks = g.rank % 4 == 0 && (reinterpret_cast<uintptr_t>(f) & 15) == 0;

    // ids: the tokens of the pieces under way; this CTA takes every `ctas`-th piece.
    __shared__ int ids[kStages + 1][kAgTokens], have[kStages + 1];
    auto produce = [&](Tokens& tokens, int at) {
        if (warp != 0) return;
        const int n = tokens.take(g, adapter, ids[at]);
        if (lane == 0) have[at] = n;
        tokens.skip(g, adapter, (ctas - 1) * kAgTokens);
    };
    float factor = 1.0f;
    if (kHalf) {
        uint32_t most = 0;
        Tokens tokens;
        if (warp == 0) tokens.skip(g, adapter, cta * kAgTokens);
        for (;;) {
            produce(tokens, 0);
            __syncthreads();
            const int n = have[0] * ranks;
            for (int i = threadIdx.x; i < n; i += kAdThreads) {
                const uint32_t v = abs_bits(f[(int64_t)ids[0][i / ranks] * g.rank + i % ranks]);
                if (v < kNonFinite) most = max(most, v);
            }
            __syncthreads();
            if (n == 0) break;
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if (lane == 0) most_of[warp] = most;
        __syncthreads();
        factor = row_factor(__reduce_max_sync(0xFFFFFFFFu, most_of[lane & 7]));
    }

    auto fetch = [&](int slot, const int* tokens, int count) {
        if (count > 0) {
            const uint32_t to = smem_u32(ring) + slot * kStage;
            if constexpr (kWords) {   // a warp a row
                const T* z0 = z - col;
                const int n = min(kAgCols, cols - col);
                for (int m = warp; m < kAgTokens; m += kAdWarps) {
                    copy_words<T, 2>(to + m * kAgStride, 0, z + (int64_t)max(tokens[m], 0) * ld, 0, 1, m < count ? n : 0, z0);
                }
                if constexpr (!kF32) {   // the 65th word of rows that begin odd
                    if (threadIdx.x < kAgTokens) {
                        const T* p = z + (int64_t)max(tokens[threadIdx.x], 0) * ld;
                        if (begins_odd(p)) copy_word(to + threadIdx.x * kAgStride, p, 64, (int)threadIdx.x < count ? n : 0, z0);
                    }
                }
            } else {
#pragma unroll
                for (int q = 0; q < kAgTokens / 16; ++q) {
                    const int m = (threadIdx.x >> 4) + 16 * q, c = kAgCols / 16 * (threadIdx.x & 15);
                    const uint32_t bytes = m < count && col + c < cols ? 16 : 0;
                    copy16(to + m * kAgStride + 16 * (threadIdx.x & 15), bytes ? z + (int64_t)tokens[m] * ld + c : z, bytes);
                }
            }
            if (even_ranks) {   // f's rows by 16 bytes
                constexpr int kLine = kR / 4;
#pragma unroll
                for (int q = 0; q < (kAgTokens * kLine + kAdThreads - 1) / kAdThreads; ++q) {
                    const int i = threadIdx.x + kAdThreads * q, m = i / kLine, k = 4 * (i % kLine);
                    const uint32_t bytes = m < count && k < ranks ? 16 : 0;
                    copy16(to + kAgTokens * kAgStride + 4 * (m * kRow + k), bytes ? f + (int64_t)tokens[m] * g.rank + k : f, bytes);
                }
            } else {
#pragma unroll
                for (int q = 0; q < kAgTokens * kR / kAdThreads; ++q) {
                    const int i = threadIdx.x + kAdThreads * q, m = i / kR, k = i % kR;
                    const uint32_t bytes = m < count && k < ranks ? 4 : 0;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + kAgTokens * kAgStride + 4 * (m * kRow + k)),
                                 "l"(bytes ? f + (int64_t)tokens[m] * g.rank + k : f), "r"(bytes) : "memory");
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Tokens tokens;
    if (warp == 0) tokens.skip(g, adapter, cta * kAgTokens);
    for (int i = 0; i < kStages; ++i) produce(tokens, i);
    __syncthreads();
    for (int i = 0; i < kStages - 1; ++i) fetch(i, ids[i], have[i]);

    float acc[kR16][kNt][4];
#pragma unroll
    for (int n = 0; n < kR16; ++n)
#pragma unroll
        for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][j][i] = 0.0f;
    float sum[kNt][4];     // of up to four pieces (one, with several blocks of ranks)
    int pieces = 0;
    int at = 0, now = 0;   // the piece's stage, and its place among the lists of tokens
    for (;;) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();   // (all warps have left the stage that is filled next, and the list that is)
        if (have[now] == 0) break;
        const int ahead = now + kStages - 1 > kStages ? now - 2 : now + kStages - 1, last = now == 0 ? kStages : now - 1;
        fetch(at == 0 ? kStages - 1 : at - 1, ids[ahead], have[ahead]);
        produce(tokens, last);
        __syncwarp();   // (lanes copied words of their own number; matrix instructions, a whole warp's, follow)
        const int* list = ids[now];
        const uint8_t* s = ring + at * kStage;
        const float* fs = reinterpret_cast<const float*>(s + kAgTokens * kAgStride);
        at = at + 1 == kStages ? 0 : at + 1;
        now = now == kStages ? 0 : now + 1;
        const bool odd = begins_odd(z), turns = kWords && (ld & 1) != 0;   // whether token 0's row begins odd, whether odd tokens' rows then differ
        constexpr int kRows = kF32 ? 2 : 4, kLine = kNt * (int)sizeof(T) / 4;          // rows of z of a lane and an instruction, words of each
        uint32_t r[kEach][kRows][kLine];
#pragma unroll
        for (int h = 0; h < kEach; ++h)
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                const int m = kTerms * (along + kAlong * h) + (kF32 ? t + 4 * q : 2 * t + (q & 1) + 8 * (q >> 1));
                ld_row<T, kWords>(s + m * kAgStride + 8 * kNt * (int)sizeof(T) * across + kNt * (int)sizeof(T) * gq, odd != (turns && (max(list[m], 0) & 1)), r[h][q]);   // (what is not there was copied like token 0)
            }
#pragma unroll
        for (int n = 0; n < kR16; ++n) {
            if (kR16 > 1 || pieces == 0)
#pragma unroll
                for (int j = 0; j < kNt; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[j][i] = 0.0f;
#pragma unroll
            for (int h = 0; h < kEach; ++h) {
                uint32_t hi[4], lo[4], rest[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // ranks g and g + 8 at the first term (or pair of terms), then at the second
                    const float* v = fs + (kTerms * (along + kAlong * h) + (kF32 ? t + 4 * (i >> 1) : 2 * t + 8 * (i >> 1))) * kRow + 16 * n + gq + 8 * (i & 1);
                    if constexpr (kF32) split(v[0], hi[i], lo[i]);
                    else if constexpr (kHalf) split16<T>(v[0] * factor, v[kRow] * factor, hi[i], lo[i]);
                    else split_three(v[0], v[kRow], hi[i], lo[i], rest[i]);
                }
                if constexpr (kF32) {
#pragma unroll
                    for (int j = 0; j < kNt; ++j) mma_split<true>(sum[j], hi, lo, __uint_as_float(r[h][0][j]), __uint_as_float(r[h][1][j]));
                } else {
                    mma_ranks<T, kNt, !kHalf>(sum, hi, lo, r[h], rest);
                }
            }
            if (kR16 > 1 || pieces == 3)
#pragma unroll
                for (int j = 0; j < kNt; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][j][i] += sum[j][i];
        }
        pieces = (pieces + 1) & 3;
    }
    if (kR16 == 1 && pieces != 0)
#pragma unroll
        for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[0][j][i] += sum[j][i];
    // The warps' sums over their tokens meet in the ring's place, those of warps on the same tokens in one slab, then the CTAs' sums.
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    constexpr int kSlabRow = kAgCols + 4, kSlab = kR * kSlabRow;
    static_assert(kAlong * kSlab * sizeof(float) <= (size_t)kStages * kStage, "the slabs take the ring's place");
    float* mine = reinterpret_cast<float*>(ring);   // [kR][kSlabRow]: the first slab, then the CTA's sums
    const float back = 1.0f / factor;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kR16; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // instruction j's columns 2 t and 2 t + 1 are 2 kNt t + j and 2 kNt t + kNt + j
            float* to = mine + along * kSlab + (16 * n + gq + 8 * (i >> 1)) * kSlabRow + 8 * kNt * across + 2 * kNt * t + kNt * (i & 1);
#pragma unroll
            for (int j = 0; j < kNt; j += 4)
                *reinterpret_cast<float4*>(to + j) = make_float4(acc[n][j][i] * back, acc[n][j + 1][i] * back, acc[n][j + 2][i] * back, acc[n][j + 3][i] * back);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < ranks * kAgCols; i += kAdThreads) {
        float* at = mine + i / kAgCols * kSlabRow + i % kAgCols;
        float v = at[0];
#pragma unroll
        for (int w = 1; w < kAlong; ++w) v += at[w * kSlab];
        at[0] = v;
    }
    __syncthreads();
    cluster_sync_all();
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    for (int i = cta * kAdThreads + threadIdx.x; i < ranks * kAgCols; i += ctas * kAdThreads) {   // each CTA finishes some rows
        const int k = i / kAgCols, c = col + i % kAgCols;
        if (c >= cols) continue;
        float v = 0.0f;
        for (int p = 0; p < ctas; ++p) v += ld_cluster(map_to_cta(smem_u32(mine + k * kSlabRow + i % kAgCols), p));
        static_cast<G*>(g.out[which])[((int64_t)adapter * g.rank + rank0 + k) * cols + c] = from_f32<G>(v * scale);
    }
    cluster_sync_all();   // nobody leaves before its sums have been fetched
}

template <typename T, typename G, int kR16, bool kWords>
static lbt_status grad_launch(AdapterGradArgs g, cudaStream_t stream) {
    constexpr int kR = 16 * kR16, kAgCols = 256 / (int)sizeof(T);
    for (int i = 0; i < 2; ++i) g.groups[i] = g.wanted[i] ? (g.cols[i] + kAgCols - 1) / kAgCols : 0;
    const int64_t blocks = (int64_t)(g.groups[0] + g.groups[1]) * g.adapters * ((g.rank + kR - 1) / kR);
    // two CTAs to an SM, and two pieces of 64 tokens for each
    g.ctas = (int)std::max<int64_t>(1, std::min<int64_t>({kAdCluster, 2 * kNumSMs / blocks, g.M / (2 * kAgTokens * std::max(1, std::min(g.adapters, g.runs)))}));
    constexpr size_t smem = (size_t)kAgStages<kR16> * kAgTokens * (kAgStride + 4 * (kR + 4));
    const dim3 grid((g.groups[0] + g.groups[1]) * g.ctas, g.adapters, (g.rank + kR - 1) / kR);
    return cluster_launch(adapter_grad_kernel<T, G, kR16, kWords>, g, grid, smem, stream, g.ctas);
}

template <typename T, typename G, bool kWords>
static lbt_status grad_rank(const AdapterGradArgs& g, cudaStream_t stream) {
    if (g.rank <= 16) return grad_launch<T, G, 1, kWords>(g, stream);
    if (g.rank <= 32) return grad_launch<T, G, 2, kWords>(g, stream);
    return grad_launch<T, G, 4, kWords>(g, stream);
}

template <typename T>
static lbt_status grad_type_of(const AdapterGradArgs& g, int grad_type, bool aligned, cudaStream_t stream) {
    if (grad_type == LBT_F32) return aligned ? grad_rank<T, float, false>(g, stream) : grad_rank<T, float, true>(g, stream);
    return aligned ? grad_rank<T, T, false>(g, stream) : grad_rank<T, T, true>(g, stream);
}

lbt_status adapter_grads(AdapterGradArgs g, int type, int grad_type, bool aligned, cudaStream_t stream) {
    if (type == LBT_F32) return grad_type_of<float>(g, grad_type, aligned, stream);
    return type == LBT_BF16 ? grad_type_of<__nv_bfloat16>(g, grad_type, aligned, stream) : grad_type_of<__half>(g, grad_type, aligned, stream);
}

}  // namespace lbt
