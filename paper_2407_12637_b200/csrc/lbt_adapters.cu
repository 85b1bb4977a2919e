// Low-rank adapters of many requests beside one linear layer, and their gradients.
//
//   h[m] = A_i x[m] (rank values);  out[m] = base[m] + s_i sum_k h[m,k] B_i[k]     for the tokens m of every run of adapter i
//
// A and B are both stored rank first, [rank, I] and [rank, O]: the gradient of x is then the same operator with A and B
// exchanged (dx = dbase + s (B dy) A), and both weight gradients have one form, G[k,c] = s sum_m f[m,k] z[m,c].
//
// Bound by memory: a token's row of x, base and out and the weights of the adapters in use, 2 rank operations an element.
// So one cluster of eight CTAs carries a tile of 16 tokens through both products: each CTA takes an eighth of x's columns,
// the partial h meet through the cluster's shared memory, then each CTA takes an eighth of the output's columns.  h never
// leaves the chip (it is written only where the backward pass asks for it).
//
// Products run as tf32 with fp32 sums: bf16 and fp16 values are exact in tf32, h enters its second product as the sum of two
// tf32 numbers (22 bits), and fp32 tensors are split the same way.  Fragments come straight from global memory: the
// reduced index may be taken in any order that both operands share, so a lane's 16 (or 32) contiguous bytes serve four
// instructions, and a lane ends up with 16 contiguous columns of the output.
#include <algorithm>

#include "lbt_sm100.cuh"
#include "lbt_types.cuh"

namespace lbt {

using namespace sm100;

constexpr int kAdTokens = 16;      // tokens of a tile
constexpr int kAdThreads = 256;
constexpr int kAdWarps = kAdThreads / 32;
constexpr int kAdCluster = 8;
constexpr int kAdMaxRank = 128;

struct AdapterArgs {
    const void* x;
    const void* a;         // [adapters, rank, I]
    const void* b;         // [adapters, rank, O]
    const float* scale;    // null: ones
    const int32_t* offsets;   // null: one run of all tokens, adapter 0
    const int32_t* index;
    const void* base;
    void* out;             // null: only h is wanted
    float* h;              // [M, rank], unscaled; null: not wanted
    int64_t M, ld_x, ld_base, ld_out;
    int I, O, runs, adapters, rank;
};

// Run r's tokens [lo, hi), cut to [0, M) whatever the offsets hold.
__device__ __forceinline__ void run_range(const int32_t* offsets, int r, int64_t M, int& lo, int& hi) {
    const int end = (int)M;
    lo = min(max(offsets[r], 0), end);
    hi = max(min(offsets[r + 1], end), lo);
}

// The run that holds a tile, by all lanes of a warp together: first token, tokens of the tile, adapter.
__device__ __forceinline__ bool run_of_tile(const AdapterArgs& g, int tile, int& row, int& rows, int& adapter) {
    if (g.offsets == nullptr) {
        row = tile * kAdTokens;
        rows = (int)min((int64_t)kAdTokens, g.M - row);
        adapter = 0;
        return rows > 0;
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int r0 = 0; r0 < g.runs; r0 += 32) {
        int lo = 0, hi = 0;
        if (r0 + lane < g.runs) run_range(g.offsets, r0 + lane, g.M, lo, hi);
        const int tiles = (hi - lo + kAdTokens - 1) / kAdTokens;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned who = __ballot_sync(0xFFFFFFFFu, tile >= before + upto - tiles && tile < before + upto);
        if (who != 0) {
            const int src = __ffs(who) - 1;
            const int at = tile - before - __shfl_sync(0xFFFFFFFFu, upto - tiles, src);
            row = __shfl_sync(0xFFFFFFFFu, lo, src) + at * kAdTokens;
            rows = min(kAdTokens, __shfl_sync(0xFFFFFFFFu, hi, src) - row);
            adapter = g.index[r0 + src];
            return true;
        }
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    return false;
}

// Eight consecutive elements of which the first `valid` exist (zeros behind them).
template <bool kAligned>
__device__ __forceinline__ void fetch8(const float* p, int valid, Vec8<float>& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.w[i] = 0;
    if (kAligned) {
        if (valid > 0) ld_vec(p, v.w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) v.w[i] = __float_as_uint(p[i]);
    }
}
template <bool kAligned, typename T>
__device__ __forceinline__ void fetch8(const T* p, int valid, Vec8<T>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = 0;
    if (kAligned) {
        if (valid > 0) ld_vec(p, v.w);
    } else {
        const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) v.w[i / 2] |= (uint32_t)u[i] << (16 * (i & 1));
    }
}

// out[0..8) = base[0..8) + d, of which the first `valid` exist
template <bool kAligned, typename T>
__device__ __forceinline__ void add8(const T* base, T* out, int valid, const float (&d)[8]) {
    if (valid <= 0) return;
    Vec8<T> v;
    float f[8];
    fetch8<kAligned>(base, valid, v);
    unpack(v, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += d[i];
    if (kAligned) {
        store8(out, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) out[i] = from_f32<T>(f[i]);
    }
}

// v = hi + lo, both tf32 (a sum of 22 bits).  An infinity or NaN is hi alone.
__device__ __forceinline__ void split(float v, uint32_t& hi, uint32_t& lo) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(v));
    const float rest = (hi & 0x7FFFFFFFu) >= kNonFinite ? 0.0f : v - __uint_as_float(hi);
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(lo) : "f"(rest));
}

// d += a b: 16 x 8 values, eight terms each.  Lane 4 g + t holds rows g, g + 8 at terms t, t + 4 of a, column g of b, and columns
// 2 t, 2 t + 1 of d.
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T> struct IsF32 { static constexpr bool value = false; };
template <> struct IsF32<float> { static constexpr bool value = true; };

// d += a b for fp32 a (two rows' values at two terms) as hi + lo, and b exact in tf32 (16-bit types) or split as well (fp32).
template <bool kSplitB>
__device__ __forceinline__ void mma_split(float (&d)[4], const uint32_t (&hi)[4], const uint32_t (&lo)[4], float b0, float b1) {
    uint32_t h0 = __float_as_uint(b0), h1 = __float_as_uint(b1), l0 = 0, l1 = 0;
    if (kSplitB) { split(b0, h0, l0); split(b1, h1, l1); }
    mma_tf32(d, lo[0], lo[1], lo[2], lo[3], h0, h1);
    if (kSplitB) mma_tf32(d, hi[0], hi[1], hi[2], hi[3], l0, l1);
    mma_tf32(d, hi[0], hi[1], hi[2], hi[3], h0, h1);
}

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// kN: blocks of eight ranks.  Shared memory: the warps' partial h, this CTA's sum of them, the tile's h.
template <typename T, int kN, bool kAligned>
__global__ void __launch_bounds__(kAdThreads) adapter_kernel(const __grid_constant__ AdapterArgs g) {
    constexpr int kR = 8 * kN, kRow = kR + 4;   // (rows 4 words apart in the banks: no two lanes of a fragment meet)
    constexpr int kSteps = kN <= 2 ? 4 : kN <= 4 ? 2 : 1;   // steps whose loads are under way together
    extern __shared__ float smem[];
    float* part = smem;                              // [warps][16][kR]
    float* mine = smem + kAdWarps * kAdTokens * kR;  // [16][kR], read by the other CTAs
    float* hs = mine + kAdTokens * kR;               // [16][kRow]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t = lane & 3;
    const int cta = (int)cluster_ctarank();
    int row, rows, adapter;
    if (!run_of_tile(g, blockIdx.x / kAdCluster, row, rows, adapter)) return;   // (all CTAs of the cluster)

    // this CTA's columns of the output, in groups of 64
    const int groups = (g.O + 63) / 64;
    const int group_lo = (int)((int64_t)groups * cta / kAdCluster), group_hi = (int)((int64_t)groups * (cta + 1) / kAdCluster);
    const T* base = static_cast<const T*>(g.base) + row * g.ld_base;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {   // no adapter: its tokens keep base
        if (g.out != nullptr && g.out != g.base)
            for (int i = threadIdx.x; i < rows * 8 * (group_hi - group_lo); i += kAdThreads) {
                const int m = i / (8 * (group_hi - group_lo)), c = 64 * group_lo + 8 * (i % (8 * (group_hi - group_lo)));
                const float zero[8] = {};
                add8<kAligned>(base + m * g.ld_base + c, out + m * g.ld_out + c, min(8, g.O - c), zero);
            }
        return;
    }

    // h of this CTA's columns of x
    const T* a = static_cast<const T*>(g.a) + (int64_t)adapter * g.rank * g.I;
    const T* x0 = static_cast<const T*>(g.x) + (row + gq) * g.ld_x;
    const T* x1 = x0 + 8 * g.ld_x;
    const bool has0 = gq < rows, has1 = gq + 8 < rows;
    float acc[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    const int steps = (g.I + 31) / 32;
    const int step_lo = (int)((int64_t)steps * cta / kAdCluster), step_hi = (int)((int64_t)steps * (cta + 1) / kAdCluster);
    for (int s0 = step_lo + warp; s0 < step_hi; s0 += kAdWarps * kSteps) {
        Vec8<T> vx0[kSteps], vx1[kSteps], va[kSteps][kN];
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int s = s0 + u * kAdWarps, k = 32 * s + 8 * t;
            const int valid = s < step_hi ? min(8, g.I - k) : 0;
            fetch8<kAligned>(x0 + k, has0 ? valid : 0, vx0[u]);
            fetch8<kAligned>(x1 + k, has1 ? valid : 0, vx1[u]);
#pragma unroll
            for (int n = 0; n < kN; ++n) fetch8<kAligned>(a + (int64_t)(8 * n + gq) * g.I + k, 8 * n + gq < g.rank ? valid : 0, va[u][n]);
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            float f0[8], f1[8];
            unpack(vx0[u], f0);
            unpack(vx1[u], f1);
#pragma unroll
            for (int p = 0; p < 4; ++p) {   // terms t and t + 4 of instruction p: the lane's elements 2 p and 2 p + 1
                uint32_t hi[4], lo[4];
                if (IsF32<T>::value) {
                    split(f0[2 * p], hi[0], lo[0]); split(f1[2 * p], hi[1], lo[1]);
                    split(f0[2 * p + 1], hi[2], lo[2]); split(f1[2 * p + 1], hi[3], lo[3]);
                } else {
                    hi[0] = __float_as_uint(f0[2 * p]); hi[1] = __float_as_uint(f1[2 * p]);
                    hi[2] = __float_as_uint(f0[2 * p + 1]); hi[3] = __float_as_uint(f1[2 * p + 1]);
                }
#pragma unroll
                for (int n = 0; n < kN; ++n) {
                    float fa[8];
                    unpack(va[u][n], fa);
                    if (IsF32<T>::value) mma_split<true>(acc[n], hi, lo, fa[2 * p], fa[2 * p + 1]);
                    else mma_tf32(acc[n], hi[0], hi[1], hi[2], hi[3], __float_as_uint(fa[2 * p]), __float_as_uint(fa[2 * p + 1]));
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        float* p = part + (warp * kAdTokens + gq) * kR + 8 * n + 2 * t;
        *reinterpret_cast<float2*>(p) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(p + 8 * kR) = make_float2(acc[n][2], acc[n][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * kR; i += kAdThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kAdWarps; ++w) v += part[w * kAdTokens * kR + i];
        mine[i] = v;
    }
    cluster_sync_all();
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    for (int i = threadIdx.x; i < kAdTokens * kR; i += kAdThreads) {
        const int m = i / kR, k = i % kR;
        float v = 0.0f;
        if (m < rows) {
#pragma unroll
            for (int c = 0; c < kAdCluster; ++c) v += ld_cluster(map_to_cta(smem_u32(mine + i), c));
            if (cta == 0 && g.h != nullptr && k < g.rank) g.h[(int64_t)(row + m) * g.rank + k] = v;
        }
        hs[m * kRow + k] = v * scale;
    }
    cluster_sync_all();   // nobody leaves, and nobody's hs is read, before the partial sums have been fetched
    if (g.out == nullptr) return;

    const T* b = static_cast<const T*>(g.b) + (int64_t)adapter * g.rank * g.O;
    for (int group = group_lo + warp; group < group_hi; group += kAdWarps) {
        const int col = 64 * group;
        float d[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[j][i] = 0.0f;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            Vec8<T> v0, v1;
            const int valid = min(8, g.O - col - 8 * gq);
            fetch8<kAligned>(b + (int64_t)(8 * n + t) * g.O + col + 8 * gq, 8 * n + t < g.rank ? valid : 0, v0);
            fetch8<kAligned>(b + (int64_t)(8 * n + t + 4) * g.O + col + 8 * gq, 8 * n + t + 4 < g.rank ? valid : 0, v1);
            float f0[8], f1[8];
            unpack(v0, f0);
            unpack(v1, f1);
            uint32_t hi[4], lo[4];
            split(hs[gq * kRow + 8 * n + t], hi[0], lo[0]);
            split(hs[(gq + 8) * kRow + 8 * n + t], hi[1], lo[1]);
            split(hs[gq * kRow + 8 * n + t + 4], hi[2], lo[2]);
            split(hs[(gq + 8) * kRow + 8 * n + t + 4], hi[3], lo[3]);
#pragma unroll
            for (int j = 0; j < 8; ++j) mma_split<IsF32<T>::value>(d[j], hi, lo, f0[j], f1[j]);   // column g of instruction j: 8 g + j
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int m = gq + 8 * half;
            if (m >= rows) continue;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = d[j][2 * half + q];
                const int c = col + 16 * t + 8 * q;
                add8<kAligned>(base + m * g.ld_base + c, out + m * g.ld_out + c, min(8, g.O - c), f);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- weight gradients
struct AdapterGradArgs {
    const float* f[2];     // [M, rank]: dh for da, h for db
    const void* z[2];      // x, dy
    void* out[2];          // da, db (null: not wanted)
    int64_t ld[2];
    int cols[2], groups[2];   // I, O; column groups of 64 (0 where not wanted)
    const float* scale;
    const int32_t* offsets;
    const int32_t* index;
    int64_t M;
    int runs, adapters, rank;
};

constexpr int kAgRanks = 32;   // ranks of a CTA: two rows of instructions

// G[k,c] = s sum_m f[m,k] z[m,c] over the tokens of one adapter's runs: 32 ranks and 64 columns a cluster, whose 64 warps take
// eight tokens at a time in turn; the partial sums meet in shared memory, in a fixed order.
template <typename T, typename G, bool kAligned>
__global__ void __launch_bounds__(kAdThreads) adapter_grad_kernel(const __grid_constant__ AdapterGradArgs g) {
    extern __shared__ float smem[];
    float* part = smem;                                // [warps][32][64]
    float* mine = smem + kAdWarps * kAgRanks * 64;     // [32][64]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t = lane & 3;
    const int cta = (int)cluster_ctarank();
    int group = blockIdx.x / kAdCluster;
    const int which = group < g.groups[0] ? 0 : 1;
    if (which == 1) group -= g.groups[0];
    const int col = 64 * group, cols = g.cols[which], adapter = blockIdx.y, rank0 = blockIdx.z * kAgRanks;
    const float* f = g.f[which];
    const T* z = static_cast<const T*>(g.z[which]);
    const int64_t ld = g.ld[which];
    const int valid = min(8, cols - col - 8 * gq);
    float d[2][8][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[n][j][i] = 0.0f;
    int at = cta * kAdWarps + warp;   // steps of eight tokens until this warp's next one
    for (int r = 0; r < g.runs; ++r) {
        int lo = 0, hi = (int)g.M;
        if (g.offsets != nullptr) {
            if (g.index[r] != adapter) continue;
            run_range(g.offsets, r, g.M, lo, hi);
        }
        const int steps = (hi - lo + 7) / 8;
        for (; at < steps; at += kAdWarps * kAdCluster) {
            const int m0 = lo + 8 * at + t, m1 = m0 + 4;
            Vec8<T> v0, v1;
            fetch8<kAligned>(z + m0 * ld + col + 8 * gq, m0 < hi ? valid : 0, v0);
            fetch8<kAligned>(z + m1 * ld + col + 8 * gq, m1 < hi ? valid : 0, v1);
            float w[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = rank0 + 16 * n + gq + 8 * (i & 1), m = i < 2 ? m0 : m1;
                    w[n][i] = k < g.rank && m < hi ? f[(int64_t)m * g.rank + k] : 0.0f;
                }
            float f0[8], f1[8];
            unpack(v0, f0);
            unpack(v1, f1);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                uint32_t h[4], l[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) split(w[n][i], h[i], l[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) mma_split<IsF32<T>::value>(d[n][j], h, l, f0[j], f1[j]);
            }
        }
        at -= steps;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // instruction j's columns 2 t and 2 t + 1 are 16 t + j and 16 t + 8 + j
            float* p = part + (warp * kAgRanks + 16 * n + gq + 8 * (i >> 1)) * 64 + 16 * t + 8 * (i & 1);
            *reinterpret_cast<float4*>(p) = make_float4(d[n][0][i], d[n][1][i], d[n][2][i], d[n][3][i]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(d[n][4][i], d[n][5][i], d[n][6][i], d[n][7][i]);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < kAgRanks * 64; i += kAdThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kAdWarps; ++w) v += part[w * kAgRanks * 64 + i];
        mine[i] = v;
    }
    cluster_sync_all();
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    const int i = cta * kAdThreads + threadIdx.x, k = rank0 + i / 64, c = col + i % 64;   // each CTA finishes four of the 32 ranks
    float v = 0.0f;
#pragma unroll
    for (int p = 0; p < kAdCluster; ++p) v += ld_cluster(map_to_cta(smem_u32(mine + i), p));
    if (k < g.rank && c < cols) static_cast<G*>(g.out[which])[((int64_t)adapter * g.rank + k) * cols + c] = from_f32<G>(v * scale);
    cluster_sync_all();
}

// ---------------------------------------------------------------------------------------------- launches
template <typename Args>
static lbt_status cluster_launch(void (*kernel)(Args), const Args& args, dim3 grid, size_t smem, cudaStream_t stream) {
    LBT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(kAdThreads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kAdCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, args));
    return launch_status();
}

template <typename T, int kN>
static lbt_status adapter_launch(const AdapterArgs& g, bool aligned, cudaStream_t stream) {
    // a run of n tokens has at most n / 16 + 1 tiles, and no more than n
    const int64_t tiles = g.offsets == nullptr ? (g.M + kAdTokens - 1) / kAdTokens : std::min<int64_t>(g.M, g.M / kAdTokens + g.runs);
    constexpr size_t smem = sizeof(float) * (kAdWarps * kAdTokens * 8 * kN + kAdTokens * 8 * kN + kAdTokens * (8 * kN + 4));
    const dim3 grid((unsigned)(tiles * kAdCluster));
    return aligned ? cluster_launch(adapter_kernel<T, kN, true>, g, grid, smem, stream) : cluster_launch(adapter_kernel<T, kN, false>, g, grid, smem, stream);
}

template <typename T>
static lbt_status adapter_run(const AdapterArgs& g, bool aligned, cudaStream_t stream) {
    if (g.rank <= 8) return adapter_launch<T, 1>(g, aligned, stream);
    if (g.rank <= 16) return adapter_launch<T, 2>(g, aligned, stream);
    if (g.rank <= 32) return adapter_launch<T, 4>(g, aligned, stream);
    if (g.rank <= 64) return adapter_launch<T, 8>(g, aligned, stream);
    return adapter_launch<T, 16>(g, aligned, stream);
}

// One pass through both products; g.M > 0 and something to do.
static lbt_status adapter_pass(const AdapterArgs& g, int type, cudaStream_t stream) {
    auto ok = [&](const void* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * type_size(type) - 1)) == 0; };
    const bool aligned = g.I % 8 == 0 && g.O % 8 == 0 && g.ld_x % 8 == 0 && g.ld_base % 8 == 0 && g.ld_out % 8 == 0 && ok(g.x) && ok(g.a) && ok(g.b) &&
                         ok(g.base) && ok(g.out);
    if (type == LBT_F32) return adapter_run<float>(g, aligned, stream);
    return type == LBT_BF16 ? adapter_run<__nv_bfloat16>(g, aligned, stream) : adapter_run<__half>(g, aligned, stream);
}

template <typename T, typename G>
static lbt_status adapter_grad_launch(const AdapterGradArgs& g, bool aligned, cudaStream_t stream) {
    constexpr size_t smem = sizeof(float) * (kAdWarps + 1) * kAgRanks * 64;
    const dim3 grid((g.groups[0] + g.groups[1]) * kAdCluster, g.adapters, (g.rank + kAgRanks - 1) / kAgRanks);
    return aligned ? cluster_launch(adapter_grad_kernel<T, G, true>, g, grid, smem, stream)
                   : cluster_launch(adapter_grad_kernel<T, G, false>, g, grid, smem, stream);
}

template <typename T>
static lbt_status adapter_grads(const AdapterGradArgs& g, bool aligned, int grad_type, cudaStream_t stream) {
    if (grad_type == LBT_F32) return adapter_grad_launch<T, float>(g, aligned, stream);
    return adapter_grad_launch<T, T>(g, aligned, stream);
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
                                           const int32_t* offsets, const int32_t* index, const void* base, void* out, float* h, void* cuda_stream) {
    lbt_adapters_desc d;
    const lbt_status rc = adapter_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (a == nullptr || b == nullptr || (d.runs > 0 && (offsets == nullptr) != (index == nullptr))) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type);
    if (off(x, e) || off(a, e) || off(b, e) || off(base, e) || off(out, e) || off(scale, 4) || off(offsets, 4) || off(index, 4) || off(h, 4))
        return LBT_ERR_ALIGNMENT;
    if (d.M == 0 || (offsets != nullptr && d.runs == 0)) return LBT_OK;
    if (x == nullptr || base == nullptr || out == nullptr) return LBT_ERR_INVALID_ARG;
    const AdapterArgs g{x, a, b, scale, offsets, index, base, out, h, d.M, d.ld_x, d.ld_base, d.ld_out, (int)d.I, (int)d.O, (int)d.runs, d.adapters, d.rank};
    return adapter_pass(g, d.type, as_stream(cuda_stream));
}

extern "C" size_t lbt_adapters_workspace_bytes(const lbt_adapters_desc* desc) {
    lbt_adapters_desc d;
    return adapter_check(desc, &d) == LBT_OK ? sizeof(float) * (size_t)std::max<int64_t>(d.M, 1) * d.rank : 0;
}

extern "C" lbt_status lbt_adapters_backward(const lbt_adapters_desc* desc, const void* dy, const void* x, const float* h, const void* a, const void* b,
                                            const float* scale, const int32_t* offsets, const int32_t* index, const void* dbase, void* dx, void* da,
                                            void* db, int grad_type, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_adapters_desc d;
    const lbt_status rc = adapter_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (a == nullptr || b == nullptr || (dx == nullptr && da == nullptr && db == nullptr) || (dx != nullptr && dbase == nullptr && d.M > 0) ||
        (d.runs > 0 && (offsets == nullptr) != (index == nullptr)) || (grad_type != LBT_F32 && grad_type != d.type))
        return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type), ge = type_size(grad_type);
    if (off(dy, e) || off(x, e) || off(a, e) || off(b, e) || off(dbase, e) || off(dx, e) || off(da, ge) || off(db, ge) || off(scale, 4) || off(h, 4) ||
        off(offsets, 4) || off(index, 4) || off(ws, 4))
        return LBT_ERR_ALIGNMENT;
    const bool any = d.M > 0 && (offsets == nullptr || d.runs > 0);
    if (any && (dy == nullptr || (da != nullptr && x == nullptr) || (db != nullptr && h == nullptr))) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_adapters_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    const cudaStream_t stream = as_stream(cuda_stream);
    float* dh = static_cast<float*>(ws);
    if (any && (dx != nullptr || da != nullptr)) {   // the same operator with A and B exchanged
        const AdapterArgs g{dy, b, a, scale, offsets, index, dbase, dx, da != nullptr ? dh : nullptr, d.M, d.ld_dy, d.ld_dbase, d.ld_dx, (int)d.O, (int)d.I,
                            (int)d.runs, d.adapters, d.rank};
        const lbt_status s = adapter_pass(g, d.type, stream);
        if (s != LBT_OK) return s;
    }
    if (da == nullptr && db == nullptr) return LBT_OK;
    AdapterGradArgs g{};
    g.f[0] = dh; g.z[0] = x; g.out[0] = da; g.ld[0] = d.ld_x; g.cols[0] = (int)d.I; g.groups[0] = da != nullptr ? (int)((d.I + 63) / 64) : 0;
    g.f[1] = h; g.z[1] = dy; g.out[1] = db; g.ld[1] = d.ld_dy; g.cols[1] = (int)d.O; g.groups[1] = db != nullptr ? (int)((d.O + 63) / 64) : 0;
    g.scale = scale; g.offsets = offsets; g.index = index; g.M = d.M;
    g.runs = offsets == nullptr ? 1 : (int)d.runs;
    g.adapters = d.adapters; g.rank = d.rank;
    auto wide = [&](const void* p) { return !off(p, 8 * e); };
    const bool aligned = (da == nullptr || (d.I % 8 == 0 && d.ld_x % 8 == 0 && wide(x))) && (db == nullptr || (d.O % 8 == 0 && d.ld_dy % 8 == 0 && wide(dy)));
    if (d.type == LBT_F32) return adapter_grads<float>(g, aligned, grad_type, stream);
    return d.type == LBT_BF16 ? adapter_grads<__nv_bfloat16>(g, aligned, grad_type, stream) : adapter_grads<__half>(g, aligned, grad_type, stream);
}
