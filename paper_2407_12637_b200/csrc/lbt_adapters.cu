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
#include <atomic>

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
    int ctas;     // of a cluster (adapter_tile_kernel)
    bool wide;    // rows of x, a, base and out begin on 32 bytes
};

// Run r's tokens [lo, hi), cut to [0, M) whatever the offsets hold.
__device__ __forceinline__ void run_range(const int32_t* offsets, int r, int64_t M, int& lo, int& hi) {
    const int end = (int)M;
    lo = min(max(offsets[r], 0), end);
    hi = max(min(offsets[r + 1], end), lo);
}

// The run that holds a tile, by all lanes of a warp together: first token, tokens of the tile, adapter.
template <int kTokens>
__device__ __forceinline__ bool run_of_tile(const AdapterArgs& g, int tile, int& row, int& rows, int& adapter) {
    if (g.offsets == nullptr) {
        row = tile * kTokens;
        rows = (int)min((int64_t)kTokens, g.M - row);
        adapter = 0;
        return rows > 0;
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int r0 = 0; r0 < g.runs; r0 += 32) {
        int lo = 0, hi = 0;
        if (r0 + lane < g.runs) run_range(g.offsets, r0 + lane, g.M, lo, hi);
        const int tiles = (hi - lo + kTokens - 1) / kTokens;
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
            row = __shfl_sync(0xFFFFFFFFu, lo, src) + at * kTokens;
            rows = min(kTokens, __shfl_sync(0xFFFFFFFFu, hi, src) - row);
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

template <typename T> struct IsHalf { static constexpr bool value = false; };
template <> struct IsHalf<__half> { static constexpr bool value = true; };
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

__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
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
    if (!run_of_tile<kAdTokens>(g, blockIdx.x / kAdCluster, row, rows, adapter)) return;   // (all CTAs of the cluster)

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

// ---------------------------------------------------------------------------------------------- 16-bit types, aligned rows
// Sixteen consecutive elements, `valid` of which exist (a multiple of eight): one 32-byte access where rows allow it.
struct Vec16 { uint32_t w[8]; };
template <typename T> __device__ __forceinline__ void fetch16(const T* p, int valid, bool wide, Vec16& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.w[i] = 0;
    if (wide) {
        if (valid > 8) ld_vec(p, v.w);
    } else if (valid > 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(p + 8);
        v.w[4] = q.x; v.w[5] = q.y; v.w[6] = q.z; v.w[7] = q.w;
    }
    if (valid > 0 && (!wide || valid == 8)) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        v.w[0] = q.x; v.w[1] = q.y; v.w[2] = q.z; v.w[3] = q.w;
    }
}

// d += a b: 16 x 8 values, sixteen terms each.  Lane 4 g + t holds rows g, g + 8 at terms 2 t, 2 t + 1 and 2 t + 8, 2 t + 9 of a, column
// g of b at the same terms, and columns 2 t, 2 t + 1 of d.
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two fp32 values as two of the 16-bit type, and what the rounding left of them as two more: 16 bits of a value together for bf16, 22
// for fp16.  An infinity or NaN is its first part alone.
template <typename T> __device__ __forceinline__ uint32_t pair16(float a, float b);
template <> __device__ __forceinline__ uint32_t pair16<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pair16<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 values16(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ float2 values16(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <typename T> __device__ __forceinline__ void split16(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pair16<T>(a, b);
    const float2 v = values16(hi, T());
    lo = pair16<T>(abs_bits(v.x) >= kNonFinite ? 0.0f : a - v.x, abs_bits(v.y) >= kNonFinite ? 0.0f : b - v.y);
}

// Three bf16 hold all of fp32's 24 bits.
__device__ __forceinline__ void split_three(float a, float b, uint32_t& hi, uint32_t& lo, uint32_t& rest) {
    hi = pair16<__nv_bfloat16>(a, b);
    float2 v = values16(hi, __nv_bfloat16());
    a = abs_bits(v.x) >= kNonFinite ? 0.0f : a - v.x;
    b = abs_bits(v.y) >= kNonFinite ? 0.0f : b - v.y;
    lo = pair16<__nv_bfloat16>(a, b);
    v = values16(lo, __nv_bfloat16());
    rest = pair16<__nv_bfloat16>(a - v.x, b - v.y);
}

// fp16 holds no more than 65504: a row of h enters its second product times a power of two that brings its largest value to
// [512, 1024), and the output's row is multiplied back.  (Rows of zeros, infinities or NaN: 1.)
__device__ __forceinline__ float row_factor(uint32_t most) {
    const int e = (int)(most >> 23);
    return most == 0 || most >= kNonFinite ? 1.0f : __uint_as_float((uint32_t)min(max(127 + 9 + 127 - e, 1), 254) << 23);
}

// Fragments are the operands as they lie in memory: a lane's 32 bytes of x and A serve four instructions without any conversion; of B a
// lane takes four ranks' 16 bytes and joins pairs of ranks.

// A lane's part of a tile's second product: rows g and g + 8 of a warp's 16 tokens (h as first and second parts), 8 kCols columns.  r:
// kCols of them, from kCols g on, of ranks 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
template <typename T, int kCols, bool kThird = false>
__device__ __forceinline__ void mma_ranks(float (&d)[kCols][4], const uint32_t (&hi)[4], const uint32_t (&lo)[4], const uint32_t (&r)[4][kCols / 2],
                                          const uint32_t* third = nullptr) {
#pragma unroll
    for (int j = 0; j < kCols; ++j) {   // column g of instruction j: kCols g + j
        const uint32_t sel = (j & 1) ? 0x7632u : 0x5410u;
        const uint32_t b0 = __byte_perm(r[0][j / 2], r[1][j / 2], sel), b1 = __byte_perm(r[2][j / 2], r[3][j / 2], sel);
        if constexpr (kThird) {
            const uint32_t rest[4] = {third[0], third[1], third[2], third[3]};
            mma16(d[j], rest, b0, b1, T());
        }
        mma16(d[j], lo, b0, b1, T());
        mma16(d[j], hi, b0, b1, T());
    }
}
__device__ __forceinline__ void ld_words(const uint8_t* p, uint32_t (&w)[2]) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
}
__device__ __forceinline__ void ld_words(const uint8_t* p, uint32_t (&w)[4]) { ld_vec(p, w); }
__device__ __forceinline__ void ld_words(const uint8_t* p, uint32_t (&w)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 16);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}
// h of rows g and g + 8 at ranks 16 k.. as fragments
template <typename T, int kR> __device__ __forceinline__ void h_parts(const float* h0, const float* h1, int k16, int t, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // both rows at the first pair of ranks, then at the second
        const int k = 16 * k16 + 2 * t + 8 * (i >> 1);
        const float2 v = kR > 16 * k16 + 8 * (i >> 1) ? *reinterpret_cast<const float2*>(((i & 1) ? h1 : h0) + k) : make_float2(0.0f, 0.0f);
        split16<T>(v.x, v.y, hi[i], lo[i]);
    }
}
// out = base + d for a row's 2 kCols columns of the lane (columns 2 j and 2 j + 1 of them: instructions' columns 2 t and 2 t + 1).
template <typename T, int kCols>
__device__ __forceinline__ void add_row(const uint32_t (&old)[kCols], const float (&d)[kCols][4], int half, float back, T* to, int valid, bool wide) {
    uint32_t w[kCols];
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
        const float2 o = values16(old[j], T());
        const int q = 2 * j / kCols, i = 2 * j % kCols;
        const float e0 = d[i][2 * half + q], e1 = d[i + 1][2 * half + q];
        w[j] = IsHalf<T>::value ? pair16<T>(fmaf(e0, back, o.x), fmaf(e1, back, o.y)) : pair16<T>(o.x + e0, o.y + e1);
    }
    if constexpr (kCols == 8) {
        if (wide && valid > 8) {
            st_vec(to, w);
            return;
        }
        if (valid > 8) *reinterpret_cast<uint4*>(to + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
    if (valid > 0) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}
// out = base for the tokens of a run without an adapter
template <typename T> __device__ __forceinline__ void copy_rows(const AdapterArgs& g, const T* base, T* out, int rows, int lo, int hi) {
    if (g.out == nullptr || g.out == g.base) return;
    for (int m = threadIdx.x >> 5; m < rows; m += kAdWarps)
        for (int c = lo + 8 * (threadIdx.x & 31); c < min(hi, g.O); c += 256)
            *reinterpret_cast<uint4*>(out + m * g.ld_out + c) = *reinterpret_cast<const uint4*>(base + m * g.ld_base + c);
}

// Few tokens a run: the weights are what is read.  The cluster of eight CTAs and its 64 warps share x's columns, then the output's.
template <typename T, int kN>
__global__ void __launch_bounds__(kAdThreads, kN <= 2 ? 4 : kN <= 8 ? 2 : 1) adapter_few_kernel(const __grid_constant__ AdapterArgs g) {
    constexpr int kR = 8 * kN, kRow = kR + 4, kK16 = (kN + 1) / 2;
    constexpr bool kHalf = IsHalf<T>::value;
    extern __shared__ float smem[];
    float* mine = smem;                            // [16][kR], read by the other CTAs
    float* hs = mine + kAdTokens * kR;             // [16][kRow]
    float* factor = hs + kAdTokens * kRow;         // [16], of fp16 rows
    float* part = factor + kAdTokens;              // [warps][16][kR]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gq = lane >> 2, t = lane & 3;
    const int cta = (int)cluster_ctarank();
    int row, rows, adapter;
    if (!run_of_tile<kAdTokens>(g, blockIdx.x / kAdCluster, row, rows, adapter)) return;   // (all CTAs of the cluster)
    const int groups = (g.O + 63) / 64;   // this CTA's columns of the output, in groups of 64
    const int group_lo = (int)((int64_t)groups * cta / kAdCluster), group_hi = (int)((int64_t)groups * (cta + 1) / kAdCluster);
    const T* base = static_cast<const T*>(g.base) + row * g.ld_base;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {
        copy_rows(g, base, out, rows, 64 * group_lo, 64 * group_hi);
        return;
    }
    const T* b = static_cast<const T*>(g.b) + (int64_t)adapter * g.rank * g.O;
    if (g.out != nullptr) {   // what the second product reads is on its way to L2 meanwhile
        const int lines = group_hi - group_lo;
        for (int i = threadIdx.x; i < (g.rank + rows) * lines; i += kAdThreads) {
            const int k = i / lines, c = 64 * (group_lo + i - k * lines);
            const T* p = k < g.rank ? b + (int64_t)k * g.O + c : base + (k - g.rank) * g.ld_base + c;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
        }
    }
    // h of this CTA's columns of x, 64 at a time
    const T* a = static_cast<const T*>(g.a) + (int64_t)adapter * g.rank * g.I;
    const T* x0 = static_cast<const T*>(g.x) + (row + gq) * g.ld_x;
    const T* x1 = x0 + 8 * g.ld_x;
    const bool has0 = gq < rows, has1 = gq + 8 < rows;
    float acc[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    const int steps = (g.I + 63) / 64;
    const int step_lo = (int)((int64_t)steps * cta / kAdCluster), step_hi = (int)((int64_t)steps * (cta + 1) / kAdCluster);
    for (int s = step_lo + warp; s < step_hi; s += kAdWarps) {
        const int k = 64 * s + 16 * t, valid = g.I - k;
        Vec16 vx0, vx1, va[kN];
        fetch16(x0 + k, has0 ? valid : 0, g.wide, vx0);
        fetch16(x1 + k, has1 ? valid : 0, g.wide, vx1);
#pragma unroll
        for (int n = 0; n < kN; ++n) fetch16(a + (int64_t)(8 * n + gq) * g.I + k, 8 * n + gq < g.rank ? valid : 0, g.wide, va[n]);
#pragma unroll
        for (int p = 0; p < 4; ++p) {   // terms 2 t, 2 t + 1 and 2 t + 8, 2 t + 9 of instruction p: the lane's words 2 p and 2 p + 1
            const uint32_t w[4] = {vx0.w[2 * p], vx1.w[2 * p], vx0.w[2 * p + 1], vx1.w[2 * p + 1]};
#pragma unroll
            for (int n = 0; n < kN; ++n) mma16(acc[n], w, va[n].w[2 * p], va[n].w[2 * p + 1], T());
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
    // Eight lanes add up a row of h from all CTAs, in each CTA (handing it round would cost another meeting).
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    if (threadIdx.x < 8 * kAdTokens) {
        const int m = threadIdx.x >> 3, j = threadIdx.x & 7;
        float v[kN];
        uint32_t most = 0;
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            v[n] = 0.0f;
            if (m < rows) {
#pragma unroll
                for (int c = 0; c < kAdCluster; ++c) v[n] += ld_cluster(map_to_cta(smem_u32(mine + m * kR + 8 * n + j), c));
                if (g.h != nullptr && 8 * n + j < g.rank && cta == 0) g.h[(int64_t)(row + m) * g.rank + 8 * n + j] = v[n];
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
    __syncwarp();
    cluster_sync_all();   // nobody leaves, and nobody's h is read, before the partial sums have been fetched
    if (g.out == nullptr) return;
    const float back0 = kHalf ? factor[gq] : 1.0f, back1 = kHalf ? factor[gq + 8] : 1.0f;
    for (int group = group_lo + warp; group < group_hi; group += kAdWarps) {
        const int col = 64 * group, valid = g.O - col - 8 * gq, c = col + 16 * t;
        float d[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[j][i] = 0.0f;
#pragma unroll
        for (int k16 = 0; k16 < kK16; ++k16) {
            uint32_t hi[4], lo[4], r[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 16 * k16 + 2 * t + (i & 1) + 8 * (i >> 1);
                r[i][0] = r[i][1] = r[i][2] = r[i][3] = 0;
                if (k < g.rank && valid > 0) ld_vec(b + (int64_t)k * g.O + col + 8 * gq, r[i]);
            }
            h_parts<T, kR>(hs + gq * kRow, hs + (gq + 8) * kRow, k16, t, hi, lo);
            mma_ranks<T>(d, hi, lo, r);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int m = gq + 8 * half;
            if (m >= rows) continue;
            Vec16 old;
            fetch16(base + m * g.ld_base + c, g.O - c, g.wide, old);
            add_row<T>(old.w, d, half, half ? back1 : back0, out + m * g.ld_out + c, g.O - c, g.wide);
        }
    }
}

// Long runs: 128 tokens a tile, a warp for each 16 of them, and a cluster of one to eight CTAs that share x's columns and then the
// output's.  Both products walk over 64 columns at a time, whose 128 rows (of x, then of base) and weights come through a ring of
// stages in shared memory (cp.async; the second product's first stages are under way while the cluster adds up h).  Rows are kStride bytes
// apart in a stage: the eight lanes of an access meet no bank twice.  Each CTA adds up its share of h's rows and hands them to the
// others: all of them everywhere would be 128 rows times the cluster.
constexpr int kTileTokens = 128, kStride = 144;
template <int kN> constexpr int kTileThreads = kN <= 4 ? 256 : 512;   // ranks above 32: two warps for each 16 tokens, half of the ranks, then of the columns each
template <int kN> constexpr int kTileStages = kN <= 2 ? 4 : kN <= 4 ? 3 : kN <= 8 ? 5 : 2;   // what fits two blocks to an SM (to rank 32), or one

template <typename T, int kN>
__global__ void __launch_bounds__(kTileThreads<kN>, kN <= 4 ? 2 : 1) adapter_tile_kernel(const __grid_constant__ AdapterArgs g) {
    constexpr int kThreads = kTileThreads<kN>, kHalves = kThreads / kAdThreads, kOwn = kN / kHalves;   // blocks of ranks of a warp's first product
    constexpr int kR = 8 * kN, kRow = kR + 4, kK16 = (kN + 1) / 2, kStage = (kTileTokens + kR) * kStride;
    constexpr int kStages = kTileStages<kN>;
    constexpr bool kHalf = IsHalf<T>::value;
    extern __shared__ __align__(16) uint8_t ring[];
    float* mine = reinterpret_cast<float*>(ring + kStages * kStage);   // [128][kR], read by the other CTAs
    float* hs = mine + kTileTokens * kR;                               // [128][kRow]
    float* factor = hs + kTileTokens * kRow;                           // [128], of fp16 rows
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 7, part = threadIdx.x >> 8, gq = lane >> 2, t = lane & 3;
    const int cta = (int)cluster_ctarank(), ctas = g.ctas;
    int row, rows, adapter;
    if (!run_of_tile<kTileTokens>(g, blockIdx.x / ctas, row, rows, adapter)) return;   // (all CTAs of the cluster)
    const int groups = (g.O + 63) / 64, steps = (g.I + 63) / 64;
    const int group_lo = (int)((int64_t)groups * cta / ctas), group_hi = (int)((int64_t)groups * (cta + 1) / ctas);
    const int step_lo = (int)((int64_t)steps * cta / ctas), n1 = (int)((int64_t)steps * (cta + 1) / ctas) - step_lo;
    const T* base = static_cast<const T*>(g.base) + row * g.ld_base;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {
        copy_rows(g, base, out, rows, 64 * group_lo, 64 * group_hi);
        return;
    }
    const T* x = static_cast<const T*>(g.x) + row * g.ld_x;
    const T* a = static_cast<const T*>(g.a) + (int64_t)adapter * g.rank * g.I;
    const T* b = static_cast<const T*>(g.b) + (int64_t)adapter * g.rank * g.O;
    const int n2 = g.out != nullptr ? group_hi - group_lo : 0, all = n1 + n2;

    // Step i's 64 columns: eight threads a row of 128 bytes.  What does not exist (rows behind the run or the rank, columns behind the
    // matrix) is zeros.
    auto fetch = [&](int i) {
        if (i < all) {
            const bool second = i >= n1;
            const int c = 64 * (second ? group_lo + i - n1 : step_lo + i) + 8 * (threadIdx.x & 7), width = second ? g.O : g.I;
            const T* left = second ? base : x;
            const T* right = second ? b : a;
            const int64_t ld = second ? g.ld_base : g.ld_x;
            const uint32_t to = smem_u32(ring) + (i % kStages) * kStage + (threadIdx.x >> 3) * kStride + 16 * (threadIdx.x & 7);
#pragma unroll
            for (int q = 0; q < kTileTokens / (kThreads / 8); ++q) {
                const int m = (threadIdx.x >> 3) + kThreads / 8 * q;
                const uint32_t bytes = m < rows && c < width ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + kThreads / 8 * q * kStride), "l"(bytes ? left + m * ld + c : left), "r"(bytes) : "memory");
            }
#pragma unroll
            for (int q = 0; q < (kR + kThreads / 8 - 1) / (kThreads / 8); ++q) {
                const int k = (threadIdx.x >> 3) + kThreads / 8 * q;
                const uint32_t bytes = k < g.rank && c < width ? 16 : 0;
                if (k < kR)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (kTileTokens + kThreads / 8 * q) * kStride), "l"(bytes ? right + (int64_t)k * width + c : right),
                                 "r"(bytes) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // Step i's stage, once it has come for all threads; the one behind the ring's end is then on its way.
    auto stage = [&](int i) -> const uint8_t* {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();   // (all warps have left the stage that is filled next)
        fetch(i + kStages - 1);
        return ring + (i % kStages) * kStage;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i);

    const int m0 = 16 * warp + gq, m1 = m0 + 8;
    float acc[kOwn][4];
#pragma unroll
    for (int n = 0; n < kOwn; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] = 0.0f;
    for (int i = 0; i < n1; ++i) {
        const uint8_t* s = stage(i) + 32 * t;
        uint4 v[4];
        v[0] = *reinterpret_cast<const uint4*>(s + m0 * kStride);
        v[1] = *reinterpret_cast<const uint4*>(s + m0 * kStride + 16);
        v[2] = *reinterpret_cast<const uint4*>(s + m1 * kStride);
        v[3] = *reinterpret_cast<const uint4*>(s + m1 * kStride + 16);
        const uint32_t w[4][4] = {{v[0].x, v[2].x, v[0].y, v[2].y}, {v[0].z, v[2].z, v[0].w, v[2].w}, {v[1].x, v[3].x, v[1].y, v[3].y}, {v[1].z, v[3].z, v[1].w, v[3].w}};
#pragma unroll
        for (int n = 0; n < kOwn; ++n) {
            const uint8_t* own = s + (kTileTokens + 8 * (kOwn * part + n) + gq) * kStride;
            const uint4 q0 = *reinterpret_cast<const uint4*>(own), q1 = *reinterpret_cast<const uint4*>(own + 16);
            float sum[4] = {};   // (the tensor core's own sums are cut off, not rounded: a step's are added up in fp32)
            mma16(sum, w[0], q0.x, q0.y, T());
            mma16(sum, w[1], q0.z, q0.w, T());
            mma16(sum, w[2], q1.x, q1.y, T());
            mma16(sum, w[3], q1.z, q1.w, T());
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[n][q] += sum[q];
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
            if (g.h != nullptr && m < last && m < rows && 8 * n + j < g.rank) g.h[(int64_t)(row + m) * g.rank + 8 * n + j] = v[n];
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
    __syncwarp();
    cluster_sync_all();   // nobody leaves before the partial sums have been fetched, nobody goes on before h is there
    if (n2 == 0) return;

    // A warp's columns: 64 of a step, or 32 where two warps share them (a lane then takes 8 bytes of each rank and 8 columns of the output).
    constexpr int kCols = 8 / kHalves;
    uint32_t hi[kK16][4], lo[kK16][4];
#pragma unroll
    for (int k = 0; k < kK16; ++k) h_parts<T, kR>(hs + m0 * kRow, hs + m1 * kRow, k, t, hi[k], lo[k]);
    const float back0 = kHalf ? factor[m0] : 1.0f, back1 = kHalf ? factor[m1] : 1.0f;
    for (int i = n1; i < all; ++i) {
        const uint8_t* s = stage(i);
        float d[kCols][4];
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) d[j][q] = 0.0f;
#pragma unroll
        for (int k = 0; k < kK16; ++k) {
            uint32_t r[4][kCols / 2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int rank = 16 * k + 2 * t + (q & 1) + 8 * (q >> 1);
                ld_words(s + (kTileTokens + min(rank, kR - 1)) * kStride + 64 * part + 2 * kCols * gq, r[q]);   // (ranks of 8: h's second half is zeros)
            }
            mma_ranks<T>(d, hi[k], lo[k], r);
        }
        const int c = 64 * (group_lo + i - n1) + 32 * part + 2 * kCols * t;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int m = half ? m1 : m0;
            if (m >= rows) continue;
            uint32_t old[kCols];
            ld_words(s + m * kStride + 64 * part + 4 * kCols * t, old);
            add_row<T>(old, d, half, half ? back1 : back0, out + m * g.ld_out + c, g.O - c, g.wide);
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
    int ctas;                 // of a cluster (adapter_grad16_kernel)
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

// The same for bf16 and fp16 rows that begin on 16 bytes.  A cluster takes 128 columns and up to 64 ranks; its CTAs take 64 tokens at a
// time in turn, z's rows and f's through a ring of stages in shared memory.  The warps of a CTA share a stage's tokens and columns: f is
// split into three bf16 or two fp16 numbers (24 or 22 bits: the gradients are fp32) as the fragments are formed, pairs of z's rows are joined as in the second product above.  fp16 holds no
// more than 65504: there f enters times a power of two that brings the largest value of the CTA's tokens to [512, 1024).
// (The tensor core's own sums are cut off, not rounded: those of a stage are added up in fp32.)
constexpr int kAgTokens = 64, kAgCols = 128, kAgStride = 2 * kAgCols + 16;
template <int kR16> constexpr int kAgStages = kR16 <= 2 ? 4 : 3;

// The 64-token pieces of an adapter's runs that one CTA takes: every `ctas`-th of them.
struct Pieces {
    int run, lo, hi, skip;   // of the current run: what is left of it; pieces to pass over
    bool there;
    __device__ __forceinline__ Pieces(const AdapterGradArgs& g, int adapter, int cta) : run(-1), lo(0), hi(0), skip(cta), there(true) { settle(g, adapter); }
    __device__ __forceinline__ void settle(const AdapterGradArgs& g, int adapter) {
        for (;;) {
            const int have = (hi - lo + kAgTokens - 1) / kAgTokens;
            if (skip < have) { lo += skip * kAgTokens; return; }
            skip -= have;
            do {
                if (++run >= g.runs) { there = false; return; }
            } while (g.offsets != nullptr && g.index[run] != adapter);
            lo = 0;
            hi = (int)g.M;
            if (g.offsets != nullptr) run_range(g.offsets, run, g.M, lo, hi);
        }
    }
    __device__ __forceinline__ void next(const AdapterGradArgs& g, int adapter, int ctas) {
        skip = ctas;
        settle(g, adapter);
    }
};

template <typename T, typename G, int kR16>
__global__ void __launch_bounds__(kAdThreads, 2) adapter_grad16_kernel(const __grid_constant__ AdapterGradArgs g) {
    constexpr int kR = 16 * kR16, kRow = kR + 4, kNt = kR16 <= 2 ? 8 : 4;      // kNt: a warp's instructions along the columns
    constexpr int kAcross = kAgCols / (8 * kNt), kAlong = kAdWarps / kAcross;  // warps along the columns, along the tokens
    constexpr int kStage = kAgTokens * (kAgStride + 4 * kRow), kStages = kAgStages<kR16>;
    constexpr bool kHalf = IsHalf<T>::value;
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

    float factor = 1.0f;
    if (kHalf) {
        uint32_t most = 0;
        for (Pieces p(g, adapter, cta); p.there; p.next(g, adapter, ctas)) {
            const int n = min(kAgTokens, p.hi - p.lo) * ranks;
            for (int i = threadIdx.x; i < n; i += kAdThreads) most = max(most, abs_bits(f[(int64_t)(p.lo + i / ranks) * g.rank + i % ranks]));
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if (lane == 0) most_of[warp] = most;
        __syncthreads();
        factor = row_factor(__reduce_max_sync(0xFFFFFFFFu, most_of[lane & 7]));
    }

    Pieces ahead(g, adapter, cta);   // the piece that is fetched next
    int slot = 0;
    auto fetch = [&]() {
        if (ahead.there) {
            const uint32_t to = smem_u32(ring) + slot * kStage;
#pragma unroll
            for (int q = 0; q < kAgTokens / 16; ++q) {
                const int m = (threadIdx.x >> 4) + 16 * q, c = 8 * (threadIdx.x & 15);
                const uint32_t bytes = ahead.lo + m < ahead.hi && col + c < cols ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + m * kAgStride + 2 * c), "l"(bytes ? z + (int64_t)(ahead.lo + m) * ld + c : z), "r"(bytes) : "memory");
            }
#pragma unroll
            for (int q = 0; q < kAgTokens * kR / kAdThreads; ++q) {
                const int i = threadIdx.x + kAdThreads * q, m = i / kR, k = i % kR;
                const uint32_t bytes = ahead.lo + m < ahead.hi && k < ranks ? 4 : 0;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + kAgTokens * kAgStride + 4 * (m * kRow + k)), "l"(bytes ? f + (int64_t)(ahead.lo + m) * g.rank + k : f),
                             "r"(bytes) : "memory");
            }
            ahead.next(g, adapter, ctas);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot = slot + 1 == kStages ? 0 : slot + 1;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch();

    float acc[kR16][kNt][4];
#pragma unroll
    for (int n = 0; n < kR16; ++n)
#pragma unroll
        for (int j = 0; j < kNt; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][j][i] = 0.0f;
    int at = 0;
    for (Pieces p(g, adapter, cta); p.there; p.next(g, adapter, ctas)) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncthreads();   // (all warps have left the stage that is filled next)
        fetch();
        const uint8_t* s = ring + at * kStage;
        const float* fs = reinterpret_cast<const float*>(s + kAgTokens * kAgStride);
        at = at + 1 == kStages ? 0 : at + 1;
        uint32_t r[4 / kAlong][4][kNt / 2];
#pragma unroll
        for (int h = 0; h < 4 / kAlong; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                ld_words(s + (16 * (along + kAlong * h) + 2 * t + (q & 1) + 8 * (q >> 1)) * kAgStride + 16 * kNt * across + 2 * kNt * gq, r[h][q]);
#pragma unroll
        for (int n = 0; n < kR16; ++n) {
            float sum[kNt][4];
#pragma unroll
            for (int j = 0; j < kNt; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j][i] = 0.0f;
#pragma unroll
            for (int h = 0; h < 4 / kAlong; ++h) {
                uint32_t hi[4], lo[4], rest[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // ranks g and g + 8 at the first pair of tokens, then at the second
                    const float* v = fs + (16 * (along + kAlong * h) + 2 * t + 8 * (i >> 1)) * kRow + 16 * n + gq + 8 * (i & 1);
                    if (kHalf) split16<T>(v[0] * factor, v[kRow] * factor, hi[i], lo[i]);
                    else split_three(v[0], v[kRow], hi[i], lo[i], rest[i]);
                }
                mma_ranks<T, kNt, !kHalf>(sum, hi, lo, r[h], rest);
            }
#pragma unroll
            for (int j = 0; j < kNt; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n][j][i] += sum[j][i];
        }
    }
    // The warps' sums over their tokens meet in the ring's place, one after the other, then the CTAs'.
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float* mine = reinterpret_cast<float*>(ring);   // [kR][128]
    const float back = 1.0f / factor;
    for (int w = 0; w < kAlong; ++w) {
        __syncthreads();
        if (along != w) continue;
#pragma unroll
        for (int n = 0; n < kR16; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // instruction j's columns 2 t and 2 t + 1 are 2 kNt t + j and 2 kNt t + kNt + j
                float* to = mine + (16 * n + gq + 8 * (i >> 1)) * kAgCols + 8 * kNt * across + 2 * kNt * t + kNt * (i & 1);
#pragma unroll
                for (int j = 0; j < kNt; ++j) to[j] = (w == 0 ? 0.0f : to[j]) + acc[n][j][i] * back;
            }
    }
    __syncthreads();
    cluster_sync_all();
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    for (int i = cta * kAdThreads + threadIdx.x; i < kR * kAgCols; i += ctas * kAdThreads) {   // each CTA finishes some rows
        const int k = i / kAgCols, c = col + i % kAgCols;
        if (k >= ranks || c >= cols) continue;
        float v = 0.0f;
        for (int p = 0; p < ctas; ++p) v += ld_cluster(map_to_cta(smem_u32(mine + i), p));
        static_cast<G*>(g.out[which])[((int64_t)adapter * g.rank + rank0 + k) * cols + c] = from_f32<G>(v * scale);
    }
    __syncwarp();
    cluster_sync_all();   // nobody leaves before its sums have been fetched
}

// ---------------------------------------------------------------------------------------------- launches
template <typename Args>
static lbt_status cluster_launch(void (*kernel)(Args), const Args& args, dim3 grid, size_t smem, cudaStream_t stream, int ctas = kAdCluster, int threads = kAdThreads) {
    LBT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, args));
    return launch_status();
}

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

template <typename T, int kN>
static lbt_status adapter_launch(const AdapterArgs& g, bool aligned, cudaStream_t stream) {
    // a run of n tokens has at most n / 16 + 1 tiles, and no more than n
    const int64_t tiles = g.offsets == nullptr ? (g.M + kAdTokens - 1) / kAdTokens : std::min<int64_t>(g.M, g.M / kAdTokens + g.runs);
    constexpr size_t smem = sizeof(float) * (kAdWarps * kAdTokens * 8 * kN + kAdTokens * 8 * kN + kAdTokens * (8 * kN + 4));
    const dim3 grid((unsigned)(tiles * kAdCluster));
    return aligned ? cluster_launch(adapter_kernel<T, kN, true>, g, grid, smem, stream) : cluster_launch(adapter_kernel<T, kN, false>, g, grid, smem, stream);
}

template <typename T, int kN>
static lbt_status adapter16_launch(AdapterArgs g, cudaStream_t stream) {
    const int64_t runs = g.offsets == nullptr ? 1 : g.runs;
    constexpr int kR = 8 * kN;
    if (g.M < 48 * runs) {   // 16 tokens a tile where runs are short on average, else 128
        constexpr size_t smem = sizeof(float) * kAdTokens * (kR + kR + 4 + 1 + kAdWarps * kR);
        const int64_t tiles = std::min<int64_t>(g.M, g.M / kAdTokens + runs);
        return cluster_launch(adapter_few_kernel<T, kN>, g, dim3((unsigned)(tiles * kAdCluster)), smem, stream);
    }
    const int64_t tiles = (g.M + (kTileTokens - 1) * runs) / kTileTokens;   // at most
    constexpr size_t smem = kTileStages<kN> * (kTileTokens + kR) * kStride + sizeof(float) * kTileTokens * (kR + kR + 4 + 1);
    // as many CTAs to a cluster as leave all clusters resident at once
    static std::atomic<int> fit[kAdCluster + 1];
    g.ctas = kAdCluster;
    while (g.ctas > 1 && tiles > clusters_fit(adapter_tile_kernel<T, kN>, smem, g.ctas, kTileThreads<kN>, fit)) --g.ctas;
    return cluster_launch(adapter_tile_kernel<T, kN>, g, dim3((unsigned)(tiles * g.ctas)), smem, stream, g.ctas, kTileThreads<kN>);
}

template <typename T>
static lbt_status adapter16(const AdapterArgs& g, cudaStream_t stream) {
    if (g.rank <= 8) return adapter16_launch<T, 1>(g, stream);
    if (g.rank <= 16) return adapter16_launch<T, 2>(g, stream);
    if (g.rank <= 32) return adapter16_launch<T, 4>(g, stream);
    if (g.rank <= 64) return adapter16_launch<T, 8>(g, stream);
    return adapter16_launch<T, 16>(g, stream);
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
static lbt_status adapter_pass(AdapterArgs g, int type, cudaStream_t stream) {
    auto ok = [&](const void* p) { return (reinterpret_cast<uintptr_t>(p) & (8 * type_size(type) - 1)) == 0; };
    const bool aligned = g.I % 8 == 0 && g.O % 8 == 0 && g.ld_x % 8 == 0 && g.ld_base % 8 == 0 && g.ld_out % 8 == 0 && ok(g.x) && ok(g.a) && ok(g.b) &&
                         ok(g.base) && ok(g.out);
    if (type == LBT_F32) return adapter_run<float>(g, aligned, stream);
    if (aligned) {
        auto wide = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; };
        g.wide = g.I % 16 == 0 && g.O % 16 == 0 && g.ld_x % 16 == 0 && g.ld_base % 16 == 0 && g.ld_out % 16 == 0 && wide(g.x) && wide(g.a) && wide(g.base) && wide(g.out);
        return type == LBT_BF16 ? adapter16<__nv_bfloat16>(g, stream) : adapter16<__half>(g, stream);
    }
    return type == LBT_BF16 ? adapter_run<__nv_bfloat16>(g, aligned, stream) : adapter_run<__half>(g, aligned, stream);
}

template <typename T, typename G>
static lbt_status adapter_grad_launch(const AdapterGradArgs& g, bool aligned, cudaStream_t stream) {
    constexpr size_t smem = sizeof(float) * (kAdWarps + 1) * kAgRanks * 64;
    const dim3 grid((g.groups[0] + g.groups[1]) * kAdCluster, g.adapters, (g.rank + kAgRanks - 1) / kAgRanks);
    return aligned ? cluster_launch(adapter_grad_kernel<T, G, true>, g, grid, smem, stream)
                   : cluster_launch(adapter_grad_kernel<T, G, false>, g, grid, smem, stream);
}

template <typename T, typename G, int kR16>
static lbt_status adapter_grad16_launch(AdapterGradArgs g, cudaStream_t stream) {
    constexpr int kR = 16 * kR16;
    for (int i = 0; i < 2; ++i) g.groups[i] = g.groups[i] > 0 ? (g.cols[i] + kAgCols - 1) / kAgCols : 0;
    const int64_t blocks = (int64_t)(g.groups[0] + g.groups[1]) * g.adapters * ((g.rank + kR - 1) / kR);
    // two CTAs to an SM, and two pieces of 64 tokens for each
    g.ctas = (int)std::max<int64_t>(1, std::min<int64_t>({kAdCluster, 2 * kNumSMs / blocks, g.M / (2 * kAgTokens * std::max(1, std::min(g.adapters, g.runs)))}));
    constexpr size_t smem = (size_t)kAgStages<kR16> * kAgTokens * (kAgStride + 4 * (kR + 4));
    static_assert(smem >= sizeof(float) * kR * kAgCols, "the sums take the ring's place");
    const dim3 grid((g.groups[0] + g.groups[1]) * g.ctas, g.adapters, (g.rank + kR - 1) / kR);
    return cluster_launch(adapter_grad16_kernel<T, G, kR16>, g, grid, smem, stream, g.ctas);
}

template <typename T, typename G>
static lbt_status adapter_grad16(const AdapterGradArgs& g, cudaStream_t stream) {
    if (g.rank <= 16) return adapter_grad16_launch<T, G, 1>(g, stream);
    if (g.rank <= 32) return adapter_grad16_launch<T, G, 2>(g, stream);
    return adapter_grad16_launch<T, G, 4>(g, stream);
}

template <typename T>
static lbt_status adapter_grads(const AdapterGradArgs& g, bool aligned, int grad_type, cudaStream_t stream) {
    if constexpr (!IsF32<T>::value)
        if (aligned) return grad_type == LBT_F32 ? adapter_grad16<T, float>(g, stream) : adapter_grad16<T, T>(g, stream);
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
