// What the kernels of the low-rank adapters share: how tiles find their runs, fragments of the matrix instructions, numbers split into
// parts that those hold, rows that begin anywhere, cluster launches.
#pragma once

#include <type_traits>

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
    int32_t* status;   // device status word (null: none)
    uint64_t limit_ns = 2000000000ull;   // after which an on-chip wait gives up (adapter_tc_kernel)
    int mute = -1;     // the CTA of each cluster whose first product is never said to be done (self-test)
    int ctas;     // of a cluster
    bool wide;    // rows of x, a, base and out begin on 32 bytes
};

// Run r's tokens [lo, hi), cut to [0, M) whatever the offsets hold.
__device__ __forceinline__ void run_range(const int32_t* offsets, int r, int64_t M, int& lo, int& hi) {
    const int end = (int)M;
    lo = min(max(offsets[r], 0), end);
    hi = max(min(offsets[r + 1], end), lo);
}

// The run that holds a tile, by all lanes of a warp together: first token, tokens of the tile, adapter.
__device__ __forceinline__ bool run_of_tile(const AdapterArgs& g, int tokens, int tile, int& row, int& rows, int& adapter) {
    if (g.offsets == nullptr) {
        row = tile * tokens;
        rows = (int)min((int64_t)tokens, g.M - row);
        adapter = 0;
        return rows > 0;
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int r0 = 0; r0 < g.runs; r0 += 32) {
        int lo = 0, hi = 0;
        if (r0 + lane < g.runs) run_range(g.offsets, r0 + lane, g.M, lo, hi);
        const int tiles = (hi - lo + tokens - 1) / tokens;
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
            row = __shfl_sync(0xFFFFFFFFu, lo, src) + at * tokens;
            rows = min(tokens, __shfl_sync(0xFFFFFFFFu, hi, src) - row);
            adapter = g.index[r0 + src];
            return true;
        }
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    return false;
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
    if (kSplitB) {   // (the instruction cuts the second part to tf32 itself; an infinity ends as NaN)
        asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(h0) : "f"(b0));
        asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(h1) : "f"(b1));
        l0 = __float_as_uint(b0 - __uint_as_float(h0));
        l1 = __float_as_uint(b1 - __uint_as_float(h1));
    }
    mma_tf32(d, lo[0], lo[1], lo[2], lo[3], h0, h1);
    if (kSplitB) mma_tf32(d, hi[0], hi[1], hi[2], hi[3], l0, l1);
    mma_tf32(d, hi[0], hi[1], hi[2], hi[3], h0, h1);
}

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void st_cluster2(uint32_t addr, uint2 v) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
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
// base += d for a row's 2 kCols columns of the lane (columns 2 j and 2 j + 1 of them: instructions' columns 2 t and 2 t + 1), as they are stored.
template <typename T, int kCols, int kWords>
__device__ __forceinline__ void add_words(uint32_t (&old)[kWords], const float (&d)[kCols][4], int half, float back) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 2 * kCols; ++j) old[j] = __float_as_uint(__uint_as_float(old[j]) + d[j % kCols][2 * half + j / kCols]);
    } else {
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            const float2 o = values16(old[j], T());
            const int q = 2 * j / kCols, i = 2 * j % kCols;
            const float e0 = d[i][2 * half + q], e1 = d[i + 1][2 * half + q];
            old[j] = IsHalf<T>::value ? pair16<T>(fmaf(e0, back, o.x), fmaf(e1, back, o.y)) : pair16<T>(o.x + e0, o.y + e1);
        }
    }
}
// kWords words of a row whose first 16 bytes begin on 16 bytes; `valid` elements exist (multiples of 16 bytes do)
template <typename T, int kWords> __device__ __forceinline__ void st_row(T* to, const uint32_t (&w)[kWords], int valid, bool wide) {
    constexpr int kEach = 16 / (int)sizeof(T);
    if constexpr (kWords == 8) {
        if (wide && valid > kEach) {
            st_vec(to, w);
            return;
        }
        if (valid > kEach) *reinterpret_cast<uint4*>(to + kEach) = make_uint4(w[4], w[5], w[6], w[7]);
    }
    if (valid > 0) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}
// out = base for the tokens of a run without an adapter, columns [lo, hi): eight loads of a lane are on their way at a time.
template <typename T, bool kWords> __device__ __forceinline__ void copy_rows(const AdapterArgs& g, const T* base, T* out, int rows, int lo, int hi, int warps) {
    if (g.out == nullptr || g.out == g.base) return;
    using V = std::conditional_t<kWords, T, uint4>;
    constexpr int kEach = sizeof(V) / sizeof(T), kDeep = 8;
    const int n = (max(min(hi, g.O) - lo, 0) + 32 * kEach - 1) / (32 * kEach), all = rows * n, end = min(hi, g.O);   // a warp takes 32 lanes' columns of a row
    for (int i0 = threadIdx.x >> 5; i0 < all; i0 += kDeep * warps) {
        V v[kDeep];
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
            const int i = i0 + q * warps, m = i / n, c = lo + kEach * (32 * (i - m * n) + (threadIdx.x & 31));
            if (i < all && c < end) v[q] = *reinterpret_cast<const V*>(base + m * g.ld_base + c);
        }
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
            const int i = i0 + q * warps, m = i / n, c = lo + kEach * (32 * (i - m * n) + (threadIdx.x & 31));
            if (i < all && c < end) *reinterpret_cast<V*>(out + m * g.ld_out + c) = v[q];
        }
    }
}

// ---------------------------------------------------------------------------------------------- rows that begin anywhere
// Rows that do not begin on 16 bytes are copied into shared memory by 4-byte words.  A 16-bit row that begins in the middle of a word
// arrives one element late (its first word holds the element ahead of it too); the fragments are shifted back as they are read.
template <typename T> __device__ __forceinline__ bool begins_odd(const T* p) { return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 2) != 0; }

// Word w of the row at p (n elements exist, 0 at least) to `to` in shared memory; begin: the tensor's first element, ahead of which nothing is read.
template <typename T> __device__ __forceinline__ void copy_word(uint32_t to, const T* p, int w, int n, const T* begin) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t bytes = w < n ? 4 : 0;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * w), "l"(bytes ? p + w : begin), "r"(bytes) : "memory");
    } else {
        const int first = 2 * w - (begins_odd(p) ? 1 : 0);   // of the word's two elements
        if (first < 0 && p == begin) {
            const uint32_t v = n > 0 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16 : 0u;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(v) : "memory");
            return;
        }
        const uint32_t bytes = n > 0 ? (uint32_t)min(max(2 * (n - first), 0), 4) : 0u;
        const uint8_t* from = bytes ? reinterpret_cast<const uint8_t*>(p + first) : reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(begin) & ~(uintptr_t)3);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * w), "l"(from), "r"(bytes) : "memory");
    }
}

// Rows p, p + step, .. (count of them, n elements each) to `to`, to + to_step, .., by a warp, a word a lane and block of 32 words.
template <typename T, int kBlocks>
__device__ __forceinline__ void copy_words(uint32_t to, uint32_t to_step, const T* p, int64_t step, int count, int n, const T* begin) {
    const int lane = threadIdx.x & 31;
    if (begins_odd(begin)) {   // (the tensor's first row may need care)
        for (int r = 0; r < count; ++r, p += step, to += to_step)
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) copy_word(to, p, lane + 32 * k, n, begin);
        return;
    }
    uint32_t even[kBlocks], odd[kBlocks];   // bytes that exist of this lane's words
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
        const int w = lane + 32 * k;
        even[k] = sizeof(T) == 4 ? (w < n ? 4 : 0) : min(max(2 * (n - 2 * w), 0), 4);
        odd[k] = min(max(2 * (n - 2 * w + 1), 0), 4);
    }
    to += 4 * lane;
#pragma unroll 4
    for (int r = 0; r < count; ++r, p += step, to += to_step) {
        const uint8_t* from = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3) + 4 * lane;
        const bool late = begins_odd(p);
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 128 * k), "l"(from + 128 * k), "r"(late ? odd[k] : even[k]) : "memory");
    }
}

// 16 bytes of a row, `bytes` (16 or 0) of which exist.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

// kWords words of a row at p in shared memory, one element further on where the row began odd.
template <int kWords> __device__ __forceinline__ void ld_shifted(const uint8_t* p, bool odd, uint32_t (&w)[kWords]) {
    ld_words(p, w);
    const uint32_t more = *reinterpret_cast<const uint32_t*>(p + 4 * kWords), sel = odd ? 0x5432u : 0x3210u;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = __byte_perm(w[i], i + 1 < kWords ? w[i + 1] : more, sel);
}
template <typename T, bool kShift, int kWords> __device__ __forceinline__ void ld_row(const uint8_t* p, bool odd, uint32_t (&w)[kWords]) {
    if constexpr (kShift && sizeof(T) == 2) ld_shifted(p, odd, w);
    else ld_words(p, w);
}

// acc += the products of a lane's 32 bytes of two rows (v0, v1) and of a row of the other operand (w), with the other lanes' (the tensor
// core's own sums are cut off, not rounded: they are added to acc in fp32).
template <typename T> __device__ __forceinline__ void mma_step(float (&acc)[4], const uint32_t (&v0)[8], const uint32_t (&v1)[8], const uint32_t (&w)[8]) {
    float sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = 0.0f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if constexpr (sizeof(T) == 4) {   // terms t and t + 4 of instruction p: the lane's elements 2 p and 2 p + 1
            uint32_t hi[4], lo[4];
            split(__uint_as_float(v0[2 * p]), hi[0], lo[0]); split(__uint_as_float(v1[2 * p]), hi[1], lo[1]);
            split(__uint_as_float(v0[2 * p + 1]), hi[2], lo[2]); split(__uint_as_float(v1[2 * p + 1]), hi[3], lo[3]);
            mma_split<true>(sum, hi, lo, __uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
        } else {                          // terms 2 t, 2 t + 1 and 2 t + 8, 2 t + 9: the lane's words 2 p and 2 p + 1
            const uint32_t v[4] = {v0[2 * p], v1[2 * p], v0[2 * p + 1], v1[2 * p + 1]};
            mma16(sum, v, w[2 * p], w[2 * p + 1], T());
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] += sum[q];
}

// Two rows of h as the fragments of the second product: 16-bit types as parts, formed once; fp32 as they lie in shared memory.
template <typename T, int kN> struct RankRows {
    const float *h0, *h1;
    uint32_t hi[sizeof(T) == 4 ? 1 : (kN + 1) / 2][4], lo[sizeof(T) == 4 ? 1 : (kN + 1) / 2][4];
    __device__ __forceinline__ RankRows(const float* h0_, const float* h1_, int t) : h0(h0_), h1(h1_) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int k = 0; k < (kN + 1) / 2; ++k) h_parts<T, 8 * kN>(h0, h1, k, t, hi[k], lo[k]);
        }
    }
};

// d = h B for two rows of h and 8 kCols columns of the weights' rows at b (144 bytes apart, `at` bytes in), `ranks` of which exist.
// odd, turns: whether the first row of B begins odd, whether every other row then differs.
template <typename T, int kN, int kCols, bool kWords>
__device__ __forceinline__ void rank_product(float (&d)[kCols][4], const RankRows<T, kN>& h, const uint8_t* b, int ranks, int gq, int t, int at, bool odd, bool turns) {
    constexpr int kLine = 144;
#pragma unroll
    for (int j = 0; j < kCols; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) d[j][q] = 0.0f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            uint32_t r0[4] = {}, r1[4] = {}, hi[4], lo[4];
            if (8 * n + t < ranks) ld_words(b + (8 * n + t) * kLine + 16 * gq, r0);
            if (8 * n + t + 4 < ranks) ld_words(b + (8 * n + t + 4) * kLine + 16 * gq, r1);
            split(h.h0[8 * n + t], hi[0], lo[0]); split(h.h1[8 * n + t], hi[1], lo[1]);
            split(h.h0[8 * n + t + 4], hi[2], lo[2]); split(h.h1[8 * n + t + 4], hi[3], lo[3]);
#pragma unroll
            for (int j = 0; j < kCols; ++j) mma_split<true>(d[j], hi, lo, __uint_as_float(r0[j]), __uint_as_float(r1[j]));   // column g of instruction j: 4 g + j
        }
    } else {
#pragma unroll
        for (int k = 0; k < (kN + 1) / 2; ++k) {
            uint32_t r[4][kCols / 2] = {};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int rank = 16 * k + 2 * t + (q & 1) + 8 * (q >> 1);
                if (rank < ranks) ld_row<T, kWords>(b + rank * kLine + at + 2 * kCols * gq, odd != (turns && (rank & 1)), r[q]);
            }
            mma_ranks<T>(d, h.hi[k], h.lo[k], r);
        }
    }
}

template <int kWords> __device__ __forceinline__ void put_words(uint8_t* to, const uint32_t (&w)[kWords]) {
#pragma unroll
    for (int q = 0; q < kWords / 4; ++q) *reinterpret_cast<uint4*>(to + 16 * q) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
}
// The first n of kCount neighbouring elements of up to 16 rows, by a warp, from shared memory (`at` bytes into each row) to rows that begin anywhere.
template <typename T, int kCount> __device__ __forceinline__ void store_rows(T* out, int64_t ld, const uint8_t* rows, int at, int count, int n) {
    const int lane = threadIdx.x & 31;
#pragma unroll 4
    for (int m = 0; m < min(16, count); ++m)
#pragma unroll
        for (int e = 0; e < kCount; e += 32)
            if (e + lane < n) out[m * ld + e + lane] = *reinterpret_cast<const T*>(rows + m * 144 + at + (e + lane) * (int)sizeof(T));
}

// Long runs of 16-bit rows that begin on 16 bytes (lbt_adapters_tc.cu).
lbt_status adapter_tc(const AdapterArgs& g, int type, cudaStream_t stream);

struct AdapterGradArgs {
    const float* f[2];     // [M, rank]: dh for da, h for db
    const void* z[2];      // x, dy
    void* out[2];          // da, db (null: not wanted)
    int64_t ld[2];
    int cols[2], groups[2];   // I, O; blocks of columns (0 where not wanted)
    bool wanted[2];
    const float* scale;
    const int32_t* offsets;
    const int32_t* index;
    int64_t M;
    int runs, adapters, rank;
    int ctas;                 // of a cluster
};
// aligned: rows of both z begin on 16 bytes (lbt_adapter_grads.cu)
lbt_status adapter_grads(AdapterGradArgs g, int type, int grad_type, bool aligned, cudaStream_t stream);

template <typename Args>
inline lbt_status cluster_launch(void (*kernel)(Args), const Args& args, dim3 grid, size_t smem, cudaStream_t stream, int ctas = kAdCluster, int threads = kAdThreads) {
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

}  // namespace lbt
