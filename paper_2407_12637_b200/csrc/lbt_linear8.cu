// Linear layer on 8-bit integers with a scale for each token and channel.
//
//   forward   Y[m,o]  = s_x[m] s_w[o] sum_i q_x[m,i] q_w[o,i] + bias[o]
//   backward  dX[m,i] = s_r[m] sum_o q_r[m,o] q_w[o,i]     (q_r, s_r): rows of dY[m,o] s_w[o]
//             dW[o,i] = s_c[o] sum_m q_c[m,o] q_x[m,i]     (q_c, s_c): columns of dY[m,o] s_x[m]
//
// A scale that sits on the reduced index cannot leave the integer sum, so the backward pass multiplies it into dY before
// dY is quantized: all three products are then exact sums of int8 products in int32, scaled once.
//
// Three products, one main loop: C[R, N] = sum_k A B with each operand either K-major ([row][k]) or MN-major ([k][row]);
// both are what TMA writes with the 128-byte swizzle and what a tcgen05 descriptor can name, so nothing is transposed.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <type_traits>

#include "lbt_sm100.cuh"
#include "lbt_types.cuh"

namespace lbt {

using namespace sm100;

namespace {

constexpr int kStep = 128;                       // reduction bytes of one pipeline stage
constexpr int kBox = kStep * 128;                // a 128 x 128-byte operand tile
constexpr uint64_t kLimitNs = 2000000000ull;     // every on-chip wait gives up after 2 s
constexpr int kMaxStages = 8;
constexpr int kRing = 6 * kBox;                  // operand ring of the 128 x 128 kernel: two CTAs fit one SM
constexpr int kPairStages = 6;
constexpr int kPairRing = kPairStages * 2 * kBox;
constexpr int kPairThreads = 320;                // TMA warp, MMA warp, 8 epilogue warps
constexpr int64_t kMaxReduction = 133144;        // 127 * 127 * k < 2^31

enum { kForward = 0, kDgrad = 1, kWgrad = 2 };   // A, B: K-major, K-major | K-major, MN-major | MN-major, MN-major

struct L8Args {
    int mode;
    int tiles_m, tiles_n, total, band;
    int steps;             // reduction steps of 128
    int splits;            // 128 x 128 kernel: CTAs of a cluster that share a tile, a slice of the reduction each
    int swapped;           // 128 x 128 kernel, forward: A = weights (128 channels), B = tokens (mma_n of them)
    int mma_n;             // 128 x 128 kernel: columns of the accumulator
    int stage_bytes, stages;
    int rows, cols;        // of the output as stored
    const float* row_scale;
    const float* col_scale;   // may be null: 1
    const float* bias;        // per column, may be null
    void* out;
    int64_t ldo;
    int out_type;
    int vec, vec4;         // rows of the output begin on 32-byte boundaries; four consecutive elements can be stored at once
    int wait_prev;         // chained behind the kernel that writes the operands
    int lost;              // 128 x 128 kernel: the CTA of each cluster whose first load is never signalled (self-test), -1: none
    uint64_t limit_ns;     // after which an on-chip wait gives up
    int32_t* status;
};

struct Bars {
    uint64_t full[kMaxStages], empty[kMaxStages], tmem_full[2], tmem_empty[2];
    uint32_t tmem_base;
    volatile uint32_t abort;
};

__device__ __forceinline__ bool wait_for(Bars* b, uint64_t* bar, uint32_t parity, const L8Args& a, bool relaxed = false) {
    if (b->abort) return false;
    if (relaxed ? mbar_wait_bounded_relaxed(bar, parity, a.limit_ns) : mbar_wait_bounded(bar, parity, a.limit_ns)) return true;
    b->abort = 1u;
    if (a.status != nullptr) atomicCAS(a.status, (int32_t)LBT_OK, (int32_t)LBT_ERR_TIMEOUT);
    return false;
}

// Tiles are walked in bands of `band` row tiles, rows fastest, so that the CTAs at work share few strips of A and B in L2.
__device__ __forceinline__ void tile_at(const L8Args& a, int t, int& m, int& n) {
    const int per_band = a.band * a.tiles_n;
    const int b = t / per_band, within = t - b * per_band;
    const int rows = min(a.band, a.tiles_m - b * a.band);
    n = within / rows;
    m = b * a.band + (within - n * rows);
}

__device__ __forceinline__ void put_one(const L8Args& a, int64_t row, int64_t col, float f) {
    const int64_t i = row * a.ldo + col;
    if (a.out_type == LBT_BF16) static_cast<__nv_bfloat16*>(a.out)[i] = __float2bfloat16_rn(f);
    else if (a.out_type == LBT_F16) static_cast<__half*>(a.out)[i] = __float2half_rn(f);
    else static_cast<float*>(a.out)[i] = f;
}

__device__ __forceinline__ float finish(int acc, float scale, float bias) { return __fadd_rn(__fmul_rn(__int2float_rn(acc), scale), bias); }

// 32 consecutive columns of one row (lane = row): scale, bias, round, store in 32-byte sectors.  `cs`: this warp's shared copy of the
// columns' scales and biases.
template <typename T>
__device__ __forceinline__ void put_row(const L8Args& a, int64_t row, int c0, const uint32_t (&v)[32], float rs, const float* cs) {
#pragma unroll
    for (int j = 0; j < 32; j += 16) {
        float f[16];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float4 s = *reinterpret_cast<const float4*>(cs + j + e), b = *reinterpret_cast<const float4*>(cs + 32 + j + e);
            f[e] = finish((int)v[j + e], __fmul_rn(rs, s.x), b.x);
            f[e + 1] = finish((int)v[j + e + 1], __fmul_rn(rs, s.y), b.y);
            f[e + 2] = finish((int)v[j + e + 2], __fmul_rn(rs, s.z), b.z);
            f[e + 3] = finish((int)v[j + e + 3], __fmul_rn(rs, s.w), b.w);
        }
        const int c = c0 + j;
        if (row >= a.rows || c >= a.cols) continue;
        T* dst = static_cast<T*>(a.out) + row * a.ldo + c;
        if (c + 16 <= a.cols) {
            Vec8<T> p, q;
            float lo[8], hi[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { lo[i] = f[i]; hi[i] = f[8 + i]; }
            pack(lo, p);
            pack(hi, q);
            if constexpr (sizeof(T) == 2) {
                const uint32_t w[8] = {p.w[0], p.w[1], p.w[2], p.w[3], q.w[0], q.w[1], q.w[2], q.w[3]};
                st_global_cs_v8(dst, w);
            } else {
                st_global_cs_v8(dst, p.w);
                st_global_cs_v8(dst + 8, q.w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < a.cols) dst[i] = from_f32<T>(f[i]);
        }
    }
}

// 32 consecutive columns from c0 of a warp's 32 rows, lane l holding row row0 + l in v.  Rows that begin on 32-byte
// boundaries leave straight from the registers; others are turned round in the warp's 4 KB of shared memory, so that a store covers
// consecutive addresses of one row (a lane's own row in 4-byte stores touched 32 partly written sectors each).
__device__ __forceinline__ void put_block(const L8Args& a, uint32_t* stage, int64_t row0, int c0, const uint32_t (&v)[32], float rs, int lane) {
    if (c0 >= a.cols || row0 >= a.rows) return;   // uniform over the warp
    const int c = c0 + lane;
    const float scale = c < a.cols && a.col_scale != nullptr ? __ldg(a.col_scale + c) : 1.0f;
    const float bias = c < a.cols && a.bias != nullptr ? __ldg(a.bias + c) : 0.0f;
    __syncwarp();
    if (a.vec) {
        float* cs = reinterpret_cast<float*>(stage);
        cs[lane] = scale;
        cs[32 + lane] = bias;
        __syncwarp();
        if (a.out_type == LBT_BF16) put_row<__nv_bfloat16>(a, row0 + lane, c0, v, rs, cs);
        else if (a.out_type == LBT_F16) put_row<__half>(a, row0 + lane, c0, v, rs, cs);
        else put_row<float>(a, row0 + lane, c0, v, rs, cs);
        return;
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) stage[lane * 32 + (j ^ lane)] = v[j];
    __syncwarp();
    const bool live = c < a.cols;
#pragma unroll 4
    for (int r = 0; r < 32; ++r) {
        const float s = __fmul_rn(__shfl_sync(0xFFFFFFFFu, rs, r), scale);
        if (live && row0 + r < a.rows) put_one(a, row0 + r, c, finish((int)stage[r * 32 + (lane ^ r)], s, bias));
    }
}

// ------------------------------------------------------------------------------------------ 128 x 128 tiles
// One tile per CTA, two CTAs per SM (one drains while the other multiplies).  With few tiles a cluster of `splits` CTAs shares a
// tile: each takes a slice of the reduction, leaves its int32 accumulator in shared memory, and finishes a slice of the
// tokens from all of them (integer sums: any order gives the same bits).  The accumulator is parked as [token][channel] whichever
// operand the tokens were, so that a warp finishes a token's 128 channels at a time: one coalesced access to each CTA's part, one
// store of 256 or 512 consecutive bytes, and a short loop (a kernel that runs for a few us waits for its instructions, too).
// 29 tokens 8192 -> 8192: 13 us (weights at HBM's rate 10.2), of which set-up 1.2, exchange and stores 3; 1111 x 2047 -> 1000: 12 us.
// (volatile keeps these behind the cluster's barrier; no memory clobber, so that stores of finished rows do not hold them back)
__device__ __forceinline__ uint4 ld_cluster_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint4 ld_cluster_words(uint32_t addr) {   // four words 128 bytes apart
    uint4 v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v.x) : "r"(addr));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v.y) : "r"(addr + 128));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v.z) : "r"(addr + 256));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v.w) : "r"(addr + 384));
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_word(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
constexpr int kTileWarps = 8;     // the last thousand instructions of a tile are its warps' latency: eight share them (four: +1.4 us)
constexpr int kParkPitch = 132;   // words of a parked row: 16-byte accesses of neighbouring rows without bank conflicts
static_assert(128 * kParkPitch * 4 <= kRing, "the parked accumulator takes the operand ring's place");

// What a warp needs to finish its rows [first + warp, + kTileWarps, ...) of a tile, looked up while the last products run: the scales and
// biases of the lane's four columns (consecutive ones where rows allow it, else every 32nd: neighbouring lanes store to
// neighbouring addresses either way), and the scale of the warp's l-th row in lane l.
struct TileFactors {
    int first, last, c0, step;
    float cs[4], bias[4], rows;
};

__device__ __forceinline__ TileFactors tile_factors(const L8Args& a, int first, int last, int64_t row0, int col0, int warp, int lane) {
    TileFactors f;
    f.first = first; f.last = last;
    f.step = a.vec4 ? 1 : 32;
    f.c0 = col0 + (a.vec4 ? lane * 4 : lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = f.c0 + i * f.step;
        f.cs[i] = c < a.cols && a.col_scale != nullptr ? __ldg(a.col_scale + c) : 1.0f;
        f.bias[i] = c < a.cols && a.bias != nullptr ? __ldg(a.bias + c) : 0.0f;
    }
    const int mine = first + warp + kTileWarps * lane;
    f.rows = mine < last ? a.row_scale[row0 + mine] : 0.0f;
    return f;
}

// Rows of the parked tile -> rows row0 + ... of the output.
template <typename T>
__device__ __forceinline__ void finish_rows(const L8Args& a, const TileFactors& f, const uint32_t* parked, const volatile uint32_t* abort, int64_t row0,
                                            int warp, int lane) {
    const int first = f.first, last = f.last, c0 = f.c0, step = f.step;
    const uint32_t park = smem_u32(parked);
    uint32_t from[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) from[r] = a.splits > 1 ? map_to_cta(park, (uint32_t)min(r, a.splits - 1)) : park;
    T* out = static_cast<T*>(a.out) + row0 * a.ldo;
    uint32_t lost = 0u;                         // whether CTA `lane` of the cluster lost a signal: its part is not there, no row may be stored
    constexpr int kRows = 4;                    // rows whose parts are on their way together
#pragma unroll 1
    for (int i = 0; first + warp + kTileWarps * i < last; i += kRows) {
        int sum[kRows][4] = {};
        auto take = [&](int u, const uint4& v) { sum[u][0] += (int)v.x; sum[u][1] += (int)v.y; sum[u][2] += (int)v.z; sum[u][3] += (int)v.w; };
        uint32_t at[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            at[u] = (uint32_t)((first + warp + kTileWarps * (i + u)) * kParkPitch + (a.vec4 ? lane * 4 : lane)) * 4u;
        }
        const int have = min(kRows, (last - first - warp + kTileWarps - 1) / kTileWarps - i);   // rows left (uniform over the warp)
        if (a.splits == 1) {
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                if (u < have) {
                    const uint32_t* p = parked + at[u] / 4;
                    take(u, a.vec4 ? *reinterpret_cast<const uint4*>(p) : make_uint4(p[0], p[32], p[64], p[96]));
                }
        } else {
            // (loaded and looked at beside the first rows' parts: 0.1 us of 11.5; an abort word pushed to all CTAs and read behind the barrier 0.2)
            if (i == 0 && lane < a.splits) lost = ld_cluster_word(map_to_cta(smem_u32(const_cast<const uint32_t*>(abort)), (uint32_t)lane));
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < a.splits) {
                    uint4 v[kRows];
#pragma unroll
                    for (int u = 0; u < kRows; ++u)
                        if (u < have) v[u] = a.vec4 ? ld_cluster_v4(from[r] + at[u]) : ld_cluster_words(from[r] + at[u]);
#pragma unroll
                    for (int u = 0; u < kRows; ++u)
                        if (u < have) take(u, v[u]);
                }
        }
        if (i == 0 && __any_sync(0xFFFFFFFFu, lost != 0u)) return;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int m = first + warp + kTileWarps * (i + u);
            const float rs = __shfl_sync(0xFFFFFFFFu, f.rows, (i + u) & 31);
            if (u >= have) break;
            alignas(16) T v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = from_f32<T>(finish(sum[u][k], __fmul_rn(rs, f.cs[k]), f.bias[k]));
            T* dst = out + m * a.ldo;
            if (a.vec4 && c0 + 3 < a.cols) {
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst + c0) = *reinterpret_cast<const uint2*>(v);
                else *reinterpret_cast<uint4*>(dst + c0) = *reinterpret_cast<const uint4*>(v);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c0 + k * step < a.cols) dst[c0 + k * step] = v[k];
            }
        }
    }
}

__global__ void __launch_bounds__(kTileWarps * 32, 2)
l8_tile_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ L8Args a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ Bars bars;
    Bars* b = &bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = a.splits > 1 ? (int)cluster_ctarank() : 0;
    int tm, tn;
    tile_at(a, (int)blockIdx.x / a.splits, tm, tn);
    const int per = (a.steps + a.splits - 1) / a.splits;
    const int k0 = split * per, k1 = min(k0 + per, a.steps), n_steps = max(k1 - k0, 0);
    const int m0 = tm * 128, n0 = tn * a.mma_n;
    const bool a_mn = a.mode == kWgrad, b_mn = a.mode != kForward;

    auto load_a = [&](int i, int s) {
        const int k = (k0 + i) * kStep;
        uint8_t* dst = ring + s * a.stage_bytes;
        if (a_mn) tma_load_2d(dst, &tmA, &b->full[s], m0, k); else tma_load_2d(dst, &tmA, &b->full[s], k, m0);
    };
    auto load_b = [&](int i, int s) {
        const int k = (k0 + i) * kStep;
        uint8_t* dst = ring + s * a.stage_bytes + kBox;
        if (b_mn) tma_load_2d(dst, &tmB, &b->full[s], n0, k); else tma_load_2d(dst, &tmB, &b->full[s], k, n0);
    };
    // One operand (weights, or wgrad's token codes) never comes from the kernel ahead: its first loads wait for nothing.
    const int ahead = min(a.stages, n_steps);
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) { mbar_init(&b->full[s], 1); mbar_init(&b->empty[s], 1); }
        mbar_init(&b->tmem_full[0], 1);
        b->abort = 0u;
        fence_mbar_init();
        for (int i = 0; i < ahead; ++i) {
            mbar_arrive_expect_tx(&b->full[i], (uint32_t)a.stage_bytes + (i == 0 && split == a.lost ? 16u : 0u));
            if (a.swapped) load_a(i, i); else load_b(i, i);
        }
    }
    if (warp == 1) { tmem_alloc(&b->tmem_base, 128); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = b->tmem_base;

    if (warp == 0) {
        if (lane == 0) {
            if (a.wait_prev) griddep_wait();
            for (int i = 0; i < ahead; ++i)
                if (a.swapped) load_b(i, i); else load_a(i, i);
            for (int i = ahead; i < n_steps; ++i) {
                const int s = i % a.stages;
                if (!wait_for(b, &b->empty[s], (uint32_t)((i / a.stages) & 1) ^ 1u, a)) break;
                mbar_arrive_expect_tx(&b->full[s], (uint32_t)a.stage_bytes);
                load_a(i, s);
                load_b(i, s);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = idesc_i8(128, a.mma_n, true, true, a_mn, b_mn);
            bool ok = true;
            for (int i = 0; i < n_steps && ok; ++i) {
                const int s = i % a.stages;
                ok = wait_for(b, &b->full[s], (uint32_t)(i / a.stages) & 1u, a);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t pa = smem_u32(ring + s * a.stage_bytes), pb = pa + kBox;
                const uint64_t da = a_mn ? smem_desc_sw128(pa, kBox, 1024) : smem_desc_sw128(pa, 16, 1024);
                const uint64_t db = b_mn ? smem_desc_sw128(pb, kBox, 1024) : smem_desc_sw128(pb, 16, 1024);
#pragma unroll
                for (int k = 0; k < kStep / 32; ++k)
                    mma_i8_ss(tmem, da + (uint64_t)(k * (a_mn ? 256 : 2)), db + (uint64_t)(k * (b_mn ? 256 : 2)), idesc, (i > 0 || k > 0) ? 1u : 0u);
                mma_commit(&b->empty[s]);
            }
            if (ok) mma_commit(&b->tmem_full[0]);
        }
        __syncwarp();
    }
    if (a.wait_prev) griddep_wait();   // the scales come from the kernel ahead too, and nothing is written before it has ended
    const int64_t row0 = a.swapped ? n0 : m0;
    const int each = (a.swapped ? a.mma_n : 128) / a.splits;
    const TileFactors factors =
        tile_factors(a, split * each, (int)min((int64_t)(split * each + each), a.rows - row0), row0, a.swapped ? m0 : n0, warp, lane);
    bool ok = true;
    if (n_steps > 0 && warp == 1) ok = wait_for(b, &b->tmem_full[0], 0u, a);   // one warp polls, the others rest at the barrier
    ok = __syncthreads_and(ok) != 0;   // uniform; without it a lost signal ends in the error word and no output of the cluster
    tc_fence_after_sync();
    const int quarter = warp & 3, tmem_lane = quarter * 32 + lane;   // the TMEM lanes a warp may read; warps 4..7 take every other 32 columns
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t* park = reinterpret_cast<uint32_t*>(ring);
#pragma unroll 1
    for (int c = (warp >> 2) * 32; c < a.mma_n && ok; c += 64) {
        uint32_t v[32];
        if (n_steps > 0) {
            tmem_ld_32x32(lanes + (uint32_t)c, v);
            tmem_ld_wait();
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0u;
        }
        if (a.swapped) {   // a lane holds a channel
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c + j < a.mma_n) park[(c + j) * kParkPitch + tmem_lane] = v[j];
        } else {           // a lane holds a token
#pragma unroll
            for (int j = 0; j < 32; j += 4)
                *reinterpret_cast<uint4*>(park + tmem_lane * kParkPitch + c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
    }
    if (a.splits > 1) cluster_sync_all(); else __syncthreads();
    if (ok) {
        if (a.out_type == LBT_BF16) finish_rows<__nv_bfloat16>(a, factors, park, &b->abort, row0, warp, lane);
        else if (a.out_type == LBT_F16) finish_rows<__half>(a, factors, park, &b->abort, row0, warp, lane);
        else finish_rows<float>(a, factors, park, &b->abort, row0, warp, lane);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (b->abort && threadIdx.x == 0) {   // copies in flight land before the CTA's shared memory goes
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 20000000ull) __nanosleep(1000);
    }
    if (a.splits > 1) cluster_sync_all();   // no CTA leaves while another reads its shared memory
    else __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, 128);
}

// ------------------------------------------------------------------------------------------ 256 x 256 tiles, CTA pairs
// Persistent: pair p works on tiles p, p + pairs, ...; two accumulators of 256 TMEM columns let the epilogue of one tile run under
// the main loop of the next.  Each CTA loads its 128 rows of A and its half of B's columns (32 KB a step), rank 0 issues the MMAs
// of both: 8 KB of shared-memory operand reads per SM and MMA instead of the 12 KB a single CTA would need.  Bound by the operands' way
// from L2 and, over seconds, by the power cap: 8192^3 forward 320 us, dgrad 310, wgrad 347 (3.2-3.6 POPS); 2048 x 4096 -> 16384 85 us.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
l8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ L8Args a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ Bars bars;
    Bars* b = &bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const bool a_mn = a.mode == kWgrad, b_mn = a.mode != kForward;

    if (threadIdx.x == 0) {
        prefetch_tensormap(&tmA);
        prefetch_tensormap(&tmB);
        for (int s = 0; s < kPairStages; ++s) { mbar_init(&b->full[s], 1); mbar_init(&b->empty[s], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&b->tmem_full[i], 1); mbar_init(&b->tmem_empty[i], 16); }
        b->abort = 0u;
        fence_mbar_init();
    }
    if (warp == 1) { tmem_alloc_pair(&b->tmem_base, 512); tmem_relinquish_pair(); }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after_sync();
    if (a.wait_prev) griddep_wait();
    const uint32_t tmem = b->tmem_base;

    if (warp == 0) {
        if (elect_one()) {
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int t = pair; t < a.total && ok; t += pairs) {
                int tm, tn;
                tile_at(a, t, tm, tn);
                const int m0 = tm * 256 + (int)rank * 128, n0 = tn * 256 + (int)rank * 128;
                for (int i = 0; i < a.steps; ++i) {
                    ok = wait_for(b, &b->empty[s], ph ^ 1u, a);
                    if (!ok) break;
                    uint8_t* dst = ring + s * 2 * kBox;
                    if (rank == 0) mbar_arrive_expect_tx(&b->full[s], 4u * kBox);   // the bytes of both CTAs
                    const uint32_t full0 = map_to_cta(smem_u32(&b->full[s]), 0);
                    const int k = i * kStep;
                    if (a_mn) tma_load_2d_pair(dst, &tmA, full0, m0, k); else tma_load_2d_pair(dst, &tmA, full0, k, m0);
                    if (b_mn) tma_load_2d_pair(dst + kBox, &tmB, full0, n0, k); else tma_load_2d_pair(dst + kBox, &tmB, full0, k, n0);
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = idesc_i8(256, 256, true, true, a_mn, b_mn);
            const uint32_t base = smem_u32(ring);
            const uint64_t da0 = a_mn ? smem_desc_sw128(base, kBox, 1024) : smem_desc_sw128(base, 16, 1024);
            const uint64_t db0 = b_mn ? smem_desc_sw128(base + kBox, kBox, 1024) : smem_desc_sw128(base + kBox, 16, 1024);
            const uint64_t ka = a_mn ? 256 : 2, kb = b_mn ? 256 : 2;
            int s = 0;
            uint32_t ph = 0, acc = 0;
            bool ok = true;
            for (int t = pair; t < a.total && ok; t += pairs, ++acc) {
                const uint32_t buf = acc & 1u;
                ok = wait_for(b, &b->tmem_empty[buf], ((acc >> 1) & 1u) ^ 1u, a);
                if (!ok) break;
                tc_fence_after_sync();
                for (int i = 0; i < a.steps; ++i) {
                    ok = wait_for(b, &b->full[s], ph, a);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint64_t da = da0 + (uint64_t)(s * (2 * kBox >> 4)), db = db0 + (uint64_t)(s * (2 * kBox >> 4));
#pragma unroll
                    for (int k = 0; k < kStep / 32; ++k)
                        mma_i8_ss_pair(tmem + buf * 256u, da + k * ka, db + k * kb, idesc, (i > 0 || k > 0) ? 1u : 0u);
                    mma_commit_pair(&b->empty[s]);
                    if (++s == kPairStages) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_pair(&b->tmem_full[buf]);
            }
        }
        __syncwarp();
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;   // the TMEM lanes a warp may read; half of the columns each
        uint32_t* stage = reinterpret_cast<uint32_t*>(ring + kPairRing + (warp - 2) * 4096);
        uint32_t acc = 0;
        for (int t = pair; t < a.total; t += pairs, ++acc) {
            int tm, tn;
            tile_at(a, t, tm, tn);
            const uint32_t buf = acc & 1u;
            bool ok = wait_for(b, &b->tmem_full[buf], (acc >> 1) & 1u, a, true);
            ok = __all_sync(0xFFFFFFFFu, ok) != 0;
            if (!ok) break;
            tc_fence_after_sync();
            const int64_t row = (int64_t)tm * 256 + rank * 128 + quarter * 32 + lane;
            const float rs = row < a.rows ? a.row_scale[row] : 0.0f;
            for (int c = half * 128; c < half * 128 + 128; c += 32) {
                uint32_t v[32];
                tmem_ld_32x32(tmem + buf * 256u + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c, v);
                tmem_ld_wait();
                put_block(a, stage, row - lane, tn * 256 + c, v, rs, lane);
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_relaxed(map_to_cta(smem_u32(&b->tmem_empty[buf]), 0));
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (b->abort && threadIdx.x == 0) {
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 20000000ull) __nanosleep(1000);
    }
    cluster_sync_all();
    if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ------------------------------------------------------------------------------------------ quantizers
// Eight consecutive elements [c, c + 8) of a row of `cols`, zeros behind its end.
template <typename T>
__device__ __forceinline__ void load_group(const T* row, int64_t c, int64_t cols, bool vec, float (&f)[8]) {
    if (vec && c + 8 <= cols) {
        load8(row + c, f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
    }
}

__device__ __forceinline__ uint2 codes8(const float (&f)[8], float factor) {
    return make_uint2(pack4(code8(f[0], factor), code8(f[1], factor), code8(f[2], factor), code8(f[3], factor)),
                      pack4(code8(f[4], factor), code8(f[5], factor), code8(f[6], factor), code8(f[7], factor)));
}

// The largest magnitude of eight raw elements as fp32 bits; for 16-bit types two at a time on the bits without their signs (which
// order like the magnitudes, infinities and NaN on top), kept apart until the end of the row.
template <typename T> struct RowMost {
    uint32_t v = 0;
    __device__ __forceinline__ void add(const Vec8<T>& r) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v = max(v, r.w[i] & 0x7FFFFFFFu);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v = __vmaxu2(v, r.w[i] & 0x7FFF7FFFu);
        }
    }
    __device__ __forceinline__ uint32_t bits() const {
        if constexpr (sizeof(T) == 4) return v;
        const uint16_t top = (uint16_t)max(v & 0xFFFFu, v >> 16);
        return __float_as_uint(to_f32(*reinterpret_cast<const T*>(&top))) & 0x7FFFFFFFu;
    }
};

// Eight consecutive elements [c, c + 8) as they are stored, zeros behind the row's end.
template <typename T>
__device__ __forceinline__ void load_raw(const T* row, int64_t c, int64_t cols, bool vec, Vec8<T>& r) {
    if (vec && c + 8 <= cols) {
        ld_vec(row + c, r.w);
    } else {
        float f[8];
        load_group(row, c, cols, false, f);
        pack(f, r);   // (exact: the values came from this type)
    }
}

// Row quantizer: kPerRow threads (a warp or the block of 256) own a row, eight columns at a time; the first four groups of a
// thread stay in registers, as stored, between the maximum and the codes (8192 columns for a block), the rest is read again.
// One reading of the elements and one byte written for each: bound by memory (8192 x 8192: fp32 52 us = 6.4 TB/s, bf16 35 us = 5.8 TB/s).
template <typename T, int kPerRow>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 6 : 4)
rows8_kernel(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld, bool vec, uint8_t* __restrict__ q, int64_t ldq,
             int64_t end, float* __restrict__ scale) {   // end: columns and padding (what lies behind them in a row is not this matrix's)
    constexpr int kHeld = 4;
    griddep_launch_dependents();
    const int64_t row = kPerRow == 256 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int t = kPerRow == 256 ? threadIdx.x : threadIdx.x & 31;
    if (row >= rows) return;
    const T* src = x + row * ld;
    Vec8<T> held[kHeld];
    RowMost<T> top;
#pragma unroll
    for (int g = 0; g < kHeld; ++g) {
        const int64_t c = (int64_t)(g * kPerRow + t) * 8;
        held[g] = Vec8<T>{};
        if (c < cols) load_raw(src, c, cols, vec, held[g]);
    }
#pragma unroll
    for (int g = 0; g < kHeld; ++g) top.add(held[g]);
    for (int64_t c = (int64_t)(kHeld * kPerRow + t) * 8; c < cols; c += kPerRow * 8) {
        Vec8<T> r;
        load_raw(src, c, cols, vec, r);
        top.add(r);
    }
    uint32_t most = __reduce_max_sync(0xFFFFFFFFu, top.bits());
    if (kPerRow == 256) {
        __shared__ uint32_t part[8];
        if ((t & 31) == 0) part[t >> 5] = most;
        __syncthreads();
        most = __reduce_max_sync(0xFFFFFFFFu, part[t & 7]);
    }
    float s, factor;
    scale8(most, s, factor);
    if (t == 0) scale[row] = s;
    uint8_t* dst = q + row * ldq;
#pragma unroll
    for (int g = 0; g < kHeld; ++g) {
        const int64_t c = (int64_t)(g * kPerRow + t) * 8;
        float f[8];
        unpack(held[g], f);
        if (c < end) *reinterpret_cast<uint2*>(dst + c) = codes8(f, factor);
    }
    for (int64_t c = (int64_t)(kHeld * kPerRow + t) * 8; c < end; c += kPerRow * 8) {
        float f[8];
        load_group(src, c, cols, vec, f);
        *reinterpret_cast<uint2*>(dst + c) = codes8(f, factor);
    }
}

// ------------------------------------------------------------------------------------------ few tokens
// A handful of tokens: the time is the weights' way from memory, each byte used once.  A tile is 16 output channels; a block's
// warps take 64-byte pieces of their rows in turn as the fragments of m16n8k32 products (A: channels, B: tokens; the reduction may
// be dealt out in any order as long as both operands agree, so a lane's 16 consecutive bytes are two fragments).  A lane copies its
// own pieces ahead (cp.async, eight of them in flight, on into the block's next tile) into slots that only it reads: no barrier
// but one a tile, where the warps' integer sums meet.  (Refilling registers instead halved the rate: a warp has six scoreboards.)
// With T a type (one token) every block quantizes the token for itself under the first weights' latency: one launch in all.
// One token 4096 -> 4096: 5.3 us (weights at HBM's rate 2.6); 8192 -> 8192: 17 us (10.2); 32768 x 8192: 51 us = 5.4 TB/s.
constexpr int kFewTokens = 16;
constexpr int kFewAhead = 8;               // pieces in flight per lane
constexpr int kFewCodes = 60 * 1024;       // codes of all tokens, kept by each block

struct FewArgs {
    const void* x;
    int64_t ldx;
    bool vec;
    uint8_t* q_x;
    float* s_x;
    const uint8_t* q_w;
    int64_t pitch;
    int I, M, tokens_pitch;   // tokens_pitch: bytes of a token's codes in shared memory, an odd multiple of 64 (no bank conflicts)
    bool wait_prev;
    L8Args out;               // rows, cols, scales, bias, output
};

__device__ __forceinline__ void mma_16832(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T, int kTiles, int kWarps>   // T void: codes come from q_x; kTiles: groups of eight tokens
__global__ void __launch_bounds__(kWarps * 32) l8_few_kernel(const __grid_constant__ FewArgs a) {
    constexpr bool kQuantize = !std::is_void<T>::value;
    constexpr int kThreads = kWarps * 32;
    extern __shared__ uint8_t few_smem[];
    uint8_t* codes = few_smem + kFewAhead * 2 * kThreads * 16;
    __shared__ int sums[2][kWarps][kTiles * 8][17];
    __shared__ float scales[kTiles * 8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tiles = (a.out.cols + 15) / 16;
    const int pieces = ((int)a.pitch + 63) / 64;
    const int mine = warp < pieces ? (pieces - warp + kWarps - 1) / kWarps : 0;   // pieces of a tile that this warp takes
    // what is being fetched: its tile, its piece and this lane's two rows of it
    int f_tile = blockIdx.x, f_piece = 0, f_stage = 0;
    const uint8_t *w0, *w1;
    auto rows_of = [&](int tile) {
        const int64_t o = (int64_t)tile * 16 + g, last = a.out.cols - 1;   // (rows past the last channel repeat it and are not stored)
        w0 = a.q_w + min(o, last) * a.pitch + 64 * warp + 16 * t;
        w1 = a.q_w + min(o + 8, last) * a.pitch + 64 * warp + 16 * t;
    };
    auto slot = [&](int stage, int half) { return few_smem + ((stage * 2 + half) * kThreads + threadIdx.x) * 16; };
    auto fetch = [&]() {
        if (f_tile < tiles && mine > 0) {
            const int k = f_piece * (64 * kWarps);
            // a lane whose 16 bytes lie behind the row's end copies zeros
            const uint32_t bytes = k + 64 * warp + 16 * t < a.pitch ? 16u : 0u;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(slot(f_stage, 0))), "l"(bytes ? w0 + k : a.q_w), "r"(bytes) : "memory");
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(slot(f_stage, 1))), "l"(bytes ? w1 + k : a.q_w), "r"(bytes) : "memory");
            if (++f_piece == mine) {
                f_piece = 0;
                f_tile += gridDim.x;
                rows_of(f_tile);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        f_stage = f_stage + 1 == kFewAhead ? 0 : f_stage + 1;
    };
    rows_of(f_tile);
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i) fetch();
    if constexpr (kQuantize) {
        __shared__ uint32_t part[kWarps];
        const T* row = static_cast<const T*>(a.x);
        uint32_t most = 0;
        for (int c = threadIdx.x * 8; c < a.I; c += kThreads * 8) {
            float f[8];
            load_group(row, c, a.I, a.vec, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, abs_bits(f[i]));
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if (lane == 0) part[warp] = most;
        __syncthreads();
        float scale, factor;
        scale8(__reduce_max_sync(0xFFFFFFFFu, part[lane & (kWarps - 1)]), scale, factor);
        for (int c = threadIdx.x * 8; c < a.tokens_pitch; c += kThreads * 8) {
            float f[8];
            load_group(row, c, a.I, a.vec, f);
            const uint2 q = codes8(f, factor);
            *reinterpret_cast<uint2*>(codes + c) = q;
            if (blockIdx.x == 0 && c < a.pitch) *reinterpret_cast<uint2*>(a.q_x + c) = q;
        }
        if (threadIdx.x == 0) scales[0] = scale;
        if (blockIdx.x == 0 && threadIdx.x == 0) a.s_x[0] = scale;
    } else {
        if (a.wait_prev) griddep_wait();
        const int chunks = (int)(a.tokens_pitch >> 4);
        for (int i = threadIdx.x; i < a.M * chunks; i += kThreads) {
            const int m = i / chunks, c = (i - m * chunks) * 16;
            const uint4 v = c < a.pitch ? *reinterpret_cast<const uint4*>(a.q_x + m * a.pitch + c) : make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(codes + m * a.tokens_pitch + c) = v;
        }
        if (threadIdx.x < a.M) scales[threadIdx.x] = a.s_x[threadIdx.x];
    }
    __syncthreads();
    int turn = 0, stage = 0;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
        int acc[kTiles][4];
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[n][i] = 0;
        for (int i = 0; i < mine; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kFewAhead - 1) : "memory");
            const uint4 lo = *reinterpret_cast<const uint4*>(slot(stage, 0)), hi = *reinterpret_cast<const uint4*>(slot(stage, 1));
            const int k = (i * kWarps + warp) * 64 + 16 * t;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const int m = min(n * 8 + g, a.M - 1);    // (columns past M are not stored)
                const uint4 b = *reinterpret_cast<const uint4*>(codes + m * a.tokens_pitch + k);
                mma_16832(acc[n], lo.x, hi.x, lo.y, hi.y, b.x, b.y);
                mma_16832(acc[n], lo.z, hi.z, lo.w, hi.w, b.z, b.w);
            }
            fetch();
            stage = stage + 1 == kFewAhead ? 0 : stage + 1;
        }
#pragma unroll
        for (int n = 0; n < kTiles; ++n) {
            sums[turn][warp][n * 8 + 2 * t][g] = acc[n][0];
            sums[turn][warp][n * 8 + 2 * t + 1][g] = acc[n][1];
            sums[turn][warp][n * 8 + 2 * t][g + 8] = acc[n][2];
            sums[turn][warp][n * 8 + 2 * t + 1][g + 8] = acc[n][3];
        }
        __syncthreads();
        const int m = threadIdx.x >> 4, r = threadIdx.x & 15;
        const int64_t o = (int64_t)tile * 16 + r;
        if (m < a.M && o < a.out.cols) {
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kWarps; ++i) sum += sums[turn][i][m][r];
            const float bias = a.out.bias != nullptr ? __ldg(a.out.bias + o) : 0.0f;
            put_one(a.out, m, o, __fadd_rn(__fmul_rn(__int2float_rn(sum), __fmul_rn(scales[m], __ldg(a.out.col_scale + o))), bias));
        }
    }
}

// Gradient quantizer, two passes over dY in tiles of 256 columns x 64 rows (a warp owns 256 columns and every eighth row).  First pass:
// the largest |dY s_w| of each row, the largest |dY s_x| of each column (as integers: order-free), and with dbias the column sums of
// each strip.  Second pass, from the last strip back (the first pass left that end in L2): both code matrices and their scales.
// Between memory and instruction issue (0.6-0.7 instructions a cycle and scheduler), so: kEven (aligned rows, O a multiple of 8) has no test per column, the row's scale
// and factor are formed once in a lane and handed round, and columns without a usable scale take a way of their own.  8192 x 8192 bf16:
// 34 us (4.0 TB/s) and 60 us (4.5 TB/s).
constexpr int kStrip = 64;
constexpr int kStripRows = kStrip / 8;   // rows of a warp

// max(m, |a|, |b|) that keeps a NaN
__device__ __forceinline__ float most3(float m, float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

template <typename T, bool kEven, bool kSums>
__global__ void __launch_bounds__(256)
grad8_stats_kernel(const T* __restrict__ dY, int64_t M, int64_t O, int64_t ld, bool vec, const float* __restrict__ s_w,
                   const float* __restrict__ s_x, uint32_t* __restrict__ row_most, uint32_t* __restrict__ col_most, float* __restrict__ sums) {
    __shared__ float most[8][256];
    __shared__ float sum[kSums ? 8 : 1][256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * 256 + lane * 8, m0 = (int64_t)blockIdx.y * kStrip + warp;
    const int rows = (int)min((int64_t)kStripRows, (M - m0 + 7) / 8);   // of this warp (may be <= 0)
    const bool live = c < O;
    float w[8], total[8], cm[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) { w[i] = c + i < O ? s_w[c + i] : 0.0f; total[i] = cm[i] = 0.0f; }
    const float sx_all = lane < rows ? s_x[m0 + 8 * lane] : 0.0f;
    const T* row = dY + m0 * ld;
    // all rows' loads of an aligned strip are on their way before the first is looked at
    Vec8<T> raw[kStripRows];
    if (kEven) {
#pragma unroll
        for (int k = 0; k < kStripRows; ++k) {
            raw[k] = Vec8<T>{};
            if (live && k < rows) ld_vec(row + k * 8 * ld + c, raw[k].w);
        }
    }
#pragma unroll
    for (int k = 0; k < kStripRows; ++k) {
        if (k >= rows) break;   // uniform over the warp
        const float sx = __shfl_sync(0xFFFFFFFFu, sx_all, k);
        float f[8], rm = 0.0f;
        if (kEven) unpack(raw[k], f);
        else load_group(row + k * 8 * ld, c, O, vec, f);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            rm = most3(rm, __fmul_rn(f[i], w[i]), __fmul_rn(f[i + 1], w[i + 1]));
            if (kEven || live) {   // (a lane behind the end: 0 times a NaN scale; its columns are not stored)
                cm[i] = most3(cm[i], __fmul_rn(f[i], sx), 0.0f);
                cm[i + 1] = most3(cm[i + 1], __fmul_rn(f[i + 1], sx), 0.0f);
            }
            if (kSums) { total[i] += f[i]; total[i + 1] += f[i + 1]; }
        }
        const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(rm) & 0x7FFFFFFFu);
        if (lane == 0) atomicMax(row_most + m0 + 8 * k, top);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        most[warp][lane * 8 + i] = cm[i];
        if (kSums) sum[warp][lane * 8 + i] = total[i];
    }
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= O) return;
    uint32_t top = 0;
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top = max(top, __float_as_uint(most[i][threadIdx.x]) & 0x7FFFFFFFu);
        if (kSums) all += sum[i][threadIdx.x];
    }
    atomicMax(col_most + col, top);
    if (kSums) sums[(int64_t)blockIdx.y * O + col] = all;
}

// code8 where the factor is known not to be 0
__device__ __forceinline__ uint32_t code8_live(float t, float factor) { return __float_as_uint(__fadd_rn(__fmul_rn(t, factor), 12582912.0f)); }

template <typename T, bool kEven>
__global__ void __launch_bounds__(256)
grad8_codes_kernel(const T* __restrict__ dY, int64_t M, int64_t O, int64_t ld, bool vec, const float* __restrict__ s_w,
                   const float* __restrict__ s_x, const uint32_t* __restrict__ row_most, const uint32_t* __restrict__ col_most,
                   const float* __restrict__ sums, uint8_t* __restrict__ q_r, uint8_t* __restrict__ q_c, int64_t ldq,
                   float* __restrict__ s_r, float* __restrict__ s_c, float* __restrict__ dbias) {
    griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int strip = gridDim.y - 1 - blockIdx.y;
    const int64_t c = (int64_t)blockIdx.x * 256 + lane * 8, m0 = (int64_t)strip * kStrip + warp;
    const int rows = (int)min((int64_t)kStripRows, (M - m0 + 7) / 8);
    float w[8], fc[8];
    bool dead = false;   // a column without a usable scale
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float s = 0.0f;
        w[i] = fc[i] = 0.0f;
        if (c + i < O) {
            w[i] = s_w[c + i];
            scale8(col_most[c + i], s, fc[i]);
            if (strip == 0 && warp == 0) s_c[c + i] = s;
        }
        dead |= fc[i] == 0.0f;
    }
    if (sums != nullptr && strip == 0) {
        const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (col < O) {
            float all = 0.0f;
            for (int64_t z = 0; z * kStrip < M; ++z) all += sums[z * O + col];
            dbias[col] = all;
        }
    }
    dead = __any_sync(0xFFFFFFFFu, dead && c < ldq);
    float sx_all = 0.0f, fr_all = 0.0f;
    if (lane < rows) {
        float s;
        sx_all = s_x[m0 + 8 * lane];
        scale8(row_most[m0 + 8 * lane], s, fr_all);
        if (blockIdx.x == 0) s_r[m0 + 8 * lane] = s;
    }
    const T* row = dY + m0 * ld;
    uint8_t *to_r = q_r != nullptr ? q_r + m0 * ldq + c : nullptr, *to_c = q_c != nullptr ? q_c + m0 * ldq + c : nullptr;
    constexpr int kBatch = 4;   // rows whose loads are on their way together
    for (int k0 = 0; k0 < rows; k0 += kBatch) {
        Vec8<T> raw[kBatch];
        if (kEven) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                raw[k] = Vec8<T>{};
                if (c < O && k0 + k < rows) ld_vec(row + (k0 + k) * 8 * ld + c, raw[k].w);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int k = k0 + b;
            if (k >= rows) break;   // uniform over the warp
            const float sx = __shfl_sync(0xFFFFFFFFu, sx_all, k), fr = __shfl_sync(0xFFFFFFFFu, fr_all, k);
            float f[8];
            if (kEven) unpack(raw[b], f);
            else load_group(row + k * 8 * ld, c, O, vec, f);
            uint32_t q[8], p[8];
            if (fr != 0.0f && !dead) {   // uniform over the warp
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[i] = code8_live(__fmul_rn(f[i], w[i]), fr);
                    p[i] = code8_live(__fmul_rn(f[i], sx), fc[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[i] = code8(__fmul_rn(f[i], w[i]), fr);
                    p[i] = code8(__fmul_rn(f[i], sx), fc[i]);
                }
            }
            if (c < ldq) {
                if (to_r != nullptr) *reinterpret_cast<uint2*>(to_r + k * 8 * ldq) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
                if (to_c != nullptr) *reinterpret_cast<uint2*>(to_c + k * 8 * ldq) = make_uint2(pack4(p[0], p[1], p[2], p[3]), pack4(p[4], p[5], p[6], p[7]));
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ host
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                             CUtensorMapFloatOOBfill);

EncodeFn encoder() {
    static EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeFn>(p);
    });
    return fn;
}

// int8 codes [rows][pitch], boxes of `box_rows` rows x 128 bytes, 128-byte swizzle, zeros outside
bool code_map(CUtensorMap* tm, const void* base, int64_t pitch, int64_t rows, int box_rows) {
    EncodeFn fn = encoder();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kTileSmem = kRing + 1024;
constexpr int kPairSmem = kPairRing + 8 * 4096 + 1024;

lbt_status allow_smem() {
    constexpr int kDevices = 64;
    static std::mutex mu;
    static bool known[kDevices];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return LBT_ERR_CUDA;
    std::lock_guard<std::mutex> lock(mu);
    if (!known[dev]) {
        if (cudaFuncSetAttribute(l8_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileSmem) != cudaSuccess ||
            cudaFuncSetAttribute(l8_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem) != cudaSuccess)
            return LBT_ERR_CUDA;
        known[dev] = true;
    }
    return LBT_OK;
}

int64_t pitch16(int64_t n) { return (n + 15) / 16 * 16; }

bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

struct Product {
    int mode;
    const void* A; int64_t a_pitch, a_rows;   // as stored
    const void* B; int64_t b_pitch, b_rows;
    int64_t rows, cols, red;                  // C[rows, cols] = sum over red
    const float *row_scale, *col_scale, *bias;
    void* out; int out_type; int64_t ldo;
    bool behind;                              // the launch ahead writes operands of this one
    int lost = -1;                            // self-test: L8Args
    uint64_t limit_ns = kLimitNs;
};

lbt_status launch(const Product& p, int32_t* status, cudaStream_t stream) {
    lbt_status rc = allow_smem();
    if (rc != LBT_OK) return rc;
    L8Args a{};
    a.mode = p.mode;
    a.steps = (int)((p.red + kStep - 1) / kStep);
    a.rows = (int)p.rows; a.cols = (int)p.cols;
    a.row_scale = p.row_scale; a.col_scale = p.col_scale; a.bias = p.bias;
    a.out = p.out; a.out_type = p.out_type; a.ldo = p.ldo; a.status = status;
    a.vec = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0 && (p.ldo * type_size(p.out_type)) % 32 == 0;
    a.vec4 = misaligned(p.out, 4 * type_size(p.out_type)) || p.ldo % 4 != 0 ? 0 : 1;
    a.wait_prev = p.behind ? 1 : 0;
    a.lost = p.lost; a.limit_ns = p.limit_ns;
    a.splits = 1;
    CUtensorMap tmA, tmB;
    const int64_t big = ((p.rows + 255) / 256) * ((p.cols + 255) / 256);
    cudaLaunchAttribute attr[2];
    int n_attr = 0;
    cudaLaunchConfig_t cfg{};
    cfg.stream = stream;
    cfg.attrs = attr;
    if (p.behind) {
        attr[n_attr].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n_attr++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (big > kNumSMs / 2) {
        if (p.lost >= 0) return LBT_ERR_UNSUPPORTED;
        a.tiles_m = (int)((p.rows + 255) / 256);
        a.tiles_n = (int)((p.cols + 255) / 256);
        a.total = a.tiles_m * a.tiles_n;
        a.band = std::min(a.tiles_m, 8);
        if (!code_map(&tmA, p.A, p.a_pitch, p.a_rows, 128) || !code_map(&tmB, p.B, p.b_pitch, p.b_rows, 128)) return LBT_ERR_CUDA;
        cfg.gridDim = dim3((unsigned)(2 * std::min(a.total, kNumSMs / 2)));
        cfg.blockDim = dim3(kPairThreads);
        cfg.dynamicSmemBytes = kPairSmem;
        cfg.numAttrs = n_attr;
        return cudaLaunchKernelEx(&cfg, l8_pair_kernel, tmA, tmB, a) == cudaSuccess ? LBT_OK : LBT_ERR_CUDA;
    }
    // Up to 64 tokens the weights are the rows of the product and the tokens its columns: the tokens' share of the operand
    // traffic and of the products shrinks with their number.
    a.swapped = p.mode == kForward && p.rows <= 64;
    a.mma_n = a.swapped ? (int)pitch16(p.rows) : 128;
    a.stage_bytes = kBox + a.mma_n * kStep;
    a.stages = std::min(kMaxStages, kRing / a.stage_bytes);
    a.tiles_m = (int)(((a.swapped ? p.cols : p.rows) + 127) / 128);
    a.tiles_n = a.swapped ? 1 : (int)((p.cols + 127) / 128);
    a.total = a.tiles_m * a.tiles_n;
    a.band = std::min(a.tiles_m, 8);
    // Clusters share a tile while all their CTAs are resident at once (256: 288 CTAs in clusters of four left some for a second
    // round, 11 us late) and each has four steps of the reduction.
    while (a.splits < 8 && a.total * a.splits * 2 <= 256 && a.steps >= a.splits * 2 * 4) a.splits *= 2;
    if (p.lost >= a.splits) return LBT_ERR_UNSUPPORTED;
    const void* A = a.swapped ? p.B : p.A;
    const void* B = a.swapped ? p.A : p.B;
    if (!code_map(&tmA, A, a.swapped ? p.b_pitch : p.a_pitch, a.swapped ? p.b_rows : p.a_rows, 128) ||
        !code_map(&tmB, B, a.swapped ? p.a_pitch : p.b_pitch, a.swapped ? p.a_rows : p.b_rows, a.mma_n))
        return LBT_ERR_CUDA;
    if (a.splits > 1) {
        attr[n_attr].id = cudaLaunchAttributeClusterDimension;
        attr[n_attr].val.clusterDim.x = (unsigned)a.splits;
        attr[n_attr].val.clusterDim.y = attr[n_attr].val.clusterDim.z = 1;
        ++n_attr;
    }
    cfg.gridDim = dim3((unsigned)(a.total * a.splits));
    cfg.blockDim = dim3(kTileWarps * 32);
    cfg.dynamicSmemBytes = kTileSmem;
    cfg.numAttrs = n_attr;
    return cudaLaunchKernelEx(&cfg, l8_tile_kernel, tmA, tmB, a) == cudaSuccess ? LBT_OK : LBT_ERR_CUDA;
}

bool vec_rows(const void* p, int64_t ld, int type) {
    const size_t bytes = 8 * type_size(type);
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * type_size(type)) % bytes == 0;
}

template <typename T>
lbt_status quantize_rows(const T* x, int type, int64_t rows, int64_t cols, int64_t ld, void* q, int64_t ldq, float* scale, cudaStream_t stream) {
    const bool vec = vec_rows(x, ld, type);
    uint8_t* dst = static_cast<uint8_t*>(q);
    if (cols <= 1024) rows8_kernel<T, 32><<<(unsigned)((rows + 7) / 8), 256, 0, stream>>>(x, rows, cols, ld, vec, dst, ldq, pitch16(cols), scale);
    else rows8_kernel<T, 256><<<(unsigned)rows, 256, 0, stream>>>(x, rows, cols, ld, vec, dst, ldq, pitch16(cols), scale);
    return launch_status();
}

lbt_status quantize_rows_any(const void* x, int type, int64_t rows, int64_t cols, int64_t ld, void* q, int64_t ldq, float* scale, cudaStream_t stream) {
    if (rows == 0) return LBT_OK;
    if (type == LBT_F32) return quantize_rows(static_cast<const float*>(x), type, rows, cols, ld, q, ldq, scale, stream);
    if (type == LBT_BF16) return quantize_rows(static_cast<const __nv_bfloat16*>(x), type, rows, cols, ld, q, ldq, scale, stream);
    return quantize_rows(static_cast<const __half*>(x), type, rows, cols, ld, q, ldq, scale, stream);
}

// Bytes of a token's codes in the few-token kernel's shared memory.
int few_pitch(int64_t I) { return (int)((I + 127) / 128 * 128 + 64); }
bool few_fits(int64_t M, int64_t I) { return M <= kFewTokens && M * ((I + 127) / 128 * 128 + 64) <= kFewCodes; }

// Few tokens, from their codes (the quantizer may be the launch ahead) or from x.
FewArgs few_args(void* q_x, float* s_x, const void* q_w, const float* s_w, const float* bias, void* y, int y_type, int64_t ldy, int64_t M,
                 int64_t O, int64_t I) {
    FewArgs a{};
    a.q_x = static_cast<uint8_t*>(q_x); a.s_x = s_x; a.q_w = static_cast<const uint8_t*>(q_w);
    a.pitch = pitch16(I); a.I = (int)I; a.M = (int)M;
    a.tokens_pitch = few_pitch(I);
    a.out.rows = (int)M; a.out.cols = (int)O; a.out.col_scale = s_w; a.out.bias = bias;
    a.out.out = y; a.out.out_type = y_type; a.out.ldo = ldy;
    return a;
}

// Blocks of eight warps, two to an SM, while two blocks' codes, pieces and sums fit its 228 KB (each block takes 1 KB more); else of
// sixteen, one to an SM.  (16 tokens 2048 -> 8192, just beyond: 14.4 us, in blocks of eight that lie alone 16.4; 9 tokens 4096 -> 8192:
// 18.5 and 20.5.)
constexpr int few_pieces(int warps) { return kFewAhead * 2 * warps * 32 * 16; }
constexpr int few_sums(int tiles, int warps) { return 2 * warps * tiles * 8 * 17 * 4; }   // (the kernel's own)
template <int kTiles> constexpr int kFewCodesOfTwo = 228 * 1024 / 2 - 1024 - 256 - few_pieces(8) - few_sums(kTiles, 8);
static_assert(few_pieces(16) + few_sums(2, 16) + kFewCodes + 256 <= 227 * 1024, "one block of sixteen warps fits");
template <typename T, int kTiles, int kWarps>
lbt_status few_launch(const FewArgs& a, bool behind, cudaStream_t stream) {
    constexpr int pieces = few_pieces(kWarps);
    constexpr int kDevices = 64;
    static std::atomic<bool> known[kDevices];   // the attribute belongs to the device that is current when it is set
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return LBT_ERR_CUDA;
    if (!known[dev].load()) {
        if (cudaFuncSetAttribute(l8_few_kernel<T, kTiles, kWarps>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 pieces + (kWarps == 8 ? kFewCodesOfTwo<kTiles> : kFewCodes)) != cudaSuccess)
            return LBT_ERR_CUDA;
        known[dev].store(true);
    }
    const int smem = pieces + a.M * a.tokens_pitch;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)std::min((a.out.cols + 15) / 16, kNumSMs * (16 / kWarps)));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = behind ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, l8_few_kernel<T, kTiles, kWarps>, a) == cudaSuccess ? LBT_OK : LBT_ERR_CUDA;
}

template <typename T, int kTiles>
lbt_status few_any(const FewArgs& a, bool behind, cudaStream_t stream) {
    return a.M * a.tokens_pitch <= kFewCodesOfTwo<kTiles> ? few_launch<T, kTiles, 8>(a, behind, stream) : few_launch<T, kTiles, 16>(a, behind, stream);
}

lbt_status few_from_codes(FewArgs a, bool behind, cudaStream_t stream) {
    a.wait_prev = behind;
    return a.M <= 8 ? few_any<void, 1>(a, behind, stream) : few_any<void, 2>(a, behind, stream);
}

lbt_status few_from_x(FewArgs a, const void* x, int x_type, int64_t ldx, cudaStream_t stream) {
    a.x = x; a.ldx = ldx; a.vec = vec_rows(x, ldx, x_type);
    if (x_type == LBT_F32) return few_any<float, 1>(a, false, stream);
    if (x_type == LBT_BF16) return few_any<__nv_bfloat16, 1>(a, false, stream);
    return few_any<__half, 1>(a, false, stream);
}

lbt_status check_sizes(int64_t M, int64_t O, int64_t I) {
    if (M < 0 || O <= 0 || I <= 0) return LBT_ERR_INVALID_ARG;
    if (M >= (1ll << 31) - 256 || O >= (1ll << 31) - 256 || I >= (1ll << 31) - 256) return LBT_ERR_UNSUPPORTED;
    return LBT_OK;
}

struct BackwardSpace {
    size_t row_most, col_most, cleared, s_r, s_c, sums, q_r, q_c, total;
};

BackwardSpace backward_space(int64_t M, int64_t O) {
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    BackwardSpace w{};
    size_t at = 256;   // slack to align the caller's pointer
    w.row_most = at; at += up((size_t)M * 4);
    w.col_most = at; at += up((size_t)O * 4);
    w.cleared = at - w.row_most;
    w.s_r = at; at += up((size_t)M * 4);
    w.s_c = at; at += up((size_t)O * 4);
    w.sums = at; at += up((size_t)((M + kStrip - 1) / kStrip) * O * 4);
    w.q_r = at; at += up((size_t)M * pitch16(O));
    w.q_c = at; at += up((size_t)M * pitch16(O));
    w.total = at;
    return w;
}

template <typename T>
lbt_status quantize_gradient(const T* dY, int type, int64_t M, int64_t O, int64_t ld, const float* s_w, const float* s_x, uint8_t* base,
                             const BackwardSpace& w, bool need_r, bool need_c, float* dbias, cudaStream_t stream) {
    const int64_t ldq = pitch16(O);
    const bool vec = vec_rows(dY, ld, type);
    uint32_t* row_most = reinterpret_cast<uint32_t*>(base + w.row_most);
    uint32_t* col_most = reinterpret_cast<uint32_t*>(base + w.col_most);
    float* sums = dbias != nullptr ? reinterpret_cast<float*>(base + w.sums) : nullptr;
    LBT_CUDA_TRY(cudaMemsetAsync(row_most, 0, w.cleared, stream));
    const dim3 grid((unsigned)((ldq + 255) / 256), (unsigned)((M + kStrip - 1) / kStrip));
    const bool even = vec && O % 8 == 0;
    auto stats = even ? (sums != nullptr ? grad8_stats_kernel<T, true, true> : grad8_stats_kernel<T, true, false>)
                      : (sums != nullptr ? grad8_stats_kernel<T, false, true> : grad8_stats_kernel<T, false, false>);
    stats<<<grid, 256, 0, stream>>>(dY, M, O, ld, vec, s_w, s_x, row_most, col_most, sums);
    auto codes = even ? grad8_codes_kernel<T, true> : grad8_codes_kernel<T, false>;
    codes<<<grid, 256, 0, stream>>>(dY, M, O, ld, vec, s_w, s_x, row_most, col_most, sums, need_r ? base + w.q_r : nullptr,
                                    need_c ? base + w.q_c : nullptr, ldq, reinterpret_cast<float*>(base + w.s_r),
                                    reinterpret_cast<float*>(base + w.s_c), dbias);
    return launch_status();
}

}  // namespace
}  // namespace lbt

using namespace lbt;

extern "C" lbt_status lbt_rows8_quantize(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ld, void* q, int64_t ldq,
                                         float* scale, void* cuda_stream) {
    if (rows < 0 || cols <= 0 || ld < cols || ldq < cols || !type_ok(x_type)) return LBT_ERR_INVALID_ARG;
    if (rows > 0 && (x == nullptr || q == nullptr || scale == nullptr)) return LBT_ERR_INVALID_ARG;
    if (ldq % 16 != 0 || misaligned(q, 16) || misaligned(x, type_size(x_type)) || misaligned(scale, 4)) return LBT_ERR_ALIGNMENT;
    if (rows >= (1ll << 31) || cols >= (1ll << 31) - 256) return LBT_ERR_UNSUPPORTED;
    return quantize_rows_any(x, x_type, rows, cols, ld, q, ldq, scale, as_stream(cuda_stream));
}

static Product forward_operands(const void* q_x, const float* s_x, const void* q_w, const float* s_w, const float* bias, void* y, int y_type,
                                int64_t ldy, int64_t M, int64_t O, int64_t I, bool behind) {
    Product p{};
    p.mode = kForward;
    p.A = q_x; p.a_pitch = pitch16(I); p.a_rows = M;
    p.B = q_w; p.b_pitch = pitch16(I); p.b_rows = O;
    p.rows = M; p.cols = O; p.red = I;
    p.row_scale = s_x; p.col_scale = s_w; p.bias = bias;
    p.out = y; p.out_type = y_type; p.ldo = ldy;
    p.behind = behind;
    return p;
}

static lbt_status forward_product(const void* q_x, const float* s_x, const void* q_w, const float* s_w, const float* bias, void* y, int y_type,
                                  int64_t ldy, int64_t M, int64_t O, int64_t I, bool behind, int32_t* status, cudaStream_t stream) {
    if (few_fits(M, I))
        return few_from_codes(few_args(const_cast<void*>(q_x), const_cast<float*>(s_x), q_w, s_w, bias, y, y_type, ldy, M, O, I), behind, stream);
    return launch(forward_operands(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I, behind), status, stream);
}

static lbt_status check_forward(const void* q_x, const float* s_x, const void* q_w, const float* s_w, const float* bias, const void* y,
                                int y_type, int64_t ldy, int64_t M, int64_t O, int64_t I) {
    const lbt_status rc = check_sizes(M, O, I);
    if (rc != LBT_OK) return rc;
    if (!type_ok(y_type) || ldy < O || q_w == nullptr || s_w == nullptr) return LBT_ERR_INVALID_ARG;
    if (M > 0 && (q_x == nullptr || s_x == nullptr || y == nullptr)) return LBT_ERR_INVALID_ARG;
    if (misaligned(q_x, 16) || misaligned(q_w, 16) || misaligned(s_x, 4) || misaligned(s_w, 4) || misaligned(bias, 4) ||
        misaligned(y, type_size(y_type)))
        return LBT_ERR_ALIGNMENT;
    return I > kMaxReduction ? LBT_ERR_ACC_RANGE : LBT_OK;
}

extern "C" lbt_status lbt_linear8_forward(const void* x, int x_type, int64_t ldx, const void* q_w, const float* s_w, const float* bias,
                                          void* y, int y_type, int64_t ldy, int64_t M, int64_t O, int64_t I, void* q_x, float* s_x,
                                          int32_t* dev_status, void* cuda_stream) {
    lbt_status rc = check_forward(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I);
    if (rc != LBT_OK) return rc;
    if (!type_ok(x_type) || ldx < I || (M > 0 && x == nullptr)) return LBT_ERR_INVALID_ARG;
    if (misaligned(x, type_size(x_type))) return LBT_ERR_ALIGNMENT;
    if (M == 0) return LBT_OK;
    const cudaStream_t stream = as_stream(cuda_stream);
    // One token: every block quantizes it for itself, one launch.  (Two tokens that way measured as slow as a launch ahead, four slower.)
    if (M == 1 && few_fits(M, I))
        return few_from_x(few_args(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I), x, x_type, ldx, stream);
    rc = quantize_rows_any(x, x_type, M, I, ldx, q_x, pitch16(I), s_x, stream);
    if (rc != LBT_OK) return rc;
    return forward_product(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I, true, dev_status, stream);
}

extern "C" lbt_status lbt_linear8_matmul(const void* q_x, const float* s_x, const void* q_w, const float* s_w, const float* bias, void* y,
                                         int y_type, int64_t ldy, int64_t M, int64_t O, int64_t I, int32_t* dev_status, void* cuda_stream) {
    const lbt_status rc = check_forward(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I);
    if (rc != LBT_OK || M == 0) return rc;
    return forward_product(q_x, s_x, q_w, s_w, bias, y, y_type, ldy, M, O, I, false, dev_status, as_stream(cuda_stream));
}

extern "C" lbt_status lbt_selftest_linear8_timeout(const void* q_x, const float* s_x, const void* q_w, const float* s_w, float* y, int64_t M,
                                                   int64_t O, int64_t I, int rank, uint32_t limit_us, int32_t* dev_status, void* cuda_stream) {
    if (dev_status == nullptr || rank < 0 || limit_us == 0 || limit_us > 1000000u) return LBT_ERR_INVALID_ARG;
    const lbt_status rc = check_forward(q_x, s_x, q_w, s_w, nullptr, y, LBT_F32, O, M, O, I);
    if (rc != LBT_OK) return rc;
    if (M == 0) return LBT_ERR_UNSUPPORTED;
    Product p = forward_operands(q_x, s_x, q_w, s_w, nullptr, y, LBT_F32, O, M, O, I, false);
    p.lost = rank;
    p.limit_ns = (uint64_t)limit_us * 1000ull;
    return launch(p, dev_status, as_stream(cuda_stream));
}

extern "C" size_t lbt_linear8_workspace_bytes(int64_t M, int64_t O, int64_t I) {
    return check_sizes(M, O, I) == LBT_OK ? backward_space(M, O).total : 0;
}

extern "C" lbt_status lbt_linear8_backward(const void* dY, int dy_type, int64_t lddy, const void* q_w, const float* s_w, const void* q_x,
                                           const float* s_x, void* dX, int dx_type, int64_t lddx, void* dW, int dw_type, int64_t lddw,
                                           float* dbias, int64_t M, int64_t O, int64_t I, int32_t* dev_status, void* ws, size_t ws_bytes,
                                           void* cuda_stream) {
    lbt_status rc = check_sizes(M, O, I);
    if (rc != LBT_OK) return rc;
    if (!type_ok(dy_type) || lddy < O || (dX == nullptr && dW == nullptr && dbias == nullptr)) return LBT_ERR_INVALID_ARG;
    if (s_w == nullptr || (M > 0 && (dY == nullptr || s_x == nullptr))) return LBT_ERR_INVALID_ARG;
    if (dX != nullptr && (!type_ok(dx_type) || lddx < I || q_w == nullptr)) return LBT_ERR_INVALID_ARG;
    if (dW != nullptr && (!type_ok(dw_type) || lddw < I || (M > 0 && q_x == nullptr))) return LBT_ERR_INVALID_ARG;
    if (misaligned(dY, type_size(dy_type)) || misaligned(q_w, 16) || misaligned(q_x, 16) || misaligned(s_w, 4) || misaligned(s_x, 4) ||
        (dX != nullptr && misaligned(dX, type_size(dx_type))) || (dW != nullptr && misaligned(dW, type_size(dw_type))) || misaligned(dbias, 4))
        return LBT_ERR_ALIGNMENT;
    if ((dX != nullptr && O > kMaxReduction) || (dW != nullptr && M > kMaxReduction)) return LBT_ERR_ACC_RANGE;
    const BackwardSpace w = backward_space(M, O);
    if (ws == nullptr || ws_bytes < w.total) return LBT_ERR_WORKSPACE;
    const cudaStream_t stream = as_stream(cuda_stream);
    if (M > 65535 * (int64_t)kStrip) return LBT_ERR_UNSUPPORTED;
    if (M == 0) {   // no tokens: dX is empty, the sums are zero
        if (dW != nullptr) LBT_CUDA_TRY(cudaMemset2DAsync(dW, (size_t)lddw * type_size(dw_type), 0, (size_t)I * type_size(dw_type), (size_t)O, stream));
        if (dbias != nullptr) LBT_CUDA_TRY(cudaMemsetAsync(dbias, 0, (size_t)O * 4, stream));
        return LBT_OK;
    }
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255) - 256;   // offsets begin at 256
    if (dy_type == LBT_F32)
        rc = quantize_gradient(static_cast<const float*>(dY), dy_type, M, O, lddy, s_w, s_x, base, w, dX != nullptr, dW != nullptr, dbias, stream);
    else if (dy_type == LBT_BF16)
        rc = quantize_gradient(static_cast<const __nv_bfloat16*>(dY), dy_type, M, O, lddy, s_w, s_x, base, w, dX != nullptr, dW != nullptr, dbias, stream);
    else
        rc = quantize_gradient(static_cast<const __half*>(dY), dy_type, M, O, lddy, s_w, s_x, base, w, dX != nullptr, dW != nullptr, dbias, stream);
    if (rc != LBT_OK) return rc;
    Product p{};
    if (dX != nullptr) {
        p.mode = kDgrad;
        p.A = base + w.q_r; p.a_pitch = pitch16(O); p.a_rows = M;
        p.B = q_w; p.b_pitch = pitch16(I); p.b_rows = O;
        p.rows = M; p.cols = I; p.red = O;
        p.row_scale = reinterpret_cast<const float*>(base + w.s_r);
        p.behind = true;   // (the weights, its other operand, are older)
        p.out = dX; p.out_type = dx_type; p.ldo = lddx;
        rc = launch(p, dev_status, stream);
        if (rc != LBT_OK) return rc;
    }
    if (dW != nullptr) {
        p = Product{};
        p.mode = kWgrad;
        p.A = base + w.q_c; p.a_pitch = pitch16(O); p.a_rows = M;
        p.B = q_x; p.b_pitch = pitch16(I); p.b_rows = M;
        p.rows = O; p.cols = I; p.red = M;
        p.row_scale = reinterpret_cast<const float*>(base + w.s_c);
        p.behind = dX == nullptr;   // the quantizer is the launch ahead; dgrad does not release its successor early
        p.out = dW; p.out_type = dw_type; p.ldo = lddw;
        rc = launch(p, dev_status, stream);
    }
    return rc;
}
