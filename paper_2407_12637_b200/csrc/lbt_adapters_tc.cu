// Long runs of low-rank adapters on the fifth-generation tensor cores: bf16 and fp16 rows that begin on 16 bytes, any rank to 128.
//
//   h[m] = A_i x[m] (rank values);  out[m] = base[m] + s_i sum_k h[m,k] B_i[k]
//
// A tile is 128 tokens of one run; a cluster of one to eight CTAs shares x's columns, then the output's, 64 at a time.  Both products take
// their operands as TMA leaves them: x (or base) and the weights come through a ring of stages, 128 bytes a row, swizzled; ranks are filled up with
// zeros to a multiple of 16.  The first product's sums lie in four accumulators in turn (two above 64 ranks), which are added up in fp32 (an
// accumulator's own additions are cut off, not rounded: a chain a quarter as long loses a quarter); the CTAs' partial h meet in
// shared memory, each CTA adding up its share of the rows for all.  h enters the second product as two 16-bit numbers (K-major tiles
// that the CTAs write into each other's memory: 16 bits of h for bf16, 22 for fp16, after a power of two for each row), B as it lies: ranks are the reduced index, columns
// contiguous (MN-major).  Its sums go to one of two accumulators; four warps each add them to base's stage, in place, and store whole 128 bytes of a row.
// Roles: a thread for each side's copies, one that issues products, two times four warps of the epilogue; all warps add up h.
//
// 4096 -> 4096, bf16, replayed on the same inputs, against fragments in registers: 8192 tokens, rank 16 43 us (45), rank 64 43 (84), rank 128 59 (127), with
// nothing of them in L2 beforehand 50, 51 and 65; 2085 tokens in 11 runs, rank 64 20 (37); 16384 tokens, rank 16 78 (79): 5.2 TB/s of the 6.6 that a copy reaches.  What is left is the time in which nothing
// streams: 13000 clocks a tile (start 2000, first columns 3000, h through the cluster 6000, the last columns 2000).
// One thread's instructions are what the products wait for: descriptors are made once a stage and stepped by constants (rank 64: 48 -> 44 us).
// Tiles of fewer tokens, so that clusters of two fill all SMs, gained nothing (8192 tokens: 43).
//
// Every wait on a barrier is bounded: where one runs out, the status word says so, what is in flight is waited for, and the kernel ends.  In the first
// product no CTA of the cluster goes on to the second one; in the second one the warps that waited store nothing more.
#include <algorithm>
#include <atomic>
#include <mutex>

#include "lbt_adapters.cuh"

namespace lbt {

constexpr int kTcTokens = 128;   // of a tile at most
constexpr int kTcLeft = kTcTokens * 128;
constexpr int kTcThreads = 384;   // a warp that loads, one that issues products, two idle; two times four of the epilogue

// Ranks to kMax: bytes of a stage, stages, accumulators of the first product (the second one's two lie behind them in TMEM).
template <int kMax> struct TcSizes {
    static constexpr int kStage = kTcLeft + kMax * 128, kStages = kMax == 64 ? 6 : 3, kSums = kMax == 64 ? 4 : 2;
    static constexpr int kPart = kTcLeft * (kMax / 64);
    static constexpr int kBytes = kStages * kStage + 2 * kPart + (int)sizeof(float) * kTcTokens * (kMax + 1) + 256 + 1024;
};
template <int kStages> struct TcBarriers {
    uint64_t full[kStages], used[kStages], done[kStages];   // a stage is filled; the first product has read it; the epilogue has
    uint64_t h_sums, sums[2], taken[2];                     // the first product's sums are there; the second one's; they have been read
    uint32_t tmem, lost, dead;
};
static_assert(sizeof(TcBarriers<6>) <= 256 && TcSizes<64>::kBytes <= 232448 && TcSizes<128>::kBytes <= 232448, "");

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// fp32 accumulators; both operands bf16 or both fp16; B K-major or MN-major
template <typename T> __device__ __forceinline__ uint32_t idesc_16(int m, int n, bool b_mn_major) {
    const uint32_t format = IsHalf<T>::value ? 0u : 1u;
    return 1u << 4 | format << 7 | format << 10 | (b_mn_major ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

template <int kStages> __device__ __forceinline__ bool tc_wait(uint64_t* bar, uint32_t parity, TcBarriers<kStages>* b, uint64_t limit_ns) {
    if (mbar_wait_bounded(bar, parity, limit_ns)) return true;
    *reinterpret_cast<volatile uint32_t*>(&b->lost) = 1u;
    return false;
}

template <typename T, int kMax>
__global__ void __launch_bounds__(kTcThreads, 1)
adapter_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_base,
                  const __grid_constant__ CUtensorMap map_b, const __grid_constant__ AdapterArgs g) {
    using S = TcSizes<kMax>;
    constexpr bool kHalf = IsHalf<T>::value;
    constexpr int kStages = S::kStages;
    extern __shared__ uint8_t raw[];
    uint8_t* ring = raw + (1024 - (smem_u32(raw) & 1023)) % 1024;      // (the swizzle counts from 1024 bytes; the same place in every CTA)
    uint8_t* parts = ring + kStages * S::kStage;                       // h's first and second parts: each 64 ranks [128] rows of 128 bytes
    float* mine = reinterpret_cast<float*>(parts + 2 * S::kPart);      // [128][kMax], read by the other CTAs; four ranks c of row m lie at c ^ (m & 7)
    float* factor = mine + kTcTokens * kMax;                           // [128], of fp16 rows
    auto* b = reinterpret_cast<TcBarriers<kStages>*>(factor + kTcTokens);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int cta = (int)cluster_ctarank(), ctas = g.ctas;
    int row, rows, adapter;
    if (!run_of_tile(g, kTcTokens, blockIdx.x / ctas, row, rows, adapter)) return;   // (all CTAs of the cluster)
    const int groups = (g.O + 63) / 64, steps = (g.I + 63) / 64;
    const int group_lo = (int)((int64_t)groups * cta / ctas), group_hi = (int)((int64_t)groups * (cta + 1) / ctas);
    const int step_lo = (int)((int64_t)steps * cta / ctas), n1 = (int)((int64_t)steps * (cta + 1) / ctas) - step_lo;
    T* out = static_cast<T*>(g.out) + row * g.ld_out;
    if (adapter < 0 || adapter >= g.adapters) {
        copy_rows<T, false>(g, static_cast<const T*>(g.base) + row * g.ld_base, out, rows, 64 * group_lo, 64 * group_hi, kTcThreads / 32);
        return;
    }
    const int n2 = g.out != nullptr ? group_hi - group_lo : 0, all = n1 + n2, rank = g.rank, ranks = (rank + 15) / 16 * 16;   // (of the products: the weights' rows behind `rank` are zeros)

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(&b->full[s], 2); mbar_init(&b->used[s], 1); mbar_init(&b->done[s], 4); }
        mbar_init(&b->h_sums, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&b->sums[i], 1); mbar_init(&b->taken[i], 4); }
        b->lost = 0u;
        fence_mbar_init();
    }
    for (int i = threadIdx.x; i < kStages * (ranks - rank) * 8; i += kTcThreads) {
        const int s = i / ((ranks - rank) * 8), at = i % ((ranks - rank) * 8);
        *reinterpret_cast<uint4*>(ring + s * S::kStage + kTcLeft + rank * 128 + at * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    if (ranks > rank) fence_proxy_async_smem();
    if (warp == 1) { tmem_alloc(&b->tmem, 512); tmem_relinquish(); }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = b->tmem;

    // This thread's side (the tokens or the weights) of step i, once the stage's last reader has left it: the first product for n1 steps, then the epilogue.
    auto load = [&](int i) {
        const int s = i % kStages, before = i - kStages;
        if (before >= n1) {
            const int first = n1 + (s - n1 % kStages + kStages) % kStages;   // the first of the second product's steps in this stage
            if (!tc_wait(&b->done[s], ((before - first) / kStages) & 1, b, g.limit_ns)) return false;
        } else if (before >= 0 && !tc_wait(&b->used[s], (before / kStages) & 1, b, g.limit_ns)) {
            return false;
        }
        const bool second = i >= n1;
        const int c = 64 * (second ? group_lo + i - n1 : step_lo + i);
        uint8_t* to = ring + s * S::kStage;
        if (warp == 0) {
            mbar_arrive_expect_tx(&b->full[s], kTcLeft);
            tma_load_2d(to, second ? &map_base : &map_x, &b->full[s], c, row);
        } else {
            mbar_arrive_expect_tx(&b->full[s], rank * 128);
            tma_load_2d(to + kTcLeft, second ? &map_b : &map_a, &b->full[s], c, adapter * rank);
        }
        return true;
    };
    int loaded = 0;   // (of a thread that loads)
    bool ok = true;

    // h of this CTA's columns of x
    if (warp == 0 || warp == 2) {
        if (lane == 0)
            for (const int end = min(all, n1 + kStages); loaded < end && (ok = load(loaded)); ++loaded) {}
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = idesc_16<T>(kTcTokens, ranks, false);
            for (int i = 0; i < n1 && ok; ++i) {
                const int s = i % kStages;
                ok = tc_wait(&b->full[s], (i / kStages) & 1, b, g.limit_ns);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t left = smem_desc_sw128(smem_u32(ring + s * S::kStage), 16, 1024), right = left + (kTcLeft >> 4);   // (addresses in 16 bytes)
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_f16(tmem + kMax * (i % S::kSums), left + 2 * k, right + 2 * k, idesc, i >= S::kSums || k > 0);
                mma_commit(&b->used[s]);
            }
            if (ok && cta != g.mute) mma_commit(&b->h_sums);
        }
    } else if (warp >= 4) {
        const int m = 32 * (warp & 3) + lane;
        ok = tc_wait(&b->h_sums, 0, b, g.limit_ns);
        __syncwarp();
        tc_fence_after_sync();
        for (int c0 = warp >= 8 ? 32 : 0; c0 < ranks; c0 += 64) {
            float sum[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) sum[c] = 0.0f;
            for (int q = 0; q < min(S::kSums, n1); ++q) {
                uint32_t v[32];
                tmem_ld_32x32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kMax * q + c0, v);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 32; ++c) sum[c] += __uint_as_float(v[c]);
            }
#pragma unroll
            for (int c = 0; c < 32; c += 4)
                if (c0 + c < ranks) *reinterpret_cast<float4*>(mine + m * kMax + (((c0 + c) / 4 ^ (m & 7)) << 2)) = make_float4(sum[c], sum[c + 1], sum[c + 2], sum[c + 3]);
        }
        tc_fence_before_sync();
    }
    cluster_sync_all();
    if (threadIdx.x == 0) {
        uint32_t lost = 0;
        for (int c = 0; c < ctas; ++c) lost |= __float_as_uint(ld_cluster(map_to_cta(smem_u32(&b->lost), c)));
        b->dead = lost;
    }
    __syncwarp();
    // A lane adds up four ranks of a row of h, and writes its parts where every CTA's second product reads them.
    constexpr int kLanes = kMax / 4;
    const float scale = g.scale != nullptr ? g.scale[adapter] : 1.0f;
    const int last = rows * (cta + 1) / ctas, j = threadIdx.x % kLanes;
    for (int m0 = rows * cta / ctas; m0 < last; m0 += kTcThreads / kLanes) {
        const int m = m0 + threadIdx.x / kLanes;
        const bool here = m < last && 4 * j < ranks;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (here) {
            const uint32_t from = smem_u32(mine + m * kMax + ((j ^ (m & 7)) << 2));
            float4 w[kAdCluster];
#pragma unroll
            for (int c = 0; c < kAdCluster; ++c)
                if (c < ctas) w[c] = ld_cluster4(map_to_cta(from, c));
#pragma unroll
            for (int c = 0; c < kAdCluster; ++c)
                if (c < ctas) { v.x += w[c].x; v.y += w[c].y; v.z += w[c].z; v.w += w[c].w; }
            v.x = 4 * j < rank ? v.x : 0.0f;
            v.y = 4 * j + 1 < rank ? v.y : 0.0f;
            v.z = 4 * j + 2 < rank ? v.z : 0.0f;
            v.w = 4 * j + 3 < rank ? v.w : 0.0f;
            if (g.h != nullptr) {
                float* to = g.h + (int64_t)(row + m) * rank + 4 * j;
                if (4 * j < rank) to[0] = v.x;
                if (4 * j + 1 < rank) to[1] = v.y;
                if (4 * j + 2 < rank) to[2] = v.z;
                if (4 * j + 3 < rank) to[3] = v.w;
            }
        }
        v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
        if (kHalf) {
            uint32_t most = max(max(abs_bits(v.x), abs_bits(v.y)), max(abs_bits(v.z), abs_bits(v.w)));
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            const float f = row_factor(most);
            v.x *= f; v.y *= f; v.z *= f; v.w *= f;
            if (here && j == 0)
                for (int c = 0; c < ctas; ++c) st_cluster(map_to_cta(smem_u32(factor + m), c), 1.0f / f);
        }
        if (here) {
            uint2 hi, lo;
            split16<T>(v.x, v.y, hi.x, lo.x);
            split16<T>(v.z, v.w, hi.y, lo.y);
            const uint32_t to = smem_u32(parts + j / 16 * kTcLeft + m * 128 + ((j % 16 / 2 ^ (m & 7)) << 4) + (j & 1) * 8);
            for (int c = 0; c < ctas; ++c) {
                const uint32_t at = map_to_cta(to, c);
                st_cluster2(at, hi);
                st_cluster2(at + S::kPart, lo);
            }
        }
    }
    fence_proxy_async();
    cluster_sync_all();   // nobody leaves before the partial sums have been fetched, nobody goes on before h is there
    fence_proxy_async();
    const bool go_on = b->dead == 0;
    __syncthreads();

    if (go_on && n2 > 0) {
        if (warp == 0 || warp == 2) {
            if (lane == 0)
                for (; loaded < all && (ok = load(loaded)); ++loaded) {}
        } else if (warp == 1) {
            if (lane == 0) {
                tc_fence_after_sync();
                const uint32_t idesc = idesc_16<T>(kTcTokens, 64, true);
                const uint64_t h = smem_desc_sw128(smem_u32(parts), 16, 1024);
                for (int j = 0; j < n2 && ok; ++j) {
                    const int i = n1 + j, s = i % kStages, buffer = j & 1;
                    ok = (j < 2 || tc_wait(&b->taken[buffer], (j / 2 - 1) & 1, b, g.limit_ns)) && tc_wait(&b->full[s], (i / kStages) & 1, b, g.limit_ns);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t d = tmem + S::kSums * kMax + 64 * buffer;
                    const uint64_t right = smem_desc_sw128(smem_u32(ring + s * S::kStage) + kTcLeft, 8192, 1024);
#pragma unroll
                    for (int part = 1; part >= 0; --part)   // the smaller part first
#pragma unroll
                        for (int k = 0; k < kMax / 16; ++k)
                            if (16 * k < ranks) mma_f16(d, h + ((part * S::kPart + k / 4 * kTcLeft + k % 4 * 32) >> 4), right + (2048 * k >> 4), idesc, part == 0 || k > 0);
                    mma_commit(&b->sums[buffer]);
                }
            }
        } else if (warp >= 4) {
            const int m = 32 * (warp & 3) + lane;
            const float back = kHalf ? factor[m] : 1.0f;
            const int buffer = warp >= 8, sub = lane >> 3, chunk = lane & 7;   // four warps take every other step
            for (int j = buffer; j < n2 && ok; j += 2) {
                const int i = n1 + j, s = i % kStages, col = 64 * (group_lo + j);
                ok = tc_wait(&b->full[s], (i / kStages) & 1, b, g.limit_ns) && tc_wait(&b->sums[buffer], (j / 2) & 1, b, g.limit_ns);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                uint8_t* base = ring + s * S::kStage;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t v[32];
                    tmem_ld_32x32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + S::kSums * kMax + 64 * buffer + 32 * half, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 4; ++q) {   // eight columns; the sums take base's place
                        uint4* at = reinterpret_cast<uint4*>(base + m * 128 + (((4 * half + q) ^ (m & 7)) << 4));
                        const uint4 o = *at;
                        uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float2 f = values16(w[c], T());
                            const float e0 = __uint_as_float(v[8 * q + 2 * c]), e1 = __uint_as_float(v[8 * q + 2 * c + 1]);
                            w[c] = kHalf ? pair16<T>(fmaf(e0, back, f.x), fmaf(e1, back, f.y)) : pair16<T>(f.x + e0, f.y + e1);
                        }
                        *at = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&b->taken[buffer]);
                T* to = out + col + 8 * chunk;
                const bool inside = col + 8 * chunk < g.O;
#pragma unroll
                for (int q = 0; q < 8; ++q) {   // four rows' 128 bytes at a time
                    const int mm = 32 * (warp & 3) + 4 * q + sub;
                    const uint4 o = *reinterpret_cast<const uint4*>(base + mm * 128 + ((chunk ^ (mm & 7)) << 4));
                    if (inside && mm < rows) *reinterpret_cast<uint4*>(to + mm * g.ld_out) = o;
                }
                fence_proxy_async_smem();   // the stage's next tile is written behind these stores
                __syncwarp();
                if (lane == 0) mbar_arrive(&b->done[s]);
            }
        }
    }
    __syncwarp();
    tc_fence_before_sync();
    __syncthreads();
    // What was asked for and not waited for (a wait has run out) arrives before this CTA's memory goes.
    if ((warp == 0 || warp == 2) && lane == 0 && (!go_on || *reinterpret_cast<volatile uint32_t*>(&b->lost) != 0)) {
        if (g.status != nullptr) atomicCAS(g.status, (int32_t)LBT_OK, (int32_t)LBT_ERR_TIMEOUT);
        for (int i = max(0, loaded - kStages); i < loaded; ++i) mbar_wait_bounded(&b->full[i % kStages], (i / kStages) & 1, g.limit_ns);
    }
    if (warp == 1) { tc_fence_after_sync(); tmem_dealloc(tmem, 512); }
}

// ---------------------------------------------------------------------------------------------- host
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeFn tc_encoder() {
    static EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) fn = reinterpret_cast<EncodeFn>(p);
    });
    return fn;
}

// 16-bit rows, boxes of `box` rows x 64 columns, 128-byte swizzle, zeros outside.
static bool tc_map(CUtensorMap* map, const void* p, int64_t cols, int64_t rows, int64_t ld, int box) {
    EncodeFn fn = tc_encoder();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, each[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(p), dims, strides, boxes, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kMax> static lbt_status tc_launch(AdapterArgs g, cudaStream_t stream) {
    auto kernel = adapter_tc_kernel<T, kMax>;
    constexpr int kBytes = TcSizes<kMax>::kBytes;
    LBT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes));
    const int64_t runs = g.offsets == nullptr ? 1 : g.runs;
    cudaLaunchConfig_t config{};
    config.blockDim = dim3(kTcThreads);
    config.dynamicSmemBytes = kBytes;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    // As many CTAs to a cluster as leave all clusters resident at once, where a run ends on average a little ahead of the middle of a tile.
    static std::atomic<int> fit[kAdCluster + 1];
    for (g.ctas = kAdCluster;; --g.ctas) {
        attr[0].val.clusterDim.x = g.ctas;
        config.gridDim = dim3(g.ctas);
        int n = fit[g.ctas].load(std::memory_order_relaxed);
        if (n == 0) {
            if (cudaOccupancyMaxActiveClusters(&n, kernel, &config) != cudaSuccess || n < 1) {
                cudaGetLastError();
                n = 1;
            }
            fit[g.ctas].store(n, std::memory_order_relaxed);
        }
        if (g.ctas == 1 || (g.M + (runs == 1 ? kTcTokens - 1 : 5 * kTcTokens / 8 * runs)) / kTcTokens <= n) break;
    }
    config.gridDim = dim3((unsigned)((g.M + (kTcTokens - 1) * runs) / kTcTokens * g.ctas));
    CUtensorMap x, a, base, b;
    const int64_t rows = (int64_t)g.adapters * g.rank;   // of the weights
    const bool out = g.out != nullptr;
    if (!tc_map(&x, g.x, g.I, g.M, g.ld_x, kTcTokens) || !tc_map(&a, g.a, g.I, rows, g.I, g.rank) ||
        !tc_map(&base, out ? g.base : g.x, out ? g.O : g.I, g.M, out ? g.ld_base : g.ld_x, kTcTokens) || !tc_map(&b, g.b, g.O, rows, g.O, g.rank))
        return LBT_ERR_CUDA;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, x, a, base, b, g));
    return launch_status();
}

lbt_status adapter_tc(const AdapterArgs& g, int type, cudaStream_t stream) {
    if (g.rank <= 64) return type == LBT_BF16 ? tc_launch<__nv_bfloat16, 64>(g, stream) : tc_launch<__half, 64>(g, stream);
    return type == LBT_BF16 ? tc_launch<__nv_bfloat16, 128>(g, stream) : tc_launch<__half, 128>(g, stream);
}

}  // namespace lbt
