// AdamW over many tensors in one launch, moments in fp32 or in 8 bits.
//
//   g' = g * grad_scale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;
//   p = (1 - lr wd) p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments: a tensor's elements fall into blocks of 256; m and u = sqrt(v) are kept as e4m3 codes of x * 448 / max|x|
// with the block's scale max|x| / 448 in fp32.  The root is stored because its ratios are the square roots of v's: e4m3
// spans 2^17.8 from its smallest to its largest number, so a block holds v's that differ by 2^35.  A positive root never
// becomes code 0 (it takes the smallest one): a vanished denominator would turn a small step into m / eps.  All of the
// arithmetic is fp32 with each operation rounded once (no contraction), so a step is reproducible operation for operation.
//
// The step is bound by memory: 14 bytes per element with fp32 parameters, bf16 gradients and 8-bit moments, 28 with all of
// it in fp32.  A block of 256 elements is one warp's work (8 consecutive elements a lane: 32-byte accesses of fp32, 16 of
// bf16, 8 of codes), so that a block's maximum is one warp reduction and nothing is shared between warps.  The table of
// tensors travels as a kernel argument: no device memory, no copy ahead of the launch.
#include <math.h>

#include <algorithm>

#include "lbt_types.cuh"

namespace lbt {

constexpr int kAdamBlock = 256;
constexpr int kAdamMax = 400;       // tensors per launch: the table fits the 32 764 bytes of a kernel's arguments
constexpr int kAdamFew = 40;        // a small table for few tensors: a launch that copies 3 KB of arguments instead of 30
constexpr int kAdamThreads = 256;

struct AdamEntry {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    uint64_t n;
    float step_size;   // lr / (1 - b1^t)
    float decay;       // 1 - lr wd
    int types;         // p type | g type << 4 | aligned << 8
};

template <int kCap>
struct AdamTable {
    AdamEntry e[kCap];
    uint32_t first[kCap + 1];   // first block of 256 of each tensor; first[count] = all of them
    int count;
    int run;                    // consecutive blocks a warp takes at a time
    float b1, omb1, b2, omb2, inv_c2, eps;
    const float* grad_scale;
    const int32_t* skip;
};

__device__ __forceinline__ float adam_load(const void* p, int type, uint64_t i) {
    if (type == LBT_F32) return static_cast<const float*>(p)[i];
    if (type == LBT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void adam_store(void* p, int type, uint64_t i, float v) {
    if (type == LBT_F32) static_cast<float*>(p)[i] = v;
    else if (type == LBT_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
__device__ __forceinline__ void adam_load8(const void* p, int type, uint64_t i, float (&f)[8]) {
    if (type == LBT_F32) load8(static_cast<const float*>(p) + i, f);
    else if (type == LBT_BF16) load8(static_cast<const __nv_bfloat16*>(p) + i, f);
    else load8(static_cast<const __half*>(p) + i, f);
}
__device__ __forceinline__ void adam_store8(void* p, int type, uint64_t i, const float (&f)[8]) {
    if (type == LBT_F32) store8(static_cast<float*>(p) + i, f);
    else if (type == LBT_BF16) store8(static_cast<__nv_bfloat16*>(p) + i, f);
    else store8(static_cast<__half*>(p) + i, f);
}

// e4m3 code (nearest, ties to even, saturating; NaN stays NaN) and back
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 e4m3_values(uint32_t pair) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)pair));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

struct AdamConst {
    float b1, omb1, b2, omb2, inv_c2, eps, gs;
};

// one element; returns u = sqrt(v)
__device__ __forceinline__ float adam_update(const AdamConst& c, float step_size, float decay, float g, float& p, float& m, float& v) {
    g = __fmul_rn(g, c.gs);
    m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.omb1, g));
    v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(c.omb2, __fmul_rn(g, g)));
    const float u = __fsqrt_rn(v);
    p = __fsub_rn(__fmul_rn(decay, p), __fdiv_rn(__fmul_rn(step_size, m), __fadd_rn(__fmul_rn(u, c.inv_c2), c.eps)));
    return u;
}

// The block's scale and factor from its largest finite magnitude (as bits).
__device__ __forceinline__ void block_scale(uint32_t most_bits, float& scale, float& factor) {
    const float most = __uint_as_float(most_bits);
    scale = __fmul_rn(most, 1.0f / 448.0f);
    factor = most > 1e-36f ? __fmul_rn(__frcp_rn(most), 448.0f) : 0.0f;
}
// what is stored of one element: NaN where it is not finite
__device__ __forceinline__ float scaled(float x, float factor, bool root) {
    if (abs_bits(x) >= kNonFinite) return __uint_as_float(0x7FC00000u);
    const float s = __fmul_rn(x, factor);
    return root && x > 0.0f ? fmaxf(s, 0.001953125f) : s;   // 2^-9, the smallest positive e4m3
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t b = abs_bits(x);
    return b < kNonFinite ? b : 0u;
}

// One block of 256 elements of one tensor, kN of them present (kFull: all 256, aligned, eight consecutive ones a lane;
// else element 32 j + lane, one by one).
template <int kBits, bool kFull>
__device__ __forceinline__ void adam_block(const AdamEntry& e, const AdamConst& c, uint64_t block, int lane) {
    const uint64_t base = block * kAdamBlock;
    const int p_type = e.types & 15, g_type = (e.types >> 4) & 15;
    float p[8], g[8], m[8], v[8];
    const uint64_t at = base + (kFull ? lane * 8 : lane);
    const int have = kFull ? 8 : (e.n > at ? (int)min((e.n - at + 31) / 32, (uint64_t)8) : 0);
    float ms = 0.0f, vs = 0.0f;
    if (kBits == 8) { ms = e.m_scale[block]; vs = e.v_scale[block]; }
    if (kFull) {
        adam_load8(e.p, p_type, at, p);
        adam_load8(e.g, g_type, at, g);
        if (kBits == 32) {
            load8(static_cast<const float*>(e.m) + at, m);
            load8(static_cast<const float*>(e.v) + at, v);
        } else {
            const uint2 mc = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.m) + at);
            const uint2 vc = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.v) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 a = e4m3_values(((i < 2 ? mc.x : mc.y) >> (16 * (i & 1))) & 0xFFFFu);
                const float2 b = e4m3_values(((i < 2 ? vc.x : vc.y) >> (16 * (i & 1))) & 0xFFFFu);
                m[2 * i] = a.x; m[2 * i + 1] = a.y; v[2 * i] = b.x; v[2 * i + 1] = b.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = g[i] = m[i] = v[i] = 0.0f;
            if (i < have) {
                const uint64_t k = at + 32 * i;
                p[i] = adam_load(e.p, p_type, k);
                g[i] = adam_load(e.g, g_type, k);
                if (kBits == 32) {
                    m[i] = static_cast<const float*>(e.m)[k];
                    v[i] = static_cast<const float*>(e.v)[k];
                } else {
                    m[i] = e4m3_values(static_cast<const uint8_t*>(e.m)[k]).x;
                    v[i] = e4m3_values(static_cast<const uint8_t*>(e.v)[k]).x;
                }
            }
        }
    }
    float u[8];
    uint32_t most_m = 0, most_u = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (kBits == 8) {
            m[i] = __fmul_rn(m[i], ms);
            v[i] = __fmul_rn(v[i], vs);
            v[i] = __fmul_rn(v[i], v[i]);
        }
        u[i] = adam_update(c, e.step_size, e.decay, g[i], p[i], m[i], v[i]);
        if (kBits == 8 && (kFull || i < have)) {
            most_m = max(most_m, finite_bits(m[i]));
            most_u = max(most_u, finite_bits(u[i]));
        }
    }
    if (kFull) adam_store8(e.p, p_type, at, p);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) adam_store(e.p, p_type, at + 32 * i, p[i]);
    if (kBits == 32) {
        if (kFull) {
            store8(static_cast<float*>(e.m) + at, m);
            store8(static_cast<float*>(e.v) + at, v);
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) {
                    static_cast<float*>(e.m)[at + 32 * i] = m[i];
                    static_cast<float*>(e.v)[at + 32 * i] = v[i];
                }
        return;
    }
    float fm, fu;
    block_scale(__reduce_max_sync(0xFFFFFFFFu, most_m), ms, fm);
    block_scale(__reduce_max_sync(0xFFFFFFFFu, most_u), vs, fu);
#pragma unroll
    for (int i = 0; i < 8; ++i) { m[i] = scaled(m[i], fm, false); u[i] = scaled(u[i], fu, true); }
    if (kFull) {
        uint32_t mc[2], vc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mc[i] = e4m3_pair(m[4 * i], m[4 * i + 1]) | e4m3_pair(m[4 * i + 2], m[4 * i + 3]) << 16;
            vc[i] = e4m3_pair(u[4 * i], u[4 * i + 1]) | e4m3_pair(u[4 * i + 2], u[4 * i + 3]) << 16;
        }
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.m) + at) = make_uint2(mc[0], mc[1]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.v) + at) = make_uint2(vc[0], vc[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) {
                static_cast<uint8_t*>(e.m)[at + 32 * i] = (uint8_t)e4m3_pair(m[i], 0.0f);
                static_cast<uint8_t*>(e.v)[at + 32 * i] = (uint8_t)e4m3_pair(u[i], 0.0f);
            }
    }
    if (lane == 0) { e.m_scale[block] = ms; e.v_scale[block] = vs; }
}

template <int kBits, int kCap>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamTable<kCap> t) {
    __shared__ uint32_t first[kCap + 1];
    if (t.skip != nullptr && *t.skip != 0) return;
    for (int i = threadIdx.x; i <= t.count; i += kAdamThreads) first[i] = t.first[i];
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const AdamConst c{t.b1, t.omb1, t.b2, t.omb2, t.inv_c2, t.eps, t.grad_scale != nullptr ? *t.grad_scale : 1.0f};
    const uint64_t all = first[t.count], stride = (uint64_t)gridDim.x * (kAdamThreads / 32) * t.run;
    for (uint64_t b0 = ((uint64_t)blockIdx.x * (kAdamThreads / 32) + (threadIdx.x >> 5)) * t.run; b0 < all; b0 += stride) {
        int lo = 0, hi = t.count;   // the tensor of block b0: the last with first <= b0 (empty tensors share their successor's first)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= b0) lo = mid; else hi = mid;
        }
        const uint64_t end = min(b0 + t.run, all);
        for (uint64_t b = b0; b < end; ++b) {
            while (b >= first[lo + 1]) ++lo;
            const AdamEntry& e = t.e[lo];
            const uint64_t block = b - first[lo];
            if ((e.types >> 8) != 0 && (block + 1) * kAdamBlock <= e.n) adam_block<kBits, true>(e, c, block, lane);
            else adam_block<kBits, false>(e, c, block, lane);
        }
    }
}

template <int kBits, int kCap>
static lbt_status adamw_launch(AdamTable<kCap>& t, cudaStream_t stream) {
    const uint64_t blocks = t.first[t.count];
    if (blocks == 0) return LBT_OK;
    // Few blocks: one a warp, spread over the SMs; many: runs of four, which amortise the search for the tensor.
    constexpr int warps = kAdamThreads / 32;
    t.run = blocks <= (uint64_t)kNumSMs * warps * 8 ? 1 : 4;
    const uint64_t want = (blocks + (uint64_t)warps * t.run - 1) / ((uint64_t)warps * t.run);
    const int grid = (int)std::min<uint64_t>(want, (uint64_t)kNumSMs * 32);
    adamw_kernel<kBits, kCap><<<grid, kAdamThreads, 0, stream>>>(t);
    return launch_status();
}

template <int kCap>
static lbt_status adamw_run(const lbt_adamw_tensor* tensors, int count, const lbt_adamw_hyper* h, const float* grad_scale,
                            const int32_t* skip, cudaStream_t stream) {
    AdamTable<kCap> t{};
    const double c1 = 1.0 - pow(h->beta1, (double)h->step), c2 = sqrt(1.0 - pow(h->beta2, (double)h->step));
    t.b1 = (float)h->beta1; t.omb1 = (float)(1.0 - h->beta1);
    t.b2 = (float)h->beta2; t.omb2 = (float)(1.0 - h->beta2);
    t.inv_c2 = 1.0f / (float)c2;
    t.eps = (float)h->eps;
    t.grad_scale = grad_scale;
    t.skip = skip;
    t.count = count;
    uint64_t at = 0;
    for (int i = 0; i < count; ++i) {
        const lbt_adamw_tensor& s = tensors[i];
        AdamEntry& e = t.e[i];
        e.p = s.p; e.g = s.g; e.m = s.m; e.v = s.v; e.m_scale = s.m_scale; e.v_scale = s.v_scale; e.n = s.n;
        e.step_size = (float)(s.lr / c1);
        e.decay = (float)(1.0 - s.lr * s.weight_decay);
        // eight elements in one access: 32 bytes of fp32, 16 of a 16-bit type, 8 of codes
        auto ok = [](const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; };
        const size_t state = h->state_bits == 8 ? 8 : 32;
        const bool aligned = ok(s.p, 8 * type_size(s.p_type)) && ok(s.g, 8 * type_size(s.g_type)) && ok(s.m, state) && ok(s.v, state);
        e.types = s.p_type | s.g_type << 4 | (aligned ? 1 << 8 : 0);
        t.first[i] = (uint32_t)at;
        at += (s.n + kAdamBlock - 1) / kAdamBlock;
        if (at > 0xFFFFFFFFull) return LBT_ERR_UNSUPPORTED;
    }
    t.first[count] = (uint32_t)at;
    return h->state_bits == 8 ? adamw_launch<8, kCap>(t, stream) : adamw_launch<32, kCap>(t, stream);
}

}  // namespace lbt

using namespace lbt;

extern "C" lbt_status lbt_adamw_step(const lbt_adamw_tensor* tensors, int count, const lbt_adamw_hyper* h,
                                     const float* d_grad_scale, const int32_t* d_skip, void* cuda_stream) {
    if (count < 0 || (count > 0 && tensors == nullptr) || h == nullptr || h->step < 1) return LBT_ERR_INVALID_ARG;
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && h->eps >= 0.0)) return LBT_ERR_INVALID_ARG;
    if (h->state_bits != 8 && h->state_bits != 32) return LBT_ERR_UNSUPPORTED_BITS;
    uint64_t blocks = 0;
    for (int i = 0; i < count; ++i) {
        const lbt_adamw_tensor& s = tensors[i];
        if (!type_ok(s.p_type) || !type_ok(s.g_type)) return LBT_ERR_INVALID_ARG;
        if (s.n == 0) continue;
        if (s.p == nullptr || s.g == nullptr || s.m == nullptr || s.v == nullptr) return LBT_ERR_INVALID_ARG;
        if (h->state_bits == 8 && (s.m_scale == nullptr || s.v_scale == nullptr)) return LBT_ERR_INVALID_ARG;
        // each tensor has its element type's own alignment at least
        auto off = [](const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; };
        if (off(s.p, type_size(s.p_type)) || off(s.g, type_size(s.g_type)) || off(s.m_scale, 4) || off(s.v_scale, 4) ||
            (h->state_bits == 32 && (off(s.m, 4) || off(s.v, 4))))
            return LBT_ERR_ALIGNMENT;
        if (s.n > (1ull << 40)) return LBT_ERR_UNSUPPORTED;
        blocks += (s.n + kAdamBlock - 1) / kAdamBlock;
    }
    if (blocks > 0xFFFFFFFFull) return LBT_ERR_UNSUPPORTED;
    const cudaStream_t stream = as_stream(cuda_stream);
    for (int i = 0; i < count; i += kAdamMax) {
        const int n = std::min(count - i, kAdamMax);
        const lbt_status rc = n <= kAdamFew ? adamw_run<kAdamFew>(tensors + i, n, h, d_grad_scale, d_skip, stream)
                                            : adamw_run<kAdamMax>(tensors + i, n, h, d_grad_scale, d_skip, stream);
        if (rc != LBT_OK) return rc;
    }
    return LBT_OK;
}
