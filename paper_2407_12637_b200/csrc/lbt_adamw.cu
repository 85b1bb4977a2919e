// AdamW over many tensors in one launch, moments in fp32 or in 8 bits.
//
//   g' = g * grad_scale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;
//   p = (1 - lr wd) p - (lr / (1 - b1^t)) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments: a tensor's elements fall into blocks of 256; m and u = sqrt(v) are kept as e4m3 codes of x * 448 / max|x|
// with the block's scale max|x| / 448 in fp32.  The root is stored because its ratios are the square roots of v's: e4m3
// spans 2^17.8 from its smallest to its largest number, so a block holds v's that differ by 2^35.  A positive root never
// becomes code 0 (it takes the smallest one): a vanished denominator would turn a small step into m / eps.  The moments are
// fp32 with each operation rounded once (no contraction), so their codes are reproducible operation for operation; the
// quotient of the update is good to 2 ulp.
//
// The step is bound by memory: 14 bytes per element with fp32 parameters, bf16 gradients and 8-bit moments, 28 with all of
// it in fp32.  A block of 256 elements is one warp's work (8 consecutive elements a lane: 32-byte accesses of fp32, 16 of
// bf16, 8 of codes), so that a block's maximum is one warp reduction and nothing is shared between warps; 64 registers keep 32
// warps on an SM, which hide the loads better than copies ahead through shared memory did with 24 (fp32 states: 55 against 80 us).  The table of tensors travels as a kernel
// argument: no device memory, no copy ahead of the launch.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "lbt_types.cuh"

namespace lbt {

constexpr int kAdamBlock = 256;
constexpr int kAdamMax = 400;       // tensors per launch: the table fits the 32 764 bytes of a kernel's arguments
constexpr int kAdamFew = 40;        // smaller tables for fewer tensors: a launch copies 3 or 10 KB of arguments instead of 30
constexpr int kAdamSome = 128;      //   (the call takes 4.5, 5.5 and 7.5 us of the host's time)
constexpr int kAdamThreads = 256;
constexpr int kAdamRun = 8;         // blocks a warp takes at a time: their scales are one 32-byte sector

struct AdamEntry {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    uint64_t n;
    double step_size;  // lr / (1 - b1^t), t the host's step
    float decay;       // 1 - lr wd
    int types;         // p type | g type << 4 | aligned << 8
};

template <int kCap>
struct AdamTable {
    AdamEntry e[kCap];
    uint32_t first[kCap + 1];   // first run of blocks of each tensor; first[count] = all of them
    int count;
    int run;                    // blocks of a run: kAdamRun, or 1
    float b1, omb1, b2, omb2, inv_c2, eps;
    const float* grad_scale;
    const int32_t* skip;
    int64_t* skipped;           // steps held back so far (null: none), added to by this launch if `counts`
    int counts;
    int64_t step;               // the host's step: t = step - *skipped
    double beta1, beta2, c1;    // c1 = 1 - b1^step
};
static_assert(sizeof(AdamTable<kAdamMax>) <= 32764, "the table is a kernel argument");

// b^t by squaring (t >= 1): a rounding for each of its at most 2 log2 t products, in 64 bits
__device__ __forceinline__ double adam_power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

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
    float step_size;   // of the tensor at work
};

// sqrt(v) by Markstein's correction (Computation of Elementary Functions on the IBM RISC System/6000, 1990): s = v y with y a
// hardware reciprocal root, then s + (v - s s) y / 2 with the residual exact in one fused operation.  Rounds as sqrtf does but
// for about one v in 2^22; below the normal range (v < 2^-126, where eps is all of the denominator) the root is underestimated.
// sqrtf's own special cases took a fifth of the step's instructions.  (An infinity or NaN comes out as NaN: adam_update.)
__device__ __forceinline__ float adam_root(float v) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaxf(v, 1.17549435e-38f)));
    const float s = __fmul_rn(v, y);
    return __fmaf_rn(__fmaf_rn(-s, s, v), __fmul_rn(0.5f, y), s);
}

// One element; returns u = sqrt(v).  An infinite v (a finite gradient beyond 1.8e19 squared) has the root infinity and the update 0.
// 8 bits have no code for infinity: it is stored as NaN, and a NaN there is read as infinity (a gradient that is not finite shows in m).
enum RootOf { kOf32, kOf8, kLeft };   // kLeft: an infinite or NaN v leaves NaN in the root and in p, which the caller mends
template <RootOf kOdd>
__device__ __forceinline__ float adam_update(const AdamConst& c, float decay, float g, float& p, float& m, float& v) {
    g = __fmul_rn(g, c.gs);
    m = __fadd_rn(__fmul_rn(c.b1, m), __fmul_rn(c.omb1, g));
    v = __fadd_rn(__fmul_rn(c.b2, v), __fmul_rn(c.omb2, __fmul_rn(g, g)));
    // (fminf passes over one NaN: v + 1 is above every finite root, infinite with v, and NaN with it)
    const float root = adam_root(v), u = kOdd == kLeft ? root : fminf(root, kOdd == kOf8 ? __uint_as_float(kNonFinite) : __fadd_rn(v, 1.0f));
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__fadd_rn(__fmul_rn(u, c.inv_c2), c.eps)));
    p = __fsub_rn(__fmul_rn(decay, p), __fmul_rn(__fmul_rn(c.step_size, m), inv));
    return u;
}

// The block's scale and factor from its largest finite magnitude (as bits).
__device__ __forceinline__ void block_scale(uint32_t most_bits, float& scale, float& factor) {
    const float most = __uint_as_float(most_bits);
    scale = __fmul_rn(most, 1.0f / 448.0f);
    factor = most > 1e-36f ? __fmul_rn(__frcp_rn(most), 448.0f) : 0.0f;
}
// The largest of a lane's eight roots as bits (NaN above infinity above all others).
__device__ __forceinline__ uint32_t largest(const float (&u)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(u[i]));
    return most;
}
// The moments of a lane's eight elements as the block stores them: scales, and codes ready to be rounded.  Every warp takes the
// short way unless its block has a root of 0 or something that is not finite: then the largest finite magnitude decides the
// scale, what is not finite is stored as NaN, and a root of 0 stays 0.
__device__ __forceinline__ void block_codes(float (&m)[8], float (&u)[8], uint32_t most_u, float& ms, float& vs) {
    float top_m = 0.0f, low_u = 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top_m = fmaxf(top_m, fabsf(m[i]));   // (passes over NaN)
        low_u = fminf(low_u, u[i]);
    }
    uint32_t most_m = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top_m));
    most_u = __reduce_max_sync(0xFFFFFFFFu, most_u & 0x7FFFFFFFu);
    const bool odd = max(most_m, most_u) >= kNonFinite || __any_sync(0xFFFFFFFFu, !(low_u > 0.0f));
    if (odd) {
        most_m = most_u = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (abs_bits(m[i]) >= kNonFinite) m[i] = __uint_as_float(0x7FC00000u); else most_m = max(most_m, abs_bits(m[i]));
            if (abs_bits(u[i]) >= kNonFinite) u[i] = __uint_as_float(0x7FC00000u); else most_u = max(most_u, abs_bits(u[i]));
        }
        most_m = __reduce_max_sync(0xFFFFFFFFu, most_m);
        most_u = __reduce_max_sync(0xFFFFFFFFu, most_u);
    }
    float fm, fu;
    block_scale(most_m, ms, fm);
    block_scale(most_u, vs, fu);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        m[i] = __fmul_rn(m[i], fm);
        const float s = __fmul_rn(u[i], fu);   // a positive root takes at least 2^-9, the smallest positive e4m3
        u[i] = !odd || u[i] > 0.0f ? fmaxf(s, 0.001953125f) : s;
    }
}

// What a lane reads of an aligned block.  kTail: the block that a tensor ends in; a lane past the end holds zeros, the one that the end
// falls into reads its elements one by one.
template <int kBits, typename P, typename G>
struct AdamRaw {
    Vec8<P> p;
    Vec8<G> g;
    uint32_t m[kBits / 4], v[kBits / 4];   // 8 bytes of codes, or 32 of fp32

    template <bool kTail>
    __device__ __forceinline__ void load(const AdamEntry& e, uint64_t at) {
        const P* ps = static_cast<const P*>(e.p) + at;
        const G* gs = static_cast<const G*>(e.g) + at;
        if (kTail && at + 8 > e.n) {
            p = Vec8<P>{};
            g = Vec8<G>{};
#pragma unroll
            for (int i = 0; i < kBits / 4; ++i) m[i] = v[i] = 0u;
            const int have = e.n > at ? (int)(e.n - at) : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) {
                    put(p.w, i, ps[i]);
                    put(g.w, i, gs[i]);
                    if constexpr (kBits == 32) {
                        m[i] = static_cast<const uint32_t*>(e.m)[at + i];
                        v[i] = static_cast<const uint32_t*>(e.v)[at + i];
                    } else {
                        m[i >> 2] |= (uint32_t)static_cast<const uint8_t*>(e.m)[at + i] << (8 * (i & 3));
                        v[i >> 2] |= (uint32_t)static_cast<const uint8_t*>(e.v)[at + i] << (8 * (i & 3));
                    }
                }
            return;
        }
        ld_vec(ps, p.w);
        ld_vec(gs, g.w);
        if constexpr (kBits == 32) {
            ld_vec(static_cast<const float*>(e.m) + at, m);
            ld_vec(static_cast<const float*>(e.v) + at, v);
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.m) + at);
            const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.v) + at);
            m[0] = a.x; m[1] = a.y; v[0] = b.x; v[1] = b.y;
        }
    }
    template <typename T, int kWords>
    static __device__ __forceinline__ void put(uint32_t (&w)[kWords], int i, T x) {
        if constexpr (sizeof(T) == 4) w[i] = *reinterpret_cast<const uint32_t*>(&x);
        else w[i >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t*>(&x) << (16 * (i & 1));
    }
};

template <int kBits, bool kTail, typename P, typename G>
__device__ __forceinline__ void adam_whole(const AdamEntry& e, const AdamConst& c, const AdamRaw<kBits, P, G>& raw, float& ms, float& vs, uint64_t at) {
    const int have = !kTail || at + 8 <= e.n ? 8 : e.n > at ? (int)(e.n - at) : 0;
    float p[8], g[8], m[8], v[8], u[8];
    unpack(raw.p, p);
    unpack(raw.g, g);
    if constexpr (kBits == 32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { m[i] = __uint_as_float(raw.m[i]); v[i] = __uint_as_float(raw.v[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = e4m3_values(raw.m[i >> 1] >> (16 * (i & 1))), b = e4m3_values(raw.v[i >> 1] >> (16 * (i & 1)));
            m[2 * i] = __fmul_rn(a.x, ms); m[2 * i + 1] = __fmul_rn(a.y, ms);
            v[2 * i] = __fmul_rn(b.x, vs); v[2 * i + 1] = __fmul_rn(b.y, vs);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = adam_update<kBits == 32 ? kOf32 : kLeft>(c, e.decay, g[i], p[i], m[i], v[i]);
    uint32_t most_u = 0;
    if constexpr (kBits == 8) {
        // An instruction an element costs this form 2 % of the step (0.4 G elements), so what has no finite root is mended on a way of its own.
        most_u = largest(u);
        if (most_u >= kNonFinite) {
            most_u = kNonFinite;
            const P* old = static_cast<const P*>(e.p) + at;   // (not written yet)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have && __float_as_uint(u[i]) >= kNonFinite) {
                    u[i] = __uint_as_float(kNonFinite);
                    p[i] = __fsub_rn(__fmul_rn(e.decay, to_f32(old[i])), __fmul_rn(__fmul_rn(c.step_size, m[i]), 0.0f));
                }
        }
    }
    if (kTail && have < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) {
                static_cast<P*>(e.p)[at + i] = from_f32<P>(p[i]);
                if constexpr (kBits == 32) {
                    static_cast<float*>(e.m)[at + i] = m[i];
                    static_cast<float*>(e.v)[at + i] = v[i];
                }
            }
    } else {
        store8(static_cast<P*>(e.p) + at, p);
        if constexpr (kBits == 32) {
            store8(static_cast<float*>(e.m) + at, m);
            store8(static_cast<float*>(e.v) + at, v);
        }
    }
    if constexpr (kBits == 8) {
        __syncwarp();
        block_codes(m, u, most_u, ms, vs);   // (an absent element's moments are 0)
        uint32_t mc[2], vc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mc[i] = e4m3_pair(m[4 * i], m[4 * i + 1]) | e4m3_pair(m[4 * i + 2], m[4 * i + 3]) << 16;
            vc[i] = e4m3_pair(u[4 * i], u[4 * i + 1]) | e4m3_pair(u[4 * i + 2], u[4 * i + 3]) << 16;
        }
        if (kTail && have < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) {
                    static_cast<uint8_t*>(e.m)[at + i] = (uint8_t)(mc[i >> 2] >> (8 * (i & 3)));
                    static_cast<uint8_t*>(e.v)[at + i] = (uint8_t)(vc[i >> 2] >> (8 * (i & 3)));
                }
        } else {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.m) + at) = make_uint2(mc[0], mc[1]);
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.v) + at) = make_uint2(vc[0], vc[1]);
        }
    }
}

// Blocks [b, end) of one aligned tensor, at most kAdamRun of them; the tensor may end in the last.  Their scales are read and written
// together, block b + l's by lane l: warps that wrote four bytes each into a sector they shared with others' cost the 0.4 G
// element step 410 of 1315 us.
template <int kBits, typename P, typename G>
__device__ __forceinline__ void adam_run(const AdamEntry& e, const AdamConst& c, uint64_t b, uint64_t end, int lane) {
    const int count = (int)(end - b), whole = (int)(min(end, e.n / kAdamBlock) - b);   // (end - b or one less)
    float old_ms = 0.0f, old_vs = 0.0f, new_ms = 0.0f, new_vs = 0.0f;
    if (kBits == 8 && lane < count) { old_ms = e.m_scale[b + lane]; old_vs = e.v_scale[b + lane]; }
    auto one = [&](auto tail, int k) {
        const uint64_t at = (b + k) * kAdamBlock + lane * 8;
        AdamRaw<kBits, P, G> now;
        now.template load<decltype(tail)::value>(e, at);
        float ms = 0.0f, vs = 0.0f;
        if (kBits == 8) { ms = __shfl_sync(0xFFFFFFFFu, old_ms, k); vs = __shfl_sync(0xFFFFFFFFu, old_vs, k); }
        adam_whole<kBits, decltype(tail)::value>(e, c, now, ms, vs, at);
        if (lane == k) { new_ms = ms; new_vs = vs; }
    };
#pragma unroll 1
    for (int k = 0; k < whole; ++k) one(std::false_type{}, k);
    if (whole < count) one(std::true_type{}, whole);
    if (kBits == 8 && lane < count) { e.m_scale[b + lane] = new_ms; e.v_scale[b + lane] = new_vs; }
}

// A block of a tensor that is not aligned, element by element (32 j + lane).
template <int kBits>
__device__ __forceinline__ void adam_ragged(const AdamEntry& e, const AdamConst& c, uint64_t block, int lane) {
    const int p_type = e.types & 15, g_type = (e.types >> 4) & 15;
    const uint64_t at = block * kAdamBlock + lane;
    const int have = e.n > at ? (int)min((e.n - at + 31) / 32, (uint64_t)8) : 0;
    const float ms = kBits == 8 ? e.m_scale[block] : 0.0f, vs = kBits == 8 ? e.v_scale[block] : 0.0f;
    float p[8], m[8], v[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float g = 0.0f;
        p[i] = m[i] = v[i] = u[i] = 0.0f;
        if (i < have) {
            const uint64_t k = at + 32 * i;
            p[i] = adam_load(e.p, p_type, k);
            g = adam_load(e.g, g_type, k);
            if (kBits == 32) {
                m[i] = static_cast<const float*>(e.m)[k];
                v[i] = static_cast<const float*>(e.v)[k];
            } else {
                m[i] = __fmul_rn(e4m3_values(static_cast<const uint8_t*>(e.m)[k]).x, ms);
                v[i] = __fmul_rn(e4m3_values(static_cast<const uint8_t*>(e.v)[k]).x, vs);
                v[i] = __fmul_rn(v[i], v[i]);
            }
            u[i] = adam_update<kBits == 32 ? kOf32 : kOf8>(c, e.decay, g, p[i], m[i], v[i]);
            adam_store(e.p, p_type, k, p[i]);
            if (kBits == 32) {
                static_cast<float*>(e.m)[k] = m[i];
                static_cast<float*>(e.v)[k] = v[i];
            }
        }
    }
    if (kBits == 32) return;
    float new_ms, new_vs;
    __syncwarp();
    block_codes(m, u, largest(u), new_ms, new_vs);   // (an absent element's moments are 0)
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < have) {
            static_cast<uint8_t*>(e.m)[at + 32 * i] = (uint8_t)e4m3_pair(m[i], 0.0f);
            static_cast<uint8_t*>(e.v)[at + 32 * i] = (uint8_t)e4m3_pair(u[i], 0.0f);
        }
    if (lane == 0) { e.m_scale[block] = new_ms; e.v_scale[block] = new_vs; }
}

template <int kBits, typename P>
__device__ __forceinline__ void adam_run_g(const AdamEntry& e, const AdamConst& c, uint64_t b, uint64_t end, int lane) {
    const int g_type = (e.types >> 4) & 15;
    if (g_type == LBT_F32) adam_run<kBits, P, float>(e, c, b, end, lane);
    else if (g_type == LBT_BF16) adam_run<kBits, P, __nv_bfloat16>(e, c, b, end, lane);
    else adam_run<kBits, P, __half>(e, c, b, end, lane);
}

template <int kBits, int kCap>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ AdamTable<kCap> t) {
    __shared__ uint32_t first[kCap + 1];
    __shared__ double correct;   // what the host's step sizes are multiplied by
    __shared__ float inv_c2;
    if (t.skip != nullptr && *t.skip != 0) {
        if (t.counts && blockIdx.x == 0 && threadIdx.x == 0) *t.skipped += 1;   // (nobody reads it in a launch that is held back)
        return;
    }
    for (int i = threadIdx.x; i <= t.count; i += kAdamThreads) first[i] = t.first[i];
    if (threadIdx.x == 0) {
        // The corrections are the host's, for its own step; once steps have been held back they are formed here for the smaller t.
        const int64_t missed = t.skipped != nullptr ? *t.skipped : 0, step = max(t.step - missed, (int64_t)1);
        correct = missed == 0 ? 1.0 : t.c1 / (1.0 - adam_power(t.beta1, step));
        inv_c2 = missed == 0 ? t.inv_c2 : 1.0f / (float)sqrt(1.0 - adam_power(t.beta2, step));
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    AdamConst c{t.b1, t.omb1, t.b2, t.omb2, inv_c2, t.eps, t.grad_scale != nullptr ? *t.grad_scale : 1.0f, 0.0f};
    const uint32_t all = first[t.count];
    const uint64_t stride = (uint64_t)gridDim.x * (kAdamThreads / 32);
    for (uint64_t r = (uint64_t)blockIdx.x * (kAdamThreads / 32) + (threadIdx.x >> 5); r < all; r += stride) {
        int lo = 0, hi = t.count;   // the tensor of run r: the last with first <= r (empty tensors share their successor's first)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= r) lo = mid; else hi = mid;
        }
        const AdamEntry& e = t.e[lo];
        c.step_size = (float)(e.step_size * correct);
        const uint64_t b = (r - first[lo]) * t.run, end = min(b + t.run, (e.n + kAdamBlock - 1) / kAdamBlock);
        if ((e.types >> 8) != 0) {
            const int p_type = e.types & 15;
            if (p_type == LBT_F32) adam_run_g<kBits, float>(e, c, b, end, lane);
            else if (p_type == LBT_BF16) adam_run_g<kBits, __nv_bfloat16>(e, c, b, end, lane);
            else adam_run_g<kBits, __half>(e, c, b, end, lane);
        } else {
            for (uint64_t k = b; k < end; ++k) adam_ragged<kBits>(e, c, k, lane);
        }
    }
}

template <int kBits, int kCap>
static lbt_status adamw_launch(const AdamTable<kCap>& t, cudaStream_t stream) {
    const uint64_t runs = t.first[t.count];
    if (runs == 0) return LBT_OK;
    constexpr int warps = kAdamThreads / 32;
    const int grid = (int)std::min<uint64_t>((runs + warps - 1) / warps, (uint64_t)kNumSMs * 32);
    adamw_kernel<kBits, kCap><<<grid, kAdamThreads, 0, stream>>>(t);
    return launch_status();
}

template <int kCap>
static lbt_status adamw_run(const lbt_adamw_tensor* tensors, int count, const lbt_adamw_hyper* h, const float* grad_scale,
                            const int32_t* skip, int64_t* skipped, bool* counted, cudaStream_t stream) {
    AdamTable<kCap> t{};
    const double c1 = 1.0 - pow(h->beta1, (double)h->step), c2 = sqrt(1.0 - pow(h->beta2, (double)h->step));
    t.b1 = (float)h->beta1; t.omb1 = (float)(1.0 - h->beta1);
    t.b2 = (float)h->beta2; t.omb2 = (float)(1.0 - h->beta2);
    t.inv_c2 = 1.0f / (float)c2;
    t.eps = (float)h->eps;
    t.grad_scale = grad_scale;
    t.skip = skip;
    t.skipped = skipped;
    t.step = h->step;
    t.beta1 = h->beta1; t.beta2 = h->beta2; t.c1 = c1;
    t.count = count;
    uint64_t blocks = 0, at = 0;
    for (int i = 0; i < count; ++i) blocks += (tensors[i].n + kAdamBlock - 1) / kAdamBlock;
    // Runs of eight where there are scales and blocks enough to fill the SMs four times over (0.4 G elements: 890 us where one
    // by one took 1209; 940-970 us on other boards); else block by block (fp32 states, 11.7 M elements: 55 us, in runs of eight 60 us; few blocks: all warps at work).
    t.run = h->state_bits == 8 && blocks > (uint64_t)kNumSMs * 32 * 4 ? kAdamRun : 1;
    for (int i = 0; i < count; ++i) {
        const lbt_adamw_tensor& s = tensors[i];
        AdamEntry& e = t.e[i];
        e.p = s.p; e.g = s.g; e.m = s.m; e.v = s.v; e.m_scale = s.m_scale; e.v_scale = s.v_scale; e.n = s.n;
        e.step_size = s.lr / c1;
        e.decay = (float)(1.0 - s.lr * s.weight_decay);
        // eight elements in one access: 32 bytes of fp32, 16 of a 16-bit type, 8 of codes
        auto ok = [](const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; };
        const size_t state = h->state_bits == 8 ? 8 : 32;
        const bool aligned = ok(s.p, 8 * type_size(s.p_type)) && ok(s.g, 8 * type_size(s.g_type)) && ok(s.m, state) && ok(s.v, state);
        e.types = s.p_type | s.g_type << 4 | (aligned ? 1 << 8 : 0);
        t.first[i] = (uint32_t)at;
        at += ((s.n + kAdamBlock - 1) / kAdamBlock + t.run - 1) / t.run;
    }
    t.first[count] = (uint32_t)at;
    // a step that is held back is counted once, by its first launch (the others only return)
    t.counts = skipped != nullptr && skip != nullptr && at > 0 && !*counted;
    *counted |= at > 0;
    return h->state_bits == 8 ? adamw_launch<8, kCap>(t, stream) : adamw_launch<32, kCap>(t, stream);
}

}  // namespace lbt

using namespace lbt;

extern "C" lbt_status lbt_adamw_step_ex(const lbt_adamw_tensor* tensors, int count, const lbt_adamw_hyper* h,
                                        const float* d_grad_scale, const int32_t* d_skip, int64_t* d_skipped, void* cuda_stream) {
    if (count < 0 || (count > 0 && tensors == nullptr) || h == nullptr || h->step < 1) return LBT_ERR_INVALID_ARG;
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && h->eps >= 0.0)) return LBT_ERR_INVALID_ARG;
    if (h->state_bits != 8 && h->state_bits != 32) return LBT_ERR_UNSUPPORTED_BITS;
    if ((reinterpret_cast<uintptr_t>(d_skipped) & 7) != 0) return LBT_ERR_ALIGNMENT;
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
    bool counted = false;
    for (int i = 0; i < count; i += kAdamMax) {
        const int n = std::min(count - i, kAdamMax);
        const lbt_status rc = n <= kAdamFew    ? adamw_run<kAdamFew>(tensors + i, n, h, d_grad_scale, d_skip, d_skipped, &counted, stream)
                              : n <= kAdamSome ? adamw_run<kAdamSome>(tensors + i, n, h, d_grad_scale, d_skip, d_skipped, &counted, stream)
                                               : adamw_run<kAdamMax>(tensors + i, n, h, d_grad_scale, d_skip, d_skipped, &counted, stream);
        if (rc != LBT_OK) return rc;
    }
    return LBT_OK;
}

extern "C" lbt_status lbt_adamw_step(const lbt_adamw_tensor* tensors, int count, const lbt_adamw_hyper* h,
                                     const float* d_grad_scale, const int32_t* d_skip, void* cuda_stream) {
    return lbt_adamw_step_ex(tensors, count, h, d_grad_scale, d_skip, nullptr, cuda_stream);
}
