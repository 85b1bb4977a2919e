// Element types of the transformer-side operators (linear8, resnorm, adamw): fp32, bf16 and fp16 tensors read
// and written as fp32 values, eight at a time where they are aligned.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lbt_common.cuh"

namespace lbt {

static inline bool type_ok(int t) { return t == LBT_F32 || t == LBT_BF16 || t == LBT_F16; }
static inline size_t type_size(int t) { return t == LBT_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Eight consecutive elements as raw words: one 16-byte access for a 16-bit type, one 32-byte access for fp32.
template <typename T> struct Vec8 { uint32_t w[sizeof(T) * 2]; };

__device__ __forceinline__ void ld_vec(const void* p, uint32_t (&w)[4]) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
__device__ __forceinline__ void ld_vec(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p) : "memory");
}
__device__ __forceinline__ void st_vec(void* p, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void st_vec(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

__device__ __forceinline__ void unpack(const Vec8<float>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v.w[i]);
}
__device__ __forceinline__ void unpack(const Vec8<__nv_bfloat16>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // a bf16 is the upper half of the fp32 with the same value
        f[2 * i] = __uint_as_float(v.w[i] << 16);
        f[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const Vec8<__half>& v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&v.w[i]));
        f[2 * i] = t.x; f[2 * i + 1] = t.y;
    }
}
__device__ __forceinline__ void pack(const float (&f)[8], Vec8<float>& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.w[i] = __float_as_uint(f[i]);
}
__device__ __forceinline__ void pack(const float (&f)[8], Vec8<__nv_bfloat16>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        v.w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
}
__device__ __forceinline__ void pack(const float (&f)[8], Vec8<__half>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 t = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        v.w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
}

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
    Vec8<T> v;
    ld_vec(p, v.w);
    unpack(v, f);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
    Vec8<T> v;
    pack(f, v);
    st_vec(p, v.w);
}

// |v| as an integer that orders like the magnitude: infinities and NaN are the largest (>= kNonFinite).
constexpr uint32_t kNonFinite = 0x7F800000u;
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Symmetric 8-bit quantizer of a row (or column) whose largest magnitude is `most`: scale = most / 127, factor = 127 / most,
// each as a rounded reciprocal times the other number; a row of (nearly) zeros has scale 0 and codes 0, a row that holds
// an infinity or NaN has scale NaN and codes 0.  `most` below 1e-36 would make the factor overflow.
__device__ __forceinline__ void scale8(uint32_t most_bits, float& scale, float& factor) {
    const float most = __uint_as_float(most_bits);
    factor = 0.0f;
    scale = most_bits >= kNonFinite ? __uint_as_float(0x7FC00000u) : 0.0f;
    if (most_bits < kNonFinite && most > 1e-36f) {
        scale = __fmul_rn(most, 1.0f / 127.0f);
        factor = __fmul_rn(__frcp_rn(most), 127.0f);
    }
}
// Code of t: t * factor rounded to nearest even by adding and subtracting 1.5 * 2^23 (|t * factor| <= 127.00002); the
// low byte of the sum is the two's-complement code.  factor 0 (a row without a usable scale) gives code 0 for any t,
// an infinity or NaN included.
__device__ __forceinline__ uint32_t code8(float t, float factor) {
    return factor != 0.0f ? __float_as_uint(__fadd_rn(__fmul_rn(t, factor), 12582912.0f)) : 0u;
}
// four codes (their low bytes) as one word
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

}  // namespace lbt
