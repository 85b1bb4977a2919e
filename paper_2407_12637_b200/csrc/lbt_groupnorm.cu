// Group norm with an activation on channels-last images, and its gradients.
//
//   per image and group: mean and variance over the group's channels at all pixels
//   k = (x - mean) rstd,  z = k w + b,  y = act(z);   e = dy act'(z),  db = sum e,  dw = sum e k,
//   dx = rstd (w e - mean_g(w e) - k mean_g(w e k))
//
// Bound by memory: x and y, then x, dy and dx.  Two kernels a direction: the first leaves sums of its share of an image's pixels for each
// channel, the second adds them up for its image (a few KB from L2), and streams.  Sums are kept by channel, whatever groups
// the channels fall into, so a thread owns eight (or, where rows are not aligned, one) neighbouring channels and
// walks over pixels.  The variance must not lose itself in a mean far from 0: a thread sums differences from the first value it
// reads of each channel, and shares are combined from their means and centred sums of squares.
#include <math.h>

#include <algorithm>

#include "lbt_sm100.cuh"
#include "lbt_types.cuh"

namespace lbt {

constexpr int kGnThreads = 256;
constexpr int kGnAhead = 4;             // pixels whose loads a thread has under way together
constexpr int kGnMaxChunks = 148;       // shares of an image's pixels

struct GroupNormArgs {
    const void* x;
    const void* w;          // null: ones
    const void* b;          // null: zeros
    void* y;                // null: codes alone
    uint8_t* q;             // unsigned codes of y (null: none)
    const float* clip;
    float* q_scale;
    float* stats;           // [N, G, 2] mean, rstd (null: not kept)
    const void* dy;
    void* dx;
    float* partial;         // [N, chunks, C, 2]
    int64_t ld_x, ld_y, ld_dy, ld_dx;
    int P, C, G, chunks, act, bits, param_type;
    float eps;
};

// kVec consecutive values of a row.
template <typename T, int kVec> struct Pack;
template <typename T> struct Pack<T, 8> {
    Vec8<T> v;
    __device__ __forceinline__ void load(const T* p) { ld_vec(p, v.w); }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack(v, f); }
    static __device__ __forceinline__ void store(T* p, const float (&f)[8]) { store8(p, f); }
};
template <typename T> struct Pack<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(v); }
    static __device__ __forceinline__ void store(T* p, const float (&f)[1]) { *p = from_f32<T>(f[0]); }
};

__device__ __forceinline__ float gn_param(const void* p, int type, int i, float none) {
    if (p == nullptr) return none;
    if (type == LBT_F32) return static_cast<const float*>(p)[i];
    if (type == LBT_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

// 1 / (1 + exp(-z)).  16-bit results (8 or 11 bits) take the hardware's exp2 and reciprocal (about 2^-21), fp32 the exact functions.
template <typename T> __device__ __forceinline__ float sigmoid(float z) {
    if (sizeof(T) == 4) return __frcp_rn(1.0f + expf(-z));
    return __fdividef(1.0f, 1.0f + __expf(-z));
}

// How a thread block covers rows of `vecs` packs: this block's first pack, its packs, and pixels side by side.
template <int kVec> struct Cover {
    int vec0, vecs, lanes, vec, lane;
    bool active;
    __device__ __forceinline__ Cover(int C) {
        const int all = (C + kVec - 1) / kVec;
        vec0 = blockIdx.z * kGnThreads;
        vecs = min(kGnThreads, all - vec0);
        lanes = kGnThreads / vecs;
        vec = threadIdx.x % vecs;
        lane = threadIdx.x / vecs;
        active = lane < lanes;
    }
    __device__ __forceinline__ int channel() const { return (vec0 + vec) * kVec; }
};

// Pixels [lo, hi) of share c.
__device__ __forceinline__ void gn_share(int P, int chunks, int c, int& lo, int& hi) {
    lo = (int)((int64_t)P * c / chunks);
    hi = (int)((int64_t)P * (c + 1) / chunks);
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kGnThreads) groupnorm_stats_kernel(const __grid_constant__ GroupNormArgs g) {
    __shared__ float2 part[kGnThreads * kVec];   // mean and centred sum of squares by pixel lane and channel
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, chunk = blockIdx.x;
    int lo, hi;
    gn_share(g.P, g.chunks, chunk, lo, hi);
    const T* x = static_cast<const T*>(g.x) + (int64_t)n * g.P * g.ld_x + cover.channel();
    if (cover.active) {
        float first[kVec], s1[kVec], s2[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) first[i] = s1[i] = s2[i] = 0.0f;
        int p = lo + cover.lane;
        const int count = max(0, (hi - p + cover.lanes - 1) / cover.lanes);
        if (p < hi) {
            Pack<T, kVec> v;
            v.load(x + p * g.ld_x);
            v.get(first);
        }
        for (; p < hi; p += kGnAhead * cover.lanes) {
            Pack<T, kVec> v[kGnAhead];
#pragma unroll
            for (int u = 0; u < kGnAhead; ++u) {
                const int at = p + u * cover.lanes;
                v[u].load(x + (at < hi ? at : p) * g.ld_x);
            }
#pragma unroll
            for (int u = 0; u < kGnAhead; ++u) {
                if (p + u * cover.lanes >= hi) break;
                float f[kVec];
                v[u].get(f);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float d = f[i] - first[i];
                    s1[i] += d;
                    s2[i] = fmaf(d, d, s2[i]);
                }
            }
        }
        const float inv = count > 0 ? 1.0f / (float)count : 0.0f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float shift = s1[i] * inv;
            part[(cover.lane * cover.vecs + cover.vec) * kVec + i] = make_float2(first[i] + shift, fmaxf(s2[i] - s1[i] * shift, 0.0f));
        }
    }
    __syncthreads();
    const int width = cover.vecs * kVec, size = hi - lo;
    for (int i = threadIdx.x; i < width; i += kGnThreads) {
        float mean = 0.0f, m2 = 0.0f;
        for (int l = 0; l < cover.lanes; ++l) mean = fmaf((float)max(0, (size - l + cover.lanes - 1) / cover.lanes), part[l * width + i].x, mean);
        mean /= (float)size;
        for (int l = 0; l < cover.lanes; ++l) {
            const float2 v = part[l * width + i];
            const float d = v.x - mean;
            m2 += fmaf((float)max(0, (size - l + cover.lanes - 1) / cover.lanes) * d, d, v.y);
        }
        reinterpret_cast<float2*>(g.partial)[((int64_t)n * g.chunks + chunk) * g.C + cover.vec0 * kVec + i] = make_float2(mean, m2);
    }
}

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// Mean and 1 / standard deviation of one group of image n from the shares' channels, by a warp.
__device__ __forceinline__ float2 group_stats(const GroupNormArgs& g, int n, int group) {
    const int lane = threadIdx.x & 31, cg = g.C / g.G, items = g.chunks * cg;
    const float2* part = reinterpret_cast<const float2*>(g.partial) + (int64_t)n * g.chunks * g.C + group * cg;
    float mean = 0.0f, m2 = 0.0f;
    for (int i = lane; i < items; i += 32) {
        int lo, hi;
        gn_share(g.P, g.chunks, i / cg, lo, hi);
        mean = fmaf((float)(hi - lo), part[(int64_t)(i / cg) * g.C + i % cg].x, mean);
    }
    const float total = (float)g.P * (float)cg;
    mean = warp_add(mean) / total;
    for (int i = lane; i < items; i += 32) {
        int lo, hi;
        gn_share(g.P, g.chunks, i / cg, lo, hi);
        const float2 v = part[(int64_t)(i / cg) * g.C + i % cg];
        const float d = v.x - mean;
        m2 += fmaf((float)(hi - lo) * d, d, v.y);
    }
    m2 = warp_add(m2) / total;
    return make_float2(mean, rsqrtf(m2 + g.eps));
}

// The quantizer of activations (lbt_quantize_act) for one value: clip to [0, c], steps of s = c / (2^bits - 1), ties to even.
struct ActQuant {
    float c, s, levels;
    bool zero;
    __device__ __forceinline__ uint32_t operator()(float z) const {
        if (zero) return 0u;
        return (uint32_t)fminf(rintf(__fdiv_rn(fminf(fmaxf(z, 0.0f), c), s)), levels);
    }
};

template <typename T, int kVec, int kAct, bool kCodes>
__global__ void __launch_bounds__(kGnThreads) groupnorm_apply_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ float2 group[];   // mean and rstd of the groups that this block's channels belong to
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, cg = g.C / g.G;
    const int group0 = cover.vec0 * kVec / cg, group1 = min((cover.vec0 + cover.vecs) * kVec - 1, g.C - 1) / cg;
    sm100::griddep_wait();
    for (int i = group0 + (threadIdx.x >> 5); i <= group1; i += kGnThreads / 32) {
        const float2 s = group_stats(g, n, i);
        if ((threadIdx.x & 31) == 0) {
            group[i - group0] = s;
            if (g.stats != nullptr && blockIdx.x == 0) {   // (a group on the border of two blocks' channels: both write the same)
                g.stats[2 * ((int64_t)n * g.G + i)] = s.x;
                g.stats[2 * ((int64_t)n * g.G + i) + 1] = s.y;
            }
        }
    }
    ActQuant quant{};
    if (kCodes) {
        quant.c = *g.clip;
        quant.levels = (float)((1 << g.bits) - 1);
        quant.s = __fdiv_rn(quant.c, quant.levels);
        quant.zero = !(quant.s > 0.0f) || isinf(quant.s);
        if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) *g.q_scale = quant.zero ? 0.0f : quant.s;
    }
    __syncthreads();
    if (!cover.active) return;
    float mean[kVec], a[kVec], b[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = cover.channel() + i;
        const float2 s = group[c / cg - group0];
        mean[i] = s.x;
        a[i] = s.y * gn_param(g.w, g.param_type, c, 1.0f);
        b[i] = gn_param(g.b, g.param_type, c, 0.0f);
    }
    int lo, hi;
    gn_share(g.P, g.chunks, blockIdx.x, lo, hi);
    const T* x = static_cast<const T*>(g.x) + (int64_t)n * g.P * g.ld_x + cover.channel();
    T* y = static_cast<T*>(g.y) + (int64_t)n * g.P * g.ld_y + cover.channel();
    for (int p = lo + cover.lane; p < hi; p += kGnAhead * cover.lanes) {
        Pack<T, kVec> v[kGnAhead];
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u) {
            const int at = p + u * cover.lanes;
            v[u].load(x + (at < hi ? at : p) * g.ld_x);
        }
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u) {
            const int at = p + u * cover.lanes;
            if (at >= hi) break;
            float f[kVec];
            v[u].get(f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float z = fmaf(f[i] - mean[i], a[i], b[i]);
                f[i] = kAct == LBT_ACT_NONE ? z : kAct == LBT_ACT_RELU ? (z < 0.0f ? 0.0f : z) : z * sigmoid<T>(z);   // (NaN stays)
            }
            if (!kCodes || g.y != nullptr) Pack<T, kVec>::store(y + at * g.ld_y, f);
            if (kCodes && kVec == 8) {
                const int64_t at8 = ((int64_t)n * g.P + at) * g.C + cover.channel();
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < kVec; ++i) q[i] = quant(f[i]);
                if (g.bits <= 4) {
                    uint32_t word = 0;
#pragma unroll
                    for (int i = 0; i < kVec; ++i) word |= q[i] << (4 * i);
                    *reinterpret_cast<uint32_t*>(g.q + at8 / 2) = word;
                } else {
                    *reinterpret_cast<uint2*>(g.q + at8) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4 % kVec], q[5 % kVec], q[6 % kVec], q[7 % kVec]));
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- backward
template <typename T, int kAct>
__device__ __forceinline__ float act_slope(float z) {
    if (kAct == LBT_ACT_NONE) return 1.0f;
    if (kAct == LBT_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    const float s = sigmoid<T>(z);
    return s * fmaf(z, 1.0f - s, 1.0f);
}

template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kGnThreads) groupnorm_sums_kernel(const __grid_constant__ GroupNormArgs g) {
    __shared__ float2 part[kGnThreads * kVec];   // sums of e and e k by pixel lane and channel
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, cg = g.C / g.G;
    int lo, hi;
    gn_share(g.P, g.chunks, blockIdx.x, lo, hi);
    if (cover.active) {
        float mean[kVec], rstd[kVec], w[kVec], b[kVec], s1[kVec], s2[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const int c = cover.channel() + i;
            const float* s = g.stats + 2 * ((int64_t)n * g.G + c / cg);
            mean[i] = s[0];
            rstd[i] = s[1];
            w[i] = gn_param(g.w, g.param_type, c, 1.0f);
            b[i] = gn_param(g.b, g.param_type, c, 0.0f);
            s1[i] = s2[i] = 0.0f;
        }
        const T* x = static_cast<const T*>(g.x) + (int64_t)n * g.P * g.ld_x + cover.channel();
        const T* dy = static_cast<const T*>(g.dy) + (int64_t)n * g.P * g.ld_dy + cover.channel();
        for (int p = lo + cover.lane; p < hi; p += kGnAhead * cover.lanes) {
            Pack<T, kVec> v[kGnAhead], d[kGnAhead];
#pragma unroll
            for (int u = 0; u < kGnAhead; ++u) {
                const int at = p + u * cover.lanes < hi ? p + u * cover.lanes : p;
                v[u].load(x + at * g.ld_x);
                d[u].load(dy + at * g.ld_dy);
            }
#pragma unroll
            for (int u = 0; u < kGnAhead; ++u) {
                if (p + u * cover.lanes >= hi) break;
                float f[kVec], e[kVec];
                v[u].get(f);
                d[u].get(e);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float k = (f[i] - mean[i]) * rstd[i];
                    if (kAct != LBT_ACT_NONE) e[i] *= act_slope<T, kAct>(fmaf(k, w[i], b[i]));
                    s1[i] += e[i];
                    s2[i] = fmaf(e[i], k, s2[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) part[(cover.lane * cover.vecs + cover.vec) * kVec + i] = make_float2(s1[i], s2[i]);
    }
    __syncthreads();
    const int width = cover.vecs * kVec;
    for (int i = threadIdx.x; i < width; i += kGnThreads) {
        float2 sum = make_float2(0.0f, 0.0f);
        for (int l = 0; l < cover.lanes; ++l) {
            sum.x += part[l * width + i].x;
            sum.y += part[l * width + i].y;
        }
        reinterpret_cast<float2*>(g.partial)[((int64_t)n * g.chunks + blockIdx.x) * g.C + cover.vec0 * kVec + i] = sum;
    }
}

template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kGnThreads) groupnorm_dx_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ float2 group[];   // mean_g(w e) and mean_g(w e k) of this block's groups
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, cg = g.C / g.G, items = g.chunks * cg;
    const int group0 = cover.vec0 * kVec / cg, group1 = min((cover.vec0 + cover.vecs) * kVec - 1, g.C - 1) / cg;
    sm100::griddep_wait();
    for (int i = group0 + (threadIdx.x >> 5); i <= group1; i += kGnThreads / 32) {
        const float2* part = reinterpret_cast<const float2*>(g.partial) + (int64_t)n * g.chunks * g.C + i * cg;
        float e = 0.0f, ek = 0.0f;
        for (int j = threadIdx.x & 31; j < items; j += 32) {
            const float2 v = part[(int64_t)(j / cg) * g.C + j % cg];
            const float w = gn_param(g.w, g.param_type, i * cg + j % cg, 1.0f);
            e = fmaf(w, v.x, e);
            ek = fmaf(w, v.y, ek);
        }
        const float total = (float)g.P * (float)cg;
        e = warp_add(e) / total;
        ek = warp_add(ek) / total;
        if ((threadIdx.x & 31) == 0) group[i - group0] = make_float2(e, ek);
    }
    __syncthreads();
    if (!cover.active) return;
    float mean[kVec], rstd[kVec], w[kVec], b[kVec];
    float2 back[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int c = cover.channel() + i;
        const float* s = g.stats + 2 * ((int64_t)n * g.G + c / cg);
        mean[i] = s[0];
        rstd[i] = s[1];
        w[i] = gn_param(g.w, g.param_type, c, 1.0f);
        b[i] = gn_param(g.b, g.param_type, c, 0.0f);
        back[i] = group[c / cg - group0];
    }
    int lo, hi;
    gn_share(g.P, g.chunks, blockIdx.x, lo, hi);
    const T* x = static_cast<const T*>(g.x) + (int64_t)n * g.P * g.ld_x + cover.channel();
    const T* dy = static_cast<const T*>(g.dy) + (int64_t)n * g.P * g.ld_dy + cover.channel();
    T* dx = static_cast<T*>(g.dx) + (int64_t)n * g.P * g.ld_dx + cover.channel();
    constexpr int kAhead = kGnAhead / 2;
    for (int p = lo + cover.lane; p < hi; p += kAhead * cover.lanes) {
        Pack<T, kVec> v[kAhead], d[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = p + u * cover.lanes < hi ? p + u * cover.lanes : p;
            v[u].load(x + at * g.ld_x);
            d[u].load(dy + at * g.ld_dy);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = p + u * cover.lanes;
            if (at >= hi) break;
            float f[kVec], e[kVec];
            v[u].get(f);
            d[u].get(e);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float k = (f[i] - mean[i]) * rstd[i];
                if (kAct != LBT_ACT_NONE) e[i] *= act_slope<T, kAct>(fmaf(k, w[i], b[i]));
                f[i] = rstd[i] * (fmaf(e[i], w[i], -back[i].x) - k * back[i].y);
            }
            Pack<T, kVec>::store(dx + at * g.ld_dx, f);
        }
    }
}

// dw and db: sums over images and shares.  32 channels a block, eight rows of shares side by side.
__global__ void __launch_bounds__(256) groupnorm_finish_kernel(const float2* partial, int rows, int C, void* dw, void* db, int type) {
    __shared__ float2 part[8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
    float2 sum = make_float2(0.0f, 0.0f);
    sm100::griddep_wait();
    if (c < C)
        for (int r = lane; r < rows; r += 8) {
            const float2 v = partial[(int64_t)r * C + c];
            sum.x += v.x;
            sum.y += v.y;
        }
    part[lane][threadIdx.x & 31] = sum;
    __syncthreads();
    if (lane != 0 || c >= C) return;
    for (int l = 1; l < 8; ++l) {
        sum.x += part[l][threadIdx.x].x;
        sum.y += part[l][threadIdx.x].y;
    }
    auto put = [&](void* p, float v) {
        if (p == nullptr) return;
        if (type == LBT_F32) static_cast<float*>(p)[c] = v;
        else if (type == LBT_BF16) static_cast<__nv_bfloat16*>(p)[c] = from_f32<__nv_bfloat16>(v);
        else static_cast<__half*>(p)[c] = from_f32<__half>(v);
    };
    put(db, sum.x);
    put(dw, sum.y);
}

// ---------------------------------------------------------------------------------------------- launches
// Shares of an image's pixels: enough blocks to fill the SMs four times over, and four pixels a thread at least.
static int gn_chunks(int64_t N, int64_t P, int64_t C, int vec) {
    const int64_t vecs = (C + vec - 1) / vec, tiles = (vecs + kGnThreads - 1) / kGnThreads, lanes = kGnThreads / std::min<int64_t>(vecs, kGnThreads);
    const int64_t want = ((int64_t)kNumSMs * 4 + N * tiles - 1) / (N * tiles), most = (P + lanes * kGnAhead - 1) / (lanes * kGnAhead);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, kGnMaxChunks}));
}

// The second kernel of a pair may set up while the first one ends.
template <typename... Args>
static lbt_status gn_chained(void (*kernel)(Args...), dim3 grid, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(kGnThreads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, args...));
    return launch_status();
}

template <typename T, int kVec, int kAct>
static lbt_status gn_forward(const GroupNormArgs& g, dim3 grid, cudaStream_t stream) {
    groupnorm_stats_kernel<T, kVec><<<grid, kGnThreads, 0, stream>>>(g);
    if (launch_status() != LBT_OK) return LBT_ERR_CUDA;
    const size_t smem = sizeof(float2) * std::min(g.G, kGnThreads * kVec);
    if (g.q != nullptr) return gn_chained(groupnorm_apply_kernel<T, kVec, kAct, true>, grid, smem, stream, g);
    return gn_chained(groupnorm_apply_kernel<T, kVec, kAct, false>, grid, smem, stream, g);
}

template <typename T, int kVec, int kAct>
static lbt_status gn_backward(const GroupNormArgs& g, dim3 grid, cudaStream_t stream) {
    groupnorm_sums_kernel<T, kVec, kAct><<<grid, kGnThreads, 0, stream>>>(g);
    if (launch_status() != LBT_OK) return LBT_ERR_CUDA;
    if (g.dx == nullptr) return LBT_OK;
    return gn_chained(groupnorm_dx_kernel<T, kVec, kAct>, grid, sizeof(float2) * std::min(g.G, kGnThreads * kVec), stream, g);
}

template <typename T, int kVec>
static lbt_status gn_run_act(const GroupNormArgs& g, dim3 grid, bool forward, cudaStream_t stream) {
    if (forward) {
        if (g.act == LBT_ACT_NONE) return gn_forward<T, kVec, LBT_ACT_NONE>(g, grid, stream);
        if (g.act == LBT_ACT_RELU) return gn_forward<T, kVec, LBT_ACT_RELU>(g, grid, stream);
        return gn_forward<T, kVec, LBT_ACT_SILU>(g, grid, stream);
    }
    if (g.act == LBT_ACT_NONE) return gn_backward<T, kVec, LBT_ACT_NONE>(g, grid, stream);
    if (g.act == LBT_ACT_RELU) return gn_backward<T, kVec, LBT_ACT_RELU>(g, grid, stream);
    return gn_backward<T, kVec, LBT_ACT_SILU>(g, grid, stream);
}

template <typename T>
static lbt_status gn_run_vec(GroupNormArgs& g, int64_t N, bool wide, bool forward, cudaStream_t stream) {
    const int vec = wide ? 8 : 1, vecs = (g.C + vec - 1) / vec;
    g.chunks = gn_chunks(N, g.P, g.C, vec);
    const dim3 grid(g.chunks, (unsigned)N, (vecs + kGnThreads - 1) / kGnThreads);
    return wide ? gn_run_act<T, 8>(g, grid, forward, stream) : gn_run_act<T, 1>(g, grid, forward, stream);
}

static lbt_status gn_run(GroupNormArgs& g, int64_t N, int type, bool wide, bool forward, cudaStream_t stream) {
    if (type == LBT_F32) return gn_run_vec<float>(g, N, wide, forward, stream);
    return type == LBT_BF16 ? gn_run_vec<__nv_bfloat16>(g, N, wide, forward, stream) : gn_run_vec<__half>(g, N, wide, forward, stream);
}

static bool gn_off(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

static lbt_status gn_check(const lbt_groupnorm_desc* desc, lbt_groupnorm_desc* d) {
    if (desc == nullptr) return LBT_ERR_INVALID_ARG;
    *d = *desc;
    if (d->N < 0 || d->P < 1 || d->C < 1 || d->G < 1 || d->C % d->G != 0 || !type_ok(d->type) || !type_ok(d->param_type) || d->act < LBT_ACT_NONE ||
        d->act > LBT_ACT_SILU || !(d->eps >= 0.0f))
        return LBT_ERR_INVALID_ARG;
    for (int64_t* ld : {&d->ld_x, &d->ld_y, &d->ld_dy, &d->ld_dx}) {
        if (*ld == 0) *ld = d->C;
        if (*ld < d->C) return LBT_ERR_INVALID_ARG;
    }
    if (d->N > 65535 || d->P > (1 << 30) || d->C > (1 << 20)) return LBT_ERR_UNSUPPORTED;
    return LBT_OK;
}

// Whether rows of all tensors begin where packs of eight may (fp32: 32 bytes, 16-bit types: 16).
static bool gn_wide(const lbt_groupnorm_desc& d, std::initializer_list<std::pair<const void*, int64_t>> rows) {
    if (d.C % 8 != 0) return false;
    for (const auto& r : rows)
        if (r.first != nullptr && (gn_off(r.first, 8 * type_size(d.type)) || r.second % 8 != 0)) return false;
    return true;
}

}  // namespace lbt

using namespace lbt;

extern "C" size_t lbt_groupnorm_workspace_bytes(const lbt_groupnorm_desc* desc) {
    lbt_groupnorm_desc d;
    if (gn_check(desc, &d) != LBT_OK) return 0;
    // two sums for each image, share and channel (either width of access), 256 bytes at least
    const int64_t chunks = std::max(gn_chunks(std::max<int64_t>(d.N, 1), d.P, d.C, 1), gn_chunks(std::max<int64_t>(d.N, 1), d.P, d.C, 8));
    return (size_t)std::max<int64_t>(256, d.N * chunks * d.C * (int64_t)sizeof(float2));
}

extern "C" lbt_status lbt_groupnorm_forward(const lbt_groupnorm_desc* desc, const void* x, const void* w, const void* b, void* y, void* q, int bits,
                                            const float* d_clip, float* d_scale_out, float* stats, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_groupnorm_desc d;
    const lbt_status rc = gn_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if ((y == nullptr && q == nullptr) || (q != nullptr && (d_clip == nullptr || d_scale_out == nullptr))) return LBT_ERR_INVALID_ARG;
    if (q != nullptr && (bits < 2 || bits > 8)) return LBT_ERR_UNSUPPORTED_BITS;
    const size_t e = type_size(d.type), pe = type_size(d.param_type);
    if (gn_off(x, e) || gn_off(y, e) || gn_off(w, pe) || gn_off(b, pe) || gn_off(stats, 4) || gn_off(d_clip, 4) || gn_off(d_scale_out, 4) ||
        gn_off(q, 16) || gn_off(ws, 8))
        return LBT_ERR_ALIGNMENT;
    const bool wide = gn_wide(d, {{x, d.ld_x}, {y, d.ld_y}});
    if (q != nullptr && !wide) return d.C % 8 != 0 ? LBT_ERR_UNSUPPORTED : LBT_ERR_ALIGNMENT;
    if (d.N == 0) return LBT_OK;
    if (x == nullptr) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_groupnorm_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    GroupNormArgs g{};
    g.x = x; g.w = w; g.b = b; g.y = y; g.q = static_cast<uint8_t*>(q); g.clip = d_clip; g.q_scale = d_scale_out; g.stats = stats;
    g.partial = static_cast<float*>(ws);
    g.ld_x = d.ld_x; g.ld_y = d.ld_y;
    g.P = (int)d.P; g.C = (int)d.C; g.G = (int)d.G; g.act = d.act; g.bits = bits; g.param_type = d.param_type; g.eps = d.eps;
    return gn_run(g, d.N, d.type, wide, true, as_stream(cuda_stream));
}

extern "C" lbt_status lbt_groupnorm_backward(const lbt_groupnorm_desc* desc, const void* dy, const void* x, const void* w, const void* b, const float* stats,
                                             void* dx, void* dw, void* db, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_groupnorm_desc d;
    const lbt_status rc = gn_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (dx == nullptr && dw == nullptr && db == nullptr) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type), pe = type_size(d.param_type);
    if (gn_off(dy, e) || gn_off(x, e) || gn_off(dx, e) || gn_off(w, pe) || gn_off(b, pe) || gn_off(dw, pe) || gn_off(db, pe) || gn_off(stats, 4) || gn_off(ws, 8))
        return LBT_ERR_ALIGNMENT;
    if (d.N > 0 && (dy == nullptr || x == nullptr || stats == nullptr)) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_groupnorm_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    const cudaStream_t stream = as_stream(cuda_stream);
    GroupNormArgs g{};
    g.x = x; g.w = w; g.b = b; g.dy = dy; g.dx = dx; g.stats = const_cast<float*>(stats); g.partial = static_cast<float*>(ws);
    g.ld_x = d.ld_x; g.ld_dy = d.ld_dy; g.ld_dx = d.ld_dx;
    g.P = (int)d.P; g.C = (int)d.C; g.G = (int)d.G; g.act = d.act; g.param_type = d.param_type; g.eps = d.eps;
    if (d.N > 0) {
        const lbt_status s = gn_run(g, d.N, d.type, gn_wide(d, {{x, d.ld_x}, {dy, d.ld_dy}, {dx, d.ld_dx}}), false, stream);
        if (s != LBT_OK) return s;
    }
    if (dw == nullptr && db == nullptr) return LBT_OK;
    return gn_chained(groupnorm_finish_kernel, dim3((g.C + 31) / 32), 0, stream, static_cast<const float2*>(ws), (int)(d.N * g.chunks), g.C, dw, db, (int)d.param_type);
}
