// Group norm with an activation on channels-last images, and its gradients.
//
//   per image and group: mean and variance over the group's channels at all pixels
//   k = (x - mean) rstd,  z = k w + b,  y = act(z);   e = dy act'(z),  db = sum e,  dw = sum e k,
//   dx = rstd (w e - mean_g(w e) - k mean_g(w e k))
//
// Bound by memory: x and y, then x, dy and dx.  Sums are kept by channel, whatever groups the channels fall into, so a thread owns
// eight neighbouring channels (two, or one, where rows are not aligned) and walks over pixels.  Two forms:
//   an image that fits the shared memory of a cluster (8 to 16 CTAs) is read once: each CTA keeps its share of the pixels on chip, the
//   CTAs' sums of each channel meet through the cluster, and the output is formed from what is kept;
//   a larger one is read twice: the first kernel leaves the sums of its share of an image's pixels for each channel, the second adds
//   them up for its image (a few KB from L2), and streams.
// The variance must not lose itself in a mean far from 0: shares are combined from their means and centred sums of squares, which
// are formed around the share's own mean (what is kept can be read again) or around the mean of what a thread has read so far.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "lbt_sm100.cuh"
#include "lbt_types.cuh"

namespace lbt {

constexpr int kGnThreads = 256;
constexpr int kGnAhead = 4;             // pixels whose loads a thread has under way together
constexpr int kGnPairs = 2;             // the same for two tensors at once
constexpr int kGnClusters = 16;         // CTAs that keep an image on chip, at most
constexpr int kGnJoined = 8;            // blocks of a cluster that add up their sums

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
    void* dw;
    void* db;
    float* partial;         // [N, parts, C, 2]
    int64_t ld_x, ld_y, ld_dy, ld_dx;
    int N, P, C, G, act, bits, param_type;
    int chunks, share;      // blocks that share an image's pixels, pixels of each (the last ones' may be fewer, or none)
    int joined;             // neighbouring blocks whose sums are added up before they are left in partial
    int parts, part_share;  // sums left of an image, pixels of each
    float eps;
    int kept;   // where the packs that are kept begin in shared memory
};

// kVec consecutive values of a row.
template <typename T, int kVec> struct Pack;
template <typename T> struct Pack<T, 8> {
    Vec8<T> v;
    __device__ __forceinline__ void load(const T* p) { ld_vec(p, v.w); }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack(v, f); }
    static __device__ __forceinline__ void store(T* p, const float (&f)[8]) { store8(p, f); }
};
template <typename T> struct Pack<T, 2> {
    uint32_t w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    }
    __device__ __forceinline__ void get(float (&f)[2]) const { get(w, f); }
    static __device__ __forceinline__ void get(const uint32_t* w, float (&f)[2]) {
        if constexpr (sizeof(T) == 4) {
            f[0] = __uint_as_float(w[0]);
            f[1] = __uint_as_float(w[1]);
        } else {
            const T* v = reinterpret_cast<const T*>(w);
            f[0] = to_f32(v[0]);
            f[1] = to_f32(v[1]);
        }
    }
    static __device__ __forceinline__ void store(T* p, const float (&f)[2]) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]);
        } else {
            T v[2] = {from_f32<T>(f[0]), from_f32<T>(f[1])};
            *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(v);
        }
    }
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
template <int kVec, int kThreads = kGnThreads> struct Cover {
    int vec0, vecs, lanes, vec, lane;
    bool active;
    __device__ __forceinline__ Cover(int C) {
        const int all = (C + kVec - 1) / kVec;
        vec0 = blockIdx.z * kThreads;
        vecs = min(kThreads, all - vec0);
        lanes = kThreads / vecs;
        lane = threadIdx.x / vecs;
        vec = threadIdx.x - lane * vecs;
        active = lane < lanes;
    }
    __device__ __forceinline__ int channel() const { return (vec0 + vec) * kVec; }
    __device__ __forceinline__ int width() const { return vecs * kVec; }
};

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// Sums by channel from those of the pixel lanes (part[lane][channel]): several threads take a channel's lanes in turn where there are
// more threads than channels, then one joins them.
__device__ __forceinline__ void join_lanes(const float2* part, float2* joined, int width, int lanes, float2* out) {
    const int parts = max(1, kGnThreads / width);
    for (int j = threadIdx.x; j < parts * width; j += kGnThreads) {
        const int own = j / width, i = j - own * width;
        float2 sum = make_float2(0.0f, 0.0f);
        for (int l = own; l < lanes; l += parts) {
            sum.x += part[l * width + i].x;
            sum.y += part[l * width + i].y;
        }
        if (parts == 1) out[i] = sum;
        else joined[j] = sum;
    }
    if (parts == 1) return;
    __syncthreads();
    if (threadIdx.x < width) {
        float2 sum = joined[threadIdx.x];
        for (int k = 1; k < parts; ++k) {
            sum.x += joined[k * width + threadIdx.x].x;
            sum.y += joined[k * width + threadIdx.x].y;
        }
        out[threadIdx.x] = sum;
    }
}

__device__ __forceinline__ float2 ld_cluster2(const float2* p, int cta) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(sm100::map_to_cta(sm100::smem_u32(p), cta)) : "memory");
    return v;
}

// Leaves this block's sums of each channel (in shared memory) in partial, or, with clusters, those of the cluster's blocks joined one after
// the other: join(all, pixels so far, a block's, its place among the image's).
template <typename Join> __device__ __forceinline__ void join_blocks(const GroupNormArgs& g, int n, int c0, int width, const float2* sums, Join join) {
    float2* out = reinterpret_cast<float2*>(g.partial) + ((int64_t)n * g.parts + blockIdx.x / g.joined) * g.C + c0;
    const int rank = blockIdx.x % g.joined;
    if (g.joined > 1) sm100::cluster_sync_all();
    else __syncthreads();
    for (int i = rank * kGnThreads + threadIdx.x; i < width; i += g.joined * kGnThreads) {
        float2 all = make_float2(0.0f, 0.0f);
        float pixels = 0.0f;
        if (g.joined == 1) all = join(all, pixels, sums[i], blockIdx.x);
        else
            for (int c = 0; c < g.joined; ++c) all = join(all, pixels, ld_cluster2(sums + i, c), blockIdx.x - rank + c);
        out[i] = all;
    }
    if (g.joined > 1) sm100::cluster_sync_all();   // nobody leaves before its sums have been fetched
}

// The sums of differences (s1) and of their squares (s2) of a thread's `count` values, moved from the value c around which they were formed to
// the values' mean: s1 is then 0 and s2 the centred sum.
template <int kVec> __device__ __forceinline__ void move_to_mean(float (&c)[kVec], float (&s1)[kVec], float (&s2)[kVec], int count) {
    const float each = 1.0f / (float)count;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float shift = s1[i] * each;
        s2[i] = fmaf(-s1[i], shift, s2[i]);
        c[i] += shift;
        s1[i] = 0.0f;
    }
}
// Where that is done: after 4, 8, 16, 32, 64, 96, .. values.  Around a first value that lies D away from the rest n squares add up to n D^2, of which D^2 is
// the image's: n^2 2^-24 of it would be lost.  Four of them lose 2^-18; around the mean of four the next ones' differences are a quarter, and so on.
__device__ __forceinline__ bool time_to_move(int count) { return count >= 4 && (count & min(count - 1, 31)) == 0; }

// A share's mean and centred sum of squares of each channel.  A thread sums differences from the mean of what it has read; the block's
// mean is formed from the threads' means, then every thread's sum of squares is moved to that mean.
template <typename T, int kVec>
__global__ void __launch_bounds__(kGnThreads, 4) groupnorm_stats_kernel(const __grid_constant__ GroupNormArgs g) {
    __shared__ float2 joined[kGnThreads];
    __shared__ float2 part[kGnThreads * kVec];
    __shared__ float2 sums[kGnThreads * kVec];
    sm100::griddep_launch_dependents();
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, chunk = blockIdx.x, width = cover.width();
    const int lo = chunk * g.share, hi = min(lo + g.share, g.P);
    const T* x = static_cast<const T*>(g.x) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_x + cover.channel();
    const int count = cover.active ? max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes) : 0;
    const int64_t step = cover.lanes * g.ld_x;
    float first[kVec], s1[kVec], s2[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) first[i] = s1[i] = s2[i] = 0.0f;
    for (int p = 0; p < count; p += kGnAhead) {
        Pack<T, kVec> v[kGnAhead];
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u)
            if (p + u < count) v[u].load(x + (p + u) * step);
        if (p == 0) v[0].get(first);
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u) {
            if (p + u >= count) break;
            float f[kVec];
            v[u].get(f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float d = f[i] - first[i];
                s1[i] += d;
                s2[i] = fmaf(d, d, s2[i]);
            }
        }
        if (p + kGnAhead <= count && time_to_move(p + kGnAhead)) move_to_mean(first, s1, s2, p + kGnAhead);
    }
    if (count > 0) move_to_mean(first, s1, s2, count);
    if (cover.active) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {   // the thread's mean, times its count; centred squares
            s2[i] = fmaxf(s2[i], 0.0f);
            part[cover.lane * width + cover.vec * kVec + i] = make_float2(first[i] * (float)count, 0.0f);
        }
    }
    __syncthreads();
    join_lanes(part, joined, width, cover.lanes, sums);
    __syncthreads();
    const float size = hi > lo ? 1.0f / (float)(hi - lo) : 0.0f;
    if (cover.active) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = first[i] - sums[cover.vec * kVec + i].x * size;
            part[cover.lane * width + cover.vec * kVec + i] = make_float2(0.0f, fmaf((float)count * d, d, s2[i]));
        }
    }
    __syncthreads();
    float2 mean[kVec];   // (of the channels threadIdx.x, + 256, ..: read before `sums` is written again)
#pragma unroll
    for (int i = 0; i < kVec; ++i) mean[i] = threadIdx.x + i * kGnThreads < width ? sums[threadIdx.x + i * kGnThreads] : make_float2(0.0f, 0.0f);
    __syncthreads();
    join_lanes(part, joined, width, cover.lanes, sums);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (threadIdx.x + i * kGnThreads < width) sums[threadIdx.x + i * kGnThreads].x = mean[i].x * size;
    join_blocks(g, n, cover.vec0 * kVec, width, sums, [&](float2 all, float& pixels, float2 v, int c) {
        const float own = (float)max(0, min(g.share, g.P - c * g.share)), d = v.x - all.x;
        pixels += own;
        const float share = pixels > 0.0f ? own / pixels : 0.0f;
        return make_float2(fmaf(d, share, all.x), all.y + fmaf(d * d, (pixels - own) * share, v.y));
    });
}

// A group's items (share, channel) as `lanes` neighbouring threads take them in turn, eight of them under way at a time.  f(value, pixels
// of the share, channel of the group).
constexpr int kGnItems = 8;
template <typename F>
__device__ __forceinline__ void each_item(const GroupNormArgs& g, const float2* part, int cg, int lane, int lanes, F f) {
    const int whole = lanes / cg, more = lanes - whole * cg;
    int share = lane / cg, channel = lane - share * cg;
    while (share < g.parts) {
        float2 v[kGnItems];
        int s[kGnItems], c[kGnItems];
#pragma unroll
        for (int u = 0; u < kGnItems; ++u) {
            s[u] = share;
            c[u] = channel;
            if (share < g.parts) v[u] = __ldcg(part + (int64_t)share * g.C + channel);
            channel += more;
            share += whole;
            if (channel >= cg) { channel -= cg; ++share; }
        }
#pragma unroll
        for (int u = 0; u < kGnItems; ++u)
            if (s[u] < g.parts) f(v[u], (float)min(g.part_share, g.P - s[u] * g.part_share), c[u]);
    }
}

// How the threads of a block share its groups: `lanes` (a power of two) to a group, so that all groups are in hand at once where
// there are no more groups than threads.
template <int kThreads = kGnThreads> struct GroupCover {
    int first, count, lanes, lane, own;
    template <int kVec> __device__ __forceinline__ GroupCover(const Cover<kVec, kThreads>& cover, int C, int cg) {
        first = cover.vec0 * kVec / cg;
        count = min((cover.vec0 + cover.vecs) * kVec - 1, C - 1) / cg - first + 1;
        lanes = 32;
        while (lanes > 1 && lanes * count > kThreads) lanes >>= 1;
        lane = threadIdx.x & (lanes - 1);
        own = threadIdx.x / lanes;
    }
    __device__ __forceinline__ int stride() const { return kThreads / lanes; }
    __device__ __forceinline__ float add(float v) const {
        for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
        return v;
    }
};

// The quantizer of activations (lbt_quantize_act) for one value: clip to [0, c], steps of s = c / (2^bits - 1), ties to even.
struct ActQuant {
    float c, s, levels;
    bool zero;
    __device__ __forceinline__ uint32_t operator()(float z) const {
        if (zero) return 0u;
        return (uint32_t)fminf(rintf(__fdiv_rn(fminf(fmaxf(z, 0.0f), c), s)), levels);
    }
    // eight neighbouring codes, the first of them element `at` (a multiple of 8)
    __device__ __forceinline__ void store8(const float* z, int bits, uint8_t* out, int64_t at) const {
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = (*this)(z[i]);
        if (bits <= 4) {
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) word |= q[i] << (4 * i);
            *reinterpret_cast<uint32_t*>(out + at / 2) = word;
        } else {
            *reinterpret_cast<uint2*>(out + at) = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
        }
    }
};

// The groups of neighbouring channels, one channel after the other (a division once, not for each).
struct Owner {
    int group, left;
    const int cg;
    __device__ __forceinline__ Owner(int channel, int cg_) : cg(cg_) {
        group = channel / cg;
        left = (group + 1) * cg - channel;
    }
    __device__ __forceinline__ int next() {
        const int own = group;
        if (--left == 0) { left = cg; ++group; }
        return own;
    }
};

// w and b of a block's channels, in shared memory (the kernel ahead does not write them).
template <int kThreads = kGnThreads> __device__ __forceinline__ void load_params(const GroupNormArgs& g, int c0, int width, float2* params) {
    for (int i = threadIdx.x; i < width; i += kThreads)
        params[i] = make_float2(gn_param(g.w, g.param_type, c0 + i, 1.0f), gn_param(g.b, g.param_type, c0 + i, 0.0f));
}

template <typename T, int kVec, int kAct, bool kCodes>
__global__ void __launch_bounds__(kGnThreads, 4) groupnorm_apply_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ float2 group[];   // mean and rstd of the groups that this block's channels belong to
    __shared__ float2 params[kGnThreads * kVec];
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, cg = g.C / g.G;
    const GroupCover<> groups(cover, g.C, cg);
    load_params(g, cover.vec0 * kVec, cover.width(), params);
    sm100::griddep_wait();
    for (int i0 = 0; i0 < groups.count; i0 += groups.stride()) {   // (whole warps stay together)
        const int i = min(i0 + groups.own, groups.count - 1);
        const float2* part = reinterpret_cast<const float2*>(g.partial) + (int64_t)n * g.parts * g.C + (groups.first + i) * cg;
        const float total = 1.0f / ((float)g.P * (float)cg);
        float mean = 0.0f, m2 = 0.0f;
        each_item(g, part, cg, groups.lane, groups.lanes, [&](float2 v, float pixels, int) { mean = fmaf(pixels, v.x, mean); });
        mean = groups.add(mean) * total;
        each_item(g, part, cg, groups.lane, groups.lanes, [&](float2 v, float pixels, int) { m2 += fmaf(pixels * (v.x - mean), v.x - mean, v.y); });
        m2 = groups.add(m2) * total;
        if (groups.lane == 0 && i0 + groups.own < groups.count) {
            const float rstd = rsqrtf(m2 + g.eps);
            group[i] = make_float2(mean, rstd);
            if (g.stats != nullptr && blockIdx.x == 0)   // (a group on the border of two blocks' channels: both write the same)
                reinterpret_cast<float2*>(g.stats)[(int64_t)n * g.G + groups.first + i] = make_float2(mean, rstd);
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
    Owner owner(cover.channel(), cg);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float2 s = group[owner.next() - groups.first], p = params[cover.vec * kVec + i];
        mean[i] = s.x;
        a[i] = s.y * p.x;
        b[i] = p.y;
    }
    const int lo = blockIdx.x * g.share, hi = min(lo + g.share, g.P);
    const int count = max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes);
    const T* x = static_cast<const T*>(g.x) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_x + cover.channel();
    T* y = static_cast<T*>(g.y) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_y + cover.channel();
    const int64_t step = cover.lanes * g.ld_x, y_step = cover.lanes * g.ld_y;
    for (int p = 0; p < count; p += kGnAhead) {
        Pack<T, kVec> v[kGnAhead];
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u)
            if (p + u < count) v[u].load(x + (p + u) * step);
#pragma unroll
        for (int u = 0; u < kGnAhead; ++u) {
            if (p + u >= count) break;
            float f[kVec];
            v[u].get(f);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float z = fmaf(f[i] - mean[i], a[i], b[i]);
                f[i] = kAct == LBT_ACT_NONE ? z : kAct == LBT_ACT_RELU ? (z < 0.0f ? 0.0f : z) : z * sigmoid<T>(z);   // (NaN stays)
            }
            if (!kCodes || g.y != nullptr) Pack<T, kVec>::store(y + (p + u) * y_step, f);
            if (kCodes && kVec == 8) {
                const int64_t at = ((int64_t)n * g.P + lo + cover.lane + (p + u) * cover.lanes) * g.C + cover.channel();
                quant.store8(f, g.bits, g.q, at);
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

// A share's sums of e and e k of each channel.
template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kGnThreads, 3) groupnorm_sums_kernel(const __grid_constant__ GroupNormArgs g) {
    __shared__ float2 joined[kGnThreads];
    __shared__ float2 part[kGnThreads * kVec];
    __shared__ float2 params[kGnThreads * kVec];
    sm100::griddep_launch_dependents();
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y, cg = g.C / g.G, width = cover.width();
    load_params(g, cover.vec0 * kVec, width, params);
    __syncthreads();
    if (cover.active) {
        float mean[kVec], a[kVec], b[kVec], s1[kVec], s2[kVec];   // z = (x - mean) a + b; s2: of e (x - mean)
        const float2* stats = reinterpret_cast<const float2*>(g.stats) + (int64_t)n * g.G;
        Owner owner(cover.channel(), cg);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float2 s = stats[owner.next()], p = params[cover.vec * kVec + i];
            mean[i] = s.x;
            a[i] = s.y * p.x;
            b[i] = p.y;
            s1[i] = s2[i] = 0.0f;
        }
        const int lo = blockIdx.x * g.share, hi = min(lo + g.share, g.P);
        const int count = max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes);
        const T* x = static_cast<const T*>(g.x) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_x + cover.channel();
        const T* dy = static_cast<const T*>(g.dy) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_dy + cover.channel();
        const int64_t step = cover.lanes * g.ld_x, dy_step = cover.lanes * g.ld_dy;
        for (int p = 0; p < count; p += kGnPairs) {
            Pack<T, kVec> v[kGnPairs], d[kGnPairs];
#pragma unroll
            for (int u = 0; u < kGnPairs; ++u)
                if (p + u < count) {
                    v[u].load(x + (p + u) * step);
                    d[u].load(dy + (p + u) * dy_step);
                }
#pragma unroll
            for (int u = 0; u < kGnPairs; ++u) {
                if (p + u >= count) break;
                float f[kVec], e[kVec];
                v[u].get(f);
                d[u].get(e);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float k = f[i] - mean[i];
                    if (kAct != LBT_ACT_NONE) e[i] *= act_slope<T, kAct>(fmaf(k, a[i], b[i]));
                    s1[i] += e[i];
                    s2[i] = fmaf(e[i], k, s2[i]);
                }
            }
        }
        Owner again(cover.channel(), cg);
#pragma unroll
        for (int i = 0; i < kVec; ++i) part[cover.lane * width + cover.vec * kVec + i] = make_float2(s1[i], s2[i] * stats[again.next()].y);
    }
    __syncthreads();
    join_lanes(part, joined, width, cover.lanes, params);   // (in the parameters' place)
    join_blocks(g, n, cover.vec0 * kVec, width, params, [](float2 all, float&, float2 v, int) { return make_float2(all.x + v.x, all.y + v.y); });
}

// dw and db of 32 channels: sums over images and shares, eight rows of them side by side.
__device__ __forceinline__ void param_grads(const GroupNormArgs& g, int rows, int c0, float2 (*part)[32]) {
    const int lane = threadIdx.x >> 5, c = c0 + (threadIdx.x & 31);
    float2 sum = make_float2(0.0f, 0.0f);
    if (c < g.C)
        for (int r = lane; r < rows; r += kGnItems * kGnThreads / 32) {
            float2 v[kGnItems];
#pragma unroll
            for (int u = 0; u < kGnItems; ++u) {
                const int at = r + u * (kGnThreads / 32);
                v[u] = at < rows ? __ldcg(reinterpret_cast<const float2*>(g.partial) + (int64_t)at * g.C + c) : make_float2(0.0f, 0.0f);
            }
#pragma unroll
            for (int u = 0; u < kGnItems; ++u) {
                sum.x += v[u].x;
                sum.y += v[u].y;
            }
        }
    __syncthreads();
    part[lane][threadIdx.x & 31] = sum;
    __syncthreads();
    if (lane != 0 || c >= g.C) return;
    for (int l = 1; l < kGnThreads / 32; ++l) {
        sum.x += part[l][threadIdx.x].x;
        sum.y += part[l][threadIdx.x].y;
    }
    auto put = [&](void* p, float v) {
        if (p == nullptr) return;
        if (g.param_type == LBT_F32) static_cast<float*>(p)[c] = v;
        else if (g.param_type == LBT_BF16) static_cast<__nv_bfloat16*>(p)[c] = from_f32<__nv_bfloat16>(v);
        else static_cast<__half*>(p)[c] = from_f32<__half>(v);
    };
    put(g.db, sum.x);
    put(g.dw, sum.y);
}

// The first row of blocks forms the parameters' gradients, the others an image's dx each.
template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kGnThreads, 3) groupnorm_dx_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ float2 group[];   // mean_g(w e) and mean_g(w e k) of this block's groups
    __shared__ float2 params[kGnThreads * kVec];
    if (blockIdx.y == 0) {
        __shared__ float2 part[kGnThreads / 32][32];
        sm100::griddep_wait();
        for (int c = 32 * (blockIdx.x + blockIdx.z * gridDim.x); c < g.C; c += 32 * gridDim.x * gridDim.z) param_grads(g, g.N * g.parts, c, part);
        return;
    }
    const Cover<kVec> cover(g.C);
    const int n = blockIdx.y - 1, cg = g.C / g.G;
    const GroupCover<> groups(cover, g.C, cg);
    load_params(g, cover.vec0 * kVec, cover.width(), params);
    sm100::griddep_wait();
    for (int i0 = 0; i0 < groups.count; i0 += groups.stride()) {
        const int i = min(i0 + groups.own, groups.count - 1);
        const float2* part = reinterpret_cast<const float2*>(g.partial) + (int64_t)n * g.parts * g.C + (groups.first + i) * cg;
        float e = 0.0f, ek = 0.0f;
        each_item(g, part, cg, groups.lane, groups.lanes, [&](float2 v, float, int c) {
            const float w = gn_param(g.w, g.param_type, (groups.first + i) * cg + c, 1.0f);
            e = fmaf(w, v.x, e);
            ek = fmaf(w, v.y, ek);
        });
        const float total = 1.0f / ((float)g.P * (float)cg);
        e = groups.add(e) * total;
        ek = groups.add(ek) * total;
        if (groups.lane == 0 && i0 + groups.own < groups.count) group[i] = make_float2(e, ek);
    }
    __syncthreads();
    if (!cover.active) return;
    float mean[kVec], a[kVec], b[kVec], c1[kVec], c2[kVec];   // dx = e a - c1 - (x - mean) c2
    const float2* stats = reinterpret_cast<const float2*>(g.stats) + (int64_t)n * g.G;
    Owner owner(cover.channel(), cg);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const int own = owner.next();
        const float2 s = stats[own], p = params[cover.vec * kVec + i], back = group[own - groups.first];
        mean[i] = s.x;
        a[i] = s.y * p.x;
        b[i] = p.y;
        c1[i] = s.y * back.x;
        c2[i] = s.y * s.y * back.y;
    }
    const int lo = blockIdx.x * g.share, hi = min(lo + g.share, g.P);
    const int count = max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes);
    const int64_t at = (int64_t)n * g.P + lo + cover.lane, step = cover.lanes * g.ld_x, dy_step = cover.lanes * g.ld_dy, dx_step = cover.lanes * g.ld_dx;
    const T* x = static_cast<const T*>(g.x) + at * g.ld_x + cover.channel();
    const T* dy = static_cast<const T*>(g.dy) + at * g.ld_dy + cover.channel();
    T* dx = static_cast<T*>(g.dx) + at * g.ld_dx + cover.channel();
    for (int p = 0; p < count; p += kGnPairs) {
        Pack<T, kVec> v[kGnPairs], d[kGnPairs];
#pragma unroll
        for (int u = 0; u < kGnPairs; ++u)
            if (p + u < count) {
                v[u].load(x + (p + u) * step);
                d[u].load(dy + (p + u) * dy_step);
            }
#pragma unroll
        for (int u = 0; u < kGnPairs; ++u) {
            if (p + u >= count) break;
            float f[kVec], e[kVec];
            v[u].get(f);
            d[u].get(e);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float k = f[i] - mean[i];
                if (kAct != LBT_ACT_NONE) e[i] *= act_slope<T, kAct>(fmaf(k, a[i], b[i]));
                f[i] = fmaf(e[i], a[i], -fmaf(k, c2[i], c1[i]));
            }
            Pack<T, kVec>::store(dx + (p + u) * dx_step, f);
        }
    }
}

// ---------------------------------------------------------------------------------------------- images kept on chip
// kVec fp32 values.
template <int kVec> struct Vals {
    float f[kVec];
    __device__ __forceinline__ void fill(float v) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) f[i] = v;
    }
};
template <int kVec> __device__ __forceinline__ Vals<kVec> add(const Vals<kVec>& a, const Vals<kVec>& b) {
    Vals<kVec> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.f[i] = a.f[i] + b.f[i];
    return r;
}
template <int kVec> __device__ __forceinline__ Vals<kVec> mul(const Vals<kVec>& a, const Vals<kVec>& b) {
    Vals<kVec> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.f[i] = a.f[i] * b.f[i];
    return r;
}
template <int kVec> __device__ __forceinline__ Vals<kVec> fma(const Vals<kVec>& a, const Vals<kVec>& b, const Vals<kVec>& c) {
    Vals<kVec> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) r.f[i] = fmaf(a.f[i], b.f[i], c.f[i]);
    return r;
}
template <int kVec> __device__ __forceinline__ Vals<kVec> all(float v) {
    Vals<kVec> r;
    r.fill(v);
    return r;
}
// 1 / (1 + exp(-z)); see sigmoid
template <typename T, int kVec> __device__ __forceinline__ Vals<kVec> sigmoids(const Vals<kVec>& z) {
    Vals<kVec> s;
    if (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) s.f[i] = sigmoid<T>(z.f[i]);
        return s;
    }
    s = mul(z, all<kVec>(-1.4426950408889634f));
#pragma unroll
    for (int i = 0; i < kVec; ++i) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(s.f[i]) : "f"(s.f[i]));
    s = add(s, all<kVec>(1.0f));
#pragma unroll
    for (int i = 0; i < kVec; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.f[i]) : "f"(s.f[i]));
    return s;
}

// What a thread keeps of an image in shared memory: its packs, one behind the other for all threads (pack k of the thread at
// (k threads + thread)); nobody else reads them, so that they need no barrier.
template <typename T, int kVec, int kThreads> struct Kept {
    uint8_t* base;
    __device__ __forceinline__ T* at(int k) const { return reinterpret_cast<T*>(base) + (k * kThreads + (int)threadIdx.x) * kVec; }
    __device__ __forceinline__ void fetch(int k, const T* src) const {
        if constexpr (kVec == 1) *at(k) = *src;
        if constexpr (kVec == 2)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(sm100::smem_u32(at(k))), "l"(src), "n"(2 * sizeof(T)) : "memory");
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * kVec / 16; ++i)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(sm100::smem_u32(at(k)) + 16 * i), "l"(reinterpret_cast<const uint8_t*>(src) + 16 * i) : "memory");
    }
    __device__ __forceinline__ Vals<kVec> get(int k) const {
        Vals<kVec> v;
        if constexpr (kVec == 1) {
            v.f[0] = to_f32(*at(k));
        } else if constexpr (kVec == 2) {
            Pack<T, 2> w;
            w.load(at(k));
            w.get(v.f);
        } else {
            Vec8<T> w;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) * kVec / 16; ++i) {
                const uint4 q = reinterpret_cast<const uint4*>(at(k))[i];
                w.w[4 * i] = q.x; w.w[4 * i + 1] = q.y; w.w[4 * i + 2] = q.z; w.w[4 * i + 3] = q.w;
            }
            unpack(w, reinterpret_cast<float (&)[8]>(v.f));
        }
        return v;
    }
};

// A thread's `count` packs are fetched in four parts, each worked on while the next are under way.
template <typename Fetch> __device__ __forceinline__ void fetch_parts(int count, Fetch fetch) {
    const int part = (count + 3) / 4;
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
        for (int k = q * part; k < min((q + 1) * part, count); ++k) fetch(k);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
}
template <int kLeft> __device__ __forceinline__ void parts_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
// once(k): behind the first part, k packs.
template <typename F, typename Once> __device__ __forceinline__ void as_they_come(int count, F f, Once once) {
    const int part = (count + 3) / 4;
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
        if (q == 0) parts_wait<3>();
        else if (q == 1) parts_wait<2>();
        else if (q == 2) parts_wait<1>();
        else parts_wait<0>();
#pragma unroll 2
        for (int k = q * part; k < min((q + 1) * part, count); ++k) f(k);
        if (q == 0) once(part);
    }
}

// The sum over the CTA's pixel lanes of kVec values a thread, into out[2 * channel].  `rows`: [image_rows][C].
template <int kVec, int kThreads>
__device__ __forceinline__ void lanes_sum(Vals<kVec> v, const Cover<kVec, kThreads>& cover, float* rows, float* out) {
    const int width = cover.width();
    const bool even = cover.vecs <= 32 && 32 % cover.vecs == 0;   // a warp holds whole pixels
    if (even) {
        for (int d = cover.vecs; d < 32; d <<= 1)
#pragma unroll
            for (int i = 0; i < kVec; ++i) v.f[i] += __shfl_xor_sync(0xFFFFFFFFu, v.f[i], d);
        if ((threadIdx.x & 31) < cover.vecs)
#pragma unroll
            for (int i = 0; i < kVec; ++i) rows[(threadIdx.x >> 5) * width + cover.vec * kVec + i] = v.f[i];
    } else if (cover.active) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) rows[cover.lane * width + cover.vec * kVec + i] = v.f[i];
    }
    __syncthreads();
    const int count = even ? kThreads / 32 : cover.lanes;
    for (int i = threadIdx.x; i < width; i += kThreads) {
        float s = 0.0f;
#pragma unroll 4
        for (int l = 0; l < count; ++l) s += rows[l * width + i];
        out[2 * i] = s;
    }
    __syncthreads();
}
static int image_rows(int vecs, int threads) { return vecs <= 32 && 32 % vecs == 0 ? threads / 32 : threads / vecs; }

// (as cluster_sync_all: a warp's lanes come from loops of their own lengths and meet first)
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// How shared memory begins in both kernels below; the packs that are kept come behind it, at g.kept.
struct ImageSpace {
    float2* chan;     // [C] sums of this CTA's pixels by channel
    float2* params;   // [C]
    float2* own;      // [G] sums of this CTA's pixels by group: read by the other CTAs
    float2* group;    // [G] of the whole image
    float* rows;
    __device__ __forceinline__ ImageSpace(uint8_t* at, int C, int G) {
        chan = reinterpret_cast<float2*>(at);
        params = chan + C;
        own = params + C;
        group = own + G;
        rows = reinterpret_cast<float*>(group + G);
    }
};

// One cluster an image.  Forward pass, against two kernels, inputs in L2: 64 x 56 x 56 x 64 bf16 with SiLU 21 us against 26 (27 from memory), 16 x 96 x 96 x 64
// fp16 18 against 34 (24 from memory; without an activation 14: issuing the sigmoids' instructions takes the rest), 8 x 28 x 28 x 91 bf16 9 against 16.  What is left is read
// (5500 clocks of 23000), sums through the cluster (6000) and written (7500) one after the other: an image's sums need all of it.
// Two fp32 operations an instruction, and one reciprocal for two sigmoids, gained nothing.
template <typename T, int kVec, int kAct, bool kCodes, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) groupnorm_image_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ __align__(16) uint8_t image[];
    const Cover<kVec, kThreads> cover(g.C);
    const ImageSpace space(image, g.C, g.G);
    const Kept<T, kVec, kThreads> kept{image + g.kept};
    const int n = blockIdx.y, cta = blockIdx.x, ctas = gridDim.x, cg = g.C / g.G;
    const int lo = min(cta * g.share, g.P), hi = min(lo + g.share, g.P);
    const int count = cover.active ? max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes) : 0;
    const T* x = static_cast<const T*>(g.x) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_x + cover.channel();
    const int64_t step = cover.lanes * g.ld_x;
    fetch_parts(count, [&](int k) { kept.fetch(k, x + k * step); });
    load_params<kThreads>(g, 0, g.C, space.params);
    // 16-bit values: sums of differences and of their squares while the pixels come, around a thread's first value.  Of packs of eight a thread has 27
    // at most; of pairs and single values (55, 110), the sums go on around the mean of the first quarter.  So at most 28 values stand around one of
    // them, which loses 3 x 28^2 2^-24 = 2^-13 of the variance (see time_to_move), half of that in rstd: below what 16 bits show.  Moving packs of
    // eight as well costs 3 % (16 x 96 x 96 x 64 fp16: 21.4 -> 22.0 us a call), moving pairs more often 9 % (31 x 4001 x 66 bf16; once: 1.5 %).  The squares are
    // then moved to the CTA's mean.  fp32 values are read again around the CTA's mean.
    constexpr bool kOnce = sizeof(T) == 2;
    Vals<kVec> s1 = all<kVec>(0.0f), s2 = all<kVec>(0.0f), first = all<kVec>(0.0f);
    const float own = (float)count, each = count > 0 ? 1.0f / own : 0.0f;
    as_they_come(count, [&](int k) {
        const Vals<kVec> v = kept.get(k);
        if constexpr (kOnce) {
            if (k == 0) first = mul(v, all<kVec>(-1.0f));
            const Vals<kVec> d = add(v, first);
            s1 = add(s1, d);
            s2 = fma(d, d, s2);
        } else {
            s1 = add(s1, v);
        }
    }, [&](int k) {
        if constexpr (kOnce && kVec < 8) {
            const float each = __fdividef(1.0f, (float)max(k, 1));   // (2^-22: what it leaves of s1 weighs its square)
#pragma unroll
            for (int i = 0; i < kVec; ++i) {   // (`first` is minus the value)
                const float shift = s1.f[i] * each;
                s2.f[i] = fmaf(-s1.f[i], shift, s2.f[i]);
                first.f[i] -= shift;
                s1.f[i] = 0.0f;
            }
        }
    });
    Vals<kVec> mean = s1;
    if constexpr (kOnce) {
        mean = fma(s1, all<kVec>(each), mul(first, all<kVec>(-1.0f)));   // of the thread's pixels
#pragma unroll
        for (int i = 0; i < kVec; ++i) s2.f[i] = fmaxf(fmaf(-s1.f[i], s1.f[i] * each, s2.f[i]), 0.0f);
        s1 = mul(mean, all<kVec>(own));
    }
    lanes_sum(s1, cover, space.rows, &space.chan[0].x);
    const float pixels = (float)(hi - lo), inv = hi > lo ? 1.0f / pixels : 0.0f;
    Vals<kVec> centre = all<kVec>(0.0f);   // minus this CTA's mean
    if (cover.active)
#pragma unroll
        for (int i = 0; i < kVec; ++i) centre.f[i] = -space.chan[cover.vec * kVec + i].x * inv;
    if constexpr (kOnce) {
        const Vals<kVec> d = add(mean, centre);
        if (count > 0) s2 = fma(mul(d, d), all<kVec>(own), s2);
    } else {
#pragma unroll 4
        for (int k = 0; k < count; ++k) {
            const Vals<kVec> d = add(kept.get(k), centre);
            s2 = fma(d, d, s2);
        }
    }
    lanes_sum(s2, cover, space.rows, &space.chan[0].y);
    // this CTA's mean and centred sum of squares of each group, then the image's
    const GroupCover<kThreads> groups(cover, g.C, cg);
    for (int i0 = 0; i0 < groups.count; i0 += groups.stride()) {   // (whole warps stay together)
        const int i = min(i0 + groups.own, groups.count - 1);
        float mean = 0.0f, m2 = 0.0f;
        for (int c = groups.lane; c < cg; c += groups.lanes) mean += space.chan[i * cg + c].x;
        mean = groups.add(mean) * inv / (float)cg;
        for (int c = groups.lane; c < cg; c += groups.lanes) {
            const float2 v = space.chan[i * cg + c];
            const float d = v.x * inv - mean;
            m2 += fmaf(pixels * d, d, v.y);
        }
        m2 = groups.add(m2);
        if (groups.lane == 0 && i0 + groups.own < groups.count) space.own[i] = make_float2(mean, m2);
    }
    cluster_arrive();
    cluster_wait();
    const float total = 1.0f / (float)g.P;
    for (int i0 = 0; i0 < g.G; i0 += kThreads / kGnClusters) {   // a lane for each CTA's sums of a group (whole warps stay together)
        const int i = i0 + threadIdx.x / kGnClusters, c = threadIdx.x % kGnClusters;
        const bool here = i < g.G && c < ctas;
        const float2 v = here ? ld_cluster2(space.own + i, c) : make_float2(0.0f, 0.0f);
        const float size = here ? (float)max(0, min(g.share, g.P - c * g.share)) : 0.0f;
        float mean = size * v.x;
#pragma unroll
        for (int d = 1; d < kGnClusters; d <<= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, d);
        mean *= total;
        float m2 = here ? fmaf(size * (float)cg * (v.x - mean), v.x - mean, v.y) : 0.0f;
#pragma unroll
        for (int d = 1; d < kGnClusters; d <<= 1) m2 += __shfl_xor_sync(0xFFFFFFFFu, m2, d);
        if (here && c == 0) {
            space.group[i] = make_float2(mean, rsqrtf(m2 * total / (float)cg + g.eps));
            if (g.stats != nullptr && cta == 0) reinterpret_cast<float2*>(g.stats)[(int64_t)n * g.G + i] = space.group[i];
        }
    }
    __syncthreads();
    cluster_arrive();   // this CTA reads no other's sums any more
    ActQuant quant{};
    if (kCodes) {
        quant.c = *g.clip;
        quant.levels = (float)((1 << g.bits) - 1);
        quant.s = __fdiv_rn(quant.c, quant.levels);
        quant.zero = !(quant.s > 0.0f) || isinf(quant.s);
        if (cta == 0 && n == 0 && threadIdx.x == 0) *g.q_scale = quant.zero ? 0.0f : quant.s;
    }
    if (cover.active) {
        Vals<kVec> a, b;
        Owner owner(cover.channel(), cg);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float2 s = space.group[owner.next()], p = space.params[cover.vec * kVec + i];
            centre.f[i] = -s.x;
            a.f[i] = s.y * p.x;
            b.f[i] = p.y;
        }
        T* y = static_cast<T*>(g.y) + ((int64_t)n * g.P + lo + cover.lane) * g.ld_y + cover.channel();
        const int64_t y_step = cover.lanes * g.ld_y;
#pragma unroll 2
        for (int k = 0; k < count; ++k) {
            Vals<kVec> z = fma(add(kept.get(k), centre), a, b);
            if (kAct == LBT_ACT_SILU) z = mul(z, sigmoids<T>(z));
            if (kAct == LBT_ACT_RELU)
#pragma unroll
                for (int i = 0; i < kVec; ++i) z.f[i] = z.f[i] < 0.0f ? 0.0f : z.f[i];   // (NaN stays)
            if (!kCodes || g.y != nullptr) Pack<T, kVec>::store(y + k * y_step, z.f);
            if constexpr (kCodes && kVec == 8)
                quant.store8(z.f, g.bits, g.q, ((int64_t)n * g.P + lo + cover.lane + k * cover.lanes) * g.C + cover.channel());
        }
    }
    cluster_wait();
}

// dy act'(z) at k = x - mean, z = k a + b
template <typename T, int kVec, int kAct>
__device__ __forceinline__ Vals<kVec> slopes(Vals<kVec> e, const Vals<kVec>& k, const Vals<kVec>& a, const Vals<kVec>& b) {
    if constexpr (kAct == LBT_ACT_SILU) {
        const Vals<kVec> z = fma(k, a, b), s = sigmoids<T>(z);
        e = mul(e, mul(s, fma(z, fma(s, all<kVec>(-1.0f), all<kVec>(1.0f)), all<kVec>(1.0f))));
    } else if constexpr (kAct == LBT_ACT_RELU) {
        const Vals<kVec> z = fma(k, a, b);
#pragma unroll
        for (int i = 0; i < kVec; ++i) e.f[i] = z.f[i] > 0.0f ? e.f[i] : 0.0f * e.f[i];
    }
    return e;
}

// Its gradients (64 x 56 x 56 x 64 bf16 with SiLU, inputs in L2: 37 us against 49 of two kernels, 47 from memory; the sigmoids are formed twice): x and dy are kept; partial: [N, C] sums of e and e k for the parameters' gradients.
template <typename T, int kVec, int kAct, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 3 : 2) groupnorm_image_grad_kernel(const __grid_constant__ GroupNormArgs g) {
    extern __shared__ __align__(16) uint8_t image[];
    sm100::griddep_launch_dependents();
    const Cover<kVec, kThreads> cover(g.C);
    const ImageSpace space(image, g.C, g.G);   // sums of e and e k
    const int n = blockIdx.y, cta = blockIdx.x, ctas = gridDim.x, cg = g.C / g.G;
    const int lo = min(cta * g.share, g.P), hi = min(lo + g.share, g.P);
    const int count = cover.active ? max(0, (hi - lo - cover.lane + cover.lanes - 1) / cover.lanes) : 0;
    const int most = (g.share + cover.lanes - 1) / cover.lanes;   // packs that any thread keeps of one tensor
    const Kept<T, kVec, kThreads> kept{image + g.kept}, kept_dy{image + g.kept + most * kThreads * kVec * (int)sizeof(T)};
    const int64_t at = (int64_t)n * g.P + lo + cover.lane, step = cover.lanes * g.ld_x, dy_step = cover.lanes * g.ld_dy, dx_step = cover.lanes * g.ld_dx;
    const T* x = static_cast<const T*>(g.x) + at * g.ld_x + cover.channel();
    const T* dy = static_cast<const T*>(g.dy) + at * g.ld_dy + cover.channel();
    fetch_parts(count, [&](int k) { kept.fetch(k, x + k * step); kept_dy.fetch(k, dy + k * dy_step); });
    load_params<kThreads>(g, 0, g.C, space.params);
    for (int i = threadIdx.x; i < g.G; i += kThreads) space.group[i] = reinterpret_cast<const float2*>(g.stats)[(int64_t)n * g.G + i];
    __syncthreads();
    Vals<kVec> centre, a, b, rstd, s1 = all<kVec>(0.0f), s2 = all<kVec>(0.0f);
    Owner owner(cover.channel(), cg);
    if (cover.active)
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float2 s = space.group[owner.next()], p = space.params[cover.vec * kVec + i];
            centre.f[i] = -s.x;
            a.f[i] = s.y * p.x;
            b.f[i] = p.y;
            rstd.f[i] = s.y;
        }
    as_they_come(count, [&](int i) {
        const Vals<kVec> k = add(kept.get(i), centre), e = slopes<T, kVec, kAct>(kept_dy.get(i), k, a, b);
        s1 = add(s1, e);
        s2 = fma(e, k, s2);
    }, [](int) {});
    if (cover.active) s2 = mul(s2, rstd);
    lanes_sum(s1, cover, space.rows, &space.chan[0].x);
    lanes_sum(s2, cover, space.rows, &space.chan[0].y);
    const GroupCover<kThreads> groups(cover, g.C, cg);
    for (int i0 = 0; i0 < groups.count; i0 += groups.stride()) {   // (whole warps stay together)
        const int i = min(i0 + groups.own, groups.count - 1);
        float e = 0.0f, ek = 0.0f;
        for (int c = groups.lane; c < cg; c += groups.lanes) {
            e = fmaf(space.params[i * cg + c].x, space.chan[i * cg + c].x, e);
            ek = fmaf(space.params[i * cg + c].x, space.chan[i * cg + c].y, ek);
        }
        e = groups.add(e);
        ek = groups.add(ek);
        if (groups.lane == 0 && i0 + groups.own < groups.count) space.own[i] = make_float2(e, ek);
    }
    cluster_arrive();
    cluster_wait();
    if (g.dw != nullptr || g.db != nullptr)   // each CTA adds up some of the channels for its image
        for (int i = cta * kThreads + threadIdx.x; i < g.C; i += ctas * kThreads) {
            float2 sum = make_float2(0.0f, 0.0f);
            for (int c = 0; c < ctas; ++c) {
                const float2 v = ld_cluster2(space.chan + i, c);
                sum.x += v.x;
                sum.y += v.y;
            }
            reinterpret_cast<float2*>(g.partial)[(int64_t)n * g.C + i] = sum;
        }
    const float total = 1.0f / ((float)g.P * (float)cg);
    for (int i = threadIdx.x; i < g.G; i += kThreads) {   // rstd mean_g(w e), rstd^2 mean_g(w e k)
        float2 sum = make_float2(0.0f, 0.0f);
        for (int c = 0; c < ctas; ++c) {
            const float2 v = ld_cluster2(space.own + i, c);
            sum.x += v.x;
            sum.y += v.y;
        }
        const float r = space.group[i].y;
        space.group[i] = make_float2(sum.x * total * r, sum.y * total * r * r);
    }
    __syncthreads();
    cluster_arrive();   // this CTA reads no other's sums any more
    if (g.dx != nullptr && cover.active) {
        Vals<kVec> c1, c2;   // dx = e a - c1 - (x - mean) c2
        Owner again(cover.channel(), cg);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float2 back = space.group[again.next()];
            c1.f[i] = -back.x;
            c2.f[i] = -back.y;
        }
        T* dx = static_cast<T*>(g.dx) + at * g.ld_dx + cover.channel();
        for (int i = 0; i < count; ++i) {
            const Vals<kVec> k = add(kept.get(i), centre);
            const Vals<kVec> d = fma(slopes<T, kVec, kAct>(kept_dy.get(i), k, a, b), a, fma(k, c2, c1));
            Pack<T, kVec>::store(dx + i * dx_step, d.f);
        }
    }
    cluster_wait();
}

__global__ void __launch_bounds__(kGnThreads) groupnorm_params_kernel(const __grid_constant__ GroupNormArgs g) {
    __shared__ float2 part[kGnThreads / 32][32];
    sm100::griddep_wait();
    param_grads(g, g.N, 32 * blockIdx.x, part);
}

// ---------------------------------------------------------------------------------------------- launches
// How an image's pixels are shared: four blocks to an SM, all resident at once, and four pixels a thread at least.  Every block of an image
// adds up again what all of them have left: few sums, unless shares are large.
static void gn_share(GroupNormArgs& g, int64_t N, int vec) {
    const int64_t P = g.P, C = g.C, vecs = (C + vec - 1) / vec, tiles = (vecs + kGnThreads - 1) / kGnThreads, lanes = kGnThreads / std::min<int64_t>(vecs, kGnThreads);
    const int64_t width = std::min<int64_t>(C, kGnThreads * vec), few = kGnJoined * std::max<int64_t>(2048 / width, P * C >> 20);
    const int64_t want = std::min<int64_t>((int64_t)kNumSMs * 4 / (N * tiles), few), most = (P + lanes * kGnAhead - 1) / (lanes * kGnAhead);
    const int64_t chunks = std::max<int64_t>(1, std::min(want, most));
    g.share = (int)((P + chunks - 1) / chunks);
    g.chunks = (int)((P + g.share - 1) / g.share);
    g.joined = g.chunks >= 2 * kGnJoined ? kGnJoined : 1;
    g.parts = (g.chunks + g.joined - 1) / g.joined;
    g.chunks = g.parts * g.joined;
    g.part_share = g.share * g.joined;
}

static lbt_status gn_first(void (*kernel)(GroupNormArgs), const GroupNormArgs& g, dim3 grid, cudaStream_t stream) {
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(kGnThreads);
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = g.joined;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, g));
    return launch_status();
}

// The second kernel of a pair may set up while the first one ends.
template <typename... Args>
static lbt_status gn_chained(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
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

// small packs need many threads to cover a row, and few registers each
template <int kVec> constexpr int kImageThreads = kVec == 8 ? 256 : 512;
constexpr size_t kGnSmem = 110 * 1024;   // shared memory of a CTA that keeps pixels: two of them to an SM
// Clusters of so many CTAs that are resident at once, with at most four `blocks` of those to an SM: asked once for each.
template <int kThreads> static int gn_resident(void (*kernel)(GroupNormArgs), int ctas, int blocks) {
    static std::atomic<int> known[kGnClusters + 1][5];
    int n = known[ctas][blocks].load(std::memory_order_relaxed);
    if (n > 0) return n;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(ctas);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = std::min<size_t>(kGnSmem, 228 * 1024 / blocks - 1024);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGnSmem) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &config) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = 1;
    }
    known[ctas][blocks].store(n, std::memory_order_relaxed);
    return n;
}
// CTAs of the cluster that keeps an image on chip (`tensors` of its size) with blocks of so many threads, 0 if it does not fit one;
// where the kept packs begin and the bytes of shared memory.  Of eight and more those that take the images in the fewest turns: an SM group holds one
// cluster of 16 less where its SMs are no multiple of it (16 x 96 x 96 x 64 fp16 with SiLU: 24 us with 16 CTAs an image, in two turns, against 18 with 12).
template <int kThreads>
static int gn_cluster(GroupNormArgs& g, void (*kernel)(GroupNormArgs), int vec, int resident, size_t size, int tensors, size_t* smem) {
    constexpr int threads = kThreads;
    const int vecs = (g.C + vec - 1) / vec;
    if (vecs > threads) return 0;
    const int lanes = threads / vecs;
    g.kept = (int)((sizeof(float2) * 2 * (g.C + g.G) + sizeof(float) * image_rows(vecs, threads) * g.C + 15) / 16 * 16);
    int best = 0, least = 0;
    for (int ctas = 8; ctas <= kGnClusters && least != 1; ++ctas) {
        const int share = (g.P + ctas - 1) / ctas;
        const size_t bytes = g.kept + (size_t)tensors * ((share + lanes - 1) / lanes) * threads * vec * size;
        if (bytes > kGnSmem) continue;
        const int blocks = (int)std::min<size_t>(resident, 228 * 1024 / (bytes + 1024)), n = gn_resident<kThreads>(kernel, ctas, blocks), turns = (g.N + n - 1) / n;
        if (best == 0 || turns < least) {
            best = ctas;
            least = turns;
            g.share = share;
            *smem = bytes;
        }
    }
    return best;
}

static lbt_status gn_image_launch(void (*kernel)(GroupNormArgs), const GroupNormArgs& g, int ctas, int threads, size_t smem, cudaStream_t stream) {
    LBT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGnSmem));
    if (ctas > 8) LBT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(ctas, g.N);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, g));
    return launch_status();
}

// (codes are written eight at a time: only there is the kernel that writes them)
template <typename T, int kVec, int kAct> static void (*gn_image(bool codes))(GroupNormArgs) {
    if constexpr (kVec == 8)
        if (codes) return groupnorm_image_kernel<T, kVec, kAct, true, kImageThreads<kVec>>;
    return groupnorm_image_kernel<T, kVec, kAct, false, kImageThreads<kVec>>;
}

template <typename T, int kVec, int kAct>
static lbt_status gn_forward(const GroupNormArgs& args, dim3 grid, cudaStream_t stream) {
    GroupNormArgs g = args;
    size_t smem = 0;
    const auto image = gn_image<T, kVec, kAct>(g.q != nullptr);
    if (const int ctas = gn_cluster<kImageThreads<kVec>>(g, image, kVec, 1024 / kImageThreads<kVec>, sizeof(T), 1, &smem))
        return gn_image_launch(image, g, ctas, kImageThreads<kVec>, smem, stream);
    g = args;
    if (gn_first(groupnorm_stats_kernel<T, kVec>, g, grid, stream) != LBT_OK) return LBT_ERR_CUDA;
    smem = sizeof(float2) * std::min(g.G, kGnThreads * kVec);
    if constexpr (kVec == 8)
        if (g.q != nullptr) return gn_chained(groupnorm_apply_kernel<T, kVec, kAct, true>, grid, kGnThreads, smem, stream, g);
    return gn_chained(groupnorm_apply_kernel<T, kVec, kAct, false>, grid, kGnThreads, smem, stream, g);
}

template <typename T, int kVec, int kAct>
static lbt_status gn_backward(const GroupNormArgs& args, dim3 grid, cudaStream_t stream) {
    GroupNormArgs g = args;
    size_t smem = 0;
    const auto image = groupnorm_image_grad_kernel<T, kVec, kAct, kImageThreads<kVec>>;
    if (const int ctas = gn_cluster<kImageThreads<kVec>>(g, image, kVec, kVec == 8 ? 3 : 2, sizeof(T), 2, &smem)) {
        const lbt_status s = gn_image_launch(image, g, ctas, kImageThreads<kVec>, smem, stream);
        if (s != LBT_OK || (g.dw == nullptr && g.db == nullptr)) return s;
        return gn_chained(groupnorm_params_kernel, dim3((g.C + 31) / 32), kGnThreads, 0, stream, g);
    }
    g = args;
    if (gn_first(groupnorm_sums_kernel<T, kVec, kAct>, g, grid, stream) != LBT_OK) return LBT_ERR_CUDA;
    grid.y = (g.dx != nullptr ? grid.y : 0) + 1;
    return gn_chained(groupnorm_dx_kernel<T, kVec, kAct>, grid, kGnThreads, sizeof(float2) * std::min(g.G, kGnThreads * kVec), stream, g);
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
static lbt_status gn_run_vec(GroupNormArgs& g, int64_t N, int vec, bool forward, cudaStream_t stream) {
    const int vecs = (g.C + vec - 1) / vec;
    gn_share(g, N, vec);
    const dim3 grid(g.chunks, (unsigned)N, (vecs + kGnThreads - 1) / kGnThreads);
    if (vec == 8) return gn_run_act<T, 8>(g, grid, forward, stream);
    return vec == 2 ? gn_run_act<T, 2>(g, grid, forward, stream) : gn_run_act<T, 1>(g, grid, forward, stream);
}

static lbt_status gn_run(GroupNormArgs& g, int64_t N, int type, int vec, bool forward, cudaStream_t stream) {
    if (type == LBT_F32) return gn_run_vec<float>(g, N, vec, forward, stream);
    return type == LBT_BF16 ? gn_run_vec<__nv_bfloat16>(g, N, vec, forward, stream) : gn_run_vec<__half>(g, N, vec, forward, stream);
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
    if (d->N > 65534 || d->P > (1 << 30) || d->C > (1 << 20)) return LBT_ERR_UNSUPPORTED;
    return LBT_OK;
}

// Channels of a pack: eight or two where every pixel of all tensors begins on that many elements, else one.
static int gn_vec(const lbt_groupnorm_desc& d, std::initializer_list<std::pair<const void*, int64_t>> rows) {
    for (int vec : {8, 2}) {
        bool ok = d.C % vec == 0;
        for (const auto& r : rows) ok = ok && (r.first == nullptr || (!gn_off(r.first, vec * type_size(d.type)) && r.second % vec == 0));
        if (ok) return vec;
    }
    return 1;
}

}  // namespace lbt

using namespace lbt;

extern "C" size_t lbt_groupnorm_workspace_bytes(const lbt_groupnorm_desc* desc) {
    lbt_groupnorm_desc d;
    if (gn_check(desc, &d) != LBT_OK) return 0;
    // two sums for each image, share and channel (any width of access), 256 bytes at least
    int64_t parts = 1;
    for (int vec : {1, 2, 8}) {
        GroupNormArgs g{};
        g.P = (int)d.P; g.C = (int)d.C;
        gn_share(g, std::max<int64_t>(d.N, 1), vec);
        parts = std::max<int64_t>(parts, g.parts);
    }
    return (size_t)std::max<int64_t>(256, d.N * parts * d.C * (int64_t)sizeof(float2));
}

extern "C" lbt_status lbt_groupnorm_forward(const lbt_groupnorm_desc* desc, const void* x, const void* w, const void* b, void* y, void* q, int bits,
                                            const float* d_clip, float* d_scale_out, float* stats, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_groupnorm_desc d;
    const lbt_status rc = gn_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if ((d.N > 0 && y == nullptr && q == nullptr) || (q != nullptr && (d_clip == nullptr || d_scale_out == nullptr))) return LBT_ERR_INVALID_ARG;
    if (q != nullptr && (bits < 2 || bits > 8)) return LBT_ERR_UNSUPPORTED_BITS;
    const size_t e = type_size(d.type), pe = type_size(d.param_type);
    if (gn_off(x, e) || gn_off(y, e) || gn_off(w, pe) || gn_off(b, pe) || gn_off(stats, 8) || gn_off(d_clip, 4) || gn_off(d_scale_out, 4) ||
        gn_off(q, 16) || gn_off(ws, 8))
        return LBT_ERR_ALIGNMENT;
    const int vec = gn_vec(d, {{x, d.ld_x}, {y, d.ld_y}});
    if (q != nullptr && vec != 8) return d.C % 8 != 0 ? LBT_ERR_UNSUPPORTED : LBT_ERR_ALIGNMENT;
    if (d.N == 0)   // (the codes of nothing have a scale all the same)
        return d_clip != nullptr && d_scale_out != nullptr ? lbt_quantize_act(nullptr, 0, d_clip, bits, nullptr, d_scale_out, cuda_stream) : LBT_OK;
    if (x == nullptr) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_groupnorm_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    GroupNormArgs g{};
    g.x = x; g.w = w; g.b = b; g.y = y; g.q = static_cast<uint8_t*>(q); g.clip = d_clip; g.q_scale = d_scale_out; g.stats = stats;
    g.partial = static_cast<float*>(ws);
    g.ld_x = d.ld_x; g.ld_y = d.ld_y; g.N = (int)d.N;
    g.P = (int)d.P; g.C = (int)d.C; g.G = (int)d.G; g.act = d.act; g.bits = bits; g.param_type = d.param_type; g.eps = d.eps;
    return gn_run(g, d.N, d.type, vec, true, as_stream(cuda_stream));
}

extern "C" lbt_status lbt_groupnorm_backward(const lbt_groupnorm_desc* desc, const void* dy, const void* x, const void* w, const void* b, const float* stats,
                                             void* dx, void* dw, void* db, void* ws, size_t ws_bytes, void* cuda_stream) {
    lbt_groupnorm_desc d;
    const lbt_status rc = gn_check(desc, &d);
    if (rc != LBT_OK) return rc;
    if (d.N > 0 && dx == nullptr && dw == nullptr && db == nullptr) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d.type), pe = type_size(d.param_type);
    if (gn_off(dy, e) || gn_off(x, e) || gn_off(dx, e) || gn_off(w, pe) || gn_off(b, pe) || gn_off(dw, pe) || gn_off(db, pe) || gn_off(stats, 8) || gn_off(ws, 8))
        return LBT_ERR_ALIGNMENT;
    if (d.N > 0 && (dy == nullptr || x == nullptr || stats == nullptr)) return LBT_ERR_INVALID_ARG;
    if (ws == nullptr || ws_bytes < lbt_groupnorm_workspace_bytes(desc)) return LBT_ERR_WORKSPACE;
    const cudaStream_t stream = as_stream(cuda_stream);
    GroupNormArgs g{};
    g.x = x; g.w = w; g.b = b; g.dy = dy; g.dx = dx; g.stats = const_cast<float*>(stats); g.partial = static_cast<float*>(ws);
    g.ld_x = d.ld_x; g.ld_dy = d.ld_dy; g.ld_dx = d.ld_dx;
    g.P = (int)d.P; g.C = (int)d.C; g.G = (int)d.G; g.act = d.act; g.param_type = d.param_type; g.eps = d.eps;
    g.dw = dw; g.db = db; g.N = (int)d.N;
    if (d.N == 0) {   // the sums of nothing
        if (dw != nullptr) LBT_CUDA_TRY(cudaMemsetAsync(dw, 0, pe * d.C, stream));
        if (db != nullptr) LBT_CUDA_TRY(cudaMemsetAsync(db, 0, pe * d.C, stream));
        return LBT_OK;
    }
    return gn_run(g, d.N, d.type, gn_vec(d, {{x, d.ld_x}, {dy, d.ld_dy}, {dx, d.ld_dx}}), false, stream);
}
