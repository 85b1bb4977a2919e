// The norm of all gradients of a model, and clipping by it.
//
//   norm = |s| sqrt(sum over all tensors of g^2);  scale = s min(1, max_norm / norm);  out = g * scale
//
// A sum of squares of gradients spans more than fp32 holds (g beyond 1.8e19 or all below 1e-19), and 0.4 G terms in fp32 lose
// what is left.  So eight squares are added in fp32 (24 bits hold them), and these sums in 64 bits: one conversion and one
// addition for each 32-byte access.  Eight squares whose sum is too large or too small for that are formed again in 64 bits.
//
// Bound by memory: 2 or 4 bytes read an element.  A chunk of one tensor is one warp's work, whose sum goes to its own word of the
// workspace; the block that finishes last adds them in the order of the chunks, so the result does not depend on which block
// ran when.  The table of tensors travels as a kernel argument.
//
// ResNet-18 (62 tensors, 11.7 M fp32, 47 MB): 15 us from memory, whose copy rate alone would take 7.1 (the rest: start, and one block's sum of 2400 words
// behind all reading); 9.8 where they lie in L2.  0.4 G bf16 elements, norm and clipped copies: 418 us, two readings and a writing at 5.8 TB/s (the sum
// is needed before the first element is scaled).  96 ragged tensors: 11 us (in L2), the latency of two chained kernels; 16 from memory.
#include <math.h>

#include <algorithm>

#include "lbt_sm100.cuh"
#include "lbt_types.cuh"

namespace lbt {

constexpr int kNormThreads = 256;
constexpr int kNormMax = 800;       // tensors per launch: the table fits the 32 764 bytes of a kernel's arguments
constexpr int kNormFew = 40;        // smaller tables for fewer tensors (less to copy at a launch)
constexpr int kNormSome = 128;
constexpr uint64_t kNormChunk = 2048;                       // elements of the smallest chunk: eight accesses a lane
constexpr uint64_t kNormChunks = (uint64_t)kNumSMs * 16;    // chunks that fill the SMs once: larger inputs take larger chunks

struct NormEntry {
    const void* g;
    void* out;
    uint64_t n;
    int types;      // g type | out type << 4 | aligned << 8
};

template <int kCap>
struct NormTable {
    NormEntry e[kCap];
    uint32_t first[kCap + 1];   // first chunk of each tensor; first[count] = all of them
    int count;
    uint64_t chunk;             // elements, a multiple of 256
};

// Elements of a chunk: the same for all tensors of a call, whatever launch they are in.
static uint64_t norm_chunk(const lbt_grad_tensor* t, int count) {
    uint64_t total = 0;
    for (int i = 0; i < count; ++i) total += t[i].n;
    const uint64_t c = (total / kNormChunks + 255) / 256 * 256;
    return std::max(c, kNormChunk);
}

// The sum of eight squares.
__device__ __forceinline__ double squares8(const float (&g)[8]) {
    float s = 0.0f, more = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { s = fmaf(g[i], g[i], s); more = fmaf(g[4 + i], g[4 + i], more); }
    s += more;
    // (2^-90: squares that vanish next to such a sum weigh less than 2^-30 of it; the sum of all-zero gradients is 0)
    if (s >= 8.077935669463161e-28f && s <= 1.0e38f) return (double)s;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits |= abs_bits(g[i]);
    if (bits == 0) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d += (double)g[i] * (double)g[i];
    return d;
}

__device__ __forceinline__ float norm_load(const void* p, int type, uint64_t i) {
    if (type == LBT_F32) return static_cast<const float*>(p)[i];
    if (type == LBT_BF16) return to_f32(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_f32(static_cast<const __half*>(p)[i]);
}

__device__ __forceinline__ void norm_store(void* p, int type, uint64_t i, float v) {
    if (type == LBT_F32) static_cast<float*>(p)[i] = v;
    else if (type == LBT_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_f32<__half>(v);
}

// The chunk's sum over this lane's elements [at, end) of an aligned tensor; 128 bytes a lane under way at a time.
template <typename G>
__device__ __forceinline__ double chunk_squares(const G* g, uint64_t at, uint64_t end, int lane) {
    constexpr int kAhead = 16 / sizeof(G);
    double sum = 0.0;
    uint64_t i = at + 8 * lane;
    for (; i + 256 * (kAhead - 1) + 8 <= end; i += 256 * kAhead) {
        Vec8<G> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) ld_vec(g + i + 256 * k, v[k].w);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float f[8];
            unpack(v[k], f);
            sum += squares8(f);
        }
    }
    for (; i + 8 <= end; i += 256) {
        float f[8];
        load8(g + i, f);
        sum += squares8(f);
    }
    if (i < end) {   // the tensor's last elements, in one lane
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = i + k < end ? to_f32(g[i + k]) : 0.0f;
        sum += squares8(f);
    }
    return sum;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// The tensor of chunk c: the last with first <= c (empty tensors share their successor's first).
__device__ __forceinline__ int norm_owner(const uint32_t* first, int count, uint32_t c) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

// The sum over the block of one value a thread; valid in every thread.
__device__ __forceinline__ double block_sum(double v, double* space) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) space[threadIdx.x >> 5] = v;
    __syncthreads();
    v = threadIdx.x < kNormThreads / 32 ? space[threadIdx.x] : 0.0;
    if (threadIdx.x < 32) {
        v = warp_sum(v);
        if (threadIdx.x == 0) space[0] = v;
    }
    __syncthreads();
    return space[0];
}

struct NormCall {
    double* partial;        // one for each chunk of this launch
    double* launches;       // the sum of each launch
    float* norms;           // of this launch's tensors (null: not wanted)
    lbt_grad_norm_t* out;
    const float* grad_scale;
    double max_norm;
    int launch, last;       // this launch's number, the last one's
};

template <int kCap>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormTable<kCap> t, const __grid_constant__ NormCall c) {
    extern __shared__ double staged[];   // a word for each chunk
    sm100::griddep_launch_dependents();   // (the clipping behind it may set up; it waits for this grid before it reads anything)
    __shared__ uint32_t first[kCap + 1];
    __shared__ double space[kNormThreads / 32];
    __shared__ bool is_last;
    for (int i = threadIdx.x; i <= t.count; i += kNormThreads) first[i] = t.first[i];
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t all = first[t.count];
    for (uint64_t k = (uint64_t)blockIdx.x * (kNormThreads / 32) + warp; k < all; k += (uint64_t)gridDim.x * (kNormThreads / 32)) {
        const int i = norm_owner(first, t.count, (uint32_t)k);
        const NormEntry& e = t.e[i];
        const uint64_t at = (k - first[i]) * t.chunk, end = min(at + t.chunk, e.n);
        const int type = e.types & 15;
        double sum = 0.0;
        if ((e.types >> 8) != 0) {
            if (type == LBT_F32) sum = chunk_squares(static_cast<const float*>(e.g), at, end, lane);
            else if (type == LBT_BF16) sum = chunk_squares(static_cast<const __nv_bfloat16*>(e.g), at, end, lane);
            else sum = chunk_squares(static_cast<const __half*>(e.g), at, end, lane);
        } else {   // not aligned: single elements, a row of 32 of them an access
            for (uint64_t p = at + lane; p < end; p += 256) {
                float f[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) f[q] = p + 32 * q < end ? norm_load(e.g, type, p + 32 * q) : 0.0f;
                sum += squares8(f);
            }
        }
        sum = warp_sum(sum);
        if (lane == 0) c.partial[k] = sum;
    }
    // The block that arrives last finishes: every other block's sums are visible to it.
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        is_last = atomicAdd(&c.out->reserved, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!is_last) return;
    // All partial sums come on chip in one sweep, eight loads of a thread under way at a time; eight lanes then add up a tensor's.
    for (uint32_t k0 = threadIdx.x; k0 < all; k0 += 8 * kNormThreads) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = k0 + u * kNormThreads < all ? __ldcg(c.partial + k0 + u * kNormThreads) : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k0 + u * kNormThreads < all) staged[k0 + u * kNormThreads] = v[u];
    }
    __syncthreads();
    double total = 0.0;
    for (int i0 = 0; i0 < t.count; i0 += kNormThreads / 8) {   // (whole warps stay together)
        const int i = i0 + threadIdx.x / 8, j = threadIdx.x & 7;
        double sum = 0.0, more = 0.0;
        if (i < t.count) {
            uint32_t k = first[i] + j;
            const uint32_t end = first[i + 1];
            for (; k + 8 < end; k += 16) { sum += staged[k]; more += staged[k + 8]; }
            if (k < end) sum += staged[k];
        }
        sum += more;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (j == 0 && i < t.count) {
            total += sum;
            if (c.norms != nullptr) c.norms[i] = (float)sqrt(sum);
        }
    }
    total = block_sum(total, space);
    if (threadIdx.x != 0) return;
    c.out->reserved = 0;
    if (c.launch < c.last) {
        c.launches[c.launch] = total;
        return;
    }
    for (int i = 0; i < c.launch; ++i) total += __ldcg(c.launches + i);
    const float s = c.grad_scale != nullptr ? *c.grad_scale : 1.0f;
    const double norm = sqrt(total) * fabs((double)s);
    const bool bad = !(norm <= 1.7976931348623157e308);   // an infinity or NaN among the gradients, or as their scale
    c.out->norm = (float)norm;
    c.out->skip = bad ? 1 : 0;
    c.out->scale = bad ? 0.0f : norm > c.max_norm ? (float)((double)s * (c.max_norm / norm)) : s;
}

// Eight products of one access.  The last reading of g and out's only writing: neither is kept in L2.
template <typename G, typename O>
__device__ __forceinline__ void clip_chunk(const G* g, O* out, float scale, uint64_t at, uint64_t end, int lane) {
    constexpr int kAhead = 4;
    uint64_t i = at + 8 * lane;
    for (; i + 256 * (kAhead - 1) + 8 <= end; i += 256 * kAhead) {
        Vec8<G> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) ld_vec(g + i + 256 * k, v[k].w);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float f[8];
            unpack(v[k], f);
#pragma unroll
            for (int q = 0; q < 8; ++q) f[q] *= scale;
            store8(out + i + 256 * k, f);
        }
    }
    for (; i < end; i += 256) {
        if (i + 8 <= end) {
            float f[8];
            load8(g + i, f);
#pragma unroll
            for (int q = 0; q < 8; ++q) f[q] *= scale;
            store8(out + i, f);
        } else {
            for (uint64_t p = i; p < end; ++p) out[p] = from_f32<O>(to_f32(g[p]) * scale);
        }
    }
}

template <typename G>
__device__ __forceinline__ void clip_chunk_out(const NormEntry& e, float scale, uint64_t at, uint64_t end, int lane) {
    const G* g = static_cast<const G*>(e.g);
    const int type = (e.types >> 4) & 15;
    if (type == LBT_F32) clip_chunk(g, static_cast<float*>(e.out), scale, at, end, lane);
    else if (type == LBT_BF16) clip_chunk(g, static_cast<__nv_bfloat16*>(e.out), scale, at, end, lane);
    else clip_chunk(g, static_cast<__half*>(e.out), scale, at, end, lane);
}

// Chunks from the last to the first: what the norm read last is still in L2.
template <int kCap>
__global__ void __launch_bounds__(kNormThreads) grad_clip_kernel(const __grid_constant__ NormTable<kCap> t, const lbt_grad_norm_t* norm) {
    __shared__ uint32_t first[kCap + 1];
    for (int i = threadIdx.x; i <= t.count; i += kNormThreads) first[i] = t.first[i];
    sm100::griddep_wait();
    const float scale = norm->scale;
    if (norm->skip != 0) return;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const uint32_t all = first[t.count];
    for (uint64_t r = (uint64_t)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5); r < all; r += (uint64_t)gridDim.x * (kNormThreads / 32)) {
        const uint32_t k = all - 1 - (uint32_t)r;
        const int i = norm_owner(first, t.count, k);
        const NormEntry& e = t.e[i];
        if (scale == 1.0f && e.out == e.g) continue;   // in place, and nothing to do
        const uint64_t at = (uint64_t)(k - first[i]) * t.chunk, end = min(at + t.chunk, e.n);
        const int type = e.types & 15;
        if ((e.types >> 8) == 0) {
            for (uint64_t p = at + lane; p < end; p += 32) norm_store(e.out, (e.types >> 4) & 15, p, norm_load(e.g, type, p) * scale);
        } else if (type == LBT_F32) {
            clip_chunk_out<float>(e, scale, at, end, lane);
        } else if (type == LBT_BF16) {
            clip_chunk_out<__nv_bfloat16>(e, scale, at, end, lane);
        } else {
            clip_chunk_out<__half>(e, scale, at, end, lane);
        }
    }
}

// Fills the table; returns the chunks of its tensors.
template <int kCap>
static uint32_t norm_table(NormTable<kCap>& t, const lbt_grad_tensor* tensors, int count, uint64_t chunk, bool with_out) {
    uint64_t at = 0;
    t.count = count;
    t.chunk = chunk;
    for (int i = 0; i < count; ++i) {
        const lbt_grad_tensor& s = tensors[i];
        auto ok = [](const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (8 * type_size(type) - 1)) == 0; };
        const bool aligned = ok(s.g, s.g_type) && (!with_out || ok(s.out, s.out_type));
        t.e[i] = {s.g, s.out, s.n, s.g_type | s.out_type << 4 | (aligned ? 1 << 8 : 0)};
        t.first[i] = (uint32_t)at;
        at += (s.n + chunk - 1) / chunk;
    }
    t.first[count] = (uint32_t)at;
    return (uint32_t)at;
}

static int norm_grid(uint32_t chunks) {
    constexpr int warps = kNormThreads / 32;
    return (int)std::min<uint64_t>((chunks + warps - 1) / warps, (uint64_t)kNumSMs * 8);
}

template <int kCap>
static lbt_status norm_launch(const lbt_grad_tensor* tensors, int count, uint64_t chunk, const NormCall& c, uint32_t* chunks, cudaStream_t stream) {
    NormTable<kCap> t;
    *chunks = norm_table(t, tensors, count, chunk, false);
    // (chunks: kNormChunks and one more for each tensor at most: 25 KB)
    grad_norm_kernel<kCap><<<std::max(1, norm_grid(*chunks)), kNormThreads, sizeof(double) * *chunks, stream>>>(t, c);
    return launch_status();
}

template <int kCap>
static lbt_status clip_launch(const lbt_grad_tensor* tensors, int count, uint64_t chunk, const lbt_grad_norm_t* norm, cudaStream_t stream) {
    NormTable<kCap> t;
    const uint32_t chunks = norm_table(t, tensors, count, chunk, true);
    if (chunks == 0) return LBT_OK;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3(norm_grid(chunks));
    config.blockDim = dim3(kNormThreads);
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    LBT_CUDA_TRY(cudaLaunchKernelEx(&config, grad_clip_kernel<kCap>, t, norm));
    return launch_status();
}

static lbt_status norm_check(const lbt_grad_tensor* tensors, int count, bool with_out) {
    if (count < 0 || (count > 0 && tensors == nullptr)) return LBT_ERR_INVALID_ARG;
    uint64_t total = 0;
    for (int i = 0; i < count; ++i) {
        const lbt_grad_tensor& s = tensors[i];
        if (!type_ok(s.g_type) || (with_out && !type_ok(s.out_type))) return LBT_ERR_INVALID_ARG;
        if (s.n == 0) continue;
        if (s.g == nullptr || (with_out && s.out == nullptr)) return LBT_ERR_INVALID_ARG;
        auto off = [](const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (type_size(type) - 1)) != 0; };
        if (off(s.g, s.g_type) || (with_out && off(s.out, s.out_type))) return LBT_ERR_ALIGNMENT;
        if (s.n > (1ull << 40)) return LBT_ERR_UNSUPPORTED;
        total += s.n;
        if (total > (1ull << 44)) return LBT_ERR_UNSUPPORTED;
    }
    return LBT_OK;
}

}  // namespace lbt

using namespace lbt;

// One 64-bit sum for each chunk and each launch.
extern "C" size_t lbt_grad_norm_workspace_bytes(const lbt_grad_tensor* tensors, int count) {
    if (norm_check(tensors, count, false) != LBT_OK) return 0;
    const uint64_t chunk = norm_chunk(tensors, count);
    uint64_t chunks = 0;
    for (int i = 0; i < count; ++i) chunks += (tensors[i].n + chunk - 1) / chunk;
    return 8 * (chunks + (uint64_t)count / kNormMax + 1);
}

extern "C" lbt_status lbt_grad_norm(const lbt_grad_tensor* tensors, int count, double max_norm, const float* d_grad_scale,
                                    lbt_grad_norm_t* out, float* norms, void* ws, size_t ws_bytes, void* cuda_stream) {
    const lbt_status rc = norm_check(tensors, count, false);
    if (rc != LBT_OK) return rc;
    if (out == nullptr || !(max_norm > 0.0)) return LBT_ERR_INVALID_ARG;
    auto off = [](const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; };
    if (off(out, 4) || off(norms, 4) || off(d_grad_scale, 4) || off(ws, 8)) return LBT_ERR_ALIGNMENT;
    if (ws == nullptr || ws_bytes < lbt_grad_norm_workspace_bytes(tensors, count)) return LBT_ERR_WORKSPACE;
    const uint64_t chunk = norm_chunk(tensors, count);
    const int last = count > 0 ? (count - 1) / kNormMax : 0;
    double* partial = static_cast<double*>(ws) + (last + 1);
    for (int l = 0; l <= last; ++l) {
        const int at = l * kNormMax, n = std::min(count - at, kNormMax);
        const NormCall c{partial, static_cast<double*>(ws), norms != nullptr ? norms + at : nullptr, out, d_grad_scale, max_norm, l, last};
        uint32_t chunks = 0;
        const lbt_status s = n <= kNormFew    ? norm_launch<kNormFew>(tensors + at, n, chunk, c, &chunks, as_stream(cuda_stream))
                             : n <= kNormSome ? norm_launch<kNormSome>(tensors + at, n, chunk, c, &chunks, as_stream(cuda_stream))
                                              : norm_launch<kNormMax>(tensors + at, n, chunk, c, &chunks, as_stream(cuda_stream));
        if (s != LBT_OK) return s;
        partial += chunks;
    }
    return LBT_OK;
}

extern "C" lbt_status lbt_grad_clip(const lbt_grad_tensor* tensors, int count, const lbt_grad_norm_t* norm, void* cuda_stream) {
    const lbt_status rc = norm_check(tensors, count, true);
    if (rc != LBT_OK) return rc;
    if (norm == nullptr) return LBT_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(norm) & 3) != 0) return LBT_ERR_ALIGNMENT;
    const uint64_t chunk = norm_chunk(tensors, count);
    for (int at = 0; at < count; at += kNormMax) {
        const int n = std::min(count - at, kNormMax);
        const lbt_status s = n <= kNormFew    ? clip_launch<kNormFew>(tensors + at, n, chunk, norm, as_stream(cuda_stream))
                             : n <= kNormSome ? clip_launch<kNormSome>(tensors + at, n, chunk, norm, as_stream(cuda_stream))
                                              : clip_launch<kNormMax>(tensors + at, n, chunk, norm, as_stream(cuda_stream));
        if (s != LBT_OK) return s;
    }
    return LBT_OK;
}
