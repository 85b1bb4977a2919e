// The norm after a block, the block's gate and residual scale, the residual sum and the norm before the next block:
//
//   u = N_post(h),   r = scale_x x + scale_h gate u,   y = N_pre(r)
//   N(v) = w k + b,  k = (v - mu) rstd;  layer norm: mu = mean v, rstd = (mean (v - mu)^2 + eps)^-1/2;  RMS: mu = 0
//
// forward: x and h are read once, r and y (or the 8-bit codes and the scale of each row of y) written once.
// backward: from x, h and the statistics the forward pass kept (four floats a token) everything else is formed again in fp32:
//   d = dr + N_pre'(dy),  dx = scale_x d,  du = scale_h gate d,  dh = N_post'(du),
//   N'(g) = rstd (e - [mean e] - k mean(e k)),  e = g w   (the bracket for the layer norm)
//   dw = sum_rows g k,  db = sum_rows g,  dgate = sum over the gate's rows of scale_h u d.
// Memory is the floor: two reads and two writes an element forward, four and two backward.  Neither pass reaches it: on 8192 x 4096
// bf16 (gate per 2048 rows) forward takes 55-59 us = 4.6-4.9 TB/s with 0.70 instructions a cycle and scheduler, eight warps each; a warp
// waits most for its rows ahead and for its turn.  Backward takes 127 us = 3.2 TB/s with 0.56 instructions: 118 registers leave
// four warps a scheduler (one block), too few to fill the latencies of shared memory and of the arithmetic; the barriers are a
// twentieth of a warp's time.
//
// One group of threads (a warp up to 1024 columns forward and 512 backward, a block above) owns a row, eight columns of it per
// thread and vector, so a row's sums are the group's reduction and nothing is read twice.  A group works through several rows: each thread copies its own columns
// of the rows to come into its own slots of shared memory (cp.async, up to three rows ahead), so the reductions of one row run
// under the loads of the next ones and no thread waits for another's copies.  Sums over rows: a group owns consecutive rows and
// keeps its columns' sums in registers; a second kernel adds the groups' sums in a fixed order (no atomics: a run repeats bit for bit).
#include <algorithm>

#include "lbt_types.cuh"
#include "lbt_sm100.cuh"

namespace lbt {

namespace {

struct Params {   // a parameter vector (weights, biases, gate rows)
    const void* p;
    int type;
    bool vec;
};

struct NormArgs {
    int64_t M;
    int D;
    int64_t rows_per_gate;
    int64_t step_gates, step_rest;   // forward: rows from one row of a group to its next = step_gates gate rows and step_rest rows
    bool layer, post, vec, one_gate;
    int depth;              // rows a thread copies ahead
    float eps_post, eps_pre, scale_x, scale_h, inv_d;
    const void *x, *h, *dr, *dy;
    void *r, *y, *dx, *dh;
    int64_t ld_x, ld_h, ld_r, ld_y, ld_dr, ld_dy, ld_dx, ld_dh;
    Params gate, w_post, b_post, w_pre, b_pre;
    uint8_t* q;
    int64_t ldq, q_end;     // q_end: D and its padding (what lies behind them in a row is not this matrix's)
    float* q_scale;
    float4* stats;
    // backward
    int64_t rows_each;      // consecutive rows of a group
    int64_t parts;          // groups
    float *part_w_post, *part_b_post, *part_w_pre, *part_b_pre;   // [blocks][D], null where not asked for
    float *part_gate;       // [parts][2][D]
    void* dgate;
};

// The kernels come in two forms.  P a type: activation rows and parameter vectors (of type P) are aligned and D is a multiple of 8,
// so a thread has eight consecutive columns to a vector, all there or none.  P void: any alignment, any D, parameters of any type;
// a thread's columns are kG apart, so that a warp reads consecutive elements one by one, and each column is tested.
// (The tests cost about as much as the arithmetic: on 8192 x 4096 bf16 an element takes 82 instructions forward with them, 36
// without.)
template <typename P> constexpr bool kEven = true;
template <> constexpr bool kEven<void> = false;

// Column of element i of thread t's vector g, and whether the vector has one in the row.  The launch picks the smallest group that
// covers D, so the first half of a thread's vectors always does.
template <typename P, int kG> __device__ __forceinline__ int column(int g, int i, int t) { return kEven<P> ? (g * kG + t) * 8 + i : (g * 8 + i) * kG + t; }
template <typename P, int kG, int kNV> __device__ __forceinline__ bool live(int g, int t, int D) {
    return (kEven<P> && 2 * g < kNV && kNV > 1) || column<P, kG>(g, 0, t) < D;
}
template <typename P, int kG> __device__ __forceinline__ bool full(int g, int t, int D) { return kEven<P> || column<P, kG>(g, 7, t) < D; }
// Runs body(i) for the elements of a live vector that lie in the row: without a test where all do.
template <typename P, int kG, typename Body> __device__ __forceinline__ void each(int g, int t, int D, Body body) {
    if (full<P, kG>(g, t, D)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) body(i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (column<P, kG>(g, i, t) < D) body(i);
    }
}

// A vector of a row as fp32 (`fill` behind the row's end), and back.  Only for live vectors.
template <typename P, int kG, typename T>
__device__ __forceinline__ void row_load(const T* row, int g, int t, int D, float fill, float (&f)[8]) {
    if constexpr (kEven<P>) {
        load8(row + column<P, kG>(g, 0, t), f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fill;
        each<P, kG>(g, t, D, [&](int i) { f[i] = to_f32(row[column<P, kG>(g, i, t)]); });
    }
}
template <typename P, int kG, typename T>
__device__ __forceinline__ void row_store(T* row, int g, int t, int D, const float (&f)[8]) {
    if constexpr (kEven<P>) {
        store8(row + column<P, kG>(g, 0, t), f);
    } else {
        each<P, kG>(g, t, D, [&](int i) { row[column<P, kG>(g, i, t)] = from_f32<T>(f[i]); });
    }
}
template <typename P, int kG>
__device__ __forceinline__ void param_load(const Params& p, int64_t at, int g, int t, int D, float fill, float (&f)[8]) {
    if (p.p == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = fill;
    } else if constexpr (kEven<P>) {
        row_load<P, kG>(static_cast<const P*>(p.p) + at, g, t, D, fill, f);
    } else if (p.type == LBT_F32) {
        row_load<P, kG>(static_cast<const float*>(p.p) + at, g, t, D, fill, f);
    } else if (p.type == LBT_BF16) {
        row_load<P, kG>(static_cast<const __nv_bfloat16*>(p.p) + at, g, t, D, fill, f);
    } else {
        row_load<P, kG>(static_cast<const __half*>(p.p) + at, g, t, D, fill, f);
    }
}
__device__ __forceinline__ void param_store(void* p, int type, int64_t i, float v) {
    if (type == LBT_F32) static_cast<float*>(p)[i] = v;
    else if (type == LBT_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// Sums (and a maximum) over the kG threads that own a row: a tree in each warp, then one over the warps' results, which every
// warp forms for itself.  Blocks alternate between two rows of shared memory, so one barrier a reduction is enough.
template <int kG>
struct Group {
    static constexpr int kWarps = kG / 32;
    float2 (*slots)[32];   // [2 buffers][warps]
    int turn;
    __device__ __forceinline__ float2 sum(float a, float b) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
            b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
        }
        if (kWarps > 1) {
            float2* s = slots[turn & 1];
            ++turn;
            if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = make_float2(a, b);
            __syncthreads();
            const float2 v = s[threadIdx.x & (kWarps - 1)];
            a = v.x; b = v.y;
#pragma unroll
            for (int o = kWarps / 2; o > 0; o >>= 1) {
                a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
                b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
            }
        }
        return make_float2(a, b);
    }
    __device__ __forceinline__ float sum(float a) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        if (kWarps > 1) {
            float* s = reinterpret_cast<float*>(slots[turn & 1]);
            ++turn;
            if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = a;
            __syncthreads();
            a = s[threadIdx.x & (kWarps - 1)];
#pragma unroll
            for (int o = kWarps / 2; o > 0; o >>= 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        }
        return a;
    }
    __device__ __forceinline__ uint32_t most(uint32_t v) {
        v = __reduce_max_sync(0xFFFFFFFFu, v);
        if (kWarps > 1) {
            uint32_t* s = reinterpret_cast<uint32_t*>(slots[turn & 1]);
            ++turn;
            if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
            __syncthreads();
            v = __reduce_max_sync(0xFFFFFFFFu, s[threadIdx.x & (kWarps - 1)]);
        }
        return v;
    }
};

// The rows ahead of a thread: its own columns of kArrays tensors, `depth` rows deep (0: every load is direct, as it always is in the
// general form).  What the thread copies only the thread reads, so its own wait is all it needs.
template <typename T, typename P, int kThreads, int kG, int kNV, int kArrays>
struct Ahead {
    static constexpr int kPieces = (int)sizeof(T) / 2;   // 16-byte pieces of eight elements
    static constexpr int kRowBytes = kThreads * kArrays * kNV * kPieces * 16;
    const T* base[kArrays];
    int64_t ld[kArrays];
    uint8_t* mine;      // this thread's first slot of the row that is read next
    uint8_t* begin;
    uint8_t* end;
    int depth, D, t;

    __device__ __forceinline__ void set(uint8_t* slots, int rows_ahead, int d, int thread) {
        begin = mine = slots + threadIdx.x * 16;
        end = begin + rows_ahead * kRowBytes;
        depth = kEven<P> ? rows_ahead : 0; D = d; t = thread;
    }
    // starts the copies of `row` into the slots at `to` (nothing past the last row: an empty group keeps the count)
    __device__ __forceinline__ void start(int64_t row, int64_t last, uint8_t* to) const {
        if (row < last) {
#pragma unroll
            for (int g = 0; g < kNV; ++g) {
                if (live<P, kG, kNV>(g, t, D)) {
#pragma unroll
                    for (int k = 0; k < kArrays; ++k)
                        if (k < 2 || base[k] != nullptr) {
                            const uint8_t* src = reinterpret_cast<const uint8_t*>(base[k] + row * ld[k] + column<P, kG>(g, 0, t));
#pragma unroll
                            for (int p = 0; p < kPieces; ++p)
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(sm100::smem_u32(to + ((k * kNV + g) * kPieces + p) * (kThreads * 16))),
                                             "l"(src + 16 * p) : "memory");
                        }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void begin_rows(int64_t first, int64_t step, int64_t last) const {
        for (int s = 0; s < depth; ++s) start(first + s * step, last, begin + s * kRowBytes);
    }
    // waits for the oldest of the rows ahead
    __device__ __forceinline__ void wait() const {
        if (depth >= 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (depth == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (depth == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    // the row that has been read makes room for one `depth` rows on
    __device__ __forceinline__ void advance(int64_t row, int64_t last) {
        if (depth > 0) {
            start(row, last, mine);
            mine = mine + kRowBytes == end ? begin : mine + kRowBytes;
        }
    }
    __device__ __forceinline__ void read(int64_t row, int array, int g, float (&f)[8]) const {
        if ((array >= 2 && base[array] == nullptr) || !live<P, kG, kNV>(g, t, D)) {   // (x and h, the first two, are always there)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.0f;
        } else if (depth > 0) {
            Vec8<T> v;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                const uint4 w = *reinterpret_cast<const uint4*>(mine + ((array * kNV + g) * kPieces + p) * (kThreads * 16));
                v.w[4 * p] = w.x; v.w[4 * p + 1] = w.y; v.w[4 * p + 2] = w.z; v.w[4 * p + 3] = w.w;
            }
            unpack(v, f);
        } else {
            row_load<P, kG>(base[array] + row * ld[array], g, t, D, 0.0f, f);
        }
    }
};

// Mean and reciprocal deviation of a row held in registers (columns past D hold zeros and are left out); the layer norm's mean is
// taken off the row in place.  rsqrtf: 2 ulp, against a row's sums of D roundings.
template <typename P, bool kLayer, int kG, int kNV>
__device__ __forceinline__ void row_stats(Group<kG>& grp, float (&v)[kNV][8], int t, int D, float inv_d, float eps, float& mu, float& rstd) {
    float s = 0.0f;
    mu = 0.0f;
    if (kLayer) {
#pragma unroll
        for (int g = 0; g < kNV; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[g][i];
        mu = grp.sum(s) * inv_d;
        s = 0.0f;
#pragma unroll
        for (int g = 0; g < kNV; ++g)
            if (live<P, kG, kNV>(g, t, D)) each<P, kG>(g, t, D, [&](int i) { v[g][i] -= mu; });
    }
#pragma unroll
    for (int g = 0; g < kNV; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[g][i] * v[g][i];
    rstd = rsqrtf(grp.sum(s) * inv_d + eps);
}

template <int kG> constexpr int kBlock = kG < 128 ? 256 : kG;   // threads of a block: groups of a warp share one
// Blocks of the forward pass on an SM: 1024 threads of 64 registers where sixteen columns a thread fit them, else 768 of 85.
template <int kG, int kNV> constexpr int kForwardBlocks = (kG == 128 || kG == 256) && kNV <= 2 ? 1024 / kBlock<kG> : kBlock<kG> <= 768 ? 768 / kBlock<kG> : 1;

template <typename T, typename P, int kG, int kNV, bool kLayer>
__global__ void __launch_bounds__(kBlock<kG>, kForwardBlocks<kG, kNV>) resnorm_forward_kernel(const __grid_constant__ NormArgs a) {
    constexpr int kThreads = kBlock<kG>, kRows = kThreads / kG;
    extern __shared__ uint8_t ahead_slots[];
    __shared__ float2 slots[2][32];
    Group<kG> grp{slots, 0};
    // (a block that owns a row keeps everything about it uniform)
    const int t = kRows == 1 ? threadIdx.x : threadIdx.x % kG, D = a.D;
    const int64_t step = (int64_t)gridDim.x * kRows, first = kRows == 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kRows + threadIdx.x / kG;
    Ahead<T, P, kThreads, kG, kNV, 2> in{{static_cast<const T*>(a.x), static_cast<const T*>(a.h)}, {a.ld_x, a.ld_h}};
    in.set(ahead_slots, a.depth, D, t);
    in.begin_rows(first, step, a.M);
    // the gate row of `row` and the row's place in it, moved on from row to row without a division
    int64_t gate_row = 0, gate_place = 0;
    if (!a.one_gate) { gate_row = first / a.rows_per_gate; gate_place = first - gate_row * a.rows_per_gate; }
    for (int64_t row = first; row < a.M; row += step) {
        float h[kNV][8], r[kNV][8];
        in.wait();
#pragma unroll
        for (int g = 0; g < kNV; ++g) {
            in.read(row, 1, g, h[g]);
            in.read(row, 0, g, r[g]);
        }
        in.advance(row + a.depth * step, a.M);
        float mu1 = 0.0f, rstd1 = 1.0f, mu2 = 0.0f, rstd2 = 1.0f;
        if (a.post) row_stats<P, kLayer, kG, kNV>(grp, h, t, D, a.inv_d, a.eps_post, mu1, rstd1);
        T* out = static_cast<T*>(a.r) + row * a.ld_r;
#pragma unroll
        for (int g = 0; g < kNV; ++g) {
            if (!live<P, kG, kNV>(g, t, D)) continue;   // (r holds zeros there)
            if (a.post) {
                float w[8], b[8];
                param_load<P, kG>(a.w_post, 0, g, t, D, 1.0f, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[g][i] = h[g][i] * rstd1 * w[i];
                if (kLayer && a.b_post.p != nullptr) {
                    param_load<P, kG>(a.b_post, 0, g, t, D, 0.0f, b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[g][i] += b[i];
                }
            }
            if (a.gate.p != nullptr) {
                float gt[8];
                param_load<P, kG>(a.gate, gate_row * D, g, t, D, 1.0f, gt);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[g][i] *= gt[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) r[g][i] = a.scale_x * r[g][i] + a.scale_h * h[g][i];   // (x = h = 0 past the end: so are r and y)
            row_store<P, kG>(out, g, t, D, r[g]);
        }
        if (a.y != nullptr || a.q != nullptr) {
            row_stats<P, kLayer, kG, kNV>(grp, r, t, D, a.inv_d, a.eps_pre, mu2, rstd2);
            uint32_t most = 0;
#pragma unroll
            for (int g = 0; g < kNV; ++g) {
                if (!live<P, kG, kNV>(g, t, D)) continue;
                float w[8];
                param_load<P, kG>(a.w_pre, 0, g, t, D, 1.0f, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) r[g][i] = r[g][i] * rstd2 * w[i];
                if (kLayer && a.b_pre.p != nullptr) {
                    param_load<P, kG>(a.b_pre, 0, g, t, D, 0.0f, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[g][i] += w[i];
                }
                if (a.y != nullptr) row_store<P, kG>(static_cast<T*>(a.y) + row * a.ld_y, g, t, D, r[g]);
            }
            if (a.q != nullptr) {
                float s, factor;
#pragma unroll
                for (int g = 0; g < kNV; ++g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) most = max(most, abs_bits(r[g][i]));
                scale8(grp.most(most), s, factor);
                if (t == 0) a.q_scale[row] = s;
#pragma unroll
                for (int g = 0; g < kNV; ++g) {
                    uint32_t k[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) k[i] = code8(r[g][i], factor);
                    uint8_t* to = a.q + row * a.ldq;
                    if constexpr (kEven<P>) {
                        const int c = column<P, kG>(g, 0, t);
                        if (c < a.q_end) *reinterpret_cast<uint2*>(to + c) = make_uint2(pack4(k[0], k[1], k[2], k[3]), pack4(k[4], k[5], k[6], k[7]));
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (column<P, kG>(g, i, t) < a.q_end) to[column<P, kG>(g, i, t)] = (uint8_t)k[i];
                    }
                }
            }
        }
        if (a.stats != nullptr && t == 0) a.stats[row] = make_float4(mu1, rstd1, mu2, rstd2);
        if (!a.one_gate) {
            gate_row += a.step_gates;
            gate_place += a.step_rest;
            if (gate_place >= a.rows_per_gate) { gate_place -= a.rows_per_gate; ++gate_row; }
        }
    }
}

// Adds a group's column sums of one array into what the second kernel adds up: a block's warps (groups of one warp) first meet in
// shared memory, in order.
template <typename P, int kG, int kNV>
__device__ __forceinline__ void publish(float* part, const float (&acc)[kNV][8], int t, int D, float* meet) {
    if (part == nullptr) return;   // uniform
    constexpr int kRows = kBlock<kG> / kG;
    float* dst = part + (int64_t)blockIdx.x * D;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int g = 0; g < kNV; ++g)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (column<P, kG>(g, i, t) < D) dst[column<P, kG>(g, i, t)] = acc[g][i];
    } else {
        for (int w = 0; w < kRows; ++w) {
            __syncthreads();
            if ((int)threadIdx.x / kG == w) {
#pragma unroll
                for (int g = 0; g < kNV; ++g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = column<P, kG>(g, i, t);
                        meet[c] = w == 0 ? acc[g][i] : meet[c] + acc[g][i];
                    }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += blockDim.x) dst[c] = meet[c];
    }
}

template <typename T, typename P, int kG, int kNV, bool kLayer>
__global__ void __launch_bounds__(kBlock<kG>, kBlock<kG> <= 512 ? 512 / kBlock<kG> : 1) resnorm_backward_kernel(const __grid_constant__ NormArgs a) {
    constexpr int kThreads = kBlock<kG>, kRows = kThreads / kG;
    extern __shared__ uint8_t ahead_slots[];
    __shared__ float2 slots[2][32];
    __shared__ float meet[kRows > 1 ? kG * kNV * 8 : 1];
    Group<kG> grp{slots, 0};
    const int t = kRows == 1 ? threadIdx.x : threadIdx.x % kG, D = a.D;
    const int64_t part = kRows == 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kRows + threadIdx.x / kG;
    const int64_t first = part * a.rows_each, last = min(first + a.rows_each, a.M);
    Ahead<T, P, kThreads, kG, kNV, 4> in{{static_cast<const T*>(a.x), static_cast<const T*>(a.h), static_cast<const T*>(a.dy), static_cast<const T*>(a.dr)},
                                         {a.ld_x, a.ld_h, a.ld_dy, a.ld_dr}};
    in.set(ahead_slots, a.depth, D, t);
    in.begin_rows(first, 1, last);
    float dw1[kNV][8], dw2[kNV][8], dg[kNV][8], db1[kLayer ? kNV : 1][8], db2[kLayer ? kNV : 1][8];
#pragma unroll
    for (int g = 0; g < kNV; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dw1[g][i] = dw2[g][i] = dg[g][i] = 0.0f;
            if (kLayer) db1[g][i] = db2[g][i] = 0.0f;
        }
    int64_t gate_i = a.one_gate ? 0 : first / a.rows_per_gate, gate_end = a.one_gate ? a.M : (gate_i + 1) * a.rows_per_gate;
    for (int64_t row = first; row < last; ++row) {
        const float4 st = a.stats[row];
        float k1[kNV][8], k2[kNV][8], e[kNV][8], d[kNV][8];   // normalised h, normalised r, dy w_pre, dr
        float u[kNV][8], gt[kNV][8];                          // N_post(h), scale_h gate
        float s_e = 0.0f, s_ek = 0.0f;
        in.wait();
        // h of vector g -> its norm: k1, u, and the gate beside it
        auto norm_h = [&](int g) {
            float p[8];
            in.read(row, 1, g, k1[g]);
            if (a.post) {
                param_load<P, kG>(a.w_post, 0, g, t, D, 1.0f, p);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    k1[g][i] = (kLayer ? k1[g][i] - st.x : k1[g][i]) * st.y;
                    u[g][i] = k1[g][i] * p[i];
                }
                if (kLayer && a.b_post.p != nullptr) {
                    param_load<P, kG>(a.b_post, 0, g, t, D, 0.0f, p);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[g][i] += p[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) u[g][i] = k1[g][i];
            }
            param_load<P, kG>(a.gate, gate_i * D, g, t, D, 1.0f, p);
            if (full<P, kG>(g, t, D)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) gt[g][i] = a.scale_h * p[i];
            } else {   // 0 past the end: what is multiplied by it stays out of the row's sums
#pragma unroll
                for (int i = 0; i < 8; ++i) gt[g][i] = column<P, kG>(g, i, t) < D ? a.scale_h * p[i] : 0.0f;
            }
        };
#pragma unroll
        for (int g = 0; g < kNV; ++g) {
            in.read(row, 0, g, k2[g]);
            in.read(row, 2, g, e[g]);
            in.read(row, 3, g, d[g]);
            if (!live<P, kG, kNV>(g, t, D)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) k1[g][i] = u[g][i] = gt[g][i] = 0.0f;
                continue;
            }
            norm_h(g);
            float p[8];
            param_load<P, kG>(a.w_pre, 0, g, t, D, 1.0f, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                k2[g][i] = a.scale_x * k2[g][i] + gt[g][i] * u[g][i];   // r
                k2[g][i] = (kLayer ? k2[g][i] - st.z : k2[g][i]) * st.w;
                dw2[g][i] += e[g][i] * k2[g][i];
                if (kLayer) db2[g][i] += e[g][i];
                e[g][i] *= p[i];   // (0 past the end, as dy is)
                if (kLayer) s_e += e[g][i];
                s_ek += e[g][i] * k2[g][i];
            }
        }
        // One vector a thread keeps the norm of h in registers; several form it again from the row in shared memory.
        if (kNV == 1) in.advance(row + a.depth, last);
        if (a.dy != nullptr) {
            float mean_e = 0.0f, mean_ek;
            if (kLayer) {
                const float2 s = grp.sum(s_e, s_ek);
                mean_e = s.x * a.inv_d;
                mean_ek = s.y * a.inv_d;
            } else {
                mean_ek = grp.sum(s_ek) * a.inv_d;
            }
#pragma unroll
            for (int g = 0; g < kNV; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[g][i] += st.w * ((kLayer ? e[g][i] - mean_e : e[g][i]) - k2[g][i] * mean_ek);
        }
        s_e = s_ek = 0.0f;
#pragma unroll
        for (int g = 0; g < kNV; ++g) {
            if (!live<P, kG, kNV>(g, t, D)) continue;
            if (kNV > 1) norm_h(g);
            float out[8], w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = a.scale_x * d[g][i];
            row_store<P, kG>(static_cast<T*>(a.dx) + row * a.ld_dx, g, t, D, out);
            if (a.post) param_load<P, kG>(a.w_post, 0, g, t, D, 1.0f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dg[g][i] += u[g][i] * d[g][i];   // (scale_h comes on when the sum leaves)
                e[g][i] = gt[g][i] * d[g][i];
            }
            if (a.post) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dw1[g][i] += e[g][i] * k1[g][i];
                    if (kLayer) db1[g][i] += e[g][i];
                    e[g][i] *= w[i];
                    if (kLayer) s_e += e[g][i];
                    s_ek += e[g][i] * k1[g][i];
                }
            }
        }
        if (kNV > 1) in.advance(row + a.depth, last);
        if (a.post) {
            float mean_e = 0.0f, mean_ek;
            if (kLayer) {
                const float2 s = grp.sum(s_e, s_ek);
                mean_e = s.x * a.inv_d;
                mean_ek = s.y * a.inv_d;
            } else {
                mean_ek = grp.sum(s_ek) * a.inv_d;
            }
#pragma unroll
            for (int g = 0; g < kNV; ++g)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[g][i] = st.y * ((kLayer ? e[g][i] - mean_e : e[g][i]) - k1[g][i] * mean_ek);
        }
#pragma unroll
        for (int g = 0; g < kNV; ++g) {
            if (live<P, kG, kNV>(g, t, D)) row_store<P, kG>(static_cast<T*>(a.dh) + row * a.ld_dh, g, t, D, e[g]);
        }
        // the gate row's last row, or the group's: its sum leaves (whole gate rows at once, shared ones through the second kernel)
        if (row + 1 == last || row + 1 == gate_end) {
            if (a.dgate != nullptr) {
                const int64_t g0 = gate_i * a.rows_per_gate, g1 = min(g0 + a.rows_per_gate, a.M);
                const bool whole = g0 >= first && g1 <= last;
                float* shared_part = a.part_gate + (part * 2 + (gate_i == first / a.rows_per_gate ? 0 : 1)) * D;
#pragma unroll
                for (int g = 0; g < kNV; ++g)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = column<P, kG>(g, i, t);
                        if (c < D) {
                            if (whole) param_store(a.dgate, a.gate.type, gate_i * D + c, a.scale_h * dg[g][i]);
                            else shared_part[c] = a.scale_h * dg[g][i];
                        }
                        dg[g][i] = 0.0f;
                    }
            }
            ++gate_i;
            gate_end += a.rows_per_gate;
        }
    }
    publish<P, kG, kNV>(a.part_w_pre, dw2, t, D, meet);
    publish<P, kG, kNV>(a.part_w_post, dw1, t, D, meet);
    if (kLayer) {
        publish<P, kLayer ? kG : 32, kLayer ? kNV : 1>(a.part_b_pre, db2, t, D, meet);
        publish<P, kLayer ? kG : 32, kLayer ? kNV : 1>(a.part_b_post, db1, t, D, meet);
    }
}

// Second kernel of the backward pass: column sums over the blocks' partial sums, and the gate rows that several groups share.
// blockIdx.y: which array, then which gate row -- or, where there are fewer of them, which eight borders between two groups, one for
// each warp (a shared gate row belongs to the first border inside it, and then reaches over few groups); 32 columns a block, eight threads a column with eight loads in flight each, added in a fixed order.
// Launched behind the first kernel's end (its blocks are resident by then).
struct FinishArgs {
    int D;
    int blocks;
    const float* part[4];
    void* out[4];
    int arrays;
    int type;
    // gates
    const float* part_gate;
    void* dgate;
    int gate_type, by_border;
    int64_t M, rows_per_gate, rows_each, parts;
};

__global__ void __launch_bounds__(256) resnorm_finish_kernel(const __grid_constant__ FinishArgs f) {
    __shared__ float meet[8][33];
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    int64_t gate = (int64_t)blockIdx.y - f.arrays;
    sm100::griddep_wait();
    if (gate < 0) {
        const float* p = f.part[blockIdx.y];
        if (c < f.D)
#pragma unroll 8
            for (int b = y; b < f.blocks; b += 8) s += p[(int64_t)b * f.D + c];
    } else {
        const int64_t border = f.by_border ? gate * 8 + y + 1 : 0;
        if (f.by_border) {
            if (border >= f.parts) return;
            gate = border * f.rows_each / f.rows_per_gate;
        }
        const int64_t g0 = gate * f.rows_per_gate, g1 = min(g0 + f.rows_per_gate, f.M);
        const int64_t p0 = g0 / f.rows_each, p1 = (g1 - 1) / f.rows_each;
        if (p0 == p1 || (f.by_border && (g0 == border * f.rows_each || p0 != border - 1))) return;   // one group's alone, or another border's
        // only a part's first gate row can have begun before it, so of parts p0 + 1 ... it is slot 0; of part p0 it is slot 0 where
        // that part begins with it
        const float* p = f.part_gate + c;
        const int64_t at0 = (p0 * 2 + (gate == p0 * f.rows_each / f.rows_per_gate ? 0 : 1)) * f.D;
        if (f.by_border) {
            if (c >= f.D) return;
            s = p[at0];
            for (int64_t i = p0 + 1; i <= p1; ++i) s += p[i * 2 * f.D];
            param_store(f.dgate, f.gate_type, gate * f.D + c, s);
            return;
        }
        if (c < f.D) {
            if (y == 0) s = p[at0];
#pragma unroll 8
            for (int64_t i = p0 + 1 + y; i <= p1; i += 8) s += p[i * 2 * f.D];
        }
    }
    meet[y][lane] = s;
    __syncthreads();
    if (y != 0 || c >= f.D) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += meet[i][lane];
    if ((int)blockIdx.y < f.arrays) param_store(f.out[blockIdx.y], f.type, c, s);
    else param_store(f.dgate, f.gate_type, gate * f.D + c, s);
}

// ------------------------------------------------------------------------------------------ host
constexpr int kMaxD = 32768;

// Threads of a row in the backward pass.
int group_threads(int D) { return D <= 512 ? 32 : D <= 1024 ? 128 : D <= 2048 ? 256 : D <= 8192 ? 512 : 1024; }

struct Split {
    int64_t rows_each, parts;
    int blocks;
};
// How the backward pass deals rows out: consecutive rows to each group, 512 threads (of 128 registers) to an SM.
Split split_rows(int64_t M, int D) {
    const int g = group_threads(D), threads = g < 128 ? 256 : g, rows = threads / g;
    const int64_t most = (int64_t)kNumSMs * std::max(1, 512 / threads) * rows;
    Split s;
    s.rows_each = std::max<int64_t>(1, (M + most - 1) / most);
    s.parts = (M + s.rows_each - 1) / s.rows_each;
    s.blocks = (int)((s.parts + rows - 1) / rows);
    return s;
}

struct NormSpace {
    size_t w_post, b_post, w_pre, b_pre, gate, total;
};
NormSpace norm_space(int64_t M, int D) {
    const Split s = split_rows(M, D);
    auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
    const size_t one = up((size_t)s.blocks * D * 4);
    NormSpace w{};
    size_t at = 256;
    w.w_post = at; at += one;
    w.b_post = at; at += one;
    w.w_pre = at; at += one;
    w.b_pre = at; at += one;
    w.gate = at; at += up((size_t)s.parts * 2 * D * 4);
    w.total = at;
    return w;
}

// Rows ahead that fit the shared memory of a block when `resident` of them share an SM.
int depth_for(int row_bytes, int resident, bool even, int64_t rows_each) {
    if (!even || rows_each < 2) return 0;   // (one row a group: nothing to run ahead of)
    return (int)std::min<int64_t>(3, 200 * 1024 / resident / row_bytes);
}

// The attribute for more than 48 KB of shared memory (it belongs to the current device).
template <typename K>
lbt_status allow_smem(K kernel, int bytes) {
    if (bytes <= 40 * 1024) return LBT_OK;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess ? LBT_OK : LBT_ERR_CUDA;
}

template <typename T, typename P, int kG, int kNV>
lbt_status forward_launch(NormArgs a, cudaStream_t stream) {
    constexpr int threads = kBlock<kG>, rows = threads / kG, resident = kForwardBlocks<kG, kNV>;
    const int64_t blocks = std::min<int64_t>((a.M + rows - 1) / rows, (int64_t)kNumSMs * resident);
    constexpr int row_bytes = Ahead<T, P, threads, kG, kNV, 2>::kRowBytes;
    a.depth = depth_for(row_bytes, resident, kEven<P>, (a.M + blocks * rows - 1) / (blocks * rows));
    a.step_gates = blocks * rows / a.rows_per_gate;
    a.step_rest = blocks * rows % a.rows_per_gate;
    auto kernel = a.layer ? resnorm_forward_kernel<T, P, kG, kNV, true> : resnorm_forward_kernel<T, P, kG, kNV, false>;
    const lbt_status rc = allow_smem(kernel, a.depth * row_bytes);
    if (rc != LBT_OK) return rc;
    kernel<<<(unsigned)blocks, threads, a.depth * row_bytes, stream>>>(a);
    return launch_status();
}

// Sixteen columns a thread where a block owns a row: half the reductions' instructions for each element.
template <typename T, typename P>
lbt_status run_forward(const NormArgs& a, cudaStream_t stream) {
    if (a.D <= 256) return forward_launch<T, P, 32, 1>(a, stream);
    if (a.D <= 512) return forward_launch<T, P, 32, 2>(a, stream);
    if (a.D <= 1024) return forward_launch<T, P, 32, 4>(a, stream);
    if (a.D <= 2048) return forward_launch<T, P, 128, 2>(a, stream);
    if (a.D <= 4096) return forward_launch<T, P, 256, 2>(a, stream);
    if (a.D <= 8192) return forward_launch<T, P, 512, 2>(a, stream);
    if (a.D <= 16384) return forward_launch<T, P, 1024, 2>(a, stream);
    if constexpr (!kEven<P>) return forward_launch<T, P, 1024, 4>(a, stream);
    return LBT_ERR_UNSUPPORTED;   // (not reached: even() refuses such rows)
}

template <typename T, typename P, int kG, int kNV, bool kLayer>
lbt_status backward_launch(NormArgs a, const Split& s, cudaStream_t stream) {
    constexpr int threads = kBlock<kG>, resident = threads <= 512 ? 512 / threads : 1;
    constexpr int row_bytes = Ahead<T, P, threads, kG, kNV, 4>::kRowBytes;
    a.depth = depth_for(row_bytes, resident, kEven<P>, s.rows_each);
    const lbt_status rc = allow_smem(resnorm_backward_kernel<T, P, kG, kNV, kLayer>, a.depth * row_bytes);
    if (rc != LBT_OK) return rc;
    resnorm_backward_kernel<T, P, kG, kNV, kLayer><<<(unsigned)s.blocks, threads, a.depth * row_bytes, stream>>>(a);
    return launch_status();
}

template <typename T, typename P, bool kLayer>
lbt_status run_backward_kind(const NormArgs& a, const Split& s, cudaStream_t stream) {
    if (a.D <= 256) return backward_launch<T, P, 32, 1, kLayer>(a, s, stream);
    if (a.D <= 512) return backward_launch<T, P, 32, 2, kLayer>(a, s, stream);
    if (a.D <= 1024) return backward_launch<T, P, 128, 1, kLayer>(a, s, stream);
    if (a.D <= 2048) return backward_launch<T, P, 256, 1, kLayer>(a, s, stream);
    if (a.D <= 4096) return backward_launch<T, P, 512, 1, kLayer>(a, s, stream);
    if (a.D <= 8192) return backward_launch<T, P, 512, 2, kLayer>(a, s, stream);
    if (a.D <= 16384) return backward_launch<T, P, 1024, 2, kLayer>(a, s, stream);
    if constexpr (!kEven<P>) return backward_launch<T, P, 1024, 4, kLayer>(a, s, stream);
    return LBT_ERR_UNSUPPORTED;   // (not reached: even() refuses such rows)
}
template <typename T, typename P>
lbt_status run_backward(const NormArgs& a, const Split& s, cudaStream_t stream) {
    return a.layer ? run_backward_kind<T, P, true>(a, s, stream) : run_backward_kind<T, P, false>(a, s, stream);
}

// The form for aligned rows where everything is aligned, D is a multiple of 8 and the parameters are fp32 or of the
// activations' type.  (Past 16384 columns rows are rare and the general form serves them.)
bool even(const NormArgs& a, int type, int param_type) {
    return a.vec && a.D % 8 == 0 && a.D <= 16384 && a.gate.vec && a.w_post.vec && a.b_post.vec && a.w_pre.vec && a.b_pre.vec &&
           (param_type == LBT_F32 || param_type == type);
}
#define LBT_RESNORM_DISPATCH(RUN, a, type, ptype, ...)                                                                        \
    do {                                                                                                                      \
        const bool e = even(a, type, ptype);                                                                                  \
        if (type == LBT_F32) return e ? RUN<float, float>(a, __VA_ARGS__) : RUN<float, void>(a, __VA_ARGS__);                 \
        if (type == LBT_BF16) {                                                                                               \
            if (!e) return RUN<__nv_bfloat16, void>(a, __VA_ARGS__);                                                          \
            return ptype == LBT_F32 ? RUN<__nv_bfloat16, float>(a, __VA_ARGS__) : RUN<__nv_bfloat16, __nv_bfloat16>(a, __VA_ARGS__); \
        }                                                                                                                     \
        if (!e) return RUN<__half, void>(a, __VA_ARGS__);                                                                     \
        return ptype == LBT_F32 ? RUN<__half, float>(a, __VA_ARGS__) : RUN<__half, __half>(a, __VA_ARGS__);                   \
    } while (0)

lbt_status forward_any(const NormArgs& a, int type, int ptype, cudaStream_t stream) { LBT_RESNORM_DISPATCH(run_forward, a, type, ptype, stream); }
lbt_status backward_any(const NormArgs& a, const Split& s, int type, int ptype, cudaStream_t stream) {
    LBT_RESNORM_DISPATCH(run_backward, a, type, ptype, s, stream);
}

bool off(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// What forward and backward check and set up alike.
lbt_status common(const lbt_resnorm_desc* d, NormArgs* a) {
    if (d == nullptr || d->M < 0 || d->D <= 0 || !type_ok(d->type) || !type_ok(d->param_type)) return LBT_ERR_INVALID_ARG;
    if (d->kind != LBT_NORM_RMS && d->kind != LBT_NORM_LAYER) return LBT_ERR_INVALID_ARG;
    if (d->rows_per_gate < 0 || !(d->eps_post >= 0.0f) || !(d->eps_pre >= 0.0f)) return LBT_ERR_INVALID_ARG;
    if (d->D > kMaxD || d->M >= (1ll << 40)) return LBT_ERR_UNSUPPORTED;
    a->M = d->M;
    a->D = (int)d->D;
    a->rows_per_gate = d->rows_per_gate == 0 ? std::max<int64_t>(d->M, 1) : d->rows_per_gate;
    a->one_gate = a->rows_per_gate >= d->M;
    a->layer = d->kind == LBT_NORM_LAYER;
    a->post = d->post_norm != 0;
    a->eps_post = d->eps_post; a->eps_pre = d->eps_pre; a->scale_x = d->scale_x; a->scale_h = d->scale_h;
    a->inv_d = 1.0f / (float)d->D;
    const int64_t* ld = &d->ld_x;
    int64_t* to[8] = {&a->ld_x, &a->ld_h, &a->ld_r, &a->ld_y, &a->ld_dr, &a->ld_dy, &a->ld_dx, &a->ld_dh};
    for (int i = 0; i < 8; ++i) {
        if (ld[i] != 0 && ld[i] < d->D) return LBT_ERR_INVALID_ARG;
        *to[i] = ld[i] != 0 ? ld[i] : d->D;
    }
    a->vec = true;
    return LBT_OK;
}

bool vec_ok(const void* p, int64_t ld, int type) {
    const size_t bytes = 8 * type_size(type);
    return p == nullptr || (!off(p, bytes) && (ld * type_size(type)) % bytes == 0);
}
Params make_param(const void* p, int type, int64_t D) {
    return Params{p, type, vec_ok(p, D, type)};
}

}  // namespace
}  // namespace lbt

using namespace lbt;

extern "C" lbt_status lbt_resnorm_forward(const lbt_resnorm_desc* d, const void* x, const void* h, const void* gate, const void* w_post,
                                          const void* b_post, const void* w_pre, const void* b_pre, void* r, void* y, void* q, int64_t ldq,
                                          float* q_scale, float* stats, void* cuda_stream) {
    NormArgs a{};
    const lbt_status rc = common(d, &a);
    if (rc != LBT_OK) return rc;
    if (q != nullptr && (q_scale == nullptr || ldq < a.D)) return LBT_ERR_INVALID_ARG;
    if (!a.layer && (b_post != nullptr || b_pre != nullptr)) return LBT_ERR_INVALID_ARG;
    if (a.M > 0 && (x == nullptr || h == nullptr || r == nullptr)) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d->type), pe = type_size(d->param_type);
    if (off(x, e) || off(h, e) || off(r, e) || off(y, e) || off(gate, pe) || off(w_post, pe) || off(b_post, pe) || off(w_pre, pe) ||
        off(b_pre, pe) || off(q, 16) || (q != nullptr && ldq % 16 != 0) || off(q_scale, 4) || off(stats, 16))
        return LBT_ERR_ALIGNMENT;
    if (a.M == 0) return LBT_OK;
    a.x = x; a.h = h; a.r = r; a.y = y;
    a.vec = vec_ok(x, a.ld_x, d->type) && vec_ok(h, a.ld_h, d->type) && vec_ok(r, a.ld_r, d->type) && vec_ok(y, a.ld_y, d->type);
    a.gate = make_param(gate, d->param_type, a.D);
    a.w_post = make_param(w_post, d->param_type, a.D); a.b_post = make_param(b_post, d->param_type, a.D);
    a.w_pre = make_param(w_pre, d->param_type, a.D); a.b_pre = make_param(b_pre, d->param_type, a.D);
    // codes: a row is padded with zeros up to the next multiple of 16 columns
    a.q = static_cast<uint8_t*>(q); a.ldq = ldq; a.q_end = (d->D + 15) / 16 * 16; a.q_scale = q_scale;
    a.stats = reinterpret_cast<float4*>(stats);
    const cudaStream_t stream = as_stream(cuda_stream);
    return forward_any(a, d->type, d->param_type, stream);
}

extern "C" size_t lbt_resnorm_workspace_bytes(const lbt_resnorm_desc* d) {
    NormArgs a{};
    return common(d, &a) == LBT_OK ? norm_space(a.M, a.D).total : 0;
}

extern "C" lbt_status lbt_resnorm_backward(const lbt_resnorm_desc* d, const void* dr, const void* dy, const void* x, const void* h,
                                           const void* gate, const void* w_post, const void* b_post, const void* w_pre, const float* stats,
                                           void* dx, void* dh, void* dgate, void* dw_post, void* db_post, void* dw_pre, void* db_pre,
                                           void* ws, size_t ws_bytes, void* cuda_stream) {
    NormArgs a{};
    lbt_status rc = common(d, &a);
    if (rc != LBT_OK) return rc;
    if (a.M > 0 && (x == nullptr || h == nullptr || stats == nullptr || dx == nullptr || dh == nullptr || (dr == nullptr && dy == nullptr)))
        return LBT_ERR_INVALID_ARG;
    if (dgate != nullptr && gate == nullptr) return LBT_ERR_INVALID_ARG;
    if (!a.post && (dw_post != nullptr || db_post != nullptr)) return LBT_ERR_INVALID_ARG;
    if (!a.layer && (b_post != nullptr || db_post != nullptr || db_pre != nullptr)) return LBT_ERR_INVALID_ARG;
    const size_t e = type_size(d->type), pe = type_size(d->param_type);
    if (off(dr, e) || off(dy, e) || off(x, e) || off(h, e) || off(dx, e) || off(dh, e) || off(gate, pe) || off(w_post, pe) || off(b_post, pe) ||
        off(w_pre, pe) || off(dgate, pe) || off(dw_post, pe) || off(db_post, pe) || off(dw_pre, pe) || off(db_pre, pe) || off(stats, 16))
        return LBT_ERR_ALIGNMENT;
    const NormSpace w = norm_space(a.M, a.D);
    if (ws == nullptr || ws_bytes < w.total) return LBT_ERR_WORKSPACE;
    const cudaStream_t stream = as_stream(cuda_stream);
    void* outs[4] = {dw_post, db_post, dw_pre, db_pre};
    if (a.M == 0) {   // no rows: the sums are zero (there is a gate row only where it is one for all)
        for (void* o : {dw_post, db_post, dw_pre, db_pre, d->rows_per_gate == 0 ? dgate : nullptr})
            if (o != nullptr) LBT_CUDA_TRY(cudaMemsetAsync(o, 0, (size_t)a.D * pe, stream));
        return LBT_OK;
    }
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255) - 256;
    const Split s = split_rows(a.M, a.D);
    a.dr = dr; a.dy = dy; a.x = x; a.h = h; a.dx = dx; a.dh = dh;
    a.vec = vec_ok(dr, a.ld_dr, d->type) && vec_ok(dy, a.ld_dy, d->type) && vec_ok(x, a.ld_x, d->type) && vec_ok(h, a.ld_h, d->type) &&
            vec_ok(dx, a.ld_dx, d->type) && vec_ok(dh, a.ld_dh, d->type);
    a.gate = make_param(gate, d->param_type, a.D);
    a.w_post = make_param(w_post, d->param_type, a.D); a.b_post = make_param(b_post, d->param_type, a.D);
    a.w_pre = make_param(w_pre, d->param_type, a.D); a.b_pre = make_param(nullptr, d->param_type, a.D);
    a.stats = reinterpret_cast<float4*>(const_cast<float*>(stats));
    a.rows_each = s.rows_each; a.parts = s.parts;
    auto at = [&](size_t o, void* wanted) { return wanted != nullptr ? reinterpret_cast<float*>(base + o) : nullptr; };
    a.part_w_post = at(w.w_post, dw_post); a.part_b_post = at(w.b_post, db_post);
    a.part_w_pre = at(w.w_pre, dw_pre); a.part_b_pre = at(w.b_pre, db_pre);
    a.part_gate = reinterpret_cast<float*>(base + w.gate);
    a.dgate = dgate;
    rc = backward_any(a, s, d->type, d->param_type, stream);
    if (rc != LBT_OK) return rc;
    FinishArgs f{};
    f.D = a.D; f.blocks = s.blocks; f.type = d->param_type;
    const float* parts[4] = {a.part_w_post, a.part_b_post, a.part_w_pre, a.part_b_pre};
    for (int i = 0; i < 4; ++i)
        if (outs[i] != nullptr) { f.part[f.arrays] = parts[i]; f.out[f.arrays++] = outs[i]; }
    int64_t shared = 0;   // blocks for the gate rows that may lie in several groups: all of them, or at most one for each border
    if (dgate != nullptr) {
        const int64_t gates = (a.M + a.rows_per_gate - 1) / a.rows_per_gate;
        f.by_border = gates > s.parts - 1;
        shared = f.by_border ? (s.parts - 1 + 7) / 8 : gates;
        f.part_gate = a.part_gate; f.dgate = dgate; f.gate_type = d->param_type;
        f.M = a.M; f.rows_per_gate = a.rows_per_gate; f.rows_each = a.rows_each; f.parts = s.parts;
    }
    if (f.arrays + shared == 0) return LBT_OK;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((a.D + 31) / 32), (unsigned)(f.arrays + shared));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, resnorm_finish_kernel, f) != cudaSuccess) return LBT_ERR_CUDA;
    return launch_status();
}
