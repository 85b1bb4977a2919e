/*
 * lbt.h -- C ABI of the B200 (sm_100a) library for the quantized backward pass of
 * arXiv 2407.12637, "Toward INT4 Fixed-Point Training via Exploring Quantization
 * Error for Gradients".
 *
 * One layer, one training iteration:
 *   1. statistics of the full-precision output gradient dY (abs-max; clip-out count),
 *   2. the clipping-factor ("interval") update of Sec. 3.3,
 *   3. b-bit fixed-point quantization of dY (Sec. 3.1),
 *   4. the integer backward contractions dX = Q(dY) Q(W) and dW = Q(dY)^T Q(X), with a
 *      dequantising fp32 epilogue.
 *
 * Conventions, valid for every entry point unless it says otherwise
 *   - Every tensor / struct pointer is a DEVICE pointer owned by the caller and 16-byte aligned.
 *     Only `lbt_conv_desc` / `lbt_gemm_desc` arguments are HOST pointers (read during the call).
 *   - The library allocates no device memory and never synchronises the device: each call
 *     enqueues kernels on `cuda_stream` (a cudaStream_t passed as void*; NULL = default stream)
 *     and returns.  Scratch memory is passed in as `ws` / `ws_bytes`; its size comes from
 *     lbt_workspace_bytes().  Workspace contents are undefined between calls.
 *   - Errors the host can see (bad arguments, unsupported sizes, launch failures) are returned
 *     and nothing is enqueued.  Conditions only the device can see (non-finite gradients, a
 *     bounded wait that ran out) are recorded in a device status word (sticky: the first
 *     non-zero value stays until the caller clears it) and outputs stay defined.
 *   - Layouts: linear layers are row-major, Y[M,O] = X[M,I] W[O,I]^T.  Convolutions use NHWC
 *     activations / gradients and KRSC weights,
 *         Y[n,p,q,k] = sum_{r,s,c} X[n, p*stride + r - pad, q*stride + s - pad, c] W[k,r,s,c].
 *   - Code storage: bit-widths <= 4 are packed two per byte as 4-bit fields, element 2j in bits
 *     0-3 and element 2j+1 in bits 4-7 of byte j (two's complement for signed codes), an odd
 *     tail padded with 0; bit-widths 5..8 take one byte per element.  "Element index" is the
 *     linear index in the buffer as given.
 */
#ifndef LBT_H_
#define LBT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t lbt_status;
enum {
    LBT_OK                   = 0,
    LBT_ERR_INVALID_ARG      = -1,  /* null pointer, non-positive size, inconsistent description */
    LBT_ERR_ALIGNMENT        = -2,  /* a pointer is not 16-byte aligned                            */
    LBT_ERR_UNSUPPORTED_BITS = -3,  /* bit-width outside 2..8                                      */
    LBT_ERR_ACC_RANGE        = -4,  /* the worst-case accumulator does not fit int32              */
    LBT_ERR_WORKSPACE        = -5,  /* ws is null or smaller than lbt_workspace_bytes()           */
    LBT_ERR_CUDA             = -6,  /* a CUDA runtime / driver call failed                        */
    LBT_ERR_NONFINITE        = -7,  /* device-reported: dY holds NaN or Inf                       */
    LBT_ERR_TIMEOUT          = -8,  /* device-reported: a bounded on-chip wait ran out            */
    LBT_ERR_UNSUPPORTED      = -9,  /* a shape this build does not cover (e.g. stride > 2)        */
    LBT_ERR_SCRATCH_LIMIT    = -10, /* the problem needs more than the library's built-in scratch */
    LBT_ERR_BITS_MISMATCH    = -11  /* device-reported: bits_g of lbt_qconv_backward differs from st->bits */
};

enum { LBT_ROUND_NEAREST = 0, LBT_ROUND_STOCHASTIC = 1 };

/*
 * Per-layer interval state (Algorithm 1: hyperparameters b, alpha, beta; input gamma_{i-1};
 * output gamma_i).  Lives in device memory; a plain copy is a checkpoint.
 */
typedef struct lbt_interval_state {
    float    gamma;       /* clipping factor, c_g = gamma * g_max (Sec. 3.1); start at 1.0        */
    float    alpha;       /* ratio of large gradients N(G_L)/N(G) (Sec. 3.2); paper's best 1e-3   */
    float    beta;        /* step of the update, Eq. (15); the paper fixes 1e-3                   */
    float    gamma_min;   /* gamma is clamped to [gamma_min, gamma_max]; the paper keeps gamma in */
    float    gamma_max;   /*   (0, 1]; gamma_max = +inf reproduces the unclamped rule             */
    int32_t  bits;        /* gradient bit-width b, 2..8                                           */
    uint32_t rounding;    /* LBT_ROUND_NEAREST (ties to even) or LBT_ROUND_STOCHASTIC             */
    uint32_t reserved;    /* keeps `seed` 8-byte aligned; write 0                                  */
    uint64_t seed;        /* Philox key                                                           */
    uint64_t iter;        /* Philox stream of the next quantization; ++ in lbt_update_interval    */
    int32_t  dev_status;  /* sticky device-side status word (LBT_OK, LBT_ERR_NONFINITE, ...)      */
    int32_t  reserved2;
} lbt_interval_state;     /* 56 bytes */

/* Per-call statistics of one gradient tensor (device memory). */
typedef struct lbt_grad_stats_t {
    float    g_max;        /* max |dY_i| over the finite elements (Sec. 3.1)                      */
    float    c;            /* clipping value c_g = gamma * g_max                                  */
    float    scale;        /* s = c_g / (2^(b-1) - 1), Eq. (2)                                    */
    uint32_t reserved;     /* scratch of the one-launch quantizer (block counter); 0 between calls   */
    uint64_t n;            /* N(G)                                                                */
    uint64_t n_out;        /* #{ |dY_i| > c_g }, numerator of R(G_out, gamma), Eq. (9)            */
    uint64_t n_nonfinite;  /* #{ dY_i is NaN or Inf }                                             */
} lbt_grad_stats_t;        /* 40 bytes */

/* Linear layer: dY[M,O], W[O,I], X[M,I].  (HOST struct.) */
typedef struct lbt_gemm_desc {
    int64_t M, O, I;
} lbt_gemm_desc;

/* Convolution: X[N,H,W,C], W[K,R,S,C], dY[N,P,Q,K], P = (H + 2 pad - R)/stride + 1.  (HOST struct.) */
typedef struct lbt_conv_desc {
    int32_t N, C, H, W, K, R, S, stride, pad;
} lbt_conv_desc;

enum {
    LBT_OP_GRAD_STATS    = 0,  /* desc ignored                        */
    LBT_OP_QUANTIZE      = 1,  /* desc ignored                        */
    LBT_OP_GEMM_DGRAD    = 2,  /* desc: const lbt_gemm_desc*          */
    LBT_OP_GEMM_WGRAD    = 3,  /* desc: const lbt_gemm_desc*          */
    LBT_OP_CONV_BACKWARD = 4,  /* desc: const lbt_conv_desc*          */
    LBT_OP_GEMM_FORWARD  = 5,  /* desc: const lbt_gemm_desc*          */
    LBT_OP_CONV_FORWARD  = 6   /* desc: const lbt_conv_desc*          */
};

/* Bytes of workspace the operation needs for this description (0 when none; also 0 for an
 * invalid description, which the operation itself then rejects).  Host-only, no CUDA call.
 * The sizes differ by operation: the wgrad contraction (LBT_OP_GEMM_WGRAD, and LBT_OP_CONV_BACKWARD,
 * which covers lbt_qconv_dgrad_wgrad and lbt_qconv_backward) adds room for the int32 partial sums of
 * its split reduction (at most ~20 MB) to what dgrad and the forward product need. */
size_t lbt_workspace_bytes(int op, const void *desc);

/*
 * Statistics, first half (Sec. 3.1: g_max = max(|G|) of one layer).
 * Writes out->g_max, out->n = n, out->n_nonfinite, and clears out->n_out, out->c, out->scale.
 * `st` is not read by this call (it is part of the signature so that the three calls of one
 * iteration take the same arguments); it may be NULL.  n = 0 is valid and gives g_max = 0.
 */
lbt_status lbt_grad_stats(const float *dY, uint64_t n, const lbt_interval_state *st,
                          lbt_grad_stats_t *out, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Quantizer, Eq. (1), (2), (4) with c_g = gamma * g_max, fused with the clip-out count of
 * Sec. 3.3 / Algorithm 1 (the gradients that this very quantization clips):
 *   c = fl32(gamma * g_max); s = fl32(c / qmax), qmax = 2^(b-1) - 1;
 *   x = clamp(fl32(dY_i / s), -qmax, qmax);
 *   nearest:    q = rint(x) (ties to even);
 *   stochastic: q = floor(x) + [u < t], t = trunc(frac(x) * 2^16) with frac(x) = x - floor(x)
 *               taken exactly (no rounding), u = the 16-bit field of
 *               Philox4x32-10(key = seed, counter = (i >> 3, iter)) that belongs to i & 7
 *               (low half of word 0 first);
 *   q_out[i] = clamp(q, -qmax, qmax), packed as the header describes.
 * In:  stats->g_max, stats->n_nonfinite (from lbt_grad_stats on the same dY); st->gamma, bits,
 *      rounding, seed, iter (all read on the device; bits outside 2..8 are clamped into it).
 * Out: stats->c, stats->scale, stats->n_out; q_out (ceil(n/2) bytes for b <= 4, else n bytes).
 * If s == 0 (an all-zero gradient) or n_nonfinite != 0 every code is 0.
 */
lbt_status lbt_quantize_grad(const float *dY, uint64_t n, const lbt_interval_state *st,
                             lbt_grad_stats_t *stats, void *q_out, void *ws, size_t ws_bytes,
                             void *cuda_stream);

/*
 * lbt_grad_stats + lbt_quantize_grad + lbt_update_interval as ONE cooperative launch (Sec. 3.1, 3.3,
 * Eq. 1, 2, 4, 15, 16): every block reduces its share of |dY|, the blocks meet at a bounded grid barrier,
 * quantize with the global g_max and count the clipped elements, and the block that finishes last applies
 * the update.  Same arguments, results (bit for bit) and device-reported conditions as the three calls in
 * sequence; dev_status also becomes LBT_ERR_TIMEOUT if the barrier's 2 s bound runs out.  Meant for
 * gradient tensors that fit L2 (the second reading of dY is then served on-chip and two launches are
 * saved); correct at any size.  With stochastic rounding the random words of each thread's first groups
 * are generated while the first phase waits on memory and kept in up to 36 KB of dynamic shared memory
 * per block.  On a device without cooperative launch it runs the three launches.
 * lbt_qconv_backward takes this path by itself for tensors of at most 112 MiB.
 */
lbt_status lbt_quantize_grad_fused(const float *dY, uint64_t n, lbt_interval_state *st,
                                   lbt_grad_stats_t *stats, void *q_out, void *cuda_stream);

/*
 * Clipping-factor update, Eq. (15), (16) / Algorithm 1:
 *   gamma <- clamp(gamma + beta * sign(n_out / n - alpha / (2^b - 1)), gamma_min, gamma_max),
 * the sign decided on n_out * (2^b - 1) versus alpha * n in binary64, sign(0) = 0; iter <- iter + 1.
 * With stats->n_nonfinite != 0, gamma is left alone and dev_status becomes LBT_ERR_NONFINITE.
 * One thread on the device; no host round trip.
 */
lbt_status lbt_update_interval(lbt_interval_state *st, const lbt_grad_stats_t *stats,
                               void *cuda_stream);

/*
 * Linear-layer backward contractions on the integer tensor cores (the paper motivates integer
 * arithmetic for the backward pass in Sec. 1 and specifies no kernel):
 *   dgrad: dX[m,i] = fl32(s_g * s_w) * sum_o q_dY[m,o] q_W[o,i]
 *   wgrad: dW[o,i] = fl32(s_g * s_x) * sum_m q_dY[m,o] q_X[m,i]
 * q_dY: signed codes of bits_g bits ([M,O]); q_W: signed codes of bits_w bits ([O,I]); q_X:
 * UNSIGNED codes of bits_x bits ([M,I]); storage as the header describes.  d_scale_*: device
 * pointers to one float each.  dX / dW: fp32 outputs.  acc_out (optional, may be NULL): the raw
 * int32 accumulators, same shape as the fp32 output.  dev_status (optional device int32, may be
 * NULL) receives LBT_ERR_TIMEOUT if a bounded wait inside a kernel ran out.
 * LBT_ERR_ACC_RANGE if (reduction length) * max|code_a| * max|code_b| >= 2^31.
 */
lbt_status lbt_qgemm_dgrad(const void *q_dY, const void *q_W, const float *d_scale_g,
                           const float *d_scale_w, float *dX, int32_t *acc_out,
                           int64_t M, int64_t O, int64_t I, int bits_g, int bits_w,
                           int32_t *dev_status, void *ws, size_t ws_bytes, void *cuda_stream);

lbt_status lbt_qgemm_wgrad(const void *q_dY, const void *q_X, const float *d_scale_g,
                           const float *d_scale_x, float *dW, int32_t *acc_out,
                           int64_t M, int64_t O, int64_t I, int bits_g, int bits_x,
                           int32_t *dev_status, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * lbt_qgemm_dgrad for callers that cannot hand over a workspace (the paper has no counterpart;
 * this is a convenience of the library).  Who needs it: code that must not allocate device memory
 * where it calls the library -- a layer hosted inside a framework whose own allocator owns every
 * byte of HBM, a latency-critical loop in which cudaMalloc / cudaFree would stall the device, a
 * process whose memory was reserved in full at start-up so that a later allocation would fail.
 * Same arguments, results and error codes as lbt_qgemm_dgrad, minus `ws` / `ws_bytes`: the scratch
 * is a fixed LBT_STATIC_SCRATCH_BYTES array inside the library's device image (so every GPU that
 * loads the library gives up that much memory until the process exits).
 *   - Returns LBT_ERR_SCRATCH_LIMIT, enqueuing nothing, when
 *     lbt_workspace_bytes(LBT_OP_GEMM_DGRAD, {M,O,I}) exceeds LBT_STATIC_SCRATCH_BYTES
 *     (for instance M = O = I = 1024 fits, 2048 does not).
 *   - It calls no cudaMalloc, cudaFree or other allocating routine.
 *   - The first call on each device looks up the array's device address (with that device
 *     current); make that first call before starting any stream capture.
 *   - All calls on a device share the one array.  Each call rewrites every part of it that it later
 *     reads, so nothing needs clearing by the caller and a previous call's leftovers are harmless;
 *     but two calls that overlap on the GPU (different streams, or threads) race on it: keep calls
 *     to this entry point ordered on one stream per device.
 */
#define LBT_STATIC_SCRATCH_BYTES (8u << 20)
lbt_status lbt_qgemm_dgrad_static(const void *q_dY, const void *q_W, const float *d_scale_g,
                                  const float *d_scale_w, float *dX, int32_t *acc_out,
                                  int64_t M, int64_t O, int64_t I, int bits_g, int bits_w,
                                  int32_t *dev_status, void *cuda_stream);

/*
 * Convolution backward contractions alone (codes already quantized), implicit GEMM:
 *   dgrad: dX[n,h,w,c] = fl32(s_g*s_w) * sum_{k,r,s} q_dY[n,p,q,k] q_W[k,r,s,c],
 *          p = (h + pad - r)/stride, q = (w + pad - s)/stride where integral and in range;
 *   wgrad: dW[k,r,s,c] = fl32(s_g*s_x) * sum_{n,p,q} q_dY[n,p,q,k] q_X[n, p*stride + r - pad,
 *          q*stride + s - pad, c], taps outside the image contributing 0.
 * Either output (with its operand) may be NULL to skip that contraction.  stride 1 or 2.
 */
lbt_status lbt_qconv_dgrad_wgrad(const lbt_conv_desc *d, const void *q_dY, const void *q_W,
                                 const void *q_X, const float *d_scale_g, const float *d_scale_w,
                                 const float *d_scale_x, float *dX, float *dW, int32_t *accX,
                                 int32_t *accW, int bits_g, int bits_w, int bits_x,
                                 int32_t *dev_status, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The whole hot path for one convolution layer and one iteration, in stream order:
 *   lbt_grad_stats(dY) -> lbt_quantize_grad (with gamma_{i-1}; counts what it clips)
 *   -> lbt_update_interval (gamma_i for the next iteration) -> dgrad -> wgrad.
 * dY is fp32 [N,P,Q,K]; q_W / q_X are 4-bit codes (signed / unsigned); q_dY_out receives the
 * gradient codes; dX / dW (and their operands) may be NULL to skip a contraction.
 * bits_g must equal st->bits (the host needs it to size q_dY_out and the integer pipeline; the state
 * itself stays on the device).  If the device finds another st->bits, dev_status becomes
 * LBT_ERR_BITS_MISMATCH, the codes are written as zeros in the layout of bits_g (so dX and dW are zero and
 * nothing is written out of bounds) and gamma is left alone.
 * A linear layer is the case H = W = R = S = 1, N = M, C = I, K = O.
 */
lbt_status lbt_qconv_backward(const lbt_conv_desc *d, const float *dY, const void *q_W,
                              const void *q_X, const float *d_scale_w, const float *d_scale_x,
                              lbt_interval_state *st, lbt_grad_stats_t *stats, void *q_dY_out,
                              float *dX, float *dW, int32_t *accX, int32_t *accW, int bits_g,
                              void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * lbt_qconv_backward with the statistics of the NEXT gradient taken where they cost nothing (Sec. 3.1: the
 * quantizer of every layer needs g_max = max |G| over the layer's whole gradient tensor before it can
 * quantize one element, which is a second reading of that tensor).  The gradient a layer receives is the dX
 * the layer behind it has just produced -- directly, where no element-wise operation sits between the two
 * layers -- and the dgrad epilogue holds every element of dX in registers:
 *   dx_stats (device, optional, 8-byte aligned, not the same struct as `stats`): receives g_max = max |dX_i| over
 *     the finite elements, n = the element count of dX and n_nonfinite, exactly as lbt_grad_stats(dX, ...) would
 *     write them (n_out, c, scale cleared); needs dX != NULL.
 *   dy_stats_ready != 0: `stats` already holds g_max, n and n_nonfinite of THIS call's dY (an earlier call's
 *     dx_stats): the abs-max pass over dY is skipped, so dY is read once (4 B + codes per element instead of 8 B).
 *     The caller vouches that they belong to dY; everything else is as in lbt_qconv_backward.
 */
lbt_status lbt_qconv_backward_ex(const lbt_conv_desc *d, const float *dY, const void *q_W,
                                 const void *q_X, const float *d_scale_w, const float *d_scale_x,
                                 lbt_interval_state *st, lbt_grad_stats_t *stats, void *q_dY_out,
                                 float *dX, float *dW, int32_t *accX, int32_t *accW, int bits_g,
                                 void *ws, size_t ws_bytes, int dy_stats_ready,
                                 lbt_grad_stats_t *dx_stats, void *cuda_stream);

/*
 * Forward side of the same layer (Sec. 3.1, Eq. 1-4): the weight and activation quantizers with a
 * clipping value the caller owns (the paper learns it per layer), rounding to nearest (ties to
 * even), and the integer forward product on the same tensor-core kernels.
 *
 * lbt_quantize_weight: zero-centred input, Eq. (2): clip to [-c, c], s = c / (2^(b-1) - 1),
 *   signed codes in [-qmax, qmax].
 * lbt_quantize_act: input after a ReLU, Eq. (3): clip to [0, c], s = c / (2^b - 1), UNSIGNED codes in
 *   [0, 2^b - 1].
 * x: device, n fp32 elements, 16-byte aligned.  d_clip: device pointer to c (one float).  bits: 2..8.
 * q_out: device, 16-byte aligned, the header's storage format (bits <= 4: two codes per byte,
 * (n + 1) / 2 bytes; else n bytes) -- exactly what the q_W / q_X arguments of the contractions take.
 * d_scale_out: device pointer that receives s.  If s is not a positive finite number (c <= 0,
 * infinite or not a number) every code is 0 and s is reported as 0.  min / max drop a NaN operand, so
 * a NaN input takes the lower end of the interval; +-Inf saturate.  One pass: 4 bytes read and 0.5 or
 * 1 byte written per element.
 */
lbt_status lbt_quantize_weight(const float *w, uint64_t n, const float *d_clip, int bits,
                               void *q_out, float *d_scale_out, void *cuda_stream);
lbt_status lbt_quantize_act(const float *x, uint64_t n, const float *d_clip, int bits,
                            void *q_out, float *d_scale_out, void *cuda_stream);

/*
 * Forward product on codes:
 *   linear: Y[m,o]     = fl32(s_x * s_w) * sum_i q_X[m,i] q_W[o,i]
 *   conv:   Y[n,p,q,k] = fl32(s_x * s_w) * sum_{r,s,c} q_X[n, p*st + r - pad, q*st + s - pad, c] q_W[k,r,s,c]
 *           (taps outside the image contribute 0; NHWC / KRSC / NPQK as for the backward calls).
 * q_X: UNSIGNED codes of bits_x bits; q_W: signed codes of bits_w bits.  Y: fp32 output; acc_out
 * (optional): the raw int32 accumulators, same shape.  Workspace: lbt_workspace_bytes with
 * LBT_OP_GEMM_FORWARD / LBT_OP_CONV_FORWARD.  Errors as for the backward contractions
 * (LBT_ERR_ACC_RANGE if C*R*S * (2^bits_x - 1) * 2^(bits_w - 1) >= 2^31).
 */
lbt_status lbt_qgemm_forward(const void *q_X, const void *q_W, const float *d_scale_x,
                             const float *d_scale_w, float *Y, int32_t *acc_out,
                             int64_t M, int64_t O, int64_t I, int bits_x, int bits_w,
                             int32_t *dev_status, void *ws, size_t ws_bytes, void *cuda_stream);
lbt_status lbt_qconv_forward(const lbt_conv_desc *d, const void *q_X, const void *q_W,
                             const float *d_scale_x, const float *d_scale_w, float *Y,
                             int32_t *acc_out, int bits_x, int bits_w, int32_t *dev_status,
                             void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Pieces for batch-sharded (data-parallel) layers that must reproduce the one-GPU result bit for bit.
 * Sec. 3.1 defines g_max, and Sec. 3.3 / Eq. (9) the clip-out ratio, over ALL gradients of a layer, so
 * a layer whose batch is split over ranks reduces them over the ranks (max of g_max, sums of n,
 * n_nonfinite and n_out: plain collectives on the fields of lbt_grad_stats_t, done by the caller between
 * these calls) and sums the integer wgrad accumulators before the dequantising multiply:
 *
 * lbt_quantize_grad_shard: lbt_quantize_grad for a shard whose first element is element
 *   `index_offset` (a multiple of 8, else LBT_ERR_INVALID_ARG) of the whole tensor: the stochastic-
 *   rounding bits of dY[i] are those of element index_offset + i, so the codes equal the matching
 *   slice of the unsharded quantization.  stats->g_max and stats->n_nonfinite must already hold the
 *   reduced values; stats->n_out receives this shard's count.
 * lbt_dequantize_acc: out[i] = (float)acc[i] * fl32(*d_scale_a * *d_scale_b) for n int32 accumulators
 *   (the epilogue of the contractions, applied after the accumulators of all shards have been summed).
 *   acc, out: device, 16-byte aligned.
 */
lbt_status lbt_quantize_grad_shard(const float *dY, uint64_t n, uint64_t index_offset,
                                   const lbt_interval_state *st, lbt_grad_stats_t *stats,
                                   void *q_out, void *cuda_stream);
lbt_status lbt_dequantize_acc(const int32_t *acc, uint64_t n, const float *d_scale_a,
                              const float *d_scale_b, float *out, void *cuda_stream);

/*
 * Diagnostics of Sec. 3.2-3.3 for one quantized gradient tensor (not part of a training step):
 *   E(G)   = sum |g - Q(g)| / (N(G) g_max)                                   Eq. (5)
 *   E(G_L) = the same over the large gradients G_L, split into clip-in / clip-out   Eq. (6), (7)
 *   U(G_L) = (gamma / (2^b - 2) R_in + (1 - gamma) R_out) / (R_in + R_out)    Eq. (8)-(10)
 * G_L is the N(G_L) = alpha N (rounded to nearest, halves to even) gradients of largest magnitude; among
 * equal magnitudes the earlier elements (memory order) belong to it first.  Q(g) = scale * code with the
 * codes and the scale of the quantization being examined; a large gradient is clip-out when |g| > c;
 * gamma is taken as c / g_max.  dY: device, n >= 1 fp32 values (all finite), 16-byte aligned; q_codes:
 * the packed codes lbt_quantize_grad wrote for dY with `bits`; stats: that call's statistics (g_max, c,
 * scale); alpha: host value in [0, 1]; out: device struct; ws: at least lbt_diagnostics_workspace_bytes().
 * Sums are accumulated in binary64 (their last bits depend on the order of accumulation).
 */
typedef struct lbt_grad_diag_t {
    uint64_t n, n_large, n_in, n_out;               /* N(G), N(G_L), N(G_in), N(G_out)              */
    double   sum_all, sum_large_in, sum_large_out;  /* sums of |g - Q(g)|                           */
    double   e_all, e_large, u_large;               /* Eq. (5), Eq. (6) = (7), Eq. (8)              */
    float    threshold;                             /* smallest magnitude in G_L (0 if G_L is empty) */
    uint32_t reserved;
} lbt_grad_diag_t;                                  /* 88 bytes */
size_t lbt_diagnostics_workspace_bytes(void);
lbt_status lbt_grad_diagnostics(const float *dY, uint64_t n, const void *q_codes, int bits, float alpha,
                                const lbt_grad_stats_t *stats, lbt_grad_diag_t *out, void *ws,
                                size_t ws_bytes, void *cuda_stream);

/*
 * Transformer-side operators (the paper trains convolutional networks; these carry its low-bit training to a residual block
 * of a language model): a linear layer on 8-bit integers, the norms, gate and residual sum between two blocks, and the
 * optimizer's step.  Element types of their tensors: */
enum { LBT_F32 = 0, LBT_BF16 = 1, LBT_F16 = 2 };
/*
 * Matrices are row-major with a leading dimension ld (elements from one row to the next, >= the row's length).  Activation and
 * gradient tensors need only their element type's alignment; rows that begin on 32-byte (fp32) or 16-byte boundaries are read
 * in wide accesses.  Zero tokens (M = 0) are valid.  Outputs overlap no input unless a call says so.
 *
 * 8-bit rows: q[m,i] = rint(x[m,i] * fl(127 fl(1 / a_m))), a_m = max_i |x[m,i]|, scale[m] = fl(a_m fl(1/127)); ties to even,
 * codes in [-127, 127].  a_m <= 1e-36: scale 0, codes 0.  A row that holds an infinity or NaN: scale NaN, codes 0 (its row of
 * a product is NaN and no other).  Code rows are 16-byte aligned, ldq a multiple of 16; columns up to the next multiple of 16 hold 0.
 * Weights [O,I] give one scale per output channel, activations [M,I] one per token.
 */
lbt_status lbt_rows8_quantize(const void *x, int x_type, int64_t rows, int64_t cols, int64_t ld, void *q, int64_t ldq,
                              float *scale, void *cuda_stream);

/*
 * Y[m,o] = s_x[m] s_w[o] sum_i q_x[m,i] q_w[o,i] (+ bias[o], fp32, may be NULL).  q_x, q_w: code rows with ldq = I rounded up
 * to 16.  lbt_linear8_forward quantizes x first and leaves its codes and scales in q_x and s_x (caller's buffers: scratch, or
 * kept for the backward pass); lbt_linear8_matmul starts from codes.  I <= 133144 (127 * 127 * I < 2^31), else
 * LBT_ERR_ACC_RANGE.  dev_status (device int32, may be NULL) receives LBT_ERR_TIMEOUT if a bounded on-chip wait ran out;
 * the outputs that hang on it are not written.
 */
lbt_status lbt_linear8_forward(const void *x, int x_type, int64_t ldx, const void *q_w, const float *s_w, const float *bias,
                               void *y, int y_type, int64_t ldy, int64_t M, int64_t O, int64_t I, void *q_x, float *s_x,
                               int32_t *dev_status, void *cuda_stream);
lbt_status lbt_linear8_matmul(const void *q_x, const float *s_x, const void *q_w, const float *s_w, const float *bias, void *y,
                              int y_type, int64_t ldy, int64_t M, int64_t O, int64_t I, int32_t *dev_status, void *cuda_stream);

/*
 * Gradients of that layer, every product on 8-bit codes.  The scale of the reduced index is multiplied into dY before dY is
 * quantized:
 *   dX[m,i] = s_r[m] sum_o q_r[m,o] q_w[o,i]   (q_r, s_r) = 8-bit rows    of fl(dY[m,o] s_w[o])
 *   dW[o,i] = s_c[o] sum_m q_c[m,o] q_x[m,i]   (q_c, s_c) = 8-bit columns of fl(dY[m,o] s_x[m])
 *   dbias[o] = sum_m dY[m,o] (fp32)
 * Any of dX, dW, dbias may be NULL.  q_x, s_x: what the forward pass left.  O <= 133144 for dX, M <= 133144 for dW
 * (LBT_ERR_ACC_RANGE), M <= 4194240 in any case.  ws: lbt_linear8_workspace_bytes(M, O, I).
 */
size_t lbt_linear8_workspace_bytes(int64_t M, int64_t O, int64_t I);
lbt_status lbt_linear8_backward(const void *dY, int dy_type, int64_t lddy, const void *q_w, const float *s_w, const void *q_x,
                                const float *s_x, void *dX, int dx_type, int64_t lddx, void *dW, int dw_type, int64_t lddw,
                                float *dbias, int64_t M, int64_t O, int64_t I, int32_t *dev_status, void *ws, size_t ws_bytes,
                                void *cuda_stream);

/*
 * Between two residual blocks: u = N_post(h), r = scale_x x + scale_h gate u, y = N_pre(r), for M rows of D columns (D <= 32768).
 *   N(v) = w (v - mu) rstd + b; LBT_NORM_LAYER: mu = mean v, rstd = (mean (v - mu)^2 + eps)^(-1/2); LBT_NORM_RMS: mu = 0.
 * y is formed from r before r is rounded to its type.  Optional (NULL): gate (1), w_* (1), b_* (0; layer norms only), y and q (no second norm),
 * stats.  gate: [ceil(M / rows_per_gate), D], gate row m / rows_per_gate for row m; rows_per_gate 0 = one gate row for all.
 * q, q_scale: y's 8-bit rows as lbt_linear8_matmul takes them (codes of the fp32 y; q and y may both be asked for).
 * stats: [M,4] floats, 16-byte aligned, kept for the backward pass (mu and rstd of both norms).  r may be x, y may be h.
 */
enum { LBT_NORM_RMS = 0, LBT_NORM_LAYER = 1 };
typedef struct lbt_resnorm_desc {   /* HOST struct */
    int64_t M, D, rows_per_gate;
    int32_t type, param_type;       /* of x, h, r, y and their gradients; of gate, w, b and their gradients */
    int32_t kind, post_norm;        /* LBT_NORM_*; post_norm 0: u = h                                       */
    float eps_post, eps_pre, scale_x, scale_h;
    int64_t ld_x, ld_h, ld_r, ld_y, ld_dr, ld_dy, ld_dx, ld_dh;   /* 0 = D */
} lbt_resnorm_desc;
lbt_status lbt_resnorm_forward(const lbt_resnorm_desc *d, const void *x, const void *h, const void *gate, const void *w_post,
                               const void *b_post, const void *w_pre, const void *b_pre, void *r, void *y, void *q, int64_t ldq,
                               float *q_scale, float *stats, void *cuda_stream);

/*
 * Its gradients, from dr (of r) and dy (of y); either may be NULL (0).  x, h, gate, the parameters and stats are the forward
 * pass's (x and h unchanged: r is formed again in fp32).  dx, dh: [M,D]; dgate (needs gate), dw_post, db_post, dw_pre, db_pre:
 * param_type, NULL where not wanted; a gate row's gradient is the sum over its rows.  dx may be dr, dh may be dy.
 * ws: lbt_resnorm_workspace_bytes(d).  Sums are fp32 in an order fixed by M and D.
 */
size_t lbt_resnorm_workspace_bytes(const lbt_resnorm_desc *d);
lbt_status lbt_resnorm_backward(const lbt_resnorm_desc *d, const void *dr, const void *dy, const void *x, const void *h,
                                const void *gate, const void *w_post, const void *b_post, const void *w_pre, const float *stats,
                                void *dx, void *dh, void *dgate, void *dw_post, void *db_post, void *dw_pre, void *db_pre,
                                void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * One AdamW step (decoupled weight decay) over `count` tensors, one launch per 400 of them:
 *   g' = g * *d_grad_scale (1 if NULL);  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2;
 *   p = (1 - lr wd) p - (lr / (1 - b1^step)) m / (sqrt(v) / sqrt(1 - b2^step) + eps)
 * in fp32: the moments with every operation rounded once, the quotient of p's update within 2 ulp (v below 2^-126 counts as
 * nearly 0 there); p is rounded to its type once.  step counts from 1.  *d_skip != 0 (device int32, may be
 * NULL): nothing changes (a step whose gradients overflowed).
 * state_bits 32: m, v fp32.  state_bits 8: m and the root of v as e4m3 codes, one byte an element, in blocks of 256 consecutive
 * elements of a tensor: value = code * scale, scale = fl(max / 448) over the block's finite values, m_scale / v_scale:
 * ceil(n / 256) floats.  A positive root is never stored as code 0.  All-zero codes and scales are the state before step 1.
 * A non-finite gradient makes its own element's p, m and v non-finite and no other element's.  A finite one whose square
 * overflows makes v infinite and its element's updates 0; with state_bits 8 such a v is kept as NaN, which is read as infinity.
 * `tensors` (HOST) is read during the call.  Tensors need their element type's alignment; 32 bytes (fp32), 16 (16-bit) and
 * 8 (codes) are read in wide accesses.  n = 0 is valid.
 */
typedef struct lbt_adamw_tensor {
    void *p;            /* parameters, p_type          */
    const void *g;      /* gradients, g_type           */
    void *m, *v;        /* moments                     */
    float *m_scale, *v_scale;
    uint64_t n;
    double lr, weight_decay;
    int32_t p_type, g_type;
} lbt_adamw_tensor;     /* 80 bytes */
typedef struct lbt_adamw_hyper {
    double beta1, beta2, eps;
    int64_t step;
    int32_t state_bits, reserved;
} lbt_adamw_hyper;      /* 40 bytes */
lbt_status lbt_adamw_step(const lbt_adamw_tensor *tensors, int count, const lbt_adamw_hyper *h, const float *d_grad_scale,
                          const int32_t *d_skip, void *cuda_stream);
/*
 * The same with the held-back steps counted on the device, where alone they are known.  d_skipped (device int64, 8-byte aligned,
 * 0 before the first step; NULL: lbt_adamw_step): a call that *d_skip holds back adds 1 to it and changes nothing else, and a
 * call that is taken corrects with h->step - *d_skipped in place of h->step.  So h->step counts the calls, whatever became of them
 * (a call in a captured graph keeps the h->step of its capture: taking 1 from *d_skipped behind it makes each replay the next step).
 */
lbt_status lbt_adamw_step_ex(const lbt_adamw_tensor *tensors, int count, const lbt_adamw_hyper *h, const float *d_grad_scale,
                             const int32_t *d_skip, int64_t *d_skipped, void *cuda_stream);

/*
 * The norm of all gradients, and clipping by it, over `count` tensors (one launch each per 800 of them):
 *   norm = |s| (sum over all tensors of g^2)^(1/2),  s = *d_grad_scale (1 if NULL);   scale = s min(1, max_norm / norm)
 * summed in 64 bits in an order fixed by the sizes.  out->scale and &out->skip are what lbt_adamw_step takes as d_grad_scale and
 * d_skip: an infinity or NaN among the gradients (or as s) makes skip 1 and scale 0 (norm is then infinite or NaN), else skip is 0.
 * max_norm > 0 (infinity: measure only).  norms (may be NULL): the norm of each tensor, without s, count floats.
 * out (device, 4-byte aligned): `reserved` is 0 before the first call and between calls; a struct belongs to one call at a time.
 * ws: lbt_grad_norm_workspace_bytes(tensors, count) bytes, 8-byte aligned.
 * lbt_grad_clip: out_i = g_i * norm->scale in fp32, rounded to out's type once, for every tensor of the table; skip != 0: nothing is
 * written.  out may be g (then a scale of 1 writes nothing) and may have another type where it is not; it overlaps no other tensor of the table.
 * `tensors` (HOST) is read during the call.  Tensors need their element type's alignment; 32 bytes (fp32) and 16 (16-bit types) are
 * read in wide accesses.  n = 0 and count = 0 are valid (the norm of nothing is 0).
 */
typedef struct lbt_grad_tensor {
    const void *g;      /* gradients, g_type                    */
    void *out;          /* clipped, out_type (lbt_grad_clip)    */
    uint64_t n;
    int32_t g_type, out_type;
} lbt_grad_tensor;      /* 32 bytes */
typedef struct lbt_grad_norm_t {
    float norm, scale;
    int32_t skip;
    uint32_t reserved;
} lbt_grad_norm_t;      /* 16 bytes */
size_t lbt_grad_norm_workspace_bytes(const lbt_grad_tensor *tensors, int count);
lbt_status lbt_grad_norm(const lbt_grad_tensor *tensors, int count, double max_norm, const float *d_grad_scale, lbt_grad_norm_t *out,
                         float *norms, void *ws, size_t ws_bytes, void *cuda_stream);
lbt_status lbt_grad_clip(const lbt_grad_tensor *tensors, int count, const lbt_grad_norm_t *norm, void *cuda_stream);

/*
 * Low-rank adapters beside one linear layer: the tokens of run k, offsets[k] <= m < offsets[k+1], take adapter i = index[k]:
 *   h[m] = A_i x[m],  out[m,o] = base[m,o] + s_i sum_r h[m,r] B_i[r,o]
 * a: [adapters, rank, I], b: [adapters, rank, O] (both rank first, contiguous; an adapter of lower rank has rows of zeros); scale: s, one
 * float an adapter (NULL: ones).  x, base, out, a and b have one type.  offsets: runs + 1 ascending device ints, index: one for each run; both NULL: one run
 * of all M tokens with adapter 0.  An index outside [0, adapters) is a run without an adapter: out = base.  Rows of no run (ahead of
 * offsets[0], from offsets[runs] on) are not written; offsets are cut to [0, M].  out may be base.
 * h (may be NULL): [M, rank] floats, kept for the backward pass (rows without an adapter are not written).
 * Sums are fp32 in an order fixed by the sizes; h enters its second product with 16 (bf16) or 22 bits.  rank <= 128, adapters <= 65535, M and
 * runs <= 2^28, I and O <= 2^30 (LBT_ERR_UNSUPPORTED above).  dev_status (device int32,
 * may be NULL) receives LBT_ERR_TIMEOUT if a bounded on-chip wait ran out: out (dx) and h are then not complete, nor is what is formed from them.
 */
typedef struct lbt_adapters_desc {   /* HOST struct */
    int64_t M, I, O, runs;
    int32_t adapters, rank, type, reserved;
    int64_t ld_x, ld_base, ld_out, ld_dy, ld_dbase, ld_dx;   /* 0 = the row's length */
} lbt_adapters_desc;
lbt_status lbt_adapters_forward(const lbt_adapters_desc *d, const void *x, const void *a, const void *b, const float *scale,
                                const int32_t *offsets, const int32_t *index, const void *base, void *out, float *h, int32_t *dev_status,
                                void *cuda_stream);

/*
 * Its gradients: dh[m] = B_i dy[m], dx[m] = dbase[m] + s_i dh[m] A_i (dx may be dbase; rows as for out), and over all runs of adapter i
 * dA_i = s_i sum_m dh[m] x[m]^T, dB_i = s_i sum_m h[m] dy[m]^T: whole tensors like a and b of grad_type (LBT_F32, or the type of a), zeros
 * for an adapter without tokens.  Any of dx, da, db may be NULL; dx is written first, so it is not x where da is wanted, nor dy where db is.  x, h, runs: the forward pass's.  ws: lbt_adapters_workspace_bytes(d).
 */
size_t lbt_adapters_workspace_bytes(const lbt_adapters_desc *d);
lbt_status lbt_adapters_backward(const lbt_adapters_desc *d, const void *dy, const void *x, const float *h, const void *a, const void *b,
                                 const float *scale, const int32_t *offsets, const int32_t *index, const void *dbase, void *dx, void *da,
                                 void *db, int grad_type, int32_t *dev_status, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Group norm with an activation on channels-last images x[N,P,C] (P pixels, ld elements from one pixel to the next, images P ld apart):
 * for each image and each group of C / G neighbouring channels, mean and (biased) variance over the group's P C / G values,
 *   k = (x - mean) rstd, rstd = (var + eps)^(-1/2);  z = k w + b;  y = act(z): z, max(z, 0) or z / (1 + exp(-z)).
 * w, b: [C] of param_type (NULL: ones, zeros).  y or q may be NULL.  q: what lbt_quantize_act makes of the fp32 y with `bits` and d_clip
 * (dense, the storage of this header's codes: what lbt_qconv_forward takes), d_scale_out: its scale (of no images too); needs C a multiple of 8 and aligned rows.
 * stats (may be NULL): [N,G,2] floats, 8-byte aligned, mean and rstd, kept for the backward pass.  ws: lbt_groupnorm_workspace_bytes(d), 8-byte aligned.
 * N <= 65534, P <= 2^30, C <= 2^20 (LBT_ERR_UNSUPPORTED above).  No sum crosses images.  Sums are fp32 (of differences from a mean or a value of the channel) in an order fixed by the sizes.  y may be x (which
 * the backward pass reads, though).
 */
enum { LBT_ACT_NONE = 0, LBT_ACT_RELU = 1, LBT_ACT_SILU = 2 };
typedef struct lbt_groupnorm_desc {   /* HOST struct */
    int64_t N, P, C, G;
    int32_t type, param_type;   /* of x, y and their gradients; of w, b and their gradients */
    int32_t act;
    float eps;
    int64_t ld_x, ld_y, ld_dy, ld_dx;   /* 0 = C */
} lbt_groupnorm_desc;
size_t lbt_groupnorm_workspace_bytes(const lbt_groupnorm_desc *d);
lbt_status lbt_groupnorm_forward(const lbt_groupnorm_desc *d, const void *x, const void *w, const void *b, void *y, void *q, int bits,
                                 const float *d_clip, float *d_scale_out, float *stats, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Its gradients from dy; x, w, b, stats are the forward pass's.  dx, dw, db: any may be NULL.  dx may be dy.  The slope of a ReLU at 0 is 0.
 */
lbt_status lbt_groupnorm_backward(const lbt_groupnorm_desc *d, const void *dy, const void *x, const void *w, const void *b, const float *stats,
                                  void *dx, void *dw, void *db, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Measurement taps (no counterpart in the paper).  After this call the library records the two
 * events (cudaEvent_t passed as void*, created by the caller) on the call's stream immediately
 * before and after every launch of the named kernel class, so that a benchmark can time one
 * kernel inside a fused call with cudaEventElapsedTime.  Passing NULL for both removes the tap.
 * Process-wide and not thread-safe: meant for a benchmark's single thread.
 */
enum {
    LBT_TIME_STATS = 0,     /* abs-max reduction                   */
    LBT_TIME_QUANTIZE = 1,  /* quantize + clip-out count           */
    LBT_TIME_EXPAND = 2,    /* code expansion (all three operands) */
    LBT_TIME_DGRAD = 3,     /* tensor-core contraction for dX      */
    LBT_TIME_WGRAD = 4,     /* tensor-core contraction for dW      */
    LBT_TIME_FORWARD = 5,   /* tensor-core contraction for Y       */
    LBT_TIME_FWD_QUANT = 6, /* weight / activation quantizer       */
    LBT_TIME_CLASSES = 7
};
lbt_status lbt_set_timing_events(int kernel_class, void *ev_start, void *ev_stop);

/*
 * Self-test of the bounded on-chip waits (no counterpart in the paper).  Every wait inside the
 * contraction kernels gives up after a time limit, records LBT_ERR_TIMEOUT and lets the kernel end
 * in an orderly way.  This call runs that very wait routine in a one-thread kernel on a barrier
 * that nothing signals, with a limit of `limit_us` microseconds (1 .. 1 000 000), and stores
 * LBT_ERR_TIMEOUT in *dev_status (device int32, sticky like the other status words) when it
 * expires -- so a deployment can check that a lost signal ends in an error code and a usable
 * context, not in a hang.  Nothing faults and nothing is left running.
 */
lbt_status lbt_selftest_wait_timeout(int32_t *dev_status, uint32_t limit_us, void *cuda_stream);

/*
 * The same self-test for the other kind of bounded wait in the library: the grid barrier of the one-launch
 * quantizer (lbt_quantize_grad_fused), a counter in memory that every block adds to and then polls.  One
 * block arrives at a barrier that expects two, with a limit of `limit_us` microseconds (1 .. 1 000 000);
 * *dev_status becomes LBT_ERR_TIMEOUT when the wait gives up.  Nothing faults and nothing is left running.
 */
lbt_status lbt_selftest_barrier_timeout(int32_t *dev_status, uint32_t limit_us, void *cuda_stream);

/*
 * The same for the 8-bit layer's product whose reduction a cluster of CTAs shares: CTA `rank` of each cluster waits for a signal
 * that never comes, with a limit of `limit_us`.  *dev_status becomes LBT_ERR_TIMEOUT and y stays as it was, in the parts that the
 * other CTAs finish too.  y: fp32 [M,O]; codes and scales as lbt_linear8_matmul takes them.  LBT_ERR_UNSUPPORTED where the product of
 * this size is not cut into more than `rank` slices.
 */
lbt_status lbt_selftest_linear8_timeout(const void *q_x, const float *s_x, const void *q_w, const float *s_w, float *y, int64_t M,
                                        int64_t O, int64_t I, int rank, uint32_t limit_us, int32_t *dev_status, void *cuda_stream);

/*
 * The same for the adapters' kernel of long runs (bf16 or fp16, rows that begin on eight elements, one run of all M tokens with adapter 0): CTA
 * `rank` (0 .. 7) of each cluster is never told that its first product is done.  Where clusters have that CTA, *dev_status becomes
 * LBT_ERR_TIMEOUT and their rows of out stay as they were.
 */
lbt_status lbt_selftest_adapters_timeout(const lbt_adapters_desc *d, const void *x, const void *a, const void *b, const void *base, void *out,
                                         int rank, uint32_t limit_us, int32_t *dev_status, void *cuda_stream);

/* Static, NUL-terminated name of a status code. */
const char *lbt_status_string(lbt_status status);

#ifdef __cplusplus
}
#endif
#endif /* LBT_H_ */
