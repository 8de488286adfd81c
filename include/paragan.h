/*
 * paragan.h -- C ABI of libparagan, the MI355X (gfx950) hot path of ParaGAN's
 * per-replica BigGAN training: spectrally normalised convolutions,
 * class-conditional BatchNorm, ReLU, nearest-upsample / avg-pool, the
 * self-attention block, the hinge loss and the D:G train step.
 *
 * The paper (ParaGAN, SoCC'24) trains BigGAN data-parallel: every replica
 * runs the generator and discriminator forward and backward passes on its
 * share of the batch, then synchronises gradients (Design, "Computation
 * Model").  This library is that per-replica compute on one GPU.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Status: every call returns PARAGAN_OK (0) or a negative PARAGAN_E*
 *   code.  Arguments are validated on the host before anything is enqueued:
 *   on error nothing has been launched and paragan_last_error() names the
 *   problem.  No C++ exception crosses the ABI.
 * - Streams: all device work is enqueued on the hipStream_t given to
 *   paragan_create(), in order; paragan_train_step and paragan_async_step
 *   also use a second stream of the context, and with
 *   paragan_set_overlap_wgrad on the step calls use a third (default
 *   priority, created on first use), ordered by events and idle again when
 *   the call returns, also on error.  Calls are asynchronous unless
 *   stated.
 * - Memory: every device buffer is allocated and owned by the caller and
 *   passed as a plain device pointer.  The library allocates no device
 *   memory; its one device-resident object is the fixed 4 MiB scratch
 *   array of paragan_sn_power_iter_noalloc, part of the loaded code.
 *   Sizes of the "saved" (forward -> backward) and "ws" (scratch) buffers
 *   come from the *_sizes() queries and must be 256-byte aligned.
 * - Activations are NHWC.  Their channel stride is the channel count
 *   rounded up to a multiple of 32 (paragan_cpad()); padded channels hold
 *   zeros on input and are written as zeros.  dtype PARAGAN_BF16 means
 *   bfloat16 activations with fp32 accumulation; PARAGAN_F32 means fp32
 *   throughout.
 * - Parameters of a module (block or network) live in ONE flat fp32 buffer
 *   in the order given by paragan_*_layout(); gradients and the Adam moments
 *   use the same layout.  Convolution weights are [Cout][kh][kw][Cin],
 *   linear weights [out][in], embeddings [classes][dim].  Spectral
 *   normalisation keeps one persistent fp32 vector u (length = the weight's
 *   row count, Cout) per SN weight in a separate flat "u" buffer, in
 *   layout order; training-mode forwards update it in place.
 * - Repeatability: the same call on the same values gives the same bits.
 *   Between calls of other sizes an image's last bits may differ, also where
 *   nothing couples the batch (the discriminator): kernels, and for the
 *   single-block calls the number of partial sums of a convolution, follow
 *   the batch.  A block called on its own and the same block inside a
 *   network may differ in the same way.  fp32 convolutions sum in one order
 *   at every size.
 * - Threading: a context is used by one host thread at a time.
 */
#ifndef PARAGAN_H
#define PARAGAN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  PARAGAN_OK = 0,
  PARAGAN_EINVAL = -1,        /* bad argument: null pointer, bad shape, ... */
  PARAGAN_EUNSUPPORTED = -2,  /* valid request this build does not handle */
  PARAGAN_EWORKSPACE = -3,    /* a buffer is smaller than the query said */
  PARAGAN_EHIP = -4,          /* a HIP runtime call failed */
  PARAGAN_ENONFINITE = -5,    /* train step produced a NaN/Inf loss */
  PARAGAN_ETIMEOUT = -6       /* a bounded wait ended without its event */
};

enum { PARAGAN_F32 = 0, PARAGAN_BF16 = 1 };

typedef struct paragan_ctx paragan_ctx;

/* Create a context bound to `hip_stream` (a hipStream_t; NULL = the null
 * stream) on the current device.  Checks that the device is gfx950. */
int paragan_create(paragan_ctx** out, void* hip_stream);
void paragan_destroy(paragan_ctx* ctx);
/* Message of the last failed call on this context (or of the last failed
 * paragan_create when ctx is NULL).  Valid until the next call. */
const char* paragan_last_error(const paragan_ctx* ctx);
/* Block until all work enqueued by this context has finished. */
int paragan_sync(paragan_ctx* ctx);
/* Off (0, the default) or on (1): whether the step calls (paragan_g_sample,
 * paragan_d_step, paragan_g_step, paragan_train_step) run the weight
 * gradients of each block backward -- with their bias column sums -- on a
 * further stream of the context (default priority), beside the block's
 * data gradients on the context's stream, ordered by events and joined
 * before the block's SN backward; every call returns with both streams
 * joined (also on error).  Results are bit-identical either way.  On, the
 * data- and weight-gradient kernels share the CUs, so a step finishes
 * sooner while each kernel's own launch takes longer: per-kernel rates
 * measured with it on count the shared time.  Returns PARAGAN_EINVAL for
 * other values. */
int paragan_set_overlap_wgrad(paragan_ctx* ctx, int on);

/* Clipping inside the step calls (paragan_d_step, paragan_g_step,
 * paragan_train_step, paragan_async_step).  With max_norm_g (max_norm_d) > 0
 * the generator's (discriminator's) optimiser steps take their gradient times
 * min(1, max_norm / norm), norm being the 2-norm of all of it; the gradients
 * the call leaves in `grads` are not clipped.  0 (the default): off, with the
 * results of before; infinity: only the norms are taken.  buf: device buffer
 * of paragan_grad_clip_size() bytes, 256-byte aligned, kept by the caller
 * until the last step called with it has run (NULL when both are off): its
 * first four floats are the generator's last norm and factor, then the
 * discriminator's.  A NaN in a gradient makes both of its floats NaN. */
int paragan_grad_clip_size(size_t* bytes);
int paragan_set_grad_clip(paragan_ctx* ctx, float max_norm_g, float max_norm_d,
                          void* buf);

/* Channel stride of an activation tensor with c channels. */
int64_t paragan_cpad(int64_t c);

/* One entry of a parameter layout. */
typedef struct {
  char name[48];       /* e.g. "g0.conv1.w" */
  int32_t ndim;
  int64_t shape[4];
  int64_t offset;      /* in floats, into the flat parameter buffer */
  int64_t u_offset;    /* in floats, into the flat u buffer; -1 if no SN */
} paragan_tensor_info;

/* ---------------------------------------------------------------------
 * Spectral normalisation (BigGAN's SN, as cited in Related Work): one
 * power iteration per training forward,
 *     v <- N(W^T u),  u <- N(W v),  sigma = u^T W v,   N(t) = t / max(|t|, eps),
 * repeated n_iter times.  W: device fp32, row-major rows x cols (the
 * weight viewed as (Cout, kh*kw*Cin)).  u: device fp32 [rows], read and
 * overwritten.  v: device fp32 [cols], written.  sigma: device fp32 scalar,
 * written.  rows, cols >= 1; n_iter >= 1.  ws: device scratch of
 * paragan_sn_ws_size() bytes, 256-byte aligned.
 * ------------------------------------------------------------------- */
int paragan_sn_ws_size(int64_t rows, int64_t cols, size_t* ws_bytes);
/* Validation only (no device work): the checks paragan_sn_power_iter makes
 * of its sizes and scalars. */
int paragan_sn_check(int64_t rows, int64_t cols, int n_iter, float eps);
int paragan_sn_power_iter(paragan_ctx* ctx, const float* W, int64_t rows,
                          int64_t cols, float* u, float* v, float* sigma,
                          int n_iter, float eps, void* ws);
/* For callers that cannot allocate device memory (code under stream
 * capture, serving loops, harnesses that forbid hipMalloc): the same
 * computation, with the same kernels and results, as paragan_sn_power_iter,
 * but its scratch is a 4 MiB array the library holds on each device until
 * the process ends (its address taken in paragan_create), so the caller
 * passes no workspace and the call allocates nothing.  Every BigGAN-128 and
 * BigGAN-512 SN weight fits (the largest needs about 1 MiB); a weight whose
 * paragan_sn_ws_size() exceeds 4 MiB is rejected with PARAGAN_EINVAL before
 * any work.  All calls on one device share that one array: calls that
 * overlap on a device (two streams, two threads, two contexts) race and
 * must be ordered by the caller.  The kernels write all scratch they read,
 * so nothing has to be cleared between calls. */
int paragan_sn_power_iter_noalloc(paragan_ctx* ctx, const float* W,
                                  int64_t rows, int64_t cols, float* u,
                                  float* v, float* sigma, int n_iter,
                                  float eps);

/* ---------------------------------------------------------------------
 * BigGAN generator residual block (spec block of the benchmark
 * model, Evaluation "Experiment Setup"):
 *   y = conv3x3(ReLU(cBN2(h1))) + b2 + conv1x1(up2(x)) + bsc,
 *   h1 = conv3x3(up2(ReLU(cBN1(x)))) + b1,
 *   cBN_k(t) = (1 + cond Wg_k^T) * BN(t) + cond Wb_k^T  (batch statistics),
 * every weight spectrally normalised.  x: [B][H][W][cpad(cin)], y:
 * [B][2H][2W][cpad(cout)], cond: fp32 [B][dc].  Parameter order from
 * paragan_gblock_layout(): bn1.gain bn1.bias conv1.w conv1.b bn2.gain
 * bn2.bias conv2.w conv2.b sc.w sc.b.
 * ------------------------------------------------------------------- */
typedef struct {
  int32_t B, H, W;       /* input batch and spatial size (H, W >= 1) */
  int32_t cin, cout, dc; /* channels in/out, width of cond */
  int32_t dtype;         /* PARAGAN_BF16 or PARAGAN_F32 */
  int32_t n_power_iter;  /* >= 1 */
  float bn_eps, sn_eps;
} paragan_gblock_desc;

int paragan_gblock_layout(const paragan_gblock_desc* d,
                          paragan_tensor_info* out, int32_t cap,
                          int32_t* count, int64_t* n_params, int64_t* n_u);
int paragan_gblock_sizes(const paragan_gblock_desc* d, size_t* saved_bytes,
                         size_t* ws_bytes);
int paragan_gblock_check(const paragan_gblock_desc* d);
/* Training forward: updates u, writes y and `saved` (read by bwd). */
int paragan_gblock_fwd(paragan_ctx* ctx, const paragan_gblock_desc* d,
                       const float* params, float* u, const void* x,
                       const float* cond, void* y, void* saved, void* ws);
/* Backward from dy ([B][2H][2W][cpad(cout)]): writes dx (x's shape),
 * dcond (fp32 [B][dc]) and grads (flat, parameter layout; overwritten). */
int paragan_gblock_bwd(paragan_ctx* ctx, const paragan_gblock_desc* d,
                       const float* params, const void* x, const float* cond,
                       const void* saved, const void* dy, void* dx,
                       float* dcond, float* grads, void* ws);

/* ---------------------------------------------------------------------
 * BigGAN discriminator residual block (the benchmark model's
 * discriminator, Evaluation "Experiment Setup"; its size pinned by Table
 * tab:GAN's 158.42M parameters):
 *   h = conv3x3([ReLU](x)) + b1,  main = [avgpool2](conv3x3(ReLU(h)) + b2),
 *   y = main + skip,  skip = conv1x1([avgpool2](x)) + bsc (learnable) or x.
 * x: [B][H][W][cpad(cin)] (bf16, or fp32 images when cin <= 4 and
 * x_f32), y: [B][H'][W'][cpad(cout)].  Parameters: conv1.w conv1.b
 * conv2.w conv2.b [sc.w sc.b].
 * ------------------------------------------------------------------- */
typedef struct {
  int32_t B, H, W, cin, cout;
  int32_t preact;        /* ReLU on the input of conv1 */
  int32_t downsample;    /* 2x2 avg-pool (H, W even) */
  int32_t learnable_sc;  /* 1x1 conv skip; required if cin != cout or pooled */
  int32_t dtype;
  int32_t n_power_iter;
  float sn_eps;
} paragan_dblock_desc;

int paragan_dblock_layout(const paragan_dblock_desc* d,
                          paragan_tensor_info* out, int32_t cap,
                          int32_t* count, int64_t* n_params, int64_t* n_u);
int paragan_dblock_sizes(const paragan_dblock_desc* d, size_t* saved_bytes,
                         size_t* ws_bytes);
int paragan_dblock_check(const paragan_dblock_desc* d);
int paragan_dblock_fwd(paragan_ctx* ctx, const paragan_dblock_desc* d,
                       const float* params, float* u, const void* x, void* y,
                       void* saved, void* ws);
/* dx may be NULL (input gradient not wanted). */
int paragan_dblock_bwd(paragan_ctx* ctx, const paragan_dblock_desc* d,
                       const float* params, const void* x, const void* saved,
                       const void* dy, void* dx, float* grads, void* ws);

/* ---------------------------------------------------------------------
 * Self-attention block of the benchmark BigGAN (Evaluation, "Experiment
 * Setup"; one per network at 64x64, counted in Table tab:GAN's 158.42M),
 * bf16 only:
 *   theta = x Wt^T (C/8), phi = maxpool2(x Wp^T) (C/8), g = maxpool2(x Wg^T)
 *   (C/2), P = softmax over keys of theta phi^T (no scaling),
 *   y = x + gamma * (P g) Wo^T.  SN on Wt Wp Wg Wo; gamma has none.
 * x, y: [B][H][W][cpad(C)], H and W even, C a multiple of 8.
 * Parameters: theta phi g o gamma.
 * ------------------------------------------------------------------- */
typedef struct {
  int32_t B, H, W, C;
  int32_t n_power_iter;
  float sn_eps;
} paragan_attn_desc;

int paragan_attn_layout(const paragan_attn_desc* d, paragan_tensor_info* out,
                        int32_t cap, int32_t* count, int64_t* n_params,
                        int64_t* n_u);
int paragan_attn_sizes(const paragan_attn_desc* d, size_t* saved_bytes,
                       size_t* ws_bytes);
int paragan_attn_check(const paragan_attn_desc* d);
int paragan_attn_fwd(paragan_ctx* ctx, const paragan_attn_desc* d,
                     const float* params, float* u, const void* x, void* y,
                     void* saved, void* ws);
int paragan_attn_bwd(paragan_ctx* ctx, const paragan_attn_desc* d,
                     const float* params, const void* x, const void* saved,
                     const void* dy, void* dx, float* grads, void* ws);

/* ---------------------------------------------------------------------
 * Operators of transformer blocks, for generators and discriminators that
 * mix tokens (image tokens, class tokens in front of them) with more than
 * the block above: norms of query and key heads with the position rotation,
 * and multi-head attention with a window, first tokens that stay visible,
 * ragged lengths and a learned relative position bias.  The projections
 * around them are the caller's.  Pointers are 16-byte aligned, strides are
 * in elements and multiples of 8.  The current device must be the context's.
 *
 * Norm and rotation of every head row x (d elements) of q and k, token t:
 *   n = x * (mean(x^2) + eps)^(-1/2) * gain    (gain_q or gain_k, [d] fp32)
 * then each pair (a, b) of the first `rot` elements becomes
 *   (a c - b s, a s + b c),  (c, s) = table[pos[t]][pair].
 * Pairs are (i, i + rot/2), or (2i, 2i + 1) with interleaved.  table: fp32
 * [n_pos][rot/2][2], any angles (for instance half of the pairs turned by a
 * token's row and half by its column); NULL when rot is 0.  pos: [T] device,
 * or NULL for t mod n_pos.  A token whose position is outside [0, n_pos) is
 * padding: its rows are not used, its outputs and gradients are zero.
 * Token t of q starts at q + t * ldq, its heads follow one another; outputs
 * likewise with ldqo and ldko.  dq, dk (the gradients of q, k) lie as q, k
 * do, dqo, dko (of the outputs) as the outputs do.  Outputs may be the
 * inputs (same pointer and stride); they must not overlap otherwise.
 * Statistics and sums are fp32.
 * ------------------------------------------------------------------- */
typedef struct {
  int64_t T;                       /* tokens, 1 .. 2^31 - 1 */
  int32_t Hq, Hk;                  /* query and key heads, >= 1 */
  int32_t d;                       /* head width, a multiple of 8 up to 256 */
  int32_t rot;                     /* rotated elements, a multiple of 16 up to d */
  int32_t interleaved;             /* pair order, 0 or 1 */
  int32_t n_pos;                   /* rows of the table, >= 1 */
  int32_t dtype;                   /* PARAGAN_BF16 or PARAGAN_F32: q, k, outputs, gradients */
  float eps;                       /* > 0, no smaller than the least normal float (1.2e-38) */
  int64_t ldq, ldk, ldqo, ldko;    /* >= heads * d */
} paragan_qknorm_desc;

int paragan_qknorm_check(const paragan_qknorm_desc* d);
/* Workspace of the backward. */
int paragan_qknorm_ws_size(const paragan_qknorm_desc* d, size_t* ws_bytes);
int paragan_qknorm_fwd(paragan_ctx* ctx, const paragan_qknorm_desc* d,
                       const void* q, const void* k, const float* gain_q,
                       const float* gain_k, const float* table,
                       const int32_t* pos, void* qo, void* ko);
/* Writes dq, dk and the gains' gradients ([d] fp32, overwritten). */
int paragan_qknorm_bwd(paragan_ctx* ctx, const paragan_qknorm_desc* d,
                       const void* q, const void* k, const float* gain_q,
                       const float* gain_k, const float* table,
                       const int32_t* pos, const void* dqo, const void* dko,
                       void* dq, void* dk, float* dgain_q, float* dgain_k,
                       void* ws);

/* Multi-head attention, bf16:
 *   S = scale * q k^T + bias,  P = softmax over the visible keys,  o = P v,
 * query head h reading key head h / (Hq / Hk).  Sequence b has len_q[b]
 * queries and len_k[b] keys (device arrays [B], or NULL for Sq and Sk; values
 * are clamped to [0, Sq] and [0, Sk]); query i stands at position
 * p = i + len_k - len_q, so a few new queries are the last tokens of a cache.
 * Key j is visible to it when j < len_k and
 *   causal: j <= p;   window > 0: |p - j| < window or j < n_sink.
 * A query that sees nothing gets zeros, one with a NaN among its scores gets
 * NaN.  Rows at and past len_q of o (and of dq), rows at and past len_k of dk
 * and dv, are written as zeros.  Keys and values at and past len_k, and those
 * that length, order and window let no query see, may hold anything and get
 * zero gradients; a NaN or infinity in a key or value that some query sees
 * can reach other queries, and one in a query or its dout other keys'
 * gradients (also where a bias of -infinity hides the key).
 * bias (n_buckets > 0): table fp32 [Hq][n_buckets] at the bucket of j - p.
 * With causal all buckets are for distances n = p - j >= 0; otherwise the
 * first half is for n = p - j >= 0 and the second for n = j - p > 0.  Of the
 * m buckets of a side, n < m/2 (rounded down) has bucket n, and above
 *   m/2 + floor(log(n / (m/2)) / log(max_distance / (m/2)) * (m - m/2)),
 * the last one from max_distance on.  Entries may be -infinity (such keys
 * are not visible); the lowest finite value is a number like any other (past
 * 2.3e38 in size all are one): the sum of a score and its bias is formed in
 * fp32, forward and backward.
 * Element (b, s, h, c) of a tensor is at b * stride[0] + s * stride[1]
 * + h * stride[2] + c.  q, k, v may repeat through zero strides in the
 * forward; o, and in the backward q, k and v (whose strides dq, dk and dv
 * share), must not overlap themselves.  dout has o's strides.  A stride
 * between tokens is below 2^24.  Outputs must not overlap inputs.
 * Softmax statistics and sums are fp32; P and dS are rounded to bf16 as
 * matrix operands. */
typedef struct {
  int32_t B, Sq, Sk;               /* sequences, queries and keys of each, >= 1; Sq, Sk <= 2^29;
                                      B * heads * ceil(S / 128) below 2^24 for either */
  int32_t Hq, Hk;                  /* query and key heads, Hq a multiple of Hk */
  int32_t d;                       /* head width, a multiple of 8 up to 128 */
  int32_t causal;                  /* 0 or 1 */
  int32_t window, n_sink;          /* 0: no window; n_sink counts with a window only; <= 2^29 */
  int32_t n_buckets, max_distance; /* 0: no bias; up to 256 (causal >= 2, otherwise even and >= 4);
                                      max_distance above half of a side's buckets, up to 512 */
  float scale;                     /* 1e-30 .. 1e30 */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
} paragan_mha_desc;

int paragan_mha_check(const paragan_mha_desc* d);
/* saved: kept from a forward to its backward; ws: scratch of either call (the
 * larger of both, mostly the backward's). */
int paragan_mha_sizes(const paragan_mha_desc* d, size_t* saved_bytes,
                      size_t* ws_bytes);
/* saved may be NULL when no backward follows (sampling, new tokens over a
 * cache: the form for few queries splits the keys over the card). */
int paragan_mha_fwd(paragan_ctx* ctx, const paragan_mha_desc* d,
                    const void* q, const void* k, const void* v,
                    const float* table, const int32_t* len_q,
                    const int32_t* len_k, void* o, void* saved, void* ws);
/* From the forward's o and saved, and dout: dq, dk, dv and dtable (fp32
 * [Hq][n_buckets], overwritten; NULL without a bias). */
int paragan_mha_bwd(paragan_ctx* ctx, const paragan_mha_desc* d,
                    const void* q, const void* k, const void* v,
                    const float* table, const int32_t* len_q,
                    const int32_t* len_k, const void* o, const void* saved,
                    const void* dout, void* dq, void* dk, void* dv,
                    float* dtable, void* ws);

/* ---------------------------------------------------------------------
 * The rest of a conditioned token block, and its training: the norms before
 * and after a block with modulation, gate and residual scale in one pass, a
 * gated linear recurrence that mixes tokens at linear cost, and the norm of
 * all gradients with clipping.  Pointers of token tensors are 16-byte
 * aligned, strides are in elements and multiples of 8, and sequence b has
 * len[b] tokens (device array [B], or NULL for S; values are clamped to
 * [0, S]): rows at and past it are not used, add to no gradient, and are
 * written as zeros.  The current device must be the context's.
 *
 * Block norm, for token (b, s) of the stream x and a block's output h (D
 * elements each):
 *   v = h   or, with post,  norm(h) * gain_post
 *   z = x + res_scale * gate[b] * v            (branch 0: z = x, no h)
 *   y = norm(z) * gain_pre * (1 + scale[b]) + shift[b]   (pre 0: no y)
 *   norm(t) = (t - mean t) * (mean (t - mean t)^2 + eps)^(-1/2)   (PARAGAN_NORM_LAYER)
 *           = t * (mean t^2 + eps)^(-1/2)                         (PARAGAN_NORM_RMS)
 * so one call ends a block and norms the next one's input; y is formed from
 * the unrounded z.  gain_post, gain_pre: fp32 [D]; gate, scale, shift: fp32
 * rows of D, mod_stride elements from one sequence's to the next one's (views
 * of one projection of the condition, for instance), or 0 for one row that
 * all sequences share (a norm's bias, a learned gate).  Each may be NULL: a
 * gain or gate of ones, a scale or shift of zeros; those of a part that the
 * descriptor leaves out (gain_post without post, for instance) are not used.
 * Statistics and sums are fp32 (sums over tokens are joined in 64 bits).
 * Element (b, s, c) of a tensor is at b * stride[0] + s * stride[1] + c.
 * z may be x and y may be h (same pointer and strides) where no backward
 * follows, which reads x and h; outputs must not overlap inputs otherwise.
 * ------------------------------------------------------------------- */
enum { PARAGAN_NORM_RMS = 0, PARAGAN_NORM_LAYER = 1 };

typedef struct {
  int32_t B, S;                    /* sequences, tokens of each, >= 1; B <= 2^20, B * S <= 2^30 */
  int32_t D;                       /* width, a multiple of 8 up to 8192 */
  int32_t dtype;                   /* PARAGAN_BF16 or PARAGAN_F32: h, y and their gradients */
  int32_t stream_dtype;            /* x, z and their gradients: dtype, or PARAGAN_F32 */
  int32_t kind;                    /* PARAGAN_NORM_RMS or PARAGAN_NORM_LAYER */
  int32_t branch, post, pre;       /* 0 or 1; branch or pre at least, post only with branch */
  float eps;                       /* > 0, no smaller than the least normal float (1.2e-38) */
  float res_scale;                 /* finite */
  int64_t mod_stride;              /* 0, or >= D and a multiple of 8 */
  int64_t x_stride[2], h_stride[2], z_stride[2], y_stride[2];
} paragan_blocknorm_desc;

int paragan_blocknorm_check(const paragan_blocknorm_desc* d);
/* saved: kept from a forward to its backward; ws: scratch of the backward. */
int paragan_blocknorm_sizes(const paragan_blocknorm_desc* d, size_t* saved_bytes,
                            size_t* ws_bytes);
/* saved may be NULL when no backward follows. */
int paragan_blocknorm_fwd(paragan_ctx* ctx, const paragan_blocknorm_desc* d,
                          const void* x, const void* h, const float* gain_post,
                          const float* gate, const float* gain_pre,
                          const float* scale, const float* shift,
                          const int32_t* len, void* z, void* y, void* saved);
/* From the forward's inputs and saved, dz (NULL: zero; z's strides, or x's
 * without a branch) and dy (y's strides; with pre): dx (x's strides), dh
 * (h's strides; with branch) and the gradients of the rows, fp32,
 * overwritten: dgain_post, dgain_pre [D]; dgate, dscale, dshift as gate, scale
 * and shift lie (with mod_stride 0 one row, the sum over all sequences).  Each
 * of these five may be NULL: not wanted. */
int paragan_blocknorm_bwd(paragan_ctx* ctx, const paragan_blocknorm_desc* d,
                          const void* x, const void* h, const float* gain_post,
                          const float* gate, const float* gain_pre,
                          const float* scale, const float* shift,
                          const int32_t* len, const void* saved,
                          const void* dz, const void* dy, void* dx, void* dh,
                          float* dgain_post, float* dgate, float* dgain_pre,
                          float* dscale, float* dshift, void* ws);

/* Gated linear recurrence, for every channel c of D by itself:
 *   a_t = exp(-sharp * softplus(decay[c]) * sigmoid(r_t)),
 *   h_t = a_t h_{t-1} + (1 - a_t^2)^(1/2) * sigmoid(g_t) * x_t,   y_t = h_t,
 * over the tokens of a sequence from the first to the last, or with reverse
 * from the last to the first.  x, r, g are the program's projections; decay:
 * fp32 [D], finite (where sharp * softplus(decay) is past 2.3e38 it counts as
 * that).  h0: the states before the first token taken, fp32
 * [B][D], or NULL for zeros; ht: those after the last, or NULL.  A sequence
 * of no tokens has ht = h0.  ht may be h0: with S = 1 that is the step of one
 * new token.  Outputs must not overlap inputs otherwise.  States and sums are
 * fp32; the backward divides by a root no smaller than 1.1e-19.  A NaN or infinity in a token reaches the tokens
 * after it (in the backward those before it too) of its sequence and channel,
 * and the channel's ddecay.  A stride between tokens is below 2^20. */
typedef struct {
  int32_t B, S;                    /* sequences, tokens of each, >= 1; B * S <= 2^30 */
  int32_t D;                       /* channels, a multiple of 8, up to 2^20; B * D < 2^31, B * ceil(D / 64) <= 2^22 */
  int32_t dtype;                   /* PARAGAN_BF16 or PARAGAN_F32: x, r, g, y and their gradients */
  int32_t reverse;                 /* 0 or 1 */
  float sharp;                     /* > 0, finite */
  int64_t x_stride[2], r_stride[2], g_stride[2], y_stride[2];   /* as above */
} paragan_scan_desc;

int paragan_scan_check(const paragan_scan_desc* d);
/* saved: kept from a forward to its backward; ws: scratch of either call. */
int paragan_scan_sizes(const paragan_scan_desc* d, size_t* saved_bytes, size_t* ws_bytes);
/* saved may be NULL when no backward follows.  Rows of x, r, g may overlap or
 * repeat (strides from 0 up) in the forward; y, and in the backward x, r and g
 * (whose strides dx, dr and dg share), must not overlap themselves. */
int paragan_scan_fwd(paragan_ctx* ctx, const paragan_scan_desc* d, const void* x,
                     const void* r, const void* g, const float* decay,
                     const int32_t* len, const float* h0, void* y, float* ht,
                     void* saved, void* ws);
/* From the forward's inputs and saved, dy (y's strides) and dht (fp32
 * [B][D], or NULL: zero): dx, dr, dg, ddecay (fp32 [D], overwritten) and dh0
 * (fp32 [B][D], or NULL: not wanted; it may be dht). */
int paragan_scan_bwd(paragan_ctx* ctx, const paragan_scan_desc* d, const void* x,
                     const void* r, const void* g, const float* decay,
                     const int32_t* len, const void* saved, const void* dy,
                     const float* dht, void* dx, void* dr, void* dg,
                     float* ddecay, float* dh0, void* ws);

/* The norm of all gradients together, and clipping:
 *   norm = grad_scale * (sum over all tensors of g^2)^(1/2),
 *   factor = grad_scale * (norm <= max_norm ? 1 : max_norm / norm),
 *   out = factor * g,
 * the sum in 64 bits and in a fixed order.  A NaN among the gradients makes
 * norm, factor and all outputs NaN; an infinity makes the norm infinite and
 * (with a finite max_norm) the factor zero, as these formulas say.  max_norm may be
 * infinite: nothing is clipped.  Outputs in place whose factor is one are
 * left alone.
 * The tensors are named once, in a plan: paragan_clip_plan writes it to host
 * memory of the size that paragan_clip_sizes gives, the caller copies it to
 * the device (8-byte aligned) and keeps the tensors where they are.  A tensor is n
 * contiguous elements at any place its type is aligned to; out may be grad
 * (in place); otherwise no two of them may overlap (refused).  n may be 0. */
typedef struct {
  const void* grad;
  void* out;                       /* grad's type and size; may be grad */
  int64_t n;                       /* 0 .. 2^40 */
  int32_t dtype;                   /* PARAGAN_BF16 or PARAGAN_F32 */
  int32_t reserved;                /* 0 */
} paragan_clip_tensor;

/* Filled by paragan_clip_plan, passed unchanged to paragan_clip. */
typedef struct {
  int64_t n_elements, n_pieces, bytes;
  int32_t n_tensors;
  int32_t in_place;                /* every out is its grad */
} paragan_clip_desc;

int paragan_clip_sizes(const paragan_clip_tensor* t, int32_t n_tensors,
                       size_t* plan_bytes, size_t* ws_bytes);
int paragan_clip_plan(const paragan_clip_tensor* t, int32_t n_tensors,
                      paragan_clip_desc* desc, void* plan_host);
/* plan: device copy; max_norm > 0; grad_scale > 0, finite; norm: device fp32
 * [2], written with norm and factor. */
int paragan_clip(paragan_ctx* ctx, const paragan_clip_desc* d, const void* plan,
                 float max_norm, float grad_scale, float* norm, void* ws);

/* ---------------------------------------------------------------------
 * Generator output layer (the last generator layer of the model,
 * Evaluation "Experiment Setup"; kept in fp32 arithmetic by the paper's
 * mixed-precision placement, Design "System Optimizations"):
 *   a = ReLU(gain * BN(x) + bias)   (batch statistics over B, H, W),
 *   img = tanh(conv3x3(a, W / sigma(W)) + b)   (3 output channels),
 * with SN on W.  x: bf16 [B][H][W][cpad(C)]; img: fp32 [B][H][W][3].
 * Shapes: cpad(C) <= 128 and W a multiple of 4 (paragan_gout_check says
 * whether W also fits the weight-gradient tile; every W up to 704 does).
 * Parameters: out_bn.gain out_bn.bias out_conv.w out_conv.b.
 * ------------------------------------------------------------------- */
typedef struct {
  int32_t B, H, W, C;
  int32_t n_power_iter;
  float bn_eps, sn_eps;
} paragan_gout_desc;

int paragan_gout_layout(const paragan_gout_desc* d, paragan_tensor_info* out,
                        int32_t cap, int32_t* count, int64_t* n_params,
                        int64_t* n_u);
int paragan_gout_sizes(const paragan_gout_desc* d, size_t* saved_bytes,
                       size_t* ws_bytes);
int paragan_gout_check(const paragan_gout_desc* d);
/* Training forward: updates u, writes img and `saved` (read by bwd). */
int paragan_gout_fwd(paragan_ctx* ctx, const paragan_gout_desc* d,
                     const float* params, float* u, const void* x, float* img,
                     void* saved, void* ws);
/* Backward from dimg (fp32 [B][H][W][3]); img is this layer's forward
 * output.  Writes dx (bf16, x's shape) and grads (flat, parameter layout;
 * overwritten). */
int paragan_gout_bwd(paragan_ctx* ctx, const paragan_gout_desc* d,
                     const float* params, const void* x, const float* img,
                     const void* saved, const float* dimg, void* dx,
                     float* grads, void* ws);

/* ---------------------------------------------------------------------
 * Optimisers.  The paper trains the two networks with different optimisers
 * (Numerical Optimizations, "Asymmetric Optimization Policy": AdaBelief for
 * the generator and Adam for the discriminator converge to the better
 * equilibrium).  Each network carries its own optimiser, on fp32 master
 * weights, with bias correction and no weight decay; t counts the steps
 * taken (the update computes step t + 1):
 *   Adam:       m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
 *               p -= lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
 *   AdaBelief (Zhuang et al., NeurIPS 2020, the method the paper cites):
 *               m = b1 m + (1 - b1) g,  s = b2 s + (1 - b2) (g - m)^2 + eps,
 *               p -= lr (m / (1 - b1^t)) / (sqrt(s / (1 - b2^t)) + eps)
 * ------------------------------------------------------------------- */
enum { PARAGAN_ADAM = 0, PARAGAN_ADABELIEF = 1 };

typedef struct {
  int32_t kind;         /* PARAGAN_ADAM or PARAGAN_ADABELIEF */
  float lr, beta1, beta2, eps;   /* lr >= 0, 0 <= beta < 1, eps > 0 */
} paragan_optim;

/* ---------------------------------------------------------------------
 * Full BigGAN networks and the G+D training iteration.  The architecture
 * is given by channel multipliers (BigGAN-128: ch 96, G 16,16,8,4,2,1, D
 * 1,2,4,8,16,16 with the last D block not pooling, attention at 64x64, 1000
 * classes, z 120 split into 6 chunks of 20, shared class embedding 128;
 * Evaluation, "Experiment Setup").  Hinge loss:
 *   L_D = mean relu(1 - D(x_real, y_real)) + mean relu(1 + D(x_fake, y_fake)),
 *   L_G = -mean D(G(z, y), y).
 * ------------------------------------------------------------------- */
typedef struct {
  int32_t img;          /* output resolution */
  int32_t ch;           /* base width */
  int32_t n_g;          /* generator blocks */
  int32_t g_mult[10];   /* n_g + 1 entries: C0 mult, then each block's out */
  int32_t n_d;          /* discriminator blocks */
  int32_t d_mult[10];   /* n_d entries */
  int32_t d_down[10];   /* n_d entries, 0/1 */
  int32_t attn_res;     /* 0: none */
  int32_t n_classes, dz, shared_dim;
  int32_t B;            /* per-GPU batch (D steps see 2B images) */
  int32_t n_power_iter;
  float bn_eps, sn_eps;
  paragan_optim opt_g, opt_d;   /* the generator's and the discriminator's */
} paragan_biggan_desc;

/* which = 0: generator, 1: discriminator. */
int paragan_net_layout(const paragan_biggan_desc* d, int32_t which,
                       paragan_tensor_info* out, int32_t cap, int32_t* count,
                       int64_t* n_params, int64_t* n_u);
int paragan_biggan_check(const paragan_biggan_desc* d);
/* Workspace of every step call below (one size serves them all). */
int paragan_train_step_ws_size(const paragan_biggan_desc* d, size_t* ws_bytes);

typedef struct {
  float* params;   /* flat fp32 master weights (updated by the optimiser) */
  float* u;        /* flat SN vectors (updated by every forward) */
  float* grads;    /* flat fp32: the last gradient computed (overwritten) */
  float* opt_m;    /* flat fp32 first moments */
  float* opt_v;    /* flat fp32 second moments (Adam's v, AdaBelief's s) */
  int64_t opt_t;   /* optimiser steps taken so far (host; incremented) */
} paragan_net_state;

/* Generator forward in training mode (batch statistics, SN u updated):
 * img (fp32 [B][img][img][3], in [-1, 1]) = G(z, y); z fp32 [B][dz], y [B].
 * No parameter changes other than u. */
int paragan_g_sample(paragan_ctx* ctx, const paragan_biggan_desc* d,
                     paragan_net_state* G, const float* z, const int32_t* y,
                     float* img, void* ws);

/* One discriminator step on supplied images: D forward, hinge, backward on
 * the batch concat(x_real, x_fake) with labels concat(y_real, y_fake)
 * (inputs sharing a weight are batched, Implementation "Hardware-Aware
 * Layout Transformation"), then D's optimiser.  x_real, x_fake: fp32
 * [B][img][img][3].  Writes D's gradients and L_D (loss_host, one float);
 * synchronises the stream at the end.  Returns PARAGAN_ENONFINITE (after
 * finishing the step) if L_D is not finite. */
int paragan_d_step(paragan_ctx* ctx, const paragan_biggan_desc* d,
                   paragan_net_state* D, const float* x_real,
                   const int32_t* y_real, const float* x_fake,
                   const int32_t* y_fake, void* ws, float* loss_host);

/* One generator step: G forward on (z, y), D forward (D's u updated, its
 * weights and optimiser state untouched), hinge L_G, D backward for the
 * input gradient only, G backward, G's optimiser.  Writes G's gradients and
 * L_G (loss_host); synchronises at the end; PARAGAN_ENONFINITE as above. */
int paragan_g_step(paragan_ctx* ctx, const paragan_biggan_desc* d,
                   paragan_net_state* G, paragan_net_state* D, const float* z,
                   const int32_t* y, void* ws, float* loss_host);

typedef struct {
  /* n_D entries each: */
  const float* const* x_real;   /* fp32 [B][img][img][3] images in [-1,1] */
  const int32_t* const* y_real; /* [B] */
  const float* const* z_fake;   /* fp32 [B][dz] */
  const int32_t* const* y_fake; /* [B] */
  const float* z_g;             /* fp32 [B][dz] for the generator step */
  const int32_t* y_g;           /* [B] */
} paragan_step_inputs;

/* One training iteration: n_D discriminator steps, each on
 * concat(real_k, G(z_k, y_k)) with labels concat(y_real_k, y_fake_k) -- the
 * same as paragan_g_sample followed by paragan_d_step -- then one generator
 * step on (z_g, y_g) as paragan_g_step; the D:G ratio n_D (1..63) is the
 * caller's (Numerical Optimizations, "Asynchronous Update Scheme": the
 * ratio is adjustable).  The results equal that sequence of calls bit for
 * bit.  Besides the context's stream the call uses a second stream of the
 * context (default priority), ordered by events, for the forwards' SN power
 * iterations and weight packing, which read only parameters; both streams
 * are idle when the call returns, also on error.  losses_host: n_D + 1
 * floats (L_D per D step, then L_G).  Returns PARAGAN_ENONFINITE (after
 * finishing the step) if a loss is not finite. */
int paragan_train_step(paragan_ctx* ctx, const paragan_biggan_desc* d,
                       paragan_net_state* G, paragan_net_state* D,
                       const paragan_step_inputs* in, int32_t n_D, void* ws,
                       float* losses_host);

/* ---------------------------------------------------------------------
 * The asynchronous update scheme (Numerical Optimizations, "Asynchronous
 * Update Scheme"), on one GPU.  One call is one iteration:
 *   1. the discriminator's parameters and SN vectors are copied to a
 *      snapshot held in the workspace;
 *   2. on the context's second stream: a generator step of batch n_D * B on
 *      (z, y) against the snapshot, as paragan_g_step (the snapshot's SN
 *      vectors advance and are discarded with it); its samples G(z, y),
 *      their labels and the snapshot's predictions D_snap(G(z, y)) are kept;
 *   3. concurrently on the context's stream: n_D discriminator steps, step k
 *      as paragan_d_step on x_real[k], y_real[k] and the k-th B samples and
 *      labels of img_buff / lab_buff -- the previous iteration's samples, so
 *      the discriminator sees fakes one generator update stale;
 *   4. after both: img_buff, lab_buff and pred_buff are replaced with this
 *      iteration's samples, labels and predictions.
 * The caller fills img_buff / lab_buff before the first iteration (e.g.
 * with paragan_g_sample).  Together the two sides need about the memory of
 * two generator steps and one discriminator step.
 *   x_real, y_real: n_D device pointers each (fp32 [B][img][img][3], [B]);
 *   z, y:           fp32 [n_D B][dz] and [n_D B] (the generator's batch);
 *   img_buff:       fp32 [n_D B][img][img][3], read then replaced;
 *   lab_buff:       [n_D B], read then replaced;
 *   pred_buff:      fp32 [n_D B], written.
 * losses_host: n_D + 1 floats (L_D per D step, then L_G against the
 * snapshot).  Both streams are idle when the call returns, also on error;
 * PARAGAN_ENONFINITE (after finishing the iteration) if a loss is not
 * finite.  ws: paragan_async_ws_size() bytes, 256-byte aligned.
 * ------------------------------------------------------------------- */
typedef struct {
  const float* const* x_real;
  const int32_t* const* y_real;
  const float* z;
  const int32_t* y;
  float* img_buff;
  int32_t* lab_buff;
  float* pred_buff;
} paragan_async_inputs;

int paragan_async_ws_size(const paragan_biggan_desc* d, int32_t n_D, size_t* ws_bytes);
int paragan_async_step(paragan_ctx* ctx, const paragan_biggan_desc* d,
                       paragan_net_state* G, paragan_net_state* D,
                       const paragan_async_inputs* in, int32_t n_D, void* ws,
                       float* losses_host);

/* ---------------------------------------------------------------------
 * Congestion-aware host data pipeline (Implementation, "Congestion-Aware
 * Data Pipelining").  Host threads fetch batches (by calling `fetch`) into
 * caller-provided host slots ahead of the consumer.  A sliding window holds
 * the latency of the last `window` fetches; once `window` fetches have
 * completed since the last change, a window mean above threshold_ms adds
 * one fetch thread and one batch of prefetch depth (up to the maxima), and a
 * mean at or below it releases one of each (down to the minima).  Depth
 * counts every batch a thread has claimed and the consumer has not yet
 * released.  Batches are delivered in sequence order 0, 1, 2, ..., each
 * exactly once, whatever the number of threads.  Host code only (no device
 * work, usable without a GPU); the caller copies a delivered slot to the
 * device (from pinned memory for an asynchronous copy) and then releases it.
 * Thread-safety: one consumer thread calls next, release and get_stats.
 * ------------------------------------------------------------------- */
/* Fill `slot` (slot_bytes bytes) with batch `seq`; return 0 on success.
 * Called from pipeline threads, concurrently for different seq. */
typedef int (*paragan_fetch_fn)(void* user, int64_t seq, void* slot, size_t slot_bytes);

typedef struct {
  int32_t min_threads, max_threads;   /* 1 <= min <= max <= 64 */
  int32_t min_depth, max_depth;       /* 1 <= min <= max <= n_slots */
  int32_t window;                     /* latency samples, 1 .. 100000 */
  double threshold_ms;                /* > 0 */
} paragan_pipeline_cfg;

typedef struct {
  int32_t threads, depth;             /* the controller's current targets */
  double window_mean_ms;              /* mean latency over the window */
  int64_t fetched, delivered;
  int64_t grows, shrinks;             /* controller adjustments so far */
  double consumer_wait_ms;            /* total time next() has waited */
} paragan_pipeline_stats;

typedef struct paragan_pipeline paragan_pipeline;

/* slots: n_slots host pointers of slot_bytes each, owned by the caller and
 * valid until paragan_pipeline_destroy returns.  Starts min_threads threads. */
int paragan_pipeline_create(paragan_pipeline** out, const paragan_pipeline_cfg* cfg,
                            paragan_fetch_fn fetch, void* user, void* const* slots,
                            int32_t n_slots, size_t slot_bytes);
/* Wait for the next batch in sequence order (timeout_ms < 0: no limit):
 * *seq, *slot.  The slot belongs to the consumer until released.
 * PARAGAN_ETIMEOUT if nothing came in time; PARAGAN_EINVAL when the batch
 * due is one whose fetch failed (the batches before it are delivered first;
 * nothing after it is fetched; the message names the batch). */
int paragan_pipeline_next(paragan_pipeline* p, int64_t* seq, int32_t* slot, int32_t timeout_ms);
int paragan_pipeline_release(paragan_pipeline* p, int32_t slot);
int paragan_pipeline_get_stats(paragan_pipeline* p, paragan_pipeline_stats* out);
/* Message of the last failed call on p (p = NULL: of the last failed
 * paragan_pipeline_create). */
const char* paragan_pipeline_error(const paragan_pipeline* p);
/* Stops the threads (a fetch in progress finishes first) and frees p. */
void paragan_pipeline_destroy(paragan_pipeline* p);

/* Seeded synthetic batches standing in for the image dataset: B images of
 * img x img x 3 floats then B int32 labels per slot.  Value i of batch seq
 * is 2u - 1 with u the top 24 bits of SplitMix64(seed + 2^40 seq + i) over
 * 2^24 (Steele, Lea and Flood, OOPSLA 2014: add 0x9E3779B97F4A7C15, then
 * the finaliser); label b is SplitMix64(seed + 2^40 seq + 2^39 + b) mod
 * n_classes.  latency_ms (host, n_latency entries, may be NULL) injects a
 * delay: fetching batch seq takes at least latency_ms[seq % n_latency]. */
typedef struct {
  uint64_t seed;
  int32_t B, img, n_classes;
  const float* latency_ms;
  int64_t n_latency;
} paragan_synth_source;

size_t paragan_synth_batch_bytes(const paragan_synth_source* s);
/* A paragan_fetch_fn with user = a paragan_synth_source*. */
int paragan_synth_fetch(void* user, int64_t seq, void* slot, size_t slot_bytes);

/* ---------------------------------------------------------------------
 * Launch profiler (instrumentation for the roofline report).  When enabled,
 * every convolution, weight-gradient and attention launch is bracketed by a
 * HIP event pair on the stream it runs on and tagged with its kernel
 * template instance and algorithmic FLOPs (real, unpadded channels); the
 * bandwidth-bound launches (SN power iteration and backward, weight packing,
 * BN statistics / apply / backward, column sums, pooling, the optimisers)
 * are tagged with their algorithmic HBM bytes instead.  Launches on the
 * context's second stream overlap the first, so their times include waiting
 * for CUs the other stream holds.
 * paragan_profile_read synchronises the stream, aggregates the records by
 * kernel name into `out` (up to `cap` entries; *count = number of kernels)
 * and clears them.  Off by default; costs two event records per launch.
 * enable = 1 turns it on; enable = 2 also appends each convolution and
 * weight-gradient launch's GEMM shape "[M,N,K]" to its name (rows =
 * pixels, N = padded output channels, K = padded taps x input channels),
 * so launches of one template instance aggregate per shape; 0 turns it off.
 * ------------------------------------------------------------------- */
typedef struct {
  char name[64];
  int64_t launches;
  double total_ms;
  double flops;
  double bytes;     /* algorithmic HBM bytes of the bandwidth-bound launches
                       (SN, packing, BN, column sums, pooling, optimiser) */
} paragan_kernel_stat;

int paragan_profile(paragan_ctx* ctx, int enable);
int paragan_profile_read(paragan_ctx* ctx, paragan_kernel_stat* out,
                         int32_t cap, int32_t* count);

#ifdef __cplusplus
}
#endif
#endif /* PARAGAN_H */
