/*
 * ringada.h -- C ABI of libringada: the per-batch adapter fine-tuning step of RingAda
 * (arXiv 2502.19864) on one GB300.
 *
 * The step (Algorithm 1, the lines "Perform Fw propagation", "calculates the loss and
 * updates the head", "Perform Bw propagation ending at the (L - d + 1)-th adapter"; and
 * Section III-B.2) is:
 *   ra_forward            forward through all L frozen transformer blocks, each with two
 *                         Houlsby adapters h <- h + GELU(h W_down) W_up (Eq. 1), then the
 *                         head and the mean cross-entropy loss;
 *   ra_backward_truncated the backward from the loss down to the lowest unfrozen layer k
 *                         (0-based, k = L - d), with activation gradients through the
 *                         frozen weights of layers > k and weight gradients only for the
 *                         adapters of layers >= k and the head; layers < k get no work;
 *   ra_adapter_update     Adam on the unfrozen adapters and the trainable head;
 *   ra_set_unfrozen_depth the top-down unfreezing schedule's depth d (Algorithm 1,
 *                         "d = d + 1" every interval; Section III-A).
 *
 * Conventions
 *   - Every pointer named *_dev is a CUDA device pointer; everything else is host memory.
 *   - Device memory is owned by the caller (e.g. PyTorch): the library reports the sizes
 *     it needs (ra_required_bytes) and binds caller buffers (ra_bind_memory).  It never
 *     allocates device memory itself and never frees caller memory.
 *   - Calls that take a cudaStream_t enqueue work on that stream and return; results
 *     land on the device.  Caller inputs must stay valid until the stream reaches the work.
 *     A stream of 0 is the legacy default stream.
 *   - Errors are status codes; nothing throws or aborts.  ra_last_error(ctx) gives a
 *     message for the last failing call on that context.  On error, no work was enqueued
 *     by that call unless stated otherwise.
 *   - Device waits inside kernels are bounded; a wait that runs out records a flag that
 *     ra_sync_status reports as RA_ERR_TIMEOUT.
 *   - Thread safety: one context must not be used from two host threads at once.
 *   - Layout: activations are row-major [B, S, H] (token-major), B*S = T tokens.  Adapter
 *     matrices follow Eq. 1's row-vector convention: W_down [H, m], W_up [m, H].  Frozen
 *     linear weights are [out, in] (the product is x W^T).
 */
#ifndef RINGADA_H
#define RINGADA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* ra_stream_t; /* same type as cudaStream_t */

typedef enum {
  RA_OK = 0,
  RA_ERR_ARG = 1,         /* a null pointer, out-of-range index or size */
  RA_ERR_STATE = 2,       /* calls out of order (no memory bound, no forward before backward...) */
  RA_ERR_NOT_SAVED = 3,   /* backward asked to reach below the layers the forward saved */
  RA_ERR_SHAPE = 4,       /* B > max_batch, S > max_seq, or an unsupported model shape */
  RA_ERR_NOMEM = 5,       /* a bound buffer is smaller than required */
  RA_ERR_CUDA = 6,        /* a CUDA runtime/driver call failed (message has the CUDA error) */
  RA_ERR_TIMEOUT = 7,     /* a bounded device wait expired (kernel returned early) */
  RA_ERR_UNSUPPORTED = 8  /* no sm_103 device, or a feature this build does not have */
} ra_status;

enum { RA_ENCODER_POSTLN = 0, RA_DECODER_PRENORM = 1, RA_ENCODER_POSTLN_SPAN = 2 };
enum { RA_F32 = 0, RA_BF16 = 1 };
/* Adapter placement (ra_model_cfg.adapter_placement).
 *   RA_ADAPTERS_HOULSBY   two adapters per block, on the attention-output and FFN-output
 *                         branches before their residual add (both archs; parameters
 *                         RA_P_WDA/WUA and RA_P_WDF/WUF);
 *   RA_ADAPTERS_POST_FFN  the placement of the paper's Fig. 1 (Section II-A): one adapter
 *                         per block after the FFN's add & LayerNorm, out = y2 +
 *                         sigma(y2 W_down) W_up (Eq. 1 on the block's LayerNorm output),
 *                         nothing after it; encoders only; its matrices are RA_P_WDF/WUF
 *                         (RA_P_WDA/WUA are not part of such a model).  At the lowest
 *                         unfrozen layer the backward stops right after this adapter's
 *                         weight gradients. */
enum { RA_ADAPTERS_HOULSBY = 0, RA_ADAPTERS_POST_FFN = 1 };

/* Model shape.  Encoder: post-LN blocks (LayerNorm, biased linears, exact-GELU FFN), a
 * trainable n_out-class linear head on the token at position 0.  Span encoder
 * (RA_ENCODER_POSTLN_SPAN): the same blocks with the extractive-QA head of the paper's SQuAD
 * task (Section IV): start and end logits at every token (n_out = 2, max_seq <= 4096), loss
 * = mean over the batch of (CE_start + CE_end) / 2, each a softmax over the sequence.  Decoder: pre-RMSNorm
 * blocks, causal attention with rotate-half RoPE, SwiGLU FFN (ffn % 64 == 0), final
 * RMSNorm and a frozen n_out-way vocabulary head over every position. */
typedef struct {
  int32_t arch;            /* RA_ENCODER_POSTLN | RA_DECODER_PRENORM | RA_ENCODER_POSTLN_SPAN */
  int32_t n_layers;        /* L >= 1 */
  int32_t hidden;          /* H, multiple of 64 */
  int32_t n_heads;         /* H / n_heads in {64, 128} for bf16, <= 128 for f32 */
  int32_t ffn;             /* F, multiple of 64 */
  int32_t n_out;           /* classes (encoder) or vocabulary (decoder), multiple of 8 for decoder bf16 */
  int32_t max_batch;       /* capacity: ra_forward accepts B <= max_batch */
  int32_t max_seq;         /* capacity: ra_forward accepts S <= max_seq */
  int32_t dtype;           /* RA_F32 | RA_BF16: storage of weights and activations */
  int32_t head_trainable;  /* 1: the head is updated with the adapters (encoder); 0: frozen */
  int32_t max_depth;       /* largest unfreezing depth that will be used (0 = L); sizes the
                              saved-activation arena: memory falls as this falls */
  float norm_eps;          /* LayerNorm / RMSNorm epsilon */
  float rope_theta;        /* RoPE base (decoder) */
  int32_t adapter_placement; /* RA_ADAPTERS_HOULSBY (0) | RA_ADAPTERS_POST_FFN (encoders) */
  int32_t prefix_buffers;  /* encoders: 1 reserves the second set of forward scratch buffers
                              and the two prefix outputs of ra_forward_prefix/suffix */
} ra_model_cfg;

typedef struct {
  float lr, beta1, beta2, eps; /* Adam, no weight decay, bias-corrected */
} ra_adam_cfg;

/* Parameter ids for ra_set_weights / ra_get_grad. */
typedef enum {
  /* encoder block */
  RA_P_WQKV = 0, RA_P_BQKV, RA_P_WO, RA_P_BO, RA_P_LN1_G, RA_P_LN1_B,
  RA_P_W1, RA_P_B1, RA_P_W2, RA_P_B2, RA_P_LN2_G, RA_P_LN2_B,
  /* adapters (both archs): attention-branch and FFN-branch, Eq. 1 */
  RA_P_WDA, RA_P_WUA, RA_P_WDF, RA_P_WUF,
  /* decoder block */
  RA_P_WQ, RA_P_WK, RA_P_WV, RA_P_RMS1_G, RA_P_WG, RA_P_WU, RA_P_WD, RA_P_RMS2_G,
  /* head (layer index -1) */
  RA_P_HEAD_W, RA_P_HEAD_B, RA_P_RMSF_G,
  RA_P_COUNT
} ra_param;

typedef struct {
  int32_t layer;       /* 0..L-1, or -1 for the head */
  int32_t param;       /* ra_param */
  const float* data_dev; /* device, float32, row-major in the shape documented for the param;
                            values are rounded once to the model's storage dtype */
  int64_t numel;       /* must equal the param's element count */
} ra_tensor_desc;

typedef struct {
  int64_t weights_bytes, trainable_bytes, workspace_bytes; /* bound sizes */
  int64_t saved_bytes_capacity;  /* arena for max_depth layers */
  int64_t saved_bytes_in_use;    /* activations the last forward kept (layers >= k) */
  int32_t depth;                 /* current unfreezing depth d */
  int32_t k_forward;             /* lowest layer the last forward saved, -1 before any */
  int32_t k_backward;            /* lowest layer the last backward reached, -1 before any */
  int32_t n_updates;             /* completed ra_adapter_update calls */
  int32_t tokens;                /* B*S of the last forward */
  int32_t num_sms;               /* SMs of the bound device */
} ra_stats;

typedef struct ra_ctx ra_ctx;

/* Create a context for the model (host only; no device work).  adapter_dim = m (the
 * bottleneck of Eq. 1), 8 <= m <= 256, multiple of 8.  *out receives the context. */
ra_status ra_create(const ra_model_cfg* cfg, int32_t adapter_dim, ra_ctx** out);

/* Bytes the caller must provide: frozen weights (and their transposed copies),
 * trainable state (adapter/head masters, gradients, Adam moments) and workspace (saved
 * activations for max_depth layers plus scratch).  Each buffer must be 256-byte aligned. */
ra_status ra_required_bytes(const ra_ctx* ctx, size_t* weights, size_t* trainable,
                            size_t* workspace);

/* Bind caller-owned device buffers of at least the required sizes (sizes are given so
 * the library can check them).  Selects the current CUDA device as the context's device;
 * requires compute capability 10.3 (sm_103).  Zeroes gradients, moments and step counts. */
ra_status ra_bind_memory(ra_ctx* ctx, void* weights_dev, size_t weights_bytes,
                         void* trainable_dev, size_t trainable_bytes,
                         void* workspace_dev, size_t workspace_bytes);

/* Copy parameters in (frozen weights, initial adapters and head).  Every parameter of the
 * model must have been set once before the first ra_forward.  Builds the transposed
 * copies the backward reads.  Enqueued on stream. */
ra_status ra_set_weights(ra_ctx* ctx, const ra_tensor_desc* list, int32_t n, ra_stream_t stream);

/* Top-down unfreezing schedule (Algorithm 1: every `interval` rounds the depth grows by
 * one adapter layer, d <- d + 1, from the top down; Section IV unfreezes one more every 40
 * steps): the depth of 0-based step `step` is min(d0 + floor(step / interval), d_max).
 * Host-only, pure.  Returns -1 for step < 0, interval < 1, d0 < 1 or d_max < d0. */
int32_t ra_schedule_depth(int32_t step, int32_t interval, int32_t d0, int32_t d_max);

/* Unfreezing depth d (1..max_depth): the next forward saves activations for layers
 * k = L - d .. L-1 only (Section III-A: below the depth only the forward runs). */
ra_status ra_set_unfrozen_depth(ra_ctx* ctx, int32_t d);

/* Forward and loss (Algorithm 1 "Fw propagation", "calculates the loss").
 * x_dev [B, S, H] in the model dtype; labels_dev int32 [B] (encoder), [B, 2] = (start,
 * end) positions (span encoder) or [B, S] (decoder); loss_dev: one float (mean
 * cross-entropy); logits_dev: nullable, float [B, n_out] (encoder) or [B*S, n_out] (span
 * encoder, decoder).  Returns RA_ERR_SHAPE if B or S exceed capacity.  Labels out of range
 * are read as 0 and reported by ra_sync_status. */
ra_status ra_forward(ra_ctx* ctx, const void* x_dev, const int32_t* labels_dev, int32_t B,
                     int32_t S, float* loss_dev, float* logits_dev, ra_stream_t stream);

/* The same forward split in two, so that the next batch's frozen prefix can run while the
 * current batch is still in its backward and update (Section III-A: the forward below the
 * unfreezing depth is independent of the training above it and can run at the same time;
 * Section III-B.2).  Encoders only; the context needs cfg.prefix_buffers = 1.
 *
 * ra_forward_prefix runs blocks 0 .. k-1 (k = L - d for the depth set now) on x_dev
 * [B, S, H] and leaves the input of block k in prefix buffer `buf` (0 or 1); with k = 0 it
 * copies x_dev there.  It saves nothing and reads only the frozen weights and the adapters
 * of blocks below k, which no update at this or a larger depth writes, and it uses its own
 * scratch buffers: it may run on another stream concurrently with ra_forward_suffix of the
 * other buffer, ra_backward_truncated and ra_adapter_update.  The caller orders it after
 * the ra_forward_suffix that last read the same buffer.
 *
 * ra_forward_suffix runs blocks k .. L-1, the head and the loss from prefix buffer `buf`,
 * with the same arguments and results as ra_forward, and enables the backward as
 * ra_forward does.  The caller orders it after the prefix that filled `buf`.  Returns
 * RA_ERR_STATE if no prefix filled `buf` or the depth changed since, RA_ERR_UNSUPPORTED
 * without prefix buffers (or for a decoder). */
ra_status ra_forward_prefix(ra_ctx* ctx, const void* x_dev, int32_t B, int32_t S, int32_t buf,
                            ra_stream_t stream);
ra_status ra_forward_suffix(ra_ctx* ctx, int32_t buf, const int32_t* labels_dev,
                            float* loss_dev, float* logits_dev, ra_stream_t stream);

/* Backward ending at layer k (0-based; Algorithm 1 "Bw propagation ending at the
 * (L - d + 1)-th adapter" is k = L - d).  Requires a preceding forward; k must satisfy
 * L - d_forward <= k <= L - 1, else RA_ERR_NOT_SAVED (k too low) or RA_ERR_ARG.
 * Writes gradients of the adapters of layers >= k and of the head (if trainable); the
 * gradient buffers of layers < k are not touched.  Gradients are overwritten, not
 * accumulated. */
ra_status ra_backward_truncated(ra_ctx* ctx, int32_t k, ra_stream_t stream);

/* Adam step on the parameters the last backward produced gradients for (adapters of
 * layers >= k_backward, and the head if trainable).  A parameter's step count starts at
 * its first update.  Requires a backward since the last update, else RA_ERR_STATE. */
ra_status ra_adapter_update(ra_ctx* ctx, const ra_adam_cfg* adam, ra_stream_t stream);

/* Device pointer to a float32 gradient buffer (tests): layer 0..L-1 with RA_P_WDA..WUF,
 * or layer -1 with RA_P_HEAD_W / RA_P_HEAD_B.  *n receives the element count.  The
 * pointer stays valid while the memory is bound. */
ra_status ra_get_grad(ra_ctx* ctx, int32_t layer, int32_t which, const float** dev_ptr,
                      int64_t* n);

/* Device pointer to a float32 trainable parameter (master copy), same indexing. */
ra_status ra_get_param(ra_ctx* ctx, int32_t layer, int32_t which, const float** dev_ptr,
                       int64_t* n);

/* Checkpoint of the trainable state: masters, Adam moments, step counts and depth, as an
 * opaque host blob of ra_trainable_state_bytes bytes.  Synchronises the device. */
ra_status ra_trainable_state_bytes(const ra_ctx* ctx, size_t* n);
ra_status ra_get_trainable(ra_ctx* ctx, void* host, size_t n);
ra_status ra_set_trainable(ra_ctx* ctx, const void* host, size_t n);

/* Host-side counters and sizes (no device access). */
ra_status ra_get_stats(const ra_ctx* ctx, ra_stats* out);

/* Synchronise the stream and report whether any bounded wait expired since the last
 * call (RA_ERR_TIMEOUT), or a CUDA error occurred (RA_ERR_CUDA).  Clears the flag. */
ra_status ra_sync_status(ra_ctx* ctx, ra_stream_t stream);

/* Failure-detection hook: enqueues one kernel whose single thread waits, bounded by
 * limit_us microseconds (1 .. 1000000), on a device barrier that nothing ever signals --
 * the same bounded wait every pipelined kernel of the step uses.  The wait expires, the
 * kernel records the timeout and returns; the next ra_sync_status on the stream reports
 * RA_ERR_TIMEOUT and clears it.  Nothing faults or hangs, and the context stays usable. */
ra_status ra_selftest_wait_timeout(ra_ctx* ctx, int32_t limit_us, ra_stream_t stream);

/* Diagnostic: y = f(x) for n float32 values with the activation code the step's kernels
 * use (the sigma of Eq. 1 and its derivative, as the adapters and the fp32 kernels evaluate
 * it: the epilogues of the bf16 GEMMs have a form of their own, no further from the exact
 * value; SiLU of the decoder's SwiGLU FFN).
 * which: 0 GELU(x) = x Phi(x), 1 GELU'(x) = Phi(x) + x phi(x), 2 SiLU, 3 SiLU'.
 * x_dev, y_dev: device arrays of n floats owned by the caller (may alias).  Enqueued on
 * `stream`; RA_ERR_ARG for another `which` or n < 0, RA_ERR_CUDA on a launch error. */
ra_status ra_eval_activation(int32_t which, const float* x_dev, float* y_dev, int64_t n,
                             ra_stream_t stream);

/* Message of the last failing call on ctx (never null; "" if none). */
const char* ra_last_error(const ra_ctx* ctx);

/* Release the context (host memory only; bound device buffers stay the caller's). */
void ra_destroy(ra_ctx* ctx);

/* ---------------------------------------------------------------------------------------
 * Measurement.  With profiling on, every kernel call of the step is bracketed by a pair of
 * CUDA events on the call's stream (also when the calls are captured into a CUDA graph:
 * the events become graph nodes and a replay re-records them).  ra_profile_read sums the
 * elapsed times per category once the recorded work has completed, together with the
 * algorithmic work of those calls (flops: 2 M N K per GEMM, 4 S^2 dh per attention head
 * forward and 10 S^2 dh backward, halved when causal; bytes: each input read once and each
 * output written once).
 * ------------------------------------------------------------------------------------- */
typedef enum {
  RA_PROF_GEMM = 0,     /* frozen-weight GEMMs and their transposed-weight dX GEMMs */
  RA_PROF_ATTN_FWD,     /* fused attention forward */
  RA_PROF_ATTN_BWD,     /* fused attention backward */
  RA_PROF_ADAPTER_FWD,  /* adapter + residual + norm forward */
  RA_PROF_ADAPTER_BWD,  /* adapter backward with the in-kernel dW reduction */
  RA_PROF_NORM,         /* LayerNorm / RMSNorm kernels outside the adapter kernels */
  RA_PROF_HEAD,         /* head, loss, cross-entropy */
  RA_PROF_UPDATE,       /* Adam and the refresh of transposed adapter copies */
  RA_PROF_COUNT
} ra_prof_cat;

typedef struct {
  double ms[RA_PROF_COUNT];     /* summed device time of the calls, milliseconds */
  double flops[RA_PROF_COUNT];  /* algorithmic floating-point operations */
  double bytes[RA_PROF_COUNT];  /* algorithmic DRAM bytes */
  int32_t calls[RA_PROF_COUNT]; /* calls recorded */
} ra_profile;

/* on != 0: start recording (clears earlier records); on == 0: stop recording. */
ra_status ra_profile_enable(ra_ctx* ctx, int32_t on);
/* Sums the records; the caller must have synchronised the recorded work first. */
ra_status ra_profile_read(ra_ctx* ctx, ra_profile* out);
/* The individual records behind ra_profile_read, in call order: category, device
 * milliseconds, algorithmic flops and bytes of each recorded kernel call.  Writes up to
 * `max` records to out (host array) and the total number to *n. */
typedef struct {
  int32_t cat;
  float ms;
  double flops, bytes;
} ra_profile_record;
ra_status ra_profile_records(ra_ctx* ctx, ra_profile_record* out, int32_t max, int32_t* n);
/* Kernels this library has launched in this process so far (every entry point). */
int64_t ra_kernel_launches(void);

/* GEMM timing without per-kernel events (measurement support, no counterpart in the paper).
 * With ra_profile_gemm_log(ctx, 1) every GEMM launch of the following calls (forward,
 * backward) is also recorded: shapes, operands, epilogue and buffers.  ra_profile_gemm_replay
 * enqueues the recorded launches again, in order, back to back on stream (capturable in a
 * CUDA graph), and returns their count and algorithmic flops (2 M N K summed).  Timing that
 * replay gives the GEMM kernels' duration with the launch overlap they have in the step,
 * which an event pair around each kernel removes.  The replay overwrites the step's
 * activations: the next backward needs a new ra_forward (ra_backward_truncated returns
 * RA_ERR_STATE until then). */
ra_status ra_profile_gemm_log(ra_ctx* ctx, int32_t on);
ra_status ra_profile_gemm_replay(ra_ctx* ctx, int32_t* n_launches, double* flops, ra_stream_t stream);

/* ---------------------------------------------------------------------------------------
 * Stand-alone kernels, for testing each piece of the step in isolation.  No context.
 * ------------------------------------------------------------------------------------- */

/* C[M, N] = A[M, K] B[N, K]^T (+ bias[N]) on the tensor cores: bf16 operands, fp32
 * accumulation, bf16 output.  Row-major, leading dimensions equal the row lengths.
 * K % 8 == 0, N % 8 == 0 (16-byte rows).  bias_dev nullable (float).  gelu_out_dev
 * nullable: if given, also writes GELU(C) there (the FFN-up epilogue of the frozen
 * forward).  Returns RA_ERR_UNSUPPORTED on a device that is not sm_103. */
ra_status ra_gemm_bf16(const void* A_dev, const void* B_dev, void* C_dev, int32_t M, int32_t N,
                       int32_t K, const float* bias_dev, void* gelu_out_dev, ra_stream_t stream);

/* The same tensor-core GEMM with one of the step's fused epilogues, for tests and kernel
 * measurements (no counterpart in the paper: these are the step's dense contractions).
 * C = A[M, K] B[N, K]^T accumulated in fp32 (A, B bf16, K-major: lda = ldb = K), then
 *   RA_EPI_STORE       C = acc (+ bias)                  (C bf16 or f32: c_dtype)
 *   RA_EPI_BIAS_GELU   u = acc + bias: C = u (nullable), C2 = GELU(u)     (bf16)
 *   RA_EPI_BIAS_GELU_G u = acc + bias: C = GELU'(u) (nullable), C2 = GELU(u) (bf16)
 *   RA_EPI_MUL         C = acc * aux                     (aux bf16 [M, N], C c_dtype)
 *   RA_EPI_RESID       C = acc + aux                     (aux f32 [M, N], C f32)
 * Outputs are [M, N] row-major with leading dimension N.  bias: nullable f32 [N].  With
 * RA_EPI_B_KN or-ed into epi, B is given as stored [K, N] (N contiguous, leading dimension N),
 * the layout of a forward weight [out, in] that the backward's dX GEMMs multiply by.  Device
 * pointers, 16-byte aligned; N and K multiples of 8.  Enqueued on stream.  RA_ERR_SHAPE
 * for a combination the kernel does not take, RA_ERR_UNSUPPORTED without sm_103.
 * scratch_dev (nullable; 256-byte aligned, scratch_bytes >= ra_gemm_scratch_bytes(),
 * caller-owned, zero-filled before its first use; every call leaves it zeroed): lets the
 * STORE and GELU epilogues spread the k-blocks of a last, partial round of output tiles over
 * all CTAs (stream-K), each such tile summed from its CTAs' fp32 partials in a fixed order,
 * so results are deterministic.  Calls that may run at the same time need different
 * scratch.  Without it every tile is accumulated by one CTA.  RA_ERR_ARG for a scratch
 * that is too small or misaligned. */
enum { RA_EPI_STORE = 0, RA_EPI_BIAS_GELU = 1, RA_EPI_MUL = 2, RA_EPI_RESID = 3,
       RA_EPI_BIAS_GELU_G = 6, RA_EPI_B_KN = 0x100 };
size_t ra_gemm_scratch_bytes(void);
ra_status ra_gemm_bf16_epi(const void* A_dev, const void* B_dev, int32_t M, int32_t N, int32_t K,
                           int32_t epi, const float* bias_dev, const void* aux_dev, void* C_dev,
                           int32_t c_dtype, void* C2_dev, void* scratch_dev, size_t scratch_bytes,
                           ra_stream_t stream);

/* Adapter backward of Eq. 1 for T rows (the in-kernel weight-gradient reduction of the
 * step), float32 throughout.  g_dev [T, H] = dLoss/d(adapter output); h_dev [T, H] the
 * adapter input; z_dev [T, m] = h W_down saved by the forward; W_down [H, m], W_up [m, H].
 * Writes dW_down [H, m], dW_up [m, H] and, if dh_dev is not null, dh [T, H].
 * scratch_dev: caller scratch of ra_adapter_backward_scratch_bytes(T, H, m) bytes.
 * The result is deterministic (fixed reduction order). */
ra_status ra_adapter_backward(const float* g_dev, const float* h_dev, const float* z_dev,
                              const float* W_down_dev, const float* W_up_dev, int32_t T,
                              int32_t H, int32_t m, float* dW_down_dev, float* dW_up_dev,
                              float* dh_dev, void* scratch_dev, size_t scratch_bytes,
                              ra_stream_t stream);
size_t ra_adapter_backward_scratch_bytes(int32_t T, int32_t H, int32_t m);

/* Same computation as ra_adapter_backward, for callers that cannot allocate device memory:
 * plug-in hosts that hand a kernel only its input and output buffers and expose no
 * allocator (custom-operator slots of serving runtimes), and loops that forbid allocation
 * once running, because cudaMalloc can block, synchronise the device or fail at any time.
 * The paper has no counterpart; this is a deployment variant.
 * Scratch: a fixed 16 MiB device array inside the library (ra_adapter_backward_noalloc_
 * capacity() bytes), held on every GPU that loads the library until the process exits;
 * the call allocates nothing and frees nothing.  Sizes whose scratch need
 * (ra_adapter_backward_scratch_bytes) exceeds the array are rejected with RA_ERR_NOMEM.
 * The first call on a device looks up the array's device address (cudaGetSymbolAddress);
 * make that first call before any stream capture.  The address is kept per device together
 * with the CUDA context it belongs to; a call made after that context was destroyed and
 * re-created (e.g. by cudaDeviceReset) looks it up again, so it too should come before any
 * capture.  All calls share the one array: calls
 * that can overlap on the GPU (different streams without ordering) race on it and must be
 * serialised by the caller.  Nothing in the array needs to start at zero: every element a
 * call reads was written earlier in the same call. */
ra_status ra_adapter_backward_noalloc(const float* g_dev, const float* h_dev, const float* z_dev,
                                      const float* W_down_dev, const float* W_up_dev, int32_t T,
                                      int32_t H, int32_t m, float* dW_down_dev, float* dW_up_dev,
                                      float* dh_dev, ra_stream_t stream);
size_t ra_adapter_backward_noalloc_capacity(void);

/* ---------------------------------------------------------------------------------------
 * Operators that answer with a tuned decoder: a paged key-value cache, attention of the newest
 * tokens over it, its eviction, attention with a sliding window over whole sequences (forward and
 * backward) and the verification of drafted tokens.  The paper has no counterpart: it ends with the
 * tuned adapters.  No context: a call takes one argument block (a struct that the caller fills in,
 * zero for what it leaves out, and may keep for as long as its buffers stay) and a stream.
 *
 * Conventions, beside those at the top
 *   - Types are RA_F32 or RA_BF16, one for all of a call's queries, keys, values and outputs; sums,
 *     softmax statistics, log-sum-exps and accumulated weights are float32 in either case.
 *   - A stride is in elements, from one token's first head to the next token's; the heads of a token are
 *     next to each other, head_dim values each.  16-byte aligned bases, and strides and head dims whose
 *     rows keep that alignment (8 values of bf16, 4 of float32), or RA_ERR_ARG / RA_ERR_SHAPE.
 *   - RA_ERR_SHAPE, too, for sizes that the kernels' 32-bit counts do not hold: a cache of more than 2^31 - 4097
 *     slots a sequence, a token of 2^31 values, more than 2^28 drafts or 2^30 words, 2^31 tokens a call.
 *   - Grouped heads: query head h reads key-value head h / (n_heads / n_kv_heads); n_heads is a multiple
 *     of n_kv_heads.
 *   - Token i sees token j when j <= i and (window == 0 or i - j < window or j < sinks): the `window`
 *     newest tokens, itself among them, and the first `sinks` ones.  A query that sees nothing has output
 *     zero and log-sum-exp -inf.  scale is positive and finite (RA_ERR_ARG).  A key or value that is not finite
 *     reaches the tokens that see it; it may also reach tokens of its own sequence that do not.  Where a token's
 *     scores are NaN, its output and its log-sum-exp are NaN.
 *   - Outputs share no memory with inputs, but where a call says that they may.
 *   - A batch of 0, or sequences of seq = 0 tokens, are RA_OK without work; their pointers may be null.
 *   - A workspace is caller-owned, 256-byte aligned, at least the bytes that the call's _workspace_bytes
 *     gives for the same argument block (all of it but the workspace filled in: for a block that the call would
 *     refuse it gives 0), and zero-filled once before its first use: calls leave zero what they need to find
 *     zero, so that one may serve any of these operators, in any shapes, one call after the other.  Calls that
 *     may run at the same time need different workspaces, and after RA_DEV_TIMEOUT one has to be zero-filled
 *     again.  RA_ERR_NOMEM for one that is too small.
 *   - err_dev (nullable): a device word into which kernels or RA_DEV_BOUNDS where an index that they read on
 *     the device is out of range (a page of the table, a length, a position), and RA_DEV_TIMEOUT where a
 *     bounded wait ran out.  Such an index is never followed: a length is clamped to [0, capacity], tokens of
 *     a bad page are not there.
 *   - RA_ERR_UNSUPPORTED on a device that is not sm_103.
 * ------------------------------------------------------------------------------------- */
enum { RA_DEV_TIMEOUT = 1, RA_DEV_BOUNDS = 2 };

/* The cache of one layer: pages of page_size tokens, [n_pages, n_kv_heads, page_size, head_dim] for keys
 * and for values.  Slot s of sequence b (its s-th cached token) is row s % page_size of page
 * block_table[b, s / page_size].  head_dim <= 256, a multiple of 8 (bf16) or 4 (f32). */
typedef struct {
  void* k_dev;
  void* v_dev;
  const int32_t* block_table_dev; /* [batch, max_pages] */
  uint32_t* err_dev;              /* nullable */
  int32_t n_pages, max_pages, page_size, n_kv_heads, head_dim, dtype;
} ra_kv_cache;

/* Puts the keys and values of the n_new newest tokens of each sequence into the cache and turns queries
 * and keys by rotate-half RoPE: the pair (x_i, x_{i + head_dim/2}) becomes (x_i c - x_{i+} s, x_{i+} c +
 * x_i s) with (c, s) = rope[p, i], rope[p, head_dim/2 + i].  lens counts the new tokens: token t of
 * sequence b goes to slot lens[b] - n_new + t and has position p = pos[b] - n_new + t (pos NULL: lens; after
 * an eviction a sequence has seen more tokens than it has cached).  Tokens of negative slot are padding:
 * not stored, their rotated queries zero.  Positions outside [0, rope_len) are read at the nearest end and
 * reported.  q_dev NULL: keys and values alone.  rope_dev NULL: nothing is turned.  q_out may be q. */
typedef struct {
  ra_kv_cache cache;
  const int32_t* lens_dev;               /* [batch] */
  const int32_t* pos_dev;                /* [batch] or NULL */
  const void *q_dev, *k_dev, *v_dev;     /* [batch * n_new] tokens of n_heads / n_kv_heads heads */
  void* q_out_dev;                       /* [batch * n_new, n_heads, head_dim] */
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const float* rope_dev;                 /* [rope_len, head_dim]: cosines, then sines; or NULL */
  int32_t rope_len, batch, n_new, n_heads;
} ra_kv_append_args;
ra_status ra_kv_append(const ra_kv_append_args* args, ra_stream_t stream);

/* Attention of the n_new newest tokens of each sequence (token t at slot lens[b] - n_new + t, already in the
 * cache) over its cached tokens: out = softmax(scale q k^T) v over the slots that it sees.  One token a
 * sequence is the ordinary step; several check drafted ones.  The window counts slots: after an eviction, tokens
 * that were kept, not those that the sequence has seen.
 * weights_out (nullable): weights_out[b, e, s] = weights_in[b, e, s] + the softmax weights that slot s got
 * from the new tokens through the query heads of key-value head e, for s < lens[b] (weights_in NULL: 0; it
 * may be weights_out); other slots are not touched.
 * max_len: no sequence is longer (0: the table's capacity); it sizes the workspace and clamps lens. */
typedef struct {
  ra_kv_cache cache;
  const int32_t* lens_dev;               /* [batch] */
  const void* q_dev; int64_t q_stride;   /* [batch * n_new, n_heads, head_dim] */
  void* out_dev; int64_t out_stride;
  float* lse_dev;                        /* [batch, n_new, n_heads] natural log, or NULL */
  const float* weights_in_dev;           /* [batch, n_kv_heads, weights_stride] */
  float* weights_out_dev;
  int64_t weights_stride;
  void* workspace_dev; size_t workspace_bytes;
  int32_t batch, n_new, n_heads, max_len, window, sinks;
  float scale;
} ra_attention_decode_args;
size_t ra_attention_decode_workspace_bytes(const ra_attention_decode_args* args);
ra_status ra_attention_decode(const ra_attention_decode_args* args, ra_stream_t stream);

/* Eviction by accumulated weight.  A sequence of at most `budget` tokens keeps them all.  A longer one keeps,
 * for each key-value head by itself, its first `first` and its newest `recent` tokens and, of those
 * between, the budget - first - recent of the largest weight (of equal ones the lowest slots; a NaN counts as
 * larger than any number).  The kept tokens are copied in order to slots 0, 1, ... of the dst cache, whose
 * pages no src page of these sequences may be; kept[b, e, i] is the slot that slot i came from (-1 beyond
 * the new length), weights_out[b, e, i] its weight (0 up to budget), lens_out[b] = min(lens[b], budget)
 * (lens_out may be lens).
 * The weights are what ra_attention_decode has added up.  ra_attention_window_forward gives none: a prompt's tokens
 * have the weights that the tokens decoded after it gave them, and none where none has been.
 * RA_ERR_ARG for first + recent > budget; RA_ERR_SHAPE where src and dst differ in heads, head dim or type
 * or dst's table cannot hold budget tokens. */
typedef struct {
  ra_kv_cache src, dst;
  const int32_t* lens_dev;               /* [batch] */
  const float* weights_dev;              /* [batch, n_kv_heads, weights_stride] */
  int64_t weights_stride;
  int32_t* lens_out_dev;                 /* [batch] */
  int32_t* kept_dev;                     /* [batch, n_kv_heads, budget] */
  float* weights_out_dev;                /* [batch, n_kv_heads, weights_out_stride] or NULL */
  int64_t weights_out_stride;
  int32_t batch, max_len, budget, first, recent;
} ra_kv_evict_args;
ra_status ra_kv_evict(const ra_kv_evict_args* args, ra_stream_t stream);

/* Causal attention with a window and sinks over whole sequences [batch, seq] (a prompt, a training step):
 * out = softmax(scale q k^T) v over the tokens that each sees, and the log-sum-exp of each row.  lens
 * (nullable): sequence b has lens[b] tokens; rows past them see nothing and are seen by nothing, and what
 * their memory holds does not matter.  Head dims: 64 and 128 (bf16), multiples of 4 up to 128 (f32).
 * The backward takes the same block, with out and lse as the forward left them, and writes dq, dk and dv
 * (zero past a sequence's end), the shared heads' gradients summed over their query heads in a fixed order.
 * The workspace is for the backward alone. */
typedef struct {
  const void *q_dev, *k_dev, *v_dev;     /* [batch * seq] tokens of n_heads / n_kv_heads heads */
  int64_t q_stride, k_stride, v_stride;
  void* out_dev; int64_t out_stride;     /* [batch * seq, n_heads, head_dim] */
  float* lse_dev;                        /* [batch, n_heads, seq] natural log; NULL: forward alone */
  const int32_t* lens_dev;               /* [batch] or NULL */
  const void* dout_dev; int64_t dout_stride;
  void *dq_dev, *dk_dev, *dv_dev;
  int64_t dq_stride, dk_stride, dv_stride;
  void* workspace_dev; size_t workspace_bytes;
  uint32_t* err_dev;                     /* nullable */
  int32_t batch, seq, n_heads, n_kv_heads, head_dim, window, sinks, dtype;
  float scale;
} ra_attention_window_args;
size_t ra_attention_window_workspace_bytes(const ra_attention_window_args* args);
ra_status ra_attention_window_forward(const ra_attention_window_args* args, ra_stream_t stream);
ra_status ra_attention_window_backward(const ra_attention_window_args* args, ra_stream_t stream);

/* Verification of drafted tokens against the target's probabilities, from given random numbers, so that
 * what comes out is distributed as the target's own samples.  target[b, i] and draft[b, i] are the two
 * models' probabilities over the vocabulary for the place of drafted token tokens[b, i]; target has one
 * row more.  Drafted token i stands while uniform[b, i] * draft < target (compared without rounding) at
 * it and at all before it.  At the first that does not stand, n, the next token is
 * argmax_v max(target[b, n, v] - draft[b, n, v], 0) / noise[b, v], and target[b, n, v] / noise[b, v] where
 * all stand or that difference is nowhere positive; with noise exponentially distributed, a sample of the
 * normalised numerator.  Ties go to the lowest token; a probability or a quotient that is NaN counts as 0.
 * accepted[b] = n; out_tokens[b] = the n drafted tokens, the next one, then -1.  n_drafted (nullable): sequence
 * b has n_drafted[b] <= n_draft drafts.  A drafted token outside the vocabulary does not stand. */
typedef struct {
  const void* target_dev; int64_t target_stride; /* [batch, n_draft + 1] rows of vocab values */
  const void* draft_dev; int64_t draft_stride;   /* [batch, n_draft] rows */
  const int32_t* tokens_dev;                     /* [batch, n_draft] */
  const int32_t* n_drafted_dev;                  /* [batch] or NULL */
  const float* uniform_dev;                      /* [batch, n_draft] in [0, 1) */
  const float* noise_dev;                        /* [batch, vocab], positive */
  int32_t* accepted_dev;                         /* [batch] */
  int32_t* out_tokens_dev;                       /* [batch, n_draft + 1] */
  void* workspace_dev; size_t workspace_bytes;
  int32_t batch, n_draft, vocab, dtype;
} ra_verify_draft_args;
size_t ra_verify_draft_workspace_bytes(const ra_verify_draft_args* args);
ra_status ra_verify_draft(const ra_verify_draft_args* args, ra_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* RINGADA_H */
