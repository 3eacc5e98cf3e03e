/*
 * ringattn.h -- C ABI of the MI355X (gfx950) ring-attention library.
 *
 * Ring Attention with Blockwise Transformers (Liu, Zaharia, Abbeel; arXiv 2310.01889):
 * one host's share of exact blockwise self-attention.  The sequence of length S is split
 * into n_hosts equal blocks of c = S / n_hosts tokens; host i keeps query block i
 * resident while key/value blocks reach it in ring order, block (i - t) mod n_hosts at
 * step t (Section 3, "Ring-Based Blockwise Attention"; Appendix A forward code).  Each
 * block is folded into the output with running row maximum, running denominator and a
 * rescaled output accumulator.  The backward pass (Appendix A backward code) accumulates
 * dQ on the host and dK/dV with the rotating block.  A blockwise feed-forward network
 * (Section 2 equation; Algorithm 1) follows the attention of the same query block.
 *
 * On one GPU the ring is virtual: all hosts' blocks live in device memory.  Calls over
 * the whole ring are one launch (bf16 backward: one for dK/dV, one for dQ) that folds every
 * host's blocks, in ring order, where they lie.  Every other call runs n_hosts ring steps, each one kernel launch covering every host that has work at
 * that step, and the block each host needs at the next step reaches its per-host receive
 * buffer (double buffer) during the current step by device-to-device copies on a
 * library-owned side stream, overlapping the compute of the current step.
 *
 * Conventions shared by every entry point
 *   - Pointers are DEVICE pointers unless stated.  The caller allocates and owns every
 *     input and output and keeps them alive until `stream` has finished the call.  The
 *     library keeps no pointer after returning.
 *   - Tensors are dense row-major.  q, k, v, o, dO, dq, dk, dv: [B, S, H, D] (batch,
 *     position, head, dim per head; the layout of the paper's code).  lse: float32
 *     [B, H, S], holding max + ln(denominator) of the scaled scores (natural log).
 *   - Every tensor except lse (and the optional per-row rstd of rms_norm_fwd) starts on a
 *     16-byte boundary; lse and rstd on a 4-byte one.  Other pointers give RA_EINVAL.
 *   - "bf16" tensors hold IEEE bfloat16 (hip_bfloat16 / torch.bfloat16).  Products are
 *     taken in bf16 with float32 accumulation (the paper's float32-logits option);
 *     softmax statistics, accumulators and weight gradients are float32; outputs are
 *     rounded to bf16 with round-to-nearest-even.
 *   - Scores are scaled by 1/sqrt(D) (Section 2 equation).  With causal != 0, query at
 *     global position p sees key at global position p' iff p' <= p; masked keys
 *     contribute exactly zero and fully masked blocks are skipped.
 *   - Calls are asynchronous and stream-ordered on `stream` (a hipStream_t; NULL means
 *     the legacy default stream).  Work on a side stream is joined back to `stream`
 *     by events, so callers see single-stream semantics.  Distinct streams may be used
 *     from distinct threads concurrently.
 *   - Workspace (receive buffers, float32 accumulators) is allocated stream-ordered on
 *     `stream` from a memory pool the library owns on each device, and freed back to that
 *     pool at the end of the call (stream-ordered).  The pool keeps freed memory cached for
 *     later calls until the process ends or ring_attn_release_workspace() is called; the
 *     device's default memory pool and its settings are not touched.  Blocks of up to 64 MiB
 *     (256 MiB a device in all) of the NULL stream are kept for its next call instead.
 *   - Return value: RA_OK or an ra_status error code.  Arguments are validated before
 *     anything is enqueued: on error nothing is enqueued and outputs are untouched.
 *     ring_attn_last_error() describes the last error on the calling thread.  NaN or
 *     Inf inputs are not checked; they propagate.
 *
 * Supported shapes: D in {64, 128}; 1 <= n_hosts <= 64; S % n_hosts == 0; the block
 * c = S / n_hosts a multiple of 128 (bf16 attention) or 64 (float32 attention); B, H >= 1;
 * B * S * H * D < 2^31 elements per tensor.  ring_attn_fwd_varlen / ring_attn_bwd_varlen
 * (causal, bf16) take any S >= 1; the limits then hold for the padded length.
 */
#ifndef RINGATTN_H
#define RINGATTN_H

#include <hip/hip_runtime.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RA_OK = 0,
  RA_EINVAL = 1,        /* null pointer, non-positive size, bad enum value         */
  RA_EUNSUPPORTED = 2,  /* shape outside the supported set listed above            */
  RA_EHIP = 3,          /* a HIP launch, copy or event call failed                 */
  RA_ENOMEM = 4         /* workspace allocation failed                             */
} ra_status;

/* Activation of the feed-forward network. */
typedef enum { RA_ACT_GELU_ERF = 0, RA_ACT_RELU = 1, RA_ACT_GELU_TANH = 2 } ra_act;

/*
 * Ring attention forward (Section 3; Appendix A forward code), bf16.
 *   q, k, v  in   bf16 [B, S, H, D]
 *   o        out  bf16 [B, S, H, D]      softmax(q k^T / sqrt(D)) v, row by row
 *   lse      out  f32  [B, H, S]         log-sum-exp of each query's scaled scores
 *   n_hosts       number of virtual hosts of the ring; block c = S / n_hosts
 *   causal        0 or 1
 */
int ring_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                  int B, int H, int S, int D, int n_hosts, int causal, hipStream_t stream);

/*
 * Ring attention backward (Appendix A backward code), bf16.
 *   q, k, v, o, lse   the forward inputs and outputs (o, lse as written by ring_attn_fwd)
 *   dO        in   bf16 [B, S, H, D]   upstream gradient of o
 *   dq, dk, dv out bf16 [B, S, H, D]   gradients of sum(dO * o); accumulated in float32
 *                                      (dq with the host, dk/dv with their block)
 *                                      and rounded once at the end.
 */
int ring_attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                  const void* dO, void* dq, void* dk, void* dv,
                  int B, int H, int S, int D, int n_hosts, int causal, hipStream_t stream);

/*
 * Causal ring attention for any sequence length S >= 1 (Section 3: the sequence is cut into
 * one block per host; here the last blocks may be short or empty), bf16.  The block is
 * c = the smallest multiple of 128 with n_hosts * c >= S.  Rows past S count as zero.  Padded
 * keys lie after every real query, so the causal mask hides them; padded query rows add
 * exactly zero to dK and dV.  Arguments, layouts and outputs as ring_attn_fwd /
 * ring_attn_bwd with causal = 1; S need not be a multiple of n_hosts or of 128; nothing is
 * copied.  Errors: RA_EINVAL for null pointers or
 * non-positive sizes, RA_EUNSUPPORTED when the padded shape is outside the supported set.
 */
int ring_attn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                         int B, int H, int S, int D, int n_hosts, hipStream_t stream);
int ring_attn_bwd_varlen(const void* q, const void* k, const void* v, const void* o,
                         const float* lse, const void* dO, void* dq, void* dk, void* dv,
                         int B, int H, int S, int D, int n_hosts, hipStream_t stream);

/* float32 twins of ring_attn_fwd / ring_attn_bwd: every tensor is float32, products and
 * accumulation are float32 (no bf16 rounding anywhere). */
int ring_attn_fwd_f32(const float* q, const float* k, const float* v, float* o, float* lse,
                      int B, int H, int S, int D, int n_hosts, int causal, hipStream_t stream);
int ring_attn_bwd_f32(const float* q, const float* k, const float* v, const float* o,
                      const float* lse, const float* dO, float* dq, float* dk, float* dv,
                      int B, int H, int S, int D, int n_hosts, int causal, hipStream_t stream);

/*
 * One host's share of the ring (Section 3; the per-host view of Figure 2 and of the
 * Appendix A scan), bf16: query block `host_idx` against every key/value block, the
 * blocks arriving in ring order (host_idx - t) mod n_hosts, step 0 being the host's own
 * block, each later block prefetched into the host's receive buffer on the side stream.
 *   q_blk     in   bf16 [B, c, H, D]    query block host_idx (global positions host_idx*c + r)
 *   k_all, v_all in bf16 [B, S, H, D]   all key/value blocks, S = n_hosts * c
 *   o_blk     out  bf16 [B, c, H, D]
 *   lse_blk   out  f32  [B, H, c]
 */
int ring_attn_fwd_host(const void* q_blk, const void* k_all, const void* v_all, void* o_blk,
                       float* lse_blk, int B, int H, int S, int D, int n_hosts, int host_idx,
                       int causal, hipStream_t stream);

/*
 * One host's share of the ring backward (Appendix A backward code seen from host
 * host_idx), bf16: dq of query block host_idx, and this host's contribution to the float32
 * dK_j, dV_j that travel with every key/value block j.  Blocks arrive in ring order
 * (host_idx - t) mod n_hosts; from step 1 on, K_j, V_j and the gradients dK_j, dV_j they carry
 * are received into the host's double buffer on the side stream, the host adds its
 * contribution, and the gradients are passed on (copied out) -- three times the bytes of
 * the forward rotation.
 *   q_blk, o_blk, dO_blk  in  bf16 [B, c, H, D];  lse_blk in f32 [B, H, c] (ring_attn_fwd_host)
 *   k_all, v_all          in  bf16 [B, S, H, D]
 *   dq_blk                out bf16 [B, c, H, D]
 *   dk_acc, dv_acc        in/out f32 [B, S, H, D]: the gradients the blocks carry when they
 *                         reach this host; this host's contributions are added.
 */
int ring_attn_bwd_host(const void* q_blk, const void* k_all, const void* v_all, const void* o_blk,
                       const float* lse_blk, const void* dO_blk, void* dq_blk, float* dk_acc,
                       float* dv_acc, int B, int H, int S, int D, int n_hosts, int host_idx,
                       int causal, hipStream_t stream);

/*
 * Ring attention forward with an explicit block order, bf16 (checks the permutation
 * invariance that Section 3 relies on: blocks may be folded in any order).
 *   kv_order  HOST pointer, int[n_hosts * n_hosts]; row i is the sequence of key/value
 *             blocks host i folds in, a permutation of 0..n_hosts-1.  Copied before return.
 * Otherwise as ring_attn_fwd.  Returns RA_EINVAL if a row is not a permutation.
 */
int ring_attn_fwd_ordered(const void* q, const void* k, const void* v, void* o, float* lse,
                          int B, int H, int S, int D, int n_hosts, int causal,
                          const int* kv_order, hipStream_t stream);

/*
 * Ring decode (the paper's appendix on the inference requirement), bf16: the Tq newest
 * tokens attend to a key/value cache of S tokens that stays split in n_hosts blocks of
 * c = S / n_hosts over the ring.  The queries sit at global positions S - Tq .. S - 1
 * (their own keys and values are the last Tq rows of the cache) on the last host, and the
 * blocks are folded into their running maximum / numerator / denominator in ring order,
 * block n_hosts-1 first, then n_hosts-2, ..., 0 (Section 3), with the online-softmax
 * recurrence of Section 2.  With causal != 0 query t sees cache positions <= S - Tq + t;
 * otherwise the whole cache.  On one GPU all blocks are resident: one launch computes the
 * partial state of every block (each split in chunks, one wave per chunk; the step reads
 * the whole cache once and is bound by HBM bandwidth) and a second folds them in ring
 * order.
 *   q        in   bf16 [B, Tq, H, D]
 *   k_cache, v_cache in bf16 [B, S, H, D]
 *   o        out  bf16 [B, Tq, H, D]
 *   lse      out  f32  [B, H, Tq]      max + ln(denominator) of each query's scaled scores
 *   1 <= Tq <= min(32, S); D in {64, 128}; S % n_hosts == 0 and c a multiple of 32;
 *   n_hosts <= 64.  Workspace: B * H * (S / chunk) * Tq * (D + 2) floats, stream-ordered.
 */
int ring_attn_decode(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                     int B, int H, int S, int D, int Tq, int n_hosts, int causal,
                     hipStream_t stream);

/*
 * ring_attn_decode for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same arguments, same
 * kernels and the same result as ring_attn_decode, bit for bit, but no allocation of any
 * kind: the chunk partial states live in a fixed 32 MiB device array (8388608 floats) that
 * the library holds on every device it runs on until the process ends.  The call is held to
 * B * H * nch * Tq * (D + 2) floats of it, with nch = S / kch chunks, kch = the block
 * S / n_hosts halved while B * H * nch < 4096 and the half stays a multiple of 32 (e.g.
 * B = 1, H = 32, D = 128, S = 262144 over 8 hosts: nch = 128, Tq <= 15); larger shapes
 * return RA_EUNSUPPORTED before anything is enqueued.  Every call on a device uses that
 * device's one array (nothing in it has to start at zero: each call writes every entry it
 * reads), so calls that overlap on one device -- on different streams, or from different
 * threads without ordering -- race and give wrong results; order them on one stream.
 */
int ring_attn_decode_noalloc(const void* q, const void* k_cache, const void* v_cache, void* o,
                             float* lse, int B, int H, int S, int D, int Tq, int n_hosts,
                             int causal, hipStream_t stream);

/*
 * Blockwise feed-forward network (Section 2 equation and "Blockwise Parallel
 * Transformers"; Algorithm 1's feed-forward step), bf16:
 *   y = act(x W1 + b1) W2 + b2, computed in groups of whole `block`s: as many as fill the chip
 *   twice, 2^25 / min(d_model, d_ff) rows, and 1.25 GiB of [rows, d_ff] intermediates hold,
 *   one block at least.  The intermediates are 2 bytes a hidden unit and row here, 8 in the
 *   backward; 2 and 14 in swiglu_ffn and its backward.  Weight gradients sum each block by
 *   itself and add up the blocks in order, whatever the groups.
 *   x  in bf16 [T, d_model];  w1 in bf16 [d_model, d_ff];  b1 in bf16 [d_ff] or NULL
 *   w2 in bf16 [d_ff, d_model];  b2 in bf16 [d_model] or NULL;  y out bf16 [T, d_model]
 *   act: an ra_act value.   T % block == 0, block % 256 == 0, d_model % 256 == 0,
 *   d_ff % 256 == 0.
 */
int blockwise_ffn(const void* x, const void* w1, const void* b1, const void* w2, const void* b2,
                  void* y, int T, int d_model, int d_ff, int block, int act, hipStream_t stream);

/*
 * Backward of blockwise_ffn for upstream dy (bf16 [T, d_model]).  The pre-activation
 * x W1 + b1 is recomputed group by group (gradient checkpointing, Section 4 setting).
 *   dx  out bf16 [T, d_model]
 *   dw1 out f32 [d_model, d_ff], db1 out f32 [d_ff] (may be NULL),
 *   dw2 out f32 [d_ff, d_model], db2 out f32 [d_model] (may be NULL).
 * Weight and bias gradients are overwritten (not accumulated into) and kept in float32.
 */
int blockwise_ffn_bwd(const void* x, const void* w1, const void* b1, const void* w2,
                      const void* dy, void* dx, float* dw1, float* db1, float* dw2, float* db2,
                      int T, int d_model, int d_ff, int block, int act, hipStream_t stream);

/*
 * Per-block projection used by Algorithm 1 (query/key/value of each input block and the
 * output projection), bf16:  y = x W (+ residual).
 *   x in bf16 [T, d_in]; w in bf16 [d_in, d_out]; residual in bf16 [T, d_out] or NULL;
 *   y out bf16 [T, d_out].  T % block == 0, block % 256 == 0, d_in, d_out % 256 == 0.
 */
int blockwise_linear(const void* x, const void* w, const void* residual, void* y, int T,
                     int d_in, int d_out, int block, hipStream_t stream);

/* Backward of blockwise_linear without residual: dx = dy W^T (bf16 [T, d_in], may be
 * NULL), dw = x^T dy (f32 [d_in, d_out], overwritten). */
int blockwise_linear_bwd(const void* x, const void* w, const void* dy, void* dx, float* dw,
                         int T, int d_in, int d_out, int block, hipStream_t stream);

/*
 * One transformer layer as Algorithm 1 composes it, bf16, batch 1: the query, key and value
 * of each host's input block, ring attention over the n_hosts hosts, the output projection
 * with residual, and the blockwise feed-forward network on each host's block with residual:
 *     Q, K, V = X Wq, X Wk, X Wv;  A = RingAttention(Q, K, V);  Y = X + A Wo;
 *     Z = Y + act(Y W1) W2          (no biases, no normalisation, no positional encoding)
 *   x  in bf16 [S, d_model];  wq, wk, wv, wo in bf16 [d_model, d_model];
 *   w1 in bf16 [d_model, d_ff]; w2 in bf16 [d_ff, d_model];  z out bf16 [S, d_model]
 *   Heads: d_model = n_heads * D with D in {64, 128}; head h owns columns [h D, (h+1) D).
 *   The host block c = S / n_hosts (a multiple of 256) is also the projection / FFN block.
 */
int ring_layer_fwd(const void* x, const void* wq, const void* wk, const void* wv, const void* wo,
                   const void* w1, const void* w2, void* z, int S, int d_model, int n_heads,
                   int d_ff, int n_hosts, int causal, int act, hipStream_t stream);

/*
 * Backward of ring_layer_fwd for upstream dz (bf16 [S, d_model]).  Every activation is
 * recomputed from x (full gradient checkpointing, the paper's training setting).
 *   dx out bf16 [S, d_model]; dwq, dwk, dwv, dwo out f32 [d_model, d_model];
 *   dw1 out f32 [d_model, d_ff]; dw2 out f32 [d_ff, d_model] (overwritten).
 */
int ring_layer_bwd(const void* x, const void* wq, const void* wk, const void* wv, const void* wo,
                   const void* w1, const void* w2, const void* dz, void* dx, float* dwq, float* dwk,
                   float* dwv, float* dwo, float* dw1, float* dw2, int S, int d_model, int n_heads,
                   int d_ff, int n_hosts, int causal, int act, hipStream_t stream);

/*
 * LLaMA-style layer (the architecture the paper trains, Section 4 model configuration)
 * and its pieces.  The pieces are not defined by the paper; these entry points implement
 * the usual definitions, stated here:
 *   RMSNorm   y = x / sqrt(mean(x^2) + 1e-6) * g   (row-wise; gain g bf16 [d])
 *   RoPE      in each head, pair (2i, 2i+1) at global position p rotated by the angle
 *             p * 10000^(-2i/D)
 *   SwiGLU    (silu(x W1) * (x W3)) W2,  silu(u) = u / (1 + e^-u)
 *   layer     n1 = RMSNorm(x; g1);  h = x + Attn(RoPE(n1 Wq), RoPE(n1 Wk), n1 Wv) Wo;
 *             z = h + SwiGLU(RMSNorm(h; g2))
 * with Attn the ring attention of this library (causal by global position).
 */

/* RMSNorm forward.  x in bf16 [T, d]; g in bf16 [d]; y out bf16 [T, d]; rstd out f32 [T]
 * (1 / sqrt(mean(x^2) + eps)) or NULL.  d % 8 == 0, d <= 8192. */
int rms_norm_fwd(const void* x, const void* g, void* y, float* rstd, int T, int d, hipStream_t stream);

/* RMSNorm backward for upstream dy (f32 [T, d]): dx out bf16 [T, d] = dres + dx_norm (dres
 * bf16 [T, d] or NULL: a residual gradient added before the one rounding); dg out f32 [d]
 * (overwritten; summed over rows in a fixed order). */
int rms_norm_bwd(const void* x, const void* g, const float* dy, const void* dres, void* dx, float* dg,
                 int T, int d, hipStream_t stream);

/* Rotary position embedding in place on x bf16 [S, H, D] (rows at global positions
 * pos0 .. pos0 + S - 1); inverse = 1 applies the transpose (rotation by minus the angle),
 * which is the backward pass.  D % 4 == 0.  Angles are formed in double precision. */
int rope_apply(void* x, int S, int H, int D, int pos0, int inverse, hipStream_t stream);

/* SwiGLU feed-forward over row blocks of `block`:
 *   y = (silu(x W1) * (x W3)) W2 (+ residual)
 *   x in bf16 [T, d_model]; w1, w3 in bf16 [d_model, d_ff]; w2 in bf16 [d_ff, d_model];
 *   residual bf16 [T, d_model] or NULL; y out bf16 [T, d_model].  Shapes as blockwise_ffn. */
int swiglu_ffn(const void* x, const void* w1, const void* w3, const void* w2, const void* residual,
               void* y, int T, int d_model, int d_ff, int block, hipStream_t stream);

/* Backward of swiglu_ffn (no residual) for upstream dy bf16 [T, d_model], recomputing
 * x W1 and x W3 group by group: dx out bf16 [T, d_model]; dw1, dw3 out f32 [d_model, d_ff],
 * dw2 out f32 [d_ff, d_model] (overwritten). */
int swiglu_ffn_bwd(const void* x, const void* w1, const void* w3, const void* w2, const void* dy,
                   void* dx, float* dw1, float* dw3, float* dw2, int T, int d_model, int d_ff,
                   int block, hipStream_t stream);

/*
 * One LLaMA-style layer, forward (batch 1).
 *   x       in  bf16 [S, d_model]
 *   params  HOST array of 9 device pointers, in this order:
 *           g1 [d_model], wq, wk, wv, wo [d_model, d_model], g2 [d_model],
 *           w1, w3 [d_model, d_ff], w2 [d_ff, d_model]       (all bf16)
 *   z       out bf16 [S, d_model]
 * d_model = n_heads * D with D in {64, 128}, d_model <= 8192; S % n_hosts == 0; the host
 * block S / n_hosts (the projection and feed-forward block) and d_model, d_ff multiples of 256.
 */
int llama_layer_fwd(const void* x, const void* const* params, void* z, int S, int d_model,
                    int n_heads, int d_ff, int n_hosts, int causal, hipStream_t stream);

/*
 * Backward of llama_layer_fwd for upstream dz (bf16 [S, d_model]); the forward is
 * recomputed from x (full gradient checkpointing, the paper's training setting).
 *   dx     out bf16 [S, d_model]
 *   grads  HOST array of 9 device pointers (f32, overwritten) matching params:
 *          dg1, dwq, dwk, dwv, dwo, dg2, dw1, dw3, dw2
 */
int llama_layer_bwd(const void* x, const void* const* params, const void* dz, void* dx,
                    float* const* grads, int S, int d_model, int n_heads, int d_ff, int n_hosts,
                    int causal, hipStream_t stream);

/*
 * One training step of a stack of n_layers LLaMA-style layers: the forward pass keeps only
 * each layer's input, the backward pass runs the layers last to first, each recomputing
 * its own forward (the paper's full recomputation of attention and feed-forward).
 *   x       in  bf16 [S, d_model]
 *   params  HOST array of 9 * n_layers device pointers (layer l at params + 9 l, as above)
 *   dz      in  bf16 [S, d_model]: gradient of the loss with respect to the stack output
 *   z       out bf16 [S, d_model]: the stack output
 *   dx      out bf16 [S, d_model]
 *   grads   HOST array of 9 * n_layers device pointers (f32, overwritten)
 */
int llama_stack_train_step(const void* x, const void* const* params, const void* dz, void* z,
                           void* dx, float* const* grads, int n_layers, int S, int d_model,
                           int n_heads, int d_ff, int n_hosts, int causal, hipStream_t stream);

/*
 * A decode step over a paged key/value cache, for a batch of requests of different lengths.
 *
 * The cache is n_pages pages of page_size tokens: k_pages, v_pages [n_pages, page_size, Hkv, D].
 * Request r owns the pages its row of block_table int32 [R, max_pages] lists, in order; its token
 * at position p lies in slot block_table[r][p / page_size] * page_size + p % page_size.  The new
 * tokens of a step lie packed in T rows, request after request; cu_rows[r] is the first row of
 * request r, cu_rows[R] their number; T may be larger, rows from there on are padding.
 *   paged_plan         pages for the new tokens, cu_rows, slots and positions of the rows
 *   paged_append       rotary embedding of q and k; k and v into their slots
 *   paged_attn_decode  attention of the new tokens over each request's pages
 * kv_type:
 *   RA_KV_BF16  pages hold bf16; k_scales, v_scales NULL
 *   RA_KV_E4M3  pages hold 8-bit floats (OCP e4m3) and k_scales, v_scales uint8 [n_pages,
 *               page_size, Hkv] the exponents of their scales: element times 2^(scale - 127).
 *               paged_append takes the smallest power of two with which every finite element of
 *               the token's head is at most 448 in magnitude, 2^-126 at least (1 where all are
 *               zero), so that what a page stands for is exact in bf16 (above bf16's smallest
 *               numbers).  e4m3 has no infinity: infinite elements are stored as NaN.  Scales
 *               are 1 .. 254 of keys and 1 .. 247, the largest paged_append writes, of values.
 * page_size: a power of two, at most 1024; n_pages * page_size < 2^31; R <= 4096; heads <= 1024;
 * D in {64, 128}.  Device-side integers are not trusted: what lies out of range is left out, as
 * said at each call, and nothing out of bounds is read or written.
 */
typedef enum { RA_KV_BF16 = 0, RA_KV_E4M3 = 1 } ra_kv;

/* Flags that paged_plan leaves in counts[3]. */
enum {
  RA_PLAN_PAGES = 1,     /* the free list ran out */
  RA_PLAN_CAPACITY = 2,  /* a request is longer than max_pages pages */
  RA_PLAN_ROWS = 4,      /* more new tokens than T rows */
  RA_PLAN_BAD_INPUT = 8  /* a negative length, number of tokens or free_head (taken as 0) */
};

/*
 * Pages, slots and positions of a step's new tokens, on the device (no host synchronisation).
 *   lens        in  int32 [R]  tokens in the cache;  n_new in int32 [R]  new tokens of this step
 *   free_pages  in  int32 [n_free]  ids of free pages, taken in order from entry *free_head on;
 *               n_free >= 1 (an empty list: any one entry, with *free_head = 1)
 *   free_head   in  int32 [1], or NULL for 0; not inside counts
 *   block_table in/out int32 [R, max_pages]: request r holds ceil(lens[r] / page_size) pages; the
 *               entries of the pages it needs on top are written, in request order, no others
 *   cu_rows     out int32 [R + 1]    new_lens out int32 [R] = lens + n_new (not lens itself)
 *   slots, positions out int32 [T]  of each row; both -1 in padding rows
 *   counts      out int32 [4]: rows, pages taken, the free_head of the next step, flags
 * Where the free list runs out, an id in it or an entry held lies outside [0, n_pages) or a
 * request outgrows max_pages, the entry (if there is one) and the slots of its tokens are -1.
 * Tokens that T rows do not hold are not taken: cu_rows ends at T, new_lens counts those taken.
 * Lengths and positions end at 2^31 - 1.
 * Outputs do not overlap inputs or one another.  Calling again with the same inputs gives the
 * same outputs.
 */
int paged_plan(const int* lens, const int* n_new, const int* free_pages, const int* free_head, int* block_table,
               int* cu_rows, int* new_lens, int* slots, int* positions, int* counts, int R, int page_size,
               int max_pages, int n_pages, int n_free, int T, hipStream_t stream);

/*
 * The new tokens' keys and values into the cache, after the rotary embedding of rope_apply.
 *   q         in  bf16 [T, Hq, D], k, v in bf16 [T, Hkv, D], rows q_stride, k_stride, v_stride
 *             elements apart (multiples of 8: they may be parts of one projection's output);
 *             q and q_out both NULL: keys and values alone
 *   q_out     out bf16 [T, Hq, D], dense: q rotated (may be q itself where q is dense)
 *   k_pages, v_pages (and scales) in/out: the slots of the rows are written, nothing else
 *   slots, positions in int32 [T] (paged_plan).  A row of a negative position is left out; one
 *             whose slot lies outside the cache has q rotated and nothing stored.  Two rows with
 *             one slot leave elements of either in it.
 *   Outputs overlap no input, but q_out that is q.
 *   rotate    1: q and k are rotated by their positions (angles formed in double); 0: copied
 * T < 2^24.
 */
int paged_append(const void* q, const void* k, const void* v, void* q_out, void* k_pages, void* v_pages,
                 unsigned char* k_scales, unsigned char* v_scales, const int* slots, const int* positions, int T,
                 int Hq, int Hkv, int D, int q_stride, int k_stride, int v_stride, int n_pages, int page_size,
                 int kv_type, int rotate, hipStream_t stream);

/*
 * Attention of the new tokens over their requests' pages: o = softmax(q K^T / sqrt(D)) V, query
 * head i reading key head i / (Hq / Hkv).
 *   q          in  bf16 [T, Hq, D];  o out bf16 [T, Hq, D];  lse out f32 [T, Hq]
 *   lens       in  int32 [R]: tokens in the cache, this step's among them (new_lens of paged_plan)
 *   cu_rows    in  int32 [R + 1] ascending, or NULL: row r is the one new token of request r
 *   max_new    the most new tokens of a request, <= 32; later rows of a longer one are not computed
 *   max_pages * page_size < 2^30.  How the work is split up goes by this product, the keys that a row of
 *   the table can hold: where all requests are short, a table of no more columns than the longest
 *   one needs is faster (16 groups of requests and key heads, 120 keys: 8 us for 11).
 *   Row t of the n of request r sits at position lens[r] - n + t and sees keys up to its own.
 *   Sums are float32 and relative to a maximum that may lag by up to 2^8: values of a magnitude
 *   past 2^119 divided by the number of keys may come out infinite.
 *   Keys past max_pages pages, or in pages outside [0, n_pages), are masked.  A masked key counts
 *   for nothing, whatever its row holds; a row that sees no key has o = 0, lse = -inf.  Rows of
 *   no request are left as they are.
 *   workspace  workspace_bytes of device memory on a 16-byte boundary, or NULL: allocated by the
 *              library like every other call's, if the call needs one.  With a workspace of its own a call allocates
 *              nothing and can be captured into a HIP graph; calls that may overlap, and graphs
 *              that may run at once, need one each.  Its contents before the call do not matter.
 * paged_attn_workspace gives the bytes that calls of this shape (and any lengths) need.
 */
int paged_attn_workspace(int R, int Hq, int Hkv, int D, int max_new, size_t* bytes);
int paged_attn_decode(const void* q, const void* k_pages, const void* v_pages, const unsigned char* k_scales,
                      const unsigned char* v_scales, const int* block_table, const int* lens, const int* cu_rows,
                      void* o, float* lse, void* workspace, size_t workspace_bytes, int T, int R, int Hq, int Hkv,
                      int D, int n_pages, int page_size, int max_pages, int max_new, int kv_type,
                      hipStream_t stream);

/*
 * Products of a few rows with weights in 4 bits (blockwise_linear's product, for decode steps):
 *   y = x W (+ residual);  x in bf16 [T, d_in], residual in bf16 [T, d_out] or NULL, y out bf16
 * W in the MX format: elements e2m1 (sign bit, then 0, 0.5, 1, 1.5, 2, 3, 4, 6), one scale
 * 2^(byte - 127) for 32 inputs of an output (byte 1 .. 254; 255 makes the group NaN).  Products
 * are exact in bf16 operands and summed in float32.  With nb = ceil(d_out / 16), kb =
 * ceil(d_in / 128):
 *   w4      uint8 [nb, kb, 64, 16]: byte j of entry l of block (i, b) holds output 16 i + l % 16,
 *           inputs 128 b + 32 (j / 4) + 8 (l / 16) + 2 (j % 4) (low four bits) and the next (high)
 *   scales  uint8 [nb, kb, 16, 4]: output 16 i + r, inputs 128 b + 32 g ... + 31
 * Places past d_out and d_in hold zero codes.  mx4_pack fills both from w bf16 [d_in, d_out]: the
 * scale is the smallest power of two (2^-126 at least) with which the group is at most 6 in
 * magnitude, codes are rounded to nearest, ties to the even code; a group with an infinity or NaN
 * has scale 255.
 * d_in % 32 == 0, d_in <= 2^29 - 128, d_in * d_out < 2^31, T <= 512.  y may be residual; it overlaps no other input.
 */
int mx4_pack(const void* w, void* w4, unsigned char* scales, int d_in, int d_out, hipStream_t stream);
int mx4_linear(const void* x, const void* w4, const unsigned char* scales, const void* residual, void* y, int T,
               int d_in, int d_out, hipStream_t stream);

/* Description of the last error returned on the calling thread ("" if none).  Valid
 * until the next library call on that thread. */
const char* ring_attn_last_error(void);

/*
 * Return the cached workspace of the current device's library pool to the driver
 * (hipMemPoolTrimTo to zero bytes).  Memory still in use by calls whose stream has not
 * reached the end of the call stays allocated, except on the NULL stream, which is waited for
 * if blocks of it are kept.  Not part of the method.  Returns RA_OK,
 * or RA_EHIP if the pool cannot be created or trimmed.
 */
int ring_attn_release_workspace(void);

/*
 * Kernel timing for benchmarks and profiling (not part of the method).
 * ring_attn_timing_enable(1) makes every later launch of the library's hot kernels be
 * bracketed by timing events on the stream it runs on (an attention backward's two as one);
 * what is launched does not change. ring_attn_timing_read(kind, ...)
 * waits for the recorded launches of that kind, returns their summed duration in
 * milliseconds and their number, and forgets them.  Kinds:
 */
enum { RA_KERNEL_ATTN_FWD = 0, RA_KERNEL_ATTN_BWD = 1, RA_KERNEL_GEMM = 2, RA_KERNEL_DECODE = 3 };
void ring_attn_timing_enable(int on);
int ring_attn_timing_read(int kind, double* total_ms, int* launches);

/*
 * Matrix-core calibration for benchmarks (not part of the method): launches 512
 * workgroups of 256 threads (two waves per SIMD on 256 compute units); every wave issues
 * iters x 32 bf16 32x32x16 matrix products (4 independent accumulator chains) and writes
 * one float to sink[wave].  The caller times the launch on `stream`: the work is
 * 2048 * iters * 32 * 32768 flop.
 *   iters            in [1, 2^20] (else RA_EINVAL)
 *   random_operands  0: the same two operands in every product (the headline rate);
 *                    1: random signs and mantissas (magnitudes in [0.5, 8)) that change
 *                    from one product to the next, as real data does (else RA_EINVAL)
 *   sink             device float[2048], overwritten
 */
int ring_attn_mfma_probe(int iters, int random_operands, float* sink, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RINGATTN_H */
