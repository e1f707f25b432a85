/*
 * mebp.h — C ABI of the MeBP checkpointed LoRA training step on AMD Instinct MI355X
 * (gfx950).
 *
 * MeBP (memory-efficient backpropagation, Sec. 3 and Algorithm 1 of the paper) trains
 * LoRA adapters of a decoder-only transformer with gradient checkpointing at every block
 * boundary. The forward loop stores only the block-boundary activations ("checkpoints");
 * the backward loop walks the blocks in reverse, decompresses each block's int4 base
 * weights just before use, recomputes the block's forward from its checkpoint, and
 * backpropagates into the LoRA A/B gradients and the block-input gradient (the backward
 * graph B_i(x, dE/dy, w) -> (dE/dx, dE/dw) of Sec. 3). Blocks are every transformer
 * layer plus the final linear layer and the cross-entropy loss (Sec. 4.2), the last two
 * fused into one call here.
 *
 * Conventions shared by every entry point:
 *  - Tensor arguments are DEVICE pointers owned by the caller; structs are host memory
 *    read during the call only. Nothing is allocated by the library: all scratch lives in
 *    the caller's workspace `ws` of at least mebp_workspace_bytes() bytes.
 *  - Activations are fp32, token-major: row n = b*T + t of a [B*T][hidden] matrix.
 *    Attention columns are head-major (column h*head_dim + e).
 *  - Compressed base weights (Sec. 3, 4-bit symmetric INT4 of every non-LoRA parameter
 *    incl. the embedding): per projection `q4` uint8 [out][in/2] (two's-complement
 *    nibbles, element 2j of a row in the low nibble of byte j) and `scale` raw fp16 bits
 *    [out][ceil(in/group)]; dequantised value W[o][i] = q[o][i] * scale[o][i/group].
 *    The last group of a row may be shorter than `group`.
 *  - LoRA: y = x W^T + (alpha/rank) (x A^T) B^T with A fp32 [rank][in], B fp32 [out][rank].
 *  - Every call validates all arguments first. On error it enqueues nothing, records a
 *    message for mebp_last_error() and returns a negative mebp_status. On success it
 *    enqueues work on `stream` and returns MEBP_OK without synchronising; outputs are
 *    valid once the stream reaches that point. Calls on one stream are ordered; two calls
 *    sharing one workspace must not run concurrently.
 *  - Results are deterministic: the same inputs give bit-identical outputs (no atomics
 *    in any reduction).
 */
#ifndef MEBP_H
#define MEBP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* A hipStream_t passed as an opaque pointer; NULL selects the null stream. */
typedef void* mebp_stream_t;

typedef enum {
  MEBP_OK = 0,
  MEBP_EINVAL = -1,       /* null pointer, negative size, inconsistent config            */
  MEBP_EUNSUPPORTED = -2, /* valid but unsupported shape (head_dim, rank, alignment)     */
  MEBP_EWORKSPACE = -3,   /* ws_bytes smaller than mebp_workspace_bytes()                */
  MEBP_EHIP = -4          /* a HIP runtime call or kernel launch failed                  */
} mebp_status;

/* Projection indices used by every per-projection array. */
enum { MEBP_Q = 0, MEBP_K = 1, MEBP_V = 2, MEBP_O = 3, MEBP_GATE = 4, MEBP_UP = 5, MEBP_DOWN = 6,
       MEBP_NPROJ = 7 };

typedef struct {
  int32_t n_layers;      /* L >= 1                                                        */
  int32_t hidden;        /* d, multiple of 32                                             */
  int32_t n_heads;       /* Hq                                                            */
  int32_t n_kv_heads;    /* Hkv, divides Hq (grouped-query attention, consecutive heads)  */
  int32_t head_dim;      /* 64, 128 or 256                                                */
  int32_t ffn;           /* F, multiple of 16                                             */
  int32_t vocab;         /* V, multiple of 32; 0 when no LM head is used                  */
  int32_t act;           /* 0 = SwiGLU (SiLU gate), 1 = GeGLU (tanh-approximated GELU)    */
  float rms_eps;         /* RMSNorm epsilon                                               */
  float rope_theta_global; /* RoPE base of global layers                                  */
  float rope_theta_local;  /* RoPE base of sliding-window layers                          */
  int32_t window;        /* sliding window W of local layers: key j visible to query i    */
                         /* iff i-W < j <= i; 0 = no window                               */
  int32_t global_every;  /* 0: every layer global; k > 0: layer l global iff (l+1)%k == 0 */
  int32_t group;         /* int4 scale group along the input dim; must be 32              */
  int32_t lora_rank;     /* r: 8 or 16                                                    */
  float lora_alpha;      /* LoRA scale s = alpha / r                                      */
  uint32_t lora_mask;    /* bit p set: projection p carries a LoRA adapter                */
  uint32_t arch;         /* architecture details beyond the shapes (MEBP_ARCH_* bits); 0 =  */
                         /* the plain pre-norm block                                      */
} mebp_config;

/* mebp_config.arch bits (Sec. 4 trains Qwen2.5 and Gemma3 models; these are the parts of
 * their blocks beyond a plain pre-norm Llama-style block). The extra frozen weights are
 * fp32 vectors in mebp_layer_base.                                                      */
enum {
  MEBP_ARCH_QKV_BIAS = 1,     /* Qwen2.5: q, k, v projections add a bias                   */
  MEBP_ARCH_QK_NORM = 2,      /* Gemma3: RMSNorm over each head of q and of k, before RoPE */
  MEBP_ARCH_SANDWICH = 4,     /* Gemma3: RMSNorm on the attention output and on the MLP    */
                              /* output before each residual add                          */
  MEBP_ARCH_EMBED_SCALE = 8   /* Gemma3: embedding output times sqrt(hidden) (the tied LM  */
                              /* head uses the table unscaled)                            */
};

typedef struct {
  const uint8_t* q4;        /* [out][in/2]                                                */
  const uint16_t* scale;    /* [out][ceil(in/group)] fp16 bits                            */
} mebp_q4;

typedef struct {
  mebp_q4 w[MEBP_NPROJ];    /* q [Hq*dh][d], k,v [Hkv*dh][d], o [d][Hq*dh],               */
                            /* gate,up [F][d], down [d][F]                                */
  const float* norm_attn;   /* [d] fp32 RMSNorm weight before attention (frozen)          */
  const float* norm_mlp;    /* [d] fp32 RMSNorm weight before the MLP (frozen)            */
  const float* bias[3];     /* MEBP_ARCH_QKV_BIAS: q [Hq*dh], k, v [Hkv*dh]; else unused  */
  const float* q_norm;      /* MEBP_ARCH_QK_NORM: [dh] weights of the q and k head norms  */
  const float* k_norm;
  const float* post_attn_norm; /* MEBP_ARCH_SANDWICH: [d] weights of the norms on the    */
  const float* post_mlp_norm;  /* attention output and on the MLP output                  */
} mebp_layer_base;

typedef struct {
  const float* A[MEBP_NPROJ]; /* [r][in]; NULL where the projection is not adapted        */
  const float* B[MEBP_NPROJ]; /* [out][r]                                                 */
} mebp_layer_lora;

typedef struct {
  float* dA[MEBP_NPROJ];    /* [r][in], overwritten (not accumulated); NULL if not adapted */
  float* dB[MEBP_NPROJ];    /* [out][r]                                                   */
} mebp_layer_lora_grad;

/* Bytes of workspace every entry point below needs for this config and batch shape
 * (B sequences of T tokens). Pure host computation; returns 0 for an invalid config. */
size_t mebp_workspace_bytes(const mebp_config* cfg, int32_t B, int32_t T);

/* forward_i of Algorithm 1 for transformer layer `layer` (Sec. 3, "Runtime
 * implementation"): x_out = F(x_in) with the int4 weights decompressed inside the GEMMs.
 *   x_in  [B*T][d] fp32 checkpoint of the layer input (read only)
 *   x_out [B*T][d] fp32 checkpoint of the layer output (written; must not alias x_in)   */
int mebp_layer_forward_ckpt(const mebp_config* cfg, int32_t layer, const mebp_layer_base* base,
                            const mebp_layer_lora* lora, const float* x_in, float* x_out,
                            int32_t B, int32_t T, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* backward_i of Algorithm 1 (Sec. 3 backward graph B_i(x, dE/dy, w) -> (dE/dx, dE/dw)):
 * recomputes the layer forward from its checkpoint and backpropagates.
 *   x_ckpt [B*T][d] fp32 layer input checkpoint
 *   dy     [B*T][d] fp32 gradient of the loss w.r.t. the layer output
 *   dx     [B*T][d] fp32 gradient w.r.t. the layer input, or NULL to skip it; may alias dy
 *   grads  LoRA gradients of the adapted projections (overwritten)                       */
int mebp_layer_recompute_backward(const mebp_config* cfg, int32_t layer, const mebp_layer_base* base,
                                  const mebp_layer_lora* lora, const float* x_ckpt, const float* dy,
                                  float* dx, const mebp_layer_lora_grad* grads, int32_t B, int32_t T,
                                  void* ws, size_t ws_bytes, mebp_stream_t stream);

/* Final block (Sec. 4.2: the final linear layer and the cross-entropy loss layer):
 * RMSNorm, logits against the tied int4 embedding, next-token cross-entropy averaged over
 * the B*(T-1) positions that have a target (position T-1 of each sequence has none), and
 * the gradient w.r.t. the last checkpoint.
 *   emb        tied embedding [V][d/2] / [V][d/32]
 *   norm_final [d] fp32
 *   x_last     [B*T][d] fp32 output checkpoint of the last layer
 *   ids        [B][T] int32 token ids in [0, V)
 *   loss       one fp32 on the device (written)
 *   dx_last    [B*T][d] fp32 (written)                                                    */
int mebp_lm_head_ce_backward(const mebp_config* cfg, const mebp_q4* emb, const float* norm_final,
                             const float* x_last, const int32_t* ids, int32_t B, int32_t T,
                             float* loss, float* dx_last, void* ws, size_t ws_bytes,
                             mebp_stream_t stream);

/* Embedding lookup with decompression of the tied int4 table (Sec. 3: the embeddings are
 * INT4 too): x0[b*T+t][:] = E[ids[b][t]][:] in fp32.                                    */
int mebp_embed(const mebp_config* cfg, const mebp_q4* emb, const int32_t* ids, int32_t B, int32_t T,
               float* x0, mebp_stream_t stream);

/* Backpropagation(x) of Algorithm 1 for one batch of token ids: embedding, forward loop
 * storing every checkpoint, final block, reverse loop recomputing each layer.
 *   layers, lora, grads  host arrays of cfg->n_layers entries
 *   ckpt  [(L+1)][B*T][d] fp32 checkpoint storage (written; ckpt[l] is the input of layer l)
 *   loss  one fp32 on the device (written)
 *   dx0   [B*T][d] fp32 gradient w.r.t. the embedding output, or NULL to skip layer 0's
 *         input gradient (the embedding is frozen)                                       */
int mebp_train_step(const mebp_config* cfg, const mebp_q4* emb, const mebp_layer_base* layers,
                    const float* norm_final, const mebp_layer_lora* lora, const int32_t* ids,
                    int32_t B, int32_t T, float* ckpt, float* loss, const mebp_layer_lora_grad* grads,
                    float* dx0, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* ---------------- optimizer step on the LoRA parameters ------------------------------
 * Sec. 3 ("Runtime implementation"): the gradient of a batch may be obtained by gradient
 * accumulation over smaller inputs, and only the LoRA weights, their gradients and the
 * optimizer state are kept for the optimizer; Sec. 4.1: the optimizer is AdamW.        */

typedef struct {
  float* A[MEBP_NPROJ];     /* [r][in] fp32, updated in place; NULL if not adapted      */
  float* B[MEBP_NPROJ];     /* [out][r]                                                 */
} mebp_layer_lora_state;    /* writable LoRA-shaped tensors: parameters or moments      */

typedef struct {
  float lr, beta1, beta2, eps, weight_decay;
  float grad_scale;         /* the gradients are multiplied by this first               */
  int32_t step;             /* t >= 1, the index of this update (bias corrections)      */
} mebp_adamw_hparams;

/* acc = (first ? 0 : acc) + scale * grads for every adapted LoRA tensor of every layer
 * (with scale = 1/k over k micro-batches of equal size: the gradient of their mean loss).
 *   grads, acc  host arrays of cfg->n_layers entries; device tensors 16-byte aligned;
 *               acc may alias grads. Enqueued on stream; returns < 0 on invalid input.  */
int mebp_lora_grad_accumulate(const mebp_config* cfg, const mebp_layer_lora_grad* grads,
                              const mebp_layer_lora_grad* acc, float scale, int32_t first,
                              mebp_stream_t stream);

/* One AdamW update (decoupled weight decay) of every adapted LoRA tensor of every layer,
 * elementwise in fp32:
 *   g = grad_scale * grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2;
 *   p = p - lr (weight_decay p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)).
 *   params, m, v  host arrays of cfg->n_layers entries, device tensors updated in place
 *                 (callers start with m = v = 0); grads: host array, tensors read only.
 * All device tensors 16-byte aligned and distinct. Requires 0 <= beta1, beta2 < 1,
 * eps >= 0, step >= 1 and finite values; returns < 0 and enqueues nothing otherwise.     */
int mebp_lora_adamw_step(const mebp_config* cfg, const mebp_layer_lora_state* params,
                         const mebp_layer_lora_grad* grads, const mebp_layer_lora_state* m,
                         const mebp_layer_lora_state* v, const mebp_adamw_hparams* hp,
                         mebp_stream_t stream);

/* Backpropagation(x) of Algorithm 1 with the checkpoints kept in host memory (Sec. 3,
 * "Runtime implementation": the checkpoints are memory-mapped during the forward pass
 * instead of being kept in memory). Same kernels, order and results as mebp_train_step,
 * bit for bit; only where the checkpoints live differs. Checkpoint x_i is computed into
 * device ring slot i % ring_slots, copied to ckpt_host[i] by a copy stream as soon as it is
 * written, and copied back into its slot ring_slots - 1 layers before the reverse loop
 * recomputes layer i (the last ring_slots checkpoints never leave the ring). Device memory
 * for checkpoints drops from (L+1) to ring_slots activations of [B*T][d] fp32.
 *   ckpt_host  [(L+1)][B*T][d] fp32 pinned host memory (hipHostMalloc; pageable memory is
 *              refused), written; complete when the stream reaches the end of the step
 *   ring       [ring_slots][B*T][d] fp32 device memory, 16-byte aligned (scratch)
 *   ring_slots 4 .. 16
 * Other arguments as mebp_train_step. Calls on one device share its copy stream and are
 * serialised on the host.                                                              */
int mebp_train_step_offload(const mebp_config* cfg, const mebp_q4* emb, const mebp_layer_base* layers,
                            const float* norm_final, const mebp_layer_lora* lora, const int32_t* ids, int32_t B,
                            int32_t T, float* ckpt_host, float* ring, int32_t ring_slots, float* loss,
                            const mebp_layer_lora_grad* grads, float* dx0, void* ws, size_t ws_bytes,
                            mebp_stream_t stream);

/* ---------------- entry point for callers that cannot allocate ----------------------
 * For callers that can neither allocate device memory nor hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * mebp_layer_recompute_backward with its scratch in a buffer of MEBP_STATIC_SCRATCH_BYTES
 * that the library holds on every device it runs on (reserved with the library's code on
 * that device and kept until the process ends) instead of a caller workspace: same kernels,
 * same order, same results. The call allocates nothing; arguments as
 * mebp_layer_recompute_backward without ws / ws_bytes. The layer must fit:
 * mebp_workspace_bytes() of the same config with vocab = 0 must not exceed
 * MEBP_STATIC_SCRATCH_BYTES (a Qwen2.5-0.5B-shaped layer at 256 tokens does), else the
 * call returns MEBP_EWORKSPACE and enqueues nothing. Every call on a device shares that
 * device's buffer and leaves its contents behind (no result depends on them): calls that
 * overlap on one device, from two streams or two host threads, race and must be
 * serialised by the caller.                                                            */
#define MEBP_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int mebp_layer_recompute_backward_static(const mebp_config* cfg, int32_t layer, const mebp_layer_base* base,
                                         const mebp_layer_lora* lora, const float* x_ckpt, const float* dy,
                                         float* dx, const mebp_layer_lora_grad* grads, int32_t B, int32_t T,
                                         mebp_stream_t stream);

/* ---------------- operators on logits ------------------------------------------------
 * What is trained on, or read off, a matrix of logits z [rows][vocab] beside the fused
 * next-token loss above. Numbers per row are fp32, sums are fp32; a temperature tau divides
 * the logits first. Logits of -inf are columns masked off: probability 0, gradient 0.
 * All calls take rows = 0 (nothing is enqueued). What a call writes lies apart from what it
 * reads, but for a gradient in place of its logits.                                        */

/* Element type of a matrix of logits or of their gradient. */
enum { MEBP_F32 = 0, MEBP_F16 = 1, MEBP_BF16 = 2 };

typedef struct {
  void* data;      /* [rows][ld], aligned to its element's size                            */
  int64_t ld;      /* elements from one row to the next, >= vocab; those behind a row's     */
                   /* vocab are neither read nor written                                   */
  int32_t rows;    /* 0 .. 2^22                                                             */
  int32_t vocab;   /* 1 .. 2^30                                                             */
  int32_t dtype;   /* MEBP_F32, MEBP_F16 or MEBP_BF16                                      */
} mebp_logits;

/* Bytes of workspace that mebp_token_logprobs (with this top_k) and mebp_distill_topk (top_k
 * = 0) need for logits of this shape. Pure host computation; 0 for an invalid one.         */
size_t mebp_logits_workspace_bytes(int32_t rows, int32_t vocab, int32_t top_k);

/* Outputs of mebp_token_logprobs, each one NULL where it is not wanted. With q = softmax(z /
 * tau): */
typedef struct {
  float* logp;      /* [rows] ln q[target]; 0 where the target is < 0                       */
  float* lse;       /* [rows] ln sum exp(z / tau)                                           */
  float* entropy;   /* [rows] -sum q ln q                                                   */
  int32_t* top_ids; /* [rows][top_k] the columns of the largest logits, in falling order,    */
                    /* of equal ones the lower column first                                 */
  float* top_logp;  /* [rows][top_k] their ln q                                             */
} mebp_token_scores;

/* Log probabilities of given tokens, with the entropy of the distribution and its top
 * alternatives: the score of a text, or a teacher's record for mebp_distill_topk.
 *   targets  [rows] int32 token ids; < 0: none; >= vocab: logp is NaN. NULL without logp
 *   top_k    0 .. 64 (0: top_ids and top_logp are NULL)
 * Logits of -inf and NaN are no alternatives: where a row has fewer than top_k others, the
 * remaining ids are -1 and their ln q is -inf. A row of nothing but -inf has lse -inf, logp
 * -inf and entropy 0; a NaN or +inf logit makes lse, logp, entropy and top_logp NaN.       */
int mebp_token_logprobs(const mebp_logits* z, const int32_t* targets, float temperature, int32_t top_k,
                        const mebp_token_scores* out, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* Gradient of sum_n d_logp[n] logp[n] + d_entropy[n] entropy[n] w.r.t. the logits:
 *   dz[n][v] = (d_logp (1[v = target] - q[v]) - d_entropy q[v] (ln q[v] + entropy)) / tau.
 *   lse, entropy   [rows] as mebp_token_logprobs wrote them for the same logits (entropy is
 *                  read only with d_entropy)
 *   d_logp, d_entropy  [rows] fp32; either may be NULL (0). targets may be NULL without d_logp
 *   dz   of the logits' rows and vocab, any type and ld. May be the logits themselves (same
 *        data, type and ld); otherwise the two must lie apart, also where rows of one would fit
 *        between rows of the other
 * A target < 0 gives its row no d_logp term, one >= vocab makes the row NaN; at a target whose logit
 * is -inf the gradient is d_logp / tau. A row whose lse is -inf gets zeros, whatever its target
 * (nothing but -inf, or logits whose quotients by tau are below fp32's lowest); a NaN or +inf logit
 * makes its row NaN. Beyond 128 in magnitude an fp32 lse has too few bits for q: such a row's sum is
 * taken anew, in a pass of its own (rows masked by a finite value, small temperatures). No workspace. */
int mebp_token_logprobs_backward(const mebp_logits* z, const int32_t* targets, float temperature, const float* lse,
                                 const float* entropy, const float* d_logp, const float* d_entropy,
                                 const mebp_logits* dz, mebp_stream_t stream);

/* What a student's logits are distilled from. Per row, with p = softmax(logits / tau) over
 * its entries, q = softmax(z / tau) and q1 = softmax(z) over the whole vocabulary:
 *   loss = w (alpha tau^2 sum_k p_k (ln p_k - ln q[id_k]) - (1 - alpha) ln q1[target]).
 * The teacher's top log probabilities serve as its logits as well. What alpha leaves unread may be
 * NULL; at alpha 0 the temperature changes nothing.                                        */
typedef struct {
  const int32_t* ids;      /* [rows][k] the teacher's token ids, read if alpha > 0; < 0: no    */
                           /* entry; an id may occur twice (its probabilities add); >= vocab: */
                           /* the row is NaN                                                 */
  const float* logits;     /* [rows][k], read if alpha > 0; -inf: no entry; NaN or +inf: the */
                           /* row is NaN                                                     */
  const int32_t* targets;  /* [rows] hard labels, read if alpha < 1; < 0: no such term here;  */
                           /* >= vocab: the row is NaN                                      */
  const float* row_weight; /* [rows] w, e.g. 1 / rows for a mean; NULL: 1. A row of weight 0 */
                           /* has loss and gradient 0 whatever its logits are               */
  int32_t k;               /* 1 .. 64                                                       */
  float temperature;       /* tau, 1e-6 .. 1e6                                              */
  float alpha;             /* 0 .. 1                                                        */
} mebp_distill;

/* Distillation from a teacher's top logits: the loss of each row and, unless dz is NULL, the
 * gradient of their sum w.r.t. the student's logits,
 *   dz = w (alpha tau (q - p) + (1 - alpha) (q1 - 1[target])).
 *   row_loss [rows] fp32 (written)
 *   dz       as in mebp_token_logprobs_backward
 * A row without entries has no distillation term, one without a label either loss and gradient 0.
 * Where the student's logit of an entry or of the label is -inf the loss is +inf, and that column's
 * gradient is its term of p (of the label) alone.
 * Else a row of nothing but -inf has loss +inf and gradient 0, and a NaN or +inf logit makes a row
 * NaN.                                                                                    */
int mebp_distill_topk(const mebp_logits* z, const mebp_distill* d, float* row_loss, const mebp_logits* dz, void* ws,
                      size_t ws_bytes, mebp_stream_t stream);

/* ---------------- the LM head's logits ------------------------------------------------
 * z = rmsnorm(x) E^T of the final norm and the tied int4 embedding for `rows` hidden states
 * x [rows][d] fp32 (what the last layer's checkpoint holds, or any of its rows), and the
 * operators above on them. Operands and products as in mebp_lm_head_ce_backward: fp16 forward,
 * bf16 backward, fp32 sums. Rows go in blocks, so that the logits and the gradient of a block (fp32
 * and bf16) take at most MEBP_LM_CHUNK_MB (environment, default 512) MiB, or those of 64 rows.
 * Vocabularies below 2^20, tables up to 4 GiB. x, dx, norm_final 16-byte aligned; dx must not
 * overlap x. rows = 0 enqueues nothing.                                                   */

/* Bytes of workspace for the four calls below (top_k: that of mebp_lm_head_logprobs, else 0).
 * Pure host computation; 0 for an invalid config or shape.                               */
size_t mebp_head_workspace_bytes(const mebp_config* cfg, int32_t rows, int32_t top_k);

/* The logits themselves: z of `rows` rows and cfg->vocab columns, MEBP_F32 or MEBP_F16 (rounded to
 * it), ld a multiple of 8 below 2^20 (a block's rows times ld below 2^31), data 16-byte aligned
 * (written).                                                                             */
int mebp_lm_head_logits(const mebp_config* cfg, const mebp_q4* emb, const float* norm_final, const float* x,
                        int32_t rows, const mebp_logits* z, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* Their gradient back to the hidden states: dx [rows][d] fp32 from dz MEBP_BF16 of the same
 * shape rules.                                                                           */
int mebp_lm_head_logits_backward(const mebp_config* cfg, const mebp_q4* emb, const float* norm_final, const float* x,
                                 int32_t rows, const mebp_logits* dz, float* dx, void* ws, size_t ws_bytes,
                                 mebp_stream_t stream);

/* mebp_token_logprobs of the head's logits: scores a text, or records a teacher's alternatives. */
int mebp_lm_head_logprobs(const mebp_config* cfg, const mebp_q4* emb, const float* norm_final, const float* x,
                          int32_t rows, const int32_t* targets, float temperature, int32_t top_k,
                          const mebp_token_scores* out, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* mebp_distill_topk of the head's logits: the sum of the rows' losses and its gradient w.r.t. x.
 *   loss  one fp32 on the device (written);  row_loss [rows] fp32 (written), or NULL
 *   dx    [rows][d] fp32 (written)                                                        */
int mebp_lm_head_distill_backward(const mebp_config* cfg, const mebp_q4* emb, const float* norm_final, const float* x,
                                  int32_t rows, const mebp_distill* d, float* loss, float* row_loss, float* dx,
                                  void* ws, size_t ws_bytes, mebp_stream_t stream);

/* mebp_train_step with mebp_lm_head_distill_backward as its final block: row n = b*T + t of `d` is
 * position t of sequence b (its entries and its target are of the token that follows there, and its
 * weight makes the sum a mean); T may be 1. Other arguments as in mebp_train_step; the workspace is
 * that of mebp_distill_step_workspace_bytes: mebp_workspace_bytes where a block of the head's logits fits where
 * mebp_train_step has its own or its copy of the table (many tokens), and the head's added to it else. */
size_t mebp_distill_step_workspace_bytes(const mebp_config* cfg, int32_t B, int32_t T);
int mebp_train_step_distill(const mebp_config* cfg, const mebp_q4* emb, const mebp_layer_base* layers,
                            const float* norm_final, const mebp_layer_lora* lora, const int32_t* ids, int32_t B,
                            int32_t T, const mebp_distill* d, float* ckpt, float* loss, float* row_loss,
                            const mebp_layer_lora_grad* grads, float* dx0, void* ws, size_t ws_bytes,
                            mebp_stream_t stream);

/* ---------------- a forward pass over a cache ------------------------------------------
 * What a trained model answers with: rotary positions by themselves, a paged cache of keys and values
 * in 8 bits, attention of new tokens over it, and a layer's forward pass with them in the place of
 * mebp_layer_forward_ckpt's attention. Numbers of sequences, lengths and pages are read on the
 * device, so that a captured call serves as they change. tokens = 0 and seqs = 0 enqueue nothing; the layer's
 * call refuses rows = 0 and seqs = 0. */

/* Heads of some tokens (queries, keys, values or their gradients). */
typedef struct {
  void* data;        /* element e of head h of token n at n * ld + h * head_ld + e, aligned to its size */
  int64_t ld;        /* elements from one token to the next, 0 .. 2^32                      */
  int64_t head_ld;   /* from one head to the next. Of outputs no two elements share a place */
  int32_t tokens;    /* 0 .. 2^24                                                           */
  int32_t heads;     /* 1 .. 1024                                                           */
  int32_t dim;       /* 1 .. 1024                                                           */
  int32_t dtype;     /* MEBP_F32, MEBP_F16 or MEBP_BF16                                     */
} mebp_heads;

/* Rotary positions: (cos, sin) of every position and pair, which a program keeps. */
typedef struct {
  float* table;      /* [n_pos][rot / 2][2] fp32, 8-byte aligned                            */
  int32_t rot;       /* the first `rot` elements of a head turn, the others stay: even, >= 2 */
  int32_t n_pos;     /* positions 0 .. n_pos - 1, up to 2^28                                */
  int32_t interleaved; /* pairs are 0: elements (j, j + rot / 2), 1: (2 j, 2 j + 1)         */
} mebp_rope;

/* Its frequencies, f_j = theta^(-2 j / rot) where nothing is scaled. */
typedef struct {
  float theta;
  float factor;      /* s >= 1 by which a context is longer: f_j / s, or by parts            */
  int32_t original;  /* 0: every frequency. Else by parts: the length of the original context. A pair that */
                     /* turns r = original f_j / 2 pi times in it gets f_j (g + (1 - g) / s),  */
  float low, high;   /* g = clamp((r - low) / (high - low), 0, 1); 0 <= low < high            */
  float gain;        /* cos and sin are multiplied by this (1: a rotation)                   */
} mebp_rope_scaling;

/* Fills rope->table (written): gain (cos, sin)(p f_j), angles in 64 bits, rounded to fp32. */
int mebp_rope_positions(const mebp_rope* rope, const mebp_rope_scaling* scaling, mebp_stream_t stream);

/* y = x with its pairs turned: y_a = x_a cos - x_b sin, y_b = x_b cos + x_a sin; in fp32, rounded once.
 *   positions [tokens] int32; one outside the table makes its token's pairs NaN
 *   y         of x's tokens, heads, dim and dtype; x itself (same data and strides), or apart from it
 *   backward  1: the transposed map, the gradient w.r.t. x of one w.r.t. y
 * Up to 2^31 elements.                                                                      */
int mebp_rope_apply(const mebp_rope* rope, const mebp_heads* x, const int32_t* positions, const mebp_heads* y,
                    int32_t backward, mebp_stream_t stream);

/* The cache: a pool of pages. Of every 16 tokens and head there is a block of keys [16][dim] and one of
 * values [dim][16] in int8, with an fp32 scale each: a number is its code times its block's scale. */
typedef struct {
  int8_t* pages;     /* [n_pages][heads][page_tokens / 16][2][16 * dim], 16-byte aligned     */
  float* scales;     /* [n_pages][heads][page_tokens / 16][2], 8-byte aligned                */
  int32_t n_pages;   /* n_pages * heads * page_tokens / 16 below 2^31                       */
  int32_t page_tokens; /* a power of two, 16 .. 65536                                       */
  int32_t heads;     /* kv heads, up to 1024                                                */
  int32_t dim;       /* 64, 128 or 256                                                      */
} mebp_kv_cache;

/* Bytes of one page's codes (its scales: page_tokens / 16 * heads * 8). 0 for an invalid shape. */
size_t mebp_kv_page_bytes(int32_t page_tokens, int32_t heads, int32_t dim);

/* New tokens of some sequences: rows start[s] .. start[s + 1] - 1 of a call's operands are the tokens
 * past[s], past[s] + 1, .. of sequence s. Rows behind start[seqs] belong to none, and what a call
 * writes is left as it was there. */
typedef struct {
  const int32_t* start;  /* [seqs + 1], not falling (device memory, as the two below)       */
  const int32_t* past;   /* [seqs] tokens that were in the cache before                     */
  const int32_t* table;  /* [seqs][table_ld]: the page of tokens p * page_tokens .. of a sequence at  */
                         /* column p                                                        */
  int64_t table_ld;      /* >= max_pages                                                    */
  int32_t max_pages;     /* columns of the table                                            */
  int32_t seqs;          /* 0 .. 65534                                                      */
  int32_t max_new;       /* no sequence has more new tokens (rows beyond are left as they were) */
  int32_t max_len;       /* none is longer with them (rows from there on are NaN in an attention); up to */
                         /* 2^30. The call's launches are laid out for these two, for all sequences alike: */
                         /* single tokens behind long texts are quicker in a call without long prompts */
} mebp_kv_batch;

/* Appends keys and values, the keys turned by their positions (rope NULL: as they are), and turns queries
 * beside them. A block's scale is max(|scale before|, max |x| / 127 in fp32), "before" 0 where the block's
 * first token is new; codes are round(x / scale) to nearest even, and where the scale changes the block's
 * earlier ones round(code before / after). Scales and codes are those of 64-bit arithmetic.
 *   k, v       of the cache's heads and dim, any dtype
 *   q, q_out   [tokens][any heads][dim] of that dtype, together and with a rope, or both NULL; q_out may be q
 * A NaN or an infinity makes its block's scale NaN. Where the table has no page of the pool (an id outside
 * 0 .. n_pages - 1, a column beyond max_pages) nothing is stored. Blocks that are written belong to one
 * sequence of the call; whole ones before them may be shared.                               */
int mebp_kv_append(const mebp_kv_cache* cache, const mebp_kv_batch* batch, const mebp_rope* rope, const mebp_heads* k,
                   const mebp_heads* v, const mebp_heads* q, const mebp_heads* q_out, mebp_stream_t stream);

/* Reads tokens back as numbers, code times scale: here `past` is the first token that is read of a
 * sequence, and its rows are as many as are read. k or v may be NULL. No page: NaN.          */
int mebp_kv_read(const mebp_kv_cache* cache, const mebp_kv_batch* batch, const mebp_heads* k, const mebp_heads* v,
                 mebp_stream_t stream);

/* Attention of the rows over what their sequences have in the cache, their own tokens included (append
 * them first): out = softmax(scale q k^T) v over the keys j <= i of the token at position i, with a window
 * W > 0 over i - W < j <= i; query heads of one kv head are consecutive.
 *   q, out  fp16 or bf16 [tokens][a multiple of the cache's heads][dim]; out apart from q
 *   lse     [tokens][q heads] fp32 log-sum-exp of the scaled scores, or NULL
 * Scores by products in the queries' type (exact there, as codes are), outputs by products in bf16 (codes are
 * exact there too; weights times their block's scale go in as two of them, off by 2^-17 at most); sums and
 * softmax in fp32. A row depends on the blocks that it sees alone: one whose scale is NaN or infinite, or
 * whose page the table does not have, makes it NaN. Sums of values beyond 10^33 may overflow, and beside
 * values' scales above 10^-6 those below 10^-27 lose bits.                                  */
int mebp_kv_attention(const mebp_kv_cache* cache, const mebp_kv_batch* batch, const mebp_heads* q, const mebp_heads* out,
                      float* lse, float scale, int32_t window, void* ws, size_t ws_bytes, mebp_stream_t stream);

/* Bytes of workspace of such a call. Pure host computation; 0 for an invalid shape.         */
size_t mebp_kv_attention_workspace_bytes(int32_t seqs, int32_t max_new, int32_t max_len, int32_t q_heads, int32_t heads,
                                         int32_t dim, int32_t window);

/* mebp_layer_forward_ckpt of `rows` new tokens of the batch's sequences: their keys and values join the
 * layer's cache, and attention is over it (scale 1 / sqrt(head_dim), the layer's window).
 *   x_in, x_out  [rows][d] fp32, apart from each other. Rows of no sequence, and those behind a
 *                sequence's max_new, go through the layer without attention
 *   cache        this layer's, of the config's n_kv_heads and head_dim
 *   rope         of the layer's theta; positions beyond its table give NaN
 *   ws           mebp_cached_workspace_bytes                                                */
int mebp_layer_forward_cached(const mebp_config* cfg, int32_t layer, const mebp_layer_base* base, const mebp_layer_lora* lora,
                              const float* x_in, float* x_out, int32_t rows, const mebp_kv_cache* cache,
                              const mebp_kv_batch* batch, const mebp_rope* rope, void* ws, size_t ws_bytes,
                              mebp_stream_t stream);
size_t mebp_cached_workspace_bytes(const mebp_config* cfg, int32_t rows, int32_t seqs, int32_t max_new, int32_t max_len);

/* Message for the last non-zero status returned on the calling thread ("" if none). */
const char* mebp_last_error(void);

/* ---------------- test and diagnostic entry points ---------------------------------- */

/* Workspace guards, a debug mode (also on when MEBP_WS_GUARD=1 is in the environment when
 * the library loads). On, every workspace slot is followed by a guard region of at least
 * 256 bytes holding a known pattern, so mebp_workspace_bytes() returns more (size the
 * workspace with the mode already set; a workspace sized without it is refused with
 * MEBP_EWORKSPACE) and mebp_workspace_offset() moves. Every entry point that takes a
 * workspace (the static-scratch one included) then fills the guards before its first
 * kernel, checks them after its last one on the caller's stream and waits for that stream
 * (so a guarded call cannot be captured into a graph); an overwritten guard fails the call
 * with MEBP_EWORKSPACE, the message naming the slot. Results are those of the unguarded
 * call. mebp_set_workspace_guards returns the previous mode (0 off, 1 on); switch it only
 * while no call is in flight. mebp_workspace_guard_check checks the guards of a workspace
 * that a guarded call used, without filling them first: MEBP_OK, MEBP_EWORKSPACE (names
 * the slot), or MEBP_EINVAL when the mode is off or an argument is bad.                  */
int mebp_set_workspace_guards(int32_t on);
int mebp_workspace_guard_check(const mebp_config* cfg, int32_t B, int32_t T, void* ws, size_t ws_bytes,
                               mebp_stream_t stream);

/* Decompression alone (Algorithm 1, decompress): out_f32[r][c] = q*s exactly and/or
 * out_bf16[r][c] = bf16 bits of that value rounded to nearest even (either may be NULL).
 * cols must be a multiple of 8; group as in mebp_config.                                 */
int mebp_dequant_q4(const mebp_q4* w, int32_t rows, int32_t cols, int32_t group, float* out_f32,
                    uint16_t* out_bf16, mebp_stream_t stream);

/* One dequant-GEMM kernel of the library on caller operands (test aid for the bit-exact check of
 * the decompression fused into the products, Algorithm 1's LazyLoadAndDecompressWeights):
 * one split, no LoRA term, no residual, fp32 outputs.
 *   forward kinds (the layer projections and the LM-head logits):
 *     out[m][n] = sum_k X[m][k] * fp16_rne(W[n][k]),   X fp16 [M][n_in], out [M][n_out]
 *   transposed kinds (the input gradients and the LM head's dH):
 *     out[m][c] = sum_n G[m][n] * bf16_rne(W[n][c]),   G bf16 [M][n_out], out [M][n_in]
 * with W [n_out][n_in] the decompressed weight (int4 codes times fp16 scale per 32 inputs).
 * A one-hot X (or G) makes each output one decompressed weight in the kernel's operand
 * type, exactly. n_in and n_out multiples of 16, 1 <= M <= 65536, n_in, n_out <= 65536,
 * x and out 16-byte aligned; MEBP_EINVAL / MEBP_EUNSUPPORTED otherwise.                  */
enum {
  MEBP_TEST_GEMM_NT = 0,        /* forward, 128 x 128 tiles (few tokens)                  */
  MEBP_TEST_GEMM_NT_BIG128 = 1, /* forward, 256 x 128 tiles, weights staged in registers  */
  MEBP_TEST_GEMM_NT_BIG256 = 2, /* forward, 256 x 256 tiles, weights staged in registers  */
  MEBP_TEST_GEMM_NT_LDS = 3,    /* forward, 256 x 256 tiles, activations loaded into LDS  */
  MEBP_TEST_GEMM_TN = 4,        /* transposed, 128 x 128 tiles                            */
  MEBP_TEST_GEMM_TN_BIG = 5,    /* transposed, 256 x 128 tiles                            */
  MEBP_TEST_GEMM_NT_LDS_W16 = 6, /* MEBP_TEST_GEMM_NT_LDS on plain fp16 weights: w->q4      */
                                 /* points at W fp16 [n_out][n_in], w->scale is unused (the */
                                 /* same kernel without the decompression, to measure it)   */
  MEBP_TEST_GEMM_TN_BIG_W16 = 7, /* MEBP_TEST_GEMM_TN_BIG on plain bf16 weights, likewise   */
  /* the kernels that the configured shapes run on: add the tile configuration (0 .. 5       */
  /* forward, 0 .. 6 transposed) or MEBP_TEST_GEMM_PLANNED for the one the library picks     */
  MEBP_TEST_GEMM_NT_MID = 16,    /* forward; n_in a multiple of 64, scales 4-byte aligned    */
  MEBP_TEST_GEMM_TN_FRAG = 32,   /* transposed, on a bf16 copy of the weights in operand     */
                                 /* order that the call writes into the library's buffer     */
                                 /* (MEBP_STATIC_SCRATCH_BYTES; shared as described there)   */
  MEBP_TEST_GEMM_TN_FRAG_AGAIN = 48, /* the same without writing the copy: on the one that   */
                                 /* the previous call of that kind left                      */
  MEBP_TEST_GEMM_PLANNED = 15
};
int mebp_test_gemm(int32_t kind, const mebp_q4* w, int32_t n_out, int32_t n_in, const void* x, int32_t M,
                   float* out, mebp_stream_t stream);

/* Byte offset inside the workspace of an intermediate kept by the last
 * mebp_layer_recompute_backward / mebp_layer_forward_ckpt on that workspace (for tests).
 * Returns (size_t)-1 for an unknown slot. Slots are listed by mebp_workspace_slot_name. */
size_t mebp_workspace_offset(const mebp_config* cfg, int32_t B, int32_t T, int32_t slot);
const char* mebp_workspace_slot_name(int32_t slot);

/* Diagnostic per-kernel timing. mebp_kernel_timing(1) creates a pool of HIP events
 * (no device memory is allocated) and from then on brackets every kernel launch of this
 * library with an event pair tagged by kernel name and algorithmic flops / bytes;
 * mebp_kernel_timing(0) stops and frees the pool. Records beyond the pool's capacity
 * (`capacity` launches) are not timed. mebp_kernel_timing_report synchronises on the
 * recorded events and writes a JSON array
 *   [{"kernel": name, "launches": n, "ms": total, "flops": total, "bytes": total}, ...]
 * into buf (truncated to len); it returns the length the full report needs including the
 * terminating NUL, or a negative mebp_status. Host-thread-unsafe; for benchmarks only.  */
int mebp_kernel_timing(int32_t enable, int32_t capacity);
int mebp_kernel_timing_report(char* buf, size_t len);

/* Measurement aid. From this call on, every launch of the kernel named `kernel` (a name
 * as it appears in the timing report) is issued `times` times back to back on its stream;
 * kernel = NULL or times <= 1 switches it off. Results are unchanged, since every kernel
 * that may be repeated computes its outputs from inputs it does not overwrite; the kernels
 * that update a buffer in place are refused with MEBP_EINVAL ("gemm_tn_act_bwd",
 * "splitk_finalize_actbwd", "rope_fwd", "qkv_post", "headnorm_bwd", "ce_chunk_stats",
 * "ce_probs", "ce_dh_accum", "ce_final", "token_scores_grad_inplace", "distill_grad_inplace",
 * "distill_row_inplace", "rope_apply_inplace", "kv_append_inplace", "lora_adamw",
 * "lora_grad_accumulate"). With timing enabled, each burst of repeated launches is bracketed by one
 * event pair and reported as `times` launches, so the report's average is the kernel's
 * back-to-back in-stream duration. Host-thread-unsafe; for benchmarks only. */
int mebp_kernel_repeat(const char* kernel, int32_t times);

#ifdef __cplusplus
}
#endif
#endif /* MEBP_H */
