/*
 * nmt.h — C ABI of the MI355X (gfx950) reduced-precision NMT training-step library.
 *
 * The library runs the data-parallel hot path of "Scaling Neural Machine Translation" on one
 * GPU: Transformer encoder-decoder forward and backward in fp16 with fp32 accumulation,
 * label-smoothed cross-entropy, loss scaling with overflow detection, fp32 master weights and
 * Adam, and gradient accumulation over several sub-batches.
 *
 * Conventions
 *  - Every function returns int: NMT_OK (0) or a negative NMT_E* code; nmt_last_error() gives
 *    the message of the last failure on the calling thread.  No C++ exception crosses the ABI.
 *  - Pointers named d_* (and all buffers handed to nmt_bind) are DEVICE pointers owned by the
 *    caller; they must stay valid until the work enqueued on them has finished.  The library
 *    never allocates or frees device memory.  A forward or backward pass large enough to use a second
 *    stream creates it, and seven events, on the context's first such pass; every pass ends with the
 *    caller's stream waiting for it.  Host pointers are marked "host".
 *  - `stream` is a hipStream_t passed as void*; all kernels are enqueued on it and no function
 *    synchronises unless it says so.
 *  - fp16 buffers are IEEE binary16 (passed as void*).  Matrices are row-major.
 *  - Linear weights are stored [out, in]; y = x W^T + b.
 */
#ifndef NMT_H_
#define NMT_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NMT_OK 0
#define NMT_EINVAL (-1) /* bad argument or unsupported shape */
#define NMT_ESTATE (-2) /* call out of order (e.g. backward before forward) */
#define NMT_ENOMEM (-3) /* caller's workspace too small */
#define NMT_EHIP (-4)   /* HIP runtime error */

typedef struct nmt_ctx nmt_ctx;

/* Model and regularisation hyper-parameters (section "Models and Hyperparameters"). */
typedef struct {
  int32_t enc_layers, dec_layers; /* blocks in the encoder / decoder                     */
  int32_t d_model, n_heads, d_ff; /* d_model % n_heads == 0, head size in {16,32,64,128}  */
  int32_t vocab;                  /* shared vocabulary, multiple of 8, <= 65536           */
  int32_t pad_id;                 /* id of the padding symbol                              */
  float dropout;                  /* on each sub-layer output before the residual add, and
                                     on the embedding + position sum                       */
  float attn_dropout;             /* on the attention probabilities: not built, must be 0
                                     (nmt_create returns NMT_EINVAL otherwise)             */
  float act_dropout;              /* after the ReLU of the feed-forward layer              */
  float label_smoothing;          /* weight of the uniform prior over the vocabulary       */
  float ln_eps;                   /* variance floor of layer normalisation                 */
  uint64_t seed;                  /* Philox key of the dropout streams                     */
  int32_t max_sentences, max_len; /* limits for B (<= 2^20) and for S, T (<= 1024)        */
} nmt_config;

const char* nmt_last_error(void);

/* Host only.  Validates the configuration and builds the parameter layout. */
int nmt_create(const nmt_config* cfg, nmt_ctx** out);
void nmt_destroy(nmt_ctx* ctx);

/* Flat parameter layout: P scalars; tensor idx occupies [offset, offset + rows*cols).
 * Biases and LayerNorm vectors have rows == 1.  idx past the end returns NMT_EINVAL.
 * *name points into storage owned by ctx.  Every tensor offset is a multiple of 8. */
int64_t nmt_param_count(const nmt_ctx* ctx);
int32_t nmt_param_tensors(const nmt_ctx* ctx);
int nmt_param_info(const nmt_ctx* ctx, int32_t idx, const char** name, int64_t* offset,
                   int32_t* rows, int32_t* cols);

/* Bytes of workspace nmt_forward_loss / nmt_backward need for a batch of B sentences padded to
 * S source and T target positions (negative on invalid shapes). */
int64_t nmt_workspace_bytes(const nmt_ctx* ctx, int32_t B, int32_t S, int32_t T);

/* Attach the caller's device buffers.  w16, g16: fp16[P] weights and per-sub-batch gradients;
 * master32, acc32, adam_m, adam_v: fp32[P]; workspace: ws_bytes bytes, 256-byte aligned.
 * Any of master32/acc32/adam_m/adam_v may be NULL if the calls using them are not made. */
int nmt_bind(nmt_ctx* ctx, void* d_w16, void* d_g16, float* d_master32, float* d_acc32,
             float* d_adam_m, float* d_adam_v, void* d_workspace, int64_t ws_bytes);

/* Forward pass in fp16 and the label-smoothed loss in fp32 (sections "Models and
 * Hyperparameters", "Half-Precision Training").  d_src [B,S], d_tgt_in [B,T], d_tgt_out [B,T]:
 * int32 ids right-padded with pad_id; every sentence has at least one token.
 * The gradient of loss_scale * (sum of token losses) with respect to the logits is left in
 * the workspace for nmt_backward: the loss is scaled at the end of the forward pass, before any
 * fp16 gradient exists ("Half-Precision Training").
 * step (< 2^24) and micro_idx (< 256) select the dropout streams; d_sent_uid [B] (uint32, may
 * be NULL = row index) names each sentence so its dropout mask does not depend on batching.
 * training == 0 disables dropout and computes the loss alone: the logits stay, and an nmt_backward that follows all the
 * same first forms that gradient from them and from the log-sum-exps and targets the forward pass kept in the workspace
 * (the same bits; one more read of the logits than with training != 0).
 * An nmt_backward that follows reads d_src and d_tgt_in again, never d_tgt_out.
 * Outputs: *d_loss_sum = sum over non-pad target tokens of the UNSCALED loss in nats,
 * *d_ntok = number of non-pad target tokens. */
int nmt_forward_loss(nmt_ctx* ctx, const int32_t* d_src, const int32_t* d_tgt_in,
                     const int32_t* d_tgt_out, int32_t B, int32_t S, int32_t T, float loss_scale,
                     uint32_t step, uint32_t micro_idx, const uint32_t* d_sent_uid, int32_t training,
                     float* d_loss_sum, int32_t* d_ntok, void* stream);

/* The same for a group of n_seg (1 .. NMT_MAX_SEGMENTS) sub-batches of different padded shapes in
 * one pass ("Training with Larger Batches": the gradients of the sub-batches of one update are
 * summed; here the sum over the sub-batches of a group is already formed, in fp32, inside the
 * weight-gradient products of the one backward pass that follows, before the gradient is rounded
 * to fp16).  segs (host, read before the call returns) gives every sub-batch's B, S, T and micro
 * index; the id buffers hold the sub-batches one after another (d_src: sum of B*S ids, d_tgt_in /
 * d_tgt_out: sum of B*T ids) and d_sent_uid one entry per sentence in the same order (NULL: a
 * sentence's index within its sub-batch).  Dropout masks, loss and gradients are those of the
 * sub-batches processed one by one and accumulated.  *d_loss_sum and *d_ntok are totals over the
 * group.  A group may hold at most 2^20 source and 2^20 target positions.
 * The overflow decision of a pass over several sub-batches is that of ITS fp16 gradient, fp16(s * sum over the
 * sub-batches), s = nmt_grad_scale(): one sub-batch whose own gradient would leave the fp16 range can be hidden
 * by the others, and a sum of gradients that each fit can leave it.  Decisions equal to the method's order
 * (every sub-batch's gradient rounded to fp16 on its own, "Half-Precision Training" / "Training with Larger
 * Batches") are guaranteed for one sub-batch per pass only; a pass of several follows its own predicate
 * exactly, and the dynamic loss scale settles where that predicate puts it. */
#define NMT_MAX_SEGMENTS 64
typedef struct {
  int32_t B, S, T;    /* sentences, padded source and target length */
  uint32_t micro_idx; /* index of the sub-batch within its update (< 256): selects its dropout streams */
} nmt_segment;
int64_t nmt_workspace_bytes_group(const nmt_ctx* ctx, int32_t n_seg, const nmt_segment* segs /*host*/);
int nmt_forward_loss_group(nmt_ctx* ctx, int32_t n_seg, const nmt_segment* segs /*host*/, const int32_t* d_src,
                           const int32_t* d_tgt_in, const int32_t* d_tgt_out, float loss_scale, uint32_t step,
                           const uint32_t* d_sent_uid, int32_t training, float* d_loss_sum, int32_t* d_ntok,
                           void* stream);

/* The same for sentences PACKED back to back, without padding: d_sentences (device, n_sent entries,
 * read by the kernels of this call) gives every sentence's source and target length, its uid and
 * the micro index of the sub-batch it belongs to; d_src holds n_src_tokens ids (the source sentences
 * one after another), d_tgt_in / d_tgt_out n_tgt_tokens ids.  n_src_tokens, n_tgt_tokens (host) must
 * be the sums of the lengths and max_src_len, max_tgt_len (host) at least the longest ones: the
 * library sizes its launches from them and clamps what it reads from d_sentences to them, so
 * inconsistent values give undefined results but no access outside the caller's buffers.  Padding
 * positions carry no loss and no gradient, so loss, token count and gradients equal those of the
 * padded sub-batches; only the rows that do nothing are gone. */
typedef struct {
  int32_t src_len, tgt_len; /* >= 1 */
  uint32_t uid;             /* names the sentence's dropout streams */
  uint32_t micro_idx;       /* < 256 */
} nmt_sentence;
int64_t nmt_workspace_bytes_packed(const nmt_ctx* ctx, int32_t n_sent, int64_t n_src_tokens, int64_t n_tgt_tokens);
int nmt_forward_loss_packed(nmt_ctx* ctx, int32_t n_sent, const nmt_sentence* d_sentences, int64_t n_src_tokens,
                            int64_t n_tgt_tokens, int32_t max_src_len, int32_t max_tgt_len, const int32_t* d_src,
                            const int32_t* d_tgt_in, const int32_t* d_tgt_out, float loss_scale, uint32_t step,
                            int32_t training, float* d_loss_sum, int32_t* d_ntok, void* stream);

/* Backward pass in fp16 of the last nmt_forward_loss / nmt_forward_loss_group /
 * nmt_forward_loss_packed; writes every element of g16 with nmt_grad_scale(ctx) times the gradient
 * of loss_scale * loss_sum.  Nothing in it knows about the scale: it is an ordinary reverse pass over
 * fp16 tensors ("Half-Precision Training"). */
int nmt_backward(nmt_ctx* ctx, void* stream);

/* Gradient accumulation over sub-batches ("Training with Larger Batches"):
 * first != 0: acc32 = float(g16) / s; else acc32 += float(g16) / s, where s = nmt_grad_scale(ctx). */
int nmt_accumulate(nmt_ctx* ctx, int32_t first, void* stream);

/* Running totals over the sub-batches of one update, kept on the device so that the caller's loop needs no
 * host arithmetic: adds the loss sum and token count the last forward call wrote (its d_loss_sum / d_ntok)
 * to *d_loss_total / *d_ntok_total (first != 0: overwrites them).  Call after the forward call, on its stream. */
int nmt_accumulate_loss(nmt_ctx* ctx, int32_t first, float* d_loss_total, int32_t* d_ntok_total, void* stream);

/* The power-of-two factor s <= 1 by which the last forward call's pass scales what it writes to g16:
 * g16 = fp16(s * gradient of loss_scale * loss_sum).  s = 1 for passes of fewer than 8192 target
 * positions (any single sub-batch of the paper's size) and halves with every doubling beyond that, so
 * that the sum over a group of sub-batches reaches the fp16 range at the same loss scale as a single
 * sub-batch's gradient would.  nmt_accumulate divides it out again (exactly). */
float nmt_grad_scale(const nmt_ctx* ctx);

/* Overflow detection on the accumulated gradients and their conversion to the original scale ("Half-Precision
 * Training": after accumulation the fp16 gradients, by then fp32 sums, are brought back to the scale of the
 * loss before the weights are updated).  *d_flag = 1 iff any element of acc32 is inf or NaN, else 0, in one
 * read-only pass over acc32; inv_scale = 1 / (loss_scale * total n_tok) is remembered by the context and applied
 * by nmt_adam_step to every element as it reads it (acc32 itself keeps the scaled sums: the unscaled gradient is
 * never written out, which saves one 4-byte write and one 4-byte read per parameter). */
int nmt_check_overflow(nmt_ctx* ctx, float inv_scale, int32_t* d_flag, void* stream);

/* Adam ("Models and Hyperparameters": beta1 0.9, beta2 0.98, epsilon 1e-8) on the fp32 master weights
 * with gradient acc32 * inv_scale (the factor of the last nmt_check_overflow; 1 if none was made) -- the optimizer
 * runs in fp32 ("Half-Precision Training") -- then w16 =
 * round-to-nearest-even of the new master weights.  t is the 1-based update count.  If *d_flag != 0 the
 * call changes nothing (the update is skipped on overflow). */
int nmt_adam_step(nmt_ctx* ctx, float lr, float beta1, float beta2, float eps, int32_t t,
                  const int32_t* d_flag, void* stream);

/* nmt_accumulate of an update's last pass, nmt_check_overflow and nmt_adam_step as one call, for callers that do nothing with
 * acc32 in between (several GPUs: the sum over ranks lies there): every buffer and *d_flag end up with the same bits, in fewer
 * passes over them. */
int nmt_finish_update(nmt_ctx* ctx, int32_t first, float inv_scale, float lr, float beta1, float beta2, float eps, int32_t t,
                      int32_t* d_flag, void* stream);

/* Host helpers holding the scalar decision logic.
 * Dynamic loss scaling: overflow -> scale /= 2, clean = 0; otherwise clean += 1 and when clean
 * reaches `window` (2000 in the paper) scale *= 2, clean = 0.  Returns NMT_EINVAL if the scale
 * would fall below 2^-14. */
int nmt_scaler_update(float* scale /*host*/, int32_t* clean /*host*/, int32_t overflow, int32_t window);
/* Learning rate of update t (1-based) as in "Models and Hyperparameters": linear warm-up to `peak`
 * (5e-4, or 1e-3 with large batches) over `warmup` (4000) updates, then proportional to the inverse
 * square root of t. */
double nmt_lr_schedule(int64_t t, double peak, int64_t warmup);

/* Host only.  Debug export for the parity tests: the place, inside the caller's workspace, of an activation the
 * last forward call saved for its backward pass.  name: "enc<l>.ffn.h" / "dec<l>.ffn.h" (the feed-forward
 * hidden activation after ReLU and dropout, fp16 [rows, d_ff]; an element > 0 is an open ReLU gate) or
 * "enc<l>.out" / "dec<l>.out" (the block's output, fp16 [rows, d_model]); rows = source / target positions of
 * the pass, in its row order.  The memory stays the caller's; it is overwritten by the next forward call. */
int nmt_debug_activation(const nmt_ctx* ctx, const char* name, const void** d_ptr, int64_t* rows, int64_t* cols);

/* Host only.  Process-wide switches of launch forms, for tests and profiling; none of them changes a
 * result bit but "row_chain", which changes the order in which the gradients of gains, shifts and output biases are summed over the rows.  name: "gemm_group" (tile rows swept together, >= 1; default 4), "gemm_persist" (0: never the
 * persistent GEMM form / 1: for 256 x 256 tiles with one of its epilogues; default 1),
 * "attn_persist" (0: one attention work item per work-group; default 1), "worklists" (0: attention
 * kernels enumerate every (sentence, tile); default 1), "one_stream" (1: forward and backward passes enqueue everything
 * on the caller's stream; default 0), "gemm_share" (1..16, default 1: the number of products a
 * caller keeps running side by side on streams of its own; large tiles are then chosen as if each product had
 * that fraction of the compute units), "gemm_tile" (0: tile shape chosen per product, the default; 1..5: every
 * product that is not cut along k, except a layer's weight gradients, takes 256x256 / 128x128 / 128x64 / 64x128 / 64x64
 * tiles), "row_chain" (0: the operations between two attentions of a narrow model are launches of their own; 1, the default: one launch
 * each way for models 64, 128 or 256 wide with d_ff = 1 to 4 times d_model, act_dropout = 0 and at most four, 256 wide one, work-groups of 16 rows to a
 * compute unit; not to be changed between a forward call and its backward call), "gemm_timing" (1: every GEMM product, and every launch of a layer's weight gradients, is bracketed by a pair of
 * HIP events on the stream it is launched on; default 0), "defaults" (value ignored: all of the above back to
 * default).  Unknown names and values out of range return NMT_EINVAL. */
int nmt_tuning(const char* name, int32_t value);
/* Host only; waits for the products concerned.  With "gemm_timing" on: the sum of the event-bracketed durations
 * (milliseconds) of the GEMM products launched since the last call, their number, and their algorithmic FLOPs
 * (2 M N K each); any of the three pointers may be NULL.  The measurement behind the benchmark's roofline figure. */
int nmt_gemm_timing(double* ms /*host*/, int64_t* products /*host*/, double* flops /*host*/);

/* ------------------------------------------------------------------------------------------
 * Kernel-level entry points (used by the per-kernel parity tests and by profiling).
 * ------------------------------------------------------------------------------------------ */

/* Dropout description for the kernels that draw masks.  Element (row r, column c) of a
 * [rows, n_cols] activation whose row r is position r % n_pos of sentence r / n_pos is kept iff
 * the 16-bit word  (Philox4x32-10(counter = (c >> 3, uid, site << 16 | pos, step << 8 | micro),
 * key = seed)[(c >> 1) & 3] >> 16 * (c & 1)) & 0xffff  is >= ceil(p * 2^16); kept values are
 * multiplied by 1 / (1 - p).  uid = d_sent_uid[sentence] or the sentence index if NULL. */
typedef struct {
  float p;
  uint32_t site, step, micro;
  uint64_t seed;
  int32_t n_pos;
  const uint32_t* d_sent_uid;
} nmt_dropout;

/* C[M,N] = epilogue(sum_k A(m,k) B(n,k)), fp16 operands, fp32 accumulation, fp16 result.
 * a_t == 0: A stored [M,K] (lda >= K); a_t != 0: stored [K,M] (lda >= M).
 * b_t == 0: B stored [N,K]; b_t != 0: stored [K,N].  The contiguous dimension of each operand,
 * N, and all leading dimensions must be multiples of 8; pointers 16-byte aligned.
 * Epilogue, in this order: + bias[n] (fp16, or NULL); ReLU if relu != 0; dropout if drop != NULL
 * and drop->p > 0; + add[m,n] (fp16 with leading dimension ldc, may alias C; or NULL);
 * if relu_src != NULL (fp16 [M,N], ld = ldc): result = relu_src > 0 ? result * mask_scale : 0. */
int nmt_op_gemm(const void* d_A, int32_t a_t, int32_t lda, const void* d_B, int32_t b_t, int32_t ldb,
                void* d_C, int32_t ldc, int32_t M, int32_t N, int32_t K, const void* d_bias,
                int32_t relu, const nmt_dropout* drop, const void* d_add, const void* d_relu_src,
                float mask_scale, void* stream);

/* The same product without epilogue, with the contraction cut into `splits` (1..64; 0 = chosen by
 * the library) equal pieces whose fp32 partial results go to d_partial (partial_floats >= splits *
 * M * N floats, 16-byte aligned) and are summed in increasing k order by a second kernel.  (The backward pass
 * uses it for the vocabulary's input gradient, with a number of its own; a layer's weight gradients are nmt_op_wgrad_group.) */
int nmt_op_gemm_splitk(const void* d_A, int32_t a_t, int32_t lda, const void* d_B, int32_t b_t, int32_t ldb,
                       void* d_C, int32_t ldc, int32_t M, int32_t N, int32_t K, float* d_partial,
                       int64_t partial_floats, int32_t splits, void* stream);

/* The weight gradients of several linear layers in one launch (the form the backward pass uses for a layer): for each
 * product g_w[out, in] = out_scale * sum_r dy[r, out] x[r, in] and, if d_gb is not null, g_b[out] = out_scale *
 * sum_r dy[r, out].  out and in are multiples of 8, matrices 16-byte aligned.  With more than one split (0 = chosen by the
 * library) the rows are cut into that many pieces whose fp32 sums go to d_partial (partial_floats >= splits * sum over
 * the products of out * (in + 1); may be null: never cut) and are added in increasing order by a second kernel.  tile:
 * 0 = chosen by the library; 1..4 force 256 x 256, 128 x 128 (two work-groups per compute unit), 128 x 128 and 64 x 64. */
typedef struct nmt_wgrad {
  const void* d_dy;
  const void* d_x;
  void* d_gw;
  void* d_gb;
  int32_t ld_dy, ld_x, ld_gw;
  int32_t out, in, rows;
} nmt_wgrad;
int nmt_op_wgrad_group(int32_t n, const nmt_wgrad* products, float out_scale, float* d_partial, int64_t partial_floats, int32_t tile,
                       int32_t splits, void* stream);

/* The same product with fp32 operands and an fp32 result, no epilogue: C[M,N] = sum_k A(m,k) B(n,k) on the fp32
 * matrix instructions.  Benchmark only -- the training step never calls it: it times what the step's products cost
 * without half precision ("Half-Precision Training" compares fp32 and fp16 training at equal settings; Table 1,
 * rows "Our reimplementation" and "16-bit").  Operands 16-byte aligned, leading dimensions multiples of 4.
 * splits (1..64) > 1 cuts the contraction into that many pieces (the form a weight gradient over many positions
 * needs to fill the chip): piece z writes its partial product to rows [z*M, (z+1)*M) of d_C, which then holds
 * splits * M rows; the caller sums them. */
int nmt_op_gemm_f32(const float* d_A, int32_t a_t, int32_t lda, const float* d_B, int32_t b_t, int32_t ldb,
                    float* d_C, int32_t ldc, int32_t M, int32_t N, int32_t K, int32_t splits, void* stream);

/* Masked multi-head attention forward.  Q [B*Tq, *] with row stride ldq (head h at columns
 * h*dh..), K, V [B*Tk, *]; O [B*Tq, *]; d_lse fp32 = log-sum-exp of the scaled
 * scores, stored [H, B*Tq] (head-major).  Key j of sentence b is hidden iff d_key_ids[b*Tk + j] == pad_id, or causal != 0 and
 * j > query index.  Scores are scaled by 1/sqrt(dh). */
int nmt_op_attention_fwd(const void* d_Q, int32_t ldq, const void* d_K, int32_t ldk, const void* d_V,
                         int32_t ldv, void* d_O, int32_t ldo, float* d_lse, const int32_t* d_key_ids,
                         int32_t pad_id, int32_t causal, int32_t B, int32_t H, int32_t dh, int32_t Tq,
                         int32_t Tk, void* stream);
/* Backward of the above: dQ, dK, dV from dO (and the forward's Q, K, V, O, lse). */
int nmt_op_attention_bwd(const void* d_Q, int32_t ldq, const void* d_K, int32_t ldk, const void* d_V,
                         int32_t ldv, const void* d_O, int32_t ldo, const void* d_dO, int32_t lddo,
                         const float* d_lse, void* d_dQ, int32_t lddq, void* d_dK, int32_t lddk,
                         void* d_dV, int32_t lddv, const int32_t* d_key_ids, int32_t pad_id,
                         int32_t causal, int32_t B, int32_t H, int32_t dh, int32_t Tq, int32_t Tk,
                         void* stream);

/* out = LayerNorm(resid + dropout(sub)) * gamma + beta per row of [rows, d] (fp16 in/out, fp32
 * math); d_stats fp32 [rows, 2] receives (mean, 1/sqrt(var + eps)). */
int nmt_op_residual_layernorm_fwd(const void* d_sub, const void* d_resid, const void* d_gamma,
                                  const void* d_beta, void* d_out, float* d_stats, int32_t rows,
                                  int32_t d, float eps, const nmt_dropout* drop, void* stream);
/* Backward: from d_dout (gradient at the LayerNorm output) computes d_dy (gradient at the
 * pre-normalisation sum), d_dym = dropout-masked d_dy (gradient at the sub-layer output),
 * and the fp16 vectors dgamma, dbeta and dbias = column sums of d_dym.  d_partial: fp32 scratch
 * of nmt_op_layernorm_bwd_scratch(d) floats. */
int64_t nmt_op_layernorm_bwd_scratch(int32_t d);
int nmt_op_residual_layernorm_bwd(const void* d_dout, const void* d_sub, const void* d_resid,
                                  const void* d_gamma, const float* d_stats, void* d_dy, void* d_dym,
                                  void* d_dgamma, void* d_dbeta, void* d_dbias, float* d_partial,
                                  int32_t rows, int32_t d, const nmt_dropout* drop, void* stream);

/* x[r, :] = dropout(sqrt(d) * E[ids[r], :] + PE(r % n_pos, :)), sinusoidal positions. */
int nmt_op_embed_fwd(const int32_t* d_ids, const void* d_E, void* d_x, int32_t rows, int32_t d,
                     int32_t vocab, const nmt_dropout* drop, void* stream);

/* Per row of fp16 logits [rows, V]: label-smoothed loss against d_targets (pad_id rows count
 * nothing), written to d_row_loss (fp32 [rows]); logits are overwritten in place by
 * loss_scale * (softmax - smoothed target) (zeros on pad rows).  Then *d_loss_sum, *d_ntok are
 * reduced deterministically. */
int nmt_op_softmax_xent(void* d_logits, const int32_t* d_targets, float* d_row_loss, int32_t rows,
                        int32_t V, int32_t pad_id, float label_smoothing, float loss_scale,
                        float* d_loss_sum, int32_t* d_ntok, void* stream);

/* dst[c] = fp16(sum_r src[r, c]) for fp16 src [rows, cols] (ld); d_partial: fp32 scratch of
 * nmt_op_colsum_scratch(cols) floats. */
int64_t nmt_op_colsum_scratch(int32_t cols);
int nmt_op_colsum(const void* d_src, int32_t ld, void* d_dst, float* d_partial, int32_t rows,
                  int32_t cols, void* stream);

/* nmt_op_colsum for callers that cannot allocate device memory and have no scratch buffer to pass: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same kernels and same
 * result bits; the partial sums live in a fixed device array of the library (8 MiB per GPU, held until the
 * process ends) instead of d_partial, so cols is limited to 4096 (NMT_EINVAL beyond that, before anything
 * is launched).  The call allocates and frees nothing.  All calls on one GPU share the array: calls that
 * overlap on one GPU (different streams) race; calls on one stream are ordered and need no clearing in
 * between (every partial sum read is written by the same call first). */
int nmt_op_colsum_static(const void* d_src, int32_t ld, void* d_dst, int32_t rows, int32_t cols, void* stream);

/* Embedding backward: d_gE[v, :] = fp16(float(d_gE[v, :]) + sqrt(d) * sum over positions r with
 * ids[r] == v of dropout-masked d_dx[r, :]), for two id streams (source then target) at once.
 * Deterministic: every sum is formed in a fixed order (the positions, sorted by id, in pieces of 16:
 * increasing position within a piece, then the pieces of an id in a fixed order).  d_scratch: 16-byte aligned int32 scratch of
 * nmt_op_embed_bwd_scratch(vocab, rows_a + rows_b, d) int32 elements.  vocab <= 65536. */
int64_t nmt_op_embed_bwd_scratch(int32_t vocab, int32_t rows_total, int32_t d);
int nmt_op_embed_bwd(const int32_t* d_ids_a, const void* d_dx_a, int32_t rows_a, const nmt_dropout* drop_a,
                     const int32_t* d_ids_b, const void* d_dx_b, int32_t rows_b, const nmt_dropout* drop_b,
                     void* d_gE, int32_t d, int32_t vocab, int32_t* d_scratch, void* stream);

/* Element-wise update kernels on n scalars (the bodies of nmt_accumulate, nmt_check_overflow
 * and nmt_adam_step). */
int nmt_op_accumulate(const void* d_g16, float* d_acc32, int64_t n, int32_t first, void* stream);
/* nmt_op_check_overflow is the single-pass form that also unscales in place: *d_flag as above and
 * d_acc32 *= inv_scale.  nmt_op_adam updates with d_g32 * grad_scale. */
int nmt_op_check_overflow(float* d_acc32, int64_t n, float inv_scale, int32_t* d_flag, void* stream);
int nmt_op_adam(float* d_master32, float* d_m, float* d_v, const float* d_g32, float grad_scale, void* d_w16, int64_t n,
                float lr, float beta1, float beta2, float eps, int32_t t, const int32_t* d_flag,
                void* stream);

/* Writes the dropout keep decisions (1 / 0 bytes) of a [rows, n_cols] activation. */
int nmt_op_dropout_mask(uint8_t* d_keep, int32_t rows, int32_t n_cols, const nmt_dropout* drop,
                        void* stream);

/* ------------------------------------------------------------------------------------------
 * Operators for models beyond the step above: deeper ones (norms around a gated residual block), sparse ones (tokens
 * sorted by expert and back) and larger ones (AdamW over many tensors, its states in 8 bits if wanted).
 * Rows are fp16, bf16 or fp32; sums, statistics and norms are fp32.  Rows may lie any distance >= d apart (ld, in
 * elements), and d and every address may be any that the type itself allows.  The same inputs give the same bits.
 * No rows and no tokens are a call like any other: sums over none are zero, ranges are empty.
 * ------------------------------------------------------------------------------------------ */
#define NMT_F16 0
#define NMT_BF16 1
#define NMT_F32 2
#define NMT_NORM_LAYER 0 /* (a - mean) / sqrt(mean((a - mean)^2) + eps) */
#define NMT_NORM_RMS 1   /* a / sqrt(mean(a^2) + eps)                     */
#define NMT_ONE_GATE 0x7FFFFFFF /* rows_per_gate: one gate for all rows, also for none */

/* The norms after one block and before the next, with the block's gate and the scale of its residual, row by row:
 *   h = resid_scale * x + gate * post(y),  post(y) = norm(y) * post_gain + post_shift   (y itself if d_post_gain is NULL)
 *   n = norm(h) * pre_gain + pre_shift                                              (not wanted if d_n is NULL)
 * y: the block's output, x: the residual stream before it, n: the next block's input.  n is formed from h before h is
 * rounded.  d_gate NULL: 1; otherwise row r takes row r / rows_per_gate of d_gate [ceil(rows / rows_per_gate), d] (rows_per_gate >= rows: one
 * gate for all; 1: a gate for every element).  No rows have no gates and nothing is written to their gradient, unless rows_per_gate is NMT_ONE_GATE: then there is one, whose gradient is zero.  Shifts may be NULL (0).  Gains, shifts and gates are contiguous, of the rows' type.
 * d_y NULL: the norm before the first block, n = norm(x) * pre_gain + pre_shift; d_h, d_post_gain, d_gate are then NULL too, and resid_scale is 1.
 * d_stats: fp32 [rows, 4] = mean and 1 / sqrt(.) of y, then of h (0 and 1 where there is no norm; RMS: mean 0), for the backward call; may be
 * NULL.  d_h may be d_x, and d_n may be d_y, with the same distance between rows; otherwise what is written overlaps nothing else.
 * d <= 16384, rows < 2^31 - 65536. */
typedef struct nmt_gated_norm {
  int32_t rows, d, type, kind; /* type: NMT_F16 / NMT_BF16 / NMT_F32; kind: NMT_NORM_LAYER / NMT_NORM_RMS */
  float eps, resid_scale;
  int32_t rows_per_gate;
  int64_t ld_x, ld_y, ld_h, ld_n;
  const void *d_x, *d_y;
  const void *d_post_gain, *d_post_shift, *d_gate, *d_pre_gain, *d_pre_shift;
  void *d_h, *d_n;
  float* d_stats;
} nmt_gated_norm;
int nmt_op_gated_norm_fwd(const nmt_gated_norm* a /*host*/, void* stream);
/* Host only.  Debug export: the work-groups of that call's launch and the threads of each, for tests of sizes that no test can allocate. */
int nmt_debug_gated_norm_grid(int32_t rows, int32_t d, int32_t type, int64_t* groups, int32_t* threads);

/* Backward of the above.  Read from `a`: rows, d, type, kind, resid_scale, rows_per_gate, the gains, shifts and gate, d_y, d_h (without d_y: the x
 * of the forward call), ld_y, ld_h and d_stats; its x, n and eps are not used.  Without d_y resid_scale is 1 for the gradient at the forward call's x; a caller that made this x
 * by itself as some factor times a tensor of its own gives the factor, and d_dx is the gradient at that tensor.  d_dh: gradient that reaches h from elsewhere (NULL: none);
 * d_dn: gradient at n (NULL: none); one of the two is there, and d_pre_gain with d_dn.  Written: d_dx (resid_scale times the gradient at h) and, with d_y, d_dy, of the
 * rows' type, and the gradients of gains, shifts and gate (sums over the rows in fp32, rounded once to the rows' type; each may be NULL).  d_dx may be d_dh and
 * d_dy may be d_dn with the same distance between rows.
 * d_scratch: 16-byte aligned, of nmt_op_gated_norm_bwd_scratch(rows, d, rows_per_gate) floats, which serve fewer rows too. */
typedef struct nmt_gated_norm_grad {
  int64_t ld_dh, ld_dn, ld_dx, ld_dy;
  const void *d_dh, *d_dn;
  void *d_dx, *d_dy;
  void *d_dpost_gain, *d_dpost_shift, *d_dgate, *d_dpre_gain, *d_dpre_shift;
  float* d_scratch;
  int64_t scratch_floats;
} nmt_gated_norm_grad;
int64_t nmt_op_gated_norm_bwd_scratch(int32_t rows, int32_t d, int32_t rows_per_gate);
int nmt_op_gated_norm_bwd(const nmt_gated_norm* a /*host*/, const nmt_gated_norm_grad* g /*host*/, void* stream);

/* Tokens to their experts.  d_expert [tokens, k]: the experts of every token (a value outside [0, experts) is none: the choice is
 * dropped); the same expert twice takes two rows.  The choices are sorted by expert, those of one expert in the order of d_expert, and row
 * d_slot[t, j] of d_rows becomes row t of d_x.
 *   capacity == 0: the experts' rows lie back to back; d_rows has tokens * k rows, and those behind the last are left as they were.
 *   capacity  > 0: expert e has the rows [e * capacity, (e + 1) * capacity) of d_rows, so that products of a size the host knows can be
 *                  enqueued; choices beyond them are dropped, and rows without a token are set to zero.
 * d_slot [tokens, k]: the row of every choice, -1 if it was dropped (another buffer than d_expert).  d_ranges [experts, 2]: first row and number of rows of every expert.
 * d_x NULL: the lists alone (d_rows is then NULL too).  d_scratch: scratch_ints >= nmt_op_expert_dispatch_scratch int32 elements.
 * k <= 64, experts <= 1024, tokens * k and experts * capacity <= 2^29, d <= 2^20. */
int64_t nmt_op_expert_dispatch_scratch(int32_t tokens, int32_t k, int32_t experts);
int nmt_op_expert_dispatch(const int32_t* d_expert, int32_t tokens, int32_t k, int32_t experts, int32_t capacity, const void* d_x,
                           int64_t ld_x, int32_t d, int32_t type, void* d_rows, int64_t ld_rows, int32_t* d_slot, int32_t* d_ranges,
                           int32_t* d_scratch, int64_t scratch_ints, void* stream);

/* And back: out[t] = add[t] + sum over j of weights[t, j] * rows[slot[t, j]], in fp32 in the order of j, rounded once.  A choice whose slot lies
 * outside [0, n_rows) adds nothing, whatever its weight.  d_weights fp32 [tokens, k], NULL: 1 (with the slots of nmt_op_expert_dispatch this is its
 * gradient: d_x from d_rows).  d_add may be NULL, or d_out with the same distance between rows. */
int nmt_op_expert_combine(const void* d_rows, int64_t ld_rows, int32_t n_rows, const int32_t* d_slot, const float* d_weights,
                          const void* d_add, int64_t ld_add, void* d_out, int64_t ld_out, int32_t tokens, int32_t k, int32_t d,
                          int32_t type, void* stream);
/* Gradients of the above: d_drows[slot[t, j]] = weights[t, j] * dout[t] and d_dweights[t, j] = the inner product of dout[t] and rows[slot[t, j]]
 * (0 for a dropped choice).  capacity and d_ranges as in nmt_op_expert_dispatch: rows without a token become zero where capacity > 0 and stay
 * as they were otherwise (d_ranges may then be NULL).  d_weights NULL: 1.  d_rows and d_dweights may both be NULL.  d_drows may be d_rows with
 * the same distance between rows; n_rows rows each.  No two choices
 * share a slot (those of nmt_op_expert_dispatch do not).  The gradient of `add` is dout. */
int nmt_op_expert_combine_bwd(const void* d_dout, int64_t ld_dout, const void* d_rows, int64_t ld_rows, int32_t n_rows,
                              const int32_t* d_slot, const float* d_weights, void* d_drows, int64_t ld_drows, float* d_dweights,
                              const int32_t* d_ranges, int32_t experts, int32_t capacity, int32_t tokens, int32_t k, int32_t d,
                              int32_t type, void* stream);

/* AdamW (Adam with decoupled weight decay) over many tensors in one launch:
 *   g = grad * grad_scale,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   master -= lr * lr_factor * (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay * master),  weights = master, rounded.
 * state_bits 32: d_m, d_v fp32 [n].  state_bits 8: one byte each, in blocks of 256 elements counted from the tensor's first (the last may be
 * shorter): m / m_scale and sqrt(v) / v_scale in OCP e4m3 (4 exponent and 3 mantissa bits), nearest, ties to even, the scale of a block being its
 * largest magnitude / 448, fp32 [ceil(n / 256)]; a sqrt(v) that is not zero is never rounded to zero, so that no step is divided by eps alone.
 * The step itself uses m and v before they are rounded.  Zeros everywhere are the states to start from.  What is inf or NaN stays so in its own element and
 * does not reach its block's scale (in 8 bits both are NaN). */
typedef struct nmt_adamw_tensor {
  int64_t n;
  float weight_decay, lr_factor;
  float* d_master;
  void *d_m, *d_v;
  float *d_m_scale, *d_v_scale; /* state_bits 8 only */
  const void* d_grad;           /* of type grad_type */
  void* d_weights;              /* of type weights_type, or NULL: no copy of this tensor */
} nmt_adamw_tensor;
typedef struct nmt_adamw nmt_adamw;
/* Bytes of the device table that nmt_adamw_create fills (host only). */
int64_t nmt_adamw_table_bytes(int32_t n, const nmt_adamw_tensor* tensors /*host*/);
/* Checks the tensors and writes the table of their pieces to d_table (16-byte aligned), which belongs to the handle until nmt_adamw_destroy.  Waits for the
 * stream, so it cannot be captured.  `tensors` itself is not kept; the buffers it names must stay where they are.  A buffer that a step writes
 * overlaps no other of the list, so no tensor is in it twice; gradients may be shared.  The table overlaps none of them. */
int nmt_adamw_create(int32_t n, const nmt_adamw_tensor* tensors /*host*/, int32_t state_bits, int32_t grad_type, int32_t weights_type,
                     void* d_table, int64_t table_bytes, void* stream, nmt_adamw** out);
void nmt_adamw_destroy(nmt_adamw* plan);
/* One step of all tensors; t >= 1 is the number of this update.  If d_flag is not NULL and *d_flag != 0 the call changes nothing, as in
 * nmt_adam_step.  lr, t and grad_scale are taken when the call is made: a captured graph repeats them. */
int nmt_adamw_step(const nmt_adamw* plan, double lr, double beta1, double beta2, double eps, int32_t t, float grad_scale,
                   const int32_t* d_flag, void* stream);

/* ------------------------------------------------------------------------------------------
 * Matrices held in 8 bits.  A matrix [rows, d] is codes in OCP e4m3 (4 exponent and 3 mantissa bits, no infinity), one byte each, rows `ld` bytes apart, and
 * fp32 scales: value = code * scale.  128 elements of a row share a scale (the last block of a row may be shorter), scale (row r, block b) at b * ld_scales + r:
 * the scales of one block of columns lie side by side.  Or, `square`, 128 x 128 elements share one: that of rows 128 q ... and block b at b * ld_scales + q.
 * Bytes behind a row's last code are neither written nor used.  Scratch belongs to one call at a time: calls that may overlap, captured ones among them, take one each.
 * ------------------------------------------------------------------------------------------ */

/* x (fp16, bf16 or fp32, any distance between rows, any address) into 8 bits.  scale = the block's largest magnitude / 448, code = x / scale, nearest, ties to
 * even; a block of nothing larger than 2^-100 is zeros.  What is inf or NaN becomes NaN in its own element and does not count for the scale.
 * d_codes, d_scales: as x lies.  d_codes_t [d, rows], d_scales_t: its transpose, whose blocks are 128 rows of x in one column (square: the same codes and scales, transposed); what
 * the products of a backward pass read.  Either pair may be NULL.  What is written overlaps nothing else. */
int nmt_op_quantize8(const void* d_x, int64_t ld_x, int32_t rows, int32_t d, int32_t type, int32_t square, void* d_codes, int64_t ld_codes,
                     float* d_scales, int64_t ld_scales, void* d_codes_t, int64_t ld_codes_t, float* d_scales_t, int64_t ld_scales_t, void* stream);

/* The norm before a block whose products take 8 bits, with the residual's addition, row by row:
 *   h = resid_scale * x + y,  n = norm(h) * gain + shift,
 * n in 8 bits to d_codes, d_scales (blocks of a row) as nmt_op_quantize8 makes them of n before it is rounded, and, if d_n is not NULL, rounded to the rows' type as well.  n is formed from h before h is
 * rounded.  d_y NULL: h is x, resid_scale is 1 and d_h NULL.  d_h may be NULL: not wanted.  d_shift may be NULL.  d_stats: fp32 [rows, 4] = 0, 1, mean and 1 / sqrt(.) of h (RMS:
 * mean 0), may be NULL: what nmt_op_gated_norm_bwd takes, with d_y as its block's output without norm or gate; the gradient passes the rounding to
 * 8 bits as if it were none.  d_h may be d_x, and d_n may be d_y, with the same distance between rows; otherwise what is written overlaps nothing else.
 * d <= 16384, rows < 2^31 - 65536. */
typedef struct nmt_norm8 {
  int32_t rows, d, type, kind; /* type: NMT_F16 / NMT_BF16 / NMT_F32; kind: NMT_NORM_LAYER / NMT_NORM_RMS */
  float eps, resid_scale;
  int64_t ld_x, ld_y, ld_h, ld_n, ld_codes, ld_scales;
  const void *d_x, *d_y, *d_gain, *d_shift;
  void *d_h, *d_n, *d_codes;
  float *d_scales, *d_stats;
} nmt_norm8;
int nmt_op_norm8(const nmt_norm8* a /*host*/, void* stream);

/* C[M, N] = A B^T + bias + add for A [M, K] and B [N, K] in 8 bits: products of codes are summed in fp32 over each block of 128 k and times its scales added up in fp32, in increasing k
 * (a long contraction of a small C in pieces, in a fixed order), rounded once to `type`.  A block's two scales are multiplied by each other first: one may be as large as the other is small, but their product is to
 * be 0 or a normal number of fp32.  (Beyond fp32 what comes of the block is infinite, or NaN where its sum is 0; below 2^-126 it is off by up to 2^-125.)  For results of 16 bits the matrix instruction adds eight products of codes at a time, to 13 bits below the largest one's power of two
 * (some 1.5e-5 of a result, at most 2^-10 of the sum of the terms' magnitudes); for fp32 results every product counts in full.  a_square, b_square: whether 128 x 128 elements share a scale.  d_bias [N] and d_add [M, N], of C's type, may be
 * NULL; d_add may be d_c with the same distances.  y = x W^T: A = x, B = W; the input's gradient: A = dy, B = W transposed; the weight's: A = dy transposed, B = x transposed.
 * batch products lie stride_* apart (bytes of A and B, elements of the others; 0: the same for all; of C not).
 * d_ranges NULL: `batch` products of M x N x K each.  Otherwise d_ranges [batch, 2] (nmt_op_expert_dispatch): expert e's rows are the ranges[e, 1] rows of A, of the scales and of C from ranges[e, 0] on, M is
 * the number of rows of A and C in all, its B, scales of B and bias lie e strides on, the other strides are not used, and a_square is 0.  Rows that no expert has are left as they
 * were; ranges do not overlap, and what of them lies outside [0, M) is cut off.  Ranges are of A's rows, never of k: the weights' gradients of experts are a batch, each expert's rows with room of their own
 * (a multiple of 128, and the rows behind an expert's last zero), since 128 rows that share a scale would reach from one expert into the next.
 * Rows of A and B begin at multiples of 16 bytes; C, bias and add have any address that their type allows and any distance.  K = 0: bias + add.  batch <= 1024; lda, ldb <= 2^22.
 * d_scratch: 16-byte aligned, scratch_floats >= nmt_op_gemm8_scratch(M, N, K, batch, ranges != NULL), which may be 0. */
typedef struct nmt_gemm8 {
  int32_t M, N, K, batch, type, a_square, b_square;
  int64_t lda, ldb, ldc, ld_add, ld_sa, ld_sb;
  int64_t stride_a, stride_b, stride_c, stride_add, stride_bias, stride_sa, stride_sb;
  const void *d_a, *d_b;
  const float *d_sa, *d_sb;
  const void *d_bias, *d_add;
  void* d_c;
  const int32_t* d_ranges;
  float* d_scratch;
  int64_t scratch_floats;
} nmt_gemm8;
int64_t nmt_op_gemm8_scratch(int32_t M, int32_t N, int32_t K, int32_t batch, int32_t ranges);
int nmt_op_gemm8(const nmt_gemm8* a /*host*/, void* stream);
/* Host only.  Debug export: the edge of the tiles that such a call is cut into and its pieces along k, for tests that are to reach every form. */
int nmt_debug_gemm8_form(int32_t M, int32_t N, int32_t K, int32_t batch, int32_t ranges, int32_t type, int32_t b_square, int32_t* tile, int32_t* splits);

/* A sparse layer as a whole over few tokens (at most 64; more: nmt_op_expert_dispatch, nmt_op_gemm8, nmt_op_expert_combine), as when one token of each sentence is at hand:
 *   hidden[t, j] = act(up[expert[t, j]] x[t]),  out[t] = add[t] + sum over j of weights[t, j] * down[expert[t, j]] hidden[t, j].
 * act NMT_ACT_RELU: up [experts, ff, d], max(., 0).  NMT_ACT_SILU_GATE: up [experts, 2 ff, d], g / (1 + exp(-g)) * u of its rows r (g) and ff + r (u).  down [experts, d, ff].  Weights in 8 bits with
 * square scales, experts stride_* apart (bytes; floats of the scales), rows at multiples of 16 bytes.  x, add and out are of `type`; products are of the inputs as they are (not in
 * 8 bits), sums fp32, out rounded once.  hidden goes from one product to the next rounded to within 2^-17 of itself (fp32: as it is).  What of x or hidden is below 2^-80, and what a block of 128 adds below 2^-109, may count with
 * fewer bits.  d_expert [tokens, k]: a value outside [0, experts) is none and adds nothing, whatever its weight; only experts that are chosen are read.
 * d_weights fp32 [tokens, k], NULL: 1.  d_add may be NULL, or d_out with the same distance.
 * d_scratch: 16-byte aligned, scratch_floats >= nmt_op_expert_layer8_scratch.  k <= 64, experts <= 1024, d and ff <= 2^20. */
#define NMT_ACT_RELU 0
#define NMT_ACT_SILU_GATE 1
typedef struct nmt_expert_layer8 {
  int32_t tokens, k, experts, d, ff, type, act;
  int64_t ld_x, ld_add, ld_out;
  int64_t ld_up, stride_up, ld_up_scales, stride_up_scales, ld_down, stride_down, ld_down_scales, stride_down_scales;
  const void* d_x;
  const int32_t* d_expert;
  const float* d_weights;
  const void* d_up;
  const float* d_up_scales;
  const void* d_down;
  const float* d_down_scales;
  const void* d_add;
  void* d_out;
  float* d_scratch;
  int64_t scratch_floats;
} nmt_expert_layer8;
int64_t nmt_op_expert_layer8_scratch(int32_t tokens, int32_t k, int32_t experts, int32_t d, int32_t ff);
int nmt_op_expert_layer8(const nmt_expert_layer8* a /*host*/, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NMT_H_ */
