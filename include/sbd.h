/*
 * sbd.h - C ABI of the MI355X (gfx950) Set Block Decoding decode step.
 *
 * One decode step of Set Block Decoding (SBD, arXiv 2509.04185) is one forward pass
 * of the SBD network f_theta over a block of k rows against an exact KV cache
 * (Sec. 2.3, eq. (hybrid_block); Alg. 3), followed by one step of the entropy-bounded
 * (EB) sampler (Sec. 2.2, eq. (eb_sampler)).  This library runs both on one GPU with
 * hand-written HIP kernels.
 *
 * Conventions shared by every entry point
 *  - Every function returns an sbd_status; no exception crosses the ABI.
 *  - Arguments and state are validated on the host before anything is enqueued; on
 *    any error nothing is enqueued and no state changes.  sbd_last_error() then gives
 *    a one-line reason.
 *  - "device" pointers are GPU global memory (e.g. torch CUDA tensors); "host"
 *    pointers are ordinary CPU memory that is read before the call returns.
 *  - All GPU work is enqueued on the context's stream and is asynchronous: outputs are
 *    valid once that stream has been synchronised.  An asynchronous device fault is
 *    reported as SBD_ERR_HIP by a later call.
 *  - Row-major layouts throughout; bf16 means IEEE bfloat16 (1/8/7 bits).
 *  - A context is used by one host thread at a time.  The library keeps no global
 *    state other than the thread-local error text of context-less calls.
 */
#ifndef SBD_H_
#define SBD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SBD_OK = 0,
  SBD_ERR_INVALID_ARG = 1,   /* a pointer, size, id or value is out of its documented range */
  SBD_ERR_STATE = 2,         /* the call is not allowed in the context's current state */
  SBD_ERR_CAPACITY = 3,      /* a sequence would exceed max_seq_len */
  SBD_ERR_OUT_OF_MEMORY = 4, /* the workspace is smaller than sbd_workspace_bytes() */
  SBD_ERR_HIP = 5,           /* a HIP runtime call or an earlier kernel failed */
  SBD_ERR_UNSUPPORTED = 6    /* the model shape is outside what the kernels implement */
} sbd_status;

typedef struct sbd_ctx sbd_ctx; /* opaque, created by sbd_create */

/* Selection rules of one sampling step (sbd_select, sbd_block_step). */
enum { SBD_SELECT_EB_ENTROPY = 0, SBD_SELECT_EB_CONFIDENCE = 1, SBD_SELECT_FACTOR = 2 };

/*
 * Decoder shape (Llama-3.1 / Qwen-3 style; the SBD network has no architectural
 * changes, Sec. 1) plus capacity limits.
 *   n_q_heads % n_kv_heads == 0; query head h reads KV head h / (n_q_heads/n_kv_heads).
 *   head_dim is 64 or 128.  d_model, n_q_heads*head_dim and ffn_dim are multiples of 256;
 *   vocab and (n_q_heads + 2 n_kv_heads) * head_dim are multiples of 128.  mask_id in
 *   [0, vocab) is the input-only mask token 'm'.
 *   qk_norm != 0 enables the per-head RMSNorm of q and k before RoPE (Qwen-3).
 *   max_batch: number of sequence slots (ids 0..max_batch-1).
 *   max_seq_len: tokens per slot, including the k rows staged by a block forward.
 *   max_block: largest k accepted by sbd_block_forward / sbd_eb_select (<= 64).
 *   prefill_chunk: rows per forward inside sbd_prefill at most (0: the library chooses, up to
 *   1024).
 */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab, mask_id;
  int32_t qk_norm;
  float rms_eps, rope_theta;
  int32_t max_batch, max_seq_len, max_block, prefill_chunk;
  int32_t weight_format;  /* SBD_WEIGHTS_BF16 (0) or SBD_WEIGHTS_FP8_E4M3 (1), see sbd_weights */
  int32_t kv_format;      /* SBD_KV_BF16 (0) or SBD_KV_FP8_E4M3 (1), see below */
  int32_t kv_scale_exp;   /* SBD_KV_FP8_E4M3 only (else ignored): scale exponent e in [-100, 100] */
} sbd_model_config;

/*
 * Formats of the projection and LM-head matrices (wq, wk, wv, wo, w_gate, w_up, w_down,
 * lm_head).  The embedding and every norm gain are bf16 in both.
 *   SBD_WEIGHTS_BF16      bf16 values.
 *   SBD_WEIGHTS_FP8_E4M3  OCP e4m3 bytes (1 sign, 4 exponent bits of bias 7, 3 mantissa
 *                         bits; no infinities, 0x7f / 0xff NaN) with a power-of-two scale per
 *                         matrix: the weight is e4m3(q) * 2^e (the FP8 weights of the
 *                         paper's timing model, Sec. 4.1).  Every forward streams the bytes
 *                         and widens them to bf16 in registers (exactly), except the fused
 *                         decode path, which streams a bf16 copy of the same values made in
 *                         sbd_create.
 */
enum { SBD_WEIGHTS_BF16 = 0, SBD_WEIGHTS_FP8_E4M3 = 1 };

/*
 * Formats of the KV cache (the cache of exact KV caching, Sec. 1 and Alg. 3).
 *   SBD_KV_BF16      each cached key (after RoPE) and value is the bf16 rounding (nearest,
 *                    ties to even) of the float the forward computes.
 *   SBD_KV_FP8_E4M3  one byte per element (the 1-byte KV of the paper's timing model,
 *                    Sec. 4.1): the e4m3 code of v * 2^-e, e = kv_scale_exp, rounded to the
 *                    nearest code with ties to even and saturated at +-448 (NaN stays NaN),
 *                    read back as e4m3 * 2^e.  The rows a forward stages are rounded so
 *                    before its own attention reads them.  sbd_kv_import rounds its bf16
 *                    input the same way; sbd_kv_export returns the stored values, which
 *                    bf16 holds exactly.  The fused decode path reads bf16 caches only
 *                    (UNSUPPORTED here); the other paths read both formats.
 */
enum { SBD_KV_BF16 = 0, SBD_KV_FP8_E4M3 = 1 };

/*
 * Weights: device memory, borrowed (they must outlive the context and not change); bf16,
 * or for the projection and LM-head matrices the format of cfg->weight_format.
 * Matrices are logical [out][in] row-major.  Per-layer fields are host arrays of
 * n_layers device pointers.  q_norm / k_norm may be NULL when qk_norm == 0.
 *   embed [vocab][d_model], lm_head [vocab][d_model], final_norm [d_model]
 *   attn_norm [d_model], wq [n_q_heads*head_dim][d_model], wk, wv [n_kv_heads*head_dim][d_model],
 *   wo [d_model][n_q_heads*head_dim], q_norm, k_norm [head_dim], mlp_norm [d_model],
 *   w_gate, w_up [ffn_dim][d_model], w_down [d_model][ffn_dim]
 */
typedef struct {
  const void *embed, *lm_head, *final_norm;
  const void *const *attn_norm, *const *wq, *const *wk, *const *wv, *const *wo;
  const void *const *q_norm, *const *k_norm, *const *mlp_norm;
  const void *const *w_gate, *const *w_up, *const *w_down;
  /* SBD_WEIGHTS_FP8_E4M3 only (else ignored): host int32 [n_layers * 7 + 1], the scale
   * exponents e of wq, wk, wv, wo, w_gate, w_up, w_down of layer 0, of layer 1, ..., then
   * of lm_head; each in [-100, 100]. */
  const int32_t* fp8_scale_exp;
} sbd_weights;

/* Bytes of device workspace sbd_create needs for this config (KV cache, activations,
 * partial results, RoPE table, and a copy of every weight matrix repacked into the
 * order the GEMM kernels stream).  *bytes is set only on SBD_OK. */
sbd_status sbd_workspace_bytes(const sbd_model_config* cfg, size_t* bytes);

/*
 * Create a context on the current HIP device.  workspace: device memory of at least
 * sbd_workspace_bytes() bytes, 256-byte aligned, caller-owned, not touched by anyone
 * else while the context lives.  stream: a hipStream_t (NULL = the null stream).
 * Every sequence slot starts empty.  The weights are read here once, to repack them into
 * the workspace (the originals must still outlive the context: the embedding and norm
 * gains are read from them).  The library allocates no device memory itself; it
 * allocates a small pinned host staging buffer here.
 */
sbd_status sbd_create(const sbd_model_config* cfg, const sbd_weights* w, void* workspace,
                      size_t workspace_bytes, void* stream, sbd_ctx** out);
sbd_status sbd_destroy(sbd_ctx* ctx);
/* Replace the stream later calls enqueue on (e.g. torch's current stream). */
sbd_status sbd_set_stream(sbd_ctx* ctx, void* stream);

/* Empty one sequence slot (cache length 0, nothing staged). */
sbd_status sbd_reset(sbd_ctx* ctx, int32_t seq);
/* Number of committed tokens in a slot. */
sbd_status sbd_cache_len(const sbd_ctx* ctx, int32_t seq, int32_t* len);

/*
 * Prefill (Alg. 2, first step): a causal forward f_theta(x;) over n prompt tokens
 * (host int32 ids in [0, vocab), mask id excluded) appended after the slot's cache,
 * committing all n rows.  Runs in forwards of at most prefill_chunk rows.
 * last_logits: device fp32 [vocab] receiving the logits of the last prompt row, or NULL.
 * Errors: CAPACITY if cache_len + n > max_seq_len.
 */
sbd_status sbd_prefill(sbd_ctx* ctx, int32_t seq, const int32_t* tokens, int32_t n,
                       float* last_logits);

/*
 * Block forward (eq. (hybrid_block); one iteration of Alg. 3) for `batch` sequences.
 *   seq_ids  host [batch], distinct slot ids.
 *   tokens   host [batch][k] ids in [0, vocab); mask rows hold mask_id.
 *   is_mask  host [batch][k] or NULL; when given it must equal (tokens == mask_id).
 *   n_causal host [batch] or NULL (= all 1).  Rows j < n_causal[b] are committed but
 *            not yet cached tokens and attend causally; rows j >= n_causal[b] form the
 *            prediction block and see every row (App. A inference mask: key kv is
 *            visible to query q iff kv <= q or q >= the first prediction index).
 *            Causal rows may not be masks.
 *   pos_ids  host [batch][k] or NULL (= cache_len + j).  RoPE positions; causal rows
 *            must keep cache_len + j.  Values in [0, max_seq_len).
 *   logits   device fp32 [batch][k][vocab], all rows, all vocab columns (row j's
 *            logits predict the token at its own position, eq. (p_theta_masked)).
 * The K/V of all k rows are staged in cache slots [cache_len, cache_len + k); the
 * first n_causal of them become permanent with sbd_commit.
 * Errors: CAPACITY if cache_len + k > max_seq_len for some sequence.
 */
sbd_status sbd_block_forward(sbd_ctx* ctx, int32_t batch, const int32_t* seq_ids, int32_t k,
                             const int32_t* tokens, const uint8_t* is_mask,
                             const int32_t* n_causal, const int32_t* pos_ids, float* logits);

/*
 * One decode step in one call: sbd_block_forward followed by the selection rule `rule`
 * (SBD_SELECT_*, threshold as for sbd_select) over the masked rows, with the selection's
 * softmax statistics taken from the LM head itself (Sec. 2.2, eq. (eb_sampler): only each
 * row's entropy, confidence and argmax are needed, not its logits).  The LM head's epilogue
 * reduces every 64-column chunk of every row to (max, argmax, Z, S) in float64; a merge
 * forms each row's entropy, confidence and token; the logits are written only when
 * `logits` is not NULL, and never read back.
 *   Arguments as sbd_block_forward and sbd_select; is_mask may be NULL (then the masked
 *   set is tokens == mask_id); the column mask_id of the config is excluded.
 *   logits    device fp32 [batch][k][vocab] or NULL.
 *   outputs   n_accepted [batch], accepted_pos [batch][k] (row indices of the block,
 *             ascending, then -1), accepted_tok [batch][k], entropy and confidence
 *             [batch][k] (nullable): as sbd_select.
 * The entropies equal sbd_select's on the same logits up to float64 summation order (the
 * chunks differ; ~1e-12 relative); the accepted rows and tokens are the same except where
 * a decision is that close.  Limits: batch * k <= 512 (INVALID_ARG beyond).  On the fused
 * decode path (SBD_DECODE_FUSED) the statistics come from the stored logits, which must
 * then be given (UNSUPPORTED otherwise).  The staged K/V and sbd_commit are as for
 * sbd_block_forward.
 */
sbd_status sbd_block_step(sbd_ctx* ctx, int32_t rule, int32_t batch, const int32_t* seq_ids, int32_t k,
                          const int32_t* tokens, const uint8_t* is_mask, const int32_t* n_causal,
                          const int32_t* pos_ids, double threshold, float* logits, int32_t* n_accepted,
                          int32_t* accepted_pos, int32_t* accepted_tok, double* entropy,
                          double* confidence);

/*
 * Exact KV caching (Sec. 1, advantages; Alg. 3): make the K/V staged by the last block
 * forward of each listed sequence permanent for its first n_commit[b] rows
 * (cache_len += n_commit[b]).  n_commit[b] <= that forward's n_causal[b], else STATE.
 * Host arrays seq_ids, n_commit [batch].  Bookkeeping only: no data moves.
 */
sbd_status sbd_commit(sbd_ctx* ctx, int32_t batch, const int32_t* seq_ids,
                      const int32_t* n_commit);

/*
 * EB-Sampler step (Sec. 2.2, eq. (eb_sampler)) on fp32 logits.
 *   logits   device fp32 [batch][k][vocab] (any logits; vocab <= the config's vocab).
 *   is_mask  host [batch][k]: the masked set M of each block.
 *   gamma    >= 0, may be +INFINITY; NaN is rejected.
 *   mask_id  column excluded from the distribution, or -1 for none.
 * For each masked row: H = entropy (nats, float64) of softmax over the vocabulary
 * without mask_id, tok = smallest id attaining the maximum logit.  Masked rows are
 * ordered by (H, row) ascending; with c_r the float64 running sum of the first r
 * entropies (c_0 = 0), s = largest r in [1, |M|] with c_{r-1} <= gamma.
 * Outputs (device): n_accepted [batch] = s (0 if M is empty); accepted_pos
 * [batch][k] = the s rows ascending, then -1; accepted_tok [batch][k] = their tokens,
 * then -1; entropy [batch][k] (nullable) = H for masked rows, NaN otherwise.
 * A masked row whose softmax is undefined (no finite logit outside mask_id, or a NaN or
 * infinite logit) has H = NaN (tok = -1 when no logit is finite), is ordered after every
 * other row and is never accepted: s runs over the other masked rows only, and is 0 when
 * there are none.
 */
sbd_status sbd_eb_select(sbd_ctx* ctx, int32_t batch, int32_t k, int32_t vocab,
                         const float* logits, const uint8_t* is_mask, double gamma,
                         int32_t mask_id, int32_t* n_accepted, int32_t* accepted_pos,
                         int32_t* accepted_tok, double* entropy);

/*
 * One sampling step under a selection rule (Sec. 2.2 and App. B), on fp32 logits.
 * Arguments and outputs as sbd_eb_select, plus:
 *   rule       SBD_SELECT_EB_ENTROPY: exactly sbd_eb_select (threshold = gamma).
 *              SBD_SELECT_EB_CONFIDENCE: App. B, EB-Sampler with the confidence error
 *              proxy: masked rows ordered by (confidence descending, row); s = largest r
 *              in [1, |M|] with sum_{j<=r} H - max_{j<=r} H <= threshold (float64,
 *              summed in that order).
 *              SBD_SELECT_FACTOR: App. B, Factor parallel decoding: the same order; s =
 *              largest r with (r + 1) * (1 - c_r) < threshold, at least 1 (c_r the r-th
 *              confidence; App. B prints the condition without the 1 -, which would
 *              reveal fewer rows the more confident they are).
 *   threshold  gamma (EB rules) or f (Factor): >= 0, may be +INFINITY; NaN is rejected.
 *   confidence device float64 [batch][k] (nullable) = max_v p_v = 1 / Z of each masked
 *              row (the softmax without mask_id), NaN otherwise.
 * As for sbd_eb_select, a row with NaN statistics is never accepted.
 * Errors: INVALID_ARG for an unknown rule, otherwise as sbd_eb_select.
 */
sbd_status sbd_select(sbd_ctx* ctx, int32_t rule, int32_t batch, int32_t k, int32_t vocab,
                      const float* logits, const uint8_t* is_mask, double threshold, int32_t mask_id,
                      int32_t* n_accepted, int32_t* accepted_pos, int32_t* accepted_tok, double* entropy,
                      double* confidence);

/*
 * sbd_eb_select for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, hosts that forbid hipMalloc): no context and no workspace.
 * The chunk statistics live in a fixed scratch array of the library (1.75 MiB per device,
 * held until the process ends; its device address is looked up on the first call on each
 * device).  No hipMalloc, hipFree or other allocating call is made.
 *   stream   hipStream_t to enqueue on (NULL = the null stream); the current device's
 *            scratch is used.
 *   Other arguments, outputs and the selection rule exactly as sbd_eb_select, with
 *   is_mask a host array [batch][k].
 * Limits: batch * k <= 1024, k <= 64, vocab <= 262144; beyond them INVALID_ARG (and
 * nothing is enqueued).  Errors are reported through sbd_last_error(NULL).
 * All calls on one device share its scratch: two calls that overlap in time on one device
 * (different streams, or different host threads) race and give wrong results.
 */
sbd_status sbd_eb_select_noalloc(void* stream, int32_t batch, int32_t k, int32_t vocab,
                                 const float* logits, const uint8_t* is_mask, double gamma,
                                 int32_t mask_id, int32_t* n_accepted, int32_t* accepted_pos,
                                 int32_t* accepted_tok, double* entropy);

/*
 * The selection part of sbd_eb_select alone, on given entropies (device float64
 * [batch][k]); same ordering, rule and outputs (no tokens); a NaN entropy is never accepted.
 */
sbd_status sbd_eb_select_entropies(sbd_ctx* ctx, int32_t batch, int32_t k,
                                   const double* entropy, const uint8_t* is_mask, double gamma,
                                   int32_t* n_accepted, int32_t* accepted_pos);

/*
 * Write n cached rows of a slot from device bf16 K, V [n_layers][n][n_kv_heads][head_dim]
 * (K after RoPE), starting at position pos0 <= cache_len; the slot's cache length
 * becomes pos0 + n and nothing stays staged.  Restores a saved cache, or installs a
 * cache produced elsewhere.  An SBD_KV_FP8_E4M3 cache stores the rounding of the values
 * described with that format.  Errors: CAPACITY if pos0 + n > max_seq_len.
 */
sbd_status sbd_kv_import(sbd_ctx* ctx, int32_t seq, int32_t pos0, int32_t n, const void* k,
                         const void* v);
/* Read rows [pos0, pos0 + n) of a slot (committed or staged) into the same layout. */
sbd_status sbd_kv_export(sbd_ctx* ctx, int32_t seq, int32_t pos0, int32_t n, void* k, void* v);

/*
 * Byte offset and size inside the workspace of a named internal buffer, for
 * inspection by tests: "x" (fp32 residual [rows][d_model]), "qkv" (fp32 projections),
 * "q" (rotated, scaled queries), "attn" (attention output), "act" (SwiGLU output), "xn"
 * (gain-scaled residual).  The last four hold bf16 pairs: [2][rows][width], the value
 * being hi + lo.  rows is the workspace's row capacity, max(max_batch * max_block,
 * prefill chunk).  Values are those of the last layer of the last forward.  INVALID_ARG
 * for an unknown name.
 */
sbd_status sbd_workspace_region(const sbd_model_config* cfg, const char* name, size_t* offset,
                                size_t* bytes);

/*
 * Which kernels run a decode-sized forward (at most 16 rows: sbd_block_forward with
 * batch * k <= 16, and prefill chunks that small).
 *   SBD_DECODE_AUTO     the library's choice (the default): SBD_DECODE_LAYERS where it
 *                       applies, otherwise one kernel per step.
 *   SBD_DECODE_FUSED    the fused forward: every layer and the LM head in one launch of one
 *                       persistent workgroup per CU.  A forward it cannot take fails with
 *                       SBD_ERR_UNSUPPORTED: it needs d_model a multiple of 128 and head_dim
 *                       64 or 128.
 *   SBD_DECODE_KERNELS  one kernel per step.
 *   SBD_DECODE_LAYERS   two launches per layer (QKV + attention + O projection; gate/up +
 *                       down), each XCD of the chip owning one KV head's share.  Needs a
 *                       device of 256 CUs in 8 XCDs, n_kv_heads 8, head_dim 128, d_model
 *                       4096, ffn_dim 12288, 14336 or 16384, batch * k <= 16 and
 *                       (n_q_heads / n_kv_heads) * k <= 64; a forward it cannot take fails
 *                       with SBD_ERR_UNSUPPORTED.
 * All give the same results up to float summation order.  Larger forwards always run one
 * kernel per step.  INVALID_ARG for another value.
 */
typedef enum {
  SBD_DECODE_AUTO = 0,
  SBD_DECODE_FUSED = 1,
  SBD_DECODE_KERNELS = 2,
  SBD_DECODE_LAYERS = 3
} sbd_decode_path;
sbd_status sbd_set_decode_path(sbd_ctx* ctx, int32_t path);
/*
 * Testing aid: the number of polls after which a dependency wait inside a launch gives up:
 * those of the per-XCD layer kernels (decode-sized forwards), and the wait of a split GEMM's
 * K slices for each other (forwards and prefill chunks of more than 16 rows).  A negative
 * value restores the default of about two million, which no correct launch comes near.  A
 * wait that gives up raises the sticky error that every later call on the context reports
 * as SBD_ERR_HIP, with a task code (layer * 16 + phase for a layer kernel, 65536 + the
 * epilogue for GEMM slices); the launch still runs to its end (on wrong data), it never
 * hangs.  With a small limit a test can take that path on purpose.  INVALID_ARG for a null
 * context.
 */
sbd_status sbd_set_wait_limit(sbd_ctx* ctx, int32_t polls);
/*
 * *fits = 1 when `path` can run a decode-sized forward of `batch` sequences of `k` rows on
 * this context's model and device, else 0 (SBD_DECODE_AUTO and SBD_DECODE_KERNELS always
 * can).  INVALID_ARG for a null pointer or an unknown path.
 */
sbd_status sbd_decode_path_fits(const sbd_ctx* ctx, int32_t path, int32_t batch, int32_t k, int32_t* fits);

/*
 * The per-XCD layer kernels and the K-split GEMMs hand partial results between workgroups
 * through one XCD's L2 and rely on workgroup i of a launch running on XCD i % 8 (256 CUs in
 * 8 XCDs).  sbd_create checks this with a probe kernel that reads each workgroup's XCC_ID
 * register (grids of 256, 1000 and 2048 workgroups); where it does not hold, the layer
 * kernels are not used (SBD_DECODE_LAYERS fails with UNSUPPORTED, AUTO takes one kernel per
 * step) and no GEMM splits K, so no hand-off between XCDs is needed.
 *   sbd_xcd_map_ok: *ok = 1 when the probe found the mapping.
 *   sbd_xcd_map_check: the decision itself on given per-workgroup XCD ids (host only):
 *   *ok = 1 iff xcc_ids[i] == i % n_xcd for every i < n.
 */
sbd_status sbd_xcd_map_ok(const sbd_ctx* ctx, int32_t* ok);
sbd_status sbd_xcd_map_check(const int32_t* xcc_ids, int32_t n, int32_t n_xcd, int32_t* ok);

/*
 * Per-kernel timing, for measurement tools.  While enabled, every kernel launch the
 * context makes is bracketed by a pair of HIP events on its stream (this adds a little
 * time between kernels).  sbd_profile_read waits for the recorded work, adds up the
 * elapsed times of all launches of one kernel kind since the previous read of that kind,
 * and returns the launch count and the total in milliseconds.
 */
typedef enum {
  SBD_KERNEL_EMBED = 0,      /* embedding gather + first RMSNorm inputs */
  SBD_KERNEL_QKV = 1,        /* QKV projection */
  SBD_KERNEL_ROPE = 2,       /* q/k norm, RoPE, KV staging */
  SBD_KERNEL_ATTENTION = 3,  /* split-KV block-hybrid attention */
  SBD_KERNEL_ATTN_MERGE = 4, /* merge of the attention splits */
  SBD_KERNEL_O_PROJ = 5,     /* output projection + residual */
  SBD_KERNEL_GATE_UP = 6,    /* gate/up projection + SwiGLU */
  SBD_KERNEL_DOWN = 7,       /* down projection + residual */
  SBD_KERNEL_LM_HEAD = 8,    /* final norm + LM head */
  SBD_KERNEL_EB_PARTIAL = 9, /* EB per-chunk softmax statistics */
  SBD_KERNEL_EB_SELECT = 10, /* EB merge, sort and select */
  SBD_KERNEL_FUSED = 11,     /* fused decode forward: all layers + LM head in one launch */
  SBD_KERNEL_LAYER_ATTN = 12,/* per-XCD layer kernel: QKV + attention + O projection */
  SBD_KERNEL_LAYER_MLP = 13, /* per-XCD layer kernel: gate/up + down projection */
  SBD_KERNEL_LAYER_FINAL = 14, /* per-XCD layer kernels: final norm inputs from the residual */
  SBD_KERNEL_COUNT = 15
} sbd_kernel;
sbd_status sbd_profile_enable(sbd_ctx* ctx, int32_t enable);
/*
 * Measurement aid: one read of `bytes` of device memory at `buf` (a positive multiple of
 * 16) by a plain streaming kernel on `stream` (NULL = the null stream), the device's
 * achievable read rate to compare the block forward's weight streams with.  sink: device
 * uint32 [64], written practically never (it keeps the loads from being dropped).  No
 * context needed; errors through sbd_last_error(NULL).
 */
sbd_status sbd_stream_probe(void* stream, const void* buf, size_t bytes, uint32_t* sink);
sbd_status sbd_profile_read(sbd_ctx* ctx, int32_t kernel, int32_t* launches, double* total_ms);

/*
 * ---------------------------------------------------------------------------------------
 * Operators of an attention layer in 8-bit formats with a scale for each block, without a
 * context: page tables of a serving batch, a paged e4m3 cache (written and read), and the
 * e4m3 product of the projections around it with the quantiser that makes its operands.
 *
 * Conventions of these calls, besides the ones at the top of this file:
 *  - stream is a hipStream_t of the current device (NULL = the null stream); every pointer
 *    in the arguments and structs is device memory of that device unless it says host.  No
 *    memory is allocated and nothing is copied to the host, so every call can be captured
 *    into a HIP graph.  Two calls may run at once if neither writes what the other uses.
 *  - Sequence lengths, tables and slots live on the device and are not checked on the host:
 *    the kernels check every page id, slot and row against the sizes given here, so wrong
 *    ones give wrong values (or rows left out), never an access outside the buffers.
 *  - Errors are reported through sbd_last_error(NULL).
 *  - Strides are in elements; a matrix or row named contiguous has none.
 */
/* Element types of 16- and 32-bit operands. */
enum { SBD_TYPE_BF16 = 0, SBD_TYPE_FP16 = 1, SBD_TYPE_FP32 = 2 };

/*
 * Page tables of `batch` sequences that share n_pages pages of page_size tokens (a power of
 * two from 16 to 256).  n_pages * page_size < 2^31 and max_pages * page_size <= 2^30.
 *   table      [batch][max_pages]: the pages of each sequence, in order of position, then -1
 *   held       [batch]: pages in each row of the table
 *   cached     [batch]: tokens of each sequence that are cached (committed); the caller adds
 *              to it, as sbd_commit does for the slots of a context
 *   free_list  [n_pages], free_count [1]: the pages that no sequence holds, first free_count
 *              entries; a permutation of all pages, and held = 0, to begin with
 */
typedef struct {
  int32_t batch, max_pages, n_pages, page_size;
  int32_t *table, *held, *cached, *free_list, *free_count;
} sbd_page_table;

/*
 * The tables of the next step, in which sequence b adds n_new[b] rows after its cached ones.
 *   n_new    [batch], 0 for a sequence that sits the step out
 *   release  [batch] or NULL: where it is not 0 the sequence has ended.  Before anything
 *            else its pages go back to the end of the free list (in order of sequence and
 *            position), its table row becomes -1, held and cached 0; n_new[b] is then the
 *            beginning of another sequence.
 *   rows     rows that the step's tensors have (at least the sum of n_new; what is over is
 *            padding)
 * A sequence needs the pages that cover cached + n_new tokens and does not hold yet.
 * Sequences are served in order: each gets all that it needs or nothing, and after the first
 * that the free list cannot serve none that needs a page is served.  The pages taken are the
 * last ones of the free list, in order.  A sequence of more than max_pages * page_size tokens
 * or with a negative length is not served and takes nothing from others.
 * Outputs: row_start [batch + 1] (rows of sequence b: row_start[b] .. row_start[b + 1], those
 * of sequences that are not served too; a negative n_new counts as 0), kv_len [batch] (cached
 * + n_new, or 0 where not served), slots [rows] (page * page_size + offset of each row's
 * token; -1 for rows of a sequence that is not served and for padding).  table, held,
 * free_list and free_count are updated; a sequence keeps the pages of rows that are not
 * committed, for the next plan.
 *   scratch  [3 * batch + 2], written before it is read
 */
sbd_status sbd_paged_plan(void* stream, const sbd_page_table* t, const int32_t* n_new, const uint8_t* release,
                          int32_t rows, int32_t* row_start, int32_t* kv_len, int32_t* slots, int32_t* scratch);

/*
 * One layer's paged cache: e4m3 codes (SBD_KV_FP8_E4M3's) with a power of two for each page
 * and KV head, keys and values apart: a value is e4m3(code) * 2^exp.
 *   k_codes  [n_pages][n_kv_heads][page_size][head_dim]
 *   v_codes  [n_pages][n_kv_heads][head_dim][page_size] (transposed: attention reads 16
 *            tokens of one dimension at a time)
 *   k_exp, v_exp  [n_pages][n_kv_heads], in [-100, 100]
 * head_dim is 64 or 128; page_size as in sbd_page_table; codes 16-byte aligned.
 */
typedef struct {
  int32_t n_pages, page_size, n_kv_heads, head_dim;
  uint8_t *k_codes, *v_codes;
  int8_t *k_exp, *v_exp;
} sbd_paged_kv;

/*
 * Write a step's keys (after RoPE) and values into their pages.
 *   k, v       SBD_TYPE_BF16 or _FP16 [rows][n_kv_heads][head_dim], rows k_stride / v_stride
 *              elements apart (a multiple of 8; base 16-byte aligned)
 *   row_start, slots  as sbd_paged_plan leaves them for this step
 * Per page and head: e is the smallest whole number in [-100, 100] with |x| <= 448 * 2^e for
 * every finite x written, and not below the page's exponent where the page keeps earlier
 * tokens of the sequence (those before the first row written); where it grows, the kept codes
 * are rounded again to the new scale.  Codes are the nearest e4m3 values, ties to even; what
 * exceeds 448 * 2^e (infinities) saturates, NaN stays NaN.  Codes behind the last row written
 * are left as they were.  Rows with a slot outside the cache, and padding, are left out.  No
 * two sequences of a step may write into one page.
 */
sbd_status sbd_paged_append(void* stream, const sbd_paged_kv* c, int32_t dtype, int32_t batch, int32_t rows,
                            const int32_t* row_start, const int32_t* slots, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride);

/*
 * Attention of a step's rows over the paged cache (which holds the step's own rows already).
 *   q, out     SBD_TYPE_BF16 or _FP16 [rows][n_q_heads][head_dim], rows q_stride / out_stride
 *              elements apart (a multiple of 8; bases 16-byte aligned).  n_q_heads is a
 *              multiple of n_kv_heads; query head h reads KV head h / (n_q_heads / n_kv_heads).
 *   row_start, kv_len  as sbd_paged_plan leaves them
 *   table      [batch][max_pages]; a position whose entry is outside [0, n_pages) is seen by
 *              no row
 *   n_causal   [batch] or NULL.  Row j of sequence b is the token at position
 *              kv_len[b] - n_new[b] + j and sees the keys up to itself if j < n_causal[b],
 *              else all kv_len[b] keys (the block-hybrid mask of sbd_block_forward).  NULL:
 *              every row is causal.
 *   scale      of the products q.k, finite
 *   max_kv     what the longest kv_len is about, in [1, max_pages * page_size]: it decides
 *              into how many parts keys are split at most, not the result beyond summation order
 * out = sum_i softmax_i(scale * q.k_i) v_i over the keys a row sees; a row that sees no key
 * (its sequence was not served) gets zeros.  Sums and softmax statistics are fp32; a key
 * whose weight is below 2^-36 of the row's largest may count as zero.  Values of keys that a
 * row does not see never reach it, NaN included.  Rows behind row_start[batch] are left as
 * they were.
 *   workspace  sbd_paged_attention_workspace() bytes, 16-byte aligned (NULL if that is 0),
 *              used by this call alone until it has ended
 */
sbd_status sbd_paged_attention_workspace(const sbd_paged_kv* c, int32_t batch, int32_t rows, int32_t n_q_heads,
                                         int32_t max_kv, size_t* bytes);
sbd_status sbd_paged_attention(void* stream, const sbd_paged_kv* c, int32_t dtype, int32_t batch, int32_t rows,
                               int32_t n_q_heads, const int32_t* row_start, const int32_t* kv_len,
                               const int32_t* table, int32_t max_pages, const int32_t* n_causal, float scale,
                               int32_t max_kv, const void* q, int64_t q_stride, void* out, int64_t out_stride,
                               void* workspace, size_t workspace_bytes);

/*
 * e4m3 codes of a matrix with a power of two for each block of block_rows x 128 elements
 * (block_rows 1: activations; 128: weights): scale = 2^e, e the smallest whole number in
 * [-100, 100] with |x| <= 448 * 2^e for every finite x of the block; code = the e4m3 value
 * nearest to x / scale (ties to even, saturating, NaN stays NaN).
 *   x       SBD_TYPE_* [rows][cols], rows x_stride elements apart; cols a multiple of 16, rows
 *           16-byte aligned, rows * cols at most 2^36
 *   codes   [rows][cols], contiguous, 16-byte aligned
 *   scales  float, block_rows 1: [ceil(cols / 128)][rows] (the scales of one block of columns
 *           lie together); block_rows 128: [ceil(rows / 128)][ceil(cols / 128)]
 */
sbd_status sbd_scaled_quantize(void* stream, int32_t dtype, int32_t rows, int32_t cols, const void* x,
                               int64_t x_stride, int32_t block_rows, uint8_t* codes, float* scales);

/*
 * Product of e4m3 matrices with a scale for each block of 128 along K:
 *   out[m][n] = sum_c a_scale[c][m] * b_scale[n / 128][c] * sum_{k in [128 c, 128 c + 128)} a[m][k] * b[n][k]
 *   a        e4m3 codes [m][k], rows a_stride elements apart (a multiple of 16, at most 2^22;
 *            16-byte aligned)
 *   a_scale  float [ceil(k / 128)][m] (any values)
 *   b        e4m3 codes [n][k], contiguous, 16-byte aligned (the weights, [out][in])
 *   b_scale  float [ceil(n / 128)][ceil(k / 128)] (any values)
 *   k        a multiple of 16, at most 2^22; m * n at most 2^36
 *   out      SBD_TYPE_* [m][n], rows out_stride elements apart, aligned to its type
 * The sums are fp32 and out is rounded once.  For 16-bit outputs the e4m3 matrix instruction
 * makes the products: of each eight neighbours along k it adds what is at least 2^-13 of the
 * largest product's power of two (each is cut off there), so that the sum of a group may be
 * off by 2^-10 of its largest product; fp32 outputs have exact products.
 *   workspace  sbd_scaled_matmul_workspace() bytes, 16-byte aligned (NULL if that is 0), used
 *              by this call alone until it has ended
 */
sbd_status sbd_scaled_matmul_workspace(int32_t m, int32_t n, int32_t k, size_t* bytes);
sbd_status sbd_scaled_matmul(void* stream, int32_t m, int32_t n, int32_t k, const uint8_t* a, int64_t a_stride,
                             const float* a_scale, const uint8_t* b, const float* b_scale, int32_t out_type,
                             void* out, int64_t out_stride, void* workspace, size_t workspace_bytes);

const char* sbd_status_string(sbd_status s);
/* Reason for the last failed call on ctx; ctx == NULL gives the calling thread's last
 * context-less failure (e.g. of sbd_create). */
const char* sbd_last_error(const sbd_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* SBD_H_ */
