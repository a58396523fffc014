/*
 * axon.h -- C ABI of the GB300 (sm_103a) Llama-family decoder forward.
 *
 * The operation behind these calls is the forward pass that the Axon paper
 * (arxiv 2608.19889) compiles to its backends: a model definition plus a
 * safetensors checkpoint go in (Fig. 1; Sec. "The Axon Compiler", Phase 3:
 * backends implement `forward` and `generate` with static-cache scaffolding),
 * logits and greedy next tokens come out (Sec. "Results", Measures). The
 * per-layer math is the pre-norm block of Sec. "The Axon Language" (RMSNorm,
 * grouped-query causal attention with rotary positions and a KV cache,
 * residual add, SwiGLU MLP) built from the library of Sec. "Built-In
 * Libraries"; the model skeleton follows the appendix causal_lm listing
 * (embedding, layer loop threading the cache, final norm, tied or untied
 * LM head).
 *
 * Conventions for every call
 *   - Return value: AXON_OK (0) or one AXON_ERR_* code. Nothing aborts or
 *     throws across the ABI. axon_status_string() names a code.
 *   - Pointers named d_* are DEVICE pointers (CUDA global memory of the
 *     device current when the model was created). The caller owns them.
 *   - Work is enqueued asynchronously on `stream` (a cudaStream_t; NULL =
 *     the legacy default stream). Argument errors are reported
 *     synchronously; device-side range checks (token ids, block-table
 *     entries, positions) set a device error word that
 *     axon_check_device() reads, and the offending access is skipped.
 *   - Token ids, context lengths and block tables are int32.
 *   - Floating point: weights bf16 (or fp32 widened in AXON_FP32_DEBUG),
 *     fp32 accumulation everywhere, fp32 residual stream and logits.
 */
#ifndef AXON_H
#define AXON_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes. */
enum {
  AXON_OK = 0,
  AXON_ERR_INVALID_ARG = 1,    /* null pointer, bad enum, B or S out of range */
  AXON_ERR_SHAPE_MISMATCH = 2, /* a weight's shape disagrees with the config */
  AXON_ERR_MISSING_WEIGHT = 3, /* a required weight name is absent */
  AXON_ERR_UNSUPPORTED = 4,    /* config outside what the kernels implement */
  AXON_ERR_OOM = 5,            /* device allocation failed */
  AXON_ERR_CUDA = 6,           /* a CUDA runtime call failed */
  AXON_ERR_TIMEOUT = 7,        /* a bounded device wait expired */
  AXON_ERR_DEVICE_CHECK = 8    /* a device-side range check fired */
};

/* KV cache layouts (Sec. Built-In Libraries: a static, preallocated cache
 * overlay; vLLM's PagedAttention manager, Sec. Related Work). */
enum { AXON_KV_CONTIGUOUS = 0, AXON_KV_PAGED = 1 };

/* Arithmetic mode (Sec. Results: bf16 primary, fp32 fallback):
 *   AXON_BF16        bf16 weights, bf16 GEMM operands and KV cache, fp32
 *                    accumulation, fp32 residual stream and logits;
 *   AXON_FP32_DEBUG  everything fp32 (CUDA-core GEMMs), for checking;
 *   AXON_FP16        the bf16 checkpoint converted exactly to fp16 (every
 *                    bf16 value of magnitude 2^-14 .. 65504 is an fp16
 *                    value), fp16 GEMM operands and KV cache, fp32
 *                    accumulation and residual: same speed as AXON_BF16, 8x
 *                    smaller operand rounding (10- vs 7-bit mantissa).
 *                    Operands saturate at +-65504; a weight beyond that
 *                    range makes axon_model_create return
 *                    AXON_ERR_UNSUPPORTED. */
enum { AXON_BF16 = 0, AXON_FP32_DEBUG = 1, AXON_FP16 = 2 };

/* Gate activation of the gated MLP (Activations built-ins, Sec. Built-In
 * Libraries): silu (SwiGLU, Llama / Qwen / Mistral) or the tanh form of
 * GELU, gelu_new of the appendix GPT-2 listing (gated GELU). */
enum { AXON_ACT_SILU = 0, AXON_ACT_GELU_TANH = 1 };

/* Element types of weight tensors handed to axon_model_create. */
enum { AXON_DTYPE_BF16 = 0, AXON_DTYPE_F32 = 1 };

/* Which positions of a prefill get logits written. */
enum { AXON_LOGITS_LAST = 0, AXON_LOGITS_ALL = 1 };

/* Model configuration: HF config.json equivalents (the appendix causal_lm
 * listing reads hidden size, layer and head counts and vocabulary size
 * through `Config.dim @@key`), plus capacity and layout fields. The struct
 * carries neither a size nor a version and has grown at its end (sink_tokens is
 * the newest field): compile callers against the header of the library that
 * they load, and zero the struct before filling it. */
typedef struct axon_config {
  int32_t num_hidden_layers;   /* L */
  int32_t hidden_size;         /* D, multiple of 64 */
  int32_t num_attention_heads; /* H, multiple of num_key_value_heads */
  int32_t num_key_value_heads; /* G */
  int32_t head_dim;            /* d: 64 or 128 */
  int32_t intermediate_size;   /* F, multiple of 64 */
  int32_t vocab_size;          /* V */
  int32_t tie_word_embeddings; /* 1: LM head = embedding matrix */
  int32_t attention_bias;      /* 1: q, k, v projections carry biases */
  float rope_theta;            /* rotary base */
  float rms_norm_eps;          /* RMSNorm epsilon */
  int32_t max_batch;           /* sequences (contiguous cache slots) */
  int32_t max_context;         /* tokens per sequence, multiple of 16 */
  int32_t max_prefill_tokens;  /* largest B*S per axon_prefill; 0 = max_batch*max_context */
  int32_t kv_layout;           /* AXON_KV_CONTIGUOUS or AXON_KV_PAGED */
  int32_t kv_block_size;       /* tokens per block: must be 16 */
  int32_t kv_num_blocks;       /* paged pool size in blocks (ignored if contiguous) */
  int32_t precision;           /* AXON_BF16, AXON_FP16 or AXON_FP32_DEBUG */
  int32_t sliding_window;      /* W > 0: a query at position p attends only to
                                  keys p-W+1 .. p (the `window=` argument of
                                  causal_mask_for_input, appendix GPT-2
                                  listing); 0: full causal attention */
  /* RoPE frequency scaling of Llama-3.1-family checkpoints (HF
   * rope_scaling {"rope_type": "llama3", ...}); rope_scaling_factor 0 =
   * none. A rotary frequency f with wavelength w = 2 pi / f is kept when
   * w < original / high_freq_factor, divided by the factor when
   * w > original / low_freq_factor, and blended linearly in
   * t = (original / w - low) / (high - low) between: (1-t) f / factor + t f. */
  float rope_scaling_factor;
  float rope_low_freq_factor;
  float rope_high_freq_factor;
  int32_t rope_original_max_position;
  int32_t hidden_act;          /* AXON_ACT_SILU or AXON_ACT_GELU_TANH: u = act(h W_gate^T) * (h W_up^T) */
  int32_t qk_norm;             /* 1: each head's q and k (after the projection and its bias) go
                                  through RMSNorm over their head_dim values, with rms_norm_eps and
                                  the gains model.layers.{i}.self_attn.{q,k}_norm.weight [head_dim],
                                  before RoPE (Qwen3-family layers); 0: none. Decode then always
                                  takes the launch chain. */
  /* Mixture of experts (the MoE built-ins: softmax top-k router, grouped
   * experts; DeepSeek-MoE layout). n_routed_experts E > 0: layers from
   * first_k_dense_replace on replace the MLP by
   *   p = softmax(h W_router^T) over the E experts (fp32 router),
   *   the num_experts_per_tok experts with the largest p (lowest index on
   *   ties), weights p (divided by their sum when norm_topk_prob),
   *   y = sum_j w_j * SwiGLU-MLP_j(h) + SwiGLU-MLP_shared(h),
   * with experts of width moe_intermediate_size and, when
   * n_shared_experts > 0, one shared MLP of width n_shared_experts *
   * moe_intermediate_size. E <= 256, 1 <= num_experts_per_tok <= min(8, E),
   * 16-bit modes only; decode takes the launch chain. */
  int32_t n_routed_experts;
  int32_t num_experts_per_tok;
  int32_t moe_intermediate_size;
  int32_t n_shared_experts;
  int32_t first_k_dense_replace;
  int32_t norm_topk_prob;
  int32_t sink_tokens;         /* with a sliding window: the first sink_tokens positions stay visible to
                                  every query (0: none; without a window it must be 0). 16-bit modes
                                  only; decode takes the launch chain. Cache blocks that neither the
                                  window nor the sinks reach are not read (axon_kv_release). */
} axon_config;

/* One named checkpoint tensor, HF Llama naming and [out, in] matrices, as a
 * safetensors file stores them (Fig. 1; weights looked up by flat dotted
 * path, appendix "Python Overhead"):
 *   model.embed_tokens.weight                       [V, D]
 *   model.layers.{i}.input_layernorm.weight         [D]
 *   model.layers.{i}.self_attn.{q,k,v}_proj.weight  [H*d | G*d | G*d, D]
 *   model.layers.{i}.self_attn.{q,k,v}_proj.bias    (if attention_bias)
 *   model.layers.{i}.self_attn.o_proj.weight        [D, H*d]
 *   model.layers.{i}.post_attention_layernorm.weight[D]
 *   model.layers.{i}.mlp.{gate,up}_proj.weight      [F, D]
 *   model.layers.{i}.mlp.down_proj.weight           [D, F]
 *   model.layers.{i}.self_attn.{q,k}_norm.weight    [d] (if qk_norm)
 *   mixture-of-experts layers (i >= first_k_dense_replace when
 *   n_routed_experts > 0) carry instead of mlp.{gate,up,down}_proj:
 *   model.layers.{i}.mlp.gate.weight                [E, D] (router)
 *   model.layers.{i}.mlp.experts.{e}.{gate,up}_proj.weight [Fe, D]
 *   model.layers.{i}.mlp.experts.{e}.down_proj.weight      [D, Fe]
 *   model.layers.{i}.mlp.shared_experts.{gate,up}_proj.weight [Fs, D]
 *   model.layers.{i}.mlp.shared_experts.down_proj.weight   [D, Fs]
 *     (Fe = moe_intermediate_size, Fs = n_shared_experts * Fe; shared only
 *     when n_shared_experts > 0)
 *   model.norm.weight                               [D]
 *   lm_head.weight                                  [V, D] (absent if tied)
 * `data` may be a host or a device pointer (unified addressing); it is
 * only read during axon_model_create. Row-major, contiguous. */
typedef struct axon_tensor {
  const char* name;
  const void* data;
  int32_t dtype; /* AXON_DTYPE_BF16 or AXON_DTYPE_F32 */
  int32_t ndim;  /* 1 or 2 */
  int64_t shape[4];
} axon_tensor;

typedef struct axon_model axon_model;

/* Build a model: validate the config against the named weights (symbolic
 * dimensions, Sec. The Axon Language, Types), allocate and repack weights
 * into the kernels' layout (fused QKV, interleaved gate/up), allocate the KV
 * cache and workspace. The weight table is copied; the caller may free it
 * on return. Work is done on `stream` and synchronised before returning.
 * *out receives the model, or NULL on error. */
int axon_model_create(const axon_config* cfg, const axon_tensor* weights, int32_t n_weights,
                      void* stream, axon_model** out);

/* Prompt pass (Positions.position_ids with past_length 0; Cache.update of
 * every prompt token; Sec. Built-In Libraries).
 *   d_ids          [B, S] token ids.
 *   B              1 .. max_batch; sequence b uses contiguous slot b, or the
 *                  blocks named by row b of d_block_table.
 *   S              1 .. max_context, B*S <= max_prefill_tokens.
 *   d_block_table  paged layout: [B, ceil(max_context/16)] pool block ids,
 *                  row b for sequence b (entries past the prompt unused);
 *                  must be NULL for the contiguous layout.
 *   logits_mode    AXON_LOGITS_LAST: d_logits is [B, V], the last position;
 *                  AXON_LOGITS_ALL: d_logits is [B, S, V].
 *   d_logits       fp32 output, or NULL to skip storing logits.
 *   d_next         [B] greedy next token (argmax of the last position's
 *                  logits, lowest index on ties), or NULL.
 * Previous contents of the used cache slots are overwritten. */
int axon_prefill(axon_model* m, const int32_t* d_ids, int32_t B, int32_t S,
                 const int32_t* d_block_table, int32_t logits_mode, float* d_logits,
                 int32_t* d_next, void* stream);

/* Variable-length batch: B sequences each append one chunk of new tokens
 * after the tokens they already hold in the cache -- a whole prompt, the
 * next piece of a long prompt (chunked prefill), or a single decode token
 * -- packed row after row into one forward pass (Positions.position_ids
 * with a per-sequence past_length and Cache.update, Sec. Built-In
 * Libraries; the continuous batching of vLLM's PagedAttention manager,
 * Sec. Related Work). Every chunk attends causally to its own sequence's
 * cached tokens and to the earlier tokens of the chunk.
 *   d_ids           [T] token ids, sequence b's chunk at rows
 *                   cu_seqlens[b] .. cu_seqlens[b+1]-1.
 *   B               1 .. max_batch; sequence b uses contiguous slot b, or
 *                   the blocks named by row b of d_block_table.
 *   T               total new tokens, B .. max_prefill_tokens.
 *   d_cu_seqlens    [B+1] row offsets: cu[0] = 0, cu[B] = T, every chunk
 *                   1 .. max_chunk tokens long.
 *   d_context_lens  [B] IN/OUT: tokens already cached for sequence b (0 for
 *                   a new prompt); chunk token i takes position
 *                   context_lens[b] + i, which must stay below
 *                   max_context. The call adds each chunk's length (in
 *                   stream order, after all reads), so the next call --
 *                   another chunk or axon_decode_step -- can follow
 *                   without host work.
 *   max_chunk       host bound on the longest chunk, 1 .. min(T,
 *                   max_context); it sizes the attention grid.
 *   d_block_table   paged layout: [B, ceil(max_context/16)], else NULL.
 *   logits_mode     AXON_LOGITS_LAST: d_logits is [B, V], the last token of
 *                   each chunk; AXON_LOGITS_ALL: d_logits is [T, V].
 *   d_logits        fp32 output, or NULL.
 *   d_next          [B] greedy next token after each chunk's last token
 *                   (lowest index on ties), or NULL.
 * Offsets and lengths are read on the device: inconsistent ones (cu not
 * starting at 0, not ending at T, a chunk outside 1 .. max_chunk) or
 * positions past max_context set the device error word
 * (AXON_ERR_DEVICE_CHECK from axon_check_device) and the rows they affect
 * are skipped. Cache slots at the chunk's positions are overwritten. */
int axon_prefill_varlen(axon_model* m, const int32_t* d_ids, int32_t B, int32_t T, const int32_t* d_cu_seqlens,
                        int32_t* d_context_lens, int32_t max_chunk, const int32_t* d_block_table,
                        int32_t logits_mode, float* d_logits, int32_t* d_next, void* stream);

/* One KV-cached greedy decode step for B sequences (generate loop, Sec.
 * Results; Cache.append in the appendix causal_lm listing).
 *   d_tokens        [B] the newest token of each sequence.
 *   d_context_lens  [B] IN/OUT: tokens already cached for sequence b; the
 *                   new token takes position context_lens[b]. The step adds
 *                   1 to every entry (in stream order, after all reads), so
 *                   consecutive steps can be replayed without host work.
 *   d_block_table   paged layout: [B, ceil(max_context/16)], else NULL.
 *   d_logits        [B, V] fp32 output, or NULL.
 *   d_next          [B] greedy next token; may alias d_tokens.
 * With B <= 8 (16-bit modes, head_dim 64 or 128) the whole step is one
 * cooperative launch with one CTA per SM (the persistent decode step); if
 * the device cannot hold that grid co-resident, or with AXON_NO_PERSIST=1
 * set when the model was created, the step is a chain of 5L+3 kernels,
 * recorded once per (B, pointer set) into a CUDA graph and replayed
 * afterwards (AXON_NO_GRAPH=1: launched directly). Both paths compute the
 * same operations; their fp32 summation orders differ. */
int axon_decode_step(axon_model* m, const int32_t* d_tokens, int32_t B, int32_t* d_context_lens,
                     const int32_t* d_block_table, float* d_logits, int32_t* d_next, void* stream);

/* Forget cached sequences: zero the KV cache and clear the device error
 * word. Synchronous. */
int axon_reset(axon_model* m);

/* Synchronise `stream` and read the device error word. Returns AXON_OK,
 * AXON_ERR_DEVICE_CHECK (a range check fired) or AXON_ERR_TIMEOUT (a
 * bounded wait expired). *bits (optional) receives the raw word; the word
 * is cleared. */
int axon_check_device(axon_model* m, void* stream, int32_t* bits);

/* Read-only view of the KV pools for inspection (tests check cache
 * placement through it). Layout of either pool: [L][num_blocks][G][16][d],
 * element type bf16 (fp32 in AXON_FP32_DEBUG). In the contiguous layout,
 * sequence b's logical block j is pool block b*blocks_per_seq + j. */
typedef struct axon_kv_view {
  void* k_pool;
  void* v_pool;
  int64_t num_blocks;
  int32_t blocks_per_seq;
  int32_t block_size;
  int32_t elem_bytes;
} axon_kv_view;
int axon_kv_view_get(const axon_model* m, axon_kv_view* out);

/* Per-kernel timing of one pass (tracing hook; the paper profiles its
 * generate loop's GPU kernels, appendix "Python Overhead", Table 5).
 * The pass runs exactly as axon_prefill / axon_decode_step would (same
 * kernels, same side effects on the cache and, for decode, on
 * d_context_lens), but launched one kernel at a time with a CUDA event pair
 * around each launch and no CUDA graph or programmatic overlap, then
 * synchronised. Entries aggregate launches of one kind:
 *   name       kernel kind ("decode_gateup", "prefill_qkv", ...)
 *   launches   number of launches in the pass
 *   total_ms   summed event time of those launches
 *   bytes      algorithmic HBM bytes of those launches (weights once, KV
 *              cache reads/writes, activations in/out)
 *   flops      algorithmic floating-point operations
 * `out` receives at most max_out entries (16 suffice); *n_out their count.
 * Prefill logits are not stored (LAST mode, next tokens only). */
typedef struct axon_kernel_time {
  char name[32];
  int32_t launches;
  float total_ms;
  double bytes;
  double flops;
} axon_kernel_time;
int axon_profile_decode_step(axon_model* m, const int32_t* d_tokens, int32_t B, int32_t* d_context_lens,
                             const int32_t* d_block_table, int32_t* d_next, void* stream, axon_kernel_time* out,
                             int32_t max_out, int32_t* n_out);
int axon_profile_prefill(axon_model* m, const int32_t* d_ids, int32_t B, int32_t S, const int32_t* d_block_table,
                         int32_t* d_next, void* stream, axon_kernel_time* out, int32_t max_out, int32_t* n_out);

/* Decode step that allocates nothing (no counterpart in the paper; a
 * deployment affordance of this library). Same arguments, results and
 * side effects as axon_decode_step, for callers that must not allocate on
 * the call path -- for example a serving loop running while another
 * component owns the device memory pool, or a caller whose allocator is
 * locked after start-up: axon_decode_step instantiates a CUDA graph the
 * first time it meets a new (B, pointer set), and instantiation allocates.
 * This entry point instead launches the step's kernels directly, and the
 * split-KV attention takes its merge scratch from a fixed, library-owned
 * device array (256 merge slots, about 2.1 MB, resident on every device
 * that loads the library until the process exits) instead of from memory
 * allocated per call. It calls no cudaMalloc, cudaFree or graph
 * instantiation.
 *   Limits: B * num_key_value_heads <= 256 (not with sink_tokens, whose
 *   attention merges in the model's own memory) and head_dim <= 128, else
 *   AXON_ERR_UNSUPPORTED; the 16-bit modes AXON_BF16 and AXON_FP16 only
 *   (AXON_ERR_UNSUPPORTED in AXON_FP32_DEBUG). The attention keeps at most
 *   256 / (B * num_key_value_heads) key splits per sequence and kv head.
 *   First call on a device (and the first after the device's context was
 *   torn down, e.g. by cudaDeviceReset): resolves the array's device address
 *   in the current context, with that device current -- make that first
 *   call before any stream capture.
 *   Every call shares the one array and clears the parts that must start
 *   at zero: calls that overlap on the GPU (different streams, or several
 *   models at once) race on it and must be serialised by the caller. (With
 *   sink_tokens that holds for the calls of one model.)
 * The key-split count may differ from axon_decode_step's, so logits can
 * differ from it by floating-point rounding of the merge. */
int axon_decode_step_noalloc(axon_model* m, const int32_t* d_tokens, int32_t B, int32_t* d_context_lens,
                             const int32_t* d_block_table, float* d_logits, int32_t* d_next, void* stream);

/* Inspection hook for mixture-of-experts models (the routing is decided on
 * the device; tests compare it with the oracle's). With d_experts non-NULL,
 * every later prefill or decode pass writes, for each MoE layer l and each
 * of its first `rows` token rows t (in the pass's row order: b * S + s for
 * axon_prefill, b for axon_decode_step, packed rows for
 * axon_prefill_varlen), the chosen experts in rank order into
 * d_experts[(l * rows + t) * num_experts_per_tok + j] (int32, device
 * memory owned by the caller, L * rows * num_experts_per_tok entries;
 * rows of dense layers are not written). NULL turns recording off.
 * AXON_ERR_UNSUPPORTED for models without experts. Decode graphs recorded
 * before the call are dropped. */
int axon_moe_routing_record(axon_model* m, int32_t* d_experts, int32_t rows);

/* ---------------------------------------------------------------------
 * Operators on a paged key/value cache, without a model pass: attention that
 * reads the cache, and the management of its blocks (vLLM's PagedAttention
 * manager, Sec. Related Work; causal masks with a window, appendix GPT-2
 * listing). All of them only enqueue work on `stream`, allocate nothing and
 * keep nothing: every buffer is the caller's and every pointer except the
 * three descriptor structs is a device pointer.
 *
 * Errors. What the host can see is refused at once (AXON_ERR_INVALID_ARG,
 * AXON_ERR_UNSUPPORTED). What only the device can see -- a block number, a
 * length or a row out of range -- sets a bit of the caller's error word
 * *d_err (one int32, zeroed by the caller; NULL: not reported) and the access
 * is skipped; axon_check_error reads and clears the word. An attention row that would
 * have read a block out of range then holds finite numbers of no meaning (the one-token
 * form leaves its keys out, the chunk form takes them for zeros); other rows are right. With shared
 * prefixes an entry out of range in the blocks in common, where the first live row's are read for
 * all, spoils every row of its group (taken for zeros there, left out elsewhere).
 *
 * Workspaces are device memory, 16-byte aligned, of at least the size that
 * the matching query returns. The attention's must be zero before its first
 * use and every call leaves it fit for the next one, of any shape and batch that
 * it is large enough for; the block operators' may hold anything. Calls that may
 * overlap (different streams) need their own. The first attention call on a device
 * sets its kernels' limits: make it before a stream capture. */

/* The pools of all layers: [num_layers][num_blocks][num_kv_heads][16][head_dim],
 * keys after RoPE, 16-byte aligned. Block numbers are common to all layers. */
typedef struct axon_kv_cache {
  void* k_pool;
  void* v_pool;
  int32_t num_layers;
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t block_size; /* 16 */
  int32_t head_dim;   /* 64 or 128 */
  int32_t precision;  /* element type: AXON_BF16, AXON_FP16, or AXON_FP32_DEBUG (block operators only) */
} axon_kv_cache;

/* The cache of a model, either layout (the pools stay the model's). */
int axon_kv_cache_get(const axon_model* m, axon_kv_cache* out);

/* Who holds which block. A block is free when its count is 0; the counts
 * are the number of table entries that name it. */
typedef struct axon_kv_seqs {
  int32_t* block_table;   /* [max_seqs][blocks_per_seq] block numbers, -1: none */
  int32_t* context_lens;  /* [max_seqs] tokens in the cache, as axon_decode_step advances them */
  int32_t* refs;          /* [num_blocks] */
  int32_t max_seqs;       /* at most 8192; times blocks_per_seq below 2^31 */
  int32_t blocks_per_seq;
} axon_kv_seqs;

/* Attention of one new token per row, split over the cache's length and
 * joined. Row b's query stands at position p = context_lens[b], whose key and
 * value are in the cache already, as everything before them; key t is visible
 * when t <= p and (window = 0 or t > p - window or t < sinks):
 *   o = sum_t softmax_t(scale q.k_t) v_t,   lse = log sum_t exp(scale q.k_t).
 *   d_q, d_out      [B][num_heads][head_dim] of the cache's type, last
 *                   dimension dense, the others with strides in elements
 *                   (multiples of 8, at least head_dim; 16-byte aligned
 *                   base; a row's heads may not overlap in d_out).
 *   B               1 .. 2048 (and B * num_kv_heads * the blocks that a row can see
 *                   below 2^31)
 *   num_heads       a multiple of num_kv_heads, at most 16 times as many;
 *                   head h reads kv head h / (num_heads / num_kv_heads)
 *   d_context_lens  [B]; negative: an idle row, o = 0 and lse = -infinity
 *   d_block_table   [B][blocks_per_seq], or NULL: row b holds blocks
 *                   b * blocks_per_seq onward
 *   window, sinks   0: none; sinks only count under a window. Blocks that
 *                   the mask hides are not looked at (-1 will do).
 *   scale           0: 1 / sqrt(head_dim)
 *   d_lse           [B][num_heads] fp32, or NULL
 * P enters the product with V in two 16-bit terms; sums, maxima and lse are
 * fp32. The result does not depend on timing. Cache slots that the mask hides
 * from a row never reach its output, whatever they hold; a visible value that is
 * infinite or not a number leaves its dim of the output not finite. */
int axon_attn_decode(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride,
                     int64_t q_head_stride, int32_t B, int32_t num_heads, const int32_t* d_context_lens,
                     const int32_t* d_block_table, int32_t blocks_per_seq, int32_t window, int32_t sinks, float scale,
                     void* d_out, int64_t out_row_stride, int64_t out_head_stride, float* d_lse, void* d_workspace,
                     int64_t workspace_bytes, int32_t* d_err, void* stream);
int axon_attn_decode_workspace(const axon_kv_cache* cache, int32_t num_heads, int32_t B, int64_t* bytes);

/* axon_attn_decode for rows that come in groups whose first blocks are the same: samples of one prompt or beams
 * (axon_kv_fork), requests with one system prompt. The blocks that all live rows of a group see whole are read once for
 * the group, the rest row by row; the result is axon_attn_decode's but for the order of its sums.
 *   d_group_offsets [num_groups + 1], ascending: group n is rows group_offsets[n] .. group_offsets[n+1]-1 (a group may be
 *                   empty); rows of no group share nothing. Inconsistent offsets are reported and nothing is shared
 *   d_prefix_lens   [num_groups] tokens whose whole blocks (prefix_lens / 16, rounded down) the tables of the
 *                   group's live rows name alike, in all their rows: the first live row's entries are read for all, which the call
 *                   does not check. It may be longer than a row's context; negative: reported, nothing is shared
 *   num_groups      1 .. 1024
 *   d_block_table   [B][blocks_per_seq]; entries of shared blocks that only idle rows (context_lens negative) hold may be anything
 * The rest as in axon_attn_decode, the workspace among it: one of axon_attn_shared_workspace's size serves axon_attn_decode
 * of the same heads and cache too. num_blocks * num_kv_heads * 16 stays below 2^31.
 * Where reading shared blocks once would spare less than 128 MB of reads the rows read them for themselves, which is faster.
 * The environment variable AXON_SHARED_MIN_BYTES (digits; anything else is ignored) sets another limit: it is read with every
 * call, and a captured call keeps what it was then. */
int axon_attn_shared(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                     int32_t B, int32_t num_heads, const int32_t* d_context_lens, const int32_t* d_block_table,
                     int32_t blocks_per_seq, const int32_t* d_group_offsets, const int32_t* d_prefix_lens, int32_t num_groups,
                     int32_t window, int32_t sinks, float scale, void* d_out, int64_t out_row_stride, int64_t out_head_stride,
                     float* d_lse, void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream);
int axon_attn_shared_workspace(const axon_kv_cache* cache, int32_t num_heads, int32_t B, int64_t* bytes);

/* axon_attn_decode for chunks of tokens, packed row after row as in
 * axon_prefill_varlen: chunk b is rows cu_seqlens[b] .. cu_seqlens[b+1]-1 of
 * d_q and d_out (T rows in all; a chunk may be empty), its row i stands at
 * position context_lens[b] + i, and the chunk's keys and values are in the
 * cache already. max_chunk bounds the longest chunk. context_lens is not
 * advanced. num_blocks * num_kv_heads * 16 stays below 2^31. Slots past a chunk's
 * last token never reach an output, whatever they hold. Tokens that the mask hides
 * from some rows only (later ones of the chunk, ones before a window in a block that it
 * reaches) have to be finite: the products add zero times their values. P has two
 * 16-bit terms here too. */
int axon_attn_prefill(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride,
                      int64_t q_head_stride, int32_t B, int32_t T, int32_t num_heads, const int32_t* d_cu_seqlens,
                      const int32_t* d_context_lens, int32_t max_chunk, const int32_t* d_block_table,
                      int32_t blocks_per_seq, int32_t window, int32_t sinks, float scale, void* d_out,
                      int64_t out_row_stride, int64_t out_head_stride, int32_t* d_err, void* stream);

/* Rotary table of the first `rotary_dim` dims of a head (a multiple of 16, at most 128): d_rope
 * [positions][rotary_dim / 2][2] fp32, (cos a, sin a) of a = position * f_j,
 * f_j = theta^(-2j / rotary_dim), the angle in 64 bits. factor > 0: the frequency scaling of
 * axon_config (low and high as rope_low_freq_factor and rope_high_freq_factor), else f_j as they are. d_rope
 * is 16-byte aligned. A table made in any other way serves as well. */
int axon_rope_table(float* d_rope, int32_t positions, int32_t rotary_dim, float theta, float factor, float low, float high,
                    int32_t original_positions, void* stream);

/* Which dims of the rotated part make a pair: (j, j + rotary_dim / 2), or (2j, 2j + 1). */
enum { AXON_ROPE_HALF = 0, AXON_ROPE_INTERLEAVED = 1 };

/* New tokens into a layer of the cache: keys rotated to their positions and values go to the
 * tokens' slots, rotated queries to d_q_out, for axon_attn_decode, axon_attn_shared or axon_attn_prefill with the same
 * lengths afterwards. A pair (x, y) becomes (x cos a - y sin a, y cos a + x sin a) in fp32, rounded once (fp16:
 * saturated at 65504); what is not rotated is copied bit for bit.
 *   d_q, d_q_out    [T][num_heads][head_dim] of the cache's type, strides as in axon_attn_decode; both NULL: keys and
 *                   values only (num_heads 0). d_q_out may be d_q with the same strides; else they may not overlap.
 *   d_k, d_v        [T][num_kv_heads][head_dim], likewise (parts of one projection's output, for instance)
 *   d_cu_seqlens    [B + 1]: chunk b is rows cu_seqlens[b] .. cu_seqlens[b+1]-1 (a chunk may be empty), its row i stands
 *                   at position context_lens[b] + i. NULL: one token per row, T = B, at position context_lens[b];
 *                   negative: an idle row, which is left out
 *   d_context_lens  [B], not advanced
 *   d_block_table   [B][blocks_per_seq], or NULL: row b holds blocks b * blocks_per_seq onward
 *   d_rope          [rope_positions][rotary_dim / 2][2] as axon_rope_table makes it; NULL with rotary_dim 0: no rotation
 *   rotary_dim      a multiple of 16, at most head_dim
 * All caches, AXON_FP32_DEBUG too. Left out are idle rows, rows beyond the table of blocks or the rotary table, and, with
 * offsets, whole chunks: one takes part with all its tokens or, if its last one lies beyond either table, its context
 * length is negative (reported, since an empty chunk is the idle one) or its offsets are inconsistent, with none. What is
 * left out leaves d_q_out and the cache as they are; a block out of range keeps the
 * token's key and value out, its query is written. Two tokens may not go to one slot: fork before rows part. */
int axon_kv_append(const axon_kv_cache* cache, int32_t layer, const void* d_q, int64_t q_row_stride, int64_t q_head_stride,
                   const void* d_k, int64_t k_row_stride, int64_t k_head_stride, const void* d_v, int64_t v_row_stride,
                   int64_t v_head_stride, int32_t B, int32_t T, int32_t num_heads, const int32_t* d_cu_seqlens,
                   const int32_t* d_context_lens, const int32_t* d_block_table, int32_t blocks_per_seq, const float* d_rope,
                   int32_t rope_positions, int32_t rotary_dim, int32_t rope_layout, void* d_q_out, int64_t out_row_stride,
                   int64_t out_head_stride, int32_t* d_err, void* stream);

/* Block dst[i] becomes a copy of block src[i], in all layers, for i < n. No
 * block may be a destination twice, or a source and a destination. */
int axon_kv_copy_blocks(const axon_kv_cache* cache, const int32_t* d_src, const int32_t* d_dst, int32_t n,
                        int32_t* d_err, void* stream);

/* Rows dst[i] take over what rows src[i] hold, for i < n (n <= max_seqs): parallel
 * samples of one prompt, or the beams that survive a step. Every row is taken as it
 * was before the call; a row may be a source any number of times, a
 * destination once. A destination first gives back what it holds. Whole blocks are
 * shared; a last block that is only part-filled is copied into a free one, so
 * that each row can be appended to. src[i] = dst[i] changes nothing. Copies take
 * the lowest free numbers in the order of i; blocks that the call gives back are free to
 * them. Blocks reserved beyond the length are not shared. A row whose
 * copy finds no free block keeps the whole blocks only (its length rounded down to
 * them) and the call reports it. */
int axon_kv_fork(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_src, const int32_t* d_dst,
                 int32_t n, void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream);

/* Rows give blocks back (d_rows [n], or NULL: rows 0 .. n-1; n <= max_seqs).
 * window = 0: everything, and the row's length becomes 0. window > 0: the blocks that no
 * query from position context_lens[r] on can see under that window and these
 * sinks; their table entries become -1, the length stays. */
int axon_kv_release(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_rows, int32_t n,
                    int32_t window, int32_t sinks, int32_t* d_err, void* stream);

/* Rows (each at most once) take blocks for d_new_tokens[i] more tokens after their
 * context_lens, the lowest free numbers in the order of the rows; blocks that a row
 * has beyond its length already are kept and counted, from the front. When the pool
 * runs out, the rows served first keep theirs, the entries left over stay
 * -1, and the call reports it. Lengths are not advanced. */
int axon_kv_reserve(const axon_kv_cache* cache, const axon_kv_seqs* seqs, const int32_t* d_rows,
                    const int32_t* d_new_tokens, int32_t n, void* d_workspace, int64_t workspace_bytes,
                    int32_t* d_err, void* stream);

/* Blocks in use move to the front: the k-th one whose number is at least their count
 * goes to the k-th free number below it, in all layers, and the table and the
 * counts follow. d_moved [num_blocks] (or NULL) gets each block's
 * number afterwards, -1 for free ones, and d_live [1] (or NULL) their count. */
int axon_kv_compact(const axon_kv_cache* cache, const axon_kv_seqs* seqs, int32_t* d_moved, int32_t* d_live,
                    void* d_workspace, int64_t workspace_bytes, int32_t* d_err, void* stream);

/* Workspace of axon_kv_fork, axon_kv_reserve and axon_kv_compact. */
int axon_kv_workspace(const axon_kv_cache* cache, const axon_kv_seqs* seqs, int64_t* bytes);

/* A token per row from its logits, for B rows of V (1 .. 524288). With m the largest logit of the row,
 * w_i = exp((logit_i - m) / temperature), and tokens in the order of their logits, equal ones by number:
 *   top-k: the first top_k stay (0 or less, V or more: all);
 *   top-p: of these the fewest, from the front, whose weights reach top_p times the sum of them all (1 or more, or
 *          not a number: all; 0 or less: the first);
 *   min-p: of these the ones with w_i >= min_p (0 or less, or not a number: all).
 * The first token always stays. d_tokens[b] is the first, by number, at which the running sum of the weights that
 * stay passes u times their sum, d_prob[b] (fp32, or NULL) its weight over that sum. u is clamped to [0, 1 - 2^-24].
 * temperature 0 (or less, or not a number): the largest logit, the lowest number among equals, d_prob 1. Logits that are not numbers
 * count as -infinity, which is never chosen; a row of nothing else gets token -1 and d_prob 0. Infinite logits share
 * everything.
 * Weights are integers in units of 2^-44 of the largest weight, and their sums are exact. So a weight is off by up to about 2^-45
 * of the largest and 2^-41 of itself (one below half a unit is 0 and never drawn), and a sum of n weights by n * 2^-45 of the
 * largest weight (2^-28 for 128256, 2^-26 for the longest vocabulary, if all were off the same way) and 2^-41 of itself. The
 * token is that of 64-bit arithmetic unless u or top_p falls that near to a border, or min_p that near to a weight, and does
 * not depend on timing; d_prob is off by its weight's error over the sum, besides its rounding to fp32.
 *   d_logits        [B][V] of type `precision` (AXON_BF16, AXON_FP16; AXON_FP32_DEBUG: fp32, as the model's logits),
 *                   row stride in elements, at least V
 *   d_temperature, d_top_k, d_top_p, d_min_p  [B], or NULL: 1, all, 1, 0
 *   d_u             [B], uniform in [0, 1)
 * No error word: nothing is indexed by what the device holds. The first call on a device sets its kernel's limits: make
 * it before a stream capture. */
int axon_sample(const void* d_logits, int64_t row_stride, int32_t precision, int32_t B, int32_t V, const float* d_temperature,
                const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, const float* d_u, int32_t* d_tokens,
                float* d_prob, void* stream);

/* Synchronise `stream` and read and clear an operator's error word: AXON_OK,
 * AXON_ERR_DEVICE_CHECK or AXON_ERR_TIMEOUT; *bits (optional) receives it. Bits:
 * 2 block number, 4 position, 8 wait expired, 16 row or row offsets, 32 no free block. */
int axon_check_error(int32_t* d_err, void* stream, int32_t* bits);

/* Release everything the model owns. NULL is a no-op. */
void axon_free(axon_model* m);

/* Static string naming a status code. */
const char* axon_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* AXON_H */
