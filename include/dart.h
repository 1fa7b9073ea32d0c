/*
 * dart.h -- C ABI of the B200 (sm_100a) implementation of DART's drafting step.
 *
 * One call of dart_draft_step followed by one call of dart_build_tree is one "draft step":
 * target hidden states -> one draft decoder layer over the prefix KV cache plus K query rows
 * -> LM head -> per-position log-softmax + top-k -> N-gram-scored tree pruning -> a
 * fixed-budget draft token tree (token ids, parents, tree-attention mask).
 *
 * Conventions
 *   - Every pointer is labelled HOST or DEVICE.  Device buffers are caller-owned unless stated.
 *   - bf16 tensors are row-major with the last index fastest; weight matrices are [out, in];
 *     weight pointers and `feats` must be 32-byte aligned and their row strides multiples of 16 bytes
 *     (they are read by TMA tile loads, or by 256-bit loads in the fallback kernels), every other device
 *     pointer 16-byte aligned.
 *   - All GPU work is enqueued on the CUDA stream passed as `void* cuda_stream` (a cudaStream_t;
 *     NULL = the legacy default stream).  dart_draft_step and dart_build_tree do not
 *     synchronise, allocate, or copy between host and device.
 *   - Return value: DART_OK (0) or a negative dart_status.  Argument errors are reported
 *     synchronously and enqueue nothing.  Errors that only the device can detect (a lookup
 *     that ran past its probe bound, a bounded wait on a barrier or on another CTA's flag that ran
 *     out) set a status word read by dart_last_device_status; the kernels never wait without a limit.
 *   - One handle may be used from one host thread and one stream at a time.
 *   - There is no CPU fallback: on a machine without an sm_100 device dart_draft_init fails.
 */
#ifndef DART_H_
#define DART_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dart_status {
  DART_OK = 0,
  DART_ERR_INVALID_ARG = -1,      /* NULL/misaligned pointer, shape the kernels do not support */
  DART_ERR_UNSUPPORTED_ARCH = -2, /* current device is not compute capability 10.x */
  DART_ERR_CUDA = -3,             /* a CUDA runtime call failed; see dart_last_cuda_error */
  DART_ERR_CAPACITY = -4,         /* batch > max_batch, or prefix + K > max_prefix */
  DART_ERR_TIMEOUT = -5,          /* a bounded device-side loop gave up (device status word) */
  DART_ERR_INTERNAL = -6
} dart_status;

typedef struct dart_handle dart_handle; /* opaque; owns workspace + the device N-gram table */

/*
 * Shapes and hyper-parameters, fixed for the lifetime of a handle.
 * Layer shapes follow Appendix B ("hyperparameters ... aligned with the target model");
 * topk/beam/tree_budget and the Combine weights are Appendix D's k_i, w, theta+1, w_ng,
 * 0.9^level, (level+1)^-0.7.
 */
typedef struct dart_config {
  uint32_t struct_size;  /* = sizeof(dart_config); guards against layout mismatch */
  int32_t hidden;        /* h; multiple of 64 */
  int32_t n_q_heads;     /* H_q */
  int32_t n_kv_heads;    /* H_kv; H_q % H_kv == 0 and (H_q/H_kv)*K <= 64 */
  int32_t head_dim;      /* d_h: 64 or 128 */
  int32_t mlp_inter;     /* I; multiple of 16 */
  int32_t vocab;         /* V; multiple of 16, < 2^21 */
  int32_t feat_in;       /* width of the concatenated target features (3h); multiple of 16.  0: the caller fuses the
                            features itself and passes g [.., hidden] as `feats`; w_fc is unused, no prefill */
  int32_t max_batch;     /* sequences per call; <= 32 and max_batch * K <= 128 */
  int32_t max_prefix;    /* P_cap: rows per sequence in the caller's KV cache */
  int32_t K;             /* query rows per sequence = future positions d (Section 3.2); 1..8 */
  int32_t topk;          /* k_i: candidates kept per position, 1..32 (Appendix D: 25) */
  int32_t beam;          /* w: beam width, 1..32 (Appendix D: 20) */
  int32_t tree_budget;   /* nodes in the output tree including the root, 2..64 (theta + 1 = 60) */
  int32_t ngram_order;   /* 2 or 3 (Appendix C: 3) */
  float rope_theta;      /* RoPE base (1e6) */
  float rms_eps;         /* RMSNorm epsilon (1e-6) */
  float w_ng;            /* Combine: N-gram weight (0.5) */
  float logit_decay;     /* Combine: w_logit = logit_decay^level (0.9) */
  float level_exp;       /* Combine: w_level = (level+1)^-level_exp (0.7) */
  float eps_logit;       /* epsilon inside s_logit = log(softmax + eps) */
  float eps_ng;          /* epsilon of a missing N-gram: s_ng = log(eps_ng) */
  float temperature;     /* 0 = deterministic top-k; > 0 = Gumbel-top-k on logits / temperature */
  uint64_t philox_seed;  /* key of the Philox4x32-10 stream used when temperature > 0 */
  int32_t ngram_layout;  /* device layout of the N-gram: DART_NGRAM_HASH or DART_NGRAM_TRIE (Appendix C) */
  int32_t reserved0;     /* 0 */
} dart_config;

/*
 * Draft-model parameters (Appendix B "Trainable parameters": FC, decoder layer, LM head, mask
 * representation; the embedding is the target's).  DEVICE pointers to bf16, row-major
 * [out, in]; caller-owned, never written, must outlive the handle.
 */
typedef struct dart_weights {
  const void* w_fc;       /* [h, feat_in]   fusion of the three target layers' hidden states */
  const void* embed;      /* [V, h]         target embedding table (shifted token embedding) */
  const void* mask_vec;   /* [2h]           learned <mask> representation, stands for [g ; e] */
  const void* norm_g;     /* [h]            RMSNorm gain on g */
  const void* norm_e;     /* [h]            RMSNorm gain on e */
  const void* w_q;        /* [H_q*d_h, 2h]  */
  const void* w_k;        /* [H_kv*d_h, 2h] */
  const void* w_v;        /* [H_kv*d_h, 2h] */
  const void* w_o;        /* [h, H_q*d_h]   */
  const void* norm_post;  /* [h]            RMSNorm gain before the MLP */
  const void* w_gate;     /* [I, h] */
  const void* w_up;       /* [I, h] */
  const void* w_down;     /* [h, I] */
  const void* norm_final; /* [h]            RMSNorm gain before the LM head */
  const void* w_lm;       /* [V, h]         the drafter's own LM head */
} dart_weights;

/*
 * N-gram rows (Appendix C), HOST arrays of length n_rows, copied into a library-owned
 * device hash table by dart_draft_init.  Row i says: after context (ctx0[i], ctx1[i]) the
 * token next[i] has continuity score score[i] = log(Pr(next | context) + eps), Appendix D's
 * s_ng.  order[i] is 3 (trigram) or 2 (bigram; ctx0[i] ignored).  Of duplicate rows the first wins.
 */
#define DART_NGRAM_HASH 0 /* open-addressing table, one 16-byte slot per row at load <= 0.5: one probe per lookup */
#define DART_NGRAM_TRIE 1 /* child lists (Appendix C): the context's node is located once, its children are then
                             searched for every candidate; 8 bytes per row plus 8 per distinct 3-gram context */
typedef struct dart_ngram_host {
  int64_t n_rows;
  const uint8_t* order;
  const int32_t* ctx0;
  const int32_t* ctx1;
  const int32_t* next;
  const float* score;
} dart_ngram_host;

/*
 * Inputs of one forward pass (Section 3.2).  Per sequence b the K query rows are
 * r = 0..K-1 at absolute positions P_b + r, P_b = seq_lens[b]; rows r < n_fresh carry fresh
 * target features and the id of the token that follows them (shifted embedding), the rest
 * are <mask> rows.  The canonical step is n_fresh = 1: the last prefix position plus d-1 masks.
 * After a verification that accepted a different number of tokens per sequence the counts differ:
 * fresh_counts_host[b] = F_b then replaces n_fresh, and the fresh rows' features and token ids are
 * packed in sequence order (sequence 0's F_0 rows, then sequence 1's, ...).
 */
typedef struct dart_step_in {
  int32_t batch;          /* B <= max_batch */
  int32_t n_fresh;        /* F, 0..K (0: K mask rows, feats/tokens unused) */
  const void* feats;      /* DEVICE bf16 [B, F, feat_in]  (packed [sum F_b, feat_in] with fresh_counts_host); with
                             feat_in = 0 the fused features g, [B, F, hidden] */
  const int32_t* tokens;  /* DEVICE i32  [B, F] next-token ids, 0 <= id < V  (packed [sum F_b]) */
  const int32_t* seq_lens;      /* DEVICE i32 [B]  P_b: rows already in the cache */
  const int32_t* seq_lens_host; /* HOST   i32 [B]  same values; used for capacity checks and launch sizing */
  void* k_cache;          /* DEVICE bf16 [max_batch, H_kv, max_prefix, d_h], post-RoPE keys */
  void* v_cache;          /* DEVICE bf16, same layout.  The call appends the fresh positions' k, v: it writes
                             rows P_b .. P_b+F-1 of both caches and nothing else (the <mask> rows' k, v
                             are transient); the caller advances seq_lens.  Needs P_b + F <= max_prefix. */
  uint64_t step_counter;  /* Philox counter word; change it every call when temperature > 0 */
  const int32_t* fresh_counts_host; /* HOST i32 [B] per-sequence fresh-row counts F_b in 0..K, or NULL: every
                                       sequence has n_fresh.  With it the call appends rows P_b .. P_b+F_b-1. */
} dart_step_in;

/*
 * Outputs of one forward pass: Algorithm 1 lines 6-8 for every logit row.  Row r predicts
 * the token after position P_b + r (shifted logits); rows r >= max(F,1)-1 are the d logit
 * rows of Section 3.2, earlier rows are computed as well.
 */
typedef struct dart_step_out {
  int32_t* topk_ids;      /* DEVICE i32 [B, K, topk]  S_i, by selection value desc, ties lower id */
  float* topk_slogit;     /* DEVICE f32 [B, K, topk]  s_logit = log(softmax(logits/T) + eps_logit) */
  float* logits;          /* DEVICE f32 [B, K, V] or NULL.  Full logits (before 1/T), for checking only */
} dart_step_out;

/* Inputs of Algorithm 1 for B sequences. */
typedef struct dart_tree_in {
  int32_t batch;
  int32_t first_row;          /* first logit row used as level 0 (= max(F,1)-1) */
  int32_t n_levels;           /* d = number of levels, first_row + n_levels <= K */
  const int32_t* topk_ids;    /* DEVICE i32 [B, K, topk] as written by dart_draft_step */
  const float* topk_slogit;   /* DEVICE f32 [B, K, topk] */
  const int32_t* ctx_tail;    /* DEVICE i32 [B, 2]: the last two known tokens (c_-2, c_-1); -1 = absent */
  const int32_t* first_rows_host; /* HOST i32 [B] per-sequence first logit row (= max(F_b,1)-1), or NULL: first_row for
                                     all.  Sequence b then has min(n_levels, K - first_rows_host[b]) levels. */
} dart_tree_in;

/*
 * The pruned draft tree per sequence.  Slot 0 is the root (token c_-1, parent -1, depth 0);
 * slots 1..n_nodes-1 are the selected nodes by score descending.  parents[x] < x.
 * mask[x][y] = 1 iff y == x or y is an ancestor of x (the tree-attention mask).
 * Unused slots: token -1, parent -1, depth -1, mask row 0.
 */
typedef struct dart_tree_out {
  int32_t* tokens;   /* DEVICE i32 [B, tree_budget] */
  int32_t* parents;  /* DEVICE i32 [B, tree_budget] */
  int32_t* depth;    /* DEVICE i32 [B, tree_budget] */
  uint8_t* mask;     /* DEVICE u8  [B, tree_budget, tree_budget] */
  int32_t* n_nodes;  /* DEVICE i32 [B] */
  float* scores;     /* DEVICE f32 [B, tree_budget] or NULL: the (ancestor-clamped) node scores */
} dart_tree_out;

/*
 * Create a handle (Section 3.2 + Section 4 set-up): validates cfg, records the weight
 * pointers, builds the device N-gram hash table from the host rows (ngram may be NULL or
 * empty: every lookup then misses), allocates the workspace (the only allocation the library
 * ever makes) and precomputes Appendix D's per-level weights.  Synchronous.
 * Errors: INVALID_ARG, UNSUPPORTED_ARCH, CUDA.  *out is NULL on failure.
 */
int dart_draft_init(const dart_config* cfg, const dart_weights* weights, const dart_ngram_host* ngram,
                    dart_handle** out);

/*
 * One forward pass of the draft layer and LM head with fused log-softmax/top-k
 * (Section 3.2; Algorithm 1 lines 6-8; Appendix D s_logit).  Asynchronous on `cuda_stream`.
 * Errors: INVALID_ARG (NULL pointers, a fresh-row count out of range), CAPACITY (batch > max_batch or
 * seq_lens_host[b] + F_b > max_prefix).
 */
int dart_draft_step(dart_handle* h, const dart_step_in* in, const dart_step_out* out, void* cuda_stream);

/*
 * Continuity-aware tree pruning (Algorithm 1, Appendix D) for B sequences, one thread block
 * per sequence.  Asynchronous on `cuda_stream`.  Bit-exact with a sequential fp32 evaluation
 * of Algorithm 1 that breaks ties by generation order.  Errors: INVALID_ARG, CAPACITY.
 */
int dart_build_tree(dart_handle* h, const dart_tree_in* in, const dart_tree_out* out, void* cuda_stream);

/*
 * One whole draft step for a caller whose step inputs and tree outputs live in HOST memory (Section 3.2 followed by
 * Algorithm 1, as one call): copies `in_bytes` from `in_host` to `in_dev`, runs dart_draft_step(in, out) and
 * dart_build_tree(tree_in, tree_out), copies `out_bytes` from `out_dev` to `out_host` and waits for `cuda_stream`.
 * The device pointers of `in` / `tree_in` (feats, tokens, seq_lens, ctx_tail) are expected to point into
 * [in_dev, in_dev + in_bytes) and those of `tree_out` into [out_dev, out_dev + out_bytes): the layout inside the two
 * buffers is the caller's.  Host buffers should be page-locked (pageable memory works, more slowly).  All buffers
 * are caller-owned; nothing is allocated.  Synchronous: on return the tree is in `out_host`.
 * Errors: those of the two calls; INVALID_ARG for a NULL buffer with a non-zero size; CUDA if a copy or the wait fails.
 */
typedef struct dart_host_io {
  const void* in_host;   /* HOST   step inputs, in_bytes */
  void* in_dev;          /* DEVICE their home on the device */
  size_t in_bytes;
  const void* out_dev;   /* DEVICE tree outputs, out_bytes */
  void* out_host;        /* HOST   where the caller reads them */
  size_t out_bytes;
} dart_host_io;
int dart_draft_step_host(dart_handle* h, const dart_host_io* io, const dart_step_in* in, const dart_step_out* out,
                         const dart_tree_in* tree_in, const dart_tree_out* tree_out, void* cuda_stream);

/* Free the workspace and the N-gram table.  The caller's buffers are untouched. */
int dart_draft_destroy(dart_handle* h);

/* Device-side status word since the last call of this function: DART_OK or DART_ERR_TIMEOUT.
 * Synchronises `cuda_stream`.  After DART_ERR_TIMEOUT the outputs of the calls since the previous check are void;
 * the call has then also cleared the handle's internal work counters (a kernel that gives up on a wait leaves
 * them half counted), so the handle stays usable: the next dart_draft_step starts from a clean state. */
int dart_last_device_status(dart_handle* h, void* cuda_stream);

/*
 * Self-test of the time-out path (the paper has no counterpart).  Every device-side wait of this library is
 * bounded: when it runs out the kernel records DART_ERR_TIMEOUT in the handle's status word and returns.  This call
 * enqueues a one-block kernel that runs exactly that path on purpose -- a wait of `spin_limit` tries (1 .. 100000,
 * each at most 2 microseconds) on a barrier that nothing signals -- so that a caller (or a test) can see the error
 * arrive through dart_last_device_status and the handle recover.  leave_ticket != 0 additionally leaves one work
 * counter of the QKV projection half counted, as a kernel that gave up mid-way would.  Faults nothing, hangs nothing.
 * Asynchronous on `cuda_stream`.  Errors: INVALID_ARG, CUDA.
 */
int dart_selftest_bounded_wait(dart_handle* h, int32_t spin_limit, int32_t leave_ticket, void* cuda_stream);

/* The cudaError_t (as int) behind the last DART_ERR_CUDA of this handle; with h = NULL, of the last call that has no
 * handle (dart_draft_init, dart_train_attention_fwd, dart_topk_rows_noalloc, dart_kv8_*, dart_qk_norm_rope, dart_token_logprobs). */
int dart_last_cuda_error(const dart_handle* h);

/* Human-readable name of a dart_status. */
const char* dart_status_string(int status);

/* Bytes of device workspace a handle for `cfg` allocates (excluding the N-gram table); 0 if cfg is invalid. */
size_t dart_workspace_bytes(const dart_config* cfg);

/*
 * Forward attention under the prefix-shared training mask (Section 3.3 "Prefix-shared masked training", Appendix B).
 * A packed row has L = prompt_len * (1 + draft_len) slots: prompt_len clean positions, then one block of draft_len
 * masked positions per prefix position n.  Clean slot q reads clean slots <= q; block n reads clean slots 0..n and
 * its own slots up to the reading one; blocks never read each other.  Slots past seq_lens_host[b] (clean slots >= it,
 * blocks of prefix positions >= it) read nothing and give zero rows.  Grouped-query heads: head j reads KV head
 * j / (n_q_heads / n_kv_heads).  Softmax scale 1 / sqrt(head_dim).
 */
typedef struct dart_train_attn_in {
  int32_t batch;             /* 1..64 */
  int32_t n_q_heads, n_kv_heads;
  int32_t head_dim;          /* 128 */
  int32_t prompt_len;        /* clean positions per packed row, >= 1 */
  int32_t draft_len;         /* d, 1..16 */
  const void* q;             /* DEVICE bf16 [batch, n_q_heads, L, head_dim], 16-byte aligned; RoPE already applied */
  const void* k;             /* DEVICE bf16 [batch, n_kv_heads, L, head_dim] */
  const void* v;             /* DEVICE bf16 [batch, n_kv_heads, L, head_dim] */
  const int32_t* seq_lens_host; /* HOST [batch]: valid prompt slots, 0..prompt_len */
  void* out;                 /* DEVICE bf16 [batch, n_q_heads, L, head_dim]; every row is written */
  int32_t* status;           /* DEVICE, may be NULL: set to a negative code if a bounded wait inside the kernel ran out */
} dart_train_attn_in;

/*
 * Enqueues the attention on `cuda_stream` (one kernel; no workspace, no handle).  Errors: INVALID_ARG (NULL or
 * misaligned pointers, sizes out of range, head_dim != 128), UNSUPPORTED_ARCH, CUDA.
 */
int dart_train_attention_fwd(const dart_train_attn_in* in, void* cuda_stream);

/* Bytes of device memory the N-gram of this handle occupies in its layout (0 without an N-gram or handle). */
size_t dart_ngram_bytes(const dart_handle* h);

/* Number of kernels one dart_draft_step / dart_build_tree call enqueues for this batch size
 * (used by benchmarks to report launch counts). */
int dart_step_launch_count(const dart_handle* h, int batch, int n_fresh);

/*
 * Verification inputs of a draft tree (Section 3, Figure 2: the tree is verified by the target model in one
 * forward pass with tree attention; the attention mask is dart_tree_out.mask).  The paper names the step, not
 * its encoding; this one is the usual pair: node x sits at absolute position root_pos[b] + depth[x] (root_pos =
 * position of the root token c_-1), and a candidate continuation is a root-to-leaf path given as the slots of its
 * nodes.  retrieve row j = path of the j-th leaf (leaves in ascending slot order), root first, padded with -1;
 * rows past n_leaves and position ids of unused slots are -1.  One small kernel, asynchronous on `cuda_stream`.
 * Errors: INVALID_ARG, CAPACITY (batch > max_batch).
 */
typedef struct dart_verify_in {
  int32_t batch;
  int32_t max_levels;         /* columns of retrieve minus one: >= the deepest node's depth (K is always enough) */
  const int32_t* parents;     /* DEVICE i32 [B, tree_budget] as written by dart_build_tree */
  const int32_t* depth;       /* DEVICE i32 [B, tree_budget] */
  const int32_t* n_nodes;     /* DEVICE i32 [B] */
  const int32_t* root_pos;    /* DEVICE i32 [B] absolute position of each sequence's root token */
} dart_verify_in;
typedef struct dart_verify_out {
  int32_t* position_ids;      /* DEVICE i32 [B, tree_budget] */
  int32_t* retrieve;          /* DEVICE i32 [B, tree_budget, max_levels + 1] */
  int32_t* n_leaves;          /* DEVICE i32 [B] */
} dart_verify_out;
int dart_tree_verify_inputs(dart_handle* h, const dart_verify_in* in, const dart_verify_out* out, void* cuda_stream);

/*
 * Draft-side prefill (Section 3.2: the draft layer attends over its own KV cache of the prefix, which has to
 * exist before the first drafting step).  A single layer's keys and values depend on nothing but the layer's
 * input, so building the cache for new prefix positions needs no attention: for every new row the call
 * computes z = [RMSNorm(W_fc f) ; RMSNorm(E[token])], k = RoPE(W_k z) and v = W_v z at the row's absolute
 * position and stores them.  Sequence b gets new_rows_host[b] rows at positions seq_lens_host[b] ..; their
 * features and next-token ids are packed in sequence order.  The caller then advances its sequence lengths and
 * runs dart_draft_step as usual (whose own fresh rows are appended by that call).  No logits are produced.
 * Asynchronous on `cuda_stream`; the packed rows are processed in passes of up to 4096 rows (three kernel launches
 * per pass: token embeddings, feature FC, k / v projection), a sequence may straddle two passes.
 * Errors: INVALID_ARG (also with feat_in = 0: the prefill needs the fusion matrix), CAPACITY (batch > max_batch or
 * seq_lens_host[b] + new_rows_host[b] > max_prefix).
 */
typedef struct dart_prefill_in {
  int32_t batch;                  /* B <= max_batch */
  const void* feats;              /* DEVICE bf16 [sum N_b, feat_in], 32-byte aligned */
  const int32_t* tokens;          /* DEVICE i32  [sum N_b] id of the token that follows each row */
  const int32_t* seq_lens_host;   /* HOST i32 [B] rows already in the cache */
  const int32_t* new_rows_host;   /* HOST i32 [B] N_b >= 0 rows to add */
  void* k_cache;                  /* DEVICE bf16 [max_batch, H_kv, max_prefix, d_h]; rows P_b .. P_b+N_b-1 are written */
  void* v_cache;                  /* DEVICE bf16, same layout */
} dart_prefill_in;
int dart_draft_prefill(dart_handle* h, const dart_prefill_in* in, void* cuda_stream);

/*
 * Measurement aid (the paper has no counterpart): the next dart_draft_step (stages 0..7) or
 * dart_build_tree (stage 8) records the caller-owned CUDA events `start_event` / `stop_event`
 * (cudaEvent_t handles) on the stream immediately before and after the kernels of `stage`,
 * then forgets them.  Stages: 0 feature FC + input staging, 1 QKV + RoPE, 2 attention,
 * 3 o_proj + norm, 4 gate/up, 5 down + norm, 6 LM-head kernel alone, 7 top-k merge, 8 tree.
 * Errors: INVALID_ARG.
 */
int dart_set_profile_events(dart_handle* h, int stage, void* start_event, void* stop_event);

/*
 * Per-row log-softmax + top-k of caller-provided logits without any allocation (the paper has no
 * counterpart: this is the candidate selection of Algorithm 1 lines 6-8 at temperature 0, offered to
 * callers that cannot allocate device memory -- a process whose own pool already owns all of HBM, a
 * latency-critical loop where cudaMalloc's implicit synchronisation is not allowed, a plug-in without a
 * dart_handle to hold a workspace).  Needs no handle.
 *   logits      DEVICE f32 [rows, vocab], row-major            (in)
 *   out_ids     DEVICE i32 [rows, topk]   value desc, ties to the lower id   (out)
 *   out_slogit  DEVICE f32 [rows, topk]   log(softmax(logits)[id] + eps_logit) (out)
 * Limits: 1 <= rows <= 128 (more: DART_ERR_CAPACITY), 1 <= topk <= min(32, vocab).
 * Scratch: a fixed 1.6 MB array inside the library's device image, one per GPU, which every GPU that
 * loads the library holds until the process exits.  All calls on a GPU share it and it keeps the last
 * call's contents (every call overwrites what it reads, nothing needs clearing): calls that overlap on
 * the same GPU -- different streams or host threads -- race; serialise them.
 * The first call on each device (made with that device current) looks up the array's device address
 * (two host threads making it together both cache the same address, which is harmless);
 * make that first call before any CUDA stream capture.  Calls cudaMalloc/cudaFree never.
 * Asynchronous on `cuda_stream`.  Errors: INVALID_ARG, CAPACITY, UNSUPPORTED_ARCH (not sm_100),
 * CUDA (the cudaError_t is then returned by dart_last_cuda_error(NULL)).
 */
int dart_topk_rows_noalloc(const float* logits, int32_t rows, int32_t vocab, int32_t topk, float eps_logit,
                           int32_t* out_ids, float* out_slogit, void* cuda_stream);

/*
 * ---- The target's KV cache in 8 bits, in pages -------------------------------------------------------------------
 * The draft tree is verified by the target model in one forward pass with tree attention (Section 3, Figure 2).  The
 * paper leaves the target's cache to its serving stack; these calls are that cache: attention of a step's new rows
 * (a tree, a prompt's chunk, a single token) over pages of 8-bit keys and values, the append that commits the accepted
 * rows, and the page operations of a process that serves many sequences.  None needs a handle; nothing is allocated;
 * everything is asynchronous on `cuda_stream` and may be captured into a CUDA graph (lengths, tables and counts are read
 * on the DEVICE when the kernels run; the HOST arguments only bound them).
 *
 * A page holds `page_tokens` consecutive tokens of one sequence for every layer and KV head.  Value = scale * code,
 * one fp32 scale per (layer, page, KV head) for keys and one for values: code e4m3 (DART_KV8_E4M3) or a two's-
 * complement integer -127 .. 127 (DART_KV8_INT8).  Position t of the sequence in slot i is token t % page_tokens of page
 * page_table[i][t / page_tokens].
 *
 * Device-detected errors go to the caller's `status` word (DEVICE i32, may be NULL; never cleared by the calls):
 * DART_ERR_INVALID_ARG for a length, count, slot or page id out of its bounds (the sequence's outputs are then void,
 * nothing outside the buffers is touched), DART_ERR_CAPACITY for a pool without enough free pages, DART_ERR_TIMEOUT
 * for a bounded wait that ran out.
 */
#define DART_KV8_E4M3 0
#define DART_KV8_INT8 1
typedef struct dart_kv8_cache {
  int32_t format;        /* DART_KV8_E4M3 or DART_KV8_INT8 */
  int32_t n_layers;      /* 1..1024 */
  int32_t n_pages;       /* 1..2^24 */
  int32_t n_kv_heads;    /* 1..256 */
  int32_t page_tokens;   /* 16, 32, 64 or 128 */
  int32_t head_dim;      /* 64 or 128 */
  void* k_pages;         /* DEVICE u8  [n_layers, n_pages, n_kv_heads, page_tokens, head_dim], 16-byte aligned */
  void* v_pages;         /* DEVICE u8, same layout */
  float* k_scale;        /* DEVICE f32 [n_layers, n_pages, n_kv_heads]; for pages in use 2^-100 .. 2^120 (the append writes
                            powers of two from 2^-64 on) */
  float* v_scale;        /* DEVICE f32, same layout */
} dart_kv8_cache;

/*
 * Attention of `rows` new rows per sequence over the cache and over each other.  Row r of batch entry b sits in sequence
 * slot slots[b] (or b), reads the slot's seq_lens cached positions and the new rows y <= r (mask == NULL) or those with
 * mask[b][r][y] != 0 (a draft tree's attention mask as dart_build_tree writes it, self included); new rows from
 * n_rows[b] on do not exist.  Without k_new / v_new the rows read the cache alone.  Grouped-query heads: head j reads KV
 * head j / (n_q_heads / n_kv_heads).  Softmax scale 1 / sqrt(head_dim), keys post-RoPE.  Every row of `out` is written;
 * rows that see no key and rows from n_rows[b] on are zero.  Sums are fp32; weights enter the second product as fp16, relative to
 * what a key contributes (weight times value scale), so the scales of a sequence may lie far apart (a span of 2^90 is safe):
 * each is off by at most 2^-11 of itself or 2^-34 of the largest, whichever is more.  Queries and new rows enter the products
 * as fp16 multiples of a power of two near the row's largest element: elements below 2^-17 of it are off by up to 2^-25 of it (new values: 2^-23 and 2^-31).
 * What hidden rows, rows that do not exist and positions
 * behind a sequence's length hold (infinities and NaN included) does not reach the output.
 */
typedef struct dart_kv8_attn_in {
  int32_t layer;
  int32_t batch;             /* 1..1024 */
  int32_t rows;              /* R: 1..4096; with a mask 1..64 */
  int32_t n_q_heads;         /* a multiple of n_kv_heads, at most 128 per KV head */
  int32_t max_seqs;          /* rows of page_table and seq_lens; >= batch without slots */
  int32_t max_pages;         /* columns of page_table */
  int32_t max_len;           /* HOST bound of seq_lens, 0 .. max_pages * page_tokens: sizes the launch and the workspace; keep it
                                near the longest length (dart_kv8_attention_plan) */
  const void* q;             /* DEVICE bf16 [batch, R, n_q_heads, head_dim], RoPE applied */
  const void* k_new;         /* DEVICE bf16 [batch, R, n_kv_heads, head_dim] or NULL (then v_new and mask are NULL too) */
  const void* v_new;
  int64_t q_stride;          /* elements from one row to the next, >= n_q_heads * head_dim, a multiple of 8; entries of
                                the batch are R rows apart (so q, k_new, v_new may be slices of one QKV matrix) */
  int64_t new_stride;        /* the same for k_new and v_new, >= n_kv_heads * head_dim */
  const int32_t* slots;      /* DEVICE i32 [batch] or NULL (slot b) */
  const int32_t* seq_lens;   /* DEVICE i32 [max_seqs] */
  const int32_t* page_table; /* DEVICE i32 [max_seqs, max_pages] */
  const int32_t* n_rows;     /* DEVICE i32 [batch], 0..R, or NULL (R) */
  const uint8_t* mask;       /* DEVICE u8 [batch, R, R] or NULL (causal) */
  void* out;                 /* DEVICE bf16 [batch, R, n_q_heads, head_dim] */
  void* workspace;           /* DEVICE, 16-byte aligned, dart_kv8_attention_workspace_bytes; calls that may overlap (other
                                streams, other graphs) need one each */
  size_t workspace_bytes;
  int32_t* status;
} dart_kv8_attn_in;
int dart_kv8_attention(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, void* cuda_stream);
/* Workspace for this shape and any smaller max_len; 0 for arguments dart_kv8_attention refuses. */
size_t dart_kv8_attention_workspace_bytes(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len);/*
 * How such a call is cut into CTAs.  The key axis is split by max_len, not by the lengths on the device: with a bound far above
 * them the parts are as long as the bound asks for and few of them have work, so a tight max_len is a faster call.
 */
typedef struct dart_kv8_plan {
  int32_t many_rows;         /* 1: the tcgen05 kernel, 0: the streaming kernel for few rows of a KV head */
  int32_t row_tiles;         /* many rows: tiles of 128 (row, head of the group) pairs */
  int32_t paired;            /* many rows: two tiles share a CTA (an odd last one has its own, with twice the keys) */
  int32_t keys_per_part;     /* keys, new rows included where many_rows, that a CTA takes at most */
  int32_t max_parts;         /* CTAs that share a KV head's keys at length max_len; 1: no join */
} dart_kv8_plan;
int dart_kv8_attention_plan(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len, int32_t with_new_rows,
                            dart_kv8_plan* out);

/*
 * Self-test of the time-out path, as dart_selftest_bounded_wait: an attention call for many rows (the tcgen05 kernel; others
 * are refused) in which the keys of every CTA stop arriving at their missing_from-th group of 64, and every wait gives up after
 * spin_limit tries (1 .. 100000, of up to about 1.3 microseconds each).  in->status becomes DART_ERR_TIMEOUT, `out` is void, the
 * next call is unharmed.  Faults nothing, hangs nothing.
 */
int dart_selftest_kv8_wait(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, int32_t spin_limit, int32_t missing_from, void* cuda_stream);

/*
 * Append: row j < n_append[b] of batch entry b -- source row row_index[b][j] of k_new / v_new, or row j -- goes to position
 * seq_lens + j of its slot, for layers first_layer .. first_layer + n_layers - 1 at once.  After a verification the
 * source rows are the accepted path: row_index = its row of dart_verify_out.retrieve.  The pages must be the sequence's
 * own (dart_kv8_reserve): this call has no counts to see whether they are, and after a reserve that did not fit they may not
 * be (dart_kv8_append_owned checks).  The caller advances seq_lens afterwards.
 * Scale of a page and head: the smallest power of two s >= 2^-64 with |x| <= qmax * s (qmax 448 or 127) over the finite
 * new values that the call writes there, or the page's scale if the sequence already has rows in it and that is larger;
 * codes are x / s rounded to nearest even (exact division, one rounding).  A scale that grows re-rounds the page's
 * older codes to it.  Infinities become the largest code; NaN becomes e4m3's NaN, or 0 in int8.
 * A slot that two entries with rows name is written once (the first time) and reported; an entry with n_append 0 claims no slot.
 */
typedef struct dart_kv8_append_in {
  int32_t first_layer, n_layers;
  int32_t batch;             /* 1..1024 */
  int32_t rows;              /* R: source rows per batch entry, 1..2^20 */
  int32_t max_append;        /* HOST bound of n_append, 1..2^20 (<= R without row_index); columns of row_index */
  int32_t max_seqs, max_pages;
  const void* k_new;         /* DEVICE bf16 [n_layers, batch, R, n_kv_heads, head_dim] */
  const void* v_new;
  int64_t row_stride;        /* elements from one row to the next, a multiple of 8; batch entries are R rows apart */
  int64_t layer_stride;      /* elements from one layer to the next, a multiple of 8 */
  const int32_t* slots;      /* DEVICE i32 [batch] or NULL */
  const int32_t* seq_lens;   /* DEVICE i32 [max_seqs] */
  const int32_t* page_table; /* DEVICE i32 [max_seqs, max_pages] */
  const int32_t* n_append;   /* DEVICE i32 [batch], 0..max_append, or NULL (max_append) */
  const int32_t* row_index;  /* DEVICE i32 [batch, max_append], entries 0..R-1, or NULL */
  int32_t* status;
} dart_kv8_append_in;
int dart_kv8_append(const dart_kv8_cache* cache, const dart_kv8_append_in* in, void* cuda_stream);

/*
 * Bookkeeping of a pool: which pages each sequence slot holds, and how many table entries name each page (0: free).
 * All three arrays are the caller's; a pool starts with table -1, lengths 0, counts 0.  Sequences share pages after a
 * fork; a shared page is not to be written (reserve replaces it first; dart_kv8_append_owned leaves it alone).  Lists name slots; a slot or pair that is out of
 * range, named twice, or (fork) has a source that is also a destination or a destination in use, is skipped and reported.
 */
typedef struct dart_kv8_pages {
  int32_t n_pages, page_tokens;
  int32_t max_seqs;          /* 1..65536 */
  int32_t max_pages;
  int32_t* page_table;       /* DEVICE i32 [max_seqs, max_pages], -1 = no page */
  int32_t* seq_lens;         /* DEVICE i32 [max_seqs] */
  int32_t* ref_count;        /* DEVICE i32 [n_pages] */
} dart_kv8_pages;
/*
 * dart_kv8_append that looks at the counts: rows go only into pages that no other slot names (count 1); the others are left
 * as they are and reported (DART_ERR_INVALID_ARG, unless the status word already holds an error).  For callers that do not
 * wait for the status of the dart_kv8_reserve before it: when that did not fit, the table still names the shared page.
 * in->page_table, max_seqs and max_pages are those of `pages`.
 */
int dart_kv8_append_owned(const dart_kv8_cache* cache, const dart_kv8_pages* pages, const dart_kv8_append_in* in, void* cuda_stream);
/* Slot dst[i] becomes a copy of slot src[i] (length, and the pages that hold its tokens, shared).  n: 1..1024 pairs. */
int dart_kv8_fork(const dart_kv8_pages* pages, const int32_t* src, const int32_t* dst, int32_t n, int32_t* status, void* cuda_stream);
/*
 * Makes positions seq_len .. seq_len + n_new[i] - 1 of the slots seqs[i] writable: missing pages are taken from the free
 * ones (lowest ids first, in list order), a page in that range that other slots share is replaced by a copy of all
 * layers (when every slot that shares it is listed, the last one keeps it).  An entry with n_new 0 asks for nothing and may name a
 * slot again.  seq_lens stay.  All or nothing: without
 * enough free pages nothing changes and the status is DART_ERR_CAPACITY.  n: 1..1024.
 */
int dart_kv8_reserve(const dart_kv8_pages* pages, const dart_kv8_cache* cache, const int32_t* seqs, const int32_t* n_new, int32_t n,
                     void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream);
/* The slots give back all their pages; a page that nobody else names is free again.  n: 1..1024. */
int dart_kv8_release(const dart_kv8_pages* pages, const int32_t* seqs, int32_t n, int32_t* status, void* cuda_stream);
/*
 * Moves the pages in use to the front of the pool: with n_live pages in use, those with ids >= n_live go to the free ids
 * below n_live (ascending to ascending; all layers), and tables and counts follow.  n_live_out: DEVICE i32 or NULL.
 */
int dart_kv8_compact(const dart_kv8_pages* pages, const dart_kv8_cache* cache, int32_t* n_live_out, void* workspace, size_t workspace_bytes,
                     int32_t* status, void* cuda_stream);
/* Workspace of reserve and compact (16-byte aligned; one call at a time). */
size_t dart_kv8_pages_workspace_bytes(const dart_kv8_pages* pages);

/*
 * ---- Around the target's attention: rotation, windows, log probabilities --------------------------------------------
 * What a verification step computes in front of dart_kv8_attention (norms and rotation of the new rows' queries and keys), its form for
 * models that attend to a window, and what is read off the target's logits behind it.  The paper leaves the target to its serving
 * stack.  As with the calls above: no handle, nothing allocated, everything on `cuda_stream`, counts and lengths read on the
 * DEVICE; device-detected errors go to `status` (DART_ERR_INVALID_ARG; the entry's outputs are then void).
 */
#define DART_BF16 0
#define DART_FP16 1
#define DART_FP32 2
/*
 * Frequencies for dart_qk_norm_rope: inv_freq (HOST, n of them, radians per position, |f| <= pi; rope_theta^(-2i / rotary_dim), or
 * any scaled form of it) as turns per position in 64-bit fractions (out, HOST), which the caller copies to the device once.
 * An angle modulo a turn is then off by at most 2^-26 of a turn (9.4e-8 radians) at every position below 2^31.  Errors: INVALID_ARG (NULL, n outside
 * 1..64, a frequency out of range).
 */
int dart_rope_frequencies(const double* inv_freq, int32_t n, uint64_t* out);
/*
 * RMS norm of every query and key head over its head_dim elements with gains q_norm / k_norm, and the rotation of its first rotary_dim
 * elements by the row's position, in one pass: fp32 inside (squares are summed in fp32: |x| < 2^60), one rounding at the end.  Pairs are
 * (i, i + rotary_dim / 2), or (2i, 2i + 1) with interleaved; pair i turns by position * f_i; elements from rotary_dim on are only normed.
 * The position of row r of batch entry b is positions[b][r] (a draft tree: dart_verify_out.position_ids) or, without positions,
 * seq_lens + r of its slot.  Rows with a negative position and rows from n_rows[b] on do not exist: their outputs are left as they were.
 * In place (q_out == q with its stride, k_out == k) is allowed; other overlaps are not.
 */
typedef struct dart_qk_rope_in {
  int32_t batch;             /* batch * rows <= 2^24 */
  int32_t rows;              /* R >= 1 */
  int32_t n_q_heads;         /* 1..1024 */
  int32_t n_k_heads;         /* 0..1024; 0: queries alone, k / k_out / k_norm unused */
  int32_t head_dim;          /* 64 or 128 */
  int32_t rotary_dim;        /* 16..head_dim, a multiple of 16 */
  int32_t interleaved;       /* 0 or 1 */
  int32_t dtype;             /* of q, k, gains and outputs: DART_BF16, DART_FP16 or DART_FP32 */
  int32_t max_seqs;          /* rows of seq_lens (without positions); >= batch without slots */
  float eps;                 /* >= 0 */
  const void* q;             /* DEVICE [batch, R, n_q_heads, head_dim], 16-byte aligned, as all of these */
  const void* k;             /* DEVICE [batch, R, n_k_heads, head_dim] */
  void* q_out;               /* DEVICE, q's shape */
  void* k_out;               /* DEVICE, k's shape */
  int64_t q_stride, k_stride, q_out_stride, k_out_stride; /* elements from one row to the next, multiples of 16 bytes; entries of the
                                batch are R rows apart (so q and k may be slices of one QKV matrix) */
  const void* q_norm;        /* DEVICE [head_dim] gains, or NULL: no norm (then k_norm is NULL too) */
  const void* k_norm;
  const uint64_t* freqs;     /* DEVICE [rotary_dim / 2] of dart_rope_frequencies */
  const int32_t* positions;  /* DEVICE i32 [batch, R] or NULL */
  const int32_t* seq_lens;   /* DEVICE i32 [max_seqs]; NULL with positions */
  const int32_t* slots;      /* DEVICE i32 [batch] or NULL (slot b); NULL with positions */
  const int32_t* n_rows;     /* DEVICE i32 [batch], 0..R, or NULL (R) */
  int32_t* status;
} dart_qk_rope_in;
int dart_qk_norm_rope(const dart_qk_rope_in* in, void* cuda_stream);

/*
 * dart_kv8_attention for models that attend to a sliding window and a few first tokens (sinks): the row at position p sees the cached
 * position t, or the new row at position t that the causal order or the mask shows it, iff t < sinks or t > p - window.  Without a
 * mask row r sits at seq_len + r.  With a mask its position is positions[b][r] (dart_verify_out.position_ids: seq_len + depth), within
 * seq_len .. seq_len + R - 1 (others are reported); a row with a negative position does not exist: zero, and seen by nobody.
 * Pages that no row of the sequence can see are not read and may have been given back (dart_kv8_trim).  Everything else, accuracy and what hidden
 * keys may hold included, is as for dart_kv8_attention.
 */
typedef struct dart_kv8_window {
  int32_t window;            /* >= 1; 1: a row sees itself and the sinks */
  int32_t sinks;             /* >= 0 */
  const int32_t* positions;  /* DEVICE i32 [batch, R]; needed with a mask, NULL without */
} dart_kv8_window;
int dart_kv8_attention_window(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* window, void* cuda_stream);
/* Workspace for this shape and any smaller max_len; 0 for arguments dart_kv8_attention_window refuses. */
size_t dart_kv8_attention_window_workspace_bytes(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len,
                                                 int32_t window, int32_t sinks);
/* How such a call is cut, as dart_kv8_attention_plan tells it: by max_len or the window, whichever is less. */
int dart_kv8_attention_window_plan(const dart_kv8_cache* cache, int32_t batch, int32_t rows, int32_t n_q_heads, int32_t max_len, int32_t window,
                                   int32_t sinks, int32_t with_new_rows, dart_kv8_plan* out);
/* dart_selftest_kv8_wait of such a call: the kernel's instances with a window wait for the new rows' tiles as well. */
int dart_selftest_kv8_window_wait(const dart_kv8_cache* cache, const dart_kv8_attn_in* in, const dart_kv8_window* window, int32_t spin_limit,
                                  int32_t missing_from, void* cuda_stream);
/*
 * The slots give back the pages that lie wholly behind the window of every row to come (positions <= seq_len - window) and hold no sink
 * (positions >= sinks); their table entries become DART_KV8_GIVEN_BACK, the other slots that share them keep them.  For pools whose layers all attend to
 * a window.  Fork copies such entries, release clears them; dart_kv8_attention of such a slot is an error (reported).  seq_lens stay and must not
 * shrink behind the next position to come.  n: 1..1024; a slot that is out of range or named twice is skipped and reported.
 */
#define DART_KV8_GIVEN_BACK (-2)
int dart_kv8_trim(const dart_kv8_pages* pages, const int32_t* seqs, int32_t n, int32_t window, int32_t sinks, int32_t* status, void* cuda_stream);

/*
 * Log probabilities of given tokens under softmax(logits / temperature), with the entropy and the most likely alternatives of every
 * row, in one pass over the logits.  Batch entry b has R rows of logits and n_tokens tokens: token j is scored by row
 * token_row[b][j] (a draft tree: tokens = dart_tree_out.tokens, token_row = dart_tree_out.parents) or, without token_row, by row j
 * (n_tokens == R).  A token or row of -1 asks for nothing: log probability 0, so that a path's sum may run over its root.
 * Rows from n_rows[b] on do not exist and are not read: their outputs, and tokens that they score, are 0, alternatives' ids -1.
 *   lse = log sum_v exp(x_v), x = logits / temperature;   token_logprob = x_token - lse;   entropy = -sum_v p_v log p_v
 * Alternatives are by logit descending, ties to the lower id.  Sums are fp32.  A logit of -infinity has probability 0; a row of nothing else has
 * lse, its log probabilities -infinity and entropy 0.  A NaN or +infinity makes the row's lse, entropy and log probabilities NaN; its alternatives
 * are still by value, NaN as -infinity.
 */
typedef struct dart_logprobs_in {
  int32_t batch;             /* batch * rows <= 2^22 */
  int32_t rows;              /* R >= 1 */
  int32_t vocab;             /* V: 1..2^22 */
  int32_t dtype;             /* of logits: DART_BF16, DART_FP16 or DART_FP32 */
  int32_t n_tokens;          /* 0..2^22 / batch; R without token_row (or 0) */
  int32_t topk;              /* 0..min(32, V) */
  float temperature;         /* 2^-100 .. 2^100 */
  const void* logits;        /* DEVICE [batch, R, V], aligned to an element */
  int64_t row_stride;        /* elements from one row to the next, >= V; entries of the batch are R rows apart */
  const int32_t* tokens;     /* DEVICE i32 [batch, n_tokens], -1..V-1 (others are reported, and NaN) */
  const int32_t* token_row;  /* DEVICE i32 [batch, n_tokens], -1..R-1 (likewise), or NULL */
  const int32_t* n_rows;     /* DEVICE i32 [batch], 0..R, or NULL (R) */
  float* token_logprob;      /* DEVICE f32 [batch, n_tokens] */
  float* lse;                /* DEVICE f32 [batch, R] or NULL */
  float* entropy;            /* DEVICE f32 [batch, R] or NULL */
  int32_t* top_ids;          /* DEVICE i32 [batch, R, topk] */
  float* top_logprobs;       /* DEVICE f32 [batch, R, topk] */
  void* workspace;           /* DEVICE, 16-byte aligned, dart_token_logprobs_workspace_bytes; calls that may overlap need one each */
  size_t workspace_bytes;
  int32_t* status;
} dart_logprobs_in;
int dart_token_logprobs(const dart_logprobs_in* in, void* cuda_stream);
/* Workspace of a call of this shape; 0 for a shape that dart_token_logprobs refuses. */
size_t dart_token_logprobs_workspace_bytes(int32_t batch, int32_t rows, int32_t vocab, int32_t dtype, int32_t topk);

#ifdef __cplusplus
}
#endif
#endif /* DART_H_ */
