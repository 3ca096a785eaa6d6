/*
 * sled.h -- C boundary of the batched verification step of SLED's edge server.
 *
 * The paper (Section 3.2) states the server's job: edge devices send the draft
 * tokens they generated, one shared target model verifies the drafts of many
 * devices together (Section 3.4), and each device gets back the position of its
 * first rejected token and the corrective token.  Acceptance follows Eq. 1 of
 * Section 3.1 (accept a draft x with probability min(1, p_target(x)/p_draft(x)),
 * on a rejection draw the replacement from the normalised positive part of
 * p_target - p_draft); when every draft is accepted one more token is drawn from
 * the target distribution that follows them.
 *
 * All entry points are plain C: fixed-width integers, raw pointers, an opaque
 * engine handle.  Unless a parameter says otherwise a pointer is a HOST pointer.
 * Every function returns SLED_OK (0) or a negative sled_status; a failed call
 * changes no context, page or counter.  An engine is used by one thread at a
 * time.  All device work is issued on the engine's stream, which does not wait for
 * any other stream: a DEVICE pointer passed in must refer to data that is already
 * complete (synchronise the stream that produced it first).
 */
#ifndef SLED_H_
#define SLED_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sled_engine sled_engine;
typedef struct sled_kvm sled_kvm;
typedef struct sled_planner sled_planner;

enum sled_status {
  SLED_OK = 0,
  SLED_ERR_ARG = -1,          /* null pointer, bad size, unsupported shape */
  SLED_ERR_UNKNOWN_CTX = -2,  /* ctx_id not open */
  SLED_ERR_DUP_CTX = -3,      /* ctx_id twice in one batch, or opened twice */
  SLED_ERR_K_RANGE = -4,      /* k < 0 or k > max_k */
  SLED_ERR_TOKEN_RANGE = -5,  /* token id outside [0, vocab) */
  SLED_ERR_NO_PAGES = -6,     /* KV pool exhausted */
  SLED_ERR_BATCH_TOO_LARGE = -7, /* n_reqs > max_batch or sum(k_i + 1) > max_step_tokens */
  SLED_ERR_NONFINITE = -8,    /* per-request status: a logit that had to be read was NaN or Inf */
  SLED_ERR_DEVICE = -9,       /* CUDA error, or a bounded device-side wait ran out */
  SLED_ERR_NO_DEVICE = -10,   /* no usable CUDA device: there is no CPU fallback */
  SLED_ERR_BASE_LEN = -11     /* base_len beyond the context's end, or before the start of its known token history */
};

/* returned by sled_poll while a request is still queued (not an error) */
#define SLED_PENDING 1

/* SLED_E4M3 (1 sign, 4 exponent bits with bias 7, 3 mantissa bits, subnormals, no infinities, 0x7f and 0xff no numbers) is a
 * type of caches that sled_append_keys writes and sled_attention_scaled reads, nothing else. */
enum sled_dtype { SLED_F32 = 0, SLED_BF16 = 1, SLED_E4M3 = 2 };

/* How the server forms batches (Section 3.4).  STATIC is the paper's scheme: requests wait until a fixed number
 * of them is there.  CONTINUOUS runs whatever has arrived, up to the capacity of a step. */
enum sled_batching { SLED_BATCH_STATIC = 0, SLED_BATCH_CONTINUOUS = 1 };

/* Shape of the Llama-style target model and the engine's capacities.
 * (The paper fixes only "Llama family", Section 4; shapes come from the workload.) */
typedef struct sled_config {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rms_eps;          /* RMSNorm epsilon */
  float rope_theta;       /* rotary base; pairs (2i, 2i+1) rotate by pos * theta^(-2i/head_dim) */
  int32_t weight_dtype;   /* sled_dtype of every array in sled_weights; SLED_BF16 runs the linear
                             layers on the tensor cores with bf16 activations and fp32 accumulation,
                             SLED_F32 keeps everything in fp32 */
  int32_t kv_dtype;       /* sled_dtype of the cached keys and values */
  int32_t page_size;      /* tokens per KV page (16) */
  int32_t n_pages;        /* pages in the pool; one page holds page_size tokens of every layer */
  int32_t max_batch;      /* most requests per sled_verify_batch */
  int32_t max_k;          /* most draft tokens per request */
  int32_t max_step_tokens;/* most sum(k_i + 1) per step; also the prefill chunk */
  float temperature;      /* divides the target logits before the softmax (> 0) */
  int32_t greedy;         /* 1: accept iff the draft equals the argmax, emit the argmax */
  int32_t probs_on_device;/* 1: every sled_request.draft_probs will be a DEVICE pointer (no staging buffer is
                             allocated, host rows are then refused); 0: host or device, found out per request */
  int32_t device_index;   /* CUDA device ordinal */
  void* stream;           /* cudaStream_t to launch on; NULL: the engine creates one */
  int32_t draft_probs_dtype; /* sled_dtype of every sled_request.draft_probs row.  SLED_F32: exact.  SLED_BF16: rows
                             rounded to 16 bits by the device, half the bytes per request (Section 3.2 wants requests
                             small).  Eq. 1 is then applied with the rounded q: the output follows the target's
                             distribution up to the rounding of q (relative 2^-9 per entry), no longer exactly. */
  int32_t attention_impl; /* 0: the library's choice (the warp-level tensor-core kernel).  1: the tcgen05 kernel where it
                             applies (bf16 cache, 16-token pages, head_dim 128, requests of at most 48 query rows, i.e.
                             (k + 1) * n_q_heads / n_kv_heads <= 48); other steps fall back to 0.  Same results within
                             the attention tolerance; measured slower than 0 on the workloads here. */
  int32_t linear_weight_bits; /* 0 or 16: the linear layers' matrices are of weight_dtype.  8 (needs weight_dtype =
                             SLED_BF16): wq, wk, wv, wo, w_gate, w_up, w_down and lm_head are e4m3 bytes (1 sign, 4
                             exponent bits with bias 7, 3 mantissa bits, subnormals, no infinities; the patterns 0x7f and
                             0xff must not occur) and every output row has an fp32 scale: W[n][k] = scale[n] *
                             e4m3(byte[n][k]).  Half the weight bytes per step (the paper sweeps 16-, 8- and 4-bit
                             precision, Section 4).  The linear layers then run on fp8 tensor-core instructions, which
                             take both operands in 8 bits: every bf16 activation goes in as the sum of two e4m3 numbers
                             times a per-token scale - eight significant bits, as in bf16 - and the products are summed
                             in fp32; embedding, norms, attention and cache are as with 16-bit weights.  d_model, ffn_dim
                             and n_q_heads * head_dim must be multiples of 16.
                             4: the same with 4-bit weights - e2m1 codes (1 sign, 2 exponent bits with bias 1, 1 mantissa
                             bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the even column in the
                             low half, rows of in/2 bytes: W[n][k] = scale[n] * e2m1(code[n][k]).  A quarter of the
                             weight bytes per step; only the weight operand of the fp8 instructions changes. */
} sled_config;

/* Target weights, row-major [out][in], all of type weight_dtype.  HOST or DEVICE
 * pointers (found out per pointer).  Copied during sled_init: the caller may free
 * them when it returns.  Per-layer members point to arrays of n_layers pointers. */
typedef struct sled_weights {
  const void* tok_emb;            /* [vocab][d_model] */
  const void* final_norm;         /* [d_model] */
  const void* lm_head;            /* [vocab][d_model] */
  const void* const* attn_norm;   /* [d_model] */
  const void* const* wq;          /* [n_q_heads*head_dim][d_model] */
  const void* const* wk;          /* [n_kv_heads*head_dim][d_model] */
  const void* const* wv;          /* [n_kv_heads*head_dim][d_model] */
  const void* const* wo;          /* [d_model][n_q_heads*head_dim] */
  const void* const* ffn_norm;    /* [d_model] */
  const void* const* w_gate;      /* [ffn_dim][d_model] */
  const void* const* w_up;        /* [ffn_dim][d_model] */
  const void* const* w_down;      /* [d_model][ffn_dim] */
  /* linear_weight_bits = 8 or 4 only (ignored otherwise): fp32 scales, one per output row of the matrix of the same name */
  const float* lm_head_scale;         /* [vocab] */
  const float* const* wq_scale;       /* [n_q_heads*head_dim] */
  const float* const* wk_scale;       /* [n_kv_heads*head_dim] */
  const float* const* wv_scale;       /* [n_kv_heads*head_dim] */
  const float* const* wo_scale;       /* [d_model] */
  const float* const* w_gate_scale;   /* [ffn_dim] */
  const float* const* w_up_scale;     /* [ffn_dim] */
  const float* const* w_down_scale;   /* [d_model] */
} sled_weights;

/* One device's verification request (Section 3.2: the draft tokens it sends;
 * Eq. 1 needs the draft model's distribution at each of them as well).  All
 * devices share the target's tokenizer (Section 3.4), so a row of draft_probs
 * has exactly `vocab` entries.  Borrowed for the duration of the call. */
typedef struct sled_request {
  uint64_t ctx_id;             /* context opened by sled_prefill */
  const int32_t* draft_tokens; /* [k], host */
  const void* draft_probs;     /* [k][vocab] of cfg.draft_probs_dtype (fp32 unless set otherwise), rows sum to 1; host
                                  (copied in during the forward pass) or device (read in place); may be NULL when
                                  k == 0 or in greedy mode */
  int32_t k;                   /* 0 <= k <= max_k; k = 0 is an ordinary decoding step */
  int64_t base_len;            /* 0: the drafts continue the context's current end.  m > 0: they continue its first m
                                  committed tokens - the length the device knew when it drafted.  Section 3.3: a device
                                  whose timer ran out sends its drafts again, extended; if the server had processed the
                                  first copy after all, it goes back to m before verifying, so the same request may be
                                  sent any number of times.  m may reach back as far as the context's tokens are known
                                  (everything for a context opened by sled_prefill) and not beyond its current end:
                                  SLED_ERR_BASE_LEN otherwise.  The cut is made once the whole call has passed
                                  validation and reservation; a device failure later leaves the context at m. */
} sled_request;

/* The feedback of Section 3.2: how many drafts were accepted (the first rejected
 * one is draft n_accepted + 1) and the corrective token, or the bonus token when
 * n_accepted == k. */
typedef struct sled_result {
  int32_t n_accepted;
  int32_t next_token;
  int32_t status;   /* SLED_OK or SLED_ERR_NONFINITE (then nothing of this request is committed) */
} sled_result;

typedef struct sled_stats {
  int64_t steps, requests, tokens_scored, drafts_accepted, tokens_committed;
  int32_t pages_total, pages_free, contexts_open;
  int64_t kernels_launched;    /* device kernels launched by this engine so far */
  int64_t kernels_last_step;   /* ... by the last sled_verify_batch */
  /* device time of the last step by kind of kernel, filled while sled_debug_set_timing is on; ms_idle: stretches of
   * the step in which no kernel ran (mode 1 only) */
  float ms_linear, ms_attention, ms_accept, ms_other, ms_step;
  int32_t linear_launches_last_step, attention_launches_last_step;
  float ms_idle;
} sled_stats;

/* ---- the three calls of the verification service ---------------------------------- */

/* Creates an engine around the one target model that all devices share (Section 3.2: the
 * server holds a single large model; Section 3.4: it verifies the drafts of many devices
 * together): checks cfg, allocates weights, KV pool and workspaces on
 * cfg->device_index, copies the weights.  Errors: SLED_ERR_ARG, SLED_ERR_NO_DEVICE,
 * SLED_ERR_DEVICE (allocation failed: nothing is left allocated). */
int sled_init(const sled_weights* w, const sled_config* cfg, sled_engine** out);

/* One batched verification step (Sections 3.1, 3.4).  For request i the target is
 * evaluated at the k_i + 1 tokens [pending_i, d_1..d_k] in one ragged pass over all
 * requests (no padding to a common length); draft j of context i is decided with the
 * Philox4x32-10 uniforms of (seed, ctx_id, absolute position of that token), so a
 * request's outcome does not depend on its batch slot or on the other requests.
 * Afterwards the KV entries of pending_i and of the accepted drafts are kept, those
 * of the rejected drafts are dropped, pages left empty return to the pool, and
 * next_token becomes the context's pending token.  results: caller-allocated [n_reqs].
 * All requests are validated and all pages reserved before anything changes. */
int sled_verify_batch(sled_engine* e, const sled_request* reqs, int32_t n_reqs, uint64_t seed,
                      sled_result* results);

/* Closes a context - a device's conversation has ended, or the device has left (Section 3.2:
 * each device is served on its own sequence) - and returns its pages to the pool.  The paper
 * leaves cache management to future work (Section 5); this call is what frees it here.
 * Errors: SLED_ERR_UNKNOWN_CTX. */
int sled_release(sled_engine* e, uint64_t ctx_id);

/* ---- what makes the three usable --------------------------------------------------- */

/* Opens a context from a device's prompt (Section 3.2: prompts are tokenised on the
 * device): caches the keys/values of tokens[0..n-2]; tokens[n-1] becomes the pending
 * token, fed first by the next verification.  n >= 1. */
int sled_prefill(sled_engine* e, uint64_t ctx_id, const int32_t* tokens, int32_t n);

int sled_set_sampling(sled_engine* e, float temperature, int32_t greedy);
int sled_get_stats(sled_engine* e, sled_stats* out);
/* cudaStream_t all work of this engine is issued on (for timing with events). */
void* sled_get_stream(sled_engine* e);
void sled_shutdown(sled_engine* e);
const char* sled_strerror(int status);

/* ---- the server loop around the step (Section 3.4, Fig. 2: queue -> batch planner -> target model) -------- */

/* Batching policy of sled_step; batch_size is the fixed size a STATIC batch waits for (<= max_batch; ignored by
 * CONTINUOUS, the default).  Only while nothing is queued. */
int sled_server_config(sled_engine* e, int32_t policy, int32_t batch_size);
/* Queues one device's request and returns a ticket for it.  The draft tokens are copied; req->draft_probs is
 * borrowed until the ticket's result has been polled.  Checked here: k, token ids, that the context is open. */
int sled_submit(sled_engine* e, const sled_request* req, uint64_t* ticket);
/* Lets the batch planner take the next batch out of the queue (arrival order; one request per context and step;
 * at most max_batch requests and max_step_tokens tokens - the paper pads a batch to a common length, here it is
 * ragged) and verifies it with sled_verify_batch.  STATIC: does nothing while fewer than batch_size requests wait,
 * unless flush != 0.  *n_verified (may be NULL): requests verified by this call.  A request whose context has been
 * released or cut back since it was queued gets its own error status and does not stop the others; if the step
 * itself fails, every request of the batch is answered with that code, which is also returned. */
int sled_step(sled_engine* e, uint64_t seed, int32_t flush, int32_t* n_verified);
/* SLED_OK and the result if the ticket's request has been verified (the ticket is then forgotten), SLED_PENDING
 * while it is queued, SLED_ERR_ARG for an unknown ticket. */
int sled_poll(sled_engine* e, uint64_t ticket, sled_result* out);
/* Requests waiting in the queue. */
int32_t sled_queued(sled_engine* e);

/* The queue and batch planner alone (host only, no device needed): what sled_submit / sled_step use. */
sled_planner* sled_planner_create(int32_t policy, int32_t batch_size, int32_t max_batch, int32_t max_step_tokens);
void sled_planner_destroy(sled_planner* p);
int sled_planner_push(sled_planner* p, uint64_t ticket, uint64_t ctx_id, int32_t k);
/* Next batch, whole or not at all: its tickets into tickets_out (cap entries); returns their number, 0 if no
 * batch is due, SLED_ERR_BATCH_TOO_LARGE (queue unchanged) if cap is too small. */
int32_t sled_planner_next_batch(sled_planner* p, int32_t flush, uint64_t* tickets_out, int32_t cap);
int32_t sled_planner_queued(sled_planner* p);

/* Host only: how a step's requests are cut into attention work items (request, KV head, chunk of keys) - the paper's
 * batched verification (Section 3.4) leaves the scheduling of the batch on the GPU open.  n_keys[i]: keys request i
 * attends to (cached prefix + its k_i + 1 new tokens), q_tokens[i] = k_i + 1, group: query heads per KV head,
 * resident_blocks: blocks of the attention kernel the GPU holds at once (two per SM), part_rows_cap: most rows of
 * partial results.  chunk_keys_out[i] (caller-allocated, n_reqs entries): keys per item of request i, a multiple of 64;
 * a request is cut into ceil(n_keys / chunk) equal parts.  Returns SLED_ERR_ARG on null pointers or non-positive sizes. */
int sled_debug_plan_attention(const int64_t* n_keys, const int32_t* q_tokens, int32_t n_reqs, int32_t n_kv_heads,
                              int32_t group, int32_t resident_blocks, int64_t part_rows_cap, int64_t* chunk_keys_out);

/* ---- stand-alone pieces of the step (device-resident operands) ---------------------- */

/* Acceptance only (Eq. 1 + residual / bonus draw) on logits already in device memory.
 *   logits   DEVICE [n_rows][vocab] fp32, request i owns rows cu_rows[i] .. cu_rows[i+1]-1
 *            (k_i + 1 rows: row j scores draft j+1, the last one the bonus token)
 *   cu_rows  HOST [n_reqs+1];  drafts HOST [n_rows - n_reqs] packed request after request
 *   q_rows   DEVICE [sum k_i][vocab] fp32 packed the same way (NULL if greedy)
 *   ctx_ids, pos0 HOST [n_reqs]: Philox counter words; pos0 = index of the pending token
 *   results  HOST [n_reqs]
 * stream: cudaStream_t or NULL for the default stream.  device_ms (may be NULL) receives the
 * kernel's duration measured with events on that stream.  Synchronises before returning. */
int sled_accept_rows(const float* logits, const int32_t* cu_rows, const int32_t* drafts, const float* q_rows,
                     const uint64_t* ctx_ids, const int64_t* pos0, int32_t n_reqs, int32_t vocab,
                     float temperature, int32_t greedy, uint64_t seed, sled_result* results, void* stream,
                     float* device_ms);

/* The same acceptance as sled_accept_rows for callers that must not allocate device memory
 * (the paper has no counterpart: this is a property of the library, not of the method).
 * A process whose GPU memory is wholly owned by another allocator, a latency path on which an
 * allocation would stall the device, or a caller between two points of a fixed schedule cannot
 * afford the cudaMalloc / cudaFree pair that sled_accept_rows performs for its small device-side
 * description of the batch.  Here that description lives in a fixed array inside the library
 * image: SLED_STATIC_MAX_REQS requests and SLED_STATIC_MAX_ROWS rows at most (just under 69 KB, held
 * by every GPU that loads the library until the process ends; the call also builds a host image
 * of that size on the caller's stack).  Larger batches are refused with
 * SLED_ERR_BATCH_TOO_LARGE.  The call allocates nothing on the device and nothing on the host
 * heap; it does not measure time.  Arguments and results are those of sled_accept_rows.
 * Every call must be made with the device that holds `logits` current (checked: SLED_ERR_ARG
 * otherwise).  The first call on a device looks up the array's device address; make that first
 * call before starting any stream capture, and from one thread.  All calls on a device share the one
 * array and every call rewrites it completely, so two calls must not overlap on the GPU: issue
 * them from one thread, one after the other (the call synchronises `stream` before returning). */
#define SLED_STATIC_MAX_REQS 1024
#define SLED_STATIC_MAX_ROWS 8192
int sled_accept_rows_static(const float* logits, const int32_t* cu_rows, const int32_t* drafts, const float* q_rows,
                            const uint64_t* ctx_ids, const int64_t* pos0, int32_t n_reqs, int32_t vocab,
                            float temperature, int32_t greedy, uint64_t seed, sled_result* results, void* stream);

/* Ragged verification attention only, over the engine's paged cache: request i's last
 * q_len[i] cached tokens are taken as the new ones; query j of request i attends to the
 * keys 0 .. n_kv_i - q_len_i + j of ctx_ids[i] in layer `layer`.
 *   q    DEVICE [sum q_len][n_q_heads][head_dim] in the activation type (bf16 with bf16 weights)
 *   out  DEVICE same shape and type.
 * device_ms (may be NULL) receives the duration of the attention kernels (events on the
 * engine's stream).  Synchronises before returning. */
int sled_attention_ragged(sled_engine* e, int32_t layer, const uint64_t* ctx_ids, const int32_t* q_len,
                          int32_t n_reqs, const void* q, void* out, float* device_ms);

/* ---- operators over a paged cache (device-resident operands) ------------------------- */

/* A cache that the caller owns, in the layout of the engine's pool: K and V are [n_layers][n_pages][n_kv_heads][page_size]
 * [head_dim], contiguous, 16-byte aligned; key x of request i lies in page page_table[i][x / page_size] at slot
 * x % page_size, for every layer and KV head.  The paper leaves the cache to future work (Section 5); these operators are
 * what a server needs of it beyond the chain drafts of sled_verify_batch.  They serve a caller that holds its cache and runs
 * its model itself: the pool of a sled_engine has no address outside, and its calls know chains only.
 *
 * All arrays, the request descriptions included, are DEVICE memory of one GPU; the calls enqueue their kernels on `stream`
 * (cudaStream_t or NULL for the default stream) and return without waiting, so they can be captured into a CUDA graph.
 * The GPU that holds k is used, whichever device is current.  What the host can see is checked before anything is
 * launched (SLED_ERR_ARG; SLED_ERR_NO_DEVICE without a GPU).  What only the GPU can see is checked by the kernels: a
 * request whose numbers do not hold together - n_kv beyond its table row, fewer keys than rows, rows outside the call, a
 * tree of more than SLED_MAX_TREE_NODES nodes - is left out; a page outside the pool is read as page 0 and never written
 * (eviction leaves its request out), and a parent that is not an earlier node makes its node unused.  Each of these, and a
 * device-side wait that runs out, sets *status (DEVICE, one int32, may be NULL) to the sled_status if it was 0; no call
 * clears it.  Entries of a table row behind the request's
 * last page, slots behind its last key and pages of nobody are never looked at, or do not change results whatever they
 * hold.  A page belongs to at most one request, once, of a call that writes to the cache or to key_weights (others may share
 * pages; of a page that requests share with different numbers of keys sled_block_bounds leaves the bounds of either); out,
 * lse and key_weights share no memory with what the call reads.  n_reqs, n_layers, n_kv_heads and n_q_heads are at most
 * 65535; arrays without entries may be NULL.
 * Scores, their maxima and sums, results and weights are held in fp32; over a bf16 cache the softmax's numerators are rounded
 * to bf16 before they meet V (their sum is not), one rounding of at most 2^-8 of each.
 * workspace: at least the bytes that the call's _workspace function names, 256-byte aligned, used from the call until its
 * kernels have run: calls (or captured graphs) that may run at the same time need a workspace each.  It need not be
 * cleared and nothing in it outlives the call.  Its size goes by table_cols * page_size, and so does how the weights of keys
 * are formed: scores of all rows over so many keys are kept up to 512 MiB, beyond that they are formed anew key by key, which
 * takes many times as long.  A table should be about as wide as its longest request. */
#define SLED_MAX_TREE_NODES 128
typedef struct sled_paged_kv {
  void* k;
  void* v;                    /* may be NULL for sled_block_bounds */
  int32_t dtype;              /* sled_dtype of k and v, and of q, out and bounds */
  int32_t n_layers;           /* 1, but for sled_evict_keys */
  int32_t n_pages, n_kv_heads;
  int32_t page_size;          /* a multiple of 16, at most 256 */
  int32_t head_dim;           /* 32, 64 or 128 */
  const int32_t* page_table;  /* [n_reqs] rows of table_cols entries, table_stride entries apart */
  int32_t table_stride, table_cols;   /* table_cols * page_size at most 2^31 - 1025 */
  const int32_t* n_kv;        /* [n_reqs] cached keys */
  int32_t n_reqs;
} sled_paged_kv;

/* Attention of drafted trees.  Request i's newest cu_q[i+1] - cu_q[i] keys are the nodes of a tree of drafted tokens,
 * parents before children; row cu_q[i] + j is node j.  It sees the request's older keys, itself and its ancestors.
 * parents[cu_q[i] + j]: node j's parent as an index among the request's nodes, -1: it follows the older keys directly,
 * -2: the node is unused - its row is 0 (lse -infinity) and nobody sees it, nor those that hang on it.  parents NULL: every request is a
 * chain (row j sees the keys up to its own), of any length.  Softmax in fp32 over scale * q.k; scale 0: 1/sqrt(head_dim).
 *   q, out  [n_rows][n_q_heads][head_dim], rows q_stride / out_stride elements apart (even numbers of bf16 elements,
 *           4-byte aligned), n_rows * n_q_heads below 2^31; rows that belong to no request are left alone
 *   lse     [n_rows][n_q_heads] fp32: natural logarithm of the sum of exponentials; may be NULL
 *   key_weights  may be NULL; [n_pages][n_kv_heads][page_size] fp32: every key's attention weight, summed over the
 *           request's rows and the heads that share the KV head, is added to its entry */
int sled_attention_tree_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t weigh, int64_t* bytes);
int sled_attention_tree(const sled_paged_kv* kv, const void* q, int64_t q_stride, const int32_t* cu_q, const int32_t* parents,
                        int32_t n_rows, int32_t n_q_heads, float scale, void* out, int64_t out_stride, float* lse,
                        float* key_weights, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream);

/* Eviction by accumulated attention weight, in all layers at once.  Where request i has more than `budget` keys, every
 * (layer, KV head) keeps for itself its first n_sink slots, its last n_recent and, of those between, the
 * budget - n_sink - n_recent with the largest key_weights (the lower slot among equals; a NaN counts as the largest).
 * They end up in the slots 0 .. budget-1: kept keys below budget - n_recent stay where they are, the places that became
 * free there take the other kept ones, both in ascending order, and the last n_recent follow in their order.  The order of the
 * older keys is of no consequence (a key carries its position).  Requests within the budget are left as they are.  The
 * caller goes on with min(n_kv, budget) keys.
 *   key_weights      [n_layers][n_pages][n_kv_heads][page_size] fp32
 *   key_weights_out  the weights of the kept keys, at their new slots: key_weights itself, or an array that does not
 *                    overlap it (then requests within the budget are copied).  Entries of slots behind the kept keys are left
 *                    as they are: a caller that adds weights up clears those of the keys it appends */
int sled_evict_keys_workspace(const sled_paged_kv* kv, int64_t* bytes);
int sled_evict_keys(const sled_paged_kv* kv, float* key_weights, float* key_weights_out, int32_t budget, int32_t n_sink,
                    int32_t n_recent, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream);

/* Smallest and largest key of every block (page), per KV head and dimension: bounds [n_pages][n_kv_heads][2][head_dim] of
 * the cache's type, 16-byte aligned.  Written for the blocks that hold any of request i's keys first[i] .. n_kv[i]-1 (first
 * NULL: all; none where first[i] >= n_kv[i]); a NaN among the keys gives NaN. */
int sled_block_bounds(const sled_paged_kv* kv, const int32_t* first, void* bounds, int32_t* status, void* stream);

/* Attention over the blocks that a cheap score selects for each query.  Chains as in sled_attention_tree without parents:
 * row j of request i is the key x = n_kv[i] - q_len + j and sees no key behind it.  It reads the n_local blocks that end
 * with its own and, of the earlier ones, the n_blocks - n_local of largest score - the largest, over the heads that share
 * the KV head, of sum_d max(q_d low_d, q_d high_d), which no q.k of the block exceeds - the lower block among equals, a
 * NaN being the largest.  Scores are fp32 sums: blocks whose scores are nearer than their rounding may change places.
 * Where there are no more than n_blocks blocks the result is that of full attention.
 *   bounds  as sled_block_bounds leaves them, for every block before a query's last n_local
 *   1 <= n_local <= n_blocks
 *   blocks  may be NULL; [n_rows][n_kv_heads][n_blocks]: the blocks that were read, ascending; entries behind a row's own
 *           block count are left alone */
int sled_attention_blocks_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int32_t n_blocks, int64_t* bytes);
int sled_attention_blocks(const sled_paged_kv* kv, const void* bounds, const void* q, int64_t q_stride, const int32_t* cu_q,
                          int32_t n_rows, int32_t n_q_heads, float scale, int32_t n_blocks, int32_t n_local, void* out,
                          int64_t out_stride, int32_t* blocks, int32_t* status, void* workspace, int64_t workspace_bytes,
                          void* stream);

/* ---- a decoding step over a cache of one's own: places, positions, keys, attention ------------------------------- */

/* What a step does with a caller's cache besides its model: sled_page_slots gives the new tokens their places,
 * sled_rotary turns their queries and keys, sled_append_keys writes keys and values into the cache, sled_attention_tree (or,
 * for caches in 8 bits, sled_attention_scaled) reads it.  As above: DEVICE memory of one GPU unless said otherwise, enqueued
 * on `stream` without waiting, capturable, *status for what only the GPU sees, nothing kept from call to call. */

/* Places of a step's tokens, from lengths that only the GPU knows.  Request i has n_kv[i] keys in the pages of its table row;
 * n_keep[i] of them stay (those of rejected drafts go; n_keep NULL: all stay), n_new[i] tokens follow.  Pages that a request
 * no longer needs go onto the stack of free pages, request by request, a request's in ascending order; then pages that
 * requests need come off its top, request by request.  (A page belongs to one request.)
 *   page_size    1 or more;  page_table [n_reqs] rows of table_cols entries, table_stride apart, entries written where a
 *                request gets a page; entries of pages that went back are left as they are
 *   free_pages   [free_cap], the first *n_free of them free, the top last.  Returned pages are written at *n_free and on;
 *                nothing else of it is.  free_cap has to hold the free and the returned ones together
 *   n_kv_out     [n_reqs]  n_keep + n_new
 *   n_free_out   [1]
 *   cu_q         [n_reqs + 1]  row offsets of the new tokens
 *   positions    [n_rows]  n_keep[i] + j of token j of request i; may be NULL
 *   slots        [n_rows]  page * page_size + offset within the page; may be NULL
 *   n_rows       room for the tokens of the call; rows behind the last token get position 0 and slot -1
 * All or nothing: where *n_free or any request's numbers do not hold together (negative, n_keep above n_kv, more keys than
 * its table row has room for, more tokens than n_rows) - SLED_ERR_ARG - or the free pages do not suffice -
 * SLED_ERR_NO_PAGES -, *status is set, no page moves, n_kv_out is n_kv, n_free_out is *n_free and nobody has a row.
 * Outputs share no memory with inputs or each other: the same call can be made, or replayed, again. */
int sled_page_slots(const int32_t* n_kv, const int32_t* n_keep, const int32_t* n_new, int32_t n_reqs, int32_t page_size,
                    int32_t* page_table, int32_t table_stride, int32_t table_cols, int32_t* free_pages, int32_t free_cap,
                    const int32_t* n_free, int32_t* n_kv_out, int32_t* n_free_out, int32_t* cu_q, int32_t* positions,
                    int64_t* slots, int32_t n_rows, int32_t* status, void* stream);

/* Radians per position of the pairs of rotary embeddings: f[i] = theta^(-2i/rot_dim), i < rot_dim/2, scaled for contexts
 * longer than those of the training.  Host only, needs no device.
 *   SLED_ROTARY_PLAIN    f
 *   SLED_ROTARY_LINEAR   f / factor
 *   SLED_ROTARY_BASE     theta * factor^(d/(d-2)) in theta's place (rot_dim d above 2): the lowest frequency is f / factor
 *   SLED_ROTARY_BANDS    f (s + (1 - s) / factor), s = clamp((t - low) / (high - low), 0, 1) of the turns t = length f / 2 pi that
 *                        the pair makes in the context length of the training; 0 <= low < high
 *   SLED_ROTARY_RAMP     the same with s falling from 1 to 0 along the pairs' index, between the (rounded down) index of the
 *                        pair that makes `high` turns and the (rounded up) one of `low` turns; 0 < low < high, theta above 1.
 *                        amplitude is 0.1 ln(factor) + 1 for factor above 1
 * rot_dim: even, 2 .. 512; factor, length above 0 (factor for all but PLAIN, length for the last two).  frequencies: HOST [rot_dim/2]; amplitude: HOST,
 * receives what cosine and sine are multiplied by (1 but for RAMP); may be NULL. */
enum sled_rotary_scaling { SLED_ROTARY_PLAIN = 0, SLED_ROTARY_LINEAR = 1, SLED_ROTARY_BASE = 2, SLED_ROTARY_BANDS = 3, SLED_ROTARY_RAMP = 4 };
int sled_rotary_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double length, double low, double high,
                            double* frequencies, double* amplitude);

/* Rows of heads: element d of head g of row t lies at t * row + g * head + d.  `out` may be `in`, with the same strides;
 * otherwise they, and the elements of out among each other, share no memory. */
typedef struct sled_heads {
  const void* in;
  int64_t in_row, in_head;
  void* out;
  int64_t out_row, out_head;
  int32_t n_heads;
} sled_heads;

/* Rotary positions of queries and keys.  The first rot_dim dimensions of every head are pairs - (2i, 2i+1) or the two halves
 * (i, i + rot_dim/2) -, and pair i of row t is turned by the angle positions[t] * frequencies[i]:
 *   (a, b) -> amplitude (a cos - b sin, a sin + b cos);  dimensions behind rot_dim are copied.
 * transpose: the angle is taken negative, which is the gradient of the call without it (and, with amplitude 1, undoes it).
 * Angles are formed in 64 bits, whatever the position: off by 3 2^-53 of their size, 2^-20.4 at 2^31.  A pair is turned in 32 bits
 * and rounded once.
 *   dtype        SLED_F32 or SLED_BF16, of all of q and k;  k may be NULL
 *   positions    [n_rows], any numbers
 *   frequencies  [rot_dim/2] fp64
 *   head_dim     even, at most 512; rot_dim even, 2 .. head_dim */
enum sled_rotary_pairs { SLED_ROTARY_PAIRS = 0, SLED_ROTARY_HALVES = 1 };
int sled_rotary(const sled_heads* q, const sled_heads* k, int32_t n_rows, int32_t head_dim, int32_t dtype, const int32_t* positions,
                const double* frequencies, int32_t rot_dim, int32_t pairs, float amplitude, int32_t transpose, void* stream);

/* New keys and values into the cache: row cu_q[i] + j of k and v is request i's key n_kv[i] - q_len + j (n_kv counts the new
 * ones), as in the attention calls.  Rows of k and v [n_rows][n_kv_heads][head_dim], k_stride / v_stride elements apart.
 * A cache of the rows' type (rows_dtype SLED_F32 or SLED_BF16) receives them as they are; k_scale and v_scale are then NULL.
 * A cache in 8 bits (SLED_E4M3) holds codes and a scale for every block of 16 slots of a page and KV head, k_scale and
 * v_scale [n_pages][n_kv_heads][page_size / 16] fp32: a key is scale * code.  The scale of a block that receives keys becomes
 * the smallest power of two, at least 2^-126, of which 448 times is no less than any new finite element of the block or, where
 * the block has older keys of the request, the size of the scale that it had, if that is larger; older keys are coded anew where
 * the scale changes.  A code is the nearest to element / scale, ties to the even one (a quotient by a caller's own scale that is no
 * power of two is rounded to 32 bits first); infinities and NaN become NaN.  What a rejected draft did to a
 * scale stays until its block is begun anew.
 * Slots behind the last key and other pages are left as they are; the rows lie outside of the cache, and no two requests of a
 * call write into one page.  A request whose numbers do not hold together is left out, a
 * page outside the pool is not written; *status says so. */
#define SLED_SCALE_BLOCK 16
int sled_append_keys(const sled_paged_kv* kv, float* k_scale, float* v_scale, const void* k, int64_t k_stride, const void* v,
                     int64_t v_stride, int32_t rows_dtype, const int32_t* cu_q, int32_t n_rows, int32_t* status, void* stream);

/* sled_attention_tree over a cache in 8 bits (kv->dtype SLED_E4M3, with its scales as in sled_append_keys: any finite
 * numbers).  q and out are bf16; parents, lse, status and workspace as there.  Scores, their maxima and sums are held in fp32, of
 * queries whose elements below 2^-31 of their row's largest in size are off by up to 2^-39 of that (the others are exact);
 * the softmax's numerators, times their block's scale, are rounded to fp16 before they meet V (their sum is not): by 2^-11 of
 * each at most, or by 2^-32 of the row's largest where that is more.  Keys of less than 2^-111 of the row's largest probability may
 * count as less than that.  Outputs are sums of exponentials, of 2^8 at most, times values until they are divided by the sum of the
 * exponentials: these sums must be below 2^128. */
int sled_attention_scaled_workspace(const sled_paged_kv* kv, int32_t n_rows, int32_t n_q_heads, int64_t* bytes);
int sled_attention_scaled(const sled_paged_kv* kv, const float* k_scale, const float* v_scale, const void* q, int64_t q_stride,
                          const int32_t* cu_q, const int32_t* parents, int32_t n_rows, int32_t n_q_heads, float scale, void* out,
                          int64_t out_stride, float* lse, int32_t* status, void* workspace, int64_t workspace_bytes, void* stream);

/* ---- test and benchmark hooks ------------------------------------------------------- */

/* Opens a context with given cache content instead of a prefill.  K, V: HOST or DEVICE,
 * [n_layers][n_tokens][n_kv_heads][head_dim] of kv_dtype. */
int sled_debug_load_kv(sled_engine* e, uint64_t ctx_id, const void* K, const void* V, int32_t n_tokens,
                       int32_t pending);
/* Reads one layer's cache of a context back: K, V HOST [n_tokens][n_kv_heads][head_dim] of kv_dtype. */
int sled_debug_read_kv(sled_engine* e, uint64_t ctx_id, int32_t layer, void* K, void* V, int32_t n_tokens);
/* Copies the logits of the last step, rows [0, n_rows), to dst (HOST or DEVICE) [n_rows][vocab] fp32. */
int sled_debug_copy_logits(sled_engine* e, float* dst, int32_t n_rows);
/* Sets a context back to n_kv cached tokens (<= its current count) and a pending token. */
int sled_debug_truncate(sled_engine* e, uint64_t ctx_id, int64_t n_kv, int32_t pending);
/* The same for n contexts in one call (ctx_ids, n_kv, pending: HOST arrays [n]); stops at the first error. */
int sled_debug_truncate_batch(sled_engine* e, const uint64_t* ctx_ids, const int64_t* n_kv, const int32_t* pending,
                              int32_t n);
/* Self-test of the recovery from a device-side wait that runs out (engines with bf16 weights).  Every wait inside
 * the tensor-core and attention kernels is bounded: when one expires the kernel records a code, kernels that follow
 * return early, and sled_verify_batch returns SLED_ERR_DEVICE with every context, page and counter as before.  This
 * call arms that path without any fault: the next sled_verify_batch starts with a small kernel that waits limit_us
 * microseconds (<= 100000) on a barrier nobody signals, using the kernels' own bounded wait.  That step fails as
 * described; the one after it runs normally. */
int sled_debug_arm_wait_timeout(sled_engine* e, int32_t limit_us);
/* commit = 0: verification steps leave every context as it was (repeatable timing). */
int sled_debug_set_commit(sled_engine* e, int32_t commit);
/* Device time per kind of kernel into sled_stats.  mode 0: off.  mode 1: every launch stamps the GPU's global timer
 * when its first block begins and its last block ends; launches keep overlapping as they do untimed, and a launch
 * is charged the time by which it extends the step beyond all earlier launches (the parts add up to ms_step).
 * mode 2: CUDA events between kernel groups, which serialises neighbouring launches (each kernel's stand-alone
 * duration; the parts add up to more than an untimed step). */
int sled_debug_set_timing(sled_engine* e, int32_t mode);
/* Context state: cached tokens, pending token, owned pages (ids into pages_out, up to cap). */
int sled_debug_query_ctx(sled_engine* e, uint64_t ctx_id, int64_t* n_kv, int32_t* pending, int32_t* n_pages,
                         int32_t* pages_out, int32_t cap);

/* Permutes the free-page list (seeded), so contexts opened afterwards get physically scattered pages. */
int sled_debug_shuffle_pages(sled_engine* e, uint64_t seed);

/* ---- host-side KV page manager (no device needed) ----------------------------------- */
/* The bookkeeping the engine uses for commit / rollback, exported so it can be
 * exercised alone.  A context owns ceil(tokens / page_size) pages; pages are handed out
 * and returned whole; a batch reservation either fits entirely or changes nothing. */
sled_kvm* sled_kvm_create(int32_t n_pages, int32_t page_size);
void sled_kvm_destroy(sled_kvm* m);
int sled_kvm_open(sled_kvm* m, uint64_t ctx_id, int64_t n_kv, int32_t pending);
/* Reserves room for extra[i] more tokens behind the cached ones of each context. */
int sled_kvm_reserve_batch(sled_kvm* m, const uint64_t* ctx_ids, const int32_t* extra, int32_t n);
/* Keeps n_keep of the reserved tokens, returns pages that no longer hold any, sets pending. */
int sled_kvm_commit(sled_kvm* m, uint64_t ctx_id, int32_t n_keep, int32_t pending);
int sled_kvm_release(sled_kvm* m, uint64_t ctx_id);
int sled_kvm_query(sled_kvm* m, uint64_t ctx_id, int64_t* n_kv, int32_t* pending, int32_t* n_pages,
                   int32_t* pages_out, int32_t cap);
int32_t sled_kvm_free_pages(sled_kvm* m);
/* As sled_kvm_reserve_batch, with request i continuing the first base_len[i] committed tokens of its context
 * (0: its current end; see sled_request.base_len): the context is cut back first.  All or nothing. */
int sled_kvm_reserve_batch_at(sled_kvm* m, const uint64_t* ctx_ids, const int32_t* extra, const int64_t* base_len,
                              int32_t n);
/* As sled_kvm_commit, recording the kept tokens: kept[0 .. n_keep-2] are the tokens behind the old pending one
 * whose cache entries stay (the accepted drafts), then `pending`. */
int sled_kvm_commit_tokens(sled_kvm* m, uint64_t ctx_id, int32_t n_keep, int32_t pending, const int32_t* kept);
/* The known committed tokens of a context: they start at sequence index *hist_start, the last one is pending. */
int sled_kvm_history(sled_kvm* m, uint64_t ctx_id, int64_t* hist_start, int32_t* n_tokens, int32_t* tokens_out,
                     int32_t cap);
/* Ragged packing of one step: for request i with k[i] drafts, writes token rows
 * cu_q[i] .. cu_q[i+1]-1 (row 0 = pending token, then the drafts): ids, owning request,
 * absolute position and physical cache slot (page * page_size + offset).  Pages must have
 * been reserved.  Output arrays: cu_q [n+1], others [sum(k_i+1)]. */
int sled_kvm_pack(sled_kvm* m, const uint64_t* ctx_ids, const int32_t* k, const int32_t* const* drafts, int32_t n,
                  int32_t* cu_q, int32_t* ids, int32_t* tok_req, int32_t* tok_pos, int32_t* tok_slot);

#ifdef __cplusplus
}
#endif
#endif /* SLED_H_ */
