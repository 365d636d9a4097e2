/*
 * crf.h -- C ABI of the GB300 bounded KV-cache recomputation library
 * (CacheReforge, arXiv 2609.30884).
 *
 * The library executes the data-parallel hot path of stale-KV-cache recovery
 * under an evolving LoRA adapter:
 *
 *   crf_recompute_window  Section 4.2 "Executable restart": feed the retained
 *                         boundary state H_{s-1} (the token embedding when
 *                         s = 0; H_{-1} in Section S1.1) to layers s..e-1 over
 *                         the complete prefix under the current adapter, and
 *                         overwrite exactly those layers' K/V (Eq. 1 cache,
 *                         Eq. S1 per-layer maps F_l / G_l, Eq. S3 projections).
 *                         Optionally continues the last prefix row through
 *                         layers e..N-1 against the historical cache, which
 *                         gives the first-step next-token state used for
 *                         fidelity (Section 3.1, Section S2.1).
 *   crf_drift             Eq. 8: per (layer, module) squared displacement of
 *                         the current adapter from each layer's anchor.
 *   crf_kl                Section S2.1: forward KL(p* || p) at the first
 *                         generated-token step, fresh logits as reference.
 *   crf_decode_step       one generated token per request on the recovered
 *                         (mixed-version) paged cache: the step that consumes
 *                         the refreshed cache (Section 3.1, first generated
 *                         tokens); greedy next token and optional logits.
 *
 * Conventions (every entry point):
 *   - Device pointers are CUDA device memory on the context's device; host
 *     arrays (the per-layer pointer tables) are read during the call only.
 *     The caller owns every buffer. The library keeps no pointer after it
 *     returns and allocates no device memory inside these calls: temporaries
 *     live in the caller's workspace (see crf_workspace_size).
 *   - `stream` is a cudaStream_t (NULL = legacy default stream). Work is
 *     enqueued on it; results are valid once the stream has synchronised.
 *   - Every argument the host can see is validated before anything is
 *     launched. A non-OK status from that validation (CRF_EINVAL,
 *     CRF_ESHAPE, CRF_EUNSUPPORTED, CRF_ENOMEM) means nothing was enqueued
 *     and nothing was written. A CRF_ECUDA from a failed launch can leave the
 *     call's earlier kernels enqueued; their outputs are then undefined.
 *     crf_last_error() returns a message in either case (thread-local).
 *   - Page tables live in device memory and the host never reads them: no
 *     call waits on its stream (crf_check alone synchronises). The first
 *     kernel of crf_recompute_window and crf_decode_step checks every page
 *     id (inside [0, num_pages), no page twice across the call's tables);
 *     a failure makes every later kernel of that call return at once, so the
 *     call writes nothing outside its workspace (pool pages, checkpoints,
 *     final rows, logits, tokens), and the next crf_check returns CRF_EINVAL.
 *   - A context is used by one host thread at a time: its device status word
 *     and timing state are shared by its calls. Separate contexts may run
 *     concurrently.
 *   - A kernel that gives up on a bounded internal wait records it in the
 *     context; crf_check() reports it as CRF_ETIMEOUT. An asynchronous CUDA
 *     error is reported as CRF_ECUDA by the next call.
 *   - Ids read from device memory are checked where they are used. A token id
 *     outside [0, vocab) is read as token 0 and recorded; crf_check() then
 *     returns CRF_EINVAL. A library built with CRF_DEBUG defined
 *     (libcrf_debug.so) also checks every page id again at each device-side
 *     use, reads or writes page 0 in place of a bad id and records it the
 *     same way.
 *   - Tensors are row-major, bf16 unless stated. Weights are [out, in].
 */
#ifndef CRF_H
#define CRF_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define CRF_API __attribute__((visibility("default")))
#else
#define CRF_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum crf_status {
  CRF_OK = 0,
  CRF_EINVAL = 1,        /* bad argument (null pointer, window out of range, ...) */
  CRF_ESHAPE = 2,        /* shapes inconsistent with each other or with the buffers */
  CRF_EUNSUPPORTED = 3,  /* valid but not implemented (head_dim, rank, alignment, ...) */
  CRF_ENOMEM = 4,        /* workspace too small */
  CRF_ECUDA = 5,         /* CUDA runtime / driver error */
  CRF_ETIMEOUT = 6       /* a kernel abandoned a bounded wait */
} crf_status;

/* Projection index order used by every per-module table. */
enum {
  CRF_MOD_Q = 0, CRF_MOD_K = 1, CRF_MOD_V = 2, CRF_MOD_O = 3,
  CRF_MOD_GATE = 4, CRF_MOD_UP = 5, CRF_MOD_DOWN = 6, CRF_NUM_MODULES = 7
};

#define CRF_PAGE_SIZE 16   /* tokens per KV page */
#define CRF_MAX_REQUESTS 32

/* Decoder shape (Qwen2.5 family, Section 5.1): pre-norm RMSNorm, rotate-half
 * RoPE, grouped-query causal attention, SwiGLU MLP. head_dim must be 64 or
 * 128; n_q_heads a multiple of n_kv_heads. */
typedef struct crf_model_dims {
  int n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab;
  float rms_eps, rope_theta;
  int qkv_bias;          /* 1: q/k/v projections carry a bias */
} crf_model_dims;

/* LoRA adapter shape: every adapted module m (bit m of module_mask) uses
 * W_m + (alpha / rank) * B_m A_m, kept unmerged. rank must be 4, 8 or 16. */
typedef struct crf_lora_dims {
  int rank;
  float alpha;
  uint32_t module_mask;
} crf_lora_dims;

/* Base weights of one layer (device pointers, bf16):
 *   W[m]    [out_m, in_m]   q:[Hq*d,h] k,v:[Hkv*d,h] o:[h,Hq*d] gate,up:[f,h] down:[h,f]
 *   bias[j] [out_j] for q,k,v (j = 0..2), used iff dims.qkv_bias
 * Every W[m] and bias[j] starts on a 16-byte boundary (CRF_EINVAL otherwise).
 *   ln1/ln2 [h] RMSNorm gains before attention / before the MLP. */
typedef struct crf_layer_weights {
  const void* W[CRF_NUM_MODULES];
  const void* bias[3];
  const void* ln1;
  const void* ln2;
} crf_layer_weights;

typedef struct crf_model {
  crf_model_dims dims;
  const crf_layer_weights* layers;  /* host array [n_layers] */
  const void* embed;                /* [vocab, h]; read when a window starts at layer 0 */
  const void* final_norm;           /* [h]; read by crf_kl with a model */
  const void* lm_head;              /* [vocab, h]; read by crf_kl with a model */
} crf_model;

/* One adapter version theta_t. A/B are host arrays [n_layers * 7] of device
 * pointers, entry l*7+m: A [rank, in_m], B [out_m, rank] (bf16); NULL for
 * modules outside module_mask. */
typedef struct crf_adapter {
  crf_lora_dims dims;
  const void* const* A;
  const void* const* B;
} crf_adapter;

/* Paged KV pool shared by all requests: per layer one K and one V pool,
 * bf16 [num_pages][n_kv_heads][16][head_dim], keys stored after rotation.
 * Token t of a request lives at page page_table[t / 16], slot t % 16. */
typedef struct crf_kv_pool {
  void* const* k_pages;   /* host array [n_layers] of device pointers */
  void* const* v_pages;   /* host array [n_layers] of device pointers */
  int num_pages;
} crf_kv_pool;

/* One cached prefix to refresh over the window [s, e) (0 <= s <= e <= N).
 *   page_table        device int32 [ceil(n_tokens/16)], distinct ids < num_pages
 *   tokens            device int32 [n_tokens]; required iff s == 0; ids in [0, vocab)
 *   hidden_in         device [n_tokens, h] = H_{s-1}; required iff s > 0
 *   hidden_out        NULL, or host array [e-s] of device [n_tokens, h]
 *                     buffers receiving H_s..H_{e-1} (refreshed checkpoints)
 *   final_hidden_out  NULL, or device [h]: the last prefix row carried
 *                     through layers e..N-1 against those layers' cached K/V
 *                     (reads the pool, writes nothing to it). s == e is
 *                     allowed only with final_hidden_out (direct reuse).
 * Pages of different requests must not overlap. */
typedef struct crf_request {
  int n_tokens, s, e;
  const int32_t* page_table;
  const int32_t* tokens;
  const void* hidden_in;
  void* const* hidden_out;
  void* final_hidden_out;
} crf_request;

typedef struct crf_ctx crf_ctx;

/* Create a context bound to CUDA device `device` (allocates a small status
 * word and queries device properties). */
CRF_API crf_status crf_create(crf_ctx** out, int device);
CRF_API crf_status crf_destroy(crf_ctx* ctx);

/* Message for the last non-OK status returned on this thread. */
CRF_API const char* crf_last_error(void);

/* Synchronise `stream`, then report what the kernels recorded since the last
 * check: a rejected page table or a failed device-side bounds check
 * (CRF_EINVAL, which takes precedence) or an abandoned bounded wait
 * (CRF_ETIMEOUT); else a pending CUDA error (CRF_ECUDA). The record is
 * cleared. */
CRF_API crf_status crf_check(crf_ctx* ctx, void* stream);

/* Failure-path self-test (no counterpart in the paper): launches one block on
 * `stream` whose wait on a barrier that nothing completes runs out after the
 * library's bounded-wait limit (2 s), exactly as a stalled kernel of the hot
 * path would; the next crf_check then returns CRF_ETIMEOUT and clears the
 * report, and the context stays usable. No fault is raised on the GPU. */
CRF_API crf_status crf_selftest_timeout(crf_ctx* ctx, void* stream);

/* Workspace bytes crf_recompute_window needs for these requests. */
CRF_API crf_status crf_workspace_size(crf_ctx* ctx, const crf_model* model, const crf_lora_dims* lora,
                              const crf_request* reqs, int n_req, size_t* bytes);

/* Bounded recomputation of every request's window (Section 4.2), batched:
 * at each layer the rows of all requests whose window covers it run as one
 * set of GEMMs; attention, RoPE and the page writes are per request.
 * `workspace` is device memory of at least crf_workspace_size bytes, 256-byte
 * aligned. */
CRF_API crf_status crf_recompute_window(crf_ctx* ctx, const crf_model* model, const crf_adapter* cur,
                                const crf_kv_pool* pool, const crf_request* reqs, int n_req,
                                void* workspace, size_t ws_bytes, void* stream);

/* One generation step for each row (the decoding that consumes the recovered
 * cache, Section 2.1; the first generated token is where Section S2.1 measures
 * KL and top-1): the token at position `pos` (the number
 * of positions already cached for that request) is embedded and carried through
 * layers 0..N-1 under `cur`; at every layer it attends to the cached keys and
 * values at positions 0..pos-1 of its page table plus its own, and its post-RoPE
 * K and V are written into slot pos % 16 of page page_table[pos / 16] of that
 * layer (so the next step sees them). The final row goes through the final norm
 * and the LM head; next_tokens[i] = argmax of row i's logits (lowest index
 * among equal maxima).
 *   page_table: device int32 [pos / 16 + 1]; pages must be distinct across rows.
 *   token:      device int32, one entry: the input token id of the row, in [0, vocab).
 * next_tokens: device int32 [n_rows]. logits: NULL or device fp32 [n_rows][vocab].
 * The model needs embed, final_norm and lm_head; 1 <= n_rows <= CRF_MAX_REQUESTS.
 * `workspace` >= crf_decode_workspace_size bytes, 256-byte aligned. */
typedef struct {
  int pos;
  const int32_t* page_table;
  const int32_t* token;
} crf_decode_row;
CRF_API crf_status crf_decode_workspace_size(crf_ctx* ctx, const crf_model* model, const crf_lora_dims* lora,
                                     const crf_decode_row* rows, int n_rows, size_t* bytes);
CRF_API crf_status crf_decode_step(crf_ctx* ctx, const crf_model* model, const crf_adapter* cur,
                           const crf_kv_pool* pool, const crf_decode_row* rows, int n_rows,
                           int32_t* next_tokens, float* logits, void* workspace, size_t ws_bytes,
                           void* stream);

/* Eq. 8 drift. anchors: host array [n_layers] of adapters (anchors[l] is the
 * version that produced layer l's cache; all of the same lora dims as cur).
 * out_sq: device fp32 [n_layers][7][2]: {||B1 A1 - B0 A0||_F^2 (unscaled),
 * ||A1 - A0||_F^2 + ||B1 - B0||_F^2}, zeros for modules not in the mask.
 * Every projection width (hidden, ffn, query and key/value widths) must be a
 * multiple of 8 (CRF_EUNSUPPORTED otherwise); every factor 16-byte aligned.
 * `workspace` >= crf_drift_workspace_size bytes. */
CRF_API crf_status crf_drift_workspace_size(crf_ctx* ctx, const crf_model_dims* dims,
                                    const crf_lora_dims* lora, size_t* bytes);
CRF_API crf_status crf_drift(crf_ctx* ctx, const crf_model_dims* dims, const crf_adapter* cur,
                     const crf_adapter* const* anchors, float* out_sq, void* workspace,
                     size_t ws_bytes, void* stream);

/* Forward KL(p* || p), p* = softmax(z_ref), p = softmax(z_cur), one value per row.
 * With model == NULL, ref/cur are device fp32 logits [n_rows, vocab].
 * With a model, ref/cur are device bf16 final hidden rows [n_rows, h]; the
 * logits z = lm_head * (rmsnorm(h) * final_norm) are formed first (model->dims.vocab
 * must equal `vocab`) and, if logits_out != NULL, stored there as fp32
 * [2 * n_rows, vocab] (ref rows first). out_kl: device fp32 [n_rows].
 * `workspace` >= crf_kl_workspace_size bytes. */
CRF_API crf_status crf_kl_workspace_size(crf_ctx* ctx, int n_rows, int vocab, int hidden, size_t* bytes);
CRF_API crf_status crf_kl(crf_ctx* ctx, const crf_model* model, const void* ref, const void* cur,
                  int n_rows, int vocab, float* out_kl, float* logits_out, void* workspace,
                  size_t ws_bytes, void* stream);

/* Allocation-free first-step KL from logits (no counterpart in the paper; an
 * interface for callers that cannot allocate device memory when they need the
 * number, such as a serving loop under a fixed device-memory budget or a C
 * host without its own device allocator).
 * Same arithmetic as crf_kl with model == NULL (the same vocabulary splits,
 * reduced in the same order), but its scratch is a fixed device array inside
 * the library (160 KiB, held by every GPU that loads it until the process
 * exits) instead of a caller workspace, so the call allocates nothing.
 * z_ref, z_cur: device fp32 [n_rows, vocab]; out_kl: device fp32 [n_rows].
 * n_rows must be 1..32 (CRF_EUNSUPPORTED beyond). `device` is made current for
 * the call and restored after. The first call on a device (and the first after
 * that device's context is recreated, e.g. after cudaDeviceReset) looks up the
 * array's device address; make that first call before any stream capture.
 * All calls share the one array: calls whose kernels overlap on the GPU
 * (different streams, or different host threads) race and must be serialised
 * by the caller. */
CRF_API crf_status crf_kl_logits_noalloc(int device, const float* z_ref, const float* z_cur,
                                         int n_rows, int vocab, float* out_kl, void* stream);

/* ------------------------------------------------------------------------
 * Extending a recovered cache with new tokens (a conversation's next turn, a
 * run of drafted tokens, one generated token for each row of a batch): calls
 * of one layer, and calls on the pages of the pool. They have no counterpart
 * in the paper, whose recovered cache is consumed by an ordinary decoder. They
 * keep the conventions above, with these differences:
 *   - crf_rotary, crf_cache_append and crf_chunk_attention check every page id
 *     where they use it: a write through an id outside [0, num_pages) is left
 *     out, a read goes to page 0, and crf_check then returns CRF_EINVAL.
 *   - crf_pages_* check their tables and counts in the call's first kernel; a
 *     call that it rejects writes nothing outside its workspace.
 *   - The current device is the same after the call as before it.
 * They may be captured into a CUDA graph; lengths and positions, which the
 * host passes, are then fixed, while the contents of tables, positions and
 * counts are read at every replay. Calls whose kernels overlap on the GPU
 * need workspaces of their own. */

#define CRF_MAX_CHUNKS 128  /* requests of one append or attention call */
#define CRF_MAX_TABLES 512  /* page tables of one crf_pages_* call */
#define CRF_MAX_KEYS (1 << 26)  /* cached positions of a request that attention sees */

enum { CRF_BF16 = 0, CRF_FP16 = 1, CRF_FP32 = 2 };                  /* element types of crf_rotary */
enum { CRF_ROPE_HALF = 0, CRF_ROPE_INTERLEAVED = 1 };               /* pairs (i, i + rot/2) or (2i, 2i + 1) */
enum { CRF_ROPE_PLAIN = 0, CRF_ROPE_LINEAR = 1, CRF_ROPE_BASE = 2, CRF_ROPE_BANDS = 3 };

/* Rotary positions. Pair i of the first rot_dim elements of a head (the rest
 * pass through) turns by p f_i at position p:
 *   (x, y) -> magnitude (x cos - y sin, y cos + x sin),  f_i = theta^(-2 i / rot_dim),
 * and for contexts `factor` (>= 1) times as long as the trained ones
 *   CRF_ROPE_LINEAR  f_i / factor (interpolated positions)
 *   CRF_ROPE_BASE    theta factor^(rot_dim / (rot_dim - 2)) in theta's place (rot_dim > 2)
 *   CRF_ROPE_BANDS   f_i (g + (1 - g) / factor), g = clamp((r - low) / (high - low), 0, 1) of the
 *                    r = original f_i / (2 pi) turns that the pair makes over the `original` trained
 *                    positions (0 <= low < high): fast pairs stay, slow ones are interpolated.
 *                    g is a ramp over turns. Models whose ramp runs over the pair's index i between two
 *                    rounded bounds have other frequencies, which this scaling does not give.
 * head_dim 2..256; rot_dim even, 2..head_dim. `factor` is not read with
 * CRF_ROPE_PLAIN; low, high and original are read with CRF_ROPE_BANDS alone. */
typedef struct crf_rope {
  int head_dim, rot_dim, layout, scaling;
  double theta, factor, low, high, original, magnitude;
} crf_rope;

/* Heads of a batch of rows: element e of head h of row r of `x` is at
 * x[r x_row + h x_head + e] (strides in elements, >= 0; that of an axis of one
 * row or head is not read), `out` likewise. `out` may be `x` itself with the
 * same strides; otherwise the two do not overlap. */
typedef struct crf_heads {
  const void* x;
  void* out;
  int heads;
  int64_t x_row, x_head, out_row, out_head;
} crf_heads;

/* Rotates n_parts (1 or 2: queries, keys) sets of heads of n_rows rows (0: the
 * call does nothing) at positions[r] (device int32, of any sign; angles are formed in 64-bit fixed
 * point). `inverse` != 0 applies the transposed map (the rotation back,
 * times magnitude): the gradient of the call without it. Arithmetic is fp32,
 * rounded once to `type`. Elements are aligned to their size; rows of
 * 16-byte aligned heads take the vector form. */
CRF_API crf_status crf_rotary(crf_ctx* ctx, const crf_rope* rope, const crf_heads* parts, int n_parts,
                              int type, int n_rows, const int32_t* positions, int inverse, void* stream);

/* New rows of one request: n_new (>= 0) rows at positions pos .. pos + n_new - 1.
 * The rows of a call's requests are packed in order. page_table: device int32,
 * ceil((pos + n_new) / 16) entries to append, ceil(n_keys / 16) to attend.
 * n_keys: cached positions that attention may see, the new rows' own (appended
 * before) among them; usually pos + n_new, at most CRF_MAX_KEYS. pos + n_new <= 2^30. */
typedef struct crf_chunk {
  int n_new, pos, n_keys;
  const int32_t* page_table;
} crf_chunk;

/* Writes the rows' keys and values (bf16) into the pages of `layer`, k rotated
 * at the row's position first when `rope` is given; with `q` (which needs
 * `rope`) the query heads are rotated into q->out in the same launch. The
 * `out` members of k and v are not read; k->heads == v->heads == n_kv_heads.
 * rope->head_dim == head_dim. head_dim 64 or 128. No two rows may share a
 * slot. Every other slot of the pool is left as it was. */
CRF_API crf_status crf_cache_append(crf_ctx* ctx, const crf_rope* rope, const crf_kv_pool* pool, int layer,
                                    int n_kv_heads, int head_dim, const crf_chunk* chunks, int n_chunks,
                                    const crf_heads* q, const crf_heads* k, const crf_heads* v, void* stream);

/* Attention of the rows over their requests' cached keys of `layer`. Row r of a
 * request (position p = pos + r) sees the keys
 *   j < n_keys, and j <= p unless causal == 0, and j > p - window if window > 0,
 * and o = softmax(scale q k) v over them, query head h reading kv head
 * h / (heads / n_kv_heads). A row that sees no key gives o = 0 and lse = -inf.
 *   q: x bf16 [rows] x heads, out the same shape (not overlapping x); heads a
 *      multiple of n_kv_heads; head_dim 64 or 128; strides multiples of 8, 16-byte aligned.
 *   lse: NULL, or device fp32 [rows][heads]: log of the sum of exp(scale q k).
 *   scale: > 0, or 0 for 1 / sqrt(head_dim); scores are kept as scale log2(e) q k in fp32, and both the
 *      factor and the scores have to be in its range.
 * Slots that a row does not see may hold anything, infinities and NaN
 * included. Softmax weights enter the product with v in bf16; sums, maxima
 * and o are fp32, and weights of up to 2^8 are summed before the division: 2^8 times
 * the sum of |v| over a row's keys has to be in fp32's range. `workspace` >=
 * crf_chunk_attention_workspace_size bytes for these chunks, 256-byte aligned.
 * Pages may be shared by requests. */
CRF_API crf_status crf_chunk_attention_workspace_size(crf_ctx* ctx, int n_q_heads, int n_kv_heads, int head_dim,
                                                      const crf_chunk* chunks, int n_chunks, int causal,
                                                      int window, size_t* bytes);
CRF_API crf_status crf_chunk_attention(crf_ctx* ctx, const crf_kv_pool* pool, int layer, int n_kv_heads,
                                       int head_dim, const crf_chunk* chunks, int n_chunks,
                                       const crf_heads* q, float* lse, float scale, int causal, int window,
                                       void* workspace, size_t ws_bytes, void* stream);

/* Pages are shared through a reference count a page (device int32 [num_pages];
 * 0: free). One table of a request of n_tokens (>= 0) tokens: `table` device int32
 * [ceil(n_tokens / 16)], `out` of the same length (see the calls). The counts go from refs_in to
 * refs_out, which may be the same array; otherwise the two do not overlap. */
typedef struct crf_pages {
  int n_tokens;
  const int32_t* table;
  int32_t* out;
} crf_pages;

/* A second continuation of every request: `out` receives the child's table. Whole pages are
 * shared (their count rises by one); a last page that is part filled, or with deep != 0 every
 * page, gets a page of its own, count 1, into which the live slots of all n_layers layers are copied
 * (the slots behind them are left as they were). New pages are the lowest free ones, dealt
 * in order of tables and entries. The call is rejected (CRF_EINVAL from crf_check) by a table id
 * outside the pool or of count 0, a negative count, and, where pages are shared, a table id whose
 * count is over 2^31 - 1 less the call's entries; and by too few free pages (CRF_ENOMEM from crf_check).
 * `out` overlaps no table of the call and no other `out`. */
CRF_API crf_status crf_pages_fork(crf_ctx* ctx, const crf_kv_pool* pool, int n_layers, int n_kv_heads,
                                  int head_dim, const int32_t* refs_in, int32_t* refs_out,
                                  const crf_pages* tables, int n_tables, int deep, void* workspace,
                                  size_t ws_bytes, void* stream);

/* Moves the live pages (count > 0) to the front of the pool: with L of them, the k-th lowest page at or
 * above L moves into the k-th lowest free one below L, in all layers; `out` receives each
 * table with the new ids (it may be `table` itself) and refs_out the moved counts, 0 from L on. The moved
 * pages' old places keep their contents. Every reference must be in a table of the call: a
 * page whose count is not the number of its entries rejects the call, as do ids outside the pool. */
CRF_API crf_status crf_pages_compact(crf_ctx* ctx, const crf_kv_pool* pool, int n_layers, int n_kv_heads,
                                     int head_dim, const int32_t* refs_in, int32_t* refs_out,
                                     const crf_pages* tables, int n_tables, void* workspace,
                                     size_t ws_bytes, void* stream);

/* Gives back every entry of the tables: each lowers its page's count by one (a page several
 * times if its entries are several). A count that would fall below zero, or an id outside the pool, rejects
 * the call. `out` is not read. */
CRF_API crf_status crf_pages_release(crf_ctx* ctx, int num_pages, const int32_t* refs_in, int32_t* refs_out,
                                     const crf_pages* tables, int n_tables, void* workspace,
                                     size_t ws_bytes, void* stream);

/* Workspace bytes (256-byte aligned) of any crf_pages_* call on these tables. */
CRF_API crf_status crf_pages_workspace_size(crf_ctx* ctx, int num_pages, const crf_pages* tables, int n_tables,
                                            size_t* bytes);

/* Per-kernel timing, for measurement: while enabled, every kernel launch and
 * device copy the library issues is bracketed by CUDA events recorded on the
 * caller's stream (the events are created here, up to `max_launches` launches
 * between reads; later launches are counted as dropped).
 * crf_profile_read synchronises those events and returns, per kernel kind,
 * its name (NUL-terminated, at most 31 chars, in names[i*32]), total device
 * milliseconds and number of kernel launches; then it clears the record.
 * Kinds with no launches are omitted. *n_kinds receives the number written. */
CRF_API crf_status crf_profile_enable(crf_ctx* ctx, int on, int max_launches);
CRF_API crf_status crf_profile_read(crf_ctx* ctx, int max_kinds, char* names, double* total_ms,
                                    int* launches, int* n_kinds, int* dropped);

#ifdef __cplusplus
}
#endif
#endif /* CRF_H */
