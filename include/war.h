/*
 * war.h -- C ABI of the MI355X speculative-verification decode step.
 *
 * The operation (WAR, arXiv 2607.17299):
 *  - Rollout is batched LLM inference over multi-turn trajectories whose KV
 *    cache is kept and reused from turn to turn (Background, "Rollout
 *    Bottlenecks"; System Design, "Overview of WAR").
 *  - Under low load the model-free suffix drafter proposes draft tokens.  The
 *    target model verifies them in one forward pass and advances several tokens
 *    when they are accepted (System Design, "SuffixDecoding").
 *  - Under high load speculation is off and the same step is plain batched
 *    decode (System Design, "SuffixDecoding": adaptive enabling, stateless
 *    mode switching).
 *  - Speculation must be lossless (Introduction; Background, "Why Workload
 *    Matters").  Here that means greedy verification:
 *      - row 0 of request b is its pending token x_b at position ctx_b;
 *      - rows 1..n_b are its drafts d_1..d_n;
 *      - g_i is the argmax of row i (ties go to the lowest id);
 *      - accept_b is the largest a with d_m == g_{m-1} for all m <= a;
 *      - next_b is g_{accept_b}.
 *    war_kv_commit then keeps the KV of rows 0..accept_b, sets
 *    ctx_b += accept_b + 1, and returns the pages reserved for rejected
 *    slots (rollback).
 *
 * Conventions
 *  - Every array argument is a DEVICE pointer owned by the caller, unless its
 *    comment says "host".  The library never frees caller memory.
 *  - Every call is ordered on the given HIP stream (a hipStream_t passed as
 *    void*; NULL = the null stream).  Nothing waits for the device unless the
 *    comment says so.
 *  - Calls on one model or one pool are not thread-safe: use one stream per
 *    model and pool.
 *  - Arguments are checked on the host before anything is enqueued.  On error
 *    the call returns a negative status, enqueues nothing and changes no
 *    state.  war_last_error() describes the last failure of the calling
 *    thread.
 */
#ifndef WAR_H
#define WAR_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t war_status;
#define WAR_OK                0
#define WAR_ERR_INVALID_ARG  (-1)
#define WAR_ERR_OUT_OF_PAGES (-2)
#define WAR_ERR_HIP          (-3)
#define WAR_ERR_UNSUPPORTED  (-4)
#define WAR_ERR_DEVICE       (-5) /* the device flagged bad input (war_pool_state) */

/* Decoder shape.
 * Layers: RMSNorm -> QKV -> rotate-half RoPE -> grouped-query attention -> O-proj,
 * then residual -> RMSNorm -> SwiGLU FFN -> residual; final RMSNorm; untied LM head.
 * Constraints: d_model, ffn_dim, vocab and (n_q_heads + 2 n_kv_heads) * head_dim
 * are multiples of 128; head_dim is 64 or 128; n_q_heads / n_kv_heads is 1..8;
 * page_size is 16. */
typedef struct war_model_config {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rms_eps;     /* RMSNorm epsilon                                        */
  float rope_base;   /* RoPE base: pair j of a head turns by pos * base^(-2j/D) */
  int32_t page_size; /* KV tokens per page (16)                                */
  int32_t max_rows;  /* most rows one forward pass holds (verify: B*(k_max+1)) */
} war_model_config;

typedef struct war_model war_model;     /* opaque: owned weight copy + owned workspace */
typedef struct war_kv_pool war_kv_pool; /* opaque: owned allocator state, borrowed KV */

/* Number of weight pointers a model takes: 3 + 7 * n_layers. */
int32_t war_weight_count(const war_model_config* cfg);

/* Create a model over caller-owned bf16 weights (device pointers, row-major [out, in]).
 * Canonical order:
 *   embed [V, d];
 *   then for each layer:
 *     attn_norm [d];
 *     w_qkv [(nq + 2 nkv) * hd, d]  (query rows head-major, then key rows, then value rows);
 *     w_o [d, nq * hd];
 *     ffn_norm [d];
 *     w_gate [F, d];
 *     w_up [F, d];
 *     w_down [d, F];
 *   then final_norm [d];
 *   then w_lm [V, d].
 * The model copies every weight into device memory it owns, the projection
 * and LM-head matrices repacked into the order its GEMM kernel streams
 * (16-row by 64-column MFMA fragments, each 16-byte lane chunk contiguous), so
 * the caller's buffers are not read after this call returns and may be freed.
 * The copy costs as much device memory as the weights themselves.  The model
 * also allocates its own device workspace (sized by max_rows).  Returns WAR_ERR_UNSUPPORTED for shapes
 * outside the constraints above. */
war_status war_model_create(const war_model_config* cfg, const void* const* weights,
                            int32_t n_weights, war_model** out);
void war_model_destroy(war_model* m);

/* Create a KV page pool over caller-owned storage.
 *   kv_pages     bf16, n_layers * num_pages * n_kv_heads * 2 * page_size * head_dim
 *                elements.  Page p of layer l, kv-head h starts at element
 *                ((l * num_pages + p) * n_kv_heads + h) * 2 * page_size * head_dim.
 *                It holds the keys (page_size * head_dim elements, in the
 *                fragment order below), then the values transposed as
 *                [head_dim][page_size].  page_size is 16.  Key slot s, dim d
 *                sits at element ((t * head_dim/32 + d/32) * 8 + s8) * 32 + d%32
 *                of the key region, with t = (s/4) % 2 and s8 = 4 (s/8) + s%4:
 *                one 512-byte run per (slot group t, 32-dim step), which is
 *                what one attention operand load reads.
 *   block_tables int32 [max_seqs][max_pages_per_seq].  Entry [s][j] is the
 *                physical page of sequence s's logical page j, or -1.
 *                Initialised to -1 here.
 * The pool owns its free stack, reference counts and per-sequence page counts.
 * Free pages pop as 0, 1, 2, ...  Pops go in batch order, logical pages
 * ascending.  Pushes go in reverse batch order, logical pages descending.  So
 * reserving and then discarding a step restores the stack exactly. */
war_status war_kv_pool_create(const war_model_config* cfg, void* kv_pages, int32_t num_pages,
                              int32_t* block_tables, int32_t max_seqs, int32_t max_pages_per_seq,
                              void* stream, war_kv_pool** out);
void war_kv_pool_destroy(war_kv_pool* p);

/* A pool that holds keys and values in 8 bits: half the bytes that attention reads and
 * twice the tokens in a replica's memory, which is what limits its requests
 * (Background, "Rollout Bottlenecks").  Every call that takes a pool takes either kind.
 * One token's head_dim keys (or values) of one kv-head are a block: codes c (OCP e4m3)
 * with a power-of-two scale 2^e, e the smallest integer with max |x| <= 448 * 2^e, at
 * least -117.  c is x / 2^e rounded to nearest even, and stands for c * 2^e, which
 * bf16 holds exactly (from 1.9375 * 2^127 on it is infinite).  A block belongs to one
 * token so that a rejected draft leaves no trace in the tokens before it, and so that
 * a step, an append, an import and war_kv_write of the same bf16 numbers store the
 * same bytes.  Where any key or value of a token and kv-head is not finite, all of
 * them read as NaN, and rows that see the token get NaN; others do not.
 * (A finite value that reads as infinite reaches only the rows that see it, too; it
 * counts as 2^128 or as the largest bf16 there.)
 *   kv_format     WAR_KV_BF16 (as war_kv_pool_create) or WAR_KV_E4M3
 *   kv_pages      war_kv_pool_bytes(cfg, num_pages, kv_format) bytes, 16-byte aligned.
 *                 E4M3: page regions as in war_kv_pool_create but of bytes, at byte
 *                 ((l * num_pages + p) * n_kv_heads + h) * 2 * 16 * head_dim, behind
 *                 all of them 32 scale bytes (e + 127) for each (l, p, h).  Key slot
 *                 s, dim d is byte ((t * head_dim/64 + d/64) * 8 + s8) * 64 + d%64 of
 *                 the key region (t and s8 as above), its scale byte 2 s8 + t; the
 *                 value is byte ((d/32 * 2 + s/8) * 16 + d%16) * 16 + (d/16)%2 * 8 +
 *                 s%8 of the value region, its scale byte 16 + s (0: not finite). */
#define WAR_KV_BF16 0
#define WAR_KV_E4M3 1
int64_t war_kv_pool_bytes(const war_model_config* cfg, int32_t num_pages, int32_t kv_format);
war_status war_kv_pool_create_format(const war_model_config* cfg, void* kv_pages, int32_t num_pages,
                                     int32_t kv_format, int32_t* block_tables, int32_t max_seqs,
                                     int32_t max_pages_per_seq, void* stream, war_kv_pool** out);

/* Ensure capacity for n_tokens[i] slots for sequence seq_ids[i] (host arrays,
 * distinct ids).  A trajectory's KV cache grows with its length and stays
 * resident from turn to turn, so KV memory is the pressure point of rollout
 * (Background, "Rollout Bottlenecks"; System Design, "Overview of WAR").
 * Pages are popped from the free stack; nothing changes when they do not
 * suffice (WAR_ERR_OUT_OF_PAGES).  Synchronises the stream. */
war_status war_kv_alloc(war_kv_pool* p, int32_t n, const int32_t* seq_ids_host,
                        const int32_t* n_tokens_host, void* stream);

/* dst shares the first n_tokens (a multiple of page_size) of src.  dst must hold no
 * pages.  The shared pages' reference counts rise.  The caller sets dst's
 * ctx_len to n_tokens.  Cache reuse across sibling rollouts (System Design,
 * "Overview of WAR"). */
war_status war_kv_fork(war_kv_pool* p, int32_t src_seq, int32_t dst_seq, int32_t n_tokens,
                       void* stream);

/* Drop every page of each listed sequence (host array, distinct ids); a page
 * returns to the free stack when its reference count reaches 0.  A finished
 * trajectory releases the KV memory it held (Background, "Rollout
 * Bottlenecks": KV footprint limits how many requests a replica keeps).
 * Synchronises the stream. */
war_status war_kv_free(war_kv_pool* p, int32_t n, const int32_t* seq_ids_host, void* stream);

/* Write precomputed keys/values of tokens [pos0, pos0 + n) of one layer of one
 * sequence into its pages (capacity must already be there, e.g. war_kv_alloc).
 * src: bf16 [2][n_kv_heads][n][head_dim] (0 = keys after RoPE, 1 = values), 2-byte
 * aligned.
 * Imports a cached context computed elsewhere: the scheduler places a
 * request on the replica whose cache already holds its prefix, and a
 * trajectory's KV is reused across turns instead of recomputed (System
 * Design, "Overview of WAR" and the cache-aware scheduler).  Reads the
 * sequence's page count (one stream synchronisation). */
war_status war_kv_load(war_kv_pool* p, int32_t seq_id, int32_t layer, int32_t pos0, int32_t n,
                       const void* src, void* stream);

/* Keys and values of many sequences' tokens into their pages, one layer, and out of
 * them (caches move between replicas: System Design, "Overview of WAR" and the
 * cache-aware scheduler).  Unlike war_kv_load nothing waits for the device.
 *   seq_ids   device int32 [B], distinct
 *   pos0      device int32 [B]: the first token's position
 *   n_max     row b * n_max + i of k and v is token pos0[b] + i; B * n_max <= 2^26
 *   n_lens    device int32 [B] in [0, n_max], or NULL: all n_max.  Rows beyond are not
 *             read (written: left as they were).
 *   k, v      device bf16 rows of n_kv_heads * head_dim, keys after RoPE; strides in
 *             elements, multiples of 8, at least a row; 16-byte aligned
 * The tokens must lie within the sequence's pages (war_kv_alloc; a page that forked
 * sequences share changes for all of them, as under war_kv_load).  A request that does
 * not (or has a bad id, position or count) is flagged (war_pool_state) and left out. */
war_status war_kv_write(war_kv_pool* p, int32_t layer, int32_t B, const int32_t* seq_ids, const int32_t* pos0,
                        int32_t n_max, const int32_t* n_lens, const void* k, int64_t k_stride, const void* v,
                        int64_t v_stride, void* stream);
war_status war_kv_read(war_kv_pool* p, int32_t layer, int32_t B, const int32_t* seq_ids, const int32_t* pos0,
                       int32_t n_max, const int32_t* n_lens, void* k, int64_t k_stride, void* v,
                       int64_t v_stride, void* stream);

/* Attention of given rows over a pool, as the steps take it: for decoders whose other
 * layers are the caller's.  An object owns the workspace of one plan; a plan is made
 * once a step and serves all its layers.
 *   max_batch, max_rows   the most requests and rows a request: max_batch <= 1024,
 *                         max_rows <= 65536, their product <= 2^20
 * The workspace is mostly partial sums, 4 * (head_dim + 2) bytes a row and kv-head.  With
 * G = n_q_heads / n_kv_heads: 16, 32 or 48 rows (the least that holds G * max_rows, 48 at
 * most) for every request and 1024 tokens of max_pages_per_seq; where G * max_rows > 48
 * also 128 rows for each of up to max(max_batch * ceil(max_rows / (128 / G)),
 * 8192 / n_kv_heads) units, whichever is more: 17 GB for 2^20 rows of 32 heads of 128.
 * The pool must outlive the object.  Only war_attend_create and _destroy allocate and
 * wait, so update and run may be captured into a graph, both together (a plan made
 * outside describes the pool as it was then); an object holds one plan at a time, so
 * graphs that may run at the same time take an object each. */
typedef struct war_attend war_attend;
war_status war_attend_create(war_kv_pool* p, int32_t max_batch, int32_t max_rows, war_attend** out);
void war_attend_destroy(war_attend* a);

/* The plan of B requests with n_max rows each.
 *   seq_ids       device int32 [B], distinct
 *   ctx_lens      device int32 [B]: position of the request's row 0
 *   n_lens        device int32 [B] in [0, n_max]: live rows; NULL: all n_max
 *   draft_parents device int32 [B][n_max - 1]: rows are draft trees as in
 *                 war_verify_step_tree; NULL: row i is the token at ctx + i.  Trees take
 *                 n_q_heads / n_kv_heads * n_max <= 48 and n_max <= 32.
 * The keys and values of positions 0 .. ctx + n_lens - 1 (a tree's node i: ctx + i) must
 * be in the pool when the attention runs.  A bad id, position or count, an id twice, or
 * rows beyond a sequence's pages are flagged (war_pool_state), and war_attend_run then
 * writes nothing.  A plan ends when the pool gives pages back (war_kv_free,
 * war_kv_commit): war_attend_run then asks for the next update. */
war_status war_attend_update(war_attend* a, int32_t B, int32_t n_max, const int32_t* seq_ids,
                             const int32_t* ctx_lens, const int32_t* n_lens, const int32_t* draft_parents,
                             void* stream);

/* o = softmax(q k / sqrt(head_dim)) v of the planned rows in one layer; row i of request
 * b sees the keys 0 .. ctx_b + i (a tree's node the context and its root path).  Over
 * either kind of pool the weights keep 16 bits for the product with the values, and the
 * sums are fp32.
 *   q, o   device bf16, row b * n_max + i at that many strides, n_q_heads * head_dim
 *          elements; strides in elements, multiples of 8; 16-byte aligned.  Rows of o
 *          beyond n_lens are left as they were. */
war_status war_attend_run(war_attend* a, int32_t layer, const void* q, int64_t q_stride, void* o,
                          int64_t o_stride, void* stream);

/* ---- The other operators of a decoder layer, for decoders whose layers are the
 * caller's (with war_attend_* between them), their weights in 4 bits: a step of few rows
 * is bound by the bytes of its weights (Background, "Rollout Bottlenecks"). ----
 *
 * A matrix of microscaled numbers: 32 neighbouring columns of a row are a block with the
 * scale 2^e, kept as the byte e + 127; a code c stands for c * 2^e.  Writing, e is the
 * smallest integer with max |x| <= top * 2^e, at least -117 (top: 448 for e4m3, 6 for
 * e2m1), and c is x / 2^e rounded to nearest even; a block with a number that is not
 * finite gets the byte 255, and all of it reads as NaN.  Reading, any scale byte will do.
 *   format        WAR_MX_E4M3: a byte a code (OCP e4m3); WAR_MX_E2M1: 4 bits (sign, two
 *                 exponent bits, one mantissa bit), the even column in the low ones
 *   rows, cols    rows in [0, 2^20], cols a multiple of 32 in [32, 65536], rows * cols
 *                 <= 2^34
 *   codes         device; rows at code_stride bytes, a multiple of 16; 16-byte aligned
 *   scales        device; rows at scale_stride bytes, a multiple of 4 (bytes up to the
 *                 next multiple of 4 may be read, and do not count); 4-byte aligned */
#define WAR_MX_E4M3 2
#define WAR_MX_E2M1 3
#define WAR_BF16 0
#define WAR_F32 1
typedef struct war_mx {
  int32_t format, rows, cols;
  void* codes;
  int64_t code_stride;
  uint8_t* scales;
  int64_t scale_stride;
} war_mx;

/* The residual's addition and the norm behind it: h += x, then y = h / sqrt(mean(h^2) +
 * eps) * gain, rounded once to y's type.  h^2 and its sum are fp32 (h, where it is bf16, is
 * rounded as it is stored, not for y).
 *   x        device bf16 [rows][cols] at x_stride, or NULL: h stays as it is
 *   h        device [rows][cols] at h_stride, h_type WAR_BF16 or WAR_F32
 *   gain     device bf16 [cols]
 *   mx       y in codes (a HOST struct of rows by cols), or NULL and
 *   y        device bf16 [rows][cols] at y_stride (y may be x, at the same stride)
 * Strides in elements, multiples of 8; 16-byte aligned; sizes as of a war_mx. */
war_status war_residual_norm(int32_t rows, int32_t cols, const void* x, int64_t x_stride, void* h, int64_t h_stride,
                             int32_t h_type, const void* gain, float eps, const war_mx* mx, void* y, int64_t y_stride,
                             void* stream);

/* A matrix x into codes (mx, a HOST struct; its rows and cols are x's); with a gate g,
 * x * g / (1 + exp(-g)): what a SwiGLU's gate and up projections leave for the one down.
 * (Zero where exp(-g) is past fp32, g below -88.7.)
 * x and gate (NULL: none): device, type WAR_BF16 or WAR_F32, strides as above. */
war_status war_quantize(const war_mx* mx, const void* x, int64_t x_stride, const void* gate, int64_t gate_stride,
                        int32_t type, void* stream);
/* The numbers that codes stand for (exact in either type while they are in its range). */
war_status war_dequantize(const war_mx* mx, void* y, int64_t y_stride, int32_t type, void* stream);

/* y = x w^T + bias with w [N, K] in WAR_MX_E2M1: an object owns w laid out for its kernels
 * (17 bytes for 32 numbers, padded to 256 rows and 512 columns).
 *   w      HOST struct; N rows (at least 1), K cols; codes need no alignment here
 *   bias   device bf16 [N], or NULL
 * Synchronises the stream: the caller's arrays are not read afterwards. */
typedef struct war_linear war_linear;
war_status war_linear_create(const war_mx* w, const void* bias, void* stream, war_linear** out);
void war_linear_destroy(war_linear* l);
/* One product.  Any number of them may run at once (no workspace); nothing is allocated.
 *   x   HOST struct, [rows][K] in either format; strides at most 2^22
 *   y   device [rows][N] at y_stride elements, at least N; y_type WAR_BF16 or WAR_F32
 * Sums are fp32 in the matrix units, over products that are exact, but for a bf16 y of e4m3
 * activations: there eight neighbours are added without their bits more than 13 binary
 * places below the largest power of two among them (a product's is that of its two numbers',
 * a weight's code of 0.5 counted as 1).  Up to 7 x 2^-13 of that power is left out of each
 * group of eight, which is much of a y that cancels to little; an fp32 y has all of it.
 * A row's result does not depend on the other rows' numbers. */
war_status war_linear_run(const war_linear* l, const war_mx* x, void* y, int64_t y_stride, int32_t y_type, void* stream);

/* Rotary positions of several axes (HOST struct; copied by the call).  Pair j of a head
 * turns by (position of its row on axis axes[j]) * freqs[j].
 *   rotary_dim  numbers of a head that turn, the first: a multiple of 8, at most head_dim
 *   adjacent    0: pair j is (j, j + rotary_dim / 2); 1: (2 j, 2 j + 1)
 *   n_axes      in [1, 4]
 *   axes        HOST [rotary_dim / 2], each in [0, n_axes); NULL: all axis 0
 *   freqs       HOST [rotary_dim / 2], finite, |f| <= 6.3 (a turn) */
typedef struct war_rope {
  int32_t rotary_dim, adjacent, n_axes;
  const uint8_t* axes;
  const double* freqs;
} war_rope;

/* The queries and keys of many sequences' new tokens turned, keys and values into their
 * pages: war_kv_write with the rotation before it.
 *   seq_ids, pos0, n_max, n_lens   as in war_kv_write
 *   positions  device int32 [n_axes][B * n_max]: row b * n_max + i on each axis; NULL: the
 *              token's place in the cache, pos0[b] + i, on every axis
 *   q, q_out   device bf16 rows of n_q_heads * head_dim; q_out may be q (same stride),
 *              and overlaps nothing else
 *   k, v       device bf16 rows of n_kv_heads * head_dim, not written
 * Strides in elements, multiples of 8; 16-byte aligned.  Turned numbers are rounded to
 * bf16.  Rows beyond n_lens, and requests that are flagged as in war_kv_write, are left
 * out: their q_out stays as it was. */
war_status war_rope_write(war_kv_pool* p, int32_t layer, const war_rope* rope, int32_t B, const int32_t* seq_ids,
                          const int32_t* pos0, int32_t n_max, const int32_t* n_lens, const int32_t* positions,
                          const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, void* stream);

/* Append a new turn to cached trajectories (System Design, "Overview of WAR";
 * Background, "Rollout Bottlenecks").
 *   seq_ids     device int32 [n]
 *   ctx_lens    device int32 [n]; read, then += n_new
 *   n_new_host  HOST int32 [n], >= 1
 *   new_tokens  device int32, packed: sequence i's tokens at offset sum_{j<i} n_new[j]
 *   next_tokens device int32 [n]: argmax after each sequence's last new token
 *   last_logits device fp32 [n][vocab], or NULL
 * Reserves pages for ctx + n_new slots and computes the new tokens' KV (causal,
 * against the cached context).  This call synchronises the stream once to read
 * ctx_lens. */
war_status war_prefill_append(war_model* m, war_kv_pool* p, int32_t n, const int32_t* seq_ids,
                              int32_t* ctx_lens, const int32_t* n_new_host,
                              const int32_t* new_tokens, int32_t* next_tokens,
                              float* last_logits, void* stream);

/* One speculative-verification step over B requests (k_max = 0: plain decode).
 *   seq_ids      device int32 [B], distinct (checked on the device)
 *   ctx_lens     device int32 [B]  cached tokens per request (not changed here)
 *   last_tokens  device int32 [B]  pending token (previous step's next_tokens)
 *   draft_tokens device int32 [B][k_max] (may be NULL when k_max == 0)
 *   draft_lens   device int32 [B]  in [0, k_max] (NULL: all k_max)
 *   accept_lens  device int32 [B]  out
 *   next_tokens  device int32 [B]  out
 *   logits       device fp32 [B * (k_max + 1)][vocab] or NULL.  Row b*(k_max+1)+i
 *                holds request b's row i; rows with i > draft_len are unspecified.
 * Reserves the pages for ctx + draft_len + 1 slots, writes the KV of all rows,
 * and leaves the pool waiting for war_kv_commit.  Until that commit the pool
 * accepts no other call that changes pages.
 * The device checks what the host cannot see without waiting: ids in range
 * and distinct, ctx_len >= 0, ctx + draft_len + 1 within max_pages_per_seq,
 * token ids in [0, vocab), enough free pages.  On a bad id, length or page
 * count the whole step fails on the device: no page moves, accept_lens and
 * next_tokens are -1 for every request, the following war_kv_commit changes
 * nothing, and war_pool_state returns WAR_ERR_DEVICE (a bad token id is
 * flagged the same way but the step runs with token 0 in its place).  The
 * host never waits for the device here while its lower bound on the free
 * pages (kept from each commit's report) covers B * ceil((k_max+1)/16)
 * pages; otherwise it reads the exact count once. */
war_status war_verify_step(war_model* m, war_kv_pool* p, int32_t B, const int32_t* seq_ids,
                           const int32_t* ctx_lens, const int32_t* last_tokens,
                           const int32_t* draft_tokens, const int32_t* draft_lens, int32_t k_max,
                           int32_t* accept_lens, int32_t* next_tokens, float* logits,
                           void* stream);

/* The verify step with sampled verification instead of greedy acceptance (the
 * paper's rollouts sample: Evaluation, temperature 1.0, top-k 200; speculation
 * stays lossless: Introduction; Background, "Why Workload Matters").  Same
 * arguments and pool protocol as war_verify_step, plus:
 *   uniforms     device fp32 [B * (k_max + 1)][2], each in [0, 1): for row
 *                b*(k_max+1)+i, [0] is the acceptance test of draft i+1 and [1]
 *                the draw made at that row.  The caller owns the randomness.
 *   temperature  > 0
 *   top_k        in [1, vocab]
 * Row i's target distribution keeps the top_k largest logits (value
 * descending, ties to the lowest token id) and takes softmax(logit / T) over
 * them.  Draft i+1 is accepted iff uniform[0] < p_i(draft); at the first
 * rejection next_token is drawn from p_i without the rejected draft, and after
 * the last accepted draft from p_n; a draw with uniform v is the smallest token
 * id whose cumulative weight (in id order) exceeds v times the total.  The
 * logits are written to `logits` when it is not NULL, else to a workspace the
 * model allocates on first use ([B * (k_max + 1)][vocab] fp32).  Decisions are
 * taken in fp32. */
war_status war_verify_step_sampled(war_model* m, war_kv_pool* p, int32_t B, const int32_t* seq_ids,
                                   const int32_t* ctx_lens, const int32_t* last_tokens,
                                   const int32_t* draft_tokens, const int32_t* draft_lens, int32_t k_max,
                                   const float* uniforms, float temperature, int32_t top_k,
                                   int32_t* accept_lens, int32_t* next_tokens, float* logits, void* stream);

/* The verify step with a draft TREE per request (SuffixDecoding proposes
 * speculation trees; the paper counts their tree-mask handling among the
 * verification costs: Evaluation).  Greedy acceptance.  Same arguments and
 * pool protocol as war_verify_step, plus:
 *   draft_parents device int32 [B][k_max]: node 0 is last_token, node i
 *                 (1..draft_len) carries draft_tokens[b][i-1] and has parent
 *                 draft_parents[b][i-1] in [0, i).  A parent outside that range
 *                 sets the device error flag (war_pool_state) and is read as i-1.
 *   accept_path   device int32 [B][k_max] out, or NULL: the accepted nodes in
 *                 depth order, -1 beyond accept_lens[b].
 *   k_max         + 1 <= 32.
 * Node i is scored on its root-to-node path: position ctx + depth(i), and it
 * sees the cached context and the nodes of that path.  Its logits are row
 * b*(k_max+1)+i.  A node is accepted when its parent is (the root always is)
 * and its token is the parent's greedy token; the accepted path ends at the
 * deepest accepted node (lowest index among equals), accept_lens[b] is its
 * depth and next_tokens[b] its greedy token.  Before returning, the step moves
 * the KV of the accepted nodes to slots ctx + 1 .. ctx + accept_lens[b], so
 * war_kv_commit keeps exactly the accepted path. */
war_status war_verify_step_tree(war_model* m, war_kv_pool* p, int32_t B, const int32_t* seq_ids,
                                const int32_t* ctx_lens, const int32_t* last_tokens,
                                const int32_t* draft_tokens, const int32_t* draft_parents,
                                const int32_t* draft_lens, int32_t k_max, int32_t* accept_lens,
                                int32_t* next_tokens, int32_t* accept_path, float* logits, void* stream);

/* What a request's next token is held to: penalties for tokens its text holds already,
 * biases, and masks (the tool calls of an agent's answers follow a grammar: System
 * Design, "Overview of WAR").  Speculation stays lossless (Introduction): a draft is
 * judged by the logits that decoding without drafts would have at its place, so a row's
 * text is the counted tokens, the pending token and the drafts on the way to the row.
 * With n(v) the occurrences of token v in that text and s(v) whether it occurs there or
 * in the prompt, a logit z of v becomes, in fp32 and in this order:
 *   z += the sum of v's bias entries, in list order
 *   z  = z > 0 ? z / repetition : z * repetition     if s(v)
 *   z -= frequency * n(v);  z -= presence            if n(v) > 0
 *   z  = -inf                                        if the row's mask excludes v
 * All arrays are device memory; one that is NULL does nothing.
 *   counts       uint16 [n_seqs][vocab]: bit 15: v is in the prompt; the rest: its
 *                occurrences in the generated text that is in the cache, at most 32767
 *                (war_counts_begin, war_counts_add)
 *   repetition, frequency, presence   fp32 [n_seqs]; repetition > 0
 *   bias_ids     int32 [n_seqs][n_bias], bias_values fp32 the same; ids outside
 *                [0, vocab) do nothing; n_bias <= 1024
 *   masks        uint32 [n_masks][ceil(vocab / 32)]: bit v % 32 of word v / 32 is 1
 *                where v is allowed
 *   mask_index   int32, one a row: its mask; negative: every token is allowed; n_masks
 *                or more: none is.  NULL: row r takes mask r.
 * Arrays by sequence are indexed by the step's sequence ids. */
typedef struct war_constraints {
  int32_t n_seqs;
  const uint16_t* counts;
  const float* repetition;
  const float* frequency;
  const float* presence;
  int32_t n_bias;
  const int32_t* bias_ids;
  const float* bias_values;
  int32_t n_masks;
  const uint32_t* masks;
  const int32_t* mask_index;
} war_constraints;

/* Constrained logits of B requests' rows, and each row's greedy token.
 *   seq_ids, last_tokens [B], draft_tokens, draft_parents (NULL: chains) [B][k_max],
 *   draft_lens [B] (NULL: all k_max; clamped to [0, k_max])   device int32; k_max < 64
 *   logits     device fp32 [B * (k_max + 1)] rows of vocab at logits_stride
 *   out        device fp32, the same at out_stride; may be logits; NULL: not wanted
 *   greedy     device int32 [B * (k_max + 1)]: the lowest id among the largest allowed
 *              logits (a NaN is none of them), -1 where no token is allowed; NULL: not
 *              wanted
 *   workspace  device, war_constrain_workspace(B * (k_max + 1), vocab) bytes, 16-byte
 *              aligned; NULL when greedy is
 * Rows with i > draft_len are not read, and left as they were.  The rows of a request
 * whose id is outside [0, n_seqs) have no token and are not written to out.  A token id
 * outside [0, vocab) counts nowhere; a parent outside [0, i) is read as i - 1. */
int64_t war_constrain_workspace(int32_t rows, int32_t vocab);
war_status war_constrain_logits(const war_constraints* c, int32_t vocab, int32_t B, const int32_t* seq_ids,
                                const int32_t* last_tokens, const int32_t* draft_tokens,
                                const int32_t* draft_parents, const int32_t* draft_lens, int32_t k_max,
                                const float* logits, int64_t logits_stride, float* out, int64_t out_stride,
                                int32_t* greedy, void* workspace, void* stream);

/* New requests' rows of a counts table [n_seqs][vocab]: their prompts' tokens get bit
 * 15, everything else is cleared.
 *   seq_ids   device int32 [B], distinct (others than [0, n_seqs) are skipped)
 *   tokens    device int32 [n_tokens], packed; request i's at offsets[i] ..
 *             offsets[i + 1] (what lies outside [0, n_tokens) is not read)
 *   offsets   device int32 [B + 1], ascending
 * Token ids outside [0, vocab) are skipped. */
war_status war_counts_begin(uint16_t* counts, int32_t vocab, int32_t n_seqs, int32_t B, const int32_t* seq_ids,
                            const int32_t* tokens, int32_t n_tokens, const int32_t* offsets, void* stream);

/* Count what a step committed (or any generated tokens): first[b] (NULL: none), then
 * lens[b] tokens of tokens[b].
 *   first   device int32 [B]: the step's last_tokens
 *   tokens  device int32 [B][n_max]: its draft_tokens; n_max <= 4096
 *   path    device int32 [B][n_max]: a tree's accept_path, token j is
 *           tokens[path[j] - 1]; NULL: in order
 *   lens    device int32 [B]: its accept_lens; -1: nothing of the request is counted;
 *           NULL: all n_max
 * seq_ids as above.  A count stays at 32767. */
war_status war_counts_add(uint16_t* counts, int32_t vocab, int32_t n_seqs, int32_t B, const int32_t* seq_ids,
                          const int32_t* first, const int32_t* tokens, int32_t n_max, const int32_t* path,
                          const int32_t* lens, void* stream);

/* A verify step under constraints: war_verify_step (chains), war_verify_step_tree
 * (draft_parents not NULL, accept_path as there) or war_verify_step_sampled (uniforms
 * not NULL, chains; temperature and top_k as there) with every row's logits
 * constrained before its token is chosen.  n_seqs must cover the pool's sequences.
 * logits receives the constrained ones; where it is NULL the model holds as many itself,
 * in memory that grows at need (like every step's, so not under a graph capture).  In a row where no token is left (none allowed;
 * sampled: none above -inf) no draft is accepted, and next_tokens is -1 where the
 * accepted path ends there. */
war_status war_verify_step_constrained(war_model* m, war_kv_pool* p, int32_t B, const int32_t* seq_ids,
                                       const int32_t* ctx_lens, const int32_t* last_tokens,
                                       const int32_t* draft_tokens, const int32_t* draft_parents,
                                       const int32_t* draft_lens, int32_t k_max, const war_constraints* c,
                                       const float* uniforms, float temperature, int32_t top_k,
                                       int32_t* accept_lens, int32_t* next_tokens, int32_t* accept_path,
                                       float* logits, void* stream);

/* war_verify_step for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc).
 * Same arguments, pool protocol and results as war_verify_step (greedy chain
 * drafts); the step's workspace (activations, split-K partials, attention
 * work list and partials, counters) is laid over a static device array of
 * 64 MiB that the library holds on each GPU it runs on until the process
 * ends, instead of the model's own workspace.  This call allocates nothing:
 * no hipMalloc, hipFree or allocating library routine, and no host buffers.
 * It returns WAR_ERR_UNSUPPORTED (enqueuing nothing) when the step does not
 * fit: the rows B*(k_max+1) with their partials, plus the attention items of
 * B requests of max_pages_per_seq pages (longer attention chunks are taken
 * first to fit).  When the host's lower bound on free pages does not cover
 * B*ceil((k_max+1)/16) pages it reads the exact count (one stream
 * synchronisation) and returns WAR_ERR_OUT_OF_PAGES if that does not cover
 * it either.  Every call on one GPU shares that GPU's array: calls that
 * overlap on one GPU (other streams, other threads) race; the array keeps the
 * last call's contents, and the step clears what must start at zero. */
war_status war_verify_step_noalloc(war_model* m, war_kv_pool* p, int32_t B, const int32_t* seq_ids,
                                   const int32_t* ctx_lens, const int32_t* last_tokens,
                                   const int32_t* draft_tokens, const int32_t* draft_lens, int32_t k_max,
                                   int32_t* accept_lens, int32_t* next_tokens, float* logits,
                                   void* stream);

/* Commit the pending verify step.
 *   accept_lens device int32 [B]; -1 discards the step.  Values are clamped
 *               to [-1, reserved capacity].
 * Effects:
 *   ctx_lens[b] += accept_lens[b] + 1;
 *   the pages the step reserved beyond the new length go back to the free
 *   stack, and their block-table entries become -1.
 * After a step that failed on the device nothing changes.  Use the same B,
 * seq_ids and ctx_lens as the verify step (an id out of range is flagged and
 * skipped).  When the kernel ends it writes its sequence number and the free
 * page count to a host-mapped word of the pool, which later verify steps read
 * instead of waiting. */
war_status war_kv_commit(war_kv_pool* p, int32_t B, const int32_t* seq_ids, int32_t* ctx_lens,
                         const int32_t* accept_lens, void* stream);

/* Synchronise the stream.  Copy the allocator state to HOST buffers (each may
 * be NULL):
 *   free_stack      [num_pages]  (only the first *free_count entries are meaningful)
 *   refcount        [num_pages]
 *   held            [max_seqs]   pages held per sequence
 *   step_base       [max_seqs]   pages held before the last reservation
 * Returns WAR_ERR_DEVICE if a kernel flagged bad device-side input since the
 * last call (a token id outside [0, vocab), a sequence id out of range or
 * repeated within one step, a negative or too long context, a tree parent out
 * of range, or a device page shortage); the flags are then cleared. */
war_status war_pool_state(war_kv_pool* p, int32_t* free_count, int32_t* free_stack,
                          int32_t* refcount, int32_t* held, int32_t* step_base, void* stream);

/* Thread-local description of the last non-OK status ("" if none). */
const char* war_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* WAR_H */
