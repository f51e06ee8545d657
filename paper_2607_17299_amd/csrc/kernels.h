// Internal launch interface between the C-ABI runtime and the gfx950 kernels.
#pragma once

#include <algorithm>

#include "common.h"

// Geometry of the paged KV storage:
//   element offset of page `page`, layer `layer`, kv-head `kvh`, kind (0 = K, 1 = V^T)
//   = ((((layer * num_pages + page) * n_kv_heads + kvh) * 2 + kind) * page_size * head_dim
// V is stored transposed, [head_dim][page_size].  K (page_size = 16) is stored
// in the order the attention's MFMA fragments read it, so that every K load of
// a wave reads 512 contiguous bytes of a page: key slot s, dim d sits at
// key_elem(s, d) (below).
//
// A pool in e4m3 (q8 not null) has the same page regions in bytes, in the orders
// key_elem8 and val_elem8, and 32 scale bytes a page and kv-head behind all pages:
// the block of a scale is the head_dim keys (or values) of one token and kv-head, the
// byte is e + 127 for the scale 2^e.
struct KvGeom {
  bf16_t* kv;
  uint8_t* q8;     // e4m3 pages, or nullptr: bf16 in kv
  uint8_t* scale;  // scale bytes of the e4m3 pages
  int64_t num_pages;
  int n_kv_heads, head_dim, page_size;
  __host__ __device__ int64_t page_elems(int layer, int page, int kvh, int kind) const {
    return ((((int64_t)layer * num_pages + page) * n_kv_heads + kvh) * 2 + kind) *
           (int64_t)page_size * head_dim;
  }
  __host__ __device__ int64_t scale_bytes(int layer, int page, int kvh) const {
    return (((int64_t)layer * num_pages + page) * n_kv_heads + kvh) * 32;
  }
};

// Element offset of key slot s (0..15), dim d in a page's K region.  The slots
// form two groups of eight, t = (s / 4) % 2 (slots 0-3, 8-11 and 4-7, 12-15:
// the two 16-key S^T tiles of a 32-key block take one group from each of the
// block's two pages), and the dims 32-wide k-steps j = d / 32; group t, k-step
// j is one 512-byte run of eight 64-byte rows (member s8 = 4 (s / 8) + s % 4),
// which is what one MFMA operand load of a wave reads from the page.
__host__ __device__ inline int key_elem(int s, int d, int head_dim) {
  const int t = (s >> 2) & 1, s8 = ((s >> 3) << 2) | (s & 3);
  return ((t * (head_dim >> 5) + (d >> 5)) * 8 + s8) * 32 + (d & 31);
}

// The same of an e4m3 page, whose 64-byte rows hold 64 dims: one load of 16 bytes a
// lane covers two MFMA k-steps of a key.
__host__ __device__ inline int key_elem8(int s, int d, int head_dim) {
  const int t = (s >> 2) & 1, s8 = ((s >> 3) << 2) | (s & 3);
  return ((t * (head_dim >> 6) + (d >> 6)) * 8 + s8) * 64 + (d & 63);
}
// Offset of value slot s, dim d in an e4m3 page's V region: 16-byte pieces of eight
// slots of dims 32 p + r and 32 p + 16 + r, in the order p, slot half, r: one load of
// 16 bytes a lane is its 8 keys of two 16-dim output tiles.
__host__ __device__ inline int val_elem8(int s, int d) {
  return (((d >> 5) * 2 + (s >> 3)) * 16 + (d & 15)) * 16 + ((d >> 4) & 1) * 8 + (s & 7);
}
// Offsets in the 32 scale bytes: a lane of the attention's score tiles reads the pair
// (slot, slot + 4) of its two keys, and eight consecutive slots' value scales.
__host__ __device__ inline int key_scale8(int s) { return (((s >> 3) << 2) | (s & 3)) * 2 + ((s >> 2) & 1); }
__host__ __device__ inline int val_scale8(int s) { return 16 + s; }

// The attention's eight work counters are a 128-byte line apart (in ints).
constexpr int kCtrStride = 32;

struct VerifySetupArgs {
  int B, k_max, vocab;
  int32_t* unit_ctr;  // attention work counters, cleared here
  int chunk;         // keys per attention item; doubled when that still leaves
  int items_double;  // at least this many items (enough to fill the attention grid),
  int items_fill;    // halved while that leaves at most this many and no request too many partials
  int G;        // query heads per kv-head
  int rb;       // attention row block of the step (rows per unit)
  int even;     // even cuts are tried first, two units a CU from chunks of 128 times this on (0: not)
  int cascade;  // 1: plan shared-prefix attention units for forked siblings
  const int32_t* seq_ids;
  const int32_t* ctx_lens;
  const int32_t* last_tokens;
  const int32_t* draft_tokens;
  const int32_t* draft_lens;
  const int32_t* draft_parents;  // nullable: tree drafts [B][k_max], parent of node i+1
};

// C[m][n] = sum_k A[arow(m)][k] * W[n][k]   (bf16 in, fp32 accumulate)
// W rows n < n_split come from W1, rows >= n_split from W2 (row n - n_split).
struct GemmArgs {
  const bf16_t* A;
  int lda;
  const int32_t* a_rows;  // nullable: A row m -> a_rows[m]
  const bf16_t* Wp;  // weights in MFMA fragment order (launch_pack_weights)
  int M, N, K, kper;
  bf16_t* out;       // EPI_SWIGLU: silu(gate) * up, bf16 [M][ld_out]
  int64_t ld_out;
  float* P;  // partial sums [split][M][N]
  // argmax epilogue (split == 1): per (row, 128-column block) best value and index
  float* logits;  // nullable [M][ld_logits]
  int64_t ld_logits;
  float* amax_v;
  int32_t* amax_i;
  int nan_max;  // argmax epilogue: a block that holds a NaN gets a NaN best value
};

enum { EPI_PARTIAL = 0, EPI_ARGMAX = 1, EPI_SWIGLU = 2 };

struct AttnArgs {
  const bf16_t* q;  // [rows][n_q_heads * head_dim]
  int64_t q_stride;
  KvGeom kv;
  int layer;
  const int32_t* table;
  int max_pages;
  StepMeta meta;
  int G, TB, n_kv_heads;
  int prb;           // rows per (item, kv-head) in the partials (the step's row block)
  float scale_log2;  // log2(e) / sqrt(head_dim)
  float* pm;         // [item][kvh][RB]
  float* pl;         // [item][kvh][RB]
  float* po;         // [item][kvh][RB][head_dim]
  bf16_t* o;         // combine output [rows][n_q_heads * head_dim]
  int64_t o_stride;  // elements between its rows
  int32_t* unit_ctr; // attention work counters; zero before each attention
                     // launch (the combine kernel resets them)
};

// allocator / setup (alloc.hip)
void launch_pool_init(const PoolDev& p, hipStream_t st);
void launch_grow(const PoolDev& p, int n, const int32_t* seq, const int32_t* a, const int32_t* b,
                 int mode, hipStream_t st);
void launch_verify_setup(const PoolDev& p, const VerifySetupArgs& a, const StepMeta& m,
                         hipStream_t st);
// The attention plan of given rows (nothing is reserved): draft_lens holds the requests'
// row counts, 0 .. k_max + 1; a request that its pages cannot hold fails the plan.
void launch_attend_plan(const PoolDev& p, const VerifySetupArgs& a, const StepMeta& m, hipStream_t st);
// The same in blocks of `TB` tokens (k_attn_rows): segment b * blocks + i is block i of
// request b.
//
// Their contexts are cut by estimated time, in keys a workgroup: a unit costs its keys and
// kUnitKeys for its start, its end and the merge of its partials.  Units of one length run
// in rounds of the grid (`slots` items of a kv-head), others fill in behind each other and
// end half a unit apart, and nothing ends before the longest.  (From integer sums, so that
// a plan repeats itself.)  Of the cuts within kCutNear of the least time the longest is
// taken: the estimate is no better than that (against the least, 8 of 256 rows behind
// 2000-20000 tokens 484 -> 472 us, bf16 461 -> 447, 4 of 500 behind 1000-9000 265 -> 278,
// 248 -> 255, the others of 20 shapes within 2%).  A kUnitKeys of 600 or 1500 moves no
// shape of either format by more than 6%.
constexpr int kRowCuts = 20;
constexpr float kUnitKeys = 1000.f, kCutNear = 1.02f;
// 512 keys times 1, 9/8, 11/8, 13/8, 2, ... 26
inline __host__ __device__ int row_cut(int c) { return (0xdb98 >> (4 * (c % 4)) & 15) << (c / 4 + 6); }
inline __host__ __device__ float row_cut_time(int chunk, int items, int64_t keys, int longest, int slots) {
  const float n = (float)(items > 1 ? items : 1), unit = (float)(chunk < longest ? chunk : longest) + kUnitKeys;
  const float rounds = (float)((items + slots - 1) / slots) * unit;
  const float filled = ((float)keys + n * kUnitKeys) / (float)slots + (float)keys / (2.f * n);
  return fminf(rounds, fmaxf(filled, unit));
}
struct RowPlanArgs {
  int B, n_max, TB, blocks;
  int chunk;        // keys per item that fit items_cap whatever the lengths
  int items_fill;   // items (of a kv-head) of one round of the grid
  int items_cap;    // items at most,
  int most_chunks;  // of a segment
  const int32_t *seq_ids, *ctx_lens, *n_lens;
  int32_t* unit_ctr;
};
void launch_attend_plan_rows(const PoolDev& p, const RowPlanArgs& a, const StepMeta& m, hipStream_t st);
void launch_commit(const PoolDev& p, int B, const int32_t* seq, int32_t* ctx, const int32_t* acc,
                   uint32_t commit_seq, hipStream_t st);
void launch_free(const PoolDev& p, int n, const int32_t* seq, hipStream_t st);
void launch_fork(const PoolDev& p, int src, int dst, int npg, hipStream_t st);
void launch_kv_load(const PoolDev& p, const KvGeom& g, int seq, int layer, int pos0, int n,
                    const bf16_t* src, hipStream_t st);
void launch_append_read(const PoolDev& p, int n, const int32_t* seq, const int32_t* ctx, int64_t total,
                        const int32_t* tokens, int vocab, int flags, int32_t* out, hipStream_t st);
void launch_add_ctx(int n, int32_t* ctx, const int32_t* add, hipStream_t st);

// keys and values of given tokens into or out of the pages (kv8.hip)
struct KvMove {
  int layer, B, n_max;
  const int32_t *seq, *pos, *n;  // [B]; null: seq0, pos0, n_max
  int seq0, pos0;
  bf16_t *k, *v;                 // row b * n_max + i: token pos[b] + i
  int64_t k_stride, v_stride;    // elements between rows
  int64_t head_stride;           // elements between a row's kv-heads
};
void launch_kv_move(bool write, const PoolDev& p, const KvGeom& g, const KvMove& m, hipStream_t st);

// GEMM of few rows (gemm.hip): at most 80, or 96 where gemm_tiled says so
void launch_gemm(const GemmArgs& g, int epi, int splits, hipStream_t st);
// Whether splits of `steps` k-steps have a fully unrolled kernel there at M rows.
inline bool gemm_unrolled(int M, int steps) {
  for (int s : {1, 2, 4, 8, 12, 16, 24, 32, 48})
    if (steps == s) return true;
  return steps == 64 && M > 32 && M <= 64;
}
// Whether a product runs in gemm_tile.hip.  More than 80 rows do, but an LM head of
// more than 256 128-id blocks from 97 on: at 81-96 rows its tiles make a nearly
// empty second round over the CUs where the streaming kernel, several workgroups a
// CU, stays at the weights' rate.  96 rows of a 4096-wide decoder: 32,768 ids 55.6 us
// streaming, 52.5 tiled; 36,864 ids 83 and 91, 65,536 ids 96 and 137, 151,936 ids
// 216 and 289 (at 112 rows 300 and 283).
inline bool gemm_tiled(int M, int N, int epi) { return M > (epi == EPI_ARGMAX && N > 256 * 128 ? 96 : 80); }
// GEMM over tiles in LDS (gemm_tile.hip): the tile shape, splits and k range a split
// that suit a shape, with the partial sums within cap_elems; shape -1 when none fits.
struct TilePlan {
  int shape, splits, kper;
};
constexpr int kTileShapes = 6;
TilePlan plan_gemm_tile(int M, int N, int K, int epi, int64_t cap_elems);
void launch_gemm_tile(const GemmArgs& g, int epi, int shape, int splits, hipStream_t st);
// W [N][K] row-major -> dst in MFMA fragment order; N % 16 == 0, K % 64 == 0
// Repack [N][K] weights (N % 128 == 0) into the GEMM's grouped fragment order;
// W2 non-null: W and W2 are the gate and up halves ([N/2][K] each) of a SwiGLU
// pair, interleaved in groups of 4 + 4 tiles.
void launch_pack_weights(const bf16_t* W, const bf16_t* W2, int N, int K, bf16_t* dst, hipStream_t st);

// sampled verification (sample.hip)
struct SampleArgs {
  const float* logits;     // [B * kp1][V] fp32
  int V;
  const int32_t* ntok;     // per request: drafts + 1 (0: no rows)
  const int32_t* drafts;   // [B][k_max]
  int k_max, kp1, B;
  const float* uniforms;   // [B * kp1][2]: acceptance test, draw
  float temperature;
  int top_k;
  // nullable: [B * kp1][V / 128], the largest logit of each 128-id block, NaN
  // where the block holds one (the LM head's argmax partials with nan_max)
  const float* block_max;
  int32_t* row_out;        // [B * kp1][3]: accepted?, token if rejected here, token if last
  const int32_t* greedy;   // nullable: constrained rows, -1 where one has no token at all
};

// constrained logits (constrain.hip)
struct ConstrainArgs {
  const float* logits;     // row b * (k_max + 1) + i at that many strides
  float* out;              // nullable; may be logits
  int64_t stride, out_stride;
  int V, B, k_max;
  const int32_t* ntok;     // rows of a request (the step's), or:
  const int32_t* draft_lens;  // nullable: rows - 1, clamped to [0, k_max]
  const int32_t *seq_ids, *last_tokens, *draft_tokens, *parents;
  // by sequence; any array may be null
  int n_seqs;
  const uint16_t* counts;
  const float *repetition, *frequency, *presence;
  int n_bias;
  const int32_t* bias_ids;
  const float* bias_values;
  int n_masks;
  const uint32_t* masks;
  const int32_t* mask_index;  // by row
  // nullable: [B * (k_max + 1)][ceil(V / 128)] best logit and id of each block of ids
  // (-inf and 0x7fffffff: none); nan_max: NaN where an allowed logit is NaN
  float* best_v;
  int32_t* best_i;
  int nan_max;
};
void launch_constrain(const ConstrainArgs& a, hipStream_t st);
void launch_greedy(const ConstrainArgs& a, int32_t* greedy, bool finite, hipStream_t st);
void launch_counts_begin(uint16_t* counts, int V, int n_seqs, int B, const int32_t* seq_ids, const int32_t* tokens,
                         int n_tokens, const int32_t* offsets, hipStream_t st);
void launch_counts_add(uint16_t* counts, int V, int n_seqs, int B, const int32_t* seq_ids, const int32_t* first,
                       const int32_t* tokens, int n_max, const int32_t* path, const int32_t* lens, hipStream_t st);
void launch_block_max(const float* logits, int rows, int V, float* block_max, hipStream_t st);
void launch_sample(const SampleArgs& s, int32_t* accept_lens, int32_t* next_tokens, hipStream_t st);

// attention (attn.hip)
int attn_rows_per_block(int G, int k_rows);  // RB (16, 32 or 48)
void launch_attn(const AttnArgs& a, int RB, int head_dim, int grid, hipStream_t st);
// 128-row blocks of a prefill (attn_rows.hip)
void launch_attn_rows(const AttnArgs& a, int head_dim, int grid, hipStream_t st);
void launch_attn_combine(const AttnArgs& a, int RB, int head_dim, int n_segs, hipStream_t st);

// elementwise / row kernels (rows.hip)
struct ModelDims {
  int d, nq, nkv, hd, F, V, qkv;
  float eps;
};
// embeddings and first norm, and the RoPE table of the pass
void launch_embed_norm(int rows, const int32_t* tok, const bf16_t* E, const bf16_t* g, int d,
                       float eps, float* h, bf16_t* u, const int32_t* pos, const double* inv_freq,
                       int half, float* cos_t, float* sin_t, hipStream_t st);
void launch_residual_norm(int rows, int splits, const float* P, int d, const bf16_t* g, float eps,
                          float* h, bf16_t* u, hipStream_t st);
void launch_qkv_rope(int rows, int splits, const float* P, const ModelDims& md,
                     const float* cos_t, const float* sin_t, const StepMeta& meta,
                     const int32_t* row_req, const int32_t* table, int max_pages, const KvGeom& kv,
                     int layer, bf16_t* q, hipStream_t st);
// none: the greedy token of a row without any (constrained rows: -1).
// parents (nullable): tree drafts; accept_path [n_req][k_max] then receives the
// accepted nodes in depth order, -1 beyond the accept length
void launch_argmax_accept(int n_req, const int32_t* ntok, int row_stride, int n_blocks,
                          const float* amax_v, const int32_t* amax_i, const int32_t* draft_tokens,
                          const int32_t* parents, int k_max, int32_t* accept_lens, int32_t* next_tokens,
                          int32_t* accept_path, hipStream_t st, int none = 0x7fffffff);
// Tree drafts: move the KV of each request's accepted nodes (slots ctx + node)
// to slots ctx + 1 .. ctx + accept_len, every layer.
void launch_kv_compact(const KvGeom& kv, int n_layers, int B, const StepMeta& meta, const int32_t* table,
                       int max_pages, const int32_t* accept_lens, const int32_t* accept_path, int k_max,
                       hipStream_t st);
