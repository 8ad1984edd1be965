// Launchers of the token operators: attention, the gated norm coupling, dropout.
// Arguments are checked by the C entry points; these only enqueue.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace petra {

// --- coupling ---------------------------------------------------------------
struct CoupleArgs {
  long rows, rows_per_gate, gates;
  long row0;                                 // forward: the launch's first row
  int width, layer;
  int has_f, has_u;                          // backward: which parts it has
  float eps, scale, inv_scale, inv_width, inv_keep;
  uint32_t cut;
  const uint64_t* rng;                       // null: no dropout
  const void *x, *f;                         // forward's inputs (f shared with backward)
  const float *post_gamma, *post_beta, *gate, *pre_gamma, *pre_beta;
  void *y, *u;                               // forward's outputs
  const void *y_in, *dy, *du;                // backward's inputs
  void *x_out, *dx, *df;                     // backward's outputs
  float *dgate, *dpost_gamma, *dpost_beta, *dpre_gamma, *dpre_beta;
  // backward: workgroups, and how they share the rows: gates_per_block whole gates
  // each, or (chunks_per_gate > 1) rows_per_chunk rows of one gate
  long blocks, gates_per_block, chunks_per_gate, rows_per_chunk;
  float *part_gate, *part_post_gamma, *part_post_beta, *part_pre_gamma, *part_pre_beta;
};

// How the backward's workgroups share the rows (blocks and the three fields after it).
void couple_plan(CoupleArgs& a);
void couple_forward(const CoupleArgs& a, int dtype, hipStream_t s);
void couple_backward(const CoupleArgs& a, int dtype, hipStream_t s);

// --- dropout ----------------------------------------------------------------
void dropout(const void* x, const void* residual, void* y, long n, float factor, uint32_t cut,
             const uint64_t* rng, int dtype, hipStream_t s);

// --- attention --------------------------------------------------------------
// Row r of a key head's queries is token r / group of query head r % group of the
// heads that share it, so that a tile of rows is one of queries whatever the group.
struct AttnArgs {
  const void *q, *k, *v, *o, *d_o;
  void *out, *dq, *dk, *dv;
  float* lse;                                // [batch][heads][q_len]
  float *stat_lse, *stat_delta;              // backward: log2(e) lse (+inf without keys) and D, [batch x key heads][rows]
  const int32_t *q_lens, *kv_lens;
  const uint64_t* rng;                       // null: no dropout
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];   // batch, token, head
  int batch, q_len, kv_len, heads, kv_heads, group, dim, causal;
  float scale, scale_log2, inv_keep;         // scale_log2 = scale log2(e)
  uint32_t cut;
  // keys (forward, query gradient) or rows (key and value gradients) split over
  // `splits` workgroups, whose fp32 partial results go to `part`
  int splits, tiles;                         // tiles: of rows or keys, of one key head
  int bh0, bhs;                              // the launch's first (batch row, key head), and how many
  float *part, *part_ml;
};

struct AttnPlan {
  int row_tile, splits;            // forward
  size_t fwd_bytes;
  int dq_tile, key_tile, dq_splits, dkv_splits;   // backward
  size_t stat_bytes, bwd_bytes;
};

AttnPlan attn_plan(const AttnArgs& a);
void attn_forward(const AttnArgs& a, const AttnPlan& p, int dtype, void* workspace, hipStream_t s);
void attn_backward(const AttnArgs& a, const AttnPlan& p, int dtype, void* workspace, hipStream_t s);

// --- head norms and rotation ------------------------------------------------
constexpr int HEADS_AXES = 4, HEADS_PAIRS = 64;

// The queries, or the keys.
struct HeadsPart {
  const void *x, *dy;
  void *y, *dx;
  const float *gamma, *beta;                 // null gamma: no norm
  float *dgamma, *dbeta, *part_gamma, *part_beta;
  int64_t x_stride[3], y_stride[3];          // batch, token, head; dx like x, dy like y
  int heads;
  // workgroups: `groups` of tokens times `splits` of heads, each `rounds` of 2^head_bits
  int blocks, groups, splits, rounds, head_bits;
};
struct HeadsArgs {
  HeadsPart part[2];
  const int32_t* positions;                  // [axes][tokens]; null: a token's index in its sequence
  long tokens;                               // batch * len
  uint32_t len;
  int dim, pairs, axes, halves, layer;
  float eps, inv_dim;
  uint64_t freq[HEADS_PAIRS];                // 2^64 of a turn a position; 0 past the pairs
  uint32_t axes4[HEADS_PAIRS / 8];           // axes of the pairs, 4 bits each
};

// The workgroups of both parts (without tokens none).
void heads_plan(HeadsArgs& a, bool backward);
void heads_forward(const HeadsArgs& a, int dtype, hipStream_t s);
void heads_backward(const HeadsArgs& a, int dtype, hipStream_t s);

// --- loss over a vocabulary -------------------------------------------------
// A gradient: rows x cols results of the product of a (a_ld between its lines) and b (cols between its lines, b_inner
// of them) over `inner`, split over `splits` workgroups of per_split.
struct VocabGrad {
  const void *a, *b;
  void* out;
  const float *factor, *rest;                // [rows], nullable together: factors, and those of b's lines `targets` beside the product
  const int32_t* targets;
  // dw: where each column's target rows begin in `order` (nullable), the rows' terms of it, factors and x; and for columns of many
  // what rounding left of these, a sum for each run of 2^run_bits rows
  const int *start, *order;
  const float *term, *row_factor, *left;
  const void* x;
  int run_bits;
  float *part, *acc;                         // the splits' sums; sums over the pieces of rows
  long rows, cols, inner, a_ld, a_free, b_inner, per_split;   // a_free: rows, or as many as a's lines have
  int splits, tile, row_tiles, col_tiles, add, last;
};
struct VocabArgs {
  const void *x, *w;
  const int32_t* targets;
  const float* weight;                       // nullable: *mean
  float *loss, *lse;
  void *dx, *dw;
  long rows, row0, piece;                    // all rows, and those at work
  int width, vocab, vocab_padded;            // padded: of e, in which the rest is zeros
  int row_tiles, col_tiles, row_tile, col_tile;
  float scale, scale_log2;                   // scale_log2 = scale log2(e)
  // workspace: each row's reference; of a piece the tiles' sums, the references that differ and which tiles
  // have them, e, factors, x times them, and what rounding the targets' terms left
  float *ref, *sums, *shift, *mean, *factor, *rest, *term, *left, *part, *acc;
  int *slow, *start, *order;
  void *scaled, *e;
};
struct VocabPlan {
  long piece;
  bool lists;                                // rows by their targets, for dw
  int run_bits;
  int row_tile, col_tile;                    // of the scores
  VocabGrad dx, dw;                          // tile, splits and per_split
  size_t ref, sums, shift, slow, mean, factor, rest, term, start, order, left, scaled, e, part, acc, bytes;   // offsets in the workspace
};

// piece_rows: rows at a time (0: by the rule).
VocabPlan vocab_plan(const VocabArgs& a, int dtype, bool gradients, long piece_rows);
void vocab_run(VocabArgs a, const VocabPlan& p, int dtype, bool gradients, void* workspace, hipStream_t s);

// --- AdamW ------------------------------------------------------------------
constexpr int ADAMW_CHUNK = 4096;            // elements a workgroup

// A tensor of the table in device memory, and where it lies among the chunks and the generator's groups of 4 elements.
struct AdamwEntry {
  float* theta;
  void *grad, *m, *v, *copy;
  float *m_scale, *v_scale;
  int64_t n, padded, first_chunk, first_group;
  float decay;
  int32_t reserved;
};
struct AdamwArgs {
  const AdamwEntry* entries;
  const int32_t* chunk_of;                   // the tensor of each chunk
  long chunks;
  int64_t* steps;
  const float *lr, *grad_scale;
  const uint64_t* rng;
  float* hyper;                              // workspace: corrections of m and of sqrt(v)
  double log_b1, log_b2;
  float b1, c1, b2, c2, eps;                 // c = 1 - b
  int zero_grads;
};

void adamw_step(const AdamwArgs& a, bool bf16_grads, bool fp8, hipStream_t s);

}  // namespace petra
