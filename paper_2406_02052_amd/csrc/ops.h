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

}  // namespace petra
