// Passes over trees of drafted tokens: new rows into a paged cache, attention of
// a tree's rows over it, commit of the accepted path (tree.hip; entry points in
// operators.cpp).
#pragma once

#include "ctx.h"

namespace specdec {

// The rows of a pass (include/spec.h, spec_rows) over one pool of pages.
struct TreeRows {
  int B, rows, stride;
  const int32_t *first, *len, *table, *parent;
  int32_t* err;
  int pages, nkv;          // of the pool
};

struct AppendArgs {
  TreeRows t;
  bf16_t *kc, *vt;         // the layer's pools
  const bf16_t *q, *k, *v;
  int64_t q_stride, kv_stride;
  bf16_t* q_out;
  int64_t q_out_stride;
  int nq;
  const int32_t* pos;      // [3][rows] or null
  int axis_end[2];         // pairs before it are on axis T, before the second on H; interleaved: -1
  double turns[64];        // theta_d / 2 pi
  int heads;               // that a workgroup rotates
};
hipError_t launch_kv_append(AppendArgs& a, int D, hipStream_t s);

// A (sequence, kv head, chunk of query rows), as the combine needs it.
struct TreeUnit {
  int part, groups;        // its first group's number, how many
  int first, row, rows, head;   // the sequence's first row; of the kv head's query rows the chunk's first, and all; its first head
};

struct TreeAttnArgs {
  TreeRows t;
  const bf16_t *kc, *vt;
  const bf16_t* q;
  int64_t q_stride;
  bf16_t* out;
  int64_t out_stride;
  float* lse;              // [rows][nq] or null
  int nq, G;
  float scale_log2;
  int target, least;       // groups aimed at; pages of a group at least
  float __attribute__((ext_vector_type(4)))* part;   // [groups][tiles][D / 8][64] outputs of groups
  float2* ml;              // [groups][tiles][32] (maximum in log2 units, sum)
  TreeUnit* units;         // [0].first: how many; then each
};
// How a call is laid out, and its workspace: part, ml, units.
struct TreeAttnPlan {
  int tiles;               // of 32 query rows of a kv head that a workgroup has
  int units, target, least, grid;
  bool combine;            // a sequence may have several groups
  int likely;              // groups of a sequence whose pages fill the table
  size_t ml, unit, bytes;
};
TreeAttnPlan tree_attn_plan(int batch, int rows, int nkv, int G, int D, int stride, int ncu);
hipError_t launch_tree_attn(TreeAttnArgs& a, const TreeAttnPlan& p, int D, void* workspace, hipStream_t s);

struct TreeCommitArgs {
  TreeRows t;
  int layers;
  int64_t layer_stride;
  bf16_t *kc, *vt;
  const int32_t *tokens, *greedy, *budget;
  int stop;
  int32_t *path, *committed, *n, *new_len;
};
hipError_t launch_tree_commit(const TreeCommitArgs& a, int D, hipStream_t s);

}  // namespace specdec
