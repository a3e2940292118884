// Entry points of the operators that need no context (include/spec.h): pages of
// a cache held in 8 bits, attention over them, scores of logits; passes over trees.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "ctx.h"
#include "kv8.h"
#include "logprobs.h"
#include "tree.h"

using namespace specdec;

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxRowsPerHead = 16 * 65535, kMaxPageHeads = 1 << 27, kMaxPackRows = 1 << 28;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, uintptr_t a) { return p && reinterpret_cast<uintptr_t>(p) % a == 0; }

// Leaves the text for spec_last_error(NULL); nothing is thrown out of an entry.
spec_status fail(spec_status s, const char* func, const char* what) noexcept {
  try {
    set_global_error(std::string(func) + ": " + what);
  } catch (...) {
  }
  return s;
}
spec_status launched(hipError_t e, const char* func) noexcept {
  return e == hipSuccess ? SPEC_OK : fail(SPEC_E_HIP, func, hipGetErrorString(e));
}

// What is wrong with a cache's description, or null.
const char* bad_cache(const spec_kv8* c, bool bf16_too) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->kv_heads < 1) return "kv_heads must be at least 1";
  if (c->pages8 < 0 || (bf16_too && c->pages16 < 0)) return "negative page count";
  if (c->pages8 > 0 && (!aligned(c->k8, 16) || !aligned(c->v8, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)))
    return "8-bit pages or scales null or misaligned";
  if (bf16_too && c->pages16 > 0 && (!aligned(c->k16, 16) || !aligned(c->v16, 16))) return "bf16 pages null or misaligned";
  return nullptr;
}

const char* bad_pass(const spec_kv8* c, int32_t batch, int32_t rows, int32_t q_heads, int32_t table_stride) {
  if (const char* w = bad_cache(c, true)) return w;
  if (batch < 1 || rows < 1 || (int64_t)batch * rows > SPEC_MAX_ROWS) return "batch and rows must be at least 1, batch*rows at most SPEC_MAX_ROWS";
  if (q_heads < 1 || q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads";
  if ((int64_t)q_heads * c->head_dim > (1 << 20)) return "q_heads*head_dim too large";
  // (row blocks are a grid's second dimension; threads of all groups fit 32 bits)
  if (rows * (int64_t)(q_heads / c->kv_heads) > kMaxRowsPerHead) return "rows*q_heads/kv_heads too large";
  if (table_stride < 1 || table_stride > INT32_MAX / SPEC_KV_PAGE) return "table_stride out of range";
  if ((int64_t)batch * c->kv_heads * table_stride > kMaxPageHeads) return "batch*kv_heads*table_stride too large";
  return nullptr;
}

struct AttnPlan {
  int target;
  int64_t groups;
  size_t ml, bytes;   // offset of the maxima and sums; all
};
AttnPlan attn_plan(const spec_kv8* c, int batch, int rows, int q_heads, int stride) {
  const int r = rows * (q_heads / c->kv_heads);
  AttnPlan p;
  p.target = kv8_target_groups(r, num_cus());
  p.groups = kv8_max_groups(batch, c->kv_heads, stride, 0, p.target);
  p.ml = align_up(kv8_part_bytes(p.groups, r, c->head_dim));
  p.bytes = p.ml + align_up(kv8_ml_bytes(p.groups, r));
  return p;
}

const char* bad_scores(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 1 || rows > 65535) return "rows out of range";
  if (vocab < 1 || vocab > kLogprobMaxVocab) return "vocab out of range";
  if (top < 0 || top > SPEC_MAX_TOP || top > vocab) return "top must be 0..SPEC_MAX_TOP and at most vocab";
  return nullptr;
}

constexpr int32_t kMaxTable = (1 << 25) - 16;   // (slots and a tree's rows behind them fit 32 bits)

// What is wrong with a cache, or with a pass over it, or null.
const char* bad_kv(const spec_kv* c) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->kv_heads < 1 || c->kv_heads > 65535) return "kv_heads must be 1..65535";
  if (c->pages < 1) return "pages must be at least 1";
  if (c->layers < 1 || c->layers > SPEC_MAX_LAYERS) return "layers must be 1..SPEC_MAX_LAYERS";
  if (c->layers > 1 && (c->layer_stride % 8 || c->layer_stride / (SPEC_KV_PAGE * c->head_dim) < (int64_t)c->pages * c->kv_heads ||
                        c->layer_stride > INT64_MAX / (4 * SPEC_MAX_LAYERS)))
    return "layer_stride must be a multiple of 8 and at least a pool";
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return "keys or values null or misaligned";
  return nullptr;
}
const char* bad_layer(const spec_kv* c, int32_t layer) {
  if (const char* w = bad_kv(c)) return w;
  return layer < 0 || layer >= c->layers ? "no such layer" : nullptr;
}
const char* bad_rows(const spec_rows* r, int32_t most) {
  if (!r) return "null rows";
  if (r->batch < 1 || r->batch > SPEC_MAX_ROWS) return "batch must be 1..SPEC_MAX_ROWS";
  if (r->rows < 1 || r->rows > most) return "rows out of range";
  if (r->table_stride < 1 || r->table_stride > kMaxTable) return "table_stride out of range";
  if (!aligned(r->d_first, 4) || !aligned(r->d_len, 4) || !aligned(r->d_table, 4) || (r->d_parent && !aligned(r->d_parent, 4)) ||
      (r->d_err && !aligned(r->d_err, 4)))
    return "rows: null or misaligned pointer";
  return nullptr;
}
const char* bad_tree_pass(const spec_kv* c, const spec_rows* r, int32_t q_heads) {
  if (const char* w = bad_rows(r, SPEC_MAX_ROWS)) return w;
  if (q_heads < 1 || q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads";
  if ((int64_t)q_heads * c->head_dim > (1 << 20)) return "q_heads*head_dim too large";
  if ((int64_t)r->batch * c->kv_heads * r->table_stride > kMaxPageHeads) return "batch*kv_heads*table_stride too large";
  return nullptr;
}
TreeRows tree_rows(const spec_kv* c, const spec_rows* r) {
  return TreeRows{r->batch, r->rows, r->table_stride, r->d_first, r->d_len, r->d_table, r->d_parent, r->d_err, c->pages, c->kv_heads};
}
TreeAttnPlan attn_plan(const spec_kv* c, const spec_rows* r, int32_t q_heads) {
  return tree_attn_plan(r->batch, r->rows, c->kv_heads, q_heads / c->kv_heads, c->head_dim, r->table_stride, num_cus());
}
bf16_t* layer_of(const spec_kv* c, void* pool, int32_t layer) {
  return static_cast<bf16_t*>(pool) + (c->layers > 1 ? layer * c->layer_stride : 0);
}
// Whether [a, a + n) and [b, b + m) share a byte (null: nothing there).
bool overlap(const void* a, size_t n, const void* b, size_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x && y && x < y + m && y < x + n;
}

}  // namespace

extern "C" {

spec_status spec_kv8_pack(const spec_kv8* c, const void* k, const void* v, int64_t row_stride, int32_t rows,
                          const int32_t* d_pages, int32_t* d_err, hipStream_t stream) {
  const char* const f = "spec_kv8_pack";
  if (const char* w = bad_cache(c, false)) return fail(SPEC_E_INVAL, f, w);
  if (c->pages8 < 1) return fail(SPEC_E_INVAL, f, "no 8-bit pages");
  if (c->kv_heads > 65535) return fail(SPEC_E_INVAL, f, "too many kv heads");
  if (rows < 1 || rows > kMaxPackRows) return fail(SPEC_E_INVAL, f, "rows must be 1..2^28");
  if (row_stride < (int64_t)c->kv_heads * c->head_dim || row_stride % 8)
    return fail(SPEC_E_INVAL, f, "row_stride must be a multiple of 8 and at least kv_heads*head_dim");
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(d_pages, 4) || (d_err && !aligned(d_err, 4)))
    return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  Kv8PackArgs a{};
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.stride = row_stride;
  a.rows = rows;
  a.nkv = c->kv_heads;
  a.pages8 = c->pages8;
  a.to = d_pages;
  a.k8 = static_cast<uint8_t*>(c->k8);
  a.v8 = static_cast<uint8_t*>(c->v8);
  a.ks = c->k_scale;
  a.vs = c->v_scale;
  a.err = d_err;
  return launched(launch_kv8_pack(a, c->head_dim, stream), f);
}

spec_status spec_kv8_attn_workspace_bytes(const spec_kv8* c, int32_t batch, int32_t rows, int32_t q_heads,
                                          int32_t table_stride, size_t* bytes) {
  const char* const f = "spec_kv8_attn_workspace_bytes";
  if (!bytes) return fail(SPEC_E_INVAL, f, "null result");
  if (const char* w = bad_pass(c, batch, rows, q_heads, table_stride)) return fail(SPEC_E_INVAL, f, w);
  *bytes = attn_plan(c, batch, rows, q_heads, table_stride).bytes;
  return SPEC_OK;
}

spec_status spec_kv8_attn(const spec_kv8* c, int32_t batch, int32_t rows, int32_t q_heads, const int32_t* d_table,
                          int32_t table_stride, const int32_t* d_packed, const int32_t* d_visible, const void* q,
                          int64_t q_stride, float scale, void* out, int64_t out_stride, float* d_lse, int32_t* d_err,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const char* const f = "spec_kv8_attn";
  if (const char* w = bad_pass(c, batch, rows, q_heads, table_stride)) return fail(SPEC_E_INVAL, f, w);
  const int64_t width = (int64_t)q_heads * c->head_dim;
  if (q_stride < width || q_stride % 8 || out_stride < width || out_stride % 8)
    return fail(SPEC_E_INVAL, f, "q_stride and out_stride must be multiples of 8 and at least q_heads*head_dim");
  // (its product with log2 e is finite)
  if (!(scale > 0.f && scale <= 0x1p127f)) return fail(SPEC_E_INVAL, f, "scale must be positive and at most 2^127");
  if (!aligned(d_table, 4) || !aligned(d_packed, 4) || !aligned(d_visible, 4) || !aligned(q, 16) || !aligned(out, 16) ||
      (d_lse && !aligned(d_lse, 4)) || (d_err && !aligned(d_err, 4)))
    return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  const AttnPlan p = attn_plan(c, batch, rows, q_heads, table_stride);
  if (!aligned(workspace, kAlign)) return fail(SPEC_E_INVAL, f, "workspace: null or not 256-byte aligned");
  if (workspace_bytes < p.bytes) return fail(SPEC_E_CAPACITY, f, "workspace too small (query spec_kv8_attn_workspace_bytes)");
  Kv8AttnArgs a{};
  a.vis = d_visible;
  a.packed = d_packed;
  a.table = d_table;
  a.stride = table_stride;
  a.k8 = static_cast<const uint8_t*>(c->k8);
  a.v8 = static_cast<const uint8_t*>(c->v8);
  a.ks = c->k_scale;
  a.vs = c->v_scale;
  a.k16 = static_cast<const bf16_t*>(c->k16);
  a.v16 = static_cast<const bf16_t*>(c->v16);
  a.pages8 = c->pages8;
  a.pages16 = c->pages16;
  a.q = static_cast<const bf16_t*>(q);
  a.q_stride = q_stride;
  a.out = static_cast<bf16_t*>(out);
  a.out_stride = out_stride;
  a.lse = d_lse;
  a.err = d_err;
  a.B = batch;
  a.R = rows;
  a.nq = q_heads;
  a.nkv = c->kv_heads;
  a.G = q_heads / c->kv_heads;
  kv8_set_parts(a, workspace, static_cast<char*>(workspace) + p.ml, p.groups);
  a.target = p.target;
  a.many = kv8_many(p.groups, batch, c->kv_heads);
  a.scale_log2 = scale * 1.4426950408889634f;
  const spec_status s = launched(launch_kv8_attn(a, c->head_dim, p.groups, stream), f);
  return s != SPEC_OK ? s : launched(launch_kv8_combine(a, c->head_dim, stream), f);
}

spec_status spec_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top, size_t* bytes) {
  const char* const f = "spec_logprobs_workspace_bytes";
  if (!bytes) return fail(SPEC_E_INVAL, f, "null result");
  if (const char* w = bad_scores(rows, vocab, top)) return fail(SPEC_E_INVAL, f, w);
  const int splits = logprob_splits(rows, vocab, num_cus());
  *bytes = align_up(logprob_stats_bytes(rows, splits)) + align_up(logprob_key_bytes(rows, splits, top));
  return SPEC_OK;
}

spec_status spec_logprobs(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                          const int32_t* d_tokens, int32_t n_tokens, int32_t top, float* d_logprob, float* d_entropy,
                          int32_t* d_top_token, float* d_top_logprob, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  const char* const f = "spec_logprobs";
  if (const char* w = bad_scores(rows, vocab, top)) return fail(SPEC_E_INVAL, f, w);
  if (dtype != SPEC_BF16 && dtype != SPEC_F16 && dtype != SPEC_F32) return fail(SPEC_E_INVAL, f, "unknown dtype");
  if (row_stride < vocab) return fail(SPEC_E_INVAL, f, "row_stride must be at least vocab");
  if (n_tokens < 0) return fail(SPEC_E_INVAL, f, "n_tokens must not be negative");
  if (!aligned(logits, dtype == SPEC_F32 ? 4 : 2) || (d_entropy && !aligned(d_entropy, 4)) ||
      (n_tokens > 0 && (!aligned(d_tokens, 4) || !aligned(d_logprob, 4))) ||
      (top > 0 && (!aligned(d_top_token, 4) || !aligned(d_top_logprob, 4))))
    return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  const int splits = logprob_splits(rows, vocab, num_cus());
  const size_t stats = align_up(logprob_stats_bytes(rows, splits));
  if (!aligned(workspace, kAlign)) return fail(SPEC_E_INVAL, f, "workspace: null or not 256-byte aligned");
  if (workspace_bytes < stats + align_up(logprob_key_bytes(rows, splits, top)))
    return fail(SPEC_E_CAPACITY, f, "workspace too small (query spec_logprobs_workspace_bytes)");
  LogprobArgs a{};
  a.x = logits;
  a.stride = row_stride;
  a.rows = rows;
  a.V = vocab;
  a.given = d_tokens;
  a.ng = n_tokens;
  a.top = top;
  a.lp = d_logprob;
  a.entropy = d_entropy;
  a.top_i = d_top_token;
  a.top_lp = d_top_logprob;
  a.stats = static_cast<float4*>(workspace);
  a.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + stats);
  a.splits = splits;
  return launched(launch_logprobs(a, dtype, stream), f);
}

spec_status spec_kv_append(const spec_kv* c, int32_t layer, const spec_rows* r, const spec_rope* rope, const int32_t* d_pos,
                           int32_t q_heads, const void* q, int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                           void* q_out, int64_t q_out_stride, hipStream_t stream) {
  const char* const f = "spec_kv_append";
  if (const char* w = bad_layer(c, layer)) return fail(SPEC_E_INVAL, f, w);
  if (const char* w = bad_rows(r, r && r->d_parent && !d_pos ? SPEC_MAX_ROWS : kMaxPackRows)) return fail(SPEC_E_INVAL, f, w);
  if (!rope) return fail(SPEC_E_INVAL, f, "null rope");
  if (!(rope->base > 1.f) || !std::isfinite(rope->base)) return fail(SPEC_E_INVAL, f, "base must be > 1");
  if (rope->interleaved != 0 && rope->interleaved != 1) return fail(SPEC_E_INVAL, f, "interleaved must be 0 or 1");
  const int32_t *sec = rope->section, half = c->head_dim / 2;
  if (sec[0] < 0 || sec[1] < 0 || sec[2] < 0 || (int64_t)sec[0] + sec[1] + sec[2] != half)
    return fail(SPEC_E_INVAL, f, "section must be non-negative and sum to head_dim/2");
  if (q_heads < 0 || (int64_t)q_heads * c->head_dim > (1 << 20)) return fail(SPEC_E_INVAL, f, "q_heads out of range");
  if (q_heads + 2 * c->kv_heads > 65535) return fail(SPEC_E_INVAL, f, "too many heads");   // a grid's second dimension
  const int64_t width = (int64_t)q_heads * c->head_dim;
  if (q_heads > 0 && (q_stride < width || q_stride % 8 || q_out_stride < width || q_out_stride % 8))
    return fail(SPEC_E_INVAL, f, "q_stride and q_out_stride must be multiples of 8 and at least q_heads*head_dim");
  if (kv_stride < (int64_t)c->kv_heads * c->head_dim || kv_stride % 8)
    return fail(SPEC_E_INVAL, f, "kv_stride must be a multiple of 8 and at least kv_heads*head_dim");
  if (!aligned(k, 16) || !aligned(v, 16) || (q_heads > 0 && (!aligned(q, 16) || !aligned(q_out, 16))) || (d_pos && !aligned(d_pos, 4)))
    return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  if (q_heads > 0 && q == q_out && q_stride != q_out_stride) return fail(SPEC_E_INVAL, f, "q_out on q needs the same stride");
  AppendArgs a{};
  a.t = tree_rows(c, r);
  a.kc = layer_of(c, c->k, layer);
  a.vt = layer_of(c, c->v, layer);
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.q_stride = q_stride;
  a.kv_stride = kv_stride;
  a.q_out = static_cast<bf16_t*>(q_out);
  a.q_out_stride = q_out_stride;
  a.nq = q_heads;
  a.pos = d_pos;
  a.axis_end[0] = rope->interleaved ? -1 : sec[0];
  a.axis_end[1] = rope->interleaved ? -1 : sec[0] + sec[1];
  // base^(-2 d / head_dim) / 2 pi of d = 8 i + j as two factors: 16 powers a call instead of 64, which took 1.3 us
  double low[8];
  for (int j = 0; j < 8; ++j) low[j] = std::pow((double)rope->base, -2.0 * j / c->head_dim);
  for (int i = 0; i < half; i += 8) {
    const double high = std::pow((double)rope->base, -2.0 * i / c->head_dim) / 6.283185307179586476925286766559;
    for (int j = 0; j < 8; ++j) a.turns[i + j] = high * low[j];
  }
  return launched(launch_kv_append(a, c->head_dim, stream), f);
}

spec_status spec_tree_attn_workspace_bytes(const spec_kv* c, const spec_rows* r, int32_t q_heads, size_t* bytes) {
  const char* const f = "spec_tree_attn_workspace_bytes";
  if (!bytes) return fail(SPEC_E_INVAL, f, "null result");
  if (const char* w = bad_kv(c)) return fail(SPEC_E_INVAL, f, w);
  if (const char* w = bad_tree_pass(c, r, q_heads)) return fail(SPEC_E_INVAL, f, w);
  *bytes = attn_plan(c, r, q_heads).bytes;
  return SPEC_OK;
}

spec_status spec_tree_attn(const spec_kv* c, int32_t layer, const spec_rows* r, int32_t q_heads, const void* q, int64_t q_stride,
                           float scale, void* out, int64_t out_stride, float* d_lse, void* workspace, size_t workspace_bytes,
                           hipStream_t stream) {
  const char* const f = "spec_tree_attn";
  if (const char* w = bad_layer(c, layer)) return fail(SPEC_E_INVAL, f, w);
  if (const char* w = bad_tree_pass(c, r, q_heads)) return fail(SPEC_E_INVAL, f, w);
  const int64_t width = (int64_t)q_heads * c->head_dim;
  if (q_stride < width || q_stride % 8 || out_stride < width || out_stride % 8)
    return fail(SPEC_E_INVAL, f, "q_stride and out_stride must be multiples of 8 and at least q_heads*head_dim");
  // (its product with log2 e is finite)
  if (!(scale > 0.f && scale <= 0x1p127f)) return fail(SPEC_E_INVAL, f, "scale must be positive and at most 2^127");
  if (!aligned(q, 16) || !aligned(out, 16) || (d_lse && !aligned(d_lse, 4))) return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  if (!aligned(workspace, kAlign)) return fail(SPEC_E_INVAL, f, "workspace: null or not 256-byte aligned");
  const TreeAttnPlan p = attn_plan(c, r, q_heads);
  if (workspace_bytes < p.bytes) return fail(SPEC_E_CAPACITY, f, "workspace too small (query spec_tree_attn_workspace_bytes)");
  TreeAttnArgs a{};
  a.t = tree_rows(c, r);
  a.kc = layer_of(c, c->k, layer);
  a.vt = layer_of(c, c->v, layer);
  a.q = static_cast<const bf16_t*>(q);
  a.q_stride = q_stride;
  a.out = static_cast<bf16_t*>(out);
  a.out_stride = out_stride;
  a.lse = d_lse;
  a.nq = q_heads;
  a.G = q_heads / c->kv_heads;
  a.scale_log2 = scale * 1.4426950408889634f;
  return launched(launch_tree_attn(a, p, c->head_dim, workspace, stream), f);
}

spec_status spec_tree_commit(const spec_kv* c, const spec_rows* r, const int32_t* d_tokens, const int32_t* d_greedy,
                             int32_t stop_token, const int32_t* d_budget, int32_t* d_path, int32_t* d_committed, int32_t* d_n,
                             int32_t* d_new_len, hipStream_t stream) {
  const char* const f = "spec_tree_commit";
  if (const char* w = bad_kv(c)) return fail(SPEC_E_INVAL, f, w);
  if (const char* w = bad_rows(r, SPEC_MAX_ROWS)) return fail(SPEC_E_INVAL, f, w);
  if (stop_token < -1) return fail(SPEC_E_INVAL, f, "stop_token must be -1 or a token");
  const size_t rows = 4 * (size_t)r->rows, batch = 4 * (size_t)r->batch;
  const struct { const void* p; size_t n; } in[] = {{r->d_first, batch + 4}, {r->d_len, batch}, {r->d_table, batch * r->table_stride},
                                                    {r->d_parent, rows}, {d_tokens, rows}, {d_greedy, rows}, {d_budget, batch}},
                                            out[] = {{d_path, rows}, {d_committed, rows}, {d_n, batch}, {d_new_len, batch}};
  if (!aligned(d_tokens, 4) || !aligned(d_greedy, 4) || (d_budget && !aligned(d_budget, 4)))
    return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
  for (const auto& o : out) {
    if (o.p && !aligned(o.p, 4)) return fail(SPEC_E_INVAL, f, "null or misaligned pointer");
    // every workgroup reads the inputs while one writes these
    for (const auto& i : in)
      if (overlap(o.p, o.n, i.p, i.n)) return fail(SPEC_E_INVAL, f, "an output overlaps an input");
    for (const auto& p : out)
      if (&p != &o && overlap(o.p, o.n, p.p, p.n)) return fail(SPEC_E_INVAL, f, "outputs overlap");
  }
  TreeCommitArgs a{};
  a.t = tree_rows(c, r);
  a.layers = c->layers;
  a.layer_stride = c->layers > 1 ? c->layer_stride : 0;
  a.kc = static_cast<bf16_t*>(c->k);
  a.vt = static_cast<bf16_t*>(c->v);
  a.tokens = d_tokens;
  a.greedy = d_greedy;
  a.budget = d_budget;
  a.stop = stop_token;
  a.path = d_path;
  a.committed = d_committed;
  a.n = d_n;
  a.new_len = d_new_len;
  return launched(launch_tree_commit(a, c->head_dim, stream), f);
}

}  // extern "C"
