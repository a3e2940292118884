// Entry points of the operators that need no context (include/spec.h): pages of
// a cache held in 8 bits, attention over them, scores of logits.
#include <hip/hip_runtime.h>

#include <cstdio>

#include "ctx.h"
#include "kv8.h"
#include "logprobs.h"

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

}  // extern "C"
