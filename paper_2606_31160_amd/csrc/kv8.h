// Pages of a KV cache held in 8 bits, and attention over a cache whose leading
// pages are such pages (kv8.hip; entry points in operators.cpp, contexts opened
// with SPEC_FLAG_KV8 in runtime.cpp).
#pragma once

#include "ctx.h"

namespace specdec {

// One prompt's keys and values -> pages in 8 bits.
struct Kv8PackArgs {
  const bf16_t *k, *v;     // rows of [nkv][D], `stride` elements apart
  int64_t stride;
  int rows, nkv, pages8;   // rows given; pages of the pool
  const int32_t* to;       // pool page of every 64 rows
  uint8_t *k8, *v8;        // [pages8][nkv][kAttnChunk][D], [pages8][nkv][D][kAttnChunk]
  float *ks, *vs;          // [pages8][nkv]
  int32_t* err;            // or null
  // rotation of the keys (null cs: they are rotated already)
  const float2* cs;        // [cap][D/2]
  const int32_t* pos3;     // [3][cap]
  const int8_t* axis;      // [D/2]
  int cap;
};
hipError_t launch_kv8_pack(const Kv8PackArgs& a, int D, hipStream_t s);

struct Kv8AttnArgs {
  const SeqState* st;      // a context's pass, or null: vis
  const int32_t* vis;      // [B][R] slots that each row sees; negative: no such row
  const int32_t* packed;   // [B] leading pages in 8 bits
  const int32_t* table;    // [B][stride] pool page of each page
  int stride;
  const uint8_t *k8, *v8;
  const float *ks, *vs;
  const bf16_t *k16, *v16; // [pages16][nkv][kAttnChunk][D], [pages16][nkv][D][kAttnChunk]
  int pages8, pages16;
  const bf16_t* q;         // row b*R + j at q + (b*R + j) * q_stride, [nq][D]
  int64_t q_stride;
  bf16_t* out;             // as q
  int64_t out_stride;
  int opk;                 // 0, or the pass's row blocks: out is written in operand order (device.h)
  float* lse;              // [B*R][nq] or null
  int32_t* err;            // or null
  float* part;             // [groups][row blocks][D/16][64] unnormalised partial outputs
  float2* ml;              // [groups][row blocks * 16] (maximum in log2 units, sum)
  int4* seq;               // [B] first group, groups of a kv head, pages of a group (sequences with pages)
  uint64_t* odd;           // [groups][row blocks] pages with values that the combine adds
  int B, R, nq, nkv, G;
  int ppw;                 // pages of a group; 0: as many as leave about `target` groups
  int target;
  bool many;               // kv8_many(): how the combine sums
  float scale_log2;
};

constexpr int kKv8MinPages = 4, kKv8MaxPages = 64;   // pages of a group

// Groups of a call at most (the grid), the partials' bytes, the groups a call without a fixed `ppw` aims at.
int64_t kv8_max_groups(int B, int nkv, int stride, int ppw, int target);
size_t kv8_part_bytes(int64_t groups, int rows, int D);
size_t kv8_ml_bytes(int64_t groups, int rows);     // of ml, odd behind it and seq behind that
void kv8_set_parts(Kv8AttnArgs& a, void* part, void* ml, int64_t groups);
int kv8_target_groups(int rows, int ncu);   // (what runs at once)
bool kv8_many(int64_t groups, int B, int nkv);
hipError_t launch_kv8_attn(const Kv8AttnArgs& a, int D, int64_t groups, hipStream_t s, hipEvent_t e0 = nullptr,
                           hipEvent_t e1 = nullptr);
hipError_t launch_kv8_combine(const Kv8AttnArgs& a, int D, hipStream_t s, hipEvent_t e0 = nullptr, hipEvent_t e1 = nullptr);

}  // namespace specdec
