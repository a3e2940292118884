// Log probabilities, entropy and top alternatives of rows of logits (logprobs.hip;
// entry point in operators.cpp).
#pragma once

#include "ctx.h"

namespace specdec {

struct LogprobArgs {
  const void* x;           // row r at x + r * stride (elements)
  int64_t stride;
  int rows, V;
  const int32_t* given;    // [rows][ng]
  int ng, top;
  float* lp;               // [rows][ng]
  float* entropy;          // [rows] or null
  int32_t* top_i;          // [rows][top]
  float* top_lp;           // [rows][top]
  float4* stats;           // [rows][splits] (maximum, sum below it, times it occurs, sum of e d)
  uint64_t* keys;          // [rows][splits][top]
  int splits;
};

constexpr int kLogprobMaxVocab = 1 << 20;

int logprob_splits(int rows, int V, int ncu);
size_t logprob_stats_bytes(int rows, int splits);
size_t logprob_key_bytes(int rows, int splits, int top);
hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t s);

}  // namespace specdec
