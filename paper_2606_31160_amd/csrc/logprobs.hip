// Scores of rows of logits: log probabilities of given tokens, entropy, and the
// most probable tokens.  With M = max x, N the times M occurs and
//   S = sum over x < M of e^(x - M),  T = sum e^(x - M) (x - M),
//   ln sum e^(x - M) = ln(N + S) = log1p(N - 1 + S) =: Z,
//   log p(i) = (x_i - M) - Z,   entropy = Z - T / (N + S).
// S leaves the maximum out so that a sure token's log probability, -S to first
// order, keeps its digits.  A row is read once.
#include <algorithm>

#include "device.h"
#include "logprobs.h"

namespace specdec {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxSplits = 128;
constexpr int kPiece = 8;                           // consecutive logits of a thread

// An order-preserving code of a logit: larger logits have larger codes; -0 equals
// 0, NaN counts as -infinity; every code is above 0, which stands for no logit.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = x != x ? 0xff800000u : __float_as_uint(x + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

template <int DT>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if (DT == SPEC_F32) return static_cast<const float*>(p)[i];
  const uint16_t h = static_cast<const uint16_t*>(p)[i];
  return DT == SPEC_BF16 ? bf2f(h) : (float)__builtin_bit_cast(_Float16, h);
}

// The largest T with at least n lanes' keys >= T, of keys below 2^bits: the n-th
// largest key if all differ.
__device__ __forceinline__ uint64_t nth_largest(uint64_t key, int n, int bits) {
  uint64_t t = 0;
  for (int b = bits - 1; b >= 0; --b) {
    const uint64_t c = t | (1ull << b);
    if (__popcll(__ballot(key >= c)) >= n) t = c;
  }
  return t;
}

// Sorts the n largest of c distinct keys in LDS: the key of rank r goes to put(r, key).
template <class Put>
__device__ __forceinline__ void rank_keys(uint64_t* list, int c, int n, uint64_t* best, Put put) {
  if (c <= kThreads) {
    const int t = threadIdx.x;
    if (t < c) {
      const uint64_t mine = list[t];
      int r = 0;
#pragma unroll 4
      for (int j = 0; j < c; ++j) r += list[j] > mine;
      if (r < n) put(r, mine);
    }
    return;
  }
  // many keys: the largest below the last one, n times
  uint64_t below = ~0ull;
  for (int r = 0; r < n; ++r) {
    uint64_t m = 0;
    for (int j = threadIdx.x; j < c; j += kThreads) {
      const uint64_t k = list[j];
      if (k < below && k > m) m = k;
    }
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t x = __shfl_xor(m, o);
      m = x > m ? x : m;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) best[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w) m = best[w] > m ? best[w] : m;
    if (threadIdx.x == 0) put(r, m);
    below = m;
  }
}

struct Scores {
  float M, Z, entropy;
};
__device__ __forceinline__ Scores scores(float M, float S, float N, float T) {
  Scores r;
  r.M = M;
  r.Z = fabsf(M) < INFINITY ? log1pf((N - 1.f) + S) : NAN;   // only infinities, or one above all: no distribution
  r.entropy = r.Z - T / (N + S);
  return r;
}

template <int DT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int row, const Scores& z) {
  for (int g = threadIdx.x; g < a.ng; g += kThreads) {
    const int t = a.given[(size_t)row * a.ng + g];
    a.lp[(size_t)row * a.ng + g] = t >= 0 && t < a.V ? (load_one<DT>(a.x, (int64_t)row * a.stride + t) - z.M) - z.Z : NAN;
  }
  if (a.entropy && threadIdx.x == 0) a.entropy[row] = z.entropy;
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int row, int r, uint64_t key, const Scores& z) {
  a.top_i[(size_t)row * a.top + r] = (int32_t)~(uint32_t)key;
  a.top_lp[(size_t)row * a.top + r] = (value_of((uint32_t)(key >> 32)) - z.M) - z.Z;
}

// One chunk of 256 E logits of a row: grid (chunks, rows).  Its statistics and its
// `top` largest keys (order of the logit, then the complement of its index, so
// that equal logits go to the lowest index) for k_logprobs_join, or with one chunk
// a row the results themselves.
//   Candidates: n of a wave's 64 lane maxima are at least as large as the n-th
// largest of them, so what is smaller is none of the n largest.
template <int DT, int E>
__global__ __launch_bounds__(kThreads) void k_logprobs(LogprobArgs a) {
  constexpr int NP = E / kPiece, NW = kThreads / 64;
  constexpr int kLocalBits = 13;                    // 256 E <= 2^13 logits
  constexpr int kLow = DT == SPEC_BF16 ? 16 : 0;    // bits of an order code that say nothing
  __shared__ float red[NW][4];
  __shared__ uint64_t thr[NW], best[NW];
  __shared__ uint64_t list[NW * ((SPEC_MAX_TOP - 1) * E + 1)];
  __shared__ int count;
  const int row = blockIdx.y, split = blockIdx.x, wave = threadIdx.x >> 6;
  const int base = split * kThreads * E;
  const char* const p = static_cast<const char*>(a.x) + (int64_t)row * a.stride * (DT == SPEC_F32 ? 4 : 2);
  const bool aligned = (reinterpret_cast<uintptr_t>(p) & 15) == 0;   // whole pieces in one or two loads
  float x[E];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int at = base + (i * kThreads + (int)threadIdx.x) * kPiece;
    if (aligned && at + kPiece <= a.V) {
      if (DT == SPEC_F32) {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(p + 4 * (int64_t)at), hi = *reinterpret_cast<const f32x4*>(p + 4 * (int64_t)at + 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[8 * i + k] = lo[k], x[8 * i + 4 + k] = hi[k];
      } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p + 2 * (int64_t)at);
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint16_t h = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
          x[8 * i + k] = DT == SPEC_BF16 ? bf2f(h) : (float)__builtin_bit_cast(_Float16, h);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < kPiece; ++k) x[8 * i + k] = at + k < a.V ? load_one<DT>(p, at + k) : -INFINITY;
    }
  }
  if (threadIdx.x == 0) count = 0;
  float m = x[0];
#pragma unroll
  for (int i = 1; i < E; ++i) m = fmaxf(m, x[i]);
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) red[wave][0] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[1][0]), fmaxf(red[2][0], red[3][0]));
  const float mm = m == -INFINITY ? 0.f : m;
  float s = 0.f, n = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x[i] - mm;
    const float e = x[i] == mm ? 0.f : __builtin_amdgcn_exp2f(d * kLog2e);
    n += x[i] == mm ? 1.f : 0.f;
    s += e;
    t = __builtin_fmaf(e, fmaxf(d, -200.f), t);     // (where e is zero, no matter how far below)
  }
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o);
    n += __shfl_xor(n, o);
    t += __shfl_xor(t, o);
  }
  if ((threadIdx.x & 63) == 0) red[wave][1] = s, red[wave][2] = n, red[wave][3] = t;

  // keys of this thread's logits within the chunk; 0: none
  auto key_of = [&](int i) -> uint64_t {
    const int local = ((i / kPiece) * kThreads + (int)threadIdx.x) * kPiece + i % kPiece;
    return base + local < a.V ? ((uint64_t)(order_of(x[i]) >> kLow) << kLocalBits) | (uint32_t)((1 << kLocalBits) - 1 - local) : 0ull;
  };
  if (a.top) {
    uint64_t big = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint64_t k = key_of(i);
      big = k > big ? k : big;
    }
    const uint64_t w = nth_largest(big, a.top, 32 - kLow + kLocalBits);
    if ((threadIdx.x & 63) == 0) thr[wave] = w;
  }
  __syncthreads();
  s = red[0][1] + red[1][1] + red[2][1] + red[3][1];
  n = red[0][2] + red[1][2] + red[2][2] + red[3][2];
  t = red[0][3] + red[1][3] + red[2][3] + red[3][3];
  const bool one = gridDim.x == 1;
  const size_t at = (size_t)row * a.splits + split;
  Scores z{};
  if (one) {
    z = scores(m, s, n, t);
    write_row<DT>(a, row, z);
  } else if (threadIdx.x == 0) {
    a.stats[at] = make_float4(m, s, n, t);
  }
  if (!a.top) return;
  uint64_t least = 1;                               // (0 is no logit)
#pragma unroll
  for (int w = 0; w < NW; ++w) least = thr[w] > least ? thr[w] : least;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint64_t k = key_of(i);
    if (k >= least) {
      const uint32_t local = (1u << kLocalBits) - 1 - (uint32_t)(k & ((1u << kLocalBits) - 1));
      list[atomicAdd(&count, 1)] = ((uint64_t)order_of(x[i]) << 32) | (uint32_t)~(base + local);
    }
  }
  __syncthreads();
  const int c = count;
  // a chunk at the end of the row may hold fewer logits than `top`
  if (!one && (int)threadIdx.x < a.top && (int)threadIdx.x >= c) a.keys[at * a.top + threadIdx.x] = 0;
  rank_keys(list, c, min(a.top, c), best, [&](int r, uint64_t k) {
    if (one)
      write_top(a, row, r, k, z);
    else
      a.keys[at * a.top + r] = k;
  });
}

// Joins the chunks of a row: grid (rows).
template <int DT>
__global__ __launch_bounds__(kThreads) void k_logprobs_join(LogprobArgs a) {
  __shared__ uint64_t list[kMaxSplits * SPEC_MAX_TOP], few[kThreads], best[kThreads / 64];
  __shared__ int count;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const float4* st = a.stats + (size_t)row * a.splits;
  if (threadIdx.x == 0) count = 0;
  // every wave sums the statistics for itself
  float M = -INFINITY;
  for (int i = lane; i < a.splits; i += 64) M = fmaxf(M, st[i].x);
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  float S = 0.f, N = 0.f, T = 0.f;
  for (int i = lane; i < a.splits; i += 64) {
    const float4 c = st[i];
    if (c.x == M) {
      S += c.y, N += c.z, T += c.w;
    } else if (c.x > -INFINITY) {
      const float d = c.x - M, e = expf(d), k = c.y + c.z;
      S += e * k;
      T += e * (c.w + fmaxf(d, -200.f) * k);
    } else {
      S += c.y;                                     // zero, or NaN
    }
  }
  for (int o = 32; o > 0; o >>= 1) {
    S += __shfl_xor(S, o);
    N += __shfl_xor(N, o);
    T += __shfl_xor(T, o);
  }
  const Scores z = scores(M, S, N, T);
  write_row<DT>(a, row, z);
  if (!a.top) return;
  const int c = a.splits * a.top;
  for (int i = threadIdx.x; i < c; i += kThreads) list[i] = a.keys[(size_t)row * c + i];
  __syncthreads();
  // as in a chunk, with all keys spread over every wave's lanes
  uint64_t big = 0;
  for (int i = lane; i < c; i += 64) big = list[i] > big ? list[i] : big;
  uint64_t least = nth_largest(big, a.top, 64);
  if (least == 0) least = 1;
  for (int i = threadIdx.x; i < c; i += kThreads)
    if (list[i] >= least) {
      const int k = atomicAdd(&count, 1);
      if (k < kThreads) few[k] = list[i];
    }
  __syncthreads();
  const bool fits = count <= kThreads;
  rank_keys(fits ? few : list, fits ? count : c, a.top, best, [&](int r, uint64_t k) { write_top(a, row, r, k, z); });
}

// Logits of a thread: as many as leave two chunks per CU, 8 to 32.
int per_thread(int rows, int V, int ncu) {
  for (int e = 32; e > kPiece; e /= 2)
    if ((int64_t)rows * ((V + kThreads * e - 1) / (kThreads * e)) >= 2 * ncu || V > kMaxSplits * kThreads * (e / 2)) return e;
  return kPiece;
}

template <int DT>
hipError_t launch(const LogprobArgs& a, hipStream_t s) {
  const dim3 grid(a.splits, a.rows);
  const int e = (a.V + a.splits * kThreads - 1) / (a.splits * kThreads);
  if (e <= 8)
    hipLaunchKernelGGL((k_logprobs<DT, 8>), grid, dim3(kThreads), 0, s, a);
  else if (e <= 16)
    hipLaunchKernelGGL((k_logprobs<DT, 16>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_logprobs<DT, 32>), grid, dim3(kThreads), 0, s, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || a.splits == 1) return err;
  hipLaunchKernelGGL(k_logprobs_join<DT>, dim3(a.rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int logprob_splits(int rows, int V, int ncu) {
  const int chunk = kThreads * per_thread(rows, V, ncu);
  return (V + chunk - 1) / chunk;
}
size_t logprob_stats_bytes(int rows, int splits) { return (size_t)rows * splits * sizeof(float4); }
size_t logprob_key_bytes(int rows, int splits, int top) { return (size_t)rows * splits * top * sizeof(uint64_t); }

hipError_t launch_logprobs(const LogprobArgs& a, int dtype, hipStream_t s) {
  return dtype == SPEC_BF16 ? launch<SPEC_BF16>(a, s) : dtype == SPEC_F16 ? launch<SPEC_F16>(a, s) : launch<SPEC_F32>(a, s);
}

}  // namespace specdec
