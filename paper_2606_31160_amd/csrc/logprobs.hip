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
template <class K>
__device__ __forceinline__ K nth_largest(K key, int n, int bits) {
  K t = 0;
  for (int b = bits - 1; b >= 0; --b) {
    const K c = t | ((K)1 << b);
    if (__popcll(__ballot(key >= c)) >= n) t = c;
  }
  return t;
}

// Sum and maximum over a wave, in every lane, by lane moves within the vector unit.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float x, float other) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(other), (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float last_lane(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}
__device__ __forceinline__ float wave_add(float x) {
  x += dpp<0x111, 0xf>(x, 0.f);
  x += dpp<0x112, 0xf>(x, 0.f);
  x += dpp<0x114, 0xf>(x, 0.f);
  x += dpp<0x118, 0xf>(x, 0.f);
  x += dpp<0x142, 0xa>(x, 0.f);
  x += dpp<0x143, 0xc>(x, 0.f);
  return last_lane(x);
}
// NaN if a lane holds one.
__device__ __forceinline__ float wave_max(float x) {
  x = __builtin_elementwise_maximum(x, dpp<0x111, 0xf>(x, -INFINITY));
  x = __builtin_elementwise_maximum(x, dpp<0x112, 0xf>(x, -INFINITY));
  x = __builtin_elementwise_maximum(x, dpp<0x114, 0xf>(x, -INFINITY));
  x = __builtin_elementwise_maximum(x, dpp<0x118, 0xf>(x, -INFINITY));
  x = __builtin_elementwise_maximum(x, dpp<0x142, 0xa>(x, -INFINITY));
  x = __builtin_elementwise_maximum(x, dpp<0x143, 0xc>(x, -INFINITY));
  return last_lane(x);
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

// The logits of the given tokens, on their way while the row is summed: thread g
// has token g (further ones are loaded when they are written).
template <int DT>
__device__ __forceinline__ float given_logit(const LogprobArgs& a, int row, int g) {
  const int t = a.given[(size_t)row * a.ng + g];
  return t >= 0 && t < a.V ? load_one<DT>(a.x, (int64_t)row * a.stride + t) : NAN;
}
template <int DT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int row, const Scores& z, float first) {
  for (int g = threadIdx.x; g < a.ng; g += kThreads)
    a.lp[(size_t)row * a.ng + g] = ((g < kThreads ? first : given_logit<DT>(a, row, g)) - z.M) - z.Z;
  if (a.entropy && threadIdx.x == 0) a.entropy[row] = z.entropy;
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int row, int r, uint64_t key, const Scores& z) {
  a.top_i[(size_t)row * a.top + r] = (int32_t)~(uint32_t)key;
  a.top_lp[(size_t)row * a.top + r] = (value_of((uint32_t)(key >> 32)) - z.M) - z.Z;
}

// Keys that a chunk's list has room for: (n - 1) E + 1 may pass a wave's threshold.
__host__ __device__ constexpr int list_keys(int top, int E) {
  return top == 0 ? 1 : kThreads / 64 * ((top - 1) * E + 1) > kThreads ? kThreads / 64 * ((top - 1) * E + 1) : kThreads;
}

// One chunk of 256 E logits of a row: grid (chunks, rows).  Its statistics and its
// `top` largest keys (order of the logit, then the complement of its index, so
// that equal logits go to the lowest index) for k_logprobs_join, or with one chunk
// a row the results themselves.
//   Candidates: n of a wave's 64 lane maxima are at least as large as the n-th
// largest of them, so what is smaller is none of the n largest.  That takes one
// comparison a logit; only the few that pass are put in order.  Where too many pass
// (equal or masked logits) or too few (NaN), the same is done with whole keys, which
// all differ.
//   Bound by its vector instructions (about eight a logit, one of them an exponential,
// and a chunk's fixed part: maxima compared, sums joined, candidates): 144 rows of
// 152064 bf16 logits, 44 MB that take 6.3 us to read, take 17.9 us with their join.
//   Logits stay in registers as they lie in memory.  What only the few lanes with the
// maximum or with candidates do is done for one such lane's logits by as many lanes,
// read again: it takes few registers, so that 32 a thread leave 8 waves a SIMD.
template <int DT, int E>
__global__ __launch_bounds__(kThreads) void k_logprobs(LogprobArgs a) {
  constexpr int NP = E / kPiece, NW = kThreads / 64;
  constexpr int kLocalBits = 13;                    // 256 E <= 2^13 logits
  constexpr int kLow = DT == SPEC_BF16 ? 16 : 0;    // bits of an order code that say nothing
  __shared__ float red[NW][4];
  __shared__ uint64_t thr[NW], best[NW];
  extern __shared__ uint64_t list[];                // list_keys(top, E)
  __shared__ int count;
  const int row = blockIdx.y, split = blockIdx.x, wave = threadIdx.x >> 6;
  const int base = split * kThreads * E;
  const bool one = gridDim.x == 1;
  const char* const p = static_cast<const char*>(a.x) + (int64_t)row * a.stride * (DT == SPEC_F32 ? 4 : 2);
  const bool aligned = (reinterpret_cast<uintptr_t>(p) & 15) == 0;   // whole pieces in one or two loads
  // logits as they lie in memory: half the registers of their values where they are 16 bits wide
  constexpr int kWords = DT == SPEC_F32 ? 8 : 4;    // of a piece
  uint32_t raw[NP][kWords];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int at = base + (i * kThreads + (int)threadIdx.x) * kPiece;
    if (aligned && at + kPiece <= a.V) {
#pragma unroll
      for (int h = 0; h < kWords / 4; ++h) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p + (DT == SPEC_F32 ? 4 : 2) * (int64_t)at + 16 * h);
        raw[i][4 * h] = w.x, raw[i][4 * h + 1] = w.y, raw[i][4 * h + 2] = w.z, raw[i][4 * h + 3] = w.w;
      }
    } else {
      constexpr uint32_t kNone = DT == SPEC_F32 ? 0xff800000u : DT == SPEC_BF16 ? 0xff80u : 0xfc00u;   // -infinity
#pragma unroll
      for (int k = 0; k < kPiece; ++k) {
        if (DT == SPEC_F32) {
          raw[i][k] = at + k < a.V ? reinterpret_cast<const uint32_t*>(p)[at + k] : kNone;
        } else {
          const uint32_t h = at + k < a.V ? reinterpret_cast<const uint16_t*>(p)[at + k] : kNone;
          raw[i][k >> 1] = k & 1 ? raw[i][k >> 1] | h << 16 : h;
        }
      }
    }
  }
  auto x = [&](int i) -> float {
    const int k = i % kPiece;
    if (DT == SPEC_F32) return __uint_as_float(raw[i / kPiece][k % kWords]);
    const uint32_t w = raw[i / kPiece][(k >> 1) % kWords];
    if (DT == SPEC_BF16) return __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(k & 1 ? w >> 16 : w));
  };
  // the place of thread t's i-th logit within the chunk
  auto place_of = [](int i, int t) { return ((i / kPiece) * kThreads + t) * kPiece + i % kPiece; };
  // f(place) for every logit of the given lanes of this wave, a lane each
  auto each_of = [&](uint64_t lanes, auto f) {
    const int lane = threadIdx.x & 63;
    while (lanes) {
      int from = -1;
#pragma unroll
      for (int k = 0; k < 64 / E; ++k)
        if (lanes) {
          if (lane / E == k) from = __builtin_ctzll(lanes);
          lanes &= lanes - 1;
        }
      const int l = place_of(lane % E, 64 * wave + from);
      if (from >= 0 && base + l < a.V) f(l);
    }
  };
  const float given = one && (int)threadIdx.x < a.ng ? given_logit<DT>(a, row, threadIdx.x) : 0.f;
  if (threadIdx.x == 0) count = 0;
  float lm = x(0);                                  // the lane's maximum; NaN if there is one
#pragma unroll
  for (int i = 1; i < E; ++i) lm = __builtin_elementwise_maximum(lm, x(i));
  float m = wave_max(lm);
  if ((threadIdx.x & 63) == 0) red[wave][0] = m;
  if (a.top) {
    const uint32_t w = nth_largest(order_of(lm) >> kLow, a.top, 32 - kLow);
    if ((threadIdx.x & 63) == 0) thr[wave] = w;
  }
  __syncthreads();
  m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(red[0][0], red[1][0]),
                                    __builtin_elementwise_maximum(red[2][0], red[3][0]));
  const bool nan = m != m;                          // workgroup-uniform
  const float mm = m == -INFINITY ? 0.f : m;
  float s = 0.f, n = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x(i) - mm, e = __builtin_amdgcn_exp2f(d * kLog2e);
    s += e;
    t = __builtin_fmaf(e, d, t);
  }
  if (t != t) {                                     // 0 times -infinity, of logits that are it
#pragma unroll
    for (int i = 0; i < NP * kWords; ++i) asm volatile("" : "+v"(raw[i / kWords][i % kWords]));   // (formed again, not kept)
    t = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = x(i) - mm, e = __builtin_amdgcn_exp2f(d * kLog2e);
      t = __builtin_fmaf(e, fmaxf(d, -200.f), t);   // (e is zero there, no matter how far below)
    }
  }
  // S without the maximum itself, and how often it occurs: the few lanes that hold it, again
  const bool has_max = lm == m;
  if (has_max) s = 0.f;
  each_of(__ballot(has_max), [&](int l) {
    const float v = load_one<DT>(p, base + l);
    n += v == m ? 1.f : 0.f;
    s += v == m ? 0.f : __builtin_amdgcn_exp2f((v - mm) * kLog2e);
  });
  s = wave_add(s);
  n = wave_add(n);
  t = wave_add(t);
  if ((threadIdx.x & 63) == 0) red[wave][1] = s, red[wave][2] = n, red[wave][3] = t;

  // the key of a place within the chunk, from memory; 0: none
  auto key_of = [&](int l) -> uint64_t {
    return base + l < a.V ? ((uint64_t)(order_of(load_one<DT>(p, base + l)) >> kLow) << kLocalBits) | (uint32_t)((1 << kLocalBits) - 1 - l) : 0ull;
  };
  auto listed = [&](float v, int l) { return ((uint64_t)order_of(v) << 32) | (uint32_t)~(base + l); };
  bool plain = false;                               // candidates by value; uniform
  if (a.top) {
    uint32_t w = (uint32_t)thr[0];
#pragma unroll
    for (int k = 1; k < NW; ++k) w = max(w, (uint32_t)thr[k]);
    // (-0 and 0 are equal in floating point; below the lowest number all pass)
    const float least = w > 0 ? value_of(w << kLow | (kLow && !(w >> 15) ? 0xffffu : 0u)) : -INFINITY;
    plain = !nan && least > -INFINITY;
    if (plain)
      each_of(__ballot(lm >= least), [&](int l) {
        const float v = load_one<DT>(p, base + l);
        if (v >= least) {
          const int at = atomicAdd(&count, 1);
          if (at < kThreads) list[at] = listed(v, l);
        }
      });
  }
  __syncthreads();
  s = red[0][1] + red[1][1] + red[2][1] + red[3][1];
  n = red[0][2] + red[1][2] + red[2][2] + red[3][2];
  t = red[0][3] + red[1][3] + red[2][3] + red[3][3];
  const size_t at = (size_t)row * a.splits + split;
  Scores z{};
  if (one) {
    z = scores(m, s, n, t);
    write_row<DT>(a, row, z, given);
  } else if (threadIdx.x == 0) {
    a.stats[at] = make_float4(m, s, n, t);
  }
  if (!a.top) return;
  int c = count;
  const int have = min(a.V - base, kThreads * E);   // logits of the chunk
  if (!plain || c > kThreads || c < min(a.top, have)) {
    uint64_t big = 0;
#pragma unroll 1
    for (int i = 0; i < E; ++i) big = max(big, key_of(place_of(i, threadIdx.x)));
    const uint64_t w = nth_largest(big, a.top, 32 - kLow + kLocalBits);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) thr[wave] = w;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    uint64_t least = 1;                             // (0 is no logit)
#pragma unroll
    for (int k = 0; k < NW; ++k) least = thr[k] > least ? thr[k] : least;
#pragma unroll 1
    for (int i = 0; i < E; ++i) {
      const int l = place_of(i, threadIdx.x);
      if (key_of(l) >= least) list[atomicAdd(&count, 1)] = listed(load_one<DT>(p, base + l), l);
    }
    __syncthreads();
    c = count;
  }
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
  constexpr int kLow = DT == SPEC_BF16 ? 16 : 0;
  __shared__ uint64_t list[kMaxSplits * SPEC_MAX_TOP], few[kThreads], best[kThreads / 64];
  __shared__ int count;
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const float4* st = a.stats + (size_t)row * a.splits;
  const int c = a.splits * a.top;
  const float given = (int)threadIdx.x < a.ng ? given_logit<DT>(a, row, threadIdx.x) : 0.f;
  if (threadIdx.x == 0) count = 0;
  // every wave sums the statistics for itself: at most 128 chunks
  float4 ch[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) ch[i] = lane + 64 * i < a.splits ? st[lane + 64 * i] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  for (int i = threadIdx.x; i < c; i += kThreads) list[i] = a.keys[(size_t)row * c + i];
  const float M = wave_max(__builtin_elementwise_maximum(ch[0].x, ch[1].x));
  float S = 0.f, N = 0.f, T = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ch[i].x > -INFINITY) {
      const float d = ch[i].x - M, e = d == 0.f ? 1.f : expf(d), k = ch[i].y + (d == 0.f ? 0.f : ch[i].z);
      S += e * k;
      N += d == 0.f ? ch[i].z : 0.f;
      T += e * (ch[i].w + (d == 0.f ? 0.f : fmaxf(d, -200.f) * k));
    }
  S = wave_add(S);
  N = wave_add(N);
  T = wave_add(T);
  const Scores z = scores(M, S, N, T);
  write_row<DT>(a, row, z, given);
  if (!a.top) return;
  __syncthreads();
  // as in a chunk, by the order alone, with all keys spread over every wave's lanes
  uint32_t big = 0;
  for (int i = lane; i < c; i += 64) big = max(big, (uint32_t)(list[i] >> (32 + kLow)));
  const uint32_t least = max(nth_largest(big, a.top, 32 - kLow), 1u);
  for (int i = threadIdx.x; i < c; i += kThreads)
    if ((uint32_t)(list[i] >> (32 + kLow)) >= least) {
      const int k = atomicAdd(&count, 1);
      if (k < kThreads) few[k] = list[i];
    }
  __syncthreads();
  const bool fits = count <= kThreads && count >= a.top;
  rank_keys(fits ? few : list, fits ? count : c, a.top, best, [&](int r, uint64_t k) { write_top(a, row, r, k, z); });
}

// Logits of a thread: 32, half the fixed parts of 16, where that leaves four chunks a
// CU (or a row has more logits than a join holds chunks of 16), else 16 where that
// leaves one a CU, else 8.  Measured for bf16 rows of 152064, five alternatives, at
// 16 and 32: 9 rows (0.7 chunks of 32 a CU) 8.7, 9.2 us, 36 rows (2.7) 10.9, 10.8, 72
// rows (5.3) 14.1, 13.1, 144 rows 20.3, 17.9; at 8, of an earlier form, 9 rows took 14.0
// where 16 took 12.9.
int per_thread(int rows, int V, int ncu) {
  auto chunks = [&](int e) { return (int64_t)rows * ((V + kThreads * e - 1) / (kThreads * e)); };
  if (chunks(32) >= 4 * ncu || V > kMaxSplits * kThreads * 16) return 32;
  return chunks(16) >= ncu || V > kMaxSplits * kThreads * 8 ? 16 : kPiece;
}

template <int DT, int E>
void launch_chunks(const LogprobArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_logprobs<DT, E>), dim3(a.splits, a.rows), dim3(kThreads), list_keys(a.top, E) * sizeof(uint64_t), s, a);
}

template <int DT>
hipError_t launch(const LogprobArgs& a, hipStream_t s) {
  const int e = (a.V + a.splits * kThreads - 1) / (a.splits * kThreads);
  if (e <= 8)
    launch_chunks<DT, 8>(a, s);
  else if (e <= 16)
    launch_chunks<DT, 16>(a, s);
  else
    launch_chunks<DT, 32>(a, s);
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
