// A KV cache whose leading pages are held in 8 bits: packing a prompt into such
// pages, and split attention over them.
//
// A page holds kAttnChunk = 64 slots of every kv head of one layer, keys
// [nkv][64][D] and values transposed, [nkv][D][64], as the bf16 pages do, in e4m3
// (no infinity; largest 448) with one scale per page, kv head and operand:
//   s = the smallest power of two with max |x| <= 448 s (at least 2^-126; 1 for a page of zeros)
//   code = e4m3(x / s), to nearest even
// A power of two costs a floating format nothing but range, and what a code stands
// for, s e4m3, is a bf16 number: reading a page in bf16 rounds nothing.
#include <hip/hip_ext.h>

#include <algorithm>
#include <cfloat>

#include "device.h"
#include "kv8.h"

namespace specdec {

namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// e with 2^e the smallest power of two such that big <= 448 2^e (0 for big = 0); big = f
// 2^x with f in [1/2, 1), and 448 = 7/8 2^9.
__device__ __forceinline__ int scale_exponent(float big) {
  int x;
  const float f = frexpf(big, &x);
  return big > 0.f ? max(f <= 0.875f ? x - 9 : x - 8, -126) : 0;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }   // |e| <= 126

// ---------------------------------------------------------------------------
// Packing: one workgroup of 256 threads per (page, kv head, keys / values).  Keys
// may be rotated on the way (a context's prompt), rounded to bf16 as the bf16
// cache would hold them.  Infinities become NaN and count for no scale.  Slots
// past the rows are zero.  Bound by memory: 4096 tokens of 8 heads of 128, 17 MB read
// and 8 MB written, 6.4 us a call in graphs (3.9 TB/s; a copy of 4 GiB reaches 4.7).
// With rotation, in a trace, 10.4 us where 7.6 without: a table's row for each pair.
// ---------------------------------------------------------------------------
template <int D, bool ROT>
__global__ __launch_bounds__(256) void k_kv8_pack(Kv8PackArgs a) {
  constexpr int KC = D / 8, U = KC / 4;             // 16-byte chunks of a row; chunks of a thread
  constexpr int kVs = kAttnChunk + 4;               // LDS row of a value dimension
  __shared__ float red[4];
  __shared__ __align__(16) uint8_t vs[D * kVs];
  const int h = blockIdx.y, s0 = blockIdx.x * kAttnChunk;
  const bool val = blockIdx.z != 0;
  const int page = a.to[blockIdx.x];
  if (page < 0 || page >= a.pages8) {               // workgroup-uniform
    if (a.err && threadIdx.x == 0) *a.err = SPEC_E_INVAL;
    return;
  }
  const bf16_t* src = val ? a.v : a.k;
  float x[U][8];
  float big = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + 256 * u, off = i / KC, c = i % KC, s = s0 + off;
    u32x4 r = ld16(src + (int64_t)min(s, a.rows - 1) * a.stride + (int64_t)h * D + 8 * c);
    if (s >= a.rows) r = u32x4{0, 0, 0, 0};
    uint32_t w[4] = {r.x, r.y, r.z, r.w};
    if (ROT && !val && s < a.rows) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int d = 4 * c + k;
        const float2 t = a.cs[(size_t)a.pos3[a.axis[d] * a.cap + s] * (D / 2) + d];
        const float e = __uint_as_float(w[k] << 16), o = __uint_as_float(w[k] & 0xffff0000u);
        w[k] = pack2(e * t.x - o * t.y, e * t.y + o * t.x);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[u][e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
      const float m = fabsf(x[u][e]);
      big = fmaxf(big, m < INFINITY ? m : 0.f);     // neither infinities nor NaN
    }
  }
  for (int o = 32; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor(big, o));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = big;
  __syncthreads();
  big = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const int e = scale_exponent(big);                // in [-126, 120]
  const float inv = power_of_two(-e);
  const size_t pg = (size_t)page * a.nkv + h;
  if (threadIdx.x == 0) (val ? a.vs : a.ks)[pg] = power_of_two(e);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + 256 * u, off = i / KC, c = i % KC;
    uint32_t code[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float v = x[u][4 * q + k];
        y[k] = v * inv;                             // (infinities become NaN: e4m3 has none)
      }
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      code[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
    if (!val) {
      *reinterpret_cast<u32x2*>(a.k8 + (pg * kAttnChunk + off) * D + 8 * c) = u32x2{code[0], code[1]};
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) vs[(8 * c + k) * kVs + off] = (uint8_t)(code[k >> 2] >> (8 * (k & 3)));
    }
  }
  if (!val) return;
  __syncthreads();
  for (int i = threadIdx.x; i < D * 4; i += 256) {
    const int d = i >> 2, c = i & 3;
    const uint32_t* r = reinterpret_cast<const uint32_t*>(vs + d * kVs + 16 * c);
    *reinterpret_cast<u32x4*>(a.v8 + (pg * D + d) * kAttnChunk + 16 * c) = u32x4{r[0], r[1], r[2], r[3]};
  }
}

// ---------------------------------------------------------------------------
// Attention.  Rows r = j G + g of a kv head (pass row j, query head g of the
// group) stand against the head's pages in groups of ppw pages; a group's
// workgroup leaves unnormalised sums, which k_kv8_combine joins.  With running
// maximum m, sum l and output O of the softmax in log2 units,
//   m' = max(m, max s),  l' = 2^(m - m') l + sum 2^(s - m'),  O' = 2^(m - m') O + sum 2^(s - m') v.
// ---------------------------------------------------------------------------

constexpr int kKeyWaves = 4;    // waves that share a group's pages: wave w takes pages w, w + 4, ..

// Sums and maxima over a wave, and its running sum, by lane moves within the
// vector unit (row shifts, then the last lane of each row of 16 to the next rows).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_max(int x) {   // x >= 0
  return max(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
}
__device__ __forceinline__ int wave_max(int x) {
  x = dpp_max<0x111, 0xf>(x);
  x = dpp_max<0x112, 0xf>(x);
  x = dpp_max<0x114, 0xf>(x);
  x = dpp_max<0x118, 0xf>(x);
  x = dpp_max<0x142, 0xa>(x);
  return __builtin_amdgcn_readlane(dpp_max<0x143, 0xc>(x), 63);
}
// Over the 16 lanes of a row, in all of them.
__device__ __forceinline__ int row_max(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
  return max(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));
}

// The groups of a call.  They are numbered sequence by sequence, then by pages,
// then by kv head.  Every wave of a workgroup counts them for itself, lane l
// sequences l, l + 64 and l + 128; vis: LDS of SPEC_MAX_ROWS words of its own.
struct Groups {
  int ppw;
  int pages[3], first[3];   // of sequence lane + 64 i: pages, number of its first group
  int total;
  int base, count, causal;  // of sequence lane (a context's)
};

__device__ __forceinline__ Groups count_groups(const Kv8AttnArgs& a, int* vis) {
  const int lane = threadIdx.x & 63;
  Groups g;
  int end[3] = {0, 0, 0};
  if (a.st) {
    const SeqState& s = a.st[min(lane, a.B - 1)];
    g.base = s.base, g.count = s.count, g.causal = s.causal;
    end[0] = lane < a.B && g.count > 0 ? g.base + g.count : 0;
  } else {
    const int n = a.B * a.R;
    int v[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = lane + 64 * i < n ? a.vis[lane + 64 * i] : 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (lane + 64 * i < n) vis[lane + 64 * i] = v[i];
    if (a.R == 1) {
#pragma unroll
      for (int i = 0; i < 3; ++i) end[i] = max(v[i], 0);
    } else if (a.B == 1) {
      const int m = wave_max(max(max(v[0], v[1]), max(v[2], 0)));
      end[0] = lane == 0 ? m : 0;
    } else {                                        // at most 80 sequences
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (lane + 64 * i < a.B)
          for (int j = 0; j < a.R; ++j) end[i] = max(end[i], vis[(lane + 64 * i) * a.R + j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    g.pages[i] = min((int)(((unsigned)end[i] + kAttnChunk - 1) / kAttnChunk), a.stride);
  auto sum = [&](int ppw) {                         // groups of ppw pages; first[] on the way
    int before = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      g.first[i] = before;
      if (64 * i >= a.B) continue;
      const int n = a.nkv * (int)(((unsigned)g.pages[i] + ppw - 1) / ppw), x = wave_scan(n);
      g.first[i] = before + x - n;
      before += __builtin_amdgcn_readlane(x, 63);
    }
    return before;
  };
  g.ppw = a.ppw;
  if (g.ppw == 0) {
    // as few pages as leave no more groups than run at once
    g.ppw = kKv8MinPages;
    g.total = sum(g.ppw);
    if (g.total > a.target) {
      g.ppw = min(max(g.total / a.target, 1) * kKv8MinPages, kKv8MaxPages);
      while ((g.total = sum(g.ppw)) > a.target && g.ppw < kKv8MaxPages && a.B * a.nkv <= a.target) g.ppw += kKv8MinPages;
    }
  } else {
    g.total = sum(g.ppw);
  }
  g.ppw = __builtin_amdgcn_readfirstlane(g.ppw);    // (all uniform, as the compiler cannot see)
  g.total = __builtin_amdgcn_readfirstlane(g.total);
  return g;
}

// Slots that row j of sequence b sees; negative: no such row.
__device__ __forceinline__ int row_vis(const Kv8AttnArgs& a, const Groups& g, const int* vis, int b, int j) {
  if (!a.st) return vis[b * a.R + j];
  const int base = __builtin_amdgcn_readlane(g.base, b), count = __builtin_amdgcn_readlane(g.count, b);
  const int causal = __builtin_amdgcn_readlane(g.causal, b);
  return j < count ? base + (j < causal ? j + 1 : count) : -1;
}

// scale: a power of two
__device__ __forceinline__ u32x4 bf16_of_e4m3(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 r[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)};
  return __builtin_bit_cast(u32x4, r);
}
// A scale as 2^e times a rest: e is its exponent as far as the bounds reach.
__device__ __forceinline__ int exponent_of(float scale, int least, int most) {
  int x;
  frexpf(scale, &x);
  return min(max(x - 1, least), most);
}

// x0, x1 as two bf16 numbers each: h the nearest, l what is left of them (2^-16 of x at most is lost).
__device__ __forceinline__ void split2(float x0, float x1, uint32_t& h, uint32_t& l) {
  h = pack2(x0, x1);
  l = pack2(x0 - __uint_as_float(h << 16), x1 - __uint_as_float(h & 0xffff0000u));
}
// Bit 7 of every byte that is a NaN code / bits 15 and 31 for bf16 numbers that are
// not finite.
__device__ __forceinline__ uint32_t nan8(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t not_finite16(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ float lane_f(float x, int l) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l));
}

// A barrier for data in LDS that leaves loads from memory in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The softmax state of a wave's rows (lane: row lane & 15 of each block).
template <int NRB, int NDT>
struct RowState {
  float m[NRB], l[NRB];
  f32x4 o[NRB][NDT];
};

// Scores s of 16 keys per lane -> probabilities 2^(s sc - m + off), handed to put, and
// l.  m is kAbove over the row's maximum when it is set, and set again only when a row's
// scores pass it: until then O is not rescaled and lanes are not compared, and a
// probability is at most 2^off, so that O keeps within the values' range.  A row's sums depend
// on no other row.  (A maximum that passes NaN on, as the row's sums do anyway, takes one
// instruction for three.)
constexpr float kLeast = 1.4e-45f;   // factors of scores are positive and finite: -infinity times one is -infinity, zero is zero
constexpr float kAbove = 8.f, kAboveFactor = 256.f;   // 2^kAbove
template <int NRB, int NDT, class Put>
__device__ __forceinline__ void soft(RowState<NRB, NDT>& st, const float (&s)[NRB][16], const float (&sc)[NRB], float off,
                                     Put put) {
  float pm[NRB];
  bool grow = false;
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    float x = s[rb][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) x = __builtin_elementwise_maximum(x, s[rb][i]);
    pm[rb] = x * sc[rb];
    grow |= pm[rb] > st.m[rb];
  }
  if (__any(grow)) {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      pm[rb] = fmaxf(pm[rb], __shfl_xor(pm[rb], 16));
      pm[rb] = fmaxf(pm[rb], __shfl_xor(pm[rb], 32));
      if (pm[rb] > st.m[rb]) {
        const float m = pm[rb] + kAbove, alpha = st.m[rb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m[rb] - m);
        st.m[rb] = m;
        st.l[rb] *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) st.o[rb][dt] *= alpha;
      }
    }
  }
  const float back = __builtin_amdgcn_exp2f(-off);
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    const float c = off - (st.m[rb] == -INFINITY ? 0.f : st.m[rb]);   // no key seen yet: all probabilities zero
    float p[16], ls = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][i], sc[rb], c));
      ls += p[i];
    }
    put(rb, p);
    st.l[rb] = __builtin_fmaf(ls, back, st.l[rb]);
  }
}

// grid (groups, row blocks / (NRB WR)), WR x 4 waves: wave w has row blocks NRB (w %
// WR) .. and pages w / WR, + 4, .. of the group.
//
// S^T = K Q^T and O^T = V^T P^T, lane (n = lane & 15, g = lane >> 4) holding row n.  Row
// i of key tile t is key 16 (i >> 2) + 4 t + (i & 3): the 16 scores of a lane belong to
// the consecutive keys 16 g .. 16 g + 15, one 16-byte read of a value row; and a
// lane's 16 bytes of a key row serve whatever part of the head dimension, whose order
// is the same in Q's operand.
//   The next page's keys are loaded while this one's softmax runs, its values while
// the next scores are formed.  (Pages by way of LDS, for the two waves of WR = 2 at
// once, took longer: 33 us where registers took 29.5, the waves in step at its barriers.)
//   Keys are read as bf16, like Q: an e4m3 code is exact in it, also times its scale's
// power of two (what is left of a scale is part of the scores' factor).  (16x16x128 MFMA
// of e4m3 numbers, against Q in two parts of four bits each, took as long, and their
// sums drop what is some 2^-16 of the largest product: scores 1e-5 off, not 1e-7.)
//   Values are read as bf16 in the same way (with the rest of a scale in the
// probability's exponent), and each probability as the sum of two bf16 numbers, 16 bits
// of it in 32 bits' range: O is in its true unit, whatever the scales of other pages.
// (One fp16 number, in a unit common to a group's pages, keeps 11 bits, and fewer on
// pages whose scale is below the largest; with half the value products it took 34.3 us a
// call where this takes 35.1, 16 scenes of 9 rows, and 15.0 for 15.3, one scene.)
//   Bound by a wave's own chain, scores to softmax to value product, with two waves a
// SIMD (of 16 scenes of 2 to 8 thousand tokens, 80 MB: 9 rows each 31.2 us, vector
// unit 39% busy, matrix unit 21%; one row each 18.5 us, 4.3 TB/s), and where a wave has
// a page or two by the loads before the first product, each waiting for the last:
// about 5 us of 11.8 for 9 rows of one sequence of 4096.
//   Which pages share a wave depends on the group only, and a row's sums on no
// other row, so contexts that differ in K, and so in NRB and WR, sum alike.
template <int D, int NRB, int WR>
__global__ __launch_bounds__(64 * WR * kKeyWaves, 2) void k_kv8_attn(Kv8AttnArgs a) {
  constexpr int NDT = D / 16, KH = D / 64, ND4 = NDT / kKeyWaves;
  constexpr int kOp = kAttnChunk * D;               // bytes of a page's keys (or values)
  __shared__ f32x4 s_o[WR][kKeyWaves][NDT][64];
  __shared__ float s_m[kKeyWaves][WR][NRB * 16], s_l[kKeyWaves][WR][NRB * 16];
  __shared__ int s_vis[WR * kKeyWaves][SPEC_MAX_ROWS];
  __shared__ uint64_t s_odd[kKeyWaves][WR];
  __shared__ u32x4 s_q[WR][NRB][2 * KH][64];        // Q's operands: in registers they would not leave room for two pages
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int wr = wave % WR, wk = wave / WR;
  const int n16 = lane & 15, g4 = lane >> 4;
  const Groups gr = count_groups(a, s_vis[wave]);
  const int id = blockIdx.x;
  if (id >= gr.total) return;
  int b = 0, pages = 0, first = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    // the last sequence whose first group is not after this one, of those that have any
    const uint64_t m = __ballot(gr.pages[i] > 0 && gr.first[i] <= id);
    if (m) {
      const int l = 63 - __builtin_clzll(m);
      b = l + 64 * i;
      pages = __builtin_amdgcn_readlane(gr.pages[i], l);
      first = __builtin_amdgcn_readlane(gr.first[i], l);
    }
  }
  b = __builtin_amdgcn_readfirstlane(b);
  pages = __builtin_amdgcn_readfirstlane(pages);
  first = __builtin_amdgcn_readfirstlane(first);
  const int grp = __builtin_amdgcn_readfirstlane((unsigned)(id - first) / (unsigned)a.nkv), kvh = id - first - grp * a.nkv;
  const int p0 = grp * gr.ppw;                      // first page
  const int np = min(gr.ppw, pages - p0);
  const int packed = min(max(a.packed[b], 0), a.stride);
  const int n8 = a.pages8 > 0 ? min(max(packed - p0, 0), np) : 0;
  const int n16p = max(packed - p0, 0);             // the first bf16 page
  if (id == first && threadIdx.x == 0 && blockIdx.y == 0) a.seq[b] = make_int4(first, (pages + gr.ppw - 1) / gr.ppw, gr.ppw, 0);

  // lane l: the group's l-th page
  int page = -1;
  if (lane < np) page = a.table[(size_t)b * a.stride + p0 + lane];

  // rows of this wave
  const int rows = a.R * a.G, r0 = (blockIdx.y * WR + wr) * NRB * 16;
  int vis[NRB], vmin = INT32_MAX, vmax = 0;
  u32x4 q[2 * KH];                                  // of row block wk
  // (a row that is not there reads one that is)
  auto q_at = [&](int rb, int& j) {
    const int r = r0 + 16 * rb + n16;
    j = r < rows ? (unsigned)r / (unsigned)a.G : 0;
    const int g = r < rows ? r - j * a.G : 0;
    return a.q + (int64_t)(b * a.R + j) * a.q_stride + (int64_t)(kvh * a.G + g) * D + 16 * g4;
  };
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    int j;
    const bf16_t* const qp = q_at(rb, j);
    int v = r0 + 16 * rb + n16 < rows ? row_vis(a, gr, s_vis[wave], b, j) : -1;
    if (v > a.stride * kAttnChunk) {                // (no more than the table has: sums with it stay below 2^31)
      if (a.err) *a.err = SPEC_E_INVAL;
      v = a.stride * kAttnChunk;
    }
    vis[rb] = v < 0 ? INT32_MAX : v;                // rows that nobody asked for need no mask
    vmin = min(vmin, vis[rb]);
    vmax = max(vmax, v);
    if (rb == wk)
#pragma unroll
      for (int t = 0; t < 2 * KH; ++t) q[t] = ld16(qp + 64 * (t >> 1) + 8 * (t & 1));
  }
  vmin = ~__builtin_amdgcn_readfirstlane(row_max(~vmin));
  vmax = __builtin_amdgcn_readfirstlane(row_max(vmax));      // slots that no row of this wave sees: from here

  // pages that may be read, and those that this wave has to
  if (page < 0 || page >= (lane < n16p ? a.pages8 : a.pages16)) page = -1;
  if (lane < np && page < 0 && a.err) *a.err = SPEC_E_INVAL;
  const int seen = vmax <= p0 * kAttnChunk ? 0 : min(np, (vmax - p0 * kAttnChunk + kAttnChunk - 1) / kAttnChunk);
  const uint64_t todo = __ballot(lane < seen && page >= 0 && lane % kKeyWaves == wk);

  RowState<NRB, NDT> st;
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    st.m[rb] = -INFINITY;
    st.l[rb] = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) st.o[rb][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int krow = 16 * (n16 >> 2) + (n16 & 3);     // key of this lane in tile 0
  auto at_of = [&](int p) {                         // element of the page's first key or value
    return ((size_t)max(__builtin_amdgcn_readlane(page, p), 0) * a.nkv + kvh) * kOp;
  };
  auto mask = [&](float (&s)[NRB][16], int k0, int end) {
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 16 * g4 + i >= min(vis[rb], end)) s[rb][i] = -INFINITY;
  };
  // Pages with values that are not finite: these are taken as zero here, as zero
  // probability times one is not zero, and the combine gives them to the rows that see
  // their slots.  (8-bit pages that every row sees keep theirs, which are all NaN.)
  uint64_t odd_pages = 0;

  if (n8 > 0) {                                     // workgroup-uniform
    const bool own = lane < n8 && page >= 0;
    const size_t sl = (size_t)(own ? page : 0) * a.nkv + kvh;
    const float ks = a.ks[sl], vsc = a.vs[sl];
    uint64_t t8 = todo & (n8 >= 64 ? ~0ull : (1ull << n8) - 1);

    // a page on its way
    u32x4 kr[4][KH];
    u32x4 vr[NDT];
    auto load_k = [&](size_t at) {
      const uint8_t* kp = a.k8 + at + krow * D + 16 * g4;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int h = 0; h < KH; ++h) kr[t][h] = *reinterpret_cast<const u32x4*>(kp + 4 * t * D + 64 * h);
      }
    };
    auto load_v = [&](size_t at) {
      const uint8_t* vp = a.v8 + at + n16 * kAttnChunk + 16 * g4;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) vr[dt] = *reinterpret_cast<const u32x4*>(vp + 16 * dt * kAttnChunk);
    };
    int p = t8 ? __builtin_ctzll(t8) : 64;
    {
      // (without a page to do, the group's first: loads outside a branch can be awaited one by one)
      const size_t at = at_of(p < 64 ? p : 0);
      load_k(at);
      load_v(at);
    }
    if (wk < NRB)
#pragma unroll
      for (int t = 0; t < 2 * KH; ++t) s_q[wr][wk][t][lane] = q[t];
    lds_barrier();                                  // with pages on their way
    // (the scales arrive before the pages)
    const bool fine = ks > 0.f && ks < INFINITY && vsc > 0.f && vsc < INFINITY;
    if (own && !fine && a.err) *a.err = SPEC_E_INVAL;
    const uint64_t good = __ballot(own && fine);
    // lane l: the l-th page's scales, kp krest and vp 2^lv (kp, vp powers of two; every code times vp is a normal
    // bf16 number, and kp leaves some range to queries of any magnitude)
    const int ek = own && fine ? exponent_of(ks, -60, 60) : 0, ev = own && fine ? exponent_of(vsc, -116, 118) : 0;
    const float krest = own && fine ? ks * power_of_two(-ek) : 1.f, kp = power_of_two(ek);
    const float lv = own && fine ? __builtin_amdgcn_logf(vsc * power_of_two(-ev)) : 0.f, vp = power_of_two(ev);

    while (p < 64) {
      t8 &= t8 - 1;
      const int next = t8 ? __builtin_ctzll(t8) : 64;
      // (the last page loads itself again, out of the caches: under a branch the loads were moved ahead of the
      // products and took registers of their own)
      const size_t nat = at_of(next < 64 ? next : p);
      const int k0 = (p0 + p) * kAttnChunk;
      const bool sound = good >> p & 1;           // else a page without scales: not visible
      const bool full = sound && k0 + kAttnChunk <= vmin;
      float s[NRB][16];                           // scores of keys 16 g4 + i
      u32x4 qf[NRB][2 * KH];
      int ql = lane;
      asm volatile("" : "+v"(ql));                // (read again for every page)
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
        for (int h = 0; h < 2 * KH; ++h) qf[rb][h] = s_q[wr][rb][h][ql];
      const float kpp = lane_f(kp, p);
      // (products on one accumulator stand apart, or the second waits for the first)
      f32x4 acc[4][NRB];
#pragma unroll
      for (int t = 0; t < 4; t += 2)
#pragma unroll
        for (int h = 0; h < 2 * KH; ++h)
#pragma unroll
          for (int k = t; k < t + 2; ++k) {
            const u32x4 w = kr[k][h >> 1];
            const u32x4 x = h & 1 ? bf16_of_e4m3(w.z, w.w, kpp) : bf16_of_e4m3(w.x, w.y, kpp);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) acc[k][rb] = mfma16x16x32(x, qf[rb][h], h ? acc[k][rb] : f32x4{0.f, 0.f, 0.f, 0.f});
          }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rb][4 * t + i] = acc[t][rb][i];
      __builtin_amdgcn_sched_barrier(0);
      load_k(nat);
      if (!full) mask(s, k0, sound ? INT32_MAX : 0);
      float sc[NRB];
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) sc[rb] = fminf(fmaxf(a.scale_log2 * lane_f(krest, p), kLeast), FLT_MAX);
      u32x4 pb[NRB][2][2];                        // the parts of the probabilities of keys 8 e ..
      soft(st, s, sc, lane_f(lv, p), [&](int rb, float (&x)[16]) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t h, l;
            split2(x[8 * e + 2 * k], x[8 * e + 2 * k + 1], h, l);
            pb[rb][e][0][k] = h, pb[rb][e][1][k] = l;
          }
      });
      if (!full) {
        const int valid = (sound ? min(vmax - k0, kAttnChunk) : 0) - 16 * g4;   // of this lane's 16 keys
        uint32_t m[4], odd = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int c = min(max(valid - 4 * k, 0), 4);
          m[k] = (uint32_t)((1ull << (8 * c)) - 1);
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t w = vr[dt][k] & m[k], x = nan8(w);
            odd |= x;
            vr[dt][k] = w & ~((x >> 7) * 0xffu);
          }
        if (__any(odd != 0)) odd_pages |= 1ull << p;
      }
      const float vpp = lane_f(vp, p);
#pragma unroll
      for (int dt = 0; dt < NDT; dt += 2)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          u32x4 v[2];
#pragma unroll
          for (int k = 0; k < 2; ++k)
            v[k] = e ? bf16_of_e4m3(vr[dt + k].z, vr[dt + k].w, vpp) : bf16_of_e4m3(vr[dt + k].x, vr[dt + k].y, vpp);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int rb = 0; rb < NRB; ++rb) st.o[rb][dt + k] = mfma16x16x32(v[k], pb[rb][e][h], st.o[rb][dt + k]);
        }
      __builtin_amdgcn_sched_barrier(0);
      load_v(nat);
      p = next;
    }
  }

  for (uint64_t t16 = n16p >= 64 ? 0 : todo & ~((1ull << n16p) - 1); t16; t16 &= t16 - 1) {
    const int p = __builtin_ctzll(t16);
    const size_t at = at_of(p);
    const int k0 = (p0 + p) * kAttnChunk;
    const bool full = k0 + kAttnChunk <= vmin;
    float s[NRB][16];
    // Q again and all of the page's keys, then all of its values, in flight at once
    u32x4 w[16 * KH], qw[NRB][2 * KH];
    const bf16_t* kp = a.k16 + at + krow * D + 16 * g4;
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      int j;
      const bf16_t* const qp = q_at(rb, j);
#pragma unroll
      for (int t = 0; t < 2 * KH; ++t) qw[rb][t] = ld16(qp + 64 * (t >> 1) + 8 * (t & 1));
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < 2 * KH; ++h) w[2 * KH * t + h] = ld16(kp + 4 * t * D + 64 * (h >> 1) + 8 * (h & 1));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 acc[NRB];
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) acc[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < 2 * KH; ++h)
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) acc[rb] = mfma16x16x32(w[2 * KH * t + h], qw[rb][h], acc[rb]);
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[rb][4 * t + i] = acc[rb][i];
    }
    const bf16_t* vp = a.v16 + at + n16 * kAttnChunk + 16 * g4;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int e = 0; e < 2; ++e) w[2 * dt + e] = ld16(vp + 16 * dt * kAttnChunk + 8 * e);
    if (!full) mask(s, k0, INT32_MAX);
    float sc[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) sc[rb] = a.scale_log2;
    u32x4 ph[NRB][2], pl[NRB][2];
    soft(st, s, sc, 0.f, [&](int rb, float (&x)[16]) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t h, l;
          split2(x[8 * e + 2 * k], x[8 * e + 2 * k + 1], h, l);
          ph[rb][e][k] = h, pl[rb][e][k] = l;
        }
    });
    if (!full) {
      const int valid = min(vmax - k0, kAttnChunk) - 16 * g4;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t m = (uint32_t)((1ull << (16 * min(max(valid - 8 * e - 2 * k, 0), 2))) - 1);
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) w[2 * dt + e][k] &= m;
        }
    }
    // an infinity times both parts of a probability would be NaN: left to the combine even if all rows see it
    u16x2 most = {0, 0};
#pragma unroll
    for (int i = 0; i < 2 * NDT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w[i][k] & 0x7fff7fffu));
    if (__any(most.x >= 0x7f80 || most.y >= 0x7f80)) {
      odd_pages |= 1ull << p;
#pragma unroll
      for (int i = 0; i < 2 * NDT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) w[i][k] &= ~((not_finite16(w[i][k]) >> 15) * 0xffffu);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          st.o[rb][dt] = mfma16x16x32(w[2 * dt + e], ph[rb][e], st.o[rb][dt]);
          st.o[rb][dt] = mfma16x16x32(w[2 * dt + e], pl[rb][e], st.o[rb][dt]);
        }
  }

  // Join the four key waves' sums: key wave w the head dimensions of tiles ND4 w ..
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    st.l[rb] += __shfl_xor(st.l[rb], 16);
    st.l[rb] += __shfl_xor(st.l[rb], 32);
    // (of a sum near 1 the logarithm is exact to more digits; O stays as it is)
    st.m[rb] -= kAbove;
    st.l[rb] *= kAboveFactor;
    if (g4 == 0) {
      s_m[wk][wr][16 * rb + n16] = st.m[rb];
      s_l[wk][wr][16 * rb + n16] = st.l[rb];
    }
  }
  if (lane == 0) s_odd[wk][wr] = odd_pages;
  lds_barrier();
  const int nrb = gridDim.y * WR * NRB;             // row blocks of the partials
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    float mx[kKeyWaves], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kKeyWaves; ++w) {
      mx[w] = s_m[w][wr][16 * rb + n16];
      M = fmaxf(M, mx[w]);
    }
#pragma unroll
    for (int w = 0; w < kKeyWaves; ++w) {
      const float f = mx[w] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mx[w] - M);
      L = __builtin_fmaf(f, s_l[w][wr][16 * rb + n16], L);
    }
    const float f = st.m[rb] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[rb] - M);
    if (rb) lds_barrier();                          // the last block's tiles have been read
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) s_o[wr][wk][dt][lane] = st.o[rb][dt] * f;
    lds_barrier();
    const size_t blk = (size_t)id * nrb + (blockIdx.y * WR + wr) * NRB + rb;
#pragma unroll
    for (int d = 0; d < ND4; ++d) {
      const int dt = wk * ND4 + d;
      f32x4 v = s_o[wr][0][dt][lane];
#pragma unroll
      for (int k = 1; k < kKeyWaves; ++k) v += s_o[wr][k][dt][lane];
      *reinterpret_cast<f32x4*>(a.part + ((blk * NDT + dt) * 64 + lane) * 4) = v;
    }
    if (wk == 0 && g4 == 0) a.ml[blk * 16 + n16] = make_float2(M, L);
    if (wk == 0 && lane == 0) {
      uint64_t w = 0;
#pragma unroll
      for (int k = 0; k < kKeyWaves; ++k) w |= s_odd[k][wr];
      a.odd[blk] = w;
    }
  }
}

// Joins the groups of a (sequence, kv head): grid (sequences x kv heads, row
// blocks, D / 16 tiles x T), NW waves.  A lane holds four columns of one row, as the
// partials do.  T = 1: a wave has a tile's 16 columns, waves take groups w, w + NW, ..
// T = 4, for many groups: a wave has four columns of four groups at once, groups 4 w ..
// 4 w + 3, then 4 NW on, so that few (sequence, kv head) pairs reach four times as many
// CUs.  Bound by latency: 144 rows of 16 scenes, 8 MB of partials, 4.9 us; 63 rows of one
// scene of 131 thousand tokens, 256 groups, 8.4 MB, 5.4 us (7.7 with T = 1).
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void k_kv8_combine(Kv8AttnArgs a, int nrb) {
  // groups of a wave loaded at once: no more than there are of few, as what is beyond is
  // loaded all the same (4: 36.5 us a call for 16 scenes of 9 rows, not 34.2)
  constexpr int NDT = D / 16, U = NW == 16 ? 4 : 2, T = NW == 16 ? 4 : 1;
  __shared__ f32x4 s_o[NW][64];
  __shared__ f32x4 s_x[NW][64];
  __shared__ float s_m[NW][16], s_l[NW][16];
  __shared__ int s_has[NW];                         // waves that have an s_x
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int n16 = lane & 15, g4 = T == 1 ? lane >> 4 : blockIdx.z % 4, sub = T == 1 ? 0 : lane >> 4;
  const int b = blockIdx.x / a.nkv, kvh = blockIdx.x % a.nkv, rb = blockIdx.y, dt = blockIdx.z / T;
  const int r = 16 * rb + n16;
  const bool in_row = r < a.R * a.G;
  const int j = in_row ? r / a.G : 0, hq = kvh * a.G + (in_row ? r % a.G : 0);
  const int4 seq = a.seq[b];                        // (of no meaning if no row of the sequence sees anything)
  int vis;
  if (a.st) {
    const SeqState& s = a.st[b];
    vis = j < s.count ? s.base + (j < s.causal ? j + 1 : s.count) : -1;
  } else {
    vis = a.vis[b * a.R + j];
  }
  if (!in_row) vis = -1;
  const int per = __any(vis > 0) ? seq.y : 0, ppw = seq.z;
  const int first = seq.x + kvh;
  float M = -INFINITY, L = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  // values that are not finite: apart from o, whose factors can round to zero
  f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
  bool has = false;
  for (int i0 = T * wave; i0 < per; i0 += T * NW * U) {
    const int i = i0 + sub;
    float2 ml[U];
    f32x4 v[U];
    uint64_t odd[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool in = i + T * NW * k < per;
      const size_t blk = ((size_t)first + (size_t)(in ? i + T * NW * k : i0) * a.nkv) * nrb + rb;
      ml[k] = a.ml[blk * 16 + n16];
      odd[k] = a.odd[blk];
      v[k] = *reinterpret_cast<const f32x4*>(a.part + ((blk * NDT + dt) * 64 + 16 * g4 + n16) * 4);
      if (!in) {
        ml[k] = make_float2(-INFINITY, 0.f);
        v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        odd[k] = 0;
      }
    }
    for (int k = 0; k < U; ++k)
      for (uint64_t w = odd[k]; w; w &= w - 1) {    // for the rows that see them
        has = true;
        const int p = (i + T * NW * k) * ppw + __builtin_ctzll(w);
        const bool in8 = p < a.packed[b];
        const size_t at = ((size_t)a.table[(size_t)b * a.stride + p] * a.nkv + kvh) * kAttnChunk * D;
        for (int key = 0; key < kAttnChunk; ++key)
          for (int e = 0; e < 4; ++e) {
            const size_t c = at + (size_t)(16 * dt + 4 * g4 + e) * kAttnChunk + key;
            const float v = in8 ? ((a.v8[c] & 0x7f) == 0x7f ? NAN : 0.f) : bf2f(a.v16[c]);
            if (!(fabsf(v) < INFINITY) && p * kAttnChunk + key < vis) x[e] += v;
          }
      }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float mn = fmaxf(M, ml[k].x);
      const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - mn);
      const float f1 = ml[k].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[k].x - mn);
      o = o * f0 + v[k] * f1;
      L = L * f0 + ml[k].y * f1;
      M = mn;
    }
  }
#pragma unroll
  for (int d = 16; T == 4 && d < 64; d *= 2) {      // the wave's four groups
    const float m = __shfl_xor(M, d), l = __shfl_xor(L, d), mn = fmaxf(M, m);
    const float f0 = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - mn);
    const float f1 = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * f0 + __shfl_xor(o[e], d) * f1;
    L = L * f0 + l * f1;
    M = mn;
  }
  has = __any(has);
  if (has) {
#pragma unroll
    for (int d = 16; T == 4 && d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], d);
    s_x[wave][lane] = x;
  }
  if (lane == 0) s_has[wave] = has;
  s_o[wave][lane] = o;
  if (lane < 16) {
    s_m[wave][n16] = M;
    s_l[wave][n16] = L;
  }
  __syncthreads();
  if (wave != 0) return;
  const uint64_t having = __ballot(lane < NW && s_has[lane % NW]);
  if (sub != 0 || vis < 0) return;                  // no such row: left as it was
  M = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, s_m[w][n16]);
  o = x = f32x4{0.f, 0.f, 0.f, 0.f};
  L = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float m = s_m[w][n16], f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - M);
    o += s_o[w][lane] * f;
    L += s_l[w][n16] * f;
  }
  for (uint64_t w = having; w; w &= w - 1) x += s_x[__builtin_ctzll(w)][lane];
  if (vis == 0) {
    o = f32x4{0.f, 0.f, 0.f, 0.f};
  } else {
    o = o * (kAboveFactor / L) + x;
  }
  const int row = b * a.R + j, d = hq * D + 16 * dt + 4 * g4;
  bf16_t* out = a.out + (a.opk ? (int64_t)xop_at(row, d, a.opk) : (int64_t)row * a.out_stride + d);
  *reinterpret_cast<u32x2*>(out) = u32x2{pack2(o.x, o.y), pack2(o.z, o.w)};
  if (a.lse && dt == 0 && g4 == 0)
    a.lse[(size_t)row * a.nq + hq] = vis == 0 ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

int row_blocks(int rows) { return (rows + 15) / 16; }

// How a workgroup takes a pass's row blocks: NRB x WR of them, y workgroups.
struct Shape {
  int nrb, wr, y;
};
Shape shape_of(int rows) {
  const int n = row_blocks(rows);
  if (n <= 2) return {n, 1, 1};
  return {2, 2, (n + 3) / 4};
}
int padded_blocks(int rows) {
  const Shape s = shape_of(rows);
  return s.nrb * s.wr * s.y;
}

}  // namespace

hipError_t launch_kv8_pack(const Kv8PackArgs& a, int D, hipStream_t s) {
  const dim3 grid((a.rows + kAttnChunk - 1) / kAttnChunk, a.nkv, 2);
  if (a.cs)
    hipLaunchKernelGGL((D == 128 ? k_kv8_pack<128, true> : k_kv8_pack<64, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((D == 128 ? k_kv8_pack<128, false> : k_kv8_pack<64, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

// One workgroup per CU: fewer pages each, in two workgroups of 4 waves per CU or one
// after another, cost their prologues (about 5 us before the first product).  Per call
// (with an earlier combine), groups aimed at 256 / 512 / 1024: 16 scenes of 2 to 8
// thousand tokens, one row each, 21.8 / 23.7 / 25.4 us, 9 rows 35.3 / 43.8 / 51.0; one of
// 131 thousand tokens 27.7 / 40.1 / 40.0.
int kv8_target_groups(int rows, int ncu) { return std::max(1, ncu / shape_of(rows).y); }

// Few (sequence, kv head) pairs have many groups each: 16 waves join them, not 4.  A
// context asks this of its prompts alone, as the order of its sums depends on it.
bool kv8_many(int64_t groups, int B, int nkv) { return groups >= (int64_t)32 * B * nkv; }

// Where the lengths decide, count_groups stops at `target`, or at kKv8MaxPages, or
// (with more heads of sequences than that) takes 4 floor(n / target) pages where n
// groups of 4 were: at most 2 target and one shorter group for each of them.
int64_t kv8_max_groups(int B, int nkv, int stride, int ppw, int target) {
  const int64_t most = ppw ? ppw : kKv8MaxPages, least = ppw ? ppw : kKv8MinPages;
  const int64_t fixed = (int64_t)B * nkv * ((stride + most - 1) / most);
  if (ppw) return fixed;
  return std::min((int64_t)B * nkv * ((stride + least - 1) / least), std::max<int64_t>(fixed, 2 * (int64_t)target + (int64_t)B * nkv));
}

size_t kv8_part_bytes(int64_t groups, int rows, int D) { return (size_t)groups * padded_blocks(rows) * 16 * D * sizeof(float); }
size_t kv8_ml_bytes(int64_t groups, int rows) {
  return (size_t)groups * padded_blocks(rows) * (16 * sizeof(float2) + sizeof(uint64_t)) + SPEC_MAX_ROWS * sizeof(int4) + 16;
}
void kv8_set_parts(Kv8AttnArgs& a, void* part, void* ml, int64_t groups) {
  const size_t n = (size_t)groups * padded_blocks(a.R * a.G);
  a.part = static_cast<float*>(part);
  a.ml = static_cast<float2*>(ml);
  a.odd = reinterpret_cast<uint64_t*>(a.ml + 16 * n);
  a.seq = reinterpret_cast<int4*>(a.odd + (n + 1) / 2 * 2);
}

hipError_t launch_kv8_attn(const Kv8AttnArgs& a, int D, int64_t groups, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const Shape h = shape_of(a.R * a.G);
  void (*f)(Kv8AttnArgs) = nullptr;
  if (D == 128)
    f = h.wr == 2 ? k_kv8_attn<128, 2, 2> : h.nrb == 2 ? k_kv8_attn<128, 2, 1> : k_kv8_attn<128, 1, 1>;
  else
    f = h.wr == 2 ? k_kv8_attn<64, 2, 2> : h.nrb == 2 ? k_kv8_attn<64, 2, 1> : k_kv8_attn<64, 1, 1>;
  hipExtLaunchKernelGGL(f, dim3((unsigned)groups, h.y), dim3(64 * h.wr * kKeyWaves), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}

hipError_t launch_kv8_combine(const Kv8AttnArgs& a, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const int rows = a.R * a.G;
  const dim3 grid(a.B * a.nkv, row_blocks(rows), a.many ? D / 4 : D / 16);
  void (*f)(Kv8AttnArgs, int) = nullptr;
  if (D == 128)
    f = a.many ? k_kv8_combine<128, 16> : k_kv8_combine<128, 4>;
  else
    f = a.many ? k_kv8_combine<64, 16> : k_kv8_combine<64, 4>;
  hipExtLaunchKernelGGL(f, grid, dim3(a.many ? 1024 : 256), 0, s, e0, e1, 0, a, padded_blocks(rows));
  return hipGetLastError();
}

}  // namespace specdec
