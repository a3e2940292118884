// A pass over trees of drafted tokens: its rows' keys and values into their slots of a
// paged cache, attention of the rows over it, and the commit of the accepted paths.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "device.h"
#include "tree.h"

namespace specdec {

namespace {

__device__ __forceinline__ void flag(const TreeRows& t) {
  if (t.err) *t.err = SPEC_E_INVAL;
}

// Whether d_first makes sense; the whole wave asks.
__device__ bool sound(const TreeRows& t) {
  const int lane = threadIdx.x & 63;
  bool bad = false;
  for (int b = lane; b < t.B; b += 64) {
    const int lo = t.first[b], hi = t.first[b + 1];
    bad |= lo < 0 || hi < lo || hi > t.rows;
  }
  return !__any(bad);
}

// p[i] for an i that all lanes share, by a scalar load: a vector load could not be awaited apart from a wave's
// loads into LDS.
__device__ __forceinline__ int shared_at(const int32_t* p, int64_t i) {
  const uint64_t at = (uint64_t)(p + i);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
  return *(const __attribute__((address_space(4))) int32_t*)((uint64_t)hi << 32 | lo);
}

struct Seq {
  int first, rows, len;
};
// Sequence b of a pass whose d_first makes sense.
__device__ __forceinline__ Seq sequence(const TreeRows& t, int b) {
  Seq s{t.first[b], t.first[b + 1], t.len[b]};
  s.rows = s.len < 0 || s.len > t.stride * SPEC_KV_PAGE ? 0 : s.rows - s.first;
  return s;
}

// The page of a slot, or -1.
__device__ __forceinline__ int page_of(const TreeRows& t, int b, int slot) {
  const int i = slot / SPEC_KV_PAGE;
  const int page = i < t.stride ? t.table[(int64_t)b * t.stride + i] : -1;
  return page < t.pages ? page : -1;
}

__device__ __forceinline__ int parent_of(const TreeRows& t, const Seq& s, int j) {
  if (!t.parent) return j - 1;
  const int p = t.parent[s.first + j];
  if (p >= -1 && p < j) return p;
  flag(t);
  return -1;
}

// Sum over the lanes up to and including each.
template <class T>
__device__ __forceinline__ T scan(T x) {
#define SD_STEP(ctrl, rows) x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, false))
  SD_STEP(0x111, 0xf);                              // row_shr:1, 2, 4, 8
  SD_STEP(0x112, 0xf);
  SD_STEP(0x114, 0xf);
  SD_STEP(0x118, 0xf);
  SD_STEP(0x142, 0xa);                              // row_bcast:15, rows 1 and 3
  SD_STEP(0x143, 0xc);                              // row_bcast:31, rows 2 and 3
#undef SD_STEP
  return x;
}
template <class T>
__device__ __forceinline__ T lane_of(T x, int l) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
}
template <class T>
__device__ __forceinline__ T total(T x) {
  return lane_of(scan(x), 63);
}

// ---------------------------------------------------------------------------
// Append.  The rows of a sequence that share a page are a tile.  A workgroup has a tile and either up to `heads` of the
// heads that are rotated (queries, then keys) or one head of the values.
//   Rotation: a thread has 8 dimensions of every 2048 / D-th row of the tile, whose 4 angles a row it forms once for all
// heads: the turn theta_d p / 2 pi in 64 bits, of which the fraction remains, then sine and cosine in 32.
//   Values: rows through LDS, columns out, 8 slots of a dimension in one store; the ends of a sequence's slots
// one by one.
// Bound by memory: 4096 rows of 32 + 2 x 8 heads of 128, 100 MB, 22.1 us a call in graphs (4.6 TB/s; a copy of 4 GiB
// reaches 4.78), 29.1 with outputs left to the caches; 20 thousand rows of 28 + 2 x 4 heads 86.1 and 88.8.  One
// head a workgroup, which forms every angle anew: 33.6 and 121.
// ---------------------------------------------------------------------------

// The tile of workgroup x: its sequence, its page's index there.  `one` wave reports what is wrong with the pass.
__device__ bool tile_of(const TreeRows& t, int x, bool one, Seq& s, int& b, int& index) {
  const int lane = threadIdx.x & 63;
  if (!sound(t)) {
    if (one) flag(t);
    return false;
  }
  if (one)
    for (int k = lane; k < t.B; k += 64)
      if ((t.len[k] < 0 || t.len[k] > t.stride * SPEC_KV_PAGE) && t.first[k + 1] > t.first[k]) flag(t);
  int at = 0;
  for (int b0 = 0; b0 < t.B; b0 += 64) {
    const int k = min(b0 + lane, t.B - 1);
    Seq q{t.first[k], t.first[k + 1], t.len[k]};
    const bool in = b0 + lane < t.B, off = q.len < 0 || q.len > t.stride * SPEC_KV_PAGE;
    q.rows = in && !off ? q.rows - q.first : 0;
    const int begin = q.len / SPEC_KV_PAGE;
    const int tiles = q.rows > 0 ? (int)(((int64_t)q.len + q.rows - 1) / SPEC_KV_PAGE) - begin + 1 : 0;
    const int ends = at + scan(tiles);
    if (x < lane_of(ends, 63)) {
      const int l = __builtin_ctzll(__ballot(ends > x));
      b = b0 + l;
      s = Seq{lane_of(q.first, l), lane_of(q.rows, l), lane_of(q.len, l)};
      index = lane_of(begin, l) + x - (lane_of(ends, l) - lane_of(tiles, l));
      return true;
    }
    at = lane_of(ends, 63);
  }
  return false;
}

// A pass of several heads a workgroup streams its outputs past the caches, which its inputs then keep.
template <bool STREAM>
__device__ __forceinline__ void store16(bf16_t* to, u32x4 x) {
  if (STREAM)
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to));
  else
    *reinterpret_cast<u32x4*>(to) = x;
}

template <int D, bool STREAM>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  constexpr int P = SPEC_KV_PAGE, C = D / 8, R = 256 / C, U = P / R;   // chunks of a row; rows at once; rows of a thread
  constexpr int kRow = D / 2 + 1;                   // LDS words of a row: odd, so that 8 rows on is 8 banks on
  __shared__ uint32_t lds[P * kRow];
  __shared__ int16_t s_up[SPEC_MAX_ROWS];
  const TreeRows& t = a.t;
  const int rotated = a.nq + t.nkv, groups = (rotated + a.heads - 1) / a.heads;
  const int tid = threadIdx.x, y = blockIdx.y;
  const bool one = y == 0 && tid < 64;              // the wave that reports
  Seq s;
  int b, index;
  if (!tile_of(t, blockIdx.x, one && blockIdx.x == 0, s, b, index)) return;
  // the tile's rows [j0, j1) of the sequence, in slots from `off` on
  const int64_t begin = (int64_t)index * P - s.len;
  const int j0 = (int)max(begin, (int64_t)0), j1 = (int)min((int64_t)s.rows, begin + P), n = j1 - j0, off = (int)(j0 - begin);
  int page = index < t.stride ? t.table[(int64_t)b * t.stride + index] : -1;
  if (page >= t.pages) page = -1;
  if (page < 0 && one) flag(t);
  const int c = tid % C, r0 = tid / C;

  if (y >= groups) {                                // values
    if (page < 0) return;
    const int h = y - groups;
    const bf16_t* src = a.v + (int64_t)(s.first + j0) * a.kv_stride + (int64_t)h * D + 8 * c;
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + R * u < n) x[u] = ld16(src + (int64_t)(r0 + R * u) * a.kv_stride);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + R * u < n)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[(off + r0 + R * u) * kRow + 4 * c + e] = x[u][e];
    __syncthreads();
    bf16_t* const to = a.vt + ((int64_t)page * t.nkv + h) * D * P;
    const int c0 = off >> 3, c1 = (off + n - 1) >> 3;
    if (c0 == 0 && c1 == 7 && n == P) {
#pragma unroll
      for (int i = tid; i < D / 2 * 8; i += 256) {
        const int k = i & 7, d = i >> 3;            // slots 8 k .., dimensions 2 d and 2 d + 1
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = lds[(8 * k + e) * kRow + d];
        u32x4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100);
          hi[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302);
        }
        store16<STREAM>(to + (2 * d) * P + 8 * k, lo);
        store16<STREAM>(to + (2 * d + 1) * P + 8 * k, hi);
      }
    } else {
      for (int i = tid; i < n * (D / 2); i += 256) {
        const int d = i / n, slot = off + i - d * n;
        const uint32_t w = lds[slot * kRow + d];
        to[(2 * d) * P + slot] = (bf16_t)w;
        to[(2 * d + 1) * P + slot] = (bf16_t)(w >> 16);
      }
    }
    return;
  }

  if (!a.pos && t.parent) {                         // workgroup-uniform: rows <= SPEC_MAX_ROWS
    for (int j = tid; j < s.rows; j += 256) s_up[j] = (int16_t)parent_of(t, s, j);
    __syncthreads();
  }
  double turns[4];
  int axis[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int d = 4 * c + k;
    turns[k] = a.turns[d];
    axis[k] = a.axis_end[0] < 0 ? d % 3 : (d >= a.axis_end[0]) + (d >= a.axis_end[1]);
  }
  float cs[U][4], sn[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + r0 + R * u;
    if (j >= j1) continue;
    double p[3];
    if (a.pos) {
      const int e0 = a.axis_end[0], e1 = a.axis_end[1];   // an axis without pairs is not read
      const int32_t* at = a.pos + s.first + j;
      p[0] = e0 ? at[0] : 0;
      p[1] = e0 < 0 || e1 > e0 ? at[t.rows] : 0;
      p[2] = e1 < D / 2 ? at[2 * (int64_t)t.rows] : 0;
    } else {
      int deep = j;
      if (t.parent) {
        deep = 0;
        for (int i = s_up[j]; i >= 0; i = s_up[i]) ++deep;
      }
      p[0] = p[1] = p[2] = (double)s.len + deep;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const double x = axis[k] == 0 ? p[0] : axis[k] == 1 ? p[1] : p[2];
      sincospif(2.f * (float)__builtin_amdgcn_fract(turns[k] * x), &sn[u][k], &cs[u][k]);
    }
  }
  const int h1 = min((y + 1) * a.heads, rotated);
  for (int h = y * a.heads; h < h1; ++h) {          // workgroup-uniform
    const bool query = h < a.nq;
    if (!query && page < 0) break;
    const bf16_t* src = query ? a.q + (int64_t)(s.first + j0) * a.q_stride + (int64_t)h * D + 8 * c
                              : a.k + (int64_t)(s.first + j0) * a.kv_stride + (int64_t)(h - a.nq) * D + 8 * c;
    bf16_t* to = query ? a.q_out + (int64_t)(s.first + j0) * a.q_out_stride + (int64_t)h * D + 8 * c
                       : a.kc + (((int64_t)page * t.nkv + h - a.nq) * P + off) * D + 8 * c;
    const int64_t step = query ? a.q_stride : a.kv_stride, step_to = query ? a.q_out_stride : D;
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + R * u < n) x[u] = ld16(src + (r0 + R * u) * step);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + R * u < n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float e = __uint_as_float(x[u][k] << 16), o = __uint_as_float(x[u][k] & 0xffff0000u);
          x[u][k] = pack2(e * cs[u][k] - o * sn[u][k], e * sn[u][k] + o * cs[u][k]);
        }
        store16<STREAM>(to + (r0 + R * u) * step_to, x[u]);
      }
  }
}

// ---------------------------------------------------------------------------
// Attention.  A kv head's query rows r = j G + g of a sequence (pass row j, query head g of the kv head's G) are cut
// into chunks of RW tiles of 32.  A workgroup has one chunk and a group of consecutive pages, whose halves (32 slots)
// its eight waves take in turn, each with a running maximum and sum of its tile's rows:
//   RW = 1  wave w takes halves w, w + 8, ..., loads them itself, and waits for no other before the end;
//   RW = 2  waves kw and kw + 4 share halves kw, kw + 4, ..., a tile each; two more waves load all keys and all
//           values, a step ahead, as a wave that loads stands still until its loads have gone out.
// Per half page
//   S^T = K Q^T   (32x32x16 bf16 products, keys down, query rows across)
//   p = 2^(scale log2e s - m), l += p
//   O^T += V^T P^T, p as the sum of two bf16 numbers
// and the waves' (m, l, O) are joined in LDS: the group gives O / L, (m, L) of every row.  One group of a
// sequence is its result; several are joined by k_tree_combine.
//
// Halves lie in LDS, copied there by loads that pass no register.  RW = 1: keys and values each in one buffer, the
// next keys while these probabilities meet their values, the next values while the next scores are formed.  The
// 16-byte chunks of a row are permuted by an xor, so that the sixteen lanes that an LDS read serves together (of 32
// those whose number has an even number of ones in bits 2 to 4, then the others) fall in distinct banks: 215 bytes a
// cycle and CU, where 136 were read with a permutation for eight lanes at a time.  Row m of a score tile is key
// (m & 3) + 4 ((m >> 3) & 1) + 8 ((m >> 2) & 1) + 16 (m >> 4): a lane's eight scores of a 16-key step are then eight
// consecutive keys, one 16-byte read of a value row.
//
// Masks: halves below the sequence's length are seen whole.  In the others a lane has 32 bits, one for each key: in a
// chain by its row's number, in a tree two words of its ancestors' bits, which wave 0 makes while the first pages come
// (a walk up the tree: a chain of 160 rows over 2000 slots 36.6 us in graphs, where it takes 22.8).  Values of slots that
// no row sees are set to zero there.
//
// What is not finite.  A value that is not finite (or sums that leave the range, of values near its end) makes a sum
// that is not finite, which the end of the loop sees.  The wave then goes over its halves once more, with such values
// taken as zero: sums that had none are the same bits again, and so are those of a row that does not see them as without them; the
// others are infinite or NaN.  Where a sum still leaves the range, one of values 2^40 lower, formed beside it, does not.
//
// What bounds it (in graphs, with the combine).  16 scenes of 2 to 8 thousand slots, one row each, 158 MB: 37 us, of
// which a group's loads take 28 (5.6 TB/s) and the rest are the chain lengths -> plan -> page table -> first page,
// joins and the combine; 144 rows of them 46, as chunks of more than 64 query rows are read twice.  25 rows over 131
// thousand slots: 32, of which 18 are 13 steps at 1.07 PFLOP/s of matrix operations (a large library product: 1.35), as
// much with half of the operands' LDS reads and 2.4 less without any load.  40 rows over 4096 slots 16.5: three such
// steps, and 9 us that do not depend on the cache.
// ---------------------------------------------------------------------------

typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma32x32x16(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Waves of an attention workgroup that multiply, that load (RW = 2), query rows of a tile.
constexpr int kWaves = 8, kLoaders = 2, kTileRows = 32;

// What workgroup i of an attention call does.
struct Work {
  int b, kvh, chunk, chunks, groups, lo, hi;   // chunk of so many; pages [lo, hi) of the sequence's
  int part;                            // this group's number
  Seq s;
};

// Groups of a sequence of so many pages, `per` to a group: one more than needed at most where the division rounds, and
// the same for every workgroup that asks.
__device__ __forceinline__ int groups_of(int pages, int per) {
  return min((int)ceilf((float)pages * __builtin_amdgcn_rcpf((float)per)), pages);
}

// Workgroup x of a sequence's nc chunks x `groups` groups x nkv kv heads; its unit's first group and unit are numbered from
// `part` and `unit` on.
template <int RW>
__device__ __forceinline__ void work_at(const TreeAttnArgs& a, int x, int nc, int pages, int part, int unit, Work& w) {
  const int nkv = a.t.nkv, keys = nkv * w.groups;   // key: (group, kv head)
  const int whole = (keys & ~7) * nc;
  w.chunks = nc;
  int key;
  if (nc == 1) {
    w.chunk = 0;
    key = x;
  } else if (x < whole) {
    const int o = x / (8 * nc);
    x -= o * 8 * nc;
    w.chunk = x >> 3;
    key = 8 * o + (x & 7);
  } else {
    x -= whole;
    w.chunk = x / (keys & 7);
    key = (keys & ~7) + x - w.chunk * (keys & 7);
  }
  const int group = key / nkv, q = pages / w.groups, r = pages - q * w.groups;
  w.kvh = key - group * nkv;
  w.lo = group * q + min(group, r);
  w.hi = w.lo + q + (group < r);
  const int u = w.kvh * nc + w.chunk;
  w.part = part + u * w.groups + group;
  if (group == 0 && threadIdx.x == 0)
    a.units[1 + unit + u] = TreeUnit{part + u * w.groups, w.groups, w.s.first, w.chunk * kTileRows * RW, w.s.rows * a.G, w.kvh * a.G};
}

// Whether there is a workgroup i.  Every (sequence, kv head, chunk) has as many groups, of equal size or one page
// less, as leave at most `target` workgroups, and none fewer than `least` pages.  The chunks of one group are eight
// workgroups apart, where its size allows: on one XCD, whose L2 gives its pages to all of them.
template <int RW>
__device__ bool work_of(const TreeAttnArgs& a, int i, Work& w) {
  constexpr int NS = (SPEC_MAX_ROWS + 63) / 64, C = kTileRows * RW;
  const TreeRows& t = a.t;
  const bool one = i == 0 && threadIdx.x == 0;
  if (t.B == 1) {                                   // nothing to look up
    const int first = shared_at(t.first, 0), end = shared_at(t.first, 1), len = shared_at(t.len, 0);
    const bool bad = first < 0 || end < first || end > t.rows, off = len < 0 || len > t.stride * SPEC_KV_PAGE;
    const int n = bad || off ? 0 : end - first;
    if (one && (bad || (end > first && (off || len + n > t.stride * SPEC_KV_PAGE)))) flag(t);
    const int nc = (n * a.G + C - 1) / C, units = nc * t.nkv;
    const int pages = min((len + n + SPEC_KV_PAGE - 1) / SPEC_KV_PAGE, t.stride);
    if (one) a.units[0].first = units;
    if (i >= units && (i >= a.target || units == 0)) return false;
    w.b = 0;
    w.s = Seq{first, n, len};
    w.groups = max(min(groups_of(pages, a.least), a.target / units), 1);
    if (i >= units * w.groups) return false;
    work_at<RW>(a, i, nc, pages, 0, 0, w);
    return true;
  }
  const int lane = threadIdx.x & 63;
  int first[NS], n[NS], len[NS], chunks[NS], pages[NS];
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    first[k] = n[k] = len[k] = chunks[k] = pages[k] = 0;
    if (64 * k < t.B) {
      const int b = min(64 * k + lane, t.B - 1);
      first[k] = t.first[b], n[k] = t.first[b + 1], len[k] = t.len[b];
    }
  }
  bool bad = false, off_table = false;
#pragma unroll
  for (int k = 0; k < NS; ++k)
    if (64 * k < t.B) {
      const bool in = 64 * k + lane < t.B;
      bad |= in && (first[k] < 0 || n[k] < first[k] || n[k] > t.rows);
      const bool off = len[k] < 0 || len[k] > t.stride * SPEC_KV_PAGE;
      off_table |= in && n[k] > first[k] && (off || len[k] + n[k] - first[k] > t.stride * SPEC_KV_PAGE);
      n[k] = in && !off ? n[k] - first[k] : 0;
      chunks[k] = (n[k] * a.G + C - 1) / C * t.nkv;  // of all kv heads
      pages[k] = n[k] ? min((len[k] + n[k] + SPEC_KV_PAGE - 1) / SPEC_KV_PAGE, t.stride) : 0;
    }
  bad = __any(bad);
  if (i == 0 && threadIdx.x < 64 && (bad || off_table)) flag(t);
  if (bad) {
    if (one) a.units[0].first = 0;
    return false;
  }
  int units = 0;
  float all = 0;                                    // pages of all units
#pragma unroll
  for (int k = 0; k < NS; ++k)
    if (64 * k < t.B) {
      units += total(chunks[k]);
      all += total((float)chunks[k] * (float)pages[k]);
    }
  if (one) a.units[0].first = units;
  // pages of a group: from a guess on (a sequence's last group is half full) the first that leaves at most `target` groups
  int per = max((int)(all / ((float)a.target - 0.5f * (float)units)), a.least);
  if (units >= a.target) per = INT32_MAX / 2;       // one group each
  while (units < a.target) {
    int g = 0;
#pragma unroll
    for (int k = 0; k < NS; ++k)
      if (64 * k < t.B) g += total(chunks[k] * groups_of(pages[k], per));
    if (g <= a.target) break;
    per += max(per / 16, 1);
  }
  int at = 0, unit = 0;                             // workgroups and units of the sequences before
#pragma unroll
  for (int k = 0; k < NS; ++k)
    if (64 * k < t.B) {
      const int g = groups_of(pages[k], per), mine = chunks[k] * g;
      const int ends = at + scan(mine), uends = unit + scan(chunks[k]);
      if (i < lane_of(ends, 63)) {
        const int l = __builtin_ctzll(__ballot(ends > i));
        auto of = [&](int x) { return lane_of(x, l); };
        w.b = 64 * k + l;
        w.s = Seq{of(first[k]), of(n[k]), of(len[k])};
        w.groups = of(g);
        const int begin = of(ends) - of(mine);
        work_at<RW>(a, i - begin, of(chunks[k]) / t.nkv, of(pages[k]), begin, of(uends) - of(chunks[k]), w);
        return true;
      }
      at = lane_of(ends, 63), unit = lane_of(uends, 63);
    }
  return false;
}

// What a bf16 pair holds that is not finite: 0x8000 in those halves.
__device__ __forceinline__ uint32_t not_finite16(uint32_t w) {
  return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// (hi, lo) bf16 pairs whose sums are x and y within 2^-16.  A matrix operand holds eight bits of p; one alone would be off as much
// as the result's own rounding to bf16, two are far below it, and three would take a third more products in all.  Sums of p are of
// p as it is.
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = pack2(x, y);
  asm("" : "+v"(hi));                               // (else the compiler rounds x a second time on its own)
  lo = pack2(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
}

__device__ __forceinline__ float other_half(float x) {   // of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// 4 KB of a page, from byte `step` on, to `lds`: lane l's 16 bytes of the i-th KB to 1024 i + 16 l, from an offset o0 .. o3 of its
// own in that KB.  Written out, as the compiler would wait for all such loads before every LDS read; a load
// has no register to write.  (An instruction's offset counts at both ends.)  The first load is five wait states into the
// block, as a vector instruction (a lane's read for instance) may have written `page` or `step` right before it.  `once`: nobody
// else reads the page.
#define SD_PAGE_TO_LDS(hint)                                                  \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\t"                             \
               "buffer_load_dwordx4 %3, %1, %2 offen " hint "lds\n\t"         \
               "buffer_load_dwordx4 %4, %1, %2 offen offset:1024 " hint "lds\n\t" \
               "buffer_load_dwordx4 %5, %1, %2 offen offset:2048 " hint "lds\n\t" \
               "buffer_load_dwordx4 %6, %1, %2 offen offset:3*1024 " hint "lds" ::"s"(lds), \
               "s"(page), "s"(step), "v"(o0), "v"(o1), "v"(o2), "v"(o3)       \
               : "m0", "memory")
__device__ __forceinline__ void page_to_lds(bool once, __amdgpu_buffer_rsrc_t page, uint32_t lds, uint32_t step, uint32_t o0, uint32_t o1,
                                            uint32_t o2, uint32_t o3) {
  if (once)
    SD_PAGE_TO_LDS("nt ");
  else
    SD_PAGE_TO_LDS("");
}
#undef SD_PAGE_TO_LDS
// All LDS reads have returned (before their source is overwritten).
__device__ __forceinline__ void lds_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void loads_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// What the chunks of row r of a half's keys are permuted by.
template <int D>
__device__ __forceinline__ int key_swizzle(int r) {
  return D == 128 ? (r & 3) + 4 * ((r >> 3) & 1) + 8 * ((r >> 2) & 1) : ((r >> 1) & 1) + 2 * ((r >> 3) & 1) + 4 * ((r >> 2) & 1);
}

// The rows that each row of a sequence's tree sees, itself and its ancestors, as bits, by one wave whose lane l has the
// parents of rows l, l + 64, ...  A row takes the bits of its ancestor 1, 2, 4, ... above: a chain of 160 rows takes 8
// steps.  Words behind the last row are not written.
constexpr int kLineWords = SPEC_MAX_ROWS / 32, kLaneRows = (SPEC_MAX_ROWS + 63) / 64;
template <int K>
__device__ __forceinline__ void lines_step(int rows, int (&up)[kLaneRows], uint32_t (&x)[kLaneRows][kLineWords]) {
  if (64 * K >= rows) return;
  const int from = up[K];
  int next = -1;
  uint32_t y[kLineWords] = {};
#pragma unroll
  for (int u = 0; u <= K; ++u) {
    const bool here = from >= 0 && from >> 6 == u;
    const int n = __builtin_amdgcn_ds_bpermute(4 * (from & 63), up[u]);
    next = here ? n : next;
#pragma unroll
    for (int e = 0; e < kLineWords; ++e)
      if (e < 2 * u + 2 && 32 * e < rows) {         // (a row of the u-th 64 has no others)
        const uint32_t z = __builtin_amdgcn_ds_bpermute(4 * (from & 63), x[u][e]);
        y[e] = here ? z : y[e];
      }
  }
  up[K] = next;
#pragma unroll
  for (int e = 0; e < kLineWords; ++e) x[K][e] |= y[e];
}
__device__ __forceinline__ void lines(const TreeRows& t, int rows, int (&up)[kLaneRows], uint32_t (*line)[kLineWords]) {
  constexpr int NS = kLaneRows;
  const int lane = threadIdx.x & 63;
  uint32_t x[NS][kLineWords];
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int j = 64 * k + lane;
    if (j >= rows) up[k] = -1;
    if (up[k] < -1 || up[k] >= j) {
      flag(t);
      up[k] = -1;
    }
#pragma unroll
    for (int e = 0; e < kLineWords; ++e) x[k][e] = j >> 5 == e ? 1u << (j & 31) : 0;
  }
  for (;;) {
    bool more = up[0] >= 0;
#pragma unroll
    for (int k = 1; k < NS; ++k) more |= up[k] >= 0;
    if (!__any(more)) break;
    static_assert(NS == 3, "one call for every 64 rows, parents behind their children");
    lines_step<2>(rows, up, x);
    lines_step<1>(rows, up, x);
    lines_step<0>(rows, up, x);
  }
#pragma unroll
  for (int k = 0; k < NS; ++k)
    if (64 * k + lane < rows)
#pragma unroll
      for (int e = 0; e < kLineWords; ++e)
        if (32 * e < rows) line[64 * k + lane][e] = x[k][e];
}

template <int D, int RW>
__global__ __launch_bounds__(64 * (kWaves + (RW == 2 ? kLoaders : 0)), RW == 2 ? 3 : 2) void k_tree_attn(TreeAttnArgs a) {
  constexpr int DT = D / 32, KS = D / 16, H = 32, kHalf = H * D * 2;   // slots of a half, bytes of its keys or values
  constexpr int kLoads = kHalf / 1024, KC = D / 8, KW = kWaves / RW;   // KW waves share a group's halves
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ uint32_t s_line[SPEC_MAX_ROWS][kLineWords];
  __shared__ float s_m[kWaves][kTileRows], s_l[kWaves][kTileRows];
  const TreeRows& t = a.t;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int kw = wave % KW, rw = wave / KW, n32 = lane & 31, half = lane >> 5;
  Work w;
  if (!work_of<RW>(a, blockIdx.x, w)) return;
  auto shared = [](int& x) __attribute__((always_inline)) { x = __builtin_amdgcn_readfirstlane(x); };   // known to the compiler only so
  shared(w.b), shared(w.kvh), shared(w.chunk), shared(w.groups), shared(w.lo), shared(w.hi), shared(w.part);
  shared(w.chunks), shared(w.s.first), shared(w.s.rows), shared(w.s.len);
  // (a page that one workgroup reads past the caches: 16 scenes of one row 38.7 -> 37.1 us a call; pages of several chunks so: 40
  // rows over 4096 slots 18.5 -> 20.1, 25 over 131 thousand 39.6 -> 44.7)
  const bool once = w.chunks == 1;
  const int row0 = (w.chunk * RW + rw) * kTileRows, rows = w.s.rows * a.G;
  const int last = min(2 * w.hi, (w.s.len + w.s.rows + H - 1) / H), tail = w.s.len / H;   // halves: the group's end; seen whole before
  const int32_t* const table = t.table + (int64_t)w.b * t.stride;
  auto page_at = [&](int hp) __attribute__((always_inline)) {   // pool page of a half, or -1
    const int x = shared_at(table, hp >> 1);
    return x < t.pages ? max(x, -1) : -1;
  };

  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds);
  // a lane's chunk of each KB: keys' row lane / KC, values' row lane / 4
  uint32_t koff[4];                                 // of the x-th KB of four
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const int r = 64 / KC * x + lane / KC;
    koff[x] = (lane / KC) * D * 2 + ((lane % KC) ^ key_swizzle<D>(r)) * 16;
  }
  const uint32_t voff = (lane >> 2) * 128 + ((lane & 3) ^ (lane >> 4)) * 16;
  auto resource = [&](const bf16_t* pool, int page) __attribute__((always_inline)) {
    const uint64_t at = (uint64_t)(pool + ((int64_t)max(page, 0) * t.nkv + w.kvh) * (2 * H * D));
    // (the compiler does not see that it is the same for all lanes)
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, 2 * kHalf, 0x00020000);
  };
  auto load_k = [&](int page, int to, int odd_half) __attribute__((always_inline)) {   // to `to` bytes into LDS
    const auto r = resource(a.kc, page);
#pragma unroll
    for (int i = 0; i < kLoads; i += 4)
      page_to_lds(once, r, lds0 + to + 1024 * i, odd_half * kHalf + 1024 * i, koff[0], koff[1], koff[2], koff[3]);
  };
  auto load_v = [&](int page, int to, int odd_half) __attribute__((always_inline)) {
    const auto r = resource(a.vt, page);
    // 16 rows of 64 bytes a KB, 128 bytes apart in the page
#pragma unroll
    for (int i = 0; i < kLoads; i += 4)
      page_to_lds(once, r, lds0 + to + kHalf + 1024 * i, odd_half * 64 + 2048 * i, voff, voff + 1024, voff + 2 * 1024, voff + 3 * 1024);
  };
  const bool loader = RW == 2 && wave >= kWaves;    // wave-uniform
  // Buffers of 2 kHalf bytes, keys and then values.  RW = 1: a wave's own one.  RW = 2: two for each kw, which take turns.
  int ids[KW];                                      // a loader's pages of the step to come
  auto ids_of = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KW; ++k) ids[k] = p0 + k < last ? page_at(p0 + k) : -1;
  };
  auto load_step = [&](int p0, int turn) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KW; ++k)
      if (p0 + k < last) {
        const int to = 2 * kHalf * (2 * k + turn);
        if (wave == kWaves)
          load_k(ids[k], to, k & 1);
        else
          load_v(ids[k], to, k & 1);
      }
  };
  int p = 2 * w.lo + kw, page = -1, next = -1;      // half pages
  const int mine = 2 * kHalf * (RW == 1 ? wave : 2 * kw);
  if (loader) {
    ids_of(2 * w.lo);
    load_step(2 * w.lo, 0);
    ids_of(2 * w.lo + KW);
  }
  if (!loader && p < last) {
    page = page_at(p);
    if (RW == 1) {
      load_k(page, mine, wave & 1);
      load_v(page, mine, wave & 1);
    }
    if (p + KW < last) next = page_at(p + KW);
  }
  const bool trees = last > tail && t.parent && wave == 0;   // wave-uniform
  int up[kLaneRows];
  if (trees)
#pragma unroll
    for (int k = 0; k < kLaneRows; ++k) up[k] = 64 * k + lane < w.s.rows ? t.parent[w.s.first + 64 * k + lane] : -1;
  // Q operands, zeros for rows that there are not
  const int r = row0 + n32, qj = r < rows ? r / a.G : 0, head = w.kvh * a.G + (r < rows ? r % a.G : 0);
  u32x4 q[KS];
  u32x4* const sq = reinterpret_cast<u32x4*>(lds + kWaves * 2 * kHalf) + (rw & 1) * KS * 64 + lane;   // RW = 2: in LDS
  if (!loader) {
    const bf16_t* src = a.q + (int64_t)(w.s.first + qj) * a.q_stride + (int64_t)head * D + 8 * half;
    constexpr int QS = RW == 1 ? KS : KS / KW;      // a wave's operands
#pragma unroll
    for (int k = 0; k < QS; ++k) q[k] = ld16(src + 16 * (RW == 1 ? k : kw + KW * k));
    if (trees) lines(t, w.s.rows, up, s_line);
#pragma unroll
    for (int k = 0; k < QS; ++k) {
      if (r >= rows) q[k] = u32x4{0, 0, 0, 0};
      if (RW == 2) sq[(kw + KW * k) * 64] = q[k];
    }
  }
  __syncthreads();
  if (RW == 1)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" ::"v"(q[k]));   // awaited here, not among the loads of the loop
  if (loader) {
    int turn = 0;
    for (int p0 = 2 * w.lo; p0 < last; p0 += KW) {
      loads_but<0>();
      asm volatile("s_barrier" ::: "memory");       // this step's halves have come, and the last one's have been read
      turn ^= 1;
      load_step(p0 + KW, turn);
      ids_of(p0 + 2 * KW);
    }
    return;
  }

  // this lane's operand rows in LDS
  const int krow = (n32 & 3) + 4 * ((n32 >> 3) & 1) + 8 * ((n32 >> 2) & 1) + 16 * (n32 >> 4);
  const int kswz = key_swizzle<D>(krow);
  const int kat = krow * D * 2, vat = kHalf + n32 * 64;
  u32x4 kx[KS], vx[2][DT];
  auto keys = [&](int from) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k) kx[k] = *reinterpret_cast<const u32x4*>(lds + from + kat + (((2 * k + half) ^ kswz) * 16));
  };
  auto value = [&](int from, int dt, int step) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4*>(lds + from + vat + dt * 32 * 64 + (((2 * step + half) ^ ((n32 >> 2) & 3)) * 16));
  };

  float m, l;
  f32x16 o[DT], s;
  u32x4 ph[2], pl[2];
  auto zero = [&](f32x16& x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  };
  auto scores = [&]() __attribute__((always_inline)) {
    zero(s);
#pragma unroll
    for (int k = 0; k < KS; ++k) s = mfma32x32x16(kx[k], RW == 1 ? q[k] : sq[k * 64], s);
  };
  // A half that not every row sees whole: which of its slots the lane's row sees, bit 16 y + e this lane's score 8 y + e; slots
  // from `end` on are nobody's.
  uint32_t mask;
  int end;
  auto masks = [&]() __attribute__((always_inline)) {
    const int seen = page < 0 ? 0 : min(max(w.s.len - p * H, 0), H);   // slots below are everybody's
    end = page < 0 ? 0 : min(w.s.len + w.s.rows - p * H, H);
    uint32_t x = seen >= H ? ~0u : (1u << seen) - 1;
    if (page >= 0 && seen < H) {
      const int off = p * H - w.s.len;              // wave-uniform: the first slot's row, or what is missing to row 0
      if (!t.parent) {
        x |= (uint32_t)((1ull << min(max(qj - off + 1, 0), H)) - 1);
      } else if (off < 0) {
        x |= s_line[qj][0] << -off;
      } else {
        const uint32_t lo = s_line[qj][off >> 5], hi = (off | 31) + 1 < w.s.rows ? s_line[qj][(off >> 5) + 1] : 0;
        x |= (uint32_t)(((uint64_t)hi << 32 | lo) >> (off & 31));
      }
    }
    mask = x >> (8 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(mask >> (16 * (i >> 3) + (i & 7)) & 1)) s[i] = -INFINITY;
  };
  // Scores to probabilities, the parts of the keys of step 16 k in ph, pl[k]; grow(f) is called where sums have
  // to follow a maximum: when it has grown by 2^8.
  auto soft = [&](auto grow) __attribute__((always_inline)) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = fmaxf(mx, other_half(mx)) * a.scale_log2;
    const bool grown = mx > m + 8.f;
    if (__any(grown)) {
      // (each row by its own scores: no bit of it follows from what its siblings' slots hold)
      const float f = grown && m != -INFINITY ? __builtin_amdgcn_exp2f(m - mx) : 1.f;   // (-infinity: sums are zero yet)
      m = grown ? mx : m;
      if (__any(f != 1.f)) {
        l *= f;
        grow(f);
      }
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 8 * k + 2 * e;
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2, -ref));
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], a.scale_log2, -ref));
        sum += x + y;
        uint32_t h, g;
        split2(x, y, h, g);
        ph[k][e] = h, pl[k][e] = g;
      }
    l += sum;
  };

  m = -INFINITY, l = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) zero(o[dt]);
  // of a half in LDS: its values' operands
  auto values = [&](int from, bool whole) __attribute__((always_inline)) {
    if (!whole) {
      if (page < 0) flag(t);
      // nobody's slots may hold anything, and zero times that is not zero
      end = page < 0 ? 0 : min(w.s.len + w.s.rows - p * H, H);
      for (int d = lane; d < D; d += 64)
        for (int c = end >> 3; c < 4; ++c) {
          u32x4* const at = reinterpret_cast<u32x4*>(lds + from + kHalf + d * 64 + ((c ^ ((d >> 2) & 3)) * 16));
          u32x4 v = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] &= (uint32_t)((1ull << (16 * min(max(end - 8 * c - 2 * e, 0), 2))) - 1);
          *at = v;
        }
    }
#pragma unroll
    for (int step = 0; step < 2; ++step)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) vx[step][dt] = value(from, dt, step);
  };
  auto rest = [&](bool whole) __attribute__((always_inline)) {
    if (!whole) masks();
    soft([&](float f) __attribute__((always_inline)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
    });
#pragma unroll
    for (int step = 0; step < 2; ++step) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32x32x16(vx[step][dt], ph[step], o[dt]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32x32x16(vx[step][dt], pl[step], o[dt]);
    }
  };
  if (RW == 1) {
    while (p < last) {
      const bool more = p + KW < last, whole = p < tail && page >= 0;
      loads_but<kLoads>();                          // the keys have come
      keys(mine);
      scores();
      lds_read();
      if (more) {
        load_k(next, mine, wave & 1);
        loads_but<kLoads>();                        // the values have come
      } else {
        loads_but<0>();
      }
      values(mine, whole);
      lds_read();
      if (more) load_v(next, mine, wave & 1);
      rest(whole);
      p += KW;
      page = next;
      if (p + KW < last) next = page_at(p + KW);
    }
  } else {
    const bool busy = row0 < rows;                  // wave-uniform: the chunk's last tiles may have no rows
    int at = mine;
    for (int p0 = 2 * w.lo; p0 < last; p0 += KW) {  // workgroup-uniform
      const bool whole = p < tail && page >= 0;
      asm volatile("s_barrier" ::: "memory");       // the halves have come
      const int other = at ^ 2 * kHalf;
      if (p < last && busy) {
        keys(at);
        scores();
        values(at, whole);
        rest(whole);
      }
      p += KW;
      page = next;
      at = other;
      if (p + KW < last) next = page_at(p + KW);
      lds_read();
    }
  }

  // join the waves: each scales its sums by its part of the group's, then each adds up its share
  l += other_half(l);
  if (half == 0) s_m[wave][n32] = m, s_l[wave][n32] = l;
  __syncthreads();                                  // (every buffer has been read, too)
  f32x4* const sums = reinterpret_cast<f32x4*>(lds);   // [waves][DT][4][64], each in the place of a wave's pages
  constexpr int Q = DT * 4;
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int k = 0; k < KW; ++k) M = fmaxf(M, s_m[rw * KW + k][n32]);
#pragma unroll
  for (int k = 0; k < KW; ++k) {
    const float x = s_m[rw * KW + k][n32];
    L = __builtin_fmaf(x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - M), s_l[rw * KW + k][n32], L);
  }
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M) / L;   // at most one

  float x0[4] = {0.f, 0.f, 0.f, 0.f};               // 0 times what is not finite is NaN
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) x0[i & 3] = __builtin_fmaf(o[dt][i], 0.f, x0[i & 3]);
  const bool slow = __any(r < rows && (x0[0] + x0[1]) + (x0[2] + x0[3]) != 0.f);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    o[dt] *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sums[(wave * Q + dt * 4 + i) * 64 + lane] = f32x4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
  }
  if (slow) {
    // Once more, 32 dimensions at a time, operands straight from the pages.  Beside each sum one of lower values: a slot adds up
    // to 2^8 times the largest value, and a wave has fewer than 2^31.
    constexpr float kLow = 0x1p-40f;
#pragma unroll 1
    for (int dt = 0; dt < DT; ++dt) {
      bool open = false;                            // one of these dimensions' sums is not finite
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = sums[(wave * Q + dt * 4 + g) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) open |= !finite(v[e]);
      }
      if (!__any(r < rows && open)) continue;
      f32x16 z, low;
      uint64_t seen = 0;                            // of each dimension 1: infinity, 2: minus infinity, 4: NaN
      m = -INFINITY, l = 0.f;                       // (they become what they were)
      zero(z);
      zero(low);
#pragma unroll 1
      for (p = 2 * w.lo + kw; p < last; p += KW) {
        page = page_at(p);
        const int64_t at = ((int64_t)max(page, 0) * t.nkv + w.kvh) * (2 * H * D);
        const bf16_t* const pk = a.kc + at + (p & 1) * H * D + krow * D + 8 * half;
        const bf16_t* const pv = a.vt + at + (dt * 32 + n32) * SPEC_KV_PAGE + (p & 1) * H + 8 * half;
        u32x4 x[2] = {ld16(pv), ld16(pv + 16)};
#pragma unroll
        for (int k = 0; k < KS; ++k) kx[k] = ld16(pk + 16 * k);
        scores();
        masks();
        soft([&](float f) __attribute__((always_inline)) { z *= f, low *= f; });
        uint32_t odd = 0;
#pragma unroll
        for (int step = 0; step < 2; ++step) {
          const int valid = end - 16 * step - 8 * half;
          u32x4 y, y2;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[step][e] &= (uint32_t)((1ull << (16 * min(max(valid - 2 * e, 0), 2))) - 1);
            const uint32_t b = not_finite16(x[step][e]);
            odd |= b;
            y[e] = x[step][e] & ~((b >> 15) * 0xffffu);
            y2[e] = pack2(__uint_as_float(y[e] << 16) * kLow, __uint_as_float(y[e] & 0xffff0000u) * kLow);
          }
          z = mfma32x32x16(y, ph[step], z);
          z = mfma32x32x16(y, pl[step], z);
          low = mfma32x32x16(y2, ph[step], low);
          low = mfma32x32x16(y2, pl[step], low);
        }
        if (__any(odd != 0)) {
          // how many infinities, negative infinities and NaN of each dimension a row sees: 1, 2^8 and 2^16 for each
          // against a one for each slot that it sees
          f32x16 c;
          zero(c);
#pragma unroll
          for (int step = 0; step < 2; ++step) {
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t k = 0;
              y[e] = 0;
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const uint32_t v = x[step][e] >> (16 * b) & 0xffff;
                k |= (v == 0x7f80 ? 0x3f80u : v == 0xff80 ? 0x4380u : (v & 0x7fff) > 0x7f80 ? 0x4780u : 0u) << (16 * b);
                y[e] |= (mask >> (16 * step + 2 * e + b) & 1 ? 0x3f80u : 0u) << (16 * b);
              }
              x[step][e] = k;
            }
            c = mfma32x32x16(x[step], y, c);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int k = (int)c[i];
            seen |= (uint64_t)((k & 0xff ? 1 : 0) | (k & 0xff00 ? 2 : 0) | (k >> 16 ? 4 : 0)) << (3 * i);
          }
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * g + e, k = (int)(seen >> (3 * i)) & 7;
          v[e] = k             ? (k == 1 ? INFINITY : k == 2 ? -INFINITY : NAN) + 0.f * f   // (f is NaN where a score is)
                 : finite(z[i]) ? z[i] * f
                                : low[i] * (f * (1.f / kLow));
        }
        sums[(wave * Q + dt * 4 + g) * 64 + lane] = v;
      }
    }
  }
  __syncthreads();
  if (r >= rows) return;
#pragma unroll
  for (int k = 0; k < Q / KW; ++k) {
    const int g = k * KW + kw;
    f32x4 v = sums[(rw * KW * Q + g) * 64 + lane];
#pragma unroll
    for (int x = 1; x < KW; ++x) v += sums[((rw * KW + x) * Q + g) * 64 + lane];
    if (w.groups == 1) {
      if (L == 0.f) v = f32x4{NAN, NAN, NAN, NAN};
      bf16_t* to = a.out + (int64_t)(w.s.first + qj) * a.out_stride + (int64_t)head * D + 8 * g + 4 * half;
      *reinterpret_cast<u32x2*>(to) = u32x2{pack2(v.x, v.y), pack2(v.z, v.w)};
    } else {
      a.part[(((int64_t)w.part * RW + rw) * Q + g) * 64 + lane] = v;
    }
  }
  if (kw == 0 && half == 0) {
    if (w.groups > 1)
      a.ml[((int64_t)w.part * RW + rw) * kTileRows + n32] = make_float2(M, L);
    else if (a.lse)
      a.lse[(int64_t)(w.s.first + qj) * a.nq + head] = (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
  }
}

// Joins the groups of a (sequence, kv head, chunk): grid (units, tiles x eights of the dimensions), W waves to an
// eight.  A lane has four dimensions of a row, as it was written, of every (W subs)-th group: where there are many
// groups of tiles of at most 8 or 16 rows, a wave has subs = 4 or 2 of them at once.  Bound by the latency of its rounds
// of loads, of which the next is asked for before one is summed: one row of 7 query heads over 131 thousand slots, 256 groups,
// takes 21.7 us in graphs with the attention, 29.5 without these two and with a quotient for every group.
template <int D, int RW, int W>
__global__ __launch_bounds__(64 * (W < 4 ? 4 : W)) void k_tree_combine(TreeAttnArgs a) {
  constexpr int Q = D / 8, U = 4, GB = W < 4 ? 4 / W : 1;   // GB eights of the dimensions a workgroup
  __shared__ f32x4 s_o[GB * W][64];
  __shared__ float s_m[GB * W][64], s_a[GB * W][64];
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int rw = blockIdx.y / (Q / GB);
  const int g = blockIdx.y % (Q / GB) * GB + wave / W, w0 = wave % W;
  const int units = a.units[0].first;
  const TreeUnit u = a.units[1 + blockIdx.x];
  if ((int)blockIdx.x >= units || u.groups < 2) return;
  const int rows = u.rows - u.row - rw * kTileRows; // of this tile
  if (rows <= 0) return;
  const int bits = u.groups <= W * U || rows > 16 ? 5 : rows > 8 ? 4 : 3, subs = 32 >> bits;
  const int row = lane & ((1 << bits) - 1), half = lane >> bits & 1, sub = lane >> (bits + 1);
  const bool live = row < rows;
  float M = -INFINITY, A = 0.f;                     // maximum and sum of the groups' weights
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  f32x4 x[U] = {}, y[U] = {};
  float2 ml[U], next[U];
  auto load = [&](int k0, f32x4 (&o)[U], float2 (&ml)[U]) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int group = k0 + W * subs * k + sub;
      const int64_t tile = (int64_t)(u.part + group) * RW + rw;
      ml[k] = make_float2(-INFINITY, 0.f);
      if (live && group < u.groups) {
        ml[k] = a.ml[tile * kTileRows + row];
        o[k] = a.part[(tile * Q + g) * 64 + row + 32 * half];
      }
    }
  };
  if (w0 * subs < u.groups) load(w0 * subs, x, ml);
  for (int k0 = w0 * subs; k0 < u.groups; k0 += W * subs * U) {
    if (k0 + W * subs * U < u.groups) load(k0 + W * subs * U, y, next);
    float now = M, c[U];
#pragma unroll
    for (int k = 0; k < U; ++k) now = ml[k].y == 0.f ? now : fmaxf(now, ml[k].x);   // (0: a group without slots that the row sees)
    const float f = M == -INFINITY ? 0.f : A * __builtin_amdgcn_exp2f(M - now);
    float sum = f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      c[k] = ml[k].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - now) * ml[k].y;
      sum += c[k];
    }
    if (sum != 0.f) {
      // o stays the average of the groups so far: sums of large values stay in range
      const float r = 1.f / sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = finite(o[e]) ? o[e] * (f * r) : o[e];
#pragma unroll
      for (int k = 0; k < U; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += ml[k].y == 0.f ? 0.f : finite(x[k][e]) ? x[k][e] * (c[k] * r) : x[k][e];
      A = sum;
      M = now;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) x[k] = y[k], ml[k] = next[k];
  }
  for (int d = 2 << bits; d < 64; d <<= 1) {        // the groups that a wave had at once
    const float m2 = __shfl_xor(M, d), a2 = __shfl_xor(A, d), now = fmaxf(M, m2);
    const float f = A == 0.f ? 0.f : A * __builtin_amdgcn_exp2f(M - now), c = a2 == 0.f ? 0.f : a2 * __builtin_amdgcn_exp2f(m2 - now);
    const float r = 1.f / (f + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float o2 = __shfl_xor(o[e], d);
      o[e] = (A == 0.f ? 0.f : finite(o[e]) ? o[e] * (f * r) : o[e]) + (a2 == 0.f ? 0.f : finite(o2) ? o2 * (c * r) : o2);
    }
    M = now, A = f + c;
  }
  float mx = M, sum = A;
  if (W > 1) {
    s_o[wave][lane] = o, s_m[wave][lane] = M, s_a[wave][lane] = A;
    __syncthreads();
    if (w0 || sub) return;
    float c[W];
#pragma unroll
    for (int k = 1; k < W; ++k) mx = fmaxf(mx, s_m[wave + k][lane]);
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float x = s_a[wave + k][lane];
      c[k] = x == 0.f ? 0.f : __builtin_amdgcn_exp2f(s_m[wave + k][lane] - mx) * x;
      sum += c[k];
    }
    const float r = 1.f / sum;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const f32x4 x = s_o[wave + k][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += finite(x[e]) ? x[e] * (c[k] * r) : x[e];
    }
  }
  if (!live || sub) return;
  if (sum == 0.f) o = f32x4{NAN, NAN, NAN, NAN};
  const int at = u.row + rw * kTileRows + row, j = at / a.G, h = u.head + at % a.G;
  bf16_t* to = a.out + (int64_t)(u.first + j) * a.out_stride + (int64_t)h * D + 8 * g + 4 * half;
  *reinterpret_cast<u32x2*>(to) = u32x2{pack2(o.x, o.y), pack2(o.z, o.w)};
  if (a.lse && g == 0 && half == 0) a.lse[(int64_t)(u.first + j) * a.nq + h] = (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------
// Commit.  One workgroup per layer, sequence and kv head.  Each wave walks the tree, a lane having every 64th row: the
// row's children that hold its greedy token by one vote, the lowest of them next.  The rows move to lower slots only,
// in their order, 16 at a time: what a step reads lies above everything that earlier ones wrote, and what it
// overwrites was read by this step or earlier ones, the same dimensions by the same wave.  A small commit is bound by
// latency, the chain first rows -> tree -> page table -> slots: one launch, 3.3 us in graphs.  16 sequences of 28
// layers and 4 kv heads of 128 take 10.4 for 5 MB: a slot's values are one element of each of 128 lines, so 26 MB are
// fetched.  The page table's part in LDS first: 10.9.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void k_tree_commit(TreeCommitArgs a) {
  constexpr int P = SPEC_KV_PAGE, NS = (SPEC_MAX_ROWS + 63) / 64;
  const TreeRows& t = a.t;
  __shared__ int16_t s_path[4][SPEC_MAX_ROWS];
  const int layer = blockIdx.x, b = blockIdx.y, kvh = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool first = layer == 0 && kvh == 0 && wave == 0;
  int16_t* const path = s_path[wave];
  const bool ok = sound(t);
  Seq s = ok ? sequence(t, b) : Seq{0, 0, 0};
  s.first = __builtin_amdgcn_readfirstlane(s.first), s.rows = __builtin_amdgcn_readfirstlane(s.rows), s.len = __builtin_amdgcn_readfirstlane(s.len);
  if (first && (!ok || (!s.rows && t.first[b + 1] > t.first[b]))) flag(t);
  int up[NS], token[NS], greedy[NS];
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int j = 64 * k + lane;
    up[k] = -2, token[k] = greedy[k] = 0;
    if (j < s.rows) {
      up[k] = t.parent ? t.parent[s.first + j] : j - 1;
      token[k] = a.tokens[s.first + j], greedy[k] = a.greedy[s.first + j];
    }
  }
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    const int j = 64 * k + lane;
    if (j < s.rows && (up[k] < -1 || up[k] >= j)) {
      if (first) flag(t);
      up[k] = -1;
    }
  }
  const int most = min(s.rows, a.budget ? __builtin_amdgcn_readfirstlane(a.budget[b]) : s.rows);
  auto greedy_of = [&](int j) __attribute__((always_inline)) {
    int x = lane_of(greedy[0], j & 63);
#pragma unroll
    for (int k = 1; k < NS; ++k)
      if (j >= 64 * k) x = lane_of(greedy[k], j & 63);
    return x;
  };
  int n = 0;
  for (int j = 0; j >= 0 && n < most;) {            // wave-uniform
    if (lane == 0) path[n] = (int16_t)j;
    ++n;
    const int want = greedy_of(j);
    if (want == a.stop && a.stop != -1) break;
    int to = -1;
#pragma unroll
    for (int k = NS - 1; k >= 0; --k) {
      const uint64_t fit = __ballot(up[k] == j && token[k] == want && 64 * k + lane < s.rows);
      if (fit) to = 64 * k + __builtin_ctzll(fit);
    }
    j = to;
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's path is in LDS
  if (first) {
    for (int i = lane; i < n; i += 64) {
      const int j = path[i];
      if (a.path) a.path[s.first + i] = j;
      if (a.committed) a.committed[s.first + i] = a.greedy[s.first + j];
    }
    if (lane == 0) {
      if (a.n) a.n[b] = n;
      if (a.new_len) a.new_len[b] = t.len[b] + n;
    }
  }
  // step i of 16, and a sixteenth of the dimensions: of keys C consecutive ones, of values every 16th
  constexpr int C = D / 16;
  bf16_t *const kc = a.kc + layer * a.layer_stride, *const vt = a.vt + layer * a.layer_stride;
  const int i16 = tid & 15, d0 = tid >> 4;
  for (int n0 = 0; n0 < n; n0 += 16) {
    const int i = n0 + i16;
    if (i >= n || path[i] == i) continue;
    const int from = s.len + path[i], to = s.len + i;
    const int pf = page_of(t, b, from), pt = page_of(t, b, to);
    if (pf < 0 || pt < 0) {
      flag(t);
      continue;
    }
    const int64_t hf = ((int64_t)pf * t.nkv + kvh) * P * D, ht = ((int64_t)pt * t.nkv + kvh) * P * D;
    const int sf = from % P, st = to % P;
    uint32_t k[C / 2];
    bf16_t v[C];
#pragma unroll
    for (int u = 0; u < C / 2; ++u) k[u] = reinterpret_cast<const uint32_t*>(kc + hf + sf * D + d0 * C)[u];
#pragma unroll
    for (int u = 0; u < C; ++u) v[u] = vt[hf + (d0 + 16 * u) * P + sf];
#pragma unroll
    for (int u = 0; u < C / 2; ++u) reinterpret_cast<uint32_t*>(kc + ht + st * D + d0 * C)[u] = k[u];
#pragma unroll
    for (int u = 0; u < C; ++u) vt[ht + (d0 + 16 * u) * P + st] = v[u];
  }
}

}  // namespace

hipError_t launch_kv_append(AppendArgs& a, int D, hipStream_t s) {
  // a tile at least for every sequence and 64 rows; at most two ends more for every sequence
  const int64_t tiles = (int64_t)a.t.rows / SPEC_KV_PAGE + 2 * std::min(a.t.B, a.t.rows), rotated = a.nq + a.t.nkv;
  // Heads of a workgroup, from the tiles that there may be at most: long passes have several, and so have passes of one row of many
  // sequences (32 of them with 32 rotated heads).  More heads share their angles, but leave fewer workgroups: 2 heads here 29.1 us
  // for the 4096 rows, 4 34.3, 8 45.4; for the 20 thousand 8 heads 88.9, 4 94.2, 1 121.
  a.heads = (int)std::min<int64_t>(8, std::max<int64_t>(1, tiles * rotated / 1024));
  const dim3 grid((unsigned)tiles, (unsigned)((rotated + a.heads - 1) / a.heads + a.t.nkv));
  if (D == 128)
    hipLaunchKernelGGL((a.heads > 1 ? k_kv_append<128, true> : k_kv_append<128, false>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((a.heads > 1 ? k_kv_append<64, true> : k_kv_append<64, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

namespace {
template <int D, int RW>
hipError_t attn(const TreeAttnArgs& a, const TreeAttnPlan& p, hipStream_t s) {
  constexpr int lds = kWaves * 2 * 32 * D * 2 + (RW == 2 ? 64 * D * 2 : 0), threads = 64 * (kWaves + (RW == 2 ? kLoaders : 0));   // half pages, Q
  static std::atomic<uint64_t> ready{0};            // devices that know of the LDS it needs
  int dev = 0;
  if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
  if (dev >= 64 || !(ready >> dev & 1)) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&k_tree_attn<D, RW>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    if (dev < 64) ready |= 1ull << dev;
  }
  hipLaunchKernelGGL((k_tree_attn<D, RW>), dim3(p.grid), dim3(threads), lds, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.combine) return e;
  // (one wave to an eighth where sequences have few groups, eight where they have many.  Us in graphs with the attention, W = 1
  // and 4: 16 sequences of one row over 5000 slots, 3 groups, 36.2 and 36.6, 8 of 5 rows over 3000, 4 groups, 20.5 and 21.0; W = 4 and
  // 8: one row over 20 thousand, 32 groups, 15.8 and 16.3, 63 over 20 thousand, 106 groups, 18.0 and 16.3, 175 over 131 thousand, 85
  // groups, 33.9 and 32.3)
  const auto combine = p.likely > 32 ? k_tree_combine<D, RW, 8> : p.likely > 4 ? k_tree_combine<D, RW, 4> : k_tree_combine<D, RW, 1>;
  const int waves = p.likely > 32 ? 8 : 4, eights = p.likely > 4 ? 1 : 4;
  hipLaunchKernelGGL(combine, dim3(p.units, RW * (D / 8) / eights), dim3(64 * waves), 0, s, a);
  return hipGetLastError();
}
}  // namespace

TreeAttnPlan tree_attn_plan(int batch, int rows, int nkv, int G, int D, int stride, int ncu) {
  TreeAttnPlan p;
  // Two tiles of an average sequence (the host knows no other; those without rows count too) share a workgroup's pages: 144
  // rows of 16 scenes 59.5 -> 50 us a call, 25 rows over 131 thousand slots 38.6 -> 34.2, 64 rows of the paper's heads over 4117
  // 20.4 -> 18.3.
  p.tiles = (int64_t)((rows + batch - 1) / batch) * G > kTileRows ? 2 : 1;
  const int64_t chunk = kTileRows * p.tiles;
  // (every sequence may end inside a chunk)
  p.units = (int)(nkv * std::min<int64_t>(((int64_t)rows * G + chunk - 1) / chunk + batch, (int64_t)rows * G));
  p.target = ncu;
  p.grid = std::max(p.target, p.units);
  // Pages of a group at least; short tables make one group, which needs no second kernel.  (The table's width bounds the
  // lengths, which only the device knows: short sequences in a wide table take several groups and the second kernel.)  Us in
  // graphs, 28 + 2 x 4 heads of 128, at least 2, 3 and 4 pages: 4 rows over 450, 1000, 4000 slots 11.1, 11.1, 11.8; 11.4, 11.3,
  // 11.9; 13.4, 13.5, 12.6; 40 rows over 1000 and 2000 14.1, 13.7, 14.3; 15.9, 15.6, 14.5.  One group up to 8 pages and up to 6:
  // 40 rows over 300 10.8 and 12.0, 4 rows over 380 9.2 and 10.7; up to 24: 5 rows over 700 and 960 13.7 and 16.1, several 12.2
  // and 12.4.
  // (a group of so many that the reciprocal's rounding leaves no second one, which nothing would join)
  const int least = 3, whole = 8;
  p.combine = stride > whole;
  p.least = p.combine ? least : 1 << 30;
  p.likely = std::min(stride / p.least, p.target / std::max(p.units, 1));
  const size_t part = (size_t)p.target * chunk * D * 4, ml = (size_t)p.target * chunk * 8,
               units = (size_t)(1 + p.units) * sizeof(TreeUnit);
  p.ml = (part + 255) / 256 * 256;
  p.unit = p.ml + (ml + 255) / 256 * 256;
  p.bytes = p.unit + (units + 255) / 256 * 256;
  return p;
}

hipError_t launch_tree_attn(TreeAttnArgs& a, const TreeAttnPlan& p, int D, void* workspace, hipStream_t s) {
  char* const w = static_cast<char*>(workspace);
  a.part = reinterpret_cast<f32x4*>(w);
  a.ml = reinterpret_cast<float2*>(w + p.ml);
  a.units = reinterpret_cast<TreeUnit*>(w + p.unit);
  a.target = p.target;
  a.least = p.least;
  if (p.tiles == 2) return D == 128 ? attn<128, 2>(a, p, s) : attn<64, 2>(a, p, s);
  return D == 128 ? attn<128, 1>(a, p, s) : attn<64, 1>(a, p, s);
}

hipError_t launch_tree_commit(const TreeCommitArgs& a, int D, hipStream_t s) {
  hipLaunchKernelGGL(D == 128 ? k_tree_commit<128> : k_tree_commit<64>, dim3(a.layers, a.t.B, a.t.nkv), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace specdec
