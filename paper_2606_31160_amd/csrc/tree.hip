// A pass over trees of drafted tokens: its rows' keys and values into their slots of a
// paged cache, attention of the rows over it, and the commit of the accepted paths.
#include <hip/hip_runtime.h>

#include "device.h"
#include "tree.h"

namespace specdec {

namespace {

constexpr int kWords = (SPEC_MAX_ROWS + 63) / 64;   // of a row's ancestors
constexpr float kAbove = 24.f;

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

struct Seq {
  int first, rows, len;
};
// Sequence b of a pass whose d_first makes sense.
__device__ __forceinline__ Seq sequence(const TreeRows& t, int b) {
  Seq s{t.first[b], t.first[b + 1], t.len[b]};
  s.rows = s.len < 0 || s.len > t.stride * SPEC_KV_PAGE ? 0 : s.rows - s.first;
  return s;
}

// The sequence of row r, or -1; the whole wave asks, of a pass whose d_first makes sense.
__device__ int sequence_of(const TreeRows& t, int r) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < t.B; b0 += 64) {
    const int b = b0 + lane;
    const uint64_t in = __ballot(b < t.B && t.first[min(b, t.B - 1)] <= r && r < t.first[min(b, t.B - 1) + 1]);
    if (in) return b0 + __builtin_ctzll(in);
  }
  return -1;
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

// One workgroup of 256 threads per row.
template <int D>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a) {
  const TreeRows& t = a.t;
  const int r = blockIdx.x;
  if (!sound(t)) return flag(t);
  const int b = sequence_of(t, r);
  if (b < 0) return;
  const Seq s = sequence(t, b);
  if (!s.rows) return flag(t);
  const int j = r - s.first, slot = s.len + j, page = page_of(t, b, slot), off = slot % SPEC_KV_PAGE;
  if (page < 0) flag(t);
  int p[3];
  if (a.pos) {
    const int e0 = a.axis_end[0], e1 = a.axis_end[1];   // an axis without pairs is not read
    p[0] = e0 ? a.pos[r] : 0;
    p[1] = e0 < 0 || e1 > e0 ? a.pos[t.rows + (int64_t)r] : 0;
    p[2] = e1 < D / 2 ? a.pos[2 * (int64_t)t.rows + r] : 0;
  } else {
    int deep = 0;
    if (t.parent)
      for (int i = parent_of(t, s, j); i >= 0; i = parent_of(t, s, i)) ++deep;
    else
      deep = j;
    p[0] = p[1] = p[2] = s.len + deep;
  }
  const int nr = a.nq + t.nkv;
  for (int e = threadIdx.x; e < nr * (D / 2); e += 256) {
    const int h = e / (D / 2), d = e % (D / 2);
    const int axis = a.axis_end[0] < 0 ? d % 3 : (d >= a.axis_end[0]) + (d >= a.axis_end[1]);
    const double x = a.turns[d] * p[axis];
    float sn, cs;
    sincospif(2.f * (float)(x - floor(x)), &sn, &cs);
    const bf16_t* src = (h < a.nq ? a.q + (int64_t)r * a.q_stride + (int64_t)h * D : a.k + (int64_t)r * a.kv_stride + (int64_t)(h - a.nq) * D) + 2 * d;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(src);
    const float x0 = __uint_as_float(w << 16), x1 = __uint_as_float(w & 0xffff0000u);
    const uint32_t y = pack2(x0 * cs - x1 * sn, x0 * sn + x1 * cs);
    if (h < a.nq)
      *reinterpret_cast<uint32_t*>(a.q_out + (int64_t)r * a.q_out_stride + (int64_t)h * D + 2 * d) = y;
    else if (page >= 0)
      *reinterpret_cast<uint32_t*>(a.kc + (((int64_t)page * t.nkv + h - a.nq) * SPEC_KV_PAGE + off) * D + 2 * d) = y;
  }
  if (page >= 0)
    for (int e = threadIdx.x; e < t.nkv * D; e += 256)
      a.vt[((int64_t)page * t.nkv * D + e) * SPEC_KV_PAGE + off] = a.v[(int64_t)r * a.kv_stride + e];
}

// One workgroup of 4 waves per row and query head; wave w takes pages w, w + 4, ...  A lane has one
// key of a page, then D / 64 dimensions of the output.
template <int D>
__global__ __launch_bounds__(256) void k_tree_attn(TreeAttnArgs a) {
  const TreeRows& t = a.t;
  constexpr int P = SPEC_KV_PAGE, U = D / 64;
  __shared__ float s_q[D], s_p[4][P], s_m[4], s_l[4], s_o[4][D];
  __shared__ uint64_t s_up[kWords + 1];
  const int r = blockIdx.x, h = blockIdx.y, kvh = h / a.G;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (!sound(t)) return flag(t);
  const int b = sequence_of(t, r);
  if (b < 0) return;
  const Seq s = sequence(t, b);
  if (!s.rows) return flag(t);
  if (threadIdx.x == 0) {
    for (int i = 0; i <= kWords; ++i) s_up[i] = 0;
    for (int i = r - s.first; i >= 0; i = parent_of(t, s, i)) s_up[i >> 6] |= 1ull << (i & 63);
  }
  for (int d = threadIdx.x; d < D; d += 256) s_q[d] = bf2f(a.q[(int64_t)r * a.q_stride + (int64_t)h * D + d]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[U] = {};
  const int end = s.len + s.rows;
  for (int pg = wave; pg * P < end; pg += 4) {
    const int page = page_of(t, b, pg * P), slot = pg * P + lane;
    if (page < 0) {
      flag(t);
      continue;
    }
    const int i = slot - s.len;
    const bool see = i < 0 || (i < s.rows && (s_up[i >> 6] >> (i & 63) & 1));
    const bf16_t* k = a.kc + (((int64_t)page * t.nkv + kvh) * P + lane) * D;
    float z = 0.f;
    for (int d = 0; d < D; ++d) z += s_q[d] * bf2f(k[d]);
    z = see ? z * a.scale_log2 : -INFINITY;
    float mx = z;
    for (int x = 32; x; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
    mx = fmaxf(mx + kAbove, m);                    // so that sums of the largest values stay in range
    const float e = see ? exp2f(z - (mx == -INFINITY ? 0.f : mx)) : 0.f, f = m == -INFINITY ? 0.f : exp2f(m - mx);
    float sum = e;
    for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
    l = l * f + sum;
    m = mx;
    s_p[wave][lane] = e;
    const uint64_t seen = __ballot(see);
    const bf16_t* v = a.vt + ((int64_t)page * t.nkv + kvh) * D * P;
    for (int u = 0; u < U; ++u) {
      float acc = isfinite(o[u]) ? o[u] * f : o[u];
      for (int c = 0; c < P; ++c) {
        const float x = bf2f(v[(lane + 64 * u) * P + c]);
        if (seen >> c & 1) acc += isfinite(x) ? s_p[wave][c] * x : x;
      }
      o[u] = acc;
    }
  }
  if (lane == 0) s_m[wave] = m, s_l[wave] = l;
  for (int u = 0; u < U; ++u) s_o[wave][lane + 64 * u] = o[u];
  __syncthreads();
  const float M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float L = 0.f, w[4];
  for (int i = 0; i < 4; ++i) {
    w[i] = s_m[i] == -INFINITY ? 0.f : exp2f(s_m[i] - M);
    L += w[i] * s_l[i];
  }
  for (int d = threadIdx.x; d < D; d += 256) {
    float x = 0.f;
    for (int i = 0; i < 4; ++i) x += isfinite(s_o[i][d]) ? s_o[i][d] * (w[i] / L) : s_o[i][d];
    a.out[(int64_t)r * a.out_stride + (int64_t)h * D + d] = f2bf(L == 0.f ? NAN : x);
  }
  if (a.lse && threadIdx.x == 0) a.lse[(int64_t)r * a.nq + h] = (M - kAbove + log2f(L * 0x1p24f)) * 0.6931471805599453f;
}

// One workgroup of 256 threads per layer, sequence and kv head, and keys or values.  Every
// one walks the tree.  The rows move to lower slots only, in their order, 16 at a time: what a
// step reads lies above everything that earlier ones wrote, and what it overwrites was
// read by this step or earlier ones, the same dimension by the same wave.
template <int D>
__global__ __launch_bounds__(256) void k_tree_commit(TreeCommitArgs a) {
  const TreeRows& t = a.t;
  __shared__ int s_path[SPEC_MAX_ROWS], s_n;
  const int layer = blockIdx.x, b = blockIdx.y, kvh = blockIdx.z >> 1, tid = threadIdx.x;
  const bool val = blockIdx.z & 1, first = layer == 0 && blockIdx.z == 0;
  const bool ok = sound(t);
  const Seq s = ok ? sequence(t, b) : Seq{0, 0, 0};
  if (!ok || (!s.rows && t.first[b + 1] > t.first[b])) flag(t);
  if (tid == 0) {
    const int most = min(s.rows, a.budget ? a.budget[b] : s.rows);
    int n = 0;
    for (int j = 0; j >= 0 && n < most;) {
      s_path[n++] = j;
      const int want = a.greedy[s.first + j];
      if (want == a.stop && a.stop != -1) break;
      int to = -1;
      for (int i = s.rows - 1; i > j; --i)
        if (parent_of(t, s, i) == j && a.tokens[s.first + i] == want) to = i;
      j = to;
    }
    s_n = n;
  }
  __syncthreads();
  const int n = s_n;
  if (first) {
    for (int i = tid; i < n; i += 256) {
      if (a.path) a.path[s.first + i] = s_path[i];
      if (a.committed) a.committed[s.first + i] = a.greedy[s.first + s_path[i]];
    }
    if (tid == 0) {
      if (a.n) a.n[b] = n;
      if (a.new_len) a.new_len[b] = t.len[b] + n;
    }
  }
  bf16_t* pool = (val ? a.vt : a.kc) + layer * a.layer_stride;
  const int i16 = tid & 15;
  for (int n0 = 0; n0 < n; n0 += 16) {
    const int i = n0 + i16;
    bool move = i < n && s_path[min(i, n - 1)] != i;
    int from = 0, to = 0;
    if (move) {
      from = s.len + s_path[i], to = s.len + i;
      const int pf = page_of(t, b, from), pt = page_of(t, b, to);
      if (pf < 0 || pt < 0) move = false, flag(t);
      from = from % SPEC_KV_PAGE, to = to % SPEC_KV_PAGE;
      const int64_t head_f = ((int64_t)pf * t.nkv + kvh) * SPEC_KV_PAGE * D, head_t = ((int64_t)pt * t.nkv + kvh) * SPEC_KV_PAGE * D;
      bf16_t x[D / 16];
      const int64_t step = val ? SPEC_KV_PAGE : 1;
      if (move)
        for (int u = 0; u < D / 16; ++u) x[u] = pool[head_f + (val ? from : from * D) + ((tid >> 4) + 16 * u) * step];
      if (move)
        for (int u = 0; u < D / 16; ++u) pool[head_t + (val ? to : to * D) + ((tid >> 4) + 16 * u) * step] = x[u];
    }
  }
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, int D, hipStream_t s) {
  hipLaunchKernelGGL(D == 128 ? k_kv_append<128> : k_kv_append<64>, dim3(a.t.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, int D, hipStream_t s) {
  hipLaunchKernelGGL(D == 128 ? k_tree_attn<128> : k_tree_attn<64>, dim3(a.t.rows, a.nq), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_tree_commit(const TreeCommitArgs& a, int D, hipStream_t s) {
  hipLaunchKernelGGL(D == 128 ? k_tree_commit<128> : k_tree_commit<64>, dim3(a.layers, a.t.B, 2 * a.t.nkv), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace specdec
