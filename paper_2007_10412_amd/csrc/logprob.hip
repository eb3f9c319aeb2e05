// Log probabilities of given classes, entropies and the likeliest classes of rows of logits, and the logits' gradient from those of
// the first two.
//
// q = softmax(z / T).  With m a row's maximum, l_v = (z_v - m) log2(e) / T, s = sum_v 2^l_v and u = sum_v 2^l_v l_v:
//   log q_v = (z_v - m) / T - ln s,   H = - sum_v q_v log q_v = ln s - ln 2 u / s,
//   dz_v = (a (1[v = token] - q_v) - h q_v (log q_v + H)) / T = 2^l_v (A + B l_v) + (a / T) 1[v = token]
// for the gradients a of log q[token] and h of H, A = (h ln 2 u / s - a) / (T s), B = - h ln 2 / (T s).  Forward a row is streamed once, 16 bytes a
// lane, and not kept (rows of up to four vectors a thread are); vectors that may hold a listed class are read again, from a cache.  Backward it is kept
// between its statistics and its gradient, in registers and, of the longer rows, in LDS; rows in parts are read twice, once in each of two launches.
//
// The k likeliest classes.  Any class of the list is at least as large as the k-th largest of the maxima of disjoint groups of
// the row (k groups then hold one such class each).  A thread's maxima are there already; one wave finds that bound of them bit by
// bit, and the few classes that reach it (of n groups some -n ln(1 - k / n): 1.4 k where n = 2 k) are placed by counting those before them.  Rows of which too
// many reach it (equal logits above all) are searched digit by digit, as often as it takes: the list is exact for every row.
#include <algorithm>

#include "vocab_row.hpp"

namespace rad {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;

// ------------------------------------------------------------------ selection
// Logits as whole numbers in their order (-0 as 0); 0 for -infinity and NaN, which are not listed.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return z > -INFINITY ? u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
constexpr uint32_t kLowestKey = 0x00800000u;            // of -FLT_MAX
// of two classes the one that comes first in a list has the larger entry; 0 is none
__device__ __forceinline__ uint64_t make_entry(uint32_t key, int index) { return key ? ((uint64_t)key << 32) | (uint32_t)~index : 0ull; }
__device__ __forceinline__ uint32_t entry_key(uint64_t e) { return (uint32_t)(e >> 32); }
__device__ __forceinline__ int entry_index(uint64_t e) { return (int)~(uint32_t)e; }

// entries that may wait for their places, at most kCand; counting takes their number squared over the threads
template <int NT> constexpr int cand_max() { return NT <= 128 ? 384 : NT <= 256 ? 512 : 1024; }
constexpr int kStrips = 512;
template <int NT, int GROUPS> struct TopLds {
  uint64_t cand[cand_max<NT>()];
  uint32_t group[GROUPS];
  uint32_t hist[256];
  int wave_n[NT / 64];
  uint16_t strip[kStrips];      // parts of a row that are to be looked at again
  int n, strips; uint32_t bound; int digit, need;
  __device__ __forceinline__ void begin() { if (threadIdx.x == 0) n = strips = 0; }     // (a barrier ahead of the first entry)
};

// wave 0: the 16 upper bits (0 below) of the k-th largest of 64 R maxima, each of `GROUPS` / (64 R) groups; at least kLowestKey
template <int GROUPS, int R>
__device__ __forceinline__ uint32_t group_bound(const uint32_t* group, int k) {
  static_assert(GROUPS % (64 * R) == 0, "whole waves");
  uint32_t m[R];
#pragma unroll
  for (int r = 0; r < R; ++r) m[r] = 0u;
#pragma unroll
  for (int j = 0; j < GROUPS / 64; ++j) m[j % R] = max(m[j % R], group[j * 64 + (int)threadIdx.x]);
  uint32_t p = 0u;
  for (int b = 31; b >= 16; --b) {
    const uint32_t with = p | (1u << b);
    int n = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) n += __popcll(__ballot(m[r] >= with));
    if (n >= k) p = with;
  }
  return max(p, kLowestKey);
}

template <int NT, int GROUPS> __device__ __forceinline__ void append(TopLds<NT, GROUPS>& lds, uint32_t key, int index) {
  const int at = atomicAdd(&lds.n, 1);
  if (at < cand_max<NT>()) lds.cand[at] = make_entry(key, index);
}

// after the groups' maxima are in place (a barrier): the bound, the same for the workgroup
template <int NT, int GROUPS> __device__ __forceinline__ uint32_t find_bound(TopLds<NT, GROUPS>& lds, int k) {
  if (threadIdx.x < 64) {
    constexpr int R = GROUPS >= 512 ? 8 : GROUPS / 64;
    const uint32_t b = R > 4 && k <= 128 ? group_bound<GROUPS, 4>(lds.group, k) : group_bound<GROUPS, R>(lds.group, k);
    if (threadIdx.x == 0) lds.bound = b;
  }
  __syncthreads();
  return lds.bound;
}

// The k largest of n entries, more than k of which are there, wherever equal keys come with ascending indexes: the k-th key digit
// by digit, then those above it and the first that equal it, in any order into cand.
template <int NT, int GROUPS, class F> __device__ __forceinline__ void select_exact(TopLds<NT, GROUPS>& lds, F entry, int64_t n, int k) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  uint32_t kth = 0u;
  int need = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int t = tid; t < 256; t += NT) lds.hist[t] = 0u;
    __syncthreads();
    for (int64_t i = tid; i < n; i += NT) {
      const uint32_t key = entry_key(entry(i));
      if (key && (shift == 24 || (key >> (shift + 8)) == (kth >> (shift + 8)))) atomicAdd(&lds.hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 64) {                                     // lane l: digits 255 - 4 l and the three below
      int c[4], sum = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) { c[q] = (int)lds.hist[255 - 4 * lane - q]; sum += c[q]; }
      int up = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(up, o); if (lane >= o) up += v; }
      int before = up - sum;
      if (before < need && need <= up) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (before < need && need <= before + c[q]) { lds.digit = 255 - 4 * lane - q; lds.need = need - before; }
          before += c[q];
        }
      }
    }
    __syncthreads();
    kth |= (uint32_t)lds.digit << shift;
    need = lds.need;
    __syncthreads();
  }
  if (tid == 0) lds.n = 0;
  __syncthreads();
  int taken = 0;                                        // entries of the k-th key: the first `need` belong to the list
  for (int64_t i0 = 0; i0 < n; i0 += NT) {
    const int64_t i = i0 + tid;
    const uint64_t e = i < n ? entry(i) : 0ull;
    const uint32_t key = entry_key(e);
    if (key > kth) lds.cand[atomicAdd(&lds.n, 1)] = e;
    if (taken >= need) continue;
    const uint64_t ties = __ballot(e != 0ull && key == kth);
    if (lane == 0) lds.wave_n[w] = __popcll(ties);
    __syncthreads();
    int before = taken + lanes_below(ties), all = taken;
#pragma unroll
    for (int q = 0; q < NT / 64; ++q) { if (q < w) before += lds.wave_n[q]; all += lds.wave_n[q]; }
    if (e != 0ull && key == kth && before < need) lds.cand[k - need + before] = e;
    taken = all;
    __syncthreads();
  }
  __syncthreads();
}

// the first k of the n entries in cand (a barrier before): put(place, entry) for those that are there.  Several neighbouring lanes
// count for one entry, as many as the workgroup has for each.
template <int NT, int GROUPS, class F> __device__ __forceinline__ void place_entries(const TopLds<NT, GROUPS>& lds, int n, int k, F put) {
  int lanes = 1;
  while (lanes < 64 && 2 * lanes * n <= NT) lanes *= 2;
  const int sub = (int)threadIdx.x & (lanes - 1);
  for (int i0 = 0; i0 < n; i0 += NT / lanes) {           // (the same for all lanes: shuffles below)
    const int i = i0 + (int)threadIdx.x / lanes;
    const uint64_t e = i < n ? lds.cand[i] : ~0ull;
    int before = 0;
#pragma unroll 4
    for (int j = sub; j < n; j += lanes) before += lds.cand[j] > e ? 1 : 0;
    for (int o = 1; o < lanes; o <<= 1) before += __shfl_xor(before, o);
    if (i < n && sub == 0 && before < k) put(before, e);
  }
  for (int i = n + (int)threadIdx.x; i < k; i += NT) put(i, 0ull);
}

// ------------------------------------------------------------------ statistics
// Sums and maxima of a wave by moves between its lanes' rows: 6 operations of a few cycles each, where shuffles take a trip through LDS.
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float none, float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(none), __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float of_lane(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }
constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, moved<kRowShr + 1, 0xf>(-INFINITY, v));
  v = fmaxf(v, moved<kRowShr + 2, 0xf>(-INFINITY, v));
  v = fmaxf(v, moved<kRowShr + 4, 0xf>(-INFINITY, v));
  v = fmaxf(v, moved<kRowShr + 8, 0xf>(-INFINITY, v));
  v = fmaxf(v, moved<kRowBcast15, 0xa>(-INFINITY, v));
  v = fmaxf(v, moved<kRowBcast31, 0xc>(-INFINITY, v));
  return of_lane(v, 63);
}
__device__ __forceinline__ float lanes_sum(float v) {
  v += moved<kRowShr + 1, 0xf>(0.f, v);
  v += moved<kRowShr + 2, 0xf>(0.f, v);
  v += moved<kRowShr + 4, 0xf>(0.f, v);
  v += moved<kRowShr + 8, 0xf>(0.f, v);
  v += moved<kRowBcast15, 0xa>(0.f, v);
  v += moved<kRowBcast31, 0xc>(0.f, v);
  return of_lane(v, 63);
}

// (m, s, u) of parts of a row; one with nothing in it adds its 0, or its NaN
struct RowStats {
  float m = -INFINITY, s = 0.f, u = 0.f;
  // as they are from another maximum: M >= m, neither it nor c infinite
  __device__ __forceinline__ void rebase(float M, float c) {
    if (m == -INFINITY) { u += s; m = M; return; }
    const float l = (m - M) * c, f = __builtin_amdgcn_exp2f(l);
    u = f * (u + s * fmaxf(l, kNoPower));
    s *= f;
    m = M;
  }
  __device__ __forceinline__ void join(float m2, float s2, float u2, float c) {
    RowStats o;
    o.m = m2; o.s = s2; o.u = u2;
    const float M = fmaxf(m, m2);
    rebase(M, c); o.rebase(M, c);
    s += o.s; u += o.u;
  }
  __device__ __forceinline__ void join_wave(float c) {
    rebase(lanes_max(m), c);
    s = lanes_sum(s); u = lanes_sum(u);
  }
};
// a workgroup's, the same for all of its threads; s_w: a triple a wave
template <int NT> __device__ __forceinline__ RowStats block_join(RowStats r, bool wave_joined, float c, float3* s_w) {
  constexpr int NW = NT / 64;
  if (!wave_joined) r.join_wave(c);
  if constexpr (NW == 1) return r;
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = make_float3(r.m, r.s, r.u);
  __syncthreads();
  RowStats all, of[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    of[w].m = s_w[w].x; of[w].s = s_w[w].y; of[w].u = s_w[w].z;
    all.m = fmaxf(all.m, of[w].m);
  }
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    of[w].rebase(all.m, c);
    all.s += of[w].s; all.u += of[w].u;
  }
  return all;
}

// what a row's statistics say
struct RowEnd {
  float base, log_s, inv_t, entropy;
  __device__ __forceinline__ RowEnd(const RowStats& r, float T) {
    base = exp_base(r.m); log_s = logf(r.s); inv_t = 1.f / T;
    entropy = log_s - kLn2 * (r.u / r.s);
  }
  __device__ __forceinline__ float log_q(float z) const { return (z - base) * inv_t - log_s; }
};

__device__ __forceinline__ bool token_counts(const int32_t* token, int row, int classes) {
  return !token || (uint32_t)token[row] < (uint32_t)classes;
}

// a row that does not count
template <int NT> __device__ __forceinline__ void leave_row(float* logprob, float* entropy, int k, int32_t* top_index, float* top_logprob, int row) {
  if (threadIdx.x == 0) {
    if (logprob) logprob[row] = 0.f;
    if (entropy) entropy[row] = 0.f;
  }
  for (int i = threadIdx.x; i < k; i += NT) {
    top_index[(int64_t)row * k + i] = -1;
    top_logprob[(int64_t)row * k + i] = -INFINITY;
  }
}
__device__ __forceinline__ void put_top(int32_t* top_index, float* top_logprob, int64_t at, uint64_t e, const RowEnd& end) {
  top_index[at] = e ? entry_index(e) : -1;
  top_logprob[at] = e ? end.log_q(key_value(entry_key(e))) : -INFINITY;
}

// ------------------------------------------------------------------ dense rows
// Forward.  A row is read once and not kept: each thread runs over its vectors with a maximum and sums of its own, whose base
// moves up when a larger logit comes (l = z c - m c is one operation so, with m c rounded once for all and what that rounding
// moved put right at the end), and reads those of its vectors again, from a cache, of which a logit may be on the list.
// Bases lie within +-2^24 T ln 2, where m c is rounded by one power of two at most; rows whose largest logit does not, and such as hold
// infinities or NaN, are done again, maximum first, by slow_stats.  (A row whose largest logit is just below the lowest base has a good sum
// from there, but that base would pass for its maximum, which a list of one class begins from: it is done again too.)  Bound by memory without lists, by the vector units with them (11 operations a
// logit at 32000 classes, 4 of them a row's share of bound and list): bf16 4096 x 32000 44 us (5.9 TB/s), with lists of 5 50; fp32 777 x 50257 with
// lists of 64 37 (4.3 TB/s).
constexpr float kFar = 0x1p24f;
constexpr int kAhead = 4, kSlots = 8;                   // vectors in flight
template <int NT> constexpr int groups_of() { return NT >= 512 ? 1 : NT == 256 ? 2 : 4; }   // a thread's, for a list's bound

__device__ __forceinline__ bool plain_stats(const RowStats& r, float lowest, float c) {
  return r.s > 0.5f && r.s < INFINITY && r.m > lowest && r.m * c <= kFar;
}

template <typename T, int NT> __device__ __noinline__ RowStats slow_stats(const T* z, int lo, int hi, float c, float3* s_w) {
  RowStats r;
  for (int v = lo + (int)threadIdx.x; v < hi; v += NT) r.m = fmaxf(r.m, ld_elem(z + v));
  __syncthreads();
  r = block_join<NT>(r, false, c, s_w);
  const float b = exp_base(r.m);
  r.s = r.u = 0.f;
  for (int v = lo + (int)threadIdx.x; v < hi; v += NT) {
    const float l = (ld_elem(z + v) - b) * c, e = __builtin_amdgcn_exp2f(l);
    r.s += e; r.u += e * fmaxf(l, kNoPower);
  }
  __syncthreads();
  return block_join<NT>(r, false, c, s_w);              // (all from one maximum)
}

template <typename T> struct Stream {
  static constexpr int VPL = 16 / (int)sizeof(T);
  static constexpr uint32_t kEmpty = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;     // -inf
  static __device__ __forceinline__ float at(const u32x4& v, int q) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[q]);
    else return __uint_as_float(q & 1 ? v[q >> 1] & 0xFFFF0000u : v[q >> 1] << 16);
  }
  static __device__ __forceinline__ float most(const u32x4& v) {
    float m = at(v, 0);
#pragma unroll
    for (int q = 1; q < VPL; ++q) m = fmaxf(m, at(v, q));
    return m;
  }
};
__device__ __forceinline__ float rounded_product(float m, float c) {   // (the same everywhere: never part of a fused operation)
#pragma clang fp contract(off)
  return m * c;
}

// a row's parts joined, by the last of its workgroups to be done
template <int NT, int GROUPS>
__device__ __forceinline__ void join_parts(const LogprobRows& a, int row, int parts, float z_token, TopLds<NT, GROUPS>& top, float3* s_w) {
  constexpr int kKept = 4;                               // entries of a thread that wait in registers
  const float c = kLog2e / a.temperature;
  const float* const st = static_cast<const float*>(a.ws) + (int64_t)row * parts * 3;
  const uint64_t* const list = reinterpret_cast<const uint64_t*>(static_cast<const char*>(a.ws) + logprob_stats_bytes(a.rows, parts)) +
                               (int64_t)row * parts * a.k;
  const int n_all = parts * a.k, tid = threadIdx.x;
  top.begin();
  uint64_t kept[kKept];
#pragma unroll
  for (int q = 0; q < kKept; ++q) { const int i = tid + q * NT; kept[q] = i < n_all ? load_of_all(list + i) : 0ull; }
  RowStats r;
  for (int p = tid; p < parts; p += NT) r.join(load_of_all(st + 3 * p), load_of_all(st + 3 * p + 1), load_of_all(st + 3 * p + 2), c);
  if (a.k > 0) {
#pragma unroll
    for (int g = 0; g < GROUPS / NT; ++g) {              // (entry i belongs to group i mod GROUPS)
      uint32_t m = 0u;
#pragma unroll
      for (int q = g; q < kKept; q += GROUPS / NT) m = max(m, entry_key(kept[q]));
      for (int i = tid + g * NT + (kKept + GROUPS / NT - 1) / (GROUPS / NT) * GROUPS; i < n_all; i += GROUPS) m = max(m, entry_key(load_of_all(list + i)));
      top.group[g * NT + tid] = m;
    }
  }
  r = block_join<NT>(r, false, c, s_w);
  const RowEnd end(r, a.temperature);
  if (tid == 0) {
    if (a.logprob) a.logprob[row] = end.log_q(z_token);
    if (a.entropy) a.entropy[row] = end.entropy;
  }
  if (a.k == 0) return;
  const uint32_t bound = find_bound(top, a.k);
  auto look = [&](uint64_t e) { if (entry_key(e) >= bound) append(top, entry_key(e), entry_index(e)); };
#pragma unroll
  for (int q = 0; q < kKept; ++q) look(kept[q]);
  for (int i = tid + kKept * NT; i < n_all; i += NT) look(load_of_all(list + i));
  __syncthreads();
  int n = top.n;
  __syncthreads();
  if (n > cand_max<NT>()) {
    select_exact(top, [&](int64_t i) { return load_of_all(list + i); }, n_all, a.k);       // (parts lie in the order of their classes)
    n = a.k;
  }
  place_entries(top, n, a.k, [&](int at, uint64_t e) { put_top(a.top_index, a.top_logprob, (int64_t)row * a.k + at, e, end); });
}

// SPLIT: the row's vectors are dealt to gridDim.x workgroups, part_vecs each; the last one to be done joins what all have left
// ONE: kAhead vectors a thread are all, and stay in registers; PAST: rows are read past the caches
template <typename T, int NT, bool SPLIT, bool ONE, bool PAST>
__global__ __launch_bounds__(NT) void logprob_rows_kernel(LogprobRows a, int part_vecs) {
  typedef Stream<T> S;
  constexpr int VPL = S::VPL, G = groups_of<NT>();
  __shared__ float3 s_w[NT / 64];
  __shared__ TopLds<NT, NT * G> top;
  __shared__ float s_most[ONE ? 1 : kSlots][ONE ? 1 : NT];         // of a thread's kAhead vectors at a time, in turn
  __shared__ bool s_last;
  const int row = SPLIT ? blockIdx.y : blockIdx.x + blockIdx.y * kRowsX;
  if (row >= a.rows) return;
  const int part = SPLIT ? blockIdx.x : 0, classes = a.classes, tid = threadIdx.x;
  if (!token_counts(a.token, row, classes)) {
    if (part == 0) leave_row<NT>(a.logprob, a.entropy, a.k, a.top_index, a.top_logprob, row);
    return;
  }
  const T* const z = static_cast<const T*>(a.z) + (int64_t)row * classes;
  const float c = kLog2e / a.temperature;
  const int head = min(classes, RowPart<T, 64, 1>::head(z)), whole = (classes - head) / VPL;      // whole vectors from `head` on
  const int v_lo = SPLIT ? min(part * part_vecs, whole) : 0, v_hi = SPLIT ? min(v_lo + part_vecs, whole) : whole;
  const bool first = part == 0, last = !SPLIT || part == (int)gridDim.x - 1;
  const T* const zv = z + head;
  // the elements before the first vector and behind the last one: one of each to a thread
  int single_col = -1;
  if (first && tid < head) single_col = tid;
  else if (last && tid >= VPL && tid < 2 * VPL && head + whole * VPL + tid - VPL < classes) single_col = head + whole * VPL + tid - VPL;
  float z_token = 0.f;
  if (a.logprob && tid == 0) z_token = ld_elem(z + a.token[row]);
  const float single = single_col >= 0 ? ld_elem(z + single_col) : -INFINITY;

  float g[G];
#pragma unroll
  for (int q = 0; q < G; ++q) g[q] = -INFINITY;
  g[0] = single;
  const float lowest = -kFar / c;
  float m = fmaxf(single, lowest), mc = rounded_product(m, c);
  const float l0 = fmaf(single, c, -mc), e0 = __builtin_amdgcn_exp2f(l0);
  float s = e0, u = e0 * fmaxf(l0, kNoPower);
  u32x4 raw[kAhead];
  auto load = [&](int v0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      raw[i] = u32x4{S::kEmpty, S::kEmpty, S::kEmpty, S::kEmpty};
      if (v0 + i * NT < v_hi) {
        const u32x4* const from = reinterpret_cast<const u32x4*>(zv + (int64_t)(v0 + i * NT) * VPL);
        if constexpr (PAST) raw[i] = __builtin_nontemporal_load(from); else raw[i] = *from;
      }
    }
  };
  const bool list = a.k > 1;                             // (the first place alone takes no search)
  top.begin();
  int turn = 0;
  for (int v0 = v_lo + tid; ONE ? v0 == v_lo + tid : v0 < v_hi; v0 += NT * kAhead) {
    load(v0);
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float mi = S::most(raw[i]);
      g[i % G] = fmaxf(g[i % G], mi);
      most = fmaxf(most, mi);
    }
    if (!ONE && a.k > 0) {
      float* const slot = &s_most[turn % kSlots][tid];
      *slot = turn < kSlots ? most : fmaxf(*slot, most);
      ++turn;
    }
    if (most > m) {
      const float mc2 = rounded_product(most, c), d = mc - mc2, f = __builtin_amdgcn_exp2f(d);
      u = f * (u + s * fmaxf(d, kNoPower));
      s *= f;
      m = most; mc = mc2;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
#pragma unroll
      for (int q = 0; q < VPL; ++q) {
        const float l = fmaf(S::at(raw[i], q), c, -mc), e = __builtin_amdgcn_exp2f(l);
        s += e; u = fmaf(e, fmaxf(l, kNoPower), u);
      }
      asm volatile("" : "+v"(s), "+v"(u));              // (both sums move on: the exponents of one are not kept for the other)
    }
  }
  RowStats r;
  {
    const float moved = fmaf(m, c, -mc), f = __builtin_amdgcn_exp2f(-moved);
    r.m = m; r.s = f * s; r.u = f * (u - moved * s);
  }
  float most = g[0];
#pragma unroll
  for (int q = 1; q < G; ++q) most = fmaxf(most, g[q]);
  if (list) {
#pragma unroll
    for (int q = 0; q < G; ++q) top.group[q * NT + tid] = order_key(g[q]);
  }
  r = block_join<NT>(r, false, c, s_w);
  if (NT == 64) __syncthreads();                        // (a larger workgroup has had one)
  const int c_lo = first ? 0 : head + v_lo * VPL, c_hi = last ? classes : head + v_hi * VPL;
  if (!plain_stats(r, lowest, c)) r = slow_stats<T, NT>(z, c_lo, c_hi, c, s_w);
  const RowEnd end(r, a.temperature);
  if (tid == 0) {
    if (SPLIT) {
      float* const st = static_cast<float*>(a.ws) + ((int64_t)row * gridDim.x + part) * 3;
      store_for_all(st, r.m); store_for_all(st + 1, r.s); store_for_all(st + 2, r.u);
    } else {
      if (a.logprob) a.logprob[row] = end.log_q(z_token);
      if (a.entropy) a.entropy[row] = end.entropy;
    }
  }
  if (a.k > 0) {
    const float least = list ? key_value(find_bound(top, a.k)) : fmaxf(r.m, key_value(kLowestKey));
    auto look = [&](const u32x4& v, int col) {
      if (S::most(v) < least) return;
      uint32_t hits = 0u;
#pragma unroll
      for (int q = 0; q < VPL; ++q) hits |= S::at(v, q) >= least ? 1u << q : 0u;
      while (hits) {                                     // (nearly always one)
        const int q = __ffs(hits) - 1, w = sizeof(T) == 2 ? q >> 1 : q;
        const uint32_t word = w == 0 ? v[0] : w == 1 ? v[1] : w == 2 ? v[2] : v[3];
        append(top, order_key(__uint_as_float(sizeof(T) == 4 ? word : q & 1 ? word & 0xFFFF0000u : word << 16)), col + q);
        hits &= hits - 1u;
      }
    };
    if (single >= least) append(top, order_key(single), single_col);
    if constexpr (ONE) {
      if (most >= least) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) look(raw[i], head + (v_lo + tid + i * NT) * VPL);
      }
    } else {
      // Slots that hold such an element, by four lanes each: a lane has a vector.
      if (most >= least)
        for (int q = 0; q < min(turn, kSlots); ++q)
          if (s_most[q][tid] >= least) {
            const int at = atomicAdd(&top.strips, 1);
            if (at < kStrips) top.strip[at] = (uint16_t)(q * NT + tid);
          }
      __syncthreads();
      const int strips = min(top.strips, kStrips);
      for (int t = tid / kAhead; t < strips; t += NT / kAhead) {
        const int q = top.strip[t];
        for (int v = v_lo + q % NT + (q / NT * kAhead + tid % kAhead) * NT; v < v_hi; v += kSlots * kAhead * NT)
          look(*reinterpret_cast<const u32x4*>(zv + (int64_t)v * VPL), head + v * VPL);
      }
      if (tid == 0 && top.strips > kStrips) atomicAdd(&top.n, cand_max<NT>() + 1);    // (too many: as if all were there)
    }
    __syncthreads();
    int n = top.n;
    __syncthreads();
    if (n > cand_max<NT>()) {
      select_exact(top, [&](int64_t i) { return make_entry(order_key(ld_elem(z + c_lo + i)), c_lo + (int)i); }, c_hi - c_lo, a.k);
      n = a.k;
    }
    if constexpr (SPLIT) {
      uint64_t* const list = reinterpret_cast<uint64_t*>(static_cast<char*>(a.ws) + logprob_stats_bytes(a.rows, (int)gridDim.x)) +
                             ((int64_t)row * gridDim.x + part) * a.k;
      place_entries(top, n, a.k, [&](int at, uint64_t e) { store_for_all(list + at, e); });
    } else {
      place_entries(top, n, a.k, [&](int at, uint64_t e) { put_top(a.top_index, a.top_logprob, (int64_t)row * a.k + at, e, end); });
    }
  }
  if constexpr (SPLIT) {
    stores_done();
    __syncthreads();
    if (tid == 0) s_last = count_done(a.done + row) == gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    if (tid == 0) a.done[row] = 0u;
    join_parts(a, row, (int)gridDim.x, z_token, top, s_w);
  }
}

// Backward: a row stays in registers between its sums and its gradient, from one maximum m, with l = z c - m c in one operation as
// above; where m lies too far from zero for that, from memory element by element.  Bound by memory, with the vector units at work for most of that time
// (exponentials are taken twice): bf16 4096 x 32000 95 us (5.5 TB/s read and written), fp32 333 x 50257 24.5-26.7 (5.1-5.5).  SPLIT: PASS 0 leaves the parts' statistics, PASS 1
// joins them (each workgroup for itself) and writes.
template <int NT> __device__ __forceinline__ float block_max(float m, float3* s_w) {
  m = lanes_max(m);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6].x = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, s_w[w].x);
  }
  __syncthreads();
  return m;
}
// sums of what threads have from one maximum
template <int NT> __device__ __forceinline__ RowStats block_sums(float m, float s, float u, float3* s_w) {
  RowStats r;
  r.m = m; r.s = lanes_sum(s); r.u = lanes_sum(u);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = make_float3(0.f, r.s, r.u);
    __syncthreads();
    r.s = r.u = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) { r.s += s_w[w].y; r.u += s_w[w].z; }
  }
  return r;
}
template <int NT> __device__ __forceinline__ RowStats joined_parts(const float* st, float c, float3* s_w) {
  RowStats r;
  for (int q = threadIdx.x; q < (int)gridDim.x; q += NT) r.join(st[3 * q], st[3 * q + 1], st[3 * q + 2], c);
  return block_join<NT>(r, false, c, s_w);
}
__device__ __forceinline__ void put_part(float* st, const RowStats& r) {
  float* const mine = st + blockIdx.x * 3;
  mine[0] = r.m; mine[1] = r.s; mine[2] = r.u;
}
// what multiplies a row's exponentials (factor + slope l), and what its token's element has besides
struct RowGrad {
  float slope, factor, token;
  __device__ __forceinline__ RowGrad(float ga, float gh, const RowStats& r) {
    token = ga;
    slope = -(gh * kLn2) / r.s;
    factor = (gh * kLn2 * (r.u / r.s) - token) / r.s;
  }
  __device__ __forceinline__ float operator()(float l) const { return __builtin_amdgcn_exp2f(l) * fmaf(fmaxf(l, kNoPower), slope, factor); }
};

template <typename T, int NT, bool SPLIT, int PASS>
__device__ __forceinline__ void slow_gradient(const T* z, T* dz, float* st, int lo, int hi, float c, float ga, float gh, float m, int token,
                                           float token_logit, float3* s_w) {
  const float b = exp_base(m);
  RowStats r;
  if constexpr (SPLIT && PASS == 1) r = joined_parts<NT>(st, c, s_w);
  else {
    float s = 0.f, u = 0.f;
    for (int v = lo + (int)threadIdx.x; v < hi; v += NT) {
      const float l = (ld_elem(z + v) - b) * c, e = __builtin_amdgcn_exp2f(l);
      s += e; u += e * fmaxf(l, kNoPower);
    }
    r = block_sums<NT>(m, s, u, s_w);
  }
  if constexpr (SPLIT && PASS == 0) { if (threadIdx.x == 0) put_part(st, r); return; }
  const RowGrad grad(ga, gh, r);
  for (int v = lo + (int)threadIdx.x; v < hi; v += NT)
    if (v != token) st_elem(dz + v, grad((ld_elem(z + v) - b) * c));
  if (token >= 0 && threadIdx.x == 0) st_elem(dz + token, grad((token_logit - b) * c) + grad.token);
}

// PAST: stored past the caches.  NL: vectors of a thread that wait in LDS beside the NV in its registers, so that two rows of up to 13248
// vectors share a CU and one row's loads pass while the other is summed (kLdsLess fewer than there is room for leave its LDS a little for
// the rest).  us with 16 vectors in registers, one row a CU / with 8 and 5: fp32 333 x 50257 30.5 / 24.5, 1300 x 50257 132 / 115, bf16
// 1300 x 100000 154 / 117, 150 x 50257 fp32 16.1 / 15.6.
constexpr int kLdsLess = 64;
static __device__ __align__(16) const uint32_t kEmpty16[4] = {0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u};     // -infinity
static __device__ __align__(16) const uint32_t kEmpty32[4] = {0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
template <typename T, int NT, int NV, int NL, bool SPLIT, int PASS, bool PAST>
__global__ __launch_bounds__(NT, NL > 0 ? 8 : 1) void logprob_grad_kernel(LogprobRows a) {
  typedef RowPart<T, NT, NV> Part;
  typedef Stream<T> S;
  static_assert(NL == 0 || !SPLIT, "whole rows");
  constexpr int VPL = Part::VPL, kVecs = NT * (NV + NL);
  constexpr int kLds = NL > 0 ? NL * NT - kLdsLess : 1;
  __shared__ u32x4 s_row[kLds];
  __shared__ float3 s_w[NT / 64];
  __shared__ float s_token;
  const int row = SPLIT ? blockIdx.y + blockIdx.z * 65535 : blockIdx.x + blockIdx.y * kRowsX;
  if (row >= a.rows) return;
  const int part = SPLIT ? blockIdx.x : 0, v0 = part * kVecs, classes = a.classes, tid = threadIdx.x;
  const T* const z = static_cast<const T*>(a.z) + (int64_t)row * classes;
  T* const dz = static_cast<T*>(a.dz) + (int64_t)row * classes;
  const int head = Part::head(z), c_lo = part == 0 ? 0 : head + v0 * VPL, c_hi = min(classes, head + (v0 + kVecs) * VPL);
  if (!token_counts(a.token, row, classes)) {
    if (!(SPLIT && PASS == 0)) for (int q = c_lo + tid; q < c_hi; q += NT) st_elem(dz + q, 0.f);
    return;
  }
  const float c = kLog2e / a.temperature, inv_t = 1.f / a.temperature;
  float* const st = SPLIT ? static_cast<float*>(a.ws) + (int64_t)row * gridDim.x * 3 : nullptr;
  Part p;
  p.template load<PAST>(z, v0, head, classes);
  auto lds_col = [&](int i) { return Part::col(NV * NT, i, head); };
  auto lds_vec = [&](int i) {                            // (each thread's own: no barriers)
    const u32x4 none = {S::kEmpty, S::kEmpty, S::kEmpty, S::kEmpty};
    return (i + 1) * NT <= kLds || i * NT + tid < kLds ? s_row[i * NT + tid] : none;
  };
  if constexpr (NL > 0) {
    // (from memory into LDS, past the registers: lane l's 16 bytes go to a wave's 1 KB at 16 l)
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) * 64;
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if ((i + 1) * NT <= kLds || i * NT + wave + 64 <= kLds) {
        const T* const from = lds_col(i) + VPL <= classes ? z + lds_col(i) : reinterpret_cast<const T*>(sizeof(T) == 2 ? kEmpty16 : kEmpty32);
        __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) const uint32_t*)from,
                                         (__attribute__((address_space(3))) uint32_t*)&s_row[i * NT + wave], 16, 0, 0);
      }
    const int tail = head + max(0, classes - head) / VPL * VPL + tid - VPL;    // (the elements behind the last vector, if Part has left them)
    if (tid >= VPL && tid < 2 * VPL && p.single_col < 0 && tail < classes && tail >= head + NT * NV * VPL) {
      p.single_col = tail;
      p.single = ld_elem(z + tail);
    }
  }
  const float ga = a.d_logprob ? a.d_logprob[row] * inv_t : 0.f, gh = a.d_entropy ? a.d_entropy[row] * inv_t : 0.f;
  int token = a.d_logprob ? a.token[row] : -1;
  if (token < c_lo || token >= c_hi) token = -1;
  if (token >= 0 && tid == 0) s_token = ld_elem(z + token);    // (a barrier ahead of any store: dz may be z)
  float m = p.single;
  if constexpr (SPLIT && PASS == 1) {
    for (int q = tid; q < (int)gridDim.x; q += NT) m = fmaxf(m, st[3 * q]);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int q = 0; q < VPL; ++q) m = fmaxf(m, p.at(i, q));
      if (i % 2) __builtin_amdgcn_sched_barrier(0);
    }
    p.forget();
    if constexpr (NL > 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // (what went into LDS has arrived)
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      m = fmaxf(m, S::most(lds_vec(i)));
      asm volatile("" : "+v"(m) :: "memory");            // (a vector of them in registers at a time)
    }
  }
  m = block_max<NT>(m, s_w);
  const float mc = rounded_product(m, c), moved = fmaf(m, c, -mc);
  if (!(fabsf(mc) <= kFar)) {
    slow_gradient<T, NT, SPLIT, PASS>(z, dz, st, c_lo, c_hi, c, ga, gh, m, token, s_token, s_w);
    return;
  }
  RowStats r;
  if constexpr (SPLIT && PASS == 1) {
    r = joined_parts<NT>(st, c, s_w);
    const float f = __builtin_amdgcn_exp2f(moved);       // (from m to the base)
    r.u = f * (r.u + moved * r.s); r.s *= f;
  } else {
    const float l0 = fmaf(p.single, c, -mc), e0 = __builtin_amdgcn_exp2f(l0);
    float s = e0, u = e0 * fmaxf(l0, kNoPower);
    auto add = [&](float v) {
      const float l = fmaf(v, c, -mc), e = __builtin_amdgcn_exp2f(l);
      s += e; u = fmaf(e, fmaxf(l, kNoPower), u);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int q = 0; q < VPL; ++q) add(p.at(i, q));
      asm volatile("" : "+v"(s), "+v"(u));              // (both sums move on: the exponents of one are not kept for the other)
    }
    p.forget();
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const u32x4 v = lds_vec(i);
#pragma unroll
      for (int q = 0; q < VPL; ++q) add(S::at(v, q));
      asm volatile("" : "+v"(s), "+v"(u));
    }
    r = block_sums<NT>(m, s, u, s_w);
    if constexpr (SPLIT) {
      const float f = __builtin_amdgcn_exp2f(-moved);
      r.u = f * (r.u - moved * r.s); r.s *= f;
      if (tid == 0) put_part(st, r);
      return;
    }
  }
  const RowGrad grad(ga, gh, r);
  const float single = grad(fmaf(p.single, c, -mc));
  store_part<T, NT, NV, PAST>(dz, p, v0, head, classes, single, [&](int i, int q) { return grad(fmaf(p.at(i, q), c, -mc)); });
#pragma unroll
  for (int i = 0; i < NL; ++i)
    if (lds_col(i) + VPL <= classes) {
      const u32x4 v = lds_vec(i);
      store_vector<T, PAST>(dz + lds_col(i), [&](int q) { return grad(fmaf(S::at(v, q), c, -mc)); });
    }
  __threadfence_block();
  __syncthreads();                                      // the token's element is written again, after its vector
  if (token >= 0 && tid == 0) st_elem(dz + token, grad(fmaf(s_token, c, -mc)) + grad.token);
}

// ------------------------------------------------------------------ after a layer's product
constexpr int kJoinThreads = 512;
// A chain of loads, a bound and a list: bf16 1 x 128000 (2000 parts) with lists of 20 6.2 us, 300 x 32000 with lists of 5 9.2.
// A workgroup a place: its parts' statistics joined, and of its logits (in fp32) those of the parts that may hold a listed one; where the
// parts are too few for a tight bound, all of them twice.
__global__ __launch_bounds__(kJoinThreads) void logprob_finish_kernel(LogprobFinish a) {
  constexpr int NT = kJoinThreads, kKept = 4;            // parts of a thread that wait in registers
  __shared__ float3 s_w[NT / 64];
  __shared__ TopLds<NT, NT> top;
  const int place = blockIdx.x, tid = threadIdx.x;
  const int row = a.list[place], live = *a.live;
  auto stats_of = [&](int p) { return *reinterpret_cast<const float2*>(a.stats + ((int64_t)p * a.stats_ld + place) * 2); };
  auto spread_of = [&](int p) { return a.spread[(int64_t)p * a.stats_ld + place]; };
  float2 ms[kKept];
  float u[kKept];
#pragma unroll
  for (int q = 0; q < kKept; ++q) {                      // (all on their way at once, whether the place counts or not)
    const int p = tid + q * NT;
    ms[q] = p < a.parts ? stats_of(p) : make_float2(-INFINITY, 0.f);
    u[q] = p < a.parts ? spread_of(p) : 0.f;
  }
  const float target = a.logprob && tid == 0 ? a.target[place] : 0.f;
  if (place >= live) {
    leave_row<NT>(a.logprob, a.entropy, a.k, a.top_index, a.top_logprob, row);
    return;
  }
  top.begin();
  const float c = kLog2e / a.temperature;
  const float* const z = a.z + (int64_t)place * a.z_ld;
  const bool list = a.k > 1, by_part = a.parts >= 2 * a.k;
  const int vecs = (a.classes + 3) / 4;                  // (rows are whole 256-byte pieces, -infinity behind the classes)
  auto vec = [&](int v) { return *reinterpret_cast<const u32x4*>(z + 4 * (int64_t)v); };
  RowStats r;
#pragma unroll
  for (int q = 0; q < kKept; ++q) r.m = fmaxf(r.m, ms[q].x);
  for (int p = tid + kKept * NT; p < a.parts; p += NT) r.m = fmaxf(r.m, stats_of(p).x);
  const float mine = r.m;
#pragma unroll
  for (int q = 0; q < kKept; ++q) {
    RowStats o;
    o.m = ms[q].x; o.s = ms[q].y; o.u = u[q];
    o.rebase(mine, c);
    r.s += o.s; r.u += o.u;
  }
  for (int p = tid + kKept * NT; p < a.parts; p += NT) r.join(stats_of(p).x, stats_of(p).y, spread_of(p), c);
  float most = mine;
  if (a.k > 0) {
    if (!by_part) {
      most = -INFINITY;
#pragma unroll 4
      for (int v = tid; v < vecs; v += NT) most = fmaxf(most, Stream<float>::most(vec(v)));
    }
    if (list) top.group[tid] = order_key(most);
  }
  r = block_join<NT>(r, false, c, s_w);
  const RowEnd end(r, a.temperature);
  if (tid == 0) {
    if (a.logprob) a.logprob[row] = end.log_q(target);
    if (a.entropy) a.entropy[row] = end.entropy;
  }
  if (a.k == 0) return;
  const float least = list ? key_value(find_bound(top, a.k)) : fmaxf(r.m, key_value(kLowestKey));
  auto look = [&](int v) {
    const u32x4 w = vec(v);
    if (Stream<float>::most(w) < least) return;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (__uint_as_float(w[q]) >= least && 4 * v + q < a.classes) append(top, order_key(__uint_as_float(w[q])), 4 * v + q);
  };
  if (by_part) {
    auto note = [&](float m, int p) {
      if (!(m >= least)) return;
      const int at = atomicAdd(&top.strips, 1);
      if (at < kStrips) top.strip[at] = (uint16_t)p;
    };
    if (most >= least) {
#pragma unroll
      for (int q = 0; q < kKept; ++q) note(ms[q].x, tid + q * NT);
      for (int p = tid + kKept * NT; p < a.parts; p += NT) note(stats_of(p).x, p);
    }
    __syncthreads();
    const int strips = min(top.strips, kStrips), lanes = a.part / 4;      // 16 or 32 for a part
    for (int t = tid / lanes; t < strips; t += NT / lanes) {
      const int v = (int)top.strip[t] * lanes + tid % lanes;
      if (v < vecs) look(v);
    }
    if (tid == 0 && top.strips > kStrips) atomicAdd(&top.n, cand_max<NT>() + 1);        // (too many: as if all were there)
  } else if (most >= least) {
#pragma unroll 4
    for (int v = tid; v < vecs; v += NT) look(v);
  }
  __syncthreads();
  int n = top.n;
  __syncthreads();
  if (n > cand_max<NT>()) {
    select_exact(top, [&](int64_t i) { return make_entry(order_key(z[i]), (int)i); }, a.classes, a.k);
    n = a.k;
  }
  place_entries(top, n, a.k, [&](int at, uint64_t e) { put_top(a.top_index, a.top_logprob, (int64_t)row * a.k + at, e, end); });
}

// ------------------------------------------------------------------ launches
template <typename T> int64_t row_vectors(int classes) { return (int64_t)classes / (16 / (int)sizeof(T)) + 1; }   // (one for the single elements at the end)

// Logits and gradients that the last-level cache (256 MB) cannot hold beside anything else go past the caches, others stay there for whoever
// reads them next.  us through / past: forward bf16 4096 x 32000 (262 MB) with lists of 5 55.0 / 51.1, 2000 x 50257 (201) 46 / 43, fp32 3000 x
// 50257 108 / 100, but 777 x 50257 (156, a third of the rows left out) 28.3 / 29.4; backward, stores alone, bf16 4096 x 32000 109 / 101, 2000 x
// 50257 100 / 92, but 8192 x 8000 (131) 47 / 49, fp32 600 x 50257 (121) 61 / 64, and loads too 101 / 97, fp32 2000 x 32000 98.7 / 94.4.
constexpr int64_t kPastBytes = 160 << 20;
template <typename T> bool past_caches(const LogprobRows& a) { return (int64_t)a.rows * a.classes * (int)sizeof(T) >= kPastBytes; }

// forward: workgroups that a row is dealt to.  A few of the longest rows, longer ones where lists are long (every part makes one).  us of the kernel in
// one / in parts: bf16 without lists 1 x 50257 7.4 / 6.2, 128 x 128000 13.5 / 11.4, but 64 x 20000 5.6 / 6.5, 256 x 128000 15.0 / 17.0; lists of 20 1 x
// 100000 13.0 / 11.7, 128 x 200000 24.7 / 21.4, but 64 x 20000 8.9 / 11.6, 1 x 50257 11.0 / 11.8, 256 x 200000 26.0 / 30.4; lists of 200 64 x 128000
// 24.4 / 35.6; fp32, of whose vectors each holds half as many, lists of 20 64 x 50257 11.6 / 13.6.
template <typename T> int forward_parts(const LogprobRows& a) {
  const int64_t vecs = row_vectors<T>(a.classes);
  if (a.rows > kLogprobSplitRows || vecs <= (a.k == 0 ? 4096 : a.k > 32 ? 65536 : sizeof(T) == 2 ? 12000 : 14000)) return 1;
  return (int)std::min<int64_t>(std::max<int64_t>(1, 512 / a.rows), (vecs + 256 * kAhead - 1) / (256 * kAhead));
}
template <typename T, int NT> hipError_t forward_whole(const LogprobRows& a, hipStream_t st) {
  const dim3 grid(a.rows < kRowsX ? a.rows : kRowsX, (a.rows + kRowsX - 1) / kRowsX);
  auto kern = row_vectors<T>(a.classes) <= NT * kAhead
                  ? past_caches<T>(a) ? logprob_rows_kernel<T, NT, false, true, true> : logprob_rows_kernel<T, NT, false, true, false>
                  : past_caches<T>(a) ? logprob_rows_kernel<T, NT, false, false, true> : logprob_rows_kernel<T, NT, false, false, false>;
  hipLaunchKernelGGL(kern, grid, dim3(NT), 0, st, a, 0);
  return hipGetLastError();
}
template <typename T> hipError_t forward(const LogprobRows& a, hipStream_t st) {
  const int64_t vecs = row_vectors<T>(a.classes);
  const int parts = forward_parts<T>(a);
  if (parts > 1) {
    const int part_vecs = (int)((vecs + parts - 1) / parts);
    auto kern = part_vecs <= 256 * kAhead ? logprob_rows_kernel<T, 256, true, true, false> : logprob_rows_kernel<T, 256, true, false, false>;
    hipLaunchKernelGGL(kern, dim3(parts, a.rows), dim3(256), 0, st, a, part_vecs);
    return hipGetLastError();
  }
  // Many rows of middling width: what a row takes besides its logits is least in one wave, or two.  us with 256 threads (128 up to 1024 vectors) /
  // by this rule: bf16, lists of 5, 4096 x 6000 19.5 / 15.5, 4096 x 10000 28.0 / 20.4, 16384 x 10000 94 / 68, 1200 x 10000 13.6 / 12.7, 16384 x 16000
  // 104 / 99, 2048 x 16000 18.7 / 17.5, fp32 4096 x 5000 23.3 / 19.0; but in one wave 1200 x 20000 17.4 / 20.7, 600 x 16000 12.8 / 13.5, and lists of
  // 64 of 1200 x 10000 16.0 / 20.1.
  if (a.k <= 32 && a.rows >= 1024) {
    if (vecs <= 64 * 20 || (a.rows >= 4096 && vecs <= 64 * 40)) return forward_whole<T, 64>(a, st);
    if (vecs <= 128 * 20) return forward_whole<T, 128>(a, st);
  }
  if (vecs <= 64 * kAhead && a.k <= 128) return forward_whole<T, 64>(a, st);
  if (vecs <= 2 * 128 * kAhead) return forward_whole<T, 128>(a, st);
  if (vecs <= 32 * 256) return forward_whole<T, 256>(a, st);
  return forward_whole<T, 512>(a, st);
}

template <typename T, int NT, int NV, int NL = 0> hipError_t backward_whole(const LogprobRows& a, hipStream_t st) {
  const dim3 grid(a.rows < kRowsX ? a.rows : kRowsX, (a.rows + kRowsX - 1) / kRowsX);
  auto kern = past_caches<T>(a) ? logprob_grad_kernel<T, NT, NV, NL, false, 1, true> : logprob_grad_kernel<T, NT, NV, NL, false, 1, false>;
  hipLaunchKernelGGL(kern, grid, dim3(NT), 0, st, a);
  return hipGetLastError();
}
// Few of the longest rows go in parts too, which takes a launch and a second read but gives each row more than a CU.  us whole / in parts:
// bf16 1 x 128000 19.6 / 11.0, 64 x 128000 24.9 / 14.8, 128 x 128000 26.0 / 22.9, 256 x 128000 29.4 / 38.9; fp32 64 x 50257 14.9 / 12.0, 128 x 50257
// 15.9 / 16.3; shorter ones bf16 64 x 50257 12.1 / 11.1, but fp32 64 x 20000 8.1 / 10.9.
template <typename T> int backward_parts(const LogprobRows& a) {
  const int64_t vecs = row_vectors<T>(a.classes);
  if (!(vecs > 1024 * 16 || (vecs > 512 * 16 && a.rows <= 128))) return 1;
  return (int)((vecs + kPartThreads * kPartVecs - 1) / (kPartThreads * kPartVecs));
}
template <typename T> hipError_t backward(const LogprobRows& a, hipStream_t st) {
  const int64_t vecs = row_vectors<T>(a.classes);
  const int parts = backward_parts<T>(a);
  if (parts > 1) {
    const dim3 grid((unsigned)parts, (unsigned)(a.rows < 65535 ? a.rows : 65535), (unsigned)((a.rows + 65534) / 65535));
    hipLaunchKernelGGL((logprob_grad_kernel<T, kPartThreads, kPartVecs, 0, true, 0, false>), grid, dim3(kPartThreads), 0, st, a);
    hipLaunchKernelGGL((logprob_grad_kernel<T, kPartThreads, kPartVecs, 0, true, 1, false>), grid, dim3(kPartThreads), 0, st, a);
    return hipGetLastError();
  }
  if (vecs <= 64 * 4) return backward_whole<T, 64, 4>(a, st);
  if (vecs <= 128 * 4) return backward_whole<T, 128, 4>(a, st);
  if (vecs <= 256 * 4) return backward_whole<T, 256, 4>(a, st);
  if (vecs <= 256 * 8) return backward_whole<T, 256, 8>(a, st);
  if (vecs <= 512 * 8) return backward_whole<T, 512, 8>(a, st);
  // (us with 512 x 16 / 1024 x 8: bf16 1300 x 50257 67 / 62, 333 x 50257 22.8 / 23.5; fp32 150 x 32000 13.2 / 11.6, 333 x 32000 17.8 / 18.3)
  if (vecs <= 1024 * 8) return backward_whole<T, 1024, 8>(a, st);
  if (vecs <= 1024 * 13 - kLdsLess) return backward_whole<T, 1024, 8, 5>(a, st);
  return backward_whole<T, 1024, 16>(a, st);
}

template <typename T> size_t rows_bytes(const LogprobRows& a) {
  const int parts = a.dz ? backward_parts<T>(a) : forward_parts<T>(a);
  if (parts <= 1) return 0;
  return logprob_stats_bytes(a.rows, parts) + (a.dz ? 0 : (size_t)a.rows * parts * a.k * 8);
}

}  // namespace

size_t logprob_rows_bytes(const LogprobRows& a) { return a.dtype == kBF16 ? rows_bytes<uint16_t>(a) : rows_bytes<float>(a); }

hipError_t launch_logprob_rows(const LogprobRows& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.k < 0 || a.k > kTopMax) return hipErrorInvalidValue;
  if (a.dz) return a.dtype == kBF16 ? backward<uint16_t>(a, st) : backward<float>(a, st);
  return a.dtype == kBF16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}

hipError_t launch_logprob_finish(const LogprobFinish& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  if (a.k < 0 || a.k > kTopMax || (a.k > 0 && !a.z)) return hipErrorInvalidValue;
  hipLaunchKernelGGL(logprob_finish_kernel, dim3((unsigned)a.rows), dim3(kJoinThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace rad
