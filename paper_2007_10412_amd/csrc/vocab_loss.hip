// Losses over a vocabulary, and their gradients, from logits that are there: softmax cross entropy and distillation from
// a teacher's most likely tokens.
//
// With q = softmax(z / T) and a list of targets (i_j, p_j), sum p_j = 1, a row's loss is T^2 sum_j p_j log(p_j / q_{i_j})
// = T^2 (sum_j p_j log p_j + lse(z / T) - sum_j p_j z_{i_j} / T), and its gradient T (q_v - sum_{j: i_j = v} p_j): dense
// in q, with k corrections.  A row is read once, 16 bytes a lane, and kept in registers between the statistics and the
// gradient; the targets' logits are read beside it, and the corrections written over the row's vectors after them.
#include <math.h>

#include <algorithm>

#include "head_epilogue.hpp"
#include "kernels.hpp"

namespace rad {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float ld_elem(const float* p) { return *p; }
__device__ __forceinline__ float ld_elem(const uint16_t* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ uint16_t to_bf16(float v) { uint16_t p[2]; put_pair(p, v, 0.f); return p[0]; }
__device__ __forceinline__ void st_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_elem(uint16_t* p, float v) { *p = to_bf16(v); }
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// sum over a workgroup of NT threads, the same for all of them; s_w: NT / 64 floats
template <int NT> __device__ __forceinline__ float block_sum(float v, float* s_w) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) t += s_w[w];
  return t;
}

// exp((v - m) / T) with c = log2(e) / T; m is finite.  (The product's rounding is an error of |v - m| c 2^-24 of the exponential, more than
// expf's: gradients of 4 x 128000 fp32 logits are off by 1.3e-7 rms, where expf with a division gives 0.8e-7.)
__device__ __forceinline__ float exp_from(float v, float m, float c) { return __builtin_amdgcn_exp2f((v - m) * c); }
// what exponentials are taken from: the maximum, or 0 where nothing is left of a row (every exponential is 0 then)
__device__ __forceinline__ float exp_base(float m) { return m == -INFINITY ? 0.f : m; }

// a part's sum of exponentials (from exp_base of its maximum m) as one from b; a part with nothing in it adds its 0, or its NaN
__device__ __forceinline__ float rebased(float s, float m, float b, float c) { return m == -INFINITY ? s : s * exp_from(m, b, c); }

__device__ __forceinline__ bool row_counts(const VocabTargets& t, int row, int classes) {
  return t.labels ? (uint32_t)t.labels[row] < (uint32_t)classes : t.counts[row] != 0;
}

// a wave's LDS writes before, its reads after (LDS serves a wave in order: only the compiler has to keep it)
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------ targets
// A wave per row.  Keys (index, place in the list) are sorted in LDS by a bitonic network over P >= k places, which puts
// entries of one index side by side; they become one of their probabilities' sum.  Missing entries sort to the end.  The chain of
// exchanges bounds it (4 lists of 128 5.7 us) until its loads do (4096 of 64 8.3).
template <int P>
__global__ __launch_bounds__(256) void teacher_kernel(const int32_t* __restrict__ index, const float* __restrict__ logit, int rows,
                                                      int k, int classes, float inv_t, int32_t* __restrict__ index_out,
                                                      float* __restrict__ prob, float* __restrict__ entropy,
                                                      int32_t* __restrict__ counts, uint16_t* __restrict__ first, int part, int parts) {
  __shared__ uint64_t s_key[4][P];
  __shared__ float s_p[4][P];
  constexpr uint64_t kNone = ~0ull;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int row = blockIdx.x * 4 + w;
  const bool live = row < rows;
  uint64_t* const key = s_key[w];
  float* const p = s_p[w];
  const int64_t at = (int64_t)(live ? row : 0) * k;
  float m = -INFINITY;
  bool bad = false;
  for (int j = lane; j < P; j += 64) {
    uint64_t kj = kNone;
    float t = -INFINITY;
    if (live && j < k) {
      const int32_t i = index[at + j];
      const float l = logit[at + j];
      if ((uint32_t)i < (uint32_t)classes && l != -INFINITY) { kj = ((uint64_t)(uint32_t)i << 32) | (uint32_t)j; t = l; }
    }
    key[j] = kj;
    p[j] = t;
    bad = bad || t != t;
    m = fmaxf(m, t);
  }
  m = wave_max(m);
  if (__any(bad)) m = NAN;
  float s = 0.f, h = 0.f;
  for (int j = lane; j < P; j += 64)
    if (key[j] != kNone) s += expf((p[j] - m) * inv_t);   // (divided by T after the maximum is off: the logits may be fp32's last)
  s = wave_sum(s);
  const float log_s = logf(s), inv_s = 1.f / s;
  for (int j = lane; j < P; j += 64) {
    float pj = 0.f;
    if (key[j] != kNone) {
      const float d = (p[j] - m) * inv_t;
      pj = expf(d) * inv_s;
      if (pj != 0.f) h += pj * (d - log_s);             // p log p -> 0
    }
    p[j] = pj;
  }
  h = wave_sum(h);
  wave_lds_fence();
  for (int size = 2; size <= P; size <<= 1)
    for (int d = size >> 1; d > 0; d >>= 1) {
      for (int q = lane; q < P / 2; q += 64) {
        const int a = (q / d) * 2 * d + q % d, b = a + d;
        const bool up = (a & size) == 0;
        const uint64_t ka = key[a], kb = key[b];
        if ((ka > kb) == up) { key[a] = kb; key[b] = ka; }
      }
      wave_lds_fence();
    }
  if (!live) return;
  const bool some = key[0] != kNone;
  // Entries of one index become one, in the first places; the places behind the last one hold none.  (64 of them at a time: an
  // entry moves to a place at or before its own, once all of the 64 are read.)
  int kept = 0;
  for (int j0 = 0; j0 < k; j0 += 64) {
    const int j = j0 + lane;
    const uint64_t kj = j < k ? key[j] : kNone;
    const bool head = kj != kNone && (j == 0 || (key[j - 1] >> 32) != (kj >> 32));
    float sum = 0.f;
    if (head)
      for (int q = j; q < k && (key[q] >> 32) == (kj >> 32) && key[q] != kNone; ++q) sum += p[(uint32_t)key[q]];
    const uint64_t heads = __ballot(head);
    const int to = kept + __popcll(heads & ((1ull << lane) - 1));
    wave_lds_fence();
    if (head) {
      key[to] = kj;
      index_out[at + to] = (int32_t)(kj >> 32);
      prob[at + to] = sum;
    }
    wave_lds_fence();
    kept += __popcll(heads);
  }
  for (int j = kept + lane; j < k; j += 64) { index_out[at + j] = -1; prob[at + j] = 0.f; }
  if (lane == 0) { entropy[row] = some ? h : 0.f; counts[row] = some ? 1 : 0; }
  if (!first) return;
  // entries before class part t (missing ones lie after all); a kernel of its own for this: 200 x 768 x 10007, k = 16 174 us, not 170
  for (int t = lane; t <= parts; t += 64) {
    int lo = 0, hi = kept;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((uint32_t)(key[mid] >> 32) < (uint32_t)t * (uint32_t)part) lo = mid + 1; else hi = mid;
    }
    first[(int64_t)row * (parts + 1) + t] = (uint16_t)lo;
  }
}

// (one workgroup, as its sum has to be there before the rows that need it: 4096 rows 4.2 us, nearly all of it the launch)
__global__ __launch_bounds__(1024) void count_rows_kernel(VocabTargets t, int rows, int classes, float* __restrict__ inv_count) {
  __shared__ int s_n[16];
  int n = 0;
  for (int r = threadIdx.x; r < rows; r += 1024) n += row_counts(t, r, classes) ? 1 : 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
  if ((threadIdx.x & 63) == 0) s_n[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x != 0) return;
  int all = 0;
  for (int w = 0; w < 16; ++w) all += s_n[w];
  *inv_count = all > 0 ? 1.f / (float)all : 0.f;
}

// thread i adds rows i, i + 1024, ...; then a fixed tree.  Without weights: the mean over the rows that count.  4096 rows 5 us.
__global__ __launch_bounds__(1024) void weighted_loss_kernel(VocabTargets t, const float* __restrict__ row_loss, int rows,
                                                             int classes, float* __restrict__ loss) {
  __shared__ float s_w[16];
  float acc = 0.f, n = 0.f;
  for (int r = threadIdx.x; r < rows; r += 1024)
    if (row_counts(t, r, classes)) { acc += (t.weight ? t.weight[r] : 1.f) * row_loss[r]; n += 1.f; }
  acc = block_sum<1024>(acc, s_w);
  n = block_sum<1024>(n, s_w);
  if (threadIdx.x == 0) *loss = t.weight ? acc : n > 0.f ? acc / n : 0.f;
}

// ------------------------------------------------------------------ dense rows
// A workgroup's part of a row: vectors v0 .. v0 + NT NV - 1 of 16 bytes, counted from the row's first 16-byte boundary (rows of
// odd widths start anywhere; 4096 x 32001 bf16 with vectors from the row's start: 132 us, of which unaligned stores are 20).
// The up to VPL - 1 elements before it, and those that the last vector lacks, are single ones, one to a thread of the first part
// and of the part that the next vector would belong to.
template <typename T, int NT, int NV> struct RowPart {
  static constexpr int VPL = 16 / (int)sizeof(T);
  // Parts of up to 64 values a lane keep their exponentials (from the wave's maximum), of which the gradient is a multiple;
  // longer ones their packed logits, and take the exponentials again.  4096 x 32000 bf16 (64 values): 105 us, 120 the other way.
  static constexpr bool kKeep = NV * VPL <= 64;
  u32x4 raw[NV];
  float e[kKeep ? NV * VPL : 1];
  float single; int single_col;                         // -1: none
  static __device__ __forceinline__ int head(const T* row) {
    return (int)((16u - ((uint32_t)reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / (int)sizeof(T);
  }
  static __device__ __forceinline__ int col(int v0, int i, int head) { return head + (v0 + i * NT + (int)threadIdx.x) * VPL; }
  static constexpr uint32_t kEmpty = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;     // -inf
  __device__ __forceinline__ void load(const T* row, int v0, int head, int classes) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col(v0, i, head);
      raw[i] = u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
      if (c + VPL <= classes) raw[i] = *reinterpret_cast<const u32x4*>(row + c);
    }
    const int whole = max(0, classes - head) / VPL, t = (int)threadIdx.x;
    single_col = -1;
    if (t < VPL) { if (v0 == 0 && t < head && t < classes) single_col = t; }
    else if (t < 2 * VPL && whole >= v0 && whole < v0 + NT * NV) {
      const int c = head + whole * VPL + t - VPL;
      if (c < classes) single_col = c;
    }
    single = single_col >= 0 ? ld_elem(row + single_col) : -INFINITY;
  }
  __device__ __forceinline__ float at(int i, int q) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[i][q]);
    else return __uint_as_float(q & 1 ? raw[i][q >> 1] & 0xFFFF0000u : raw[i][q >> 1] << 16);
  }
  // The compiler forgets what it has unpacked of the vectors: each pass over them unpacks again (an instruction a value),
  // where it would otherwise keep two registers for every packed one.
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(raw[i][0]), "+v"(raw[i][1]), "+v"(raw[i][2]), "+v"(raw[i][3]));
  }
  // maximum and sum of exponentials of the whole wave
  __device__ __forceinline__ void stats(float c, float* m_out, float* s_out) {
    float m = single;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int q = 0; q < VPL; ++q) m = fmaxf(m, at(i, q));
      if (i % 2) __builtin_amdgcn_sched_barrier(0);     // (the vectors stay packed: few of their values at a time)
    }
    m = wave_max(m);
    if (sizeof(T) == 2 && !kKeep) forget();
    const float b = exp_base(m);
    float s = exp_from(single, b, c);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int q = 0; q < VPL; ++q) {
        const float v = exp_from(at(i, q), b, c);
        if (kKeep) e[kKeep ? i * VPL + q : 0] = v;
        s += v;
      }
      if (i % 2) __builtin_amdgcn_sched_barrier(0);
    }
    *m_out = m;
    *s_out = wave_sum(s);
  }
};

// stores a part of a row: f(i, q) is element q of vector i, single what the single element becomes
template <typename T, int NT, int NV, class F>
__device__ __forceinline__ void store_part(T* out, const RowPart<T, NT, NV>& p, int v0, int head, int classes, float single, F f) {
  constexpr int VPL = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = RowPart<T, NT, NV>::col(v0, i, head);
    if (c + VPL <= classes) {
      u32x4 w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (sizeof(T) == 4) w[q] = __float_as_uint(f(i, q));
        else w[q] = bf16_pair(f(i, 2 * q), f(i, 2 * q + 1));
      }
      __builtin_memcpy(out + c, &w, 16);                // (dz may be aligned otherwise)
    }
    if (i % 2) __builtin_amdgcn_sched_barrier(0);
  }
  if (p.single_col >= 0) st_elem(out + p.single_col, single);
}

// SPLIT: the row's parts are dealt to gridDim.x workgroups.  PASS 0 leaves each part's maximum and sum in stats
// [rows][parts][2] and, with part 0, the targets' largest logit z_0 and sum_j p_j (z_{i_j} - z_0) in dots [rows][2]; PASS 1 joins
// them, part by part in order, and writes.  Without SPLIT one workgroup has the whole row in its registers, and memory bounds it:
// 4096 x 32000 bf16 101 us (5.2 TB/s), 777 x 50257 40 (3.9; three rows a CU).  4 x 128000 fp32 takes 4 + 9 in parts.
// count: the rows that count are counted here (by every workgroup for itself).
constexpr int kRowsX = 1 << 20;                         // (a grid's x times its workgroup stays below 2^32)
template <typename T, int NT, int NV, bool SPLIT, int PASS>
__global__ __launch_bounds__(NT) void vocab_rows_kernel(VocabRows a, float* __restrict__ dots, int count) {
  typedef RowPart<T, NT, NV> Part;
  constexpr int VPL = Part::VPL, NW = NT / 64;
  __shared__ float s_m[NW], s_s[NW], s_w[NW], s_tz[kTeacherMax];
  __shared__ float3 s_t[NW];
  const int row = SPLIT ? blockIdx.y + blockIdx.z * 65535 : blockIdx.x + blockIdx.y * kRowsX;
  if (row >= a.rows) return;
  const int part = SPLIT ? blockIdx.x : 0, v0 = part * NT * NV;
  const VocabTargets& t = a.t;                          // (lists: a call with labels has a layer with it)
  const int32_t* const index = t.index + (int64_t)row * t.k;
  const float* const prob = t.prob + (int64_t)row * t.k;
  const int classes = a.classes;
  const T* const z = static_cast<const T*>(a.z) + (int64_t)row * classes;
  T* const dz = static_cast<T*>(a.dz) + (int64_t)row * classes;
  const float c = kLog2e / t.temperature;
  const bool counts = row_counts(t, row, classes);
  const int head = Part::head(z), c_lo = part == 0 ? 0 : head + v0 * VPL, c_hi = min(classes, head + (v0 + NT * NV) * VPL);

  if (!counts) {                                        // (the same for the whole workgroup)
    if (a.row_loss && part == 0 && threadIdx.x == 0 && !(SPLIT && PASS == 0)) a.row_loss[row] = 0.f;
    if (a.dz && !(SPLIT && PASS == 0))
      for (int q = c_lo + (int)threadIdx.x; q < c_hi; q += NT) st_elem(dz + q, 0.f);
    return;
  }

  Part p;
  p.load(z, v0, head, classes);
  float inv_count = 0.f;
  if (count) {
    float n = 0.f;
    for (int q = threadIdx.x; q < a.rows; q += NT) n += row_counts(t, q, classes) ? 1.f : 0.f;
    inv_count = 1.f / block_sum<NT>(n, s_w);            // (this row counts)
  }
  // The targets' logits: all of them for the loss (one part of a row), those of this part for the gradient.  They are read
  // here, ahead of any store: dz may be z.
  TargetSum sum;
  for (int j = threadIdx.x; j < t.k; j += NT) {
    const int i = index[j];
    const float pj = prob[j];
    const bool mine = i >= c_lo && i < c_hi;
    if (i < 0 || pj == 0.f || (!mine && (PASS == 1 && SPLIT ? true : part != 0))) continue;
    const float v = ld_elem(z + i);
    if (!(SPLIT && PASS == 1)) sum.add(pj, v);
    s_tz[j] = v;
  }
  if (!(SPLIT && PASS == 1) && part == 0) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum.join_lane(o);
    if ((threadIdx.x & 63) == 0) sum.put(&s_t[threadIdx.x >> 6]);
  }

  float m = -INFINITY, s = 0.f, wm = -INFINITY;
  if (!SPLIT || PASS == 0) {
    float ws;
    p.stats(c, &wm, &ws);
    if ((threadIdx.x & 63) == 0) { s_m[threadIdx.x >> 6] = wm; s_s[threadIdx.x >> 6] = ws; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, s_m[w]);
    const float b = exp_base(m);
#pragma unroll
    for (int w = 0; w < NW; ++w) s += rebased(s_s[w], s_m[w], b, c);
  }
  float z0 = 0.f, dot = 0.f;
  if (!(SPLIT && PASS == 1) && part == 0 && threadIdx.x == 0) {
    TargetSum all;
    for (int w = 0; w < NW; ++w) all.join(s_t[w]);
    z0 = all.from(); dot = all.dot;
  }
  if (SPLIT && PASS == 0) {
    if (threadIdx.x == 0) {
      float* const st = a.stats + ((int64_t)row * gridDim.x + part) * 2;
      st[0] = m; st[1] = s;
      if (part == 0) { dots[2 * row] = z0; dots[2 * row + 1] = dot; }
    }
    return;
  }
  if (SPLIT) {
    const float* const st = a.stats + (int64_t)row * gridDim.x * 2;
    for (int w = 0; w < (int)gridDim.x; ++w) m = fmaxf(m, st[2 * w]);
    const float b = exp_base(m);
    for (int w = 0; w < (int)gridDim.x; ++w) s += rebased(st[2 * w + 1], st[2 * w], b, c);
    if (part == 0) { z0 = dots[2 * row]; dot = dots[2 * row + 1]; }
    __syncthreads();                                    // every target's logit has been read
  }
  const float b = exp_base(m);
  if (a.row_loss && part == 0 && threadIdx.x == 0) {
    const float T1 = t.temperature;
    // lse - sum_j p_j z_j / T, from differences of logits (the probabilities' sum is 1)
    a.row_loss[row] = T1 * T1 * (t.entropy[row] + (logf(s) + ((b - z0) - dot) / T1));
  }
  if (!a.dz) return;
  const float weight = t.weight ? t.weight[row] : count ? inv_count : *t.inv_count;
  const float wt = weight * t.temperature, f = wt / s;
  const float single = exp_from(p.single, b, c) * f;
  if constexpr (Part::kKeep && !SPLIT) {
    const float fw = wm == -INFINITY ? f : f * exp_from(wm, b, c);
    store_part<T, NT, NV>(dz, p, v0, head, classes, single, [&](int i, int q) { return p.e[i * VPL + q] * fw; });
  } else {
    if (sizeof(T) == 2) p.forget();
    store_part<T, NT, NV>(dz, p, v0, head, classes, single, [&](int i, int q) { return exp_from(p.at(i, q), b, c) * f; });
  }
  __threadfence_block();
  __syncthreads();                                      // the targets' elements are written again, after their vectors
  for (int j = threadIdx.x; j < t.k; j += NT) {
    const int i = index[j];
    const float pj = prob[j];
    if (i >= c_lo && i < c_hi && pj != 0.f) st_elem(dz + i, exp_from(s_tz[j], b, c) * f - wt * pj);
  }
}

// out (+)= in, rounded once: 4096 x 32000 with beta = 1 187 us (5.6 TB/s)
__global__ __launch_bounds__(256) void cast_add_kernel(const float* __restrict__ in, uint16_t* __restrict__ out, int64_t n, int beta) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i + 8 <= n && (reinterpret_cast<uintptr_t>(out) & 15) == 0) {
    const floatx4 a = *reinterpret_cast<const floatx4*>(in + i), b = *reinterpret_cast<const floatx4*>(in + i + 4);
    float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    u32x4 o = {0u, 0u, 0u, 0u};
    if (beta) o = *reinterpret_cast<const u32x4*>(out + i);
    u32x4 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (beta) { v[2 * q] += __uint_as_float(o[q] << 16); v[2 * q + 1] += __uint_as_float(o[q] & 0xFFFF0000u); }
      r[q] = bf16_pair(v[2 * q], v[2 * q + 1]);
    }
    *reinterpret_cast<u32x4*>(out + i) = r;
    return;
  }
  for (int64_t j = i; j < n && j < i + 8; ++j) out[j] = to_bf16(in[j] + (beta ? bf16_bits_to_f32(out[j]) : 0.f));
}

constexpr int kPartThreads = 256, kPartVecs = 4;

template <typename T, int NT, int NV>
hipError_t rows_whole(const VocabRows& a, hipStream_t st) {
  hipLaunchKernelGGL((vocab_rows_kernel<T, NT, NV, false, 1>), dim3(std::min(a.rows, kRowsX), (a.rows + kRowsX - 1) / kRowsX), dim3(NT), 0, st, a, (float*)nullptr, vocab_rows_count(a) ? 1 : 0);
  return hipGetLastError();
}
// Long rows that are few go in parts too, which takes a launch and a second read but gives them more than a CU each.  us of a call
// with lists of 16, whole / in parts.  bf16 with gradients: 1 x 128000 24.9 / 16.4, 64 x 128000 29.4 / 22.3, 128 x 66000 26.5 / 22.8,
// 128 x 128000 33.2 / 32.5, but 200 x 128000 34.8 / 47.3; 1 x 33000 16.2 / 14.8, 64 x 33000 17.9 / 17.0, but 256 x 33000 20.4 / 22.0,
// 1 x 20000 12.0 / 14.4.  The loss alone: 1 x 128000 17.9 / 14.9, 64 x 128000 19.4 / 17.7, but 128 x 128000 22.5 / 24.8, 64 x 33000
// 15.0 / 15.1.  fp32 (half the exponentials in a vector) with gradients: 1 x 65000 16.4 / 15.4, 16 x 33000 16.1 / 16.0, but
// 64 x 33000 17.2 / 17.8, 1 x 25000 12.6 / 14.0; the loss alone 1 x 65000 12.8 / 13.8.
template <typename T> bool few_long_rows(int rows, int64_t vecs, bool gradient) {
  const bool longest = vecs > 512 * 16;                               // (they take 1024 threads a row)
  if (sizeof(T) == 4) return gradient && longest && rows <= 16;
  return longest ? rows <= (gradient ? 128 : 64) : gradient && vecs > 512 * 8 && rows <= 64;
}
template <typename T>
hipError_t rows_any(const VocabRows& a, hipStream_t st) {
  constexpr int VPL = 16 / (int)sizeof(T);
  const int64_t vecs = (int64_t)a.classes / VPL + 1;                  // (one for the single elements at the end)
  const bool whole = !few_long_rows<T>(a.rows, vecs, a.dz != nullptr);
  if (vecs <= 64 * 4) return rows_whole<T, 64, 4>(a, st);
  if (vecs <= 128 * 4) return rows_whole<T, 128, 4>(a, st);
  if (vecs <= 256 * 4) return rows_whole<T, 256, 4>(a, st);
  if (vecs <= 256 * 8) return rows_whole<T, 256, 8>(a, st);
  if (vecs <= 512 * 8) return rows_whole<T, 512, 8>(a, st);
  if (vecs <= 512 * 16 && whole) return rows_whole<T, 512, 16>(a, st);
  if (vecs <= 1024 * 16 && whole) return rows_whole<T, 1024, 16>(a, st);
  const int64_t parts = (vecs + kPartThreads * kPartVecs - 1) / (kPartThreads * kPartVecs);
  float* const dots = a.stats + (int64_t)a.rows * parts * 2;
  const dim3 grid((unsigned)parts, (unsigned)(a.rows < 65535 ? a.rows : 65535), (unsigned)((a.rows + 65534) / 65535));
  hipLaunchKernelGGL((vocab_rows_kernel<T, kPartThreads, kPartVecs, true, 0>), grid, dim3(kPartThreads), 0, st, a, dots, 0);
  hipLaunchKernelGGL((vocab_rows_kernel<T, kPartThreads, kPartVecs, true, 1>), grid, dim3(kPartThreads), 0, st, a, dots, vocab_rows_count(a) ? 1 : 0);
  return hipGetLastError();
}

template <int P>
hipError_t teacher_of(const int32_t* index, const float* logit, int rows, int k, int classes, float temperature, int32_t* index_out,
                      float* prob, float* entropy, int32_t* counts, uint16_t* first, int part, int parts, hipStream_t st) {
  hipLaunchKernelGGL(teacher_kernel<P>, dim3((rows + 3) / 4), dim3(256), 0, st, index, logit, rows, k, classes,
                     1.f / temperature, index_out, prob, entropy, counts, first, part, parts);
  return hipGetLastError();
}

}  // namespace

bool vocab_rows_count(const VocabRows& a) { return a.dz && !a.t.weight && a.rows <= 2048; }

hipError_t launch_teacher(const int32_t* index, const float* logit, int rows, int k, int classes, float temperature, int32_t* index_out,
                          float* prob, float* entropy, int32_t* counts, uint16_t* first, int part, int parts, hipStream_t st) {
  if (k < 1 || k > kTeacherMax) return hipErrorInvalidValue;
  auto of = k <= 64 ? teacher_of<64> : k <= 128 ? teacher_of<128> : k <= 256 ? teacher_of<256> : teacher_of<1024>;
  return of(index, logit, rows, k, classes, temperature, index_out, prob, entropy, counts, first, part, parts, st);
}

hipError_t launch_count_rows(const VocabTargets& t, int rows, int classes, float* inv_count, hipStream_t st) {
  hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, st, t, rows, classes, inv_count);
  return hipGetLastError();
}

hipError_t launch_weighted_loss(const VocabTargets& t, const float* row_loss, int rows, int classes, float* loss, hipStream_t st) {
  hipLaunchKernelGGL(weighted_loss_kernel, dim3(1), dim3(1024), 0, st, t, row_loss, rows, classes, loss);
  return hipGetLastError();
}

int64_t vocab_rows_stats_floats(int rows, int classes) {
  const int64_t parts = (classes / 4 + 2 + kPartThreads * kPartVecs) / (kPartThreads * kPartVecs) + 1;   // (fp32 vectors)
  return (int64_t)rows * (parts * 2 + 2);
}

hipError_t launch_vocab_rows(const VocabRows& a, hipStream_t st) {
  if (a.rows <= 0) return hipSuccess;
  return a.dtype == kBF16 ? rows_any<uint16_t>(a, st) : rows_any<float>(a, st);
}

hipError_t launch_cast_add(const float* in, uint16_t* out, int64_t n, int beta, hipStream_t st) {
  hipLaunchKernelGGL(cast_add_kernel, dim3((unsigned)((n + 2047) / 2048)), dim3(256), 0, st, in, out, n, beta);
  return hipGetLastError();
}

}  // namespace rad
