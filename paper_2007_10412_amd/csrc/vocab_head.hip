// What surrounds the three products of a layer under a loss over its classes.  Those products take the rows that have a target
// only (row_list), so that a batch of which half are prompts costs half.  The logits' product leaves the logits (bf16: each in
// 16 bits) and the softmax's statistics per part of a row (epilogue_vocab); with a row's sum known, one pass leaves dz in
// their place.
#include <math.h>

#include "head_epilogue.hpp"
#include "kernels.hpp"

namespace rad {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// ------------------------------------------------------------------ the list of rows
// One workgroup: a thread has 8 consecutive rows of 8192 at a time, and places them by a count over the threads before it.  A
// launch and the latency of a few dependent steps: 2000 rows 5 us, 4096 7.
__global__ __launch_bounds__(1024) void row_list_kernel(VocabTargets t, int rows, int classes, int32_t* __restrict__ list,
                                                        int32_t* __restrict__ live, float* __restrict__ inv_count,
                                                        float* __restrict__ common) {
  __shared__ int s_n[16];
  __shared__ float2 s_w[16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  auto counts = [&](int r) { return t.labels ? (uint32_t)t.labels[r] < (uint32_t)classes : t.counts[r] != 0; };
  int total = 0;                                        // rows that count (of one block of rows: below)
  if (rows > 8192) {
    for (int r = threadIdx.x; r < rows; r += 1024) total += counts(r) ? 1 : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) s_n[w] = total;
    __syncthreads();
    total = 0;
    for (int q = 0; q < 16; ++q) total += s_n[q];
  }
  int before = 0;                                       // rows that count before this block of 8192
  for (int r0 = 0; r0 < rows; r0 += 8192) {
    uint32_t mine = 0u;
    const int r1 = r0 + (int)threadIdx.x * 8;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (r1 + q < rows && counts(r1 + q)) mine |= 1u << q;
    int n = __popc(mine), up = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(up, o); if (lane >= o) up += v; }
    __syncthreads();
    if (lane == 63) s_n[w] = up;
    __syncthreads();
    int at = before + up - n, all = 0;
    for (int q = 0; q < 16; ++q) { if (q < w) at += s_n[q]; all += s_n[q]; }
    if (rows <= 8192) total = all;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = r1 + q;
      if (r >= rows) break;
      const bool c = (mine >> q) & 1u;
      list[c ? at : total + (r - at)] = r;              // (r - at rows before this one do not count)
      at += c ? 1 : 0;
    }
    before += all;
  }
  WeightRange of;
  if (t.weight) {
    for (int r = threadIdx.x; r < rows; r += 1024) if (counts(r)) of.add(t.weight[r]);
    of.join_wave();
    if (lane == 0) s_w[w] = make_float2(of.most, of.least);
    __syncthreads();
    for (int q = 0; q < 16; ++q) of.join(s_w[q].x, s_w[q].y);
  }
  if (threadIdx.x == 0) {
    const float inv = inv_count ? (total > 0 ? 1.f / (float)total : 0.f) : t.weight ? 0.f : *t.inv_count;
    *live = total;
    if (inv_count) *inv_count = inv;
    *common = t.weight ? of.common(t.temperature) : t.temperature * inv;
  }
}

// ------------------------------------------------------------------ between the products
// What epilogue_vocab does, on partial sums: 16 lanes have 64 columns of a row, four each.  40 x 2000 of 13 splits 5.3 us,
// the launch and two loads after one another.
template <typename T>
__global__ __launch_bounds__(256) void vocab_join_kernel(GemmArgs g) {
  const HeadArgs& h = g.head;
  const int l = threadIdx.x & 15, place = (int)blockIdx.y * 16 + (threadIdx.x >> 4), live = *h.live;
  if (place >= live) return;
  const int part = blockIdx.x, col = part * 64 + l * 4;
  const float* const in = static_cast<const float*>(g.C) + (int64_t)place * g.ldc + col;
  floatx4 z = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < g.k_splits; s += 4) {
    floatx4 v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = s + q < g.k_splits ? *reinterpret_cast<const floatx4*>(in + (s + q) * g.split_stride) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] += v[q][e];
  }
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (g.bias) z[e] += g.bias[min(col + e, g.N - 1)];
    if (col + e >= g.N) z[e] = -INFINITY;
    m = fmaxf(m, z[e]);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float from = m == -INFINITY ? 0.f : m;
  float below[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) { below[e] = z[e] - from; s += __builtin_amdgcn_exp2f(below[e] * h.c); }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (l == 0) *reinterpret_cast<float2*>(h.stats + ((int64_t)part * h.stats_ld + place) * 2) = make_float2(m, s);
  if (g.y) {
    T* const y = static_cast<T*>(g.y) + (int64_t)place * g.ldy + col;
    const float k = -h.c / kCodeRange;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(y) = u32x2{code_pair(below[0] * k, below[1] * k), code_pair(below[2] * k, below[3] * k)};
    else *reinterpret_cast<floatx4*>(y) = z;
  }
  const int row = h.row_map[place];
  int t0 = 0, t1 = 0;
  if (h.labels) t1 = 1;
  else { t0 = h.first[(int64_t)row * h.first_ld + part]; t1 = h.first[(int64_t)row * h.first_ld + part + 1]; }
  for (int t = t0; t < t1; ++t) {
    const int at = (h.labels ? h.labels[row] : h.index[(int64_t)row * h.k + t]) - col;
    if (at >= 0 && at < 4) h.target[(int64_t)place * h.k + t] = at == 0 ? z[0] : at == 1 ? z[1] : at == 2 ? z[2] : z[3];
  }
}

// a row's share of *common (with weights never zero)
__device__ __forceinline__ float row_share(const VocabTargets& t, int row, float common) {
  return !t.weight ? 1.f : t.weight[row] * t.temperature / common;
}

// (maximum, sum of exponentials from it) of two parts; one with nothing in it adds its 0, or its NaN
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
  if (m2 == -INFINITY) { s += s2; return; }
  if (m == -INFINITY) { m = m2; s += s2; return; }
  const float M = fmaxf(m, m2);
  s = s * __builtin_amdgcn_exp2f((m - M) * c) + s2 * __builtin_amdgcn_exp2f((m2 - M) * c);
  m = M;
}

// R = 2^shift places a workgroup, 1024 / R threads for the parts of each: the statistics of neighbouring places lie side by
// side, so a load brings R rows' pairs of several parts.  4096 rows of 1000 parts 15 us (2.2 TB/s), of 8 parts 6, the launch and
// its chain of loads (list, statistics, probabilities).
constexpr int kFinishThreads = 1024, kFinishRows = 16, kFinishAhead = 4;
template <typename T>
__global__ __launch_bounds__(kFinishThreads) void vocab_finish_kernel(VocabFinish a, int shift) {
  __shared__ float s_m[16][kFinishRows], s_s[16][kFinishRows];
  __shared__ float3 s_t[16][kFinishRows];
  __shared__ int s_row[kFinishRows];
  const int R = 1 << shift, r = (int)threadIdx.x & (R - 1), grp = (int)threadIdx.x >> shift, groups = kFinishThreads >> shift;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int place0 = (int)blockIdx.x << shift, place = place0 + r;
  const int live = *a.live;
  const VocabTargets& t = a.t;
  const float c = kLog2e / t.temperature;
  const bool counts = place < live;
  const int row = place < a.rows ? a.list[place] : -1;

  float m = -INFINITY, s = 0.f;
  TargetSum sum;
  if (counts) {
    for (int p = grp; p < a.parts; p += groups * kFinishAhead) {
      float2 v[kFinishAhead];
#pragma unroll
      for (int q = 0; q < kFinishAhead; ++q) {
        const int pq = p + q * groups;
        v[q] = pq < a.parts ? *reinterpret_cast<const float2*>(a.stats + ((int64_t)pq * a.stats_ld + place) * 2) : make_float2(-INFINITY, 0.f);
      }
#pragma unroll
      for (int q = 0; q < kFinishAhead; ++q) join(m, s, v[q].x, v[q].y, c);
    }
    for (int j = grp; j < t.k; j += groups) {
      const float pj = t.labels ? 1.f : t.prob[(int64_t)row * t.k + j];
      if (pj != 0.f) sum.add(pj, a.target[(int64_t)place * t.k + j]);
    }
  }
  for (int o = R; o < 64; o <<= 1) {
    join(m, s, __shfl_xor(m, o), __shfl_xor(s, o), c);
    sum.join_lane(o);
  }
  if (lane < R) { s_m[wave][r] = m; s_s[wave][r] = s; sum.put(&s_t[wave][r]); }
  __syncthreads();
  if ((int)threadIdx.x < R) {
    for (int w = 1; w < 16; ++w) { join(m, s, s_m[w][r], s_s[w][r], c); sum.join(s_t[w][r]); }
    s_row[r] = row;
    float part = 0.f;                                   // of the batch's loss
    if (counts) {
      const float T1 = t.temperature, top = m == -INFINITY ? 0.f : m;
      const float weight = t.weight ? t.weight[row] : *t.inv_count;
      const float loss = T1 * T1 * ((t.labels ? 0.f : t.entropy[row]) + (logf(s) + ((top - sum.from()) - sum.dot) / T1));
      a.row_loss[row] = loss;
      a.top[place] = top;
      a.factor[place] = row_share(t, row, *a.common) / s;
      part = weight * loss;
    } else if (place < a.rows) {
      a.row_loss[row] = 0.f;
    }
    if (a.loss && !a.z) *a.loss = part;                 // (of one row: vocab_loss_inside)
  }
  __syncthreads();
  if (a.xs && live < a.rows) {
    const int64_t bytes = a.x_ld * (int64_t)sizeof(T);
    const int vecs = (int)(bytes / 16);
    for (int q = threadIdx.x; q < R * vecs; q += kFinishThreads) {
      const int rr = q / vecs, v = q - rr * vecs;
      if (place0 + rr < live)
        *reinterpret_cast<u32x4*>(static_cast<char*>(a.xs) + (place0 + rr) * bytes + v * 16) =
            *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.x) + s_row[rr] * bytes + v * 16);
    }
  }
  if (a.dx)
    for (int rr = 0; rr < R; ++rr) {
      if (place0 + rr < live || place0 + rr >= a.rows) continue;
      T* const d = static_cast<T*>(a.dx) + (int64_t)s_row[rr] * a.d_in;
      for (int v = threadIdx.x; v < a.d_in; v += kFinishThreads) d[v] = 0;
    }
}

// 16 rows x kSteps 16-byte vectors of 16 lanes a workgroup.  Reads and writes a logit, and is bound by that: 4096 x 128000 bf16
// 404 us (5.2 TB/s), 4096 x 32000 97, 1024 x 8003 fp32 12.  The last column of
// workgroups (where there is a loss to sum) has no logits: its first one adds the rows' losses.
constexpr int kGradRows = 16;
template <typename T, int kGradSteps>
__global__ __launch_bounds__(256) void vocab_gradient_kernel(VocabFinish a, int sum_column) {
  constexpr int VPL = 16 / (int)sizeof(T), kCols = 16 * VPL * kGradSteps;
  __shared__ float s_w[4];
  const int live = *a.live;
  const VocabTargets& t = a.t;
  if ((int)blockIdx.x == sum_column) {
    if (blockIdx.y != 0) return;
    float sum = 0.f;
    for (int p = threadIdx.x; p < live; p += 256) {
      const int row = a.list[p];
      sum += (t.weight ? t.weight[row] : *t.inv_count) * a.row_loss[row];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) *a.loss = (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
    return;
  }
  if ((int)blockIdx.y * kGradRows >= live) return;
  const int l = threadIdx.x & 15, place = (int)blockIdx.y * kGradRows + (threadIdx.x >> 4);
  const float c = kLog2e / t.temperature;
  const int c0 = (int)blockIdx.x * kCols, shift = a.part == 64 ? 6 : 7;
  const bool counts = place < live;
  T* const zr = static_cast<T*>(a.z) + (int64_t)place * a.z_ld;
  float top = 0.f, f = 0.f;
  if (counts) {
    top = a.top[place]; f = a.factor[place];
    u32x4 w[kGradSteps];
    float m[kGradSteps];
#pragma unroll
    for (int q = 0; q < kGradSteps; ++q) {
      const int64_t col = (int64_t)c0 + (q * 16 + l) * VPL;
      w[q] = u32x4{0u, 0u, 0u, 0u};
      m[q] = -INFINITY;
      if (col < a.z_ld) w[q] = *reinterpret_cast<const u32x4*>(zr + col);
      if (sizeof(T) == 2 && col < a.classes) m[q] = a.stats[((col >> shift) * a.stats_ld + place) * 2];
    }
#pragma unroll
    for (int q = 0; q < kGradSteps; ++q) {
      const int64_t col = (int64_t)c0 + (q * 16 + l) * VPL;
      if (col >= a.z_ld) continue;
      u32x4 o;
      if constexpr (sizeof(T) == 2) {
        const float off = m[q] == -INFINITY ? 0.f : (m[q] - top) * c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = w[q][e] & 0xFFFFu, hi = w[q][e] >> 16;
          const float e0 = __builtin_amdgcn_exp2f(fmaf((float)lo, -kCodeRange / 65535.f, off));
          const float e1 = __builtin_amdgcn_exp2f(fmaf((float)hi, -kCodeRange / 65535.f, off));
          o[e] = bf16_pair((lo == kCodeLast ? 0.f : e0) * f, (hi == kCodeLast ? 0.f : e1) * f);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(__builtin_amdgcn_exp2f((__uint_as_float(w[q][e]) - top) * c) * f);
      }
      *reinterpret_cast<u32x4*>(zr + col) = o;
    }
  }
  __threadfence_block();
  __syncthreads();                                      // the targets' elements are written again, after their vectors
  if (!counts) return;
  const int row = a.list[place];
  int t0 = 0, t1 = 0;
  if (t.labels) t1 = (uint32_t)(t.labels[row] - c0) < (uint32_t)kCols ? 1 : 0;
  else {
    const uint16_t* const fr = a.first + (int64_t)row * a.first_ld;
    t0 = fr[c0 >> shift]; t1 = fr[min((c0 + kCols) >> shift, a.parts)];
  }
  const float wt = row_share(t, row, *a.common);
  for (int j = t0 + l; j < t1; j += 16) {
    const float pj = t.labels ? 1.f : t.prob[(int64_t)row * t.k + j];
    if (pj == 0.f) continue;
    const int col = t.labels ? t.labels[row] : t.index[(int64_t)row * t.k + j];
    const float g = __builtin_amdgcn_exp2f((a.target[(int64_t)place * t.k + j] - top) * c) * f - wt * pj;
    if constexpr (sizeof(T) == 2) zr[col] = (uint16_t)bf16_pair(g, 0.f);
    else zr[col] = g;
  }
}

// ------------------------------------------------------------------ sums
// Partial sums of a split product, split by split in order, four columns a thread: 4096 x 2048 to bf16 15 us, 1024 x 512 5.
__global__ __launch_bounds__(256) void split_sum_kernel(SplitSum a) {
  const int row = blockIdx.y;
  const int rows = a.live ? min(a.rows, *a.live) : a.rows;
  if (row >= rows) return;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= a.cols) return;
  const float* const in = a.in + (int64_t)row * a.in_ld + c;          // (rows are padded to whole vectors)
  floatx4 v = *reinterpret_cast<const floatx4*>(in);
  for (int s = 1; s < a.splits; ++s) {
    const floatx4 w = *reinterpret_cast<const floatx4*>(in + s * a.stride);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += w[e];
  }
  const int64_t at = (int64_t)(a.map ? a.map[row] : row) * a.out_ld + c;
  const float f = *a.scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= f;
  if (a.out_dtype == kF32) {
    float* const o = static_cast<float*>(a.out) + at;
    if (c + 4 <= a.cols && !a.beta) { __builtin_memcpy(o, &v, 16); return; }
#pragma unroll
    for (int e = 0; e < 4; ++e) if (c + e < a.cols) o[e] = a.beta ? o[e] + v[e] : v[e];
    return;
  }
  uint16_t* const o = static_cast<uint16_t*>(a.out) + at;
  if (c + 4 <= a.cols && !a.beta) {
    const u32x2 w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    __builtin_memcpy(o, &w, 8);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (c + e < a.cols) o[e] = (uint16_t)bf16_pair(a.beta ? bf16_bits_to_f32(o[e]) + v[e] : v[e], 0.f);
}

// (the sum is of dz as the products take it, in the layer's type, as rad_backward_dW's is of the dy that it is given)
// 64 lanes' vectors of columns and one range of rows a workgroup, its four waves every fourth row: 1024 x 8003 fp32 6 us (5.4
// TB/s) and 4.6 for the ranges' sum; in one range 512 x 1024 x 8192 took 110 us instead of 80
template <typename T>
__global__ __launch_bounds__(256) void head_colsum_kernel(const T* __restrict__ g, int64_t g_ld, const int32_t* __restrict__ live,
                                                          int cols, float* __restrict__ part) {
  constexpr int VPL = 16 / (int)sizeof(T), W = 64 * VPL;
  __shared__ float s_sum[4][W];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int n = *live, per = (n + kHeadColsumSplits - 1) / kHeadColsumSplits;
  const int r0 = (int)blockIdx.y * per, r1 = min(n, r0 + per);
  const int c = (int)blockIdx.x * W + lane * VPL;
  float sum[VPL] = {};
  if (c < g_ld)
    for (int r = r0 + w; r < r1; r += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(g + (int64_t)r * g_ld + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) { sum[2 * e] += __uint_as_float(v[e] << 16); sum[2 * e + 1] += __uint_as_float(v[e] & 0xFFFF0000u); }
        else sum[e] += __uint_as_float(v[e]);
      }
    }
#pragma unroll
  for (int e = 0; e < VPL; ++e) s_sum[w][lane * VPL + e] = sum[e];
  __syncthreads();
  for (int q = threadIdx.x; q < W; q += 256) {
    const int col = (int)blockIdx.x * W + q;
    if (col < cols) part[(int64_t)blockIdx.y * cols + col] = (s_sum[0][q] + s_sum[1][q]) + (s_sum[2][q] + s_sum[3][q]);
  }
}
__global__ __launch_bounds__(256) void head_colsum_final_kernel(const float* __restrict__ part, int cols, const float* __restrict__ scale,
                                                                float* __restrict__ out, int beta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float s = 0.f;
  for (int q = 0; q < kHeadColsumSplits; ++q) s += part[(int64_t)q * cols + c];
  out[c] = (beta ? out[c] : 0.f) + *scale * s;
}

// a vector a thread: 1000 x 50257 bf16 34 us (5.9 TB/s)
template <typename T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const T* __restrict__ in, int64_t rows, int cols, T* __restrict__ out, int vecs) {
  constexpr int VPL = 16 / (int)sizeof(T);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * vecs) return;
  const int64_t row = i / vecs;
  const int c = (int)(i - row * vecs) * VPL;
  const T* const src = in + row * cols + c;
  u32x4 w = {0u, 0u, 0u, 0u};
  if (c + VPL <= cols) __builtin_memcpy(&w, src, 16);
  else {
    T* we = reinterpret_cast<T*>(&w);
#pragma unroll
    for (int e = 0; e < VPL; ++e) if (c + e < cols) we[e] = src[e];
  }
  *reinterpret_cast<u32x4*>(out + i * VPL) = w;
}

}  // namespace

hipError_t launch_row_list(const VocabTargets& t, int rows, int classes, int32_t* list, int32_t* live, float* inv_count, float* common,
                           hipStream_t st) {
  hipLaunchKernelGGL(row_list_kernel, dim3(1), dim3(1024), 0, st, t, rows, classes, list, live, inv_count, common);
  return hipGetLastError();
}
hipError_t launch_vocab_join(int dtype, const GemmArgs& g, hipStream_t st) {
  const dim3 grid((g.N + 63) / 64, (g.M + 15) / 16);
  if (grid.y > 65535 || g.ldc % 64) return hipErrorInvalidValue;
  if (dtype == kBF16) hipLaunchKernelGGL(vocab_join_kernel<uint16_t>, grid, dim3(256), 0, st, g);
  else hipLaunchKernelGGL(vocab_join_kernel<float>, grid, dim3(256), 0, st, g);
  return hipGetLastError();
}
// places of a finishing workgroup: up to 16, while there is a workgroup for every other CU
static int finish_shift(int rows) {
  int shift = 4;
  while (shift > 0 && (rows >> shift) < 128) --shift;
  return shift;
}
// 16 vectors a lane where that makes a workgroup for every other CU, 4 where it does not
template <typename T> static hipError_t gradient_of(const VocabFinish& a, hipStream_t st) {
  const unsigned rows = (unsigned)((a.rows + kGradRows - 1) / kGradRows);
  if (rows > 65535) return hipErrorInvalidValue;
  const int64_t width = 16 * (16 / (int)sizeof(T));
  const bool wide = rows * ((a.z_ld + 16 * width - 1) / (16 * width)) >= 128;
  const unsigned cols = (unsigned)((a.z_ld + (wide ? 16 : 4) * width - 1) / ((wide ? 16 : 4) * width));
  const dim3 grid(cols + (a.loss ? 1 : 0), rows);
  const int sum_column = a.loss ? (int)cols : -1;
  if (wide) hipLaunchKernelGGL((vocab_gradient_kernel<T, 16>), grid, dim3(256), 0, st, a, sum_column);
  else hipLaunchKernelGGL((vocab_gradient_kernel<T, 4>), grid, dim3(256), 0, st, a, sum_column);
  return hipGetLastError();
}
bool vocab_loss_inside(const VocabFinish& a) { return a.z || a.rows == 1; }
hipError_t launch_vocab_finish(const VocabFinish& a, hipStream_t st) {
  const int shift = finish_shift(a.rows);
  const dim3 grid((a.rows + (1 << shift) - 1) >> shift);
  if (a.dtype == kBF16) hipLaunchKernelGGL(vocab_finish_kernel<uint16_t>, grid, dim3(kFinishThreads), 0, st, a, shift);
  else hipLaunchKernelGGL(vocab_finish_kernel<float>, grid, dim3(kFinishThreads), 0, st, a, shift);
  return hipGetLastError();
}
hipError_t launch_vocab_gradient(const VocabFinish& a, hipStream_t st) {
  return a.dtype == kBF16 ? gradient_of<uint16_t>(a, st) : gradient_of<float>(a, st);
}
hipError_t launch_split_sum(const SplitSum& a, hipStream_t st) {
  if (a.rows > 65535 || a.in_ld % 4) return hipErrorInvalidValue;
  hipLaunchKernelGGL(split_sum_kernel, dim3((a.cols + 1023) / 1024, a.rows), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_head_colsum(int dtype, const void* g, int64_t g_ld, const int32_t* live, const float* scale, int cols, float* part,
                              float* out, int beta, hipStream_t st) {
  const int W = dtype == kBF16 ? 512 : 256;
  const dim3 grid((cols + W - 1) / W, kHeadColsumSplits);
  if (dtype == kBF16) hipLaunchKernelGGL(head_colsum_kernel<uint16_t>, grid, dim3(256), 0, st, (const uint16_t*)g, g_ld, live, cols, part);
  else hipLaunchKernelGGL(head_colsum_kernel<float>, grid, dim3(256), 0, st, (const float*)g, g_ld, live, cols, part);
  hipLaunchKernelGGL(head_colsum_final_kernel, dim3((cols + 255) / 256), dim3(256), 0, st, part, cols, scale, out, beta);
  return hipGetLastError();
}
hipError_t launch_pad_rows(int dtype, const void* in, int64_t rows, int cols, void* out, int64_t out_ld, hipStream_t st) {
  const int vecs = (int)(out_ld / (dtype == kBF16 ? 8 : 4));
  const dim3 grid((unsigned)((rows * vecs + 255) / 256));
  if (dtype == kBF16) hipLaunchKernelGGL(pad_rows_kernel<uint16_t>, grid, dim3(256), 0, st, (const uint16_t*)in, rows, cols, (uint16_t*)out, vecs);
  else hipLaunchKernelGGL(pad_rows_kernel<float>, grid, dim3(256), 0, st, (const float*)in, rows, cols, (float*)out, vecs);
  return hipGetLastError();
}

}  // namespace rad
