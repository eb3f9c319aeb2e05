// A small layer under a loss over up to 16 classes, where launches are most of the time: two kernels instead of five
// (150 x 300 x 10 with all gradients, against the general route: fp32 with biases 43 -> 15 us, bf16 28 -> 16).  What bounds
// them is latency: two launches, the loads' way from memory (labels, weights and biases are asked for before the products) and
// the exchanges between lanes.
//
// The first has a workgroup for 4 rows: its threads share the d_in products of a logit, and a transposing reduction leaves lane
// 16 r + v of every wave with z_v of row r, so the softmax is a few exchanges among the 16 lanes of a row.
// dX follows at once, the layer's few weights coming from the caches.  The second forms dW from dz, 64 rows of it a workgroup,
// with the bias gradient as the row of a column of ones, and sums the loss.
#include <math.h>

#include "head_epilogue.hpp"
#include "kernels.hpp"

namespace rad {
namespace {

constexpr int VP = kFewClasses, R = 64 / VP;           // places for classes, rows of a workgroup

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float ld_elem(const float* p) { return *p; }
__device__ __forceinline__ float ld_elem(const uint16_t* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ void st_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_elem(uint16_t* p, float v) { *p = (uint16_t)bf16_pair(v, 0.f); }

__device__ __forceinline__ bool row_counts(const VocabTargets& t, int row, int classes) {
  return t.labels ? (uint32_t)t.labels[row] < (uint32_t)classes : t.counts[row] != 0;
}

// 64 sums over the lanes of a wave, one to a lane: in step o a lane keeps the half of its values whose number has its bit o
template <int N> __device__ __forceinline__ void reduce_scatter(float (&v)[64], int lane) {
  if constexpr (N >= 1) {
    const bool up = (lane & N) != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float send = up ? v[i] : v[i + N], keep = up ? v[i + N] : v[i];
      v[i] = keep + __shfl_xor(send, N);
    }
    reduce_scatter<N / 2>(v, lane);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void few_classes_kernel(FewClasses a) {
  __shared__ float s_w[4], s_z[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const VocabTargets& t = a.t;
  const int V = a.classes;
  const int row0 = (int)blockIdx.x * R;
  const int r = lane / VP, v = lane % VP, row = row0 + r;
  // (what the softmax needs is asked for before the products, whose loads it then does not follow)
  float n = 0.f;
  if (!t.weight)
    for (int q = threadIdx.x; q < a.rows; q += 256) n += row_counts(t, q, V) ? 1.f : 0.f;
  const bool counts = row < a.rows && row_counts(t, row, V);
  const int label = t.labels && row < a.rows ? t.labels[row] : -1;
  const float weight = t.weight && row < a.rows ? t.weight[row] : 0.f;
  const float bias = a.bias && v < V ? a.bias[v] : 0.f;
  const T* const W = static_cast<const T*>(a.W);
  float acc[64];
#pragma unroll
  for (int i = 0; i < 64; ++i) acc[i] = 0.f;
  for (int d = threadIdx.x; d < a.d_in; d += 256) {
    float x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = row0 + r < a.rows ? ld_elem(static_cast<const T*>(a.x) + (int64_t)(row0 + r) * a.d_in + d) : 0.f;
#pragma unroll
    for (int v = 0; v < VP; ++v) {                      // (classes past the last: what it has, never used)
      const float wv = ld_elem(W + (int64_t)d * V + min(v, V - 1));
#pragma unroll
      for (int r = 0; r < R; ++r) acc[r * VP + v] += x[r] * wv;
    }
  }
  reduce_scatter<32>(acc, lane);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
  s_z[w][lane] = acc[0];
  if (lane == 0) s_w[w] = n;
  __syncthreads();
  n = (s_w[0] + s_w[1]) + (s_w[2] + s_w[3]);
  const float inv_count = n > 0.f ? 1.f / n : 0.f;
  float z = (s_z[0][lane] + s_z[1][lane]) + (s_z[2][lane] + s_z[3][lane]);     // (the same in all waves from here on)
  z = v < V ? z + bias : -INFINITY;
  float p = 0.f;
  if (counts) {
    if (t.labels) p = label == v ? 1.f : 0.f;
    else
      for (int j = 0; j < t.k; ++j) {                   // (sorted, each class once)
        const int i = t.index[(int64_t)row * t.k + j];
        if (i < 0) break;
        if (i == v) p += t.prob[(int64_t)row * t.k + j];
      }
  }
  const float c = kLog2e / t.temperature;
  float m = z;
#pragma unroll
  for (int o = VP / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float top = m == -INFINITY ? 0.f : m;
  const float e = __builtin_amdgcn_exp2f((z - top) * c);
  float s = e, dot = p != 0.f ? p * (z - top) : 0.f;
#pragma unroll
  for (int o = VP / 2; o > 0; o >>= 1) { s += __shfl_xor(s, o); dot += __shfl_xor(dot, o); }
  const float T1 = t.temperature;
  if (w == 0 && v == 0 && row < a.rows)
    a.row_loss[row] = counts ? T1 * T1 * ((t.labels ? 0.f : t.entropy[row]) + (logf(s) - dot / T1)) : 0.f;
  const float wt = counts ? (t.weight ? weight : inv_count) * T1 : 0.f;
  const float g = counts && v < V ? wt / s * e - wt * p : 0.f;
  if (a.dz && w == 0 && row < a.rows) a.dz[(int64_t)row * VP + v] = g;
  if (!a.dx) return;
  const uint64_t live = __ballot(counts);               // (a row that does not count: zeros, also where W holds what 0 times is NaN)
  for (int d0 = 0; d0 < a.d_in; d0 += 256) {
    const int d = d0 + (int)threadIdx.x;
    float sum[R];
#pragma unroll
    for (int q = 0; q < R; ++q) sum[q] = 0.f;
#pragma unroll
    for (int q = 0; q < VP; ++q) {                      // (g is zero in classes past the last)
      const float wv = d < a.d_in && q < V ? ld_elem(W + (int64_t)d * V + q) : 0.f;
#pragma unroll
      for (int rr = 0; rr < R; ++rr) sum[rr] += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), rr * VP + q)) * wv;
    }
    if (d < a.d_in) {
#pragma unroll
      for (int rr = 0; rr < R; ++rr)
        if (row0 + rr < a.rows) st_elem(static_cast<T*>(a.dx) + (int64_t)(row0 + rr) * a.d_in + d, (live >> (rr * VP)) & 1u ? sum[rr] : 0.f);
    }
  }
}

// dW rows d0 .. d0 + 63 (and, as row d_in, the bias gradient): a lane has one, the 16 waves share the batch.  The last
// workgroup, where a loss is asked for, adds the rows' losses.
template <typename T, typename O>
__global__ __launch_bounds__(1024) void few_classes_dw_kernel(FewClasses a, int blocks) {
  __shared__ float s_sum[16][VP][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const VocabTargets& t = a.t;
  const int V = a.classes;
  if ((int)blockIdx.x == blocks) {
    float sum = 0.f, n = 0.f;
    for (int r = threadIdx.x; r < a.rows; r += 1024)
      if (row_counts(t, r, V)) { sum += (t.weight ? t.weight[r] : 1.f) * a.row_loss[r]; n += 1.f; }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { sum += __shfl_xor(sum, o); n += __shfl_xor(n, o); }
    if (lane == 0) { s_sum[0][0][w] = sum; s_sum[0][1][w] = n; }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int q = 1; q < 16; ++q) { sum += s_sum[0][0][q]; n += s_sum[0][1][q]; }
    *a.loss = t.weight ? sum : n > 0.f ? sum / n : 0.f;
    return;
  }
  static_assert(VP == 16, "a wave of the 16 for each class");
  const int d = (int)blockIdx.x * 64 + lane;
  float acc[VP];
#pragma unroll
  for (int v = 0; v < VP; ++v) acc[v] = 0.f;
#pragma unroll 4
  for (int r = w; r < a.rows; r += 16) {
    const float* const g = a.dz + (int64_t)r * VP;      // (the same for the wave, as is whether the row counts)
    float x = d < a.d_in ? ld_elem(static_cast<const T*>(a.x) + (int64_t)r * a.d_in + d) : 1.f;
    if (!row_counts(t, r, V)) x = 0.f;
#pragma unroll
    for (int v = 0; v < VP; ++v) acc[v] += x * g[v];
  }
#pragma unroll
  for (int v = 0; v < VP; ++v) s_sum[w][v][lane] = acc[v];
  __syncthreads();
  if (w >= V) return;                                   // a wave joins a class
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < 16; ++q) sum += s_sum[q][w][lane];
  if (d < a.d_in && a.dw) {
    O* const o = static_cast<O*>(a.dw) + (int64_t)d * V + w;
    st_elem(o, a.beta ? ld_elem(o) + sum : sum);
  } else if (d == a.d_in && a.dbias) {
    a.dbias[w] = a.beta ? a.dbias[w] + sum : sum;
  }
}

template <typename T> hipError_t few_of(const FewClasses& a, hipStream_t st) {
  hipLaunchKernelGGL(few_classes_kernel<T>, dim3((a.rows + R - 1) / R), dim3(256), 0, st, a);
  if (!a.dz && !a.loss) return hipGetLastError();
  // (the bias gradient's row is one past the others)
  const int blocks = !a.dz ? 0 : (a.d_in + (a.dbias ? 1 : 0) + 63) / 64;
  const dim3 grid(blocks + (a.loss ? 1 : 0));
  if (sizeof(T) == 2 && a.dw_dtype == kBF16) hipLaunchKernelGGL((few_classes_dw_kernel<T, uint16_t>), grid, dim3(1024), 0, st, a, blocks);
  else hipLaunchKernelGGL((few_classes_dw_kernel<T, float>), grid, dim3(1024), 0, st, a, blocks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_few_classes(const FewClasses& a, hipStream_t st) {
  if (a.classes < 1 || a.classes > kFewClasses) return hipErrorInvalidValue;
  return a.dtype == kBF16 ? few_of<uint16_t>(a, st) : few_of<float>(a, st);
}

}  // namespace rad
