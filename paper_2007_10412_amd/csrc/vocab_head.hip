// What surrounds the three bf16 products of a layer under a loss over its classes.  Those products take the rows that have a
// target only (row_list), so that a batch of which half are prompts costs half.  The logits' product leaves each logit in 16
// bits and the softmax's statistics per 128 columns (epilogue_vocab); with a row's sum known, one pass over those codes leaves
// dz in their place.
#include <math.h>

#include "head_epilogue.hpp"
#include "kernels.hpp"

namespace rad {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// ------------------------------------------------------------------ the list of rows
// One workgroup: a thread has 8 consecutive rows of 8192 at a time, and places them by a count over the threads before it.
__global__ __launch_bounds__(1024) void row_list_kernel(VocabTargets t, int rows, int classes, int32_t* __restrict__ list,
                                                        int32_t* __restrict__ live) {
  __shared__ int s_n[16];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int total = 0;                                        // rows that count, first of all
  for (int r = threadIdx.x; r < rows; r += 1024) total += (t.labels ? (uint32_t)t.labels[r] < (uint32_t)classes : t.counts[r] != 0) ? 1 : 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
  if (lane == 0) s_n[w] = total;
  __syncthreads();
  total = 0;
  for (int q = 0; q < 16; ++q) total += s_n[q];
  int before = 0;                                       // rows that count before this block of 8192
  for (int r0 = 0; r0 < rows; r0 += 8192) {
    uint32_t mine = 0u;
    const int r1 = r0 + (int)threadIdx.x * 8;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (r1 + q < rows && (t.labels ? (uint32_t)t.labels[r1 + q] < (uint32_t)classes : t.counts[r1 + q] != 0)) mine |= 1u << q;
    int n = __popc(mine), up = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(up, o); if (lane >= o) up += v; }
    __syncthreads();
    if (lane == 63) s_n[w] = up;
    __syncthreads();
    int at = before + up - n, all = 0;
    for (int q = 0; q < 16; ++q) { if (q < w) at += s_n[q]; all += s_n[q]; }
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
  if (threadIdx.x == 0) *live = total;
}

// a wave per row: entry j (ascending, -1 at the end) is before class 128 t for every t past its part
__global__ __launch_bounds__(256) void list_parts_kernel(const int32_t* __restrict__ index, int rows, int k, int parts,
                                                         uint16_t* __restrict__ first, int first_ld) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int32_t* const e = index + (int64_t)row * k;
  for (int t = lane; t <= parts; t += 64) {
    int lo = 0, hi = k;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if ((uint32_t)e[mid] < (uint32_t)t * 128u) lo = mid + 1; else hi = mid;     // (-1 lies after every class)
    }
    first[(int64_t)row * first_ld + t] = (uint16_t)lo;
  }
}

// ------------------------------------------------------------------ between the products
// 16 places a workgroup.  Their parts' statistics lie side by side, so a load brings 16 rows' pairs of one part.
constexpr int kFinishRows = 16, kFinishGroups = 64;
__global__ __launch_bounds__(kFinishRows * kFinishGroups) void vocab_finish_kernel(VocabFinish a) {
  __shared__ float s_m[kFinishGroups][kFinishRows], s_s[kFinishGroups][kFinishRows];
  __shared__ int s_row[kFinishRows];
  const int r = threadIdx.x % kFinishRows, grp = threadIdx.x / kFinishRows;
  const int place0 = blockIdx.x * kFinishRows, place = place0 + r;
  const int live = *a.live;
  const VocabTargets& t = a.t;
  const float c = kLog2e / t.temperature;
  const bool counts = place < live;

  float m = -INFINITY, s = 0.f;
  if (counts)
    for (int p = grp; p < a.parts; p += kFinishGroups) {
      const float2 v = *reinterpret_cast<const float2*>(a.stats + ((int64_t)p * a.stats_ld + place) * 2);
      if (v.x == -INFINITY) { s += v.y; continue; }     // nothing there (or a NaN)
      if (v.x > m) { s = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - v.x) * c); m = v.x; }
      s += v.x == m ? v.y : v.y * __builtin_amdgcn_exp2f((v.x - m) * c);
    }
  s_m[grp][r] = m; s_s[grp][r] = s;
  if (grp == 0) s_row[r] = place < a.rows ? a.list[place] : -1;
  __syncthreads();
  if (grp == 0) {
    float M = -INFINITY, S = 0.f;
    for (int q = 0; q < kFinishGroups; ++q) M = fmaxf(M, s_m[q][r]);
    const float b = M == -INFINITY ? 0.f : M;
    for (int q = 0; q < kFinishGroups; ++q) S += s_m[q][r] == -INFINITY ? s_s[q][r] : s_s[q][r] * __builtin_amdgcn_exp2f((s_m[q][r] - b) * c);
    if (counts) {
      const int row = s_row[r];
      float dot = 0.f;
      for (int j = 0; j < t.k; ++j) {
        const float pj = t.labels ? 1.f : t.prob[(int64_t)row * t.k + j];
        if (pj != 0.f) dot += pj * (a.target[(int64_t)place * t.k + j] - b);
      }
      const float T = t.temperature;
      if (a.row_loss) a.row_loss[row] = T * T * ((t.labels ? 0.f : t.entropy[row]) + (logf(S) - dot / T));
      a.top[place] = b;
      a.log2_sum[place] = log2f(S);
      a.factor[place] = (t.weight ? t.weight[row] : *t.inv_count) * T;
    } else if (place < a.rows && a.row_loss) {
      a.row_loss[s_row[r]] = 0.f;
    }
  }
  if (a.xs && live < a.rows) {
    const int vecs = (int)(a.xs_ld / 8);
    for (int q = threadIdx.x; q < kFinishRows * vecs; q += kFinishRows * kFinishGroups) {
      const int rr = q / vecs, v = q - rr * vecs;
      if (place0 + rr < live)
        *reinterpret_cast<u32x4*>(a.xs + (int64_t)(place0 + rr) * a.xs_ld + v * 8) =
            *reinterpret_cast<const u32x4*>(a.x + (int64_t)s_row[rr] * a.x_ld + v * 8);
    }
  }
  if (a.dx)
    for (int rr = 0; rr < kFinishRows; ++rr) {
      if (place0 + rr < live || place0 + rr >= a.rows) continue;
      uint16_t* const d = a.dx + (int64_t)s_row[rr] * a.d_in;
      for (int v = threadIdx.x; v < a.d_in; v += kFinishRows * kFinishGroups) d[v] = 0;
    }
}

// 16 rows x 2048 columns a workgroup: 16 lanes have a row's 128 columns of one part.  Reads and writes two bytes a logit, and is
// bound by that.
constexpr int kGradRows = 16, kGradParts = 16;
__global__ __launch_bounds__(256) void vocab_gradient_kernel(VocabFinish a) {
  const int l = threadIdx.x & 15, place = (int)blockIdx.y * kGradRows + (threadIdx.x >> 4);
  const int live = *a.live;
  if ((int)blockIdx.y * kGradRows >= live) return;
  const VocabTargets& t = a.t;
  const float c = kLog2e / t.temperature;
  const int p0 = (int)blockIdx.x * kGradParts;
  const bool counts = place < live;
  uint16_t* const zr = a.z + (int64_t)place * a.z_ld;
  float top = 0.f, log2_sum = 0.f, f = 0.f;
  if (counts) {
    top = a.top[place]; log2_sum = a.log2_sum[place]; f = a.factor[place];
    u32x4 w[kGradParts];
    float m[kGradParts];
#pragma unroll
    for (int q = 0; q < kGradParts; ++q) {
      const int64_t col = (int64_t)(p0 + q) * 128 + l * 8;
      w[q] = u32x4{0u, 0u, 0u, 0u};
      m[q] = -INFINITY;
      if (col < a.z_ld) w[q] = *reinterpret_cast<const u32x4*>(zr + col);
      if (p0 + q < a.parts) m[q] = a.stats[((int64_t)(p0 + q) * a.stats_ld + place) * 2];
    }
#pragma unroll
    for (int q = 0; q < kGradParts; ++q) {
      const int64_t col = (int64_t)(p0 + q) * 128 + l * 8;
      if (col >= a.z_ld) continue;
      const float off = (m[q] == -INFINITY ? 0.f : (m[q] - top) * c) - log2_sum;
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = w[q][e] & 0xFFFFu, hi = w[q][e] >> 16;
        const float a0 = f * __builtin_amdgcn_exp2f(fmaf((float)lo, -kCodeRange / 65535.f, off));
        const float a1 = f * __builtin_amdgcn_exp2f(fmaf((float)hi, -kCodeRange / 65535.f, off));
        o[e] = bf16_pair(lo == kCodeLast ? 0.f * log2_sum : a0, hi == kCodeLast ? 0.f * log2_sum : a1);   // (a NaN row stays one)
      }
      *reinterpret_cast<u32x4*>(zr + col) = o;
    }
  }
  __threadfence_block();
  __syncthreads();                                      // the targets' elements are written again, after their vectors
  if (!counts) return;
  const int row = a.list[place];
  int t0 = 0, t1 = 0;
  if (t.labels) t1 = (t.labels[row] >> 7) >= p0 && (t.labels[row] >> 7) < p0 + kGradParts ? 1 : 0;
  else {
    const uint16_t* const fr = a.first + (int64_t)row * a.first_ld;
    t0 = fr[p0]; t1 = fr[min(p0 + kGradParts, a.parts)];
  }
  for (int j = t0 + l; j < t1; j += 16) {
    const float pj = t.labels ? 1.f : t.prob[(int64_t)row * t.k + j];
    if (pj == 0.f) continue;
    const int col = t.labels ? t.labels[row] : t.index[(int64_t)row * t.k + j];
    const float e = __builtin_amdgcn_exp2f((a.target[(int64_t)place * t.k + j] - top) * c - log2_sum);
    zr[col] = (uint16_t)bf16_pair(f * (e - pj), 0.f);
  }
}

// ------------------------------------------------------------------ sums
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

// 512 columns and one range of rows a workgroup, its four waves every fourth row
__global__ __launch_bounds__(256) void head_colsum_kernel(const uint16_t* __restrict__ g, int64_t g_ld, const int32_t* __restrict__ live,
                                                          int cols, float* __restrict__ part) {
  __shared__ float s_sum[4][512];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int n = *live, per = (n + kHeadColsumSplits - 1) / kHeadColsumSplits;
  const int r0 = (int)blockIdx.y * per, r1 = min(n, r0 + per);
  const int c = (int)blockIdx.x * 512 + lane * 8;
  float sum[8] = {};
  if (c < g_ld)
    for (int r = r0 + w; r < r1; r += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(g + (int64_t)r * g_ld + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) { sum[2 * e] += __uint_as_float(v[e] << 16); sum[2 * e + 1] += __uint_as_float(v[e] & 0xFFFF0000u); }
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_sum[w][lane * 8 + e] = sum[e];
  __syncthreads();
  for (int q = threadIdx.x; q < 512; q += 256) {
    const int col = (int)blockIdx.x * 512 + q;
    if (col < cols) part[(int64_t)blockIdx.y * cols + col] = (s_sum[0][q] + s_sum[1][q]) + (s_sum[2][q] + s_sum[3][q]);
  }
}
__global__ __launch_bounds__(256) void head_colsum_final_kernel(const float* __restrict__ part, int cols, float* __restrict__ out, int beta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float s = beta ? out[c] : 0.f;
  for (int q = 0; q < kHeadColsumSplits; ++q) s += part[(int64_t)q * cols + c];
  out[c] = s;
}

__global__ __launch_bounds__(256) void pad_rows_kernel(const uint16_t* __restrict__ in, int64_t rows, int cols, uint16_t* __restrict__ out,
                                                       int vecs) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * vecs) return;
  const int64_t row = i / vecs;
  const int c = (int)(i - row * vecs) * 8;
  const uint16_t* const src = in + row * cols + c;
  u32x4 w = {0u, 0u, 0u, 0u};
  if (c + 8 <= cols) __builtin_memcpy(&w, src, 16);
  else {
    uint16_t* we = reinterpret_cast<uint16_t*>(&w);
#pragma unroll
    for (int e = 0; e < 8; ++e) if (c + e < cols) we[e] = src[e];
  }
  *reinterpret_cast<u32x4*>(out + i * 8) = w;
}

}  // namespace

hipError_t launch_row_list(const VocabTargets& t, int rows, int classes, int32_t* list, int32_t* live, hipStream_t st) {
  hipLaunchKernelGGL(row_list_kernel, dim3(1), dim3(1024), 0, st, t, rows, classes, list, live);
  return hipGetLastError();
}
hipError_t launch_list_parts(const int32_t* index, int rows, int k, int parts, uint16_t* first, int first_ld, hipStream_t st) {
  hipLaunchKernelGGL(list_parts_kernel, dim3((rows + 3) / 4), dim3(256), 0, st, index, rows, k, parts, first, first_ld);
  return hipGetLastError();
}
hipError_t launch_vocab_finish(const VocabFinish& a, hipStream_t st) {
  hipLaunchKernelGGL(vocab_finish_kernel, dim3((a.rows + kFinishRows - 1) / kFinishRows), dim3(kFinishRows * kFinishGroups), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_vocab_gradient(const VocabFinish& a, hipStream_t st) {
  const unsigned cols = (unsigned)((a.z_ld + 128 * kGradParts - 1) / (128 * kGradParts));
  const unsigned rows = (unsigned)((a.rows + kGradRows - 1) / kGradRows);
  if (rows > 65535) return hipErrorInvalidValue;
  hipLaunchKernelGGL(vocab_gradient_kernel, dim3(cols, rows), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_split_sum(const SplitSum& a, hipStream_t st) {
  if (a.rows > 65535 || a.in_ld % 4) return hipErrorInvalidValue;
  hipLaunchKernelGGL(split_sum_kernel, dim3((a.cols + 1023) / 1024, a.rows), dim3(256), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_head_colsum(const uint16_t* g, int64_t g_ld, const int32_t* live, int cols, float* part,
                              float* out, int beta, hipStream_t st) {
  hipLaunchKernelGGL(head_colsum_kernel, dim3((cols + 511) / 512, kHeadColsumSplits), dim3(256), 0, st, g, g_ld, live, cols, part);
  hipLaunchKernelGGL(head_colsum_final_kernel, dim3((cols + 255) / 256), dim3(256), 0, st, part, cols, out, beta);
  return hipGetLastError();
}
hipError_t launch_pad_rows(const uint16_t* in, int64_t rows, int cols, uint16_t* out, int64_t out_ld, hipStream_t st) {
  const int64_t n = rows * (out_ld / 8);
  hipLaunchKernelGGL(pad_rows_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, in, rows, cols, out, (int)(out_ld / 8));
  return hipGetLastError();
}

}  // namespace rad
