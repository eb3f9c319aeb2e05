// A layer's logits for a few rows, with what their log probabilities need (kEpiLogprob's outputs), without matrix instructions: W is
// read once from where it lies, whatever its rows' alignment, 16 bytes a lane.
//
//   z[r][v] = bias[v] + sum_k x[r][k] W[k][v]
//
// A workgroup has 16 neighbouring vectors of W's rows (256 bytes of each: 128 classes of bf16, 64 of fp32) and all of K, dealt to its 16
// waves 32 rows of W at a time: a wave's four quarters take 8 rows each, so that 8 loads of a lane are on their way at once and the 8
// values of x that they meet are one or two loads.  The quarters' and the waves' sums meet in LDS, in an order that is always the same.
//
// Bound by W's way from memory: bf16 1 x 4096 x 128000 167 us (6.3 TB/s), fp32 337 (6.2), bf16 1 x 2048 x 32000 21 (6.2).  A wave's step of
// one row takes 16 operations per 16 bytes in bf16 (4 in fp32), each further row 8 (4) more, of which a CU has time for some 40.
#include <algorithm>

#include "vocab_row.hpp"

namespace rad {
namespace {

constexpr int kFewThreads = 1024, kFewWaves = kFewThreads / 64, kFewBlock = 32;      // rows of W of a wave's step

template <typename T> struct FewTypes {
  static constexpr int VPL = 16 / (int)sizeof(T), C = 16 * VPL;                      // classes of a lane, of a workgroup
  typedef u32x4 any __attribute__((aligned(sizeof(uint16_t))));
};
template <typename T> __device__ __forceinline__ float few_at(const u32x4& v, int q) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v[q]);
  else return __uint_as_float(q & 1 ? v[q >> 1] & 0xFFFF0000u : v[q >> 1] << 16);
}

// PAST: W past the caches
template <typename T, int R, bool PAST>
__global__ __launch_bounds__(kFewThreads, R <= 2 ? 8 : 4) void few_rows_kernel(FewRows a) {
  constexpr int VPL = FewTypes<T>::VPL, C = FewTypes<T>::C, XV = 8 / VPL;            // vectors of x that meet 8 rows of W
  typedef typename FewTypes<T>::any vec;
  __shared__ float s_z[R][kFewWaves][C];
  const int tid = threadIdx.x, lane = tid & 63, slot = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = a.K, N = a.N, c0 = blockIdx.x * C;
  int row[R], live = 0;                                  // the rows that count, in order
#pragma unroll
  for (int p = 0; p < R; ++p) row[p] = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool counts = r < a.rows && (!a.token || (uint32_t)a.token[r] < (uint32_t)N);
#pragma unroll
    for (int p = 0; p <= r; ++p) row[p] = counts && live == p ? r : row[p];
    live += counts ? 1 : 0;
  }
  if (blockIdx.x == 0 && tid == 0) {
    *a.live = live;
    int yes = 0, no = live;
    for (int r = 0; r < a.rows; ++r) {
      const bool counts = !a.token || (uint32_t)a.token[r] < (uint32_t)N;
      a.list[counts ? yes++ : no++] = r;
    }
  }
  if (live == 0) return;

  // (the last vectors begin so early that they end with the row)
  const uint32_t at = ((uint32_t)(quarter * 8) * (uint32_t)a.w_ld + (uint32_t)min(c0 + slot * VPL, N - VPL)) * (uint32_t)sizeof(T);
  const int64_t line = a.w_ld * (int64_t)sizeof(T);
  const T* x[R];
#pragma unroll
  for (int p = 0; p < R; ++p) x[p] = static_cast<const T*>(a.x) + (int64_t)row[p] * a.x_ld;
  float acc[R][VPL];
#pragma unroll
  for (int p = 0; p < R; ++p)
#pragma unroll
    for (int e = 0; e < VPL; ++e) acc[p][e] = 0.f;
  const int whole = K / kFewBlock;
  for (int b = wave; b < whole; b += kFewWaves) {
    const unsigned char* const from = static_cast<const unsigned char*>(a.W) + (int64_t)b * kFewBlock * line;
    u32x4 w[8], xv[R][XV];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const vec* const p = reinterpret_cast<const vec*>(from + j * line + at);
      if constexpr (PAST) w[j] = __builtin_nontemporal_load(p); else w[j] = *p;
    }
#pragma unroll
    for (int p = 0; p < R; ++p)
#pragma unroll
      for (int h = 0; h < XV; ++h) xv[p][h] = *reinterpret_cast<const vec*>(x[p] + b * kFewBlock + quarter * 8 + h * VPL);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int p = 0; p < R; ++p) {
        const float f = few_at<T>(xv[p][j / VPL], j % VPL);
#pragma unroll
        for (int e = 0; e < VPL; ++e) acc[p][e] = fmaf(f, few_at<T>(w[j], e), acc[p][e]);
      }
  }
  if (K % kFewBlock && wave == whole % kFewWaves) {
    const unsigned char* const from = static_cast<const unsigned char*>(a.W) + (int64_t)whole * kFewBlock * line;
    for (int j = 0; j < 8; ++j) {
      const int k = whole * kFewBlock + quarter * 8 + j;
      if (k >= K) break;
      const u32x4 w = *reinterpret_cast<const vec*>(from + j * line + at);
#pragma unroll
      for (int p = 0; p < R; ++p) {
        const float f = ld_elem(x[p] + k);
#pragma unroll
        for (int e = 0; e < VPL; ++e) acc[p][e] = fmaf(f, few_at<T>(w, e), acc[p][e]);
      }
    }
  }

  // the quarters' sums: a lane gives half of its own away and then half of what is left, and has VPL / 4 classes in the end
  const bool upper = quarter & 2, odd = quarter & 1;
#pragma unroll
  for (int p = 0; p < R; ++p) {
    float half[VPL / 2], mine[VPL / 4];
#pragma unroll
    for (int e = 0; e < VPL / 2; ++e) {
      const float lo = acc[p][e], hi = acc[p][e + VPL / 2];
      half[e] = (upper ? hi : lo) + __shfl_xor(upper ? lo : hi, 32);
    }
#pragma unroll
    for (int e = 0; e < VPL / 4; ++e) {
      mine[e] = (odd ? half[e + VPL / 4] : half[e]) + __shfl_xor(odd ? half[e] : half[e + VPL / 4], 16);
      s_z[p][wave][slot * VPL + (upper ? VPL / 2 : 0) + (odd ? VPL / 4 : 0) + e] = mine[e];
    }
  }
  __syncthreads();

  // 64 classes of a place a wave
  const int place = __builtin_amdgcn_readfirstlane(tid / C), i = tid % C, v = c0 + i;
  if (place >= live) return;
  float z = -INFINITY;
  if (v < N) {
    const int first = i / VPL * VPL, in = first + (v - min(c0 + first, N - VPL));
    z = a.bias ? a.bias[v] : 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) z += s_z[place][w][in];
  }
  if (a.z && v < a.z_ld) a.z[(int64_t)place * a.z_ld + v] = z;
  int r = 0;
#pragma unroll
  for (int p = 0; p < R; ++p) r = place == p ? row[p] : r;
  if (a.token && v < N && a.token[r] == v) a.target[place] = z;
  const float m = wave_max(z), base = exp_base(m), l = (z - base) * a.c, e = __builtin_amdgcn_exp2f(l);
  const float s = wave_sum(e), u = wave_sum(e * fmaxf(l, kNoPower));
  const int part = (v - lane) / 64;
  if (lane == 0 && v < N) {
    *reinterpret_cast<float2*>(a.stats + ((int64_t)part * a.stats_ld + place) * 2) = make_float2(m, s);
    a.spread[(int64_t)part * a.stats_ld + place] = u;
  }
}

// A W of whole lines that is not in the last-level cache anyhow is read past the caches.  us through / past them: bf16 1 x 4096 x 128000 188 / 171,
// 1 x 2048 x 32000 (131 MB) 27.7 / 25.5, fp32 1 x 2048 x 16000 (128 MB) 27.4 / 25.2; but where lines are shared between neighbours bf16 1 x 1024 x 50257
// (103 MB) 28.0 / 29.1, and 1 x 2048 x 16000 (66 MB) 15.5 / 17.9.
constexpr int64_t kPastBytes = 96 << 20;
template <typename T, int R> hipError_t few_rows(const FewRows& a, hipStream_t st) {
  const int64_t line = a.w_ld * (int64_t)sizeof(T);
  const bool past = line * a.K >= kPastBytes && ((reinterpret_cast<uintptr_t>(a.W) | (uintptr_t)line) & 127) == 0;
  auto kern = past ? few_rows_kernel<T, R, true> : few_rows_kernel<T, R, false>;
  hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + FewTypes<T>::C - 1) / FewTypes<T>::C)), dim3(kFewThreads), 0, st, a);
  return hipGetLastError();
}
template <typename T> hipError_t few_rows(const FewRows& a, hipStream_t st) {
  if (a.rows <= 1) return few_rows<T, 1>(a, st);
  if (a.rows <= 2) return few_rows<T, 2>(a, st);
  if (a.rows <= 4) return few_rows<T, 4>(a, st);
  if constexpr (sizeof(T) == 4) return few_rows<T, 8>(a, st);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_few_rows(const FewRows& a, hipStream_t st) {
  if (a.rows < 1 || a.K < 1 || a.N < 16 || (int64_t)kFewBlock * a.w_ld * 4 >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  return a.dtype == kBF16 ? few_rows<uint16_t>(a, st) : few_rows<float>(a, st);
}

}  // namespace rad
