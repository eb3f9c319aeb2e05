// Rows of logits in registers: what the kernels that take dense logits share.
#pragma once
#include <math.h>

#include "head_epilogue.hpp"
#include "kernels.hpp"

namespace rad {

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
  // PAST: past the caches
  template <bool PAST = false> __device__ __forceinline__ void load(const T* row, int v0, int head, int classes) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = col(v0, i, head);
      raw[i] = u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
      if (c + VPL <= classes) {
        if constexpr (PAST) raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + c));
        else raw[i] = *reinterpret_cast<const u32x4*>(row + c);
      }
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

// stores a vector of a row: f(q) is its element q; PAST: past the caches
template <typename T, bool PAST, class F> __device__ __forceinline__ void store_vector(T* out, F f) {
  typedef u32x4 u32x4_any __attribute__((aligned(2)));
  u32x4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (sizeof(T) == 4) w[q] = __float_as_uint(f(q));
    else w[q] = bf16_pair(f(2 * q), f(2 * q + 1));
  }
  u32x4_any* const to = reinterpret_cast<u32x4_any*>(out);              // (dz may be aligned otherwise)
  if constexpr (PAST) __builtin_nontemporal_store(w, to); else *to = w;
}

// stores a part of a row: f(i, q) is element q of vector i, single what the single element becomes
template <typename T, int NT, int NV, bool PAST = false, class F>
__device__ __forceinline__ void store_part(T* out, const RowPart<T, NT, NV>& p, int v0, int head, int classes, float single, F f) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = RowPart<T, NT, NV>::col(v0, i, head);
    if (c + RowPart<T, NT, NV>::VPL <= classes) store_vector<T, PAST>(out + c, [&](int q) { return f(i, q); });
    if (i % 2) __builtin_amdgcn_sched_barrier(0);
  }
  if (p.single_col >= 0) st_elem(out + p.single_col, single);
}

// a grid's x times its workgroup stays below 2^32
constexpr int kRowsX = 1 << 20;
// rows in parts: threads of a workgroup and their vectors
constexpr int kPartThreads = 256, kPartVecs = 4;

}  // namespace rad
