// Parameter updates (Section 4.3 and Appendix A, training details): plain SGD for the recurrent model, Adam for the
// feedforward ones, each with an l2 term added to the gradient as l2 * w; and the norm of many gradients together, by which
// they are clipped.  One pass over a tensor: every operand is read once and every result written once, so the kernels are HBM
// streams (SGD 8 bytes read + 4 written per fp32 parameter; Adam 16 read + 12 written, 2 more written when a bf16 copy of the
// parameter is kept; a norm reads its gradients, and the step that follows applies the clipping factor as it reads them again).
// A launch takes many tensors: each is cut into chunks, which the workgroups take in turn.
#include "kernels.hpp"

namespace rad {

namespace {

__device__ __forceinline__ uint16_t to_bf16(float f) {      // round to nearest even
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40u);
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}

// (Which product of a moment's sum is rounded ahead of it differs between whole vectors and single elements, and is spelled out: a
// parameter gets the same bits in every build.)
template <bool ADAM, bool VECTOR>
__device__ __forceinline__ float update_one(float w, float g, float& m, float& v, const OptimArgs& a) {
#pragma clang fp contract(off)
  g = fmaf(a.l2, w, g);
  if constexpr (ADAM) {
    m = VECTOR ? fmaf(a.omb1, g, a.beta1 * m) : fmaf(a.beta1, m, a.omb1 * g);
    v = VECTOR ? fmaf(g, a.omb2 * g, a.beta2 * v) : fmaf(a.beta2, v, g * (a.omb2 * g));
    const float m_hat = m * a.inv_bc1, v_hat = v * a.inv_bc2;
    return w - a.lr * m_hat / (sqrtf(v_hat) + a.eps);
  } else {
    return fmaf(-a.lr, g, w);
  }
}

// Elements of a chunk.  A step takes one vector a lane: with four, the loads of each wait behind the stores of the one before, which
// steps past the caches do not hide (us with four / one, steps after their gradients were written: SGD bf16 2400 MB 830 / 778, 6400 MB 2225 /
// 2080, fp32 545 MB 160 / 152, 6400 MB 1914 / 1790, Adam bf16 545 MB 123 / 114, 2400 MB 583 / 558).
constexpr int kStepChunk = 1024;
constexpr int kClipChunk = 4096;
constexpr int kNormThreads = 1024, kNormChunk = 16384;

// the tensor that chunk c lies in
__device__ __forceinline__ int tensor_of(const int32_t* chunk_end, int n, int c) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (c < chunk_end[mid]) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// Chunks of tensors in whole 16-byte vectors; what is left of a tensor, or a tensor at another address, element by element.
// PAST: past the caches, for steps that these cannot hold, whatever came before them.  us through / past:
//   with the norm ahead: Adam bf16 4096-4096-4096-1000 (1.1 GB) 248 / 197, 8192-8192-4096 628 / 543, SGD fp32 8192-8192-8192 387 / 334, 8192-8192-4096 295 / 246;
//   alone, after their gradients were written (the writing included): SGD fp32 of 545 MB 168 / 152, 1600 MB 483 / 444, bf16 545 MB 187 / 165, Adam bf16
//   545 MB 133 / 113, 2400 MB 604 / 552; the same step again and again: 85 / 83, 283 / 252, 113 / 95, 93 / 93, 475 / 402;
//   but SGD 4096-4096-4096-1000 in fp32 (0.45 GB), again and again, 68 / 77 (with four vectors a lane).
// Bound by memory.  (The loads alone or the stores alone gain nothing; the gradients through the caches and the rest past them: the first of these
// 191, but 8192-8192-4096 553, SGD fp32 8192-8192-8192 348.)
template <bool ADAM, bool SCALED, bool PAST>
__global__ __launch_bounds__(256) void optim_kernel(OptimList l) {
  float scale = 1.f;
  if constexpr (SCALED) {
    scale = *l.scale;
    if (scale == 0.f) return;
  }
  // (Adam after a norm begins with the gradients that the norm read last, of which the last-level cache still holds the most:
  // bf16 8192-8192-4096 with its norm 552 us from the first, 543 from the last, 4096-4096-4096-1000 200 and 197; SGD, which needs less of it
  // besides, fp32 8192-8192-4096 245 and 246.)
  const int b = ADAM && SCALED ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x;
  const int t = tensor_of(l.chunk_end, l.n, b), c = b - (t ? l.chunk_end[t - 1] : 0);
  float* const w = l.w[t]; float* const m = l.m[t]; float* const v = l.v[t];
  const float* const g = l.g[t];
  uint16_t* const lo = l.lo[t];
  const int64_t i0 = (int64_t)c * kStepChunk, n = l.count[t];
  const uintptr_t align = reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(m) |
                          reinterpret_cast<uintptr_t>(v) | (reinterpret_cast<uintptr_t>(lo) << 1);   // (8-byte vectors of the bf16 copy)
  const OptimArgs& a = l.a;
  auto grad = [&](float x) {                            // (rounded, as if the scaled gradient had been stored)
#pragma clang fp contract(off)
    if constexpr (SCALED) return x * scale; else return x;
  };
  auto ld = [](const float* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(p));
    else return *reinterpret_cast<const floatx4*>(p);
  };
  auto st = [](float* p, floatx4 x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<floatx4*>(p));
    else *reinterpret_cast<floatx4*>(p) = x;
  };
  const int64_t i = i0 + (int)threadIdx.x * 4;
  if (i >= n) return;
  if (i + 4 <= n && (align & 15) == 0) {
    floatx4 wv = ld(w + i), gv = ld(g + i), mv = {0.f, 0.f, 0.f, 0.f}, vv = mv;
    if constexpr (ADAM) { mv = ld(m + i); vv = ld(v + i); }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float me = mv[e], ve = vv[e];
      wv[e] = update_one<ADAM, true>(wv[e], grad(gv[e]), me, ve, a);
      mv[e] = me; vv[e] = ve;
    }
    st(w + i, wv);
    if constexpr (ADAM) { st(m + i, mv); st(v + i, vv); }
    if (lo) {
      const u32x2 p = {(uint32_t)to_bf16(wv[0]) | ((uint32_t)to_bf16(wv[1]) << 16), (uint32_t)to_bf16(wv[2]) | ((uint32_t)to_bf16(wv[3]) << 16)};
      *reinterpret_cast<u32x2*>(lo + i) = p;
    }
    return;
  }
  for (int64_t j = i; j < n && j < i + 4; ++j) {
    float mm = 0.f, vv = 0.f;
    if constexpr (ADAM) { mm = m[j]; vv = v[j]; }
    const float wn = update_one<ADAM, false>(w[j], grad(g[j]), mm, vv, a);
    w[j] = wn;
    if constexpr (ADAM) { m[j] = mm; v[j] = vv; }
    if (lo) lo[j] = to_bf16(wn);
  }
}

// a sum over the workgroup in a fixed order
__device__ __forceinline__ double block_sum(double s, double* s_w) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = s;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < kNormThreads / 64; ++w) all += s_w[w];
  return all;
}

// Squares and their sums are fp64: fp32's largest gradients do not overflow them, nor do its smallest vanish, and a sum of 10^9
// squares is as good as one of ten.  Each workgroup takes chunks gridDim.x apart, the same ones in every call, and the last one to
// be done adds what all have left, in their order, so that the norm takes no launch of its own.  Bound by memory: 150 MB of fp32 31 us (4.8 TB/s),
// 117 MB of bf16 out of the last-level cache 24; six small tensors 6.5, a launch and two trips to memory.
__global__ __launch_bounds__(kNormThreads) void square_sums_kernel(NormList l) {
  __shared__ double s_w[kNormThreads / 64];
  __shared__ bool s_last;
  double sum = 0.0;
  const int chunks = l.n > 0 ? l.chunk_end[l.n - 1] : 0;
  for (int b = blockIdx.x; b < chunks; b += gridDim.x) {
    const int t = tensor_of(l.chunk_end, l.n, b), c = b - (t ? l.chunk_end[t - 1] : 0);
    const int64_t i0 = (int64_t)c * kNormChunk, n = l.count[t];
    const bool half = (l.bf16[t >> 5] >> (t & 31)) & 1u, aligned = (reinterpret_cast<uintptr_t>(l.g[t]) & 15) == 0;
    if (half) {
      const uint16_t* const g = static_cast<const uint16_t*>(l.g[t]);
      auto add = [&](u32x4 v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double x = __uint_as_float(v[e] << 16), y = __uint_as_float(v[e] & 0xFFFF0000u);
          sum += x * x; sum += y * y;
        }
      };
      if (i0 + kNormChunk <= n && aligned) {                 // (all loads of a chunk in flight at once)
        u32x4 v[kNormChunk / (8 * kNormThreads)];
#pragma unroll
        for (int q = 0; q < kNormChunk / (8 * kNormThreads); ++q) v[q] = *reinterpret_cast<const u32x4*>(g + i0 + q * 8 * kNormThreads + (int)threadIdx.x * 8);
#pragma unroll
        for (int q = 0; q < kNormChunk / (8 * kNormThreads); ++q) add(v[q]);
      } else {
        for (int64_t i = i0 + (int)threadIdx.x; i < n && i < i0 + kNormChunk; i += kNormThreads) { const double x = bf16_bits_to_f32(g[i]); sum += x * x; }
      }
    } else {
      const float* const g = static_cast<const float*>(l.g[t]);
      if (i0 + kNormChunk <= n && aligned) {
        floatx4 v[kNormChunk / (4 * kNormThreads)];
#pragma unroll
        for (int q = 0; q < kNormChunk / (4 * kNormThreads); ++q) v[q] = *reinterpret_cast<const floatx4*>(g + i0 + q * 4 * kNormThreads + (int)threadIdx.x * 4);
#pragma unroll
        for (int q = 0; q < kNormChunk / (4 * kNormThreads); ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) { const double x = v[q][e]; sum += x * x; }
      } else {
        for (int64_t i = i0 + (int)threadIdx.x; i < n && i < i0 + kNormChunk; i += kNormThreads) { const double x = g[i]; sum += x * x; }
      }
    }
  }
  sum = block_sum(sum, s_w);
  double* const mine = l.partial + l.first + blockIdx.x;
  if (!l.done) { if (threadIdx.x == 0) *mine = sum; return; }
  if (threadIdx.x == 0) {
    store_for_all(mine, sum);
    stores_done();
    s_last = count_done(l.done) == gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  const int all = l.first + (int)gridDim.x;
  double total = 0.0;
  for (int i = threadIdx.x; i < all; i += kNormThreads) total += load_of_all(l.partial + i);
  __syncthreads();
  total = block_sum(total, s_w);
  if (threadIdx.x != 0) return;
  *l.done = 0u;
  const double r = sqrt(total);
  const float f = (float)r;
  if (l.norm) *l.norm = f;
  const bool finite = f < INFINITY, over = finite && r > l.max_norm;
  // (0 says that the norm is not finite, so the least scale of one that is, is the smallest subnormal number)
  if (l.scale) *l.scale = !finite ? 0.f : over ? fmaxf((float)(l.max_norm / r), 0x1p-149f) : 1.f;
  if (l.factors) {
    const int e = over && l.max_norm / r < 0x1p-126 ? max(-126, min(126, ilogb(r))) : 0;
    l.factors[0] = (float)ldexp(1.0, -e);
    l.factors[1] = over ? (float)(l.max_norm / ldexp(r, -e)) : 1.f;
  }
}

// Elements times two factors whose product is the scale: the first is 1, or, where the scale would be a subnormal number of few bits (or none:
// max_norm is less than 2^-126 of the norm), a power of two that brings them to the norm's size.  It is exact but for elements below 2^-126 of
// that, and the second, at most twice max_norm, has all its bits but where max_norm is subnormal itself.
// (Stored past the caches: 1023-4097-1000-50257 in bf16 61 us with the norm, 71 where the end of the kernel waits for them; with a kernel that reads
// the clipped gradients next, us through / past: fp32 60 MB 61 / 62, 117 MB 121 / 115, 200 MB 225 / 211, 600 MB 614 / 613, bf16 60 MB 104 / 82,
// 200 MB 296 / 287, in place the same.)  PAST: read past
// them too, where they cannot hold them: bf16 2048-4096-50000 (0.8 GB read and written) 219 us through them, 197 past, but the first 61 and 62.
template <bool PAST> __global__ __launch_bounds__(256) void clip_kernel(ClipList l) {
  const float lift = l.factors[0], f = l.factors[1];    // (1 and 1 for a norm that is not finite: the gradients as they are)
  const int t = tensor_of(l.chunk_end, l.n, blockIdx.x), c = (int)blockIdx.x - (t ? l.chunk_end[t - 1] : 0);
  if (lift == 1.f && f == 1.f && l.out[t] == l.g[t]) return;
  const int64_t i0 = (int64_t)c * kClipChunk, n = l.count[t];
  const bool half = (l.bf16[t >> 5] >> (t & 31)) & 1u;
  const bool aligned = ((reinterpret_cast<uintptr_t>(l.g[t]) | reinterpret_cast<uintptr_t>(l.out[t])) & 15) == 0;
  if (half) {
    const uint16_t* const g = static_cast<const uint16_t*>(l.g[t]);
    uint16_t* const o = static_cast<uint16_t*>(l.out[t]);
#pragma unroll
    for (int q = 0; q < kClipChunk / 2048; ++q) {
      const int64_t i = i0 + q * 2048 + (int)threadIdx.x * 8;
      if (i + 8 <= n && aligned) {
        u32x4 v;
        if constexpr (PAST) v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(g + i)); else v = *reinterpret_cast<const u32x4*>(g + i);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = (uint32_t)to_bf16(__uint_as_float(v[e] << 16) * lift * f) | ((uint32_t)to_bf16(__uint_as_float(v[e] & 0xFFFF0000u) * lift * f) << 16);
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(o + i));
      } else {
        for (int64_t j = i; j < n && j < i + 8; ++j) o[j] = to_bf16(bf16_bits_to_f32(g[j]) * lift * f);
      }
    }
    return;
  }
  const float* const g = static_cast<const float*>(l.g[t]);
  float* const o = static_cast<float*>(l.out[t]);
#pragma unroll
  for (int q = 0; q < kClipChunk / 1024; ++q) {
    const int64_t i = i0 + q * 1024 + (int)threadIdx.x * 4;
    if (i + 4 <= n && aligned) {
      floatx4 v;
      if constexpr (PAST) v = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(g + i)); else v = *reinterpret_cast<const floatx4*>(g + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * lift * f;
      __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(o + i));
    } else {
      for (int64_t j = i; j < n && j < i + 4; ++j) o[j] = g[j] * lift * f;
    }
  }
}

template <bool PAST> void optim_run(bool adam, const OptimList& l, unsigned chunks, hipStream_t st) {
  auto kern = adam ? l.scale ? optim_kernel<true, true, PAST> : optim_kernel<true, false, PAST>
                   : l.scale ? optim_kernel<false, true, PAST> : optim_kernel<false, false, PAST>;
  hipLaunchKernelGGL(kern, dim3(chunks), dim3(256), 0, st, l);
}

// fills chunk_end; their number, or -1 where a grid cannot have so many
int64_t count_chunks(int n, const int64_t* count, int32_t* chunk_end, int chunk) {
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    chunks += (count[i] + chunk - 1) / chunk;
    if (chunks >= (int64_t(1) << 24)) return -1;        // (a grid of 256 threads a workgroup: 2^32 at most)
    chunk_end[i] = (int32_t)chunks;
  }
  return chunks;
}

}  // namespace

hipError_t launch_optim(bool adam, bool past, OptimList* l, hipStream_t st) {
  const int64_t chunks = count_chunks(l->n, l->count, l->chunk_end, kStepChunk);
  if (chunks < 0) return hipErrorInvalidValue;
  if (chunks == 0) return hipSuccess;
  if (past) optim_run<true>(adam, *l, (unsigned)chunks, st); else optim_run<false>(adam, *l, (unsigned)chunks, st);
  return hipGetLastError();
}

hipError_t launch_square_sums(NormList* l, int* partials, hipStream_t st) {
  const int64_t chunks = count_chunks(l->n, l->count, l->chunk_end, kNormChunk);
  *partials = 0;
  if (chunks < 0) return hipErrorInvalidValue;
  if (chunks == 0 && !l->done) return hipSuccess;
  *partials = chunks < 1 ? 1 : chunks < kNormBlocks ? (int)chunks : kNormBlocks;
  hipLaunchKernelGGL(square_sums_kernel, dim3(*partials), dim3(kNormThreads), 0, st, *l);
  return hipGetLastError();
}

hipError_t launch_clip(bool past, ClipList* l, hipStream_t st) {
  const int64_t chunks = count_chunks(l->n, l->count, l->chunk_end, kClipChunk);
  if (chunks < 0) return hipErrorInvalidValue;
  if (chunks == 0) return hipSuccess;
  if (past) hipLaunchKernelGGL(clip_kernel<true>, dim3((unsigned)chunks), dim3(256), 0, st, *l);
  else hipLaunchKernelGGL(clip_kernel<false>, dim3((unsigned)chunks), dim3(256), 0, st, *l);
  return hipGetLastError();
}

}  // namespace rad
