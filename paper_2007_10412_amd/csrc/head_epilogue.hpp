// Epilogues of the products of a layer under a loss over its classes (see HeadArgs): four waves, two by two on a tile.
#pragma once
#include "gemm.hpp"

namespace rad {

// What row gradients are divided by and the products multiplied by at their ends (row weights w of the rows that count): T x the
// largest |w|.  Not where that is infinite or NaN, whose rows would take the others' gradients with them, nor where rows whose
// weight is below 2^-60 of a factor above 1 would lose theirs to underflow; then 1, and each row has its own weight.
struct WeightRange {
  float most = 0.f, least = INFINITY;                      // of |w|; infinite or NaN: infinity; zeros are not among the least
  __device__ __forceinline__ void add(float w) {
    w = fabsf(w);
    most = fmaxf(most, w < INFINITY ? w : INFINITY);
    if (w > 0.f) least = fminf(least, w);
  }
  __device__ __forceinline__ void join(float m, float l) { most = fmaxf(most, m); least = fminf(least, l); }
  __device__ __forceinline__ void join_wave() {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) join(__shfl_xor(most, o), __shfl_xor(least, o));
  }
  __device__ __forceinline__ float common(float T) const {
    const float f = T * most;
    return f > 0.f && f < INFINITY && (f <= 1.f || least >= most * 0x1p-60f) ? f : 1.f;
  }
};

// sum_j p_j (z_j - base) over a row's targets of p > 0, base the largest of their logits: with it a loss is (lse - base) minus this
// sum, and nothing large cancels, whichever targets a mask of the type's lowest value has taken out (from the first target's
// logit, masked so and of probability 0, the loss came out as -8e31).
struct TargetSum {
  float base = -INFINITY, mass = 0.f, dot = 0.f;
  __device__ __forceinline__ void add(float p, float z) {
    if (z == -INFINITY) { dot = -INFINITY; return; }       // (such a target costs infinity)
    if (z > base) {
      if (mass > 0.f) dot += mass * (base - z);
      base = z;
    }
    mass += p;
    dot += p * (z - base);
  }
  __device__ __forceinline__ void join(float b, float m, float d) {
    const float most = fmaxf(base, b);
    if (mass > 0.f) dot += mass * (base - most);
    if (m > 0.f) d += m * (b - most);
    base = most; mass += m; dot += d;
  }
  __device__ __forceinline__ void join_lane(int o) { join(__shfl_xor(base, o), __shfl_xor(mass, o), __shfl_xor(dot, o)); }
  __device__ __forceinline__ void put(float3* to) const { *to = make_float3(base, mass, dot); }
  __device__ __forceinline__ void join(const float3& o) { join(o.x, o.y, o.z); }
  __device__ __forceinline__ float from() const { return base == -INFINITY ? 0.f : base; }
};

// The rows that count, made into a list by a workgroup for itself: a thread has PER consecutive rows, of which `mine` count, the
// first of them at place `at`.  Returns their number; the workgroup that writes leaves the whole list in memory.
// s_n: a word a wave; s_w: a pair.
template <int PER>
__device__ __forceinline__ int own_rows(const HeadArgs& h, int classes, int32_t* s_n, float2* s_w, bool write, uint32_t* mine_out, int* at_out) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r0 = (int)threadIdx.x * PER;
  uint32_t mine = 0u;
#pragma unroll
  for (int q = 0; q < PER; ++q)
    if (r0 + q < h.rows && (h.labels ? (uint32_t)h.labels[r0 + q] < (uint32_t)classes : h.counts[r0 + q] != 0)) mine |= 1u << q;
  const int n = __popc(mine);
  int up = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(up, o); if (lane >= o) up += v; }
  if (lane == 63) s_n[w] = up;
  if (write && h.weight) {
    WeightRange of;
#pragma unroll
    for (int q = 0; q < PER; ++q) if ((mine >> q) & 1u) of.add(h.weight[r0 + q]);
    of.join_wave();
    if (lane == 0) s_w[w] = make_float2(of.most, of.least);
  }
  __syncthreads();
  int at = up - n, all = 0;
#pragma unroll
  for (int q = 0; q < kGemmThreads / 64; ++q) { if (q < w) at += s_n[q]; all += s_n[q]; }
  *mine_out = mine; *at_out = at;
  if (write) {
    if (threadIdx.x == 0) {
      const float inv = h.inv_count_out ? (all > 0 ? 1.f / (float)all : 0.f) : h.weight ? 0.f : *h.inv_count;
      WeightRange of;
      if (h.weight) for (int q = 0; q < kGemmThreads / 64; ++q) of.join(s_w[q].x, s_w[q].y);
      *h.live_out = all;
      if (h.inv_count_out) *h.inv_count_out = inv;
      *h.common_out = h.weight ? of.common(h.temperature) : h.temperature * inv;
    }
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int r = r0 + q;
      if (r >= h.rows) break;
      const bool c = (mine >> q) & 1u;
      h.list_out[c ? at : all + (r - at)] = r;                 // (r - at rows before this one do not count)
      at += c ? 1 : 0;
    }
  }
  return all;
}

// fp32 pair -> two bf16 (round to nearest even) in one word
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  uint16_t p[2];
  put_pair(p, a, b);
  return (uint32_t)p[0] | ((uint32_t)p[1] << 16);
}

// two distances below a maximum, as shares of the range, to 16 bits each (round to nearest; clamped to [0, 1])
constexpr float kCodeRange = 128.f;
constexpr uint32_t kCodeLast = 65535u;
__device__ __forceinline__ uint32_t code_pair(float a, float b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  union { u16x2 v; uint32_t w; } u;
  u.v = __builtin_amdgcn_cvt_pknorm_u16(a, b);
  return u.w;
}

// rows and columns of a tile in LDS to global memory, 16 bytes a lane: row r of the tile goes to row place(r) of C
template <typename T, int BM, int BN, class PLACE>
__device__ __forceinline__ void store_tile(const T* ct, T* C, int64_t ldc, int rows, int n0, int N, PLACE place) {
  constexpr int VPL = 16 / (int)sizeof(T), CP = BN + VPL, CPR = BN / VPL, NV = BM * CPR / kGemmThreads;
#pragma unroll
  for (int it = 0; it < NV; ++it) {
    const int c = (int)threadIdx.x + it * kGemmThreads;
    const int r = c / CPR, ch = c % CPR, col = n0 + ch * VPL;
    if (r >= rows || col >= N) continue;
    const u32x4 v = *reinterpret_cast<const u32x4*>(&ct[r * CP + ch * VPL]);
    T* const dst = C + (int64_t)place(r) * ldc + col;
    if (col + VPL <= N) {
      __builtin_memcpy(dst, &v, 16);                       // (at element alignment: rows of any width)
    } else {
      const T* ve = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int e = 0; e < VPL; ++e) if (col + e < N) dst[e] = ve[e];
    }
  }
}

// bf16: the logits z = acc + bias never leave the registers.  What does, per row and part of its columns (a wave's: 128, or 64 in
// smaller tiles): their maximum m and the sum of
// 2^((z - m) c) in fp32, the targets' logits, and, where there is a backward pass, how far every logit lies below m, as
// 16 bits of a range of 128 powers of two (y, rows ldy apart, columns up to ldy; the last code stands for anything lower,
// whose exponential is zero in fp32 too).  A step of that code is 2^-9 of a power of two, 0.04 % rms of a probability, a
// quarter of what rounding the exponentials themselves to bf16 would cost, and they would be rounded once more when their
// row's sum is known: dW of 4096 x 4096 x 128000 was 0.29 % rms off that way, against 0.17 % of a sum rounded once.
// fp32: the logits themselves take the place of the codes.
// The product is transposed (lane = row of the tile): a row's 64 values are one lane's, so maximum and sum take one exchange
// between the two lanes that share the row.
template <typename T, int BM, int BN, int TM, int TN>
__device__ __forceinline__ void epilogue_vocab(const GemmArgs& g, floatx16 (&acc)[TM][TN], T* ct, int m0, int n0, int wm0,
                                               int wn0, int live, const int32_t* tile_rows) {
  constexpr bool kCodes = sizeof(T) == 2;
  constexpr int CP = BN + 16 / (int)sizeof(T), kPart = 32 * TN;            // a wave's columns are one part of a row
  const HeadArgs& h = g.head;
  const int lane = threadIdx.x & 63, lr = lane & 31, hh = lane >> 5;
  const int nw = n0 + wn0, part = nw / kPart;
  const float c = h.c, c_code = -c / kCodeRange;
  if (g.bias) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int cb = nw + j * 32 + q * 8 + hh * 4;
        float b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = g.bias[min(cb + e, g.N - 1)];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
        if (q & 1) __builtin_amdgcn_sched_barrier(0);        // (a few values of the bias in registers at a time)
      }
  }
  if (nw + kPart > g.N) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool out = nw + j * 32 + acc_row(e, lane) >= g.N;
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j][e] = out ? -INFINITY : acc[i][j][e];
      }
  }
  // Targets t0 .. t1 - 1 of each row lie among these columns, the first of them in column next.  That takes three loads, each of
  // which waits for the one before: in bf16 they are made for all rows at once, as a wave has nothing else to do meanwhile
  // (4096 x 2048 x 32000 with lists of 32 1536 -> 1524 us); in fp32 the registers for it cost more (1024 x 512 x 8003 254 -> 266).
  int row[TM], t0[TM], t1[TM], next[TM];
  auto find = [&](int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; ++i) {
      const int r = wm0 + i * 32 + lr;
      row[i] = m0 + r < live && nw < g.N ? tile_rows[r] : -1;   // (the last tile may reach a whole part past the classes)
      t0[i] = 0; t1[i] = 0; next[i] = -1;
    }
    if (h.labels) {
#pragma unroll
      for (int i = i0; i < i1; ++i) {
        if (row[i] >= 0) next[i] = h.labels[row[i]] - nw;
        t1[i] = (uint32_t)next[i] < (uint32_t)kPart ? 1 : 0;
      }
      return;
    }
#pragma unroll
    for (int i = i0; i < i1; ++i)
      if (row[i] >= 0) {
        const uint16_t* const f = h.first + (int64_t)row[i] * h.first_ld + part;
        t0[i] = f[0]; t1[i] = f[1];
      }
#pragma unroll
    for (int i = i0; i < i1; ++i)
      if (t0[i] < t1[i]) next[i] = h.index[(int64_t)row[i] * h.k + t0[i]] - nw;
  };
  if constexpr (kCodes) find(0, TM);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if constexpr (!kCodes) find(i, i + 1);
    const int place = m0 + wm0 + i * 32 + lr;
    for (int t = t0[i]; __any(t < t1[i]); ++t) {
      const int col = t < t1[i] ? next[i] : -1;
      if (t + 1 < t1[i]) next[i] = h.index[(int64_t)row[i] * h.k + t + 1] - nw;
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) z = col == j * 32 + acc_row(e, lane) ? acc[i][j][e] : z;
      if (col >= 0 && ((col >> 2) & 1) == hh) h.target[(int64_t)place * h.k + t] = z;
    }
    float m = -INFINITY, s = 0.f;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
    m = fmaxf(m, __shfl_xor(m, 32));
    const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float d = acc[i][j][e] - from;
        s += __builtin_amdgcn_exp2f(d * c);
        if (kCodes) acc[i][j][e] = d * c_code;
      }
    s += __shfl_xor(s, 32);
    if (row[i] >= 0 && hh == 0) *reinterpret_cast<float2*>(h.stats + ((int64_t)part * h.stats_ld + place) * 2) = make_float2(m, s);
    if (g.y) {
      T* const crow = ct + (wm0 + i * 32 + lr) * CP + wn0 + hh * 4;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float v0 = acc[i][j][4 * q], v1 = acc[i][j][4 * q + 1], v2 = acc[i][j][4 * q + 2], v3 = acc[i][j][4 * q + 3];
          if constexpr (kCodes) *reinterpret_cast<u32x2*>(crow + j * 32 + q * 8) = u32x2{code_pair(v0, v1), code_pair(v2, v3)};
          else *reinterpret_cast<floatx4*>(crow + j * 32 + q * 8) = floatx4{v0, v1, v2, v3};
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (!g.y) return;
  __syncthreads();
  store_tile<T, BM, BN>(ct, static_cast<T*>(g.y), g.ldy, live - m0, n0, (int)g.ldy, [&](int r) { return m0 + r; });
}

// a transposed tile's partial sums, four columns of a row a lane (rows are whole vectors)
template <int TM, int TN>
__device__ __forceinline__ void store_partial_rows(const GemmArgs& g, floatx16 (&acc)[TM][TN], int m0, int n0, int wm0, int wn0, int live,
                                                   int split) {
  const int lane = threadIdx.x & 63, lr = lane & 31, hh = lane >> 5;
  float* const C = static_cast<float*>(g.C) + (int64_t)split * g.split_stride;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int place = m0 + wm0 + i * 32 + lr;
    if (place >= live) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = n0 + wn0 + j * 32 + q * 8 + hh * 4;
        if (col < g.ldc)
          *reinterpret_cast<floatx4*>(C + (int64_t)place * g.ldc + col) =
              floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      }
  }
}

// dX (rows sent to their places in the batch) and dW in bf16 through LDS, or in fp32 as they are
template <bool X, int BM, int BN, int TM, int TN>
__device__ __forceinline__ void epilogue_head(const GemmArgs& g, floatx16 (&acc)[TM][TN], uint16_t* ct, int m0, int n0, int wm0,
                                              int wn0, int rows) {
  const int lane = threadIdx.x & 63;
  const float common = *g.head.common;                   // (partial sums of either return before)
  if (g.c_dtype == kF32) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int place = m0 + wm0 + i * 32 + acc_row(e, lane);
        if (place >= rows) continue;
        float* const dst = static_cast<float*>(g.C) + (int64_t)(X ? g.head.row_map[place] : place) * g.ldc + n0 + wn0 + (lane & 31);
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if (n0 + wn0 + j * 32 + (lane & 31) < g.N) dst[j * 32] = acc[i][j][e] * common + (!X && g.beta ? dst[j * 32] : 0.f);
      }
    return;
  }
  constexpr int CP = BN + 8;
  uint16_t* const cbase = ct + (wm0 + 4 * (lane >> 5)) * CP + wn0 + (lane & 31);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const int r0 = i * 32 + (e >> 2) * 8 + (e & 3);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        uint16_t st[2];
        put_pair(st, acc[i][j][e] * common, acc[i][j][e + 1] * common);
        cbase[r0 * CP + j * 32] = st[0];
        cbase[(r0 + 1) * CP + j * 32] = st[1];
      }
    }
  __syncthreads();
  store_tile<uint16_t, BM, BN>(ct, static_cast<uint16_t*>(g.C), g.ldc, rows - m0, n0, g.N,
                                    [&](int r) { return X ? g.head.row_map[m0 + r] : m0 + r; });
}

}  // namespace rad
