// Products of a layer under a loss over its classes (HeadArgs), bf16 and fp32: 128 x 128 or 64 x 128 tiles, operands straight
// into LDS as in gemm_bf16_dma.hpp, slices of 128 bytes of K (64 bf16, 32 fp32) in a ring of S stages, S - 1 of them on their way.
//
// bf16: the 256 x 256 kernel needs 256 tiles to give every CU work.  100 rows x 1024 x 10000 are 40 of them, for whose 16
// slices each CU waits alone (28 us, of which the weights' way from memory is 4); here they are 79 or 158, two to a CU, and a
// slice of the weights is asked for S - 1 slices ahead: 16 us in 128-row tiles, 13 in 64-row ones.
// fp32: bound by the matrix cores (16 products of 32 x 32 x 2 per four 16-byte reads of LDS).
#pragma once
#include "gemm_bf16_dma.hpp"

namespace rad {

// loads of one slice of an operand of R rows (256 threads, R / 32 loads of 16 bytes each):
//   K contiguous: rows of 128 bytes, chunks swizzled as in Lds64
//   M/N contiguous: k-rows of the tile's R elements as they lie in memory; bf16 ones in LdsMN's order, for the transposing reads
template <typename T, int R, bool MN> struct TileOperand {
  static constexpr int ES = sizeof(T), BK = 128 / ES;
  static constexpr int CPR = MN ? R * ES / 16 : 8, NI = R / 32, EPC = 16 / ES;     // chunks per row, loads, elements per chunk
  static_assert(!MN || ES == 4 || R >= 128, "four k-rows of a bf16 tile differ by four chunks each");
  uint32_t voff[NI];
  const unsigned char* base;
  int64_t slice_bytes;
  uint32_t wave_lds;
  static __device__ __forceinline__ int unit(int i) { return i * kGemmThreads + (int)threadIdx.x; }
  static __device__ __forceinline__ int line(int u) { return u / CPR; }            // row of the tile, or k-row of the slice
  static __device__ __forceinline__ int chunk(int u) {
    const int r = u / CPR, c = u % CPR;
    return !MN ? c ^ ((r >> 1) & 7) : ES == 2 ? c ^ (4 * (r & 3)) : c;
  }
  // rows past rmax (K contiguous; row r0 + r is row map[r] of p, where there is a map) and chunks past it (M/N contiguous, rmax whole
  // chunks) read the last one instead
  __device__ __forceinline__ void init(const void* p, int64_t ld, int r0, int kbeg, int rmax, const int32_t* map) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int u = unit(i), r = line(u);
      const uint32_t pitch = (uint32_t)ld * ES;
      if (MN) voff[i] = (uint32_t)r * pitch + (uint32_t)min(chunk(u), (rmax - r0) / EPC - 1) * 16u;
      else if (map) voff[i] = (uint32_t)map[min(r, rmax - 1 - r0)] * pitch + (uint32_t)chunk(u) * 16u;
      else voff[i] = (uint32_t)min(r, rmax - 1 - r0) * pitch + (uint32_t)chunk(u) * 16u;
    }
    base = static_cast<const unsigned char*>(p) + (MN ? (int64_t)kbeg * ld + r0 : (map ? 0 : (int64_t)r0 * ld) + kbeg) * ES;
    slice_bytes = MN ? BK * ld * ES : 128;
    wave_lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) * 1024u;
  }
  // slice s into the tile at LDS byte lds; krem: valid k from its start on (zeros behind them)
  __device__ __forceinline__ void issue(uint32_t lds, int s, int krem) const {
    const unsigned char* const from = base + (int64_t)s * slice_bytes;
    if (krem >= BK) {
#pragma unroll
      for (int i = 0; i < NI; ++i) dma16(from, voff[i], lds + wave_lds + (uint32_t)i * 4096u);
      return;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int u = unit(i);
      const bool in = MN ? line(u) < krem : chunk(u) * EPC < krem;
      dma16_aim(lds + wave_lds + (uint32_t)i * 4096u);
      asm volatile("s_nop 0");
      dma16_go_at(in ? from + voff[i] : reinterpret_cast<const unsigned char*>(kZeroChunk));
    }
  }
};

// offset of this lane's first transposing read of k-step 0 in an M/N-contiguous tile of R rows (see mn_frag_byte)
template <int R> __device__ __forceinline__ uint32_t tile_frag_byte(int row0, int lane) {
  const int s = lane & 15, grp = lane >> 4;
  const int row = row0 + 16 * (grp & 1) + 4 * (s & 3), k = 8 * (grp >> 1) + (s >> 2);
  return (uint32_t)(k * (R * 2) + (((row >> 3) ^ (4 * (k & 3))) << 4) + (row & 7) * 2);
}

template <typename T, int BM, int BN, int S> struct TileSmem {
  static constexpr int STAGE = (BM + BN) * 128, CT = BM * (BN + 16 / (int)sizeof(T)) * (int)sizeof(T);
  static constexpr int BYTES = S * STAGE > CT ? S * STAGE : CT;
};

// the matrix instructions of one slice: acc (+)= A B, or its transpose (SWAP)
template <typename T, bool AT, bool BT, int BM, int BN, int TM, int TN, bool SWAP> struct TileMma;

template <bool AT, bool BT, int BM, int BN, int TM, int TN, bool SWAP> struct TileMma<uint16_t, AT, BT, BM, BN, TM, TN, SWAP> {
  uint32_t fa[TM], fb[TN];
  __device__ __forceinline__ void init(int wm0, int wn0, int lane) {
    const int lr = lane & 31;
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i] = AT ? tile_frag_byte<BM>(wm0 + i * 32, lane) : (uint32_t)(wm0 + i * 32 + lr);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = BT ? tile_frag_byte<BN>(wn0 + j * 32, lane) : (uint32_t)(wn0 + j * 32 + lr);
  }
  __device__ __forceinline__ void run(const unsigned char* A, const unsigned char* B, int lane, floatx16 (&acc)[TM][TN]) const {
    const int lk = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      bf16x8 a[TM], b[TN];
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if constexpr (AT) a[i] = mn_frag_read(A, fa[i], ks, BM * 2);
        else a[i] = *reinterpret_cast<const bf16x8*>(A + Lds64<BM>::unit((int)fa[i], 2 * ks + lk) * 16);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        if constexpr (BT) b[j] = mn_frag_read(B, fb[j], ks, BN * 2);
        else b[j] = *reinterpret_cast<const bf16x8*>(B + Lds64<BN>::unit((int)fb[j], 2 * ks + lk) * 16);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          if constexpr (SWAP) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
          else acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
        }
    }
  }
};

// fp32: a product's order of k is free, so a lane takes four consecutive ones (lanes 0 .. 31 the first four of eight, the
// others the last four) with one read from a K-contiguous tile, one per k from an M/N-contiguous one
template <bool AT, bool BT, int BM, int BN, int TM, int TN, bool SWAP> struct TileMma<float, AT, BT, BM, BN, TM, TN, SWAP> {
  int ra, rb;
  __device__ __forceinline__ void init(int wm0, int wn0, int lane) { ra = wm0 + (lane & 31); rb = wn0 + (lane & 31); }
  template <bool MN, int R> static __device__ __forceinline__ floatx4 read(const unsigned char* tile, int row, int ks, int lk) {
    if constexpr (MN) {
      const float* const p = reinterpret_cast<const float*>(tile) + (8 * ks + 4 * lk) * R + row;
      return floatx4{p[0], p[R], p[2 * R], p[3 * R]};
    } else {
      return *reinterpret_cast<const floatx4*>(tile + Lds64<R>::unit(row, 2 * ks + lk) * 16);
    }
  }
  __device__ __forceinline__ void run(const unsigned char* A, const unsigned char* B, int lane, floatx16 (&acc)[TM][TN]) const {
    const int lk = lane >> 5;
    floatx4 a[2][TM], b[2][TN];
    auto fetch = [&](int set, int ks) {
#pragma unroll
      for (int i = 0; i < TM; ++i) a[set][i] = read<AT, BM>(A, ra + i * 32, ks, lk);
#pragma unroll
      for (int j = 0; j < TN; ++j) b[set][j] = read<BT, BN>(B, rb + j * 32, ks, lk);
    };
    fetch(0, 0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks < 3) fetch((ks + 1) & 1, ks + 1);
      const int q = ks & 1;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            if constexpr (SWAP) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[q][j][e], a[q][i][e], acc[i][j], 0, 0, 0);
            else acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[q][i][e], b[q][j][e], acc[i][j], 0, 0, 0);
          }
    }
  }
};

// workgroup `block` of split `split` of a product
template <typename T, int AKIND, int BKIND, int EPI, int BM, int BN, int S>
__device__ __forceinline__ void tile_product(const GemmArgs& g, unsigned char* smem_raw, int block, int split) {
  constexpr int TM = BM / 64, TN = BN / 64;
  constexpr bool kAT = AKIND == kOpMN, kBT = BKIND == kOpMN, kSwap = EPI == kEpiVocab;
  typedef TileOperand<T, BM, kAT> LoadA;
  typedef TileOperand<T, BN, kBT> LoadB;
  typedef TileSmem<T, BM, BN, S> Smem;
  constexpr int BK = LoadA::BK, kLoads = LoadA::NI + LoadB::NI;
  const uint32_t smem_lds = (uint32_t)reinterpret_cast<uintptr_t>(smem_raw);

  // the workgroups of an XCD (ids equal mod 8) take neighbouring tiles, in columns of up to 8 tile rows; the grid is made for
  // all rows, the tiles dealt out are those of the rows that count
  int live;
  uint32_t mine = 0u;
  int mine_at = 0;
  if (EPI == kEpiVocab && g.head.list_out) {
    __shared__ int32_t s_n[kGemmThreads / 64];
    __shared__ float2 s_w[kGemmThreads / 64];
    const bool write = block == 0 && split == 0;
    live = g.head.rows <= 4 * kGemmThreads ? own_rows<4>(g.head, g.N, s_n, s_w, write, &mine, &mine_at)
                                           : own_rows<kOwnListRows / kGemmThreads>(g.head, g.N, s_n, s_w, write, &mine, &mine_at);
  } else {
    live = *g.head.live;
  }
  const int tiles_n = (g.N + BN - 1) / BN, tiles_m = ((EPI == kEpiHeadW ? g.M : live) + BM - 1) / BM, tiles = tiles_m * tiles_n;
  if (block >= tiles) return;
  const int x = block & 7, lin = x * (tiles >> 3) + min(x, tiles & 7) + (block >> 3);
  constexpr int GM = 8;
  const int grp = lin / (GM * tiles_n), within = lin - grp * (GM * tiles_n), gh = min(GM, tiles_m - grp * GM);
  const int m0 = (grp * GM + within % gh) * BM, n0 = (within / gh) * BN;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wm0 = (w >> 1) * (BM / 2), wn0 = (w & 1) * (BN / 2);
  const int32_t* tile_rows = nullptr;                   // rows of the batch of the tile's rows
  if (EPI == kEpiVocab && g.head.list_out) {
    __shared__ int32_t s_list[BM];
    const int per = g.head.rows <= 4 * kGemmThreads ? 4 : kOwnListRows / kGemmThreads;
    for (int q0 = 0; q0 < per; q0 += 4) {
#pragma unroll
      for (int q = q0; q < q0 + 4; ++q) {
        const int at = mine_at + __popc(mine & ((1u << q) - 1u)) - m0;
        if (((mine >> q) & 1u) && (uint32_t)at < (uint32_t)BM) s_list[at] = (int)threadIdx.x * per + q;
      }
    }
    __syncthreads();
    tile_rows = s_list;
  } else if (EPI == kEpiVocab) {
    tile_rows = g.head.row_map + m0;
  }

  floatx16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int kbeg = g.k_splits > 1 ? split * g.k_split : 0;
  const int k_all = EPI == kEpiHeadW ? min(g.K, live) : g.K;
  const int kend = g.k_splits > 1 ? min(k_all, kbeg + g.k_split) : k_all;
  const int KT = max(0, (kend - kbeg + BK - 1) / BK);
  LoadA la; LoadB lb;
  if (EPI == kEpiVocab) la.init(g.A, g.lda, m0, kbeg, live, tile_rows);
  else if (EPI == kEpiHeadW) la.init(live == g.head.rows ? g.head.whole : g.A, g.lda, m0, kbeg, g.m_load, nullptr);
  else la.init(g.A, g.lda, m0, kbeg, g.M, nullptr);
  lb.init(g.B, g.ldb, n0, kbeg, kBT ? g.head.n_load : g.N, nullptr);
  auto issue = [&](int s) {
    const uint32_t at = smem_lds + (uint32_t)(s % S) * Smem::STAGE;
    const int krem = kend - kbeg - s * BK;
    la.issue(at, s, krem);
    lb.issue(at + BM * 128, s, krem);
  };
  TileMma<T, kAT, kBT, BM, BN, TM, TN, kSwap> mma;
  mma.init(wm0, wn0, lane);

#pragma unroll
  for (int s = 0; s < S - 1; ++s) if (s < KT) issue(s);
  for (int kt = 0; kt < KT; ++kt) {
    // slice kt has landed (this thread's part of it; S - 2 slices may still be on their way), and everybody is done with the
    // stage that slice kt + S - 1 goes to
    if (kt + S - 2 < KT) dma_wait<(S - 2) * kLoads>(); else dma_wait<0>();
    __syncthreads();
    if (kt + S - 1 < KT) issue(kt + S - 1);
    const unsigned char* const A = smem_raw + (kt % S) * Smem::STAGE;
    mma.run(A, A + BM * 128, lane, acc);
  }
  __syncthreads();                                      // the stages become the output tile
  T* const ct = reinterpret_cast<T*>(smem_raw);
  if constexpr (EPI == kEpiVocab) {
    if (g.k_splits > 1) { store_partial_rows<TM, TN>(g, acc, m0, n0, wm0, wn0, live, split); return; }
    epilogue_vocab<T, BM, BN, TM, TN>(g, acc, ct, m0, n0, wm0, wn0, live, tile_rows);
  } else {
    if (g.k_splits > 1) {                               // this split's partial sums, in fp32
      GemmArgs gs = g;
      gs.C = static_cast<float*>(g.C) + (int64_t)split * g.split_stride;
      epilogue_store<TM, TN, float, true, false, false, false>(gs, acc, m0, n0, wm0, wn0);
      return;
    }
    epilogue_head<EPI == kEpiHeadX, BM, BN, TM, TN>(g, acc, reinterpret_cast<uint16_t*>(ct), m0, n0, wm0, wn0,
                                                    EPI == kEpiHeadX ? live : g.M);
  }
}

template <typename T, int AKIND, int BKIND, int EPI, int BM, int BN, int S>
__global__ __launch_bounds__(kGemmThreads) void gemm_tile_kernel(GemmArgs g) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  tile_product<T, AKIND, BKIND, EPI, BM, BN, S>(g, smem_raw, blockIdx.x, blockIdx.y);
}

// dX and dW in one launch: neither waits for the other, and where rows are few neither fills the chip.  The first w_blocks
// workgroups (a multiple of 8) have dW's tiles, split by split; the others dX's.
template <typename T, int BM, int S>
__global__ __launch_bounds__(kGemmThreads) void gemm_tile_pair_kernel(GemmArgs x, GemmArgs w, int w_blocks, int w_tiles8, int x_tiles8) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  const int b = blockIdx.x;
  if (b < w_blocks) tile_product<T, kOpMN, kOpMN, kEpiHeadW, 128, 128, 2>(w, smem_raw, b % w_tiles8, b / w_tiles8);
  else tile_product<T, kOpK, kOpK, kEpiHeadX, BM, 128, S>(x, smem_raw, (b - w_blocks) % x_tiles8, (b - w_blocks) / x_tiles8);
}

}  // namespace rad
