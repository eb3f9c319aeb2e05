// Products of a layer under a loss over its classes (see HeadArgs in kernels.hpp): the logits with what a softmax needs of
// them, dX and dW, on the direct-to-LDS kernels.
#include "gemm_launch.hpp"
#include "gemm_tile.hpp"

namespace rad {
namespace {

template <class K> hipError_t launch_sized(K kern, bool* prepared, int smem, int bm, int bn, const GemmArgs& g, hipStream_t st) {
  if (!*prepared) {               // one host thread drives a context
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
    *prepared = true;
  }
  return launch_gemm_kernel(kern, dim3(tiles_of(g, bm, bn), g.k_splits > 1 ? g.k_splits : 1), smem, st, g);
}
template <typename T, int AKIND, int BKIND, int EPI, int BM, int S> hipError_t run_tile(const GemmArgs& g, hipStream_t st) {
  static bool prepared = false;
  return launch_sized(gemm_tile_kernel<T, AKIND, BKIND, EPI, BM, 128, S>, &prepared, TileSmem<T, BM, 128, S>::BYTES, BM, 128, g, st);
}

template <typename T, int BM, int S> hipError_t run_pair(const GemmArgs& x, const GemmArgs& w, hipStream_t st) {
  auto kern = gemm_tile_pair_kernel<T, BM, S>;
  constexpr int sx = TileSmem<T, BM, 128, S>::BYTES, sw = TileSmem<T, 128, 128, 2>::BYTES, smem = sx > sw ? sx : sw;
  static bool prepared = false;
  if (!prepared) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
    prepared = true;
  }
  const int w8 = (tiles_of(w, 128, 128) + 7) / 8 * 8, x8 = (tiles_of(x, BM, 128) + 7) / 8 * 8;
  const int w_blocks = w8 * (w.k_splits > 1 ? w.k_splits : 1), x_blocks = x8 * (x.k_splits > 1 ? x.k_splits : 1);
  hipLaunchKernelGGL(kern, dim3(w_blocks + x_blocks), dim3(kGemmThreads), smem, st, x, w, w_blocks, w8, x8);
  return hipGetLastError();
}

// rows of any number; whole 16-byte vectors in every row (the caller pads copies where a tensor has others), per-thread
// offsets of 32 bits
template <typename T, int AKIND, int BKIND> hipError_t check_head(const GemmArgs& g) {
  constexpr int EPC = 16 / (int)sizeof(T);
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || !(g.head.live || (g.head.list_out && g.head.rows <= kOwnListRows)) || g.lda % EPC || g.ldb % EPC) return hipErrorInvalidValue;
  if ((reinterpret_cast<uintptr_t>(g.A) | reinterpret_cast<uintptr_t>(g.B)) & 15) return hipErrorInvalidValue;
  if (BKIND == kOpMN && (g.head.n_load % EPC || g.head.n_load < g.N)) return hipErrorInvalidValue;
  if (AKIND == kOpMN && (g.m_load % EPC || g.m_load < g.M)) return hipErrorInvalidValue;
  if (g.k_splits > 1 && (g.k_split % 64 || g.split_stride <= 0)) return hipErrorInvalidValue;
  if (256 * g.lda * (int64_t)sizeof(T) >= (int64_t(1) << 32) || 256 * g.ldb * (int64_t)sizeof(T) >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  return hipSuccess;
}
template <typename T, int AKIND, int BKIND, int EPI> hipError_t run_head(const GemmArgs& g, hipStream_t st) {
  const hipError_t e = check_head<T, AKIND, BKIND>(g);
  if (e != hipSuccess || g.dry_run) return e;
  if constexpr (sizeof(T) == 2) {
    if (g.head.tile == 256) {
      if (EPI == kEpiVocab && (g.head.list_out || g.k_splits > 1)) return hipErrorInvalidValue;
      static bool prepared = false;
      return launch_sized(gemm_dma64_bf16_kernel<AKIND, BKIND, EPI, 256, 256>, &prepared, GemmDma64Smem<EPI, 256, 256>::BYTES, 256, 256, g, st);
    }
  }
  // A workgroup alone on its CU has room for four stages, two for two each: x W of 4096 x 4096 x 1000 63 -> 57 us.  (In fp32
  // a slice's products take longer than its way from memory.)
  if constexpr (sizeof(T) == 2) {
    if (g.head.tile == 128 && (int64_t)tiles_of(g, 128, 128) * (g.k_splits > 1 ? g.k_splits : 1) <= 256)
      return run_tile<T, AKIND, BKIND, EPI, 128, 4>(g, st);
  }
  if (g.head.tile == 128) return run_tile<T, AKIND, BKIND, EPI, 128, 2>(g, st);
  if constexpr (AKIND == kOpK || sizeof(T) == 4) { if (g.head.tile == 64) return run_tile<T, AKIND, BKIND, EPI, 64, 3>(g, st); }
  return hipErrorInvalidValue;
}
template <typename T> hipError_t run_any(int epi, const GemmArgs& g, hipStream_t st) {
  if (epi == kEpiVocab) return run_head<T, kOpK, kOpMN, kEpiVocab>(g, st);
  if (epi == kEpiHeadX) return run_head<T, kOpK, kOpK, kEpiHeadX>(g, st);
  if (epi == kEpiHeadW) return run_head<T, kOpMN, kOpMN, kEpiHeadW>(g, st);
  return hipErrorInvalidValue;
}

template <typename T> hipError_t run_pair_any(const GemmArgs& x, const GemmArgs& w, hipStream_t st) {
  hipError_t e = check_head<T, kOpK, kOpK>(x);
  if (e == hipSuccess) e = check_head<T, kOpMN, kOpMN>(w);
  if (e != hipSuccess) return e;
  return x.head.tile == 64 ? run_pair<T, 64, 3>(x, w, st) : run_pair<T, 128, 2>(x, w, st);
}

}  // namespace

hipError_t launch_gemm_head_pair(int dtype, const GemmArgs& x, const GemmArgs& w, hipStream_t st) {
  if (x.head.tile == 256 || w.head.tile != 128) return hipErrorInvalidValue;
  return dtype == kBF16 ? run_pair_any<uint16_t>(x, w, st) : run_pair_any<float>(x, w, st);
}

hipError_t launch_gemm_head(int dtype, int epi, const GemmArgs& g, hipStream_t st, const char** name) {
  static const char* const names[2][3] = {{"gemm_f32_head_fwd", "gemm_f32_head_dx", "gemm_f32_head_dw"},
                                          {"gemm_bf16_head_fwd", "gemm_bf16_head_dx", "gemm_bf16_head_dw"}};
  if (name) *name = names[dtype == kBF16][epi == kEpiVocab ? 0 : epi == kEpiHeadX ? 1 : 2];
  return dtype == kBF16 ? run_any<uint16_t>(epi, g, st) : run_any<float>(epi, g, st);
}

}  // namespace rad
