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

// rows of any number; whole 16-byte vectors in every row (the caller pads copies where a tensor has others), per-thread
// offsets of 32 bits
template <typename T, int AKIND, int BKIND, int EPI> hipError_t run_head(const GemmArgs& g, hipStream_t st) {
  constexpr int EPC = 16 / (int)sizeof(T);
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || !g.head.live || g.lda % EPC || g.ldb % EPC) return hipErrorInvalidValue;
  if ((reinterpret_cast<uintptr_t>(g.A) | reinterpret_cast<uintptr_t>(g.B)) & 15) return hipErrorInvalidValue;
  if (BKIND == kOpMN && (g.head.n_load % EPC || g.head.n_load < g.N)) return hipErrorInvalidValue;
  if (AKIND == kOpMN && (g.m_load % EPC || g.m_load < g.M)) return hipErrorInvalidValue;
  if (g.k_splits > 1 && (g.k_split % 64 || g.split_stride <= 0)) return hipErrorInvalidValue;
  if (256 * g.lda * (int64_t)sizeof(T) >= (int64_t(1) << 32) || 256 * g.ldb * (int64_t)sizeof(T) >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  if (g.dry_run) return hipSuccess;
  if constexpr (sizeof(T) == 2) {
    if (g.head.tile == 256) {
      static bool prepared = false;
      return launch_sized(gemm_dma64_bf16_kernel<AKIND, BKIND, EPI, 256, 256>, &prepared, GemmDma64Smem<EPI, 256, 256>::BYTES, 256, 256, g, st);
    }
  }
  if (g.head.tile == 128) return run_tile<T, AKIND, BKIND, EPI, 128, 2>(g, st);
  if constexpr (AKIND == kOpK) { if (g.head.tile == 64) return run_tile<T, AKIND, BKIND, EPI, 64, 3>(g, st); }
  return hipErrorInvalidValue;
}
template <typename T> hipError_t run_any(int epi, const GemmArgs& g, hipStream_t st) {
  if (epi == kEpiVocab) return run_head<T, kOpK, kOpMN, kEpiVocab>(g, st);
  if (epi == kEpiHeadX) return run_head<T, kOpK, kOpK, kEpiHeadX>(g, st);
  if (epi == kEpiHeadW) return run_head<T, kOpMN, kOpMN, kEpiHeadW>(g, st);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_gemm_head(int dtype, int epi, const GemmArgs& g, hipStream_t st, const char** name) {
  static const char* const names[2][3] = {{"gemm_f32_head_fwd", "gemm_f32_head_dx", "gemm_f32_head_dw"},
                                          {"gemm_bf16_head_fwd", "gemm_bf16_head_dx", "gemm_bf16_head_dw"}};
  if (name) *name = names[dtype == kBF16][epi == kEpiVocab ? 0 : epi == kEpiHeadX ? 1 : 2];
  return dtype == kBF16 ? run_any<uint16_t>(epi, g, st) : run_any<float>(epi, g, st);
}

}  // namespace rad
