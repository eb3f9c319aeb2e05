// bf16 products of a layer under a loss over its classes (see HeadArgs in kernels.hpp): the logits with the softmax's
// exponentials, dX and dW, on the direct-to-LDS kernels.
#include "gemm_launch.hpp"

namespace rad {
namespace {

// rows of any number; whole 16-byte vectors in every row (the caller pads copies where a tensor has others), per-thread
// offsets of 32 bits
template <int AKIND, int BKIND, int EPI> hipError_t run_head(const GemmArgs& g, hipStream_t st) {
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || !g.head.live || g.lda % 8 || g.ldb % 8) return hipErrorInvalidValue;
  if ((reinterpret_cast<uintptr_t>(g.A) | reinterpret_cast<uintptr_t>(g.B)) & 15) return hipErrorInvalidValue;
  if (BKIND == kOpMN && (g.head.n_load % 8 || g.head.n_load < g.N)) return hipErrorInvalidValue;
  if (AKIND == kOpMN && (g.m_load % 8 || g.m_load < g.M)) return hipErrorInvalidValue;
  if (g.k_splits > 1 && (g.k_split % 64 || g.split_stride <= 0)) return hipErrorInvalidValue;
  if (256 * g.lda * 2 >= (int64_t(1) << 32) || 256 * g.ldb * 2 >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  if (g.dry_run) return hipSuccess;
  auto kern = gemm_dma64_bf16_kernel<AKIND, BKIND, EPI, 256, 256>;
  constexpr int smem = GemmDma64Smem<EPI, 256, 256>::BYTES;
  static bool prepared = false;   // one host thread drives a context
  if (!prepared) {
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
    prepared = true;
  }
  return launch_gemm_kernel(kern, dim3(tiles_of(g, 256, 256), g.k_splits > 1 ? g.k_splits : 1), smem, st, g);
}

}  // namespace

hipError_t launch_gemm_bf16_head(int epi, const GemmArgs& g, hipStream_t st, const char** name) {
  if (epi == kEpiVocab) { if (name) *name = "gemm_bf16_head_fwd"; return run_head<kOpK, kOpMN, kEpiVocab>(g, st); }
  if (epi == kEpiHeadX) { if (name) *name = "gemm_bf16_head_dx"; return run_head<kOpK, kOpK, kEpiHeadX>(g, st); }
  if (epi == kEpiHeadW) { if (name) *name = "gemm_bf16_head_dw"; return run_head<kOpMN, kOpMN, kEpiHeadW>(g, st); }
  return hipErrorInvalidValue;
}

}  // namespace rad
