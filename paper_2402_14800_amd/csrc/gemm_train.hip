// The bf16 GEMMs of an expert's training step: gemm_packed_kernel with the epilogues that only this needs.  EPI_SWIGLU_KEEP also stores
// both branches before the activation, fp32, which the backward pass would otherwise have to multiply out again (4 of its 12 T H F
// flop; in bf16 they would make the gradients' error twice that of one rounding).  EPI_STORE_F32 stores the sums themselves: of a GEMM
// with too few tiles for the chip its ranges of K are taken as a batch and summed afterwards, in order.
#include "gemm_packed_kernel.h"

namespace moep {

int allow_train_gemms() {
  for (auto allow : {allow_lds<EPI_SWIGLU_KEEP, false, true>, allow_lds<EPI_STORE_F32, false, false>, allow_lds<EPI_STORE_F32, false, true>})
    if (int st = allow()) return st;
  return MOEP_OK;
}

int launch_gemm_bf16_train(const PackedGemmArgs& g, hipStream_t s, const char* name) {
  KArgs k;
  if (int st = gemm_arguments(g, name, &k)) return st;
  if (!k.m_tiles) return MOEP_OK;
  if (g.tile_expert) return fail(MOEP_EINVAL, "%s: no grouped form", name);
  Timed t(name, s);
  if (g.epilogue == EPI_SWIGLU_KEEP && g.b_row_major) return launch<EPI_SWIGLU_KEEP, false, true>(k, s);
  if (g.epilogue == EPI_STORE_F32) return g.b_row_major ? launch<EPI_STORE_F32, false, true>(k, s) : launch<EPI_STORE_F32, false, false>(k, s);
  return fail(MOEP_EINVAL, "%s: unsupported epilogue %d", name, g.epilogue);
}

}  // namespace moep
