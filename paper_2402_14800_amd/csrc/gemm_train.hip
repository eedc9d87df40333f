// The bf16 GEMMs of an expert's training step: gemm_packed_kernel with the epilogues that only this needs.  EPI_SWIGLU_KEEP also stores
// both branches before the activation, fp32, which the backward pass would otherwise have to multiply out again (4 of its 12 T H F
// flop; in bf16 they would make the gradients' error twice that of one rounding).  EPI_STORE_F32 stores the sums themselves: of a GEMM
// with too few tiles for the chip its ranges of K are taken as a batch and summed afterwards, in order.  EPI_SEVERAL: several GEMMs in one
// launch (tile_plan.h).
//
// Bound by the matrix rate under the power cap where the product is large, 8192 rows of H 4096, F 14336: gate/up with the branches 1410 to
// 1475 us (1.30 to 1.36 PFLOP/s; about 225 us of it are the 0.94 GB of branches in its epilogue), dh 655 to 705 us (1.36 to 1.47, its
// result in fp32); dx 1165 to 1210 (1.6), dW1 and dW3 1200 to 1240 (1.6), dW2 672 to 705 (1.4) have the plain epilogue.  777 rows of H 1024, F 3584: 24, 17 and 47
// us (dx and the three gradients in one launch, 0.61), one round of tiles with its fill and drain.
#include "gemm_packed_kernel.h"

namespace moep {

int allow_train_gemms() {
  for (auto allow : {allow_lds<EPI_SWIGLU_KEEP, false, true>, allow_lds<EPI_STORE_F32, false, false>, allow_lds<EPI_STORE_F32, false, true>,
                     allow_lds<EPI_SEVERAL, false, false>})
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

int launch_gemm_bf16_several(const PackedProduct* q, int n, hipStream_t s, const char* name) {
  if (n < 1 || n > SEVERAL_MAX) return fail(MOEP_EINVAL, "%s: %d GEMMs", name, n);
  KArgs k = {};
  int order[SEVERAL_MAX];
  int64_t full = 0, rows = 0;
  for (int i = 0; i < n; ++i) {
    if (q[i].M <= 0 || q[i].N <= 0 || q[i].N % 32 || q[i].ranges < 1 || q[i].K <= 0 || q[i].K % ((int64_t)64 * q[i].ranges))
      return fail(MOEP_EINVAL, "%s: M=%lld, N=%d, K=%d in %d ranges", name, (long long)q[i].M, q[i].N, q[i].K, q[i].ranges);
    if (((uintptr_t)q[i].A | (uintptr_t)q[i].B | (uintptr_t)q[i].C) & 15) return fail(MOEP_EUNSUPPORTED, "%s: operands must be 16-byte aligned", name);
    full += ceil_div(q[i].M, 256) * ceil_div(q[i].N, GEMM_BN_STORE) * q[i].ranges;
    if (q[i].M > rows) rows = q[i].M;
    int at = i;
    for (; at > 0 && q[order[at - 1]].K / q[order[at - 1]].ranges < q[i].K / q[i].ranges; --at) order[at] = order[at - 1];
    order[at] = i;
  }
  const bool half = half_width_pays(full);
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) {
    const PackedProduct& g = q[order[i]];
    KProblem& d = k.several[i];
    d.A = (const char*)g.A; d.B = (const char*)g.B; d.C = g.C;
    d.M = g.M; d.ldc = g.N; d.N = g.N; d.c_range_bytes = g.M * g.N * 4; d.f32 = g.ranges > 1;
    d.wide_nsl = g.K / 32; d.nsl = d.wide_nsl / g.ranges;
    d.m_tiles = (int)ceil_div(g.M, 256); d.n_tiles = (int)ceil_div(g.N, gemm_tile_columns(false, half));
    tiles += (int64_t)d.m_tiles * d.n_tiles * g.ranges;
    if (tiles >= (int64_t)1 << 31 || g.ranges >= 1 << 28) return fail(MOEP_EUNSUPPORTED, "%s: too many tiles", name);
    d.end = (uint32_t)tiles;
  }
  k.problems = n;
  k.m_tiles = (int)tiles; k.n_tiles = 1; k.experts = 1;      // (what the grid is made from)
  k.half_width = half ? 1 : 0;
  k.row_groups = gemm_row_groups(rows);
  Timed t(name, s);
  return launch<EPI_SEVERAL, false, false>(k, s);
}

}  // namespace moep
