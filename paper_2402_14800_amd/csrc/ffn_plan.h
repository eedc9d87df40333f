// The plan of an expert block's training step.  Host arithmetic only, without HIP, so that a program built on the CPU can check it.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "moeprune.h"
#include "tile_plan.h"

namespace moep {

constexpr int64_t whole_steps(int64_t n, int64_t step) { return (n + step - 1) / step; }

// Bytes of an operand [rows, K] as the GEMMs read it: bf16 in blocks of 256 rows, fp32 row-major.
constexpr size_t operand_bytes(int64_t rows, int64_t K, moep_dtype dt) {
  return dt == MOEP_BF16 ? (size_t)whole_steps(rows, 256) * 256 * (size_t)K * 2 : (size_t)rows * (size_t)K * 4;
}
// Of the fp32 sums of a product in ranges of K, one [M, N] each; in one range there are none.
constexpr size_t part_bytes(int64_t M, int64_t N, int ranges) {
  return ranges > 1 ? ((size_t)ranges * (size_t)M * (size_t)N * 4 + 255) & ~(size_t)255 : 0;
}

// Ranges of K for a product of `M` x `N` outputs (tile_plan.h): bf16 tiles of 256 x 256 on as many compute units, ranges of at least
// 512; fp32 tiles of 32 x 64, four to a compute unit, ranges of at least 128.
constexpr int ranges_of(int64_t M, int64_t N, int64_t K, moep_dtype dt, bool any) {
  if (dt == MOEP_BF16) return (int)k_ranges(whole_steps(M, 256) * whole_steps(N, 256), 256, whole_steps(K, 64), 8, any);
  if (!any && K % 32) return 1;
  return (int)k_ranges(whole_steps(M, 32) * whole_steps(N, 64), 1024, whole_steps(K, 32), 4, any);
}

// The backward call's workspace.  `t_parts` ranges along the tokens for dW2, half as many (where even) for dW1 and dW3, which have
// twice the tiles; K of the transposed operands is T padded to whole ranges.
struct FfnBackwardPlan {
  bool together;                                  // the last three products in one launch (tile_plan.h)
  int dh_parts, dx_parts, t_parts, t_parts13;
  int64_t Tp, rows13;                             // rows13: rows of da^T | db^T as one operand
  size_t dy, w2t, dh, dab, w13t, x_t, dy_t, dadb_t, h_t, dx_part, w13_part, w2_part, total;
};
// false: T is too large
inline bool plan_ffn_backward(int64_t T, int H, int F, moep_dtype dt, FfnBackwardPlan* p) {
  p->dh_parts = ranges_of(T, F, H, dt, false);
  p->dx_parts = ranges_of(T, H, 2 * (int64_t)F, dt, false);
  p->t_parts = ranges_of(H, F, T, dt, true);
  p->t_parts13 = p->t_parts % 2 ? p->t_parts : p->t_parts / 2;
  const BackwardCut cut = cut_backward(T, H, F);
  p->together = dt == MOEP_BF16 && cut.together;
  if (p->together) {
    p->dx_parts = (int)cut.dx_ranges;
    p->t_parts = p->t_parts13 = (int)cut.t_ranges;
  }
  const int64_t unit = (dt == MOEP_BF16 ? 64 : p->t_parts > 1 ? 32 : 4) * (int64_t)p->t_parts;
  p->Tp = whole_steps(T, unit) * unit;
  if (p->Tp >= (int64_t)1 << 31) return false;
  p->rows13 = dt == MOEP_BF16 ? 2 * whole_steps(F, 256) * 256 : 2 * (int64_t)F;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
  p->dy = take(dt == MOEP_BF16 ? operand_bytes(T, H, dt) : 0);
  p->w2t = take(operand_bytes(F, H, dt));
  p->dh = take((size_t)p->dh_parts * T * F * 4);
  p->dab = take(operand_bytes(T, 2 * (int64_t)F, dt));
  p->w13t = take(operand_bytes(H, 2 * (int64_t)F, dt));
  p->x_t = take(operand_bytes(H, p->Tp, dt));
  p->dy_t = take(operand_bytes(H, p->Tp, dt));
  p->dadb_t = take(operand_bytes(p->rows13, p->Tp, dt));
  p->h_t = take(operand_bytes(F, p->Tp, dt));
  p->dx_part = take(part_bytes(T, H, p->dx_parts));
  p->w13_part = take(part_bytes(p->rows13, H, p->t_parts13));
  p->w2_part = take(part_bytes(H, F, p->t_parts));
  p->total = at;
  return true;
}

}  // namespace moep
