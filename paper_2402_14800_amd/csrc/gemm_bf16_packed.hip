// The bf16 GEMMs of the expert pass and of the routed layers (gemm_packed_kernel.h), the packing of their operands, and the
// launches' arguments.
#include "gemm_packed_kernel.h"

namespace moep {
namespace {

// ---- packing ---------------------------------------------------------------------------------
// mode 0: A operand, block row p of tile t = source row 256 t + p.
// mode 1: weight, 256 output columns per tile: block row p = row 256 t + perm32(p) of W0.
// mode 2: gate/up weight pair, 128 output columns per tile: block row p < 128 = row 128 t + perm32(p) of
//         W0, block row p >= 128 = row 128 t + perm32(p - 128) of W1.
// mode 3: gathered A operand of a grouped GEMM: block row p of tile t = source row rows_of[tile_row0[t] + p]
//         (the rows routed to the tile's expert, Sec. 3.3); tiles beyond the number in use are left alone, and so are
//         the rows that the launch's bodies do not fetch (16 rows x 2 for each of tile_order's row groups).
// Rows beyond the last one re-read the last row (their products are never stored).
// One workgroup moves a pair of slices (64 k-values) of one tile, so that whole 128-byte lines are read;
// blockIdx.z selects the expert of a weight stack.
struct PackArgs {
  const u32x4* W0; const u32x4* W1;
  u32x4* dst;
  int64_t ld_chunks;      // source leading dimension in 16-byte chunks
  int64_t rows;           // valid source rows (modes 0..2)
  int64_t src_expert_chunks, dst_expert_chunks;   // per-expert strides (blockIdx.z)
  const int32_t* rows_of; const int32_t* tile_expert; const int32_t* tile_row0; const int32_t* seg_end;
  const int32_t* tiles_in_use; const uint32_t* tile_order;
  int nsl;                // K / 32
  int mode;
};

__global__ __launch_bounds__(256) void pack_kernel(PackArgs p) {
  const int t = blockIdx.x;
  const int sp = blockIdx.y;                 // slice pair
  const u32x4* W0 = p.W0 + (int64_t)blockIdx.z * p.src_expert_chunks;
  const u32x4* W1 = p.W1 + (int64_t)blockIdx.z * p.src_expert_chunks;
  u32x4* dst = p.dst + (int64_t)blockIdx.z * p.dst_expert_chunks;
  int64_t g_row0 = 0, g_end = 0;
  int groups = 8;
  if (p.mode == 3) {
    if (t >= *p.tiles_in_use) return;
    groups = (int)p.tile_order[TILE_ORDER_ROW_GROUPS];
    g_row0 = p.tile_row0[t];
    g_end = p.seg_end[p.tile_expert[t]];
  }
  auto move = [&](auto pieces) {             // of 32 rows; a loop of its own for each number, all its loads in flight together
#pragma unroll
    for (int it = 0; it < decltype(pieces)::value; ++it) {
      const int q = it * 256 + threadIdx.x;    // 2048 chunks: 256 rows x 8 chunks of a 128-byte line
      const int row = q >> 3, c8 = q & 7;
      const u32x4* src = W0;
      int64_t r;
      if (p.mode == 3) {
        int64_t slot = g_row0 + row;
        if (slot >= g_end) slot = g_end - 1;
        r = p.rows_of[slot];
      } else {
        if (p.mode == 0) r = (int64_t)t * 256 + row;
        else if (p.mode == 1) r = (int64_t)t * 256 + perm32(row);
        else {
          r = (int64_t)t * 128 + perm32(row & 127);
          if (row >= 128) src = W1;
        }
        if (r >= p.rows) r = p.rows - 1;
      }
      const u32x4 v = src[r * p.ld_chunks + (int64_t)sp * 8 + c8];
      const int s = 2 * sp + (c8 >> 2);
      const int pos = (c8 & 3) ^ ((row >> 2) & 3);
      dst[((int64_t)t * p.nsl + s) * 1024 + row * 4 + pos] = v;
    }
  };
  if (groups > 6) move(std::integral_constant<int, 8>{});
  else if (groups > 4) move(std::integral_constant<int, 6>{});
  else move(std::integral_constant<int, 4>{});
}

// Per-device launch state, filled on a device's first launch under a mutex (first calls from several host threads are
// safe): the compute-unit count, and whether the dynamic LDS limits have been raised.  They are raised for EVERY expert
// GEMM at once, so that after one call at any size a call at any other only launches (and can be captured).
constexpr int kMaxDevices = 64;
struct DeviceState {
  int compute_units = 0;
  bool ready = false;
};
std::mutex g_dev_mu;
DeviceState g_dev[kMaxDevices];

int launch_pack(PackArgs p, int64_t tiles, int K, int experts, hipStream_t s, const char* name) {
  if (K <= 0 || K % 64) return fail(MOEP_EUNSUPPORTED, "%s: K=%d must be a positive multiple of 64", name, K);
  if (tiles <= 0 || experts <= 0) return MOEP_OK;
  if (((uintptr_t)p.W0 | (uintptr_t)p.W1 | (uintptr_t)p.dst) & 15)
    return fail(MOEP_EUNSUPPORTED, "%s: operands must be 16-byte aligned", name);
  if (tiles >= ((int64_t)1 << 31) || K / 64 > 65535 || experts > 65535) return fail(MOEP_EUNSUPPORTED, "%s: too large", name);
  p.nsl = K / 32;
  Timed t(name, s);
  hipLaunchKernelGGL(pack_kernel, dim3((unsigned)tiles, K / 64, experts), dim3(256), 0, s, p);
  MOEP_HIP(hipGetLastError());
  return MOEP_OK;
}

}  // namespace

int gemm_device_ready(int* compute_units) {
  int dev = 0;
  MOEP_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(MOEP_EUNSUPPORTED, "device ordinal %d beyond %d", dev, kMaxDevices - 1);
  std::lock_guard<std::mutex> lk(g_dev_mu);
  DeviceState& d = g_dev[dev];
  if (!d.ready) {
    int v = 0;
    MOEP_HIP(hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev));
    d.compute_units = v > 0 ? v : 256;
    for (auto allow : {allow_lds<EPI_STORE, false, false>, allow_lds<EPI_STORE, false, true>, allow_lds<EPI_STORE, true, false>,
                       allow_lds<EPI_STORE, true, true>, allow_lds<EPI_SWIGLU, false, false>, allow_lds<EPI_SWIGLU, false, true>,
                       allow_lds<EPI_SWIGLU, true, false>, allow_lds<EPI_SWIGLU, true, true>,
                       allow_lds<EPI_ROWSCALE_F32, true, false>, allow_lds<EPI_ROWSCALE_F32, true, true>})
      if (int st = allow()) return st;
    if (int st = allow_train_gemms()) return st;
    d.ready = true;
  }
  if (compute_units) *compute_units = d.compute_units;
  return MOEP_OK;
}

size_t packed_a_bytes(int64_t rows, int K) {
  return (size_t)ceil_div(rows, 256) * 256 * (size_t)K * 2;
}

size_t packed_b_bytes(int N, int K, bool gate_up_pair) {
  return (size_t)ceil_div(N, gate_up_pair ? 128 : 256) * 256 * (size_t)K * 2;
}

int launch_pack_a_bf16(const void* X, int64_t ld, int64_t rows, int K, void* dst, hipStream_t s, const char* name) {
  if (ld % 8) return fail(MOEP_EUNSUPPORTED, "%s: leading dimension must be a multiple of 8", name);
  PackArgs p = {};
  p.W0 = (const u32x4*)X; p.dst = (u32x4*)dst; p.ld_chunks = ld / 8; p.rows = rows; p.mode = 0;
  return launch_pack(p, ceil_div(rows, 256), K, 1, s, name);
}

int launch_pack_a_gathered_bf16(const void* X, int64_t ld, const int32_t* rows_of, const int32_t* tile_expert,
                                const int32_t* tile_row0, const int32_t* seg_end, const int32_t* tiles_in_use,
                                const uint32_t* tile_order, int64_t max_tiles, int K, void* dst, hipStream_t s, const char* name) {
  if (ld % 8) return fail(MOEP_EUNSUPPORTED, "%s: leading dimension must be a multiple of 8", name);
  PackArgs p = {};
  p.W0 = (const u32x4*)X; p.dst = (u32x4*)dst; p.ld_chunks = ld / 8; p.mode = 3;
  p.rows_of = rows_of; p.tile_expert = tile_expert; p.tile_row0 = tile_row0; p.seg_end = seg_end;
  p.tiles_in_use = tiles_in_use; p.tile_order = tile_order;
  return launch_pack(p, max_tiles, K, 1, s, name);
}

int launch_pack_b_bf16(const void* W0, const void* W1, int N, int K, int experts, void* dst, hipStream_t s,
                       const char* name) {
  PackArgs p = {};
  p.W0 = (const u32x4*)W0; p.W1 = (const u32x4*)W1; p.dst = (u32x4*)dst;
  p.ld_chunks = K / 8; p.rows = N; p.mode = W1 ? 2 : 1;
  p.src_expert_chunks = (int64_t)N * (K / 8);
  p.dst_expert_chunks = (int64_t)(packed_b_bytes(N, K, W1 != nullptr) / 16);
  return launch_pack(p, ceil_div(N, W1 ? 128 : 256), K, experts, s, name);
}

int launch_gemm_bf16_packed(const PackedGemmArgs& g, hipStream_t s, const char* name) {
  KArgs k;
  if (int st = gemm_arguments(g, name, &k)) return st;
  if (!k.m_tiles) return MOEP_OK;
  const bool grouped = g.tile_expert != nullptr;
  Timed t(name, s);
#define MOEP_GEMM_CASE(EPI, GROUPED) \
  return g.b_row_major ? launch<EPI, GROUPED, true>(k, s) : launch<EPI, GROUPED, false>(k, s)
  if (grouped) {
    switch (g.epilogue) {
      case EPI_STORE: MOEP_GEMM_CASE(EPI_STORE, true);
      case EPI_SWIGLU: MOEP_GEMM_CASE(EPI_SWIGLU, true);
      case EPI_ROWSCALE_F32: MOEP_GEMM_CASE(EPI_ROWSCALE_F32, true);
    }
  } else {
    switch (g.epilogue) {
      case EPI_STORE: MOEP_GEMM_CASE(EPI_STORE, false);
      case EPI_SWIGLU: MOEP_GEMM_CASE(EPI_SWIGLU, false);
    }
  }
#undef MOEP_GEMM_CASE
  return fail(MOEP_EINVAL, "%s: unsupported epilogue %d", name, g.epilogue);
}

}  // namespace moep
