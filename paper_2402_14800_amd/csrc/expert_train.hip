// What an expert's training step needs beside the GEMMs: operands transposed into the GEMMs' layouts, and the pass over the branches
// between the two halves of the backward GEMMs.
//
// With g = x W1^T, u = x W3^T, h = silu(g) u, y = h W2^T and the gradient dy of y:
//   dh = dy W2,  da = dh u s (1 + g (1 - s)) with s = 1 / (1 + exp(-g)),  db = dh g s,
//   dx = da W1 + db W3,  dW1 = da^T x,  dW3 = db^T x,  dW2 = dy^T h.
// The GEMMs multiply A B^T with both operands contiguous along the summed dimension, so every product but the forward's needs one or
// both operands transposed: the weights for dh and dx, and x, dy, da, db and h along the tokens for the weights' gradients.  All of
// these are passes bound by memory, over matrices that a GEMM reads many times.
//
// A thread takes a block of N x N elements (N = 8 bf16, 4 fp32: N rows of one 16-byte chunk) and transposes it in registers; lanes lie
// so that a wavefront reads whole 128-byte lines (8 or 16 chunks side by side) and writes whole 64-byte rows of the operand's blocks.
#include "common.h"

namespace moep {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;   // one 16-byte chunk
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

template <typename S> constexpr int N_OF = 16 / sizeof(S);         // elements of a chunk

// Chunk of row `row` that begins at k (a multiple of N) of an operand.  bf16: blocks of 256 rows x 32 k (gemm_packed_kernel.h), a weight's
// rows reordered inside every 32: row 8 q + 4 b + f of them lies at 16 b + 4 q + f.
template <typename S>
__device__ __forceinline__ u32x4* chunk_of(const Operand& o, int64_t row, int64_t k) {
  if constexpr (sizeof(S) == 4) return (u32x4*)(o.p + (row * o.K + k) * 4);
  int p = (int)(row & 255);
  if (o.weight) p = (p & ~31) | ((p & 4) << 2) | ((p & 24) >> 1) | (p & 3);
  const int64_t block = (row >> 8) * (o.K >> 5) + (k >> 5);
  return (u32x4*)(o.p + (block << 14) + p * 64 + ((((int)(k >> 3) & 3) ^ ((p >> 2) & 3)) << 4));
}

// in[i] = row i of the block, out[j] = its column j
template <typename S>
__device__ __forceinline__ void transposed(const u32x4 (&in)[N_OF<S>], u32x4 (&out)[N_OF<S>]) {
  if constexpr (sizeof(S) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = u32x4{in[0][j], in[1][j], in[2][j], in[3][j]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)                            // (bytes of the first row's element below those of the second's)
        out[j][q] = __builtin_amdgcn_perm(in[2 * q + 1][j >> 1], in[2 * q][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
  }
}

// Where a thread's block lies: a workgroup's wavefronts each take 64 columns x N^2 rows, 64 / N chunks side by side.
template <typename S, int THREADS = 256>
struct Place {
  int64_t r0;
  int c0;
  __device__ Place(unsigned row_block, unsigned column_block) {
    constexpr int N = N_OF<S>, SIDE = 64 / N;
    const int lane = threadIdx.x & 63;
    r0 = (int64_t)row_block * (N * N) + (lane / SIDE) * N;
    c0 = (int)column_block * THREADS + (int)(threadIdx.x >> 6) * 64 + (lane % SIDE) * N;
  }
};
template <typename S> int64_t row_blocks(int64_t rows) { return ceil_div(rows, (int64_t)N_OF<S> * N_OF<S>); }
int64_t column_blocks(int64_t columns) { return ceil_div(columns, 256); }

// Several jobs in one launch: workgroups end[j - 1] .. end[j] - 1 work on job j.  (A launch of its own each costs 2 to 4 us, as much as
// the job itself takes with a few hundred rows.)  `first`: of a launch that begins further on, where one grid does not hold them all.
template <typename J>
struct Jobs {
  J job[MAX_JOBS];
  unsigned end[MAX_JOBS];
  int n;
  unsigned first;
};
template <typename J>
__device__ __forceinline__ int find_job(const Jobs<J>& p, unsigned* block) {
  const unsigned b = blockIdx.x + p.first;
  int j = 0;
  while (j + 1 < p.n && b >= p.end[j]) ++j;
  *block = b - (j ? p.end[j - 1] : 0u);
  return j;
}
// `launch(first, n)`: workgroups of 256 first .. first + n - 1 of `blocks`, in as many launches as the grids' limit takes.
template <typename F>
int in_launches(int64_t blocks, F launch) {
  constexpr int64_t MOST = most_workgroups(256);
  for (int64_t first = 0; first < blocks; first += MOST) {
    launch(first, (unsigned)(blocks - first < MOST ? blocks - first : MOST));
    MOEP_HIP(hipGetLastError());
  }
  return MOEP_OK;
}

struct TransposeArgs {
  TransposeJob t;
  unsigned rows;                             // row blocks
};

// Reads and writes each matrix once: the two gate/up weights and the down weight of 4096 x 14336 with 8192 rows of tokens and of dy
// take 181 to 193 us, 5.4 to 5.7 TB/s, no less than a copy (5.1).  Six waves a SIMD cover a block's eight loads.
template <typename S>
__global__ __launch_bounds__(256, 6) void transpose_kernel(Jobs<TransposeArgs> jobs) {
  constexpr int N = N_OF<S>;
  unsigned block;
  const TransposeArgs& a = jobs.job[find_job(jobs, &block)];
  const TransposeJob& p = a.t;
  const Place<S> at(block % a.rows, block / a.rows);
  if (at.c0 >= p.C) return;
  u32x4 in[N], out[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    in[i] = u32x4{0, 0, 0, 0};
    const int64_t r = at.r0 + i;
    if (r < p.R) in[i] = *(const u32x4*)((const char*)p.X + (r * p.C + at.c0) * sizeof(S));
  }
  if (p.straight.p)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at.r0 + i < p.R) *chunk_of<S>(p.straight, at.r0 + i, at.c0) = in[i];
  if (p.k0 + at.r0 >= p.k_end) return;
  transposed<S>(in, out);
#pragma unroll
  for (int j = 0; j < N; ++j) *chunk_of<S>(p.out, at.c0 + j, p.k0 + at.r0) = out[j];
}

struct BranchArgs {
  const float* dh; const float* g; const float* u;
  int parts, F;
  int64_t T, part_stride;
  unsigned first;                            // row block that the launch begins with
  Operand dab, da_t, db_t, h_t;
};

template <typename S>
__device__ __forceinline__ u32x4 rounded(const float (&x)[N_OF<S>]) {
  u32x4 v;
  if constexpr (sizeof(S) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, bf16x2));
  }
  return v;
}

// Reads 12 bytes an element (dh, g, u in fp32: rounded to bf16 before this pass they would leave the gradients with twice the error of
// one rounding) and writes five chunks' worth: da, db as the A operand of dx, da, db, h along the tokens.  Bound by that, 22 bytes an
// element of bf16: 8192 x 14336 at 4.9 TB/s.  ROWS of a thread's block are asked for together, and without branches between them (rows beyond
// the last one repeat it, and are cleared): with a branch for each row and its stores in front of the next row's loads it was 4.2 TB/s.
// All rows in flight take 256 registers, one wave a SIMD; held to two waves it spills (597 us instead of 524).
// SUMMED: dh comes in several parts; few rows then, whose loads are all that the launch waits for, and workgroups of one wave, which
// reach more compute units: 8 rows of 4096 x 14336 20.7 us in workgroups of 256, 15.9 so; 8 of 1024 x 3584 18.7 / 12.6 (with its launch's
// events).  8192 x 14336 in one part is 524 / 540.
template <bool SUMMED> constexpr int BRANCH_THREADS = SUMMED ? 64 : 256;
template <typename S, bool SUMMED>
__global__ __launch_bounds__(BRANCH_THREADS<SUMMED>) void branch_gradients_kernel(BranchArgs p) {
  constexpr int N = N_OF<S>, ROWS = SUMMED ? 4 : 2;
  const Place<S, BRANCH_THREADS<SUMMED>> at(blockIdx.x + p.first, blockIdx.y);
  if (at.c0 >= p.F || at.r0 >= p.da_t.K) return;
  u32x4 a[N], b[N], h[N], out[N];
#pragma unroll
  for (int i0 = 0; i0 < N; i0 += ROWS) {
    float dh[ROWS][N], g[ROWS][N], u[ROWS][N];
    auto row = [&](int i) {
      const int64_t t = at.r0 + i0 + i;
      return (t < p.T ? t : p.T - 1) * p.F + at.c0;
    };
    auto load = [&](const float* from, int64_t e, float (&to)[N]) {
#pragma unroll
      for (int j = 0; j < N; j += 4) *(f32x4*)(to + j) = *(const f32x4*)(from + e + j);
    };
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      load(p.dh, row(i), dh[i]);
      load(p.g, row(i), g[i]);
      load(p.u, row(i), u[i]);
    }
    if (SUMMED)
#pragma unroll 2
      for (int q = 1; q < p.parts; ++q) {
        float x[ROWS][N];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) load(p.dh + q * p.part_stride, row(i), x[i]);
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) dh[i][j] += x[i][j];
      }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      float xa[N], xb[N], xh[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float s = 1.f / (1.f + __expf(-g[i][j])), silu = g[i][j] * s;
        xa[j] = dh[i][j] * u[i][j] * (s * (1.f + g[i][j] * (1.f - s)));
        xb[j] = dh[i][j] * silu;
        xh[j] = silu * u[i][j];
      }
      const bool there = at.r0 + i0 + i < p.T;
      const u32x4 zero = {0, 0, 0, 0};
      a[i0 + i] = there ? rounded<S>(xa) : zero;
      b[i0 + i] = there ? rounded<S>(xb) : zero;
      h[i0 + i] = there ? rounded<S>(xh) : zero;
    }
  }
  // (all stores after all loads: a row's would have to stay behind the stores of the row before)
  if (p.dab.p)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (at.r0 + i < p.T) {
        *chunk_of<S>(p.dab, at.r0 + i, at.c0) = a[i];
        *chunk_of<S>(p.dab, at.r0 + i, p.F + at.c0) = b[i];
      }
  if (!p.da_t.p) return;
  auto put = [&](const u32x4 (&in)[N], const Operand& o) {
    transposed<S>(in, out);
#pragma unroll
    for (int j = 0; j < N; ++j) *chunk_of<S>(o, at.c0 + j, at.r0) = out[j];
  };
  put(a, p.da_t);
  put(b, p.db_t);
  put(h, p.h_t);
}

__global__ __launch_bounds__(256) void silu_product_kernel(const f32x4* g, const f32x4* u, int64_t n, f32x4* h) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const f32x4 a = g[i], b = u[i];
  f32x4 o;
#pragma unroll
  for (int v = 0; v < 4; ++v) o[v] = a[v] / (1.f + expf(-a[v])) * b[v];
  h[i] = o;
}

template <typename S>
__global__ __launch_bounds__(256) void sum_parts_kernel(Jobs<SumJob> jobs) {
  constexpr int N = N_OF<S>;
  unsigned block;
  const SumJob& p = jobs.job[find_job(jobs, &block)];
  const int64_t i = ((int64_t)block * 256 + threadIdx.x) * N;
  if (i >= p.n) return;
  float x[N];
#pragma unroll
  for (int j = 0; j < N; j += 4) *(f32x4*)(x + j) = *(const f32x4*)(p.part + i + j);
#pragma unroll 4
  for (int q = 1; q < p.parts; ++q)
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const f32x4 y = *(const f32x4*)(p.part + q * p.stride + i + j);
#pragma unroll
      for (int v = 0; v < 4; ++v) x[j + v] += y[v];
    }
  *(u32x4*)((S*)p.out + i) = rounded<S>(x);
}

__global__ __launch_bounds__(256) void clear_kernel(u32x4* p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = u32x4{0, 0, 0, 0};
}

}  // namespace

int launch_transposes(const TransposeJob* jobs, int n, moep_dtype dt, hipStream_t s) {
  if (n < 1 || n > MAX_JOBS) return fail(MOEP_EINVAL, "transposes: %d jobs", n);
  Jobs<TransposeArgs> p = {};
  p.n = n;
  int64_t blocks = 0;
  for (int j = 0; j < n; ++j) {
    const int64_t rows = dt == MOEP_BF16 ? row_blocks<uint16_t>(jobs[j].k_end - jobs[j].k0) : row_blocks<float>(jobs[j].k_end - jobs[j].k0);
    p.job[j] = {jobs[j], (unsigned)rows};
    blocks += rows * column_blocks(jobs[j].C);
    if (blocks >= (int64_t)1 << 31) return fail(MOEP_EUNSUPPORTED, "transposes: too large");
    p.end[j] = (unsigned)blocks;
  }
  Timed t("transpose", s);
  return in_launches(blocks, [&](int64_t first, unsigned n) {
    p.first = (unsigned)first;
    if (dt == MOEP_BF16) hipLaunchKernelGGL(transpose_kernel<uint16_t>, dim3(n), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(transpose_kernel<float>, dim3(n), dim3(256), 0, s, p);
  });
}

int launch_gradients_of_branches(const float* dh, int parts, const float* g, const float* u, int64_t T, int F, moep_dtype dt, const Operand& dab,
                                 const Operand& da_t, const Operand& db_t, const Operand& h_t, hipStream_t s) {
  BranchArgs p = {dh, g, u, parts, F, T, T * (int64_t)F, 0, dab, da_t, db_t, h_t};
  if (!p.da_t.p) p.da_t.K = T;
  Timed t("branch_gradients", s);
  const int64_t rows = dt == MOEP_BF16 ? row_blocks<uint16_t>(p.da_t.K) : row_blocks<float>(p.da_t.K);
  return in_launches(rows, [&](int64_t first, unsigned n) {  // (along the rows; columns are few)
    p.first = (unsigned)first;
#define MOEP_BRANCH(S, SUMMED)                                                                                                    \
  hipLaunchKernelGGL((branch_gradients_kernel<S, SUMMED>), dim3(n, (unsigned)ceil_div(F, BRANCH_THREADS<SUMMED>)), dim3(BRANCH_THREADS<SUMMED>), 0, s, p)
    if (dt == MOEP_BF16) { if (parts > 1) MOEP_BRANCH(uint16_t, true); else MOEP_BRANCH(uint16_t, false); }
    else if (parts > 1) MOEP_BRANCH(float, true);
    else MOEP_BRANCH(float, false);
#undef MOEP_BRANCH
  });
}

int launch_silu_product(const float* g, const float* u, int64_t n, float* h, hipStream_t s) {
  Timed t("silu_product", s);
  return in_launches(ceil_div(n / 4, 256), [&](int64_t first, unsigned blocks) {
    const int64_t i = first * 256;
    hipLaunchKernelGGL(silu_product_kernel, dim3(blocks), dim3(256), 0, s, (const f32x4*)g + i, (const f32x4*)u + i, n / 4 - i, (f32x4*)h + i);
  });
}

int launch_sums(const SumJob* jobs, int n, moep_dtype dt, hipStream_t s) {
  if (n < 1) return MOEP_OK;
  if (n > MAX_JOBS) return fail(MOEP_EINVAL, "sums: %d jobs", n);
  Jobs<SumJob> p = {};
  p.n = n;
  int64_t blocks = 0;
  for (int j = 0; j < n; ++j) {
    p.job[j] = jobs[j];
    blocks += ceil_div(jobs[j].n, 256 * (dt == MOEP_BF16 ? 8 : 4));
    if (blocks >= (int64_t)1 << 31) return fail(MOEP_EUNSUPPORTED, "sums: too large");
    p.end[j] = (unsigned)blocks;
  }
  Timed t("sum_parts", s);
  return in_launches(blocks, [&](int64_t first, unsigned n) {
    p.first = (unsigned)first;
    if (dt == MOEP_BF16) hipLaunchKernelGGL(sum_parts_kernel<uint16_t>, dim3(n), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(sum_parts_kernel<float>, dim3(n), dim3(256), 0, s, p);
  });
}

int launch_clear(void* p, size_t bytes, hipStream_t s) {
  const int64_t n = (int64_t)(bytes / 16);
  if (!n) return MOEP_OK;
  const int64_t blocks = ceil_div(n, 256);
  hipLaunchKernelGGL(clear_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, (u32x4*)p, n);
  MOEP_HIP(hipGetLastError());
  return MOEP_OK;
}

}  // namespace moep
