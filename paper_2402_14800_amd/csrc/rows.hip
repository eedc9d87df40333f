// A token's row on its way to the experts and back (moe_dispatch_rows, moe_combine_rows, and their gradients).
//
// Slot (t, j) of a token that uses it gets a number slot(t, j), counted by expert, within an expert by token, within a token by j:
//   dispatch: rows[slot(t, j)] = x[t]             gradient: dx[t] = sum_j drows[slot(t, j)]
//   combine:  out[t] = sum_j w[t, j] y[slot(t, j)]   gradients: dy[slot(t, j)] = w[t, j] dout[t],  dw[t, j] = <dout[t], y[slot(t, j)]>
// All of it is bound by memory: a token's row is read once and written k times, or the other way round.  The numbers come from counting
// alone (integers: the same whatever the order).  Where rows are many, counting, placing and copying are kernels of their own: the copy then needs no
// LDS and no registers to speak of and runs at the memory's rate, while one kernel for all of it spent 8 to 10 us of every workgroup on the counting
// (200000 tokens of 256 bf16, 2 slots 122 us, 52 now).  Where they are few, one launch does all, every workgroup counting for itself.
// us and bytes read and written, 32768 tokens of 4096 bf16, 2 slots: count 4.6, place 4.9, copy 138 (5.8 TB/s), its gradient 120 (6.7); combine 121
// (6.6), its gradients 231 (5.8).  777 tokens of 1012 fp32, 4 slots: dispatch 7.1; one token of 4096, 2 slots: 2.6, combine 2.1.
#include <type_traits>

#include "common.h"

namespace moep {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;   // one 16-byte chunk
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int MAX_E = 32, MAX_K = 16;

// STREAM: past the caches.
template <bool STREAM> __device__ __forceinline__ u32x4 load(const u32x4* p) { return STREAM ? __builtin_nontemporal_load(p) : *p; }
template <bool STREAM> __device__ __forceinline__ void store(u32x4* p, const u32x4& v) {
  if (STREAM) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// ---- dispatch --------------------------------------------------------------------------------------
struct DispatchArgs {
  const char* x;
  const int32_t* experts;                    // [T, k]
  const int32_t* used;                       // [T], may be NULL: all k
  int64_t T;
  int k, E, chunks;                          // chunks of 16 bytes to a row
  int32_t* counts;                           // [pieces, E]: ids of each expert in pieces of `piece` tokens
  int piece, pieces;
  char* rows;
  int32_t* slot_of;                          // [T, k]
  int32_t* offsets;                          // [E + 1]
};

// Slots i, i + B, .. as they are in memory (beyond `end` slot end - 1 again: all loads at once, and no lane's waits for another's),
// and the expert of each: -1 if the slot is not used, or beyond the end.
template <int DEEP, int B>
struct Ids {
  int expert[DEEP], used[DEEP], j[DEEP];
  __device__ __forceinline__ void request(const DispatchArgs& p, unsigned i, unsigned end) {
#pragma unroll
    for (int q = 0; q < DEEP; ++q) expert[q] = p.experts[min(i + q * B, end - 1)];
    if (!p.used) return;
    const unsigned k = (unsigned)p.k, last = (end - 1) / k, t_step = B / k, j_step = B - t_step * k;
    unsigned t = i / k, slot = i - t * k;    // (of the next ones without a division)
#pragma unroll
    for (int q = 0; q < DEEP; ++q) {
      j[q] = (int)slot;
      used[q] = p.used[min(t, last)];
      t += t_step;
      slot += j_step;
      if (slot >= k) { slot -= k; ++t; }
    }
  }
  __device__ __forceinline__ int at(const DispatchArgs& p, int q, unsigned i, unsigned end) const {
    bool there = i + q * B < end && (unsigned)expert[q] < (unsigned)p.E;
    if (p.used) there = there && j[q] < used[q];
    return there ? expert[q] : -1;
  }
};

// Counts in LDS, eight copies so that the lanes of a wavefront seldom meet at one.
constexpr int COPIES = 8;
struct Counts { int n[COPIES][MAX_E + 1]; };
__device__ __forceinline__ void clear(Counts* c) {
  for (int i = threadIdx.x; i < COPIES * (MAX_E + 1); i += THREADS) (&c->n[0][0])[i] = 0;
}
__device__ __forceinline__ int total(const Counts& c, int e) {
  int n = 0;
#pragma unroll
  for (int q = 0; q < COPIES; ++q) n += c.n[q][e];
  return n;
}

__global__ __launch_bounds__(THREADS) void count_rows_kernel(DispatchArgs p) {
  __shared__ Counts c;
  clear(&c);
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * p.piece, t1 = min(p.T, t0 + p.piece);
  const unsigned i0 = (unsigned)(t0 * p.k), i1 = (unsigned)(t1 * p.k);
  constexpr int DEEP = 4;
  for (unsigned i = i0 + threadIdx.x; i < i1; i += DEEP * THREADS) {
    Ids<DEEP, THREADS> ids;
    ids.request(p, i, i1);
#pragma unroll
    for (int q = 0; q < DEEP; ++q) {
      const int e = ids.at(p, q, i, i1);
      if (e >= 0) atomicAdd(&c.n[threadIdx.x & (COPIES - 1)][e], 1);
    }
  }
  __syncthreads();
  if ((int)threadIdx.x < p.E) p.counts[(int64_t)blockIdx.x * p.E + threadIdx.x] = total(c, threadIdx.x);
}

// Among the wavefront's slots of the same expert e (-1: none) how many come before this lane's; and how many there are, to of_wave[e].
__device__ __forceinline__ int rank_in_wave(int e, int* of_wave) {
  int rank = 0;
  for (unsigned long long left = __ballot(e >= 0); left;) {
    const int of = __builtin_amdgcn_readlane(e, __ffsll((long long)left) - 1);
    const unsigned long long same = __ballot(e == of);
    if (e == of) {
      rank = __builtin_amdgcn_mbcnt_hi((unsigned)(same >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)same, 0u));
      of_wave[e] = __popcll(same);
    }
    left &= ~same;
  }
  return rank;
}
// Sum of the lanes' numbers up to and with this one, over the first 32 lanes.
__device__ __forceinline__ int running_sum(int n, int lane) {
#pragma unroll
  for (int d = 1; d < MAX_E; d <<= 1) {
    const int from = __shfl_up(n, d);
    if (lane >= d) n += from;
  }
  return n;
}
__device__ __forceinline__ void write_offsets(const DispatchArgs& p, int e, int upto) {
  if (blockIdx.x != 0 || e >= p.E) return;
  p.offsets[e + 1] = upto;
  if (e == 0) p.offsets[0] = 0;
}

// Up to THREADS slots: every workgroup works them all out, one to a thread, and copies one token's row.
__global__ __launch_bounds__(THREADS) void dispatch_few_rows_kernel(DispatchArgs p) {
  constexpr int B = THREADS, W = WAVES;
  __shared__ int next[MAX_E];
  __shared__ int of_wave[W][MAX_E];
  __shared__ int slots[B];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t = (int)blockIdx.x, n = (int)p.T * p.k;
  const u32x4* const from = (const u32x4*)p.x + (int64_t)t * p.chunks;
  Ids<1, B> ids;
  u32x4 v = {0, 0, 0, 0};                    // (the row's first chunks are asked for with the ids)
  if (n > 0) {
    ids.request(p, tid, n);
    if (tid < p.chunks) v = from[tid];
  }
  for (int i = tid; i < W * MAX_E; i += B) (&of_wave[0][0])[i] = 0;
  __syncthreads();
  const int e = n > 0 ? ids.at(p, 0, tid, n) : -1;
  const int rank = rank_in_wave(e, of_wave[wave]);
  __syncthreads();
  if (tid < 64) {                            // rows in front of each wavefront's, of its expert and of those before
    int all = 0;
    if (tid < MAX_E)
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const int m = of_wave[w][tid];
        of_wave[w][tid] = all;
        all += m;
      }
    const int upto = running_sum(all, lane);
    if (tid < MAX_E) next[tid] = upto - all;
    write_offsets(p, tid, upto);
  }
  __syncthreads();
  const int slot = e >= 0 ? next[e] + of_wave[wave][e] + rank : -1;
  slots[tid] = slot;
  if (blockIdx.x == 0 && tid < n) p.slot_of[tid] = slot;
  if (n == 0) return;
  __syncthreads();
  for (int c = tid; c < p.chunks; c += B) {
    if (c >= B) v = from[c];
    for (int j = 0; j < p.k; ++j) {
      const int to = slots[t * p.k + j];
      if (to >= 0) ((u32x4*)p.rows)[(int64_t)to * p.chunks + c] = v;
    }
  }
}

// Beyond, up to MANY_THREADS x DEEP slots: every workgroup counts them all, and places and copies those of `piece` tokens, 64 slots at most.
constexpr int MANY_THREADS = 1024;
template <int DEEP>
__global__ __launch_bounds__(MANY_THREADS) void dispatch_many_rows_kernel(DispatchArgs p) {
  __shared__ Counts before, rest;
  __shared__ int slots[64];
  const int tid = threadIdx.x;
  const int t0 = (int)blockIdx.x * p.piece, tokens = min(p.piece, (int)p.T - t0), n = tokens * p.k;
  const unsigned i0 = (unsigned)(t0 * p.k), all = (unsigned)((int)p.T * p.k);
  const int work = tokens * p.chunks;
  const u32x4* const from = (const u32x4*)p.x + (int64_t)t0 * p.chunks;
  Ids<DEEP, MANY_THREADS> ids;
  Ids<1, 64> own;
  ids.request(p, tid, all);
  if (tid < 64) own.request(p, i0 + tid, i0 + n);
  u32x4 v = {0, 0, 0, 0};                    // (the first chunks of the rows are asked for with the ids)
  if (tid < work) v = from[tid];
  for (int i = tid; i < COPIES * (MAX_E + 1); i += MANY_THREADS) { (&before.n[0][0])[i] = 0; (&rest.n[0][0])[i] = 0; }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < DEEP; ++q) {
    const int e = ids.at(p, q, tid, all);
    if (e >= 0) atomicAdd(&((unsigned)(tid + q * MANY_THREADS) < i0 ? before : rest).n[tid & (COPIES - 1)][e], 1);
  }
  __syncthreads();
  if (tid < 64) {
    const int b = tid < p.E ? total(before, tid) : 0, m = tid < p.E ? b + total(rest, tid) : 0;
    const int upto = running_sum(m, tid);
    write_offsets(p, tid, upto);
    const int first = upto - m + b;          // of expert `tid`
    const int e = own.at(p, 0, i0 + tid, i0 + n);
    __shared__ int unused[MAX_E];
    const int rank = rank_in_wave(e, unused);
    const int slot = __shfl(first, e >= 0 ? e : 0) + rank;
    slots[tid] = e >= 0 ? slot : -1;
    if (tid < n) p.slot_of[i0 + tid] = slots[tid];
  }
  __syncthreads();
  for (int i = tid; i < work; i += MANY_THREADS) {
    if (i >= MANY_THREADS) v = from[i];
    const int token = i / p.chunks, c = i - token * p.chunks;
    for (int j = 0; j < p.k; ++j) {
      const int to = slots[token * p.k + j];
      if (to >= 0) ((u32x4*)p.rows)[(int64_t)to * p.chunks + c] = v;
    }
  }
}

// The slots' numbers, a piece of the tokens to a workgroup.
__global__ __launch_bounds__(THREADS) void place_rows_kernel(DispatchArgs p) {
  __shared__ Counts before, rest;
  __shared__ int next[MAX_E];                // the number of the next row of each expert
  __shared__ int of_wave[WAVES][MAX_E];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t0 = (int64_t)blockIdx.x * p.piece, t1 = min(p.T, t0 + p.piece);
  const unsigned i0 = (unsigned)(t0 * p.k), i1 = (unsigned)(t1 * p.k);
  Ids<1, THREADS> ids;                       // (asked for before the counting, which takes longer than they do)
  ids.request(p, i0 + tid, i1);
  clear(&before);
  clear(&rest);
  __syncthreads();
  {
    const unsigned mine = blockIdx.x * (unsigned)p.E, n = (unsigned)p.pieces * (unsigned)p.E, e_step = THREADS % (unsigned)p.E;
    constexpr int DEEP = 8;
    unsigned e = tid % (unsigned)p.E;
    for (unsigned i = tid; i < n; i += DEEP * THREADS) {
      int c[DEEP];
#pragma unroll
      for (int q = 0; q < DEEP; ++q) c[q] = p.counts[min(i + q * THREADS, n - 1)];
#pragma unroll
      for (int q = 0; q < DEEP; ++q) {
        if (i + q * THREADS < n) atomicAdd(&(i + q * THREADS < mine ? before : rest).n[(tid >> 3) & (COPIES - 1)][e], c[q]);
        e += e_step;
        if (e >= (unsigned)p.E) e -= p.E;
      }
    }
  }
  __syncthreads();
  if (tid < 64) {                            // rows of the experts in front, and of this one in front of the workgroup's
    const int b = tid < p.E ? total(before, tid) : 0, n = tid < p.E ? b + total(rest, tid) : 0;
    const int upto = running_sum(n, lane);
    if (tid < MAX_E) next[tid] = upto - n + b;
    write_offsets(p, tid, upto);
  }
  for (unsigned i = i0; i < i1; i += THREADS) {
    if (i > i0) ids.request(p, i + tid, i1);
    if (tid < WAVES * MAX_E) (&of_wave[0][0])[tid] = 0;
    __syncthreads();                         // (`next` is there too)
    const int e = ids.at(p, 0, i + tid, i1);
    const int rank = rank_in_wave(e, of_wave[wave]);
    __syncthreads();
    int slot = -1;
    if (e >= 0) {
      slot = next[e] + rank;
#pragma unroll
      for (int w = 0; w < WAVES - 1; ++w) slot += w < wave ? of_wave[w][e] : 0;
    }
    if (i + tid < i1) p.slot_of[i + tid] = slot;
    __syncthreads();
    if (tid < MAX_E)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) next[tid] += of_wave[w][tid];
    __syncthreads();                         // (`next` and `of_wave` begin anew)
  }
}
static_assert(WAVES * MAX_E <= THREADS, "of_wave is cleared at once");

// The rows: a thread takes one chunk of a token's row (2^shift lanes to a row) and stores it k times.
template <int KG, bool STREAM>
__global__ __launch_bounds__(THREADS) void copy_rows_kernel(DispatchArgs p, int shift) {
  const int lane = threadIdx.x & 63;
  const int side = 64 >> shift, parts = (p.chunks + (1 << shift) - 1) >> shift;
  const int64_t item = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const int64_t group = item / parts;
  const int64_t t = group * side + (lane >> shift);
  const int c = (int)(item - group * parts) * (1 << shift) + (lane & ((1 << shift) - 1));
  if (t >= p.T || c >= p.chunks) return;
  const u32x4 v = load<STREAM>((const u32x4*)p.x + t * p.chunks + c);
  for (int j0 = 0; j0 < p.k; j0 += KG) {
    int slot[KG];
#pragma unroll
    for (int j = 0; j < KG; ++j) slot[j] = j0 + j < p.k ? p.slot_of[t * p.k + j0 + j] : -1;
#pragma unroll
    for (int j = 0; j < KG; ++j)
      if (slot[j] >= 0) {
        store<STREAM>((u32x4*)p.rows + (int64_t)slot[j] * p.chunks + c, v);
      }
  }
}

// ---- combine ---------------------------------------------------------------------------------------
// Elements of a chunk: 4 fp32 or 8 bf16.
template <typename S> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int N = 4;
  __device__ static float get(const u32x4& v, int j) { return __uint_as_float(v[j]); }
  __device__ static u32x4 pack(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
template <> struct Chunk<uint16_t> {
  static constexpr int N = 8;
  __device__ static float get(const u32x4& v, int j) { return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16); }
  __device__ static u32x4 pack(const float (&x)[8]) {              // (to the nearest, ties to even: the only rounding of a result)
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, bf16x2));
    return v;
  }
};

struct CombineArgs {
  const char* y;                             // [R, H]
  const int32_t* slot_of;                    // [T, k]; outside [0, R): not there
  const float* weights;                      // [T, k], may be NULL (1)
  int64_t T;
  int k, chunks, R;
  char* out;                                 // [T, H]
  // backward
  const char* dout;                          // [T, H]
  char* dy;                                  // [R, H]
  float* dweights;                           // [T, k], may be NULL: not wanted
};

// A thread takes one chunk of a token's row, KG slots' at once, so that their loads are in flight together; the sum goes in the slots' order, in 32
// bits.
template <typename S, int KG, bool STREAM>
__global__ __launch_bounds__(THREADS) void combine_rows_kernel(CombineArgs p, int shift) {
  constexpr int N = Chunk<S>::N;
  const int lane = threadIdx.x & 63;
  const int side = 64 >> shift, parts = (p.chunks + (1 << shift) - 1) >> shift;
  const int64_t item = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const int64_t group = item / parts;
  const int64_t t = group * side + (lane >> shift);
  const int c = (int)(item - group * parts) * (1 << shift) + (lane & ((1 << shift) - 1));
  if (t >= p.T || c >= p.chunks) return;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  for (int j0 = 0; j0 < p.k; j0 += KG) {
    int slot[KG];
    float w[KG];
    u32x4 v[KG];
#pragma unroll
    for (int j = 0; j < KG; ++j) {
      slot[j] = j0 + j < p.k ? p.slot_of[t * p.k + j0 + j] : -1;
      w[j] = j0 + j < p.k && p.weights ? p.weights[t * p.k + j0 + j] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < KG; ++j)
      if ((unsigned)slot[j] < (unsigned)p.R) {
        v[j] = load<STREAM>((const u32x4*)p.y + (int64_t)slot[j] * p.chunks + c);
      }
#pragma unroll
    for (int j = 0; j < KG; ++j)
      if ((unsigned)slot[j] < (unsigned)p.R)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = fmaf(w[j], Chunk<S>::get(v[j], i), sum[i]);
  }
  ((u32x4*)p.out)[t * p.chunks + c] = Chunk<S>::pack(sum);
}

// dy and dw of a token by 2^shift lanes, or by all of a workgroup of W wavefronts: each goes through its chunks of dout and of the k rows of y,
// adding up k products in 32 bits, which are then joined in a fixed order.  A workgroup to a token has all of its loads in flight at once: rows of 8 KB,
// 32768 tokens of 2 slots 277 us by wavefronts, 251 by workgroups, 231 past the caches.  Shorter rows (bf16, 2 slots) by wavefronts / by workgroups: 1024
// tokens of 576 6.4 / 6.4, of 1024 6.6 / 6.5, of 1536 7.6 / 6.8, of 1984 8.4 / 7.6; 2048 tokens 6.8 / 6.9, 8.6 / 8.6, 9.2 / 8.9, 10.6 / 10.4; 4096 tokens 8.9 / 9.9,
// 11.0 / 11.4, 13.6 / 14.1, 19.3 / 19.4; 16384 tokens of 576 23 / 32, of 1984 66.6 / 65.6.
template <typename S, int KG, int W, bool STREAM>
__global__ __launch_bounds__(THREADS) void combine_rows_backward_kernel(CombineArgs p, int shift) {
  constexpr int N = Chunk<S>::N, U = KG > 4 ? 1 : 2;
  __shared__ float joined[WAVES][KG];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int side = W > 1 ? 1 : 64 >> shift;
  const int64_t t = W > 1 ? (int64_t)blockIdx.x : ((int64_t)blockIdx.x * WAVES + wave) * side + (lane >> shift);
  const int c0 = W > 1 ? threadIdx.x : lane & ((1 << shift) - 1), step = W > 1 ? THREADS : 1 << shift;
  const bool mine = t < p.T;
  for (int j0 = 0; j0 < p.k; j0 += KG) {
    int slot[KG];
    float w[KG], dot[KG];
#pragma unroll
    for (int j = 0; j < KG; ++j) {
      const bool there = mine && j0 + j < p.k;
      slot[j] = there ? p.slot_of[t * p.k + j0 + j] : -1;
      if ((unsigned)slot[j] >= (unsigned)p.R) slot[j] = -1;
      w[j] = there && p.weights ? p.weights[t * p.k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    if (mine)
      for (int c = c0; c < p.chunks; c += U * step) {
        u32x4 d[U], v[U][KG];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c + u * step < p.chunks) {
            d[u] = load<STREAM>((const u32x4*)p.dout + t * p.chunks + c + u * step);
            if (p.dweights)
#pragma unroll
              for (int j = 0; j < KG; ++j)
                if (slot[j] >= 0) v[u][j] = load<STREAM>((const u32x4*)p.y + (int64_t)slot[j] * p.chunks + c + u * step);
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c + u * step < p.chunks) {
#pragma unroll
            for (int j = 0; j < KG; ++j)
              if (slot[j] >= 0) {
                float x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                  const float g = Chunk<S>::get(d[u], i);
                  if (p.dweights) dot[j] = fmaf(g, Chunk<S>::get(v[u][j], i), dot[j]);
                  x[i] = w[j] * g;
                }
                store<STREAM>((u32x4*)p.dy + (int64_t)slot[j] * p.chunks + c + u * step, Chunk<S>::pack(x));
              }
          }
      }
    if (!p.dweights) continue;
#pragma unroll
    for (int j = 0; j < KG; ++j)
      for (int d = (W > 1 ? 64 : 1 << shift) >> 1; d > 0; d >>= 1) dot[j] += __shfl_xor(dot[j], d);
    if (W > 1) {
      if (j0) __syncthreads();
      if (lane == 0)
#pragma unroll
        for (int j = 0; j < KG; ++j) joined[wave][j] = dot[j];
      __syncthreads();
      if (threadIdx.x == 0)
#pragma unroll
        for (int j = 0; j < KG; ++j) dot[j] = (joined[0][j] + joined[1][j]) + (joined[2][j] + joined[3][j]);
    }
    if (mine && c0 == 0)
#pragma unroll
      for (int j = 0; j < KG; ++j)
        if (j0 + j < p.k) p.dweights[t * p.k + j0 + j] = dot[j];
  }
}

// ---- host ------------------------------------------------------------------------------------------
int check_rows_shape(const char* who, int64_t T, int k, int H, moep_dtype dt) {
  if (dt != MOEP_F32 && dt != MOEP_BF16) return fail(MOEP_EINVAL, "%s: unknown dtype %d", who, (int)dt);
  if (k < 1 || k > MAX_K) return fail(MOEP_EINVAL, "%s: k=%d out of range [1, %d]", who, k, MAX_K);
  if (T < 0 || T > ((int64_t)1 << 30) / k) return fail(MOEP_EINVAL, "%s: T=%lld out of range [0, 2^30 / k]", who, (long long)T);
  if (H < 1 || H > 1 << 24) return fail(MOEP_EINVAL, "%s: H=%d out of range [1, 2^24]", who, H);
  if (H % (dt == MOEP_BF16 ? 64 : 4)) return fail(MOEP_EUNSUPPORTED, "%s: H=%d must be a multiple of %d", who, H, dt == MOEP_BF16 ? 64 : 4);
  return MOEP_OK;
}
int check_16(const char* who, std::initializer_list<const void*> pointers) {
  for (const void* q : pointers)
    if ((uintptr_t)q & 15) return fail(MOEP_EUNSUPPORTED, "%s: rows must be 16-byte aligned", who);
  return MOEP_OK;
}
int check_4(const char* who, std::initializer_list<const void*> pointers) {
  for (const void* q : pointers)
    if ((uintptr_t)q & 3) return fail(MOEP_EUNSUPPORTED, "%s: slots, experts, offsets and weights must be 4-byte aligned", who);
  return MOEP_OK;
}

// What the caches behind the XCDs' hold: where a call reads and writes more, its large streams go past them (a result that the next call reads
// stays, if it is the smaller one).  us without / with, 32768 tokens of 4096 bf16, 2 slots: combine 143 / 123, dispatch and its gradient in turn 290 / 264
// (the tokens' rows alone past them or not; what was left in the caches to be written back is not pushed out by what is read).
constexpr double HELD_BYTES = 268.5e6;
inline bool past_caches(int64_t rows, int64_t row_bytes) { return (double)rows * (double)row_bytes > HELD_BYTES; }
// Slots up to which one launch does all of it, in either of two ways.  us with the launch, in one / in three launches without the gaps between them:
// 1024 tokens of 4096, 2 slots 9.1 / 11.0; 1999 of 2048, 4 slots (7996) 12.5 / 14.5; 4096 of 4096, 2 slots 20.7 / 22.3; 4096 of 1024, 4 slots 18.2 / 14.1.
constexpr int FEW_SLOTS = THREADS, MANY_SLOTS = 8 * MANY_THREADS;
constexpr int64_t MOST_COUNTS = 8192;        // of pieces and experts that a workgroup adds up
struct DispatchPlan { int piece = 1; int64_t pieces = 0; };
DispatchPlan plan_dispatch(int64_t T, int k, int E) {
  if (T * k <= FEW_SLOTS) return {1, T > 0 ? T : 1};
  if (T * k <= MANY_SLOTS) {                 // (as many workgroups as fit the chip; their slots are one wavefront's)
    int piece = (int)ceil_div(T, 512);
    return {piece, ceil_div(T, piece)};
  }
  int64_t piece = THREADS / k;               // (a slot to a thread)
  while (ceil_div(T, piece) * E > MOST_COUNTS) piece *= 2;
  return {(int)piece, ceil_div(T, piece)};
}
static_assert(MANY_SLOTS / 512 + MAX_K <= 64, "slots of a piece");

int row_shift(int chunks) {                  // lanes to a row, as a power of two
  int s = 6;
  while (s > 0 && chunks <= 1 << (s - 1)) --s;
  return s;
}

template <typename F>
void with_slots(int k, F launch) {
  if (k == 1) launch(std::integral_constant<int, 1>{});
  else if (k == 2) launch(std::integral_constant<int, 2>{});
  else if (k <= 4) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 8>{});
}

// A wavefront to every 64 chunks of a row (of short rows to several): launch(first token, tokens, workgroups, lanes to a row as a power of two),
// in as many launches as the grids' limit takes.
template <typename F>
int in_launches(int64_t T, int chunks, F launch) {
  const int shift = row_shift(chunks), side = 64 >> shift;
  const int64_t parts = ceil_div(chunks, 1 << shift), most = (most_workgroups(THREADS) * WAVES / parts - 1) * side;
  for (int64_t t = 0; t < T; t += most) {
    const int64_t tokens = T - t < most ? T - t : most;
    launch(t, tokens, (unsigned)ceil_div(ceil_div(tokens, side) * parts, WAVES), shift);
    MOEP_HIP(hipGetLastError());
  }
  return MOEP_OK;
}

int launch_combine(const CombineArgs& p, moep_dtype dt, hipStream_t s, const char* name) {
  Timed timed(name, s);
  const int64_t row = (int64_t)p.chunks * 16;
  const bool stream = past_caches(p.R + p.T, row);
  return in_launches(p.T, p.chunks, [&](int64_t t, int64_t tokens, unsigned blocks, int shift) {
    CombineArgs a = p;
    a.T = tokens;
    a.slot_of += t * p.k;
    if (a.weights) a.weights += t * p.k;
    a.out += t * row;
    with_slots(p.k, [&](auto kg) {
      constexpr int KG = decltype(kg)::value;
      auto with = [&](auto streams) {
        constexpr bool STREAM = decltype(streams)::value;
        if (dt == MOEP_BF16) hipLaunchKernelGGL((combine_rows_kernel<uint16_t, KG, STREAM>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
        else hipLaunchKernelGGL((combine_rows_kernel<float, KG, STREAM>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
      };
      if (stream) with(std::true_type{});
      else with(std::false_type{});
    });
  });
}

}  // namespace
}  // namespace moep

using namespace moep;

extern "C" {

size_t moe_dispatch_rows_workspace(int64_t T, int k, int E) {
  if (k < 1 || k > MAX_K || E < 1 || E > MAX_E || T < 0 || T > ((int64_t)1 << 30) / k) return 0;
  return T * k > MANY_SLOTS ? (size_t)plan_dispatch(T, k, E).pieces * E * sizeof(int32_t) : 0;
}

int moe_dispatch_rows(const void* x, const int32_t* experts, const int32_t* used, int64_t T, int k, int E, int H, moep_dtype dt, void* rows,
                      int32_t* slot_of, int32_t* offsets, void* ws, size_t ws_bytes, void* hip_stream) {
  const char* who = "moe_dispatch_rows";
  if (int st = check_rows_shape(who, T, k, H, dt)) return st;
  if (E < 1 || E > MAX_E) return fail(MOEP_EINVAL, "%s: E=%d out of range [1, %d]", who, E, MAX_E);
  if (!offsets) return fail(MOEP_EINVAL, "%s: NULL offsets", who);
  if (T > 0 && (!x || !experts || !rows || !slot_of)) return fail(MOEP_EINVAL, "%s: NULL x, experts, rows or slot_of", who);
  if (int st = check_16(who, {x, rows})) return st;
  if (int st = check_4(who, {experts, used, slot_of, offsets})) return st;
  const size_t need = moe_dispatch_rows_workspace(T, k, E);
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(MOEP_EWORKSPACE, "%s: needs a 256-byte aligned workspace of %zu bytes", who, need);
  hipStream_t s = (hipStream_t)hip_stream;
  const DispatchPlan plan = plan_dispatch(T, k, E);
  const int64_t row = (int64_t)H * (int64_t)dtype_size(dt);
  const DispatchArgs p = {(const char*)x, experts, used, T, k, E, (int)(row / 16), (int32_t*)ws, plan.piece, (int)plan.pieces, (char*)rows, slot_of, offsets};
  const dim3 grid((unsigned)plan.pieces);
  if (T * k <= MANY_SLOTS) {
    Timed timed("dispatch_rows", s);
    if (T * k <= FEW_SLOTS) hipLaunchKernelGGL(dispatch_few_rows_kernel, grid, dim3(THREADS), 0, s, p);
    else if (T * k <= MANY_THREADS) hipLaunchKernelGGL(dispatch_many_rows_kernel<1>, grid, dim3(MANY_THREADS), 0, s, p);
    else if (T * k <= 4 * MANY_THREADS) hipLaunchKernelGGL(dispatch_many_rows_kernel<4>, grid, dim3(MANY_THREADS), 0, s, p);
    else hipLaunchKernelGGL(dispatch_many_rows_kernel<8>, grid, dim3(MANY_THREADS), 0, s, p);
    MOEP_HIP(hipGetLastError());
    return MOEP_OK;
  }
  {
    Timed timed("count_rows", s);
    hipLaunchKernelGGL(count_rows_kernel, grid, dim3(THREADS), 0, s, p);
    MOEP_HIP(hipGetLastError());
  }
  {
    Timed timed("place_rows", s);
    hipLaunchKernelGGL(place_rows_kernel, grid, dim3(THREADS), 0, s, p);
    MOEP_HIP(hipGetLastError());
  }
  Timed timed("copy_rows", s);
  return in_launches(T, p.chunks, [&](int64_t t, int64_t tokens, unsigned blocks, int shift) {
    DispatchArgs a = p;
    a.T = tokens;
    a.x += t * row;
    a.slot_of += t * k;
    with_slots(k, [&](auto kg) {
      constexpr int KG = decltype(kg)::value;
      if (past_caches(T * k + T, row)) hipLaunchKernelGGL((copy_rows_kernel<KG, true>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
      else hipLaunchKernelGGL((copy_rows_kernel<KG, false>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
    });
  });
}

int moe_dispatch_rows_backward(const void* drows, const int32_t* slot_of, int64_t T, int k, int H, int64_t R, moep_dtype dt, void* dx,
                               void* hip_stream) {
  const char* who = "moe_dispatch_rows_backward";
  if (int st = check_rows_shape(who, T, k, H, dt)) return st;
  if (R < 0 || R > (int64_t)1 << 30) return fail(MOEP_EINVAL, "%s: R=%lld out of range [0, 2^30]", who, (long long)R);
  if (T == 0) return MOEP_OK;
  if ((!drows && R > 0) || !slot_of || !dx) return fail(MOEP_EINVAL, "%s: NULL drows, slot_of or dx", who);
  if (int st = check_16(who, {drows, dx})) return st;
  if (int st = check_4(who, {slot_of})) return st;
  CombineArgs p = {(const char*)drows, slot_of, nullptr, T, k, (int)((int64_t)H * (int64_t)dtype_size(dt) / 16), (int)R, (char*)dx, nullptr, nullptr, nullptr};
  return launch_combine(p, dt, (hipStream_t)hip_stream, "dispatch_rows_backward");
}

int moe_combine_rows(const void* y, const int32_t* slot_of, const float* weights, int64_t T, int k, int H, int64_t R, moep_dtype dt, void* out,
                     void* hip_stream) {
  const char* who = "moe_combine_rows";
  if (int st = check_rows_shape(who, T, k, H, dt)) return st;
  if (R < 0 || R > (int64_t)1 << 30) return fail(MOEP_EINVAL, "%s: R=%lld out of range [0, 2^30]", who, (long long)R);
  if (T == 0) return MOEP_OK;
  if ((!y && R > 0) || !slot_of || !out) return fail(MOEP_EINVAL, "%s: NULL y, slot_of or out", who);
  if (int st = check_16(who, {y, out})) return st;
  if (int st = check_4(who, {slot_of, weights})) return st;
  CombineArgs p = {(const char*)y, slot_of, weights, T, k, (int)((int64_t)H * (int64_t)dtype_size(dt) / 16), (int)R, (char*)out, nullptr, nullptr, nullptr};
  return launch_combine(p, dt, (hipStream_t)hip_stream, "combine_rows");
}

int moe_combine_rows_backward(const void* dout, const void* y, const int32_t* slot_of, const float* weights, int64_t T, int k, int H, int64_t R,
                              moep_dtype dt, void* dy, float* dweights, void* hip_stream) {
  const char* who = "moe_combine_rows_backward";
  if (int st = check_rows_shape(who, T, k, H, dt)) return st;
  if (R < 0 || R > (int64_t)1 << 30) return fail(MOEP_EINVAL, "%s: R=%lld out of range [0, 2^30]", who, (long long)R);
  if (T == 0) return MOEP_OK;
  if (!dout || !slot_of || (!dy && R > 0)) return fail(MOEP_EINVAL, "%s: NULL dout, slot_of or dy", who);
  if (dweights && !y && R > 0) return fail(MOEP_EINVAL, "%s: the weights' gradient needs y", who);
  if (int st = check_16(who, {dout, y, dy})) return st;
  if (int st = check_4(who, {slot_of, weights, dweights})) return st;
  hipStream_t s = (hipStream_t)hip_stream;
  const CombineArgs p = {(const char*)y, slot_of, weights, T, k, (int)((int64_t)H * (int64_t)dtype_size(dt) / 16), (int)R, nullptr, (const char*)dout,
                         (char*)dy, dweights};
  const int shift = row_shift(p.chunks);
  const bool wide = p.chunks >= THREADS || (p.chunks > 64 && T <= 2048);   // a workgroup to a token
  const int64_t each = wide ? 1 : (int64_t)WAVES * (64 >> shift), tokens = each << 20;
  const bool stream = past_caches(2 * R + T, (int64_t)p.chunks * 16);
  Timed timed("combine_rows_backward", s);
  const int64_t row = (int64_t)p.chunks * 16;
  for (int64_t t = 0; t < T; t += tokens) {
    CombineArgs a = p;
    a.T = T - t < tokens ? T - t : tokens;
    a.slot_of += t * k;
    if (a.weights) a.weights += t * k;
    a.dout += t * row;
    if (a.dweights) a.dweights += t * k;
    const unsigned blocks = (unsigned)ceil_div(a.T, each);
    with_slots(k, [&](auto kg) {
      constexpr int KG = decltype(kg)::value;
      auto with = [&](auto w) {
        constexpr int W = decltype(w)::value;
        auto streaming = [&](auto streams) {
          constexpr bool STREAM = decltype(streams)::value;
          if (dt == MOEP_BF16) hipLaunchKernelGGL((combine_rows_backward_kernel<uint16_t, KG, W, STREAM>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
          else hipLaunchKernelGGL((combine_rows_backward_kernel<float, KG, W, STREAM>), dim3(blocks), dim3(THREADS), 0, s, a, shift);
        };
        if (stream) streaming(std::true_type{});
        else streaming(std::false_type{});
      };
      if (wide) with(std::integral_constant<int, WAVES>{});
      else with(std::integral_constant<int, 1>{});
    });
    MOEP_HIP(hipGetLastError());
  }
  return MOEP_OK;
}

}  // extern "C"
