// Rows of logits [T, V] on the GPU: how a workgroup reads one and adds it up, for the kernels of logits.hip and answers.hip.
#pragma once

#include <type_traits>

#include "common.h"

namespace moep {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;   // one 16-byte chunk
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) unsigned long long u64x2;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float NEG_INF = -__builtin_inff();
constexpr int NC = 16;                       // chunks of a tile per thread
// Elements of a chunk: 4 fp32 or 8 bf16.
template <typename S> struct Elements;
template <> struct Elements<float> {
  static constexpr int N = 4;
  static constexpr unsigned NEUTRAL = 0xff800000u;
  __device__ static float get(const u32x4& v, int j) { return __uint_as_float(v[j]); }
  __device__ static float load(const float* p) { return *p; }
  __device__ static void store(float* p, float x) { *p = x; }
  __device__ static float nothing() { return NEG_INF; }
  __device__ static u32x4 pack(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
template <> struct Elements<uint16_t> {
  static constexpr int N = 8;
  static constexpr unsigned NEUTRAL = 0xff80ff80u;
  __device__ static float get(const u32x4& v, int j) { return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16); }
  __device__ static float load(const uint16_t* p) { return __uint_as_float((unsigned)*p << 16); }
  __device__ static void store(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }   // (to the nearest, ties to even)
  __device__ static uint16_t nothing() { return 0xff80; }
  __device__ static u32x4 pack(const float (&x)[8]) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, bf16x2));
    return v;
  }
};

// The larger one, NaN if either is (fmaxf drops a NaN): a row that holds one is told by its maximum.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// Largest halves of a chunk as signed 16-bit numbers, those of even and of odd elements.
__device__ __forceinline__ s16x2 top_halves(const u32x4& v) {
  const unsigned a = v[0], b = v[1], c = v[2], d = v[3];     // (numbers of their own: __builtin_bit_cast of v[i] reads v[0])
  return __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)),
                                   __builtin_elementwise_max(__builtin_bit_cast(s16x2, c), __builtin_bit_cast(s16x2, d)));
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row seen as 16-byte chunks from the boundary at or before its first element: chunk c holds elements c N - lead .. + N - 1,
// of which those within [0, V) are the row's.  Rows need no alignment beyond their elements'.  A chunk that reaches beyond the row on
// either side is loaded whole where that stays between the first row's first element and the last row's last, and cut to the row in
// registers (what it brought of the neighbours, who may be writing theirs, goes unused); only the first row's first chunk and the last row's
// last one are put together element by element.
template <typename S>
struct Row {
  static constexpr int N = Elements<S>::N;
  const S* at;
  const char* base;                          // of chunk 0
  int V, lead, chunks, first_load, end_load;
  __device__ Row(const void* rows, int64_t ld, int V_, int64_t t, int64_t T) : at((const S*)rows + t * ld), V(V_) {
    base = (const char*)at - ((uintptr_t)at & 15);
    lead = (int)(((uintptr_t)at & 15) / sizeof(S));
    chunks = (V + lead + N - 1) / N;
    first_load = t * ld < lead ? 1 : 0;
    end_load = V == 0 ? 0 : (T - 1 - t) * ld + V >= (int64_t)chunks * N - lead ? chunks : (V + lead) / N;
  }
  __device__ bool whole(int c) const { return c * N >= lead && (c + 1) * N <= V + lead; }
  __device__ const u32x4* chunk(int c) const { return (const u32x4*)(base + (uint32_t)c * 16u); }
  __device__ bool has(int c, int j) const { const int i = c * N - lead + j; return i >= 0 && i < V; }
};

template <typename S>
__device__ __forceinline__ u32x4 neutral() {
  return u32x4{Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL};
}

// Between two branches that differ in a hint to the caches alone: the compiler would make one of both, without the hint.
__device__ __forceinline__ void apart() { asm volatile(""); }

// Chunk c (thread by thread) of a row: the request alone, nothing waits.  What is not there is -inf.  STREAM: past the caches.
template <bool STREAM = false, typename S>
__device__ __forceinline__ void request(const Row<S>& row, int c, u32x4& v) {
  v = neutral<S>();
  if (c >= row.first_load && c < row.end_load) v = STREAM ? __builtin_nontemporal_load(row.chunk(c)) : *row.chunk(c);
}
// Chunks tile B NC + n B + tid of a row
template <typename S, int B, bool STREAM = false>
__device__ __forceinline__ void request_tile(const Row<S>& row, int tile, int tid, u32x4 (&v)[NC]) {
#pragma unroll
  for (int n = 0; n < NC; ++n) request<STREAM>(row, tile * (B * NC) + n * B + tid, v[n]);
}
// The thread's index as a number that the compiler knows nothing of.  Taken anew for every row: what it can tell ahead of all rows (sixteen
// offsets, sixteen comparisons' sides) it keeps in registers from row to row.
__device__ __forceinline__ int thread_again(int tid) {
  asm volatile("" : "+v"(tid));
  return tid;
}

// A chunk as a shift register: its first element, and the others moved down by one with another at the end.  (The rare paths go through
// a chunk element by element in a loop: written out they would take registers from the common one.)
template <typename S>
__device__ __forceinline__ S shift_out(u32x4& v, S in) {
  if constexpr (sizeof(S) == 4) {
    const S first = __uint_as_float(v[0]);
    v = u32x4{v[1], v[2], v[3], __float_as_uint(in)};
    return first;
  } else {
    const S first = (S)v[0];
    v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16),
              __builtin_amdgcn_alignbit(v[3], v[2], 16), __builtin_amdgcn_alignbit((unsigned)in, v[3], 16)};
    return first;
  }
}

// The row's first and last chunk cut to the row, in the two threads that hold them.
template <typename S>
__device__ __forceinline__ u32x4 cut(const Row<S>& row, int c, u32x4 v) {
  const bool there = c >= row.first_load && c < row.end_load;
#pragma unroll 1
  for (int j = 0; j < Row<S>::N; ++j) {
    S x = shift_out<S>(v, S(0));
    if (!row.has(c, j)) x = Elements<S>::nothing();
    else if (!there) x = row.at[c * Row<S>::N - row.lead + j];
    if constexpr (sizeof(S) == 4) v[3] = __float_as_uint(x);
    else v[3] = (v[3] & 0xffffu) | ((unsigned)x << 16);
  }
  return v;
}
template <typename S, int B>
__device__ __forceinline__ void cut_ends(const Row<S>& row, int tile, int tid, u32x4 (&v)[NC]) {
  const int c0 = tile * (B * NC) + tid, last = row.chunks - 1;
  if (row.lead && c0 == 0) v[0] = cut(row, 0, v[0]);
  if (!row.whole(last) && last >= c0 && last < c0 + B * NC && (last - c0) % B == 0 && !(row.lead && last == 0)) {
    u32x4 end = neutral<S>();
#pragma unroll
    for (int n = 0; n < NC; ++n)
      if (c0 + n * B == last) end = v[n];
    end = cut(row, last, end);
#pragma unroll
    for (int n = 0; n < NC; ++n)
      if (c0 + n * B == last) v[n] = end;
  }
}

// A wavefront's values joined, the same in all lanes: over each 16 lanes, then the sixteens, from lane to lane in the registers (through LDS,
// as an exchange of any lanes goes, six steps take a microsecond).
template <typename T, typename F>
__device__ __forceinline__ T over_wave(T x, T identity, F join) {
  static_assert(sizeof(T) == 4, "");
#define MOEP_FROM(ctrl, rows) \
  x = join(x, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, identity), __builtin_bit_cast(int, x), ctrl, rows, 0xf, false)))
  MOEP_FROM(0x111, 0xf); MOEP_FROM(0x112, 0xf); MOEP_FROM(0x114, 0xf); MOEP_FROM(0x118, 0xf);   // the lane 1, 2, 4, 8 before
  MOEP_FROM(0x142, 0xa); MOEP_FROM(0x143, 0xc);                                                // lane 15 of the sixteen, 31 of the half before
#undef MOEP_FROM
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ float max_over_wave(float x) { return over_wave(x, NEG_INF, [](float a, float b) { return max_nan(a, b); }); }
__device__ __forceinline__ float sum_over_wave(float x) { return over_wave(x, 0.f, [](float a, float b) { return a + b; }); }

// A number that is the same in all lanes, moved to where it takes no register of theirs.
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// Running maximum m of the elements seen, s = sum exp2((z - m) c) and (ENTROPY, c = log2 e) w = sum exp(z - m) (z - m).  32 bits:
// sums of at most 2^28 terms in [0, 1], in groups of at most 2^20 per thread.
struct Stats { float m, s, w; };

__device__ __forceinline__ float reference(float m) { return m == NEG_INF ? 0.f : m; }   // (nothing but -inf: they stay -inf)

// The sums of `a` taken over from its maximum to `m`, which is no smaller.
template <bool ENTROPY>
__device__ __forceinline__ Stats moved(const Stats& a, float m, float c) {
  if (a.s == 0.f) return Stats{m, 0.f, 0.f};                 // nothing in it
  const float d = a.m - m, f = exp2_fast(d * c);
  // (a maximum far below: f is 0, and d can be -inf)
  return Stats{m, a.s * f, ENTROPY ? f * (a.w + a.s * fmaxf(d, -1000.f)) : 0.f};
}

// The largest element of a tile.  bf16: by the halves' bits as signed 16-bit numbers, two elements an instruction and none taken
// apart, which is the numbers' order as soon as one of them is not negative; a thread with nothing but negative ones looks again.
// (A NaN with its sign set is missed here.  Its exponential is NaN all the same, and so are the sums.)
template <typename S, int B>
__device__ __forceinline__ float largest(const u32x4 (&v)[NC], int chunks_left) {
  constexpr int N = Elements<S>::N;
  float m = NEG_INF;
  if constexpr (sizeof(S) == 2) {
    s16x2 top = {-32768, -32768};
#pragma unroll
    for (int n = 0; n < NC; ++n)
      if (n * B < chunks_left)                               // (the same for all threads)
        top = __builtin_elementwise_max(top, top_halves(v[n]));
    const short x = max(top[0], top[1]);
    if (x >= 0) return __uint_as_float((unsigned)x << 16);
  }
#pragma unroll
  for (int n = 0; n < NC; ++n)
    if (n * B < chunks_left)
#pragma unroll
      for (int j = 0; j < N; j += 2) m = max_nan(m, max_nan(Elements<S>::get(v[n], j), Elements<S>::get(v[n], j + 1)));
  return m;
}

// Before a tile is used again: its elements are taken apart anew then, instead of all of them being held taken apart in twice the
// registers (bf16: 209 registers for 128, which leaves half as many wavefronts to cover the loads).
__device__ __forceinline__ void use_again(u32x4 (&v)[NC]) {
#pragma unroll
  for (int n = 0; n < NC; ++n) asm volatile("" : "+v"(v[n]));
}

template <typename S, int B, bool ENTROPY>
__device__ __forceinline__ void add_tile(u32x4 (&v)[NC], int chunks_left, Stats& a, float c) {
  constexpr int N = Elements<S>::N;
  const float m = max_nan(a.m, largest<S, B>(v, chunks_left));
  if (!(m == a.m)) a = moved<ENTROPY>(a, m, c);
  const float r = reference(m);
  use_again(v);
  float s[2] = {0.f, 0.f}, w[2] = {0.f, 0.f};
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    if (n * B < chunks_left)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      // the difference first: a masked logit may be the type's lowest value, whose product with log2 e overflows
      float d = Elements<S>::get(v[n], j) - r;
      if (ENTROPY) d = max_nan(d, -1000.f);                  // exp is 0 there, and 0 times -inf is not
      const float e = exp2_fast(d * c);
      s[j & 1] += e;
      if (ENTROPY) w[j & 1] = fmaf(e, d, w[j & 1]);
    }
  }
  a.s += s[0] + s[1];
  a.w += w[0] + w[1];
}

// The workgroup's joint statistics, the same in every thread, in two halves with a barrier between them: each wavefront's into `shared`
// (3 floats a wavefront), then those of all, in a fixed order.
template <int B, bool ENTROPY>
__device__ __forceinline__ Stats join_wave(Stats a, float c, float* shared) {
  constexpr int WAVES = B / 64;
  a = moved<ENTROPY>(a, max_over_wave(a.m), c);
  a.s = sum_over_wave(a.s);
  if (ENTROPY) a.w = sum_over_wave(a.w);
  if (WAVES > 1 && (threadIdx.x & 63) == 0) {
    const int wave = threadIdx.x >> 6;
    shared[wave] = a.m; shared[WAVES + wave] = a.s; shared[2 * WAVES + wave] = a.w;
  }
  return a;
}
template <int B, bool ENTROPY>
__device__ __forceinline__ Stats join_all(const Stats& a, float c, const float* shared) {
  constexpr int WAVES = B / 64;
  if (WAVES == 1) return a;
  float m = shared[0];
#pragma unroll
  for (int q = 1; q < WAVES; ++q) m = max_nan(m, shared[q]);
  Stats t = {m, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < WAVES; ++q) {
    const Stats x = moved<ENTROPY>(Stats{shared[q], shared[WAVES + q], shared[2 * WAVES + q]}, m, c);
    t.s += x.s; t.w += x.w;
  }
  return t;
}

// `aligned`: whether the gradient's row starts like the logits' within 16 bytes.  Else all of a chunk's elements are stored by themselves:
// loss and gradient of 4096 rows of 32000 bf16 in rows of 32001, the gradient in rows of 32000, 225 us for 122, the gradient alone 215 for 122.
template <typename S>
__device__ __forceinline__ void store_chunk(const Row<S>& row, S* out, bool aligned, int c, u32x4 v, bool stream = false) {
  const int i0 = c * Row<S>::N - row.lead;
  if (aligned && row.whole(c)) {
    if (stream) {                                            // (past the caches)
      apart();
      __builtin_nontemporal_store(v, (u32x4*)(out + i0));
      apart();
    } else {
      *(u32x4*)(out + i0) = v;
    }
    return;
  }
#pragma unroll 1
  for (int j = 0; j < Row<S>::N; ++j) {
    const S x = shift_out<S>(v, S(0));
    if (row.has(c, j)) out[i0 + j] = x;
  }
}

// Threads per row of a loss: the fewest whose registers hold it whole, so that many rows are in flight on a compute unit at different
// points of their way, and fewer barriers stop them.  us, 4096 rows, loss and gradient, 64 / 128 / 256 / 512 / 1024 threads: V = 4096 bf16 (512
// chunks) 19 / 21 / 26 / 46 / 93; 8000 (1000) 28 / 31 / 32 / 51 / 98; 16000 (2000) - / 55 / 50 / 68 / 115; 24000 (3000) - / - / 81 / 87 / 135; 32000 (4000)
// - / - / 110 / 104 / 158 (1000 rows: 25 / 30 / 41); 65000 (8125) - / - / - / 207 / 233; 131072 (16384) held by 1024 412, not held 511.  Few rows
// get more threads, since there is nothing else for the compute units to do: 33 rows of 1003 fp32 logits 7.9 us with 64 threads, 6.6
// with 256; one of 32000 bf16 9.7 with 256, 8.4 with 512.  0: none hold it.
int threads_to_hold(int64_t T, int64_t chunks) {
  if (chunks > 1024 * NC) return 0;
  if (T <= 512) return chunks <= 512 ? 256 : chunks <= 512 * NC ? 512 : 1024;
  if (chunks <= 64 * NC) return 64;
  if (chunks <= 128 * 12) return 128;                        // (of 16 that there is room for)
  if (chunks <= 256 * (T < 2048 ? NC : 14)) return 256;
  return chunks <= 512 * NC ? 512 : 1024;
}
// Threads per row of log probabilities, which need not be held: one wavefront where that holds a row of many, else 256, or 512 where few
// rows have more than a tile.  us, 64 / 256 / 512 / 1024 threads: 8192 rows of 4096 bf16, K = 5 21 / 46 / 95 / 214; 8192 of 32000, K = 64 122 / 115 /
// 176 / 330; 777 of 50001 fp32 56 / 43 / 38 / 54; 300 of 131072 bf16 79 / 34 / 32 / 40; one of 32000 - / 9.0 / 9.3 / 10.8, of 131072 - / 23.3 / 17.6 / 16.9.
int threads_to_read(int64_t T, int64_t chunks) {
  if (chunks <= 64 * NC && T > 2048) return 64;
  return T >= 1024 || chunks <= 256 * NC ? 256 : 512;
}
// Chunks of a row at most: its elements from the 16-byte boundary before it on, which is as far for every row where `ld` is whole chunks.
int64_t most_chunks(const void* logits, int64_t ld, int64_t V, moep_dtype dt) {
  const int64_t size = (int64_t)dtype_size(dt), n = 16 / size;
  return ceil_div(V + (ld % n ? n - 1 : (int64_t)((uintptr_t)logits & 15) / size), n);
}

template <typename F>
void with_threads(int threads, F launch) {
  switch (threads) {
    case 64: launch(std::integral_constant<int, 64>{}); break;
    case 128: launch(std::integral_constant<int, 128>{}); break;
    case 256: launch(std::integral_constant<int, 256>{}); break;
    default: launch(std::integral_constant<int, 512>{});
  }
}

int check_rows(const char* who, int64_t T, int64_t V, moep_dtype dt, const void* logits, int64_t ld) {
  if (dt != MOEP_F32 && dt != MOEP_BF16) return fail(MOEP_EINVAL, "%s: unknown dtype %d", who, (int)dt);
  if (T < 0 || T > (int64_t)1 << 30) return fail(MOEP_EINVAL, "%s: T=%lld out of range [0, 2^30]", who, (long long)T);
  if (V < 1 || V > (int64_t)1 << 28) return fail(MOEP_EINVAL, "%s: V=%lld out of range [1, 2^28]", who, (long long)V);
  if (ld < V) return fail(MOEP_EINVAL, "%s: rows of %lld elements are only %lld apart", who, (long long)V, (long long)ld);
  if ((uintptr_t)logits % dtype_size(dt)) return fail(MOEP_EUNSUPPORTED, "%s: logits are not aligned to their elements", who);
  return MOEP_OK;
}

// Rows of a launch, of up to 1024 threads each.
constexpr int64_t LAUNCH_ROWS = (int64_t)1 << 21;
static_assert(LAUNCH_ROWS <= most_workgroups(1024), "one workgroup a row");

}  // namespace
}  // namespace moep
