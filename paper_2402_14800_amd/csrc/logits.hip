// Rows of logits [T, V]: log probabilities of given tokens with the entropy and the K best alternatives
// (moe_token_logprobs), and the distillation loss from a teacher's K best logits with its gradient (moe_distill_topk).
//
// With m = max_i z_i, s = sum_i exp((z_i - m) / tau):  log p_i = (z_i - m) / tau - log s, and (tau = 1) the entropy is
// log s - sum_i exp(z_i - m) (z_i - m) / s.  With q the softmax of the teacher's K logits over tau, the loss of a row is
// tau^2 sum_j q_j (log q_j - log p_id(j)) and its gradient tau (p - q).
//
// Bound by the one read of the logits (and the one write of the gradient); the lanes are close behind: an element of two
// bytes costs about ten lane operations, four of them the exponential.  One workgroup takes a row; each thread keeps its own
// running maximum and sums (a rescale per 16 chunks), so the row is read without a barrier and joined once at its end.  Up to
// 16 chunks of 16 bytes per thread stay in registers, so a row of up to 32768 bf16 logits on 256 threads is read from memory
// once also where it is used again (the gradient, the search for the best); a longer one is walked tile by tile and read
// again from the caches.
#include "common.h"

namespace moep {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;   // one 16-byte chunk
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float NEG_INF = -__builtin_inff();
constexpr int NC = 16;                       // chunks of a tile per thread
constexpr int CANDIDATES = 512;              // room for the elements that the search for the best sorts

// Elements of a chunk: 4 fp32 or 8 bf16.
template <typename S> struct Elements;
template <> struct Elements<float> {
  static constexpr int N = 4;
  static constexpr unsigned NEUTRAL = 0xff800000u;
  __device__ static float get(const u32x4& v, int j) { return __uint_as_float(v[j]); }
  __device__ static float load(const float* p) { return *p; }
  __device__ static void store(float* p, float x) { *p = x; }
  __device__ static void put(u32x4& v, int j, const float* p) { v[j] = __float_as_uint(*p); }
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
  __device__ static void put(u32x4& v, int j, const uint16_t* p) {
    v[j >> 1] = j & 1 ? (v[j >> 1] & 0xffffu) | ((unsigned)*p << 16) : (v[j >> 1] & 0xffff0000u) | *p;
  }
  __device__ static u32x4 pack(const float (&x)[8]) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, bf16x2));
    return v;
  }
};

// The larger one, NaN if either is (fmaxf drops a NaN): a row that holds one is told by its maximum.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row seen as 16-byte chunks from the boundary at or before its first element: chunk c holds elements c N - lead .. + N - 1,
// of which those within [0, V) exist.  Rows need no alignment beyond their elements'.
template <typename S>
struct Row {
  static constexpr int N = Elements<S>::N;
  const S* at;
  int V, lead, chunks, first_whole, end_whole;
  __device__ Row(const S* p, int V_) : at(p), V(V_) {
    lead = (int)(((uintptr_t)p & 15) / sizeof(S));
    chunks = (V + lead + N - 1) / N;
    first_whole = lead ? 1 : 0;
    end_whole = (V + lead) / N;
  }
  __device__ bool whole(int c) const { return c >= first_whole && c < end_whole; }
  __device__ u32x4 partial(int c) const {
    u32x4 v = {Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = c * N - lead + j;
      if (i >= 0 && i < V) Elements<S>::put(v, j, at + i);
    }
    return v;
  }
};

// Chunks tile B NC + n B + tid of a row in a thread's registers; what the row does not have is -inf.
template <typename S, int B>
__device__ __forceinline__ void load_tile(const Row<S>& row, int tile, u32x4 (&v)[NC]) {
  const int tid = threadIdx.x, c0 = tile * (B * NC) + tid;
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    v[n] = u32x4{Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL, Elements<S>::NEUTRAL};
    const int c = c0 + n * B;
    if (row.whole(c)) v[n] = *(const u32x4*)(row.at + ((int64_t)c * Row<S>::N - row.lead));
  }
  if (row.lead || row.end_whole < row.chunks) {              // the ends of the row
    if (row.lead && c0 == 0) v[0] = row.partial(0);
    const int last = row.end_whole;
    if (last < row.chunks && last >= row.first_whole && last >= c0 && last < c0 + B * NC && (last - c0) % B == 0) {
      const u32x4 end = row.partial(last);
#pragma unroll
      for (int n = 0; n < NC; ++n)
        if (c0 + n * B == last) v[n] = end;
    }
  }
}

// Running maximum m of the elements seen, s = sum exp2((z - m) c) and (ENTROPY, c = log2 e) w = sum exp(z - m) (z - m).  32 bits:
// sums of at most 2^28 terms in [0, 1], in groups of at most 2^20 per thread.
struct Stats { float m, s, w; };

__device__ __forceinline__ float reference(float m) { return m == NEG_INF ? 0.f : m; }   // (nothing but -inf: they stay -inf)

// The sums of `a` taken over from its maximum to `m`, which is no smaller.
template <bool ENTROPY>
__device__ __forceinline__ Stats moved(const Stats& a, float m, float c) {
  if (!(a.s > 0.f)) return Stats{m, 0.f, 0.f};               // nothing in it (or NaN, which m tells)
  const float d = a.m - m, f = exp2_fast(d * c);
  // (a maximum far below: f is 0, and d can be -inf)
  return Stats{m, a.s * f, ENTROPY ? f * (a.w + a.s * fmaxf(d, -1000.f)) : 0.f};
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
  float m = a.m;
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    if (n * B < chunks_left)                                 // (the same for all threads)
#pragma unroll
    for (int j = 0; j < N; j += 2) m = max_nan(m, max_nan(Elements<S>::get(v[n], j), Elements<S>::get(v[n], j + 1)));
  }
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
      if (ENTROPY) d = fmaxf(d, -1000.f);                    // exp is 0 there, and 0 times -inf is not
      const float e = exp2_fast(d * c);
      s[j & 1] += e;
      if (ENTROPY) w[j & 1] = fmaf(e, d, w[j & 1]);
    }
  }
  a.s += s[0] + s[1];
  a.w += w[0] + w[1];
}

// The workgroup's joint statistics, the same in every thread; `shared`: 3 floats per wavefront.  Joined in a fixed order.
template <int B, bool ENTROPY>
__device__ __forceinline__ Stats join(Stats a, float c, float* shared) {
  constexpr int WAVES = B / 64;
  float m = a.m;
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max_nan(m, __shfl_xor(m, o));
  a = moved<ENTROPY>(a, m, c);
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    a.s += __shfl_xor(a.s, o);
    if (ENTROPY) a.w += __shfl_xor(a.w, o);
  }
  if (WAVES == 1) return a;
  if ((threadIdx.x & 63) == 0) {
    const int wave = threadIdx.x >> 6;
    shared[wave] = a.m; shared[WAVES + wave] = a.s; shared[2 * WAVES + wave] = a.w;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < WAVES; ++q) m = max_nan(m, shared[q]);
  Stats t = {m, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < WAVES; ++q) {
    const Stats x = moved<ENTROPY>(Stats{shared[q], shared[WAVES + q], shared[2 * WAVES + q]}, m, c);
    t.s += x.s; t.w += x.w;
  }
  return t;
}

// A number whose unsigned order is the logits' (-0 as +0): 1 .. for numbers, so that 0 stands for nothing.
__device__ __forceinline__ unsigned order_key(float z) {
  const unsigned b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// ---- log probabilities ----------------------------------------------------------------------------
struct LogprobArgs {
  const void* logits; int64_t ld; int V;
  const int64_t* tokens;
  int K;
  float* logprob; float* entropy; float* top_logprob; int32_t* top_ids;
};

template <int B>
struct SearchSpace {
  unsigned key[B];                           // of each thread's largest element
  unsigned long long candidate[CANDIDATES];  // key << 32 | ~index: larger is better, and no two are alike
  unsigned hist[256];
  unsigned threshold;
  int count, need;
};

// The exact threshold where the shortcut below collects too many elements (equal logits by the thousand): the K-th largest key, eight
// bits at a time, then by the same means the index up to which elements of just that key are taken, lowest first.  Nine short walks
// of the row.
template <typename S, int B>
__device__ void select_exactly(const S* z, int V, int K, SearchSpace<B>* q) {
  const int tid = threadIdx.x;
  unsigned prefix = 0, index = 0;
  if (tid == 0) q->need = K;
  for (int pass = 0; pass < 8; ++pass) {
    const bool by_index = pass >= 4;                         // (lowest index first: counted upwards)
    const int shift = 24 - 8 * (pass & 3);
    for (int i = tid; i < 256; i += B) q->hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < V; i += B) {
      const unsigned k = order_key(Elements<S>::load(z + i));
      const unsigned x = by_index ? (unsigned)i : k;
      const unsigned seen = by_index ? index : prefix;
      if (by_index && k != prefix) continue;
      if (shift < 24 && (x >> (shift + 8)) != (seen >> (shift + 8))) continue;
      const unsigned bin = (x >> shift) & 255u;
      // (equal elements come in crowds: those of the first active lane's bin are counted together)
      const unsigned lead = (unsigned)__builtin_amdgcn_readfirstlane((int)bin);
      const unsigned long long same = __ballot(bin == lead);
      if (bin != lead) atomicAdd(&q->hist[bin], 1u);
      else if ((tid & 63) == __ffsll((long long)same) - 1) atomicAdd(&q->hist[bin], (unsigned)__popcll(same));
    }
    __syncthreads();
    if (tid == 0) {
      int need = q->need, b = by_index ? 0 : 255;
      const int step = by_index ? 1 : -1;
      while ((int)q->hist[b] < need) { need -= (int)q->hist[b]; b += step; }   // (ends: at least `need` elements are counted)
      q->need = need;
      q->threshold = (unsigned)b;
    }
    __syncthreads();
    if (by_index) index |= q->threshold << shift;
    else prefix |= q->threshold << shift;
  }
  if (tid == 0) q->count = 0;
  __syncthreads();
  for (int i = tid; i < V; i += B) {
    const unsigned k = order_key(Elements<S>::load(z + i));
    if (k > prefix || (k == prefix && (unsigned)i <= index)) {
      const int at = atomicAdd(&q->count, 1);
      if (at < CANDIDATES) q->candidate[at] = ((unsigned long long)k << 32) | (unsigned)~i;   // (K of them)
    }
  }
  __syncthreads();
}

// The K best of a row.  Every thread knows the largest of its own elements; at least K of those are no smaller than the K-th largest
// of them, which is therefore a threshold that the K best reach, and few others do (256 threads, K = 64: about 74 elements).  They are
// collected in any order and sorted by counting, each against all; no two compare equal, so the result has one order.
template <typename S, int B>
__device__ void best_of_row(const Row<S>& row, u32x4 (&held)[NC], int tiles, const LogprobArgs& p, const Stats& own, const Stats& all,
                            int64_t t, SearchSpace<B>* q) {
  constexpr int N = Elements<S>::N;
  const int tid = threadIdx.x, lane = tid & 63;
  const float log_s = logf(all.s);
  float* const out = p.top_logprob + t * p.K;
  int32_t* const ids = p.top_ids + t * p.K;
  if (!(all.m == all.m)) {                                   // NaN in the row: no order
    for (int j = tid; j < p.K; j += B) { out[j] = all.m; ids[j] = j; }
    return;
  }
  unsigned threshold;
  if (p.K == 1) {
    threshold = order_key(all.m);
    if (tid == 0) q->count = 0;
  } else {
    q->key[tid] = tid < row.chunks ? order_key(own.m) : 0u;
    if (tid == 0) q->count = 0;
    __syncthreads();
    if (tid < 64) {
      constexpr int GROUPS = B >= 256 ? 4 : 1, EACH = B / (64 * GROUPS);
      unsigned k[GROUPS];
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        k[g] = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) k[g] = max(k[g], q->key[(e * GROUPS + g) * 64 + lane]);
      }
      unsigned found = 0;                                    // the largest key that at least K groups reach, by its bits (bf16: the upper ones)
      for (int b = 31; b >= (sizeof(S) == 2 ? 16 : 0); --b) {
        const unsigned at = found | (1u << b);
        int n = 0;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) n += __popcll(__ballot(k[g] >= at));
        if (n >= p.K) found = at;
      }
      if (lane == 0) q->threshold = found;
    }
    __syncthreads();
    threshold = q->threshold;
  }
  // (fewer than K groups with elements: everything)
  const float least = threshold <= 0x007fffffu ? NEG_INF : key_value(threshold);
  if (p.K == 1) __syncthreads();                             // the count is 0
  if (own.m >= least) {
    auto collect = [&](const u32x4& v, int c) {
      float m = NEG_INF;
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, Elements<S>::get(v, j));
      if (m < least) return;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float z = Elements<S>::get(v, j);
        const int i = c * N - row.lead + j;
        if (z >= least && i >= 0 && i < row.V) {
          const int at = atomicAdd(&q->count, 1);
          if (at < CANDIDATES) q->candidate[at] = ((unsigned long long)order_key(z) << 32) | (unsigned)~i;
        }
      }
    };
    if (tiles == 1) {
      use_again(held);
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        if (n * B < row.chunks) collect(held[n], n * B + tid);
      }
    } else {
      for (int c = tid; c < row.chunks; c += B)
        collect(row.whole(c) ? *(const u32x4*)(row.at + ((int64_t)c * N - row.lead)) : row.partial(c), c);
    }
  }
  __syncthreads();
  if (q->count > CANDIDATES) {                               // (the same for all threads)
    __syncthreads();
    select_exactly<S, B>(row.at, row.V, p.K, q);
  }
  const int n = q->count;
  for (int i = tid; i < n; i += B) {
    const unsigned long long mine = q->candidate[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += q->candidate[j] > mine;
    if (rank < p.K) {
      const float z = key_value((unsigned)(mine >> 32));
      ids[rank] = (int32_t)~(unsigned)mine;
      out[rank] = all.m == NEG_INF ? NEG_INF : (z - all.m) - log_s;
    }
  }
}

template <typename S, int B>
__global__ __launch_bounds__(B) void token_logprobs_kernel(LogprobArgs p) {
  __shared__ float shared[3 * (B / 64)];
  __shared__ SearchSpace<B> search;
  const int64_t t = blockIdx.x;
  const Row<S> row((const S*)p.logits + t * p.ld, p.V);
  const int tiles = (row.chunks + B * NC - 1) / (B * NC);
  u32x4 v[NC];
  Stats own = {NEG_INF, 0.f, 0.f};
  for (int i = 0; i < tiles; ++i) {
    load_tile<S, B>(row, i, v);
    add_tile<S, B, true>(v, row.chunks - i * (B * NC), own, LOG2E);
  }
  const Stats all = join<B, true>(own, LOG2E, shared);
  if (threadIdx.x == 0) {
    const float log_s = logf(all.s);
    const int64_t y = p.tokens[t];
    float lp = 0.f;                                          // no token given
    if (y >= p.V) lp = __builtin_nanf("");
    else if (y >= 0) lp = all.m == NEG_INF ? NEG_INF : (Elements<S>::load(row.at + y) - all.m) - log_s;
    p.logprob[t] = lp;
    p.entropy[t] = all.m == NEG_INF ? 0.f : fmaxf(log_s - all.w / all.s, 0.f) + 0.f * all.m;   // (NaN and inf of m stay)
  }
  if (p.K > 0) best_of_row<S, B>(row, v, tiles, p, own, all, t, &search);
}

// ---- distillation ---------------------------------------------------------------------------------
enum DistillMode { LOSS = 0, LOSS_AND_GRADIENT = 1, GRADIENT = 2 };

struct DistillArgs {
  const void* logits; int64_t ld; int V;
  const int32_t* ids; const float* teacher; int K;
  float tau;
  const float* weights;                      // LOSS*: optional; GRADIENT: the upstream gradient of each row's loss
  float* loss; float* stats;                 // stats [T, 2]: m and log s of each row (GRADIENT reads them)
  void* grad; int64_t ld_grad;
};

constexpr int MAX_K = 128;                   // two entries per lane of the first wavefront
struct Teacher { int id[MAX_K]; float q[MAX_K]; };

// One wavefront, entries lane and lane + 64: q, the first of several entries with one id carrying their sum in `total`.
struct Entry { int id; float z, q, log_q, total; bool first; };

template <typename S>
__device__ __forceinline__ bool read_teacher(const DistillArgs& p, const Row<S>& row, int64_t t, Teacher* shared, Entry (&e)[2]) {
  const int lane = threadIdx.x & 63;
  const float c = LOG2E / p.tau;
  float x[2], m = NEG_INF;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = lane + 64 * h;
    e[h].id = -1; x[h] = NEG_INF; e[h].z = 0.f;
    if (j < p.K) { e[h].id = p.ids[t * p.K + j]; x[h] = p.teacher[t * p.K + j]; }
    if (e[h].id < 0 || e[h].id >= row.V || x[h] == NEG_INF) { e[h].id = -1; x[h] = NEG_INF; }
    if (e[h].id >= 0) e[h].z = Elements<S>::load(row.at + e[h].id);
    m = max_nan(m, x[h]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max_nan(m, __shfl_xor(m, o));
  if (m == NEG_INF) return false;                            // no alternative is there
  float s = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) { e[h].q = exp2_fast((x[h] - m) * c); s += e[h].q; }
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  const float log_s = logf(s);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    e[h].q /= s;
    e[h].log_q = (x[h] - m) / p.tau - log_s;
    const int j = lane + 64 * h;
    shared->id[j] = e[h].id; shared->q[j] = e[h].q;
    e[h].total = 0.f; e[h].first = e[h].id >= 0;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int j = 0; j < p.K; ++j) {
    const int id = shared->id[j];
    const float q = shared->q[j];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (id == e[h].id) {
        e[h].total += q;
        if (j < lane + 64 * h) e[h].first = false;
      }
  }
  return true;
}

template <typename S, int B>
__device__ __forceinline__ void store_chunk(const Row<S>& row, S* out, bool aligned, int c, const u32x4& v) {
  constexpr int N = Elements<S>::N;
  const int i0 = c * N - row.lead;
  if (aligned && row.whole(c)) {
    *(u32x4*)(out + i0) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const S x = sizeof(S) == 4 ? __builtin_bit_cast(S, (typename std::conditional<sizeof(S) == 4, unsigned, uint16_t>::type)v[sizeof(S) == 4 ? j : 0])
                               : __builtin_bit_cast(S, (typename std::conditional<sizeof(S) == 4, unsigned, uint16_t>::type)(v[j >> 1] >> (16 * (j & 1))));
    if (i0 + j >= 0 && i0 + j < row.V) out[i0 + j] = x;
  }
}

template <typename S, int B, int MODE>
__global__ __launch_bounds__(B) void distill_topk_kernel(DistillArgs p) {
  constexpr int N = Elements<S>::N;
  __shared__ float shared[3 * (B / 64)];
  __shared__ Teacher teacher;
  __shared__ int present;
  const int tid = threadIdx.x;
  const int64_t t = blockIdx.x;
  const Row<S> row((const S*)p.logits + t * p.ld, p.V);
  const int tiles = (row.chunks + B * NC - 1) / (B * NC);
  S* const out = MODE == LOSS ? nullptr : (S*)p.grad + t * p.ld_grad;
  const bool aligned = (((uintptr_t)out ^ (uintptr_t)row.at) & 15) == 0;
  const float weight = p.weights ? p.weights[t] : 1.f;
  auto write_zeros = [&]() {
    for (int c = tid; c < row.chunks; c += B) store_chunk<S, B>(row, out, aligned, c, u32x4{0, 0, 0, 0});
  };
  if (weight == 0.f) {                                       // the row is left out: its logits are not read
    if (MODE != GRADIENT && tid == 0) { p.loss[t] = 0.f; p.stats[2 * t] = 0.f; p.stats[2 * t + 1] = 0.f; }
    if (MODE != LOSS) write_zeros();
    return;
  }
  const float c = LOG2E / p.tau;
  u32x4 v[NC];
  if (tiles == 1) load_tile<S, B>(row, 0, v);                // (on its way while the teacher's entries are read)
  Entry e[2];
  if (tid < 64) {
    const bool any = read_teacher<S>(p, row, t, &teacher, e);
    if (tid == 0) present = any;
    asm volatile("" :: "v"(e[0].z), "v"(e[1].z));            // (they are here: grad may be the logits' own memory)
  }
  float m, log_s, inv_s = 1.f;
  if (MODE != GRADIENT) {
    Stats all = {NEG_INF, 0.f, 0.f};
    for (int i = 0; i < tiles; ++i) {
      if (tiles > 1) load_tile<S, B>(row, i, v);
      add_tile<S, B, false>(v, row.chunks - i * (B * NC), all, c);
    }
    all = join<B, false>(all, c, shared);
    m = all.m; log_s = logf(all.s); inv_s = 1.f / all.s;
  } else {
    m = p.stats[2 * t]; log_s = p.stats[2 * t + 1];
  }
  __syncthreads();
  // No alternative, or no logit above -inf: nothing to learn from.
  const bool nothing = !present || m == NEG_INF;
  if (MODE != GRADIENT && tid < 64) {
    float x = 0.f;
    if (!nothing)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (e[h].id >= 0 && !(e[h].q == 0.f)) x += e[h].q * (e[h].log_q - ((e[h].z - m) / p.tau - log_s));
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    if (tid == 0) {
      p.loss[t] = p.tau * p.tau * x;
      p.stats[2 * t] = m;
      p.stats[2 * t + 1] = m == NEG_INF ? 0.f : log_s;
    }
  }
  if (MODE == LOSS) return;
  if (nothing) {
    write_zeros();
    return;
  }
  // p_i = exp((z_i - m) / tau) / s, the division (GRADIENT: an exponent) once per row
  const float scale = weight * p.tau, shift = MODE == GRADIENT ? -log_s * LOG2E : 0.f;
  const float factor = MODE == GRADIENT ? scale : scale * inv_s;
  for (int i = 0; i < tiles; ++i) {
    if (tiles > 1) load_tile<S, B>(row, i, v);
    else use_again(v);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int at = i * (B * NC) + n * B;
      if (at + tid < row.chunks) {
        float x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float d = Elements<S>::get(v[n], j) - m;
          x[j] = factor * exp2_fast(MODE == GRADIENT ? fmaf(d, c, shift) : d * c);
        }
        store_chunk<S, B>(row, out, aligned, at + tid, Elements<S>::pack(x));
      }
    }
  }
  __syncthreads();                                           // the row is written: the teacher's entries go over it
  if (tid < 64)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (e[h].first) {
        const float d = e[h].z - m;
        const float pz = MODE == GRADIENT ? exp2_fast(fmaf(d, c, shift)) : exp2_fast(d * c) * inv_s;
        Elements<S>::store(out + e[h].id, scale * (pz - e[h].total));
      }
}

// Threads per row.  A row of up to 16 chunks per thread of one wavefront needs no barrier; few rows get 1024 threads, since
// there is nothing else for the compute units to do.
int threads_per_row(int64_t T, int V, moep_dtype dt) {
  const int64_t chunks = ceil_div((int64_t)V * (int64_t)dtype_size(dt), 16) + 1;
  if (T <= 512 && chunks > 256) return 1024;
  return chunks <= 512 && T > 2048 ? 64 : 256;
}

int check_rows(const char* who, int64_t T, int64_t V, moep_dtype dt, const void* logits, int64_t ld) {
  if (dt != MOEP_F32 && dt != MOEP_BF16) return fail(MOEP_EINVAL, "%s: unknown dtype %d", who, (int)dt);
  if (T < 0 || T > (int64_t)1 << 30) return fail(MOEP_EINVAL, "%s: T=%lld out of range [0, 2^30]", who, (long long)T);
  if (V < 1 || V > (int64_t)1 << 28) return fail(MOEP_EINVAL, "%s: V=%lld out of range [1, 2^28]", who, (long long)V);
  if (ld < V) return fail(MOEP_EINVAL, "%s: rows of %lld elements are only %lld apart", who, (long long)V, (long long)ld);
  if ((uintptr_t)logits % dtype_size(dt)) return fail(MOEP_EUNSUPPORTED, "%s: logits are not aligned to their elements", who);
  return MOEP_OK;
}

template <int MODE>
int launch_distill(const DistillArgs& p, int64_t T, moep_dtype dt, hipStream_t s, const char* name) {
  const int threads = threads_per_row(T, p.V, dt);
  Timed timed(name, s);
#define MOEP_DISTILL(S, B) hipLaunchKernelGGL((distill_topk_kernel<S, B, MODE>), dim3((unsigned)T), dim3(B), 0, s, p)
  if (dt == MOEP_BF16) {
    if (threads == 64) MOEP_DISTILL(uint16_t, 64);
    else if (threads == 256) MOEP_DISTILL(uint16_t, 256);
    else MOEP_DISTILL(uint16_t, 1024);
  } else {
    if (threads == 64) MOEP_DISTILL(float, 64);
    else if (threads == 256) MOEP_DISTILL(float, 256);
    else MOEP_DISTILL(float, 1024);
  }
#undef MOEP_DISTILL
  MOEP_HIP(hipGetLastError());
  return MOEP_OK;
}

int check_teacher(const char* who, int64_t T, int K, const void* ids, const void* teacher, float tau) {
  if (K < 1 || K > MAX_K) return fail(MOEP_EINVAL, "%s: K=%d out of range [1, %d]", who, K, MAX_K);
  if (!(tau > 0.f) || tau > 1e30f) return fail(MOEP_EINVAL, "%s: temperature %g must be positive and finite", who, (double)tau);
  if (T > 0 && (!ids || !teacher)) return fail(MOEP_EINVAL, "%s: NULL teacher ids or logits", who);
  return MOEP_OK;
}

}  // namespace
}  // namespace moep

using namespace moep;

extern "C" {

int moe_token_logprobs(const void* logits, int64_t ld, const int64_t* tokens, int64_t T, int64_t V, moep_dtype dt, int K,
                       float* logprob, float* entropy, float* top_logprob, int32_t* top_ids, void* hip_stream) {
  const char* who = "moe_token_logprobs";
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (K < 0 || K > MAX_K || K > V) return fail(MOEP_EINVAL, "%s: K=%d out of range [0, min(%d, V)]", who, K, MAX_K);
  if (T == 0) return MOEP_OK;
  if (!logits || !tokens || !logprob || !entropy) return fail(MOEP_EINVAL, "%s: NULL logits, tokens, logprob or entropy", who);
  if (K > 0 && (!top_logprob || !top_ids)) return fail(MOEP_EINVAL, "%s: NULL top_logprob or top_ids", who);
  LogprobArgs p = {logits, ld, (int)V, tokens, K, logprob, entropy, top_logprob, top_ids};
  hipStream_t s = (hipStream_t)hip_stream;
  int threads = threads_per_row(T, p.V, dt);
  if (threads == 64 && K > 32) threads = 256;                // (a threshold from 64 groups would let too many through)
  Timed timed("token_logprobs", s);
#define MOEP_LOGPROBS(S, B) hipLaunchKernelGGL((token_logprobs_kernel<S, B>), dim3((unsigned)T), dim3(B), 0, s, p)
  if (dt == MOEP_BF16) {
    if (threads == 64) MOEP_LOGPROBS(uint16_t, 64);
    else if (threads == 256) MOEP_LOGPROBS(uint16_t, 256);
    else MOEP_LOGPROBS(uint16_t, 1024);
  } else {
    if (threads == 64) MOEP_LOGPROBS(float, 64);
    else if (threads == 256) MOEP_LOGPROBS(float, 256);
    else MOEP_LOGPROBS(float, 1024);
  }
#undef MOEP_LOGPROBS
  MOEP_HIP(hipGetLastError());
  return MOEP_OK;
}

int moe_distill_topk(const void* logits, int64_t ld, const int32_t* ids, const float* teacher, int64_t T, int64_t V, int K,
                     moep_dtype dt, float temperature, const float* weights, float* loss, float* stats, void* grad,
                     int64_t ld_grad, void* hip_stream) {
  const char* who = "moe_distill_topk";
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (int st = check_teacher(who, T, K, ids, teacher, temperature)) return st;
  if (grad)
    if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (T == 0) return MOEP_OK;
  if (!logits || !loss || !stats) return fail(MOEP_EINVAL, "%s: NULL logits, loss or stats", who);
  DistillArgs p = {logits, ld, (int)V, ids, teacher, K, temperature, weights, loss, stats, grad, ld_grad};
  return grad ? launch_distill<LOSS_AND_GRADIENT>(p, T, dt, (hipStream_t)hip_stream, "distill_loss_gradient")
              : launch_distill<LOSS>(p, T, dt, (hipStream_t)hip_stream, "distill_loss");
}

int moe_distill_topk_backward(const void* logits, int64_t ld, const int32_t* ids, const float* teacher, const float* stats,
                              const float* grad_loss, int64_t T, int64_t V, int K, moep_dtype dt, float temperature, void* grad,
                              int64_t ld_grad, void* hip_stream) {
  const char* who = "moe_distill_topk_backward";
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (int st = check_teacher(who, T, K, ids, teacher, temperature)) return st;
  if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (T == 0) return MOEP_OK;
  if (!logits || !stats || !grad_loss || !grad) return fail(MOEP_EINVAL, "%s: NULL logits, stats, grad_loss or grad", who);
  DistillArgs p = {logits, ld, (int)V, ids, teacher, K, temperature, grad_loss, nullptr, (float*)stats, grad, ld_grad};
  return launch_distill<GRADIENT>(p, T, dt, (hipStream_t)hip_stream, "distill_gradient");
}

}  // extern "C"
