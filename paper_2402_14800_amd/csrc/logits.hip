// Rows of logits [T, V]: log probabilities of given tokens with the entropy and the K best alternatives
// (moe_token_logprobs), and the distillation loss from a teacher's K best logits with its gradient (moe_distill_topk).
//
// With m = max_i z_i, s = sum_i exp((z_i - m) / tau):  log p_i = (z_i - m) / tau - log s, and (tau = 1) the entropy is
// log s - sum_i exp(z_i - m) (z_i - m) / s.  With q the softmax of the teacher's K logits over tau, the loss of a row is
// tau^2 sum_j q_j (log q_j - log p_id(j)), added up as tau sum_j q_j (tau (log q_j + log s) + m - z_id(j)), and its gradient tau (p - q).
//
// Bound by the one read of the logits (and the one write of the gradient); the lanes are close behind: an element of two
// bytes costs about ten lane operations, four of them the exponential.  A workgroup takes a row; each thread keeps its own
// running maximum and sums (a rescale per 16 chunks), so the row is read without a barrier and joined once at its end.  Up to
// 16 chunks of 16 bytes per thread stay in registers, so a row of up to 32768 bf16 logits on 256 threads is read from memory
// once also where it is used again (the gradient, the search for the best); a longer one is walked tile by tile.
// Time and bytes read and written: 1999 rows of 32000 bf16, K = 1 32.0 us (4.0 TB/s: 1280 workgroups fit the chip, so these are 1.6 rounds of
// them), 2048 of 131072, K = 64 114 us (4.7); loss and gradient of 4096 of 32000, K = 64 103 us (5.1, the rate of a copy), of 2048 of
// 131072, K = 100 227 to 234 us (4.6 to 4.7); one row of 32000, K = 20 9 us, the workgroup's own way through it.
// (Workgroups that stay and ask for their next row while they end the present one were slower everywhere, 1.1 to 1.7 times: loads and
// stores return in order, so a row's first chunk waited for the stores before it. More workgroups than fit do the same without.)
#include "logits_rows.h"

namespace moep {
namespace {

// A number whose unsigned order is the logits' (-0 as +0): 1 .. for numbers, so that 0 stands for nothing.
__device__ __forceinline__ unsigned order_key(float z) {
  const unsigned b = __float_as_uint(z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// ---- log probabilities ----------------------------------------------------------------------------
struct LogprobArgs {
  const void* logits; int64_t ld, T; int V;
  const int64_t* tokens;
  int K;
  float* logprob; float* entropy; float* top_logprob; int32_t* top_ids;
};

template <int B>
struct SearchSpace {
  // Chunks with an element that reaches the threshold: each wavefront's in the order it met them, and where they begin in the row.
  // (one wavefront gets less room, so that twenty of them fit a compute unit)
  static constexpr int HITS = B == 64 ? 128 : 512 / (B / 64), CANDIDATES = B == 64 ? 256 : 512;
  u32x4 hit[B / 64 * HITS];
  int hit_at[B / 64 * HITS];
  unsigned threshold_of[2][B / 64];          // the wavefronts', of this tile and the one before
  __attribute__((aligned(16))) unsigned long long candidate[CANDIDATES];   // key << 32 | ~index: larger is better, and no two are alike
  unsigned hist[256];
  unsigned threshold;                        // (of the exact search)
  int count, need;
};

// The exact threshold where the shortcut below collects too many elements (equal logits by the thousand): the K-th largest key, eight
// bits at a time, then by the same means the index up to which elements of just that key are taken, lowest first.  Nine short walks
// of the row: 2048 rows of 32000 equal bf16 logits, K = 64 988 us for 43, one of them 279 for 14.  Short rows come here with ordinary logits
// too, where K comes near the threads that the threshold is taken from, whole wavefronts with a chunk each: 2100 rows of 1000, K = 20 10.5 us,
// 33 21.5, 64 118, 128 83.
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
      if (at < q->CANDIDATES) q->candidate[at] = ((unsigned long long)k << 32) | (unsigned)~i;   // (K of them)
    }
  }
  __syncthreads();
}

// The K best of a row.  Every thread knows the largest of the elements it has seen; if of each of W wavefronts K / W threads' reach a
// threshold, K elements do, the K best among them, and few others (256 threads, K = 64: about 90 elements of a tile).  After every tile
// the threshold is found anew, each wavefront's by itself and the least of them, and the tile's chunks that hold an element which reaches it
// are set aside in LDS while they are in registers; what an earlier, lower threshold let in does no harm.  At the end every lane takes such a
// chunk, and the elements that reach the last threshold are sorted by counting, each against all; no two compare equal, so the result has
// one order.

// A key that at least `need` lanes' reach, and hardly more: `need` plus an eighth.  By bits from two octaves below the largest (most often
// there), else from all of them.  0 if there are not so many.
__device__ __forceinline__ unsigned reached_by(unsigned key, int need, int lowest_bit) {
  const unsigned top = over_wave(key, 0u, [](unsigned a, unsigned b) { return max(a, b); });
  if (need == 1) return top;
  constexpr unsigned TWO_OCTAVES = 1u << 24;
  unsigned found = top > TWO_OCTAVES ? (top - TWO_OCTAVES) & ~0xffffu : 0u;
  int bit = 23;
  if (__popcll(__ballot(key >= found)) < need) { found = 0; bit = 31; }
  for (; bit >= lowest_bit; --bit) {
    const unsigned at = found + (1u << bit);
    const int n = __popcll(__ballot(key >= at));
    if (n >= need) {
      found = at;
      if (n <= need + (need >> 3)) break;
    }
  }
  return found;
}

// The threshold in two halves with a barrier between them, like the statistics.
template <typename S, int B>
__device__ __forceinline__ unsigned threshold_of_wave(float own, bool seen, int chunks, int K, int turn, SearchSpace<B>* q) {
  constexpr int WAVES = B / 64;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // the wavefronts all of whose threads have seen something; one where none has
  const int full = max(1, min(WAVES, chunks / 64));
  unsigned found = ~0u;
  if (wave < full) found = reached_by(seen ? order_key(own) : 0u, (K + full - 1) / full, sizeof(S) == 2 ? 16 : 0);
  if (WAVES > 1 && (threadIdx.x & 63) == 0) q->threshold_of[turn][wave] = found;
  return found;
}
template <int B>
__device__ __forceinline__ float threshold_of_all(unsigned found, int turn, const SearchSpace<B>* q) {
  if (B > 64)
#pragma unroll
    for (int w = 0; w < B / 64; ++w) found = min(found, q->threshold_of[turn][w]);
  found = (unsigned)__builtin_amdgcn_readfirstlane((int)found);
  return found <= 0x007fffffu ? NEG_INF : key_value(found);  // (too few: everything)
}

// Sets aside the chunks of a tile with an element that reaches `least`; `hits`: the wavefront's, before and after (beyond HITS: not kept).
template <typename S, int B>
__device__ __forceinline__ int set_aside(const Row<S>& row, const u32x4 (&v)[NC], int tile, int tid, float least, int hits, SearchSpace<B>* q) {
  constexpr int N = Elements<S>::N, HITS = SearchSpace<B>::HITS;
  const int c0 = tile * (B * NC);
  const int first = __builtin_amdgcn_readfirstlane(tid >> 6) * HITS;
  auto walk = [&](auto some) {
#pragma unroll
    for (int n = 0; n < NC; ++n)
      if (c0 + n * B < row.chunks) {                         // (the same for all threads)
        const bool mine = some(v[n]);
        const unsigned long long mask = __ballot(mine);
        const int at = hits + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
        if (mine && at < HITS) {
          q->hit[first + at] = v[n];
          q->hit_at[first + at] = (c0 + n * B + tid) * N - row.lead;
        }
        hits += __popcll(mask);
      }
  };
  if (sizeof(S) == 2 && least > 0.f) {                       // (bits of numbers that are not negative are in their order)
    const short bits = (short)(__float_as_uint(least) >> 16);
    walk([&](const u32x4& x) {
      const s16x2 top = top_halves(x);
      return max(top[0], top[1]) >= bits;
    });
  } else {
    walk([&](const u32x4& x) {
      float m = Elements<S>::get(x, 0);
#pragma unroll
      for (int j = 1; j < N; ++j) m = fmaxf(m, Elements<S>::get(x, j));
      return m >= least;
    });
  }
  return hits;
}

// The elements that reach `least` of the chunks that the wavefront has set aside: into the workgroup's list.
template <typename S, int B>
__device__ __forceinline__ void expand(int V, int hits, float least, SearchSpace<B>* q) {
  constexpr int N = Elements<S>::N, HITS = SearchSpace<B>::HITS;
  const int lane = threadIdx.x & 63, first = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * HITS;
  if (hits > HITS) {                                         // not all were kept: the exact search
    if (lane == 0) atomicAdd(&q->count, q->CANDIDATES + 1);
    return;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int h0 = 0; h0 < hits; h0 += 64) {
    const bool there = h0 + lane < hits;
    const u32x4 x = there ? q->hit[first + h0 + lane] : neutral<S>();
    const int i0 = there ? q->hit_at[first + h0 + lane] : V;
    unsigned long long mask[N];
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      mask[j] = __ballot(Elements<S>::get(x, j) >= least && i0 + j >= 0 && i0 + j < V);
      n += __popcll(mask[j]);
    }
    int at = 0;
    if (lane == 0) at = atomicAdd(&q->count, n);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if ((mask[j] >> lane) & 1) {
        const int k = at + __builtin_amdgcn_mbcnt_hi((unsigned)(mask[j] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask[j], 0u));
        if (k < q->CANDIDATES) q->candidate[k] = ((unsigned long long)order_key(Elements<S>::get(x, j)) << 32) | (unsigned)~(i0 + j);
      }
      at += __popcll(mask[j]);
    }
  }
}

template <typename S, int B>
__device__ __forceinline__ void write_best(const S* row, const LogprobArgs& p, const Stats& all, int64_t t, SearchSpace<B>* q) {
  const int tid = threadIdx.x;
  const float log_s = logf(all.s);
  float* const out = p.top_logprob + t * p.K;
  int32_t* const ids = p.top_ids + t * p.K;
  if (!(all.s == all.s)) {                                   // NaN or +inf in the row: no order
    for (int j = tid; j < p.K; j += B) { out[j] = all.s; ids[j] = j; }
    return;
  }
  if (q->count > q->CANDIDATES) {                               // (the same for all threads)
    __syncthreads();
    select_exactly<S, B>(row, p.V, p.K, q);
  }
  const int n = q->count;
  // A candidate's rank: how many are larger.  Where there are few of them, several threads share the counting.
  const int share = 4 * n <= B ? 2 : 2 * n <= B ? 1 : 0, part = tid & ((1 << share) - 1);
  for (int i0 = 0; i0 < n; i0 += B >> share) {
    const int i = i0 + (tid >> share);
    const unsigned long long mine = i < n ? q->candidate[i] : ~0ull;
    int rank = 0;
#pragma unroll 4
    for (int j = 2 * part; j < n; j += 2 << share) {
      const u64x2 x = *(const u64x2*)(q->candidate + j);
      rank += (x[0] > mine) + (j + 1 < n && x[1] > mine);
    }
    if (share > 0) rank += __shfl_xor(rank, 1);
    if (share > 1) rank += __shfl_xor(rank, 2);
    if (i < n && part == 0 && rank < p.K) {
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
  int tid = threadIdx.x;
  const int64_t t = blockIdx.x;
  const Row<S> row(p.logits, p.ld, p.V, t, p.T);
  const int64_t y = p.tokens[t];
  u32x4 v[NC];
  Stats own = {NEG_INF, 0.f, 0.f};
  if (tid == 0) search.count = 0;
  int hits = 0;
  float least = NEG_INF, zy = 0.f;
  const int tiles = (row.chunks + B * NC - 1) / (B * NC);
  for (int tile = 0; tile < tiles; ++tile) {
    tid = thread_again(tid);
    request_tile<S, B>(row, tile, tid, v);
    cut_ends<S, B>(row, tile, tid, v);
    add_tile<S, B, true>(v, row.chunks - tile * (B * NC), own, LOG2E);
    // (after the tile's own loads have been waited for one by one: a load that only some lanes make ends that)
    if (tile + 1 == tiles && tid == 0 && y >= 0 && y < p.V) zy = Elements<S>::load(row.at + y);
    unsigned found = 0;
    if (p.K > 0) found = threshold_of_wave<S, B>(own.m, tid < row.chunks, row.chunks, p.K, tile & 1, &search);
    if (tile + 1 == tiles) own = join_wave<B, true>(own, LOG2E, shared);
    else if (p.K == 0) continue;
    __syncthreads();
    if (p.K > 0) {
      least = threshold_of_all<B>(found, tile & 1, &search);
      use_again(v);
      hits = set_aside<S, B>(row, v, tile, tid, least, hits, &search);
    }
  }
  const Stats all = join_all<B, true>(own, LOG2E, shared);
  if (tid == 0) {
    const float log_s = logf(all.s);
    float lp = 0.f;                                          // no token given
    if (y >= p.V) lp = __builtin_nanf("");
    else if (y >= 0) lp = all.m == NEG_INF ? NEG_INF : (zy - all.m) - log_s;
    p.logprob[t] = lp;
    p.entropy[t] = all.m == NEG_INF ? 0.f : max_nan(log_s - all.w / all.s, 0.f);
  }
  if (p.K > 0) {
    expand<S, B>(p.V, hits, least, &search);
    __syncthreads();
    write_best<S, B>(row.at, p, all, t, &search);
  }
}

// ---- distillation ---------------------------------------------------------------------------------
enum DistillMode { LOSS = 0, LOSS_AND_GRADIENT = 1, GRADIENT = 2 };

struct DistillArgs {
  const void* logits; int64_t ld, T; int V;
  const int32_t* ids; const float* teacher; int K;
  float tau;
  const float* weights;                      // LOSS*: optional; GRADIENT: the upstream gradient of each row's loss
  float* loss; float* stats;                 // stats [T, 2]: m and log s of each row (GRADIENT reads them)
  void* grad; int64_t ld_grad;
};

constexpr int MAX_K = 128;                   // two entries per lane of the first wavefront

// A row's alternatives as they are in memory: entries lane and lane + 64 of the first wavefront.
struct Alternatives {
  int id[2];
  float x[2];
};
__device__ __forceinline__ Alternatives request_alternatives(const DistillArgs& p, int64_t t) {
  Alternatives a = {{-1, -1}, {NEG_INF, NEG_INF}};
  if (t < p.T && threadIdx.x < 64)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = threadIdx.x + 64 * h;
      if (j < p.K) { a.id[h] = p.ids[t * p.K + j]; a.x[h] = p.teacher[t * p.K + j]; }
    }
  return a;
}

// What the first wavefront keeps of them while the row is worked on, out of the way of the registers: the id (-1: not there), q, log q, the
// student's logit, and for the first of the entries with one id (ids are all different as a rule) the sum of their q, else -1.
struct __attribute__((aligned(16))) Teacher { int id[MAX_K]; float q[MAX_K], log_q[MAX_K], z[MAX_K], total[MAX_K]; };

// Entries and weights of a row into LDS; whether there is any.  One wavefront.
__device__ __forceinline__ bool weigh(const DistillArgs& p, const Alternatives& a, Teacher* e) {
  const int lane = threadIdx.x & 63;
  const float c = LOG2E / p.tau;
  float q[2], m = NEG_INF;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (a.id[h] >= 0) m = max_nan(m, a.x[h]);
  m = max_over_wave(m);
  const float r = reference(m);                              // (no alternative is there: everything below is 0)
  float s = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) { q[h] = a.id[h] >= 0 ? exp2_fast((a.x[h] - r) * c) : 0.f; s += q[h]; }
  s = sum_over_wave(s);
  const float log_s = logf(s);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = lane + 64 * h;
    q[h] /= s;
    e->id[j] = a.id[h]; e->q[j] = q[h]; e->log_q[j] = (a.x[h] - r) / p.tau - log_s;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // Is an id there twice?  (Entries that are not there have ids of their own, so that they are not found alike.)
  int mine[2], found[2] = {0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h) mine[h] = a.id[h] >= 0 ? a.id[h] : -2 - (lane + 64 * h);
  const bool many = p.K > 64;
#pragma unroll 4
  for (int j = 0; j < p.K; j += 4) {
    const i32x4 id = *(const i32x4*)(e->id + j);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      found[0] += id[k] == mine[0];
      if (many) found[1] += id[k] == mine[1];
    }
  }
  float total[2] = {q[0], q[1]};
  bool first[2] = {a.id[0] >= 0, a.id[1] >= 0};
  if (__ballot(found[0] > 1 || found[1] > 1)) {
    total[0] = total[1] = 0.f;
    for (int j = 0; j < p.K; ++j) {
      const int id = e->id[j];
      const float qj = e->q[j];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (id == a.id[h]) {
          total[h] += qj;
          if (j < lane + 64 * h) first[h] = false;
        }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) e->total[lane + 64 * h] = first[h] ? total[h] : -1.f;
  return !(m == NEG_INF);
}

// HELD: the row fits the workgroup's registers.
template <typename S, int B, int MODE, bool HELD>
__global__ __launch_bounds__(B) void distill_topk_kernel(DistillArgs p) {
  constexpr int N = Elements<S>::N;
  __shared__ float shared[3 * (B / 64)];
  __shared__ Teacher teacher;
  __shared__ int present;
  int tid = threadIdx.x;
  const int64_t t = blockIdx.x;
  const Row<S> row(p.logits, p.ld, p.V, t, p.T);
  const int tiles = HELD ? 1 : (row.chunks + B * NC - 1) / (B * NC);
  S* const out = MODE == LOSS ? nullptr : (S*)p.grad + t * p.ld_grad;
  const bool aligned = (((uintptr_t)out ^ (uintptr_t)row.at) & 15) == 0;
  const float weight = p.weights ? uniform(p.weights[t]) : 1.f;
  auto write_zeros = [&]() {
    for (int k = tid; k < row.chunks; k += B) store_chunk(row, out, aligned, k, u32x4{0, 0, 0, 0});
  };
  if (weight == 0.f) {                                       // the row is left out: its logits are not read
    // (stats of a row without a distribution: its loss is a constant, whatever gradient of it the backward call is given)
    if (MODE != GRADIENT && tid == 0) { p.loss[t] = 0.f; p.stats[2 * t] = NEG_INF; p.stats[2 * t + 1] = 0.f; }
    if (MODE != LOSS) write_zeros();
    return;
  }
  const float c = uniform(LOG2E / p.tau);
  Alternatives alt = request_alternatives(p, t);             // (in front of the row's chunks: loads return in order)
  u32x4 v[NC];
  if (HELD) request_tile<S, B>(row, 0, tid, v);
  float z[2];
  if (tid < 64) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (alt.id[h] >= p.V || alt.x[h] == NEG_INF) alt.id[h] = -1;             // not there
      z[h] = alt.id[h] >= 0 ? Elements<S>::load(row.at + alt.id[h]) : 0.f;
    }
    const bool any = weigh(p, alt, &teacher);
    if (tid == 0) present = any;
  }
  // (they are here before anybody writes: grad may be the logits' own memory)
  auto keep_logits = [&]() {
    if (tid < 64)
#pragma unroll
      for (int h = 0; h < 2; ++h) teacher.z[tid + 64 * h] = z[h];
  };
  float m, log_s, inv_s = 1.f;
  if (MODE != GRADIENT) {
    Stats all = {NEG_INF, 0.f, 0.f};
    for (int i = 0; i < tiles; ++i) {
      tid = thread_again(tid);
      if (!HELD) request_tile<S, B>(row, i, tid, v);
      cut_ends<S, B>(row, i, tid, v);
      add_tile<S, B, false>(v, row.chunks - i * (B * NC), all, c);
    }
    keep_logits();
    all = join_wave<B, false>(all, c, shared);
    __syncthreads();                                         // (`present` is there too)
    all = join_all<B, false>(all, c, shared);
    m = uniform(all.m); log_s = uniform(logf(all.s)); inv_s = uniform(1.f / all.s);
  } else {
    m = uniform(p.stats[2 * t]); log_s = uniform(p.stats[2 * t + 1]);
    keep_logits();
    __syncthreads();
  }
  // No alternative, or no logit above -inf: nothing to learn from.
  const bool nothing = !__builtin_amdgcn_readfirstlane(present) || m == NEG_INF;
  if (MODE != GRADIENT && tid < 64) {
    float x = 0.f;
    if (!nothing)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = tid + 64 * h;
        const float q = teacher.q[j];
        // (the logits' difference is not divided by the temperature: below 1 that overflows for the type's lowest value as a mask)
        if (teacher.id[j] >= 0 && !(q == 0.f)) x += q * fmaf(p.tau, teacher.log_q[j] + log_s, m - teacher.z[j]);
      }
    x = sum_over_wave(x);
    if (tid == 0) {
      p.loss[t] = p.tau * x;
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
  const float scale = uniform(weight * p.tau), shift = MODE == GRADIENT ? uniform(-log_s * LOG2E) : 0.f;
  const float factor = uniform(scale * inv_s);
  for (int i = 0; i < tiles; ++i) {
    tid = thread_again(tid);
    if (!HELD) request_tile<S, B>(row, i, tid, v);
    if (!HELD || MODE == GRADIENT) cut_ends<S, B>(row, i, tid, v);
    else use_again(v);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int at = i * (B * NC) + n * B + tid;
      if (at < row.chunks) {
        float x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float d = Elements<S>::get(v[n], j) - m;
          x[j] = factor * exp2_fast(MODE == GRADIENT ? fmaf(d, c, shift) : d * c);
        }
        store_chunk(row, out, aligned, at, Elements<S>::pack(x));
      }
    }
  }
  __syncthreads();                                           // the row is written: the teacher's entries go over it
  if (tid < 64)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = tid + 64 * h, id = teacher.id[j];
      const float total = teacher.total[j];
      if (id >= 0 && !(total == -1.f)) {
        const float d = teacher.z[j] - m;
        const float pz = MODE == GRADIENT ? exp2_fast(fmaf(d, c, shift)) : exp2_fast(d * c) * inv_s;
        Elements<S>::store(out + id, scale * (pz - total));
      }
    }
}

template <int MODE>
int launch_distill(const DistillArgs& whole, int64_t T, moep_dtype dt, hipStream_t s, const char* name) {
  const int64_t chunks = most_chunks(whole.logits, whole.ld, whole.V, dt);
  const int threads = threads_to_hold(T, chunks);
  Timed timed(name, s);
  for (int64_t t = 0; t < T; t += LAUNCH_ROWS) {
    DistillArgs p = whole;
    p.T = T - t < LAUNCH_ROWS ? T - t : LAUNCH_ROWS;
    const int64_t size = (int64_t)dtype_size(dt);
    p.logits = (const char*)whole.logits + t * whole.ld * size;
    p.ids = whole.ids + t * whole.K;
    p.teacher = whole.teacher + t * whole.K;
    if (p.weights) p.weights += t;
    if (p.loss) p.loss += t;
    p.stats += 2 * t;
    if (p.grad) p.grad = (char*)whole.grad + t * whole.ld_grad * size;
    auto with = [&](auto b, auto held) {
      constexpr int B = decltype(b)::value;
      constexpr bool HELD = decltype(held)::value;
      if (dt == MOEP_BF16) hipLaunchKernelGGL((distill_topk_kernel<uint16_t, B, MODE, HELD>), dim3((unsigned)p.T), dim3(B), 0, s, p);
      else hipLaunchKernelGGL((distill_topk_kernel<float, B, MODE, HELD>), dim3((unsigned)p.T), dim3(B), 0, s, p);
    };
    constexpr auto most = std::integral_constant<int, 1024>{};
    if (!threads) with(most, std::false_type{});
    else if (threads == 1024) with(most, std::true_type{});
    else with_threads(threads, [&](auto b) { with(b, std::true_type{}); });
    MOEP_HIP(hipGetLastError());
  }
  return MOEP_OK;
}

int check_teacher(const char* who, int64_t T, int K, const void* ids, const void* teacher, float tau) {
  if (K < 1 || K > MAX_K) return fail(MOEP_EINVAL, "%s: K=%d out of range [1, %d]", who, K, MAX_K);
  // (beyond, tau^2 or 1 / tau has no 32-bit number: the loss would be infinite or not a number)
  if (!(tau >= 0x1p-60f && tau <= 0x1p60f)) return fail(MOEP_EINVAL, "%s: temperature %g out of range [2^-60, 2^60]", who, (double)tau);
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
  hipStream_t s = (hipStream_t)hip_stream;
  int threads = threads_to_read(T, most_chunks(logits, ld, V, dt));
  if (threads == 64 && K > 32) threads = 128;                // (a threshold from few more than K threads lets too many through)
  Timed timed("token_logprobs", s);
  for (int64_t t = 0; t < T; t += LAUNCH_ROWS) {
    const int64_t rows = T - t < LAUNCH_ROWS ? T - t : LAUNCH_ROWS;
    LogprobArgs p = {(const char*)logits + t * ld * (int64_t)dtype_size(dt), ld, rows, (int)V, tokens + t, K, logprob + t, entropy + t,
                     K ? top_logprob + t * K : nullptr, K ? top_ids + t * K : nullptr};
    with_threads(threads, [&](auto b) {
      constexpr int B = decltype(b)::value;
      if (dt == MOEP_BF16) hipLaunchKernelGGL((token_logprobs_kernel<uint16_t, B>), dim3((unsigned)rows), dim3(B), 0, s, p);
      else hipLaunchKernelGGL((token_logprobs_kernel<float, B>), dim3((unsigned)rows), dim3(B), 0, s, p);
    });
    MOEP_HIP(hipGetLastError());
  }
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
  DistillArgs p = {logits, ld, T, (int)V, ids, teacher, K, temperature, weights, loss, stats, grad, ld_grad};
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
  DistillArgs p = {logits, ld, T, (int)V, ids, teacher, K, temperature, grad_loss, nullptr, (float*)stats, grad, ld_grad};
  return launch_distill<GRADIENT>(p, T, dt, (hipStream_t)hip_stream, "distill_gradient");
}

}  // extern "C"
