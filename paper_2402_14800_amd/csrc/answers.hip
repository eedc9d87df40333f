// Losses on given answers, and their gradients by the logits: the clipped policy loss of sampled tokens (moe_policy_loss) and the loss of
// paired answers (moe_preference_loss).
//
// Of a row z with its token y, lp = (z_y - m) / tau - log s (m, s as in logits.hip), and both losses reach the logits through lp alone:
// with c the loss's derivative by lp, the gradient is c (onehot_y - p) / tau.
//   policy:      r = exp(lp - old), loss = -min(r A, clip(r) A) + kl (exp(e) - e - 1) with e = ref - lp,
//                c = -r A (0 where the clip holds) - kl (exp(e) - 1)
//   preference:  D = sum over an answer's tokens of lp - ref (or their mean), h = beta (D_chosen - D_rejected),
//                loss = -(1 - ls) log sigmoid(h) - ls log sigmoid(-h), c = +-(ls - sigmoid(-h)) beta (over the number of tokens)
// Bound by the read of the logits and the write of the gradient.  The policy loss knows c as soon as its row is summed, so the row stays in
// registers and is read once; a pair's c needs all rows of both answers, so the gradient reads the logits again, last rows first.
// us and bytes read and written: policy loss and gradient of 4096 rows of 32000 bf16 93 (5.6 TB/s); loss, then gradient of 1001 of 50001 22 (4.6) and 31
// (6.5); pairs of 3333 rows of 32000 33 to 35 (6.3 where the call before left something in the caches), 4.9 for the 8 pairs, 63 (6.6).
#include "logits_rows.h"

namespace moep {
namespace {

enum AnswerMode { LOSS = 0, LOSS_AND_GRADIENT = 1, GRADIENT = 2 };

struct AnswerArgs {
  const void* logits; int64_t ld, T; int V;
  const int64_t* tokens;                     // [T]; negative: none
  float tau;
  // policy, LOSS*
  const float* old; const float* advantages; const float* ref;
  float low, high, kl;                       // 1 - clip, 1 + clip
  const float* up;                           // LOSS*: the rows' weights (optional); GRADIENT: the upstream gradient of each row's or pair's loss (optional)
  // preference
  const int64_t* offsets;                    // [2 pairs + 1]; NULL: policy
  int64_t pairs, first;                      // `first`: the launch's first row
  float* loss; float* logprob;
  float* stats;                              // [T, 3]: m, log s, c (GRADIENT reads them)
  void* grad; int64_t ld_grad;
  int64_t stream_rows;                       // the launch's first rows are read past the caches: so many of them
  bool stream_grad;                          // and the gradient is written past them
  int parts, span;                           // GRADIENT: workgroups to a row, and chunks to each of them
  bool all_rows;                             // GRADIENT, preference: rows of no answer get 0, and are not left as they were
};

// exp(x) - 1 - x without the cancellation: 0.5 x^2 and up.  (Series below 0.5: the first term left out is x^10 / 10!, at most 2.2e-9 of the sum.)
__device__ __forceinline__ float exp_beyond_line(float x) {
  if (fabsf(x) < 0.5f) {
    float s = 1.f / 362880.f;
    s = fmaf(s, x, 1.f / 40320.f);
    s = fmaf(s, x, 1.f / 5040.f);
    s = fmaf(s, x, 1.f / 720.f);
    s = fmaf(s, x, 1.f / 120.f);
    s = fmaf(s, x, 1.f / 24.f);
    s = fmaf(s, x, 1.f / 6.f);
    s = fmaf(s, x, 0.5f);
    return s * x * x;
  }
  const float e = expm1f(x);
  return e == -NEG_INF ? e : e - x;                          // (x may be infinite itself)
}

// (z - m) / tau - log s as a number and what its rounding left out: ratios and an answer's sum see differences of such numbers, which are small, and the
// logarithm's own last place is 5e-7 for the sum of a large vocabulary.  s = 2^e f with f next to 1: e log 2 in two parts, the first without
// rounding (12 bits), and a logarithm of at most 0.4.
struct LogProb { float value, rest; };
__device__ __forceinline__ LogProb log_prob(float z, float m, float s, float tau) {
  const float d = z - m, q = d / tau;
  if (!(fabsf(q) < 0x1p100f)) return {q - logf(s), 0.f};     // (-inf, or a mask of the type's lowest value)
  const float back = d - z, d_rest = (z - (d - back)) - (m + back);
  const float q_rest = (fmaf(-q, tau, d) + d_rest) / tau;
  int e;
  float f = frexpf(s, &e);
  if (f < 0.70710678f) { f *= 2.f; --e; }
  constexpr float LN2_HI = 0x1.62ep-1f, LN2_LO = 0x1.0bfbe8p-15f;
  const float hi = (float)e * LN2_HI, lo = fmaf((float)e, LN2_LO, logf(f));
  const float a = q - hi, a_back = a - q, a_rest = (q - (a - a_back)) - (hi + a_back);
  const float small = (a_rest + q_rest) - lo, value = a + small;
  return {value, small - (value - a)};
}

struct Term { float loss, slope; };
__device__ __forceinline__ Term policy_term(const AnswerArgs& p, const LogProb& lp, float old, float A, float ref) {
  Term t = {0.f, 0.f};
  if (!(A == 0.f) || lp.value != lp.value) {                 // (A = 0: nothing to gain either way, also where r is infinite)
    const float r = expf((lp.value - old) + lp.rest);
    // the ratio has gone as far as it may the way the advantage asks for
    const bool far = A > 0.f ? r > p.high : A < 0.f && r < p.low;   // (NaN asks for neither)
    t.loss = far ? -(A > 0.f ? p.high : p.low) * A : -r * A;
    t.slope = far ? 0.f : -r * A;
  }
  if (p.ref) {
    const float e = (ref - lp.value) - lp.rest;
    t.loss = fmaf(p.kl, exp_beyond_line(e), t.loss);
    t.slope = fmaf(-p.kl, expm1f(e), t.slope);
  }
  if (fabsf(t.loss) == -NEG_INF) t.slope = 0.f;              // (an exponential beyond 32 bits: no gradient that could be followed)
  return t;
}

// The answer that row t belongs to: how many of the n ascending offsets are <= t, less one.  64 of them are looked at at once, by every
// wavefront for itself: one round trip up to 63, two up to 4095.  (Offsets in any other order end as well, and within [-1, n).)
// In 32 bits (n < 2^24): of a 64-bit comparison that picked a bound and ended the loop as well, the compiler kept the loop's end alone.
__device__ __forceinline__ int answer_of(const int64_t* offsets, int n, int64_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;                                        // those in front of lo are <= t, those from hi on are not
  while (lo < hi) {
    const int step = (hi - lo + 63) >> 6, at = lo + (lane + 1) * step - 1;
    const int k = __popcll(__ballot(at < hi && offsets[at] <= t));
    hi = min(hi, lo + (k + 1) * step - 1);
    lo = min(lo + k * step, hi);
  }
  return lo - 1;
}

// ---- a row's statistics, where the row is not used again -------------------------------------------
// Four chunks at a time, the next four on their way meanwhile, each four with a running maximum of its own: a wavefront adds up what has
// come while the rest comes, and 32 registers of chunks leave room for twice as many wavefronts as a row that is held.  An element costs
// the lanes seven operations (unpacked, one FMA, the exponential's four, one sum): the exponent is z c - k with k the integer next to m c, whose
// factor exp2(k - m c) is left to the four's sum.  (c = log2(e) / tau is a number of 32 bits.  At temperature 1 it is 1.3e-8 of itself too small, and sums are
// too large by 1.3e-8 for each unit that the logits lie below the maximum; at others the division's rounding comes in: up to 7.3e-8 for each unit of
// (m - z) / tau, in either direction.  A second FMA with what c leaves out took 3 to 7 % of the loss's time for 2e-8 of a log probability at temperature 1.)
constexpr int GROUP = 4;
struct Running {
  float m = NEG_INF, s = 0.f;                // maximum, and sum of exp2((z - m) c)
  float k = 0.f, f = 1.f;                    // k: integer next to m c, f = exp2(k - m c)
  bool near = true;                          // |m c| < 2^20: k is as exact as the exponents need it
};
// (by name: of an array the compiler kept parts in memory)
struct Group {
  u32x4 a, b, c, d;
  template <typename F> __device__ __forceinline__ void each(F f) { f(a, 0); f(b, 1); f(c, 2); f(d, 3); }
};
template <typename S, int B>
__device__ __forceinline__ void request_group(const Row<S>& row, int g, int tid, bool stream, Group& v) {
  if (stream) {
    apart();
    v.each([&](u32x4& x, int n) { request<true>(row, (g * GROUP + n) * B + tid, x); });
    apart();
  } else v.each([&](u32x4& x, int n) { request(row, (g * GROUP + n) * B + tid, x); });
}
template <typename S>
__device__ __forceinline__ float largest_of(Group& v) {
  constexpr int N = Elements<S>::N;
  if constexpr (sizeof(S) == 2) {            // (as in `largest`)
    const s16x2 top = __builtin_elementwise_max(__builtin_elementwise_max(top_halves(v.a), top_halves(v.b)),
                                                __builtin_elementwise_max(top_halves(v.c), top_halves(v.d)));
    const short x = max(top[0], top[1]);
    if (x >= 0) return __uint_as_float((unsigned)x << 16);
  }
  float m = NEG_INF;
  v.each([&](u32x4& x, int) {
#pragma unroll
    for (int j = 0; j < N; ++j) m = max_nan(m, Elements<S>::get(x, j));
  });
  return m;
}
template <typename S>
__device__ __forceinline__ void add_group(Group& v, Running& a, float c) {
  constexpr int N = Elements<S>::N;
  const float m = max_nan(a.m, largest_of<S>(v));
  v.each([](u32x4& x, int) { asm volatile("" : "+v"(x)); });           // (taken apart anew, not held taken apart: see use_again)
  if (!(m == a.m)) {
    a.s = moved<false>(Stats{a.m, a.s, 0.f}, m, c).s;
    a.m = m;
    a.near = fabsf(m * c) < 0x1p20f;
    a.k = a.near ? rintf(m * c) : 0.f;
    a.f = a.near ? exp2_fast(fmaf(-m, c, a.k)) : 1.f;        // (m c is not rounded, as the elements' z c are not)
  }
  float s0 = 0.f, s1 = 0.f;
  auto add = [&](auto exponent) {
    v.each([&](u32x4& x, int) {
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        s0 += exp2_fast(exponent(Elements<S>::get(x, j)));
        s1 += exp2_fast(exponent(Elements<S>::get(x, j + 1)));
      }
    });
  };
  const float r = reference(m);
  if (a.near) add([&](float z) { return fmaf(z, c, -a.k); });
  else add([&](float z) { return (z - r) * c; });            // nothing but -inf so far, logits near the type's ends, or a cold temperature
  a.s = fmaf(s0 + s1, a.f, a.s);
}
// The group's chunks that reach beyond the row cut to it: the row's first and last one, in the threads that hold them.
template <typename S, int B>
__device__ __forceinline__ void cut_group(const Row<S>& row, int g, int tid, Group& v) {
  const int c0 = g * (GROUP * B), last = row.chunks - 1;
  if (row.lead && c0 + tid == 0) v.a = cut(row, 0, v.a);
  if (!row.whole(last) && last >= c0 && last < c0 + GROUP * B && (last - c0) % B == tid && !(row.lead && last == 0)) {
    u32x4 end = v.a;
    v.each([&](u32x4& x, int n) { if (c0 + n * B + tid == last) end = x; });
    end = cut(row, last, end);
    v.each([&](u32x4& x, int n) { if (c0 + n * B + tid == last) x = end; });
  }
}
template <typename S, int B>
__device__ __forceinline__ Stats add_row(const Row<S>& row, int tid, float c, bool stream) {
  const int groups = (row.chunks + GROUP * B - 1) / (GROUP * B);
  Running a;
  Group now, then;
  request_group<S, B>(row, 0, tid, stream, now);
  request_group<S, B>(row, 1, tid, stream, then);
  for (int g = 0; g < groups; g += 2) {
    cut_group<S, B>(row, g, tid, now);
    add_group<S>(now, a, c);
    request_group<S, B>(row, g + 2, tid, stream, now);
    if (g + 1 >= groups) break;              // (the same for all threads)
    cut_group<S, B>(row, g + 1, tid, then);
    add_group<S>(then, a, c);
    request_group<S, B>(row, g + 3, tid, stream, then);
  }
  return Stats{a.m, a.s, 0.f};
}

// HELD: the row fits the workgroup's registers (LOSS_AND_GRADIENT, the one mode that uses a row twice).
template <typename S, int B, int MODE, bool HELD>
__global__ __launch_bounds__(B, MODE != LOSS_AND_GRADIENT ? 7 : 1) void answers_kernel(AnswerArgs p) {
  constexpr int N = Elements<S>::N;
  __shared__ float shared[3 * (B / 64)];
  int tid = threadIdx.x;
  // (the gradient by itself: the rows that the loss read last are the ones that the caches still hold)
  const int64_t t = MODE == GRADIENT ? p.T - 1 - blockIdx.x / (unsigned)p.parts : blockIdx.x;
  const bool stream = MODE != GRADIENT && t < p.stream_rows, stream_grad = MODE == GRADIENT || p.stream_grad;
  const Row<S> row(p.logits, p.ld, p.V, t, p.T);
  S* const out = MODE == LOSS ? nullptr : (S*)p.grad + t * p.ld_grad;
  const bool aligned = (((uintptr_t)out ^ (uintptr_t)row.at) & 15) == 0;
  const int c_first = MODE == GRADIENT ? (int)(blockIdx.x % (unsigned)p.parts) * p.span : 0;
  const int c_end = MODE == GRADIENT ? min(row.chunks, c_first + p.span) : row.chunks;
  auto write_zeros = [&]() {
    for (int k = c_first + tid; k < c_end; k += B) store_chunk(row, out, aligned, k, u32x4{0, 0, 0, 0}, stream_grad);
  };
  const int64_t y = p.tokens[t];
  const float c = uniform(LOG2E / p.tau);
  float m, scale, factor, shift = 0.f;                       // the gradient is scale [i = y] - factor exp2((z - m) c + shift)
  u32x4 v[HELD ? NC : 1];
  if (MODE != GRADIENT) {
    bool left_out = y < 0;
    if (p.offsets) left_out = left_out || p.first + t < p.offsets[0] || p.first + t >= p.offsets[2 * p.pairs];
    const float weight = !p.offsets && p.up ? uniform(p.up[t]) : 1.f;
    if (left_out || weight == 0.f) {                         // its logits are not read
      if (tid == 0) {
        if (!p.offsets) p.loss[t] = 0.f;
        p.logprob[t] = 0.f;
        p.stats[3 * t] = NEG_INF; p.stats[3 * t + 1] = 0.f; p.stats[3 * t + 2] = 0.f;
      }
      if (MODE == LOSS_AND_GRADIENT) write_zeros();
      return;
    }
    float zy = y < p.V ? Elements<S>::load(row.at + y) : __builtin_nanf("");
    float old = 0.f, A = 0.f, ref = 0.f;
    if (!p.offsets) {
      old = p.old[t]; A = p.advantages[t];
      if (p.ref) ref = p.ref[t];
    }
    Stats all = {NEG_INF, 0.f, 0.f};
    if constexpr (!HELD) {
      all = add_row<S, B>(row, tid, c, stream);
    } else {
      if (stream) {
        apart();
        request_tile<S, B, true>(row, 0, tid, v);
        apart();
      } else {
        request_tile<S, B>(row, 0, tid, v);
      }
      cut_ends<S, B>(row, 0, tid, v);
      add_tile<S, B, false>(v, row.chunks, all, c);
    }
    zy = uniform(zy);                                        // (here before anybody writes: grad may be the logits' own memory)
    all = join_wave<B, false>(all, c, shared);
    __syncthreads();
    all = join_all<B, false>(all, c, shared);
    m = uniform(all.m);
    const float log_s = uniform(logf(all.s));
    LogProb lp = {NEG_INF, 0.f};
    if (!(y < p.V)) lp.value = __builtin_nanf("");
    else if (!(m == NEG_INF)) lp = log_prob(zy, m, uniform(all.s), p.tau);
    Term term = {0.f, 0.f};
    if (!p.offsets) term = policy_term(p, lp, old, A, ref);
    if (tid == 0) {
      if (!p.offsets) p.loss[t] = term.loss;
      p.logprob[t] = lp.value;
      // (of a pair's row what lp left out, where its derivative will be)
      p.stats[3 * t] = m; p.stats[3 * t + 1] = m == NEG_INF ? 0.f : log_s; p.stats[3 * t + 2] = p.offsets ? lp.rest : term.slope;
    }
    if (MODE == LOSS) return;
    scale = uniform(term.slope * weight / p.tau);
    factor = uniform(scale / all.s);
    if (term.slope == 0.f) {
      write_zeros();
      return;
    }
  } else {
    const float slope = uniform(p.stats[3 * t + 2]);
    m = uniform(p.stats[3 * t]);
    shift = uniform(-p.stats[3 * t + 1] * LOG2E);
    float up = 1.f;
    if (p.offsets) {
      const int pairs = (int)p.pairs, a = answer_of(p.offsets, 2 * pairs + 1, p.first + t);
      if (a < 0 || a >= 2 * pairs) {                         // a row of no answer
        if (p.all_rows) write_zeros();
        return;
      }
      if (p.up) up = uniform(p.up[a < pairs ? a : a - pairs]);
    } else if (p.up) {
      up = uniform(p.up[t]);
    }
    if (slope == 0.f || up == 0.f || m == NEG_INF || y < 0) { // (its logits are not read; nothing but -inf has no distribution)
      write_zeros();
      return;
    }
    scale = uniform(slope * up / p.tau);
    factor = scale;
  }
  const int at_y = y < p.V ? (int)((y + row.lead) / N) : -1, of_y = y < p.V ? (int)((y + row.lead) % N) : 0;
  auto write = [&](const u32x4& z, int at) {
    if (at >= c_end) return;
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = Elements<S>::get(z, j) - m;
      x[j] = -factor * exp2_fast(MODE == GRADIENT ? fmaf(d, c, shift) : d * c);
    }
    if (at == at_y)
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] += j == of_y ? scale : 0.f;
    store_chunk(row, out, aligned, at, Elements<S>::pack(x), stream_grad);
  };
  if constexpr (HELD) {
    tid = thread_again(tid);
    use_again(v);
#pragma unroll
    for (int n = 0; n < NC; ++n) write(v[n], n * B + tid);
  } else {
    const int first = c_first / (GROUP * B), end = (c_end + GROUP * B - 1) / (GROUP * B);
    Group now, then;
    request_group<S, B>(row, first, tid, false, now);
    for (int g = first; g < end; ++g) {
      if (g + 1 < end) request_group<S, B>(row, g + 1, tid, false, then);
      cut_group<S, B>(row, g, tid, now);
      now.each([&](u32x4& x, int n) { write(x, (g * GROUP + n) * B + tid); });
      now = then;
    }
  }
}

// A pair: both answers' sums of lp - ref in 64 bits, the loss, the rewards, and c of every row of theirs.
struct PairArgs {
  const int64_t* tokens; const int64_t* offsets; const float* ref; const float* logprob;
  int64_t T, pairs;
  float beta, smoothing;
  int average;
  float* loss; float* rewards; float* stats;
};
constexpr int PAIR_THREADS = 512, SIDE_WAVES = PAIR_THREADS / 128;    // half of the threads to an answer
static_assert(SIDE_WAVES == 4, "four sums are added below");

__global__ __launch_bounds__(PAIR_THREADS) void pairs_kernel(PairArgs p) {
  __shared__ double sums[2][SIDE_WAVES];
  __shared__ int64_t given[2][SIDE_WAVES];
  const int side = threadIdx.x >= PAIR_THREADS / 2 ? 1 : 0, tid = threadIdx.x & (PAIR_THREADS / 2 - 1);
  const int64_t pair = blockIdx.x;
  const int64_t* const at = p.offsets + (side ? p.pairs + pair : pair);
  const int64_t r0 = max((int64_t)0, min(p.T, at[0])), r1 = max((int64_t)0, min(p.T, at[1]));
  {
    double x = 0;
    int64_t n = 0;
    constexpr int DEEP = 4;
    for (int64_t t = r0 + tid; t < r1; t += DEEP * (PAIR_THREADS / 2)) {
      int64_t y[DEEP];
      float lp[DEEP], rest[DEEP], ref[DEEP];
#pragma unroll
      for (int q = 0; q < DEEP; ++q) {       // (beyond the end the last row again: all loads at once)
        const int64_t i = min(t + q * (PAIR_THREADS / 2), r1 - 1);
        y[q] = p.tokens[i]; lp[q] = p.logprob[i]; rest[q] = p.stats[3 * i + 2]; ref[q] = p.ref[i];
      }
#pragma unroll
      for (int q = 0; q < DEEP; ++q)
        if (t + q * (PAIR_THREADS / 2) < r1 && y[q] >= 0) {
          x += ((double)lp[q] - (double)ref[q]) + (double)rest[q];
          ++n;
        }
    }
    for (int d = 32; d > 0; d >>= 1) {
      x += __shfl_xor(x, d);
      n += __shfl_xor(n, d);
    }
    if ((tid & 63) == 0) { sums[side][tid >> 6] = x; given[side][tid >> 6] = n; }
  }
  __syncthreads();
  double reward[2], by[2];
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const double x = (sums[a][0] + sums[a][1]) + (sums[a][2] + sums[a][3]);
    const int64_t n = given[a][0] + given[a][1] + given[a][2] + given[a][3];
    by[a] = (double)p.beta / (double)(p.average && n > 0 ? n : 1);
    reward[a] = by[a] * x;
  }
  const double h = reward[0] - reward[1], ls = (double)p.smoothing;
  const double e = exp(-fabs(h)), by_h = ls - (h > 0 ? e : 1.0) / (1 + e);
  const float c = (float)((side ? -by_h : by_h) * by[side]);
  for (int64_t t = r0 + tid; t < r1; t += PAIR_THREADS / 2) p.stats[3 * t + 2] = p.tokens[t] >= 0 ? c : 0.f;
  if (threadIdx.x == 0) {
    // -log sigmoid(h) = max(-h, 0) + log(1 + exp(-|h|)), and the other one is h more
    const double away = log1p(e);
    const double loss = (1 - ls) * (fmax(-h, 0.0) + away) + (ls > 0 ? ls * (fmax(h, 0.0) + away) : 0.0);
    p.loss[pair] = (float)(h == h ? loss : h);
    p.rewards[pair] = (float)reward[0];
    p.rewards[p.pairs + pair] = (float)reward[1];
  }
}

// Threads per row where it is not held.  us, 64 / 256 / 512 threads.  The loss alone: 1 row of 32000 bf16 - / 7.9 / 7.5; 128 of 131072 - / 18.3 / 14.6; 300 of
// 50001 - / 14.9 / 15.5; 700 of 32000 - / 14.0 / 16.0; 1001 of 50001 - / 24.1 / 26.3; 4096 of 1000 8.1 / 16.8 / -; 4096 of 4000 13.1 / 16.6 / -; 8192 of 8000
// 30.2 / 32.0 / -, of 4000 fp32 28.2 / 26.7 / -; 1024 of 8000 12.1 / 9.6 / -; 2048 of 8000 11.7 / 12.5 / -, of 1000 6.9 / 11.0 / -.  The gradient alone: 5000 of 4000
// 16.5 / 18.3 / 22.5; 3256 of 32000 - / 75.5 / 72.1; 8192 of 32000 - / 198 / 195.
int threads_to_walk(int64_t T, int64_t chunks, bool gradient) {
  if (chunks <= 64 * GROUP * 4 && T > 2048) return 64;
  if (gradient) return chunks <= 512 * GROUP ? 256 : 512;
  return T >= 256 || chunks <= 256 * GROUP ? 256 : 512;
}
// Workgroups to a row of a gradient alone, of `turns` groups of chunks: as many as fill the chip where rows are few.  us, one / so many: 1 row of
// 262144 bf16 28 / 6.2, 20 31 / 8.1, 128 of 131072 19.5 / 13.6, 300 of 50001 16.3 / 14.5 (6.1 of each the time of an empty launch as measured here).
int64_t row_parts(int64_t T, int64_t turns) {
  const int64_t parts = 1024 / T;
  return parts < 1 ? 1 : parts < turns ? parts : turns;
}
// The caches (256 MB behind the XCDs') and what passes them by.  A gradient that comes by itself is written past them, so that they keep the logits that
// it has yet to read, and its lines need not be written back while the next call reads; the loss alone reads past them what they could not
// keep for the gradient.  us, without the two / with the first / with both, loss and gradient of pairs: 500 rows of 131072 bf16 92 / 75 / 75,
// 3256 of 32000 135 / 120 / 115, 8192 of 32000 311 / 292 / 290; keeping 100 MB instead of 160: 82, 119, 290.  Loss and gradient in one read: the logits are not
// read again, so those of a large batch come past the caches, and the gradient goes past them if it is more than they hold: 3256 of
// 32000 83 / 71, 4096 of 32000 101 / 88, 8192 of 32000 191 / 180 (the logits alone past them 193), 1001 of 50001 (100 MB) the same.
constexpr double HELD_BYTES = 268.5e6, LARGE_BYTES = 134e6, KEPT_BYTES = 160e6;
template <int MODE>
int launch_answers(const AnswerArgs& whole, int64_t T, moep_dtype dt, hipStream_t s, const char* name) {
  const int64_t chunks = most_chunks(whole.logits, whole.ld, whole.V, dt);
  const int threads = MODE == LOSS_AND_GRADIENT ? threads_to_hold(T, chunks) : threads_to_walk(T, chunks, MODE == GRADIENT);
  const int64_t turns = threads ? ceil_div(chunks, (int64_t)GROUP * threads) : 1;
  const int64_t parts = MODE == GRADIENT ? row_parts(T, turns) : 1;
  const double bytes = (double)whole.V * (double)dtype_size(dt);       // of a row
  // rows of the loss alone in front of those that the caches can keep for the gradient; all of a large batch whose gradient comes with it
  const int64_t streamed = MODE == LOSS ? T - (int64_t)(KEPT_BYTES / bytes) : bytes * (double)T > LARGE_BYTES ? T : 0;
  Timed timed(name, s);
  const int64_t launches = ceil_div(T, LAUNCH_ROWS);
  for (int64_t i = 0; i < launches; ++i) {
    const int64_t t = (MODE == GRADIENT ? launches - 1 - i : i) * LAUNCH_ROWS;
    AnswerArgs p = whole;
    p.T = T - t < LAUNCH_ROWS ? T - t : LAUNCH_ROWS;
    p.first = t;
    p.stream_rows = streamed - t;
    p.stream_grad = bytes * (double)T > HELD_BYTES;
    p.parts = (int)parts;
    p.span = (int)(ceil_div(turns, parts) * GROUP * threads);
    const unsigned blocks = (unsigned)(p.T * parts);
    const int64_t size = (int64_t)dtype_size(dt);
    p.logits = (const char*)whole.logits + t * whole.ld * size;
    p.tokens += t;
    if (p.old) p.old += t;
    if (p.advantages) p.advantages += t;
    if (p.ref) p.ref += t;
    if (p.up && !p.offsets) p.up += t;
    if (p.loss && !p.offsets) p.loss += t;
    if (p.logprob) p.logprob += t;
    p.stats += 3 * t;
    if (p.grad) p.grad = (char*)whole.grad + t * whole.ld_grad * size;
    auto with = [&](auto b, auto held) {
      constexpr int B = decltype(b)::value;
      constexpr bool HELD = decltype(held)::value && MODE == LOSS_AND_GRADIENT;
      if (dt == MOEP_BF16) hipLaunchKernelGGL((answers_kernel<uint16_t, B, MODE, HELD>), dim3(blocks), dim3(B), 0, s, p);
      else hipLaunchKernelGGL((answers_kernel<float, B, MODE, HELD>), dim3(blocks), dim3(B), 0, s, p);
    };
    if constexpr (MODE != LOSS_AND_GRADIENT) {
      if (threads == 64) with(std::integral_constant<int, 64>{}, std::false_type{});
      else if (threads == 256) with(std::integral_constant<int, 256>{}, std::false_type{});
      else with(std::integral_constant<int, 512>{}, std::false_type{});
    } else {
      constexpr auto most = std::integral_constant<int, 1024>{};
      if (!threads) with(most, std::false_type{});
      else if (threads == 1024) with(most, std::true_type{});
      else with_threads(threads, [&](auto b) { with(b, std::true_type{}); });
    }
    MOEP_HIP(hipGetLastError());
  }
  return MOEP_OK;
}

int check_temperature(const char* who, float tau) {
  // (as for distillation: beyond, 1 / tau or what it multiplies has no 32-bit number)
  if (!(tau >= 0x1p-60f && tau <= 0x1p60f)) return fail(MOEP_EINVAL, "%s: temperature %g out of range [2^-60, 2^60]", who, (double)tau);
  return MOEP_OK;
}
int check_scalars(const char* who, std::initializer_list<const void*> of4, std::initializer_list<const void*> of8) {
  for (const void* q : of4)
    if ((uintptr_t)q & 3) return fail(MOEP_EUNSUPPORTED, "%s: fp32 arrays must be 4-byte aligned", who);
  for (const void* q : of8)
    if ((uintptr_t)q & 7) return fail(MOEP_EUNSUPPORTED, "%s: tokens and offsets must be 8-byte aligned", who);
  return MOEP_OK;
}

// `all_rows`: the gradient's rows of no answer are written too, with 0.
int preference_loss(const char* who, const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* ref_logprob, int64_t T,
                    int64_t V, int64_t pairs, moep_dtype dt, float beta, float smoothing, int average, const float* weights, float* loss,
                    float* rewards, float* logprob, float* stats, void* grad, int64_t ld_grad, bool all_rows, hipStream_t s) {
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (pairs < 0 || pairs > (int64_t)1 << 22) return fail(MOEP_EINVAL, "%s: %lld pairs out of range [0, 2^22]", who, (long long)pairs);
  if (!(beta > 0.f && beta <= 0x1p60f)) return fail(MOEP_EINVAL, "%s: beta %g out of range (0, 2^60]", who, (double)beta);
  if (!(smoothing >= 0.f && smoothing < 1.f)) return fail(MOEP_EINVAL, "%s: smoothing %g out of range [0, 1)", who, (double)smoothing);
  if (average != 0 && average != 1) return fail(MOEP_EINVAL, "%s: average=%d is neither 0 nor 1", who, average);
  if (grad)
    if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (!offsets) return fail(MOEP_EINVAL, "%s: NULL offsets", who);
  if (pairs > 0 && (!loss || !rewards)) return fail(MOEP_EINVAL, "%s: NULL loss or rewards", who);
  if (T > 0 && (!logits || !tokens || !ref_logprob || !logprob || !stats))
    return fail(MOEP_EINVAL, "%s: NULL logits, tokens, ref_logprob, logprob or stats", who);
  if (int st = check_scalars(who, {ref_logprob, weights, loss, rewards, logprob, stats}, {tokens, offsets})) return st;
  AnswerArgs p = {logits, ld, T, (int)V, tokens, 1.f, nullptr, nullptr, nullptr, 0.f, 0.f, 0.f, nullptr, offsets, pairs, 0,
                  nullptr, logprob, stats, nullptr, 0};
  if (T > 0)
    if (int st = launch_answers<LOSS>(p, T, dt, s, "answer_logprobs")) return st;
  if (pairs > 0) {
    Timed timed("pairs", s);
    const PairArgs q = {tokens, offsets, ref_logprob, logprob, T, pairs, beta, smoothing, average, loss, rewards, stats};
    hipLaunchKernelGGL(pairs_kernel, dim3((unsigned)pairs), dim3(PAIR_THREADS), 0, s, q);
    MOEP_HIP(hipGetLastError());
  }
  if (!grad || T == 0 || (pairs == 0 && !all_rows)) return MOEP_OK;
  p.up = weights; p.grad = grad; p.ld_grad = ld_grad; p.all_rows = all_rows;
  return launch_answers<GRADIENT>(p, T, dt, s, "preference_gradient");
}

int preference_gradient(const char* who, const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* stats,
                        const float* grad_loss, int64_t T, int64_t V, int64_t pairs, moep_dtype dt, void* grad, int64_t ld_grad, bool all_rows,
                        hipStream_t s) {
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (pairs < 0 || pairs > (int64_t)1 << 22) return fail(MOEP_EINVAL, "%s: %lld pairs out of range [0, 2^22]", who, (long long)pairs);
  if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (T == 0 || (pairs == 0 && !all_rows)) return MOEP_OK;
  if (!logits || !tokens || !offsets || !stats || (pairs > 0 && !grad_loss) || !grad)
    return fail(MOEP_EINVAL, "%s: NULL logits, tokens, offsets, stats, grad_loss or grad", who);
  if (int st = check_scalars(who, {stats, grad_loss}, {tokens, offsets})) return st;
  AnswerArgs p = {logits, ld, T, (int)V, tokens, 1.f, nullptr, nullptr, nullptr, 0.f, 0.f, 0.f, grad_loss, offsets, pairs, 0,
                  nullptr, nullptr, (float*)stats, grad, ld_grad};
  p.all_rows = all_rows;
  return launch_answers<GRADIENT>(p, T, dt, s, "preference_gradient");
}

}  // namespace
}  // namespace moep

using namespace moep;

extern "C" {

int moe_policy_loss(const void* logits, int64_t ld, const int64_t* tokens, const float* old_logprob, const float* advantages,
                    const float* ref_logprob, int64_t T, int64_t V, moep_dtype dt, float clip_low, float clip_high, float kl, float temperature,
                    const float* weights, float* loss, float* logprob, float* stats, void* grad, int64_t ld_grad, void* hip_stream) {
  const char* who = "moe_policy_loss";
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (int st = check_temperature(who, temperature)) return st;
  if (!(clip_low >= 0.f && clip_low <= 1.f)) return fail(MOEP_EINVAL, "%s: clip_low %g out of range [0, 1]", who, (double)clip_low);
  if (!(clip_high >= 0.f && clip_high <= 0x1p60f)) return fail(MOEP_EINVAL, "%s: clip_high %g out of range [0, 2^60]", who, (double)clip_high);
  if (!(kl >= 0.f && kl <= 0x1p60f)) return fail(MOEP_EINVAL, "%s: kl %g out of range [0, 2^60]", who, (double)kl);
  if (grad)
    if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (T == 0) return MOEP_OK;
  if (!logits || !tokens || !old_logprob || !advantages || !loss || !logprob || !stats)
    return fail(MOEP_EINVAL, "%s: NULL logits, tokens, old_logprob, advantages, loss, logprob or stats", who);
  if (kl > 0.f && !ref_logprob) return fail(MOEP_EINVAL, "%s: the KL term needs ref_logprob", who);
  if (int st = check_scalars(who, {old_logprob, advantages, ref_logprob, weights, loss, logprob, stats}, {tokens})) return st;
  const AnswerArgs p = {logits, ld, T, (int)V, tokens, temperature, old_logprob, advantages, kl > 0.f ? ref_logprob : nullptr, 1.f - clip_low,
                        1.f + clip_high, kl, weights, nullptr, 0, 0, loss, logprob, stats, grad, ld_grad};
  return grad ? launch_answers<LOSS_AND_GRADIENT>(p, T, dt, (hipStream_t)hip_stream, "policy_loss_gradient")
              : launch_answers<LOSS>(p, T, dt, (hipStream_t)hip_stream, "policy_loss");
}

int moe_policy_loss_backward(const void* logits, int64_t ld, const int64_t* tokens, const float* stats, const float* grad_loss, int64_t T,
                             int64_t V, moep_dtype dt, float temperature, void* grad, int64_t ld_grad, void* hip_stream) {
  const char* who = "moe_policy_loss_backward";
  if (int st = check_rows(who, T, V, dt, logits, ld)) return st;
  if (int st = check_temperature(who, temperature)) return st;
  if (int st = check_rows(who, T, V, dt, grad, ld_grad)) return st;
  if (T == 0) return MOEP_OK;
  if (!logits || !tokens || !stats || !grad_loss || !grad) return fail(MOEP_EINVAL, "%s: NULL logits, tokens, stats, grad_loss or grad", who);
  if (int st = check_scalars(who, {stats, grad_loss}, {tokens})) return st;
  const AnswerArgs p = {logits, ld, T, (int)V, tokens, temperature, nullptr, nullptr, nullptr, 0.f, 0.f, 0.f, grad_loss, nullptr, 0, 0,
                        nullptr, nullptr, (float*)stats, grad, ld_grad};
  return launch_answers<GRADIENT>(p, T, dt, (hipStream_t)hip_stream, "policy_gradient");
}

int moe_preference_loss(const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* ref_logprob, int64_t T,
                        int64_t V, int64_t pairs, moep_dtype dt, float beta, float smoothing, int average, const float* weights, float* loss,
                        float* rewards, float* logprob, float* stats, void* grad, int64_t ld_grad, void* hip_stream) {
  return preference_loss("moe_preference_loss", logits, ld, tokens, offsets, ref_logprob, T, V, pairs, dt, beta, smoothing, average, weights, loss,
                         rewards, logprob, stats, grad, ld_grad, false, (hipStream_t)hip_stream);
}

int moe_preference_loss_all_rows(const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* ref_logprob,
                                 int64_t T, int64_t V, int64_t pairs, moep_dtype dt, float beta, float smoothing, int average,
                                 const float* weights, float* loss, float* rewards, float* logprob, float* stats, void* grad, int64_t ld_grad,
                                 void* hip_stream) {
  const char* who = "moe_preference_loss_all_rows";
  if (T > 0 && !grad) return fail(MOEP_EINVAL, "%s: NULL grad", who);
  return preference_loss(who, logits, ld, tokens, offsets, ref_logprob, T, V, pairs, dt, beta, smoothing, average, weights, loss, rewards, logprob,
                         stats, grad, ld_grad, true, (hipStream_t)hip_stream);
}

int moe_preference_loss_backward(const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* stats,
                                 const float* grad_loss, int64_t T, int64_t V, int64_t pairs, moep_dtype dt, void* grad, int64_t ld_grad,
                                 void* hip_stream) {
  return preference_gradient("moe_preference_loss_backward", logits, ld, tokens, offsets, stats, grad_loss, T, V, pairs, dt, grad, ld_grad, false,
                             (hipStream_t)hip_stream);
}

int moe_preference_loss_backward_all_rows(const void* logits, int64_t ld, const int64_t* tokens, const int64_t* offsets, const float* stats,
                                          const float* grad_loss, int64_t T, int64_t V, int64_t pairs, moep_dtype dt, void* grad, int64_t ld_grad,
                                          void* hip_stream) {
  return preference_gradient("moe_preference_loss_backward_all_rows", logits, ld, tokens, offsets, stats, grad_loss, T, V, pairs, dt, grad, ld_grad,
                             true, (hipStream_t)hip_stream);
}

}  // extern "C"
