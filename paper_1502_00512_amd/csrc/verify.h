// Verification of drafted words against a target model's distribution, from given random numbers.
//   p_i = softmax(target_i / tau),  q_i = softmax(draft_i / tau_d)  (no draft logits: q_i has all its mass on the draft d_i)
//   draft i is accepted iff u_i q_i(d_i) < p_i(d_i); n = drafts accepted before the first that is not
//   the word after them is drawn from r = max(p_n - q_n, 0) (all of the text's drafts accepted, or r = 0: r = p_n): the first
//   v with sum_{j <= v} r_j > u_K sum_j r_j
// Which step of a sum over the vocabulary a random number falls on depends on every term: 100000 terms of 32 bits leave the
// step open once in some hundred words, so the drawn word's row is summed in 64 bits with exponentials to 1e-14.  The
// acceptance of a draft compares two probabilities and gets by with 32-bit sums.
//   1. maximum and sum of exponentials of every row that can matter, by parts of a row (HBM-bound; all the bytes are here)
//   2. how many drafts are accepted; sums of exponentials of the one row pair that is drawn from, in 64 bits
//   3. sums of r by parts      4. the part, the thread's stretch of it and the word on which u_K falls
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int VERIFY_THREADS = 256, VERIFY_PARTS = 64;

struct VerifySeq {  // what the steps behind the second one know of a text
  int n;            // accepted
  int mixed;        // the drawn row is p - q (else p alone)
  float mp, mq;     // maxima of the drawn rows
};

struct VerifyArgs {
  const void *target, *draft;  // draft may be nullptr
  long ldt, ldd;
  const int32_t *drafts, *lengths;  // lengths may be nullptr
  const float *u;
  int V, B, K, parts, per;  // per: slots of a part
  float tau, tau_d;
  int32_t *accepted, *tokens, *range_flag;
  float2 *stat;    // [row][part], rows of the target then of the draft
  double *sums;    // [text][part][2]: sums of exponentials of p, q
  double *rest;    // [text][part]: sums of r
  VerifySeq *seq;  // [text]
};

__device__ inline int draft_length(const VerifyArgs &a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.K) : a.K;
}

// 2^x to 64 bits: x = n + f with |f| <= 1/2 and the series of 2^f, whose 12th term is below 2e-14.
__device__ inline double exp2_64(double x) {
  x = x < -1100.0 ? -1100.0 : x;  // (a NaN stays one)
  const double n = rint(x), f = (x - n) * LN2_64;
  double p = 1.0 / 39916800.0;
  p = fma(p, f, 1.0 / 3628800.0);
  p = fma(p, f, 1.0 / 362880.0);
  p = fma(p, f, 1.0 / 40320.0);
  p = fma(p, f, 1.0 / 5040.0);
  p = fma(p, f, 1.0 / 720.0);
  p = fma(p, f, 1.0 / 120.0);
  p = fma(p, f, 1.0 / 24.0);
  p = fma(p, f, 1.0 / 6.0);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}
// e^{(z - m) / tau} of a row: z c + b.
struct Exp64 {
  double c, b;
  __device__ Exp64(float m, float tau) {
    c = LOG2E_64 / (double)tau;
    b = m == -INFINITY ? 0.0 : -(double)m * c;
  }
  __device__ double operator()(float z) const { return exp2_64(fma((double)z, c, b)); }
};

template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_stats_kernel(const VerifyArgs a) {
  constexpr int N = SlotOf<T>::N, WAVES = VERIFY_THREADS / 64, FLIGHT = 4;
  __shared__ float sh_m[WAVES], sh_s[WAVES];
  const int r = blockIdx.x / a.parts, part = blockIdx.x % a.parts, targets = (a.K + 1) * a.B;
  const bool is_draft = r >= targets;
  const int row = is_draft ? r - targets : r, i = row / a.B, b = row % a.B, len = draft_length(a, b);
  if (is_draft ? i >= len : i > len) return;  // a row behind the text's drafts
  const T *z = is_draft ? static_cast<const T *>(a.draft) + row * a.ldd : static_cast<const T *>(a.target) + row * a.ldt;
  const int first = part * a.per, last = min(first + a.per, a.V / N);
  const float c = LOG2E / (is_draft ? a.tau_d : a.tau);
  const float zt = part == a.parts - 1 ? tail_elem(z, threadIdx.x, a.V) : -INFINITY;  // the last part has the row's last elements
  float mx = zt, s = zt == -INFINITY ? 0.0f : 1.0f;
  for (int j0 = first + threadIdx.x; j0 < last; j0 += FLIGHT * VERIFY_THREADS) {
    slot_t raw[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      const int j = j0 + k * VERIFY_THREADS;
      raw[k] = j < last ? load_slot(z, j) : empty_slot<T>();
    }
    float top = mx;
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) top = slot_max<T>(top, raw[k]);
    const float base = top == -INFINITY ? 0.0f : top, bias = -base * c;
    if (top > mx) {
      s *= exp2_32(fmaf(mx, c, bias));
      mx = top;
    }
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k)
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_32(fmaf(slot_elem<T>(raw[k], e), c, bias));
  }
  const float own = mx;
  mx = wave_max(mx);
  float base = mx == -INFINITY ? 0.0f : mx;
  s = wave_sum(s * exp2_32(fmaf(own, c, -base * c)));
  if ((threadIdx.x & 63) == 0) {
    sh_m[threadIdx.x >> 6] = mx;
    sh_s[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < WAVES; ++k) mx = fmaxf(mx, sh_m[k]);
    base = mx == -INFINITY ? 0.0f : mx;
    s = 0.0f;
    for (int k = 0; k < WAVES; ++k) s += sh_s[k] * exp2_32(fmaf(sh_m[k], c, -base * c));
    a.stat[(long)r * a.parts + part] = make_float2(mx, s);
  }
}

// Maximum and sum of row r, by one wave.
__device__ inline float2 verify_row(const VerifyArgs &a, long r, float tau) {
  const int lane = threadIdx.x & 63;
  const float c = LOG2E / tau;
  const float2 q = lane < a.parts ? a.stat[r * a.parts + lane] : make_float2(-INFINITY, 0.0f);
  const float m = wave_max(q.x), base = m == -INFINITY ? 0.0f : m;
  return make_float2(m, wave_sum(q.y * exp2_32(fmaf(q.x, c, -base * c))));
}

template <typename T>
__device__ inline const T *verify_target(const VerifyArgs &a, int i, int b) {
  return static_cast<const T *>(a.target) + ((long)i * a.B + b) * a.ldt;
}
template <typename T>
__device__ inline const T *verify_draft(const VerifyArgs &a, int i, int b) {
  return static_cast<const T *>(a.draft) + ((long)i * a.B + b) * a.ldd;
}

// How many drafts of text b are accepted: a wave to each draft.  All threads of the workgroup take part.
template <typename T, int THREADS>
__device__ inline VerifySeq verify_decide(const VerifyArgs &a, int b) {
  __shared__ int sh_n;
  __shared__ float2 sh_max;
  const int len = draft_length(a, b), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == 0) sh_n = len;
  __syncthreads();
  for (int i = wave; i < len; i += THREADS / 64) {
    const long at = (long)i * a.B + b;
    const int d = a.drafts[at];
    bool accept = false;
    if (d < 0 || d >= a.V) {
      if (a.range_flag) *a.range_flag = 1;
    } else {
      const float2 p = verify_row(a, at, a.tau);
      const double zp = (double)to_f32(verify_target<T>(a, i, b)[d]);
      const double pd = exp2_64((zp - (double)p.x) * (LOG2E_64 / (double)a.tau)) / (double)p.y;
      double qd = 1.0;
      if (a.draft) {
        const float2 q = verify_row(a, (long)(a.K + 1) * a.B + at, a.tau_d);
        const double zq = (double)to_f32(verify_draft<T>(a, i, b)[d]);
        qd = exp2_64((zq - (double)q.x) * (LOG2E_64 / (double)a.tau_d)) / (double)q.y;
      }
      accept = (double)a.u[at] * qd < pd;
    }
    if (!accept && (threadIdx.x & 63) == 0) atomicMin(&sh_n, i);
  }
  __syncthreads();
  VerifySeq s;
  s.n = sh_n;
  s.mixed = s.n < len;
  if (wave == 0) {
    const long at = (long)s.n * a.B + b;
    const float mp = verify_row(a, at, a.tau).x;
    const float mq = s.mixed && a.draft ? verify_row(a, (long)(a.K + 1) * a.B + at, a.tau_d).x : -INFINITY;
    if (threadIdx.x == 0) sh_max = make_float2(mp, mq);
  }
  __syncthreads();
  s.mp = sh_max.x;
  s.mq = sh_max.y;
  return s;
}

template <int THREADS>
__device__ inline double block_sum(double v) {
  __shared__ double sh[THREADS / 64];
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) v += sh[i];
  return v;
}

// One part of the drawn row pair: sums of exponentials.
template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_sums_kernel(const VerifyArgs a) {
  constexpr int N = SlotOf<T>::N;
  const int b = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const VerifySeq s = verify_decide<T, VERIFY_THREADS>(a, b);
  if (part == 0 && threadIdx.x == 0) a.seq[b] = s;
  const bool with_q = s.mixed && a.draft;
  const T *p = verify_target<T>(a, s.n, b), *q = with_q ? verify_draft<T>(a, s.n, b) : nullptr;
  const Exp64 ep(s.mp, a.tau), eq(s.mq, a.tau_d);
  const int first = part * a.per, last = min(first + a.per, (a.V + N - 1) / N);
  double sp = 0.0, sq = 0.0;
  for (int j = first + threadIdx.x; j < last; j += VERIFY_THREADS) {
    const slot_t rp = load_any_slot(p, j, a.V), rq = with_q ? load_any_slot(q, j, a.V) : empty_slot<T>();
#pragma unroll
    for (int e = 0; e < N; ++e) sp += ep(slot_elem<T>(rp, e));
    if (with_q)
#pragma unroll
      for (int e = 0; e < N; ++e) sq += eq(slot_elem<T>(rq, e));
  }
  sp = block_sum<VERIFY_THREADS>(sp);
  sq = block_sum<VERIFY_THREADS>(sq);
  if (threadIdx.x == 0) {
    a.sums[((long)b * a.parts + part) * 2] = sp;
    a.sums[((long)b * a.parts + part) * 2 + 1] = sq;
  }
}

// r of the drawn row pair, up to a common factor.
template <typename T>
struct Rest {
  const T *p, *q;
  Exp64 ep, eq;
  double sp, sq;
  int V, drop;  // drop: a word without mass (the rejected draft of a text without draft logits), or -1
  __device__ Rest(const VerifyArgs &a, int b, const VerifySeq &s, const double *sums, bool plain)
      : p(verify_target<T>(a, s.n, b)), q(nullptr), ep(s.mp, a.tau), eq(s.mq, a.tau_d), V(a.V), drop(-1) {
    sp = sq = 0.0;
    for (int i = 0; i < a.parts; ++i) {
      sp += sums[2 * i];
      sq += sums[2 * i + 1];
    }
    sp = 1.0 / sp;
    sq = 1.0 / sq;
    if (!s.mixed || plain) return;
    if (a.draft) q = verify_draft<T>(a, s.n, b);
    else drop = a.drafts[(long)s.n * a.B + b];
  }
  __device__ double one(float zp, float zq, int v) const {
    const double r = ep(zp) * sp;
    if (q) {
      const double d = r - eq(zq) * sq;
      return d < 0.0 ? 0.0 : d;  // (a NaN stays one)
    }
    return v == drop ? 0.0 : r;
  }
  __device__ void slot(int j, double (&r)[SlotOf<T>::N]) const {
    constexpr int N = SlotOf<T>::N;
    const slot_t rp = load_any_slot(p, j, V), rq = q ? load_any_slot(q, j, V) : empty_slot<T>();
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = one(slot_elem<T>(rp, e), slot_elem<T>(rq, e), j * N + e);
  }
};

template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_rest_kernel(const VerifyArgs a) {
  constexpr int N = SlotOf<T>::N;
  const int b = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const VerifySeq s = a.seq[b];
  const Rest<T> rest(a, b, s, a.sums + (long)b * a.parts * 2, false);
  const int first = part * a.per, last = min(first + a.per, (a.V + N - 1) / N);
  double sum = 0.0;
  for (int j = first + threadIdx.x; j < last; j += VERIFY_THREADS) {
    double r[N];
    rest.slot(j, r);
#pragma unroll
    for (int e = 0; e < N; ++e) sum += r[e];
  }
  sum = block_sum<VERIFY_THREADS>(sum);
  if (threadIdx.x == 0) a.rest[(long)b * a.parts + part] = sum;
}

template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_draw_kernel(const VerifyArgs a) {
  constexpr int N = SlotOf<T>::N;
  __shared__ double sh_sum[VERIFY_THREADS];
  __shared__ int sh_word;
  const int b = blockIdx.x, tid = threadIdx.x;
  const VerifySeq s = a.seq[b];
  const double *sums = a.sums + (long)b * a.parts * 2, *rests = a.rest + (long)b * a.parts;
  double total = 0.0;
  for (int i = 0; i < a.parts; ++i) total += rests[i];
  const bool plain = total == 0.0;  // p <= q everywhere: p itself
  const Rest<T> rest(a, b, s, sums, plain);
  auto of_part = [&](int i) { return plain ? sums[2 * i] * rest.sp : rests[i]; };
  if (plain) {
    total = 0.0;
    for (int i = 0; i < a.parts; ++i) total += of_part(i);
  }
  // the first part whose end lies above the number; rounding of the product can leave none: the last one with any mass
  const double goal = (double)a.u[(long)a.K * a.B + b] * total;
  double before = 0.0, sum = 0.0, mass_before = 0.0;
  int part = -1, mass = -1;
  for (int i = 0; i < a.parts; ++i) {
    const double next = of_part(i);
    if (next > 0.0) {
      mass = i;
      mass_before = sum;
    }
    if (sum + next > goal) {
      part = i;
      before = sum;
      break;
    }
    sum += next;
  }
  if (part < 0) {
    part = mass;
    before = mass_before;
  }
  if (tid == 0) sh_word = -1;
  __syncthreads();
  if (part >= 0 && total - total == 0.0) {
    // stretches of neighbouring slots, one for each thread
    const int first = part * a.per, last = min(first + a.per, (a.V + N - 1) / N);
    const int stretch = (last - first + VERIFY_THREADS - 1) / VERIFY_THREADS;
    const int j0 = min(first + tid * stretch, last), j1 = min(j0 + stretch, last);
    double mine = 0.0;
    int final = -1;  // last word with any mass
    for (int j = j0; j < j1; ++j) {
      double r[N];
      rest.slot(j, r);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        mine += r[e];
        if (r[e] > 0.0) final = j * N + e;
      }
    }
    sh_sum[tid] = mine;
    __syncthreads();
    for (int o = 1; o < VERIFY_THREADS; o <<= 1) {
      const double add = tid >= o ? sh_sum[tid - o] : 0.0;
      __syncthreads();
      sh_sum[tid] += add;
      __syncthreads();
    }
    const double upto = before + sh_sum[tid], from = before + (tid ? sh_sum[tid - 1] : 0.0);
    // sums of stretches rise from thread to thread, so one thread at most sees the number pass; where rounding lets none,
    // the part's last word with any mass
    if (from <= goal && upto > goal) {
      double c = from;
      int word = final;
      for (int j = j0; j < j1; ++j) {
        double r[N];
        rest.slot(j, r);
        bool found = false;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          c += r[e];
          if (!found && c > goal) {
            found = true;
            word = j * N + e;
          }
        }
        if (found) break;
      }
      sh_word = word | 1 << 30;
    }
    __syncthreads();
    if (sh_word < 0) {
      __syncthreads();
      if (final >= 0) atomicMax(&sh_word, final);
    }
    __syncthreads();
  }
  const int word = sh_word < 0 ? -1 : sh_word & ~(1 << 30);
  if (tid == 0) a.accepted[b] = s.n;
  for (int i = tid; i <= a.K; i += VERIFY_THREADS) {
    const long at = (long)i * a.B + b;
    a.tokens[at] = i < s.n ? a.drafts[at] : i == s.n ? word : -1;
  }
}

}  // namespace rnnlm_dev
