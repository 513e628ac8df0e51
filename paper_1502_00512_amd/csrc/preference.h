// Preference loss of pairs of texts: of streams s < P the text of stream s is preferred to that of stream P + s.
//   S_s = sum_t ln softmax(z)(y) over the positions of stream s that count (or their mean),  r = (S_c - ref_c) - (S_r - ref_r)
//   logistic: -(1 - eps) ln sigma(beta r) - eps ln sigma(-beta r);  squared: (r - 1 / (2 beta))^2;  hinge: max(0, 1 - beta r)
//   dz of a position = scale w L'(r) (+1 preferred, -1 other) (1 / count, if means) ([v = y] - softmax(z)(v))
// Every position's gradient hangs on all rows of its pair.
#pragma once
#include "word_loss.h"

namespace rnnlm_dev {

enum PreferenceKind { PREFER_LOGISTIC, PREFER_SQUARED, PREFER_HINGE };

struct PreferenceRow {  // what is kept of a row between the steps
  double l;
  WordSum sum;
  int y;  // -1: does not count
};
struct PreferencePair {
  double g_chosen, g_other;  // factors of the gradient of a position
};

template <typename T>
struct PreferenceArgs {
  WordRows<T> rows;
  const float *ref, *weight;
  float *loss, *logp;
  int Tn, P, kind;
  bool mean;
  float beta, eps, scale;
  PreferenceRow *row;
  PreferencePair *pair;
  // rows that meet (preference_meet_kernel): their words as they are published, whether the gradient is written, polls of a wait
  unsigned long long *published;
  int *done;
  int polls;
  __device__ int pair_of(long m) const {
    const int s = (int)(m % (2 * P));
    return s < P ? s : s - P;
  }
};

// The words' log-probabilities, a row a workgroup, read once.  Bound by HBM where rows are many (16384 x 64000 bf16 6.3 TB/s), else
// a chain of latencies: 160 x 10000 bf16 4.5 us.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) preference_words_kernel(const PreferenceArgs<T> a) {
  __shared__ WordShared<THREADS / 64> sh;
  const WordRows<T> &w = a.rows;
  const long m = blockIdx.x;
  PreferenceRow out = {0.0, {0.0f, 0.0f, 0.0f}, w.word(m)};
  if (a.weight && a.weight[a.pair_of(m)] == 0.0f) out.y = -1;
  if (out.y >= 0) {
    const T *row = w.z + m * w.ldz;
    const float zt = tail_elem(row, threadIdx.x, w.V), zy = to_f32(row[out.y]);
    out.sum = w.once && !w.dz ? word_sum_by_memory<T, THREADS, 4, true>(row, zt, w.V, 1.0f, sh)
                              : word_sum_by_memory<T, THREADS, 4, false>(row, zt, w.V, 1.0f, sh);
    if (threadIdx.x == 0) out.l = out.sum.logp(zy, 1.0f);
  }
  if (threadIdx.x == 0) a.row[m] = out;
}

// A word's log-probability as another workgroup reads it; two NaNs of their own kind: not published yet, and a position that
// does not count.
constexpr unsigned long long WORD_EMPTY = ~0ull, WORD_NONE = ~1ull;
__device__ inline unsigned long long word_published(double l, int y) {
  return y < 0 ? WORD_NONE : l != l ? 0x7ff8000000000000ull : __builtin_bit_cast(unsigned long long, l);
}

// Sum of the log-probabilities of a text, and number of its words.
struct PreferenceText {
  double l;
  int count;
};
// By one wave, in a fixed order, `waves` of them sharing a text 64 positions at a time.  word(t): as published.
template <class F>
__device__ inline PreferenceText preference_text(int Tn, int wave, int waves, F &&word) {
  PreferenceText s = {0.0, 0};
  for (int t = wave * 64 + (threadIdx.x & 63); t < Tn; t += 64 * waves) {
    const unsigned long long w = word(t);
    if (w != WORD_NONE) {
      s.l += __builtin_bit_cast(double, w);
      ++s.count;
    }
  }
  return {wave_sum(s.l), wave_sum(s.count)};
}

// ln(1 + e^x)
__device__ inline double softplus(double x) { return (x > 0.0 ? x : 0.0) + log1p(exp(-fabs(x))); }

// A pair's factors of the gradient, by one wave, from the sums of its preferred text and of the other one; its loss and its texts'
// log-probabilities, where asked for.
template <typename T>
__device__ inline PreferencePair preference_pair(const PreferenceArgs<T> &a, int p, bool write, const PreferenceText &chosen,
                                                 const PreferenceText &other) {
  const int nc = chosen.count, no = other.count;
  double c = chosen.l, o = other.l;
  const double sc = a.mean ? 1.0 / (nc > 0 ? nc : 1) : 1.0, so = a.mean ? 1.0 / (no > 0 ? no : 1) : 1.0;
  c *= sc;
  o *= so;
  write = write && (threadIdx.x & 63) == 0;
  if (write && a.logp) {
    a.logp[p] = (float)c;
    a.logp[a.P + p] = (float)o;
  }
  const double w = a.weight ? (double)a.weight[p] : 1.0, beta = a.beta, eps = a.eps;
  if (w == 0.0) {
    if (write) a.loss[p] = 0.0f;
    return {0.0, 0.0};
  }
  if (a.ref) {
    c -= (double)a.ref[p];
    o -= (double)a.ref[a.P + p];
  }
  const double r = c - o, x = beta * r;
  double g;
  if (a.kind == PREFER_LOGISTIC) {
    if (write) a.loss[p] = (float)(w * ((1.0 - eps) * softplus(-x) + (eps == 0.0 ? 0.0 : eps * softplus(x))));
    const double e = exp(-fabs(x)), small = e / (1.0 + e), large = 1.0 / (1.0 + e);  // sigma(-|x|), sigma(|x|)
    g = beta * (eps * (x < 0.0 ? small : large) - (1.0 - eps) * (x < 0.0 ? large : small));
  } else if (a.kind == PREFER_SQUARED) {
    const double d = r - 0.5 / beta;
    if (write) a.loss[p] = (float)(w * (d * d));
    g = 2.0 * d;
  } else {
    if (write) a.loss[p] = (float)(w * (x >= 1.0 ? 0.0 : 1.0 - x));
    g = x >= 1.0 ? 0.0 : x < 1.0 ? -beta : x;  // (no number: neither)
  }
  g *= w * (double)a.scale;
  return {g * sc, -g * so};
}
// The same by one wave that adds up the words: word(t, other).
template <typename T, class F>
__device__ inline PreferencePair preference_pair_of(const PreferenceArgs<T> &a, int p, bool write, F &&word) {
  return preference_pair(a, p, write, preference_text(a.Tn, 0, 1, [&](int t) { return word(t, 0); }),
                         preference_text(a.Tn, 0, 1, [&](int t) { return word(t, 1); }));
}
// A word of the first pass.
template <typename T>
__device__ inline unsigned long long preference_word(const PreferenceArgs<T> &a, int p, int t, int other) {
  const PreferenceRow &row = a.row[((long)t * 2 + other) * a.P + p];
  return word_published(row.l, row.y);
}

// Where texts are long, or no gradient is wanted: a workgroup a pair, half of its waves to a text (a wave alone is a chain of
// loads: 1 pair of 512 positions 5.2 us, 4 of 2048 28, 1 of 20000 133; so 2.9, 10 and 18.5).
template <typename T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) preference_pairs_kernel(const PreferenceArgs<T> a) {
  constexpr int HALF = WAVES / 2;
  __shared__ PreferenceText text[WAVES];
  const int wave = threadIdx.x >> 6, other = wave / HALF, p = blockIdx.x;
  const PreferenceText mine = preference_text(a.Tn, wave % HALF, HALF, [&](int t) { return preference_word(a, p, t, other); });
  if ((threadIdx.x & 63) == 0) text[wave] = mine;
  __syncthreads();
  if (wave != 0) return;
  PreferenceText sum[2] = {text[0], text[HALF]};
  for (int i = 1; i < HALF; ++i)
    for (int j = 0; j < 2; ++j) {
      sum[j].l += text[j * HALF + i].l;
      sum[j].count += text[j * HALF + i].count;
    }
  const PreferencePair f = preference_pair(a, p, true, sum[0], sum[1]);
  if (threadIdx.x == 0) a.pair[p] = f;
}

// The gradients, a row a workgroup, the row read again.  INSIDE: each finds its pair's factors itself, from the words of both
// texts (up to PREFERENCE_INSIDE positions: a load or two of each lane), while its row is on the way; so a small call takes two
// launches.  160 x 10000 bf16 5.0 us, 16384 x 64000 760 (5.5 TB/s).
constexpr int PREFERENCE_INSIDE = 128;
template <typename T, int THREADS, int NV, bool INSIDE>
__global__ void __launch_bounds__(THREADS) preference_row_kernel(const PreferenceArgs<T> a) {
  const WordRows<T> &w = a.rows;
  const long m = blockIdx.x;
  const PreferenceRow r = a.row[m];
  T *drow = w.dz + m * w.ldd;
  const T *row = w.z + m * w.ldz;
  const int p = a.pair_of(m), s = (int)(m % (2 * a.P));
  WordRow<T, THREADS, NV> held;
  if (r.y >= 0) held.load(row, w.V, false);
  __shared__ float g;
  if (threadIdx.x < 64) {
    const PreferencePair f = INSIDE ? preference_pair_of(a, p, m == s && s < a.P, [&](int t, int other) { return preference_word(a, p, t, other); }) : a.pair[p];
    if (threadIdx.x == 0) g = (float)(s < a.P ? f.g_chosen : f.g_other);
  }
  __syncthreads();
  if (r.y < 0 || r.l == -INFINITY) return word_no_gradient<T, THREADS>(drow, w.V);
  held.gradient(r.sum, drow, to_f32(row[r.y]), r.y, w.V, 1.0f, g);
}
// Rows that do not fit the registers: 1280 x 300000 bf16, with the words, 458 us.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) preference_stream_kernel(const PreferenceArgs<T> a) {
  const WordRows<T> &w = a.rows;
  const long m = blockIdx.x;
  const PreferenceRow r = a.row[m];
  T *drow = w.dz + m * w.ldd;
  if (r.y < 0 || r.l == -INFINITY) return word_no_gradient<T, THREADS>(drow, w.V);
  const PreferencePair p = a.pair[a.pair_of(m)];
  const T *row = w.z + m * w.ldz;
  const float g = (float)((int)(m % (2 * a.P)) < a.P ? p.g_chosen : p.g_other);
  word_gradient_by_memory<T, THREADS>(r.sum, row, drow, tail_elem(row, threadIdx.x, w.V), to_f32(row[r.y]), r.y, w.V, 1.0f, g);
}

// ---- rows that meet ----
// One pass over the logits where they are many: a workgroup holds its row, publishes its word's log-probability (the word is
// its own flag) and waits for those of its pair, which were started next to it.  A wait ends after `polls` polls, too (the rest
// of a pair may not be on the GPU yet, where other work fills it): such a row leaves its sum to preference_rest_kernel, which
// writes the same gradient.
// 2560 x 64000 bf16 (64 pairs of 20 positions) 138-141 us where a row by itself (policy_row_kernel) takes 115: a pair's rows write
// only when the last of them has been read.  Two passes: 188.
constexpr int PREFERENCE_MEET = 64;  // most positions of a text: the pair's rows are at most half of what the GPU holds

template <typename T>
__global__ void __launch_bounds__(256) preference_clear_kernel(const PreferenceArgs<T> a, long rows) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < rows; i += 256L * gridDim.x) a.published[i] = WORD_EMPTY;
}

template <typename T, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 4) preference_meet_kernel(const PreferenceArgs<T> a) {
  __shared__ WordShared<THREADS / 64> sh;
  __shared__ unsigned long long words[2 * PREFERENCE_MEET];
  __shared__ int met, masked;  // (not in sh: its sums may still be read)
  const WordRows<T> &w = a.rows;
  // workgroups in the order of the pairs
  const int p = blockIdx.x / (2 * a.Tn), k = blockIdx.x % (2 * a.Tn), s = k & 1 ? a.P + p : p;
  const long m = (long)(k >> 1) * 2 * a.P + s;
  int y = w.word(m);
  if (a.weight && a.weight[p] == 0.0f) y = -1;
  const T *row = w.z + m * w.ldz;
  T *drow = w.dz + m * w.ldd;
  WordRow<T, THREADS, NV> held;
  WordSum r = {};
  float zy = 0.0f;
  if (y >= 0) {
    held.load(row, w.V, w.once);
    zy = to_f32(row[y]);
    r = held.sum(row, w.V, 1.0f, sh);
  }
  double l = 0.0;
  if (threadIdx.x == 0) {
    if (y >= 0) l = r.logp(zy, 1.0f);
    __hip_atomic_store(a.published + m, word_published(l, y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    masked = l == -INFINITY;
  }
  if (y < 0) {
    word_no_gradient<T, THREADS>(drow, w.V);
    if (k != 0) {  // (the pair's first row sees to its loss)
      if (threadIdx.x == 0) a.done[m] = 1;
      return;
    }
  }
  for (int i = threadIdx.x; i < 2 * a.Tn; i += THREADS) {
    const unsigned long long *at = a.published + (long)(i >> 1) * 2 * a.P + (i & 1 ? a.P + p : p);
    unsigned long long v = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int n = 0; v == WORD_EMPTY && n < a.polls; ++n) {
      __builtin_amdgcn_s_sleep(4);
      v = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    words[i] = v;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    bool all = true;
    for (int i = threadIdx.x; i < 2 * a.Tn; i += 64) all = all && words[i] != WORD_EMPTY;
    all = __all(all);
    if (all) {
      const PreferencePair f = preference_pair_of(a, p, k == 0, [&](int t, int other) { return words[2 * t + other]; });
      if (threadIdx.x == 0) sh.g = (float)(k & 1 ? f.g_other : f.g_chosen);
    }
    if (threadIdx.x == 0) {
      a.done[m] = all;
      if (!all) a.row[m] = {l, r, y};
      met = all;
    }
  }
  __syncthreads();
  if (!met || y < 0) return;
  if (masked) return word_no_gradient<T, THREADS>(drow, w.V);
  held.gradient(r, drow, zy, y, w.V, 1.0f, sh.g);
}

// Rows whose wait ended early, read again (every word has been published by now): the same sum, the same steps behind it, the same
// bits.  4 us where there are none.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) preference_rest_kernel(const PreferenceArgs<T> a, long rows) {
  __shared__ float g;
  const WordRows<T> &w = a.rows;
  for (long first = blockIdx.x; first < rows; first += (long)gridDim.x * 64) {
    // (each wave looks at the same 64 rows, so that all agree)
    const long mine = first + (long)(threadIdx.x & 63) * gridDim.x;
    unsigned long long open = __ballot(mine < rows && !a.done[mine < rows ? mine : 0]);
    while (open) {
      const long m = first + (long)(__ffsll(open) - 1) * gridDim.x;
      open &= open - 1;
      const int s = (int)(m % (2 * a.P)), p = s < a.P ? s : s - a.P;
      const PreferenceRow r = a.row[m];
      if (threadIdx.x < 64) {
        const PreferencePair f = preference_pair_of(a, p, m == s && s < a.P, [&](int t, int other) { return a.published[((long)t * 2 + other) * a.P + p]; });
        if (threadIdx.x == 0) g = (float)(s < a.P ? f.g_chosen : f.g_other);
      }
      __syncthreads();
      T *drow = w.dz + m * w.ldd;
      const T *row = w.z + m * w.ldz;
      if (r.y < 0 || r.l == -INFINITY) word_no_gradient<T, THREADS>(drow, w.V);
      else word_gradient_by_memory<T, THREADS>(r.sum, row, drow, tail_elem(row, threadIdx.x, w.V), to_f32(row[r.y]), r.y, w.V, 1.0f, g);
      __syncthreads();
    }
  }
}

}  // namespace rnnlm_dev
