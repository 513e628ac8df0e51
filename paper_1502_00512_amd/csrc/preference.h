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
  __device__ int pair_of(long m) const {
    const int s = (int)(m % (2 * P));
    return s < P ? s : s - P;
  }
};

// The words' log-probabilities, a row a workgroup.
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

// Sum of the log-probabilities of stream s and number of its words: one wave, in a fixed order.
template <typename T>
__device__ inline double preference_text(const PreferenceArgs<T> &a, int s, int &count) {
  double l = 0.0;
  count = 0;
  for (int t = threadIdx.x & 63; t < a.Tn; t += 64) {
    const PreferenceRow &row = a.row[(long)t * 2 * a.P + s];
    if (row.y >= 0) {
      l += row.l;
      ++count;
    }
  }
  count = wave_sum(count);
  return wave_sum(l);
}

// ln(1 + e^x)
__device__ inline double softplus(double x) { return (x > 0.0 ? x : 0.0) + log1p(exp(-fabs(x))); }

// A pair's factors of the gradient, by one wave; its loss and its texts' log-probabilities, where asked for.
template <typename T>
__device__ inline PreferencePair preference_pair(const PreferenceArgs<T> &a, int p, bool write) {
  int nc, no;
  double c = preference_text(a, p, nc), o = preference_text(a, a.P + p, no);
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
    g = x >= 1.0 ? 0.0 : -beta;
  }
  g *= w * (double)a.scale;
  return {g * sc, -g * so};
}

// Where texts are long, or no gradient is wanted: a wave a pair.
template <typename T>
__global__ void __launch_bounds__(64) preference_pairs_kernel(const PreferenceArgs<T> a) {
  const PreferencePair p = preference_pair(a, blockIdx.x, true);
  if (threadIdx.x == 0) a.pair[blockIdx.x] = p;
}

// The gradients, a row a workgroup, the row read again.  INSIDE: each finds its pair's factors itself, from the words of both
// texts (up to PREFERENCE_INSIDE positions: a load or two of each lane), while its row is on the way.
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
    const PreferencePair f = INSIDE ? preference_pair(a, p, m == s && s < a.P) : a.pair[p];
    if (threadIdx.x == 0) g = (float)(s < a.P ? f.g_chosen : f.g_other);
  }
  __syncthreads();
  if (r.y < 0 || r.l == -INFINITY) return word_no_gradient<T, THREADS>(drow, w.V);
  held.gradient(r.sum, drow, to_f32(row[r.y]), r.y, w.V, 1.0f, g);
}
// Rows that do not fit the registers.
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

}  // namespace rnnlm_dev
