// Rows of logits whose gradient is that of a given word's log-probability, times a number g that hangs on that log-probability:
//   l = ln q(y),  q = softmax(z / tau),      dz[v] = g ([v = y] - q(v)) / tau
// What the policy loss (policy.h) and the preference loss (preference.h) share: the sum of a row's exponentials, l, and the
// gradient.  Sums are taken relative to a whole power of 2 near the row's greatest logits (rows.h), l in 64 bits from there: a
// ratio of probabilities is compared with its border, and a text's words are added up.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

template <typename T>
struct WordRows {
  const T *z;
  long ldz;
  T *dz;  // may be z (same row length); nullptr: no gradient
  long ldd;
  const int32_t *y;
  int32_t *range_flag;
  float tau;
  int V;
  bool once;  // read past the caches
  // Row m's word, -1: none.
  __device__ int word(long m) const {
    const int w = y[m];
    if (w >= V && range_flag && threadIdx.x == 0) *range_flag = 1;
    return w < V ? w : -1;
  }
};

// A row's sum of exponentials of (z - shift) c, c = log2 e / tau in 32 bits: s 2^power.
struct WordSum {
  float shift, power, s;
  // ln q of a word.  The logarithm goes back to units of a logit by the c that the sum was formed with.
  __device__ double logp(float zy, float tau) const {
    if (s == 0.0f || zy == -INFINITY) return s == s && s != INFINITY ? -INFINITY : NAN;
    const double c = (double)(LOG2E / tau);
    return (((double)zy - (double)shift) - ((double)power + log2((double)s)) / c) / (double)tau;
  }
};

// -g q(v) / tau: exponents stay whole powers away from z c, what is left of the factors is multiplied.
struct WordDense {
  float c, b, a, shift;
  __device__ WordDense(const WordSum &r, float tau, float g) : c(LOG2E / tau), shift(r.shift) {
    a = g == 0.0f || r.s == 0.0f ? 0.0f : -g / __builtin_amdgcn_frexp_mantf(r.s);
    b = -r.power - (float)__builtin_amdgcn_frexp_expf(r.s);
  }
  // SHIFT: rows whose sums have one
  template <bool SHIFT = false>
  __device__ float at(float z) const {
    if (SHIFT) z -= shift;
    return a * exp2_32(fmaf(z, c, b));
  }
};

template <int WAVES>
struct WordShared {
  float m[WAVES], s[WAVES], again[WAVES];
  float g;
};

template <typename T, int THREADS>
__device__ inline void word_no_gradient(T *drow, int V) {
  const float zero[SlotOf<T>::N] = {};
  const int full = V / SlotOf<T>::N, at = full * SlotOf<T>::N + threadIdx.x;
  for (int j = threadIdx.x; j < full; j += THREADS) store_slot(drow, j, zero);
  if (at < V) drow[at] = from_f32<T>(0.0f);
}

// The sum by a pass over memory, at z - maximum with a running maximum and sum of each thread: for logits of any size.
// zt: this thread's element behind the whole slots.
template <typename T, int THREADS, int FLIGHT, bool ONCE>
__device__ inline WordSum word_sum_by_memory(const T *row, float zt, int V, float tau, WordShared<THREADS / 64> &sh) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), full = V / N;
  const float c = LOG2E / tau;
  float mx = zt, s = zt == -INFINITY ? 0.0f : 1.0f;
  if (zt != zt) mx = -INFINITY, s = NAN;
  for (int j0 = tid; j0 < full; j0 += FLIGHT * THREADS) {
    slot_t raw[FLIGHT];
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) {
      const int j = j0 + i * THREADS;
      raw[i] = j < full ? load_slot<T, ONCE>(row, j) : empty_slot<T>();
    }
    float top = mx;
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) top = slot_max<T>(top, raw[i]);
    const float base = top == -INFINITY ? 0.0f : top;
    if (top > mx) {
      s *= exp2_32((mx - base) * c);  // (from -inf: the sum is 0, and so is the factor)
      mx = top;
    }
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_32((slot_elem<T>(raw[i], e) - base) * c);
  }
  const float top = wave_max(mx);
  if ((tid & 63) == 0) sh.m[wave] = top;
  __syncthreads();
  WordSum r = {waves_max<WAVES>(sh.m), 0.0f, 0.0f};
  if (r.shift == -INFINITY) r.shift = 0.0f;
  s *= exp2_32((mx - r.shift) * c);
  s = wave_sum(s);
  if ((tid & 63) == 0) sh.s[wave] = s;
  __syncthreads();
  r.s = waves_sum<WAVES>(sh.s);
  return r;
}

// The gradient by a pass over memory.
template <typename T, int THREADS>
__device__ inline void word_gradient_by_memory(const WordSum &r, const T *row, T *drow, float zt, float zy, int y, int V, float tau, float g) {
  constexpr int N = SlotOf<T>::N;
  const int tid = threadIdx.x, full = V / N;
  const WordDense dense(r, tau, g);
  for (int j = tid; j < full; j += THREADS) {
    const slot_t raw = load_slot(row, j);
    float d[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = dense.template at<true>(slot_elem<T>(raw, e));
    store_slot(drow, j, d);
  }
  if (full * N + tid < V) drow[full * N + tid] = from_f32<T>(dense.template at<true>(zt));
  // the word itself, by the thread that wrote it just now
  if ((y < full * N ? y / N % THREADS : y - full * N) == tid) drow[y] = from_f32<T>(g + dense.template at<true>(zy));
}

// The row in registers, NV slots of a thread, packed as stored.
template <typename T, int THREADS, int NV>
struct WordRow {
  static constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64;
  slot_t raw[NV];
  float zt;

  __device__ void load(const T *row, int V, bool once) {
    const int tid = threadIdx.x, full = V / N;
    if (once) {
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < full ? load_slot<T, true>(row + i * THREADS * N, tid) : empty_slot<T>();
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < full ? load_slot(row + i * THREADS * N, tid) : empty_slot<T>();
    }
    zt = tail_elem(row, tid, V);
  }
  // The sum while the row arrives: a wave's reference is near the greatest element of its first slots, so a later element of it
  // can only make it too large by being e^69 times greater, and the sum cannot vanish.  Where that happens, a sum is no number,
  // or a wave's first slots are masked throughout (or beyond the references' range), the row is read again by way of memory.
  __device__ WordSum sum(const T *row, int V, float tau, WordShared<WAVES> &sh) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), full = V / N;
    const float ref = wave_max(slot_max<T>(zt, raw[0])), c = LOG2E / tau, b = -whole_power(ref, c);
    float s = exp2_32(fmaf(zt, c, b));
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_32(fmaf(slot_elem<T>(raw[i], e), c, b));
    s = wave_sum(s);
    const bool holds = wave == 0 || wave * 64 < full;  // (the first wave: also a row of less than a slot)
    if ((tid & 63) == 0) {
      sh.m[wave] = s == 0.0f ? -INFINITY : -b;
      sh.s[wave] = s;
      sh.again[wave] = !joinable(s) || (holds && !near_power(ref, c)) ? 1.0f : 0.0f;
    }
    __syncthreads();
    if (waves_max<WAVES>(sh.again) != 0.0f) {
      __syncthreads();
      return word_sum_by_memory<T, THREADS, 1, false>(row, zt, V, tau, sh);
    }
    WordSum r = {};
    const float most = waves_max<WAVES>(sh.m);
    r.power = most == -INFINITY ? 0.0f : most;
    const int of = tid & (WAVES - 1);
    r.s = group_reduce<WAVES>(sh.s[of] * exp2_32(sh.m[of] - r.power), [](float x, float y) { return x + y; });
    return r;
  }
  template <bool SHIFT>
  __device__ void gradient_as(const WordSum &r, T *drow, float zy, int y, int V, float tau, float g) {
    const int tid = threadIdx.x, full = V / N;
    const WordDense dense(r, tau, g);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      keep_packed(raw[i]);
      if (i * THREADS + tid < full) {
        float d[N];
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = dense.template at<SHIFT>(slot_elem<T>(raw[i], e));
        store_slot(drow + i * THREADS * N, tid, d);
      }
    }
    if (full * N + tid < V) drow[full * N + tid] = from_f32<T>(dense.template at<SHIFT>(zt));
    // the word itself, by the thread that wrote it just now
    if ((y < full * N ? y / N % THREADS : y - full * N) == tid) drow[y] = from_f32<T>(g + dense.template at<SHIFT>(zy));
  }
  __device__ void gradient(const WordSum &r, T *drow, float zy, int y, int V, float tau, float g) {
    if (r.shift == 0.0f) gradient_as<false>(r, drow, zy, y, V, tau, g);
    else gradient_as<true>(r, drow, zy, y, V, tau, g);
  }
};

}  // namespace rnnlm_dev
