// Distillation from a teacher's list of logits: loss and gradient of a student's rows of logits.
//   t_k = val_k / tau,  p_k = exp(t_k - n),  n = the teacher's ln sum_v exp(t_v) as given, or ln sum_k exp(t_k);  pi = sum_k p_k
//   loss  = w (alpha tau^2 sum_k p_k (ln p_k - ln q_tau(id_k)) - (1 - alpha) ln q_1(y)),   q_tau = softmax(z / tau)
//   dz[v] = w g (alpha tau (pi q_tau(v) - sum_{k: id_k = v} p_k) + (1 - alpha) (q_1(v) - [v = y]))
// The sum over the list is pi (A / (tau S) + lse_tau - n) with S = sum_k e^{t_k - t_max}, A = sum_k e^{t_k - t_max} (val_k - z_k): a
// pass over the row needs a sum of exponentials only, and the listed words are read one by one.  (Logits are taken as distances, the
// list's from its greatest one, the row's from its pivot, lse_tau and n as well: what is added up is no larger than the spread.)
// A sum is taken relative to a reference; any will do that leaves it finite and far from 0.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

template <typename T>
struct DistillArgs {
  const T *z;
  long ldz;
  T *dz;  // may be z (same row length); nullptr: loss only
  long ldd;
  const int32_t *ids, *y;
  const float *vals, *lse, *weight;
  float *loss;
  int32_t *range_flag;
  float tau, alpha, scale;
  int V, K;
  bool once;  // read past the caches
  double inv_tau;
};

// Exponentials of an element.  ONE: a single temperature (tau = 1, or no labels).  SQUARE: tau = 2 and labels, whose
// exponential at 1 is the square of the one at 2 (a multiplication in place of 5 instructions' time; tau = 2 is the usual
// temperature).  TWO: any other tau, and labels.
enum DistillMode { DISTILL_ONE, DISTILL_SQUARE, DISTILL_TWO };

struct DistillEntry {  // a word of the list, or (last) the label
  int id;              // -1: absent
  float val, z, p;     // teacher's logit, student's logit, e^{t - t_max}
};

// The list in LDS: K entries and the label, behind them the entries' ids by themselves (four to a read, four reads
// at once), padded with -2.
__host__ __device__ inline int distill_ids(int K) { return (K + 15) / 16 * 16; }
__host__ __device__ inline size_t distill_lds(int K) { return (size_t)(K + 1) * sizeof(DistillEntry) + (size_t)distill_ids(K) * 4; }

// What a row's softmax is made of: sums of exponentials of z - shift at tau and at 1, relative to 2^power and 2^power1.
struct RowSums {
  float shift, power, power1, s, s1;
  // The logit that the sum at tau is relative to, as far as 32 bits go.
  __device__ float pivot(float tau) const { return shift + power * (tau / LOG2E); }
};

// Exponentials of a row that are relative to whole powers of 2 (shift = 0).
template <int MODE>
struct DistillExp {
  float c, b, b1;
  __device__ DistillExp(float m, float tau) : c(LOG2E / tau), b(-whole_power(m, c)), b1(-whole_power(m, LOG2E)) {}
  __device__ void add(float z, float &s, float &s1) const {
    const float e = exp2_32(fmaf(z, c, b));
    s += e;
    if (MODE == DISTILL_SQUARE) s1 = fmaf(e, e, s1);
    if (MODE == DISTILL_TWO) s1 += exp2_32(fmaf(z, LOG2E, b1));
  }
  __device__ float power1() const { return MODE == DISTILL_SQUARE ? -2.0f * b : -b1; }
};

// The dense part of a row's gradient: pi g alpha tau q_tau(v) + g (1 - alpha) q_1(v).  Exponents stay whole powers away from z c
// (the sum's own whole power is taken off, too: sums may be as large as fp32 goes), and what is left of the factors is multiplied:
// with the factors' logarithms in the exponent, -power + log2(a / s) was rounded at the power's size and a row's gradient off
// by 2e-4 at logits of 10^4.  (Multiplied and in the exponent: 2560 rows of 64000 bf16 words 120.6 us and 120.3; of 10000, which
// the memory-side cache holds, 21.9 and 21.2.)
template <int MODE>
struct DistillDense {
  float c, b, a, b1, a1, shift;
  __device__ DistillDense(const RowSums &r, float tau, float soft, float hard) : c(LOG2E / tau), shift(r.shift) {
    term(MODE == DISTILL_ONE ? soft + hard : soft, r.power, r.s, a, b);
    if (MODE == DISTILL_SQUARE) {  // d = e (a + a1 e), the sum of squares in the same units
      b1 = 0.0f;
      a1 = r.s1 == 0.0f ? 0.0f : hard / ldexpf(r.s1, 2 * (int)(b + r.power));
    } else {
      term(hard, r.power1, r.s1, a1, b1);
    }
  }
  // factor / s = a 2^(b + power)
  __device__ static void term(float factor, float power, float s, float &a, float &b) {
    a = s == 0.0f ? 0.0f : factor / __builtin_amdgcn_frexp_mantf(s);
    b = -power - (float)__builtin_amdgcn_frexp_expf(s);
  }
  // SHIFT: rows whose sums have one
  template <bool SHIFT = false>
  __device__ float at(float z) const {
    if (SHIFT) z -= shift;
    const float e = exp2_32(fmaf(z, c, b));
    if (MODE == DISTILL_SQUARE) return e * fmaf(a1, e, a);
    return MODE == DISTILL_TWO ? fmaf(a1, exp2_32(fmaf(z, LOG2E, b1)), a * e) : a * e;
  }
};

// Reads the list of row m: this thread's entries e = tid, tid + THREADS, ...  Returns the greatest logit among them.
template <typename T, int THREADS>
__device__ inline float distill_entries(const DistillArgs<T> &a, long m, const T *row, DistillEntry *ent) {
  float most = -INFINITY;
  const bool label = a.y && a.alpha < 1.0f;
  int *ids = reinterpret_cast<int *>(ent + a.K + 1);
  for (int e = a.K + threadIdx.x; e < distill_ids(a.K); e += THREADS) ids[e] = -2;
  for (int e = threadIdx.x; e <= a.K; e += THREADS) {
    DistillEntry d;
    d.val = -INFINITY;
    d.z = d.p = 0.0f;
    if (e < a.K) {
      d.id = a.ids[m * a.K + e];
      d.val = a.vals[m * a.K + e];
    } else {
      d.id = label ? a.y[m] : -1;
    }
    if (d.id >= a.V && a.range_flag) *a.range_flag = 1;
    if (d.id < 0 || d.id >= a.V) {
      d.id = -1;
      d.val = -INFINITY;
    } else {
      d.z = to_f32(row[d.id]);
      if (e < a.K) most = fmaxf(most, d.val);
    }
    ent[e] = d;
    if (e < a.K) ids[e] = d.id;
  }
  return most;
}

// The list's sums S and A over this thread's entries.  (Differences of logits first: neither a list's probabilities nor A hang on how
// far from zero list and row lie.  A in 64 bits: masked words may be on the list, at the type's lowest value.)
template <int THREADS>
__device__ inline void distill_list_sums(DistillEntry *ent, int K, float c, float most, float pivot, float &S, double &A) {
  for (int e = threadIdx.x; e < K; e += THREADS) {
    const DistillEntry d = ent[e];
    if (d.val == -INFINITY) continue;  // absent, or a probability of zero: no term
    const float p = exp2_32((d.val - most) * c);
    ent[e].p = p;
    if (p == 0.0f) continue;
    S += p;
    A += (double)p * (((double)d.val - (double)most) - ((double)d.z - (double)pivot));
  }
}

// Sums over the workgroup's waves, by way of LDS.
template <int WAVES>
struct DistillShared {
  float m[WAVES], m1[WAVES], t[WAVES], s[WAVES], s1[WAVES], S[WAVES], again[WAVES];
  double A[WAVES];
};

struct DistillList {
  float most, S, factor, pi;  // greatest logit; p_k = factor e^{t_k - t_max}
};

// The list's sums (the barrier in between also publishes the waves' sums of the row): all threads take part.
template <typename T, int THREADS>
__device__ inline DistillList distill_list(const DistillArgs<T> &a, long m, float pivot, DistillEntry *ent,
                                           DistillShared<THREADS / 64> &sh) {
  constexpr int WAVES = THREADS / 64;
  DistillList l;
  l.most = waves_max<WAVES>(sh.t);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float S = 0.0f;
  double A = 0.0;
  if (wave * 64 < a.K) {
    distill_list_sums<THREADS>(ent, a.K, LOG2E / a.tau, l.most, pivot, S, A);
    S = wave_sum(S);
    A = wave_sum(A);
  }
  if ((threadIdx.x & 63) == 0) {
    sh.S[wave] = S;
    sh.A[wave] = A;
  }
  __syncthreads();
  l.S = waves_sum<WAVES>(sh.S);
  // (a NaN in the list stays one)
  l.factor = l.S == 0.0f ? 0.0f : a.lse ? exp2_32((float)(((double)l.most * a.inv_tau - (double)a.lse[m]) * LOG2E_64)) : 1.0f / l.S;
  l.pi = l.S == 0.0f ? 0.0f : a.lse ? l.factor * l.S : l.S / l.S;
  return l;
}

// The row's loss, by one thread, in 64 bits.  Logarithms go back to units of a logit by the factor their sums were formed with
// (c in 32 bits is not log2 e / tau), and are distances from the row's pivot and the list's greatest logit, as A is.
template <typename T, int MODE>
__device__ inline void distill_loss(const DistillArgs<T> &a, long m, float w, const RowSums &r, const DistillList &l,
                                    const DistillEntry &label, const double *A_of_wave, int waves) {
  const bool hard = label.id >= 0;
  double loss = 0.0;
  if (r.s == 0.0f) {  // no word left
    if ((a.alpha > 0.0f && l.pi != 0.0f) || hard) loss = INFINITY;
  } else {
    const double tau = a.tau;
    if (a.alpha > 0.0f && l.pi != 0.0f) {
      double A = 0.0;
      for (int i = 0; i < waves; ++i) A += A_of_wave[i];
      const double c = (double)(LOG2E / a.tau);
      const double ln_sum = ((double)r.shift + (double)r.power / c - (double)r.pivot(a.tau)) + log2((double)r.s) / c;  // times tau
      const double n = a.lse ? (double)a.lse[m] - (double)l.most / tau : log((double)l.S);
      loss = (double)a.alpha * tau * tau * (double)l.pi * ((A / (double)l.S + ln_sum) / tau - n);
    }
    if (hard) {
      const double sum = MODE == DISTILL_ONE ? (double)r.power + log2((double)r.s) : (double)r.power1 + log2((double)r.s1);
      loss += (double)(1.0f - a.alpha) * ((double)r.shift - (double)label.z + sum / (double)LOG2E);
    }
  }
  a.loss[m] = (float)((double)w * loss);
}

// The listed words' gradients, behind the dense pass: each word is written once, with everything that the list and the label
// take off it.  Every entry looks for its like among all ids; only a word that is listed twice has its probabilities added up.
template <typename T, int THREADS, int MODE>
__device__ inline void distill_listed(const DistillArgs<T> &a, const DistillDense<MODE> &dense, float coef, float hard,
                                      const DistillEntry *ent, T *drow) {
  const int4 *ids = reinterpret_cast<const int4 *>(ent + a.K + 1);
  const int label = ent[a.K].id;
  for (int e = threadIdx.x; e <= a.K; e += THREADS) {
    const DistillEntry d = ent[e];
    if (d.id < 0) continue;
    int alike = 0;
    for (int j = 0; j < distill_ids(a.K) / 4; j += 4) {
      int4 q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = ids[j + i];
#pragma unroll
      for (int i = 0; i < 4; ++i) alike += (q[i].x == d.id) + (q[i].y == d.id) + (q[i].z == d.id) + (q[i].w == d.id);
    }
    float p = d.p;
    if (e == a.K) {
      if (alike) continue;  // the entry takes it off
      p = 0.0f;
    } else if (alike > 1) {
      p = 0.0f;
      int first = a.K;
#pragma unroll 8
      for (int j = a.K - 1; j >= 0; --j) {
        const DistillEntry x = ent[j];
        p += x.id == d.id ? x.p : 0.0f;
        first = x.id == d.id ? j : first;
      }
      if (first < e) continue;
    }
    drow[d.id] = from_f32<T>(dense.template at<true>(d.z) - (coef * p + (d.id == label ? hard : 0.0f)));
  }
}

template <typename T, int THREADS>
__device__ inline void distill_without_weight(const DistillArgs<T> &a, long m) {
  if (threadIdx.x == 0) a.loss[m] = 0.0f;
  if (!a.dz) return;
  T *drow = a.dz + m * a.ldd;
  const float zero[SlotOf<T>::N] = {};
  const int full = a.V / SlotOf<T>::N, at = full * SlotOf<T>::N + threadIdx.x;
  for (int j = threadIdx.x; j < full; j += THREADS) store_slot(drow, j, zero);
  if (at < a.V) drow[at] = from_f32<T>(0.0f);
}

// A row by two passes over memory: sums with a running maximum and sum of each thread (all at z - maximum: for logits of any
// size), then the gradient.  zt: this thread's element behind the whole slots; te: the greatest logit of its list entries.
template <typename T, int THREADS, int MODE, int FLIGHT, bool ONCE>
__device__ inline void distill_by_memory(const DistillArgs<T> &a, long m, float w, const T *row, float zt, float te, DistillEntry *ent,
                                         DistillShared<THREADS / 64> &sh) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, full = a.V / N;
  const float c = LOG2E / a.tau;
  float mx = zt, s = zt == -INFINITY ? 0.0f : 1.0f, s1 = s;
  auto move = [&](float to) {  // (from -inf: the sums are 0, and so is the factor)
    const float e = exp2_32((mx - to) * c);
    s *= e;
    if (MODE == DISTILL_SQUARE) s1 *= e * e;
    if (MODE == DISTILL_TWO) s1 *= exp2_32((mx - to) * LOG2E);
  };
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
      move(base);
      mx = top;
    }
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float z = slot_elem<T>(raw[i], e) - base, x = exp2_32(z * c);
        s += x;
        if (MODE == DISTILL_SQUARE) s1 = fmaf(x, x, s1);
        if (MODE == DISTILL_TWO) s1 += exp2_32(z * LOG2E);
      }
  }
  const float top = wave_max(mx);
  if (lane == 0) {
    sh.m[wave] = top;
    sh.t[wave] = te;
  }
  __syncthreads();
  RowSums r = {waves_max<WAVES>(sh.m), 0.0f, 0.0f, 0.0f, 0.0f};
  if (r.shift == -INFINITY) r.shift = 0.0f;
  move(r.shift);
  s = wave_sum(s);
  if (MODE != DISTILL_ONE) s1 = wave_sum(s1);
  if (lane == 0) {
    sh.s[wave] = s;
    sh.s1[wave] = s1;
  }
  const DistillList l = distill_list<T, THREADS>(a, m, r.pivot(a.tau), ent, sh);  // (a barrier)
  r.s = waves_sum<WAVES>(sh.s);
  if (MODE != DISTILL_ONE) r.s1 = waves_sum<WAVES>(sh.s1);
  if (tid == 0) distill_loss<T, MODE>(a, m, w, r, l, ent[a.K], sh.A, WAVES);
  if (!a.dz) return;
  const float coef = w * a.scale * a.alpha * a.tau, hard = ent[a.K].id >= 0 ? w * a.scale * (1.0f - a.alpha) : 0.0f;
  const DistillDense<MODE> dense(r, a.tau, coef * l.pi, hard);
  T *drow = a.dz + m * a.ldd;
  for (int j = tid; j < full; j += THREADS) {
    const slot_t raw = load_slot(row, j);
    float d[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = dense.template at<true>(slot_elem<T>(raw, e));
    store_slot(drow, j, d);
  }
  if (full * N + tid < a.V) drow[full * N + tid] = from_f32<T>(dense.template at<true>(zt));
  __syncthreads();
  distill_listed<T, THREADS, MODE>(a, dense, coef * l.factor, hard, ent, drow);
}

// A workgroup's row stays in registers between the sums and the gradient: the row is read once and its gradient written once,
// which is all that bounds the call (HBM, with the exponentials' instructions not far behind).  NV: slots of a thread.
// bf16, alpha = 0.5: 2560 rows of 64000 words (K = 64, tau = 1) 119 us (5.5 TB/s; a copy of 512 MiB reaches 5.4), 8192 of 100000
// (K = 100, tau = 2) 700 us (4.7; a copy of 2 GiB 4.9).  2560 of 10000 (K = 32, alpha = 1) 20.4 us (5.0).  fp32, 900 of 33278
// (K = 37, tau = 1.5) 46.7 us (5.1).
// The sums run while the row arrives: a wave's reference is near the greatest element of its first slots, so a later element of
// it can only make it too large by being e^69 times greater, and the sum cannot vanish.  Where that happens, a sum is no number, or a
// wave's first slots are masked throughout (or beyond the references' range), the row goes by way of memory.
template <typename T, int THREADS, int NV, int MODE>
__global__ void __launch_bounds__(THREADS, 4) distill_row_kernel(const DistillArgs<T> a) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64;
  extern __shared__ __align__(16) unsigned char lds[];
  DistillEntry *ent = reinterpret_cast<DistillEntry *>(lds);
  __shared__ DistillShared<WAVES> sh;
  const long m = blockIdx.x;
  const float w = a.weight ? a.weight[m] : 1.0f;
  if (w == 0.0f) return distill_without_weight<T, THREADS>(a, m);
  const T *row = a.z + m * a.ldz;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, full = a.V / N;
  slot_t raw[NV];
  if (a.once) {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < full ? load_slot<T, true>(row + i * THREADS * N, tid) : empty_slot<T>();
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < full ? load_slot(row + i * THREADS * N, tid) : empty_slot<T>();
  }
  const float zt = tail_elem(row, tid, a.V);
  const float te = wave_max(distill_entries<T, THREADS>(a, m, row, ent));
  const float ref = wave_max(slot_max<T>(zt, raw[0]));
  const DistillExp<MODE> ex(ref, a.tau);
  float s = 0.0f, s1 = 0.0f;
  ex.add(zt, s, s1);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) ex.add(slot_elem<T>(raw[i], e), s, s1);
  s = wave_sum(s);
  if (MODE != DISTILL_ONE) s1 = wave_sum(s1);
  const float sum = s + s1;
  const bool holds = wave == 0 || wave * 64 < full;  // (the first wave: also a row of less than a slot)
  const bool again = !joinable(sum) || (holds && !(near_power(ref, ex.c) && near_power(ref, LOG2E)));
  if (lane == 0) {
    sh.m[wave] = s == 0.0f ? -INFINITY : -ex.b;
    sh.m1[wave] = s1 == 0.0f ? -INFINITY : ex.power1();
    sh.s[wave] = s;
    sh.s1[wave] = s1;
    sh.t[wave] = te;
    sh.again[wave] = again ? 1.0f : 0.0f;
  }
  __syncthreads();
  if (waves_max<WAVES>(sh.again) != 0.0f) {
    __syncthreads();
    return distill_by_memory<T, THREADS, MODE, 1, false>(a, m, w, row, zt, te, ent, sh);
  }
  RowSums r = {};
  const float most = waves_max<WAVES>(sh.m);
  r.power = most == -INFINITY ? 0.0f : most;
  const DistillList l = distill_list<T, THREADS>(a, m, r.pivot(a.tau), ent, sh);
  const int of = tid & (WAVES - 1);
  auto join = [&](const float *power, const float *of_wave, float top) {
    return group_reduce<WAVES>(of_wave[of] * exp2_32(power[of] - top), [](float x, float y) { return x + y; });
  };
  r.s = join(sh.m, sh.s, r.power);
  if (MODE != DISTILL_ONE) {
    const float most1 = waves_max<WAVES>(sh.m1);
    r.power1 = most1 == -INFINITY ? 0.0f : most1;
    r.s1 = join(sh.m1, sh.s1, r.power1);
  }
  const float coef = w * a.scale * a.alpha * a.tau, hard = ent[a.K].id >= 0 ? w * a.scale * (1.0f - a.alpha) : 0.0f;
  const DistillDense<MODE> dense(r, a.tau, coef * l.pi, hard);
  T *drow = a.dz + m * a.ldd;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    keep_packed(raw[i]);
    if (i * THREADS + tid < full) {
      float d[N];
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = dense.at(slot_elem<T>(raw[i], e));
      store_slot(drow + i * THREADS * N, tid, d);
    }
  }
  if (full * N + tid < a.V) drow[full * N + tid] = from_f32<T>(dense.template at<true>(zt));
  if (tid == 0) distill_loss<T, MODE>(a, m, w, r, l, ent[a.K], sh.A, WAVES);
  __syncthreads();  // the dense pass first, then the listed words on top of it
  distill_listed<T, THREADS, MODE>(a, dense, coef * l.factor, hard, ent, drow);
}

// Rows that do not fit the registers, and calls without a gradient (1280 bf16 rows of 64000 words, K = 64, 28.9 us, 5.7 TB/s).
template <typename T, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS) distill_stream_kernel(const DistillArgs<T> a) {
  extern __shared__ __align__(16) unsigned char lds[];
  DistillEntry *ent = reinterpret_cast<DistillEntry *>(lds);
  __shared__ DistillShared<THREADS / 64> sh;
  const long m = blockIdx.x;
  const float w = a.weight ? a.weight[m] : 1.0f;
  if (w == 0.0f) return distill_without_weight<T, THREADS>(a, m);
  const T *row = a.z + m * a.ldz;
  const float te = wave_max(distill_entries<T, THREADS>(a, m, row, ent)), zt = tail_elem(row, threadIdx.x, a.V);
  if (a.once && !a.dz) distill_by_memory<T, THREADS, MODE, 4, true>(a, m, w, row, zt, te, ent, sh);
  else distill_by_memory<T, THREADS, MODE, 4, false>(a, m, w, row, zt, te, ent, sh);
}

// Sum of n losses in 64 bits, in a fixed order, by one workgroup.
__global__ void __launch_bounds__(1024) sum_losses_kernel(const float *__restrict__ loss, long n, double *__restrict__ out) {
  __shared__ double sh[16];
  double a = 0.0;
  for (long i = threadIdx.x; i < n; i += 1024) a += (double)loss[i];
  a = wave_sum(a);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) a += sh[i];
    *out = a;
  }
}

}  // namespace rnnlm_dev
