// Distillation from a teacher's list of logits: loss and gradient of a student's rows of logits.
//   t_k = val_k / tau,  p_k = exp(t_k - n),  n = the teacher's ln sum_v exp(t_v) as given, or ln sum_k exp(t_k);  pi = sum_k p_k
//   loss  = w (alpha tau^2 sum_k p_k (ln p_k - ln q_tau(id_k)) - (1 - alpha) ln q_1(y)),   q_tau = softmax(z / tau)
//   dz[v] = w g (alpha tau (pi q_tau(v) - sum_{k: id_k = v} p_k) + (1 - alpha) (q_1(v) - [v = y]))
// The sum over the list is pi (A / S + lse_tau - n) with S = sum_k e^{t_k - t_max}, A = sum_k e^{t_k - t_max} (t_k - z_k / tau):
// a pass over the row needs the maximum and the sum of exponentials only, and the listed words are read one by one.
// The list's sums are formed in 64 bits (a few hundred terms a row): the loss is a difference of numbers ten times its size.
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
};

struct DistillEntry {  // a word of the list, or (last) the label
  int id;              // -1: absent
  float t, z, coef;    // teacher's logit / tau, student's logit, what the word's gradient has taken off
};

// What a row's softmax is made of: maximum, and the sums of exponentials relative to it at tau and at 1.
struct RowSums {
  float m, s, s1;
};

// Reads the list of row m: this thread's entries e = tid, tid + THREADS, ...  Returns the greatest t among them.
template <typename T, int THREADS>
__device__ inline float distill_entries(const DistillArgs<T> &a, long m, const T *row, bool label, DistillEntry *ent) {
  float tmax = -INFINITY;
  const float inv_tau = 1.0f / a.tau;
  for (int e = threadIdx.x; e <= a.K; e += THREADS) {
    DistillEntry d;
    d.t = -INFINITY;
    d.z = d.coef = 0.0f;
    if (e < a.K) {
      d.id = a.ids[m * a.K + e];
      d.t = a.vals[m * a.K + e] * inv_tau;
    } else {
      d.id = label ? a.y[m] : -1;
    }
    if (d.id >= a.V && a.range_flag) *a.range_flag = 1;
    if (d.id < 0 || d.id >= a.V) {
      d.id = -1;
      d.t = -INFINITY;
    } else {
      d.z = to_f32(row[d.id]);
      if (e < a.K) tmax = fmaxf(tmax, d.t);
    }
    ent[e] = d;
  }
  return tmax;
}

// The list's sums S and A of this thread's entries.
template <int THREADS>
__device__ inline void distill_list_sums(const DistillEntry *ent, int K, float inv_tau, float tmax, double &S, double &A) {
  S = A = 0.0;
  for (int e = threadIdx.x; e < K; e += THREADS) {
    const DistillEntry d = ent[e];
    if (d.t == -INFINITY) continue;  // absent, or a probability of zero: no term
    const double p = exp((double)d.t - (double)tmax);
    if (p == 0.0) continue;
    S += p;
    A += p * ((double)d.t - (double)d.z * (double)inv_tau);
  }
}

// What the gradient of a row is made of: dz = a exp2(z c + b) + a1 exp2(z log2 e + b1) - coefficients of the listed words.
struct DistillRow {
  float c, b, a, b1, a1, hard;
  __device__ float dense(float z, bool two) const {
    const float d = a * exp2_32(fmaf(z, c, b));
    return two ? fmaf(a1, exp2_32(fmaf(z, LOG2E, b1)), d) : d;
  }
};

// Loss of the row (thread 0 writes it), the coefficients of the listed words, and the dense part's constants.
template <typename T, int THREADS, bool TWO>
__device__ inline DistillRow distill_finish(const DistillArgs<T> &a, long m, float w, RowSums r, float tmax, double S, double A,
                                            DistillEntry *ent) {
  const float inv_tau = 1.0f / a.tau, g = w * a.scale;
  const bool label = ent[a.K].id >= 0;
  const double n = a.lse ? (double)a.lse[m] : (double)tmax + log(S);
  const double pi = S == 0.0 ? 0.0 : a.lse ? exp((double)tmax - n) * S : S / S;  // (a NaN in the list stays one)
  const float s1 = TWO ? r.s1 : r.s;
  DistillRow o;
  const float base = r.m == -INFINITY ? 0.0f : r.m;  // no finite logit: every exponential below is 0
  o.c = LOG2E * inv_tau;
  o.b = -base * o.c;
  o.b1 = -base * LOG2E;
  o.hard = label ? g * (1.0f - a.alpha) : 0.0f;
  const float soft = (float)((double)(g * a.alpha * a.tau) * pi);
  o.a = r.s == 0.0f ? 0.0f : soft / r.s;
  o.a1 = s1 == 0.0f ? 0.0f : o.hard / s1;
  if (!TWO) o.a += o.a1;  // tau = 1, or no label anywhere
  for (int e = threadIdx.x; e <= a.K; e += THREADS) {
    const DistillEntry d = ent[e];
    float coef = 0.0f;
    if (e == a.K) coef = o.hard;
    else if (d.t != -INFINITY) coef = (float)((double)(g * a.alpha * a.tau) * exp((double)d.t - n));
    ent[e].coef = coef;
  }
  if (threadIdx.x == 0) {
    double loss = 0.0;
    if (r.s == 0.0f) {
      if ((a.alpha > 0.0f && pi != 0.0) || (label && a.alpha < 1.0f)) loss = INFINITY;
    } else {
      const double top = (double)r.m * (double)inv_tau;
      if (a.alpha > 0.0f && pi != 0.0) loss = (double)(a.alpha * a.tau) * (double)a.tau * pi * (A / S + top + log((double)r.s) - n);
      if (label && a.alpha < 1.0f)
        loss += (double)(1.0f - a.alpha) * ((double)r.m - (double)ent[a.K].z + log((double)s1));
    }
    a.loss[m] = (float)((double)w * loss);
  }
  return o;
}

// The listed words' gradients, behind the dense pass: each word is written once, with everything that the list takes off it.
template <typename T, int THREADS, bool TWO>
__device__ inline void distill_listed(const DistillArgs<T> &a, const DistillRow &o, const DistillEntry *ent, T *drow) {
  for (int e = threadIdx.x; e <= a.K; e += THREADS) {
    const int id = ent[e].id;
    if (id < 0) continue;
    float off = 0.0f;
    bool first = true;
    for (int j = 0; j <= a.K; ++j)
      if (ent[j].id == id) {
        off += ent[j].coef;
        first = first && j >= e;
      }
    if (first) drow[id] = from_f32<T>(o.dense(ent[e].z, TWO) - off);
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

// A workgroup's row stays in registers between the sums and the gradient: the row is read once and its gradient written once,
// which is all that bounds the call (HBM).  NV: slots of a thread.  TWO: tau != 1 and labels (two exponentials an element).
template <typename T, int THREADS, int NV, bool TWO>
__global__ void __launch_bounds__(THREADS, 4) distill_row_kernel(const DistillArgs<T> a) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64;
  extern __shared__ __align__(16) unsigned char lds[];
  DistillEntry *ent = reinterpret_cast<DistillEntry *>(lds);
  __shared__ float sh_m[WAVES], sh_t[WAVES], sh_s[WAVES], sh_s1[WAVES];
  __shared__ double sh_S[WAVES], sh_A[WAVES];
  const long m = blockIdx.x;
  const float w = a.weight ? a.weight[m] : 1.0f;
  if (w == 0.0f) return distill_without_weight<T, THREADS>(a, m);
  const T *row = a.z + m * a.ldz;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, full = a.V / N;
  slot_t raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = i * THREADS + tid;
    raw[i] = j < full ? load_slot(row, j) : empty_slot<T>();
  }
  const float zt = tail_elem(row, tid, a.V);
  const float te = distill_entries<T, THREADS>(a, m, row, a.y && a.alpha < 1.0f, ent);
  float mx = zt;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    mx = slot_max<T>(mx, raw[i]);
    keep_packed(raw[i]);
  }
  mx = wave_max(mx);
  const float tw = wave_max(te);
  if (lane == 0) {
    sh_m[wave] = mx;
    sh_t[wave] = tw;
  }
  __syncthreads();
  float tmax = sh_t[0];
  mx = sh_m[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) {
    mx = fmaxf(mx, sh_m[i]);
    tmax = fmaxf(tmax, sh_t[i]);
  }
  const float base = mx == -INFINITY ? 0.0f : mx, c = LOG2E / a.tau, b = -base * c, b1 = -base * LOG2E;
  float s = exp2_32(fmaf(zt, c, b)), s1 = TWO ? exp2_32(fmaf(zt, LOG2E, b1)) : 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (i * THREADS + wave * 64 >= full) break;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float z = slot_elem<T>(raw[i], e);
      s += exp2_32(fmaf(z, c, b));
      if (TWO) s1 += exp2_32(fmaf(z, LOG2E, b1));
    }
    keep_packed(raw[i]);
  }
  double S, A;
  distill_list_sums<THREADS>(ent, a.K, 1.0f / a.tau, tmax, S, A);
  s = wave_sum(s);
  if (TWO) s1 = wave_sum(s1);
  if (wave * 64 < a.K) {
    S = wave_sum(S);
    A = wave_sum(A);
  }
  if (lane == 0) {
    sh_s[wave] = s;
    if (TWO) sh_s1[wave] = s1;
    sh_S[wave] = S;
    sh_A[wave] = A;
  }
  __syncthreads();
  RowSums r = {mx, 0.0f, 0.0f};
  S = A = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    r.s += sh_s[i];
    if (TWO) r.s1 += sh_s1[i];
    S += sh_S[i];
    A += sh_A[i];
  }
  const DistillRow o = distill_finish<T, THREADS, TWO>(a, m, w, r, tmax, S, A, ent);
  if (!a.dz) return;
  T *drow = a.dz + m * a.ldd;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = i * THREADS + tid;
    if (j >= full) break;
    float d[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = o.dense(slot_elem<T>(raw[i], e), TWO);
    store_slot(drow, j, d);
  }
  if (full * N + tid < a.V) drow[full * N + tid] = from_f32<T>(o.dense(zt, TWO));
  __syncthreads();  // the dense pass first, then the listed words on top of it
  distill_listed<T, THREADS, TWO>(a, o, ent, drow);
}

// Rows that do not fit the registers, and calls without a gradient: one pass with a running maximum and sum of each thread,
// then (with a gradient) a second one.
template <typename T, int THREADS, bool TWO>
__global__ void __launch_bounds__(THREADS) distill_stream_kernel(const DistillArgs<T> a) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64, FLIGHT = 4;
  extern __shared__ __align__(16) unsigned char lds[];
  DistillEntry *ent = reinterpret_cast<DistillEntry *>(lds);
  __shared__ float sh_m[WAVES], sh_t[WAVES], sh_s[WAVES], sh_s1[WAVES];
  __shared__ double sh_S[WAVES], sh_A[WAVES];
  const long m = blockIdx.x;
  const float w = a.weight ? a.weight[m] : 1.0f;
  if (w == 0.0f) return distill_without_weight<T, THREADS>(a, m);
  const T *row = a.z + m * a.ldz;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, full = a.V / N;
  const float c = LOG2E / a.tau;
  const float te = distill_entries<T, THREADS>(a, m, row, a.y && a.alpha < 1.0f, ent);
  const float zt = tail_elem(row, tid, a.V);
  float mx = zt, s = zt == -INFINITY ? 0.0f : 1.0f, s1 = s;
  for (int j0 = tid; j0 < full; j0 += FLIGHT * THREADS) {
    slot_t raw[FLIGHT];
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) {
      const int j = j0 + i * THREADS;
      raw[i] = j < full ? load_slot(row, j) : empty_slot<T>();
    }
    float top = mx;
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i) top = slot_max<T>(top, raw[i]);
    const float base = top == -INFINITY ? 0.0f : top, b = -base * c, b1 = -base * LOG2E;
    if (top > mx) {  // (mx = -inf: the sums are 0, and so is the factor)
      s *= exp2_32(fmaf(mx, c, b));
      if (TWO) s1 *= exp2_32(fmaf(mx, LOG2E, b1));
      mx = top;
    }
#pragma unroll
    for (int i = 0; i < FLIGHT; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float z = slot_elem<T>(raw[i], e);
        s += exp2_32(fmaf(z, c, b));
        if (TWO) s1 += exp2_32(fmaf(z, LOG2E, b1));
      }
  }
  const float own = mx;
  mx = wave_max(mx);
  const float tw = wave_max(te);
  if (lane == 0) {
    sh_m[wave] = mx;
    sh_t[wave] = tw;
  }
  __syncthreads();
  float tmax = sh_t[0];
  mx = sh_m[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) {
    mx = fmaxf(mx, sh_m[i]);
    tmax = fmaxf(tmax, sh_t[i]);
  }
  const float base = mx == -INFINITY ? 0.0f : mx;
  s *= exp2_32(fmaf(own, c, -base * c));
  if (TWO) s1 *= exp2_32(fmaf(own, LOG2E, -base * LOG2E));
  double S, A;
  distill_list_sums<THREADS>(ent, a.K, 1.0f / a.tau, tmax, S, A);
  s = wave_sum(s);
  if (TWO) s1 = wave_sum(s1);
  if (wave * 64 < a.K) {
    S = wave_sum(S);
    A = wave_sum(A);
  }
  if (lane == 0) {
    sh_s[wave] = s;
    if (TWO) sh_s1[wave] = s1;
    sh_S[wave] = S;
    sh_A[wave] = A;
  }
  __syncthreads();
  RowSums r = {mx, 0.0f, 0.0f};
  S = A = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    r.s += sh_s[i];
    if (TWO) r.s1 += sh_s1[i];
    S += sh_S[i];
    A += sh_A[i];
  }
  const DistillRow o = distill_finish<T, THREADS, TWO>(a, m, w, r, tmax, S, A, ent);
  if (!a.dz) return;
  T *drow = a.dz + m * a.ldd;
  for (int j = tid; j < full; j += THREADS) {
    const slot_t raw = load_slot(row, j);
    float d[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = o.dense(slot_elem<T>(raw, e), TWO);
    store_slot(drow, j, d);
  }
  if (full * N + tid < a.V) drow[full * N + tid] = from_f32<T>(o.dense(zt, TWO));
  __syncthreads();
  distill_listed<T, THREADS, TWO>(a, o, ent, drow);
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
