// Clipped policy loss of drawn words, with a penalty for leaving a reference model.
//   l = ln softmax(z / tau)(y),  rho = e^{l - old},  d = ref - l
//   loss = w (-min(rho A, clamp(rho, 1 - lo, 1 + hi) A) + beta (e^d - d - 1))
//   g = d loss / dl = w (-[not clipped] rho A + beta (1 - e^d)),       dz[v] = scale g ([v = y] - softmax(z / tau)(v)) / tau
// (e^d - d - 1 is what draws from the model say of KL(model || ref), one by one, never negative.)
#pragma once
#include "word_loss.h"

namespace rnnlm_dev {

template <typename T>
struct PolicyArgs {
  WordRows<T> rows;
  const float *old_logp, *ref_logp, *advantage, *weight;
  float *loss, *logp;
  float lo, hi, beta, scale;
};

// Loss of row m and (returned) the factor of its gradient, in 64 bits, by one thread.
template <typename T>
__device__ inline float policy_terms(const PolicyArgs<T> &a, long m, double l) {
  const double w = a.weight ? (double)a.weight[m] : 1.0, A = a.advantage[m];
  const double rho = a.old_logp ? exp(l - (double)a.old_logp[m]) : 1.0, least = 1.0 - (double)a.lo, most = 1.0 + (double)a.hi;
  const double free = rho * A, held = (rho < least ? least : rho > most ? most : rho) * A;  // (a NaN stays one)
  double loss = free > held ? -held : -free, g = free > held ? 0.0 : -free;
  if (a.beta != 0.0f) {
    const double d = (double)a.ref_logp[m] - l, e = expm1(d);
    loss += (double)a.beta * (d == INFINITY ? d : e - d);
    g -= (double)a.beta * e;
  }
  a.loss[m] = (float)(w * loss);
  if (a.logp) a.logp[m] = (float)l;
  return l == -INFINITY ? 0.0f : (float)(w * g * (double)a.scale / (double)a.rows.tau);
}

template <typename T, int THREADS>
__device__ inline void policy_does_not_count(const PolicyArgs<T> &a, long m) {
  if (threadIdx.x == 0) {
    a.loss[m] = 0.0f;
    if (a.logp) a.logp[m] = 0.0f;
  }
  if (a.rows.dz) word_no_gradient<T, THREADS>(a.rows.dz + m * a.rows.ldd, a.rows.V);
}

// A workgroup's row stays in registers between the sum and the gradient: read once, written once.  Bound by HBM: 2560 x 64000
// bf16 114 us (5.7 TB/s), 8192 x 100000 bf16 650 (5.0, where a copy reaches 4.9), 900 x 33278 fp32, a quarter of whose rows do not
// count, 33; 32 x 1000 fp32 4.2, the latency of its steps.
template <typename T, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 4) policy_row_kernel(const PolicyArgs<T> a) {
  __shared__ WordShared<THREADS / 64> sh;
  const WordRows<T> &w = a.rows;
  const long m = blockIdx.x;
  const int y = w.word(m);
  if (y < 0 || (a.weight && a.weight[m] == 0.0f)) return policy_does_not_count<T, THREADS>(a, m);
  const T *row = w.z + m * w.ldz;
  WordRow<T, THREADS, NV> held;
  held.load(row, w.V, w.once);
  const float zy = to_f32(row[y]);
  const WordSum r = held.sum(row, w.V, w.tau, sh);
  if (threadIdx.x == 0) sh.g = policy_terms(a, m, r.logp(zy, w.tau));
  __syncthreads();
  held.gradient(r, w.dz + m * w.ldd, zy, y, w.V, w.tau, sh.g);
}

// Rows that do not fit the registers, and calls without a gradient.  Loss alone, 2560 x 64000 bf16: 51 us (6.4 TB/s); 1280 x 300000
// bf16 446 (two reads and a write; 5.2 TB/s of them).
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) policy_stream_kernel(const PolicyArgs<T> a) {
  __shared__ WordShared<THREADS / 64> sh;
  const WordRows<T> &w = a.rows;
  const long m = blockIdx.x;
  const int y = w.word(m);
  if (y < 0 || (a.weight && a.weight[m] == 0.0f)) return policy_does_not_count<T, THREADS>(a, m);
  const T *row = w.z + m * w.ldz;
  const float zt = tail_elem(row, threadIdx.x, w.V), zy = to_f32(row[y]);
  const WordSum r = w.once && !w.dz ? word_sum_by_memory<T, THREADS, 4, true>(row, zt, w.V, w.tau, sh)
                                    : word_sum_by_memory<T, THREADS, 4, false>(row, zt, w.V, w.tau, sh);
  if (threadIdx.x == 0) sh.g = policy_terms(a, m, r.logp(zy, w.tau));
  if (!w.dz) return;
  __syncthreads();
  word_gradient_by_memory<T, THREADS>(r, row, w.dz + m * w.ldd, zt, zy, y, w.V, w.tau, sh.g);
}

}  // namespace rnnlm_dev
