// Host side of the operators that adapt a trained model (include/rnnlm.h, "Adapting"): checks of arguments, choice of kernel,
// launches.
#include "call_checks.h"
#include "losses.h"
#include "policy.h"
#include "preference.h"

namespace {

template <typename T>
WordRows<T> word_rows(const void *logits, int64_t rows, int32_t V, int64_t ld, const int32_t *y, float tau, void *dlogits, int64_t ldd,
                      int32_t *range_flag) {
  const int32_t dtype = sizeof(T) == 4 ? RNNLM_DTYPE_FP32 : RNNLM_DTYPE_BF16;
  return {static_cast<const T *>(logits), ld, static_cast<T *>(dlogits), ldd, y, range_flag, tau, V, read_once(rows, V, dtype)};
}
// A gradient in place row by row, or apart from the logits.
bool gradient_rows_ok(const void *logits, int64_t ld, const void *dlogits, int64_t ldd, int32_t dtype, int64_t rows, int32_t V) {
  if (!dlogits) return true;
  if (!rows_ok(dlogits, dtype, rows, V, ldd)) return false;
  const size_t es = elem_bytes(dtype);
  return dlogits == logits ? ld == ldd
                           : rows == 0 || !meet(span(logits, ((size_t)(rows - 1) * ld + V) * es),
                                                span(dlogits, ((size_t)(rows - 1) * ldd + V) * es));
}

// Threads and slots of a thread that hold a row of `slots` whole slots: f(std::integral_constant...).  Many short rows: a wave
// each, since a row's time is the latency of its steps, not its bytes.
template <int THREADS, int NV>
struct RowShape {
  static constexpr int threads = THREADS, nv = NV;
};
constexpr int HELD_SLOTS = 1024 * 25;
template <class F>
void with_row_shape(int64_t rows, int slots, F &&f) {
  const bool wave_each = rows >= 1024 && slots <= 64 * 8;
  if (wave_each && slots <= 64 * 2) f(RowShape<64, 2>());
  else if (wave_each && slots <= 64 * 4) f(RowShape<64, 4>());
  else if (wave_each) f(RowShape<64, 8>());
  else if (slots <= 256) f(RowShape<256, 1>());
  else if (slots <= 256 * 2) f(RowShape<256, 2>());
  else if (slots <= 256 * 4) f(RowShape<256, 4>());
  else if (slots <= 256 * 6) f(RowShape<256, 6>());
  else if (slots <= 256 * 8) f(RowShape<256, 8>());
  else if (slots <= 512 * 6) f(RowShape<512, 6>());
  else if (slots <= 512 * 8) f(RowShape<512, 8>());
  else if (slots <= 512 * 12) f(RowShape<512, 12>());
  else if (slots <= 512 * 16) f(RowShape<512, 16>());
  else if (slots <= 512 * 20) f(RowShape<512, 20>());
  else if (slots <= 512 * 25) f(RowShape<512, 25>());
  else if (slots <= 1024 * 18) f(RowShape<1024, 18>());
  else f(RowShape<1024, 25>());
}

// ---- policy loss ----
template <typename T>
int policy_call(const PolicyArgs<T> &a, int64_t rows, hipStream_t st) {
  const int slots = a.rows.V / SlotOf<T>::N;  // whole ones: what a thread's registers hold
  if (!a.rows.dz || slots > HELD_SLOTS) {
    hipLaunchKernelGGL((policy_stream_kernel<T, 512>), dim3((unsigned)rows), dim3(512), 0, st, a);
  } else {
    with_row_shape(rows, slots, [&](auto shape) {
      hipLaunchKernelGGL((policy_row_kernel<T, decltype(shape)::threads, decltype(shape)::nv>), dim3((unsigned)rows),
                         dim3(decltype(shape)::threads), 0, st, a);
    });
  }
  LAUNCHED();
  return RNNLM_OK;
}

// ---- preference loss ----
size_t preference_rows_bytes(int64_t rows) { return align256((size_t)rows * sizeof(PreferenceRow)); }
bool preference_sizes_ok(int32_t T, int32_t pairs) {
  return T >= 0 && pairs >= 1 && pairs <= (1 << 20) && (int64_t)T * pairs * 2 <= ROWS_MAX;
}
template <typename T>
int preference_call(const PreferenceArgs<T> &a, hipStream_t st) {
  const int64_t rows = (int64_t)a.Tn * a.P * 2;
  if (rows > 0) {
    hipLaunchKernelGGL((preference_words_kernel<T, 512>), dim3((unsigned)rows), dim3(512), 0, st, a);
    LAUNCHED();
  }
  hipLaunchKernelGGL(preference_pairs_kernel<T>, dim3((unsigned)a.P), dim3(64), 0, st, a);
  LAUNCHED();
  if (rows > 0 && a.rows.dz) {
    hipLaunchKernelGGL((preference_gradient_kernel<T, 512>), dim3((unsigned)rows), dim3(512), 0, st, a);
    LAUNCHED();
  }
  return RNNLM_OK;
}

}  // namespace

extern "C" {

int rnnlm_policy_loss(const void *logits, int32_t dtype, int64_t rows, int32_t V, int64_t ld, const int32_t *y,
                      const float *old_logp, const float *ref_logp, const float *advantage, const float *weight, float tau,
                      float clip_low, float clip_high, float beta, float scale, float *loss, float *logp, double *sum_loss,
                      void *dlogits, int64_t ld_dlogits, int32_t *range_flag, void *stream) {
  if (!rows_ok(logits, dtype, rows, V, ld) || (rows > 0 && (!y || !advantage || !loss || (beta != 0.0f && !ref_logp))) || !tau_ok(tau) ||
      !(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f && std::isfinite(clip_high)) ||
      !(beta >= 0.0f && std::isfinite(beta)) || !std::isfinite(scale) ||
      !gradient_rows_ok(logits, ld, dlogits, ld_dlogits, dtype, rows, V))
    return RNNLM_ERR_ARG;
  if (!aligned(y, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(advantage, 4) || !aligned(weight, 4) ||
      !aligned(loss, 4) || !aligned(logp, 4) || !aligned(sum_loss, 8) || !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  if (rows > 0) {
    const auto call = [&](auto rows_of) {
      typedef std::remove_const_t<std::remove_pointer_t<decltype(rows_of.z)>> T;
      return policy_call<T>({rows_of, old_logp, ref_logp, advantage, weight, loss, logp, clip_low, clip_high, beta, scale}, rows, st);
    };
    const int rc = dtype == RNNLM_DTYPE_FP32 ? call(word_rows<float>(logits, rows, V, ld, y, tau, dlogits, ld_dlogits, range_flag))
                                             : call(word_rows<bf16_t>(logits, rows, V, ld, y, tau, dlogits, ld_dlogits, range_flag));
    if (rc) return rc;
  }
  if (sum_loss) {
    hipLaunchKernelGGL(sum_losses_kernel, dim3(1), dim3(1024), 0, st, loss, (long)rows, sum_loss);
    LAUNCHED();
  }
  return RNNLM_OK;
}

size_t rnnlm_preference_workspace_bytes(int32_t T, int32_t pairs) {
  return preference_sizes_ok(T, pairs) ? preference_rows_bytes((int64_t)T * pairs * 2) + align256((size_t)pairs * sizeof(PreferencePair)) : 0;
}

int rnnlm_preference_loss(const void *logits, int32_t dtype, int32_t T, int32_t pairs, int32_t V, int64_t ld, const int32_t *y,
                          const float *ref, const float *weight, int32_t kind, float beta, float smoothing, int32_t mean, float scale,
                          float *loss, float *logp, double *sum_loss, void *dlogits, int64_t ld_dlogits, int32_t *range_flag,
                          void *workspace, size_t workspace_bytes, void *stream) {
  if (!preference_sizes_ok(T, pairs)) return RNNLM_ERR_ARG;
  const int64_t rows = (int64_t)T * pairs * 2;
  if (!rows_ok(logits, dtype, rows, V, ld) || (rows > 0 && !y) || !loss || kind < RNNLM_PREFERENCE_LOGISTIC ||
      kind > RNNLM_PREFERENCE_HINGE || !(beta > 0.0f && std::isfinite(beta)) || !(smoothing >= 0.0f && smoothing <= 0.5f) ||
      (smoothing != 0.0f && kind != RNNLM_PREFERENCE_LOGISTIC) || (mean != 0 && mean != 1) || !std::isfinite(scale) ||
      !gradient_rows_ok(logits, ld, dlogits, ld_dlogits, dtype, rows, V))
    return RNNLM_ERR_ARG;
  if (!aligned(y, 4) || !aligned(ref, 4) || !aligned(weight, 4) || !aligned(loss, 4) || !aligned(logp, 4) || !aligned(sum_loss, 8) ||
      !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < rnnlm_preference_workspace_bytes(T, pairs)) return RNNLM_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  const auto call = [&](auto rows_of) {
    typedef std::remove_const_t<std::remove_pointer_t<decltype(rows_of.z)>> E;
    return preference_call<E>({rows_of, ref, weight, loss, logp, T, pairs, kind, mean != 0, beta, smoothing, scale,
                               static_cast<PreferenceRow *>(workspace),
                               reinterpret_cast<PreferencePair *>(static_cast<char *>(workspace) + preference_rows_bytes(rows))},
                              st);
  };
  const int rc = dtype == RNNLM_DTYPE_FP32 ? call(word_rows<float>(logits, rows, V, ld, y, 1.0f, dlogits, ld_dlogits, range_flag))
                                           : call(word_rows<bf16_t>(logits, rows, V, ld, y, 1.0f, dlogits, ld_dlogits, range_flag));
  if (rc) return rc;
  if (sum_loss) {
    hipLaunchKernelGGL(sum_losses_kernel, dim3(1), dim3(1024), 0, st, loss, (long)pairs, sum_loss);
    LAUNCHED();
  }
  return RNNLM_OK;
}

}  // extern "C"
