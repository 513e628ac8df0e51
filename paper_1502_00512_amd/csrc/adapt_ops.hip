// Host side of the operators that adapt a trained model (include/rnnlm.h, "Adapting"): checks of arguments, choice of kernel,
// launches.
#include "adapters.h"
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

// ---- adapters ----
constexpr int64_t ADAPTER_ROWS_MAX = 1 << 17;  // (putting the rows in order compares each with each)
constexpr int ADAPTER_GRAD_WAVES = 8;

int adapter_r_tiles(int32_t R) { return (R + 15) / 16; }
// Columns of a wave of adapter_grad_kernel, in 16s: as many as its accumulators and operands leave registers for.
int adapter_grad_tiles(int32_t R, int32_t dtype) { return dtype == RNNLM_DTYPE_BF16 && adapter_r_tiles(R) <= 2 ? 8 : 4; }

// A sum over rows for W columns: blocks of columns, positions of a chunk.  Chunks until there are some 512 workgroups.
struct GradPlan {
  int blocks, chunks, chunk;
};
GradPlan adapter_grad_plan(int64_t rows, int32_t W, int32_t R, int32_t dtype) {
  GradPlan p;
  const int cols = ADAPTER_GRAD_WAVES * 16 * adapter_grad_tiles(R, dtype);
  p.blocks = (W + cols - 1) / cols;
  const int64_t tiles = std::max<int64_t>(1, (rows + ADAPTER_TILE - 1) / ADAPTER_TILE);
  const int64_t want = std::min<int64_t>(tiles, std::max(1, 512 / p.blocks));
  p.chunk = (int)((tiles + want - 1) / want) * ADAPTER_TILE;
  p.chunks = (int)std::max<int64_t>(1, (rows + p.chunk - 1) / p.chunk);
  return p;
}

// Rows in up to this many tiles are taken as they come: an adapter is read once for each tile that has it.
constexpr int ADAPTER_UNORDERED = 4;

struct AdapterPlan {
  long Mp;
  size_t perm, start, inner, tr_inner, tr_dinner, dinner, part, split, total;
};
AdapterPlan adapter_plan(int64_t rows, int32_t K, int32_t N, int32_t n, int32_t R, int32_t dtype, bool backward) {
  AdapterPlan p = {};
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += align256(bytes);
    return at;
  };
  p.perm = take((size_t)rows * 4);
  p.start = take(((size_t)n + 1) * 4);
  if (!backward) {
    p.inner = take((size_t)rows * R * 4);
  } else {
    p.Mp = round_up(rows + ADAPTER_TILE, 64);
    const size_t turned = (size_t)p.Mp * R * (dtype == RNNLM_DTYPE_FP32 ? 4 : 6);
    const GradPlan up = adapter_grad_plan(rows, N, R, dtype), down = adapter_grad_plan(rows, K, R, dtype);
    p.tr_inner = take(turned);
    p.tr_dinner = take(turned);
    p.dinner = take((size_t)rows * R * 4);
    p.part = take((size_t)up.blocks * rows * R * 4);
    p.split = take(std::max(up.chunks > 1 ? (size_t)2 * up.chunks * N : 0, down.chunks > 1 ? (size_t)2 * down.chunks * K : 0) * R * 4);
  }
  p.total = std::max<size_t>(o, 256);
  return p;
}
bool adapter_sizes_ok(int64_t rows, int32_t K, int32_t N, int32_t n, int32_t R, int32_t dtype) {
  return rows >= 0 && rows <= ADAPTER_ROWS_MAX && K >= 1 && K <= 65536 && N >= 1 && N <= LOGITS_V_MAX && n >= 1 && n <= 65536 && R >= 1 &&
         R <= ADAPTER_R_MAX && (dtype == RNNLM_DTYPE_FP32 || dtype == RNNLM_DTYPE_BF16);
}
bool adapters_ok(const rnnlm_adapters *a, int32_t dtype) {
  return a->down && a->up && aligned(a->down, elem_bytes(dtype)) && aligned(a->up, elem_bytes(dtype)) && aligned(a->scale, 4);
}

template <typename T>
void launch_order(const AdapterRows &rows, void *perm, void *start, const float *inner, const Transposed<T> &tr, int32_t *flag, hipStream_t st) {
  hipLaunchKernelGGL(adapter_order_kernel<T>, dim3((rows.M + rows.n + 64) / 64), dim3(1024), 0, st, rows, static_cast<int32_t *>(perm),
                     static_cast<int32_t *>(start), inner, tr, flag);
}
template <typename T>
void launch_inner(const InnerArgs<T> &a, hipStream_t st) {
  const dim3 grid((a.rows.M + ADAPTER_TILE - 1) / ADAPTER_TILE, std::min(ADAPTER_TILE, a.rows.n));
  switch (adapter_r_tiles(a.R)) {
    case 1: hipLaunchKernelGGL((adapter_inner_kernel<T, 1>), grid, dim3(512), 0, st, a); break;
    case 2: hipLaunchKernelGGL((adapter_inner_kernel<T, 2>), grid, dim3(512), 0, st, a); break;
    case 3: hipLaunchKernelGGL((adapter_inner_kernel<T, 3>), grid, dim3(512), 0, st, a); break;
    default: hipLaunchKernelGGL((adapter_inner_kernel<T, 4>), grid, dim3(512), 0, st, a);
  }
}
template <typename T, int NF, bool PACKED, bool ACROSS>
void launch_outer_as(OuterArgs<T> a, hipStream_t st) {
  const int64_t tiles = (a.rows.M + ADAPTER_TILE - 1) / ADAPTER_TILE, cols = (a.N + 255) / 256;
  // a wave's rows of inner are read once for `blocks` blocks, as long as some 2048 workgroups are left
  a.blocks = (int)std::max<int64_t>(std::min<int64_t>(4, std::max<int64_t>(1, tiles * cols / 2048)), (tiles * cols * 256 + THREADS_MAX - 1) / THREADS_MAX);
  const dim3 grid((unsigned)tiles, (unsigned)((cols + a.blocks - 1) / a.blocks));
  hipLaunchKernelGGL((adapter_outer_kernel<T, NF, PACKED, ACROSS>), grid, dim3(256), 0, st, a);
}
template <typename T, bool ACROSS>
void launch_outer(const OuterArgs<T> &a, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (a.R <= 16) launch_outer_as<T, 1, true, ACROSS>(a, st);
    else if (a.R <= 32) launch_outer_as<T, 1, false, ACROSS>(a, st);
    else launch_outer_as<T, 2, false, ACROSS>(a, st);
  } else {
    switch (adapter_r_tiles(a.R)) {
      case 1: launch_outer_as<T, 1, false, ACROSS>(a, st); break;
      case 2: launch_outer_as<T, 2, false, ACROSS>(a, st); break;
      case 3: launch_outer_as<T, 3, false, ACROSS>(a, st); break;
      default: launch_outer_as<T, 4, false, ACROSS>(a, st);
    }
  }
}
template <typename T, bool INNER>
int grad_call(GradArgs<T> a, const GradPlan &p, hipStream_t st) {
  const dim3 grid(p.blocks, p.chunks), threads(64 * ADAPTER_GRAD_WAVES);
  a.chunk = p.chunk;
  if (a.rows.M > 0) {
    switch (adapter_r_tiles(a.R)) {
      case 1: hipLaunchKernelGGL((adapter_grad_kernel<T, 1, sizeof(T) == 2 ? 8 : 4, INNER>), grid, threads, 0, st, a); break;
      case 2: hipLaunchKernelGGL((adapter_grad_kernel<T, 2, sizeof(T) == 2 ? 8 : 4, INNER>), grid, threads, 0, st, a); break;
      case 3: hipLaunchKernelGGL((adapter_grad_kernel<T, 3, 4, INNER>), grid, threads, 0, st, a); break;
      default: hipLaunchKernelGGL((adapter_grad_kernel<T, 4, 4, INNER>), grid, threads, 0, st, a);
    }
    LAUNCHED();
  }
  const JoinArgs j = {a.start, a.split, a.scale, a.G, a.N, a.R, a.chunk, a.rows.n, a.across};
  const int64_t size = (int64_t)a.N * a.R, parts = std::max<int64_t>(1, std::min<int64_t>((size + 2047) / 2048, 4096 / std::min(a.rows.n, 4096)));
  hipLaunchKernelGGL(adapter_join_kernel, dim3((unsigned)parts, std::min(a.rows.n, 4096)), dim3(256), 0, st, j);
  LAUNCHED();
  return RNNLM_OK;
}

template <typename T>
int adapter_forward(const T *x, int64_t ldx, int64_t M, int32_t K, int32_t N, const rnnlm_adapters &a, const int32_t *ids, const T *base,
                    int64_t ldb, T *out, int64_t ldo, float *inner, int32_t *flag, char *ws, const AdapterPlan &p, hipStream_t st) {
  AdapterRows rows = {ids, nullptr, (int)M, a.n};
  if (M > ADAPTER_UNORDERED * ADAPTER_TILE) {
    launch_order<T>(rows, ws + p.perm, ws + p.start, nullptr, Transposed<T>{}, flag, st);
    LAUNCHED();
    rows.perm = reinterpret_cast<int32_t *>(ws + p.perm);
  }
  if (!inner) inner = reinterpret_cast<float *>(ws + p.inner);
  launch_inner<T>({rows, x, static_cast<const T *>(a.down), ldx, K, a.R, inner, flag}, st);
  LAUNCHED();
  launch_outer<T, false>({rows, inner, false, static_cast<const T *>(a.up), a.scale, base, out, ldb, ldo, N, a.R, 1}, st);
  LAUNCHED();
  return RNNLM_OK;
}

template <typename T>
int adapter_backward(const T *dout, int64_t ldd, const T *x, int64_t ldx, const float *inner, int64_t M, int32_t K, int32_t N,
                     const rnnlm_adapters &a, const int32_t *ids, float *ddown, float *dup, T *dx, int64_t lddx, int32_t *flag, char *ws,
                     const AdapterPlan &p, hipStream_t st) {
  const int32_t dtype = sizeof(T) == 4 ? RNNLM_DTYPE_FP32 : RNNLM_DTYPE_BF16;
  const AdapterRows rows = {ids, reinterpret_cast<int32_t *>(ws + p.perm), (int)M, a.n};
  const int32_t *start = reinterpret_cast<int32_t *>(ws + p.start);
  const Transposed<T> tr_inner = {reinterpret_cast<T *>(ws + p.tr_inner), p.Mp, a.R};
  const Transposed<T> tr_dinner = {reinterpret_cast<T *>(ws + p.tr_dinner), p.Mp, a.R};
  float *dinner = reinterpret_cast<float *>(ws + p.dinner), *part = reinterpret_cast<float *>(ws + p.part);
  float *split = reinterpret_cast<float *>(ws + p.split);
  launch_order<T>(rows, ws + p.perm, ws + p.start, inner, tr_inner, flag, st);
  LAUNCHED();
  const GradPlan up = adapter_grad_plan(M, N, a.R, dtype), down = adapter_grad_plan(M, K, a.R, dtype);
  int rc = grad_call<T, true>({rows, start, dout, ldd, tr_inner, static_cast<const T *>(a.up), a.scale, dup, split, part, N, a.R, 0, false}, up, st);
  if (rc) return rc;
  if (M > 0) {
    hipLaunchKernelGGL(adapter_dinner_kernel<T>, dim3((unsigned)((M * a.R + 255) / 256)), dim3(256), 0, st,
                       DinnerArgs<T>{rows, start, part, a.scale, dinner, tr_dinner, up.blocks, a.R});
    LAUNCHED();
  }
  rc = grad_call<T, false>({rows, start, x, ldx, tr_dinner, nullptr, nullptr, ddown, split, nullptr, K, a.R, 0, true}, down, st);
  if (rc) return rc;
  if (dx && M > 0) {
    launch_outer<T, true>({rows, dinner, true, static_cast<const T *>(a.down), nullptr, nullptr, dx, 0, lddx, K, a.R, 1}, st);
    LAUNCHED();
  }
  return RNNLM_OK;
}

}  // namespace

extern "C" {

size_t rnnlm_adapter_workspace_bytes(int64_t rows, int32_t K, int32_t N, int32_t n, int32_t R, int32_t dtype, int32_t backward) {
  return adapter_sizes_ok(rows, K, N, n, R, dtype) && (backward == 0 || backward == 1) ? adapter_plan(rows, K, N, n, R, dtype, backward != 0).total : 0;
}

int rnnlm_adapter_forward(const void *x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t K, int32_t N, const rnnlm_adapters *a,
                          const int32_t *ids, const void *base, int64_t ld_base, void *out, int64_t ld_out, float *inner,
                          int32_t *range_flag, void *workspace, size_t workspace_bytes, void *stream) {
  if (!a || !adapter_sizes_ok(rows, K, N, a->n, a->R, dtype) || !adapters_ok(a, dtype) || !rows_ok(x, dtype, rows, K, ld_x) ||
      !rows_ok(out, dtype, rows, N, ld_out) || (base && !rows_ok(base, dtype, rows, N, ld_base)) || (rows > 0 && !ids) || !aligned(ids, 4) ||
      !aligned(inner, 4) || !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  const size_t es = elem_bytes(dtype);
  const auto all = [&](const void *p, int64_t ld, int32_t w) { return span(p, rows > 0 ? ((size_t)(rows - 1) * ld + w) * es : 0); };
  if (base && (base == out ? ld_base != ld_out : meet(all(base, ld_base, N), all(out, ld_out, N)))) return RNNLM_ERR_ARG;
  if (meet(all(x, ld_x, K), all(out, ld_out, N))) return RNNLM_ERR_ARG;
  const AdapterPlan p = adapter_plan(rows, K, N, a->n, a->R, dtype, false);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < p.total) return RNNLM_ERR_ARG;
  if (rows == 0) return RNNLM_OK;
  hipStream_t st = (hipStream_t)stream;
  char *ws = static_cast<char *>(workspace);
  if (dtype == RNNLM_DTYPE_FP32)
    return adapter_forward<float>(static_cast<const float *>(x), ld_x, rows, K, N, *a, ids, static_cast<const float *>(base), ld_base,
                                  static_cast<float *>(out), ld_out, inner, range_flag, ws, p, st);
  return adapter_forward<bf16_t>(static_cast<const bf16_t *>(x), ld_x, rows, K, N, *a, ids, static_cast<const bf16_t *>(base), ld_base,
                                 static_cast<bf16_t *>(out), ld_out, inner, range_flag, ws, p, st);
}

int rnnlm_adapter_backward(const void *dout, int64_t ld_dout, const void *x, int64_t ld_x, const float *inner, int32_t dtype, int64_t rows,
                           int32_t K, int32_t N, const rnnlm_adapters *a, const int32_t *ids, float *ddown, float *dup, void *dx,
                           int64_t ld_dx, int32_t *range_flag, void *workspace, size_t workspace_bytes, void *stream) {
  if (!a || !adapter_sizes_ok(rows, K, N, a->n, a->R, dtype) || !adapters_ok(a, dtype) || !rows_ok(dout, dtype, rows, N, ld_dout) ||
      !rows_ok(x, dtype, rows, K, ld_x) || (dx && !rows_ok(dx, dtype, rows, K, ld_dx)) || (rows > 0 && (!ids || !inner)) || !ddown || !dup ||
      !aligned(ids, 4) || !aligned(inner, 4) || !aligned(ddown, 4) || !aligned(dup, 4) || !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  const size_t es = elem_bytes(dtype);
  const auto all = [&](const void *p, int64_t ld, int32_t w) { return span(p, rows > 0 ? ((size_t)(rows - 1) * ld + w) * es : 0); };
  if (dx && (meet(all(dx, ld_dx, K), all(x, ld_x, K)) || meet(all(dx, ld_dx, K), all(dout, ld_dout, N)))) return RNNLM_ERR_ARG;
  const AdapterPlan p = adapter_plan(rows, K, N, a->n, a->R, dtype, true);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < p.total) return RNNLM_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  char *ws = static_cast<char *>(workspace);
  if (dtype == RNNLM_DTYPE_FP32)
    return adapter_backward<float>(static_cast<const float *>(dout), ld_dout, static_cast<const float *>(x), ld_x, inner, rows, K, N, *a, ids,
                                   ddown, dup, static_cast<float *>(dx), ld_dx, range_flag, ws, p, st);
  return adapter_backward<bf16_t>(static_cast<const bf16_t *>(dout), ld_dout, static_cast<const bf16_t *>(x), ld_x, inner, rows, K, N, *a, ids,
                                  ddown, dup, static_cast<bf16_t *>(dx), ld_dx, range_flag, ws, p, st);
}

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
