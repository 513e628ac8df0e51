// Host side of the operators that adapt a trained model (include/rnnlm.h, "Adapting"): checks of arguments, choice of kernel,
// launches.
#include <atomic>

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
// each, since a row's time is the latency of its steps, not its bytes.  The shapes of 25 slots keep 36 to 100 bytes of a thread in
// scratch.  512 threads of 25 and 1024 of 13, us: rows that meet, 2560 x 100000 bf16 214 and 242, x 50000 fp32 200 and 214, but the policy
// loss, 8192 x 100000 bf16 657 and 623, 2560 x 50000 fp32 220 and 194.
template <int THREADS, int NV>
struct RowShape {
  static constexpr int threads = THREADS, nv = NV;
};
constexpr int HELD_SLOTS = 1024 * 25;
template <class F>
void with_long_row_shape(int slots, F &&f) {  // of more than 1024 slots
  if (slots <= 256 * 6) f(RowShape<256, 6>());
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
template <class F>
void with_row_shape(int64_t rows, int slots, F &&f) {
  const bool wave_each = rows >= 1024 && slots <= 64 * 8;
  if (wave_each && slots <= 64 * 2) f(RowShape<64, 2>());
  else if (wave_each && slots <= 64 * 4) f(RowShape<64, 4>());
  else if (wave_each) f(RowShape<64, 8>());
  else if (slots <= 256) f(RowShape<256, 1>());
  else if (slots <= 256 * 2) f(RowShape<256, 2>());
  else if (slots <= 256 * 4) f(RowShape<256, 4>());
  else with_long_row_shape(slots, f);
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
std::atomic<int32_t> preference_polls{256};  // of about a microsecond

struct PreferencePlan {
  size_t row, pair, published, done, total;
};
PreferencePlan preference_plan(int32_t T, int32_t pairs) {
  const size_t rows = (size_t)T * pairs * 2;
  PreferencePlan p;
  size_t o = 0;
  auto take = [&](size_t n) {
    const size_t at = o;
    o += align256(n);
    return at;
  };
  p.row = take(rows * sizeof(PreferenceRow));
  p.pair = take((size_t)pairs * sizeof(PreferencePair));
  p.published = take(rows * sizeof(unsigned long long));
  p.done = take(rows * sizeof(int));
  p.total = o;
  return p;
}
bool preference_sizes_ok(int32_t T, int32_t pairs) {
  return T >= 0 && pairs >= 1 && pairs <= (1 << 20) && (int64_t)T * pairs * 2 <= ROWS_MAX;
}
template <typename T>
int preference_call(const PreferenceArgs<T> &a, hipStream_t st) {
  const int64_t rows = (int64_t)a.Tn * a.P * 2;
  const int slots = a.rows.V / SlotOf<T>::N;
  // Rows that meet, where the logits are many and the rows long: they and two passes, us: 26 x 10 bf16 rows of 64000 (33 MB) 22.0
  // and 23.8, 128 x 10 of 33000 46 and 48, 128 x 20 of 100000 211 and 297, 32 x 20 fp32 of 33278 42 and 48; but 64 x 10 bf16 of
  // 10000 15.0 and 13.0, 128 x 10 of them 19.4 and 17.4, and 128 x 64 rows of 4000 57 and 45 (a wave a row: all of them wait).
  if (rows > 0 && a.rows.dz && slots <= HELD_SLOTS && slots > 1024 && a.Tn <= PREFERENCE_MEET && (double)rows * a.rows.V * sizeof(T) > 30e6) {
    hipLaunchKernelGGL(preference_clear_kernel<T>, dim3((unsigned)std::min<int64_t>(256, (rows + 255) / 256)), dim3(256), 0, st, a, (long)rows);
    LAUNCHED();
    with_long_row_shape(slots, [&](auto shape) {
      constexpr int THREADS = decltype(shape)::threads, NV = decltype(shape)::nv;
      hipLaunchKernelGGL((preference_meet_kernel<T, THREADS, NV>), dim3((unsigned)rows), dim3(THREADS), 0, st, a);
    });
    LAUNCHED();
    hipLaunchKernelGGL((preference_rest_kernel<T, 512>), dim3((unsigned)std::min<int64_t>(rows, 256)), dim3(512), 0, st, a, (long)rows);
    LAUNCHED();
    return RNNLM_OK;
  }
  if (rows > 0) {
    // (512 threads have eight slots each under way per round: shorter rows are left to fewer)
    if (slots <= 256) hipLaunchKernelGGL((preference_words_kernel<T, 64>), dim3((unsigned)rows), dim3(64), 0, st, a);
    else if (slots <= 1024) hipLaunchKernelGGL((preference_words_kernel<T, 256>), dim3((unsigned)rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((preference_words_kernel<T, 512>), dim3((unsigned)rows), dim3(512), 0, st, a);
    LAUNCHED();
  }
  const bool gradient = rows > 0 && a.rows.dz, held = slots <= HELD_SLOTS, inside = gradient && held && a.Tn <= PREFERENCE_INSIDE;
  if (!inside) {
    if (a.Tn <= 64) hipLaunchKernelGGL((preference_pairs_kernel<T, 2>), dim3((unsigned)a.P), dim3(128), 0, st, a);
    else hipLaunchKernelGGL((preference_pairs_kernel<T, 16>), dim3((unsigned)a.P), dim3(1024), 0, st, a);
    LAUNCHED();
  }
  if (!gradient) return RNNLM_OK;
  if (!held) {
    hipLaunchKernelGGL((preference_stream_kernel<T, 512>), dim3((unsigned)rows), dim3(512), 0, st, a);
  } else {
    with_row_shape(rows, slots, [&](auto shape) {
      constexpr int THREADS = decltype(shape)::threads, NV = decltype(shape)::nv;
      if (inside) hipLaunchKernelGGL((preference_row_kernel<T, THREADS, NV, true>), dim3((unsigned)rows), dim3(THREADS), 0, st, a);
      else hipLaunchKernelGGL((preference_row_kernel<T, THREADS, NV, false>), dim3((unsigned)rows), dim3(THREADS), 0, st, a);
    });
  }
  LAUNCHED();
  return RNNLM_OK;
}

// ---- adapters ----
constexpr int64_t ADAPTER_ROWS_MAX = 1 << 17;  // (putting the rows in order compares each with each)

int adapter_r_tiles(int32_t R) { return (R + 15) / 16; }
// Columns of a wave of adapter_grad_kernel, in 16s.  Four, even where some registers go to scratch (bf16 of R > 48: 196 bytes of a
// thread, fp32 of 16 < R <= 32: 116), since half the columns are twice the parts of dinner: four and two, us, 2560 x 64000, 16 adapters:
// bf16 R = 64 331 and 468, fp32 R = 32 356 and 396 (900 x 33278: 135 and 140, 135 and 135).
// small: half of what R <= 16 has otherwise, where that lets two workgroups share a compute unit, for gradients of up to 128 MB: they
// and the others, us: 160 x 2000 bf16 (R = 16) 29 and 32, 900 x 33278 fp32 (R = 5) 75 and 78 (but bf16, R = 16 60 and 57); 2560 x
// 64000 bf16 (R = 16, 1 and 128 adapters) 113 and 105, 301 and 271, fp32 (1 and 16 adapters) 196 and 194, 218 and 216.
constexpr int adapter_grad_tiles(int r_tiles, bool bf16, bool small) {
  return r_tiles == 1 ? (bf16 ? 8 : 4) / (small ? 2 : 1) : bf16 || r_tiles == 2 ? 4 : 2;
}
bool adapter_grad_small(int64_t rows, int32_t N, int32_t dtype) { return (double)rows * N * (double)elem_bytes(dtype) <= (double)READ_ONCE_BYTES; }
constexpr int adapter_input_tiles(int r_tiles, bool bf16) { return r_tiles <= 2 || bf16 ? 4 : 2; }

// A sum over rows for W columns: blocks of columns, positions of a chunk.  A compute unit holds `together` workgroups, each of
// which takes some 6 us and 2.5 a tile; each chunk may leave W R numbers to be written and read once more.  The chunk for which rounds of
// workgroups and that come out least (900 rows, N = 33278, R = 5, fp32: 85 us by chunks until there were 512 workgroups, which
// made 520, 3 rounds).
struct GradPlan {
  int blocks, chunks, chunk;
};
GradPlan adapter_grad_plan(int64_t rows, int32_t W, int32_t R, int tiles_of_wave, int together) {
  GradPlan p;
  const int cols = ADAPTER_GRAD_WAVES * 16 * tiles_of_wave;
  p.blocks = (W + cols - 1) / cols;
  const int64_t tiles = std::max<int64_t>(1, (rows + ADAPTER_TILE - 1) / ADAPTER_TILE);
  int64_t chunks = 1;
  double least = INFINITY;
  for (int64_t each = 1; each <= std::min<int64_t>(tiles, ADAPTER_CHUNK / ADAPTER_TILE); ++each) {
    const int64_t k = (tiles + each - 1) / each, rounds = (k * p.blocks + 256 * together - 1) / (256 * together);
    const double us = rounds * (2.5 * each + 6.0) + (double)k * W * R * 8 / 5e6;
    if (us <= least) least = us, chunks = k, p.chunk = (int)each * ADAPTER_TILE;
  }
  // Few workgroups: parts of tiles, by the same costs, since a workgroup takes its adapters one after the other (160 rows of 8
  // adapters, N = 2000: 38 us by whole tiles, 34 so; 64 rows of one adapter, N = 10000, R = 60, lose 13 us by less than the costs).
  const double rows_least = std::sqrt((double)rows * W * R * 8 / 5e6 * ADAPTER_TILE / 3.0);
  if (chunks * p.blocks < 128)
    p.chunk = (int)std::min<int64_t>(p.chunk, round_up(std::max<int64_t>({1, rows * p.blocks / 256, std::lround(rows_least)}), 8));
  p.chunks = (int)std::max<int64_t>(1, (rows + p.chunk - 1) / p.chunk);
  return p;
}
GradPlan adapter_up_plan(int64_t rows, int32_t N, int32_t R, int32_t dtype) {
  const bool small = adapter_grad_small(rows, N, dtype);
  const int r_tiles = adapter_r_tiles(R);
  return adapter_grad_plan(rows, N, R, adapter_grad_tiles(r_tiles, dtype == RNNLM_DTYPE_BF16, small), r_tiles == 1 && small ? 2 : 1);
}
GradPlan adapter_down_plan(int64_t rows, int32_t K, int32_t R, int32_t dtype) {
  return adapter_grad_plan(rows, K, R, adapter_input_tiles(adapter_r_tiles(R), dtype == RNNLM_DTYPE_BF16), 1);
}

// Rows in up to this many tiles are taken as they come: an adapter is read once for each tile that has it.
constexpr int ADAPTER_UNORDERED = 4;

// Sums of up to this many blocks of columns are formed where they are used, more in a launch of their own.
constexpr int ADAPTER_BLOCKS_INSIDE = 8;

struct AdapterPlan {
  size_t perm, sorted, start, inner, part, dinner, split_up, split_down, total;
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
  p.sorted = take((size_t)rows * 4);
  p.start = take(((size_t)n + 1) * 4);
  if (!backward) {
    p.inner = take((size_t)rows * R * 4);
  } else {
    const GradPlan up = adapter_up_plan(rows, N, R, dtype), down = adapter_down_plan(rows, K, R, dtype);
    p.part = take((size_t)up.blocks * rows * R * 4);
    p.dinner = take((size_t)rows * R * 4);
    p.split_up = take(up.chunks > 1 ? (size_t)up.chunks * N * R * 4 : 0);
    p.split_down = take(down.chunks > 1 ? (size_t)down.chunks * K * R * 4 : 0);
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

// The rows in order, and where each adapter's begin.
AdapterRows order_rows(AdapterRows rows, char *ws, const AdapterPlan &p, int32_t *flag, hipStream_t st) {
  int32_t *perm = reinterpret_cast<int32_t *>(ws + p.perm), *sorted = reinterpret_cast<int32_t *>(ws + p.sorted);
  hipLaunchKernelGGL(adapter_order_kernel, dim3((rows.M + rows.n + 64) / 64), dim3(1024), 0, st, rows, perm, sorted,
                     reinterpret_cast<int32_t *>(ws + p.start), flag);
  rows.perm = perm;
  rows.sorted = sorted;
  return rows;
}
template <class F>
void with_r_tiles(int32_t R, F &&f) {
  switch (adapter_r_tiles(R)) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 3: f(std::integral_constant<int, 3>()); break;
    default: f(std::integral_constant<int, 4>());
  }
}
template <typename T>
void launch_inner(const InnerArgs<T> &a, hipStream_t st) {
  const dim3 grid((a.rows.M + ADAPTER_TILE - 1) / ADAPTER_TILE, std::min(ADAPTER_TILE, a.rows.n));
  with_r_tiles(a.R, [&](auto r) { hipLaunchKernelGGL((adapter_inner_kernel<T, decltype(r)::value>), grid, dim3(512), 0, st, a); });
}
template <typename T, int NF, bool PACKED>
void launch_outer_as(OuterArgs<T> a, hipStream_t st) {
  // Columns of a wave, 32 and 64, us, 2560 rows of 64000, 8 adapters: R = 64 fp32 492 and 723 (64 spill), bf16 270 and 218, R = 40
  // 262 and 211; fp32 of 16 < R <= 48 would do better with 64 (R = 32 385 and 324, R = 48 437 and 359).
  constexpr int VT = NF == 1 || sizeof(T) == 2 ? 4 : 2;
  const int64_t cols = (a.N + 64 * VT - 1) / (64 * VT);
  // a wave takes the adapters of its tile one after the other: smaller tiles until there is a workgroup for every compute unit
  const auto tiles = [&]() { return (a.rows.M + a.tile - 1) / a.tile; };
  a.tile = ADAPTER_TILE;
  while (a.tile > 4 && tiles() * cols < 256) a.tile /= 2;
  // and walks over its columns with the next ones requested ahead: one round of as many workgroups as the GPU holds (512, 768 and
  // 1024 of them, us, 2560 rows of 64000: bf16 R = 16 165, 163, 183, R = 64 217, 265, 232, fp32 R = 16 298, 336, 305)
  constexpr int64_t WGS = NF == 1 && sizeof(T) == 2 ? 768 : 512;
  const int64_t side = std::max<int64_t>(1, std::min(cols, WGS / tiles()));
  a.blocks = (int)((cols + side - 1) / side);
  const dim3 grid((unsigned)tiles(), (unsigned)((cols + a.blocks - 1) / a.blocks));
  hipLaunchKernelGGL((adapter_outer_kernel<T, NF, PACKED, VT>), grid, dim3(256), 0, st, a);
}
template <typename T>
void launch_outer(const OuterArgs<T> &a, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (a.R <= 16) launch_outer_as<T, 1, true>(a, st);
    else if (a.R <= 32) launch_outer_as<T, 1, false>(a, st);
    else launch_outer_as<T, 2, false>(a, st);
  } else {
    with_r_tiles(a.R, [&](auto r) { launch_outer_as<T, decltype(r)::value, false>(a, st); });
  }
}
// (Arrays narrower than a wave's columns: one kernel of each type, whatever R.)
template <typename T>
void launch_grad(const GradArgs<T> &a, const GradPlan &p, hipStream_t st) {
  const dim3 grid(p.blocks, p.chunks), threads(64 * ADAPTER_GRAD_WAVES);
  constexpr bool BF16 = sizeof(T) == 2;
  const bool small = adapter_grad_small(a.rows.M, a.N, BF16 ? RNNLM_DTYPE_BF16 : RNNLM_DTYPE_FP32);
  if (a.N < 16 * adapter_grad_tiles(adapter_r_tiles(a.R), BF16, small)) {
    hipLaunchKernelGGL((adapter_grad_kernel<T, 4, 2, true>), grid, threads, 0, st, a);
  } else {
    with_r_tiles(a.R, [&](auto r) {
      constexpr int JT = decltype(r)::value;
      if (small) hipLaunchKernelGGL((adapter_grad_kernel<T, JT, adapter_grad_tiles(JT, BF16, true), false>), grid, threads, 0, st, a);
      else hipLaunchKernelGGL((adapter_grad_kernel<T, JT, adapter_grad_tiles(JT, BF16, false), false>), grid, threads, 0, st, a);
    });
  }
}
template <typename T>
void launch_input_grad(const InputGradArgs<T> &a, const GradPlan &p, hipStream_t st) {
  const dim3 grid(p.blocks, p.chunks), threads(64 * ADAPTER_GRAD_WAVES);
  constexpr bool BF16 = sizeof(T) == 2;
  if (a.K < 16 * adapter_input_tiles(adapter_r_tiles(a.R), BF16)) {
    hipLaunchKernelGGL((adapter_input_grad_kernel<T, 4, 2, true>), grid, threads, 0, st, a);
  } else {
    with_r_tiles(a.R, [&](auto r) {
      constexpr int JT = decltype(r)::value;
      hipLaunchKernelGGL((adapter_input_grad_kernel<T, JT, adapter_input_tiles(JT, BF16), false>), grid, threads, 0, st, a);
    });
  }
}

template <typename T>
int adapter_forward(const T *x, int64_t ldx, int64_t M, int32_t K, int32_t N, const rnnlm_adapters &a, const int32_t *ids, const T *base,
                    int64_t ldb, T *out, int64_t ldo, float *inner, int32_t *flag, char *ws, const AdapterPlan &p, hipStream_t st) {
  AdapterRows rows = {ids, nullptr, nullptr, (int)M, a.n};
  if (M > ADAPTER_UNORDERED * ADAPTER_TILE) {
    rows = order_rows(rows, ws, p, flag, st);
    LAUNCHED();
  }
  if (!inner) inner = reinterpret_cast<float *>(ws + p.inner);
  launch_inner<T>({rows, x, static_cast<const T *>(a.down), ldx, K, a.R, inner, flag}, st);
  LAUNCHED();
  launch_outer<T>({rows, inner, static_cast<const T *>(a.up), a.scale, base, out, ldb, ldo, N, a.R, 1, ADAPTER_TILE}, st);
  LAUNCHED();
  return RNNLM_OK;
}

template <typename T>
int adapter_backward(const T *dout, int64_t ldd, const T *x, int64_t ldx, const float *inner, int64_t M, int32_t K, int32_t N,
                     const rnnlm_adapters &a, const int32_t *ids, float *ddown, float *dup, T *dx, int64_t lddx, int32_t *flag, char *ws,
                     const AdapterPlan &p, hipStream_t st) {
  const int32_t dtype = sizeof(T) == 4 ? RNNLM_DTYPE_FP32 : RNNLM_DTYPE_BF16;
  const int32_t *start = reinterpret_cast<int32_t *>(ws + p.start);
  const auto floats = [&](size_t at) { return reinterpret_cast<float *>(ws + at); };
  const AdapterRows rows = order_rows({ids, nullptr, nullptr, (int)M, a.n}, ws, p, flag, st);
  LAUNCHED();
  const GradPlan up = adapter_up_plan(M, N, a.R, dtype), down = adapter_down_plan(M, K, a.R, dtype);
  if (M > 0) {
    launch_grad<T>({rows, start, dout, ldd, inner, static_cast<const T *>(a.up), a.scale, dup, floats(p.split_up), floats(p.part), N, a.R, up.chunk},
                   up, st);
    LAUNCHED();
    const bool apart = up.blocks > ADAPTER_BLOCKS_INSIDE;
    if (apart) {
      hipLaunchKernelGGL(adapter_blocks_kernel, dim3((unsigned)((M * a.R + 63) / 64)), dim3(1024), 0, st, floats(p.part), up.blocks, (long)M * a.R,
                         floats(p.dinner));
      LAUNCHED();
    }
    launch_input_grad<T>({rows, start, x, static_cast<const T *>(a.down), a.scale, floats(apart ? p.dinner : p.part), ddown, floats(p.split_down), dx,
                          ldx, lddx, K, a.R, down.chunk, apart ? 1 : up.blocks},
                         down, st);
    LAUNCHED();
  }
  const int64_t size = (int64_t)std::max(N, K) * a.R;
  const unsigned ids_y = std::min(a.n, 1024), parts = (unsigned)std::max<int64_t>(1, std::min<int64_t>((size + 1023) / 1024, 1024 / ids_y));
  hipLaunchKernelGGL(adapter_join_kernel, dim3(parts, ids_y, 2), dim3(256), 0, st, start, a.n,
                     JoinArgs{floats(p.split_up), a.scale, dup, (int64_t)N * a.R, up.chunk},
                     JoinArgs{floats(p.split_down), nullptr, ddown, (int64_t)K * a.R, down.chunk});
  LAUNCHED();
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
  return preference_sizes_ok(T, pairs) ? preference_plan(T, pairs).total : 0;
}

int rnnlm_set_preference_wait(int32_t polls) {
  if (polls < 0 || polls > (1 << 20)) return RNNLM_ERR_ARG;  // (calls that share the GPU may wait for one another's rows)
  preference_polls = polls;
  return RNNLM_OK;
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
  const PreferencePlan p = preference_plan(T, pairs);
  char *ws = static_cast<char *>(workspace);
  const auto call = [&](auto rows_of) {
    typedef std::remove_const_t<std::remove_pointer_t<decltype(rows_of.z)>> E;
    return preference_call<E>({rows_of, ref, weight, loss, logp, T, pairs, kind, mean != 0, beta, smoothing, scale,
                               reinterpret_cast<PreferenceRow *>(ws + p.row), reinterpret_cast<PreferencePair *>(ws + p.pair),
                               reinterpret_cast<unsigned long long *>(ws + p.published), reinterpret_cast<int *>(ws + p.done), preference_polls.load()},
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
