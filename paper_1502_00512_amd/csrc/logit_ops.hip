// Host side of the operators on arrays of logits (include/rnnlm.h, "Logits"): checks of arguments, choice of kernel, launches.
#include "call_checks.h"
#include "distill.h"
#include "top_logits.h"
#include "verify.h"

using namespace rnnlm_dev;

namespace {

// ---- top logits ----
struct TopPlan {
  int chunks, per, threads, nv;
};
// A workgroup holds THREADS x NV slots of a row.  The measured calls: bf16, K = 64 unless said.
// Up to 4096 slots 256 threads, with as few slots each as hold the row.  Up to 10240 one workgroup of 512, no second launch: 64000
// words, 1 row 9.4 us against 12.5 in chunks, 256 rows 14.0 and 20.3, 2560 rows 66 and 76.  Up to 20480 one of 1024, where the rows
// are no more than the compute units or the lists long.  100000 words, that and chunks: K = 200, 1 row 16.2 and 23.6, 256 rows 21.7
// and 38.5, 2560 rows 178 and 212; K = 64, 1 row 11.7 and 14.5, 256 rows 17.6 and 25.4; K = 16, 128 rows 14.9 and 15.9, 256 rows
// 18.0 and 19.9, but 512 rows 32.8 and 28.6, 2560 rows 142 and 95 (one such workgroup on a compute unit: nothing runs while it
// waits).  Short lists of few rows pay for it: K = 16, 1 to 64 rows 12.6 to 14.1 and 12.3 to 12.5, K = 3 15.2 to 15.8 and 12.3
// to 12.7 (50000 fp32 words, K = 3 and 16, do not: 10.0 to 13.3 and 12.0 to 16.2).  (The widest of these kernels keeps 10 (fp32)
// or 13 (bf16) registers of a thread in scratch.)
// Else chunks of 4096 slots.  Half or a quarter as many, until the workgroups are as many as the compute units, gain nothing: 4 rows of
// 200000 words 16.1 us and 16.3 whole, of 400000 words (K = 16) 15.6 and 12.9, one of 1000000 (K = 3) 16.3 and 13.2.
TopPlan top_plan(int64_t rows, int32_t V, int32_t K, int32_t dtype) {
  const int slots = slots_of(V, dtype);
  TopPlan p;
  p.threads = 256;
  p.nv = 16;
  auto chunks = [&]() { return (slots + p.nv * p.threads - 1) / (p.nv * p.threads); };
  if (chunks() == 1) {
    while (p.nv > 1 && p.nv / 2 * p.threads >= slots) p.nv /= 2;
  } else if (slots <= TOP_WIDE * 20) {
    p.threads = TOP_WIDE;
    if (slots > TOP_WIDE * 16) p.nv = 20;
  } else if (slots <= TOP_WIDEST * 20 && (rows <= 256 || K > TOP_COUNTED)) {
    p.threads = TOP_WIDEST;
    if (slots > TOP_WIDEST * 16) p.nv = 20;
  }
  p.chunks = chunks();
  p.per = (slots + p.chunks - 1) / p.chunks;
  p.chunks = (slots + p.per - 1) / p.per;
  return p;
}
size_t top_bytes(const TopPlan &p, int64_t rows, int32_t K) {
  if (p.chunks == 1) return 0;
  return align256((size_t)rows * p.chunks * K * 8) + align256((size_t)rows * p.chunks * 16);
}
bool top_sizes_ok(int64_t rows, int32_t V, int32_t K, int32_t dtype) {
  if (rows < 0 || rows > ROWS_MAX || V < 1 || V > TOP_V_MAX || K < 1 || K > std::min(V, TOP_K_MAX)) return false;
  if (dtype != RNNLM_DTYPE_FP32 && dtype != RNNLM_DTYPE_BF16) return false;
  const TopPlan p = top_plan(rows, V, K, dtype);
  return rows * p.chunks * p.threads <= THREADS_MAX;
}
template <typename T, int THREADS, int NV>
void launch_top_chunks(const TopArgs &a, int64_t rows, hipStream_t st) {
  hipLaunchKernelGGL((top_chunk_kernel<T, THREADS, NV>), dim3((unsigned)(rows * a.chunks)), dim3(THREADS), 0, st, a);
}
template <typename T>
void launch_top(const TopArgs &a, int64_t rows, const TopPlan &p, hipStream_t st) {
  if (p.threads == TOP_WIDEST && p.nv == 20) launch_top_chunks<T, TOP_WIDEST, 20>(a, rows, st);
  else if (p.threads == TOP_WIDEST) launch_top_chunks<T, TOP_WIDEST, 16>(a, rows, st);
  else if (p.threads == TOP_WIDE && p.nv == 20) launch_top_chunks<T, TOP_WIDE, 20>(a, rows, st);
  else if (p.threads == TOP_WIDE) launch_top_chunks<T, TOP_WIDE, 16>(a, rows, st);
  else if (p.nv == 1) launch_top_chunks<T, 256, 1>(a, rows, st);
  else if (p.nv == 2) launch_top_chunks<T, 256, 2>(a, rows, st);
  else if (p.nv == 4) launch_top_chunks<T, 256, 4>(a, rows, st);
  else if (p.nv == 8) launch_top_chunks<T, 256, 8>(a, rows, st);
  else launch_top_chunks<T, 256, 16>(a, rows, st);
}

// ---- distillation ----
template <typename T, int THREADS, int NV, int MODE>
void launch_distill_row(const DistillArgs<T> &a, int64_t rows, hipStream_t st) {
  hipLaunchKernelGGL((distill_row_kernel<T, THREADS, NV, MODE>), dim3((unsigned)rows), dim3(THREADS),
                     distill_lds(a.K), st, a);
}
template <typename T, int MODE>
void launch_distill(const DistillArgs<T> &a, int64_t rows, hipStream_t st) {
  const int slots = a.V / SlotOf<T>::N;  // whole ones: what a thread's registers hold
  // Many short rows: a wave each, four times as many in flight (a row's time is the latency of its steps, not its bytes): bf16,
  // K = 40, 6000 rows of 1000 words 14.0 us and 19.6 with four waves each, of 3000 words 21.9 and 24.1; 512 to 2048 rows 11 either
  // way.
  const bool wave_each = rows >= 1024 && slots <= 64 * 8;
  if (!a.dz || slots > 1024 * 25) {
    hipLaunchKernelGGL((distill_stream_kernel<T, 512, MODE>), dim3((unsigned)rows), dim3(512), distill_lds(a.K), st, a);
  } else if (wave_each && slots <= 64 * 2) {
    launch_distill_row<T, 64, 2, MODE>(a, rows, st);
  } else if (wave_each && slots <= 64 * 4) {
    launch_distill_row<T, 64, 4, MODE>(a, rows, st);
  } else if (wave_each) {
    launch_distill_row<T, 64, 8, MODE>(a, rows, st);
  } else if (slots <= 256) {
    launch_distill_row<T, 256, 1, MODE>(a, rows, st);
  } else if (slots <= 256 * 2) {
    launch_distill_row<T, 256, 2, MODE>(a, rows, st);
  } else if (slots <= 256 * 4) {
    launch_distill_row<T, 256, 4, MODE>(a, rows, st);
  } else if (slots <= 256 * 6) {
    launch_distill_row<T, 256, 6, MODE>(a, rows, st);
  } else if (slots <= 256 * 8) {
    launch_distill_row<T, 256, 8, MODE>(a, rows, st);
  } else if (slots <= 512 * 6) {
    launch_distill_row<T, 512, 6, MODE>(a, rows, st);
  } else if (slots <= 512 * 8) {
    launch_distill_row<T, 512, 8, MODE>(a, rows, st);
  } else if (slots <= 512 * 12) {
    launch_distill_row<T, 512, 12, MODE>(a, rows, st);
  } else if (slots <= 512 * 16) {
    launch_distill_row<T, 512, 16, MODE>(a, rows, st);
  } else if (slots <= 512 * 20) {
    launch_distill_row<T, 512, 20, MODE>(a, rows, st);
  } else if (slots <= 512 * 25) {
    launch_distill_row<T, 512, 25, MODE>(a, rows, st);
  } else if (slots <= 1024 * 18) {
    launch_distill_row<T, 1024, 18, MODE>(a, rows, st);
  } else {
    launch_distill_row<T, 1024, 25, MODE>(a, rows, st);
  }
}
template <typename T>
int distill_call(DistillArgs<T> a, int64_t rows, hipStream_t st) {
  if (!a.y || a.alpha == 1.0f || a.tau == 1.0f) launch_distill<T, DISTILL_ONE>(a, rows, st);
  else if (a.tau == 2.0f) launch_distill<T, DISTILL_SQUARE>(a, rows, st);
  else launch_distill<T, DISTILL_TWO>(a, rows, st);
  LAUNCHED();
  return RNNLM_OK;
}

// ---- verification ----
struct VerifyPlan {
  int parts, chunks;
  size_t stat, sums, rest, seq, total;
};
int verify_blocks(int32_t V, int32_t dtype) { return (slots_of(V, dtype) + 63) / 64; }
VerifyPlan verify_plan(int32_t K, int32_t B, int32_t V) {
  VerifyPlan p;
  const int slots = slots_of(V, RNNLM_DTYPE_BF16);  // (fp32 rows have twice as many: parts of twice the slots)
  // Parts of a row until there are 8192 workgroups (4096 and 16384: the same within 2 us for 128 texts x 4 drafts over 100000
  // words); shares of a text until there are 4096 (2048 and 8192 in place of it: as fast or slower).
  const int64_t rows = (int64_t)(2 * K + 1) * B, fill = 8192;
  p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({fill / std::min(rows, fill), VERIFY_PARTS, slots / VERIFY_THREADS}));
  p.chunks = (int)std::max<int64_t>(1, std::min<int64_t>({4096 / std::min<int64_t>(B, 4096), VERIFY_PARTS, slots / VERIFY_THREADS}));
  size_t o = 0;
  auto take = [&](size_t n) {
    const size_t at = o;
    o = align256(o + n);
    return at;
  };
  p.stat = take((size_t)rows * p.parts * 8);
  p.sums = take((size_t)B * p.chunks * 16);
  p.rest = take((size_t)B * verify_blocks(V, RNNLM_DTYPE_FP32) * 8);
  p.seq = take((size_t)B * sizeof(VerifySeq));
  p.total = o;
  return p;
}
bool verify_sizes_ok(int32_t K, int32_t B, int32_t V) {
  return K >= 0 && K <= 1024 && B >= 1 && B <= (1 << 20) && V >= 1 && V <= TOP_V_MAX &&
         (int64_t)(2 * K + 1) * B <= ROWS_MAX;
}
template <typename T>
int verify_call(const VerifyArgs &a, hipStream_t st) {
  const dim3 threads(VERIFY_THREADS);
  const int64_t rows = (int64_t)(a.draft ? 2 * a.K + 1 : a.K + 1) * a.B;
  hipLaunchKernelGGL(verify_stats_kernel<T>, dim3((unsigned)(rows * a.parts)), threads, 0, st, a);
  const dim3 shares((unsigned)(a.B * a.chunks));
  if (a.blocks <= (a.draft ? VERIFY_ONE_BLOCKS / 2 : VERIFY_ONE_BLOCKS)) {
    hipLaunchKernelGGL(verify_one_kernel<T>, dim3((unsigned)a.B), dim3(VERIFY_ONE_THREADS), 0, st, a);
  } else if (shares.x <= VERIFY_DECIDE_INSIDE && a.draft) {
    hipLaunchKernelGGL((verify_sums_kernel<T, true>), shares, threads, 0, st, a);
    hipLaunchKernelGGL((verify_rest_kernel<T, false>), shares, threads, 0, st, a);
  } else if (shares.x <= VERIFY_DECIDE_INSIDE) {
    hipLaunchKernelGGL((verify_rest_kernel<T, true>), shares, threads, 0, st, a);
  } else {
    hipLaunchKernelGGL(verify_decide_kernel<T>, dim3((unsigned)a.B), dim3(VERIFY_DECIDE_THREADS), 0, st, a);
    if (a.draft) hipLaunchKernelGGL((verify_sums_kernel<T, false>), shares, threads, 0, st, a);
    hipLaunchKernelGGL((verify_rest_kernel<T, false>), shares, threads, 0, st, a);
  }
  LAUNCHED();
  return RNNLM_OK;
}

}  // namespace

extern "C" {

size_t rnnlm_top_logits_workspace_bytes(int64_t rows, int32_t V, int32_t K, int32_t dtype) {
  return top_sizes_ok(rows, V, K, dtype) ? std::max<size_t>(256, top_bytes(top_plan(rows, V, K, dtype), rows, K)) : 0;
}

int rnnlm_top_logits(const void *logits, int32_t dtype, int64_t rows, int32_t V, int64_t ld, int32_t K, float tau,
                     int32_t *ids, float *vals, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
  if (!top_sizes_ok(rows, V, K, dtype) || !rows_ok(logits, dtype, rows, V, ld) || !tau_ok(tau) || (rows > 0 && (!ids || !vals)))
    return RNNLM_ERR_ARG;
  if (!aligned(ids, 4) || !aligned(vals, 4) || !aligned(lse, 4)) return RNNLM_ERR_ARG;
  const TopPlan p = top_plan(rows, V, K, dtype);
  const size_t need = top_bytes(p, rows, K);
  if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return RNNLM_ERR_ARG;
  if (rows == 0) return RNNLM_OK;
  TopArgs a = {};
  a.z = logits;
  a.ld = ld;
  a.V = V;
  a.K = K;
  a.chunks = p.chunks;
  a.per = p.per;
  a.tau = tau;
  a.ids = ids;
  a.vals = vals;
  a.lse = lse;
  a.once = read_once(rows, V, dtype);
  if (need) {
    a.part = static_cast<unsigned long long *>(workspace);
    a.stat = reinterpret_cast<double2 *>(static_cast<char *>(workspace) + align256((size_t)rows * p.chunks * K * 8));
  }
  hipStream_t st = (hipStream_t)stream;
  if (dtype == RNNLM_DTYPE_FP32) launch_top<float>(a, rows, p, st);
  else launch_top<bf16_t>(a, rows, p, st);
  LAUNCHED();
  if (p.chunks > 1) {
    hipLaunchKernelGGL(top_merge_kernel, dim3((unsigned)rows), dim3(TOP_MERGE_THREADS), 0, st, a);
    LAUNCHED();
  }
  return RNNLM_OK;
}

int rnnlm_distill_loss(const void *logits, int32_t dtype, int64_t rows, int32_t V, int64_t ld, const int32_t *ids,
                       const float *vals, int32_t K, const float *lse, const int32_t *y, const float *weight, float tau,
                       float alpha, float scale, float *loss, double *sum_loss, void *dlogits, int64_t ld_dlogits,
                       int32_t *range_flag, void *stream) {
  if (!rows_ok(logits, dtype, rows, V, ld) || (rows > 0 && (!ids || !vals || !loss || (alpha < 1.0f && !y))) || K < 1 || K > 1024 || !tau_ok(tau) ||
      !(alpha >= 0.0f && alpha <= 1.0f) || !std::isfinite(scale))
    return RNNLM_ERR_ARG;
  if (!aligned(ids, 4) || !aligned(vals, 4) || !aligned(lse, 4) || !aligned(y, 4) || !aligned(weight, 4) ||
      !aligned(loss, 4) || !aligned(sum_loss, 8) || !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  const size_t es = elem_bytes(dtype);
  const bool once = read_once(rows, V, dtype);
  const double inv_tau = 1.0 / (double)tau;
  if (dlogits) {
    if (!rows_ok(dlogits, dtype, rows, V, ld_dlogits)) return RNNLM_ERR_ARG;
    // in place row by row, or apart
    if (dlogits == logits ? ld != ld_dlogits
                          : rows > 0 && meet(span(logits, ((size_t)(rows - 1) * ld + V) * es),
                                             span(dlogits, ((size_t)(rows - 1) * ld_dlogits + V) * es)))
      return RNNLM_ERR_ARG;
  }
  hipStream_t st = (hipStream_t)stream;
  if (rows > 0) {
    int rc;
    if (dtype == RNNLM_DTYPE_FP32) {
      rc = distill_call(DistillArgs<float>{static_cast<const float *>(logits), ld, static_cast<float *>(dlogits), ld_dlogits, ids, y,
                                           vals, lse, weight, loss, range_flag, tau, alpha, scale, V, K, once, inv_tau},
                        rows, st);
    } else {
      rc = distill_call(DistillArgs<bf16_t>{static_cast<const bf16_t *>(logits), ld, static_cast<bf16_t *>(dlogits), ld_dlogits,
                                            ids, y, vals, lse, weight, loss, range_flag, tau, alpha, scale, V, K, once, inv_tau},
                        rows, st);
    }
    if (rc) return rc;
  }
  if (sum_loss) {
    hipLaunchKernelGGL(sum_losses_kernel, dim3(1), dim3(1024), 0, st, loss, (long)rows, sum_loss);
    LAUNCHED();
  }
  return RNNLM_OK;
}

size_t rnnlm_verify_workspace_bytes(int32_t K, int32_t B, int32_t V) {
  return verify_sizes_ok(K, B, V) ? verify_plan(K, B, V).total : 0;
}

int rnnlm_verify_drafts(const void *target, int64_t ld_target, const void *draft, int64_t ld_draft, int32_t dtype, int32_t K,
                        int32_t B, int32_t V, const int32_t *drafts, const int32_t *lengths, const float *u, float tau,
                        float tau_draft, int32_t *accepted, int32_t *tokens, int32_t *range_flag, void *workspace,
                        size_t workspace_bytes, void *stream) {
  if (!verify_sizes_ok(K, B, V) || !rows_ok(target, dtype, (int64_t)(K + 1) * B, V, ld_target) || !u || !accepted || !tokens ||
      (K > 0 && !drafts) || !tau_ok(tau) || !tau_ok(tau_draft))
    return RNNLM_ERR_ARG;
  if (K == 0) draft = nullptr;
  if (draft && !rows_ok(draft, dtype, (int64_t)K * B, V, ld_draft)) return RNNLM_ERR_ARG;
  if (!aligned(drafts, 4) || !aligned(lengths, 4) || !aligned(u, 4) || !aligned(accepted, 4) || !aligned(tokens, 4) ||
      !aligned(range_flag, 4))
    return RNNLM_ERR_ARG;
  const VerifyPlan p = verify_plan(K, B, V);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < p.total) return RNNLM_ERR_ARG;
  char *ws = static_cast<char *>(workspace);
  VerifyArgs a = {};
  a.target = target;
  a.draft = draft;
  a.ldt = ld_target;
  a.ldd = ld_draft;
  a.drafts = drafts;
  a.lengths = lengths;
  a.u = u;
  a.V = V;
  a.B = B;
  a.K = K;
  a.parts = p.parts;
  a.per = (slots_of(V, dtype) + p.parts - 1) / p.parts;
  a.blocks = verify_blocks(V, dtype);
  // whole rounds of a workgroup's waves
  const int waves = VERIFY_THREADS / 64;
  a.span = (a.blocks + p.chunks * waves - 1) / (p.chunks * waves) * waves;
  a.chunks = (a.blocks + a.span - 1) / a.span;
  a.tau = tau;
  a.tau_d = tau_draft;
  a.accepted = accepted;
  a.tokens = tokens;
  a.range_flag = range_flag;
  a.stat = reinterpret_cast<float2 *>(ws + p.stat);
  a.sums = reinterpret_cast<double *>(ws + p.sums);
  a.rest = reinterpret_cast<double *>(ws + p.rest);
  a.seq = reinterpret_cast<VerifySeq *>(ws + p.seq);
  hipStream_t st = (hipStream_t)stream;
  return dtype == RNNLM_DTYPE_FP32 ? verify_call<float>(a, st) : verify_call<bf16_t>(a, st);
}

}  // extern "C"
