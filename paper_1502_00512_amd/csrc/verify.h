// Verification of drafted words against a target model's distribution, from given random numbers.
//   p_i = softmax(target_i / tau),  q_i = softmax(draft_i / tau_d)  (no draft logits: q_i has all its mass on the draft d_i)
//   draft i is accepted iff u_i q_i(d_i) < p_i(d_i); n = drafts accepted before the first that is not
//   the word after them is drawn from r = max(p_n - q_n, 0) (all of the text's drafts accepted, or r = 0: r = p_n): the first
//   v with sum_{j <= v} r_j > u_K sum_j r_j
// Which step of a sum over the vocabulary a random number falls on depends on every term: 100000 terms of 32 bits leave the
// step open once in some hundred words, so the drawn word's row is summed in 64 bits with exponentials to 1e-14 (where p and q are
// not equal and yet agree to that altogether, r is rounding: a draft from q is rejected there once in 1e13).  The
// acceptance of a draft compares two probabilities and gets by with 32-bit sums.
//   1. maximum and sum of exponentials of every row that can matter, by parts of a row (HBM-bound; all the bytes are here)
//   2. how many drafts are accepted
//   3. sums of exponentials of the row pair of a text that is drawn from p - q, in 64 bits (p alone needs no sum: r may have any
//      common factor)
//   4. sums of r by blocks of one slot a lane, and by the last workgroup of a text to finish: the block on which u_K falls, and
//      the word in it
// 128 texts of up to 5 drafts over 100000 bf16 words take 34, 5, 15 and 30 us (rows behind a text's drafts are left out: 154 of 282 MB
// read), 37 without draft logits over 33278 fp32 words 6 and 10 (2 inside of 4).
// Short rows do 2 to 4 in one workgroup a text.  Steps 3 and 4 are bound by 64-bit instructions (some 23 an exponential); texts
// differ in what they need, so they are cut fine (a chunk is a few blocks) and every workgroup knows at once whether it has
// anything to do: with step 2 inside step 3 and eight chunks a text, 128 texts over 100000 words took 26 and 31 us in the two.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int VERIFY_THREADS = 256, VERIFY_PARTS = 64;
constexpr int VERIFY_DECIDE_THREADS = 512;  // a wave to each of up to eight rows
constexpr int VERIFY_STAGED = 1024;  // sums of blocks that the drawing workgroup holds in LDS
// A text in one workgroup: rows of at most so many blocks, half as many where there is a draft row (two passes over two rows).
// In one workgroup and in shares: 15 texts x 4 drafts over 22650 words 31 and 22 us, over 13250 words 23 and 23.
constexpr int VERIFY_ONE_THREADS = 1024, VERIFY_ONE_BLOCKS = 64;
// Up to so many workgroups, all at work at once, step 2 is part of the next: it takes them less than its launch does (4 drafts over
// 64000 words: 32 texts 36.0 us and 37.9 with a launch of its own, 256 texts 116.9 and 111.7).
constexpr int VERIFY_DECIDE_INSIDE = 1024;

struct VerifySeq {  // what the steps behind the second one know of a text
  int n;            // accepted
  int mixed;        // the drawn row is p - q (else p alone)
  float mp, mq;     // maxima of the drawn rows
  int ok;           // they are numbers, and p has any
  unsigned done;    // workgroups of the last step that have finished
};

struct VerifyArgs {
  const void *target, *draft;  // draft may be nullptr
  long ldt, ldd;
  const int32_t *drafts, *lengths;  // lengths may be nullptr
  const float *u;
  int V, B, K, parts, per;    // parts of a row in the first step; slots of each
  int chunks, blocks, span;   // workgroups of a text in the others; blocks of a row; blocks of each workgroup
  float tau, tau_d;
  int32_t *accepted, *tokens, *range_flag;
  float2 *stat;    // [row][part], rows of the target then of the draft
  double *sums;    // [text][chunk][2]: sums of exponentials of p, q
  double *rest;    // [text][block]: sums of r
  VerifySeq *seq;  // [text]
};

__device__ inline int draft_length(const VerifyArgs &a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.K) : a.K;
}

// e^{(z - m) / tau} of a row in 64 bits, up to a factor that the row has in common: 2^x, x = z c + b = n + f with |f| <= 1/2,
// and the polynomial of degree 9 that meets 2^f at the ten Chebyshev nodes of [-1/2, 1/2]: 1.8e-14 relative off at most, so a
// hundred thousand such terms place a step of their sum to about 1e-14.  (b = -m c is rounded: the common factor.)  n is what
// adding 1.5 * 2^52 leaves in the low word; 2^n goes into the exponent by an integer addition, which holds down to n = -1022.
// Logits more than some 690 tau (never 700) below the maximum, and masked ones, give 0.  Where m c passes 2^50 only logits equal to
// the maximum are as near: e = 1.  No NaNs: the caller knows the row.
struct Exp64 {
  double c, b;
  float least;
  __device__ Exp64(float m, float tau) {
    if (m == -INFINITY) m = 0.0f;
    c = LOG2E_64 / (double)tau;
    b = -(double)m * c;
    if (fabs(b) > 1125899906842624.0) c = b = 0.0;
    least = m - 690.0f * tau;
    if ((double)m - (double)least > 700.0 * (double)tau) least = nextafterf(least, m);  // (a step of m's size may be many tau)
  }
  __device__ double operator()(float z) const {
    constexpr double SHIFT = 6755399441055744.0;
    const double x = fma((double)z, c, b), t = x + SHIFT, f = x - (t - SHIFT);
    double p = 1.0205905413765595e-07;
    p = fma(p, f, 1.325964524488711e-06);
    p = fma(p, f, 1.5252672924850737e-05);
    p = fma(p, f, 0.0001540343375125101);
    p = fma(p, f, 0.0013333558200794592);
    p = fma(p, f, 0.009618129193934313);
    p = fma(p, f, 0.05550410866465167);
    p = fma(p, f, 0.2402265069564034);
    p = fma(p, f, 0.6931471805599462);
    p = fma(p, f, 1.0000000000000135);
    const unsigned hi = (unsigned)__double2hiint(p) + ((unsigned)__double2loint(t) << 20);
    const double e = __hiloint2double((int)hi, __double2loint(p));
    return z >= least ? e : 0.0;
  }
};

template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_stats_kernel(const VerifyArgs a) {
  constexpr int N = SlotOf<T>::N, WAVES = VERIFY_THREADS / 64, FLIGHT = 4;
  __shared__ float sh_m[WAVES], sh_s[WAVES];
  const int r = blockIdx.x / a.parts, part = blockIdx.x % a.parts, targets = (a.K + 1) * a.B;
  const bool is_draft = r >= targets;
  const int row = is_draft ? r - targets : r, i = row / a.B, b = row % a.B, len = draft_length(a, b);
  if (r < a.B && part == 0 && threadIdx.x == 0) a.seq[r].done = 0;
  if (is_draft ? i >= len : i > len) return;  // a row behind the text's drafts
  const T *z = is_draft ? static_cast<const T *>(a.draft) + row * a.ldd : static_cast<const T *>(a.target) + row * a.ldt;
  const int first = part * a.per, last = min(first + a.per, a.V / N);
  const float c = LOG2E / (is_draft ? a.tau_d : a.tau);
  const float zt = part == a.parts - 1 ? tail_elem(z, threadIdx.x, a.V) : -INFINITY;  // the last part has the row's last elements
  float mx = zt, s = zt == -INFINITY ? 0.0f : 1.0f;
  for (int j0 = first + threadIdx.x; j0 < last; j0 += FLIGHT * VERIFY_THREADS) {
    slot_t raw[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      const int j = j0 + k * VERIFY_THREADS;
      raw[k] = j < last ? load_slot(z, j) : empty_slot<T>();
    }
    float top = mx;
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) top = slot_max<T>(top, raw[k]);
    const float base = top == -INFINITY ? 0.0f : top;
    if (top > mx) {
      s *= exp2_32((mx - base) * c);
      mx = top;
    }
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k)
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_32((slot_elem<T>(raw[k], e) - base) * c);
  }
  const float own = mx;
  mx = wave_max(mx);
  float base = mx == -INFINITY ? 0.0f : mx;
  s = wave_sum(s * exp2_32((own - base) * c));
  if ((threadIdx.x & 63) == 0) {
    sh_m[threadIdx.x >> 6] = mx;
    sh_s[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < WAVES; ++k) mx = fmaxf(mx, sh_m[k]);
    base = mx == -INFINITY ? 0.0f : mx;
    s = 0.0f;
    for (int k = 0; k < WAVES; ++k) s += sh_s[k] * exp2_32((sh_m[k] - base) * c);
    a.stat[(long)r * a.parts + part] = make_float2(mx, s);
  }
}

// Maximum and sum of row r, by one wave.
__device__ inline float2 verify_row(const VerifyArgs &a, long r, float tau) {
  const int lane = threadIdx.x & 63;
  const float c = LOG2E / tau;
  const float2 q = lane < a.parts ? a.stat[r * a.parts + lane] : make_float2(-INFINITY, 0.0f);
  const float m = wave_max(q.x), base = m == -INFINITY ? 0.0f : m;
  return make_float2(m, wave_sum(q.y * exp2_32((q.x - base) * c)));
}

template <typename T>
__device__ inline const T *verify_target(const VerifyArgs &a, int i, int b) {
  return static_cast<const T *>(a.target) + ((long)i * a.B + b) * a.ldt;
}
template <typename T>
__device__ inline const T *verify_draft(const VerifyArgs &a, int i, int b) {
  return static_cast<const T *>(a.draft) + ((long)i * a.B + b) * a.ldd;
}

// How many drafts of text b are accepted: a wave to each row, all loads but the drafts' own logits at once (what is read of
// rows behind the text's drafts was never written, and counts for nothing).  All threads of the workgroup take part.
template <typename T, int THREADS>
__device__ inline VerifySeq verify_decide(const VerifyArgs &a, int b) {
  constexpr int WAVES = THREADS / 64, KEPT = 2 * WAVES;
  __shared__ float4 sh_row[KEPT];  // maximum and sum of p, of q
  __shared__ int sh_reject[WAVES];
  const int len = draft_length(a, b), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int reject = INT32_MAX;
  for (int i = wave; i <= a.K; i += WAVES) {
    const long at = (long)i * a.B + b;
    const bool drafted = i < a.K;
    const int d = drafted ? a.drafts[at] : 0;
    const bool in_range = d >= 0 && d < a.V;
    float zp = 0.0f, zq = 0.0f;
    if (drafted && in_range) {
      zp = to_f32(verify_target<T>(a, i, b)[d]);
      if (a.draft) zq = to_f32(verify_draft<T>(a, i, b)[d]);
    }
    const float2 p = verify_row(a, at, a.tau);
    const float2 q = drafted && a.draft ? verify_row(a, (long)(a.K + 1) * a.B + at, a.tau_d) : make_float2(-INFINITY, 0.0f);
    if (i < KEPT && (threadIdx.x & 63) == 0) sh_row[i] = make_float4(p.x, p.y, q.x, q.y);
    if (i >= len) continue;
    bool accept = false;
    if (in_range) {
      const double pd = exp(((double)zp - (double)p.x) / (double)a.tau) / (double)p.y;
      const double qd = !a.draft ? 1.0 : q.y == 0.0f ? 0.0 : exp(((double)zq - (double)q.x) / (double)a.tau_d) / (double)q.y;
      accept = (double)a.u[at] * qd < pd;  // (false where one is a NaN)
    } else if (a.range_flag) {
      *a.range_flag = 1;
    }
    if (!accept) reject = min(reject, i);
  }
  if ((threadIdx.x & 63) == 0) sh_reject[wave] = reject;
  __syncthreads();
  VerifySeq s = {};
  s.n = min(len, group_reduce<WAVES>(sh_reject[threadIdx.x & (WAVES - 1)], [](int x, int y) { return min(x, y); }));
  s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.mixed = s.n < len;
  if (s.n >= KEPT) {
    const long at = (long)s.n * a.B + b;
    const float2 p = verify_row(a, at, a.tau), q = s.mixed && a.draft ? verify_row(a, (long)(a.K + 1) * a.B + at, a.tau_d) : make_float2(-INFINITY, 0.0f);
    if (threadIdx.x == 0) sh_row[0] = make_float4(p.x, p.y, q.x, q.y);
    __syncthreads();
  }
  const float4 row = sh_row[s.n < KEPT ? s.n : 0];
  s.mp = row.x;
  s.mq = row.z;
  s.ok = row.y > 0.0f && row.y - row.y == 0.0f && (!s.mixed || row.w - row.w == 0.0f);
  return s;
}

template <int THREADS>
__device__ inline double block_sum(double v) {
  __shared__ double sh[THREADS / 64];
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) v += sh[i];
  return v;
}

// r of the drawn row pair of a text, and sums over it.  A block is one slot of each lane of a wave.
template <typename T>
struct Rest {
  static constexpr int N = SlotOf<T>::N;
  const T *p, *q;  // q: nullptr where p is drawn from alone
  Exp64 ep, eq;
  double sp = 1.0, sq = 1.0;  // 1 / the sums of exponentials
  int V, drop;                // drop: a word without mass (the rejected draft of a text without draft logits), or -1
  __device__ Rest(const VerifyArgs &a, int b, const VerifySeq &s)
      : p(verify_target<T>(a, s.n, b)), q(nullptr), ep(s.mp, a.tau), eq(s.mq, a.tau_d), V(a.V), drop(-1) {
    if (!s.mixed) return;
    if (a.draft) q = verify_draft<T>(a, s.n, b);
    else drop = a.drafts[(long)s.n * a.B + b];
  }
  // p alone is drawn from as it is: r may have any common factor.
  __device__ void normalise(double Sp, double Sq) {
    sp = 1.0 / Sp;
    sq = Sq == 0.0 ? 0.0 : 1.0 / Sq;  // (a draft row of nothing but masked words has no mass anywhere)
  }
  __device__ void alone() {
    q = nullptr;
    drop = -1;
  }
  struct Block {
    slot_t p, q;
  };
  // This lane's slots of block k, both loads at once.
  __device__ __forceinline__ Block load(int k) const {
    const int j = k * 64 + (threadIdx.x & 63);
    Block o;
    o.q = empty_slot<T>();
    if ((k + 1) * 64 * N <= V) {
      o.p = load_slot(p, j);
      if (q) o.q = load_slot(q, j);
    } else {
      o.p = load_any_slot(p, j, V);
      if (q) o.q = load_any_slot(q, j, V);
    }
    return o;
  }
  // Calls f(k, block) for blocks first, first + step, ... < last, the next one's loads ahead of it.
  template <class F>
  __device__ __forceinline__ void each(int first, int last, int step, F &&f) const {
    if (first >= last) return;
    Block next = load(first);
    for (int k = first; k < last; k += step) {
      const Block now = next;
      if (k + step < last) next = load(k + step);
      f(k, now);
    }
  }
  // This lane's r in block k; returns their sum.
  __device__ __forceinline__ double rest(int k, const Block &o, double (&r)[N]) const {
#pragma clang fp contract(off)  // equal probabilities leave 0: both products are rounded
    const int v0 = (k * 64 + (threadIdx.x & 63)) * N;
    double sum = 0.0;
    if (q) {
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = fmax(ep(slot_elem<T>(o.p, e)) * sp - eq(slot_elem<T>(o.q, e)) * sq, 0.0);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = v0 + e == drop ? 0.0 : ep(slot_elem<T>(o.p, e)) * sp;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sum += r[e];
    return sum;
  }
};

// The word on which goal falls in block k, `before` it the sum of the blocks in front of it; by one wave.  Where rounding
// lets no word's sum pass the goal: the block's last word with any mass (-1: it has none).
template <typename T>
__device__ inline int word_of_block(const Rest<T> &rest, int k, double before, double goal) {
  constexpr int N = SlotOf<T>::N;
  const int lane = threadIdx.x & 63;
  double r[N];
  const double mine = rest.rest(k, rest.load(k), r);
  const double upto = wave_scan(mine);
  double c = before + (upto - mine);
  int found = INT32_MAX, last = -1;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    c += r[e];
    const int v = (k * 64 + lane) * N + e;
    if (r[e] > 0.0) {
      last = v;
      if (c > goal && found == INT32_MAX) found = v;
    }
  }
  found = wave_reduce(found, [](int x, int y) { return min(x, y); });
  last = wave_reduce(last, [](int x, int y) { return max(x, y); });
  return found == INT32_MAX ? last : found;
}

// The first block whose sums up to it pass u times the whole, by one wave.  Returns the block, or the last with any mass
// where rounding lets none pass, or -1; before: the sum in front of it; total = 0: there is no mass.
template <class Load>
__device__ inline int block_of_number(int blocks, double u, Load &&load, double &before, double &goal, double &total) {
  const int lane = threadIdx.x & 63, stretch = (blocks + 63) / 64, k0 = min(lane * stretch, blocks), k1 = min(k0 + stretch, blocks);
  double mine = 0.0;
  for (int k = k0; k < k1; ++k) mine += load(k);
  const double upto = wave_scan(mine), from = upto - mine;
  total = lane_value(upto, 63);
  goal = u * total;
  double c = from, in_front = 0.0, last_front = 0.0;
  int found = INT32_MAX, last = -1;
  for (int k = k0; k < k1; ++k) {
    const double s = load(k);
    if (s > 0.0) {
      last = k;
      last_front = c;
      if (c + s > goal && found == INT32_MAX) {
        found = k;
        in_front = c;
      }
    }
    c += s;
  }
  const int first = wave_reduce(found, [](int x, int y) { return min(x, y); });
  const int end = wave_reduce(last, [](int x, int y) { return max(x, y); });
  const int k = first != INT32_MAX ? first : end;
  before = 0.0;
  if (k >= 0) before = lane_value(first != INT32_MAX ? in_front : last_front, __builtin_amdgcn_readfirstlane(k / stretch));
  return k;
}

__device__ inline void verify_store(const VerifyArgs &a, int b, int n, int word) {
  if (threadIdx.x == 0) a.accepted[b] = n;
  for (int i = threadIdx.x; i <= a.K; i += blockDim.x) {
    const long at = (long)i * a.B + b;
    a.tokens[at] = i < n ? a.drafts[at] : i == n ? word : -1;
  }
}

// The drawn word, by all threads of a workgroup: load(k) is the sum of r over block k; again(): forms the sums of p alone in
// their place.
template <typename T, class Load, class Again>
__device__ inline int verify_draw(const VerifyArgs &a, int b, Rest<T> &rest, Load &&load, Again &&again) {
  __shared__ int sh_word;
  constexpr int NONE = -2;  // no mass anywhere
  auto draw = [&]() {
    if (threadIdx.x < 64) {
      double before, goal, total;
      const int k = block_of_number(a.blocks, (double)a.u[(long)a.K * a.B + b], load, before, goal, total);
      const int word = total == 0.0 ? NONE : k < 0 ? -1 : word_of_block(rest, k, before, goal);
      if (threadIdx.x == 0) sh_word = word;
    }
    __syncthreads();
  };
  draw();
  if (sh_word == NONE) {  // p <= q everywhere: p itself
    rest.alone();
    again();
    draw();
  }
  return max(sh_word, -1);
}

// This lane's sums of exponentials over blocks [first, last) of the drawn row pair.
template <typename T, int THREADS>
__device__ __forceinline__ void verify_exponentials(const Rest<T> &rest, int first, int last, double &sp, double &sq) {
  sp = sq = 0.0;
  rest.each(first + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), last, THREADS / 64, [&](int, const typename Rest<T>::Block &o) {
#pragma unroll
    for (int e = 0; e < SlotOf<T>::N; ++e) sp += rest.ep(slot_elem<T>(o.p, e));
    if (rest.q)
#pragma unroll
      for (int e = 0; e < SlotOf<T>::N; ++e) sq += rest.eq(slot_elem<T>(o.q, e));
  });
}

template <typename T>
__global__ void __launch_bounds__(VERIFY_DECIDE_THREADS) verify_decide_kernel(const VerifyArgs a) {
  const int b = blockIdx.x;
  const VerifySeq s = verify_decide<T, VERIFY_DECIDE_THREADS>(a, b);
  if (threadIdx.x == 0) a.seq[b] = s;
}

// One share of a row pair that p - q is drawn from: sums of exponentials.  DECIDE: the workgroup works step 2 out for itself.
template <typename T, bool DECIDE>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_sums_kernel(const VerifyArgs a) {
  const int b = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  VerifySeq s;
  if constexpr (DECIDE) {
    s = verify_decide<T, VERIFY_THREADS>(a, b);
    if (chunk == 0 && threadIdx.x == 0) a.seq[b] = s;
  } else {
    s = a.seq[b];
  }
  if (!s.ok || !s.mixed) return;
  const Rest<T> rest(a, b, s);
  double sp, sq;
  verify_exponentials<T, VERIFY_THREADS>(rest, chunk * a.span, min((chunk + 1) * a.span, a.blocks), sp, sq);
  sp = block_sum<VERIFY_THREADS>(sp);
  sq = block_sum<VERIFY_THREADS>(sq);
  if (threadIdx.x == 0) {
    a.sums[((long)b * a.chunks + chunk) * 2] = sp;
    a.sums[((long)b * a.chunks + chunk) * 2 + 1] = sq;
  }
}

// Sums of r by blocks; the last workgroup of a text draws its word.  (What it reads of the others' moves with agent-scope
// accesses, each workgroup's before its arrival at the text's counter.)
template <typename T, bool DECIDE>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_rest_kernel(const VerifyArgs a) {
  __shared__ int sh_last;
  const int b = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  VerifySeq s;
  if constexpr (DECIDE) s = verify_decide<T, VERIFY_THREADS>(a, b);
  else s = a.seq[b];
  if (!s.ok) {
    if (chunk == 0) verify_store(a, b, s.n, -1);
    return;
  }
  Rest<T> rest(a, b, s);
  if (rest.q) {
    double sp = 0.0, sq = 0.0;
    for (int i = threadIdx.x & 63; i < a.chunks; i += 64) {
      sp += a.sums[((long)b * a.chunks + i) * 2];
      sq += a.sums[((long)b * a.chunks + i) * 2 + 1];
    }
    rest.normalise(wave_sum(sp), wave_sum(sq));
  }
  double *const of_block = a.rest + (long)b * a.blocks;
  auto load = [&](int k) { return __hip_atomic_load(of_block + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  __shared__ double staged[VERIFY_STAGED];
  const bool stage = a.blocks <= VERIFY_STAGED;
  auto fetch = [&] {  // all loads at once: one after the other each takes a trip to memory
    if (!stage) return;
    for (int k = threadIdx.x; k < a.blocks; k += VERIFY_THREADS) staged[k] = load(k);
    __syncthreads();
  };
  auto form = [&](int first, int last) {
    rest.each(first + wave, last, VERIFY_THREADS / 64, [&](int k, const typename Rest<T>::Block &o) {
      double r[Rest<T>::N];
      const double sum = wave_sum(rest.rest(k, o, r));
      if ((threadIdx.x & 63) == 0) __hip_atomic_store(of_block + k, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  form(chunk * a.span, min((chunk + 1) * a.span, a.blocks));
  if (threadIdx.x == 0)
    sh_last = __hip_atomic_fetch_add(&a.seq[b].done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (unsigned)a.chunks;
  __syncthreads();
  if (!sh_last) return;
  fetch();
  const int word = verify_draw<T>(a, b, rest, [&](int k) { return stage ? staged[k] : load(k); }, [&] {
    form(0, a.blocks);
    fetch();
  });
  verify_store(a, b, s.n, word);
}

// Steps 2 to 4 of a text whose rows are short.
template <typename T>
__global__ void __launch_bounds__(VERIFY_ONE_THREADS) verify_one_kernel(const VerifyArgs a) {
  __shared__ double of_block[VERIFY_ONE_BLOCKS];
  const int b = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const VerifySeq s = verify_decide<T, VERIFY_ONE_THREADS>(a, b);
  int word = -1;
  if (s.ok) {
    Rest<T> rest(a, b, s);
    if (rest.q) {
      double sp, sq;
      verify_exponentials<T, VERIFY_ONE_THREADS>(rest, 0, a.blocks, sp, sq);
      sp = block_sum<VERIFY_ONE_THREADS>(sp);
      sq = block_sum<VERIFY_ONE_THREADS>(sq);
      rest.normalise(sp, sq);
    }
    auto form = [&] {
      rest.each(wave, a.blocks, VERIFY_ONE_THREADS / 64, [&](int k, const typename Rest<T>::Block &o) {
        double r[Rest<T>::N];
        const double sum = wave_sum(rest.rest(k, o, r));
        if ((threadIdx.x & 63) == 0) of_block[k] = sum;
      });
      __syncthreads();
    };
    form();
    word = verify_draw<T>(a, b, rest, [&](int k) { return of_block[k]; }, form);
  }
  verify_store(a, b, s.n, word);
}

}  // namespace rnnlm_dev
