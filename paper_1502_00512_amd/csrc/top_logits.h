// The K greatest logits of a row, in descending order (equal ones: the lower id first), and ln sum_v exp(z_v / tau).
// A row, or a chunk of a long one, fits a workgroup's registers, so it is read once, which is what bounds calls of many rows (2560
// of 64000 bf16 words, K = 64: 66 us, 4.9 TB/s); few rows are bound by the steps' latency.  A word is ranked by one 64-bit key, the
// logit's bits in an order that integers have, above the complement of the id: keys differ, so the order is total and a result
// does not depend on which wave arrives first.  (A NaN of either kind ranks with the masked words, -inf; -0 ranks with +0.)
//   1. maxima of groups of elements (one group a thread or several), sum of exponentials of the chunk
//   2. a threshold that at least K of the maxima reach, so at least K elements do: bisection over the maxima by one wave
//   3. elements that reach it into LDS: of G groups without structure some G ln(G / (G - K)), so several a thread where one
//      a thread would leave more than 1.15 K (5968 bf16 rows of 1582 words, K = 155: 102 us with two a
//      thread, 53 with four)
//   4. their ranks among each other
// Where step 3 finds more than LDS holds, or the groups that hold a number are fewer than K, the exact K-th key is found by
// bisection over the bits of logit and id with a count of the whole chunk for each: 32 + 20 counts, right for every input.
// (Rows of few words are ranked whole then.)
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int TOP_K_MAX = 256;
constexpr int TOP_WIDE = 512, TOP_WIDEST = 1024, TOP_MERGE_THREADS = 256, TOP_CAP = 1024, TOP_MERGE_LDS = 2048;
constexpr int TOP_COUNTED = 128;  // keys that are ranked by counting
constexpr int TOP_WHOLE = 512;  // rows of so many words may be ranked as they are
constexpr int TOP_V_MAX = 1 << 20;  // ids fit 20 bits
constexpr unsigned TOP_MASKED = 0x007fffffu;  // order of -inf

// The order of a logit as an unsigned integer, and back.
__device__ inline unsigned logit_order(float z) {
  z = fmaxf(z, -INFINITY) + 0.0f;
  const unsigned u = __builtin_bit_cast(unsigned, z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float order_logit(unsigned k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ inline unsigned long long top_key(unsigned order, int id) {
  return (unsigned long long)order << 32 | (unsigned)~id;
}

struct TopArgs {
  const void *z;
  long ld;
  int V, K, chunks, per;  // per: slots of a chunk
  float tau;
  int32_t *ids;
  float *vals, *lse;
  unsigned long long *part;  // [row][chunk][K], descending; 0 behind a chunk's last element
  double2 *stat;             // [row][chunk]: base-2 logarithm of a reference, sum of exponentials at tau relative to it
  bool once;                 // read past the caches
};

__device__ inline void top_store(const TopArgs &a, long row, int rank, unsigned long long key) {
  a.ids[row * a.K + rank] = (int)~(unsigned)key;
  a.vals[row * a.K + rank] = order_logit((unsigned)(key >> 32));
}

// ln of the sum s of 2^{z c} relative to 2^ref, at tau.  (c is log2 e / tau in 32 bits: by ln 2 the logarithm of a row far from zero
// would be off by as much as c is, once more than its own rounding.)
__device__ inline float row_lse(const TopArgs &a, double ref, float s) {
  return s == 0.0f ? -INFINITY : (float)((ref + log2((double)s)) / ((double)(LOG2E / a.tau) * (double)a.tau));
}

// The value of the lane whose number differs in the bits of X.
template <int X>
__device__ inline unsigned long long lane_xor(unsigned long long v) {
  if constexpr (X == 1) return lane_swap<0xB1>(v);
  else if constexpr (X == 2) return lane_swap<0x4E>(v);
  else if constexpr (X == 3) return lane_swap<0x1B>(v);
  else if constexpr (X == 4) return lane_swap<0x1B>(lane_swap<0x141>(v));
  else if constexpr (X == 7) return lane_swap<0x141>(v);
  else if constexpr (X == 8) return lane_swap<0x128>(v);
  else if constexpr (X == 15) return lane_swap<0x140>(v);
  else return __shfl_xor(v, X);
}
// Sorts a wave's keys, descending: sorted runs of BITS lanes are joined to runs of twice as many, the first exchange of each
// join a mirrored one.
template <int X, int BIT>
__device__ inline void top_exchange(unsigned long long &key) {
  const unsigned long long other = lane_xor<X>(key);
  const bool lower = (threadIdx.x & BIT) == 0;
  key = (other > key) == lower ? other : key;
}
template <int BITS>
__device__ inline void top_settle(unsigned long long &key) {
  if constexpr (BITS >= 1) {
    top_exchange<BITS, BITS>(key);
    top_settle<BITS / 2>(key);
  }
}
template <int BITS = 1>
__device__ inline void top_sort(unsigned long long &key) {
  if constexpr (BITS <= 32) {
    top_exchange<2 * BITS - 1, BITS>(key);
    top_settle<BITS / 2>(key);
    top_sort<2 * BITS>(key);
  }
}

// store(rank, key) for the K greatest of n keys in LDS (room for whole 64s).  Few keys: eight lanes to a key, each counts an eighth
// of the others.  Many: lists of 64, sorted by a wave each; a key's rank is what bisection finds above it in every list.  (Counted
// and sorted: K = 64 of 64000 words, 2560 rows 66.7 and 69.8 us; K = 120 of 10000, one row 12.0 and 11.1; K = 155 of 1582,
// 5968 rows 54 and 40; K = 256 of 109430, 3 rows 45.8 and 30.3.)
template <int THREADS, class Store>
__device__ inline void top_ranks(unsigned long long *cand, int n, int K, Store &&store) {
  if (n > TOP_COUNTED) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lists = (n + 63) / 64;
    for (int l = wave; l < lists; l += THREADS / 64) {
      unsigned long long key = l * 64 + lane < n ? cand[l * 64 + lane] : 0;
      top_sort(key);
      cand[l * 64 + lane] = key;
    }
    __syncthreads();
    for (int l = wave; l < lists; l += THREADS / 64) {
      const unsigned long long key = cand[l * 64 + lane];
      int rank = 0;
      for (int other = 0; other < lists; other += 4) {  // (its own list among them)
        int above[4] = {};
#pragma unroll
        for (int step = 32; step; step >>= 1)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (other + i < lists && cand[(other + i) * 64 + above[i] + step - 1] > key) above[i] += step;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (other + i < lists) rank += above[i] + (cand[(other + i) * 64 + above[i]] > key);
      }
      if (key != 0 && rank < K) store(rank, key);
    }
    return;
  }
  for (int i0 = 0; i0 < n; i0 += THREADS / 8) {
    const int i = i0 + threadIdx.x / 8;
    const unsigned long long key = i < n ? cand[i] : ~0ull;
    int rank = 0;
#pragma unroll 4
    for (int j = threadIdx.x & 7; j < n; j += 8) rank += cand[j] > key;
    rank = group_reduce<8>(rank, [](int x, int y) { return x + y; });
    if (i < n && rank < K && (threadIdx.x & 7) == 0) store(rank, key);
  }
}

// A threshold that at least K of 64 G numbers reach, and few more; by one wave.  (Bisection: a count takes 2 G instructions.)
template <int G>
__device__ inline unsigned top_threshold(const unsigned *group, int K, unsigned greatest) {
  unsigned g[G], low = 0xffffffffu;
#pragma unroll
  for (int i = 0; i < G; ++i) {
    g[i] = group[i * 64 + (threadIdx.x & 63)];
    low = min(low, g[i]);
  }
  low = wave_reduce(low, [](unsigned p, unsigned q) { return min(p, q); });
  // at least K reach lo (all of them, to begin with), fewer reach hi
  unsigned lo = __builtin_amdgcn_readfirstlane(low), hi = greatest + 1;
  while (hi - lo > 1) {
    const unsigned mid = lo + (hi - lo) / 2;
    int n = 0;
#pragma unroll
    for (int i = 0; i < G; ++i) n += __popcll(__ballot(g[i] >= mid));
    if (n >= K) {
      lo = mid;
      if (n <= K + K / 8) break;
    } else {
      hi = mid;
    }
  }
  return lo;
}

template <typename T, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 4) top_chunk_kernel(const TopArgs a) {
  constexpr int N = SlotOf<T>::N, WAVES = THREADS / 64, PARTS = NV <= 8 ? 4 : 2;  // groups of a thread where they are fine
  __shared__ float sh_m[WAVES], sh_s[WAVES];
  __shared__ double sh_ref[WAVES];
  __shared__ unsigned group[PARTS * THREADS];
  __shared__ unsigned long long cand[TOP_CAP];
  __shared__ unsigned sh_t, sh_n, sh_count[2][WAVES];
  const long row = blockIdx.x / a.chunks;
  const int chunk = blockIdx.x % a.chunks, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const T *z = static_cast<const T *>(a.z) + row * a.ld;
  const int full = a.V / N, first = chunk * a.per, slots = min(a.per, full - first), K = a.K;
  slot_t raw[NV];
  if (a.once) {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < slots ? load_slot<T, true>(z + (first + i * THREADS) * N, tid) : empty_slot<T>();
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = i * THREADS + tid < slots ? load_slot(z + (first + i * THREADS) * N, tid) : empty_slot<T>();
  }
  const int tail = chunk == a.chunks - 1 ? full * N + tid : a.V;  // the last chunk has the row's last elements, one a thread
  const float zt = tail < a.V ? to_f32(z[tail]) : -INFINITY;
  if (tid == 0) sh_n = 0;
  // 1.  The sum is relative to about the greatest element of the wave's first slots (a whole power of 2), so it runs while the
  // rest arrives.
  const float c = LOG2E / a.tau, ref = wave_max(slot_max<T>(zt, raw[0])), b = -whole_power(ref, c);
  float top[NV], part[PARTS], s = exp2_32(fmaf(zt, c, b));
  auto maxima = [&](int i) {
    if constexpr (NV < 4) {  // groups of a slot's quarters
      float of_slot[4];
#pragma unroll
      for (int e = 0; e < N; e += N / 4) of_slot[e / (N / 4)] = max3(slot_elem<T>(raw[i], e), slot_elem<T>(raw[i], e + N / 4 - 1), -INFINITY);
      top[i] = max3(max3(of_slot[0], of_slot[1], of_slot[2]), of_slot[3], -INFINITY);
#pragma unroll
      for (int e = 0; e < 4; ++e) part[e] = max3(part[e], of_slot[e], -INFINITY);
    } else {
      top[i] = slot_max<T>(-INFINITY, raw[i]);
      part[i % PARTS] = max3(part[i % PARTS], top[i], -INFINITY);
    }
  };
#pragma unroll
  for (int i = 0; i < PARTS; ++i) part[i] = i == 0 ? max3(zt, -INFINITY, -INFINITY) : -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    maxima(i);
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp2_32(fmaf(slot_elem<T>(raw[i], e), c, b));
    keep_packed(raw[i]);
    keep_here(s);  // (with the exponentials of many slots put off the kernel spilled 100 registers)
  }
  const bool fine = 4 * K > min(slots, THREADS);
  auto groups = [&] {
    float all = part[0];
#pragma unroll
    for (int i = 1; i < PARTS; ++i) all = max3(all, part[i], -INFINITY);
    group[tid] = logit_order(fine ? part[0] : all);
    if (fine)
#pragma unroll
      for (int i = 1; i < PARTS; ++i) group[i * THREADS + tid] = logit_order(part[i]);
    return wave_max(all);
  };
  float mine = groups();
  s = wave_sum(s);
  double power = -(double)b;
  if (s != s) {  // NaNs: they rank as masked words, and the maxima once more without them
#pragma unroll
    for (int i = 0; i < PARTS; ++i) part[i] = i == 0 ? max3(zt, -INFINITY, -INFINITY) : -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      without_nans<T>(raw[i]);
      maxima(i);
    }
    mine = groups();
  }
  if (!joinable(s) || (!near_power(ref, c) && mine > -INFINITY)) {
    // no number or too great a one, or the first slots are masked throughout: once more, relative to the wave's maximum
    const float base = mine == -INFINITY ? 0.0f : mine;
    s = exp2_32((zt - base) * c);
    for (int j = tid; j < slots; j += THREADS) {
      const slot_t q = load_slot(z, first + j);
#pragma unroll
      for (int e = 0; e < N; ++e) s += exp2_32((slot_elem<T>(q, e) - base) * c);
    }
    s = wave_sum(s);
    power = (double)base * (double)c;
  }
  if (lane == 0) sh_ref[wave] = s == 0.0f ? -INFINITY : power;
  if (lane == 0) {
    sh_m[wave] = mine;
    sh_s[wave] = s;
  }
  __syncthreads();
  // 2.
  if (wave == 0) {
    const float mx = waves_max<WAVES>(sh_m);
    const unsigned top_order = __builtin_amdgcn_readfirstlane(logit_order(mx));
    const unsigned lo = fine ? top_threshold<PARTS * WAVES>(group, K, top_order) : top_threshold<WAVES>(group, K, top_order);
    if (lane == 0) sh_t = lo;
  }
  __syncthreads();
  // 3.
  const unsigned thr = sh_t;
  const bool few = thr <= TOP_MASKED;  // fewer than K groups with a number
  if (!few) {
    // Of its slots that reach the threshold a lane takes one at a time, each lane its own (selected from the registers): the
    // 64 lanes' few finds share the instructions.
    const float t = order_logit(thr);
    unsigned left = 0;  // slots with finds
#pragma unroll
    for (int i = 0; i < NV; ++i) left |= (top[i] >= t ? 1u : 0u) << i;
    if (zt >= t) {
      const unsigned at = atomicAdd(&sh_n, 1u);
      if (at < TOP_CAP) cand[at] = top_key(logit_order(zt), tail);
    }
    while (__any(left != 0)) {
      const int mine_at = left ? __builtin_ctz(left) : NV;
      left &= left - 1;
      slot_t q = empty_slot<T>();
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i == mine_at) q = raw[i];
      unsigned finds = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) finds |= (slot_elem<T>(q, e) >= t ? 1u : 0u) << e;
      unsigned at = finds ? atomicAdd(&sh_n, (unsigned)__popc(finds)) : 0u;
      const int id0 = (first + mine_at * THREADS + tid) * N;
      while (__any(finds != 0)) {
        if (finds) {
          const int f = __builtin_ctz(finds);
          float v = slot_elem<T>(q, 0);
#pragma unroll
          for (int e = 1; e < N; ++e) v = e == f ? slot_elem<T>(q, e) : v;
          if (at < TOP_CAP) cand[at] = top_key(logit_order(v), id0 + f);
          ++at;
          finds &= finds - 1;
        }
      }
    }
    __syncthreads();
  }
  int n = (int)sh_n;
  auto each = [&](auto &&element) {
    if (tail < a.V) element(logit_order(zt), tail);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = i * THREADS + tid;
      keep_packed(raw[i]);
      if (j < slots) {
#pragma unroll
        for (int e = 0; e < N; ++e) element(logit_order(slot_elem<T>(raw[i], e)), (first + j) * N + e);
      }
    }
  };
  if (NV == 1 && few && a.V <= TOP_WHOLE) {
    each([&](unsigned k, int id) { cand[id] = top_key(k, id); });
    __syncthreads();
    n = a.V;
  } else if (few || n > TOP_CAP) {
    // exact: the order of the K-th element, then the id up to which elements of that order belong
    int turn = 0;
    auto count = [&](auto &&reaches) {
      int mine = 0;
      each([&](unsigned k, int id) { mine += reaches(k, id); });
      mine = wave_sum(mine);
      if (lane == 0) sh_count[turn][wave] = mine;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) all += sh_count[turn][i];
      turn ^= 1;  // the next count writes the other copy, so nobody waits for this one's readers
      return all;
    };
    unsigned kth = 0;
    for (unsigned bit = 1u << 31; bit; bit >>= 1)
      if (count([&](unsigned k, int) { return k >= (kth | bit); }) >= K) kth |= bit;
    const int above = count([&](unsigned k, int) { return k > kth; });
    int bound = 0;  // greatest id below which fewer than the missing elements are found
    for (int bit = TOP_V_MAX >> 1; bit; bit >>= 1)
      if (count([&](unsigned k, int id) { return k == kth && id < (bound | bit); }) < K - above) bound |= bit;
    if (tid == 0) sh_n = 0;
    __syncthreads();
    each([&](unsigned k, int id) {
      if (k > kth || (k == kth && id <= bound)) cand[atomicAdd(&sh_n, 1u)] = top_key(k, id);
    });
    __syncthreads();
    n = (int)sh_n;
  }
  // 4.
  top_ranks<THREADS>(cand, n, K, [&](int rank, unsigned long long key) {
    if (a.chunks == 1) top_store(a, row, rank, key);
    else a.part[(long)blockIdx.x * K + rank] = key;
  });
  if (a.chunks > 1)
    for (int i = n + tid; i < K; i += THREADS) a.part[(long)blockIdx.x * K + i] = 0;
  if (wave == 0) {
    const double q = sh_ref[lane & (WAVES - 1)], top_ref = group_reduce<WAVES>(q, [](double x, double y) { return fmax(x, y); });
    const float v = group_reduce<WAVES>(sh_s[lane & (WAVES - 1)] * power_between(q, top_ref), [](float x, float y) { return x + y; });
    if (lane == 0) {
      if (a.chunks > 1) a.stat[blockIdx.x] = make_double2(top_ref, (double)v);
      else if (a.lse) a.lse[row] = row_lse(a, top_ref, v);
    }
  }
}

// Joins the chunks of a row.  Each list's K / chunks greatest are at least K keys together, so no key below the least of them
// is wanted: the others (K to 3 K of them) are ranked among each other.  Where that leaves too many, a key's rank is its place in
// its own list and how many keys of the other lists are above it, each by bisection.
__global__ void __launch_bounds__(TOP_MERGE_THREADS) top_merge_kernel(const TopArgs a) {
  __shared__ unsigned long long lds[TOP_MERGE_LDS], cand[TOP_CAP];
  __shared__ unsigned long long sh_least;
  __shared__ unsigned sh_n;
  const long row = blockIdx.x;
  const int n = a.chunks * a.K, K = a.K, tid = threadIdx.x;
  const unsigned long long *key = a.part + row * n;
  if (tid == 0) sh_n = 0;
  if (tid < 64) {
    unsigned long long least = ~0ull;
    for (int l = tid; l < a.chunks; l += 64) least = min(least, key[l * K + (K + a.chunks - 1) / a.chunks - 1]);
    least = wave_reduce(least, [](unsigned long long x, unsigned long long y) { return x < y ? x : y; });
    if (tid == 0) sh_least = least;
  }
  const bool in_lds = n <= TOP_MERGE_LDS;  // (more: the widest vocabularies with the longest lists)
  if (in_lds)
    for (int i = tid; i < n; i += TOP_MERGE_THREADS) lds[i] = key[i];
  __syncthreads();
  if (in_lds) key = lds;
  const unsigned long long least = sh_least;
  for (int i = tid; i < n; i += TOP_MERGE_THREADS) {
    const unsigned long long k = key[i];
    if (k >= least && k != 0) {
      const unsigned at = atomicAdd(&sh_n, 1u);
      if (at < TOP_CAP) cand[at] = k;
    }
  }
  __syncthreads();
  if (sh_n <= TOP_CAP) {
    top_ranks<TOP_MERGE_THREADS>(cand, (int)sh_n, K, [&](int rank, unsigned long long k) { top_store(a, row, rank, k); });
  } else {
    for (int i = tid; i < n; i += TOP_MERGE_THREADS) {
      const unsigned long long k = key[i];
      if (k == 0) continue;
      const int mine = i / K;
      int rank = i - mine * K;
      for (int l = 0; l < a.chunks && rank < K; ++l) {
        if (l == mine) continue;
        int lo = 0, hi = K;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (key[l * K + mid] > k) lo = mid + 1;
          else hi = mid;
        }
        rank += lo;
      }
      if (rank < K) top_store(a, row, rank, k);
    }
  }
  if (threadIdx.x < 64 && a.lse) {
    double ref = -INFINITY;
    float s = 0.0f;
    for (int l = threadIdx.x; l < a.chunks; l += 64) {
      const double2 q = a.stat[row * a.chunks + l];
      const double top_ref = fmax(ref, q.x);
      s = s * power_between(ref, top_ref) + (float)q.y * power_between(q.x, top_ref);
      ref = top_ref;
    }
    const double top_ref = wave_reduce(ref, [](double x, double y) { return fmax(x, y); });
    s = wave_sum(s * power_between(ref, top_ref));
    if (threadIdx.x == 0) a.lse[row] = row_lse(a, top_ref, s);
  }
}

}  // namespace rnnlm_dev
