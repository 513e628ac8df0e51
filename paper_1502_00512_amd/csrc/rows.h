// Rows of logits as the operators on arrays of logits read them (logit_ops.hip): 16-byte slots of a row that may start at
// any element, and reductions over a workgroup.
#pragma once
#include "common.h"

namespace rnnlm_dev {

// Rows of more bytes than this in a call are read past the caches: more than half of the memory-side cache's 256 MB, so little
// of them is still there from whoever wrote them.  Read so and ordinarily: 164 MB (loss only) 30.4 and 33.4 us, 328 MB (with
// gradient) 132 and 138, but 51 MB 27.8 and 24.5, 120 MB 58.3 and 54.5.
constexpr long READ_ONCE_BYTES = 128L << 20;

constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LOG2E_64 = 1.44269504088896340736;

// A row starts where the one before ends, at any element: its slots are read and written at the elements' alignment.
typedef u32x4_t slot_t;
typedef u32x4_t slot_bf16_t __attribute__((aligned(2)));
typedef u32x4_t slot_fp32_t __attribute__((aligned(4)));
template <typename T>
struct SlotOf;
template <>
struct SlotOf<float> {
  typedef slot_fp32_t type;
  static constexpr int N = 4;
};
template <>
struct SlotOf<bf16_t> {
  typedef slot_bf16_t type;
  static constexpr int N = 8;
};

// Element e of a slot.
template <typename T>
__device__ inline float slot_elem(const slot_t &s, int e);
template <>
__device__ inline float slot_elem<float>(const slot_t &s, int e) {
  const unsigned w = s[e];
  return __builtin_bit_cast(float, w);
}
template <>
__device__ inline float slot_elem<bf16_t>(const slot_t &s, int e) {
  const unsigned w = s[e >> 1];
  return __builtin_bit_cast(float, e & 1 ? w & 0xffff0000u : w << 16);
}

template <typename T>
__device__ inline slot_t empty_slot() {  // -inf in every element
  const unsigned w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return slot_t{w, w, w, w};
}

// Whole slot j of a row; the elements behind a row's last whole slot are taken one by one (tail_elem).  ONCE: nobody reads it
// again soon, it need not displace anything in the caches.
template <typename T, bool ONCE = false>
__device__ inline slot_t load_slot(const T *row, int j) {
  // (an unsigned 32-bit offset from a row that all lanes share: no 64-bit address in registers)
  const auto *p = reinterpret_cast<const typename SlotOf<T>::type *>(reinterpret_cast<const char *>(row) + (unsigned)j * 16u);
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}
// Gradients are written past the caches: they are as large as the logits, and with ordinary stores the rows that other
// workgroups are about to read were displaced (2560 rows of 10000 bf16 words 30.2 -> 24.5 us, of 64000 149 -> 138; 8192 of
// 100000 733 -> 691).
template <typename T>
__device__ inline void store_slot(T *row, int j, const float (&v)[SlotOf<T>::N]) {
  constexpr int N = SlotOf<T>::N;
  union {
    slot_t s;
    T t[N];
  } o;
#pragma unroll
  for (int e = 0; e < N; ++e) o.t[e] = from_f32<T>(v[e]);
  __builtin_nontemporal_store(o.s, reinterpret_cast<typename SlotOf<T>::type *>(reinterpret_cast<char *>(row) + (unsigned)j * 16u));
}
// Element of the row behind its whole slots that thread tid takes; -inf for the others.
template <typename T>
__device__ inline float tail_elem(const T *row, int tid, int V) {
  const int at = V / SlotOf<T>::N * SlotOf<T>::N + tid;
  return at < V ? to_f32(row[at]) : -INFINITY;
}
// Slot j of a row, whole or not: elements behind the row are -inf.
template <typename T>
__device__ inline slot_t load_any_slot(const T *row, int j, int V) {
  constexpr int N = SlotOf<T>::N;
  if (j * N + N <= V) return load_slot(row, j);
  union {
    slot_t s;
    T t[N];
  } o;
  o.s = empty_slot<T>();
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (j * N + e < V) o.t[e] = row[j * N + e];
  return o.s;
}
// Makes the compiler unpack a slot anew where it is used again: elements of a bf16 slot kept unpacked take twice its
// registers (a row that fits them spilled 280 of them).
__device__ inline void keep_packed(slot_t &s) { asm volatile("" : "+v"(s)); }

// Makes the compiler work a value out by here.
__device__ inline void keep_here(float &v) { asm volatile("" : "+v"(v)); }

// The greatest of three numbers.  Quiet NaNs lose; a signalling one makes a quiet NaN of its maximum with the number in front of
// it, which is lost then: wherever that matters the elements go through without_nans first.  (fmaxf of values from memory costs
// an instruction more for each of them, which makes signalling NaNs quiet: two and a half instructions for two elements instead
// of one.)
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// -inf in place of a slot's NaNs.
template <typename T>
__device__ inline void without_nans(slot_t &s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned w = s[i];
    if constexpr (sizeof(T) == 4) {
      w = (w & 0x7fffffffu) > 0x7f800000u ? 0xff800000u : w;
    } else {
      w = (w & 0x7fffu) > 0x7f80u ? (w & 0xffff0000u) | 0xff80u : w;
      w = (w & 0x7fff0000u) > 0x7f800000u ? (w & 0xffffu) | 0xff800000u : w;
    }
    s[i] = w;
  }
}
// The greatest of m and the elements of a slot.
template <typename T>
__device__ inline float slot_max(float m, const slot_t &s) {
#pragma unroll
  for (int e = 0; e < SlotOf<T>::N; e += 2) m = max3(m, slot_elem<T>(s, e), slot_elem<T>(s, e + 1));
  return m;
}

__device__ inline float exp2_32(float x) { return __builtin_amdgcn_exp2f(x); }

// References of a sum of exponentials 2^{z c}: whole powers of 2 near 2^{m c}, so that z c - power is rounded once and sums move
// from one to another by exact factors.  Logits whose power is beyond 2^22 (and masked ones) have none.
__device__ inline bool near_power(float m, float c) { return fabsf(m * c) < 4194304.0f; }
__device__ inline float whole_power(float m, float c) { return near_power(m, c) ? rintf(m * c) : 0.0f; }
// Sums that are formed relative to a wave's first elements may be this large: those of all waves and chunks of a row stay in range
// together, and so does what they are joined by.  (No: also where they are no numbers.)
__device__ inline bool joinable(float sum) { return sum < 0x1p100f; }
// 2^(from - to); 0 from -inf.
__device__ inline float power_between(double from, double to) { return from == -INFINITY ? 0.0f : exp2_32((float)(from - to)); }

// Exchanges within 16 lanes: a mirrored or swapped lane's value in two instructions' time, where an exchange by way of LDS takes
// about a hundred cycles.
template <int CTRL, typename X>
__device__ inline X lane_swap(X v) {
  constexpr int WORDS = sizeof(X) / 4;
  union {
    X x;
    int w[WORDS];
  } u;
  u.x = v;
#pragma unroll
  for (int i = 0; i < WORDS; ++i) u.w[i] = __builtin_amdgcn_update_dpp(0, u.w[i], CTRL, 0xf, 0xf, true);
  return u.x;
}
template <typename X>
__device__ inline X lane_value(X v, int lane) {
  constexpr int WORDS = sizeof(X) / 4;
  union {
    X x;
    int w[WORDS];
  } u;
  u.x = v;
#pragma unroll
  for (int i = 0; i < WORDS; ++i) u.w[i] = __builtin_amdgcn_readlane(u.w[i], lane);
  return u.x;
}
// Over groups of G lanes (2 to 16, aligned): every lane gets its group's.
template <int G, typename X, class Op>
__device__ inline X group_reduce(X v, Op &&op) {
  if (G >= 2) v = op(v, lane_swap<0xB1>(v));   // the neighbour
  if (G >= 4) v = op(v, lane_swap<0x4E>(v));   // the other pair of four
  if (G >= 8) v = op(v, lane_swap<0x141>(v));  // mirrored among eight
  if (G >= 16) v = op(v, lane_swap<0x140>(v)); // mirrored among sixteen
  return v;
}
// Over the 64 lanes; all of them have to be active.
template <typename X, class Op>
__device__ inline X wave_reduce(X v, Op &&op) {
  v = group_reduce<16>(v, op);
  return op(op(lane_value(v, 0), lane_value(v, 16)), op(lane_value(v, 32), lane_value(v, 48)));
}
// The same over WAVES numbers of LDS (a power of two, one a wave of the workgroup), for every lane.
template <int WAVES, class Op>
__device__ inline float waves_reduce(const float *of_wave, Op &&op) {
  return group_reduce<WAVES>(of_wave[threadIdx.x & (WAVES - 1)], op);
}
template <int WAVES>
__device__ inline float waves_max(const float *of_wave) {
  return waves_reduce<WAVES>(of_wave, [](float a, float b) { return fmaxf(a, b); });
}
template <int WAVES>
__device__ inline float waves_sum(const float *of_wave) {
  return waves_reduce<WAVES>(of_wave, [](float a, float b) { return a + b; });
}
// Sums of the lanes up to each one: within sixteen lanes, then the rows of sixteen in front.
template <typename X>
__device__ inline X wave_scan(X v) {
  v += lane_swap<0x111>(v);  // the value 1, 2, 4, 8 lanes below (0 from outside the sixteen)
  v += lane_swap<0x112>(v);
  v += lane_swap<0x114>(v);
  v += lane_swap<0x118>(v);
  const X r0 = lane_value(v, 15), r1 = r0 + lane_value(v, 31), r2 = r1 + lane_value(v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return row == 0 ? v : v + (row == 1 ? r0 : row == 2 ? r1 : r2);
}
__device__ inline float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
template <typename X>
__device__ inline X wave_sum(X v) {
  return wave_reduce(v, [](X a, X b) { return a + b; });
}

}  // namespace rnnlm_dev
