// Between a window's logits as the output layer forms and uses them (vocabulary-major, [Vp][ldz], position m = t*Bp + s) and
// the caller's rows (one a position, row t*B + s, V logits each): both directions, 64 x 64 tiles through LDS so that either
// side moves whole 128-byte lines (bf16).  Bound by HBM: V = 64000, 2560 positions, bf16 read 328 MB and write as much.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int LW_TILE = 64;

template <typename T>
struct LogitTile {
  T v[LW_TILE][LW_TILE + 16 / sizeof(T)];  // [position][word]: rows stay 16-byte aligned
};

struct LogitWindow {
  int Tn, B, Bp, V;
  long ldz, ld;
  // row of the caller's array that holds position m, or -1 on padding
  __device__ long row(int m) const {
    const int t = m / Bp, s = m % Bp;
    return t < Tn && s < B ? (long)t * B + s : -1;
  }
};

template <typename T>
__global__ void __launch_bounds__(256) logits_to_rows_kernel(const T *__restrict__ ZT, T *__restrict__ out, const LogitWindow w) {
  constexpr int N = SlotOf<T>::N, PER = LW_TILE / N;
  __shared__ LogitTile<T> tile;
  const int v0 = blockIdx.x * LW_TILE, m0 = blockIdx.y * LW_TILE;
  for (int i = threadIdx.x; i < LW_TILE * PER; i += 256) {
    const int v = i / PER, c = i % PER * N;
    union {
      slot_t s;
      T t[N];
    } in;
    in.s = *reinterpret_cast<const slot_t *>(ZT + (long)(v0 + v) * w.ldz + m0 + c);
#pragma unroll
    for (int e = 0; e < N; ++e) tile.v[c + e][v] = in.t[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < LW_TILE * PER; i += 256) {
    const int m = i / PER, c = i % PER * N;
    const long row = w.row(m0 + m);
    if (row < 0) continue;
    T *dst = out + row * w.ld + v0 + c;
    if (v0 + c + N <= w.V) {
      *reinterpret_cast<typename SlotOf<T>::type *>(dst) = *reinterpret_cast<const slot_t *>(&tile.v[m][c]);
    } else {
      for (int e = 0; e < N; ++e)
        if (v0 + c + e < w.V) dst[e] = tile.v[m][c + e];
    }
  }
}

// The way back for gradients: padding (words and positions) becomes zero.  A workgroup owns 64 words and walks a share of `per`
// positions in order.  sums[share][v] receives its sum over them (bias gradients), which bias_update_kernel joins; sums = nullptr:
// there is one share, and b_out[v] = alpha b[v] - lr sum.  With all positions of 64 words to a workgroup 10000 words ran on 157 compute units: 77 us for 2560 positions, 27 in shares.
template <typename T>
__global__ void __launch_bounds__(256) rows_to_logits_kernel(const T *__restrict__ in, T *__restrict__ ZT, int Mp, int per,
                                                             float *__restrict__ sums, long ld_sums, const float *__restrict__ b,
                                                             float *__restrict__ b_out, float alpha, float lr, const LogitWindow w) {
  constexpr int N = SlotOf<T>::N, PER = LW_TILE / N, ROWS = 256 / PER;  // positions a round
  __shared__ LogitTile<T> tile;
  __shared__ float part[ROWS][LW_TILE + 1];
  const int v0 = blockIdx.x * LW_TILE, c = threadIdx.x % PER * N, first = threadIdx.x / PER;
  float db[N];
#pragma unroll
  for (int e = 0; e < N; ++e) db[e] = 0.0f;
  const int end = min(Mp, ((int)blockIdx.y + 1) * per);
  for (int m0 = blockIdx.y * per; m0 < end; m0 += LW_TILE) {
    for (int m = first; m < LW_TILE; m += ROWS) {
      union {
        slot_t s;
        T t[N];
      } o;
      o.s = slot_t{0u, 0u, 0u, 0u};
      const long row = w.row(m0 + m);
      if (row >= 0) {
        const T *src = in + row * w.ld + v0 + c;
        if (v0 + c + N <= w.V) {
          o.s = *reinterpret_cast<const typename SlotOf<T>::type *>(src);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (v0 + c + e < w.V) o.t[e] = src[e];
        }
      }
      *reinterpret_cast<slot_t *>(&tile.v[m][c]) = o.s;
#pragma unroll
      for (int e = 0; e < N; ++e) db[e] += to_f32(o.t[e]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < LW_TILE * PER; i += 256) {
      const int v = i / PER, m = i % PER * N;
      union {
        slot_t s;
        T t[N];
      } o;
#pragma unroll
      for (int e = 0; e < N; ++e) o.t[e] = tile.v[m + e][v];
      *reinterpret_cast<slot_t *>(ZT + (long)(v0 + v) * w.ldz + m0 + m) = o.s;
    }
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < N; ++e) part[first][c + e] = db[e];
  __syncthreads();
  if (threadIdx.x < LW_TILE) {
    float d = 0.0f;
    for (int i = 0; i < ROWS; ++i) d += part[i][threadIdx.x];
    const int v = v0 + threadIdx.x;
    if (sums) sums[blockIdx.y * ld_sums + v] = d;
    else if (v < w.V) b_out[v] = (alpha != 0.0f ? alpha * b[v] : 0.0f) - lr * d;
  }
}

// b_out[v] = alpha b[v] - lr (the sums of all shares, in order).
__global__ void __launch_bounds__(256) bias_update_kernel(const float *__restrict__ sums, long ld_sums, int shares, int V,
                                                          const float *__restrict__ b, float *__restrict__ b_out, float alpha, float lr) {
  const int v = blockIdx.x * 256 + threadIdx.x;
  if (v >= V) return;
  float d = 0.0f;
  for (int i = 0; i < shares; ++i) d += sums[i * ld_sums + v];
  b_out[v] = (alpha != 0.0f ? alpha * b[v] : 0.0f) - lr * d;
}

// The window's losses summed in 64 bits (and the recurrent kernels' counters cleared between their two launches).
__global__ void __launch_bounds__(1024) losses_sum_kernel(const float *__restrict__ loss, int n, const WindowSum w) {
  window_sum(w, n, [&](int i) { return loss[i]; });
}

// h_state of every text after the inputs it keeps: the first and its accepted drafts.
template <typename T>
__global__ void __launch_bounds__(256) keep_states_kernel(const T *__restrict__ Hs, const int32_t *__restrict__ accepted, int H,
                                                          int Hp, int Bp, float *__restrict__ h_state) {
  const int s = blockIdx.x;
  const T *src = Hs + ((long)(accepted[s] + 1) * Bp + s) * Hp;
  for (int j = threadIdx.x; j < H; j += 256) h_state[(long)s * H + j] = to_f32(src[j]);
}

}  // namespace rnnlm_dev
