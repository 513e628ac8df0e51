// Low-rank adapters of many texts beside a shared projection, forward and backward.  Row m has x[K] and belongs to adapter
// a = ids[m], or to none:
//   inner = down[a] x (R numbers),                 out = base + f_a up[a] inner
//   dinner = f_a up[a]^T dout,  dup[a] = f_a sum_m dout inner^T,  ddown[a] = sum_m dinner x^T,  dx = down[a]^T dinner
// Rows are taken in the order of their adapters (adapter_order_kernel), 32 positions of that order a tile; a tile may hold rows
// of several adapters, each of which is multiplied with the whole tile and kept where it belongs (the products are few beside
// the bytes of base, out and dout, which bound all of this).
// Products: 16 x 16 tiles of the matrix cores.  bf16: inner and dinner are fp32 and go in as two parts (products that end in a
// bf16 number; 2^-17) or three (gradients in fp32; 2^-25), everything else is bf16 already; fp32: the fp32 instruction.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int ADAPTER_TILE = 32;   // rows of a tile
constexpr int ADAPTER_R_MAX = 64;

struct AdapterRows {
  const int32_t *ids, *perm;  // perm: rows in the order of their adapters; nullptr: as they are
  int M, n;
  // adapter of a row; n: none
  __device__ int key(int row) const {
    const int a = ids[row];
    return a >= 0 && a < n ? a : n;
  }
  __device__ int row(int pos) const { return perm ? perm[pos] : pos; }
};

// A lane's 16 bytes of an operand: VEC consecutive k of row (or column) l % 16, from k = (l / 16) VEC of a chunk of CHUNK on.
template <typename T>
struct Mma;
template <>
struct Mma<bf16_t> {
  static constexpr int VEC = 8, CHUNK = 32;
  __device__ static void add(f32x4_t &acc, const slot_t &a, const slot_t &b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
  }
};
template <>
struct Mma<float> {  // the e-th instruction contracts k = e, 4 + e, 8 + e, 12 + e
  static constexpr int VEC = 4, CHUNK = 16;
  __device__ static void add(f32x4_t &acc, const slot_t &a, const slot_t &b) {
    const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], acc, 0, 0, 0);
  }
};

// Orders the LDS accesses of a wave's lanes among one another.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The first `left` elements of a slot, zeros behind them.
template <typename T>
__device__ inline slot_t first_elems(slot_t s, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) s[i] = i < left ? s[i] : 0u;
    else s[i] = 2 * i + 1 < left ? s[i] : 2 * i < left ? s[i] & 0xffffu : 0u;
  }
  return s;
}
// Up to `left` elements from p on (zeros behind them), of which `there` may be read.
template <typename T>
__device__ inline slot_t load_elems(const T *p, int left, long there) {
  constexpr int N = SlotOf<T>::N;
  if (left <= 0) return slot_t{0u, 0u, 0u, 0u};
  if (there >= N) {
    const slot_t s = *reinterpret_cast<const typename SlotOf<T>::type *>(p);
    return left >= N ? s : first_elems<T>(s, left);
  }
  union {
    slot_t s;
    T t[N];
  } o;
  o.s = slot_t{0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < left) o.t[e] = p[e];
  return o.s;
}
// A number in PARTS bf16 parts, each the rest of those in front of it.
template <int PARTS>
__device__ inline void bf16_parts(float x, bf16_t (&p)[PARTS]) {
  p[0] = (bf16_t)x;
  float rest = x - (float)p[0];
  if (!(fabsf((float)p[0]) < INFINITY)) rest = 0.0f;
#pragma unroll
  for (int i = 1; i < PARTS; ++i) {
    p[i] = (bf16_t)rest;
    rest -= (float)p[i];
  }
}

// Numbers of the rows in the order of their adapters, transposed: [part][r][position].
template <typename T>
struct Transposed {
  static constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;
  T *at;
  long Mp;  // positions of a line, more than any tile reads
  int R;
  __device__ void put(int r, long pos, float v) const {
    if constexpr (PARTS == 1) {
      at[r * Mp + pos] = v;
    } else {
      bf16_t p[PARTS];
      bf16_parts<PARTS>(v, p);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) at[((long)i * R + r) * Mp + pos] = p[i];
    }
  }
};

// perm: the rows ordered by (adapter, row), rows without one last; start[a]: first position of adapter a, start[n]: of those
// rows.  64 questions a workgroup, each answered by counting all smaller keys: M (M + n) / 64 comparisons of a wave (2560 rows
// 2 us).  inner (may be nullptr) is transposed on the way.
template <typename T>
__global__ void __launch_bounds__(1024) adapter_order_kernel(const AdapterRows rows, int32_t *__restrict__ perm, int32_t *__restrict__ start,
                                                             const float *__restrict__ inner, const Transposed<T> tr, int32_t *range_flag) {
  __shared__ int32_t keys[4096];
  __shared__ int32_t cnt[16][64];
  __shared__ int32_t rank_of[64];
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, M = rows.M;
  const int q = blockIdx.x * 64 + lane;
  const int mine = q < M ? rows.key(q) : q - M;
  if (slice == 0 && q < M && rows.ids[q] >= rows.n && range_flag) *range_flag = 1;
  int rank = 0;
  for (int base = 0; base < M; base += 4096) {
    const int n = min(4096, M - base);
    for (int i = threadIdx.x; i < n; i += 1024) keys[i] = rows.key(base + i);
    __syncthreads();
    for (int i = slice; i < n; i += 16) {
      const int k = keys[i];
      rank += (k < mine) || (k == mine && base + i < q && q < M);
    }
    __syncthreads();
  }
  cnt[slice][lane] = rank;
  __syncthreads();
  if (slice == 0) {
    int r = 0;
    for (int g = 0; g < 16; ++g) r += cnt[g][lane];
    rank_of[lane] = r;
    if (q < M) perm[r] = q;
    else if (q - M <= rows.n) start[q - M] = r;
  }
  if (!inner) return;
  __syncthreads();
  const int here = min(64, M - (int)blockIdx.x * 64);
  for (int i = threadIdx.x; i < here * tr.R; i += 1024) {
    const int m = i / tr.R, r = i % tr.R;
    tr.put(r, rank_of[m], inner[((long)blockIdx.x * 64 + m) * tr.R + r]);
  }
}

// What a wave knows of a tile: lane l < 32 (and l + 32) the row at position 32 tile + l and its adapter.
struct AdapterTile {
  int row, key;  // -1, n: behind the last row
  __device__ AdapterTile(const AdapterRows &r, int first) {
    const int pos = first + (threadIdx.x & 31);
    row = pos < r.M ? r.row(pos) : -1;
    key = row >= 0 ? r.key(row) : r.n;
  }
  // The adapters of the tile one after the other, in the order of their first rows: the next one behind `left` (lanes not yet
  // dealt with), n when there is none.
  __device__ int next(unsigned &left, int n) const {
    left &= (unsigned)__ballot(key < n);
    if (!left) return n;
    const int a = __builtin_amdgcn_readlane(key, __ffs(left) - 1);
    left &= ~(unsigned)__ballot(key == a);
    return a;
  }
};

template <typename T>
struct InnerArgs {
  AdapterRows rows;
  const T *x, *down;
  long ldx;
  int K, R;
  float *inner;  // [M][R]
  int32_t *range_flag;
};

// inner: a workgroup a tile and one of its adapters (blockIdx.y-th); K over the waves, joined in LDS.
template <typename T, int RT>
__global__ void __launch_bounds__(512) adapter_inner_kernel(const InnerArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, WAVES = 8, TILE = ADAPTER_TILE;
  __shared__ float part[WAVES][RT * 16][TILE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const AdapterTile tile(a.rows, blockIdx.x * TILE);
  const int n = a.rows.n;
  unsigned left = 0xffffffffu;
  int id = tile.next(left, n);
  for (unsigned i = 0; i < blockIdx.y && id < n; ++i) id = tile.next(left, n);
  if (blockIdx.y == 0) {
    if (wave == 0 && a.range_flag && tile.row >= 0 && a.rows.ids[tile.row] >= n) *a.range_flag = 1;
    for (int i = wave; i < TILE; i += WAVES) {  // rows without an adapter
      const int row = __shfl(tile.row, i), key = __shfl(tile.key, i);
      if (row >= 0 && key == n && lane < a.R) a.inner[(long)row * a.R + lane] = 0.0f;
    }
  }
  if (id >= n) return;
  const T *down = a.down + (long)id * a.R * a.K;
  const T *xs[2];
  int ok[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = __shfl(tile.row, t * 16 + c);
    ok[t] = row >= 0 && __shfl(tile.key, t * 16 + c) == id;
    xs[t] = a.x + (ok[t] ? row : 0) * a.ldx;
  }
  f32x4_t acc[RT][2] = {};
#pragma unroll 2
  for (int k0 = wave * CHUNK; k0 < a.K; k0 += WAVES * CHUNK) {
    const int k = k0 + q * VEC, have = a.K - k;
    slot_t fx[2], fd[RT];
#pragma unroll
    for (int t = 0; t < 2; ++t) fx[t] = load_elems(xs[t] + k, ok[t] ? have : 0, have);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int j = r * 16 + c;
      fd[r] = load_elems(down + (long)j * a.K + k, j < a.R ? have : 0, have);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int t = 0; t < 2; ++t) Mma<T>::add(acc[r][t], fd[r], fx[t]);
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[wave][r * 16 + q * 4 + i][t * 16 + c] = acc[r][t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < RT * 16 * TILE; i += 512) {
    const int j = i % (RT * 16), m = i / (RT * 16), row = __shfl(tile.row, m & 31), key = __shfl(tile.key, m & 31);
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w][j][m];
    if (j < a.R && row >= 0 && key == id) a.inner[(long)row * a.R + j] = s;
  }
}

template <typename T>
struct OuterArgs {
  AdapterRows rows;
  const float *inner;  // [M][R], of rows or (by_position) of positions
  bool by_position;
  const T *up;         // [n][N][R], or (template ACROSS) [n][R][N]
  const float *scale;  // may be nullptr
  const T *base;       // may be nullptr (zeros), may be out
  T *out;
  long ldb, ldo;
  int N, R, blocks;    // blocks of 64 columns of a wave
};

// out = base + f up inner: a wave a tile and 64 columns, `blocks` times; through LDS so that base and out move in whole lines.
// Bound by HBM.  NF: operand slots of R.  PACKED (bf16, R <= 16): both parts of inner in one product, beside one another.
template <typename T, int NF, bool PACKED, bool ACROSS>
__global__ void __launch_bounds__(256, 2) adapter_outer_kernel(const OuterArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, TILE = ADAPTER_TILE, COLS = 64, PITCH = COLS + 4;
  constexpr int PARTS = sizeof(T) == 4 || PACKED ? 1 : 2, LANES = COLS / VEC, ROWS = 64 / LANES, MOVES = TILE / ROWS;
  __shared__ float turn[4][TILE][PITCH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int first = blockIdx.x * TILE, n = a.rows.n, N = a.N, R = a.R;
  const AdapterTile tile(a.rows, first);
  const int kq = (PACKED ? q & 1 : q) * VEC;
  // inner of the tile's rows (columns of the product), times the adapter's factor
  slot_t fu[2][NF][PARTS];
  int key[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int row = __shfl(tile.row, t * 16 + c);
    key[t] = __shfl(tile.key, t * 16 + c);
    const bool ok = row >= 0 && key[t] < n;
    const float f = ok && a.scale ? a.scale[key[t]] : 1.0f;
    const float *u = a.inner + (a.by_position ? (long)first + t * 16 + c : (long)row) * R;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      union {
        slot_t s[PARTS];
        T e[PARTS][VEC];
      } o;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int k = i * CHUNK + kq + e;
        const float v = ok && k < R ? u[k] * f : 0.0f;
        if constexpr (sizeof(T) == 4) {
          o.e[0][e] = v;
        } else {
          bf16_t p[2];
          bf16_parts<2>(v, p);
          if constexpr (PACKED) {
            o.e[0][e] = q < 2 ? p[0] : p[1];
          } else {
            o.e[0][e] = p[0];
            o.e[1][e] = p[1];
          }
        }
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p) fu[t][i][p] = o.s[p];
    }
  }
  const int lr = lane / LANES, lc = lane % LANES * VEC;
  int rows[MOVES];
#pragma unroll
  for (int i = 0; i < MOVES; ++i) rows[i] = __shfl(tile.row, i * ROWS + lr);
  for (int b = 0; b < a.blocks; ++b) {
    const int v0 = ((blockIdx.y * a.blocks + b) * 4 + wave) * COLS;
    if (v0 >= N) break;  // (nothing is shared between the waves)
    slot_t old[MOVES];
#pragma unroll
    for (int i = 0; i < MOVES; ++i) {
      const int have = N - (v0 + lc);
      old[i] = a.base && rows[i] >= 0 ? load_elems(a.base + rows[i] * a.ldb + v0 + lc, have, have) : slot_t{0u, 0u, 0u, 0u};
    }
    f32x4_t sum[4][2];
#pragma unroll
    for (int v = 0; v < 4; ++v) sum[v][0] = sum[v][1] = f32x4_t{-0.0f, -0.0f, -0.0f, -0.0f};  // (x + -0 is x)
    unsigned left = 0xffffffffu;
    for (int id = tile.next(left, n); id < n; id = tile.next(left, n)) {
      const T *up = a.up + (long)id * N * R;
      slot_t fa[4][NF];
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          const int col = v0 + v * 16 + c, k = i * CHUNK + kq;
          if constexpr (ACROSS) {
            union {
              slot_t s;
              T e[VEC];
            } o;
            o.s = slot_t{0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if (col < N && k + e < R) o.e[e] = up[(long)(k + e) * N + col];
            fa[v][i] = o.s;
          } else {
            fa[v][i] = load_elems(up + (long)col * R + k, col < N ? R - k : 0, (long)(N - col) * R - k);
          }
        }
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4_t acc = {};
#pragma unroll
          for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) Mma<T>::add(acc, fa[v][i], fu[t][i][p]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[v][t][e] = key[t] == id ? acc[e] : sum[v][t][e];
        }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4_t *>(&turn[wave][t * 16 + c][v * 16 + q * 4]) = sum[v][t];
    wave_sync();
#pragma unroll
    for (int i = 0; i < MOVES; ++i) {
      if (rows[i] < 0) continue;
      union {
        slot_t s;
        T t[VEC];
      } o;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o.t[e] = from_f32<T>(slot_elem<T>(old[i], e) + turn[wave][i * ROWS + lr][lc + e]);
      T *dst = a.out + rows[i] * a.ldo + v0 + lc;
      if (v0 + lc + VEC <= N) {
        *reinterpret_cast<typename SlotOf<T>::type *>(dst) = o.s;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v0 + lc + e < N) dst[e] = o.t[e];
      }
    }
    wave_sync();
  }
}

// A gradient that is a sum over rows, of all adapters: G[a][v][r] = f_a sum_m d[m][v] w[m][r], w as Transposed; and (template
// INNER) part[v block][position][r] = sum over the block's v of d[m][v] up[a][v][r].
// Workgroups: chunks of positions x blocks of columns.  A chunk may hold many adapters and an adapter lie in many chunks: where
// it has a chunk for itself or shares it whole, G is written, else a part, which adapter_join_kernel sums up.
template <typename T>
struct GradArgs {
  AdapterRows rows;
  const int32_t *start;
  const T *d;
  long ldd;
  Transposed<T> w;
  const T *up;
  const float *scale;  // may be nullptr
  float *G;            // [n][N][R], or (across) [n][R][N]
  float *split;        // [2 chunks][N][R]
  float *part;         // [blocks of columns][M][R]
  int N, R, chunk;     // positions of a chunk
  bool across;
};

// Part of adapter a in chunk i, in units of N R: an adapter that starts in front of the chunk has the first, one that goes on
// behind it the second.
__device__ inline long adapter_split(int a_start, int chunk, int i) { return 2L * i + (a_start < i * chunk ? 0 : 1); }

template <typename T, int JT, int VT, bool INNER>
__global__ void __launch_bounds__(512) adapter_grad_kernel(const GradArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, TILE = ADAPTER_TILE, WAVES = 8, COLS = 16 * VT, PARTS = Transposed<T>::PARTS;
  constexpr int PITCH = COLS + 16 / sizeof(T), LANES = COLS / VEC, ROWS = 64 / LANES, MOVES = TILE / ROWS;
  constexpr int MK = TILE / CHUNK, VK = COLS / CHUNK;  // slots of the rows, of the columns
  __shared__ __align__(16) T buf[WAVES][TILE][PITCH];
  __shared__ float red[INNER ? WAVES : 1][INNER ? TILE : 1][INNER ? JT * 16 + 4 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int N = a.N, R = a.R, n = a.rows.n, block = blockIdx.x, ci = blockIdx.y;
  const int v0 = (block * WAVES + wave) * COLS;
  const int present = a.start[n], end_chunk = min((ci + 1) * a.chunk, present);
  const int lr = lane / LANES, lc = lane % LANES * VEC, have = N - (v0 + lc);
  T(*my)[PITCH] = buf[wave];
  for (int pos = ci * a.chunk; pos < end_chunk;) {
    const int id = __builtin_amdgcn_readfirstlane(a.rows.key(a.rows.row(pos)));
    const int a_start = a.start[id], a_end = a.start[id + 1], end = min(a_end, end_chunk);
    slot_t fup[INNER ? VK : 1][INNER ? JT : 1];
    if constexpr (INNER) {
      const T *up = a.up + (long)id * N * R;
#pragma unroll
      for (int k = 0; k < VK; ++k)
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          union {
            slot_t s;
            T e[VEC];
          } o;
          o.s = slot_t{0u, 0u, 0u, 0u};
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int v = v0 + k * CHUNK + q * VEC + e, r = j * 16 + c;
            if (v < N && r < R) o.e[e] = up[(long)v * R + r];
          }
          fup[k][j] = o.s;
        }
    }
    f32x4_t g[VT][JT] = {};
    for (; pos < end; pos += TILE) {
      const int here = min(TILE, end - pos);
      const int row_of = a.rows.row(pos + min(lane & 31, here - 1));
#pragma unroll
      for (int i = 0; i < MOVES; ++i) {
        const int m = i * ROWS + lr, row = __shfl(row_of, m);
        *reinterpret_cast<slot_t *>(&my[m][lc]) = load_elems(a.d + row * a.ldd + v0 + lc, m < here ? have : 0, have);
      }
      wave_sync();
      slot_t fw[MK][JT][PARTS];
#pragma unroll
      for (int k = 0; k < MK; ++k)
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
          for (int p = 0; p < PARTS; ++p) {
            const int r = j * 16 + c, m = k * CHUNK + q * VEC;
            const T *src = a.w.at + ((long)p * R + (r < R ? r : 0)) * a.w.Mp + pos + m;
            fw[k][j][p] = load_elems(src, r < R ? here - m : 0, VEC);
          }
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int k = 0; k < MK; ++k) {
          union {
            slot_t s;
            T e[VEC];
          } o;
#pragma unroll
          for (int e = 0; e < VEC; ++e) o.e[e] = my[k * CHUNK + q * VEC + e][v * 16 + c];
#pragma unroll
          for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) Mma<T>::add(g[v][j], fw[k][j][p], o.s);
        }
      if constexpr (INNER) {
        f32x4_t acc[JT][2] = {};
#pragma unroll
        for (int k = 0; k < VK; ++k)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const slot_t fd = *reinterpret_cast<const slot_t *>(&my[t * 16 + c][k * CHUNK + q * VEC]);
#pragma unroll
            for (int j = 0; j < JT; ++j) Mma<T>::add(acc[j][t], fup[k][j], fd);
          }
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
          for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4_t *>(&red[wave][t * 16 + c][j * 16 + q * 4]) = acc[j][t];
        __syncthreads();
        for (int i = threadIdx.x; i < here * R; i += 512) {
          const int m = i / R, r = i % R;
          float s = 0.0f;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) s += red[w][m][r];
          a.part[((long)block * a.rows.M + pos + m) * R + r] = s;
        }
        __syncthreads();
      }
      wave_sync();
    }
    pos = end;
    const bool whole = a_start >= ci * a.chunk && a_end == end;
    float *G = whole ? a.G + (long)id * N * R : a.split + adapter_split(a_start, a.chunk, ci) * N * R;
    const float f = whole && a.scale ? a.scale[id] : 1.0f;
    const bool across = whole && a.across;
#pragma unroll
    for (int v = 0; v < VT; ++v) {
      const int col = v0 + v * 16 + c;
      if (col >= N) continue;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = j * 16 + q * 4 + e;
          if (r < R) G[across ? (long)r * N + col : (long)col * R + r] = g[v][j][e] * f;
        }
    }
  }
}

// Sums the parts of the adapters that lie in several chunks; zeros for those without rows.
struct JoinArgs {
  const int32_t *start;
  const float *split, *scale;
  float *G;
  int N, R, chunk, n;
  bool across;
};
static __global__ void __launch_bounds__(256) adapter_join_kernel(const JoinArgs a) {
  const long size = (long)a.N * a.R;
  for (int id = blockIdx.y; id < a.n; id += gridDim.y) {
    const int start = a.start[id], end = a.start[id + 1];
    const int c0 = start / a.chunk, c1 = end > start ? (end - 1) / a.chunk : c0;
    if (end > start && c0 == c1) continue;
    const float f = a.scale ? a.scale[id] : 1.0f;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < size; i += (long)gridDim.x * 256) {
      float s = 0.0f;
      if (end > start)
        for (int c = c0; c <= c1; ++c) s += a.split[adapter_split(start, a.chunk, c) * size + i];
      s *= f;
      a.G[(long)id * size + (a.across ? i % a.R * a.N + i / a.R : i)] = end > start ? s : 0.0f;
    }
  }
}

// dinner [position][R] = f_a sum over the blocks of columns, in order; and transposed.
template <typename T>
struct DinnerArgs {
  AdapterRows rows;
  const int32_t *start;
  const float *part, *scale;
  float *dinner;
  Transposed<T> tr;
  int blocks, R;
};
template <typename T>
__global__ void __launch_bounds__(256) adapter_dinner_kernel(const DinnerArgs<T> a) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x, size = (long)a.rows.M * a.R;
  const int pos = (int)(i / a.R), r = (int)(i % a.R);
  if (pos >= a.start[a.rows.n]) return;
  float s = 0.0f;
  for (int b = 0; b < a.blocks; ++b) s += a.part[b * size + i];
  if (a.scale) s *= a.scale[a.rows.key(a.rows.row(pos))];
  a.dinner[i] = s;
  a.tr.put(r, pos, s);
}

}  // namespace rnnlm_dev
