// Low-rank adapters of many texts beside a shared projection, forward and backward.  Row m has x[K] and belongs to adapter
// a = ids[m], or to none:
//   inner = down[a] x (R numbers),                 out = base + f_a up[a] inner
//   dinner = f_a up[a]^T dout,  dup[a] = f_a sum_m dout inner^T,  ddown[a] = sum_m dinner x^T,  dx = down[a]^T dinner
// Rows are taken in the order of their adapters (adapter_order_kernel), 32 positions of that order a tile; a tile may hold rows
// of several adapters, each of which is multiplied with the whole tile and kept where it belongs (the products are few beside
// the bytes of base, out and dout, which bound all of this).
// Products: 16 x 16 tiles of the matrix cores.  bf16: inner and dinner are fp32 and go in as two parts (products that end in a
// bf16 number; 2^-17) or three (gradients in fp32; 2^-26), everything else is bf16 already; fp32: the fp32 instruction.
#pragma once
#include "rows.h"

namespace rnnlm_dev {

constexpr int ADAPTER_TILE = 32;   // rows of a tile
constexpr int ADAPTER_R_MAX = 64;

struct AdapterRows {
  const int32_t *ids, *perm, *sorted;  // rows in the order of their adapters, and those; perm = nullptr: rows as they are
  int M, n;
  // adapter of a row; n: none
  __device__ int key(int row) const {
    const int a = ids[row];
    return a >= 0 && a < n ? a : n;
  }
  __device__ int row(int pos) const { return perm ? perm[pos] : pos; }
  __device__ int key_at(int pos) const { return perm ? sorted[pos] : key(pos); }
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
// Zeros in place of the first `gone` elements of a slot.
template <typename T>
__device__ inline slot_t last_elems(slot_t s, int gone) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) s[i] = i < gone ? 0u : s[i];
    else s[i] = 2 * i + 1 < gone ? 0u : 2 * i < gone ? s[i] & 0xffff0000u : s[i];
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
// Up to `left` elements from p on, zeros behind them; as many in front of them may be read as are missing of a slot (left < 0: p lies
// behind the end).  One load and no branch: element by element, the last columns were what small calls waited for.
template <typename T>
__device__ inline slot_t load_last(const T *p, long left) {
  constexpr int N = SlotOf<T>::N;
  const long back = left < N ? N - left : 0;
  const slot_t s = *reinterpret_cast<const typename SlotOf<T>::type *>(p - back);
  const int bits = (int)min(back, (long)N) * (128 / N);
  const unsigned long long lo = s[0] | (unsigned long long)s[1] << 32, hi = s[2] | (unsigned long long)s[3] << 32;
  const unsigned long long low = bits == 0 ? lo : bits < 64 ? lo >> bits | hi << (64 - bits) : bits < 128 ? hi >> (bits - 64) : 0;
  const unsigned long long high = bits < 64 ? hi >> bits : 0;
  return slot_t{(unsigned)low, (unsigned)(low >> 32), (unsigned)high, (unsigned)(high >> 32)};
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

// bf16 parts of a number whose products are summed in fp32.
template <typename T>
constexpr int GRAD_PARTS = sizeof(T) == 2 ? 3 : 1;

// perm: the rows ordered by (adapter, row), rows without one last; sorted: their adapters; start[a]: first position of adapter
// a, start[n]: of those rows.  64 questions a workgroup, each answered by counting smaller keys (equal ones of earlier rows,
// too): M (M + n) / 64 comparisons of a wave.  2560 rows, 16 adapters 7 us, 900 rows 5.
static __global__ void __launch_bounds__(1024) adapter_order_kernel(const AdapterRows rows, int32_t *__restrict__ perm,
                                                                    int32_t *__restrict__ sorted, int32_t *__restrict__ start,
                                                                    int32_t *range_flag) {
  constexpr int KEYS = 4096;
  __shared__ __align__(16) int32_t keys[KEYS];
  __shared__ int32_t cnt[16][64];
  const int lane = threadIdx.x & 63, slice = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), M = rows.M, first = blockIdx.x * 64;
  const int q = first + lane;
  const int mine = q < M ? rows.key(q) : q - M;
  if (slice == 0 && q < M && rows.ids[q] >= rows.n && range_flag) *range_flag = 1;
  int rank = 0;
  for (int base = 0; base < M; base += KEYS) {
    const int n = min(KEYS, M - base);
#pragma unroll
    for (int j = 0; j < KEYS / 1024; ++j) {
      const int i = j * 1024 + threadIdx.x;
      keys[i] = i < n ? rows.key(base + i) : 0x7fffffff;
    }
    __syncthreads();
    // 64 keys at a time: those in front of this workgroup's own rows count where they are equal, too
    for (int i = slice * 64; i < n; i += 1024) {
      const int4 *k = reinterpret_cast<const int4 *>(keys + i);
      const int below = q < M && base + i < first ? mine + 1 : mine;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int4 v = k[j];
        rank += (v.x < below) + (v.y < below) + (v.z < below) + (v.w < below);
      }
    }
    __syncthreads();
  }
  cnt[slice][lane] = rank;
  __syncthreads();
  if (slice != 0) return;
  int r = 0;
#pragma unroll
  for (int g = 0; g < 16; ++g) r += cnt[g][lane];
  if (q < M) {  // equal ones among this workgroup's own rows
#pragma unroll 8
    for (int j = 0; j < 63; ++j) r += __builtin_amdgcn_readlane(mine, j) == mine && j < lane;
  }
  if (q < M) perm[r] = q, sorted[r] = mine;
  else if (q - M <= rows.n) start[q - M] = r;
}

// What a wave knows of a tile of up to 32 rows from position `first` on: lane l < 32 (and l + 32) the l-th row and its adapter.
struct AdapterTile {
  int row, key;  // -1, n: behind the last row
  __device__ AdapterTile(const AdapterRows &r, int first, int rows) {
    const int l = threadIdx.x & 31, pos = first + l;
    const bool in = l < rows && pos < r.M;
    row = in ? r.row(pos) : -1;
    key = in ? r.key_at(pos) : r.n;
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

// inner: a workgroup a tile and one of its adapters (blockIdx.y-th); K over the waves, joined in LDS in order.  A chain of
// latencies (a tile has 32 K numbers): 2560 x 1024 bf16, R = 16, 8 adapters 6.6 us, 128 rows of as many adapters 7.0.  Chunks
// behind the end of short rows are branched around: 164 rows of K = 387, R = 58 9.1 us, 16.4 where the last one was loaded again
// in their place (bf16 rows of odd length: a load takes its lanes one by one).
template <typename T, int RT>
__global__ void __launch_bounds__(512) adapter_inner_kernel(const InnerArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, WAVES = 8, TILE = ADAPTER_TILE;
  __shared__ float part[WAVES][RT * 16][TILE + 1];  // (read down its columns)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const AdapterTile tile(a.rows, blockIdx.x * TILE, TILE);
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
  // Rows of other adapters, and r >= R, go along: their products are dropped.
  const T *xs[2], *ds[RT];
#pragma unroll
  for (int t = 0; t < 2; ++t) xs[t] = a.x + max(0, __shfl(tile.row, t * 16 + c)) * a.ldx + q * VEC;
#pragma unroll
  for (int r = 0; r < RT; ++r) ds[r] = a.down + ((long)id * a.R + min(r * 16 + c, a.R - 1)) * a.K + q * VEC;
  f32x4_t acc[RT][2] = {};
  typedef typename SlotOf<T>::type Slot;
  const int whole = a.K / CHUNK * CHUNK;
  constexpr int AHEAD = 4;  // chunks whose loads are under way together
  for (int k0 = wave * CHUNK; k0 < whole; k0 += AHEAD * WAVES * CHUNK) {
    slot_t fx[AHEAD][2], fd[AHEAD][RT];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int k = k0 + u * WAVES * CHUNK;
      if (k < whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t) fx[u][t] = *reinterpret_cast<const Slot *>(xs[t] + k);
#pragma unroll
        for (int r = 0; r < RT; ++r) fd[u][r] = *reinterpret_cast<const Slot *>(ds[r] + k);
      } else {  // (behind the end: nothing is added)
#pragma unroll
        for (int t = 0; t < 2; ++t) fx[u][t] = slot_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < RT; ++r) fd[u][r] = slot_t{0u, 0u, 0u, 0u};
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < 2; ++t) Mma<T>::add(acc[r][t], fd[u][r], fx[u][t]);
    }
  }
  if (whole < a.K && wave == whole / CHUNK % WAVES) {
    const int have = a.K - whole - q * VEC;
    slot_t fx[2], fd[RT];
    if (a.K >= VEC) {
#pragma unroll
      for (int t = 0; t < 2; ++t) fx[t] = load_last(xs[t] + whole, have);
#pragma unroll
      for (int r = 0; r < RT; ++r) fd[r] = load_last(ds[r] + whole, have);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) fx[t] = load_elems(xs[t], have, have);
#pragma unroll
      for (int r = 0; r < RT; ++r) fd[r] = load_elems(ds[r], have, have);
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
  const float *inner;  // [M][R]
  const T *up;         // [n][N][R]
  const float *scale;  // may be nullptr
  const T *base;       // may be nullptr (zeros), may be out
  T *out;
  long ldb, ldo;
  int N, R, blocks;    // blocks of columns of a wave
  int tile;            // rows of a tile, at most 32
};

// out = base + f up inner: a wave a tile and 16 VT columns, `blocks` times; through LDS so that base and out move in whole lines.
// Bound by HBM: 2560 x 64000 bf16, R = 16, 8 adapters 140 us (676 MB, 4.8 TB/s; workgroups dealt so that each XCD has its own
// columns took as long), 128 rows of as many adapters 50 where up stays in the memory-side cache, 62 where it does not (295 MB, 4.8
// TB/s), fp32 113 (576 MB, 5.1 TB/s).  Every tile reads all of its adapter's up again, mostly out of the memory-side cache, which
// bounds high ranks: of the 8 adapters above R = 64 (2560 rows) bf16 fetches 841 MB in place of 394, 202 us, fp32 1704 MB in place
// of 786, 478 us.
// NF: operand slots of R.  PACKED (bf16, R <= 16): both parts of inner in one product, beside one another.
template <typename T, int NF, bool PACKED, int VT>
__global__ void __launch_bounds__(256, 2) adapter_outer_kernel(const OuterArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, TILE = ADAPTER_TILE, COLS = 16 * VT, PITCH = COLS + 4;
  constexpr int PARTS = sizeof(T) == 4 || PACKED ? 1 : 2, LANES = COLS / VEC, ROWS = 64 / LANES, MOVES = TILE / ROWS;
  __shared__ float turn[4][TILE][PITCH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int n = a.rows.n, N = a.N, R = a.R;
  const AdapterTile tile(a.rows, blockIdx.x * a.tile, a.tile);
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
    const float *u = a.inner + (long)row * R;
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
  const bool wide = N >= COLS, slots = R % VEC == 0;
  typedef typename SlotOf<T>::type Slot;
  // the last block starts early enough not to stick out; its columns from `from` on are written
  const int first = (blockIdx.y * 4 * a.blocks + wave) * COLS, end = min(N, first + 4 * a.blocks * COLS);
  const auto start = [&](int from) { return wide ? min(from, N - COLS) : from; };
  const auto load_base = [&](int v0, slot_t (&old)[MOVES]) {
#pragma unroll
    for (int i = 0; i < MOVES; ++i) {
      const T *at = a.base + max(rows[i], 0) * a.ldb + v0 + lc;
      if (!a.base) old[i] = slot_t{0u, 0u, 0u, 0u};
      else if (!wide) old[i] = load_elems(at, N - (v0 + lc), N - (v0 + lc));
      else old[i] = *reinterpret_cast<const Slot *>(at);
    }
  };
  // (columns behind the last one, of narrow arrays: the last one again, dropped)
  const auto load_up = [&](int v0, int id, slot_t (&fa)[VT][NF]) {
    const T *up = a.up + (long)id * N * R;
    // (whole slots of every lane lie in up, all of the block's at once: no branch stands between the loads)
    if (slots || (long)(N - v0 - COLS) * R + 1 >= VEC) {
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int i = 0; i < NF; ++i)
          fa[v][i] = *reinterpret_cast<const Slot *>(up + (unsigned)(min(v0 + v * 16 + c, N - 1) * R + min(i * CHUNK + kq, slots ? R - VEC : R - 1)));
    } else {
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          const int col = min(v0 + v * 16 + c, N - 1), k = i * CHUNK + kq;
          fa[v][i] = load_elems(up + (unsigned)(col * R + min(k, R - 1)), R - k, (long)(N - col) * R - k);
        }
    }
  };
  if (first >= N) return;  // (nothing is shared between the waves)
  unsigned left = 0xffffffffu;
  const int id0 = tile.next(left, n);
  const unsigned left0 = left;
  constexpr bool EARLY = NF == 1 || sizeof(T) == 2;  // up is requested a step ahead, too (where registers are left for it)
  slot_t old[2][MOVES], fa[EARLY ? 2 : 1][VT][NF];
  load_base(start(first), old[0]);
  if (EARLY && id0 < n) load_up(start(first), id0, fa[0]);
  for (int from = first; from < end; from += 4 * COLS) {
    const int v0 = start(from), after = from + 4 * COLS;
    if (after < end) load_base(start(after), old[1]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
      if (key[t] >= n) {
#pragma unroll
        for (int v = 0; v < VT; ++v)  // (x + -0 is x)
          *reinterpret_cast<f32x4_t *>(&turn[wave][t * 16 + c][v * 16 + q * 4]) = f32x4_t{-0.0f, -0.0f, -0.0f, -0.0f};
      }
    left = left0;
    for (int id = id0; id < n;) {
      const int next = tile.next(left, n);
      if constexpr (!EARLY) load_up(v0, id, fa[0]);
      else if (next < n) load_up(v0, next, fa[1]);
      else if (after < end) load_up(start(after), id0, fa[1]);
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4_t acc = {};
#pragma unroll
          for (int i = 0; i < NF; ++i) {
            const slot_t f = R % CHUNK == 0 ? fa[0][v][i] : first_elems<T>(fa[0][v][i], R - (i * CHUNK + kq));
#pragma unroll
            for (int p = 0; p < PARTS; ++p) Mma<T>::add(acc, f, fu[t][i][p]);
          }
          if (key[t] == id) *reinterpret_cast<f32x4_t *>(&turn[wave][t * 16 + c][v * 16 + q * 4]) = acc;
        }
#pragma unroll
      for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int i = 0; i < NF; ++i) fa[0][v][i] = fa[EARLY][v][i];
      id = next;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < MOVES; ++i) {
      union {
        slot_t s;
        T t[VEC];
      } o;
#pragma unroll
      for (int e = 0; e < VEC; ++e) o.t[e] = from_f32<T>(slot_elem<T>(old[0][i], e) + turn[wave][i * ROWS + lr][lc + e]);
      const int col = v0 + lc;
      T *dst = a.out + max(rows[i], 0) * a.ldo + col;
      if (rows[i] < 0) {
      } else if (col >= from && col + VEC <= N) {
        *reinterpret_cast<Slot *>(dst) = o.s;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (col + e >= from && col + e < N) dst[e] = o.t[e];
      }
      old[0][i] = old[1][i];
    }
    wave_sync();
  }
}

// VEC consecutive rows from k0 + (l / 16) VEC on of column c0 + l % 16 of a tile in LDS: an operand whose k are the rows.
// bf16: the transposing read; of each 16 lanes, lane s points at 4 elements of row s / 4 and gets 4 rows of its column.
template <typename T>
__device__ inline slot_t across(const T *tile, int pitch, int k0, int c0) {
  const int lane = threadIdx.x & 63, q = lane >> 4, c = lane & 15;
  if constexpr (sizeof(T) == 2) {
    typedef short s16x4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4_t *lds_ptr_t;
    const T *p = tile + (k0 + q * 8 + (c >> 2)) * pitch + c0 + 4 * (c & 3);
    union {
      s16x4_t h[2];
      slot_t s;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p + 4 * pitch));
    return u.s;
  } else {
    const T *p = tile + (k0 + q * 4) * pitch + c0 + c;
    return slot_t{__builtin_bit_cast(unsigned, p[0]), __builtin_bit_cast(unsigned, p[pitch]), __builtin_bit_cast(unsigned, p[2 * pitch]),
                  __builtin_bit_cast(unsigned, p[3 * pitch])};
  }
}
// VEC numbers as an operand: of bf16 PARTS operands, the numbers' first parts, second ones, ...; of fp32 the numbers themselves.
template <typename T, int PARTS>
__device__ inline void operand_parts(const float (&v)[Mma<T>::VEC], slot_t (&s)[PARTS]) {
  union {
    slot_t s[PARTS];
    T e[PARTS][Mma<T>::VEC];
  } o;
#pragma unroll
  for (int e = 0; e < Mma<T>::VEC; ++e) {
    if constexpr (sizeof(T) == 4) {
      o.e[0][e] = v[e];
    } else {
      bf16_t p[PARTS];
      bf16_parts<PARTS>(v[e], p);
#pragma unroll
      for (int i = 0; i < PARTS; ++i) o.e[i][e] = p[i];
    }
  }
#pragma unroll
  for (int i = 0; i < PARTS; ++i) s[i] = o.s[i];
}

// A wave's 32 rows x COLS columns of an array, row by row by way of registers (requested early) into LDS.  The last block of
// columns starts early enough not to stick out (what it has in common with the one in front is left out where it would count
// twice); only arrays narrower than a block are fetched element by element.
template <typename T, int COLS, bool NARROW>
struct WaveTile {
  static constexpr int VEC = Mma<T>::VEC, LANES = COLS / VEC, ROWS = 64 / LANES, MOVES = ADAPTER_TILE / ROWS, PITCH = COLS + 16 / sizeof(T);
  slot_t raw[MOVES];
  int rows;  // of lane l, the row of l % 32 (the last ones may repeat one that is there)
  __device__ static int start(int v0, int N) { return max(0, min(v0, N - COLS)); }
  __device__ void load(const T *d, long ld, int rows_, int v0) {
    const int lane = threadIdx.x & 63;
    rows = rows_;
    if constexpr (!NARROW) {
      const T *at = d + v0 + lane % LANES * VEC;
#pragma unroll
      for (int i = 0; i < MOVES; ++i)
        raw[i] = *reinterpret_cast<const typename SlotOf<T>::type *>(at + __shfl(rows, i * ROWS + lane / LANES) * ld);
    }
  }
  // kept: of this lane's columns, ones
  __device__ void keep(const slot_t &kept) {
#pragma unroll
    for (int i = 0; i < MOVES; ++i) raw[i] &= kept;
  }
  // zeros in place of the rows from `here` on (of narrow arrays: and of the columns in front of `from`)
  __device__ void store(T (*tile)[PITCH], const T *d, long ld, int here, int v0, int from, int N) const {
    const int lane = threadIdx.x & 63;
    if constexpr (!NARROW) {
#pragma unroll
      for (int i = 0; i < MOVES; ++i) {
        const int m = i * ROWS + lane / LANES;
        *reinterpret_cast<slot_t *>(&tile[m][lane % LANES * VEC]) = m < here ? raw[i] : slot_t{0u, 0u, 0u, 0u};
      }
    } else {
      for (int i0 = 0; i0 < ADAPTER_TILE * COLS; i0 += 8 * 64) {
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = i0 + j * 64 + lane, m = i / COLS, col = v0 + i % COLS;
          const long row = __shfl(rows, m);
          v[j] = m < here && col >= from && col < N ? d[row * ld + col] : from_f32<T>(0.0f);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[(i0 + j * 64 + lane) / COLS][(i0 + j * 64 + lane) % COLS] = v[j];
      }
    }
  }
};

// Gradients that are sums over rows.  Workgroups: chunks of positions x blocks of columns.  A chunk may hold many adapters and
// an adapter lie in many chunks: the one it starts in writes its gradient (finished, where all of it lies there), any other
// has one such adapter, its first, and writes a part of its own; adapter_join_kernel sums up.

constexpr int ADAPTER_GRAD_WAVES = 8, ADAPTER_CHUNK = 1024;  // most positions of a chunk

// A chunk's tiles, each of rows of one adapter: first position (in the chunk), rows less one, adapter.
struct TileList {
  int row[ADAPTER_CHUNK], tile[ADAPTER_CHUNK], of_wave[2][ADAPTER_GRAD_WAVES];
  __device__ int first(int i) const { return __builtin_amdgcn_readfirstlane(tile[i]) & 1023; }
  __device__ int rows(int i) const { return (__builtin_amdgcn_readfirstlane(tile[i]) >> 10 & 31) + 1; }
  __device__ int adapter(int i) const { return __builtin_amdgcn_readfirstlane(tile[i]) >> 15; }
};
// Fills the list for positions begin .. end - 1 (more than none, at most ADAPTER_CHUNK): a workgroup of ADAPTER_GRAD_WAVES waves.
// Returns the number of tiles.
__device__ inline int list_tiles(const AdapterRows &rows, const int32_t *start, int begin, int end, TileList &list) {
  constexpr int THREADS = 64 * ADAPTER_GRAD_WAVES;
  static_assert(ADAPTER_CHUNK == 2 * THREADS, "two positions a thread");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int entry[2];
  unsigned long long heads[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int pos = begin + j * THREADS + threadIdx.x;
    const bool in = pos < end;
    const int p = in ? pos : end - 1, key = rows.sorted[p], row = rows.perm[p];
    const int from = max(start[key], begin), to = min(start[key + 1], end);
    list.row[pos - begin] = row;  // (behind the end: the last row)
    entry[j] = (pos - begin) | (min(ADAPTER_TILE, to - p) - 1) << 10 | key << 15;
    heads[j] = __ballot(in && ((p - from) & (ADAPTER_TILE - 1)) == 0);
    if (lane == 0) list.of_wave[j][wave] = __popcll(heads[j]);
  }
  __syncthreads();
  int at = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int mine = at;
#pragma unroll
    for (int w = 0; w < ADAPTER_GRAD_WAVES; ++w) {
      mine += w < wave ? list.of_wave[j][w] : 0;
      at += list.of_wave[j][w];
    }
    if (heads[j] >> lane & 1) list.tile[mine + __popcll(heads[j] & ((1ull << lane) - 1))] = entry[j];
  }
  __syncthreads();
  return at;
}

template <typename T>
struct GradArgs {
  AdapterRows rows;
  const int32_t *start;
  const T *d;
  long ldd;
  const float *inner;  // [M][R]
  const T *up;
  const float *scale;  // may be nullptr
  float *G;            // [n][N][R]
  float *split;        // [chunks][N][R]
  float *part;         // [blocks of columns][M][R]
  int N, R, chunk;     // positions of a chunk
};

// dup[a][v][r] = f_a sum_m dout[m][v] inner[m][r], and of every block of columns part[position][r] = sum_v dout[m][v] up[a][v][r]:
// dout is read once.  2560 x 64000 bf16, R = 32, 16 adapters 129 us: 397 MB read (328 of them dout, 65 up), 172 written (131
// of gradient, 41 of part), 4.4 TB/s.  900 x 33278 fp32, R = 5, 7 adapters 48: fp32 products of 16 x 16 tiles for R = 5, LDS and
// barriers.  NARROW: fewer columns than a wave's.
// Two workgroups to a compute unit where registers and LDS allow it (VT of half the size, R <= 16): each waits less for the other
// waves of its own.
template <typename T>
constexpr bool grad_by_two(int JT, int VT) { return JT == 1 && VT * sizeof(T) <= 8; }
template <typename T, int JT, int VT, bool NARROW>
__global__ void __launch_bounds__(64 * ADAPTER_GRAD_WAVES, grad_by_two<T>(JT, VT) ? 4 : 2) adapter_grad_kernel(const GradArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, TILE = ADAPTER_TILE, WAVES = ADAPTER_GRAD_WAVES, COLS = 16 * VT;
  constexpr int THREADS = 64 * WAVES, PARTS = GRAD_PARTS<T>, MK = TILE / CHUNK, VK = COLS / CHUNK;  // slots of the rows, of the columns
  constexpr int REDS = JT <= 2 && !grad_by_two<T>(JT, VT) ? 2 : 1;  // (as many as LDS holds)
  constexpr int WIDTH = JT == 3 ? 64 : JT * 16, STEP = THREADS / WIDTH, EACH = TILE / STEP;  // a tile's inner numbers over the threads
  constexpr bool EARLY = JT <= 2;        // the next adapter's up has registers of its own
  typedef WaveTile<T, COLS, NARROW> Tile;
  __shared__ __align__(16) T buf[WAVES][TILE][Tile::PITCH];
  __shared__ __align__(16) float red[REDS][WAVES][TILE][JT * 16 + 4];
  __shared__ __align__(16) T turned[2][PARTS][JT * 16][TILE + 16 / sizeof(T)];  // inner of two tiles, its parts, [r][m]
  __shared__ TileList list;
  // Ones where a wave's columns count.  What it has in common with the wave in front is zero in up and in dout: 0 times an infinity
  // is no number.  Read from here for every tile, without a branch: masks held in registers made the kernels spill, and a branch
  // for the last waves cost all others 5% (900 x 33278 bf16, R = 16: 59.7 us without zeros in dout, 60.8 so, 62.9 with the branch).
  __shared__ slot_t counted[WAVES][Tile::LANES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int N = a.N, R = a.R, n = a.rows.n, block = blockIdx.x, ci = blockIdx.y;
  const int from = (block * WAVES + wave) * COLS, v0 = Tile::start(from, N);  // the columns from `from` on count
  const int end_chunk = min((ci + 1) * a.chunk, a.start[n]);
  T(*my)[Tile::PITCH] = buf[wave];
  const int tr = threadIdx.x % WIDTH, tm = threadIdx.x / WIDTH;  // this thread's r, and first m
  const int chunk0 = ci * a.chunk;
  if (chunk0 >= end_chunk) return;
  if (lane < Tile::LANES) counted[wave][lane] = last_elems<T>(slot_t{~0u, ~0u, ~0u, ~0u}, from - (v0 + lane * VEC));
  const int count = list_tiles(a.rows, a.start, chunk0, end_chunk, list);
  // What a tile needs of memory, requested two tiles ahead (behind the last one: that again, so that no branch stands between
  // the requests and the waits can count them).
  struct Ahead {
    Tile tile;
    float in[EACH];
  };
  const auto request = [&](Ahead &x, int i) {
    const int rows = list.row[min(list.first(min(i, count - 1)) + (lane & 31), ADAPTER_CHUNK - 1)];
    x.tile.load(a.d, a.ldd, rows, v0);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const long row = __shfl(rows, tm + e * STEP);
      x.in[e] = a.inner[row * R + min(tr, R - 1)];
    }
  };
  const auto inner_store = [&](const Ahead &x, int i) {
    if (tr >= JT * 16) return;
    const int here = list.rows(min(i, count - 1));
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int m = tm + e * STEP;
      const float v = m < here ? x.in[e] : 0.0f;  // (r >= R: those rows of the product are dropped)
      if constexpr (PARTS == 1) {
        turned[i & 1][0][tr][m] = v;
      } else {
        bf16_t p[PARTS];
        bf16_parts<PARTS>(v, p);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) turned[i & 1][k][tr][m] = p[k];
      }
    }
  };
  // up[v][r], k = v (r >= R: anything).  A wave's part of up is contiguous: CHUNK R elements at a time, slot by slot first, then
  // turned by way of LDS.
  slot_t fup[VK][JT], fup2[EARLY ? VK : 1][EARLY ? JT : 1];
  const auto up_slot = [&](int j) { return min(j * 64 + lane, 4 * R - 1) * VEC; };
  const auto up_load = [&](auto &to, int id) {
    if constexpr (!NARROW) {
      const T *up = a.up + (long)id * N * R;
#pragma unroll
      for (int k = 0; k < VK; ++k)
#pragma unroll
        for (int j = 0; j < JT; ++j) to[k][j] = *reinterpret_cast<const typename SlotOf<T>::type *>(up + (unsigned)((v0 + k * CHUNK) * R + up_slot(j)));
    }
  };
  const auto up_turn = [&](const auto &raw, T *stage, int id) {
    constexpr int PITCH = JT * 16 + 16 / sizeof(T);
    static_assert(CHUNK * PITCH * sizeof(T) <= sizeof(red[0][0]), "a wave's share of red holds a step");
#pragma unroll
    for (int k = 0; k < VK; ++k) {
      if constexpr (!NARROW) {
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          const int i = up_slot(j);
          int v = i / R, r = i - v * R;
          if (R % VEC == 0) {
            *reinterpret_cast<slot_t *>(stage + v * PITCH + r) = raw[k][j];
          } else {
            union {
              slot_t s;
              T e[VEC];
            } o;
            o.s = raw[k][j];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              stage[v * PITCH + r] = o.e[e];
              r = r + 1 == R ? (++v, 0) : r + 1;
            }
          }
        }
      } else {
        const T *up = a.up + (long)id * N * R;
        const int v = v0 + k * CHUNK, there = max(0, min(CHUNK, N - v));
        for (int i = lane; i < CHUNK * R; i += 64)
          stage[i / R * PITCH + i % R] = i < there * R ? up[(unsigned)(v * R + i)] : from_f32<T>(0.0f);
      }
      wave_sync();
#pragma unroll
      for (int j = 0; j < JT; ++j) {
        fup[k][j] = across(stage, PITCH, 0, j * 16);
        fup[k][j] &= counted[wave][k * (CHUNK / VEC) + q];
      }
      wave_sync();
    }
  };
  f32x4_t g[VT][JT] = {};
  // What a tile leaves to be written, after the next one's rows have arrived and before further ones are requested (stores
  // count with the loads: behind them they would be waited for with them): the sums of `part`, and the gradient of an adapter
  // whose rows end.
  float sums[EACH];
  const auto write_sums = [&](int i) {
    float *part = a.part + ((long)block * a.rows.M + chunk0 + list.first(i)) * R;
    const int here = list.rows(i);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int m = tm + e * STEP;
      if (tr < R && m < here) part[m * R + tr] = sums[e];
    }
  };
  const auto write_gradient = [&](int id) {
    const int a_start = a.start[id], a_end = a.start[id + 1];
    const bool whole = a_start >= chunk0 && a_end <= end_chunk;
    float *G = a_start >= chunk0 ? a.G + (long)id * N * R : a.split + (long)ci * N * R;
    const float f = whole && a.scale ? a.scale[id] : 1.0f;
#pragma unroll
    for (int v = 0; v < VT; ++v) {
      const int col = v0 + v * 16 + c;
#pragma unroll
      for (int j = 0; j < JT; ++j) {
        const int r = j * 16 + q * 4;
        float *dst = G + (unsigned)(col * R + r);
        const f32x4_t x = g[v][j] * f;
        g[v][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (col < from || col >= N) {
        } else if (r + 4 <= R) {
          *reinterpret_cast<slot_fp32_t *>(dst) = __builtin_bit_cast(slot_t, x);
        } else {
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (r + e < R) dst[e] = x[e];
        }
      }
    }
  };
  int id = list.adapter(0);
  const auto step = [&](Ahead &x, const Ahead &y, int i) {
    const int here = list.rows(i), before = id;
    id = list.adapter(i);
    const int after = list.adapter(min(i + 1, count - 1));
    if constexpr (!NARROW) x.tile.keep(counted[wave][lane % Tile::LANES]);
    x.tile.store(my, a.d, a.ldd, here, v0, from, N);
    if (i > 0) write_sums(i - 1);
    if (i > 0 && id != before) write_gradient(before);
    if (i == 0 || id != before) {
      T *stage = reinterpret_cast<T *>(&red[REDS == 2 ? i & 1 : 0][wave][0][0]);
      if constexpr (EARLY) up_turn(fup2, stage, id);
      else up_turn(fup, stage, id);
    }
    if constexpr (EARLY)
      if (after != id) up_load(fup2, after);
    request(x, i + 2);
    wave_sync();
    f32x4_t acc[JT][2] = {};
#pragma unroll
    for (int k = 0; k < VK; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const slot_t fd = *reinterpret_cast<const slot_t *>(&my[t * 16 + c][k * CHUNK + q * VEC]);
#pragma unroll
        for (int j = 0; j < JT; ++j) Mma<T>::add(acc[j][t], fup[k][j], fd);
      }
    if constexpr (!EARLY)
      if (after != id) up_load(fup, after);
    float(*r_of)[TILE][JT * 16 + 4] = red[REDS == 2 ? i & 1 : 0];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4_t *>(&r_of[wave][t * 16 + c][j * 16 + q * 4]) = acc[j][t];
    // (an operand of inner at a time: all of them at once, and registers spill)
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int k = 0; k < MK; ++k) {
        slot_t fw[PARTS];  // inner[m][r]: k = m
#pragma unroll
        for (int p = 0; p < PARTS; ++p) fw[p] = *reinterpret_cast<const slot_t *>(&turned[i & 1][p][j * 16 + c][k * CHUNK + q * VEC]);
#pragma unroll
        for (int v = 0; v < VT; ++v) {
          const slot_t fd = across(&my[0][0], Tile::PITCH, k * CHUNK, v * 16);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) Mma<T>::add(g[v][j], fw[p], fd);
        }
      }
    inner_store(y, i + 1);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      sums[e] = 0.0f;
      if (tr < JT * 16) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sums[e] += r_of[w][tm + e * STEP][tr];
      }
    }
    if (REDS == 1) __syncthreads();
  };
  Ahead even, odd;
  if constexpr (EARLY) up_load(fup2, id);
  else up_load(fup, id);
  request(even, 0);
  request(odd, 1);
  inner_store(even, 0);
  __syncthreads();
  for (int i = 0; i < count; i += 2) {
    step(even, odd, i);
    if (i + 1 < count) step(odd, even, i + 1);
  }
  write_sums(count - 1);
  write_gradient(id);
}

template <typename T>
struct InputGradArgs {
  AdapterRows rows;
  const int32_t *start;
  const T *x, *down;
  const float *scale;  // may be nullptr
  const float *part;   // [blocks][M][R]
  float *G, *split;    // [n][R][K]; [chunks][R][K]
  T *dx;               // may be nullptr
  long ldx, lddx;
  int K, R, chunk, blocks;
};

// dinner of a tile from the blocks' parts, then ddown[a][r][k] = sum_m dinner[m][r] x[m][k] and dx[m][k] = sum_r down[a][r][k]
// dinner[m][r].  Sums of parts are formed once for every 512 columns of x.  A chain of latencies: 2560 x 1024 bf16, R = 32 12 us.
template <typename T, int JT, int VT, bool NARROW>
__global__ void __launch_bounds__(64 * ADAPTER_GRAD_WAVES) adapter_input_grad_kernel(const InputGradArgs<T> a) {
  constexpr int VEC = Mma<T>::VEC, CHUNK = Mma<T>::CHUNK, TILE = ADAPTER_TILE, WAVES = ADAPTER_GRAD_WAVES, COLS = 16 * VT;
  constexpr int THREADS = 64 * WAVES, PARTS = GRAD_PARTS<T>, PARTS2 = sizeof(T) == 2 ? 2 : 1, MK = TILE / CHUNK;
  constexpr int JK = (JT * 16 + CHUNK - 1) / CHUNK, RP = JK * CHUNK, DP = RP + 4;
  typedef WaveTile<T, COLS, NARROW> Tile;
  __shared__ __align__(16) T buf[WAVES][TILE][Tile::PITCH];
  __shared__ __align__(16) float dinner[TILE][DP];
  __shared__ float sums[THREADS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int K = a.K, R = a.R, n = a.rows.n, ci = blockIdx.y;
  const int from = (blockIdx.x * WAVES + wave) * COLS, k0 = Tile::start(from, K);  // the columns from `from` on count
  const int present = a.start[n], end_chunk = min((ci + 1) * a.chunk, present);
  T(*my)[Tile::PITCH] = buf[wave];
  // rows without an adapter
  if (a.dx)
    for (int pos = max(ci * a.chunk, present) + wave; pos < min((ci + 1) * a.chunk, a.rows.M); pos += WAVES) {
      const int row = a.rows.row(pos);
      const int end = min(K, (int)(blockIdx.x + 1) * WAVES * COLS);
      for (int k = blockIdx.x * WAVES * COLS + lane; k < end; k += 64) a.dx[row * a.lddx + k] = from_f32<T>(0.0f);
    }
  for (int i = threadIdx.x; i < TILE * DP; i += THREADS) dinner[i / DP][i % DP] = 0.0f;  // (behind R as well)
  __syncthreads();
  for (int pos = ci * a.chunk; pos < end_chunk;) {
    const int id = __builtin_amdgcn_readfirstlane(a.rows.key_at(pos));
    const int a_start = a.start[id], a_end = a.start[id + 1], end = min(a_end, end_chunk);
    const float f = a.scale ? a.scale[id] : 1.0f;
    const T *down = a.down + (long)id * R * K;
    const auto rows_at = [&](int at) { return a.rows.row(min(at + (lane & 31), a.rows.M - 1)); };
    Tile tile;  // of x, requested ahead
    tile.load(a.x, a.ldx, rows_at(pos), k0);
    slot_t fdown[VT][JK];  // down[r][k]: k of the product = r
    if (a.dx) {
#pragma unroll
      for (int j = 0; j < JK; j += MK) {
        const int r0 = j * CHUNK;
        Tile t;
        t.load(down, K, min(r0 + (lane & 31), R - 1), k0);
        t.store(my, down, K, R - r0, k0, k0, K);
        wave_sync();
#pragma unroll
        for (int i = 0; i < MK && j + i < JK; ++i)
#pragma unroll
          for (int v = 0; v < VT; ++v) fdown[v][j + i] = across(&my[0][0], Tile::PITCH, i * CHUNK, v * 16);
        wave_sync();
      }
    }
    f32x4_t g[VT][JT] = {};
    for (; pos < end; pos += TILE) {
      const int here = min(TILE, end - pos), rows = tile.rows;
      {  // the tile's part of every block is contiguous: groups of threads share out the blocks where it is short
        const int size = here * R;
        int width = 32;
        while (width < size && width < THREADS) width *= 2;
        const int groups = THREADS / width, group = threadIdx.x / width, at = threadIdx.x % width;
        const float *part = a.part + (long)pos * R;
        const long step = (long)a.rows.M * R;
        for (int i = at; i < size; i += width) {
          float s = 0.0f;
#pragma unroll 8
          for (int b = group; b < a.blocks; b += groups) s += part[b * step + i];
          if (groups == 1) dinner[i / R][i % R] = s * f;
          else sums[threadIdx.x] = s;
        }
        if (groups > 1) {
          __syncthreads();
          if (threadIdx.x < size) {
            float s = 0.0f;
            for (int i = 0; i < groups; ++i) s += sums[i * width + threadIdx.x];
            dinner[threadIdx.x / R][threadIdx.x % R] = s * f;
          }
        }
        for (int i = size + threadIdx.x; i < TILE * R; i += THREADS) dinner[i / R][i % R] = 0.0f;
      }
      tile.store(my, a.x, a.ldx, here, k0, k0, K);
      __syncthreads();
      if (pos + TILE < end) tile.load(a.x, a.ldx, rows_at(pos + TILE), k0);
#pragma unroll
      for (int j = 0; j < JT; ++j) {
        slot_t fw[MK][PARTS];  // dinner[m][r]: k = m
#pragma unroll
        for (int k = 0; k < MK; ++k) {
          float v[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[e] = dinner[k * CHUNK + q * VEC + e][j * 16 + c];
          operand_parts<T>(v, fw[k]);
        }
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
          for (int k = 0; k < MK; ++k) {
            const slot_t fx = across(&my[0][0], Tile::PITCH, k * CHUNK, v * 16);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) Mma<T>::add(g[v][j], fw[k][p], fx);
          }
      }
      wave_sync();
      if (a.dx) {  // by way of this wave's tile, so that rows move in whole lines
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          slot_t fd[JK][PARTS2];  // dinner[m][r]: k = r
#pragma unroll
          for (int j = 0; j < JK; ++j) {
            float v[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = dinner[t * 16 + c][j * CHUNK + q * VEC + e];
            operand_parts<T>(v, fd[j]);
          }
#pragma unroll
          for (int v = 0; v < VT; ++v) {
            f32x4_t acc = {};
#pragma unroll
            for (int j = 0; j < JK; ++j)
#pragma unroll
              for (int p = 0; p < PARTS2; ++p) Mma<T>::add(acc, fdown[v][j], fd[j][p]);
#pragma unroll
            for (int e = 0; e < 4; ++e) my[t * 16 + c][v * 16 + q * 4 + e] = from_f32<T>(acc[e]);
          }
        }
        wave_sync();
#pragma unroll
        for (int i = 0; i < Tile::MOVES; ++i) {
          const int m = i * Tile::ROWS + lane / Tile::LANES, col = lane % Tile::LANES * VEC, row = __shfl(rows, m);
          T *dst = a.dx + row * a.lddx + k0 + col;
          union {
            slot_t s;
            T e[VEC];
          } o;
          o.s = *reinterpret_cast<const slot_t *>(&my[m][col]);
          if (m < here && k0 + col + VEC <= K) {
            *reinterpret_cast<typename SlotOf<T>::type *>(dst) = o.s;
          } else if (m < here) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if (k0 + col + e < K) dst[e] = o.e[e];
          }
        }
      }
      __syncthreads();
    }
    pos = end;
    float *G = a_start >= ci * a.chunk ? a.G + (long)id * K * R : a.split + (long)ci * K * R;
#pragma unroll
    for (int v = 0; v < VT; ++v) {
      const int col = k0 + v * 16 + c;
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = j * 16 + q * 4 + e;
          if (col >= from && col < K && r < R) G[(unsigned)(r * K + col)] = g[v][j][e];
        }
    }
  }
}

// sum[i] of the blocks' parts, in a fixed order: 64 numbers a workgroup, the blocks shared out to 16 groups of its lanes.  41 MB
// (125 blocks of 2560 x 32) 14 us.
static __global__ void __launch_bounds__(1024) adapter_blocks_kernel(const float *__restrict__ part, int blocks, long size, float *__restrict__ sum) {
  __shared__ float of[16][64];
  const int lane = threadIdx.x & 63, group = threadIdx.x >> 6;
  const long i = (long)blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (i < size) {
#pragma unroll 8
    for (int b = group; b < blocks; b += 16) s += part[b * size + i];
  }
  of[group][lane] = s;
  __syncthreads();
  if (group != 0 || i >= size) return;
  s = 0.0f;
#pragma unroll
  for (int g = 0; g < 16; ++g) s += of[g][lane];
  sum[i] = s;
}

// Sums up what the chunks wrote of adapters that lie in several, in order; zeros for those without rows.  5-6 us.
struct JoinArgs {
  const float *split, *scale;  // scale may be nullptr
  float *G;
  long size;  // of an adapter's gradient
  int chunk;
};
static __global__ void __launch_bounds__(256) adapter_join_kernel(const int32_t *__restrict__ begin, int n, const JoinArgs up, const JoinArgs down) {
  const JoinArgs a = blockIdx.z ? down : up;
  for (int id = blockIdx.y; id < n; id += gridDim.y) {
    const int start = begin[id], end = begin[id + 1];
    const int c0 = start / a.chunk, c1 = end > start ? (end - 1) / a.chunk : c0;
    if (end > start && c0 == c1) continue;
    const float f = a.scale ? a.scale[id] : 1.0f;
    float *G = a.G + id * a.size;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < a.size; i += (long)gridDim.x * 256) {
      float s = 0.0f;
      if (end > start) {
        s = G[i];
#pragma unroll 8
        for (int c = c0 + 1; c <= c1; ++c) s += a.split[c * a.size + i];
        s *= f;
      }
      G[i] = s;
    }
  }
}

}  // namespace rnnlm_dev
