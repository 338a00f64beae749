// Low-rank adapters of many requests at once, beside a projection that they share, and
// their gradients.
//
// Row m of a batch has adapter a = index[m]:
//   h = x A_a^T, o = y + s_a h B_a^T
//   p = s_a g B_a, dx = d + p A_a, dA_a = sum p^T x, dB_a = s_a sum g^T h
// Three kinds of products, each with one long side that is read once: k_shrink sums over
// a long side (h, p), k_expand has the rank as its inner side (o, dx), k_outer sums over
// the rows of an adapter (dA, dB). Rows are taken in the order of their adapters
// (gptq2d_adapter_groups), in windows of fixed size, so that a window has one adapter or
// few, one after another.
//
// Inner products of 16-bit inputs are summed by the 16-bit matrix instruction in 32
// bits. h and p stay 32-bit: where the instruction takes them in, they are the sum of 16-bit
// numbers, so that no rounding of theirs shows in a result.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "codes.hpp"

namespace g2d {
namespace {

typedef bf16 b8 __attribute__((ext_vector_type(8)));

constexpr int kMaxRank = 128;

// ---------------------------------------------------------------------------
// matrix instructions: a 16 x 16 tile from K elements of 16 rows on both sides, lane l
// with E consecutive ones of row l % 16; the result has, in lane l, column l % 16 (of the
// second) and rows l / 16 * 4 + i (of the first)
// ---------------------------------------------------------------------------

template <class T>
struct Mat {
  static constexpr int E = 8, K = 32;
  typedef T F __attribute__((ext_vector_type(8)));
};
template <>
struct Mat<float> {
  static constexpr int E = 4, K = 16;
  typedef f4 F;
};
__device__ __forceinline__ f4 mma(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mma(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mma(f4 a, f4 b, f4 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

// Elements k .. k + E - 1 of a row of n, zeros past its end. WIDE: rows start on 16-byte
// boundaries and n is a multiple of E.
template <bool WIDE, class T>
__device__ __forceinline__ typename Mat<T>::F load_row(const T* row, int k, int n) {
  typedef typename Mat<T>::F F;
  F f;
  if constexpr (WIDE) {
    f = __builtin_bit_cast(F, *(const u4*)(row + (k < n ? k : 0)));
    if (k >= n) f = F{};
  } else {
#pragma unroll
    for (int i = 0; i < Mat<T>::E; ++i) f[i] = row[min(k + i, n - 1)];
#pragma unroll
    for (int i = 0; i < Mat<T>::E; ++i) f[i] = k + i < n ? f[i] : (T)0.0f;
  }
  return f;
}

// what of x (or, near the type's smallest number, of all that is summed with it) T holds
// and what it does not; infinities leave nothing
__device__ __forceinline__ float split(float& x, bf16) {
  const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  x = x == hi ? 0.0f : x - hi;
  return hi;
}
__device__ __forceinline__ float split(float& x, _Float16) {
  const float hi = (float)(_Float16)x;
  x = x == hi ? 0.0f : x - hi;
  return hi;
}

// ---------------------------------------------------------------------------
// rows in the order of their adapters
// ---------------------------------------------------------------------------

struct Groups {
  const int32_t *order, *which, *start;  // row and adapter at each place; places before an adapter's
  int rows, count;
};
__device__ __forceinline__ int row_at(const Groups& g, int i) { return min(max(g.order[min(i, g.rows - 1)], 0), g.rows - 1); }
// the adapter, `count` for none, -1 past the last row
__device__ __forceinline__ int which_at(const Groups& g, int i) {
  const int w = min(max(g.which[min(i, g.rows - 1)], 0), g.count);
  return i < g.rows ? w : -1;
}

// The places of a window (of n <= 64, from `first`) at which another adapter begins; `mine`:
// the adapter at the lane's place.
__device__ __forceinline__ uint64_t heads_of(const Groups& g, int first, int n, int& mine) {
  const int lane = threadIdx.x & 63;
  mine = which_at(g, first + min(lane, n - 1));
  const int before = __shfl_up(mine, 1);
  return __ballot(lane < n && mine >= 0 && (lane == 0 || mine != before));
}

constexpr int kGroupRows = 16;  // of a thread and turn
struct GroupArgs {
  int rows, count;
  const int32_t* index;
  int32_t *order, *which, *start;
};
// One work group for each adapter, and one for the rows that have none: how many rows lie
// before the adapter's, then the places of its own, which come in the rows' order.
__global__ __launch_bounds__(256) void k_group(GroupArgs g) {
  __shared__ int less4[4], same4[4];
  const int a = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
  auto key = [&](int m) {
    const int i = m < g.rows ? g.index[m] : -2;
    return m >= g.rows ? g.count + 1 : i < 0 || i >= g.count ? g.count : i;
  };
  int less = 0;
  for (int m = t; m < g.rows; m += 256) less += key(m) < a;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) less += __shfl_xor(less, d);
  if (lane == 0) less4[w] = less;
  __syncthreads();
  int at = less4[0] + less4[1] + less4[2] + less4[3];
  if (t == 0) {
    g.start[a] = at;
    if (a == g.count) g.start[a + 1] = g.rows;
  }
  for (int m0 = 0; m0 < g.rows; m0 += 256 * kGroupRows) {
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < kGroupRows; ++i) mine |= (uint32_t)(key(m0 + t * kGroupRows + i) == a) << i;
    const int n = __popc(mine);
    int upto = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 63) same4[w] = upto;
    __syncthreads();
    int p = at + upto - n;
    for (int k = 0; k < w; ++k) p += same4[k];
    for (uint32_t left = mine; left != 0; left &= left - 1, ++p) {
      g.order[p] = m0 + t * kGroupRows + __builtin_ctz(left);
      g.which[p] = a;
    }
    at += same4[0] + same4[1] + same4[2] + same4[3];
  }
}

// ---------------------------------------------------------------------------
// sums over a long side
// ---------------------------------------------------------------------------

struct ShrinkArgs {
  Groups g;
  int n, rank, ranks;  // inner side, rank and the rank that results have room for
  const void* X;
  int64_t ldx;
  const void* W;  // rank rows of n for each adapter
  int64_t ldw, step;
  const float* scales;  // results are multiplied by them
  float* H;             // [part][place][ranks]
  int64_t places;
};

// A work group takes a window of 16 MT rows and a part of the inner side, whose steps its
// four waves share; their sums are joined in LDS.
template <class T, int MT, int RT, bool WIDE>
__global__ __launch_bounds__(256) void k_shrink(ShrinkArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr int U = MT + RT <= 2 ? 8 : MT + RT <= 5 ? 4 : 2;
  __shared__ f4 red[4][MT * RT][64];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int first = blockIdx.x * 16 * MT;
  int mine;
  uint64_t heads = heads_of(a.g, first, 16 * MT, mine);
  const T* x[MT];
  int own[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    x[i] = (const T*)a.X + (int64_t)row_at(a.g, first + 16 * i + m) * a.ldx;
    own[i] = which_at(a.g, first + 16 * i + m);
  }
  const int steps = (a.n + M::K - 1) / M::K;
  const int s0 = (int)((int64_t)steps * blockIdx.y / gridDim.y), s1 = (int)((int64_t)steps * (blockIdx.y + 1) / gridDim.y);
  for (int z = 0; heads != 0; heads &= heads - 1, ++z) {
    if (z % gridDim.z != blockIdx.z) continue;
    const int ad = __shfl(mine, __builtin_ctzll(heads));
    if (ad >= a.g.count) continue;
    const T* wr[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) wr[j] = (const T*)a.W + ad * a.step + (int64_t)min(16 * j + m, a.rank - 1) * a.ldw;
    f4 acc[MT][RT] = {};
    for (int s = s0 + w; s < s1; s += 4 * U) {
      F fx[U][MT], fw[U][RT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (steps past the end are zeros on one side)
        const int k = s + 4 * u < s1 ? (s + 4 * u) * M::K + q * M::E : a.n;
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[u][i] = load_row<WIDE>(x[i], k, a.n);
#pragma unroll
        for (int j = 0; j < RT; ++j) fw[u][j] = load_row<WIDE>(wr[j], k, a.n);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < RT; ++j) acc[i][j] = mma(fw[u][j], fx[u][i], acc[i][j]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < RT; ++j) red[w][i * RT + j][lane] = acc[i][j];
    __syncthreads();
    const float f = a.scales ? a.scales[ad] : 1.0f;
#pragma unroll
    for (int c = 0; c < MT * RT; ++c) {
      if (c % 4 != w) continue;
      const int i = c / RT, j = c % RT;
      f4 s = (red[0][c][lane] + red[1][c][lane]) + (red[2][c][lane] + red[3][c][lane]);
      const int r = 16 * j + 4 * q;
      if (own[i] == ad && r < a.ranks) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = r + e < a.rank ? s[e] * f : 0.0f;
        *(f4*)(a.H + ((int64_t)blockIdx.y * a.places + first + 16 * i + m) * a.ranks + r) = s;
      }
    }
  }
}

// The parts' sums: to the rows themselves (rank columns) or in the places' order (ranks).
struct FoldArgs {
  Groups g;
  int rank, ranks, parts;
  const float* H;
  int64_t places;
  float* out;
  bool by_row;
};
__global__ __launch_bounds__(256) void k_fold(FoldArgs a) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int cols = a.by_row ? a.rank : a.ranks;
  const int64_t i = e / cols;
  if (i >= a.g.rows) return;
  const int r = (int)(e - i * cols);
  float s = 0.0f;
  if (which_at(a.g, (int)i) < a.g.count)
    for (int p = 0; p < a.parts; ++p) s += a.H[(p * a.places + i) * a.ranks + r];
  a.out[(a.by_row ? (int64_t)row_at(a.g, (int)i) : i) * cols + r] = s;
}

// ---------------------------------------------------------------------------
// products with the rank inside
// ---------------------------------------------------------------------------

struct ExpandArgs {
  Groups g;
  int n, rank, ranks, parts;
  const float* H;  // [part][place][ranks]
  int64_t places;
  const float* scales;
  const void* W;  // n rows of rank for each adapter
  int64_t ldw, step;
  const void* Y;  // may be NULL
  int64_t ldy;
  void* O;
  int64_t ldo;
  bool wide;  // Y and O are moved in 16-byte pieces
};

// NK: steps of the inner side, of M::K each; 0: of 16-bit types one step that has both
// halves of 16 h. A work group takes 16 WIN rows and 256 columns, a wave 64 of them. Four
// tiles' rows of W are dealt out so that a lane ends with 16 consecutive columns.
template <class T, int NK, int WIN, bool WIDE>
__global__ __launch_bounds__(256) void k_expand(ExpandArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr bool kNarrow = sizeof(T) == 2, kPacked = kNarrow && NK == 0;
  constexpr int S = kPacked ? 1 : NK, TERMS = kNarrow && !kPacked ? 2 : 1;
  constexpr int ROWS = 16 * WIN;
  // h of the window, as the instruction takes it: [term][step][row][4 pieces]
  __shared__ F hs[TERMS * S][ROWS * 4];
  __shared__ float back[ROWS];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int first = blockIdx.x * ROWS;
  int mine;
  uint64_t heads = heads_of(a.g, first, ROWS, mine);
  const int c0 = blockIdx.y * 256 + w * 64 + q * 16;  // the lane's columns
  T* out[WIN];
  int own[WIN];
  float y[WIN][16];
#pragma unroll
  for (int i = 0; i < WIN; ++i) {
    const int64_t row = row_at(a.g, first + 16 * i + m);
    own[i] = which_at(a.g, first + 16 * i + m);
    out[i] = (T*)a.O + row * a.ldo + c0;
    const T* p = (const T*)a.Y + row * a.ldy;
    if (a.Y) {
      const bool all = a.wide && c0 + 16 <= a.n;
      load8(p + c0, all, min(a.n - c0, 8), y[i], p);
      load8(p + c0 + 8, all, min(a.n - c0 - 8, 8), y[i] + 8, p);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[i][e] = 0.0f;
    }
  }
  for (int i0 = t >> 2; i0 < ROWS; i0 += 64) {
    const int place = first + i0, p = t & 3;
    const int wh = which_at(a.g, place);
    const float f = wh >= 0 && wh < a.g.count && a.scales ? a.scales[wh] : 1.0f;
    float h[S][M::E];
#pragma unroll
    for (int k = 0; k < S; ++k) {
#pragma unroll
      for (int e = 0; e < M::E; ++e) h[k][e] = 0.0f;
      const int r = kPacked ? p % 2 * 8 : k * M::K + p * M::E;
      if (r < a.ranks && wh >= 0 && wh < a.g.count)
        for (int s = 0; s < a.parts; ++s) {
          const f4* x = (const f4*)(a.H + (s * a.places + place) * a.ranks + r);
#pragma unroll
          for (int v = 0; v < M::E / 4; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[k][4 * v + e] += x[v][e];
        }
    }
    float up = 1.0f;
    if constexpr (std::is_same<T, _Float16>::value) {
      // a power of two brings the row's largest to [1, 2): halves reach from there to where it does not matter
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < S; ++k)
#pragma unroll
        for (int e = 0; e < M::E; ++e) top = max(top, mag(h[k][e]));
      top = max(top, (uint32_t)__shfl_xor((int)top, 1));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2));
      const uint32_t ex = min(max(top >> 23, 2u), 252u);
      up = __uint_as_float(ex << 23);
      const float down = __uint_as_float((254u - ex) << 23);
#pragma unroll
      for (int k = 0; k < S; ++k)
#pragma unroll
        for (int e = 0; e < M::E; ++e) h[k][e] *= down;
    }
    if (p == 0) back[i0] = up * f;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      if constexpr (!kNarrow) {
        F v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = h[k][e];
        hs[k][i0 * 4 + p] = v;
      } else {
        F hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = h[k][e];
          hi[e] = (T)split(x, T());
          lo[e] = (T)x;
        }
        if constexpr (kPacked) {
          hs[0][i0 * 4 + p] = p < 2 ? hi : lo;
        } else {
          hs[k][i0 * 4 + p] = hi;
          hs[S + k][i0 * 4 + p] = lo;
        }
      }
    }
  }
  __syncthreads();
  for (int z = 0; heads != 0; heads &= heads - 1, ++z) {
    if (z % gridDim.z != blockIdx.z) continue;
    const int ad = __shfl(mine, __builtin_ctzll(heads));
    F fw[4][S];
    if (ad < a.g.count) {
      // rows of tile j: lane m has column 16 (m / 4) + 4 j + m % 4 of the wave's
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = blockIdx.y * 256 + w * 64 + (m >> 2) * 16 + 4 * j + (m & 3);
        const T* row = (const T*)a.W + ad * a.step + (int64_t)min(c, a.n - 1) * a.ldw;
#pragma unroll
        for (int k = 0; k < S; ++k) fw[j][k] = load_row<WIDE>(row, kPacked ? q % 2 * 8 : k * M::K + q * M::E, a.rank);
      }
    }
#pragma unroll
    for (int i = 0; i < WIN; ++i) {
      if (__ballot(own[i] == ad) == 0) continue;
      f4 acc[4] = {};
      if (ad < a.g.count) {
#pragma unroll
        for (int k = 0; k < S; ++k)
#pragma unroll
          for (int u = 0; u < TERMS; ++u) {
            const F h = hs[u * S + k][(16 * i + m) * 4 + q];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = mma(fw[j][k], h, acc[j]);
          }
      }
      if (own[i] != ad || c0 >= a.n) continue;
      const float f = back[16 * i + m];
      float o[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = ad < a.g.count ? fmaf(acc[e / 4][e % 4], f, y[i][e]) : y[i][e];
      const bool all = a.wide && c0 + 16 <= a.n;
      store8(out[i], all, min(a.n - c0, 8), o);
      store8(out[i] + 8, all, min(a.n - c0 - 8, 8), o + 8);
    }
  }
}

// ---------------------------------------------------------------------------
// sums over an adapter's rows
// ---------------------------------------------------------------------------

struct OuterArgs {
  Groups g;
  int n, rank;
  const void* Z;  // rows of n
  int64_t ldz;
  const float* H;  // rows (by_row: of the batch, else places) of ldh
  int64_t ldh;
  bool by_row;
  const float* scales;
  float* out;       // [adapter][n][rank], or [adapter][rank][n] where `across`
  bool across;
  int window;       // places of a work group, a multiple of 32
  float* parts;     // [window + adapter] like an adapter's part of out
};

// A wave takes 128 columns and 16 RT ranks; lane l reads 8 (16-bit) or 4 columns of a
// row at once, whose pieces of different rows are turned in registers to runs of one column.
// Adapters whose rows lie in one window are done with it; of the others each window gives a
// part, at the number of the window and the adapter together (which grows along the
// order, so that no two are alike).
template <class T, int RT, bool WIDE>
__global__ __launch_bounds__(256) void k_outer(OuterArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr bool kNarrow = sizeof(T) == 2;
  constexpr int C = M::E;             // column tiles: columns C m + j
  constexpr int TERMS = std::is_same<T, bf16>::value ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;
  constexpr int COLS = 16 * C, STEP = kNarrow ? 32 : 4;  // rows of a step
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int c0 = (blockIdx.x * 4 + w) * COLS, r0 = blockIdx.z * 16 * RT;
  if (c0 >= a.n) return;
  const int begin = blockIdx.y * a.window, end = min(begin + a.window, a.g.rows);
  int i0 = begin;
  while (i0 < end) {
    const int ad = which_at(a.g, i0);
    if (ad >= a.g.count) break;
    const int from = max(a.g.start[ad], begin), to = min(a.g.start[ad + 1], end);
    if (to <= i0) break;  // (groups that are not this batch's)
    const float f = a.scales ? a.scales[ad] : 1.0f;
    auto h_of = [&](int i, int r) {
      const int64_t row = a.by_row ? row_at(a.g, i) : i;
      return r < a.rank ? a.H[row * a.ldh + r] * f : 0.0f;
    };
    float down[RT], up[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) down[j] = up[j] = 1.0f;
    if constexpr (std::is_same<T, _Float16>::value) {
      // a power of two for each rank: its largest h here comes to [1, 2)
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        uint32_t top = 0;
        for (int i = from + q; i < to; i += 4) top = max(top, mag(h_of(i, r0 + 16 * j + m)));
        top = quad_max(top);
        const uint32_t ex = min(max(top >> 23, 2u), 252u);
        up[j] = __uint_as_float(ex << 23);
        down[j] = __uint_as_float((254u - ex) << 23);
      }
    }
    f4 acc[C][RT] = {};
    for (int s = from; s < to; s += STEP) {
      if constexpr (kNarrow) {
        u4 z[8];
        const int i8 = s + 8 * q;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = min(i8 + e, to - 1);
          const T* row = (const T*)a.Z + (int64_t)row_at(a.g, i) * a.ldz;
          z[e] = __builtin_bit_cast(u4, load_row<WIDE>(row, c0 + C * m, a.n));
          if (i8 + e >= to) z[e] = u4{};
        }
        F h[RT][TERMS];
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x = i8 + e < to ? h_of(min(i8 + e, to - 1), r0 + 16 * j + m) * down[j] : 0.0f;
#pragma unroll
            for (int u = 0; u < TERMS; ++u) h[j][u][e] = u + 1 < TERMS ? (T)split(x, T()) : (T)x;
          }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          u4 col;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            col[p] = __builtin_amdgcn_perm(z[2 * p + 1][c / 2], z[2 * p][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
          const F fz = __builtin_bit_cast(F, col);
#pragma unroll
          for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int u = TERMS - 1; u >= 0; --u) acc[c][j] = mma(fz, h[j][u], acc[c][j]);
        }
      } else {
        const int i = s + q;
        const T* row = (const T*)a.Z + (int64_t)row_at(a.g, min(i, to - 1)) * a.ldz;
        F z = load_row<WIDE>(row, c0 + C * m, a.n);
        if (i >= to) z = F{};
#pragma unroll
        for (int j = 0; j < RT; ++j) {
          const float h = i < to ? h_of(min(i, to - 1), r0 + 16 * j + m) : 0.0f;
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[c], h, acc[c][j], 0, 0, 0);
        }
      }
    }
    const bool whole = a.g.start[ad] >= begin && a.g.start[ad + 1] <= end;
    float* o = whole ? a.out + (int64_t)ad * a.n * a.rank : a.parts + (int64_t)(blockIdx.y + ad) * a.n * a.rank;
    // lane: rank m of each tile, columns c0 + C (4 q + i) + c
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int r = r0 + 16 * j + m;
      if (r >= a.rank) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const int col = c0 + C * (4 * q + i) + c;
          if (col < a.n) o[a.across ? (int64_t)r * a.n + col : (int64_t)col * a.rank + r] = acc[c][j][i] * up[j];
        }
    }
    i0 = to;
  }
}

// The parts' sums, and zeros for adapters without rows.
struct JoinArgs {
  Groups g;
  int64_t size;  // of an adapter
  int window;
  const float* parts;
  float* out;
};
__global__ __launch_bounds__(256) void k_outer_join(JoinArgs a) {
  const int ad = blockIdx.y;
  const int from = a.g.start[ad], to = min(a.g.start[ad + 1], a.g.rows);
  const int w0 = from / a.window, w1 = to > from ? (to - 1) / a.window : w0;
  if (to > from && w0 == w1) return;  // (or it is there already)
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < a.size; e += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
    if (to > from)
      for (int w = w0; w <= w1; ++w) s += a.parts[(w + ad) * a.size + e];
    a.out[ad * a.size + e] = s;
  }
}

// Rows of W (rows x cols, of each adapter that has rows) as columns.
struct TurnArgs {
  Groups g;
  int rows, cols;
  const void* W;
  int64_t ldw, step;
  void* out;
  int64_t ldo, step_out;
};
template <class T>
__global__ __launch_bounds__(256) void k_turn(TurnArgs a) {
  __shared__ T tile[32][33];
  const int ad = blockIdx.z;
  if (a.g.start[ad] >= a.g.start[ad + 1]) return;
  const int tiles = (a.cols + 31) / 32, x = threadIdx.x & 31, y0 = threadIdx.x >> 5;
  const int r0 = blockIdx.x / tiles * 32, c0 = (blockIdx.x - r0 / 32 * tiles) * 32;
  for (int y = y0; y < 32; y += 8)
    if (r0 + y < a.rows && c0 + x < a.cols) tile[y][x] = ((const T*)a.W)[ad * a.step + (r0 + y) * a.ldw + c0 + x];
  __syncthreads();
  for (int y = y0; y < 32; y += 8)
    if (c0 + y < a.cols && r0 + x < a.rows) ((T*)a.out)[ad * a.step_out + (c0 + y) * a.ldo + r0 + x] = tile[x][y];
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t up(int64_t v, int64_t m) { return ceil_div(v, m) * m; }

int ranks_of(int rank) { return (int)up(rank, 16); }
// row tiles of a window, parts of the inner side
int shrink_tiles(int64_t rows, int rank, bool wide) { return !wide || rows < 2048 ? 1 : rank <= 64 ? 4 : 2; }
int shrink_parts(int64_t rows, int64_t n) {
  const int64_t want = ceil_div(512, ceil_div(rows, 16)), room = ceil_div(n, 256);
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, room, 16}));
}
int64_t places_of(int64_t rows) { return up(rows, 64); }
size_t h_bytes(int64_t rows, int64_t n, int rank) {
  return up256((size_t)shrink_parts(rows, n) * places_of(rows) * ranks_of(rank) * 4);
}

template <class T, int MT, int RT, bool WIDE>
void shrink_as(const ShrinkArgs& a, int parts, int z, hipStream_t s) {
  hipLaunchKernelGGL((k_shrink<T, MT, RT, WIDE>), dim3((unsigned)ceil_div(a.g.rows, 16 * MT), parts, z), dim3(256), 0, s, a);
}
template <class T>
void shrink(const ShrinkArgs& a, bool wide, int parts, hipStream_t s) {
  const int tiles = shrink_tiles(a.g.rows, a.rank, wide);
  const int z = std::min(tiles == 1 && a.g.rows <= 1024 ? 16 : 1, a.g.count);
  auto of = [&](auto rt) {
    constexpr int RT = decltype(rt)::value;
    if (!wide) return shrink_as<T, 1, RT, false>(a, parts, z, s);
    if (tiles == 1) return shrink_as<T, 1, RT, true>(a, parts, z, s);
    return shrink_as<T, RT == 8 ? 2 : 4, RT, true>(a, parts, z, s);
  };
  if (a.rank <= 16) of(std::integral_constant<int, 1>());
  else if (a.rank <= 32) of(std::integral_constant<int, 2>());
  else if (a.rank <= 64) of(std::integral_constant<int, 4>());
  else of(std::integral_constant<int, 8>());
}

template <class T>
void turn(const TurnArgs& a, hipStream_t s) {
  const int64_t tiles = ceil_div(a.rows, 32) * ceil_div(a.cols, 32);
  hipLaunchKernelGGL(k_turn<T>, dim3((unsigned)tiles, 1, a.g.count), dim3(256), 0, s, a);
}

template <class T>
void expand(const ExpandArgs& a, bool wide, hipStream_t s) {
  const bool few = a.g.rows <= 1024;
  auto of = [&](auto nk) {
    constexpr int NK = decltype(nk)::value;
    const unsigned cols = (unsigned)ceil_div(a.n, 256);
    auto as = [&](auto win, auto w) {
      constexpr int WIN = decltype(win)::value;
      const dim3 grid((unsigned)ceil_div(a.g.rows, 16 * WIN), cols, few ? std::min(16, a.g.count + 1) : 1);
      hipLaunchKernelGGL((k_expand<T, NK, WIN, decltype(w)::value>), grid, dim3(256), 0, s, a);
    };
    if (!wide) as(std::integral_constant<int, 1>(), std::false_type());
    else if (few) as(std::integral_constant<int, 1>(), std::true_type());
    else as(std::integral_constant<int, 4>(), std::true_type());
  };
  if constexpr (sizeof(T) == 4) {
    if (a.rank <= 16) of(std::integral_constant<int, 1>());
    else if (a.rank <= 32) of(std::integral_constant<int, 2>());
    else if (a.rank <= 64) of(std::integral_constant<int, 4>());
    else of(std::integral_constant<int, 8>());
  } else {
    if (a.rank <= 16) of(std::integral_constant<int, 0>());
    else if (a.rank <= 32) of(std::integral_constant<int, 1>());
    else if (a.rank <= 64) of(std::integral_constant<int, 2>());
    else of(std::integral_constant<int, 4>());
  }
}

int outer_window(int64_t rows, int64_t n) {
  // as many windows as fill the device with four waves of columns a work group
  const int64_t strips = ceil_div(n, 512), want = std::max<int64_t>(1, ceil_div(512, strips));
  return (int)std::max<int64_t>(64, up(ceil_div(rows, want), 32));
}
size_t outer_bytes(int64_t rows, int64_t n, int rank, int count) {
  const int64_t windows = ceil_div(rows, outer_window(rows, n));
  return windows <= 1 ? 0 : up256((size_t)(windows + count) * n * rank * 4);
}
template <class T>
void outer(OuterArgs a, bool wide, hipStream_t s) {
  a.window = outer_window(a.g.rows, a.n);
  const JoinArgs join = {a.g, (int64_t)a.n * a.rank, a.window, a.parts, a.out};
  const dim3 join_grid((unsigned)std::min<int64_t>(ceil_div(join.size, 1024), 1024), a.g.count);
  if (a.g.rows == 0) {  // zeros
    hipLaunchKernelGGL(k_outer_join, join_grid, dim3(256), 0, s, join);
    return;
  }
  auto of = [&](auto rt) {
    constexpr int RT = decltype(rt)::value;
    const dim3 grid((unsigned)ceil_div(a.n, 4 * 16 * Mat<T>::E), (unsigned)ceil_div(a.g.rows, a.window),
                    (unsigned)ceil_div(a.rank, 16 * RT));
    if (wide)
      hipLaunchKernelGGL((k_outer<T, RT, true>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_outer<T, RT, false>), grid, dim3(256), 0, s, a);
  };
  if (a.rank <= 16) of(std::integral_constant<int, 1>());
  else if (a.rank <= 32) of(std::integral_constant<int, 2>());
  else of(std::integral_constant<int, 4>());
  hipLaunchKernelGGL(k_outer_join, join_grid, dim3(256), 0, s, join);
}

bool bad_shape(int64_t M, int64_t N, int64_t K, int R, int count) {
  const int64_t top = (int64_t)1 << 22;
  return M < 0 || M > top || N < 1 || N > top || K < 1 || K > top || R < 1 || R > kMaxRank || count < 1 || count > 4096;
}
Groups groups_of(const int32_t* g, int64_t M, int count) { return {g, g + M, g + 2 * M, (int)M, count}; }
template <class T>
bool wide_matrix(const void* p, int64_t ld, int64_t n) {
  return wide_rows(p, ld, sizeof(T)) && n % Mat<T>::E == 0;
}

struct BackSpace {
  size_t h, p, at, bt, outer, all;
  int64_t ldat, ldbt;
};
BackSpace back_space(int64_t M, int64_t N, int64_t K, int R, int count) {
  BackSpace b;
  b.ldat = up(R, 8), b.ldbt = up(N, 8);
  b.h = 0;
  b.p = b.h + h_bytes(M, N, R);
  b.at = b.p + up256((size_t)places_of(M) * ranks_of(R) * 4);
  b.bt = b.at + up256((size_t)count * K * b.ldat * 4);
  b.outer = b.bt + up256((size_t)count * R * b.ldbt * 4);
  b.all = b.outer + std::max(outer_bytes(M, N, R, count), outer_bytes(M, K, R, count));
  return b;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

int64_t gptq2d_adapter_groups_size(int64_t M, int count) {
  if (bad_shape(M, 1, 1, 1, count)) return 0;
  return 2 * M + count + 2;
}

gptq2d_status gptq2d_adapter_groups(int64_t M, int count, const int32_t* index, int32_t* groups, void* stream) {
  if (bad_shape(M, 1, 1, 1, count)) return refuse("M must lie in [0, 2^22], count in [1, 4096]");
  if (M * (count + 1) > (int64_t)1 << 32) return refuse("M (count + 1) must not exceed 2^32");
  if (!groups || (M > 0 && !index)) return refuse("index or groups is NULL");
  if (!aligned(index, 4) || !aligned(groups, 4)) return refuse("an argument is not aligned to its elements");
  const GroupArgs a = {(int)M, count, index, groups, groups + M, groups + 2 * M};
  hipLaunchKernelGGL(k_group, dim3(count + 1), dim3(256), 0, (hipStream_t)stream, a);
  return launched("gptq2d_adapter_groups");
}

size_t gptq2d_adapters_workspace_size(int64_t M, int64_t N, int64_t K, int R, int count) {
  if (bad_shape(M, N, K, R, count) || M == 0) return 0;
  return h_bytes(M, K, R);
}

gptq2d_status gptq2d_adapters(int64_t M, int64_t N, int64_t K, int R, int count, gptq2d_dtype dt, const void* X, int64_t ldx,
                              const void* A, int64_t lda, const void* B, int64_t ldb, const float* scales,
                              const int32_t* groups, const void* Y, int64_t ldy, void* O, int64_t ldo, float* H,
                              void* workspace, size_t ws_bytes, void* stream) {
  if (bad_shape(M, N, K, R, count)) return refuse("M, N and K must lie in [1, 2^22] (M may be 0), R in [1, 128], count in [1, 4096]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (M == 0) return GPTQ2D_OK;
  if (!X || !A || !B || !groups || !O) return refuse("X, A, B, groups or O is NULL");
  if (ldx < K || lda < K || ldb < R || (Y && ldy < N) || ldo < N) return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  if (!aligned(X, es) || !aligned(A, es) || !aligned(B, es) || !aligned(Y, es) || !aligned(O, es) || !aligned(scales, 4) ||
      !aligned(groups, 4) || !aligned(H, 4))
    return refuse("an argument is not aligned to its elements");
  const size_t need = h_bytes(M, K, R);
  if (!workspace || ws_bytes < need) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const hipStream_t s = (hipStream_t)stream;
  const Groups g = groups_of(groups, M, count);
  const int parts = shrink_parts(M, K);
  float* h = (float*)workspace;
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const ShrinkArgs sh = {g, (int)K, R, ranks_of(R), X, ldx, A, lda, R * lda, nullptr, h, places_of(M)};
    shrink<T>(sh, wide_matrix<T>(X, ldx, K) && wide_matrix<T>(A, lda, K), parts, s);
    if (H) {
      const FoldArgs f = {g, R, ranks_of(R), parts, h, places_of(M), H, true};
      hipLaunchKernelGGL(k_fold, dim3((unsigned)ceil_div(M * R, 256)), dim3(256), 0, s, f);
    }
    const ExpandArgs e = {g, (int)N, R, ranks_of(R), parts, h, places_of(M), scales, B, ldb, N * ldb, Y, ldy, O, ldo,
                          (!Y || wide_rows(Y, ldy, es)) && wide_rows(O, ldo, es)};
    expand<T>(e, wide_matrix<T>(B, ldb, R), s);
  });
  return launched("gptq2d_adapters");
}

size_t gptq2d_adapters_backward_workspace_size(int64_t M, int64_t N, int64_t K, int R, int count) {
  if (bad_shape(M, N, K, R, count) || M == 0) return 0;
  return back_space(M, N, K, R, count).all;
}

gptq2d_status gptq2d_adapters_backward(int64_t M, int64_t N, int64_t K, int R, int count, gptq2d_dtype dt, const void* G,
                                       int64_t ldg, const void* X, int64_t ldx, const void* A, int64_t lda, const void* B,
                                       int64_t ldb, const float* scales, const int32_t* groups, const float* H, const void* D,
                                       int64_t ldd, void* dX, int64_t lddx, float* dA, float* dB, void* workspace,
                                       size_t ws_bytes, void* stream) {
  if (bad_shape(M, N, K, R, count)) return refuse("M, N and K must lie in [1, 2^22] (M may be 0), R in [1, 128], count in [1, 4096]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (!dX && !dA && !dB) return refuse("no gradient is asked for");
  if (!groups) return refuse("groups is NULL");
  if (M == 0) {  // nothing but zeros
    const Groups g = groups_of(groups, 0, count);
    if (dA) outer<float>({g, (int)K, R, nullptr, 0, nullptr, 0, false, nullptr, dA, true, 0, nullptr}, true, (hipStream_t)stream);
    if (dB) outer<float>({g, (int)N, R, nullptr, 0, nullptr, 0, false, nullptr, dB, false, 0, nullptr}, true, (hipStream_t)stream);
    return launched("gptq2d_adapters_backward");
  }
  if (!G) return refuse("G is NULL");
  if (dX && !A) return refuse("dX needs A");
  if ((dX || dA) && !B) return refuse("dX and dA need B");
  if (dA && !X) return refuse("dA needs X");
  if (dB && !H) return refuse("dB needs H");
  if (ldg < N || (dA && ldx < K) || (dX && (lda < K || lddx < K || (D && ldd < K))) || ((dX || dA) && ldb < R))
    return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  for (const void* p : {G, X, A, B, D, (const void*)dX})
    if (!aligned(p, es)) return refuse("an argument is not aligned to its elements");
  for (const void* p : {(const void*)scales, (const void*)groups, (const void*)H, (const void*)dA, (const void*)dB})
    if (!aligned(p, 4)) return refuse("an argument is not aligned to its elements");
  const BackSpace b = back_space(M, N, K, R, count);
  if (!workspace || ws_bytes < b.all) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const hipStream_t s = (hipStream_t)stream;
  const Groups g = groups_of(groups, M, count);
  char* ws = (char*)workspace;
  float *h = (float*)(ws + b.h), *pr = (float*)(ws + b.p), *parts = (float*)(ws + b.outer);
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const bool wide_g = wide_matrix<T>(G, ldg, N);
    if (dB) outer<T>({g, (int)N, R, G, ldg, H, R, true, scales, dB, false, 0, parts}, wide_g, s);
    if (!dX && !dA) return;
    const TurnArgs tb = {g, (int)N, R, B, ldb, N * ldb, ws + b.bt, b.ldbt, R * b.ldbt};
    turn<T>(tb, s);
    const int n = shrink_parts(M, N);
    const ShrinkArgs sh = {g, (int)N, R, ranks_of(R), G, ldg, ws + b.bt, b.ldbt, R * b.ldbt, scales, h, places_of(M)};
    shrink<T>(sh, wide_g, n, s);
    const float* ph = h;
    if (n > 1) {
      const FoldArgs f = {g, R, ranks_of(R), n, h, places_of(M), pr, false};
      hipLaunchKernelGGL(k_fold, dim3((unsigned)ceil_div(M * ranks_of(R), 256)), dim3(256), 0, s, f);
      ph = pr;
    }
    if (dA) outer<T>({g, (int)K, R, X, ldx, ph, ranks_of(R), false, nullptr, dA, true, 0, parts}, wide_matrix<T>(X, ldx, K), s);
    if (dX) {
      const TurnArgs ta = {g, R, (int)K, A, lda, R * lda, ws + b.at, b.ldat, K * b.ldat};
      turn<T>(ta, s);
      const ExpandArgs e = {g, (int)K, R, ranks_of(R), 1, ph, places_of(M), nullptr, ws + b.at, b.ldat, K * b.ldat, D, ldd, dX,
                            lddx, (!D || wide_rows(D, ldd, es)) && wide_rows(dX, lddx, es)};
      expand<T>(e, R % Mat<T>::E == 0, s);
    }
  });
  return launched("gptq2d_adapters_backward");
}

}  // extern "C"
