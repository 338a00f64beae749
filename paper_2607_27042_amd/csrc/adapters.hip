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
// bits. h and p stay 32-bit: where the instruction takes them in, each is the sum of three bf16
// numbers, which hold its 24 bits whatever its size, and an f16 number beside it is the sum of
// two, its 11 bits. (As halves of f16, relative to the largest h of a row or of an adapter's rows,
// an h 2^-25 of that was nothing, and those in between lost bits to it; six products instead of
// two: 4096 x 11008 x 4096, rank 64, f16, a call 87 us, so 77, gradients of 8192 x 4096 x 4096, rank
// 16, 110 and 101, of 2048 x 4096 x 4096, rank 128, 111 and 92.)
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

// the same with the fragments of N tiles: the 32-bit steps of one would wait for one another
template <int N, class F>
__device__ __forceinline__ void mma_each(const F (&w)[N], F x, f4 (&acc)[N]) {
  if constexpr (std::is_same<F, f4>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j][i], x[i], acc[j], 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = mma(w[j], x, acc[j]);
  }
}

// 16 bytes at any element (memory takes them off their boundary as well, in two lines)
typedef u4 u4_near __attribute__((aligned(2)));

// Elements k .. k + E - 1 of a row of n, in two halves: the load, without a branch and with
// nothing done to what it brings (a wave that would set it to zero there, or choose between two
// loads, would wait for it there), and what is left to do where it is used and the row ends
// among these elements or before them. SHORT: rows of any length, others have E elements
// at least (that instances for both have the branch took 45 instead of 34 us of 8192 x 4096
// gradients' sums over rows).
template <bool SHORT, class T>
__device__ __forceinline__ typename Mat<T>::F load_row(const T* row, int k, int n) {
  typedef typename Mat<T>::F F;
  if constexpr (SHORT) {
    if (n < Mat<T>::E) return F{};  // end_row reads what there is
  }
  return __builtin_bit_cast(F, *(const u4_near*)(row + min(k, n - Mat<T>::E)));
}
template <bool SHORT, class T>
__device__ __forceinline__ void end_row(typename Mat<T>::F& f, const T* row, int k, int n) {
  typedef unsigned __int128 B;
  constexpr int E = Mat<T>::E, bits = 8 * sizeof(T);
  if (k + E <= n) return;
  B b = __builtin_bit_cast(B, f);
  const int d = k - (n - E);  // the row's last E elements: those before k are shifted out, zeros in
  b = d < E ? b >> (bits * d) : 0;
  if constexpr (SHORT) {
    if (n < E) {
      b = 0;
#pragma unroll 1
      for (int i = n - 1; i >= k; --i) {
        typedef typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type U;
        b = b << bits | __builtin_bit_cast(U, row[i]);
      }
    }
  }
  f = __builtin_bit_cast(typename Mat<T>::F, b);
}

// Takes the first eight bits of x off it: x becomes the rest. Both have its sign and neither is
// zero unless x is (what bf16 holds whole is taken as the number before it), so that the sum
// of what an infinite factor gives with each is infinite too.
__device__ __forceinline__ float split(float& x) {
  const uint32_t b = __float_as_uint(x);
  const float hi = __uint_as_float((b - (x != 0.0f ? 1u : 0u)) & 0xffff0000u);
  x -= hi;
  return hi;
}
// eight f16 as the sums of two bf16 each
__device__ __forceinline__ void split(h8 x, b8& hi, b8& lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = (float)x[e];
    hi[e] = (bf16)split(v);
    lo[e] = (bf16)v;
  }
}

// over a wave, in every lane, without LDS
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true);
  const u2 a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = a[0] + a[1];
  const u2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return b[0] + b[1];
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

struct GroupArgs {
  int rows, count;
  const int32_t* index;
  int32_t *order, *which, *start;
};
constexpr int kGroupThreads = 1024;
constexpr int kGroupRows = 4;  // of a thread and turn
// One work group for each adapter, and one for the rows that have none: how many rows lie
// before the adapter's, and the places of its own, which come in the rows' order. Up to
// 16384 rows are looked at once (8192 rows, 4 adapters: 6.7 us; turn by turn 9.6, row by row 21).
template <int TURNS>
__global__ __launch_bounds__(kGroupThreads) void k_group(GroupArgs g) {
  __shared__ int less16[16], count64[64];
  const int a = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6, waves = blockDim.x >> 6;
  const bool many = g.rows > (int)blockDim.x * kGroupRows * TURNS;
  auto key = [&](int i) { return i < 0 || i >= g.count ? g.count : i; };
  // turn u of the rows from m0 on: rows in fours along the threads
  auto row = [&](int m0, int u, int e) { return m0 + (u * (int)blockDim.x + t) * kGroupRows + e; };
  int less = 0, at = 0;
  if (many) {
#pragma unroll 8
    for (int m = t; m < g.rows; m += blockDim.x) less += key(g.index[m]) < a;
    less = (int)wave_sum((uint32_t)less);
    if (lane == 0) less16[w] = less;
    __syncthreads();
    for (int k = 0; k < waves; ++k) at += less16[k];
  }
  for (int m0 = 0; m0 < g.rows || m0 == 0; m0 += (int)blockDim.x * kGroupRows * TURNS) {
    int k[TURNS][kGroupRows];
#pragma unroll
    for (int u = 0; u < TURNS; ++u)
#pragma unroll
      for (int e = 0; e < kGroupRows; ++e) k[u][e] = row(m0, u, e) < g.rows ? key(g.index[row(m0, u, e)]) : 0x7fffffff;
    uint32_t mine = 0;
    int before[TURNS];
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
      // the bits of the lanes of each of four rows: how many lie before the lane's, and all
      int all = 0;
      before[u] = 0;
#pragma unroll
      for (int e = 0; e < kGroupRows; ++e) {
        if (!many) less += k[u][e] < a;
        mine |= (uint32_t)(k[u][e] == a) << (u * kGroupRows + e);
        const uint64_t b = __ballot(k[u][e] == a);
        before[u] += __popcll(b & ((1ull << lane) - 1));
        all += __popcll(b);
      }
      if (m0 > 0 && u == 0) __syncthreads();
      if (lane == 0) count64[u * 16 + w] = all;
    }
    if (!many) {
      less = (int)wave_sum((uint32_t)less);
      if (lane == 0) less16[w] = less;
    }
    __syncthreads();
    if (!many)
      for (int k = 0; k < waves; ++k) at += less16[k];
    // of turns and waves, in that order, those before
    const int n = lane % 16 < waves && lane < TURNS * 16 ? count64[lane] : 0;
    int upto = n;
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xf, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x142, 0xa, 0xf, true);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x143, 0xc, 0xf, true);
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
      int p = at + before[u] + __builtin_amdgcn_readlane(upto - n, u * 16 + w);
#pragma unroll
      for (int e = 0; e < kGroupRows; ++e)
        if (mine >> (u * kGroupRows + e) & 1) {
          g.order[p] = row(m0, u, e);
          g.which[p++] = a;
        }
    }
    if (m0 == 0 && t == 0) {
      g.start[a] = at;
      if (a == g.count) g.start[a + 1] = g.rows;
    }
    at += __builtin_amdgcn_readlane(upto, 63);
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
template <class T, int MT, int RT, bool SHORT>
__global__ __launch_bounds__(256) void k_shrink(ShrinkArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr int U = MT + RT <= 3 ? 4 : 2;
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
    F fx[2][U][MT], fw[2][U][RT];
    // a wave takes two steps in a row (128 bytes of a row of 16-bit numbers), then the next one
    const int n = s1 - s0, all = (n + 7) / 8 * 2;
    auto step = [&](int i) { return (i & ~1) * 4 + 2 * w + (i & 1); };  // the wave's i-th
    auto load = [&](int i, F x_[U][MT], F w_[U][RT]) {  // steps i .. i + U - 1 of the wave's
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (s0 + min(step(i + u), n - 1)) * M::K + q * M::E;
#pragma unroll
        for (int i = 0; i < MT; ++i) x_[u][i] = load_row<SHORT>(x[i], k, a.n);
#pragma unroll
        for (int j = 0; j < RT; ++j) w_[u][j] = load_row<SHORT>(wr[j], k, a.n);
      }
    };
    auto sum = [&](int i, F x_[U][MT], F w_[U][RT]) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = step(i + u), k0 = (s0 + s) * M::K;
        if (i + u >= all || s >= n) continue;
        if (k0 + M::K > a.n) {
#pragma unroll
          for (int i = 0; i < MT; ++i) end_row<SHORT>(x_[u][i], x[i], k0 + q * M::E, a.n);
#pragma unroll
          for (int j = 0; j < RT; ++j) end_row<SHORT>(w_[u][j], wr[j], k0 + q * M::E, a.n);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          F (&rows)[RT] = *(F(*)[RT])w_[u];
          mma_each(rows, x_[u][i], acc[i]);
        }
      }
    };
    // a turn's loads are on their way while the one before is summed (the two without copies take twice the code:
    // 600 x 4096, rank 128, a call 39 us, so 30)
    load(0, fx[0], fw[0]);
#pragma unroll 1
    for (int i = 0; i < all; i += U) {
      load(i + U, fx[1], fw[1]);
      sum(i, fx[0], fw[0]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int k = 0; k < MT; ++k) fx[0][u][k] = fx[1][u][k];
#pragma unroll
        for (int k = 0; k < RT; ++k) fw[0][u][k] = fw[1][u][k];
      }
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

// The same for many rows: a work group takes 64 rows and a part of the inner side, which come
// through a ring of LDS buffers of 128 bytes of each row, loaded without registers in
// between, BUFS - 1 of them ahead; a wave sums 16 rows. The pieces of a row are dealt out so that
// the 16 rows that are read at once lie in different banks. (The rows' direct way to the
// registers takes 64 bytes of each of 16 rows at a time, and has each wave load the weights anew:
// 8192 x 4096, rank 16, 22.8 us there, 17.3 here; 4096 x 4096, rank 64, 21.9 and 15.7.)
// For rows on 16-byte boundaries, of whole pieces.
template <int N>
__device__ __forceinline__ void wait_loads() {  // until N of the wave's loads are on their way
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
}
typedef __attribute__((address_space(3))) void lds_void;
template <int RT>
constexpr int shrink_bufs() {  // two work groups' fit a compute unit (5756 x 2816, rank 64, 32 bits, a call: 77 us; one with twice the buffers 116)
  return RT == 1 ? 7 : RT == 2 ? 6 : RT == 4 ? 4 : 3;
}
template <class T, int RT>
__global__ __launch_bounds__(256) void k_shrink_many(ShrinkArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr int BUFS = shrink_bufs<RT>(), ROWS = 64 + 16 * RT;
  constexpr int CHUNK = 128 / sizeof(T);               // elements of a row in a buffer
  constexpr int XL = 2, WL = RT == 1 ? 1 : RT / 2;     // a wave's loads of X and W (eight rows each)
  __shared__ alignas(16) char ring[BUFS][ROWS * 128];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int first = blockIdx.x * 64;
  int mine;
  uint64_t heads = heads_of(a.g, first, 64, mine);
  const int own = which_at(a.g, first + 16 * w + m);
  // the lane's place in a load: row lane / 8 of eight, piece lane % 8 of it, changed by the row
  const int lr = lane >> 3, piece = (lane & 7) ^ lr;
  const char* x[XL];
#pragma unroll
  for (int i = 0; i < XL; ++i) x[i] = (const char*)((const T*)a.X + (int64_t)row_at(a.g, first + 16 * w + 8 * i + lr) * a.ldx);
  const int chunks = (a.n + CHUNK - 1) / CHUNK;
  const int s0 = (int)((int64_t)chunks * blockIdx.y / gridDim.y), s1 = (int)((int64_t)chunks * (blockIdx.y + 1) / gridDim.y);
  const int most = (int)((a.n * sizeof(T) - 16));  // the last piece of a row
  for (; heads != 0; heads &= heads - 1) {
    const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctzll(heads));
    if (ad >= a.g.count) continue;
    const char* wr[WL];
#pragma unroll
    for (int i = 0; i < WL; ++i)
      wr[i] = (const char*)((const T*)a.W + ad * a.step + (int64_t)min((w * WL + i) * 8 + lr, a.rank - 1) * a.ldw);
    auto load = [&](int s) {
      char* b = ring[(s - s0) % BUFS];
      const int at = min(s * 128 + piece * 16, most);
#pragma unroll
      for (int i = 0; i < XL; ++i)
        __builtin_amdgcn_global_load_lds((const void*)(x[i] + at), (lds_void*)(b + (16 * w + 8 * i) * 128), 16, 0, 0);
      if (RT > 1 || w < 2) {
#pragma unroll
        for (int i = 0; i < WL; ++i)
          __builtin_amdgcn_global_load_lds((const void*)(wr[i] + at), (lds_void*)(b + (64 + (w * WL + i) * 8) * 128), 16, 0, 0);
      }
    };
    f4 acc[RT] = {};
    wait_loads<0>();
    asm volatile("s_barrier" ::: "memory");  // the last adapter's buffers are read
#pragma unroll 1
    for (int s = s0; s < min(s0 + BUFS - 1, s1); ++s) load(s);
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
      if (s + BUFS - 1 > s1) wait_loads<0>();
      else if (RT > 1 || w < 2) wait_loads<(BUFS - 2) * (XL + WL)>();
      else wait_loads<(BUFS - 2) * XL>();
      // every wave's part of this buffer is there, and every wave has read the one that is filled next
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (s + BUFS - 1 < s1) load(s + BUFS - 1);
      const char* b = ring[(s - s0) % BUFS];
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // (two steps of the instruction)
        const int p = ((4 * k + q) ^ (m & 7)) * 16;
        F fx = *(const F*)(b + (16 * w + m) * 128 + p);
        F fw[RT];
#pragma unroll
        for (int j = 0; j < RT; ++j) fw[j] = *(const F*)(b + (64 + 16 * j + m) * 128 + p);
        if ((s + 1) * CHUNK > a.n && s * CHUNK + (4 * k + q) * M::E >= a.n) {
          fx = F{};
#pragma unroll
          for (int j = 0; j < RT; ++j) fw[j] = F{};
        }
        mma_each(fw, fx, acc);
      }
    }
    const float f = a.scales ? a.scales[ad] : 1.0f;
    if (own == ad) {
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const int r = 16 * j + 4 * q;
        if (r >= a.ranks) continue;
        f4 s = acc[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = r + e < a.rank ? s[e] * f : 0.0f;
        *(f4*)(a.H + ((int64_t)blockIdx.y * a.places + first + 16 * w + m) * a.ranks + r) = s;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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
};

// NK: steps of the inner side, of M::K each; 0: of 16-bit types steps that have two of the
// numbers that each of 16 h is the sum of. A work group takes 16 WIN rows and 256 columns, a wave 64 of them. Four
// tiles' rows of W are dealt out so that a lane ends with 16 consecutive columns.
// waves of a SIMD that an instance's registers are held down to (f16 has W twice as long)
template <class T, int NK>
constexpr int expand_waves() {
  return std::is_same<T, _Float16>::value ? (NK <= 1 ? 3 : 2) : sizeof(T) == 2 ? (NK == 1 ? 3 : NK <= 2 ? 4 : 2) : NK == 1 ? 4 : NK == 2 ? 3 : 2;
}
template <class T, int NK, int WIN, bool SHORT>
__global__ __launch_bounds__(256, (expand_waves<T, NK>())) void k_expand(ExpandArgs a) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr bool kNarrow = sizeof(T) == 2, kPacked = kNarrow && NK == 0;
  constexpr int S = kPacked ? 1 : NK;
  // what the instruction multiplies; the numbers that an h and an f16 of W are the sums of. Of a
  // packed step bf16 has two of an h's three in one instruction, f16 both of W's. (Two numbers of a
  // bf16 h would leave 2^-17 of it out: 4096 x 11008, rank 64, 52.5 us, three 56)
  typedef typename std::conditional<kNarrow, b8, F>::type P;
  constexpr bool kHalves = std::is_same<T, _Float16>::value;
  constexpr int NUMBERS = kNarrow ? 3 : 1, TERMS = kPacked && !kHalves ? 2 : NUMBERS, OF_W = kHalves && !kPacked ? 2 : 1;
  constexpr int ROWS = 16 * WIN, V = 16 * sizeof(T) / 16;  // rows; pieces of 16 bytes of a lane's columns
  // h of the window, as the instruction takes it: [term][step][row][4 pieces]
  __shared__ P hs[TERMS * S][ROWS * 4];
  __shared__ float back[ROWS];
  __shared__ int at[ROWS], of[ROWS];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int strips = (a.n + 255) / 256, window = blockIdx.x / (uint32_t)strips, strip = blockIdx.x - window * strips;
  const int first = window * ROWS;
  const int c0 = strip * 256 + w * 64 + q * 16;  // the lane's columns
  const bool whole = c0 + 16 <= a.n;
  if (t < ROWS) at[t] = row_at(a.g, first + t), of[t] = which_at(a.g, first + t);
  F fw[4][S];
  P numbers[4][kHalves ? S * OF_W : 1];  // of an f16 W
  int held = -1;  // the adapter whose W is in registers
  bool fresh = false;
  auto inner = [&](int k) { return kPacked ? q % 2 * 8 : k * M::K + q * M::E; };  // a lane's elements of step k
  // rows of tile j: lane m has column 16 (m / 4) + 4 j + m % 4 of the wave's
  auto w_row = [&](int j) {
    const int c = c0 - q * 16 + (m >> 2) * 16 + 4 * j + (m & 3);
    return (const T*)a.W + held * a.step + (int64_t)min(c, a.n - 1) * a.ldw;
  };
  auto take = [&]() __attribute__((always_inline)) {  // what hold has loaded
    if constexpr (kHalves) {
      if (!fresh) return;
      fresh = false;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < S; ++k) {
          P hi, lo;
          split(fw[j][k], hi, lo);
          if constexpr (kPacked) {
            const u4 first = __builtin_bit_cast(u4, hi), second = __builtin_bit_cast(u4, lo);
            numbers[j][k] = __builtin_bit_cast(P, q < 2 ? first : second);
          } else {
            numbers[j][k * OF_W] = hi, numbers[j][k * OF_W + 1] = lo;
          }
        }
    }
  };
  auto hold = [&](int ad) __attribute__((always_inline)) {
    if (ad >= a.g.count || ad == held) return;
    held = ad, fresh = true;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < S; ++k) fw[j][k] = load_row<SHORT>(w_row(j), inner(k), a.rank);
    if (a.rank % (kPacked ? 16 : M::K) != 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < S; ++k) end_row<SHORT>(fw[j][k], w_row(j), inner(k), a.rank);
    }
    if (S > 1) take();  // (as loaded and as numbers they would not fit the registers)
  };
  {
    // W of the work group's first adapter is on its way while h is laid out
    int mine;
    uint64_t heads = heads_of(a.g, first, ROWS, mine);
    for (int z = 0; z < (int)blockIdx.z && heads != 0; ++z) heads &= heads - 1;
    if (heads == 0 && gridDim.z > 1) return;  // the window has no more of them
    if (heads != 0) hold(__builtin_amdgcn_readlane(mine, __builtin_ctzll(heads)));
  }
  for (int i0 = t >> 2; i0 < ROWS; i0 += 64) {
    const int place = first + i0, p = t & 3;
    const int wh = which_at(a.g, place);
    const bool some = wh >= 0 && wh < a.g.count;
    const float f = some && a.scales ? a.scales[wh] : 1.0f;
    float h[S][M::E];
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int e = 0; e < M::E; ++e) h[k][e] = 0.0f;
    const float* from = a.H + (int64_t)place * a.ranks;  // (read where there is none, too: nothing waits for which)
    const int64_t part = a.places * a.ranks;
#pragma unroll 4
    for (int s = 0; s < a.parts; ++s)
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const int r = kPacked ? p % 2 * 8 : k * M::K + p * M::E;
        const f4* x = (const f4*)(from + s * part + (r < a.ranks ? r : 0));
#pragma unroll
        for (int v = 0; v < M::E / 4; ++v) {
          const f4 y = x[v];
#pragma unroll
          for (int e = 0; e < 4; ++e) h[k][4 * v + e] += y[e];
        }
      }
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int e = 0; e < M::E; ++e)
        if (!some || (kPacked ? p % 2 * 8 : k * M::K + p * M::E) >= a.ranks) h[k][e] = 0.0f;
    if (p == 0) back[i0] = f;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      if constexpr (!kNarrow) {
        F v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = h[k][e];
        hs[k][i0 * 4 + p] = v;
      } else {
        P v[4] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = h[k][e];
          v[0][e] = (bf16)split(x);
          v[1][e] = (bf16)split(x);
          v[2][e] = (bf16)x;
        }
#pragma unroll
        for (int u = 0; u < TERMS; ++u) {
          if constexpr (kPacked && !kHalves) {
            const u4 first = __builtin_bit_cast(u4, v[2 * u]), second = __builtin_bit_cast(u4, v[2 * u + 1]);
            hs[u * S + k][i0 * 4 + p] = __builtin_bit_cast(P, p < 2 ? first : second);
          } else {
            hs[u * S + k][i0 * 4 + p] = v[u];
          }
        }
      }
    }
  }
  __syncthreads();
  if (c0 - q * 16 >= a.n) return;
  // a window's part of Y, loaded some windows ahead
  constexpr int AHEAD = WIN == 1 || NK == 8 ? 1 : 3;
  u4 ahead[AHEAD][V];
  auto fetch = [&](int i, u4 to[V]) {
    if (!whole || !a.Y) return;
    const T* p = (const T*)a.Y + (int64_t)at[16 * min(i, WIN - 1) + m] * a.ldy + c0;
#pragma unroll
    for (int v = 0; v < V; ++v) to[v] = *(const u4_near*)((const char*)p + 16 * v);
  };
  // the window's adapters; a work group of many takes some of them
  const int mine = of[min(lane, ROWS - 1)], before = __shfl_up(mine, 1);
  uint64_t heads = __ballot(lane < ROWS && mine >= 0 && (lane == 0 || mine != before));
  for (int z = 0; heads != 0; heads &= heads - 1, ++z) {
    if (z % gridDim.z != blockIdx.z) continue;
    const int from = __builtin_ctzll(heads), ad = __builtin_amdgcn_readfirstlane(of[from]);
    const uint64_t rest = heads & (heads - 1);
    const int last = (rest ? __builtin_ctzll(rest) : ROWS) - 1;
#pragma unroll
    for (int b = 0; b < AHEAD; ++b) fetch(from / 16 + b, ahead[b]);
    hold(ad);
    take();
#pragma unroll 1
    for (int i = from / 16; i <= last / 16; ++i) {
      const int place = 16 * i + m;
      const bool own = place >= from && of[place] == ad;
      u4 y[V];
#pragma unroll
      for (int v = 0; v < V; ++v) y[v] = ahead[0][v];
#pragma unroll
      for (int b = 0; b + 1 < AHEAD; ++b)
#pragma unroll
        for (int v = 0; v < V; ++v) ahead[b][v] = ahead[b + 1][v];
      if (i + AHEAD <= last / 16) fetch(i + AHEAD, ahead[AHEAD - 1]);
      f4 acc[4] = {};
      if (ad < a.g.count) {
#pragma unroll
        for (int k = 0; k < S; ++k)
#pragma unroll
          for (int u = 0; u < TERMS; ++u) {
            const P h = hs[u * S + k][place * 4 + q];
#pragma unroll
            for (int o = 0; o < OF_W; ++o)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if constexpr (kHalves) acc[j] = mma(numbers[j][k * OF_W + o], h, acc[j]);
                else acc[j] = mma(fw[j][k], h, acc[j]);
              }
          }
      }
      if (!own || c0 >= a.n) continue;
      const float f = back[place];
      T* out = (T*)a.O + (int64_t)at[place] * a.ldo + c0;
      const T* from_y = (const T*)a.Y + (int64_t)at[place] * a.ldy + c0;
      float o[16];
      if (whole && a.Y) {
        typedef T E __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = (float)__builtin_bit_cast(E, y[e * sizeof(T) / 16])[e % (16 / sizeof(T))];
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = a.Y && c0 + e < a.n ? (float)from_y[e] : 0.0f;
      }
      if (ad < a.g.count) {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = fmaf(acc[e / 4][e % 4], f, o[e]);
      }
      if (whole) {
        typedef T E __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int v = 0; v < V; ++v) {
          E x;
#pragma unroll
          for (int e = 0; e < 16 / (int)sizeof(T); ++e) x[e] = (T)o[v * 16 / sizeof(T) + e];
          *(u4_near*)((char*)out + 16 * v) = __builtin_bit_cast(u4, x);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (c0 + e < a.n) out[e] = (T)o[e];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// sums over an adapter's rows
// ---------------------------------------------------------------------------

struct Outer {
  int n;
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
struct OuterArgs {
  Groups g;
  int rank, ranks, deal;  // rank, work groups of it, and those that share a window's adapters
  bool alone;             // one window, few adapters: nothing to join
  Outer of[2];            // those that are asked for
};

// A work group takes some columns, 16 RT ranks and a window of places, whose steps its
// four waves share; their sums are joined in LDS. Lane l reads 8 (16-bit) or 4 columns of
// a row at once; the pieces of 16-bit rows are turned in registers to runs of one
// column. Adapters whose rows lie in one window are done with it; of the others each window gives a
// part, at the number of the window and the adapter together (which grows along the
// order, so that no two are alike).
template <class T, int RT, bool SHORT>
__device__ __forceinline__ void outer_tile(const OuterArgs& a, const Outer& o, int strip, int window, int rank0, int share,
                                           float* red) {
  typedef Mat<T> M;
  typedef typename M::F F;
  constexpr bool kNarrow = sizeof(T) == 2;
  constexpr int C = M::E;             // column tiles: columns C m + j
  constexpr bool kHalves = std::is_same<T, _Float16>::value;
  constexpr int COLS = 16 * C, STEP = 32;  // columns, rows of a step
  constexpr int L = 8;                     // rows of a lane and step
  constexpr int PITCH = COLS + 4;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, m = lane & 15, q = lane >> 4;
  const int c0 = strip * COLS, r0 = rank0 * 16 * RT;
  const int begin = window * o.window, end = min(begin + o.window, a.g.rows);
  int i0 = begin;
  while (i0 < end) {
    const int ad = which_at(a.g, i0);
    if (ad >= a.g.count) break;
    const int from = max(a.g.start[ad], begin), to = min(a.g.start[ad + 1], end);
    if (to <= i0) break;  // (groups that are not this batch's)
    if (share-- != 0) {
      i0 = to;
      continue;
    }
    share = a.deal - 1;
    const float f = o.scales ? o.scales[ad] : 1.0f;
    // place of a lane's row e in the step from s on
    auto place = [&](int s, int e) { return kNarrow ? s + 8 * q + e : s + 4 * e + q; };
    struct Step {
      u4 z[L];
      float h[RT][L];
    };
    int rows[L];
    auto find = [&](int s) {
#pragma unroll
      for (int e = 0; e < L; ++e) rows[e] = row_at(a.g, min(place(s, e), to - 1));
    };
    auto load = [&](int s, Step& x) {
#pragma unroll
      for (int e = 0; e < L; ++e)
        x.z[e] = __builtin_bit_cast(u4, load_row<SHORT>((const T*)o.Z + (int64_t)rows[e] * o.ldz, c0 + C * m, o.n));
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int e = 0; e < L; ++e)
          x.h[j][e] = *(const float*)((const char*)o.H + ((uint32_t)(o.by_row ? rows[e] : min(place(s, e), to - 1)) * (uint32_t)o.ldh +
                                                          (uint32_t)min(r0 + 16 * j + m, a.rank - 1)) * 4u);
    };
    f4 acc[C][RT] = {};
    auto sum = [&](int s, Step& x) {
      if (c0 + COLS > o.n && c0 + C * m < o.n) {  // the last columns (those past them are not written)
#pragma unroll
        for (int e = 0; e < L; ++e) {
          F f = __builtin_bit_cast(F, x.z[e]);
          end_row<SHORT>(f, (const T*)o.Z + (int64_t)row_at(a.g, min(place(s, e), to - 1)) * o.ldz, c0 + C * m, o.n);
          x.z[e] = __builtin_bit_cast(u4, f);
        }
      }
      if (s + STEP > to) {
#pragma unroll
        for (int e = 0; e < L; ++e) {
          const bool in = place(s, e) < to;
          if (!in) x.z[e] = u4{};
#pragma unroll
          for (int j = 0; j < RT; ++j) x.h[j][e] = in ? x.h[j][e] : 0.0f;
        }
      }
      if constexpr (kNarrow) {
        b8 h[RT][3];
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float v = x.h[j][e] * f;
            h[j][0][e] = (bf16)split(v);
            h[j][1][e] = (bf16)split(v);
            h[j][2][e] = (bf16)v;
          }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          u4 col;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            col[p] = __builtin_amdgcn_perm(x.z[2 * p + 1][c / 2], x.z[2 * p][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
          b8 z[2];
          if constexpr (kHalves) split(__builtin_bit_cast(h8, col), z[0], z[1]);
          else z[0] = __builtin_bit_cast(b8, col);
#pragma unroll
          for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int u = 2; u >= 0; --u)
#pragma unroll
              for (int o = kHalves ? 1 : 0; o >= 0; --o) acc[c][j] = mma(z[o], h[j][u], acc[c][j]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < L; ++e) {
          const f4 z = __builtin_bit_cast(f4, x.z[e]);
#pragma unroll
          for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(z[c], x.h[j][e] * f, acc[c][j], 0, 0, 0);
        }
      }
    };
    // a step's loads are on their way while the one before is summed, its rows' numbers before that
    Step x, y;
    const int s0 = from + w * STEP;
    if (s0 < to) {
      find(s0);
      load(s0, x);
      find(s0 + 4 * STEP);
#pragma unroll 1
      for (int s = s0;;) {  // (x and y in turn, without copies: twice the code, which small calls wait for, and 80 registers more)
        if (s + 4 * STEP < to) load(s + 4 * STEP, y);
        find(s + 8 * STEP);
        sum(s, x);
        s += 4 * STEP;
        if (s >= to) break;
        x = y;
      }
    }
    // lane: rank m of each tile, columns C (4 q + i) + c: to rows of ranks
    __syncthreads();
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < C; c += 4) {
          f4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = acc[c + e][j][i];
          *(f4*)(red + ((w * RT + j) * 16 + m) * PITCH + C * (4 * q + i) + c) = v;
        }
    __syncthreads();
    const bool whole = a.g.rows <= o.window || (a.g.start[ad] >= begin && a.g.start[ad + 1] <= end);
    float* to_out = whole ? o.out + (int64_t)ad * o.n * a.rank : o.parts + (int64_t)(window + ad) * o.n * a.rank;
    for (int e = t; e < 16 * RT * COLS; e += 256) {
      const int r = o.across ? e / COLS : e % (16 * RT), c = o.across ? e % COLS : e / (16 * RT);
      const float* v = red + r * PITCH + c;
      constexpr int wave = RT * 16 * PITCH;
      const float s = (v[0] + v[wave]) + (v[2 * wave] + v[3 * wave]);
      if (r0 + r < a.rank && c0 + c < o.n)
        to_out[o.across ? (int64_t)(r0 + r) * o.n + c0 + c : (int64_t)(c0 + c) * a.rank + r0 + r] = s;
    }
    i0 = to;
  }
}
// (registers for three waves of a SIMD, two for 32 ranks: 8192 x 4096, rank 16, gradients 101.0 us, with two
// 102.6; 4096 x 2048, rank 64, 32 bits, 112, with one 129)
template <class T, int RT, bool SHORT>
__global__ __launch_bounds__(256, (RT == 1 ? 3 : 2)) void k_outer(OuterArgs a) {
  __shared__ float red[4 * RT * 16 * (16 * Mat<T>::E + 4)];
  const int which = blockIdx.z / (uint32_t)a.deal;
  const Outer o = a.of[which];
  // every eighth work group runs on the same die: the ranks of a strip follow one another there
  const int k = blockIdx.x >> 3, strip = k / a.ranks * 8 + (blockIdx.x & 7);
  if (strip * 16 * Mat<T>::E >= o.n || (int)blockIdx.y * o.window >= a.g.rows) return;
  if (a.alone) {
    // zeros for adapters without rows
    constexpr int COLS = 16 * Mat<T>::E;
    const int lane = threadIdx.x & 63, ad = min(lane, a.g.count - 1), c0 = strip * COLS, r0 = k % a.ranks * 16 * RT;
    uint64_t none = __ballot(lane < a.g.count && lane % a.deal == (int)blockIdx.z - which * a.deal &&
                             a.g.start[ad] >= a.g.start[ad + 1]);
    for (; none != 0; none &= none - 1) {
      float* out = o.out + (int64_t)__builtin_ctzll(none) * o.n * a.rank;
      for (int e = threadIdx.x; e < 16 * RT * COLS; e += 256) {
        const int r = o.across ? e / COLS : e % (16 * RT), c = o.across ? e % COLS : e / (16 * RT);
        if (r0 + r < a.rank && c0 + c < o.n) out[o.across ? (int64_t)(r0 + r) * o.n + c0 + c : (int64_t)(c0 + c) * a.rank + r0 + r] = 0.0f;
      }
    }
  }
  outer_tile<T, RT, SHORT>(a, o, strip, blockIdx.y, k % a.ranks, blockIdx.z - which * a.deal, red);
}

// The parts' sums, and zeros for adapters without rows.
__global__ __launch_bounds__(256) void k_outer_join(OuterArgs a) {
  const Outer o = a.of[blockIdx.z];
  const int ad = blockIdx.y;
  const int64_t size = (int64_t)o.n * a.rank;
  const int from = max(a.g.start[ad], 0), to = min(a.g.start[ad + 1], a.g.rows);
  const int w0 = from / o.window, w1 = to > from ? (to - 1) / o.window : w0;
  if (to > from && w0 == w1) return;  // (it is there already)
  float* out = o.out + ad * size;
  const float* parts = o.parts + (int64_t)(w0 + ad) * size;
  if (size % 4 == 0) {  // (out is aligned to its elements, the parts to 16 bytes)
    typedef f4 f4_near __attribute__((aligned(4)));
    for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < size; e += (int64_t)gridDim.x * 1024) {
      f4 s = {};
      if (to > from)
#pragma unroll 4
        for (int w = 0; w <= w1 - w0; ++w) s += *(const f4*)(parts + w * size + e);
      *(f4_near*)(out + e) = s;
    }
    return;
  }
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < size; e += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
    if (to > from)
      for (int w = 0; w <= w1 - w0; ++w) s += parts[w * size + e];
    out[e] = s;
  }
}

// Rows of W (rows x cols, of each adapter that has rows) as columns.
struct Turn {
  int rows, cols;
  const void* W;
  int64_t ldw, step;
  void* out;
  int64_t ldo, step_out;
};
struct TurnArgs {
  Groups g;
  Turn of[2];
};
template <class T>
__global__ __launch_bounds__(256) void k_turn(TurnArgs a) {
  __shared__ T tile[32][33];
  const int ad = blockIdx.z;
  const Turn u = a.of[blockIdx.y];
  const int tiles = (u.cols + 31) / 32, x = threadIdx.x & 31, y0 = threadIdx.x >> 5;
  const int r0 = blockIdx.x / tiles * 32, c0 = (blockIdx.x - r0 / 32 * tiles) * 32;
  if (r0 >= u.rows || a.g.start[ad] >= a.g.start[ad + 1]) return;
  for (int y = y0; y < 32; y += 8)
    if (r0 + y < u.rows && c0 + x < u.cols) tile[y][x] = ((const T*)u.W)[ad * u.step + (r0 + y) * u.ldw + c0 + x];
  __syncthreads();
  for (int y = y0; y < 32; y += 8)
    if (c0 + y < u.cols && r0 + x < u.rows) ((T*)u.out)[ad * u.step_out + (c0 + y) * u.ldo + r0 + x] = tile[x][y];
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t up(int64_t v, int64_t m) { return ceil_div(v, m) * m; }

int ranks_of(int rank) { return (int)up(rank, 16); }
// Sums over a long side of few rows: windows of 16 for whose adapters there are work groups each.
// Of many rows, and of fewer along so long a side that what windows of 16 read of W is most
// (1500 x 11008, rank 16, a call: 35 us so, 30 as of many; 1100 x 4096, rank 64, 28.3 and 26.6, rank 32 19.5 and 22),
// a work group takes its window's adapters one after another.
constexpr int kFew = 2048;
bool many_rows(int64_t rows, int64_t n, int rank) { return rows >= kFew || (rows >= kFew / 2 && n * rank >= 5 << 15); }
constexpr int kManyGroups = 512;  // work groups of many rows that run at once
// Work groups for the adapters of a window of 16: as many as a window has on average and one (a
// work group too many costs its launch: 1358 x 4224, 38 adapters, 27 us, with 16 for each 36).
int adapter_groups(int64_t rows, int count) {
  return (int)std::min<int64_t>({16, count, ceil_div(count, ceil_div(rows, 16)) + 1});
}
// Row tiles of a window: more rows read the weights more seldom.
int shrink_tiles(int64_t rows, int64_t n, int rank) { return !many_rows(rows, n, rank) || rank <= 16 ? 1 : 2; }
// Parts of the inner side, which fill the device. Few rows: four at most, which what reads h
// sums (64 rows of 4096, 48 adapters of rank 16, a call: 2 / 4 / 8 / 16 parts 16.0 / 14.9 / 15.7 / 17.8 us,
// one row 11.9 / 11.7 / 11.7 / 12.4).
// `apart`: their sums take a launch of their own, which a short side does without.
int shrink_parts(int64_t rows, int64_t n, int rank, int count, bool apart) {
  const bool many = many_rows(rows, n, rank);
  const int64_t room = ceil_div(n, apart && !many ? 1024 : 256);
  if (many) {
    // rounds of the work groups that run at once, each of its share of the side (in pieces
    // of 64) and what it takes to begin (4787 rows of 4096, rank 128, 32 bits, a call, with half as many at
    // once: three parts 122 us, four, which begin a second round, 156)
    int64_t best = 1, least = INT64_MAX;
    for (int64_t p = 1; p <= std::min<int64_t>(16, room); ++p) {
      const int64_t takes = ceil_div(ceil_div(rows, 64) * p, kManyGroups) * (ceil_div(n, 64 * p) + 6) + p;
      if (takes < least) least = takes, best = p;
    }
    return (int)best;
  }
  // an adapter begins inside a window or at its end
  const int64_t want = std::min<int64_t>(4, ceil_div(256, std::min(rows, ceil_div(rows, 16) + count - 1)));
  return (int)std::max<int64_t>(1, std::min(want, room));
}
int64_t places_of(int64_t rows) { return up(rows, 64); }
size_t h_bytes(int64_t rows, int64_t n, int rank, int count, bool apart) {
  return up256((size_t)shrink_parts(rows, n, rank, count, apart) * places_of(rows) * ranks_of(rank) * 4);
}

template <class T>
void shrink(const ShrinkArgs& a, int parts, hipStream_t s) {
  const bool many = many_rows(a.g.rows, a.n, a.rank);
  if (many && wide_rows(a.X, a.ldx, sizeof(T)) && wide_rows(a.W, a.ldw, sizeof(T)) && a.n % Mat<T>::E == 0 &&
      a.n >= 128) {
    const dim3 grid((unsigned)ceil_div(a.g.rows, 64), parts);
    if (a.rank <= 16) hipLaunchKernelGGL((k_shrink_many<T, 1>), grid, dim3(256), 0, s, a);
    else if (a.rank <= 32) hipLaunchKernelGGL((k_shrink_many<T, 2>), grid, dim3(256), 0, s, a);
    else if (a.rank <= 64) hipLaunchKernelGGL((k_shrink_many<T, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_shrink_many<T, 8>), grid, dim3(256), 0, s, a);
    return;
  }
  const bool brief = a.n < Mat<T>::E;
  const int tiles = brief ? 1 : shrink_tiles(a.g.rows, a.n, a.rank);
  const dim3 grid((unsigned)ceil_div(a.g.rows, 16 * tiles), parts, many ? 1 : adapter_groups(a.g.rows, a.g.count));
  auto of = [&](auto rt) {
    constexpr int RT = decltype(rt)::value;
    if (brief)
      hipLaunchKernelGGL((k_shrink<T, 1, RT, true>), grid, dim3(256), 0, s, a);
    else if (tiles == 1)
      hipLaunchKernelGGL((k_shrink<T, 1, RT, false>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_shrink<T, 2, RT, false>), grid, dim3(256), 0, s, a);
  };
  if (a.rank <= 16) of(std::integral_constant<int, 1>());
  else if (a.rank <= 32) of(std::integral_constant<int, 2>());
  else if (a.rank <= 64) of(std::integral_constant<int, 4>());
  else of(std::integral_constant<int, 8>());
}

template <class T>
void turn(const TurnArgs& a, int n, hipStream_t s) {
  int64_t tiles = 0;
  for (int i = 0; i < n; ++i) tiles = std::max(tiles, ceil_div(a.of[i].rows, 32) * ceil_div(a.of[i].cols, 32));
  hipLaunchKernelGGL(k_turn<T>, dim3((unsigned)tiles, n, a.g.count), dim3(256), 0, s, a);
}

template <class T>
void expand(const ExpandArgs& a, hipStream_t s) {
  // Windows of 64 rows (4096 x 11008, rank 64, a call: 32 / 64 rows 95 / 83 us; 128 take too many registers),
  // of 16 where that leaves the device without work (600 x 4096, rank 16, 22 us, of 64 28; 1200 x 11008 33 and 28;
  // 1100 x 2048, rank 64, 32 and 36, but of rank 128 37 and 34: so many rows of W are better read for 64).
  const bool few = ceil_div(a.g.rows, 64) * ceil_div(a.n, 256) < (a.rank > 64 ? 128 : 400);
  auto of = [&](auto nk) {
    constexpr int NK = decltype(nk)::value, WIN = 4;
    const int64_t strips = ceil_div(a.n, 256);
    auto as = [&](auto win, auto brief) {
      constexpr int W = decltype(win)::value;
      hipLaunchKernelGGL((k_expand<T, NK, W, decltype(brief)::value>),
                         dim3((unsigned)(ceil_div(a.g.rows, 16 * W) * strips), 1, few ? adapter_groups(a.g.rows, a.g.count + 1) : 1), dim3(256),
                         0, s, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, WIN> more;
    if constexpr (NK <= 1) {
      if (a.rank < Mat<T>::E) {
        few ? as(one, std::true_type()) : as(more, std::true_type());
        return;
      }
    }
    few ? as(one, std::false_type()) : as(more, std::false_type());
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

// Sums parts of h where there are many, or many work groups would do it for themselves again;
// returns how many are left. `out` may be h itself: an element's parts are one thread's.
template <class T>
int fold(const Groups& g, int rank, int parts, const float* h, float* out, hipStream_t s) {
  if (parts == 1 || (parts <= 4 && g.rows < kFew)) return parts;
  const FoldArgs f = {g, rank, ranks_of(rank), parts, h, places_of(g.rows), out, false};
  hipLaunchKernelGGL(k_fold, dim3((unsigned)ceil_div(g.rows * (int64_t)ranks_of(rank), 256)), dim3(256), 0, s, f);
  return 1;
}

// places of a window: as many windows as fill the device with strips of 128 columns, of 256
// places at least (two steps of each wave): fewer windows are fewer sums to join, and of a single one
// (up to 512 places) there is nothing to join
int outer_window(int64_t rows, int64_t n, int rank) {
  if (rows <= 512) return 512;
  const int64_t groups = 2 * ceil_div(n, 128) * (rank <= 16 ? 1 : ceil_div(rank, 32));
  return (int)std::max<int64_t>(256, up(ceil_div(rows, std::max<int64_t>(1, ceil_div(768, groups))), 128));
}
size_t outer_bytes(int64_t rows, int64_t n, int rank, int count) {
  const int64_t windows = ceil_div(rows, outer_window(rows, n, rank));
  return windows <= 1 ? 0 : up256((size_t)(windows + count) * n * rank * 4);
}
// the first n of a.of
template <class T>
void outer(OuterArgs a, int n, hipStream_t s) {
  int64_t strips = 0, windows = 0, size = 0;
  bool brief = false;
  for (int i = 0; i < n; ++i) {
    a.of[i].window = outer_window(a.g.rows, a.of[i].n, a.rank);
    strips = std::max(strips, ceil_div(a.of[i].n, 16 * Mat<T>::E));
    windows = std::max(windows, ceil_div(a.g.rows, a.of[i].window));
    size = std::max(size, (int64_t)a.of[i].n * a.rank);
    brief = brief || a.of[i].n < Mat<T>::E;
  }
  if (windows > 0) {
    a.ranks = a.rank <= 16 ? 1 : (int)ceil_div(a.rank, 32);
    // few work groups: a window's adapters at the same time
    const int64_t groups = strips * a.ranks * windows * n;
    a.alone = windows == 1 && a.g.count <= 64 && a.g.count * size <= 1 << 20;
    a.deal = (int)std::max<int64_t>(1, std::min<int64_t>({a.g.count, 8, 1024 / groups}));
    const dim3 grid((unsigned)(up(strips, 8) * a.ranks), (unsigned)windows, (unsigned)(n * a.deal));
    auto as = [&](auto rt, auto brief) {
      hipLaunchKernelGGL((k_outer<T, decltype(rt)::value, decltype(brief)::value>), grid, dim3(256), 0, s, a);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (a.rank <= 16) brief ? as(one, std::true_type()) : as(one, std::false_type());
    else brief ? as(two, std::true_type()) : as(two, std::false_type());
  }
  if (!a.alone)
    hipLaunchKernelGGL(k_outer_join, dim3((unsigned)std::min<int64_t>(ceil_div(size, 1024), 256), a.g.count, n), dim3(256), 0, s, a);
}

bool bad_shape(int64_t M, int64_t N, int64_t K, int R, int count) {
  const int64_t top = (int64_t)1 << 22, all = (int64_t)1 << 37;  // (work groups of 64 rows and 256 columns: 2^32 work items at most)
  return M < 0 || M > top || N < 1 || N > top || K < 1 || K > top || M * N > all || M * K > all || R < 1 || R > kMaxRank ||
         count < 1 || count > 4096;
}
Groups groups_of(const int32_t* g, int64_t M, int count) { return {g, g + M, g + 2 * M, (int)M, count}; }
struct BackSpace {
  size_t h, p, at, bt, outer[2], all;
  int64_t ldat, ldbt;
};
BackSpace back_space(int64_t M, int64_t N, int64_t K, int R, int count) {
  BackSpace b;
  b.ldat = up(R, 8), b.ldbt = up(N, 8);
  b.h = 0;
  b.p = b.h + h_bytes(M, N, R, count, true);
  b.at = b.p + up256((size_t)places_of(M) * ranks_of(R) * 4);
  b.bt = b.at + up256((size_t)count * K * b.ldat * 4);
  b.outer[0] = b.bt + up256((size_t)count * R * b.ldbt * 4);
  b.outer[1] = b.outer[0] + outer_bytes(M, K, R, count);
  b.all = b.outer[1] + outer_bytes(M, N, R, count);
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
  // as many threads as rows want, in one turn where that is enough
  const dim3 threads(M <= 1024 ? 256 : kGroupThreads);
  if (M <= 4096)
    hipLaunchKernelGGL(k_group<1>, dim3(count + 1), threads, 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(k_group<4>, dim3(count + 1), threads, 0, (hipStream_t)stream, a);
  return launched("gptq2d_adapter_groups");
}

size_t gptq2d_adapters_workspace_size(int64_t M, int64_t N, int64_t K, int R, int count) {
  if (bad_shape(M, N, K, R, count) || M == 0) return 0;
  return h_bytes(M, K, R, count, false);
}

gptq2d_status gptq2d_adapters(int64_t M, int64_t N, int64_t K, int R, int count, gptq2d_dtype dt, const void* X, int64_t ldx,
                              const void* A, int64_t lda, const void* B, int64_t ldb, const float* scales,
                              const int32_t* groups, const void* Y, int64_t ldy, void* O, int64_t ldo, float* H,
                              void* workspace, size_t ws_bytes, void* stream) {
  if (bad_shape(M, N, K, R, count)) return refuse("M, N and K must lie in [1, 2^22] (M may be 0), M N and M K in [0, 2^37], R in [1, 128], count in [1, 4096]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (M == 0) return GPTQ2D_OK;
  if (!X || !A || !B || !groups || !O) return refuse("X, A, B, groups or O is NULL");
  if (ldx < K || lda < K || ldb < R || (Y && ldy < N) || ldo < N) return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  if (!aligned(X, es) || !aligned(A, es) || !aligned(B, es) || !aligned(Y, es) || !aligned(O, es) || !aligned(scales, 4) ||
      !aligned(groups, 4) || !aligned(H, 4))
    return refuse("an argument is not aligned to its elements");
  const size_t need = h_bytes(M, K, R, count, false);
  if (!workspace || ws_bytes < need) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const hipStream_t s = (hipStream_t)stream;
  const Groups g = groups_of(groups, M, count);
  const int parts = shrink_parts(M, K, R, count, false);
  float* h = (float*)workspace;
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const ShrinkArgs sh = {g, (int)K, R, ranks_of(R), X, ldx, A, lda, R * lda, nullptr, h, places_of(M)};
    shrink<T>(sh, parts, s);
    if (H) {
      const FoldArgs f = {g, R, ranks_of(R), parts, h, places_of(M), H, true};
      hipLaunchKernelGGL(k_fold, dim3((unsigned)ceil_div(M * R, 256)), dim3(256), 0, s, f);
    }
    const int left = fold<T>(g, R, parts, h, h, s);
    const ExpandArgs e = {g, (int)N, R, ranks_of(R), left, h, places_of(M), scales, B, ldb, N * ldb, Y, ldy, O, ldo};
    expand<T>(e, s);
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
  if (bad_shape(M, N, K, R, count)) return refuse("M, N and K must lie in [1, 2^22] (M may be 0), M N and M K in [0, 2^37], R in [1, 128], count in [1, 4096]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (M > 0 && !dX && !dA && !dB) return refuse("no gradient is asked for");  // (of no rows dX may be NULL)
  if (!groups) return refuse("groups is NULL");
  if (M == 0) {  // nothing but zeros
    if (!dA && !dB) return GPTQ2D_OK;
    OuterArgs o = {groups_of(groups, 0, count), R, 1, 1, false, {}};
    int n = 0;
    if (dA) o.of[n].n = (int)K, o.of[n++].out = dA;
    if (dB) o.of[n].n = (int)N, o.of[n++].out = dB;
    outer<float>(o, n, (hipStream_t)stream);
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
  float *h = (float*)(ws + b.h), *pr = (float*)(ws + b.p);
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const float* ph = h;
    if (dX || dA) {
      const Turn of_b = {(int)N, R, B, ldb, N * ldb, ws + b.bt, b.ldbt, R * b.ldbt};
      const Turn of_a = {R, (int)K, A, lda, R * lda, ws + b.at, b.ldat, K * b.ldat};
      turn<T>({g, {of_b, of_a}}, dX ? 2 : 1, s);
      const int parts = shrink_parts(M, N, R, count, true);
      const ShrinkArgs sh = {g, (int)N, R, ranks_of(R), G, ldg, ws + b.bt, b.ldbt, R * b.ldbt, scales, h, places_of(M)};
      shrink<T>(sh, parts, s);
      if (parts > 1) {
        const FoldArgs f = {g, R, ranks_of(R), parts, h, places_of(M), pr, false};
        hipLaunchKernelGGL(k_fold, dim3((unsigned)ceil_div(M * ranks_of(R), 256)), dim3(256), 0, s, f);
        ph = pr;
      }
    }
    OuterArgs o = {g, R, 1, 1, false, {}};
    int n = 0;
    if (dA) o.of[n++] = {(int)K, X, ldx, ph, ranks_of(R), false, nullptr, dA, true, 0,
                         (float*)(ws + b.outer[0])};
    if (dB) o.of[n++] = {(int)N, G, ldg, H, R, true, scales, dB, false, 0, (float*)(ws + b.outer[1])};
    if (n > 0) outer<T>(o, n, s);
    if (dX) {
      const ExpandArgs e = {g, (int)K, R, ranks_of(R), 1, ph, places_of(M), nullptr, ws + b.at, b.ldat, K * b.ldat, D, ldd, dX,
                            lddx};
      expand<T>(e, s);
    }
  });
  return launched("gptq2d_adapters_backward");
}

}  // extern "C"
