// Matrices in eight-bit floating point (e4m3) with a 32-bit scale for each
// block of 128 values: the quantiser and the product
//   C[m][n] = sum_b SA[b][m] SB[b][n] sum_{k in block b} A[m][k] B[n][k].
#include <algorithm>
#include <type_traits>

#include "codes.hpp"

namespace g2d {
namespace {

constexpr int kBlock = 128;
// rows that the product quantises by itself: at 4096 x 4096 1 / 2 / 4 rows took 5.3 /
// 6.6 / 8.1 us, against 7.8 us after a launch of the quantiser
constexpr int kFusedRows = 2;

// ---------------------------------------------------------------------------
// Quantiser
// ---------------------------------------------------------------------------

struct QuantArgs {
  int64_t rows, cols;
  const void* X;
  int64_t ldx;
  uint8_t* Q;
  int64_t ldq;
  float* S;
  int64_t lds;
  uint8_t* QT;
  int64_t ldqt;
  float* ST;
  int64_t ldst;
  bool pow2, wide;
};

// Codes of the first n of eight columns; the rest up to the next multiple of
// 16 is inside the row (its leading dimension is one) and becomes code 0.
__device__ __forceinline__ void put8(uint8_t* p, u2 q) { *(u2*)p = q; }

// Blocks of 1 x 128, 16 lanes each, eight values a lane: one 16-byte load of a
// 16-bit type, the largest magnitude over the 16 lanes without LDS, one 8-byte
// store. Bound by its bytes: 8192 x 4096 bf16 25.9 us, 3.9 TB/s read and written
// (a large copy reaches 4.9).
template <class T>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantArgs a) {
  const int64_t nb = (a.cols + kBlock - 1) / kBlock, total = a.rows * nb;
  for (int64_t id = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); id < total; id += (int64_t)gridDim.x * 16) {
    const int64_t row = id / nb, b = id - row * nb;
    const int64_t c0 = b * kBlock + (threadIdx.x & 15) * 8;
    const int n = (int)min((int64_t)8, a.cols - c0);
    float x[8];
    load8((const T*)a.X + row * a.ldx + c0, a.wide && n == 8, n, x, (const T*)a.X);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, mag(x[i]));
    m = group_max<16>(m);
    const float s = block_scale(m, 1.0f / kTopE4M3, a.pow2);
    const u2 q = code8<false>(x, 1.0f / s, bad_amax(m));
    if (c0 < (a.cols + 15) / 16 * 16) put8(a.Q + row * a.ldq + c0, q);
    if ((threadIdx.x & 15) == 0) a.S[b * a.lds + row] = s;
  }
}

// One 128 x 128 tile per work group, read once: thread t holds the 8 x 8
// values of rows 8 (t / 16) and columns 8 (t % 16). TILE: one scale for the
// tile; otherwise one for each row (Q) and one for each column (QT). Codes of the
// transpose are turned through LDS, so that both directions store whole pieces.
// Bound by its bytes, with the exchange through LDS not hidden: 2047 x 11008 bf16 to
// both 25.3 us, 3.6 TB/s; 2047 x 4096 to the transpose 9.4 us, 2.7 TB/s; a few tiles
// 5 us (one way), 7.5 us (both).
template <class T, bool TILE>
__global__ __launch_bounds__(256) void k_quantize_tile(QuantArgs a) {
  __shared__ __align__(16) uint32_t colmax[4][kBlock + 4];
  __shared__ __align__(16) uint8_t turned[kBlock][kBlock + 16];
  const int t = threadIdx.x, tr = t >> 4, tc = t & 15;
  const int64_t nc = (a.cols + kBlock - 1) / kBlock, by = blockIdx.x / nc, bx = blockIdx.x - by * nc;
  const int64_t r0 = by * kBlock, c0 = bx * kBlock;
  const int64_t rows = a.rows - r0, cols = a.cols - c0;  // of the tile on
  float x[8][8];
  uint32_t rm[8], cm[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cm[i] = 0;
  // one way for the whole tile, so that no row's loads wait for another's (2405 x 768
  // bf16 10.6 us with a choice in each row)
  if (a.wide && (cols >= kBlock || cols % 8 == 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T* p = (const T*)a.X + (r0 + min((int64_t)8 * tr + i, rows - 1)) * a.ldx + c0;
      load8(p + (8 * tc < cols ? 8 * tc : 0), true, 8, x[i], p);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 8 * tr + i < rows && 8 * tc < cols ? x[i][j] : 0.0f;
  } else {
    const int n = (int)max((int64_t)0, min((int64_t)8, cols - 8 * tc));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = 8 * tr + i;
      load8((const T*)a.X + (r0 + r) * a.ldx + c0 + 8 * tc, false, r < rows ? n : 0, x[i], (const T*)a.X);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    rm[i] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = mag(x[i][j]);
      rm[i] = max(rm[i], m);
      cm[j] = max(cm[j], m);
    }
  }
  if constexpr (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, rm[i]);
    m = group_max<64>(m);
    if ((t & 63) == 0) colmax[0][t >> 6] = m;
    __syncthreads();
    m = max(max(colmax[0][0], colmax[0][1]), max(colmax[0][2], colmax[0][3]));
    const float s = block_scale(m, 1.0f / kTopE4M3, a.pow2);
    if (t == 0) {
      if (a.Q) a.S[by * a.lds + bx] = s;
      if (a.QT) a.ST[bx * a.ldst + by] = s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) rm[i] = cm[i] = m;
  }
  if (a.Q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = 8 * tr + i;
      if constexpr (!TILE) rm[i] = group_max<16>(rm[i]);
      const float s = block_scale(rm[i], 1.0f / kTopE4M3, a.pow2);
      const u2 q = code8<false>(x[i], 1.0f / s, bad_amax(rm[i]));
      if (r < rows) {
        if (8 * tc < (cols + 15) / 16 * 16) put8(a.Q + (r0 + r) * a.ldq + c0 + 8 * tc, q);
        if (!TILE && tc == 0) a.S[bx * a.lds + r0 + r] = s;
      }
    }
  }
  if (a.QT) {
    if constexpr (!TILE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {  // over the wave's 32 rows
        cm[j] = quad_max(cm[j]);
        if ((tr & 3) == 0) colmax[tr >> 2][8 * tc + j] = cm[j];
      }
      __syncthreads();
      if (t < kBlock) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, colmax[i][t]);
        colmax[0][t] = m;
        if (t < cols) a.ST[by * a.ldst + c0 + t] = block_scale(m, 1.0f / kTopE4M3, a.pow2);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) cm[j] = colmax[0][8 * tc + j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = 1.0f / block_scale(cm[j], 1.0f / kTopE4M3, a.pow2);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i][j];
      // (16-byte pieces of column c lie at piece ^ (c / 16): lanes meet twice in a bank, not eight times)
      *(u2*)&turned[8 * tc + j][8 * (tr ^ (tc & 14))] = code8<false>(y, r, bad_amax(cm[j]));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = t + 256 * i, c = e >> 3, k = (e & 7) * 16;
      if (c < cols && k < rows) *(u4*)(a.QT + (c0 + c) * a.ldqt + r0 + k) = *(const u4*)&turned[c][k ^ (c >> 4) * 16];
    }
  }
}

template <class T>
void quantize_typed(const QuantArgs& a, bool tile, hipStream_t s) {
  const int64_t nr = ceil_div(a.rows, kBlock), nc = ceil_div(a.cols, kBlock);
  if (!tile && !a.QT) {
    hipLaunchKernelGGL(k_quantize_rows<T>, dim3((unsigned)std::min<int64_t>(1 << 20, ceil_div(a.rows * nc, 16))), dim3(256), 0, s, a);
  } else {
    auto k = tile ? k_quantize_tile<T, true> : k_quantize_tile<T, false>;
    hipLaunchKernelGGL(k, dim3((unsigned)(nc * nr)), dim3(256), 0, s, a);
  }
}

void quantize(const QuantArgs& a, gptq2d_dtype dt, bool tile, hipStream_t s) {
  with_type(dt, [&](auto* p) { quantize_typed<std::remove_pointer_t<decltype(p)>>(a, tile, s); });
}

// ---------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------

struct ProductArgs {
  int M, N, K;        // Y (M x N) = X (M x K) W (N x K)^T
  const uint8_t* W;   // N x K
  int64_t ldw;
  const float* SW;    // ROWS: [block][n], otherwise [n / 128][block]
  int64_t ldsw;
  const void* X;      // M x K: codes (unless the kernel quantises by itself)
  int64_t ldx;
  bool pow2;          // what it quantises has scales of powers of two
  const float* SX;    // [block][m]
  int64_t ldsx;
  void* Y;
  int64_t ldy;
  bool ywide;         // four consecutive results of a row are aligned to be stored at once
  float* part;        // splits > 1: partial sums, [split][m][n]
  int splits;
};

typedef __attribute__((address_space(3))) void lds_void;

// Piece c of 16 codes of a row's last block at p, of whose codes n are there:
// zeros after them. (Rows reach to a multiple of 16 codes, so a piece that starts
// before the end can be read whole; for the others the first is read, so that no
// load waits for a branch.)
__device__ __forceinline__ u4 tail16(const uint8_t* p, int c, int n) {
  n -= 16 * c;
  u4 v = *(const u4*)(p + (n > 0 ? 16 * c : 0));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int keep = min(max(n - 4 * i, 0), 4);
    v[i] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1;
  }
  return v;
}

// R rows of an operand, from row r0 on, go into LDS 128 codes deep at a time, row
// by row (128 bytes each). Chunk c of 16 bytes of row r lies at chunk c ^ (r / 2 % 8),
// so that rows read at the same k spread over the banks. Rows past the
// last are the last one's (their products are not stored).
template <int R, int THREADS>
struct Stage {
  static constexpr int N = R * 8 / THREADS;
  const uint8_t* base;  // of row r0
  uint32_t at[N];       // below 2^31: up to 256 rows of up to 2^23 bytes
  __device__ __forceinline__ void init(const uint8_t* src, int64_t ld, int r0, int rows) {
    base = src + (int64_t)r0 * ld;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + i * THREADS, r = e >> 3;
      at[i] = (uint32_t)(min(r, rows - 1 - r0) * (int)ld + (((e & 7) ^ ((r >> 1) & 7)) << 4));
    }
  }
  __device__ __forceinline__ void piece(int i, uint8_t* dst, int k0) const {
    __builtin_amdgcn_global_load_lds((const void*)(base + k0 + at[i]),
                                     (lds_void*)(dst + (i * THREADS + (threadIdx.x & ~63)) * 16), 16, 0, 0);
  }
  __device__ __forceinline__ void tail(uint8_t* dst, int k0, int K) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + i * THREADS, c = (e & 7) ^ ((e >> 4) & 7);
      *(u4*)(dst + e * 16) = tail16(base + k0 + at[i] - 16 * c, c, K - k0);
    }
  }
};

// The lane's 32 codes of a row: pieces g and g + 4 of 16 (which codes of the block
// a lane holds is free, as long as both operands agree; pieces 2 g and 2 g + 1
// meet in the banks, at 8.1 cycles a read of the wave where these take 4.9)
__device__ __forceinline__ i8v frag(const uint8_t* tile, int row, int g) {
  const u4 lo = *(const u4*)(tile + row * kBlock + (g ^ ((row >> 1) & 7)) * 16);
  const u4 hi = *(const u4*)(tile + row * kBlock + ((g + 4) ^ ((row >> 1) & 7)) * 16);
  return __builtin_bit_cast(i8v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// the lane's 32 codes as four operands of eight halves
__device__ __forceinline__ void widen(i8v v, h8 h[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const h2 a = halves<false, false>(v[2 * i]), b = halves<false, true>(v[2 * i]);
    const h2 c = halves<false, false>(v[2 * i + 1]), d = halves<false, true>(v[2 * i + 1]);
    h[i] = h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
}

// The work group's tile, so that the groups of one XCD (dispatched round-robin
// over eight) take neighbouring tiles: eight rows of tiles at a time, so both
// operands' panels stay in its L2.
__device__ __forceinline__ void tile_of(int id, int total, int tn, int tm, int& bn, int& bm) {
  const int q = total / 8, r = total % 8, x = id % 8;
  int w = x * q + min(x, r) + id / 8;
  const int per = 8 * tn, grp = w / per, first = grp * 8, h = min(8, tm - first);
  w -= grp * per;
  bm = first + w % h;
  bn = w / h;
}

// acc + p a b for two scales, wherever the result is in range. Where one scale is below
// one and the other is not, their product is as well; otherwise p may take them one by one.
__device__ __forceinline__ float add_scaled(float p, float a, float b, float acc) {
  const bool first = (fabsf(a) >= 1.0f) != (fabsf(b) >= 1.0f);
  return fmaf(p * (first ? a * b : a), first ? 1.0f : b, acc);
}

template <class T>
__device__ __forceinline__ void put4(T* p, bool wide, int n, f4 v) {
  if (wide && n >= 4) {
    if constexpr (sizeof(T) == 4) {
      *(f4*)p = v;
    } else {
      typedef T V __attribute__((ext_vector_type(4)));
      *(u2*)p = __builtin_bit_cast(u2, V{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

// BN x BM tile of Y^T per work group, WN x WM waves. The weights are the
// instruction's row operand, so a lane's accumulator holds four consecutive n of
// one m: its scale is one register for X and one uniform value for W.
// Each 128-deep block is summed by itself and enters the accumulators with its scale.
// EXACT: the codes are widened to halves (which hold them exactly) and summed
// by the 16-bit instruction. The eight-bit one aligns its products to about
// 14 bits below the largest (measured 1.5e-5 rms of the sum of magnitudes, 3e-4 at
// most, where few products tower over the others). A 16-bit result's own rounding covers that: off by 2.07e-4
// (f16) and 1.65e-3 (bf16) rms where only rounded at the end, it is off by 2.07e-4 to
// 2.15e-4 and 1.65e-3 to 1.67e-3, at K = 128 and 11008 alike, with loud channels or
// magnitudes over 2^12. A 32-bit result's does not.
//
// The whole of a block's codes comes into LDS while the one before it is multiplied.
// Measured, by tile: 256 x 256 at 8192 x 11008 x 4096 bf16 356 us (2.07 PFLOP/s; a large
// library product reaches 2.67); what bounds it are issue slots: when it took 387, it
// took 278 without the scales' multiply-adds and 322 without its loads. 128 x 128 at
// 2048 x 4096 x 11008 94 us (1.97 PFLOP/s), EXACT and ROWS at 11008 x 4096 x 2047 215 us
// (0.86, of the 1.1 that a large product of 16-bit matrices reaches); 64 x 64 at 333 x
// 1000 x 700 6.8 us, which is six blocks' latency (with the loads of three blocks on
// their way no less). Tiles of 32 x 32 of the instruction were no faster (437 against 428
// us at 128 x 128).
template <class T, int BN, int BM, int WN, int WM, bool ROWS, bool EXACT>
__global__ __launch_bounds__(64 * WN * WM) void k_product(ProductArgs a, int tn, int tm) {
  constexpr int THREADS = 64 * WN * WM, TN = BN / WN / 16, TM = BM / WM / 16;
  // four arrays, not two of two: the compiler then knows that the loads into the
  // next block's do not touch what is being read
  __shared__ __align__(16) uint8_t w0[BN * kBlock], w1[BN * kBlock], x0[BM * kBlock], x1[BM * kBlock];
  // A block's scales, one a thread: X's BM, then those of W's BN rows, which come this
  // way also where they are one: read for the step from memory it costs 4 % of a
  // large product.
  __shared__ __align__(16) float s0[THREADS], s1[THREADS];
  static_assert(BM + BN <= THREADS, "one scale a thread");
  int bn, bm;
  tile_of(blockIdx.x, gridDim.x, tn, tm, bn, bm);
  const int n0 = bn * BN, m0 = bm * BM;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 15, g = l >> 4;
  const int wn = (w % WN) * (BN / WN), wm = (w / WN) * (BM / WM);
  const int nb = (a.K + kBlock - 1) / kBlock;
  const int b0 = (int)((int64_t)nb * blockIdx.y / a.splits), b1 = (int)((int64_t)nb * (blockIdx.y + 1) / a.splits);
  f4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = f4{0, 0, 0, 0};
  Stage<BN, THREADS> gw;
  Stage<BM, THREADS> gx;
  const bool xs = w < BM / 64;  // (whole waves)
  const int64_t psl = xs ? a.ldsx : ROWS ? a.ldsw : 1;
  const float* ps;
  auto init = [&](int n, int m) {
    gw.init(a.W, a.ldw, n, a.N);
    gx.init((const uint8_t*)a.X, a.ldx, m, a.M);
    const int at = xs ? min(m + (int)threadIdx.x, a.M - 1) : min(n + (int)threadIdx.x - BM, a.N - 1);
    ps = xs ? a.SX + at : ROWS ? a.SW + at : a.SW + at / kBlock * a.ldsw;
  };
  init(n0, m0);
  auto scales = [&](int b, float* ms) {
    __builtin_amdgcn_global_load_lds((const void*)(ps + b * psl), (lds_void*)(ms + (threadIdx.x & ~63)), 4, 0, 0);
  };
  // the i-th of `parts` shares of a whole block's loads
  constexpr int LOADS = Stage<BN, THREADS>::N + Stage<BM, THREADS>::N;
  auto share = [&](int b, uint8_t* lw, uint8_t* lx, int i, int parts) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      if (j < LOADS * i / parts || j >= LOADS * (i + 1) / parts) continue;
      if (j < Stage<BN, THREADS>::N)
        gw.piece(j, lw, b * kBlock);
      else
        gx.piece(j - Stage<BN, THREADS>::N, lx, b * kBlock);
    }
  };
  auto tails = [&](int b, uint8_t* lw, uint8_t* lx) {
    gw.tail(lw, b * kBlock, a.K);
    gx.tail(lx, b * kBlock, a.K);
  };
  // block b, which lies in lw, lx and ls, while the next one comes into mw, mx and
  // ms. SPREAD: it is whole, and its loads are spread over this one's products
  // (issued at once they hold up every wave until the memory pipeline has taken them).
  // CARE: sums are scaled one scale at a time where the product of the two, or one of
  // them, could leave the range; otherwise `rare` tells of scales where that may be.
  bool rare = false;
  auto step = [&](int b, const uint8_t* lw, const uint8_t* lx, const float* ls, uint8_t* mw, uint8_t* mx, float* ms,
                  auto spread, auto care) {
    constexpr bool SPREAD = decltype(spread)::value, CARE = decltype(care)::value;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this block's codes and scales are in LDS
    __syncthreads();
    float sx[TM];
    const float u = ROWS ? 1.0f : ls[BM + wn];
#pragma unroll
    for (int j = 0; j < TM; ++j) sx[j] = ls[wm + 16 * j + c] * u;
    if (SPREAD || b + 1 < b1) scales(b + 1, ms);
    if (!SPREAD && b + 1 < b1) {
      if ((b + 2) * kBlock <= a.K)
        share(b + 1, mw, mx, 0, 1);
      else
        tails(b + 1, mw, mx);
    }
    f4 sw = {1, 1, 1, 1};
    auto scaled = [&](int i, int j, f4 p) {
      if (ROWS && j == 0) sw = *(const f4*)&ls[BM + wn + 16 * i + 4 * g];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc[i][j][e] = CARE ? add_scaled(p[e], ROWS ? sw[e] : u, ls[wm + 16 * j + c], acc[i][j][e])
                            : fmaf(ROWS ? p[e] * sw[e] : p[e], sx[j], acc[i][j][e]);
    };
    if constexpr (EXACT) {
      h8 fx[TM][4];
#pragma unroll
      for (int j = 0; j < TM; ++j) widen(frag(lx, wm + 16 * j + c, g), fx[j]);
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        if constexpr (SPREAD) share(b + 1, mw, mx, i, TN);
        h8 fw[4];
        widen(frag(lw, wn + 16 * i + c, g), fw);
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          f4 p = {0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(fw[k], fx[j][k], p, 0, 0, 0);
          scaled(i, j, p);
        }
      }
    } else {
      // the sums of one row of blocks are scaled while the next one's are formed
      i8v fx[TM], fw = frag(lw, wn + c, g);
#pragma unroll
      for (int j = 0; j < TM; ++j) fx[j] = frag(lx, wm + 16 * j + c, g);
      f4 p[2][TM];
#pragma unroll
      for (int i = 0; i <= TN; ++i) {
        if (i < TN) {
          if constexpr (SPREAD) share(b + 1, mw, mx, i, TN);
          const i8v now = fw;
          if (i + 1 < TN) fw = frag(lw, wn + 16 * (i + 1) + c, g);
#pragma unroll
          for (int j = 0; j < TM; ++j)
            p[i & 1][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(now, fx[j], f4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
        }
        if (i > 0) {
#pragma unroll
          for (int j = 0; j < TM; ++j) scaled(i - 1, j, p[(i - 1) & 1][j]);
        }
        if (i > 0 && i < TN) {
#pragma unroll
          for (int j = 0; j < TM; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);             // a product
            __builtin_amdgcn_sched_group_barrier(0x002, ROWS ? 8 : 4, 0);  // and the scaling of one before it
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (!CARE) {  // (here, where no product waits for it)
      if constexpr (ROWS) {
        // (the work group's threads have them all; the place is formed anew, as 256 x 256
        // has no register left to hold it)
        int e = threadIdx.x;
        asm volatile("" : "+v"(e));
        const float v = fabsf(ls[e]);
        rare |= v < 0x1p-100f || v > 0x1p100f;
      } else {
#pragma unroll
        for (int j = 0; j < TM; ++j) rare |= !__builtin_amdgcn_classf(sx[j], 0x10b);  // neither normal nor NaN
      }
    }
  };
  auto begin = [&]() {
    if (b0 >= b1) return;
    scales(b0, s0);
    if ((b0 + 1) * kBlock <= a.K)
      share(b0, w0, x0, 0, 1);
    else
      tails(b0, w0, x0);
  };
  auto rest = [&](int b, auto care) {
    for (bool odd = false; b < b1; ++b, odd = !odd)
      step(b, odd ? w1 : w0, odd ? x1 : x0, odd ? s1 : s0, odd ? w0 : w1, odd ? x0 : x1, odd ? s0 : s1,
           std::false_type(), care);
  };
  int b = b0;
  begin();
  for (const int e = min(b1, a.K / kBlock) - 1; b + 1 < e; b += 2) {
    step(b, w0, x0, s0, w1, x1, s1, std::true_type(), std::false_type());
    step(b + 1, w1, x1, s1, w0, x0, s0, std::true_type(), std::false_type());
  }
  rest(b, std::false_type());  // up to three
  // The whole tile once more where a scale called for it, which finite values of ordinary
  // sizes never do: 8192 x 11008 x 4096 takes 348 us with and without this. (A choice in
  // every step takes 280 to 320 registers and spills at 256 x 256.)
  if (__syncthreads_or(rare)) {
    int n1 = n0, m1 = m0;  // (unknown to the compiler, which would hold addresses in registers for this)
    asm("" : "+s"(n1), "+s"(m1));
    init(n1, m1);
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = f4{0, 0, 0, 0};
    begin();
    rest(b0, std::true_type());
    __syncthreads();
  }
  // Each wave turns its results through LDS, 16 rows of Y at a time, and stores them
  // row by row, whole lines at a time. Straight from the registers, four results of a
  // lane's row: 3313 x 5770 x 482 bf16 (rows off the 16-byte boundaries) 51 us, now
  // 41; 8192 x 11008 x 4096 394 and 380 us. (Vectors from where a row's own addresses
  // allow them are no faster than one element a lane.)
  constexpr int EN = BN / WN, PITCH = EN + 4, PER = WN * WM / 4;
  static_assert(PER * 16 * PITCH * 4 <= (BN < BM ? BN : BM) * kBlock, "staged results fit");
  float* own = (float*)(w / PER == 0 ? w0 : w / PER == 1 ? w1 : w / PER == 2 ? x0 : x1) + w % PER * (16 * PITCH);
  auto store = [&](auto* y, int64_t ldy, bool wide) {
    y += (int64_t)(m0 + wm) * ldy + n0 + wn;
    const int rows = a.M - m0 - wm, cols = a.N - n0 - wn;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
#pragma unroll
      for (int i = 0; i < TN; ++i) *(f4*)&own[c * PITCH + 16 * i + 4 * g] = acc[i][j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (LDS keeps a wave's order)
      if (wide) {
#pragma unroll
        for (int e = l; e < 4 * EN; e += 64) {
          const int r = e / (EN / 4), n = e % (EN / 4) * 4;
          if (16 * j + r < rows && n < cols)
            put4(y + (16 * j + r) * ldy + n, true, cols - n, *(const f4*)&own[r * PITCH + n]);
        }
      } else {
#pragma unroll 8
        for (int e = l; e < 16 * EN; e += 64) {
          const int r = e / EN, n = e % EN;
          if (16 * j + r < rows && n < cols)
            y[(16 * j + r) * ldy + n] = (std::remove_pointer_t<decltype(y)>)own[r * PITCH + n];
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  };
  if (a.splits > 1)
    store(a.part + (int64_t)blockIdx.y * a.M * a.N, a.N, (a.N & 3) == 0);
  else
    store((T*)a.Y, a.ldy, a.ywide);
}

// Few rows (M <= 16 TM): the weights are read once, straight into the
// instruction's registers, 16 rows a work group; its eight waves take every
// eighth block of 128, the loads of four of them at once, and add up in LDS in
// the order of the waves.
// FUSED (rows of X, at least M; 0: X is codes): X comes as it is, and each wave
// quantises the blocks it takes, two values a lane (K and ldx are even), through
// LDS of its own. Every work group does that for itself, which for few rows costs
// less than a launch before this one.
// 256 work groups, one a compute unit, have all blocks of 4096 columns on their way in
// one turn: what 1 x 4096 x 4096 takes, 5.9 us (2.8 TB/s; in a loop from the last-level
// cache), is the launch, one memory latency and what follows it.
template <class T, int TM, bool ROWS, bool EXACT, int FUSED>
__global__ __launch_bounds__(512) void k_thin(ProductArgs a) {
  constexpr int U = TM == 1 ? 4 : TM == 2 ? 2 : 1;  // (with more, two work groups do not fit a compute unit's registers)
  __shared__ f4 sum[8][TM][64];
  __shared__ __align__(16) uint8_t own[FUSED ? 8 : 1][U][FUSED ? FUSED : 1][kBlock];
  const int n0 = blockIdx.x * 16, l = threadIdx.x & 63, c = l & 15, g = l >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nb = (a.K + kBlock - 1) / kBlock;
  const uint8_t* pw = a.W + (int64_t)min(n0 + c, a.N - 1) * a.ldw;
  f4 acc[TM];
#pragma unroll
  for (int j = 0; j < TM; ++j) acc[j] = f4{0, 0, 0, 0};
  // pieces 2 g and 2 g + 1 of a row's block; those past the end of the row are
  // read from the block's start, and masked once they are there
  auto load = [&](const uint8_t* row, int b) {
    const uint8_t* p = row + b * kBlock;
    const int left = a.K - b * kBlock;
    const u4 lo = *(const u4*)(p + (32 * g < left ? 32 * g : 0)), hi = *(const u4*)(p + (32 * g + 16 < left ? 32 * g + 16 : 0));
    return __builtin_bit_cast(i8v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto mask = [&](i8v& v, int b) {
    const int left = a.K - b * kBlock - 32 * g;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int keep = min(max(left - 4 * i, 0), 4);
      v[i] &= keep == 4 ? -1 : (1 << (8 * keep)) - 1;
    }
  };
  for (int b0 = w; b0 < nb; b0 += 8 * U) {
    i8v fw[U], fx[U][TM];
    f4 sw[U];
    struct alignas(2 * sizeof(T)) Pair { T v[2]; };
    Pair raw[U][FUSED ? FUSED : 1];
    float sx[U][TM];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = min(b0 + 8 * u, nb - 1);
      fw[u] = load(pw, b);
      if constexpr (ROWS) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[u][e] = a.SW[b * a.ldsw + min(n0 + 4 * g + e, a.N - 1)];
      } else {
        const float v = a.SW[(int64_t)(n0 / kBlock) * a.ldsw + b];
        sw[u] = f4{v, v, v, v};
      }
      if constexpr (FUSED) {
        const int k = min(b * kBlock + 2 * l, a.K - 2);
#pragma unroll
        for (int m = 0; m < FUSED; ++m)
          raw[u][m] = *(const Pair*)((const T*)a.X + (int64_t)min(m, a.M - 1) * a.ldx + k);
      } else {
#pragma unroll
        for (int j = 0; j < TM; ++j) {
          const int m = min(16 * j + c, a.M - 1);
          fx[u][j] = load((const uint8_t*)a.X + (int64_t)m * a.ldx, b);
          sx[u][j] = a.SX[b * a.ldsx + m];
        }
      }
    }
    if constexpr (FUSED) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = min(b0 + 8 * u, nb - 1) * kBlock + 2 * l < a.K;
#pragma unroll
        for (int m = 0; m < FUSED; ++m) {
          if (m >= a.M) break;
          const float x = in ? (float)raw[u][m].v[0] : 0.0f, y = in ? (float)raw[u][m].v[1] : 0.0f;
          const uint32_t top = group_max<64>(max(mag(x), mag(y)));
          const float s = block_scale(top, 1.0f / kTopE4M3, a.pow2), r = 1.0f / s;
          const uint32_t q = bad_amax(top) ? 0 : code4<false>(x * r, y * r, 0.0f, 0.0f);
          *(uint16_t*)&own[w][u][m][2 * l] = (uint16_t)q;
          if (m == 0 || m == min(c, a.M - 1)) sx[u][0] = s;
        }
      }
      // (the wave reads what it wrote itself: LDS keeps its order)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u4* p = (const u4*)&own[w][u][min(c, a.M - 1)][32 * g];
        const u4 lo = p[0], hi = p[1];
        fx[u][0] = __builtin_bit_cast(i8v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = b0 + 8 * u;
      if (b >= nb) break;
      if ((b + 1) * kBlock > a.K) {
        mask(fw[u], b);
#pragma unroll
        for (int j = 0; j < TM; ++j)
          if (!FUSED) mask(fx[u][j], b);
      }
      h8 hw[4];
      if constexpr (EXACT) widen(fw[u], hw);
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        f4 p = {0, 0, 0, 0};
        if constexpr (EXACT) {
          h8 hx[4];
          widen(fx[u][j], hx);
#pragma unroll
          for (int k = 0; k < 4; ++k) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(hw[k], hx[k], p, 0, 0, 0);
        } else {
          p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[u], fx[u][j], p, 0, 0, 0, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = add_scaled(p[e], sw[u][e], sx[u][j], acc[j][e]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < TM; ++j) sum[w][j][l] = acc[j];
  __syncthreads();
  for (int j = w; j < TM; j += 8) {
    f4 v = sum[0][j][l];
#pragma unroll
    for (int i = 1; i < 8; ++i) v += sum[i][j][l];
    const int m = 16 * j + c, n = n0 + 4 * g;
    if (m < a.M && n < a.N) put4((T*)a.Y + (int64_t)m * a.ldy + n, a.ywide, a.N - n, v);
  }
}

// Adds the splits' partial sums in their order. A split costs 8 bytes a result here,
// which a product of few tiles has to spare.
template <class T>
__global__ __launch_bounds__(256) void k_join(ProductArgs a) {
  const int64_t total = (int64_t)a.M * a.N;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    float v = a.part[e];
    for (int s = 1; s < a.splits; ++s) v += a.part[s * total + e];
    const int64_t m = e / a.N;
    ((T*)a.Y)[m * a.ldy + (e - m * a.N)] = (T)v;
  }
}

// Which kernel (edge of a work group's tile; 16: few rows) and how many parts of K
// (the same for the workspace's size and the launch).
struct Plan { int edge; int splits; };
Plan plan(int64_t M, int64_t N, int64_t K) {
  const int64_t nb = ceil_div(K, kBlock);
  // Few rows, against 64 x 64 tiles, at 4096 x 4096: 16 rows 6.4 and 10.2 us, 32 rows
  // 8.8 and 9.8; with more of the weights a second tile of rows, read from the caches
  // by every work group, costs more than the tiles' join (32 x 11008 x 4096 19.2 and
  // 17.7 us, 32 x 4096 x 11008 20.3 and 17.6; 16 rows 13.7 and 17.3). Four tiles of rows leave
  // registers for one block at a time, so K is to be short: 44 x 1536 x 2238 5.5 and 9.4
  // us, 64 x 2048 x 2048 7.7 and 8.2, 64 x 4096 x 4096 12.8 and 10.4, 33 x 1000 x 11008
  // 20.8 and 10.9.
  if (M <= 16 || (M <= 32 && N <= 8192 && nb <= 32) || (M <= 64 && N <= 4096 && nb <= 20)) return {16, 1};
  auto tiles = [&](int64_t e) { return ceil_div(M, e) * ceil_div(N, e); };
  // A 256 x 256 tile has a compute unit to itself, two of 128 x 128 share one; rounds of
  // them take 60 and 36 us at K = 4096. 8192 x 11008: 6 rounds, 356 us, against 11, 390
  // us; 4096 x 4096 64 and 74 us; 6000 x 6000: 3 rounds, 172 us, against 5, 164 us; 2048 x
  // 4096: 60 us (half the units idle) against 44.
  if (5 * ceil_div(tiles(256), 256) < 3 * ceil_div(tiles(128), 512)) return {256, 1};
  // Tiles of 128 that do not fill the device, along a short K or where they are few: 64 x
  // 64, which need not be split, or less. 700 x 1500 at K = 1500 8.6 us against 16.8, at
  // 4096 24 against 22, at 11008 66 against 32; 2048 x 2048 at K = 1500 15.6 against
  // 27, at 4096 30 against 35, at 6000 51 against 48; 333 x 1000 at K = 700 5.7
  // against 8.2.
  if ((tiles(128) <= 256 && nb <= 32) || (tiles(128) < 128 && tiles(64) <= 256)) {
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({512 / tiles(64), nb / 8, 16}));
    return {64, (int)splits};
  }
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({512 / tiles(128), nb / 4, 16}));
  return {128, (int)splits};
}

size_t part_bytes(const Plan& p, int64_t M, int64_t N) {
  return p.splits > 1 ? (size_t)p.splits * M * N * sizeof(float) : 0;
}

template <class T, int BN, int BM, int WN, int WM, bool ROWS, bool EXACT>
void launch_product(const ProductArgs& a, hipStream_t s) {
  const int tn = (a.N + BN - 1) / BN, tm = (a.M + BM - 1) / BM;
  hipLaunchKernelGGL((k_product<T, BN, BM, WN, WM, ROWS, EXACT>), dim3(tn * tm, a.splits), dim3(64 * WN * WM), 0, s, a,
                     tn, tm);
}

template <class T, bool ROWS>
void product_typed(ProductArgs a, const Plan& p, hipStream_t s) {
  constexpr bool EXACT = sizeof(T) == 4;
  if (p.edge == 16) {
    const dim3 grid((a.N + 15) / 16);
    if (a.M <= 16) hipLaunchKernelGGL((k_thin<T, 1, ROWS, EXACT, 0>), grid, dim3(512), 0, s, a);
    else if (a.M <= 32) hipLaunchKernelGGL((k_thin<T, 2, ROWS, EXACT, 0>), grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL((k_thin<T, 4, ROWS, EXACT, 0>), grid, dim3(512), 0, s, a);
    return;
  }
  if (p.edge == 64) {
    launch_product<T, 64, 64, 2, 2, ROWS, EXACT>(a, s);
  } else if constexpr (EXACT) {  // (widened operands of 256 x 256 do not fit the registers)
    launch_product<T, 128, 128, 2, 2, ROWS, EXACT>(a, s);
  } else {
    if (p.edge == 256)
      launch_product<T, 256, 256, 2, 4, ROWS, EXACT>(a, s);
    else
      launch_product<T, 128, 128, 2, 2, ROWS, EXACT>(a, s);
  }
  if (p.splits > 1) {
    const int64_t total = (int64_t)a.M * a.N;
    hipLaunchKernelGGL(k_join<T>, dim3((unsigned)std::min<int64_t>(2048, ceil_div(total, 256))), dim3(256), 0, s, a);
  }
}

void product(const ProductArgs& a, const Plan& p, bool rows, gptq2d_dtype dt, hipStream_t s) {
  with_type(dt, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (rows)
      product_typed<T, true>(a, p, s);
    else
      product_typed<T, false>(a, p, s);
  });
}

// ---------------------------------------------------------------------------
// Arguments
// ---------------------------------------------------------------------------

constexpr int64_t kMaxDim = (int64_t)1 << 22;
bool bad_dim(int64_t d) { return d < 1 || d > kMaxDim; }
// more entries than the device holds (and than a launch's grid can cover)
bool bad_area(int64_t r, int64_t c) { return r * c > (int64_t)1 << 37; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

bool bad_sizes(int64_t M, int64_t N, int64_t K) {
  return bad_dim(M) || bad_dim(N) || bad_dim(K) || bad_area(M, N) || bad_area(M, K) || bad_area(N, K);
}

gptq2d_status check_codes(const void* Q, int64_t ldq, int64_t cols, const void* S, int64_t lds, int64_t least) {
  if (!Q || !S) return refuse("codes or scales are NULL");
  if (!aligned(Q, 16) || ldq % 16 != 0) return refuse("codes need 16-byte aligned rows");
  if (ldq < cols || ldq > kMaxDim * 2) return refuse("leading dimension of the codes too small or too large");
  if (!aligned(S, 4) || lds < least) return refuse("leading dimension of the scales too small");
  return GPTQ2D_OK;
}

gptq2d_status check_matrix(const void* X, int64_t ldx, int64_t cols, gptq2d_dtype dt, const char* what) {
  if (!X) return refuse(what);
  if (ldx < cols) return refuse("leading dimension too small");
  if (!aligned(X, elem_size(dt))) return refuse("a matrix is not aligned to its elements");
  return GPTQ2D_OK;
}

gptq2d_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return GPTQ2D_OK;
  if (!ws || have < need) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(ws, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return GPTQ2D_OK;
}

// workspace regions of the layer's calls
struct Region {
  char* at;
  template <class P>
  P* take(size_t bytes) {
    P* p = (P*)at;
    at += up256(bytes);
    return p;
  }
};
// rows of an odd number of 128 bytes: those of a power of two would meet in one
// channel of the L2 whenever a work group reads the same block of all its rows
// (8192 x 11008 x 4096: 449 us with rows of 4096 bytes, 387 us with 4224)
int64_t code_ld(int64_t cols) { return (ceil_div(cols, kBlock) | 1) * kBlock; }
size_t code_bytes(int64_t rows, int64_t cols) { return up256((size_t)rows * code_ld(cols)); }
size_t scale_bytes(int64_t rows, int64_t cols) { return up256((size_t)rows * ceil_div(cols, kBlock) * sizeof(float)); }

ProductArgs product_args(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* SA, int64_t ldsa,
                         const void* B, int64_t ldb, const float* SB, int64_t ldsb, void* C, int64_t ldc,
                         gptq2d_dtype dt, const Plan& p, void* part) {
  ProductArgs a = {};
  a.M = (int)M, a.N = (int)N, a.K = (int)K;
  a.X = A, a.ldx = lda, a.SX = SA, a.ldsx = ldsa;
  a.W = (const uint8_t*)B, a.ldw = ldb, a.SW = SB, a.ldsw = ldsb;
  a.Y = C, a.ldy = ldc;
  const size_t es = elem_size(dt);
  a.ywide = aligned(C, 4 * es) && ldc % 4 == 0;
  a.part = (float*)part, a.splits = p.splits;
  return a;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

gptq2d_status gptq2d_block_quantize(int64_t rows, int64_t cols, gptq2d_dtype dt, const void* X, int64_t ldx,
                                    int block_rows, int pow2, void* Q, int64_t ldq, float* S, int64_t lds, void* QT,
                                    int64_t ldqt, float* ST, int64_t ldst, void* stream) {
  if (bad_dim(rows) || bad_dim(cols)) return refuse("rows and cols must lie in [1, 2^22]");
  if (bad_area(rows, cols)) return refuse("X has more than 2^37 entries");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (block_rows != 1 && block_rows != kBlock) return refuse("block_rows must be 1 or 128");
  if (!Q && !QT) return refuse("neither codes nor transposed codes are asked for");
  gptq2d_status st = check_matrix(X, ldx, cols, dt, "X is NULL");
  const bool tile = block_rows != 1;
  if (st == GPTQ2D_OK && Q) st = check_codes(Q, ldq, cols, S, lds, tile ? ceil_div(cols, kBlock) : rows);
  if (st == GPTQ2D_OK && QT) st = check_codes(QT, ldqt, rows, ST, ldst, tile ? ceil_div(rows, kBlock) : cols);
  if (st != GPTQ2D_OK) return st;
  QuantArgs a = {rows, cols, X, ldx, (uint8_t*)Q, ldq, S, lds, (uint8_t*)QT, ldqt, ST, ldst, pow2 != 0,
                 wide_rows(X, ldx, elem_size(dt))};
  quantize(a, dt, tile, (hipStream_t)stream);
  return launched("gptq2d_block_quantize");
}

size_t gptq2d_block_matmul_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (bad_sizes(M, N, K)) return 0;
  return part_bytes(plan(M, N, K), M, N);
}

gptq2d_status gptq2d_block_matmul(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* SA,
                                  int64_t ldsa, const void* B, int64_t ldb, const float* SB, int64_t ldsb,
                                  int b_block_rows, gptq2d_dtype dt, void* C, int64_t ldc, void* workspace,
                                  size_t ws_bytes, void* stream) {
  if (bad_sizes(M, N, K)) return refuse("M, N and K must lie in [1, 2^22], each matrix in 2^37 entries");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (b_block_rows != 1 && b_block_rows != kBlock) return refuse("block_rows must be 1 or 128");
  const bool rows = b_block_rows == 1;
  gptq2d_status st = check_codes(A, lda, K, SA, ldsa, M);
  if (st == GPTQ2D_OK) st = check_codes(B, ldb, K, SB, ldsb, rows ? N : ceil_div(K, kBlock));
  if (st == GPTQ2D_OK) st = check_matrix(C, ldc, N, dt, "C is NULL");
  const Plan p = plan(M, N, K);
  if (st == GPTQ2D_OK) st = check_workspace(workspace, ws_bytes, part_bytes(p, M, N));
  if (st != GPTQ2D_OK) return st;
  product(product_args(M, N, K, A, lda, SA, ldsa, B, ldb, SB, ldsb, C, ldc, dt, p, workspace), p, rows, dt,
          (hipStream_t)stream);
  return launched("gptq2d_block_matmul");
}

size_t gptq2d_block_linear_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (bad_sizes(M, N, K)) return 0;
  return code_bytes(M, K) + scale_bytes(M, K) + part_bytes(plan(M, N, K), M, N);
}

gptq2d_status gptq2d_block_linear(int64_t M, int64_t N, int64_t K, gptq2d_dtype dt, const void* X, int64_t ldx,
                                  const void* W, int64_t ldw, const float* SW, int64_t ldsw, int pow2, void* Y,
                                  int64_t ldy, void* workspace, size_t ws_bytes, void* stream) {
  if (bad_sizes(M, N, K)) return refuse("M, N and K must lie in [1, 2^22], each matrix in 2^37 entries");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  gptq2d_status st = check_matrix(X, ldx, K, dt, "X is NULL");
  if (st == GPTQ2D_OK) st = check_codes(W, ldw, K, SW, ldsw, ceil_div(K, kBlock));
  if (st == GPTQ2D_OK) st = check_matrix(Y, ldy, N, dt, "Y is NULL");
  if (st == GPTQ2D_OK) st = check_workspace(workspace, ws_bytes, gptq2d_block_linear_workspace_size(M, N, K));
  if (st != GPTQ2D_OK) return st;
  const Plan p = plan(M, N, K);
  if (M <= kFusedRows && K % 2 == 0 && ldx % 2 == 0 && aligned(X, 2 * elem_size(dt))) {
    ProductArgs a = product_args(M, N, K, X, ldx, nullptr, 0, W, ldw, SW, ldsw, Y, ldy, dt, p, nullptr);
    a.pow2 = pow2 != 0;
    with_type(dt, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      auto k = M == 1 ? k_thin<T, 1, false, sizeof(T) == 4, 1> : k_thin<T, 1, false, sizeof(T) == 4, kFusedRows>;
      hipLaunchKernelGGL(k, dim3((unsigned)ceil_div(N, 16)), dim3(512), 0, (hipStream_t)stream, a);
    });
    return launched("gptq2d_block_linear");
  }
  Region ws{(char*)workspace};
  uint8_t* q = ws.take<uint8_t>(code_bytes(M, K));
  float* sq = ws.take<float>(scale_bytes(M, K));
  QuantArgs a = {M, K, X, ldx, q, code_ld(K), sq, M, nullptr, 0, nullptr, 0, pow2 != 0, wide_rows(X, ldx, elem_size(dt))};
  quantize(a, dt, false, (hipStream_t)stream);
  product(product_args(M, N, K, q, code_ld(K), sq, M, W, ldw, SW, ldsw, Y, ldy, dt, p, ws.at), p, false, dt,
          (hipStream_t)stream);
  return launched("gptq2d_block_linear");
}

size_t gptq2d_block_linear_backward_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (bad_sizes(M, N, K)) return 0;
  return code_bytes(M, N) + scale_bytes(M, N) + code_bytes(N, M) + scale_bytes(N, M) + code_bytes(K, M) +
         scale_bytes(K, M) + std::max(part_bytes(plan(M, K, N), M, K), part_bytes(plan(N, K, M), N, K));
}

gptq2d_status gptq2d_block_linear_backward(int64_t M, int64_t N, int64_t K, gptq2d_dtype dt, const void* dY,
                                           int64_t lddy, const void* X, int64_t ldx, const void* WT, int64_t ldwt,
                                           const float* SWT, int64_t ldswt, int pow2, void* dX, int64_t lddx, float* dW,
                                           int64_t lddw, void* workspace, size_t ws_bytes, void* stream) {
  if (bad_sizes(M, N, K)) return refuse("M, N and K must lie in [1, 2^22], each matrix in 2^37 entries");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (!dX && !dW) return refuse("neither dX nor dW is asked for");
  gptq2d_status st = check_matrix(dY, lddy, N, dt, "dY is NULL");
  if (st == GPTQ2D_OK && dX) st = check_codes(WT, ldwt, N, SWT, ldswt, ceil_div(N, kBlock));
  if (st == GPTQ2D_OK && dX) st = check_matrix(dX, lddx, K, dt, "dX is NULL");
  if (st == GPTQ2D_OK && dW) st = check_matrix(X, ldx, K, dt, "X is NULL");
  if (st == GPTQ2D_OK && dW) st = check_matrix(dW, lddw, K, GPTQ2D_F32, "dW is NULL");
  if (st == GPTQ2D_OK) st = check_workspace(workspace, ws_bytes, gptq2d_block_linear_backward_workspace_size(M, N, K));
  if (st != GPTQ2D_OK) return st;
  Region ws{(char*)workspace};
  uint8_t* qy = ws.take<uint8_t>(code_bytes(M, N));
  float* sy = ws.take<float>(scale_bytes(M, N));
  uint8_t* qyt = ws.take<uint8_t>(code_bytes(N, M));
  float* syt = ws.take<float>(scale_bytes(N, M));
  uint8_t* qxt = ws.take<uint8_t>(code_bytes(K, M));
  float* sxt = ws.take<float>(scale_bytes(K, M));
  const hipStream_t s = (hipStream_t)stream;
  const size_t es = elem_size(dt);
  // dY is read once for both products that it enters
  QuantArgs a = {M, N, dY, lddy, dX ? qy : nullptr, code_ld(N), sy, M, dW ? qyt : nullptr, code_ld(M), syt, N,
                 pow2 != 0, wide_rows(dY, lddy, es)};
  quantize(a, dt, false, s);
  if (dX) {
    const Plan p = plan(M, K, N);
    product(product_args(M, K, N, qy, code_ld(N), sy, M, WT, ldwt, SWT, ldswt, dX, lddx, dt, p, ws.at), p, false, dt, s);
  }
  if (dW) {
    QuantArgs x = {M, K, X, ldx, nullptr, 0, nullptr, 0, qxt, code_ld(M), sxt, K, pow2 != 0, wide_rows(X, ldx, es)};
    quantize(x, dt, false, s);
    const Plan p = plan(N, K, M);
    product(product_args(N, K, M, qyt, code_ld(M), syt, N, qxt, code_ld(M), sxt, K, dW, lddw, GPTQ2D_F32, p, ws.at), p,
            true, GPTQ2D_F32, s);
  }
  return launched("gptq2d_block_linear_backward");
}

}  // extern "C"
