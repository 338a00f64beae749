// Attention of a tree of drafted tokens (one token: decoding) over a paged
// eight-bit cache.
//
// Sequence b has context[b] tokens in the cache and then its drafted ones. A
// drafted token t sees the whole context and the drafted tokens u whose bit is
// set in mask[b][t]. With keys k = ks ck and values v = vs cv (codes and scales),
//   z = scale ks (q . ck),  o = sum_x softmax(z)_x vs_x cv_x,  lse = log sum e^z.
#include <math.h>

#include <algorithm>

#include "codes.hpp"

namespace g2d {
namespace {

constexpr int kStep = 32;        // tokens a wave takes at a time
constexpr int kWaves = 4;
constexpr int kMaxSplits = 64;
constexpr int kBalanced = 256;   // sequences whose lengths a work group looks at
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2E = 1.44269504088896341f;

// work groups of k_tree that a compute unit's registers and LDS are to hold at once
constexpr int groups_a_unit(int dp, int tiles) { return dp < 256 && dp * tiles <= 256 ? 2 : 1; }

// The instance whose registers, kept to 128, let a compute unit hold four: one token of 40
// sequences over 300 (dim 64, f16) 10.8 us, with three 12.4.
constexpr bool four_a_unit(bool int8, int dp, int tiles, int zq, int zp) {
  return !int8 && dp == 64 && tiles == 1 && zq < zp;
}

struct TreeArgs {
  int seqs, width, kv, group, dim, rows;  // rows = width * group: queries of a sequence that share a kv head
  gptq2d_dtype dt;
  const void* Q;
  int64_t ldq;
  const uint8_t *KC, *VC;
  const float *KS, *VS;
  int64_t pages;
  int page, page16;
  uint64_t magic;  // floor(2^32 / page16) + 1
  const int32_t* table;
  int64_t ldt;
  int capacity;  // tokens that a row of the table covers
  const int32_t *context, *drafts;
  const uint64_t* mask;
  float scale;  // times log2 e
  void* O;
  int64_t ldo;
  bool qwide, owide;  // rows of Q and O start on 16-byte boundaries
  float* lse;
  int splits, rowblocks;  // parts that a sequence may have
  int mean;               // parts that one of mean length is to have
  float* part;  // splits > 1: [sequence][kv head][row][split][dim padded], then {m, l} likewise
};

// eight elements of type dt from element i on; wide: they are 16-byte aligned
__device__ __forceinline__ void load8_as(const void* p, gptq2d_dtype dt, int64_t i, bool wide, float x[8]) {
  if (dt == GPTQ2D_F32) load8((const float*)p + i, wide, 8, x, (const float*)p);
  else if (dt == GPTQ2D_F16) load8((const _Float16*)p + i, wide, 8, x, (const _Float16*)p);
  else load8((const bf16*)p + i, wide, 8, x, (const bf16*)p);
}
// N (4 or a multiple of 8) results; wide: aligned to their size, at most 16 bytes
template <int N, class T>
__device__ __forceinline__ void store_n(T* p, bool wide, const float* v) {
  if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8) store8(p + i, wide, 8, v + i);
  } else if (wide) {
    if constexpr (sizeof(T) == 4) {
      *(f4*)p = f4{v[0], v[1], v[2], v[3]};
    } else {
      typedef T V __attribute__((ext_vector_type(4)));
      *(u2*)p = __builtin_bit_cast(u2, V{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (T)v[i];
  }
}
template <int N>
__device__ __forceinline__ void store_as(void* p, gptq2d_dtype dt, int64_t i, bool wide, const float* v) {
  if (dt == GPTQ2D_F32) store_n<N>((float*)p + i, wide, v);
  else if (dt == GPTQ2D_F16) store_n<N>((_Float16*)p + i, wide, v);
  else store_n<N>((bf16*)p + i, wide, v);
}

// over the four lanes that share l % 16, in every lane: the instructions swap
// halves (rows of 16) of two registers
__device__ __forceinline__ float quad_max(float v) {
  const u2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  const u2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const u2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A value scale's level, in bits 8 to 15: log2, rounded up, plus 127. A reference takes it
// less kLevel: products of e^z and value scales reach 2^5 then, and 2^15 before a
// reference moves, which halves hold, and are normal halves down to 2^-19 of the largest.
// Scales below 2^-75 count as that, or the sum of the exponentials could overflow.
constexpr float kLevel = 132.0f;
__device__ __forceinline__ uint32_t value_level(float v) {
  return max((__float_as_uint(v) + 0x7fffffu) >> 23, 52u) << 8;
}

// One wave's 32 tokens as they lie in the cache. A lane (c = l % 16, g = l / 16)
// holds of the keys a quarter (g) of token c of each 16-token row, and of the
// values sixteenth c of tokens 4 g .. 4 g + 3 of each row: both are what the
// matrix instruction takes as its row operand once widened, with no exchange
// between lanes (the order in which it sums is free, as long as both operands
// agree).
template <int DP>
struct Tokens {
  u4 k[2][DP / 64];
  uint32_t v[2][4][DP / 64];
  f4 ks[2], vs[2];
};

// the top bits of the bytes that are e4m3's NaNs
__device__ __forceinline__ uint32_t nan_codes(uint32_t v) { return ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// The table's entries of a wave's next 32 tokens (uniform, looked up ahead of
// the tokens themselves); an entry that names no page, or tokens from `end` on: -1
struct Entry {
  int32_t page[2], off[2];
};
__device__ __forceinline__ Entry look_up(const TreeArgs& a, const int32_t* table, int tok, int end) {
  Entry r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const bool in = tok + 16 * h < end;
    const uint32_t t16 = in ? (uint32_t)(tok >> 4) + h : 0;
    const uint32_t pg = (uint32_t)((t16 * a.magic) >> 32);  // exact: t16 page16 < 2^32
    r.off[h] = (t16 - pg * a.page16) * 16;
    const int32_t e = table[pg];
    r.page[h] = in && e >= 0 && e < a.pages ? e : -1;
  }
  return r;
}

// Tokens that are not there are read from page 0 and masked later. Past the end
// of a vector any of it is read: there the query is 0 (keys) or the results are
// not stored (values).
__device__ __forceinline__ int64_t place(const TreeArgs& a, Entry e, int h, int hkv) {
  return ((int64_t)max(e.page[h], 0) * a.kv + hkv) * a.page + e.off[h];
}
template <int DP>
__device__ __forceinline__ void fetch_keys(Tokens<DP>& x, const TreeArgs& a, Entry e, int hkv, int c, int g) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint8_t* p = a.KC + place(a, e, h, hkv) * a.dim;
#pragma unroll
    for (int i = 0; i < DP / 64; ++i) {
      const int d = g * (DP / 4) + 16 * i;
      x.k[h][i] = *(const u4*)(p + (uint32_t)(c * a.dim + (d < a.dim ? d : 0)));
    }
  }
}
template <int DP>
__device__ __forceinline__ void fetch_values(Tokens<DP>& x, const TreeArgs& a, Entry e, int hkv, int c, int g) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint8_t* pv = a.VC + place(a, e, h, hkv) * a.dim;
    const int d = c * (DP / 16) < a.dim ? c * (DP / 16) : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* p = pv + (uint32_t)((4 * g + i) * a.dim + d);
      if constexpr (DP == 64) {
        x.v[h][i][0] = *(const uint32_t*)p;
      } else if constexpr (DP == 128) {
        const u2 w = *(const u2*)p;
        x.v[h][i][0] = w[0], x.v[h][i][1] = w[1];
      } else {
        const u4 w = *(const u4*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[h][i][j] = w[j];
      }
    }
  }
}
template <int DP>
__device__ __forceinline__ void fetch_scales(Tokens<DP>& x, const TreeArgs& a, Entry e, int hkv, int g) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t at = place(a, e, h, hkv) + 4 * g;
    x.ks[h] = *(const f4*)(a.KS + at);
    x.vs[h] = *(const f4*)(a.VS + at);
  }
}

// NaN in the results v of N elements from d0 on, for the NaN codes of those drafted tokens
// first .. end - 1 that query tq sees
template <int N>
__device__ __forceinline__ void put_nans(const TreeArgs& a, const int32_t* table, int b, int hkv, int tq, int ctx, int first,
                                         int end, int d0, float (&v)[N]) {
  if (d0 >= a.dim) return;
  const uint64_t sees = a.mask ? a.mask[(int64_t)b * a.width + tq] : ((uint64_t)2 << tq) - 1;
  for (int x = first; x < end; ++x) {
    const int pg = x / a.page;
    const int32_t e = table[pg];
    if (!((sees >> (x - ctx)) & 1) || e < 0 || e >= a.pages) continue;
    const uint8_t* p = a.VC + (((int64_t)e * a.kv + hkv) * a.page + (x - pg * a.page)) * a.dim + d0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if ((p[j] & 0x7f) == 0x7f) v[j] = __uint_as_float(0x7fc00000u);
  }
}

// Tokens of a part: the same for all sequences, so that the work groups of long and
// short ones take alike, as far as the longest one's parts suffice; whole steps.
// (32 trees of 8, lengths between 8192 and 32768: 278 us, in equal numbers of parts
// 311 us; 16 trees of 13, lengths between 2048 and 8192: 57 and 54 us.)
__device__ __forceinline__ int part_length(const TreeArgs& a, int total, int l) {
  int per = (total + a.splits - 1) / a.splits;
  if (a.splits > 1 && a.seqs <= kBalanced) {
    int n[kBalanced / 64];
#pragma unroll
    for (int i = 0; i < kBalanced / 64; ++i) n[i] = a.context[min(l + 64 * i, a.seqs - 1)];
    float sum = 0;  // (a mean, so 32 bits will do)
#pragma unroll
    for (int i = 0; i < kBalanced / 64; ++i)
      sum += l + 64 * i < a.seqs ? (float)(min(max(n[i], 0), a.capacity) + a.width) : 0.0f;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    per = max(per, (int)(sum / (a.seqs * (a.mean - 0.5f))));  // half a part is lost to whole ones
  }
  constexpr int whole = kWaves * kStep;
  return __builtin_amdgcn_readfirstlane((per + whole - 1) / whole * whole);
}

// 16 QT queries of one kv head and sequence over one part of its tokens. Scores
// and outputs are transposed (tokens and dimensions are the instruction's rows,
// queries its columns), so a lane's values all belong to one query: maximum,
// sum and rescaling are its own, and the scores leave the first product in the
// registers where the second one takes them.
// Codes are widened to halves, exactly. A query is scaled by a power of two so
// that its largest element is in [1, 2) and rounded to halves (which a 16-bit
// query survives, but for elements below 2^-14 of the largest); probabilities
// are taken times vs, relative to the query's largest such product so far (a bound
// of it: the largest score times the largest vs of a step), and so is their sum. Queries are kept as ZQ halves (two of them, 22 bits, for 32-bit
// queries), probabilities as ZP (one, rounded by 2^-11 at most, where the result
// is rounded by 2^-8 after it).
//
// Each wave streams its own tokens from memory to registers; LDS only joins the four
// waves at the end. One kv head's tokens are read once for all queries that share it,
// which is what bounds long contexts: 32 trees of 8 (4 queries a head) over up to
// 32768 tokens (dim 128) 281 us, 5.0 TB/s of cache. With 52 queries a head, 16 trees
// of 13 over up to 8192 (dim 64, f16) 55 us, the cache's bytes are 19 us of it and
// the instructions of the softmax and of widening the codes bound it (some 20 us of
// issue slots, 7 us of the matrix unit; the rest is not accounted for); one token over
// 4096 8.3 us, where the chain of one step does (length, table, codes, scores, values).
template <bool INT8, int DP, int QT, int ZQ, int ZP>
__global__ __launch_bounds__(64 * kWaves, four_a_unit(INT8, DP, QT, ZQ, ZP) ? 4 : groups_a_unit(DP, QT)) void k_tree(TreeArgs a) {
  constexpr int KS = DP / 32, NT = DP / 16;
  __shared__ float lm[kWaves][16 * QT], ll[kWaves][16 * QT];
  __shared__ float lo[kWaves][16 * QT][DP + 4];
  __shared__ int odd[kWaves];
  // parts are the slowest index: work groups go round the XCDs by their number, and
  // the last parts, which few sequences have, are not to meet on a few of them
  const int hkv = blockIdx.x / a.rowblocks, rb = blockIdx.x % a.rowblocks, b = blockIdx.y, split = blockIdx.z;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, c = l & 15, g = l >> 4;
  const int ctx = min(max(a.context[b], 0), a.capacity);
  const int drafted = a.drafts ? min(max(a.drafts[b], 0), a.width) : a.width;
  const int total = min(ctx + drafted, a.capacity);
  const int per = part_length(a, total, l);
  const int begin = split * per, end = min(total, begin + per);
  if (begin >= end && a.splits > 1) {  // no such part
    float* ml = a.part + (int64_t)a.seqs * a.kv * a.rows * a.splits * DP;
    for (int r = rb * 16 * QT + threadIdx.x; r < min((rb + 1) * 16 * QT, a.rows); r += 64 * kWaves) {
      const int64_t at = (((int64_t)b * a.kv + hkv) * a.rows + r) * a.splits + split;
      ml[2 * at] = -INFINITY, ml[2 * at + 1] = 0.0f;
    }
    return;
  }
  const int32_t* table = a.table + b * a.ldt;

  constexpr int kStride = kWaves * kStep;
  Tokens<DP> x;
  int tok = begin + w * kStep;
  Entry now = look_up(a, table, tok, end), next = look_up(a, table, tok + kStride, end);
  if (tok < end) {
    fetch_keys(x, a, now, hkv, c, g);
    fetch_scales(x, a, now, hkv, g);
    fetch_values(x, a, now, hkv, c, g);
  }

  h8 q[QT][KS][ZQ];
  float qs[QT], m[QT], sum[QT];
  f4 o[QT][NT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = (rb * QT + t) * 16 + c, tq = r / a.group, head = hkv * a.group + r % a.group;
    const bool live = r < a.rows;
    const int64_t at = ((int64_t)b * a.width + tq) * a.ldq + (int64_t)head * a.dim;
    float f[DP / 4];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = g * (DP / 4) + 8 * s;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[8 * s + i] = 0.0f;
      if (live && d < a.dim) load8_as(a.Q, a.dt, at + d, a.qwide, f + 8 * s);
    }
#pragma unroll
    for (int i = 0; i < DP / 4; ++i) top = max(top, mag(f[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    uint32_t e = min(top & 0x7f800000u, 253u << 23);
    if (e == 0 || bad_amax(top)) e = 127u << 23;
    // (a scale of zero is taken as queries of zero, so that qs stays positive)
    const float down = a.scale == 0.0f ? 0.0f : copysignf(__uint_as_float((254u << 23) - e), a.scale);
    qs[t] = fmaxf(fabsf(a.scale) * __uint_as_float(e), 0x1p-126f);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = f[8 * s + i] * down;
        q[t][s][0][i] = (_Float16)v;
        if constexpr (ZQ == 2) q[t][s][1][i] = (_Float16)(v - (float)q[t][s][0][i]);
      }
    m[t] = -INFINITY, sum[t] = 0;
#pragma unroll
    for (int j = 0; j < NT; ++j) o[t][j] = f4{0, 0, 0, 0};
  }
  bool found = false;  // a NaN code among the wave's drafted tokens (uniform)
  float minus = -1.0f;  // (unknown to the compiler, which would make a multiply-add with it a subtraction)
  asm("" : "+s"(minus));

  // Tokens are kept once: as soon as the keys of a step are widened, those of the
  // next one are on their way into their registers, and likewise the values. (The
  // last step fetches once more, from page 0: a branch around the loads would make
  // the compiler wait for all of them at its end.)
  for (; tok < end; tok += kStride) {
    const Entry after = look_up(a, table, tok + 2 * kStride, end);
    if constexpr (!INT8) {
      if (tok + kStep > ctx) {
        // A NaN among a drafted token's codes would reach the queries that do not see it, as
        // 0 times NaN: it is left out, and those that see it get their NaN at the end.
        auto nan = [&](int i, int e) {
          return tok + 16 * (i >> 2) + 4 * g + (i & 3) >= ctx ? nan_codes(x.v[i >> 2][i & 3][e]) : 0u;
        };
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < DP / 64; ++e) any |= nan(i, e);
        if (__any(any != 0)) {
          found = true;
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < DP / 64; ++e) {
              const uint32_t n = nan(i, e);
              x.v[i >> 2][i & 3][e] &= ~((n << 1) - (n >> 7));
            }
        }
      }
    }
    // scores
    h8 kf[2][KS];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const uint32_t w0 = x.k[h][s / 2][2 * (s & 1)], w1 = x.k[h][s / 2][2 * (s & 1) + 1];
        const h2 p0 = halves<INT8, false>(w0), p1 = halves<INT8, true>(w0);
        const h2 p2 = halves<INT8, false>(w1), p3 = halves<INT8, true>(w1);
        kf[h][s] = h8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
      }
    fetch_keys(x, a, next, hkv, c, g);
    f4 z[QT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        z[t][h] = f4{0, 0, 0, 0};
#pragma unroll
        for (int e = ZQ - 1; e >= 0; --e)
#pragma unroll
          for (int s = 0; s < KS; ++s)
            z[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[h][s], q[t][s][e], z[t][h], 0, 0, 0);
      }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) z[t][h] *= x.ks[h];
    f4 vs[2] = {x.vs[0], x.vs[1]};
    fetch_scales(x, a, next, hkv, g);
    // bit 4 h + i: token tok + 16 h + 4 g + i is seen by query t; bits 8 to 15: the level
    // of the value scales that it sees
    uint32_t ok[QT];
    const bool edge = tok + kStep > min(ctx, end) || now.page[0] < 0 || now.page[1] < 0;
    if (edge) {
      uint64_t sees[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const int tq = min((rb * QT + t) * 16 + c, a.rows - 1) / a.group;
        sees[t] = a.mask ? a.mask[(int64_t)b * a.width + tq] : ((uint64_t)2 << tq) - 1;
        ok[t] = 0;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int first = tok + 16 * h + 4 * g, past = first - ctx;
        const uint32_t in = now.page[h] < 0 ? 0 : (1u << min(max(end - first, 0), 4)) - 1;
        const uint32_t before = (1u << min(max(-past, 0), 4)) - 1;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const uint64_t tree = past >= 0 ? (past < 64 ? sees[t] >> past : 0) : past > -4 ? sees[t] << -past : 0;
          ok[t] |= (in & (before | (uint32_t)tree)) << (4 * h);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // whatever lies there, it must not meet a zero probability
          const uint32_t keep = -((in >> i) & 1);
          vs[h][i] = __uint_as_float(__float_as_uint(vs[h][i]) & keep);
#pragma unroll
          for (int e = 0; e < DP / 64; ++e) x.v[h][i][e] &= keep;
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((ok[t] >> (4 * h + i)) & 1)) z[t][h][i] = -INFINITY;
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, (ok[t] >> i) & 1 ? vs[i >> 2][i & 3] : 0.0f);
        ok[t] |= value_level(most);
      }
    }
    // A query's reference m moves when the largest score it sees, times the largest
    // value scale it sees, exceeds it by more than 2^10, which is seldom after the
    // first tokens. A value that it does not see, however large, does not move it. (One
    // reference of the value scales for all queries took 52 us where this takes 55, and gave
    // zeros to the queries beside one that saw a value 2^30 times theirs.)
    if (!edge) {
      float most = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, vs[i >> 2][i & 3]);
#pragma unroll
      for (int t = 0; t < QT; ++t) ok[t] = value_level(most);
    }
    auto most = [&](int t) {
      float v = z[t][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) v = fmaxf(v, z[t][i >> 2][i & 3]);
      return v;
    };
    auto level = [&](int t) { return (float)((ok[t] >> 8) & 0xff); };
    bool moves = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) moves |= fmaf(most(t), qs[t], level(t)) - m[t] > kLevel + 10.0f;
    if (__any(moves)) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float top = fmaxf(quad_max(most(t)) * qs[t] + (quad_max(level(t)) - kLevel), m[t]);
        const float d = __builtin_amdgcn_exp2f(m[t] - (top == -INFINITY ? 0.0f : top));
        sum[t] *= d;
        m[t] = top;
#pragma unroll
        for (int j = 0; j < NT; ++j) o[t][j] *= d;
      }
    }
    // probabilities
    h8 p[QT][ZP];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const float base = m[t] == -INFINITY ? 0.0f : m[t];
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (one rounding, of the difference; any reference would do)
        const float e = __builtin_amdgcn_exp2f(fmaf(z[t][i >> 2][i & 3], qs[t], -base));
        sum[t] += e;
        y[i] = e * vs[i >> 2][i & 3];
      }
      if (edge) {  // a probability of 0 may have met a scale that is not finite
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (ok[t] >> i) & 1 ? y[i] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const h2 hi = __builtin_convertvector(fp2{y[i], y[i + 1]}, h2);
        p[t][0][i] = hi[0], p[t][0][i + 1] = hi[1];
        if constexpr (ZP == 2) {
          // y - hi as one instruction that reads halves and writes them
          p[t][1][i] = (_Float16)fmaf((float)hi[0], minus, y[i]), p[t][1][i + 1] = (_Float16)fmaf((float)hi[1], minus, y[i + 1]);
        }
      }
    }
    // values
#pragma unroll
    for (int e = 0; e < DP / 64; ++e) {
      h8 vf[4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const uint32_t lo2 = __builtin_amdgcn_perm(x.v[h][i + 1][e], x.v[h][i][e], 0x05010400u);
          const uint32_t hi2 = __builtin_amdgcn_perm(x.v[h][i + 1][e], x.v[h][i][e], 0x07030602u);
          const h2 d0 = halves<INT8, false>(lo2), d1 = halves<INT8, true>(lo2);
          const h2 d2 = halves<INT8, false>(hi2), d3 = halves<INT8, true>(hi2);
          vf[0][4 * h + i] = d0[0], vf[0][4 * h + i + 1] = d0[1];
          vf[1][4 * h + i] = d1[0], vf[1][4 * h + i + 1] = d1[1];
          vf[2][4 * h + i] = d2[0], vf[2][4 * h + i + 1] = d2[1];
          vf[3][4 * h + i] = d3[0], vf[3][4 * h + i + 1] = d3[1];
        }
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int s = ZP - 1; s >= 0; --s)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o[t][4 * e + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], p[t][s], o[t][4 * e + j], 0, 0, 0);
    }
    fetch_values(x, a, next, hkv, c, g);
    now = next, next = after;
  }

  // the waves' parts, in their order
  if constexpr (!INT8) {
    if (l == 0) odd[w] = found;
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    sum[t] = quad_sum(sum[t]);
    if (g == 0) lm[w][16 * t + c] = m[t], ll[w][16 * t + c] = sum[t];
  }
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NT; j += 4)
        *(f4*)&lo[w][16 * t + c][(4 * g + i) * NT + j] =
            f4{o[t][j][i], o[t][j + 1][i], o[t][j + 2][i], o[t][j + 3][i]};
  __syncthreads();
  int group = a.group;
  // (its reciprocal is not to be held from the queries to here)
  if constexpr (four_a_unit(INT8, DP, QT, ZQ, ZP)) asm("" : "+s"(group));
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qr = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * NT;
    const int r = (rb * QT + t) * 16 + qr;
    if (r < a.rows) {
      float top = lm[0][16 * t + qr], L = 0, f[kWaves], v[NT];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) top = fmaxf(top, lm[i][16 * t + qr]);
#pragma unroll
      for (int j = 0; j < NT; ++j) v[j] = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        f[i] = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(lm[i][16 * t + qr] - top);
        L += ll[i][16 * t + qr] * f[i];
#pragma unroll
        for (int j = 0; j < NT; j += 4) {
          const f4 s = *(const f4*)&lo[i][16 * t + qr][d0 + j];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[j + k] = fmaf(s[k], f[i], v[j + k]);
        }
      }
      if constexpr (!INT8) {
        if (odd[0] | odd[1] | odd[2] | odd[3]) put_nans<NT>(a, table, b, hkv, r / group, ctx, max(begin, ctx), end, d0, v);
      }
      if (a.splits == 1) {
        const int tk = r / group, head = hkv * group + r % group;
        const int64_t row = (int64_t)b * a.width + tk;
        const bool none = L == 0.0f || tk >= drafted;
        const float inv = 1.0f / L;
#pragma unroll
        for (int j = 0; j < NT; ++j) v[j] = none ? 0.0f : v[j] * inv;
        if (d0 < a.dim) store_as<NT>(a.O, a.dt, row * a.ldo + (int64_t)head * a.dim + d0, a.owide, v);
        if (a.lse && d0 == 0)
          a.lse[row * (a.kv * a.group) + head] = none ? -INFINITY : (top + log2f(L)) * kLn2;
      } else {
        const int64_t at = (((int64_t)b * a.kv + hkv) * a.rows + r) * a.splits + split;
        float* ml = a.part + (int64_t)a.seqs * a.kv * a.rows * a.splits * DP;
        if (L != 0.0f) {
#pragma unroll
          for (int j = 0; j < NT; j += 4) *(f4*)(a.part + at * DP + d0 + j) = f4{v[j], v[j + 1], v[j + 2], v[j + 3]};
        }
        if (d0 == 0) ml[2 * at] = top, ml[2 * at + 1] = L;
      }
    }
  }
}

// G waves per query: each adds up every G-th split's part, eight loads at a time,
// then the waves' sums are added, all in a fixed order. Bound by latency: 32 queries
// of 33 parts 4.5 us (G = 4), 8192 of up to 4 parts 7.8 us (G = 1).
template <int DP, int G>
__global__ __launch_bounds__(64 * kWaves) void k_tree_join(TreeArgs a) {
  constexpr int E = DP / 64;  // elements of a lane
  __shared__ float lo[G][DP];
  const int wave = threadIdx.x >> 6, w = wave % G, l = threadIdx.x & 63;
  const uint32_t all = (uint32_t)a.seqs * a.kv * a.rows, id = blockIdx.x * (kWaves / G) + wave / G;
  if (id >= all) return;  // (G = 1, or a whole work group)
  const uint32_t bh = id / (uint32_t)a.rows, b = bh / (uint32_t)a.kv;
  const int r = id - bh * a.rows, hkv = bh - b * a.kv;
  const float* ml = a.part + (int64_t)all * a.splits * DP + 2 * (int64_t)id * a.splits;
  const float ms = l < a.splits ? ml[2 * l] : -INFINITY, ls = l < a.splits ? ml[2 * l + 1] : 0.0f;
  const float* part = a.part + (int64_t)id * a.splits * DP + E * l;
  float v[E], x[8][E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0;
  float top = ms;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  // (-1: an empty part, which is not written; one far below the best is, and may hold a NaN)
  const float f = ls == 0.0f ? -1.0f : top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ms - top);
  float L = ls * f;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) L += __shfl_xor(L, d);
  for (int s0 = w; s0 < a.splits; s0 += 8 * G) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) x[u][e] = part[(int64_t)min(s0 + u * G, a.splits - 1) * DP + e];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int s = s0 + u * G;
      const float fs = s < a.splits ? __shfl(f, s) : -1.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += fs < 0.0f ? 0.0f : x[u][e] * fs;
    }
  }
  if constexpr (G > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) lo[w][E * l + e] = v[e];
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 1; i < G; ++i) v[e] += lo[i][E * l + e];
  }
  const int tk = r / a.group, head = hkv * a.group + r % a.group;
  const int64_t row = (int64_t)b * a.width + tk;
  const int drafted = a.drafts ? min(max(a.drafts[b], 0), a.width) : a.width;
  const bool none = L == 0.0f || tk >= drafted;
  const int64_t at = row * a.ldo + (int64_t)head * a.dim + E * l;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (E * l + e >= a.dim) break;
    const float y = none ? 0.0f : v[e] / L;
    if (a.dt == GPTQ2D_F32) ((float*)a.O)[at + e] = y;
    else if (a.dt == GPTQ2D_F16) ((_Float16*)a.O)[at + e] = (_Float16)y;
    else ((bf16*)a.O)[at + e] = (bf16)y;
  }
  if (a.lse && l == 0) a.lse[row * (a.kv * a.group) + head] = none ? -INFINITY : (top + log2f(L)) * kLn2;
}

// bits of a token's ancestors and itself; a parent that is not an earlier token is none
__global__ __launch_bounds__(256) void k_tree_masks(int64_t count, int width, const int32_t* parents, uint64_t* masks) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= count * width) return;
  const int64_t b = i / width;
  int t = (int)(i - b * width);
  uint64_t m = (uint64_t)1 << t;
  for (;;) {
    const int p = parents[b * width + t];
    if (p < 0 || p >= t) break;
    m |= (uint64_t)1 << p;
    t = p;
  }
  masks[i] = m;
}

int padded(int dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Queries a work group takes, in tiles of 16: more of them share each read of
// the cache, as far as they and their accumulators fit the registers (a kernel
// that spills is not built: two tiles of 32-bit queries of 256 gave wrong results).
int query_tiles(int rows, int dim, bool f32) {
  const int most = f32 ? (padded(dim) == 256 ? 1 : 2) : padded(dim) == 256 ? 2 : 4;
  return std::min(most, rows <= 16 ? 1 : rows <= 32 ? 2 : 4);
}

// Parts that a sequence's tokens are split into: as many as run at once. Where a work
// group has a compute unit to itself, one more than fit would take a second round: 12
// trees of 5 (dim 256, 96 work groups a part, 256 at once) 61 us in 2 parts, 81 in 3, 85
// in 6; 20 of 40 over 308 tokens (240) 17 us whole, 35 in 2. Where two share one, a few
// more than fit do no harm: 40 tokens over 8000 (320 work groups a part, 512 at once) 116
// us whole, 98 in 2 parts, 95 in 3; 32 of 2 x 16 queries a head over 853 (416) 26 us
// whole, 38 in 2; 16 of 13 over 8192 (128) 60 / 59 / 59 / 70 us in 2 / 3 / 4 / 6; 32 of 8
// over 32768 (256) 302 / 287 / 306 us in 1 / 2 / 4. (10 trees of 32 x 8 queries a head, 80
// and 256 at once: 170 us in 3 parts, 155 in 7, 181 in 8.)
int split_count(int64_t seqs, int rows, int kv, int dim) {
  const int tiles = query_tiles(rows, dim, false), a_unit = groups_a_unit(padded(dim), tiles);
  const int64_t groups = seqs * kv * ceil_div(rows, 16 * tiles);
  const int64_t fit = a_unit == 1 ? 256 / groups : (512 + 2 * groups / 5) / groups;
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, fit));
}

// parts that the longest sequence may have: up to twice the mean's
int slot_count(int64_t seqs, int rows, int kv, int dim) {
  const int s = split_count(seqs, rows, kv, dim);
  return s == 1 || seqs == 1 ? s : std::min(2 * s, kMaxSplits);
}

size_t part_bytes(int64_t seqs, int rows, int kv, int dim) {
  const int s = slot_count(seqs, rows, kv, dim);
  return s == 1 ? 0 : (size_t)seqs * kv * rows * s * (padded(dim) + 2) * sizeof(float);
}

template <bool INT8, int DP, int QT, int ZQ, int ZP>
void launch(const TreeArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_tree<INT8, DP, QT, ZQ, ZP>), dim3(a.kv * a.rowblocks, a.seqs, a.splits), dim3(64 * kWaves), 0, s, a);
}
template <bool INT8, int DP, int ZQ, int ZP>
void launch_tiles(const TreeArgs& a, int tiles, hipStream_t s) {
  if (tiles == 1) {
    launch<INT8, DP, 1, ZQ, ZP>(a, s);
  } else if (tiles == 2) {
    if constexpr (DP != 256 || ZQ == 1) launch<INT8, DP, 2, ZQ, ZP>(a, s);
  } else {
    if constexpr (DP != 256 && ZQ == 1 && (DP != 64 || ZP == 2)) launch<INT8, DP, 4, ZQ, ZP>(a, s);
  }
  const int64_t all = (int64_t)a.seqs * a.kv * a.rows;
  if (a.splits > 8)
    hipLaunchKernelGGL((k_tree_join<DP, kWaves>), dim3((unsigned)all), dim3(64 * kWaves), 0, s, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL((k_tree_join<DP, 1>), dim3((unsigned)ceil_div(all, kWaves)), dim3(64 * kWaves), 0, s, a);
}
template <bool INT8, int DP>
void launch_type(const TreeArgs& a, int tiles, hipStream_t s) {
  if (a.dt == GPTQ2D_F32) launch_tiles<INT8, DP, 2, 2>(a, tiles, s);
  // (the kernel for four tiles of 64 and one half spills)
  else if (a.dt == GPTQ2D_F16 || (DP == 64 && tiles == 4)) launch_tiles<INT8, DP, 1, 2>(a, tiles, s);
  else launch_tiles<INT8, DP, 1, 1>(a, tiles, s);
}
template <bool INT8>
void launch_dim(const TreeArgs& a, int tiles, hipStream_t s) {
  if (a.dim <= 64) launch_type<INT8, 64>(a, tiles, s);
  else if (a.dim <= 128) launch_type<INT8, 128>(a, tiles, s);
  else launch_type<INT8, 256>(a, tiles, s);
}

bool bad_shape(int64_t seqs, int width, int heads, int kv_heads, int dim) {
  return seqs < 1 || seqs > 65535 || width < 1 || width > 64 || kv_heads < 1 || kv_heads > 1024 || heads < kv_heads ||
         heads > 4096 || heads % kv_heads != 0 || seqs * heads * width > (int64_t)1 << 24 || dim < 16 || dim > 256 || dim % 16 != 0;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

gptq2d_status gptq2d_tree_masks(int64_t seqs, int width, const int32_t* parents, uint64_t* masks, void* stream) {
  if (seqs < 0 || seqs > 65535) return refuse("seqs must lie in [0, 65535]");
  if (width < 1 || width > 64) return refuse("width must lie in [1, 64]");
  if (seqs == 0) return GPTQ2D_OK;
  if (!parents || !masks) return refuse("parents or masks are NULL");
  if (!aligned(parents, 4) || !aligned(masks, 8)) return refuse("parents or masks are not aligned");
  hipLaunchKernelGGL(k_tree_masks, dim3((unsigned)ceil_div(seqs * width, 256)), dim3(256), 0, (hipStream_t)stream, seqs,
                     width, parents, masks);
  return launched("gptq2d_tree_masks");
}

size_t gptq2d_tree_attention_workspace_size(int64_t seqs, int width, int heads, int kv_heads, int dim) {
  if (bad_shape(seqs, width, heads, kv_heads, dim)) return 0;
  return part_bytes(seqs, width * (heads / kv_heads), kv_heads, dim);
}

gptq2d_status gptq2d_tree_attention(int64_t seqs, int width, int heads, int kv_heads, int dim, gptq2d_dtype dt,
                                    const void* Q, int64_t ldq, gptq2d_code code, int64_t pages, int page_size,
                                    const void* KC, const void* VC, const float* KS, const float* VS,
                                    const int32_t* table, int64_t ldt, int64_t table_width, const int32_t* context,
                                    const int32_t* drafts, const uint64_t* masks, float scale, void* O, int64_t ldo,
                                    float* lse, void* workspace, size_t ws_bytes, void* stream) {
  if (bad_shape(seqs, width, heads, kv_heads, dim))
    return refuse("bad shape: 1 <= seqs <= 65535, 1 <= width <= 64, heads a multiple of kv_heads (up to 4096 of up to "
                  "1024), seqs x width x heads up to 2^24, dim a multiple of 16 up to 256");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  gptq2d_status st = check_cache(kv_heads, dim, code, pages, page_size, KC, VC, KS, VS);
  if (st != GPTQ2D_OK) return st;
  if (!Q || !O || !table || !context) return refuse("Q, O, table or context are NULL");
  const int64_t cols = (int64_t)heads * dim;
  if (ldq < cols || ldo < cols) return refuse("leading dimension too small");
  if (table_width < 1 || ldt < table_width || table_width > ((int64_t)1 << 28) / page_size)
    return refuse("the page table must cover 1 to 2^28 tokens a sequence");
  const size_t es = elem_size(dt);
  if (!aligned(Q, es) || !aligned(O, es) || !aligned(table, 4) || !aligned(context, 4) || !aligned(drafts, 4) ||
      !aligned(masks, 8) || !aligned(lse, 4))
    return refuse("an argument is not aligned to its elements");
  if (!isfinite(scale)) return refuse("scale is not finite");
  const int rows = width * (heads / kv_heads);
  const size_t need = part_bytes(seqs, rows, kv_heads, dim);
  if (need > 0 && (!workspace || ws_bytes < need)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (need > 0 && !aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  TreeArgs a = {};
  a.seqs = (int)seqs, a.width = width, a.kv = kv_heads, a.group = heads / kv_heads, a.dim = dim, a.rows = rows;
  a.dt = dt, a.Q = Q, a.ldq = ldq;
  a.KC = (const uint8_t*)KC, a.VC = (const uint8_t*)VC, a.KS = KS, a.VS = VS;
  a.pages = pages, a.page = page_size, a.page16 = page_size / 16, a.magic = ((uint64_t)1 << 32) / a.page16 + 1;
  a.table = table, a.ldt = ldt, a.capacity = (int)(table_width * page_size);
  a.context = context, a.drafts = drafts, a.mask = masks;
  a.scale = scale * kLog2E;
  a.qwide = wide_rows(Q, ldq, es), a.owide = wide_rows(O, ldo, es);
  a.O = O, a.ldo = ldo, a.lse = lse, a.part = (float*)workspace;
  const int tiles = query_tiles(rows, dim, dt == GPTQ2D_F32);
  a.rowblocks = (int)ceil_div(rows, 16 * tiles);
  a.mean = split_count(seqs, rows, kv_heads, dim);
  a.splits = (int)std::min<int64_t>(slot_count(seqs, rows, kv_heads, dim), ceil_div(a.capacity, kWaves * kStep));
  if (code == GPTQ2D_INT8)
    launch_dim<true>(a, tiles, (hipStream_t)stream);
  else
    launch_dim<false>(a, tiles, (hipStream_t)stream);
  return launched("gptq2d_tree_attention");
}

}  // extern "C"
