// Log probabilities of given tokens, with the entropy and the top alternatives,
// and their gradient.
//
// For a row of logits x and z = a x (a = 1 / temperature):
//   lse = log sum e^z, lp = z_y - lse, H = lse - sum p z, p = e^(z - lse)
//   dx = a (g_lp (1[y] - p) - g_H p (log p + H))
// All of them but lse are functions of the differences to the row's largest logit, and
// are computed from these.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "codes.hpp"

namespace g2d {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 16;                    // elements of a thread and step
constexpr int kChunk = kThreads * kVec;     // of a work group
constexpr int kMaxTop = 64;
constexpr int kHeld = kThreads;             // candidates that are ranked at once
constexpr int kSpare = 32;                  // candidates beyond the best that wait for that
constexpr int kMaxParts = 64;               // parts of a row
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLog2E = 1.44269504088896341f;

struct ScoreArgs {
  int64_t rows;
  int vocab, top, parts;
  const void* X;
  int64_t ldx;
  float a, a2;  // a and a log2 e
  const int64_t* target;
  float *logprob, *entropy, *lse;
  int32_t* ids;
  float* tops;
  float* stat;       // parts > 1: the Sums of each part
  uint64_t* keys;    // parts > 1: top keys of each part
};

// A candidate as one number that orders as wanted: larger values first (NaN
// above all), the lower index first among equal ones (-0 = 0). No key is 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t i) { return (uint64_t)order_of(x) << 32 | (0xffffffffu - i); }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - (uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}

// The best of a work group's candidates, with room for a whole step's.
struct Pool {
  alignas(16) uint64_t key[kHeld + kChunk];
  alignas(16) uint64_t best[kThreads];
  uint64_t limit;  // candidates below it are none of the best
  int count;
};

// Number of keys above the thread's among the first n of the group's; n <=
// kThreads, past n keys are 0 (and their threads' ranks are not wanted).
__device__ __forceinline__ int rank_in(Pool& p, uint64_t mine, int n) {
  p.best[threadIdx.x] = mine;
  __syncthreads();
  int r = 0;
  if ((int)(threadIdx.x & ~63) >= n) return r;  // (whole waves)
  // (128 bytes are read at once: the reads are to wait for one another seldom)
  for (int i = 0; i < n; i += 16) {
    uint64_t k[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) k[j] = p.best[i + j];
#pragma unroll
    for (int j = 0; j < 16; ++j) r += k[j] > mine;
  }
  return r;
}

// A first limit that at least `top` elements reach, from the largest of each lane
// (whose low bits give way to the lane's number, so that no two of a wave are equal and
// the limit is no higher): the least of the four waves' of rank top / 4, or the greatest
// of the waves' of rank top (rows that leave waves without elements). It is found without
// LDS, whose reads would take longer than all else of a row of a few steps.
__device__ __forceinline__ void first_limit(Pool& p, uint32_t most, int top) {
  const uint32_t mine = most == 0 ? 0 : (most & ~63u) | (threadIdx.x & 63);
  int above = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i) above += (uint32_t)__builtin_amdgcn_readlane((int)mine, i) > mine;
  // where there are fewer elements no lane has the rank, or one without an element: 0
  auto of_rank = [&](int r) {
    const uint64_t at = __ballot(above == r);
    const uint32_t k = at == 0 ? 0 : (uint32_t)__builtin_amdgcn_readlane((int)mine, __builtin_ctzll(at));
    return (uint64_t)(k & ~63u) << 32;
  };
  const int w = threadIdx.x >> 6;
  const uint64_t quarter = of_rank((top - 1) / 4), whole = of_rank(top - 1);
  if ((threadIdx.x & 63) == 0) p.best[w] = quarter, p.best[4 + w] = whole;
  __syncthreads();
  if (threadIdx.x == 0)
    p.limit = max(min(min(p.best[0], p.best[1]), min(p.best[2], p.best[3])),
                  max(max(p.best[4], p.best[5]), max(p.best[6], p.best[7])));
  __syncthreads();
}

// Keeps the `top` best candidates, in order, and makes the last of them the
// limit. While there are more than kHeld, the top-th of the threads' largest is
// one: candidates of `top` threads, a quarter at most, lie above it.
__device__ __forceinline__ void keep_best(Pool& p, int top) {
  const int t = threadIdx.x;
  while (p.count > kHeld) {
    const int n = p.count;
    uint64_t mine[(kHeld + kChunk) / kThreads], most = 0;
#pragma unroll
    for (int i = 0; i < (kHeld + kChunk) / kThreads; ++i) {
      mine[i] = t + i * kThreads < n ? p.key[t + i * kThreads] : 0;
      most = max(most, mine[i]);
    }
    if (rank_in(p, most, kThreads) == top - 1) p.limit = most;
    if (t == 0) p.count = 0;
    __syncthreads();
    const uint64_t limit = p.limit;
#pragma unroll
    for (int i = 0; i < (kHeld + kChunk) / kThreads; ++i)
      if (mine[i] >= limit && mine[i] != 0) p.key[atomicAdd(&p.count, 1)] = mine[i];
    __syncthreads();
  }
  const int n = p.count;
  const uint64_t mine = t < n ? p.key[t] : 0;
  const int r = rank_in(p, mine, n);
  if (mine != 0 && r < top) p.key[r] = mine;
  if (mine != 0 && r == top - 1) p.limit = mine;
  if (t == 0) p.count = min(n, top);
  __syncthreads();
}

// Running sums of a thread or more over logits of which m is the largest:
// s1 = sum 2^(a2 (x - m)), s2 = sum (x - m) 2^(a2 (x - m)). Differences are taken
// before anything is scaled: those of near logits are exact, and a logit of the
// type's lowest value cannot overflow.
struct Sums {
  float m, s1, s2;
};
__device__ __forceinline__ void move_to(Sums& s, float m, float a2) {
  if (s.m != -INFINITY) {
    const float d = s.m - m, f = __builtin_amdgcn_exp2f(a2 * d);
    // f = 0: what was summed is below the new terms' last place
    s.s2 = f == 0.0f ? 0.0f : f * fmaf(s.s1, d, s.s2);
    s.s1 *= f;
  }
  s.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b, float a2) {
  if (a.m >= b.m)
    move_to(b, a.m, a2);
  else
    move_to(a, b.m, a2);
  return Sums{a.m, a.s1 + b.s1, a.s2 + b.s2};
}
__device__ __forceinline__ Sums wave_join(Sums s, float a2) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums o{__shfl_xor(s.m, d), __shfl_xor(s.s1, d), __shfl_xor(s.s2, d)};
    s = (threadIdx.x & d) ? join(o, s, a2) : join(s, o, a2);  // the same order in both lanes
  }
  return s;
}

// A thread's elements of one step: kVec of them in pieces of 16 bytes, the
// pieces of a group side by side. Element j of the thread is element
// step + (j / W) kThreads W + t W + j % W of the row.
template <class T>
struct Piece {
  static constexpr int W = 16 / sizeof(T), N = kVec / W;
  struct alignas(16) V { T v[W]; };
};
template <class T>
__device__ __forceinline__ int64_t index_of(int64_t step, int j) {
  constexpr int W = Piece<T>::W;
  return step + (j / W) * kThreads * W + (int)threadIdx.x * W + j % W;
}
template <class T>
__device__ __forceinline__ void load_whole(const T* x, int64_t step, typename Piece<T>::V raw[Piece<T>::N]) {
#pragma unroll
  for (int i = 0; i < Piece<T>::N; ++i)
    raw[i] = *(const typename Piece<T>::V*)(x + index_of<T>(step, i * Piece<T>::W));
}

// m, l: the largest logit and the logarithm of the sum relative to it
struct Out {
  float lse, entropy, m, l;
};
__device__ __forceinline__ Out finish(const ScoreArgs& a, Sums s) {
  // every logit -inf: the sum is empty
  if (s.m == -INFINITY && s.s1 == 0.0f) return {-INFINITY, 0.0f, 0.0f, 0.0f};
  const float l = logf(s.s1), h = l - a.a * (s.s2 / s.s1);
  return {fmaf(s.m, a.a, l), h < 0.0f ? 0.0f : h, s.m, l};
}

// From the difference to the largest logit, as the sums are: a x - lse would be
// rounded at the size of lse (32000 equal logits of -1e9 would have probability 1).
__device__ __forceinline__ float logprob_of(float x, float a, Out o) { return fmaf(x - o.m, a, -o.l); }

template <class T>
__device__ __forceinline__ float target_logprob(const ScoreArgs& a, int64_t row, Out o) {
  if (!a.target) return 0.0f;
  const int64_t y = a.target[row];
  if (y < 0) return 0.0f;
  if (y >= a.vocab) return __uint_as_float(0x7fc00000u);
  return logprob_of((float)((const T*)a.X)[row * a.ldx + y], a.a, o);
}

__device__ __forceinline__ void put_best(Pool& p, const ScoreArgs& a, int64_t row, Out o) {
  const int t = threadIdx.x;
  if (t >= a.top) return;
  const uint64_t k = p.key[t];
  a.ids[row * a.top + t] = (int32_t)key_index(k);
  a.tops[row * a.top + t] = logprob_of(key_value(k), a.a, o);
}

// One work group per part of a row, one pass. Each thread sums relative to its
// own largest logit so far, which moves rarely after the first steps. At the end
// s1 >= 1 and s2 <= 0, so the entropy log s1 - s2 / s1 cancels nothing.
// TOP: an element below the limit (the top-th best so far) is none of the best; the
// first step sets a limit that few pass, so ranking is seldom. Bound by its bytes:
// 4096 x 128000 bf16 with top 8 212 us in a loop, 4.9 TB/s; 2047 x 50257 50 us, 4.1 TB/s, whose
// rows start off the 16-byte boundaries. One row of 32000 f32 with top 20, 9.0 us: the
// first limit and one ranking of candidates (without top 4.4 us).
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_score(ScoreArgs a) {
  __shared__ Sums wave[kThreads / 64];
  __shared__ typename std::conditional<TOP, Pool, int>::type pool;
  const int t = threadIdx.x;
  const int row32 = blockIdx.x / (uint32_t)a.parts, part = blockIdx.x - row32 * a.parts;
  const int64_t row = row32;
  const T* x = (const T*)a.X + row * a.ldx;
  const int lead = (int)(((uintptr_t)x & 15) / sizeof(T));  // elements from the boundary before the row to it
  const int steps = (a.vocab + lead + kChunk - 1) / kChunk;
  const int first = (uint32_t)(steps * part) / (uint32_t)a.parts, last = (uint32_t)(steps * (part + 1)) / (uint32_t)a.parts;
  Sums s{-INFINITY, 0.0f, 0.0f};
  if constexpr (TOP) {
    if (t == 0) pool.count = 0, pool.limit = 0;
    __syncthreads();
  }
  // the steps inside the row are loaded whole, one ahead; the first and the last may
  // reach past it
  const int inner = lead > 0 ? 1 : 0, outer = (a.vocab + lead) / kChunk - 1;
  typename Piece<T>::V raw[Piece<T>::N];
  const bool any = inner <= outer;
  auto ahead = [&](int c) { load_whole(x, (int64_t)max(inner, min(c, outer)) * kChunk - lead, raw); };
  if (any) ahead(first);
  for (int c = first; c < last; ++c) {
    float v[kVec];
    const int64_t at = (int64_t)c * kChunk - lead;
    if (any) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = (float)raw[i / Piece<T>::W].v[i % Piece<T>::W];
      ahead(c + 1);
    }
    if (c < inner || c > outer) {
      // pieces inside the row are loaded whole (for the others the row's first is, so that
      // no load waits for a branch), those at its ends element by element
      constexpr int W = Piece<T>::W, N = Piece<T>::N;
      const int64_t begin = lead > 0 ? W - lead : 0;
      typename Piece<T>::V some[N] = {};
      if (begin + W <= a.vocab) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int64_t e = index_of<T>(at, i * W);
          some[i] = *(const typename Piece<T>::V*)(x + (e >= 0 && e + W <= a.vocab ? e : begin));
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t e = index_of<T>(at, i * W);
        const bool inside = e >= 0 && e + W <= a.vocab;
#pragma unroll
        for (int j = 0; j < W; ++j) v[i * W + j] = inside ? (float)some[i].v[j] : -INFINITY;
        if (!inside && e + W > 0 && e < a.vocab) {
#pragma unroll
          for (int j = 0; j < W; ++j) v[i * W + j] = (float)x[max((int64_t)0, min(e + j, (int64_t)a.vocab - 1))];
#pragma unroll
          for (int j = 0; j < W; ++j) v[i * W + j] = e + j >= 0 && e + j < a.vocab ? v[i * W + j] : -INFINITY;
        }
      }
    }
    float m = v[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) m = fmaxf(m, v[i]);
    if (m > s.m) move_to(s, m, a.a2);
    const Sums old = s;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float d = v[i] - s.m, e = __builtin_amdgcn_exp2f(d * a.a2);
      s.s1 += e;
      s.s2 = fmaf(e, d, s.s2);
    }
    bool odd = false;  // a NaN, which maxima drop
    if (!(fabsf(s.s2) < 1e37f)) {
      // a difference of -inf (0 times it is NaN), or a NaN: once more with care
      s = old;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        odd |= v[i] != v[i];
        if (v[i] == -INFINITY) continue;
        // 2^(a2 d) is 0 long before d reaches the clamp
        const float d = fmaxf(v[i] - s.m, -3e38f), e = __builtin_amdgcn_exp2f(d * a.a2);
        s.s1 += e;
        s.s2 = fmaf(e, d, s.s2);
      }
      if (odd) s.s1 = s.s2 = __uint_as_float(0x7fc00000u);
    }
    if constexpr (TOP) {
      if (c == first) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const int64_t e = index_of<T>(at, i);
          if (e >= 0 && e < a.vocab) most = max(most, order_of(v[i]));
        }
        first_limit(pool, most, a.top);
      }
      const uint64_t limit = pool.limit;
      const float least = key_value(limit);  // NaN: of the start, or NaN themselves
      if (odd || !(m < least)) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          if (v[i] < least) continue;
          const int64_t e = index_of<T>(at, i);
          const uint64_t k = key_of(v[i], (uint32_t)e);
          if (k >= limit && e >= 0 && e < a.vocab) pool.key[atomicAdd(&pool.count, 1)] = k;
        }
      }
      __syncthreads();
      // a limit that keeps up spares the threads most of these
      if (pool.count > a.top + kSpare || c + 1 == last) keep_best(pool, a.top);
      __syncthreads();
    }
  }
  s = wave_join(s, a.a2);
  if ((t & 63) == 0) wave[t >> 6] = s;
  __syncthreads();
  s = join(join(wave[0], wave[1], a.a2), join(wave[2], wave[3], a.a2), a.a2);
  if (a.parts > 1) {
    if (t == 0) ((f4*)a.stat)[blockIdx.x] = f4{s.m, s.s1, s.s2, 0.0f};
    if constexpr (TOP) {
      // a part of a step's remainder may have fewer
      if (t < a.top) a.keys[(int64_t)blockIdx.x * a.top + t] = t < pool.count ? pool.key[t] : 0;
    }
    return;
  }
  const Out o = finish(a, s);
  if (t == 0) {
    a.lse[row] = o.lse;
    a.entropy[row] = o.entropy;
    a.logprob[row] = target_logprob<T>(a, row, o);
  }
  if constexpr (TOP) put_best(pool, a, row, o);
}

// One work group per row: its parts' sums, and the best of their best. One row of
// eight parts 5.4 us with top 20, 3.2 us without.
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_score_join(ScoreArgs a) {
  __shared__ typename std::conditional<TOP, Pool, int>::type pool;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  Sums s{-INFINITY, 0.0f, 0.0f};
  const int l = t & 63;
  if (l < a.parts) {
    const f4 st = ((const f4*)a.stat)[row * a.parts + l];
    s = Sums{st[0], st[1], st[2]};
  }
  s = wave_join(s, a.a2);
  const Out o = finish(a, s);
  if (t == 0) {
    a.lse[row] = o.lse;
    a.entropy[row] = o.entropy;
    a.logprob[row] = target_logprob<T>(a, row, o);
  }
  if constexpr (TOP) {
    const int n = a.parts * a.top;  // at most kMaxParts kMaxTop = kChunk
    if (t == 0) pool.count = n, pool.limit = 0;
    for (int i = t; i < n; i += kThreads) pool.key[i] = a.keys[row * n + i];
    __syncthreads();
    keep_best(pool, a.top);
    put_best(pool, a, row, o);
  }
}

struct GradArgs {
  int64_t rows;
  int vocab, parts;
  const void* X;
  int64_t ldx;
  float a, a2;
  const int64_t* target;
  const float *lse, *entropy, *gl, *gh;
  void* D;
  int64_t ldd;
  bool shared;  // the gradients share memory with the logits
};

// Past it lse, a 32-bit number, is off by more than 2^-18, and p by as much of itself.
constexpr float kNear = 128.0f;

// One pass, element by element. Rows of logits and gradients that start at the
// same distance from a 16-byte boundary are moved in 16-byte pieces. Bound by its
// bytes: 2047 x 50257 bf16 78 us, 5.3 TB/s read and written (the logits partly from the
// last-level cache, after the forward pass).
// A row whose lse is far from zero (or not a 32-bit number at all) is summed again
// first, relative to its largest logit. Every part of a row does that for itself; where
// one part's gradients would take the place of logits that another has yet to
// sum, the first part takes the whole row.
template <class T>
__global__ __launch_bounds__(kThreads) void k_score_grad(GradArgs a) {
  constexpr int W = 16 / sizeof(T);
  struct alignas(16) V { T v[W]; };
  __shared__ Sums wave[kThreads / 64];
  const int row32 = blockIdx.x / (uint32_t)a.parts, part = blockIdx.x - row32 * a.parts;
  const int64_t row = row32;
  const T* x = (const T*)a.X + row * a.ldx;
  T* d = (T*)a.D + row * a.ldd;
  const float lse = a.lse[row];
  const bool far = fabsf(lse) > kNear, whole = far && a.shared;
  if (whole && part > 0) return;
  const float gl = a.gl ? a.gl[row] : 0.0f, gh = a.gh ? a.gh[row] : 0.0f;
  const float H = gh != 0.0f ? a.entropy[row] : 0.0f;
  const int64_t y = a.gl ? a.target[row] : -1;  // (past the vocabulary it would make NaN of the entropy's part too)
  const bool given = y >= 0 && y < a.vocab;
  const float g = given ? gl : y >= a.vocab ? gl * __uint_as_float(0x7fc00000u) : 0.0f;
  const int lead = (int)(((uintptr_t)x & 15) / sizeof(T));
  const int64_t n = a.vocab + lead;
  float m = 0.0f, l = lse;  // log p = a (x - m) - l
  if (far) {
    Sums s{-INFINITY, 0.0f, 0.0f};
    auto add = [&](float v) {
      if (v > s.m) {
        s.s1 *= __builtin_amdgcn_exp2f((s.m - v) * a.a2);
        s.m = v;
      }
      if (v != -INFINITY) s.s1 += __builtin_amdgcn_exp2f((v - s.m) * a.a2);
    };
    for (int64_t e = threadIdx.x * W; e < n; e += kThreads * W) {
      const int64_t i0 = e - lead;
      if (i0 >= 0 && i0 + W <= a.vocab) {
        const V in = *(const V*)(x + i0);
#pragma unroll
        for (int j = 0; j < W; ++j) add((float)in.v[j]);
      } else {
        for (int j = 0; j < W; ++j)
          if (i0 + j >= 0 && i0 + j < a.vocab) add((float)x[i0 + j]);
      }
    }
    s = wave_join(s, a.a2);
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = s;
    __syncthreads();
    s = join(join(wave[0], wave[1], a.a2), join(wave[2], wave[3], a.a2), a.a2);
    m = s.m, l = logf(s.s1);
  }
  auto one = [&](float v, int64_t i) {
    const float q = fmaf(v - m, a.a, -l);
    const float p = __builtin_amdgcn_exp2f(q * kLog2E);
    float r = -p * (g + gh * (fmaxf(q, -700.0f) + H));
    if (i == y) r += g;
    // a row without a finite logit has no gradient
    return m == -INFINITY ? 0.0f : a.a * r;
  };
  const bool wide = (((uintptr_t)x ^ (uintptr_t)d) & 15) == 0;
  const int parts = whole ? 1 : a.parts;
  const int64_t per = (n + parts - 1) / parts;
  const int64_t span = (per + kThreads * W - 1) / (kThreads * W) * (kThreads * W);
  const int64_t end = min(n, span * (part + 1));
  for (int64_t e = span * part + threadIdx.x * W; e < end; e += kThreads * W) {
    const int64_t i0 = e - lead;
    if (wide && i0 >= 0 && i0 + W <= a.vocab) {
      const V in = *(const V*)(x + i0);
      V out;
#pragma unroll
      for (int j = 0; j < W; ++j) out.v[j] = (T)one((float)in.v[j], i0 + j);
      *(V*)(d + i0) = out;
    } else {
      for (int j = 0; j < W; ++j)
        if (i0 + j >= 0 && i0 + j < a.vocab) d[i0 + j] = (T)one((float)x[i0 + j], i0 + j);
    }
  }
}

// Parts of a row: as many as give every compute unit a work group, each of one step
// at least. At 256 / 512 / 1024 work groups: 700 rows of 32000 bf16 13.4 / 13.3 / 19.7
// us, 256 of 128000 f32 23.1 / 27.9 / 30.5, 130 of 50257 bf16 with top 20 26.3 / 25.4 /
// 29.2, 64 of 128000 12.5 / 12.2 / 13.5 (more parts are more to join).
int part_count(int64_t rows, int64_t vocab) {
  const int64_t want = ceil_div(256, rows), room = ceil_div(vocab, kChunk);
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, room, kMaxParts}));
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t stat_bytes(int64_t rows, int parts) { return up256((size_t)rows * parts * 4 * sizeof(float)); }
size_t score_bytes(int64_t rows, int64_t vocab, int top) {
  const int parts = part_count(rows, vocab);
  return parts == 1 ? 0 : stat_bytes(rows, parts) + up256((size_t)rows * parts * top * sizeof(uint64_t));
}

bool bad_sizes(int64_t rows, int64_t vocab) {
  return rows < 0 || rows > (int64_t)1 << 22 || vocab < 1 || vocab > (int64_t)1 << 28;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

size_t gptq2d_token_logprobs_workspace_size(int64_t rows, int64_t vocab, int top) {
  if (bad_sizes(rows, vocab) || rows == 0 || top < 0 || top > kMaxTop) return 0;
  return score_bytes(rows, vocab, top);
}

gptq2d_status gptq2d_token_logprobs(int64_t rows, int64_t vocab, gptq2d_dtype dt, const void* X, int64_t ldx,
                                    float scale, const int64_t* target, int top, float* logprob, float* entropy,
                                    float* lse, int32_t* ids, float* tops, void* workspace, size_t ws_bytes,
                                    void* stream) {
  if (bad_sizes(rows, vocab)) return refuse("rows must lie in [0, 2^22], vocab in [1, 2^28]");
  if (top < 0 || top > kMaxTop || top > vocab) return refuse("top must lie in [0, 64] and not exceed vocab");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (!(scale > 0.0f) || !isfinite(scale)) return refuse("scale must be positive and finite");
  if (rows == 0) return GPTQ2D_OK;
  if (!X || !logprob || !entropy || !lse) return refuse("X, logprob, entropy or lse is NULL");
  if (top > 0 && (!ids || !tops)) return refuse("ids or tops is NULL");
  if (ldx < vocab) return refuse("leading dimension too small");
  if (!aligned(X, elem_size(dt)) || !aligned(target, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
      !aligned(lse, 4) || !aligned(ids, 4) || !aligned(tops, 4))
    return refuse("an argument is not aligned to its elements");
  const size_t need = score_bytes(rows, vocab, top);
  if (need > 0 && (!workspace || ws_bytes < need)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (need > 0 && !aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int parts = part_count(rows, vocab);
  ScoreArgs a = {rows, (int)vocab, top, parts, X, ldx, scale, scale * kLog2E, target, logprob, entropy, lse, ids, tops,
                 (float*)workspace, (uint64_t*)((char*)workspace + stat_bytes(rows, parts))};
  const hipStream_t s = (hipStream_t)stream;
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    const dim3 grid((unsigned)(rows * parts));
    if (top > 0)
      hipLaunchKernelGGL((k_score<T, true>), grid, dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL((k_score<T, false>), grid, dim3(kThreads), 0, s, a);
    if (parts > 1) {
      if (top > 0)
        hipLaunchKernelGGL((k_score_join<T, true>), dim3((unsigned)rows), dim3(kThreads), 0, s, a);
      else
        hipLaunchKernelGGL((k_score_join<T, false>), dim3((unsigned)rows), dim3(kThreads), 0, s, a);
    }
  });
  return launched("gptq2d_token_logprobs");
}

gptq2d_status gptq2d_token_logprobs_backward(int64_t rows, int64_t vocab, gptq2d_dtype dt, const void* X, int64_t ldx,
                                             float scale, const int64_t* target, const float* lse, const float* entropy,
                                             const float* g_logprob, const float* g_entropy, void* dX, int64_t lddx,
                                             void* stream) {
  if (bad_sizes(rows, vocab)) return refuse("rows must lie in [0, 2^22], vocab in [1, 2^28]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (!(scale > 0.0f) || !isfinite(scale)) return refuse("scale must be positive and finite");
  if (!g_logprob && !g_entropy) return refuse("no gradient is given");
  if (rows == 0) return GPTQ2D_OK;
  if (!X || !dX || !lse) return refuse("X, dX or lse is NULL");
  if (g_logprob && !target) return refuse("g_logprob needs the targets");
  if (g_entropy && !entropy) return refuse("g_entropy needs the entropy");
  if (ldx < vocab || lddx < vocab) return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  if (!aligned(X, es) || !aligned(dX, es) || !aligned(target, 8) || !aligned(lse, 4) || !aligned(entropy, 4) ||
      !aligned(g_logprob, 4) || !aligned(g_entropy, 4))
    return refuse("an argument is not aligned to its elements");
  GradArgs a = {rows, (int)vocab, 1, X, ldx, scale, scale * kLog2E, target, lse, entropy, g_logprob, g_entropy, dX, lddx,
                (uintptr_t)X < (uintptr_t)dX + ((rows - 1) * lddx + vocab) * es &&
                    (uintptr_t)dX < (uintptr_t)X + ((rows - 1) * ldx + vocab) * es};
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(2048, rows), ceil_div(vocab, 4096)));
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    hipLaunchKernelGGL(k_score_grad<T>, dim3((unsigned)(rows * a.parts)), dim3(kThreads), 0, (hipStream_t)stream, a);
  });
  return launched("gptq2d_token_logprobs_backward");
}

}  // extern "C"
