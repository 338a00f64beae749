// Which tokens of a drafted tree are kept, and the token after them: decided from the
// target's logits and given random numbers, or greedily.
//
// p_c = softmax(a x_c) of the row of token c. The scan starts at token 0, which is
// decided already, and tests the tokens that follow the current one in their order:
//   certain drafts:  u (1 - sum of p over those rejected here) < p(token)
//   drawn from q:    u M q(token) < p(token) - beta q(token), beta = 0 and M = 1 at
//                    first; a rejection makes beta += M, M = sum max(p - beta q, 0)
//   greedy:          the token is the lowest of the largest logits
// An accepted token is the current one from there on. In the end the next token is
// the first whose sum of r, over it and the tokens before it, is above u_0 times the
// sum over all, r being what is left of p: p without the rejected tokens, or max(p -
// beta q, 0), or p where that is nothing. (max(max(p - q, 0) / M - q, 0) is max(p - (1
// + M) q, 0) / M: drafts of one distribution, rejected one after another, leave a
// single pass over the row each.)
//
// A vocabulary has as many borders between tokens as tokens: with sums that are off by
// 1e-8, one in a thousand samples of a vocabulary of 128000 would be another one. What
// decides the sample is held in 64 bits; tests of single tokens, and log probabilities,
// have 32-bit terms, summed in 32 bits by a thread and in 64 after that.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "codes.hpp"

namespace g2d {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 16;                 // elements of a thread and step
constexpr int kChunk = kThreads * kVec;  // of a work group
constexpr int kMaxWidth = 64;
constexpr int kMaxParts = 64;            // of a row
constexpr float kLog2E = 1.44269504088896341f;

// of a part of a row: its largest logit, the lowest token that has it, and sums
// relative to it
struct alignas(16) Part {
  float m;
  int32_t at;
  double sum;
};
// of a part of the last row; m, sum: as above, left: the sum of r
struct alignas(16) Last {
  double m, sum, left;
  int64_t at;
};
// what the scan ends with
struct alignas(16) State {
  int32_t node;      // -1: none
  int32_t residual;  // r is less than p
  uint64_t gone;     // rejected tokens of the node
  double beta, m, sum;  // drawn drafts: with the row's largest logit and its sum
};

struct VerifyArgs {
  int64_t seqs;
  int width, vocab, parts, chunks, per;  // parts of a row; of the last one, with `per` elements each
  const void* X;
  int64_t ldx;
  float a;
  const int64_t* tokens;
  const int32_t *parents, *drafts;
  const float* u;
  const void* D;
  int64_t ldd;
  float ad;
  const float* dlse;
  int32_t *path, *count;
  int64_t* next;
  float* logprob;
  Part* part;
  Last* last;
  State* state;
};

__device__ __forceinline__ int drafted(const VerifyArgs& v, int64_t seq) {
  return v.drafts ? min(max(v.drafts[seq], 0), v.width) : v.width;
}
__device__ __forceinline__ int parent_of(const VerifyArgs& v, int64_t seq, int t) {
  if (!v.parents) return t - 1;
  const int p = v.parents[seq * v.width + t];
  return p >= 0 && p < t ? p : -1;
}

// Elements first .. first + kVec - 1 of a row, those outside [0, n) as -inf. `first` is
// kVec elements times something behind a 16-byte boundary where the row allows it.
template <class T>
__device__ __forceinline__ void load16(const T* x, int64_t first, int n, float v[kVec]) {
  constexpr int W = 16 / sizeof(T);
  struct alignas(16) V { T v[W]; };
  if (first >= 0 && first + kVec <= n && ((uintptr_t)(x + first) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kVec / W; ++i) {
      const V p = *(const V*)(x + first + i * W);
#pragma unroll
      for (int j = 0; j < W; ++j) v[i * W + j] = (float)p.v[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)x[max((int64_t)0, min(first + i, (int64_t)n - 1))];
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = first + i >= 0 && first + i < n ? v[i] : -INFINITY;
  }
}
template <class T>
__device__ __forceinline__ int lead_of(const T* x) {
  return (int)(((uintptr_t)x & 15) / sizeof(T));
}

// Joins two parts: the lower index of equal maxima.
__device__ __forceinline__ Part join(Part p, Part q, float a) {
  if (q.m > p.m || (q.m == p.m && q.at < p.at)) {
    const Part t = p;
    p = q;
    q = t;
  }
  if (q.sum != 0.0) p.sum += q.sum * (double)__builtin_amdgcn_exp2f((q.m - p.m) * a * kLog2E);
  return p;
}
__device__ __forceinline__ Part wave_join(Part p, float a) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Part q{__shfl_xor(p.m, d), __shfl_xor(p.at, d), __shfl_xor(p.sum, d)};
    p = (threadIdx.x & d) ? join(q, p, a) : join(p, q, a);
  }
  return p;
}

// Largest logit and sum of a part of every row that tokens follow.
template <class T>
__global__ __launch_bounds__(kThreads) void k_rows(VerifyArgs v) {
  __shared__ Part wave[kThreads / 64];
  const int row32 = blockIdx.x / (uint32_t)v.parts, part = blockIdx.x - row32 * v.parts;
  const int64_t row = row32, seq = row / v.width;
  const int c = (int)(row - seq * v.width), t = threadIdx.x, lane = t & 63;
  const int n = drafted(v, seq);
  if (__ballot(lane > c && lane < n && parent_of(v, seq, lane < v.width ? lane : 0) == c) == 0) return;
  const T* x = (const T*)v.X + row * v.ldx;
  const int lead = lead_of(x);
  const int steps = (v.vocab + lead + kChunk - 1) / kChunk;
  const int first = (int)((int64_t)steps * part / v.parts), last = (int)((int64_t)steps * (part + 1) / v.parts);
  const float a2 = v.a * kLog2E;
  float m = -INFINITY, sum = 0.0f;
  int at = 0x7fffffff;
  for (int s = first; s < last; ++s) {
    float z[kVec];
    const int64_t e = (int64_t)s * kChunk + (int64_t)t * kVec - lead;
    load16(x, e, v.vocab, z);
    float top = z[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) top = fmaxf(top, z[i]);
    if (top > m) {
      sum *= __builtin_amdgcn_exp2f((m - top) * a2);
      m = top;
      int k = 0;
#pragma unroll
      for (int i = kVec - 1; i >= 0; --i) k = z[i] == top ? i : k;
      at = (int)(e + k);
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (z[i] != -INFINITY) sum += __builtin_amdgcn_exp2f((z[i] - m) * a2);  // NaN: NaN
  }
  Part p = wave_join(Part{m, at, (double)sum}, v.a);
  if (lane == 0) wave[t >> 6] = p;
  __syncthreads();
  if (t == 0) v.part[blockIdx.x] = join(join(wave[0], wave[1], v.a), join(wave[2], wave[3], v.a), v.a);
}

constexpr int kWalk = 1024;

__device__ __forceinline__ double wave_sum(double s) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
  return s;
}

// The scan of a sequence. All waves go through it alike; where a drawn draft is
// rejected they share a pass over the row.
template <class T>
__global__ __launch_bounds__(kWalk) void k_walk(VerifyArgs v) {
  __shared__ Part rows[kMaxWidth];
  __shared__ double sums[kWalk / 64];
  const int64_t seq = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int n = drafted(v, seq);
  const bool in = lane < v.width;
  const int parent = in && lane > 0 && lane < n ? parent_of(v, seq, lane) : -1;
  // the sums of the rows that tokens follow
  for (int c = w; c < v.width; c += kWalk / 64) {
    if (__ballot(parent == c) == 0) continue;
    Part p{-INFINITY, 0x7fffffff, 0.0};
    if (lane < v.parts) p = v.part[(seq * v.width + c) * v.parts + lane];
    p = wave_join(p, v.a);
    if (lane == 0) rows[c] = p;
  }
  __syncthreads();
  const int64_t token = in ? v.tokens[seq * v.width + lane] : -1;
  const T *X = (const T*)v.X + seq * v.width * v.ldx, *D = (const T*)v.D + seq * v.width * v.ldd;
  const float* dlse = v.dlse + seq * v.width;
  double p = 0.0, q = 0.0;
  float lp = 0.0f;
  bool best = false;
  if (parent >= 0) {
    const Part r = rows[parent];
    const bool ok = token >= 0 && token < v.vocab;
    const double z = ok ? ((double)(float)X[parent * v.ldx + token] - (double)r.m) * (double)v.a : -INFINITY;
    // of a row of nothing but -inf, or with a NaN or +inf: NaN
    p = exp(z) / r.sum;
    lp = (float)(z - log(r.sum));
    if (!(r.sum > 0.0)) lp = __uint_as_float(0x7fc00000u), p = (double)lp;
    if (v.D && ok) q = exp((double)(float)D[parent * v.ldd + token] * (double)v.ad - (double)dlse[parent]);
    best = p == p && token == r.at;
  }
  const double u = v.u && in ? (double)v.u[seq * v.width + lane] : 0.0;
  auto of = [&](double x, int from) { return __shfl(x, from); };
  int cur = n > 0 ? 0 : -1, kept = n > 0 ? 1 : 0;
  int way = lane == 0 && n > 0 ? 0 : -1;  // lane i: the i-th kept token
  double beta = 0.0, M = 1.0, gone_p = 0.0, total = 0.0, top = 0.0;
  uint64_t gone = 0;
  bool summed = false;
  // the sum of the current row and of max(p - beta q, 0), in 64 bits
  auto pass = [&](bool residual) {
    const T *x = X + cur * v.ldx, *d = D + cur * v.ldd;
    double s = 0.0;
    const int lead = lead_of(x);
    for (int64_t e = (int64_t)t * kVec - lead; e < v.vocab; e += kWalk * kVec) {
      float z[kVec], y[kVec];
      load16(x, e, v.vocab, z);
      if (residual) load16(d, e, v.vocab, y);
      for (int i = 0; i < kVec; ++i) {
        if (z[i] == -INFINITY) continue;
        const double f = exp(((double)z[i] - top) * (double)v.a);
        if (!residual)
          s += f;
        else
          s += fmax(f / total - beta * exp((double)y[i] * (double)v.ad - (double)dlse[cur]), 0.0);
      }
    }
    s = wave_sum(s);
    __syncthreads();
    if (lane == 0) sums[w] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kWalk / 64; ++i) s += sums[i];
    return s;
  };
  while (cur >= 0) {
    const uint64_t children = __ballot(parent == cur);
    int taken = -1;
    for (uint64_t left = children; left != 0; left &= left - 1) {
      const int c = __builtin_ctzll(left);
      const double pc = of(p, c);
      if (!v.u) {
        if (__shfl((int)best, c)) taken = c;
      } else if (v.D) {
        if (gone != 0) {
          if (!summed) top = (double)rows[cur].m, total = pass(false), summed = true;
          M = pass(true);
        }
        const double qc = of(q, c);
        if (of(u, c) * M * qc < pc - beta * qc) taken = c;
        else beta += M;
      } else {
        const int64_t mine = __shfl(token, c);
        const bool again = (__ballot(token == mine) & gone) != 0;
        if (!again && of(u, c) * (1.0 - gone_p) < pc) taken = c;
        else if (!again) gone_p += pc;
      }
      if (taken >= 0) break;
      gone |= 1ull << c;
    }
    if (taken < 0) break;
    cur = taken;
    if (lane == kept) way = cur;
    ++kept;
    gone = 0, beta = 0.0, M = 1.0, gone_p = 0.0, summed = false;
  }
  const bool residual = v.u && gone != 0;
  if (residual && v.D && !summed) top = (double)rows[cur].m, total = pass(false);
  if (w == 0) {
    if (in) {
      v.path[seq * v.width + lane] = way;
      if (lane > 0) v.logprob[seq * v.width + lane] = lp;
    }
    if (lane == 0) {
      v.count[seq] = kept;
      v.state[seq] = State{cur, residual, gone, beta, top, total};
    }
  }
}

// The tokens of the state's rejected drafts that lie in [first, first + per) of the row.
struct Gone {
  int token[kMaxWidth];
  int n;
};
__device__ __forceinline__ void find_gone(const VerifyArgs& v, const State& s, int64_t seq, int64_t first, int64_t end, Gone& g) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const int64_t token = s.gone >> lane & 1 ? v.tokens[seq * v.width + lane] : -1;
    const bool here = token >= first && token < end;
    const uint64_t all = __ballot(here);
    if (here) g.token[__popcll(all & ((1ull << lane) - 1))] = (int)token;
    if (lane == 0) g.n = __popcll(all);
  }
}

// e^(a (x - m)) and what is left of it (relative to the row's sum, for drawn drafts) of a
// thread's elements
template <class T>
__device__ __forceinline__ void remaining(const VerifyArgs& v, const State& s, const Gone& g, const T* x, const T* d, double dlse,
                                          int64_t e, const float z[kVec], double m, double f[kVec], double r[kVec]) {
  float y[kVec];
  const bool drawn = s.residual && v.D;
  if (drawn) load16(d, e, v.vocab, y);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    f[i] = z[i] == -INFINITY ? 0.0 : exp(((double)z[i] - m) * (double)v.a);
    r[i] = f[i];
    if (drawn) r[i] = z[i] == -INFINITY ? 0.0 : fmax(f[i] / s.sum - s.beta * exp((double)y[i] * (double)v.ad - dlse), 0.0);
  }
  if (s.residual && !v.D)
    for (int k = 0; k < g.n; ++k)
#pragma unroll
      for (int i = 0; i < kVec; ++i) r[i] = e + i == g.token[k] ? 0.0 : r[i];
}

// Sums of one part of the last row.
template <class T>
__global__ __launch_bounds__(kThreads) void k_last(VerifyArgs v) {
  __shared__ Gone gone;
  __shared__ float tops[kThreads / 64];
  __shared__ double sums[2][kThreads / 64];
  __shared__ int first[kThreads / 64];
  const int64_t seq = blockIdx.x / (uint32_t)v.chunks;
  const int chunk = blockIdx.x - (int)seq * v.chunks, t = threadIdx.x, lane = t & 63;
  const State s = v.state[seq];
  if (s.node < 0) return;
  const int64_t row = seq * v.width + s.node;
  const T *x = (const T*)v.X + row * v.ldx, *d = (const T*)v.D + row * v.ldd;
  const int lead = lead_of(x);
  const int64_t begin = (int64_t)chunk * v.per - lead, end = min(begin + v.per, (int64_t)v.vocab);
  find_gone(v, s, seq, begin, end, gone);
  float top = -INFINITY;
  int at = 0x7fffffff;
  for (int64_t e = begin + t * kVec; e < end; e += kChunk) {
    float z[kVec];
    load16(x, e, v.vocab, z);
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (z[i] > top) top = z[i], at = (int)(e + i);
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const float o = __shfl_xor(top, k);
    const int oa = __shfl_xor(at, k);
    if (o > top || (o == top && oa < at)) top = o, at = oa;
  }
  if (lane == 0) tops[t >> 6] = top, first[t >> 6] = at;
  __syncthreads();
  for (int k = 0; k < kThreads / 64; ++k)
    if (tops[k] > top || (tops[k] == top && first[k] < at)) top = tops[k], at = first[k];
  // the row's own largest where the scan needed it: r is relative to the whole row then
  const double m = s.residual && v.D ? s.m : (double)top;
  const double dlse = s.residual && v.D ? (double)v.dlse[row] : 0.0;
  double all = 0.0, left = 0.0;
  bool bad = false;
  for (int64_t e = begin + t * kVec; e < end; e += kChunk) {
    float z[kVec];
    double f[kVec], r[kVec];
    load16(x, e, v.vocab, z);
    remaining(v, s, gone, x, d, dlse, e, z, m, f, r);
#pragma unroll
    for (int i = 0; i < kVec; ++i) all += f[i], left += r[i], bad |= z[i] != z[i] || z[i] == INFINITY;
  }
  if (bad) all = NAN;
  all = wave_sum(all), left = wave_sum(left);
  if (lane == 0) sums[0][t >> 6] = all, sums[1][t >> 6] = left;
  __syncthreads();
  if (t == 0) {
    all = left = 0.0;
    for (int k = 0; k < kThreads / 64; ++k) all += sums[0][k], left += sums[1][k];
    v.last[blockIdx.x] = Last{m, all, left, at};
  }
}

// The next token of a sequence: its part of the row, then its place there.
template <class T>
__global__ __launch_bounds__(kThreads) void k_next(VerifyArgs v) {
  __shared__ Gone gone;
  __shared__ double sums[kThreads / 64];
  __shared__ int found;
  const int64_t seq = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63;
  State s = v.state[seq];
  if (s.node < 0) {
    if (t == 0) v.next[seq] = -1, v.logprob[seq * v.width] = 0.0f;
    return;
  }
  const int64_t row = seq * v.width + s.node;
  const T *x = (const T*)v.X + row * v.ldx, *d = (const T*)v.D + row * v.ldd;
  Last l{-INFINITY, 0.0, 0.0, 0x7fffffff};
  if (lane < v.chunks) l = v.last[seq * v.chunks + lane];
  double m = l.m, best = l.m;
  int64_t at = l.at;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const double o = __shfl_xor(best, k);
    const int64_t oa = __shfl_xor(at, k);
    if (o > best || (o == best && oa < at)) best = o, at = oa;
  }
  const double f = l.sum == 0.0 ? 0.0 : exp((m - best) * (double)v.a);
  const double total = wave_sum(l.sum * f);
  const bool drawn = s.residual && v.D;
  double left = l.left * (drawn ? 1.0 : f);
  if (l.left == 0.0) left = 0.0;
  if (!(total > 0.0)) {  // nothing but -inf, or a NaN or +inf
    if (t == 0) v.next[seq] = -1, v.logprob[seq * v.width] = __uint_as_float(0x7fc00000u);
    return;
  }
  int64_t chosen = at;
  if (v.u) {
    const double u = (double)v.u[seq * v.width];
    if (s.residual && !(wave_sum(left) > 0.0)) {  // nothing is left of p: p itself
      s.residual = 0;
      left = l.sum * f;
      if (drawn && l.sum == 0.0) left = 0.0;
    }
    // sums of the parts up to the lane's
    double upto = left;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const double o = __shfl_up(upto, k);
      if (lane >= k) upto += o;
    }
    const double aim = u * __shfl(upto, 63);
    const uint64_t over = __ballot(upto > aim && left > 0.0), some = __ballot(left > 0.0);
    const int part = over != 0 ? __builtin_ctzll(over) : some != 0 ? 63 - __builtin_clzll(some) : 0;
    const double before = __shfl(upto - left, part), aim_in = aim - before;
    const double pm = __shfl(m, part), pf = s.residual && v.D ? 1.0 : __shfl(f, part);
    const int lead = lead_of(x);
    const int64_t begin = (int64_t)part * v.per - lead, end = min(begin + v.per, (int64_t)v.vocab);
    find_gone(v, s, seq, begin, end, gone);
    if (t == 0) found = -1;
    __syncthreads();
    const double dlse = s.residual && v.D ? (double)v.dlse[row] : 0.0;
    double past = 0.0;
    int late = -1;  // the last token with something left
    for (int64_t step = begin; step < end; step += kChunk) {
      const int64_t e = step + t * kVec;
      float z[kVec];
      double g[kVec], r[kVec], mine = 0.0;
      load16(x, e, v.vocab, z);
      remaining(v, s, gone, x, d, dlse, e, z, pm, g, r);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        r[i] *= pf;
        mine += r[i];
        if (r[i] > 0.0) late = (int)(e + i);
      }
      double in = mine;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const double o = __shfl_up(in, k);
        if (lane >= k) in += o;
      }
      __syncthreads();
      if (lane == 63) sums[t >> 6] = in;
      __syncthreads();
      double ahead = past;
      for (int k = 0; k < (t >> 6); ++k) ahead += sums[k];
      double sum = ahead + (in - mine);
      int pick = -1;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        sum += r[i];
        if (pick < 0 && r[i] > 0.0 && sum > aim_in) pick = (int)(e + i);
      }
      // the first thread that has one
      const uint64_t has = __ballot(pick >= 0);
      const int mine_first = has != 0 ? __shfl(pick, __builtin_ctzll(has)) : -1;
      for (int k = 0; k < kThreads / 64; ++k) {
        __syncthreads();
        if (k == t >> 6 && lane == 0 && found < 0 && mine_first >= 0) found = mine_first;
      }
      __syncthreads();
      if (found >= 0) break;
      for (int k = 0; k < kThreads / 64; ++k) past += sums[k];
    }
    chosen = found;
    if (chosen < 0) {  // the sums' last place: the last one
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) late = max(late, __shfl_xor(late, k));
      __syncthreads();
      if (t == 0) found = -1;
      __syncthreads();
      if (lane == 0) atomicMax(&found, late);
      __syncthreads();
      chosen = found;
    }
  }
  if (t == 0) {
    v.next[seq] = chosen;
    v.logprob[seq * v.width] = chosen < 0 ? __uint_as_float(0x7fc00000u)
                                          : (float)(((double)(float)x[chosen] - best) * (double)v.a - log(total));
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// parts of a row for the first pass
int row_parts(int64_t rows, int64_t vocab) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(1024, rows), ceil_div(vocab + 7, kChunk), kMaxParts}));
}
// elements of a part of the last row: parts of whole steps, kMaxParts of them at most
int64_t last_per(int64_t vocab) { return ceil_div(ceil_div(vocab + 7, kMaxParts), kChunk) * kChunk; }

struct Space {
  size_t part, last, state, all;
};
Space space_of(int64_t seqs, int width, int64_t vocab) {
  Space s;
  s.part = 0;
  s.last = s.part + up256((size_t)seqs * width * row_parts(seqs * width, vocab) * sizeof(Part));
  s.state = s.last + up256((size_t)seqs * ceil_div(vocab + 7, last_per(vocab)) * sizeof(Last));
  s.all = s.state + up256((size_t)seqs * sizeof(State));
  return s;
}
bool bad_sizes(int64_t seqs, int width, int64_t vocab) {
  return seqs < 0 || seqs > 65535 || width < 1 || width > kMaxWidth || vocab < 1 || vocab > (int64_t)1 << 28;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

size_t gptq2d_tree_verify_workspace_size(int64_t seqs, int width, int64_t vocab) {
  if (bad_sizes(seqs, width, vocab) || seqs == 0) return 0;
  return space_of(seqs, width, vocab).all;
}

gptq2d_status gptq2d_tree_verify(int64_t seqs, int width, int64_t vocab, gptq2d_dtype dt, const void* X, int64_t ldx,
                                 float scale, const int64_t* tokens, const int32_t* parents, const int32_t* drafts,
                                 const float* uniform, const void* D, int64_t ldd, float draft_scale,
                                 const float* draft_lse, int32_t* path, int32_t* count, int64_t* next, float* logprob,
                                 void* workspace, size_t ws_bytes, void* stream) {
  if (bad_sizes(seqs, width, vocab)) return refuse("seqs must lie in [0, 65535], width in [1, 64], vocab in [1, 2^28]");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (!(scale > 0.0f) || !isfinite(scale)) return refuse("scale must be positive and finite");
  if (D && (!(draft_scale > 0.0f) || !isfinite(draft_scale))) return refuse("draft_scale must be positive and finite");
  if (D && !draft_lse) return refuse("D needs draft_lse");
  if (D && !uniform) return refuse("drawn drafts need random numbers");
  if (seqs == 0) return GPTQ2D_OK;
  if (!X || !tokens || !path || !count || !next || !logprob) return refuse("X, tokens, path, count, next or logprob is NULL");
  if (ldx < vocab || (D && ldd < vocab)) return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  if (!aligned(X, es) || !aligned(D, es) || !aligned(tokens, 8) || !aligned(parents, 4) || !aligned(drafts, 4) ||
      !aligned(uniform, 4) || !aligned(draft_lse, 4) || !aligned(path, 4) || !aligned(count, 4) || !aligned(next, 8) ||
      !aligned(logprob, 4))
    return refuse("an argument is not aligned to its elements");
  const Space sp = space_of(seqs, width, vocab);
  if (!workspace || ws_bytes < sp.all) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  char* w = (char*)workspace;
  const int64_t per = last_per(vocab);
  VerifyArgs v = {seqs, width, (int)vocab, row_parts(seqs * width, vocab), (int)ceil_div(vocab + 7, per), (int)per, X, ldx,
                  scale, tokens, parents, drafts, uniform, D, ldd, draft_scale, draft_lse, path, count, next, logprob,
                  (Part*)(w + sp.part), (Last*)(w + sp.last), (State*)(w + sp.state)};
  const hipStream_t s = (hipStream_t)stream;
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    if (width > 1) hipLaunchKernelGGL(k_rows<T>, dim3((unsigned)(seqs * width * v.parts)), dim3(kThreads), 0, s, v);
    hipLaunchKernelGGL(k_walk<T>, dim3((unsigned)seqs), dim3(kWalk), 0, s, v);
    hipLaunchKernelGGL(k_last<T>, dim3((unsigned)(seqs * v.chunks)), dim3(kThreads), 0, s, v);
    hipLaunchKernelGGL(k_next<T>, dim3((unsigned)seqs), dim3(kThreads), 0, s, v);
  });
  return launched("gptq2d_tree_verify");
}

}  // extern "C"
