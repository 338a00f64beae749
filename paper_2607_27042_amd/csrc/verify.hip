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
constexpr int kVec = 16;                 // elements of a thread and step in the first pass
constexpr int kChunk = kThreads * kVec;  // of a work group
// and step in 64-bit passes
constexpr int kFew = 4;
constexpr int kFewChunk = kThreads * kFew;
constexpr int kTurn = 4;  // steps whose loads are on their way at once
constexpr int kMaxWidth = 64;
constexpr int kMaxParts = 64;            // of a row
constexpr float kLog2E = 1.44269504088896341f;
constexpr double kLog2E64 = 1.4426950408889634;

// 2^t to about 1e-13 of itself for t in [-1000, 1000], 0 or infinity down to -5000 and up to 5000, from a
// table of 2^(k / 256). t is split at the nearest multiple of 1 / 256, which adding 1.5 2^44
// leaves in the low bits; the rest, |f| <= 1 / 512, needs four terms of its series. The 64-bit
// terms of the last rows are most of what their pass costs: 64 rows of 128000 with as many
// of the drafts 19.4 us, 18.7 with the scaled maximum rounded before it is taken off. (There, with
// a comparison in place of the lower bound and the exponent's own instruction 20.5, with a
// polynomial of degree 8 on |f| <= 1 / 2 and no table 22.)
struct Powers {
  double at[256];
  __device__ __forceinline__ void fill() {  // by the first 256 threads; a barrier follows
    if (threadIdx.x < 256) at[threadIdx.x] = exp2((double)threadIdx.x * 0x1p-8);
  }
  __device__ __forceinline__ double of(double t) const {
    const double big = t + 0x1.8p44, f = t - (big - 0x1.8p44);
    const uint32_t k = __builtin_bit_cast(u2, big)[0];
    double p = 0.05550410866482158;
    p = fma(p, f, 0.2402265069591007);
    p = fma(p, f, 0.6931471805599453);
    p *= f;
    const double e = at[k & 255];
    return __builtin_amdgcn_ldexp(fma(e, p, e), (int32_t)k >> 8);
  }
};

// Across a wave without LDS, whose answers would take longer than all else in passes of a
// few elements a lane: a value moved by a lane pattern, sums of all lanes and of those up
// to the lane, the value of one lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {  // 0 where the pattern gives none
  const u2 b = __builtin_bit_cast(u2, x);
  return __builtin_bit_cast(double, u2{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[0], CTRL, ROWS, 0xf, true),
                                       (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[1], CTRL, ROWS, 0xf, true)});
}
__device__ __forceinline__ double sum_upto(double x) {
  x += moved<0x111, 0xf>(x);  // rows of 16: 1, 2, 4, 8 lanes up
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);  // the last of rows 0 and 2 to the rows after them
  x += moved<0x143, 0xc>(x);  // the last of the first half to the second
  return x;
}
__device__ __forceinline__ double at_lane(double x, int lane) {
  const u2 b = __builtin_bit_cast(u2, x);
  return __builtin_bit_cast(double, u2{(uint32_t)__builtin_amdgcn_readlane((int)b[0], lane),
                                       (uint32_t)__builtin_amdgcn_readlane((int)b[1], lane)});
}
__device__ __forceinline__ double wave_sum(double x) { return at_lane(sum_upto(x), 63); }
// a float as a number that orders alike (NaN as -inf), and back
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x + 0.0f : -INFINITY);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }
// the largest of all lanes, and the lowest place of those that have it
__device__ __forceinline__ void wave_top(float& x, int& at) {
  const uint32_t mine = order_of(x), top = group_max<64>(mine);
  at = (int)~group_max<64>(mine == top ? ~(uint32_t)at : 0);
  x = value_of(top);
}

// of a part of a row: its largest logit, the lowest token that has it, and sums
// relative to it
struct alignas(16) Part {
  float m;
  int32_t at;
  double sum;
};
// of a part of the last row; m, sum: as above, left: the sum of r
struct alignas(16) Last {
  double m, sum, left, less;  // of drawn drafts: Residue's over and less
  int32_t at, unused[3];
};
// what the scan ends with
struct alignas(16) State {
  int32_t node;      // -1: none
  int32_t residual;  // r is less than p
  uint64_t gone;     // rejected tokens of the node
  double beta, m, sum;  // drawn drafts, rejected: beta, the row's largest logit and its sum
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
  // e^(a (x - m)) and e^(ad d - lse); of -inf both are 0. Differences first (a d is exact): with m
  // a log2(e) rounded before x was taken from it, the largest logit's own term would be 1 only as
  // long as m a is below 2^50 or so.
  __device__ __forceinline__ double p2(const Powers& of, float x, double m) const {
    return of.of(fmax(((double)x - m) * ((double)a * kLog2E64), -5000.0));  // (NaN: 0)
  }
  __device__ __forceinline__ double q2(const Powers& of, float d, double lse) const {
    return of.of(fmin(fmax(fma((double)d, (double)ad, -lse) * kLog2E64, -5000.0), 5000.0));
  }
};

// Sums for a drawn draft's residue over some terms f = e^(a (x - m)): of f, and of f and beta
// q where p > beta q. The sum of max(p - beta q, 0) is over / all - less, with `all` of the
// whole row, which is known only afterwards; which terms are over is told by a sum that is off by
// 1e-7, what matters only for terms as near to zero as that.
struct Residue {
  double all, over, less;
  __device__ __forceinline__ void add(double f, double by, double bq) {
    const bool in = f * by > bq;
    all += f;
    if (in) {  // (a branch: choosing the terms takes four instructions more than it does)
      over += f, less += bq;
      asm volatile("" : "+v"(over));
    }
  }
};

__device__ __forceinline__ int drafted(const VerifyArgs& v, int64_t seq) {
  return v.drafts ? min(max(v.drafts[seq], 0), v.width) : v.width;
}
__device__ __forceinline__ int parent_of(const VerifyArgs& v, int64_t seq, int t) {
  if (!v.parents) return t - 1;
  const int p = v.parents[seq * v.width + t];
  return p >= 0 && p < t ? p : -1;
}

// device memory (which the compiler does not see of every pointer here; what it takes for
// any memory it loads in order with LDS)
#define G2D_GLOBAL __attribute__((address_space(1)))

// N elements behind a boundary of as many bytes (16 at most), as they are loaded
template <class T, int N>
struct Raw {
  static constexpr int W = N * sizeof(T) < 16 ? N : 16 / sizeof(T);
  typedef uint32_t V __attribute__((ext_vector_type(W * sizeof(T) / 4)));
  typedef T E __attribute__((ext_vector_type(W)));
  V p[N / W];
  __device__ __forceinline__ void load(const T* x) {
#pragma unroll
    for (int i = 0; i < N / W; ++i) p[i] = *(const G2D_GLOBAL V*)(x + i * W);
  }
  __device__ __forceinline__ void values(float v[N]) const {
#pragma unroll
    for (int i = 0; i < N / W; ++i) {
      const E e = __builtin_bit_cast(E, p[i]);
#pragma unroll
      for (int j = 0; j < W; ++j) v[i * W + j] = (float)e[j];
    }
  }
  static __device__ __forceinline__ bool fits(const T* x, int first, int n) {
    return first >= 0 && first + N <= n && ((uintptr_t)(x + first) & (sizeof(V) - 1)) == 0;
  }
};
// Elements first .. first + N - 1 of a row, those outside [0, n) as -inf.
template <int N, class T>
__device__ __forceinline__ void load_some(const T* x, int first, int n, float v[N]) {
  if (Raw<T, N>::fits(x, first, n)) {
    Raw<T, N> r;
    r.load(x + first);
    r.values(v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (first + i >= 0 && first + i < n) v[i] = (float)((const G2D_GLOBAL T*)x)[first + i];
  }
}
// STEPS steps of kFew elements from e on, a group's steps behind one another
template <class T, int STEPS = kTurn>
struct Turn {
  float z[STEPS][kFew];
  __device__ __forceinline__ void load(const T* x, int e, int n) {
    typedef Raw<T, kFew> R;
    if (R::fits(x, e, n) && R::fits(x, e + (STEPS - 1) * kFewChunk, n)) {
      R r[STEPS];
#pragma unroll
      for (int k = 0; k < STEPS; ++k) r[k].load(x + e + k * kFewChunk);
#pragma unroll
      for (int k = 0; k < STEPS; ++k) r[k].values(z[k]);
    } else {
#pragma unroll
      for (int k = 0; k < STEPS; ++k) load_some<kFew>(x, e + k * kFewChunk, n, z[k]);
    }
  }
};
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
  if (q.sum != 0.0) p.sum += q.sum * exp2(((double)q.m - (double)p.m) * (double)a * kLog2E64);
  return p;
}
__device__ __forceinline__ Part wave_join(Part p, float a) {
  Part q = p;
  wave_top(q.m, q.at);
  q.sum = wave_sum(p.sum != 0.0 ? p.sum * exp2(((double)p.m - (double)q.m) * (double)a * kLog2E64) : 0.0);
  return q;
}

// Largest logit and sum of a part of every row that tokens follow. Bound by its bytes: 64
// chains of 8 over 128000 bf16 28 us for 115 MB, 4.1 TB/s (with 64-bit terms, which would spare
// the last row's own sum, 61 us).
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
  // (never infinite: the largest logit's own term would be that times 0. What is too small then matters
  // for differences below 2^-120.)
  const float a2 = fminf(v.a * kLog2E, 0x1.fffffep127f);
  float m = -INFINITY, sum = 0.0f;
  int at = 0x7fffffff;
  // a thread's elements of a step lie in pieces of 16 bytes, the pieces of a group side by
  // side; the steps inside the row are loaded one ahead
  constexpr int W = 16 / sizeof(T), N = kVec / W;
  const int inner = lead > 0 ? 1 : 0, outer = (v.vocab + lead) / kChunk - 1;
  Raw<T, W> raw[N];
  auto place = [&](int s, int i) { return s * kChunk + i * kThreads * W + t * W - lead; };
  auto ahead = [&](int s) {
    const int c = max(inner, min(s, outer));
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i].load(x + place(c, i));
  };
  if (inner <= outer) ahead(first);
#pragma unroll 1
  for (int s = first; s < last; ++s) {
    float z[kVec];
    if (s >= inner && s <= outer) {
#pragma unroll
      for (int i = 0; i < N; ++i) raw[i].values(z + i * W);
      ahead(s + 1);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) load_some<W>(x, place(s, i), v.vocab, z + i * W);
      if (inner <= outer) ahead(s + 1);
    }
    float top = z[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) top = fmaxf(top, z[i]);
    if (top > m) {
      sum *= __builtin_amdgcn_exp2f((m - top) * a2);
      m = top;
#pragma unroll
      for (int i = kVec - 1; i >= 0; --i) at = z[i] == top ? place(s, i / W) + i % W : at;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += __builtin_amdgcn_exp2f((z[i] - ref) * a2);  // NaN: NaN
  }
  Part p = wave_join(Part{m, at, (double)sum}, v.a);
  if (lane == 0) wave[t >> 6] = p;
  __syncthreads();
  if (t == 0) v.part[blockIdx.x] = join(join(wave[0], wave[1], v.a), join(wave[2], wave[3], v.a), v.a);
}

constexpr int kWalk = 512;

// The scan of a sequence. All waves go through it alike; where a drawn draft is rejected and
// another follows the same token they share a pass over the row, one work group with nothing
// loaded ahead: 16 trees of 13, three followers each, over 128000 bf16 126 us with 2.9 tokens
// kept and 195 with 1.9, over 50257 f16 50; a chain, which has no such pass, 7.7.
template <class T>
__global__ __launch_bounds__(kWalk) void k_walk(VerifyArgs v) {
  __shared__ Part rows[kMaxWidth];
  __shared__ Residue sums[kWalk / 64];
  __shared__ Powers powers;
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
  if (v.D) powers.fill();
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
    p = exp2(z * kLog2E64) / r.sum;
    lp = (float)(z - log(r.sum));
    if (!(r.sum > 0.0)) lp = __uint_as_float(0x7fc00000u), p = (double)lp;
    if (v.D && ok) q = exp2(((double)(float)D[parent * v.ldd + token] * (double)v.ad - (double)dlse[parent]) * kLog2E64);
    best = p == p && token == r.at;
  }
  const double u = v.u && in ? (double)v.u[seq * v.width + lane] : 0.0;
  auto of = [&](double x, int from) { return at_lane(x, from); };
  int cur = n > 0 ? 0 : -1, kept = n > 0 ? 1 : 0;
  int way = lane == 0 && n > 0 ? 0 : -1;  // lane i: the i-th kept token
  double beta = 0.0, M = 1.0, gone_p = 0.0;
  uint64_t gone = 0;
  // the sum of max(p - beta q, 0) of the current row
  auto remaining = [&]() {
    const T *x = X + cur * v.ldx, *d = D + cur * v.ldd;
    const int lead = lead_of(x);
    const double top = (double)rows[cur].m, by = 1.0 / rows[cur].sum, lse = (double)dlse[cur];
    Residue r{};
#pragma unroll 1
    for (int e = t * kFew - lead; e < v.vocab; e += kWalk * kFew) {
      float z[kFew], y[kFew];
      load_some<kFew>(x, e, v.vocab, z);
      load_some<kFew>(d, e, v.vocab, y);
#pragma unroll
      for (int i = 0; i < kFew; ++i) r.add(v.p2(powers, z[i], top), by, beta * v.q2(powers, y[i], lse));
    }
    r = Residue{wave_sum(r.all), wave_sum(r.over), wave_sum(r.less)};
    __syncthreads();
    if (lane == 0) sums[w] = r;
    __syncthreads();
    r = Residue{};
    for (int i = 0; i < kWalk / 64; ++i) r.all += sums[i].all, r.over += sums[i].over, r.less += sums[i].less;
    return fmax(r.over / r.all - r.less, 0.0);
  };
  while (cur >= 0) {
    // (what is no token was not drawn from q: that it does not pass says nothing of the others)
    const uint64_t children = __ballot(parent == cur && token >= 0 && token < v.vocab);
    int taken = -1;
    for (uint64_t left = children; left != 0; left &= left - 1) {
      const int c = __builtin_ctzll(left);
      const double pc = of(p, c);
      if (!v.u) {
        if (__ballot(best) >> c & 1) taken = c;
      } else if (v.D) {
        if (gone != 0) M = remaining();
        const double qc = of(q, c);
        if (of(u, c) * M * qc < pc - beta * qc) taken = c;
        else beta += M;
      } else {
        const int64_t mine = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(token >> 32), c) << 32 |
                                       (uint32_t)__builtin_amdgcn_readlane((int)token, c));
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
    gone = 0, beta = 0.0, M = 1.0, gone_p = 0.0;
  }
  const bool residual = v.u && gone != 0;
  if (w == 0) {
    if (in) {
      v.path[seq * v.width + lane] = way;
      if (lane > 0) v.logprob[seq * v.width + lane] = lp;
    }
    if (lane == 0) {
      v.count[seq] = kept;
      v.state[seq] = State{cur, residual, gone, beta, residual ? (double)rows[cur].m : 0.0, residual ? rows[cur].sum : 0.0};
    }
  }
}

// The tokens of the state's rejected drafts that lie in [first, first + per) of the row.
struct Gone {
  int token[kMaxWidth];
  int n;
};
__device__ __forceinline__ void find_gone(const VerifyArgs& v, const State& s, int64_t seq, int first, int end, Gone& g) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const int64_t token = s.gone >> lane & 1 ? v.tokens[seq * v.width + lane] : -1;
    const bool here = token >= max(first, 0) && token < end;
    const uint64_t all = __ballot(here);
    if (here) g.token[__popcll(all & ((1ull << lane) - 1))] = (int)token;
    if (lane == 0) g.n = __popcll(all);
  }
}

__device__ __forceinline__ void without(const Gone& g, int e, double f[kFew]) {
#pragma unroll 1
  for (int k = 0; k < g.n; ++k)
#pragma unroll
    for (int i = 0; i < kFew; ++i) f[i] = e + i == g.token[k] ? 0.0 : f[i];
}
// Sums of one part of the last row, STEPS steps at once.
template <class T, int STEPS>
__global__ __launch_bounds__(kThreads) void k_last(VerifyArgs v) {
  __shared__ Gone gone;
  __shared__ float tops[kThreads / 64];
  __shared__ Residue sums[kThreads / 64];
  __shared__ Powers powers;
  __shared__ int first[kThreads / 64];
  const int64_t seq = blockIdx.x / (uint32_t)v.chunks;
  const int chunk = blockIdx.x - (int)seq * v.chunks, t = threadIdx.x, lane = t & 63;
  const State s = v.state[seq];
  if (s.node < 0) return;
  const int64_t row = seq * v.width + s.node;
  const T *x = (const T*)v.X + row * v.ldx, *d = (const T*)v.D + row * v.ldd;
  const int lead = lead_of(x);
  const int begin = chunk * v.per - lead, end = min(begin + v.per, v.vocab);
  const bool drawn = s.residual && v.D;
  const float ld = drawn ? v.dlse[row] : 0.0f;
  find_gone(v, s, seq, begin, end, gone);
  powers.fill();
  const bool once = v.per <= STEPS * kFewChunk;  // all of the part in registers
  Turn<T, STEPS> turn, other;
  if (once) turn.load(x, begin + t * kFew, end);
  if (once && drawn) other.load(d, begin + t * kFew, end);
  float top = -INFINITY;
  int at = 0x7fffffff;
  bool bad = false;
  if (!drawn) {
    for (int e = begin + t * kFew; e < end; e += STEPS * kFewChunk) {
      if (e > begin + t * kFew || !once) turn.load(x, e, end);
#pragma unroll
      for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int i = 0; i < kFew; ++i)
          if (turn.z[k][i] > top) top = turn.z[k][i], at = e + k * kFewChunk + i;
    }
    wave_top(top, at);
    if (lane == 0) tops[t >> 6] = top, first[t >> 6] = at;
  }
  __syncthreads();
  if (!drawn)
    for (int k = 0; k < kThreads / 64; ++k)
      if (tops[k] > top || (tops[k] == top && first[k] < at)) top = tops[k], at = first[k];
  // drawn drafts: the row's own largest, so that its terms can be told from q
  const double m = drawn ? s.m : top == -INFINITY ? 0.0 : (double)top;
  const bool some = s.residual && !v.D && gone.n > 0;
  const double by = drawn ? 1.0 / s.sum : 0.0, lse = (double)ld;
  Residue r{};
  for (int e0 = begin + t * kFew; e0 < end; e0 += STEPS * kFewChunk) {
    if (!once) turn.load(x, e0, end);
    if (drawn && !once) other.load(d, e0, end);
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      if (e0 - t * kFew + k * kFewChunk >= end) break;
      double f[kFew];
#pragma unroll
      for (int i = 0; i < kFew; ++i) {
        const float z = turn.z[k][i];
        f[i] = v.p2(powers, z, m);
        bad |= z != z || z == INFINITY;
        if (drawn) r.add(f[i], by, s.beta * v.q2(powers, other.z[k][i], lse));
        else r.all += f[i];
      }
      if (some) {
        without(gone, e0 + k * kFewChunk, f);
#pragma unroll
        for (int i = 0; i < kFew; ++i) r.over += f[i];
      }
    }
  }
  if (bad) r.all = NAN;
  if (!drawn && !some) r.over = r.all;
  r = Residue{wave_sum(r.all), wave_sum(r.over), wave_sum(r.less)};
  if (lane == 0) sums[t >> 6] = r;
  __syncthreads();
  if (t == 0) {
    r = Residue{};
    for (int k = 0; k < kThreads / 64; ++k) r.all += sums[k].all, r.over += sums[k].over, r.less += sums[k].less;
    v.last[blockIdx.x] = Last{top == -INFINITY && !drawn ? -INFINITY : m, r.all, r.over, r.less, at, {}};
  }
}

// The next token of a sequence: its part of the row, then its place there, STEPS steps at
// once: a part of 4096 waits once for memory and for the other waves' sums (64 rows of 128000
// 7.8 us, step by step 10.0; parts of one step 3.7 us, as four 6.8).
template <class T, int STEPS>
__global__ __launch_bounds__(kThreads) void k_next(VerifyArgs v) {
  __shared__ Gone gone;
  __shared__ double sums[STEPS][kThreads / 64];
  __shared__ int found[kThreads / 64];
  __shared__ float logit;
  __shared__ Powers powers;
  const int64_t seq = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  // (parts of a sequence without a row are not what they were: they are not used)
  Last l{-INFINITY, 0.0, 0.0, 0.0, 0x7fffffff, {}};
  if (lane < v.chunks) l = v.last[seq * v.chunks + lane];
  const float u32 = v.u ? v.u[seq * v.width] : 0.0f;
  State s = v.state[seq];
  if (s.node < 0) {
    if (t == 0) v.next[seq] = -1, v.logprob[seq * v.width] = 0.0f;
    return;
  }
  const int64_t row = seq * v.width + s.node;
  const T *x = (const T*)v.X + row * v.ldx, *d = (const T*)v.D + row * v.ldd;
  bool drawn = s.residual && v.D;
  float best = (float)l.m;  // (they are 32-bit numbers)
  int at = l.at;
  if (!drawn) wave_top(best, at);
  else best = (float)s.m;
  const double f = drawn || best == -INFINITY ? 1.0 : exp2((l.m - (double)best) * ((double)v.a * kLog2E64));
  const double total = wave_sum(l.sum * f);
  if (!(total > 0.0)) {  // nothing but -inf, or a NaN or +inf
    if (t == 0) v.next[seq] = -1, v.logprob[seq * v.width] = __uint_as_float(0x7fc00000u);
    return;
  }
  int64_t chosen = at;
  float value = best;  // its logit
  if (v.u) {
    const double u = (double)u32;
    double left = drawn ? fmax(l.left / total - l.less, 0.0) : l.left * f;
    int pick;
    bool known;
#pragma unroll 1
    for (;;) {
      if (s.residual && __ballot(left > 0.0) == 0) {  // nothing is left of p: p itself
        s.residual = 0, drawn = false;
        left = l.sum * f;
      }
      // sums of the parts up to the lane's
      const double upto = sum_upto(left), aim = u * at_lane(upto, 63);
      const uint64_t over = __ballot(upto > aim && left > 0.0), some = __ballot(left > 0.0);
      const int part = over != 0 ? __builtin_ctzll(over) : 63 - __builtin_clzll(some | 1);
      const double before = at_lane(upto - left, part);
      const double pm = drawn ? s.m : at_lane(l.m, part), pf = at_lane(f, part);
      const int lead = lead_of(x);
      const int begin = part * v.per - lead, end = min(begin + v.per, v.vocab);
      const double lse = drawn ? (double)v.dlse[row] : 0.0;
      find_gone(v, s, seq, begin, end, gone);
      powers.fill();
      __syncthreads();
      const double by = 1.0 / total, aim_in = aim - before;
      double past = 0.0;
      int late = -1;  // the last token with something left
      pick = -1;
#pragma unroll 1
      for (int step = begin; step < end; step += STEPS * kFewChunk) {
        Turn<T, STEPS> turn, other;
        turn.load(x, step + t * kFew, end);
        if (drawn) other.load(d, step + t * kFew, end);
        double r[STEPS][kFew], before_in[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          const int e = step + k * kFewChunk + t * kFew;
          double mine = 0.0;
#pragma unroll
          for (int i = 0; i < kFew; ++i) r[k][i] = v.p2(powers, turn.z[k][i], pm);
          if (drawn) {
#pragma unroll
            for (int i = 0; i < kFew; ++i) r[k][i] = fmax(fma(r[k][i], by, -s.beta * v.q2(powers, other.z[k][i], lse)), 0.0);
          } else if (s.residual) {
            without(gone, e, r[k]);
          }
#pragma unroll
          for (int i = 0; i < kFew; ++i) {
            r[k][i] *= pf;
            mine += r[k][i];
            if (r[k][i] > 0.0) late = e + i;
          }
          const double in = sum_upto(mine);
          before_in[k] = in - mine;
          if (lane == 63) sums[k][w] = in;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          double sum = past + before_in[k];
          for (int i = 0; i < kThreads / 64; ++i) {
            const double all = sums[k][i];
            if (i < w) sum += all;
            past += all;
          }
#pragma unroll
          for (int i = 0; i < kFew; ++i) {
            sum += r[k][i];
            if (pick < 0 && r[k][i] > 0.0 && sum > aim_in) pick = step + k * kFewChunk + t * kFew + i;
          }
        }
        // the lowest (of none: -1, as a number without sign the largest)
        pick = (int)~group_max<64>(~(uint32_t)pick);
        if (lane == 0) found[w] = pick;
        __syncthreads();
        for (int k = 0; k < kThreads / 64; ++k) pick = (int)min((uint32_t)pick, (uint32_t)found[k]);
        if (pick >= 0) {  // (the thread that has it has its logit)
#pragma unroll
          for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int i = 0; i < kFew; ++i)
              if (step + k * kFewChunk + t * kFew + i == pick) logit = turn.z[k][i];
          break;
        }
      }
      known = pick >= 0;
      if (pick < 0) {  // the sums' last place: the last one
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) late = max(late, __shfl_xor(late, k));
        __syncthreads();
        if (lane == 0) found[w] = late;
        __syncthreads();
        for (int k = 0; k < kThreads / 64; ++k) pick = max(pick, found[k]);
      }
      __syncthreads();
      if (pick >= 0 || !s.residual) break;
      // what a part has left was the rounding of its sums (p and beta q alike to their last places): without it
      if (lane == part) left = 0.0;
    }
    chosen = pick;
    value = known ? logit : pick >= 0 ? (float)x[pick] : 0.0f;
  }
  if (t == 0) {
    v.next[seq] = chosen;
    v.logprob[seq * v.width] = chosen < 0 ? __uint_as_float(0x7fc00000u)
                                          : (float)(((double)value - (double)best) * (double)v.a - log(total));
  }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// parts of a row for the first pass
int row_parts(int64_t rows, int64_t vocab) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(4096, rows), ceil_div(vocab + 7, kChunk), kMaxParts}));
}
// elements of a part of the last row: parts of whole steps, kMaxParts of them at most
int64_t last_per(int64_t seqs, int64_t vocab) {
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(kMaxParts, ceil_div(2048, seqs)));
  return ceil_div(ceil_div(vocab + 7, parts), kFewChunk) * kFewChunk;
}

struct Space {
  size_t part, last, state, all;
};
Space space_of(int64_t seqs, int width, int64_t vocab) {
  Space s;
  s.part = 0;
  s.last = s.part + up256((size_t)seqs * width * row_parts(seqs * width, vocab) * sizeof(Part));
  s.state = s.last + up256((size_t)seqs * ceil_div(vocab + 7, last_per(seqs, vocab)) * sizeof(Last));
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
  const int64_t per = last_per(seqs, vocab);
  VerifyArgs v = {seqs, width, (int)vocab, row_parts(seqs * width, vocab), (int)ceil_div(vocab + 7, per), (int)per, X, ldx,
                  scale, tokens, parents, drafts, uniform, D, ldd, draft_scale, draft_lse, path, count, next, logprob,
                  (Part*)(w + sp.part), (Last*)(w + sp.last), (State*)(w + sp.state)};
  const hipStream_t s = (hipStream_t)stream;
  with_type(dt, [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    if (width > 1) hipLaunchKernelGGL(k_rows<T>, dim3((unsigned)(seqs * width * v.parts)), dim3(kThreads), 0, s, v);
    hipLaunchKernelGGL(k_walk<T>, dim3((unsigned)seqs), dim3(kWalk), 0, s, v);
    auto end = [&](auto steps) {
      constexpr int STEPS = decltype(steps)::value;
      hipLaunchKernelGGL((k_last<T, STEPS>), dim3((unsigned)(seqs * v.chunks)), dim3(kThreads), 0, s, v);
      hipLaunchKernelGGL((k_next<T, STEPS>), dim3((unsigned)seqs), dim3(kThreads), 0, s, v);
    };
    if (per == kFewChunk) end(std::integral_constant<int, 1>());
    else end(std::integral_constant<int, kTurn>());
  });
  return launched("gptq2d_tree_verify");
}

}  // extern "C"
