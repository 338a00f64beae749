// Keys and values of attention in eight bits: written to the pages of a cache
// with one scale for each token and head, and read back.
//
// A page holds page_size tokens head by head: codes [page][head][token][dim],
// scales [page][head][token]. A head's tokens are adjacent, so the attention
// that reads one head of a page reads whole lines.
#include <type_traits>

#include "codes.hpp"

namespace g2d {
namespace {

struct CacheArgs {
  int64_t tokens;
  int heads, dim;
  const int64_t* slots;
  uint32_t total, page, magic;  // slots, slots per page, floor(2^32 / page) + 1
  void *K, *V;                  // the vectors: tokens x (heads dim)
  int64_t ldk, ldv;
  uint8_t *KC, *VC;
  float *KS, *VS;
  bool wide;
};

// a vector's place in the cache, or -1 for a slot that is none (without branches:
// the loads of several are not to wait for one another)
__device__ __forceinline__ int64_t place(const CacheArgs& a, int64_t s, int head) {
  const bool none = s < 0 || s >= a.total;
  const uint32_t slot = none ? 0 : (uint32_t)s;
  uint32_t q = __umulhi(slot, a.magic);  // slot < 2^31: at most one too large
  q -= q * a.page > slot;
  const int64_t at = ((int64_t)q * a.heads + head) * a.page + (slot - q * a.page);
  return none ? -1 : at;
}

// L lanes hold a vector, eight values each (dim <= 8 L): one read, the largest
// magnitude over the lanes, one write. Bound by its bytes: 32768 tokens x 8 heads x
// 128 from 16 bits 52 us, 3.9 TB/s read and written; 64 tokens 2.6 us.
template <class T, int L, bool INT8>
__global__ __launch_bounds__(256) void k_append(CacheArgs a) {
  const int lane = threadIdx.x % L, head = blockIdx.y;
  const int64_t token = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int64_t at = token < a.tokens ? place(a, a.slots[token], head) : -1;
  const bool active = at >= 0 && 8 * lane < a.dim;
  const bool key = blockIdx.z == 0;
  float x[8];
  const T* p = (const T*)(key ? a.K : a.V) + token * (key ? a.ldk : a.ldv) + (int64_t)head * a.dim + 8 * lane;
  load8(p, a.wide && active, active ? 8 : 0, x, (const T*)(key ? a.K : a.V));
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, mag(x[i]));
  m = group_max<L>(m);
  const float s = block_scale(m, 1.0f / (INT8 ? kTopInt8 : kTopE4M3), false);
  const u2 q = code8<INT8>(x, 1.0f / s, bad_amax(m));
  if (!active) return;
  *(u2*)((key ? a.KC : a.VC) + at * a.dim + 8 * lane) = q;
  if (lane == 0) (key ? a.KS : a.VS)[at] = s;
}

// L lanes hold a vector, sixteen values each (dim <= 16 L), and four vectors one
// after the other: slot, codes and value wait for one another, so that the reads
// of four of them are on their way at once (32768 tokens x 8 heads x 128, int8 to
// 16 bits: 92 us one by one with eight values a lane, now 33.5 us, 6.1 TB/s, the
// codes partly from the last-level cache; 64 tokens 3.7 us, of which the chain of
// three reads is most: with one vector a lane they take 2.8 us, but the call, which
// a launch's latency bounds, no less).
template <class T, int L, bool INT8>
__global__ __launch_bounds__(256) void k_read(CacheArgs a) {
  constexpr int V = 4, P = 256 / L;  // vectors of a lane, of a work group at a time
  const int lane = threadIdx.x % L;
  const bool key = blockIdx.y == 0;
  const uint32_t all = (uint32_t)(a.tokens * a.heads), first = blockIdx.x * (P * V) + threadIdx.x / L;
  if (16 * lane >= a.dim) return;
  int64_t at[V];
  u4 q[V];
  float s[V];
  uint32_t token[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    token[v] = min(first + v * P, all - 1) / (uint32_t)a.heads;
    at[v] = a.slots[token[v]];
  }
#pragma unroll
  for (int v = 0; v < V; ++v) at[v] = place(a, at[v], (int)(min(first + v * P, all - 1) - token[v] * a.heads));
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int64_t from = max(at[v], (int64_t)0);
    q[v] = *(const u4*)((key ? a.KC : a.VC) + from * a.dim + 16 * lane);
    s[v] = (key ? a.KS : a.VS)[from];
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t vec = first + v * P;
    if (vec >= all) break;
    T* p = (T*)(key ? a.K : a.V) + token[v] * (key ? a.ldk : a.ldv) + (int64_t)(vec - token[v] * a.heads) * a.dim + 16 * lane;
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const h2 lo = halves<INT8, false>(q[v][i]), hi = halves<INT8, true>(q[v][i]);
      x[4 * i] = (float)lo[0] * s[v], x[4 * i + 1] = (float)lo[1] * s[v];
      x[4 * i + 2] = (float)hi[0] * s[v], x[4 * i + 3] = (float)hi[1] * s[v];
    }
    if (at[v] < 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.0f;
    }
    store8(p, a.wide, 8, x);
    store8(p + 8, a.wide, 8, x + 8);
  }
}

// lanes of a vector when writing (8 values each) and reading (16)
template <class T, int L, bool INT8>
void launch(const CacheArgs& a, bool append, hipStream_t s) {
  if (append)
    hipLaunchKernelGGL((k_append<T, L, INT8>), dim3((unsigned)ceil_div(a.tokens, 256 / L), a.heads, 2), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_read<T, L / 2, INT8>), dim3((unsigned)ceil_div(a.tokens * a.heads, 4 * 256 / (L / 2)), 2),
                       dim3(256), 0, s, a);
}

template <class T, bool INT8>
void launch_dim(const CacheArgs& a, bool append, hipStream_t s) {
  if (a.dim <= 32) launch<T, 4, INT8>(a, append, s);
  else if (a.dim <= 64) launch<T, 8, INT8>(a, append, s);
  else if (a.dim <= 128) launch<T, 16, INT8>(a, append, s);
  else launch<T, 32, INT8>(a, append, s);
}

gptq2d_status cache_call(int64_t tokens, int heads, int dim, gptq2d_dtype dt, void* K, int64_t ldk, void* V,
                         int64_t ldv, const int64_t* slots, gptq2d_code code, int64_t pages, int page_size, void* KC,
                         void* VC, float* KS, float* VS, bool append, hipStream_t s, const char* name) {
  const gptq2d_status st = check_cache(heads, dim, code, pages, page_size, KC, VC, KS, VS);
  if (st != GPTQ2D_OK) return st;
  if (tokens < 0 || tokens > (int64_t)1 << 26 || tokens * heads > (int64_t)1 << 30)
    return refuse("tokens must lie in [0, 2^26], and tokens x heads in 2^30");
  if (!narrow_dtype(dt)) return refuse("bad dtype");
  if (tokens == 0) return GPTQ2D_OK;
  if (!K || !V || !slots) return refuse("K, V or slots are NULL");
  if (ldk < (int64_t)heads * dim || ldv < (int64_t)heads * dim) return refuse("leading dimension too small");
  const size_t es = elem_size(dt);
  if (!aligned(K, es) || !aligned(V, es) || !aligned(slots, 8)) return refuse("K, V or slots are not aligned");
  CacheArgs a = {tokens, heads, dim, slots, (uint32_t)(pages * page_size), (uint32_t)page_size,
                 (uint32_t)(((uint64_t)1 << 32) / page_size + 1), K, V, ldk, ldv, (uint8_t*)KC, (uint8_t*)VC, KS, VS,
                 wide_rows(K, ldk, es) && wide_rows(V, ldv, es)};
  with_type(dt, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (code == GPTQ2D_INT8)
      launch_dim<T, true>(a, append, s);
    else
      launch_dim<T, false>(a, append, s);
  });
  return launched(name);
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

gptq2d_status gptq2d_cache_append(int64_t tokens, int heads, int dim, gptq2d_dtype dt, const void* K, int64_t ldk,
                                  const void* V, int64_t ldv, const int64_t* slots, gptq2d_code code, int64_t pages,
                                  int page_size, void* KC, void* VC, float* KS, float* VS, void* stream) {
  return cache_call(tokens, heads, dim, dt, (void*)K, ldk, (void*)V, ldv, slots, code, pages, page_size, KC, VC, KS, VS,
                    true, (hipStream_t)stream, "gptq2d_cache_append");
}

gptq2d_status gptq2d_cache_read(int64_t tokens, int heads, int dim, gptq2d_dtype dt, const int64_t* slots,
                                gptq2d_code code, int64_t pages, int page_size, const void* KC, const void* VC,
                                const float* KS, const float* VS, void* K, int64_t ldk, void* V, int64_t ldv,
                                void* stream) {
  return cache_call(tokens, heads, dim, dt, K, ldk, V, ldv, slots, code, pages, page_size, (void*)KC, (void*)VC,
                    (float*)KS, (float*)VS, false, (hipStream_t)stream, "gptq2d_cache_read");
}

}  // extern "C"
