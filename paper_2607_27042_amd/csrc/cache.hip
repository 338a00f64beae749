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

// the vector's place in the cache, or -1 for a slot that is none
__device__ __forceinline__ int64_t place(const CacheArgs& a, int64_t token, int head) {
  const int64_t s = a.slots[token];
  if (s < 0 || s >= a.total) return -1;
  const uint32_t slot = (uint32_t)s;
  uint32_t q = __umulhi(slot, a.magic);  // slot < 2^31: at most one too large
  if (q * a.page > slot) --q;
  return ((int64_t)q * a.heads + head) * a.page + (slot - q * a.page);
}

// L lanes hold a vector, eight values each (dim <= 8 L)
template <class T, int L, bool INT8>
__global__ __launch_bounds__(256) void k_append(CacheArgs a) {
  const int lane = threadIdx.x % L, head = blockIdx.y;
  const int64_t token = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int64_t at = token < a.tokens ? place(a, token, head) : -1;
  const bool active = at >= 0 && 8 * lane < a.dim;
  const bool key = blockIdx.z == 0;
  float x[8];
  const T* p = (const T*)(key ? a.K : a.V) + token * (key ? a.ldk : a.ldv) + (int64_t)head * a.dim + 8 * lane;
  load8(p, a.wide && active, active ? 8 : 0, x);
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

template <class T, int L, bool INT8>
__global__ __launch_bounds__(256) void k_read(CacheArgs a) {
  const int lane = threadIdx.x % L, head = blockIdx.y;
  const int64_t token = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (token >= a.tokens || 8 * lane >= a.dim) return;
  const bool key = blockIdx.z == 0;
  const int64_t at = place(a, token, head);
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  if (at >= 0) {
    const u2 q = *(const u2*)((key ? a.KC : a.VC) + at * a.dim + 8 * lane);
    const float s = (key ? a.KS : a.VS)[at];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const h2 lo = halves<INT8, false>(q[i]), hi = halves<INT8, true>(q[i]);
      x[4 * i] = (float)lo[0] * s, x[4 * i + 1] = (float)lo[1] * s;
      x[4 * i + 2] = (float)hi[0] * s, x[4 * i + 3] = (float)hi[1] * s;
    }
  }
  store8((T*)(key ? a.K : a.V) + token * (key ? a.ldk : a.ldv) + (int64_t)head * a.dim + 8 * lane, a.wide, 8, x);
}

template <class T, int L, bool INT8>
void launch(const CacheArgs& a, bool append, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(a.tokens, 256 / L), a.heads, 2);
  if (append)
    hipLaunchKernelGGL((k_append<T, L, INT8>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_read<T, L, INT8>), grid, dim3(256), 0, s, a);
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
  if (tokens < 0 || tokens > (int64_t)1 << 26) return refuse("tokens must lie in [0, 2^26]");
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
