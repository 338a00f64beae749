// Pages of the eight-bit cache between two steps of serving: the kept tokens of a
// drafted tree moved to where the next step expects them, page tables of sequences
// that were forked, cut, freed or have grown, and the copies of pages that these ask
// for. The caches of a model's layers share their tables, so a call does all layers.
#include <algorithm>

#include "codes.hpp"

namespace g2d {
namespace {

// ---------------------------------------------------------------------------
// vectors and pages moved
// ---------------------------------------------------------------------------

constexpr int kLayers = 96;  // of a launch: what its arguments have room for

struct Layers {
  uint8_t* code[kLayers][2];  // KC, VC
  float* scale[kLayers][2];   // KS, VS
};

struct CommitArgs {
  int64_t vectors;  // seqs heads
  int heads, dim, width, layers;
  uint32_t page, magic;  // tokens of a page, floor(2^32 / page) + 1
  int64_t pages;
  const int32_t* table;
  int64_t ldt, table_width;
  const int32_t *context, *path;
  Layers at;
};

// slot of a sequence's position, or -1
__device__ __forceinline__ int64_t slot_of(const CommitArgs& a, int64_t seq, int64_t pos) {
  if (pos < 0 || pos >= (int64_t)0x7fffffff) return -1;
  uint32_t q = __umulhi((uint32_t)pos, a.magic);  // pos < 2^31: at most one too large
  q -= q * a.page > (uint32_t)pos;
  if (q >= a.table_width) return -1;
  const int32_t p = a.table[seq * a.ldt + q];
  return p < 0 || p >= a.pages ? -1 : (int64_t)p * a.page + ((uint32_t)pos - q * a.page);
}

// A wave moves one head's vectors of one sequence in one layer, L lanes a vector. A
// position is written by the entry of its own number, and read by that or an earlier
// one (path[i] >= i): so all reads of a turn come before its writes, and turns may
// follow one another.
template <int L>
__global__ __launch_bounds__(256) void k_commit(CommitArgs a) {
  constexpr int P = 64 / L;
  const int lane = threadIdx.x & 63, l = lane % L, layer = blockIdx.y;
  const int64_t vec = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (vec >= a.vectors) return;
  const int64_t seq = vec / a.heads;
  const int head = (int)(vec - seq * a.heads);
  const int64_t context = a.context[seq];
  const int32_t mine = lane < a.width ? a.path[seq * a.width + lane] : -1;
  const bool moves = mine > lane && mine < a.width;
  uint64_t todo = __ballot(moves);
  if (todo == 0) return;
  const int end = 64 - __builtin_clzll(todo);
  uint8_t *const kc = a.at.code[layer][0], *const vc = a.at.code[layer][1];
  float *const ks = a.at.scale[layer][0], *const vs = a.at.scale[layer][1];
  for (int i0 = __builtin_ctzll(todo) / P * P; i0 < end; i0 += P) {
    const int i = i0 + lane / L;
    const int32_t from = __shfl(mine, i);
    int64_t src = -1, dst = -1;
    if (todo >> i & 1) src = slot_of(a, seq, context + from), dst = slot_of(a, seq, context + i);
    const bool go = src >= 0 && dst >= 0 && 16 * l < a.dim;
    // [page][head][token]
    auto place = [&](int64_t slot) {
      const int64_t p = slot / a.page;
      return (p * a.heads + head) * a.page + (slot - p * a.page);
    };
    const int64_t s = go ? place(src) : 0, d = go ? place(dst) : 0;
    u4 k{}, v{};
    float fk = 0.0f, fv = 0.0f;
    if (go) {
      k = *(const u4*)(kc + s * a.dim + 16 * l);
      v = *(const u4*)(vc + s * a.dim + 16 * l);
      if (l == 0) fk = ks[s], fv = vs[s];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (go) {
      *(u4*)(kc + d * a.dim + 16 * l) = k;
      *(u4*)(vc + d * a.dim + 16 * l) = v;
      if (l == 0) ks[d] = fk, vs[d] = fv;
    }
  }
}

struct CopyArgs {
  int heads, dim;
  int64_t pages;
  uint32_t page, pieces;  // 16-byte pieces of a head's codes
  const int32_t* copies;
  Layers at;
};

// A work group copies some pieces of one page's codes in one layer, head by head the
// first tokens; the first group the scales too.
__global__ __launch_bounds__(256) void k_copy(CopyArgs a) {
  const int64_t i = blockIdx.x;
  const int layer = blockIdx.z;
  const int32_t from = a.copies[3 * i], to = a.copies[3 * i + 1];
  const uint32_t n = (uint32_t)min(max(a.copies[3 * i + 2], 0), (int32_t)a.page);
  if (from < 0 || to < 0 || from >= a.pages || to >= a.pages || from == to || n == 0) return;
  const uint32_t some = n * (uint32_t)a.dim / 16, all = some * (uint32_t)a.heads;
  const int64_t size = (int64_t)a.heads * a.page;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    uint8_t* c = a.at.code[layer][t];
    const u4* src = (const u4*)(c + from * size * a.dim);
    u4* dst = (u4*)(c + to * size * a.dim);
    for (uint32_t e = blockIdx.y * 256 + threadIdx.x; e < all; e += gridDim.y * 256) {
      const uint32_t head = e / some;
      const uint32_t at = head * a.pieces + (e - head * some);
      dst[at] = src[at];
    }
    if (blockIdx.y == 0) {
      float* f = a.at.scale[layer][t];
      for (uint32_t e = threadIdx.x; e < n * a.heads; e += 256) {
        const uint32_t head = e / n, at = head * a.page + (e - head * n);
        f[to * size + at] = f[from * size + at];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// page tables
// ---------------------------------------------------------------------------

struct UpdateArgs {
  int64_t rows, old_rows, table_width, pages, page;
  const int32_t* table;
  int64_t ldt;
  const int32_t *length, *source, *want, *held;
  int32_t* out;
  int64_t ldo;
  int32_t *copies, *left;
  // workspace: a mark of each page (0: a row holds it whole, 1 + s: row s is the first
  // of those that end in it, kNobody), the free pages in order, the number of new
  // pages of the rows before each
  uint32_t *mark, *list, *before;
};
constexpr uint32_t kNobody = 0xffffffffu;

struct Row {
  const int32_t* old;
  int64_t whole, end;  // pages that are kept whole, pages that are wanted
  int part;            // tokens in the page after the whole ones
};
__device__ __forceinline__ Row row_of(const UpdateArgs& a, int64_t s) {
  const int64_t from = a.source ? (int64_t)a.source[s] : s;
  const bool any = from >= 0 && from < a.old_rows;
  const int64_t room = a.table_width * a.page;
  const int64_t want = min(max((int64_t)a.want[s], (int64_t)0), room);
  const int64_t kept = any ? min(max((int64_t)a.length[from], (int64_t)0), want) : 0;
  Row r;
  r.old = a.table + (any ? from : 0) * a.ldt;
  r.whole = kept / a.page;
  r.part = (int)(kept - r.whole * a.page);
  r.end = (want + a.page - 1) / a.page;
  return r;
}
__device__ __forceinline__ int32_t named(const UpdateArgs& a, int32_t p) { return p < 0 || p >= a.pages ? -1 : p; }
// whether row s gets a copy of page p, in which what it keeps ends
__device__ __forceinline__ bool copies_page(const UpdateArgs& a, const uint32_t* mark, int64_t s, int32_t p) {
  return p >= 0 && (mark[p] != (uint32_t)s + 1 || (a.held && a.held[p] != 0));
}

__device__ __forceinline__ void mark_row(const UpdateArgs& a, uint32_t* mark, int64_t s, int lane) {
  const Row r = row_of(a, s);
  const int64_t n = r.whole + (r.part > 0);
  for (int64_t j = lane; j < n; j += 64) {
    const int32_t p = named(a, r.old[j]);
    if (p >= 0) atomicMin(&mark[p], j < r.whole ? 0u : (uint32_t)s + 1);
  }
}
__device__ __forceinline__ uint32_t new_pages(const UpdateArgs& a, const uint32_t* mark, int64_t s) {
  const Row r = row_of(a, s);
  const int64_t n = r.whole + (r.part > 0);
  return (uint32_t)(max(r.end - n, (int64_t)0) + (r.part > 0 && copies_page(a, mark, s, named(a, r.old[r.whole]))));
}
__device__ __forceinline__ void write_row(const UpdateArgs& a, const uint32_t* mark, int64_t s, uint32_t free, int lane) {
  const Row r = row_of(a, s);
  const int32_t last = r.part > 0 ? named(a, r.old[r.whole]) : -1;
  const bool copied = r.part > 0 && copies_page(a, mark, s, last);
  const uint32_t first = a.before[s];
  const int64_t kept = r.whole + (r.part > 0 && !copied);  // entries that stay as they were
  for (int64_t j = lane; j < a.table_width; j += 64) {
    int32_t p = -1;
    if (j < kept) {
      p = named(a, r.old[j]);
    } else if (j < r.end) {
      const uint64_t nth = (uint64_t)first + (uint64_t)(j - kept);
      if (nth < free) p = (int32_t)a.list[nth];
    }
    a.out[s * a.ldo + j] = p;
    if (copied && j == r.whole) {
      a.copies[3 * s] = last;
      a.copies[3 * s + 1] = p;
      a.copies[3 * s + 2] = r.part;
    }
  }
  if (!copied && lane < 3) a.copies[3 * s + lane] = lane < 2 ? -1 : 0;
}

// sum of the values before the thread's, of a work group of kScan threads; `all` gets the total
constexpr int kScan = 1024;
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(s, d);
    if (lane >= d) s += o;
  }
  __syncthreads();  // (the last call's sums are read)
  if (lane == 63) waves[w] = s;
  __syncthreads();
  uint32_t b = 0, t = 0;
  for (int i = 0; i < kScan / 64; ++i) {
    const uint32_t x = waves[i];
    if (i < w) b += x;
    t += x;
  }
  all = t;
  return b + s - v;
}

__device__ __forceinline__ void scan_all(const UpdateArgs& a, const uint32_t* mark, uint32_t* waves, uint32_t& free) {
  const int t = threadIdx.x;
  uint32_t need = 0, all;
  for (int64_t s0 = 0; s0 < a.rows; s0 += kScan) {
    const int64_t s = s0 + t;
    const uint32_t b = sum_before(s < a.rows ? new_pages(a, mark, s) : 0, waves, all);
    if (s < a.rows) a.before[s] = need + b;
    need += all;
  }
  free = 0;
  for (int64_t p0 = 0; p0 < a.pages; p0 += 4 * kScan) {
    bool f[4];
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t p = p0 + 4 * t + i;
      f[i] = p < a.pages && mark[p] == kNobody && !(a.held && a.held[p] != 0);
      n += f[i];
    }
    uint32_t at = free + sum_before(n, waves, all);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (f[i]) a.list[at++] = (uint32_t)(p0 + 4 * t + i);
    free += all;
  }
  if (t == 0 && a.left) *a.left = (int32_t)free - (int32_t)need;
}

// All of it in one work group, with the marks in LDS.
constexpr int kOnePages = 32768;
__global__ __launch_bounds__(kScan) void k_update_one(UpdateArgs a) {
  __shared__ uint32_t mark[kOnePages];
  __shared__ uint32_t waves[kScan / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int p = threadIdx.x; p < a.pages; p += kScan) mark[p] = kNobody;
  __syncthreads();
  for (int64_t s = w; s < a.rows; s += kScan / 64) mark_row(a, mark, s, lane);
  __syncthreads();
  uint32_t free;
  scan_all(a, mark, waves, free);
  __syncthreads();
  for (int64_t s = w; s < a.rows; s += kScan / 64) write_row(a, mark, s, free, lane);
}

// The same in four launches.
__global__ __launch_bounds__(256) void k_update_clear(UpdateArgs a) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p < a.pages) a.mark[p] = kNobody;
}
__global__ __launch_bounds__(256) void k_update_mark(UpdateArgs a) {
  const int64_t s = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (s < a.rows) mark_row(a, a.mark, s, threadIdx.x & 63);
}
__global__ __launch_bounds__(kScan) void k_update_scan(UpdateArgs a) {
  __shared__ uint32_t waves[kScan / 64];
  uint32_t free;
  scan_all(a, a.mark, waves, free);
  if (threadIdx.x == 0) a.before[a.rows] = free;
}
__global__ __launch_bounds__(256) void k_update_write(UpdateArgs a) {
  const int64_t s = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (s < a.rows) write_row(a, a.mark, s, a.before[a.rows], threadIdx.x & 63);
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t update_bytes(int64_t rows, int64_t pages) {
  return 2 * up256((size_t)pages * 4) + up256((size_t)(rows + 1) * 4);
}

// the layers' tensors [first, first + n) for a launch
gptq2d_status check_layers(int layers, int heads, int dim, int64_t pages, int page_size, void* const* KC, void* const* VC,
                           float* const* KS, float* const* VS) {
  if (layers < 1 || layers > 4096) return refuse("layers must lie in [1, 4096]");
  if (!KC || !VC || !KS || !VS) return refuse("an array of the layers' tensors is NULL");
  for (int i = 0; i < layers; ++i) {
    const gptq2d_status st = check_cache(heads, dim, GPTQ2D_E4M3, pages, page_size, KC[i], VC[i], KS[i], VS[i]);
    if (st != GPTQ2D_OK) return st;
  }
  return GPTQ2D_OK;
}
void take_layers(Layers& at, int first, int n, void* const* KC, void* const* VC, float* const* KS, float* const* VS) {
  for (int i = 0; i < n; ++i) {
    at.code[i][0] = (uint8_t*)KC[first + i], at.code[i][1] = (uint8_t*)VC[first + i];
    at.scale[i][0] = KS[first + i], at.scale[i][1] = VS[first + i];
  }
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

}  // namespace
}  // namespace g2d

using namespace g2d;

extern "C" {

gptq2d_status gptq2d_cache_commit(int layers, int64_t seqs, int width, int heads, int dim, int64_t pages, int page_size,
                                  void* const* KC, void* const* VC, float* const* KS, float* const* VS,
                                  const int32_t* table, int64_t ldt, int64_t table_width, const int32_t* context,
                                  const int32_t* path, void* stream) {
  const gptq2d_status st = check_layers(layers, heads, dim, pages, page_size, KC, VC, KS, VS);
  if (st != GPTQ2D_OK) return st;
  if (seqs < 0 || seqs > 65535 || width < 1 || width > 64) return refuse("seqs must lie in [0, 65535], width in [1, 64]");
  if (seqs == 0) return GPTQ2D_OK;
  if (!table || !context || !path) return refuse("table, context or path is NULL");
  if (table_width < 1 || table_width > (int64_t)1 << 24 || ldt < table_width) return refuse("bad table");
  if (!aligned(table, 4) || !aligned(context, 4) || !aligned(path, 4)) return refuse("an argument is not aligned to its elements");
  CommitArgs a = {seqs * heads, heads, dim, width, 0, (uint32_t)page_size, (uint32_t)(((uint64_t)1 << 32) / page_size + 1),
                  pages, table, ldt, table_width, context, path, {}};
  for (int first = 0; first < layers; first += kLayers) {
    a.layers = std::min(kLayers, layers - first);
    take_layers(a.at, first, a.layers, KC, VC, KS, VS);
    const dim3 grid((unsigned)ceil_div(a.vectors, 4), a.layers);
    if (dim <= 64)
      hipLaunchKernelGGL(k_commit<4>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else if (dim <= 128)
      hipLaunchKernelGGL(k_commit<8>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else
      hipLaunchKernelGGL(k_commit<16>, grid, dim3(256), 0, (hipStream_t)stream, a);
  }
  return launched("gptq2d_cache_commit");
}

gptq2d_status gptq2d_cache_copy(int layers, int64_t count, int heads, int dim, int64_t pages, int page_size,
                                void* const* KC, void* const* VC, float* const* KS, float* const* VS,
                                const int32_t* copies, void* stream) {
  const gptq2d_status st = check_layers(layers, heads, dim, pages, page_size, KC, VC, KS, VS);
  if (st != GPTQ2D_OK) return st;
  if (count < 0 || count > (int64_t)1 << 22) return refuse("count must lie in [0, 2^22]");
  if (count == 0) return GPTQ2D_OK;
  if (!copies) return refuse("copies is NULL");
  if (!aligned(copies, 4)) return refuse("an argument is not aligned to its elements");
  CopyArgs a = {heads, dim, pages, (uint32_t)page_size, (uint32_t)(page_size * dim / 16), copies, {}};
  const int64_t pieces = (int64_t)heads * a.pieces;
  for (int first = 0; first < layers; first += kLayers) {
    const int n = std::min(kLayers, layers - first);
    take_layers(a.at, first, n, KC, VC, KS, VS);
    const dim3 grid((unsigned)count, (unsigned)std::min<int64_t>(ceil_div(pieces, 1024), 64), n);
    hipLaunchKernelGGL(k_copy, grid, dim3(256), 0, (hipStream_t)stream, a);
  }
  return launched("gptq2d_cache_copy");
}

size_t gptq2d_pages_update_workspace_size(int64_t rows, int64_t pages) {
  if (rows < 1 || rows > 65535 || pages < 1 || pages > (int64_t)0x7fffffff / 16) return 0;
  return update_bytes(rows, pages);
}

gptq2d_status gptq2d_pages_update(int64_t rows, int64_t old_rows, int64_t table_width, const int32_t* table, int64_t ldt,
                                  const int32_t* length, const int32_t* source, const int32_t* want, const int32_t* held,
                                  int64_t pages, int page_size, int32_t* out, int64_t ldo, int32_t* copies, int32_t* left,
                                  void* workspace, size_t ws_bytes, void* stream) {
  if (rows < 1 || rows > 65535 || old_rows < 1 || old_rows > 65535) return refuse("rows and old_rows must lie in [1, 65535]");
  if (page_size < 16 || page_size > 4096 || page_size % 16 != 0)
    return refuse("page_size must be a multiple of 16 in [16, 4096]");
  if (pages < 1 || pages > (int64_t)0x7fffffff / page_size) return refuse("the cache must hold 1 to 2^31 - 1 tokens");
  if (table_width < 1 || table_width > (int64_t)1 << 24 || ldt < table_width || ldo < table_width) return refuse("bad table");
  if (rows * table_width > (int64_t)1 << 31) return refuse("rows x table_width must not exceed 2^31");
  if (!table || !length || !want || !out || !copies) return refuse("table, length, want, out or copies is NULL");
  if (!source && rows > old_rows) return refuse("more rows than there were need their sources");
  for (const void* p : {(const void*)table, (const void*)length, (const void*)source, (const void*)want, (const void*)held,
                        (const void*)out, (const void*)copies, (const void*)left})
    if (!aligned(p, 4)) return refuse("an argument is not aligned to its elements");
  if (overlap(table, ((old_rows - 1) * ldt + table_width) * 4, out, ((rows - 1) * ldo + table_width) * 4))
    return refuse("out must not share memory with table");
  const size_t need = update_bytes(rows, pages);
  if (!workspace || ws_bytes < need) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace missing or too small");
  if (!aligned(workspace, 256)) return refuse(GPTQ2D_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  UpdateArgs a = {rows, old_rows, table_width, pages, page_size, table, ldt, length, source, want, held, out, ldo, copies, left};
  char* w = (char*)workspace;
  a.mark = (uint32_t*)w;
  a.list = (uint32_t*)(w + up256((size_t)pages * 4));
  a.before = (uint32_t*)(w + 2 * up256((size_t)pages * 4));
  const hipStream_t s = (hipStream_t)stream;
  if (rows * table_width + pages <= kOnePages) {
    hipLaunchKernelGGL(k_update_one, dim3(1), dim3(kScan), 0, s, a);
  } else {
    const unsigned waves = (unsigned)ceil_div(rows, 4);
    hipLaunchKernelGGL(k_update_clear, dim3((unsigned)ceil_div(pages, 256)), dim3(256), 0, s, a);
    hipLaunchKernelGGL(k_update_mark, dim3(waves), dim3(256), 0, s, a);
    hipLaunchKernelGGL(k_update_scan, dim3(1), dim3(kScan), 0, s, a);
    hipLaunchKernelGGL(k_update_write, dim3(waves), dim3(256), 0, s, a);
  }
  return launched("gptq2d_pages_update");
}

}  // extern "C"
