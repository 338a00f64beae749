// Pages of the eight-bit cache between two steps of serving: the kept tokens of a
// drafted tree moved to where the next step expects them, page tables of sequences
// that were forked, cut, freed or have grown, and the copies of pages that these ask
// for. The caches of a model's layers share their tables, so a call does all layers.
#include <algorithm>
#include <type_traits>

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

// A wave moves one head's vectors of one sequence in N layers, L lanes a vector; where they lie
// is found once for them. A position is written by the entry of its own number, and
// read by that or an earlier one (path[i] >= i): so all reads of a turn come before its
// writes, and turns may follow one another. Bound by the chain path, table, vector: 32
// layers of 64 trees of 64, 8 heads of 64, 8.8 us, of one tree of 8 4.0 us.
template <int L, int N>
__global__ __launch_bounds__(256) void k_commit(CommitArgs a) {
  constexpr int P = 64 / L;
  const int lane = threadIdx.x & 63, l = lane % L, layer0 = blockIdx.y * N, layers = min(N, a.layers - layer0);
  const int64_t vec = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (vec >= a.vectors) return;
  const int64_t seq = vec / a.heads;
  const int head = (int)(vec - seq * a.heads);
  const int64_t context = a.context[seq];
  const int32_t mine = lane < a.width ? a.path[seq * a.width + lane] : -1;
  const uint64_t todo = __ballot(mine > lane && mine < a.width);
  if (todo == 0) return;
  const int end = 64 - __builtin_clzll(todo);
#pragma unroll 1
  for (int i0 = __builtin_ctzll(todo) / P * P; i0 < end; i0 += P) {
    const int i = i0 + lane / L;
    const int32_t from = __shfl(mine, i);
    int64_t src = -1, dst = -1;
    if (todo >> i & 1) src = slot_of(a, seq, context + from), dst = slot_of(a, seq, context + i);
    const bool go = src >= 0 && dst >= 0 && 16 * l < a.dim;
    // [page][head][token]
    auto place = [&](int64_t slot) {
      const uint32_t p = (uint32_t)slot / a.page;
      return ((int64_t)p * a.heads + head) * a.page + ((uint32_t)slot - p * a.page);
    };
    const int64_t s = go ? place(src) : 0, d = go ? place(dst) : 0;
    u4 v[N][2];
    float f[N][2];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (go && k < layers) {
          v[k][t] = *(const u4*)(a.at.code[layer0 + k][t] + s * a.dim + 16 * l);
          if (l == 0) f[k][t] = a.at.scale[layer0 + k][t][s];
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (go && k < layers) {
          *(u4*)(a.at.code[layer0 + k][t] + d * a.dim + 16 * l) = v[k][t];
          if (l == 0) a.at.scale[layer0 + k][t][d] = f[k][t];
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

constexpr int kPieces = 4;  // of a thread and tensor

// A work group copies some pieces of one page's codes in one layer, head by head the
// first tokens; the first group the scales too. Source and copy are different pages, so
// everything is read before anything is written (4 pages of 64 tokens, 8 heads of 128, 32
// layers 7.0 us, piece by piece 7.8).
__global__ __launch_bounds__(256) void k_copy(CopyArgs a) {
  const int64_t i = blockIdx.x;
  const int layer = blockIdx.z;
  const int32_t from = a.copies[3 * i], to = a.copies[3 * i + 1];
  const uint32_t n = (uint32_t)min(max(a.copies[3 * i + 2], 0), (int32_t)a.page);
  if (from < 0 || to < 0 || from >= a.pages || to >= a.pages || from == to || n == 0) return;
  const uint32_t some = n * (uint32_t)a.dim / 16, all = some * (uint32_t)a.heads;
  const int64_t size = (int64_t)a.heads * a.page, delta = (to - (int64_t)from) * size;
  u4* c[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) c[t] = (u4*)(a.at.code[layer][t] + from * size * a.dim);
  const int64_t far = delta * a.dim / 16;
  for (uint32_t e0 = blockIdx.y * (256 * kPieces) + threadIdx.x; e0 < all; e0 += gridDim.y * (256 * kPieces)) {
    uint32_t at[kPieces];
    u4 v[kPieces][2];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const uint32_t e = min(e0 + k * 256, all - 1), head = e / some;
      at[k] = head * a.pieces + (e - head * some);
#pragma unroll
      for (int t = 0; t < 2; ++t) v[k][t] = c[t][at[k]];
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (e0 + k * 256 < all) c[t][far + at[k]] = v[k][t];
  }
  if (blockIdx.y == 0) {
    for (uint32_t e = threadIdx.x; e < n * a.heads; e += 256) {
      const uint32_t head = e / n, at = head * a.page + (e - head * n);
      float* f[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) f[t] = a.at.scale[layer][t] + from * size + at;
      const float x = *f[0], y = *f[1];
      f[0][delta] = x, f[1][delta] = y;
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
  // workspace: a mark of each page (0: it is held, or a row holds it whole, 1 + s: row s is
  // the first of those that end in it, kNobody), the free pages in order, the number of
  // new pages of the rows before each
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
__device__ __forceinline__ bool copies_page(const uint32_t* mark, int64_t s, int32_t p) {
  return p >= 0 && mark[p] != (uint32_t)s + 1;
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
  return (uint32_t)(max(r.end - n, (int64_t)0) + (r.part > 0 && copies_page(mark, s, named(a, r.old[r.whole]))));
}
__device__ __forceinline__ void write_row(const UpdateArgs& a, const uint32_t* mark, int64_t s, uint32_t free, int lane) {
  const Row r = row_of(a, s);
  const int32_t last = r.part > 0 ? named(a, r.old[r.whole]) : -1;
  const bool copied = r.part > 0 && copies_page(mark, s, last);
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
__device__ __forceinline__ uint32_t sum_upto(uint32_t v) {  // of the lanes up to this one
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, true);
  return v;
}
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* waves, uint32_t& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t s = sum_upto(v);
  __syncthreads();  // (the last call's sums are read)
  if (lane == 63) waves[w] = s;
  __syncthreads();
  const uint32_t upto = sum_upto(lane < kScan / 64 ? waves[lane] : 0);
  all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  return s - v + (w > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)upto, w - 1) : 0);
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
      f[i] = p < a.pages && mark[p] == kNobody;
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

// All of it in one launch: every work group marks all pages and finds all free ones for
// itself, in LDS, and writes its share of the rows. (Marks shared through memory have to be
// cleared, made, and looked at by launches of their own: 256 rows of 130 entries over 9281
// pages 20 us in four launches, 15 here.)
constexpr int kOnePages = 28672, kOneRows = 1024;
struct Found {
  int32_t from, whole, part, end;  // as of a Row, `from` its old sequence
  int32_t last;                    // the page that it ends in, -1: none
  uint32_t before;                 // new pages of the rows before it; the top bit: `last` is copied
};
__global__ __launch_bounds__(kScan) void k_update_one(UpdateArgs a) {
  __shared__ uint32_t mark[kOnePages];  // later: the free pages
  __shared__ Found found[kOneRows];
  __shared__ uint64_t bits[kOnePages / 64];
  __shared__ uint32_t ahead[kOnePages / 64];
  __shared__ uint32_t waves[kScan / 64];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, rows = (int)a.rows, pages = (int)a.pages;
  const int width = (int)a.table_width;
  // a row's numbers in 32 bits (table_width page <= 2^30)
  int from = t, want = 0;
  if (t < rows) {
    if (a.source) from = a.source[t];
    want = a.want[t];
  }
  if (t < rows) {
    const bool any = from >= 0 && from < a.old_rows;
    const uint32_t page = (uint32_t)a.page, room = (uint32_t)width * page;
    const uint32_t wants = min((uint32_t)max(want, 0), room);
    const uint32_t kept = any ? min((uint32_t)max(a.length[from], 0), wants) : 0, whole = kept / page;
    found[t] = Found{any ? from : 0, (int)whole, (int)(kept - whole * page), (int)((wants + page - 1) / page), -1, 0};
  }
#pragma unroll 1
  for (int p0 = t; p0 < pages; p0 += 14 * kScan) {
    int32_t held[14];
#pragma unroll
    for (int k = 0; k < 14; ++k) held[k] = a.held ? a.held[min(p0 + k * kScan, pages - 1)] : 0;
#pragma unroll
    for (int k = 0; k < 14; ++k)
      if (p0 + k * kScan < pages) mark[p0 + k * kScan] = held[k] != 0 ? 0 : kNobody;
  }
  __syncthreads();
  // A wave takes eight rows at once, 256 entries of each; its lanes hold the rows' numbers. (0 is the
  // least mark: it is stored.)
  constexpr int kBatch = 8, kWaves = kScan / 64;
#pragma unroll 1
  for (int s0 = w; s0 < rows; s0 += kBatch * kWaves) {
    const int row = s0 + (lane % kBatch) * kWaves;
    const Found f = found[min(row, rows - 1)];
    const int from_of = f.from, whole_of = row < rows ? f.whole : 0, end_of = row < rows ? f.whole + (f.part > 0) : 0;
    const int most = (int)group_max<64>((uint32_t)end_of);
#pragma unroll 1
    for (int j0 = 0; j0 < most; j0 += 256) {
      int32_t p[4][kBatch];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (j0 + 64 * c >= most) break;
        const uint32_t at = (uint32_t)min(j0 + 64 * c + lane, width - 1) * 4;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int32_t* first = a.table + (int64_t)__builtin_amdgcn_readlane(from_of, k) * a.ldt;
          p[c][k] = *(const int32_t*)((const char*)first + at);
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int first = j0 + 64 * c;
        if (first >= most) break;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int whole = __builtin_amdgcn_readlane(whole_of, k);
          const bool names = (uint32_t)p[c][k] < (uint32_t)pages;
          if (first + 64 <= whole) {  // (most of them)
            if (names) mark[p[c][k]] = 0;
          } else if (first < __builtin_amdgcn_readlane(end_of, k)) {
            const int j = first + lane;
            if (j < whole && names) mark[p[c][k]] = 0;
            if (j == whole && j < __builtin_amdgcn_readlane(end_of, k)) {
              if (names) atomicMin(&mark[p[c][k]], (uint32_t)(s0 + k * kWaves) + 1);
              found[s0 + k * kWaves].last = names ? p[c][k] : -1;
            }
          }
        }
      }
    }
  }
  __syncthreads();
  uint32_t need = 0, copied = 0, all;
  if (t < rows) {
    const Found f = found[t];
    copied = f.part > 0 && copies_page(mark, t, f.last);
    need = (uint32_t)max(f.end - f.whole - (f.part > 0), 0) + copied;
  }
  const uint32_t before = sum_before(need, waves, all);
  const uint32_t lacking = all;
  if (t < rows) found[t].before = before | copied << 31;
  // free pages, a word of 64 by each wave
  const int words = (pages + 63) / 64;
  for (int k = 0; k * kScan < pages; ++k) {
    const int p = k * kScan + t;
    const uint64_t free = __ballot(p < pages && mark[min(p, pages - 1)] == kNobody);
    if (lane == 0 && p < pages) bits[p / 64] = free;
  }
  __syncthreads();
  // the free ones in order, in the place of the marks (kOnePages / 64 <= kScan)
  const uint32_t at = sum_before(t < words ? (uint32_t)__popcll(bits[t]) : 0, waves, all);
  if (t < words) ahead[t] = at;
  const uint32_t free = all;
  __syncthreads();
  for (int k = 0; k * kScan < pages; ++k) {
    const int p = k * kScan + t, word = min(p / 64, words - 1);
    const uint64_t b = bits[word];
    if (p < pages && (b >> lane & 1)) mark[ahead[word] + __popcll(b & ((1ull << lane) - 1))] = (uint32_t)p;
  }
  __syncthreads();
  if (blockIdx.x == 0 && t == 0 && a.left) *a.left = (int32_t)free - (int32_t)lacking;
  for (int row = blockIdx.x * (kScan / 64) + w; row < rows; row += gridDim.x * (kScan / 64)) {
    const Found f = found[row];
    const bool copy = f.before >> 31;
    const uint32_t first = f.before & 0x7fffffffu;
    const int kept = f.whole + (f.part > 0 && !copy);
#pragma unroll 1
    for (int j0 = lane; j0 < width; j0 += 256) {
      int32_t old[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) old[k] = a.table[(int64_t)f.from * a.ldt + min(j0 + 64 * k, width - 1)];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + 64 * k;
        if (j >= width) break;
        int32_t p = -1;
        if (j < kept) p = named(a, old[k]);
        else if (j < f.end && first + (uint32_t)(j - kept) < free) p = (int32_t)mark[first + (uint32_t)(j - kept)];
        a.out[row * a.ldo + j] = p;
        if (copy && j == f.whole) {
          a.copies[3 * row] = f.last;
          a.copies[3 * row + 1] = p;
          a.copies[3 * row + 2] = f.part;
        }
      }
    }
    if (!copy && lane < 3) a.copies[3 * row + lane] = lane < 2 ? -1 : 0;
  }
}

// The same in four launches.
__global__ __launch_bounds__(256) void k_update_clear(UpdateArgs a) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p < a.pages) a.mark[p] = a.held && a.held[p] != 0 ? 0 : kNobody;
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
    // layers of a wave: one as long as all waves are there at once, then the way to a vector for four
    auto of = [&](auto l) {
      constexpr int L = decltype(l)::value;
      const unsigned groups = (unsigned)ceil_div(a.vectors, 4);
      if ((int64_t)groups * a.layers <= 2048)
        hipLaunchKernelGGL((k_commit<L, 1>), dim3(groups, a.layers), dim3(256), 0, (hipStream_t)stream, a);
      else
        hipLaunchKernelGGL((k_commit<L, 4>), dim3(groups, (a.layers + 3) / 4), dim3(256), 0, (hipStream_t)stream, a);
    };
    if (dim <= 64) of(std::integral_constant<int, 4>());
    else if (dim <= 128) of(std::integral_constant<int, 8>());
    else of(std::integral_constant<int, 16>());
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
    const dim3 grid((unsigned)count, (unsigned)std::min<int64_t>(ceil_div(pieces, 256 * kPieces), 64), n);
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
  if (rows <= kOneRows && pages <= kOnePages && rows * table_width <= 1 << 18) {
    hipLaunchKernelGGL(k_update_one, dim3((unsigned)ceil_div(rows, kScan / 64)), dim3(kScan), 0, s, a);
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
