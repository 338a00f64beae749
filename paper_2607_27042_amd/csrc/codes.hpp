// Building blocks of the eight-bit operators (quantiser, block product, cache,
// attention, log probabilities): element types, the scale of a block and its
// codes, cross-lane reductions, refusals.
//
// A block of values x with largest magnitude amax is held as eight-bit codes
// and one 32-bit scale s:
//   s = max(fl(amax c), 2^-126), c = fl(1 / top), top = 448 (e4m3) or 127 (int8);
//       rounded up to a power of two where asked; 1 if amax = 0
//   code = the nearest code (ties to even) to fl(x fl(1 / s)), clamped to +-top
// with fl the rounding to 32 bits, so that codes are the same on every route.
// A block that holds a NaN or an infinity gets scale NaN and codes 0: whatever
// reads it comes out as NaN, and no code is ever one of e4m3's NaNs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.hpp"

namespace g2d {

typedef float fp2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16;
typedef bf16 b4 __attribute__((ext_vector_type(4)));

constexpr float kTopE4M3 = 448.0f;
constexpr float kTopInt8 = 127.0f;
constexpr float kTinyScale = 0x1p-126f;

__device__ __forceinline__ bool bad_amax(uint32_t bits) { return bits >= 0x7f800000u; }

// bits: the largest of the magnitudes' bit patterns (ordered as the magnitudes
// are, infinity and NaN above all of them)
__device__ __forceinline__ float block_scale(uint32_t bits, float inv_top, bool pow2) {
  if (bad_amax(bits)) return __uint_as_float(0x7fc00000u);
  if (bits == 0) return 1.0f;
  float s = fmaxf(__uint_as_float(bits) * inv_top, kTinyScale);
  if (pow2) s = __uint_as_float((__float_as_uint(s) + 0x7fffffu) & 0x7f800000u);
  return s;
}

__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

__device__ __forceinline__ float clampf(float x, float top) { return fminf(fmaxf(x, -top), top); }

// four codes from four values already multiplied by 1 / s
template <bool INT8>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  if constexpr (INT8) {
    const int ia = (int)rintf(clampf(a, kTopInt8)), ib = (int)rintf(clampf(b, kTopInt8));
    const int ic = (int)rintf(clampf(c, kTopInt8)), id = (int)rintf(clampf(d, kTopInt8));
    return (ia & 255) | (ib & 255) << 8 | (ic & 255) << 16 | (uint32_t)id << 24;
  } else {
    int r = 0;
    r = __builtin_amdgcn_cvt_pk_fp8_f32(clampf(a, kTopE4M3), clampf(b, kTopE4M3), r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(clampf(c, kTopE4M3), clampf(d, kTopE4M3), r, true);
    return (uint32_t)r;
  }
}

// codes of eight values; zero where the block is not finite
template <bool INT8>
__device__ __forceinline__ u2 code8(const float x[8], float r, bool bad) {
  u2 q;
  q[0] = code4<INT8>(x[0] * r, x[1] * r, x[2] * r, x[3] * r);
  q[1] = code4<INT8>(x[4] * r, x[5] * r, x[6] * r, x[7] * r);
  if (bad) q = u2{0, 0};
  return q;
}

// the two halves that bytes 2 HI and 2 HI + 1 of w stand for, exactly
template <bool INT8, bool HI>
__device__ __forceinline__ h2 halves(uint32_t w) {
  if constexpr (INT8) {
    // 0x6400 | b is 1024 + b; b is the code plus 128
    const uint32_t p = __builtin_amdgcn_perm(0x64646464u, w ^ 0x80808080u, HI ? 0x04030402u : 0x04010400u);
    return __builtin_bit_cast(h2, p) - h2{(_Float16)1152.0f, (_Float16)1152.0f};
  } else {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI);
  }
}

// Eight consecutive elements at p as floats; `wide`: p is 16-byte aligned and
// all eight are there, otherwise the first n (which may be none) are read one by
// one, the rest are 0. (For those the last one is read, or what lies at `any`: a
// branch around a load would make the next one wait for it.)
template <class T>
__device__ __forceinline__ void load8(const T* p, bool wide, int n, float x[8], const T* any) {
  if (wide) {
    if constexpr (sizeof(T) == 4) {
      const f4 a = *(const f4*)p, b = *(const f4*)(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
      typedef T V __attribute__((ext_vector_type(8)));
      const V a = __builtin_bit_cast(V, *(const u4*)p);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
  } else {
    const T* q = n > 0 ? p : any;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)q[min(i, max(n - 1, 0))];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? x[i] : 0.0f;
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, bool wide, int n, const float x[8]) {
  if (wide) {
    if constexpr (sizeof(T) == 4) {
      *(f4*)p = f4{x[0], x[1], x[2], x[3]};
      *(f4*)(p + 4) = f4{x[4], x[5], x[6], x[7]};
    } else {
      // one piece of 16 bytes: element by element the compiler would share the
      // stores with the other branch, and write eight times as often
      typedef T V __attribute__((ext_vector_type(8)));
      V a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (T)x[i];
      *(u4*)p = __builtin_bit_cast(u4, a);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)x[i];
  }
}

// over groups of L consecutive lanes (L a power of two), in every lane, without LDS:
// lanes 1 and 2 away, then 8 and 16 lanes mirrored, then rows of 16 and halves swapped
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  static_assert(L >= 4 && L <= 64, "4 to 64 lanes");
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));
  if constexpr (L >= 8) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if constexpr (L >= 16) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  if constexpr (L >= 32) {
    const u2 a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
  }
  if constexpr (L == 64) {
    const u2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max(b[0], b[1]);
  }
  return v;
}

// over the four lanes that share lane % 16, in every lane
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const u2 a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const u2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------

inline gptq2d_status refuse(gptq2d_status s, const char* msg) noexcept {
  try {
    set_error(msg);
  } catch (...) {
  }
  return s;
}
inline gptq2d_status refuse(const char* msg) noexcept { return refuse(GPTQ2D_ERR_INVALID_ARG, msg); }

// the error of the launches before it
inline gptq2d_status launched(const char* what) noexcept {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return GPTQ2D_OK;
  try {
    return hip_fail(e, what);
  } catch (...) {
    return GPTQ2D_ERR_HIP;
  }
}

inline size_t elem_size(gptq2d_dtype dt) { return dt == GPTQ2D_F64 ? 8 : dt == GPTQ2D_F32 ? 4 : 2; }
inline bool narrow_dtype(gptq2d_dtype dt) {
  return dt == GPTQ2D_F32 || dt == GPTQ2D_F16 || dt == GPTQ2D_BF16;
}
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// every row of a matrix starts on a 16-byte boundary
inline bool wide_rows(const void* p, int64_t ld, size_t es) {
  return aligned(p, 16) && (uint64_t)ld * es % 16 == 0;
}
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The cache's shape and tensors. Slots stay below 2^31 (quotients by the page
// size are taken in 32 bits).
inline gptq2d_status check_cache(int heads, int dim, gptq2d_code code, int64_t pages, int page_size, const void* KC,
                                 const void* VC, const void* KS, const void* VS) {
  if (heads < 1 || heads > 4096) return refuse("heads must lie in [1, 4096]");
  if (dim < 16 || dim > 256 || dim % 16 != 0) return refuse("dim must be a multiple of 16 in [16, 256]");
  if (code != GPTQ2D_E4M3 && code != GPTQ2D_INT8) return refuse("bad code");
  if (page_size < 16 || page_size > 4096 || page_size % 16 != 0)
    return refuse("page_size must be a multiple of 16 in [16, 4096]");
  if (pages < 1 || pages > (int64_t)0x7fffffff / page_size) return refuse("the cache must hold 1 to 2^31 - 1 tokens");
  if (!KC || !VC || !KS || !VS) return refuse("a tensor of the cache is NULL");
  if (!aligned(KC, 16) || !aligned(VC, 16) || !aligned(KS, 16) || !aligned(VS, 16))
    return refuse("the cache's tensors must be 16-byte aligned");
  return GPTQ2D_OK;
}

// calls f with a null pointer of the element type of dt (F32, F16 or BF16)
template <class F>
inline void with_type(gptq2d_dtype dt, F&& f) {
  if (dt == GPTQ2D_F32)
    f((float*)nullptr);
  else if (dt == GPTQ2D_F16)
    f((_Float16*)nullptr);
  else
    f((bf16*)nullptr);
}

}  // namespace g2d
