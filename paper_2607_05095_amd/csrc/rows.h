// rows.h -- rows of any width and alignment: chunks of 16 bytes at the element
// type's own alignment, with a checked tail.
#pragma once

#include "common.h"

namespace fast {

// gfx950 loads and stores 16 bytes at any address; these types tell the compiler
// that only the element's alignment is known, so one instruction moves a
// chunk of a row whose width is no multiple of 16 bytes.
typedef float f32x4_e __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_e __attribute__((ext_vector_type(4), aligned(2)));

typedef float f32x2_e __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32x2_e __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_e __attribute__((aligned(2)));

// Elements of type T (float, or uint16_t holding bf16) in 16 bytes.
template <typename T> constexpr int CHUNK = 16 / int(sizeof(T));

// x[0..CHUNK) = p[0..n), zeros from n on: one load of a whole chunk (NT: streamed,
// non-temporal), else one per power of two in n.  n <= 0 reads nothing.
template <bool NT = false>
__device__ __forceinline__ void load_chunk_of(const float* __restrict__ p, int n, float* x) {
  if (n >= 4) {
    const f32x4_e v = ld_stream<f32x4_e, NT>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    return;
  }
  x[0] = x[1] = x[2] = x[3] = 0.f;
  if (n >= 2) {
    const f32x2_e v = *reinterpret_cast<const f32x2_e*>(p);
    x[0] = v.x; x[1] = v.y;
    if (n == 3) x[2] = p[2];
  } else if (n == 1) {
    x[0] = p[0];
  }
}
__device__ __forceinline__ float bf16_at(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }
template <bool NT = false>
__device__ __forceinline__ void load_chunk_of(const uint16_t* __restrict__ p, int n, float* x) {
  if (n >= 8) {
    const u32x4_e w = ld_stream<u32x4_e, NT>(p);
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = 0.f;
  auto upto3 = [&](int base, int m) {
    if (m >= 2) {
      const uint32_t w = *reinterpret_cast<const u32_e*>(p + base);
      x[base] = bf16_lo(w); x[base + 1] = bf16_hi(w);
      if (m == 3) x[base + 2] = bf16_at(p + base + 2);
    } else if (m == 1) {
      x[base] = bf16_at(p + base);
    }
  };
  if (n >= 4) {
    const u32x2_e w = *reinterpret_cast<const u32x2_e*>(p);
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    upto3(4, n - 4);
  } else {
    upto3(0, n);
  }
}
template <typename T, bool NT = false>
__device__ __forceinline__ void load_chunk(const T* __restrict__ p, int n, float* x) {
  load_chunk_of<NT>(p, n, x);
}

template <bool NT = false>
__device__ __forceinline__ void store_chunk_of(float* __restrict__ p, int n, const float* x) {
  if (n >= 4) {
    st_stream<f32x4_e, NT>(p, f32x4_e{x[0], x[1], x[2], x[3]});
  } else if (n >= 2) {
    *reinterpret_cast<f32x2_e*>(p) = f32x2_e{x[0], x[1]};
    if (n == 3) p[2] = x[2];
  } else if (n == 1) {
    p[0] = x[0];
  }
}
template <bool NT = false>
__device__ __forceinline__ void store_chunk_of(uint16_t* __restrict__ p, int n, const float* x) {
  auto upto3 = [&](int base, int m) {
    if (m >= 2) {
      *reinterpret_cast<u32_e*>(p + base) = bf16_pack(x[base], x[base + 1]);
      if (m == 3) p[base + 2] = uint16_t(bf16_rne(x[base + 2]));
    } else if (m == 1) {
      p[base] = uint16_t(bf16_rne(x[base]));
    }
  };
  if (n >= 8) {
    st_stream<u32x4_e, NT>(p, u32x4_e{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3]),
                                      bf16_pack(x[4], x[5]), bf16_pack(x[6], x[7])});
  } else if (n >= 4) {
    *reinterpret_cast<u32x2_e*>(p) = u32x2_e{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3])};
    upto3(4, n - 4);
  } else {
    upto3(0, n);
  }
}
template <typename T, bool NT = false>
__device__ __forceinline__ void store_chunk(T* __restrict__ p, int n, const float* x) {
  store_chunk_of<NT>(p, n, x);
}

// Do two arrays of as many bytes overlap other than byte on byte?  NULL: no array.
inline bool shifted(const void* a, const void* b, int64_t bytes) {
  if (!a || !b || a == b) return false;
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return (p > q ? p - q : q - p) < uint64_t(bytes);
}

// Do the elements of rows of F elements, ldx and ldy apart, overlap other than
// element on element?
inline bool rows_collide(const char* x, int64_t ldx, const char* y, int64_t ldy, int64_t n, int64_t F,
                         int64_t es) {
  const char* xe = x + ((n - 1) * ldx + F) * es;
  const char* ye = y + ((n - 1) * ldy + F) * es;
  if (x >= ye || y >= xe) return false;
  if (ldx != ldy) return true;
  if (x == y) return false;
  // the same distance apart in every row: disjoint where one lies in the other's gap
  const int64_t d = (y > x ? y - x : x - y) % (ldx * es);
  return d < F * es || ldx * es - d < F * es;
}

// Do p bytes at a and q at b meet?  NULL: no array.
inline bool meet(const void* a, int64_t p, const void* b, int64_t q) {
  if (!a || !b || p <= 0 || q <= 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < uint64_t(p) : x - y < uint64_t(q);
}
// Bytes from the first to the last element of n rows of F elements, ld apart.
inline int64_t span(int64_t n, int64_t F, int64_t ld, int64_t es) { return n > 0 ? ((n - 1) * ld + F) * es : 0; }

// A launch has fewer than 2^32 threads along an axis.
inline bool grid_fits(int64_t blocks, int64_t threads) { return blocks * threads < (int64_t(1) << 32); }

// t / d for t * d < 2^32 with the multiplier of div_magic(d): one high product.
inline uint32_t div_magic(uint32_t d) {
  return d <= 1 ? 0u : uint32_t(((uint64_t(1) << 32) + d - 1) / d);
}
__device__ __forceinline__ uint32_t div_small(uint32_t t, uint32_t magic) {
  return magic ? __umulhi(t, magic) : t;
}

}  // namespace fast
