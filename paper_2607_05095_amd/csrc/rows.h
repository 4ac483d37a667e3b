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

// Elements of type T (float, or uint16_t holding bf16) in 16 bytes.
template <typename T> constexpr int CHUNK = 16 / int(sizeof(T));

// x[0..CHUNK) = p[0..n), zeros from n on.  n <= 0 reads nothing.
template <typename T>
__device__ __forceinline__ void load_chunk(const T* __restrict__ p, int n, float* x) {
  constexpr int VE = CHUNK<T>;
  if (n >= VE) {
    if constexpr (sizeof(T) == 4) {
      const f32x4_e v = *reinterpret_cast<const f32x4_e*>(p);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      const u32x4_e w = *reinterpret_cast<const u32x4_e*>(p);
      x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
      x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    }
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      x[j] = 0.f;
      if (j < n) VecIO<T, 1>::load(p + j, x + j);
    }
  }
}

template <typename T>
__device__ __forceinline__ void store_chunk(T* __restrict__ p, int n, const float* x) {
  constexpr int VE = CHUNK<T>;
  if (n >= VE) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4_e*>(p) = f32x4_e{x[0], x[1], x[2], x[3]};
    } else {
      *reinterpret_cast<u32x4_e*>(p) = u32x4_e{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3]),
                                               bf16_pack(x[4], x[5]), bf16_pack(x[6], x[7])};
    }
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (j < n) VecIO<T, 1>::store(p + j, x + j);
  }
}

// t / d for t * d < 2^32 with the multiplier of div_magic(d): one high product.
inline uint32_t div_magic(uint32_t d) {
  return d <= 1 ? 0u : uint32_t(((uint64_t(1) << 32) + d - 1) / d);
}
__device__ __forceinline__ uint32_t div_small(uint32_t t, uint32_t magic) {
  return magic ? __umulhi(t, magic) : t;
}

}  // namespace fast
