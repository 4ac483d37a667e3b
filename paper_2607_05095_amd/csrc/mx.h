// mx.h -- cached rows in 8 or 4 bits.
//
// A record holds `parts` vectors of `width` elements: each vector's codes (e4m3
// or e2m1, padded to 8 codes), then a scale byte per vector and group of 32
// elements.  Byte b stands for 2^(b - 127), 255 for a group that is not a number;
// an element is its code's value times its group's scale.  These are the element
// and scale formats of the OCP Microscaling (MX) specification 1.0, which
// gfx950 converts in hardware.
#pragma once

#include "common.h"

namespace fast {

constexpr int MX_GROUP = 32;         // elements per scale
constexpr int MX_PIECE = 8;          // codes that a lane moves at once

struct MxRecord {
  int parts, width, groups;          // groups: scales per part
  int code_bytes;                    // bytes of a part's codes
  int scale_off;                     // where the scales start
  int64_t stride;                    // bytes from record to record
};

// Reading records at random takes time by the 128-byte lines they touch
// (2.64 M records of 216-264 bytes: 92 us where a record touches 2 lines, 137 where
// it touches 3, 117-127 in between; scales in an array of their own cost as
// much as a third line).  So the stride is the multiple of 16, up to an eighth above
// the content, whose records touch the fewest lines on average.
inline MxRecord mx_record(int parts, int width, int fmt) {
  MxRecord r = {};
  r.parts = parts;
  r.width = width;
  r.groups = (width + MX_GROUP - 1) / MX_GROUP;
  r.code_bytes = (width + MX_PIECE - 1) / MX_PIECE * (fmt == FAST_MXFP4 ? MX_PIECE / 2 : MX_PIECE);
  r.scale_off = parts * r.code_bytes;
  const int content = parts * (r.code_bytes + r.groups);
  const int first = (content + 15) / 16 * 16, limit = content + content / 8;
  int64_t best = INT64_MAX;
  for (int s = first; s == first || s <= limit; s += 16) {
    int64_t lines = 0;
    for (int k = 0; k < 8; ++k) lines += (k * s % CACHE_LINE + content + CACHE_LINE - 1) / CACHE_LINE;
    if (lines < best) {
      best = lines;
      r.stride = s;
    }
  }
  return r;
}

constexpr int MX_MAX_WIDTH = 1024, MX_MAX_PARTS = 128, MX_MAX_ELEMS = 8192;

inline fast_status_t mx_check(const char* fn, int parts, int width, fast_cache_format_t fmt) {
  if (parts <= 0 || width <= 0)
    return fail(FAST_ERR_INVALID_ARG, "%s: %d parts of %d elements", fn, parts, width);
  if (fmt != FAST_MXFP8 && fmt != FAST_MXFP4)
    return fail(FAST_ERR_INVALID_ARG, "%s: bad cache format", fn);
  if (parts > MX_MAX_PARTS || width > MX_MAX_WIDTH || int64_t(parts) * width > MX_MAX_ELEMS)
    return fail(FAST_ERR_UNSUPPORTED, "%s: %d parts of %d elements (at most %d, %d, %d together)", fn, parts,
                width, MX_MAX_PARTS, MX_MAX_WIDTH, MX_MAX_ELEMS);
  return FAST_OK;
}

// Slot of an id: through the map, or the id itself; -1 where it has none.
__device__ __forceinline__ int64_t mx_slot(int64_t id, int64_t id_bound,
                                           const int32_t* __restrict__ slot_map, int64_t rows) {
  if (id < 0 || id >= id_bound) return -1;
  const int64_t s = slot_map ? int64_t(slot_map[id]) : id;
  return s >= 0 && s < rows ? s : -1;
}

// 2^(b - 127) as the converters take it: the bits of a float's exponent field
// (0 is read as 2^-127, 255 as not a number).
__device__ __forceinline__ float mx_scale(uint32_t b) { return __uint_as_float(b << 23); }

// A piece of 4, 8 or 16 codes of one group, and its values.  Pieces of 16 may start
// at a multiple of 8 codes.
typedef uint32_t u32x4_8 __attribute__((ext_vector_type(4), aligned(8)));
typedef uint32_t u32x2_4 __attribute__((ext_vector_type(2), aligned(4)));
template <int FMT, int N> struct MxPiece;
template <int N> struct MxPiece<FAST_MXFP8, N> {
  uint32_t w[N / 4];
  __device__ void load(const uint8_t* p) {
    if constexpr (N == 16) {
      const u32x4_8 t = *reinterpret_cast<const u32x4_8*>(p);
      w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
    } else if constexpr (N == 8) {
      const uint2 t = *reinterpret_cast<const uint2*>(p);
      w[0] = t.x; w[1] = t.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  __device__ void store(uint8_t* p) const {
    static_assert(N <= 8, "pieces are written 4 or 8 codes at a time");
    if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
  __device__ void zero() {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) w[k] = 0u;
  }
  __device__ void unpack(float scale, float* x) const {
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
      const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k], scale, false);
      const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k], scale, true);
      x[4 * k] = a.x; x[4 * k + 1] = a.y; x[4 * k + 2] = b.x; x[4 * k + 3] = b.y;
    }
  }
  // round to nearest, ties to even; |x| <= 448 scale
  __device__ void pack(float scale, const float* x) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
      s16x2 t = {0, 0};
      t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, x[4 * k], x[4 * k + 1], scale, false);
      t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, x[4 * k + 2], x[4 * k + 3], scale, true);
      w[k] = __builtin_bit_cast(uint32_t, t);
    }
  }
};
template <int N> struct MxPiece<FAST_MXFP4, N> {
  static constexpr int W = N >= 8 ? N / 8 : 1, PAIRS = N >= 8 ? 4 : 2;   // words, pairs in each
  uint32_t w[W];
  __device__ void load(const uint8_t* p) {
    if constexpr (N == 16) {
      const u32x2_4 t = *reinterpret_cast<const u32x2_4*>(p);
      w[0] = t.x; w[1] = t.y;
    } else if constexpr (N == 8) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ void store(uint8_t* p) const {
    static_assert(N <= 8, "pieces are written 4 or 8 codes at a time");
    if constexpr (N == 8) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint16_t*>(p) = uint16_t(w[0]);
  }
  __device__ void zero() {
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = 0u;
  }
  __device__ void unpack(float scale, float* x) const {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], scale, 0);
      const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], scale, 1);
      float* o = x + 8 * k;
      o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
      if constexpr (PAIRS == 4) {
        const f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], scale, 2);
        const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], scale, 3);
        o[4] = c.x; o[5] = c.y; o[6] = d.x; o[7] = d.y;
      }
    }
  }
  // round to nearest, ties to even; |x| <= 6 scale
  __device__ void pack(float scale, const float* x) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      uint32_t t = 0;
      t = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(t, x[8 * k], x[8 * k + 1], scale, 0);
      t = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(t, x[8 * k + 2], x[8 * k + 3], scale, 1);
      if constexpr (PAIRS == 4) {
        t = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(t, x[8 * k + 4], x[8 * k + 5], scale, 2);
        t = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(t, x[8 * k + 6], x[8 * k + 7], scale, 3);
      }
      w[k] = t;
    }
  }
};

// Scale byte of a group from its largest magnitude: the smallest power of two
// whose multiple of the format's largest value (448 = 1.75 2^8, 6 = 1.5 2^2)
// reaches it, taken from the float's exponent and mantissa, so it is exact.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(float amax) {
  const uint32_t b = __float_as_uint(amax);
  if (b >= 0x7f800000u) return 255u;                       // an infinity or a NaN
  constexpr uint32_t top = FMT == FAST_MXFP4 ? 0x400000u : 0x600000u;   // mantissa of the largest value
  constexpr int emax = FMT == FAST_MXFP4 ? 2 : 8;
  const int e = int(b >> 23) - emax + ((b & 0x7fffffu) > top ? 1 : 0);
  return e > 0 ? uint32_t(e) : 0u;
}

// The scale byte under which the nearest code may stand for 2^128, which fp32 does not hold
// (groups of more than 448 2^119, 6 2^125), and the largest value below: 240 2^120, 3 2^126.
template <int FMT> constexpr uint32_t MX_TOP_BYTE = FMT == FAST_MXFP4 ? 253u : 247u;
template <int FMT> constexpr float MX_TOP = FMT == FAST_MXFP4 ? 0x1.8p127f : 0x1.ep127f;

}  // namespace fast
