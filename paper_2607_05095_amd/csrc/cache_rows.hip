// cache_rows.hip -- cached rows in 8 or 4 bits: written from rows, read back
// (record layout and conversions in mx.h).
//
// Bound by HBM: a write reads a row and writes its record, a read the other way
// round, at random slots.  A lane moves 8 elements; the four neighbouring lanes
// of a group of 32 find its largest magnitude with two DPP exchanges inside
// their quad, so a row is read once and no LDS is used.
#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int CR_THREADS = 256;
constexpr int CR_UNITS = 1024;       // pieces per workgroup, about

struct CacheArgs {
  const int64_t* ids;
  int64_t n, id_bound;
  const int32_t* slot_map;
  int64_t cache_rows;
  MxRecord rec;
  int rows;                          // rows per workgroup
  int upr, upp;                      // pieces per row, per part
  uint32_t mag_upr, mag_upp;
  const void* src;
  void* dst;
  const uint8_t* cache_in;
  uint8_t* cache;
  int32_t* owner;                    // last i of each slot, or NULL: no repeats
};

// 8 elements of a row: values from src, or to dst.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float* x) {
#pragma unroll
  for (int j = 0; j < 8; j += CHUNK<T>) load_chunk(p + j, n - j, x + j);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float* x) {
#pragma unroll
  for (int j = 0; j < 8; j += CHUNK<T>) store_chunk(p + j, n - j, x + j);
}

// Two passes over the ids find the last i of every slot: the first clears the
// slots that the ids name, the second takes the maximum.
__global__ void __launch_bounds__(CR_THREADS) k_cache_claim(CacheArgs a, int pass) {
  const int64_t i = int64_t(blockIdx.x) * CR_THREADS + threadIdx.x;
  if (i >= a.n) return;
  const int64_t s = mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows);
  if (s < 0) return;
  if (pass == 0) a.owner[s] = -1;
  else atomicMax(a.owner + s, int32_t(i));
}

template <typename T, int FMT>
__global__ void __launch_bounds__(CR_THREADS) k_cache_write(CacheArgs a) {
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows);
  const T* src = static_cast<const T*>(a.src);
  constexpr int PB = FMT == FAST_MXFP4 ? MX_PIECE / 2 : MX_PIECE;
  // whole quads of lanes: upp is a multiple of 4
  for (int t = threadIdx.x; t < rows * a.upr; t += CR_THREADS) {
    const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
    const int part = int(div_small(u, a.mag_upp)), c = u - part * a.upp;
    const int64_t i = row0 + r;
    int64_t slot = mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows);
    if (slot >= 0 && a.owner && a.owner[slot] != int32_t(i)) slot = -1;
    if (slot < 0) continue;            // the four lanes of a quad share a row
    float x[8];
    load8(src + (i * a.rec.parts + part) * a.rec.width + c * 8, a.rec.width - c * 8, x);
    // magnitudes as integers: their order is that of the values, NaN the largest
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
      m = m > b ? m : b;
    }
    uint32_t o = __float_as_uint(dpp_quad_xor1(__uint_as_float(m)));
    m = m > o ? m : o;
    o = __float_as_uint(dpp_quad_xor2(__uint_as_float(m)));
    m = m > o ? m : o;
    const uint32_t sb = mx_scale_byte<FMT>(__uint_as_float(m));
    MxPiece<FMT, 8> p;
    if (sb == 255u) p.zero();
    else p.pack(mx_scale(sb), x);
    uint8_t* rec = a.cache + slot * a.rec.stride;
    if (c * 8 < a.rec.width) p.store(rec + part * a.rec.code_bytes + c * PB);
    if ((c & 3) == 0) rec[a.rec.scale_off + part * a.rec.groups + (c >> 2)] = uint8_t(sb);
  }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(CR_THREADS) k_cache_gather(CacheArgs a) {
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows);
  T* dst = static_cast<T*>(a.dst);
  constexpr int PB = FMT == FAST_MXFP4 ? MX_PIECE / 2 : MX_PIECE;
  for (int t = threadIdx.x; t < rows * a.upr; t += CR_THREADS) {
    const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
    const int part = int(div_small(u, a.mag_upp)), c = u - part * a.upp;
    const int64_t i = row0 + r;
    const int64_t slot = mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows);
    if (slot < 0) continue;
    const uint8_t* rec = a.cache_in + slot * a.rec.stride;
    MxPiece<FMT, 8> p;
    p.load(rec + part * a.rec.code_bytes + c * PB);
    const uint32_t sb = rec[a.rec.scale_off + part * a.rec.groups + (c >> 2)];
    float x[8];
    p.unpack(mx_scale(sb), x);
    store8(dst + (i * a.rec.parts + part) * a.rec.width + c * 8, a.rec.width - c * 8, x);
  }
}

static fast_status_t cache_check(const char* fn, const int64_t* ids, int64_t n, int64_t id_bound,
                                 int parts, int width, fast_dtype_t dtype, const void* rows,
                                 fast_cache_format_t fmt, const void* cache, int64_t cache_rows) {
  if (n < 0 || id_bound < 0 || cache_rows < 0) return fail(FAST_ERR_INVALID_ARG, "%s: negative size", fn);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  const fast_status_t s = mx_check(fn, parts, width, fmt);
  if (s != FAST_OK) return s;
  if (n >= (int64_t(1) << 31) || cache_rows >= (int64_t(1) << 31))
    return fail(FAST_ERR_UNSUPPORTED, "%s: n or cache_rows >= 2^31", fn);
  if (n == 0 || cache_rows == 0) return FAST_OK;
  if (!ids || !rows || !cache) return fail(FAST_ERR_INVALID_ARG, "%s: NULL ids/rows/cache", fn);
  const size_t es = elem_size(dtype);
  if (!aligned(rows, es)) return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(cache, 16)) return fail(FAST_ERR_UNSUPPORTED, "%s: cache not 16-byte aligned", fn);
  if (!aligned(ids, 8)) return fail(FAST_ERR_UNSUPPORTED, "%s: ids not 8-byte aligned", fn);
  return FAST_OK;
}

static CacheArgs cache_args(const int64_t* ids, int64_t n, int64_t id_bound, const int32_t* slot_map,
                            int parts, int width, fast_cache_format_t fmt, int64_t cache_rows,
                            int quad) {
  CacheArgs a = {};
  a.ids = ids;
  a.n = n;
  a.id_bound = id_bound;
  a.slot_map = slot_map;
  a.cache_rows = cache_rows;
  a.rec = mx_record(parts, width, fmt);
  a.upp = ((width + MX_PIECE - 1) / MX_PIECE + quad - 1) / quad * quad;
  a.upr = a.upp * parts;
  a.rows = CR_UNITS / a.upr > 0 ? CR_UNITS / a.upr : 1;
  a.mag_upr = div_magic(a.upr);
  a.mag_upp = div_magic(a.upp);
  return a;
}

}  // namespace fast

using namespace fast;

extern "C" size_t fast_cache_row_bytes(int parts, int width, fast_cache_format_t format) {
  if (parts <= 0 || width <= 0 || parts > MX_MAX_PARTS || width > MX_MAX_WIDTH ||
      int64_t(parts) * width > MX_MAX_ELEMS || (format != FAST_MXFP8 && format != FAST_MXFP4))
    return 0;
  return size_t(mx_record(parts, width, format).stride);
}

extern "C" size_t fast_cache_write_workspace(int64_t n, int64_t cache_rows) {
  if (n < 0 || cache_rows < 0 || n >= (int64_t(1) << 31) || cache_rows >= (int64_t(1) << 31)) return 0;
  return align_up(size_t(cache_rows > 0 ? cache_rows : 1) * sizeof(int32_t), 16);
}

extern "C" fast_status_t fast_cache_write(const int64_t* ids, int64_t n, int64_t id_bound,
                                          const int32_t* slot_map, int parts, int width,
                                          fast_dtype_t dtype, const void* src,
                                          fast_cache_format_t format, void* cache,
                                          int64_t cache_rows, int distinct, void* ws,
                                          size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_cache_write";
  const fast_status_t s = cache_check(fn, ids, n, id_bound, parts, width, dtype, src, format, cache,
                                      cache_rows);
  if (s != FAST_OK) return s;
  if (n == 0 || cache_rows == 0) return ok();
  if (!distinct) {
    if (!ws || ws_bytes < fast_cache_write_workspace(n, cache_rows))
      return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0,
                  fast_cache_write_workspace(n, cache_rows));
    if (!aligned(ws, 16)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 16-byte aligned", fn);
  }
  CacheArgs a = cache_args(ids, n, id_bound, slot_map, parts, width, format, cache_rows, 4);
  a.src = src;
  a.cache = static_cast<uint8_t*>(cache);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!distinct) {
    a.owner = static_cast<int32_t*>(ws);
    const uint32_t g = uint32_t((n + CR_THREADS - 1) / CR_THREADS);
    hipLaunchKernelGGL(k_cache_claim, dim3(g), dim3(CR_THREADS), 0, st, a, 0);
    hipLaunchKernelGGL(k_cache_claim, dim3(g), dim3(CR_THREADS), 0, st, a, 1);
  }
  const uint32_t grid = uint32_t((n + a.rows - 1) / a.rows);
#define FAST_CW(T, F) hipLaunchKernelGGL((k_cache_write<T, F>), dim3(grid), dim3(CR_THREADS), 0, st, a)
  if (dtype == FAST_F32) {
    if (format == FAST_MXFP8) FAST_CW(float, FAST_MXFP8);
    else FAST_CW(float, FAST_MXFP4);
  } else {
    if (format == FAST_MXFP8) FAST_CW(uint16_t, FAST_MXFP8);
    else FAST_CW(uint16_t, FAST_MXFP4);
  }
#undef FAST_CW
  return check_launch(fn);
}

extern "C" fast_status_t fast_cache_gather(const int64_t* ids, int64_t n, int64_t id_bound,
                                           const int32_t* slot_map, int parts, int width,
                                           fast_cache_format_t format, const void* cache,
                                           int64_t cache_rows, fast_dtype_t dtype, void* rows,
                                           fast_stream_t stream) {
  const char* fn = "fast_cache_gather";
  const fast_status_t s = cache_check(fn, ids, n, id_bound, parts, width, dtype, rows, format, cache,
                                      cache_rows);
  if (s != FAST_OK) return s;
  if (n == 0 || cache_rows == 0) return ok();
  CacheArgs a = cache_args(ids, n, id_bound, slot_map, parts, width, format, cache_rows, 1);
  a.dst = rows;
  a.cache_in = static_cast<const uint8_t*>(cache);
  const uint32_t grid = uint32_t((n + a.rows - 1) / a.rows);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define FAST_CG(T, F) hipLaunchKernelGGL((k_cache_gather<T, F>), dim3(grid), dim3(CR_THREADS), 0, st, a)
  if (dtype == FAST_F32) {
    if (format == FAST_MXFP8) FAST_CG(float, FAST_MXFP8);
    else FAST_CG(float, FAST_MXFP4);
  } else {
    if (format == FAST_MXFP8) FAST_CG(uint16_t, FAST_MXFP8);
    else FAST_CG(uint16_t, FAST_MXFP4);
  }
#undef FAST_CG
  return check_launch(fn);
}
