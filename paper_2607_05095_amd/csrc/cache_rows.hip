// cache_rows.hip -- cached rows in 8 or 4 bits: written from rows, read back
// (record layout and conversions in mx.h).
//
// Bound by HBM: a write reads a row and writes its record, a read the other way
// round, at random slots (264,000 rows of 4 x 50 fp32 in 8 bits: 54 us = 5.1 TB/s and 45 = 6.2).  A workgroup looks up the slots of its rows once, in LDS;
// then a thread moves CR_UNROLL pieces of 16 bytes of a row (4 fp32 or 8 bf16
// elements), all of whose loads are in flight together.  The 8 or 4 neighbouring lanes of
// a group of 32 find its largest magnitude with DPP exchanges, so a row is read once.
#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int CR_THREADS = 256;
constexpr int CR_UNROLL = 4;         // pieces per thread
constexpr int CR_TILE = CR_UNROLL * CR_THREADS;
constexpr int CR_ROWS = 256;         // rows per workgroup, at most
constexpr int CR_SMALL = 1024;       // writes whose repeats a workgroup finds itself

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
  int32_t* owner;                    // write: the last i of each slot, or NULL
  int32_t* slots;                    // write with owners: the slot of each i, looked up once
  bool search;                       // write of at most CR_SMALL rows: repeats are looked for here
};

// Two passes find the last i of every slot: the first looks the slots up and clears their
// owners, the second takes the maximum.
__global__ void __launch_bounds__(CR_THREADS) k_cache_claim(CacheArgs a, int pass) {
  const int64_t i = int64_t(blockIdx.x) * CR_THREADS + threadIdx.x;
  if (i >= a.n) return;
  if (pass == 0) {
    const int64_t s = mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows);
    a.slots[i] = int32_t(s);
    if (s >= 0) a.owner[s] = -1;
  } else {
    const int32_t s = a.slots[i];
    if (s >= 0) atomicMax(a.owner + s, int32_t(i));
  }
}

// Slots of the workgroup's rows (-1: none), in LDS.
__device__ __forceinline__ void cr_slots(const CacheArgs& a, int64_t row0, int rows, int32_t* s_slot) {
  for (int r = threadIdx.x; r < rows; r += CR_THREADS) {
    const int64_t i = row0 + r;
    int32_t s;
    if (a.owner) {
      s = a.slots[i];
      if (s >= 0 && a.owner[s] != int32_t(i)) s = -1;
    } else {
      s = int32_t(mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows));
    }
    s_slot[r] = s;
  }
  __syncthreads();
}

// A row whose slot a later row has too is not written: a wave per row compares it
// with all later slots.  (n <= CR_SMALL: one launch instead of three.)
__device__ __forceinline__ void cr_search(const CacheArgs& a, int64_t row0, int rows, int32_t* s_slot) {
  __shared__ int32_t s_all[CR_SMALL];
  const int n = int(a.n), lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < n; i += CR_THREADS)
    s_all[i] = int32_t(mx_slot(a.ids[i], a.id_bound, a.slot_map, a.cache_rows));
  __syncthreads();
  for (int r = threadIdx.x >> 6; r < rows; r += CR_THREADS / 64) {
    const int i = int(row0) + r, s = s_all[i];
    bool later = false;
    for (int j = i + 1 + lane; j < n; j += 64) later |= s_all[j] == s;
    later = __any(later);
    if (lane == 0) s_slot[r] = later ? -1 : s;
  }
  __syncthreads();
}

template <typename T, int FMT>
__global__ void __launch_bounds__(CR_THREADS) k_cache_write(CacheArgs a) {
  constexpr int N = CHUNK<T>, GL = MX_GROUP / N;         // elements per piece, pieces per group
  constexpr int PB = FMT == FAST_MXFP4 ? N / 2 : N;      // bytes of a piece's codes
  __shared__ int32_t s_slot[CR_ROWS];
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows), total = rows * a.upr;
  if (a.search) cr_search(a, row0, rows, s_slot);
  else cr_slots(a, row0, rows, s_slot);
  const T* src = static_cast<const T*>(a.src) + row0 * a.rec.parts * a.rec.width;
  int slot[CR_UNROLL], part[CR_UNROLL], c[CR_UNROLL];
  float x[CR_UNROLL][N];
#pragma unroll
  for (int k = 0; k < CR_UNROLL; ++k) {
    const int t = threadIdx.x + (blockIdx.y * CR_UNROLL + k) * CR_THREADS;
    slot[k] = -1;
    if (t < total) {                 // whole groups of lanes: upp is a multiple of GL
      const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
      part[k] = int(div_small(u, a.mag_upp));
      c[k] = u - part[k] * a.upp;
      slot[k] = s_slot[r];
      if (slot[k] >= 0)
        load_chunk(src + int64_t(r * a.rec.parts + part[k]) * a.rec.width + c[k] * N, a.rec.width - c[k] * N, x[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < CR_UNROLL; ++k) {
    if (slot[k] < 0) continue;       // the lanes of a group share a row
    // magnitudes as integers: their order is that of the values, NaN the largest
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t b = __float_as_uint(x[k][j]) & 0x7fffffffu;
      m = m > b ? m : b;
    }
    uint32_t o = __float_as_uint(dpp_quad_xor1(__uint_as_float(m)));
    m = m > o ? m : o;
    o = __float_as_uint(dpp_quad_xor2(__uint_as_float(m)));
    m = m > o ? m : o;
    if constexpr (GL == 8) {
      o = __float_as_uint(dpp_row_half_mirror(__uint_as_float(m)));
      m = m > o ? m : o;
    }
    const uint32_t sb = mx_scale_byte<FMT>(__uint_as_float(m));
    if (sb == MX_TOP_BYTE<FMT>) {    // finite rows read back finite
#pragma unroll
      for (int j = 0; j < N; ++j) x[k][j] = fminf(fmaxf(x[k][j], -MX_TOP<FMT>), MX_TOP<FMT>);
    }
    MxPiece<FMT, N> p;
    if (sb == 255u) p.zero();
    else p.pack(mx_scale(sb), x[k]);
    uint8_t* rec = a.cache + int64_t(slot[k]) * a.rec.stride;
    if (c[k] * PB < a.rec.code_bytes) p.store(rec + part[k] * a.rec.code_bytes + c[k] * PB);
    if (c[k] % GL == 0) rec[a.rec.scale_off + part[k] * a.rec.groups + c[k] / GL] = uint8_t(sb);
  }
}

template <typename T, int FMT, bool NT>
__global__ void __launch_bounds__(CR_THREADS) k_cache_gather(CacheArgs a) {
  constexpr int N = CHUNK<T>, GL = MX_GROUP / N;
  constexpr int PB = FMT == FAST_MXFP4 ? N / 2 : N;
  __shared__ int32_t s_slot[CR_ROWS];
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows), total = rows * a.upr;
  cr_slots(a, row0, rows, s_slot);
  T* dst = static_cast<T*>(a.dst) + row0 * a.rec.parts * a.rec.width;
  MxPiece<FMT, N> p[CR_UNROLL];
  uint32_t sb[CR_UNROLL];
  int at[CR_UNROLL], left[CR_UNROLL];
#pragma unroll
  for (int k = 0; k < CR_UNROLL; ++k) {
    const int t = threadIdx.x + (blockIdx.y * CR_UNROLL + k) * CR_THREADS;
    left[k] = 0;
    if (t < total) {
      const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
      const int part = int(div_small(u, a.mag_upp)), c = u - part * a.upp, slot = s_slot[r];
      if (slot >= 0) {
        const uint8_t* rec = a.cache_in + int64_t(slot) * a.rec.stride;
        p[k].load(rec + part * a.rec.code_bytes + c * PB);
        sb[k] = rec[a.rec.scale_off + part * a.rec.groups + c / GL];
        at[k] = (r * a.rec.parts + part) * a.rec.width + c * N;
        left[k] = a.rec.width - c * N;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < CR_UNROLL; ++k) {
    if (left[k] <= 0) continue;
    float x[N];
    p[k].unpack(mx_scale(sb[k]), x);
    store_chunk<T, NT>(dst + at[k], left[k], x);
  }
}

static fast_status_t cache_check(const char* fn, const int64_t* ids, int64_t n, int64_t id_bound,
                                 const int32_t* slot_map, int parts, int width, fast_dtype_t dtype,
                                 const void* rows, fast_cache_format_t fmt, const void* cache,
                                 int64_t cache_rows) {
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
  if (!aligned(slot_map, 4)) return fail(FAST_ERR_UNSUPPORTED, "%s: slot_map not 4-byte aligned", fn);
  return FAST_OK;
}

static CacheArgs cache_args(const int64_t* ids, int64_t n, int64_t id_bound, const int32_t* slot_map,
                            int parts, int width, fast_cache_format_t fmt, int64_t cache_rows,
                            fast_dtype_t dtype, bool write) {
  CacheArgs a = {};
  a.ids = ids;
  a.n = n;
  a.id_bound = id_bound;
  a.slot_map = slot_map;
  a.cache_rows = cache_rows;
  a.rec = mx_record(parts, width, fmt);
  const int piece = dtype == FAST_F32 ? CHUNK<float> : CHUNK<uint16_t>;
  // a read moves the pieces that hold elements, a write whole groups of them
  a.upp = write ? a.rec.groups * (MX_GROUP / piece) : (width + piece - 1) / piece;
  a.upr = a.upp * parts;
  a.rows = a.upr < CR_TILE ? CR_TILE / a.upr : 1;
  if (a.rows > CR_ROWS) a.rows = CR_ROWS;
  a.mag_upr = div_magic(a.upr);
  a.mag_upp = div_magic(a.upp);
  return a;
}

// Workgroups over the rows, and over the pieces of rows that are more than one tile.
static dim3 cache_grid(const CacheArgs& a) {
  return dim3(uint32_t((a.n + a.rows - 1) / a.rows), uint32_t((a.rows * a.upr + CR_TILE - 1) / CR_TILE));
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
  // owners, then slots
  return align_up(size_t(cache_rows > 0 ? cache_rows : 1) * sizeof(int32_t), 16) +
         align_up(size_t(n) * sizeof(int32_t), 16);
}

extern "C" fast_status_t fast_cache_write(const int64_t* ids, int64_t n, int64_t id_bound,
                                          const int32_t* slot_map, int parts, int width,
                                          fast_dtype_t dtype, const void* src,
                                          fast_cache_format_t format, void* cache,
                                          int64_t cache_rows, int distinct, void* ws,
                                          size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_cache_write";
  const fast_status_t s = cache_check(fn, ids, n, id_bound, slot_map, parts, width, dtype, src, format,
                                      cache, cache_rows);
  if (s != FAST_OK) return s;
  if (n == 0 || cache_rows == 0) return ok();
  if (!distinct) {
    if (!ws || ws_bytes < fast_cache_write_workspace(n, cache_rows))
      return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0,
                  fast_cache_write_workspace(n, cache_rows));
    if (!aligned(ws, 16)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 16-byte aligned", fn);
  }
  CacheArgs a = cache_args(ids, n, id_bound, slot_map, parts, width, format, cache_rows, dtype, true);
  const dim3 grid = cache_grid(a);
  if (!grid_fits(grid.x, CR_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  a.src = src;
  a.cache = static_cast<uint8_t*>(cache);
  hipStream_t st = static_cast<hipStream_t>(stream);
  a.search = !distinct && n <= CR_SMALL;
  if (!distinct && !a.search) {
    a.owner = static_cast<int32_t*>(ws);
    a.slots = a.owner + align_up(size_t(cache_rows) * sizeof(int32_t), 16) / sizeof(int32_t);
    const uint32_t g = uint32_t((n + CR_THREADS - 1) / CR_THREADS);
    hipLaunchKernelGGL(k_cache_claim, dim3(g), dim3(CR_THREADS), 0, st, a, 0);
    hipLaunchKernelGGL(k_cache_claim, dim3(g), dim3(CR_THREADS), 0, st, a, 1);
  }
#define FAST_CW(T, F) hipLaunchKernelGGL((k_cache_write<T, F>), grid, dim3(CR_THREADS), 0, st, a)
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
  const fast_status_t s = cache_check(fn, ids, n, id_bound, slot_map, parts, width, dtype, rows, format,
                                      cache, cache_rows);
  if (s != FAST_OK) return s;
  if (n == 0 || cache_rows == 0) return ok();
  CacheArgs a = cache_args(ids, n, id_bound, slot_map, parts, width, format, cache_rows, dtype, false);
  a.dst = rows;
  a.cache_in = static_cast<const uint8_t*>(cache);
  const dim3 grid = cache_grid(a);
  if (!grid_fits(grid.x, CR_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // Rows that would fill a good part of the 256 MB last-level cache are streamed past it:
  // 1.3 M rows of 172 fp32 from 8 bits 280 -> 208 us; write and read of 300,000 rows of
  // 256 bf16 (154 MB) 93 -> 71.
  const bool nt = n * int64_t(parts) * width * elem_size(dtype) > (int64_t(64) << 20);
#define FAST_CG(T, F)                                                                                  \
  do {                                                                                                 \
    if (nt) hipLaunchKernelGGL((k_cache_gather<T, F, true>), grid, dim3(CR_THREADS), 0, st, a);        \
    else hipLaunchKernelGGL((k_cache_gather<T, F, false>), grid, dim3(CR_THREADS), 0, st, a);          \
  } while (0)
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
