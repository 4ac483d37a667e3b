// layer_norm.hip -- layer norm of rows, forward and backward.
//   h = x + res,  mu = mean(h),  r = 1 / sqrt(mean((h - mu)^2) + eps)
//   y = (h - mu) r gamma + beta
//   backward, with xhat = (h - mu) r and g = dy gamma:
//     dx = r (g - mean(g) - xhat mean(g xhat)) + dsum,
//     dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// Bound by HBM (about 10 flop per element moved): 40,000 rows of 2048 fp32 with residual and
// sum, forward 217 us = 6.0 TB/s, backward 247 = 5.3.  A group of G lanes (a power
// of two up to a wave; a whole workgroup for the widest rows) holds a row in
// registers, P chunks of 16 bytes a lane, so the mean and then the sum of the
// squared distances from it are formed from one read of the row.  Row sums go
// through the lanes by DPP and permlane swaps, fp32.
//
// The backward walks several rows per group: a lane owns the same columns of every
// row, so the terms of dgamma and dbeta are added in its registers, at most
// LN_ROWS of them in fp32; a workgroup joins its groups in fp64 in LDS and
// writes one partial row, and a second launch adds the partial rows in fp64 in
// their order (one workgroup writes the sums itself).  No atomics: repeated calls give the same bits.
#include <algorithm>

#include "rows.h"

namespace fast {

constexpr int LN_THREADS = 256;  // of a workgroup that holds several groups
constexpr int LN_MAX_G = 1024;   // lanes of a group, at most
constexpr int LN_ELEMS = 16;     // elements of a row per lane, at most
constexpr int64_t LN_BLOCKS = 1024;   // workgroups of the backward, about
constexpr int LN_ROWS = 32;      // rows that a lane adds up in fp32, at most
constexpr int64_t LN_ALONE = 2;  // rows per group up to which one workgroup does the backward
constexpr int64_t LN_MAX_D = 8192;

// Sums over the G lanes of a group; G > 64: over the workgroup, through
// one of two LDS buffers in turn, so that one barrier per sum is enough (a
// wave that writes a buffer again has passed the barrier behind its last readers).
struct LnSum {
  float2* buf;
  int turn;
};
__device__ __forceinline__ float2 row_sums(float x, float y, int G, LnSum& s) {
  if (G <= 64) return make_float2(group_sum(x, G), group_sum(y, G));
  x = group_sum(x, 64);
  y = group_sum(y, 64);
  float2* b = s.buf + s.turn * (LN_MAX_G / 64);
  s.turn ^= 1;
  if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = make_float2(x, y);
  __syncthreads();
  float2 t = make_float2(0.f, 0.f);
  for (int w = 0; w < G / 64; ++w) {
    t.x += b[w].x;
    t.y += b[w].y;
  }
  return t;
}

struct LnArgs {
  int64_t n;
  int D, G;
  const void* x;
  const void* res;
  const float* gamma;
  const float* beta;
  float eps;
  void* y;
  void* sum;
  float* mean;
  float* rstd;
};

// A lane's chunk p of a row.  Of a row that is no multiple of 16 bytes (TAIL) the last chunk
// starts early enough to end with it: its first `skip` elements are the
// neighbour's, and count once; loading the rest of a row one by one took 1.5 times as
// long (200,000 x 172 bf16).  Rows of less than 16 bytes are one partial chunk.
template <int VE, bool TAIL>
struct LnChunk {
  int first, n, skip;                // elements [first, first + n), n <= 0: none
  __device__ LnChunk(int c, int D) {
    first = c * VE;
    n = D - first;
    skip = 0;
    if constexpr (TAIL) {
      if (n > 0 && n < VE && D >= VE) {
        skip = VE - n;
        first = D - VE;
        n = VE;
      }
    } else if (n > VE) {
      n = VE;
    }
  }
  __device__ bool own(int j) const { return TAIL ? j >= skip && j < n : n > 0; }
};
template <typename T, bool TAIL, bool NT>
__device__ __forceinline__ void ln_load(const T* row, const LnChunk<CHUNK<T>, TAIL>& c, float* x) {
  if (TAIL || c.n > 0) {
    load_chunk<T, NT>(row + c.first, c.n, x);
  } else {
#pragma unroll
    for (int j = 0; j < CHUNK<T>; ++j) x[j] = 0.f;
  }
}
template <typename T, bool TAIL, bool NT>
__device__ __forceinline__ void ln_store(T* row, const LnChunk<CHUNK<T>, TAIL>& c, const float* x) {
  if (c.n > 0) store_chunk<T, NT>(row + c.first, c.n, x);
}
// The chunk's columns of an fp32 vector, `fill` where it is NULL.
template <int VE, bool TAIL>
__device__ __forceinline__ void ln_cols(const float* v, float fill, const LnChunk<VE, TAIL>& c, float* x) {
#pragma unroll
  for (int j = 0; j < VE; j += 4) {
    if (v) {
      load_chunk(v + c.first + j, c.n - j, x + j);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) x[j + k] = fill;
    }
  }
}

template <typename T, int P, bool TAIL, bool NT>
__global__ void __launch_bounds__(LN_MAX_G) k_ln_fwd(LnArgs a) {
  constexpr int VE = CHUNK<T>;
  typedef LnChunk<VE, TAIL> Chunk;
  __shared__ float2 s_red[2 * (LN_MAX_G / 64)];
  LnSum red = {s_red, 0};
  const int G = a.G, lane = threadIdx.x & (G - 1), sub = threadIdx.x / G;
  const int64_t row = int64_t(blockIdx.x) * (int(blockDim.x) / G) + sub;
  if (row >= a.n) return;               // whole groups; a workgroup-wide row always exists
  const int D = a.D;
  float h[P][VE], g[P][VE], b[P][VE];
#pragma unroll
  for (int p = 0; p < P; ++p)
    ln_load<T, TAIL, NT>(static_cast<const T*>(a.x) + row * D, Chunk(lane + p * G, D), h[p]);
  if (a.res) {
    float t[P][VE];
#pragma unroll
    for (int p = 0; p < P; ++p)
      ln_load<T, TAIL, NT>(static_cast<const T*>(a.res) + row * D, Chunk(lane + p * G, D), t[p]);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        h[p][j] += t[p][j];
        // the statistics are those of the stored row, which the backward reads
        if constexpr (sizeof(T) == 2) h[p][j] = __uint_as_float(bf16_rne(h[p][j]) << 16);
      }
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    ln_cols(a.gamma, 1.f, Chunk(lane + p * G, D), g[p]);
    ln_cols(a.beta, 0.f, Chunk(lane + p * G, D), b[p]);
  }
  float s = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Chunk c(lane + p * G, D);
#pragma unroll
    for (int j = 0; j < VE; ++j) s += !TAIL || c.own(j) ? h[p][j] : 0.f;   // zeros past the row
  }
  const float mean = row_sums(s, 0.f, G, red).x / float(D);
  // the row has been read by every lane: sum and y may take the place of x or res
  if (a.sum) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      ln_store<T, TAIL, NT>(static_cast<T*>(a.sum) + row * D, Chunk(lane + p * G, D), h[p]);
  }
  float q = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Chunk c(lane + p * G, D);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float d = c.own(j) ? h[p][j] - mean : 0.f;
      q = fmaf(d, d, q);
    }
  }
  const float rstd = 1.f / sqrtf(row_sums(q, 0.f, G, red).x / float(D) + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int j = 0; j < VE; ++j) g[p][j] = fmaf((h[p][j] - mean) * rstd, g[p][j], b[p][j]);
    ln_store<T, TAIL, NT>(static_cast<T*>(a.y) + row * D, Chunk(lane + p * G, D), g[p]);
  }
}

struct LnBwdArgs {
  int64_t n;
  int D, G;
  const void* h;
  const float* gamma;
  const float* mean;
  const float* rstd;
  const void* dy;
  const void* dsum;
  void* dx;
  float* part;         // [workgroups][2][D], or NULL: dx only, or one workgroup
  float* dgamma;       // one workgroup: the sums themselves, each may be NULL
  float* dbeta;
};

template <typename T, int P, bool TAIL, bool NT>
__global__ void __launch_bounds__(LN_MAX_G) k_ln_bwd(LnBwdArgs a) {
  constexpr int VE = CHUNK<T>;
  typedef LnChunk<VE, TAIL> Chunk;
  __shared__ float2 s_red[2 * (LN_MAX_G / 64)];
  LnSum red = {s_red, 0};
  extern __shared__ float s_col[];      // [groups][2][D] where the workgroup holds several groups
  const int G = a.G, lane = threadIdx.x & (G - 1), sub = threadIdx.x / G, groups = blockDim.x / G;
  const int D = a.D;
  // rows b, b + workgroups, ... (in units of a workgroup's groups), so that the chip reads
  // one stretch of memory at a time: 281 -> 272 us against a stretch per workgroup
  // (40,000 x 2048 fp32)
  const int64_t r0 = int64_t(blockIdx.x) * groups, step = int64_t(gridDim.x) * groups;
  float ga[P][VE], dg[P][VE], db[P][VE];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    ln_cols(a.gamma, 1.f, Chunk(lane + p * G, D), ga[p]);
#pragma unroll
    for (int j = 0; j < VE; ++j) dg[p][j] = db[p][j] = 0.f;
  }
  const float inv = 1.f / float(D);
  for (int64_t row = r0 + sub; row < a.n; row += step) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    float xh[P][VE], dy[P][VE], d[P][VE];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const Chunk c(lane + p * G, D);
      ln_load<T, TAIL, NT>(static_cast<const T*>(a.h) + row * D, c, xh[p]);
      ln_load<T, TAIL, NT>(static_cast<const T*>(a.dy) + row * D, c, dy[p]);   // zeros past the row
    }
    if (a.dsum) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        ln_load<T, TAIL, NT>(static_cast<const T*>(a.dsum) + row * D, Chunk(lane + p * G, D), d[p]);
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < VE; ++j) d[p][j] = 0.f;
    }
    // dx may take dsum's place, and a last chunk reads elements that another wave writes: they
    // have arrived before the barrier in row_sums lets that wave go on
    if constexpr (TAIL) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < VE; ++j) asm volatile("" : "+v"(d[p][j]));
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const Chunk c(lane + p * G, D);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        xh[p][j] = (xh[p][j] - mean) * rstd;
        dg[p][j] = fmaf(dy[p][j], xh[p][j], dg[p][j]);
        db[p][j] += dy[p][j];
        dy[p][j] *= ga[p][j];
        const float g = !TAIL || c.own(j) ? dy[p][j] : 0.f;
        s1 += g;
        s2 = fmaf(g, xh[p][j], s2);
      }
    }
    const float2 st = row_sums(s1, s2, G, red);
    s1 = st.x * inv;
    s2 = st.y * inv;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int j = 0; j < VE; ++j) d[p][j] = fmaf(rstd, dy[p][j] - s1 - xh[p][j] * s2, d[p][j]);
      ln_store<T, TAIL, NT>(static_cast<T*>(a.dx) + row * D, Chunk(lane + p * G, D), d[p]);
    }
  }
  float* og = a.part ? a.part + int64_t(blockIdx.x) * 2 * D : a.dgamma;
  float* ob = a.part ? og + D : a.dbeta;
  if (!og && !ob) return;
  if (groups == 1) {                     // the lanes of the workgroup own different columns
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const Chunk k(lane + p * G, D);
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (k.own(j)) {
          if (og) og[k.first + j] = dg[p][j];
          if (ob) ob[k.first + j] = db[p][j];
        }
    }
    return;
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const Chunk k(lane + p * G, D);
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (k.own(j)) {
        s_col[2 * sub * D + k.first + j] = dg[p][j];
        s_col[(2 * sub + 1) * D + k.first + j] = db[p][j];
      }
  }
  __syncthreads();
  for (int col = threadIdx.x; col < 2 * D; col += LN_THREADS) {   // the groups in order
    double t = 0.0;
#pragma unroll 8
    for (int k = 0; k < groups; ++k) t += s_col[2 * k * D + col];
    float* o = col < D ? og : ob;
    if (o) o[col < D ? col : col - D] = float(t);
  }
}

// dgamma and dbeta from the partial rows, added in fp64 in a fixed order: LNS_ROWS
// threads per column take every LNS_ROWS-th row, then one adds theirs.
constexpr int LNS_THREADS = 1024, LNS_COLS = 16, LNS_ROWS = LNS_THREADS / LNS_COLS;
__global__ void __launch_bounds__(LNS_THREADS) k_ln_bwd_sum(const float* __restrict__ part, int64_t nb,
                                                            int D, float* __restrict__ dgamma,
                                                            float* __restrict__ dbeta) {
  __shared__ double s[LNS_ROWS][LNS_COLS];
  const int col = threadIdx.x % LNS_COLS, r = threadIdx.x / LNS_COLS;
  const int c = blockIdx.x * LNS_COLS + col;         // of 2 D columns
  double t = 0.0;
  if (c < 2 * D) {
#pragma unroll 8
    for (int64_t b = r; b < nb; b += LNS_ROWS) t += part[b * 2 * D + c];
  }
  s[r][col] = t;
  __syncthreads();
  for (int h = LNS_ROWS / 2; h > 0; h /= 2) {
    if (r < h) s[r][col] += s[r + h][col];
    __syncthreads();
  }
  if (r == 0 && c < 2 * D) {
    float* o = c < D ? dgamma : dbeta;
    if (o) o[c < D ? c : c - D] = float(s[0][col]);
  }
}

struct LnPlan {
  int G, P;            // lanes per row, chunks per lane
  int threads;         // per workgroup: one group of more than a wave, or several
  int64_t nb;          // backward: workgroups
};

// The group with the fewest idle chunk slots that holds a row in at most LN_ELEMS
// elements a lane, and the fewest of those.  Fewer registers keep more rows in flight: 40,000
// rows of 2048 fp32, backward 444 us with a wave per row (32 elements a lane), 281 with
// 256 lanes (8); 200,000 rows of 172 bf16, 8 lanes of 24 elements 136, 32 of 8 78.
static LnPlan ln_plan(int64_t n, int D, int ve) {
  LnPlan L = {};
  const int C = (D + ve - 1) / ve;
  int best = 1 << 30;
  for (int G = 1; G <= LN_MAX_G; G *= 2)
    for (int P = 1; P <= LN_ELEMS / ve; ++P)
      if (G * P >= C && (G * P < best || (G * P == best && P < L.P))) {
        best = G * P;
        L.G = G;
        L.P = P;
      }
  L.threads = L.G > 64 ? L.G : LN_THREADS;
  // 4 workgroups per CU (4 / 6 / 8 / 16: 15.2 / 17.7 / 17.7 / 19.0 us for 66,000 rows of 128
  // bf16, and 4.0 to 5.6 for the partial rows' sums), and at most LN_ROWS rows per group
  const int64_t groups = L.threads / L.G;
  int64_t per = (n + LN_BLOCKS * groups - 1) / (LN_BLOCKS * groups);
  per = per < 1 ? 1 : (per > LN_ROWS ? LN_ROWS : per);
  L.nb = (n + per * groups - 1) / (per * groups);
  // Few rows: one workgroup, which writes the sums itself; both directions of 4 rows
  // of 54 fp32 in two launches 5.2 us, in three 7.3.  2 / 4 rows per group: 32 / 64 rows of 172
  // fp32 8.8 / 11.3, with more workgroups and a launch for their sums 9.8 / 9.7.
  if (n <= LN_ALONE * groups) L.nb = 1;
  return L;
}

// Stream rows that cover whole cache lines when a pass moves more than the 256 MB
// last-level cache holds: 40,000 x 2048 fp32, forward 223 -> 217 us, backward 272 ->
// 247; 66,000 x 128 bf16 (135 MB for both directions) 14.8 -> 14.7, 20.0 -> 21.9.
static bool ln_stream(int64_t n, int D, size_t es, int arrays, const void* const* rows, int count) {
  if ((D * es) % CACHE_LINE != 0 || n * int64_t(D * es) * arrays <= (int64_t(256) << 20)) return false;
  for (int k = 0; k < count; ++k)
    if (!aligned(rows[k], CACHE_LINE)) return false;
  return true;
}

template <typename T, bool TAIL, bool NT>
static void launch_ln(const LnArgs& a, const LnPlan& L, uint32_t grid, size_t, hipStream_t st) {
  static_assert(LN_ELEMS == 16, "chunks per lane: 1 to 4 of fp32, 1 or 2 of bf16");
#define FAST_LN(p) hipLaunchKernelGGL((k_ln_fwd<T, p, TAIL, NT>), dim3(grid), dim3(L.threads), 0, st, a)
  if (L.P == 1) FAST_LN(1);
  else if (L.P == 2) FAST_LN(2);
  else if constexpr (sizeof(T) == 4) {
    if (L.P == 3) FAST_LN(3);
    else FAST_LN(4);
  }
#undef FAST_LN
}
template <typename T, bool TAIL, bool NT>
static void launch_ln(const LnBwdArgs& a, const LnPlan& L, uint32_t grid, size_t lds, hipStream_t st) {
#define FAST_LN(p) hipLaunchKernelGGL((k_ln_bwd<T, p, TAIL, NT>), dim3(grid), dim3(L.threads), lds, st, a)
  if (L.P == 1) FAST_LN(1);
  else if (L.P == 2) FAST_LN(2);
  else if constexpr (sizeof(T) == 4) {
    if (L.P == 3) FAST_LN(3);
    else FAST_LN(4);
  }
#undef FAST_LN
}
// Streamed rows cover whole cache lines, so they have no tail.
template <typename Args>
static void launch_ln(const Args& a, const LnPlan& L, uint32_t grid, size_t lds, fast_dtype_t dtype, bool nt,
                      hipStream_t st) {
  const bool tail = a.D % (dtype == FAST_F32 ? CHUNK<float> : CHUNK<uint16_t>) != 0;
  if (dtype == FAST_F32) {
    if (nt) launch_ln<float, false, true>(a, L, grid, lds, st);
    else if (tail) launch_ln<float, true, false>(a, L, grid, lds, st);
    else launch_ln<float, false, false>(a, L, grid, lds, st);
  } else {
    if (nt) launch_ln<uint16_t, false, true>(a, L, grid, lds, st);
    else if (tail) launch_ln<uint16_t, true, false>(a, L, grid, lds, st);
    else launch_ln<uint16_t, false, false>(a, L, grid, lds, st);
  }
}

static fast_status_t ln_check(const char* fn, int64_t n, int D, fast_dtype_t dtype) {
  if (n < 0) return fail(FAST_ERR_INVALID_ARG, "%s: n = %lld < 0", fn, (long long)n);
  if (D <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: D = %d <= 0", fn, D);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (D > LN_MAX_D) return fail(FAST_ERR_UNSUPPORTED, "%s: D = %d > %lld", fn, D, (long long)LN_MAX_D);
  if (n >= (int64_t(1) << 31)) return fail(FAST_ERR_UNSUPPORTED, "%s: n >= 2^31", fn);
  return FAST_OK;
}

}  // namespace fast

using namespace fast;

extern "C" fast_status_t fast_layer_norm_fwd(int64_t n, int D, fast_dtype_t dtype, const void* x,
                                             const void* res, const float* gamma,
                                             const float* beta, float eps, void* y, void* sum,
                                             float* mean, float* rstd, fast_stream_t stream) {
  const char* fn = "fast_layer_norm_fwd";
  const fast_status_t s = ln_check(fn, n, D, dtype);
  if (s != FAST_OK) return s;
  if (!(eps >= 0.f)) return fail(FAST_ERR_INVALID_ARG, "%s: eps is negative or not a number", fn);
  if (sum && !res) return fail(FAST_ERR_INVALID_ARG, "%s: sum without res", fn);
  if (sum && sum == y) return fail(FAST_ERR_INVALID_ARG, "%s: y and sum are one array", fn);
  if (n == 0) return ok();
  if (!x || !y) return fail(FAST_ERR_INVALID_ARG, "%s: NULL x/y", fn);
  const size_t es = elem_size(dtype);
  if (!aligned(x, es) || !aligned(res, es) || !aligned(y, es) || !aligned(sum, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: gamma/beta/mean/rstd not 4-byte aligned", fn);
  const int64_t bytes = n * D * int64_t(es);
  if (shifted(y, x, bytes) || shifted(y, res, bytes) || shifted(sum, x, bytes) || shifted(sum, res, bytes) ||
      shifted(y, sum, bytes))
    return fail(FAST_ERR_INVALID_ARG, "%s: y or sum overlaps x, res or the other, shifted", fn);
  const LnPlan L = ln_plan(n, D, 16 / int(es));
  const LnArgs a = {n, D, L.G, x, res, gamma, beta, eps, y, sum, mean, rstd};
  const int64_t per = L.threads / L.G;
  const uint32_t grid = uint32_t((n + per - 1) / per);
  if (!grid_fits(grid, L.threads)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const void* rows[] = {x, res, y, sum};
  const bool nt = ln_stream(n, D, es, 2 + (res != nullptr) + (sum != nullptr), rows, 4);
  launch_ln(a, L, grid, 0, dtype, nt, st);
  return check_launch(fn);
}

extern "C" size_t fast_layer_norm_bwd_workspace(int64_t n, int D) {
  if (n < 0 || n >= (int64_t(1) << 31) || D <= 0 || D > LN_MAX_D) return 0;
  // for either type, the most workgroups of up to n rows: it grows with n, so that one for
  // the largest call serves all
  int64_t nb = 1;
  for (int ve = 4; ve <= 8; ve += 4) {
    const LnPlan L = ln_plan(n, D, ve);
    const int64_t units = (n + L.threads / L.G - 1) / (L.threads / L.G);
    nb = std::max({nb, L.nb, std::min(units, LN_BLOCKS)});
  }
  return size_t(nb) * 2 * D * sizeof(float);
}

extern "C" fast_status_t fast_layer_norm_bwd(int64_t n, int D, fast_dtype_t dtype, const void* h,
                                             const float* gamma, const float* mean,
                                             const float* rstd, const void* dy, const void* dsum,
                                             void* dx, float* dgamma, float* dbeta, void* ws,
                                             size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_layer_norm_bwd";
  const fast_status_t s = ln_check(fn, n, D, dtype);
  if (s != FAST_OK) return s;
  const bool sums = dgamma || dbeta;
  if (n > 0 && (!h || !mean || !rstd || !dy || !dx))
    return fail(FAST_ERR_INVALID_ARG, "%s: NULL h/mean/rstd/dy/dx", fn);
  const size_t es = elem_size(dtype);
  if (!aligned(h, es) || !aligned(dy, es) || !aligned(dsum, es) || !aligned(dx, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) ||
      !aligned(dbeta, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: gamma/mean/rstd/dgamma/dbeta not 4-byte aligned", fn);
  const int64_t bytes = n * D * int64_t(es);
  if (shifted(dx, h, bytes) || shifted(dx, dy, bytes) || shifted(dx, dsum, bytes))
    return fail(FAST_ERR_INVALID_ARG, "%s: dx overlaps h, dy or dsum, shifted", fn);
  if (sums) {
    if (!ws || ws_bytes < fast_layer_norm_bwd_workspace(n, D))
      return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0,
                  fast_layer_norm_bwd_workspace(n, D));
    if (!aligned(ws, 8)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 8-byte aligned", fn);
  }
  if (n == 0 && !sums) return ok();
  const LnPlan L = ln_plan(n, D, 16 / int(es));
  if (!grid_fits(L.nb, L.threads)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n > 0) {
    const LnBwdArgs a = {n, D, L.G, h, gamma, mean, rstd, dy, dsum, dx,
                         sums && L.nb > 1 ? static_cast<float*>(ws) : nullptr, dgamma, dbeta};
    // at most 32 KB: a lane owns at most LN_ELEMS columns
    const size_t lds = sums && L.G < L.threads ? size_t(L.threads / L.G) * 2 * D * sizeof(float) : 0;
    const void* rows[] = {h, dy, dsum, dx};
    const bool nt = ln_stream(n, D, es, 3 + (dsum != nullptr), rows, 4);
    launch_ln(a, L, uint32_t(L.nb), lds, dtype, nt, st);
  }
  if (sums && (n == 0 || L.nb > 1))
    hipLaunchKernelGGL(k_ln_bwd_sum, dim3((2 * D + LNS_COLS - 1) / LNS_COLS), dim3(LNS_THREADS), 0, st,
                       static_cast<const float*>(ws), n > 0 ? L.nb : 0, D, dgamma, dbeta);
  return check_launch(fn);
}
