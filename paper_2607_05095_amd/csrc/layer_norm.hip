// layer_norm.hip -- layer norm of rows, forward and backward.
//   h = x + res,  mu = mean(h),  r = 1 / sqrt(mean((h - mu)^2) + eps)
//   y = (h - mu) r gamma + beta
//   backward, with xhat = (h - mu) r and g = dy gamma:
//     dx = r (g - mean(g) - xhat mean(g xhat)) + dsum,
//     dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// Bound by HBM (about 10 flop per element moved).  A group of G lanes (a power
// of two up to a wave; a whole workgroup for the widest rows) holds a row in
// registers, P chunks of 16 bytes a lane, so the mean and then the sum of the
// squared distances from it are formed from one read of the row.  Row sums go
// through the lanes by DPP and permlane swaps, fp32.
//
// The backward walks several rows per group: a lane owns the same columns of every
// row, so the terms of dgamma and dbeta are added in its registers, at most
// LN_ROWS of them in fp32; a workgroup joins its groups in fp64 in LDS and
// writes one partial row, and a second launch adds the partial rows in fp64 in
// their order.  No atomics: repeated calls give the same bits.
#include "rows.h"

namespace fast {

constexpr int LN_THREADS = 256;
constexpr int LN_MAX_P = 8;      // chunks of a row per lane, at most
constexpr int LN_ROWS = 32;      // rows that a lane adds up in fp32, at most
constexpr int64_t LN_MAX_D = int64_t(LN_THREADS) * LN_MAX_P * 4;   // 8192

// Sum over the G lanes of a group; G = LN_THREADS: over the workgroup.
__device__ __forceinline__ float row_sum(float x, int G, float* s_red) {
  if (G <= 64) return group_sum(x, G);
  x = group_sum(x, 64);
  __syncthreads();                       // the last sum's readers are done
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = x;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < LN_THREADS / 64; ++w) t += s_red[w];
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

template <typename T, int P>
__global__ void __launch_bounds__(LN_THREADS) k_ln_fwd(LnArgs a) {
  constexpr int VE = CHUNK<T>;
  __shared__ float s_red[LN_THREADS / 64];
  const int G = a.G, lane = threadIdx.x & (G - 1), sub = threadIdx.x / G;
  const int64_t row = int64_t(blockIdx.x) * (LN_THREADS / G) + sub;
  if (row >= a.n) return;               // whole groups; a workgroup-wide row always exists
  const int D = a.D;
  const T* x = static_cast<const T*>(a.x) + row * D;
  float h[P][VE];
  float s = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) load_chunk(x + (lane + p * G) * VE, D - (lane + p * G) * VE, h[p]);
  if (a.res) {
    const T* r = static_cast<const T*>(a.res) + row * D;
    float t[P][VE];
#pragma unroll
    for (int p = 0; p < P; ++p) load_chunk(r + (lane + p * G) * VE, D - (lane + p * G) * VE, t[p]);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        h[p][j] += t[p][j];
        // the statistics are those of the stored row, which the backward reads
        if constexpr (sizeof(T) == 2) h[p][j] = __uint_as_float(bf16_rne(h[p][j]) << 16);
      }
    if (a.sum) {
      T* o = static_cast<T*>(a.sum) + row * D;
#pragma unroll
      for (int p = 0; p < P; ++p) store_chunk(o + (lane + p * G) * VE, D - (lane + p * G) * VE, h[p]);
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < VE; ++j) s += h[p][j];
  const float mean = row_sum(s, G, s_red) / float(D);
  float q = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float c = (lane + p * G) * VE + j < D ? h[p][j] - mean : 0.f;
      q = fmaf(c, c, q);
    }
  const float rstd = 1.f / sqrtf(row_sum(q, G, s_red) / float(D) + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* y = static_cast<T*>(a.y) + row * D;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c0 = (lane + p * G) * VE;
    float g[VE], b[VE];
#pragma unroll
    for (int j = 0; j < VE; j += 4) {
      if (a.gamma) load_chunk(a.gamma + c0 + j, D - c0 - j, g + j);
      else for (int k = 0; k < 4; ++k) g[j + k] = 1.f;
      if (a.beta) load_chunk(a.beta + c0 + j, D - c0 - j, b + j);
      else for (int k = 0; k < 4; ++k) b[j + k] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) g[j] = fmaf((h[p][j] - mean) * rstd, g[j], b[j]);
    store_chunk(y + c0, D - c0, g);
  }
}

struct LnBwdArgs {
  int64_t n;
  int D, G;
  int64_t rows;        // rows per workgroup
  const void* h;
  const float* gamma;
  const float* mean;
  const float* rstd;
  const void* dy;
  const void* dsum;
  void* dx;
  double* part;        // [workgroups][2][D], or NULL: dx only
};

template <typename T, int P>
__global__ void __launch_bounds__(LN_THREADS) k_ln_bwd(LnBwdArgs a) {
  constexpr int VE = CHUNK<T>;
  __shared__ float s_red[LN_THREADS / 64];
  extern __shared__ double s_col[];     // [D] where the workgroup holds several groups
  const int G = a.G, lane = threadIdx.x & (G - 1), sub = threadIdx.x / G, groups = LN_THREADS / G;
  const int D = a.D;
  const int64_t r0 = int64_t(blockIdx.x) * a.rows;
  const int64_t r1 = r0 + a.rows < a.n ? r0 + a.rows : a.n;
  float ga[P][VE], dg[P][VE], db[P][VE];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int c0 = (lane + p * G) * VE;
#pragma unroll
    for (int j = 0; j < VE; j += 4) {
      if (a.gamma) load_chunk(a.gamma + c0 + j, D - c0 - j, ga[p] + j);
      else for (int k = 0; k < 4; ++k) ga[p][j + k] = 1.f;
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) dg[p][j] = db[p][j] = 0.f;
  }
  const float inv = 1.f / float(D);
  for (int64_t row = r0 + sub; row < r1; row += groups) {
    const T* hp = static_cast<const T*>(a.h) + row * D;
    const T* yp = static_cast<const T*>(a.dy) + row * D;
    float xh[P][VE], dy[P][VE];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c0 = (lane + p * G) * VE;
      load_chunk(hp + c0, D - c0, xh[p]);
      load_chunk(yp + c0, D - c0, dy[p]);     // 0 past the row's end: those columns add nothing
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        xh[p][j] = (xh[p][j] - mean) * rstd;
        dg[p][j] = fmaf(dy[p][j], xh[p][j], dg[p][j]);
        db[p][j] += dy[p][j];
        dy[p][j] *= ga[p][j];
        s1 += dy[p][j];
        s2 = fmaf(dy[p][j], xh[p][j], s2);
      }
    s1 = row_sum(s1, G, s_red) * inv;
    s2 = row_sum(s2, G, s_red) * inv;
    T* o = static_cast<T*>(a.dx) + row * D;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c0 = (lane + p * G) * VE;
      float d[VE];
      if (a.dsum) load_chunk(static_cast<const T*>(a.dsum) + row * D + c0, D - c0, d);
      else
        for (int j = 0; j < VE; ++j) d[j] = 0.f;
#pragma unroll
      for (int j = 0; j < VE; ++j) d[j] = fmaf(rstd, dy[p][j] - s1 - xh[p][j] * s2, d[j]);
      store_chunk(o + c0, D - c0, d);
    }
  }
  if (!a.part) return;
  double* out = a.part + int64_t(blockIdx.x) * 2 * D;
  const int wave = threadIdx.x >> 6;
  for (int which = 0; which < 2; ++which) {
    double c[P][VE];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        c[p][j] = which ? db[p][j] : dg[p][j];
        for (int o = G; o < 64; o *= 2) c[p][j] += __shfl_xor(c[p][j], o);   // the groups of a wave
      }
    if (groups == 1) {                   // the lanes of the workgroup own different columns
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < VE; ++j)
          if ((lane + p * G) * VE + j < D) out[which * D + (lane + p * G) * VE + j] = c[p][j];
      continue;
    }
    for (int k = 0; k < LN_THREADS / 64; ++k) {   // the waves in order
      if (wave == k && (threadIdx.x & 63) < G) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            const int col = (lane + p * G) * VE + j;
            if (col < D) s_col[col] = (k ? s_col[col] : 0.0) + c[p][j];
          }
      }
      __syncthreads();
    }
    for (int col = threadIdx.x; col < D; col += LN_THREADS) out[which * D + col] = s_col[col];
    __syncthreads();                     // read before the next sums overwrite it
  }
}

// dgamma and dbeta from the partial rows, added in their order: LN_SUM_ROWS
// threads per column take every LN_SUM_ROWS-th row, then one adds theirs.
constexpr int LN_SUM_COLS = 16;
constexpr int LN_SUM_ROWS = LN_THREADS / LN_SUM_COLS;
__global__ void __launch_bounds__(LN_THREADS) k_ln_bwd_sum(const double* __restrict__ part, int64_t nb,
                                                           int D, float* __restrict__ dgamma,
                                                           float* __restrict__ dbeta) {
  __shared__ double s[LN_SUM_ROWS][LN_SUM_COLS];
  const int col = threadIdx.x % LN_SUM_COLS, r = threadIdx.x / LN_SUM_COLS;
  const int c = blockIdx.x * LN_SUM_COLS + col;      // of 2 D columns
  double t = 0.0;
  if (c < 2 * D)
    for (int64_t b = r; b < nb; b += LN_SUM_ROWS) t += part[b * 2 * D + c];
  s[r][col] = t;
  __syncthreads();
  if (r == 0 && c < 2 * D) {
    for (int k = 1; k < LN_SUM_ROWS; ++k) t += s[k][col];
    float* o = c < D ? dgamma : dbeta;
    if (o) o[c < D ? c : c - D] = float(t);
  }
}

struct LnPlan {
  int G, P;            // lanes per row, chunks per lane
  int64_t rows, nb;    // backward: rows per workgroup, workgroups
};

// The narrowest group that holds a row with the fewest idle chunk slots; a
// workgroup for rows past what a wave's registers hold.
static LnPlan ln_plan(int64_t n, int D, int ve) {
  LnPlan L = {};
  const int C = (D + ve - 1) / ve;
  int best = 1 << 30;
  const int ps[] = {1, 2, 3, 4, 6, 8};
  for (int G = 1; G <= 64; G *= 2)
    for (int P : ps)
      if (G * P >= C && (G * P < best || (G * P == best && P < L.P))) {
        best = G * P;
        L.G = G;
        L.P = P;
      }
  if (best == 1 << 30) {
    L.G = LN_THREADS;
    for (int P : ps)
      if (LN_THREADS * P >= C) {
        L.P = P;
        break;
      }
  }
  const int64_t groups = LN_THREADS / L.G;
  // about 2048 workgroups (8 per CU), each with at most LN_ROWS rows per group
  int64_t per = (n + 2048 * groups - 1) / (2048 * groups);
  per = per < 1 ? 1 : (per > LN_ROWS ? LN_ROWS : per);
  L.rows = per * groups;
  L.nb = (n + L.rows - 1) / L.rows;
  return L;
}

template <typename T>
static void launch_ln_fwd(const LnArgs& a, int P, uint32_t grid, hipStream_t st) {
#define FAST_LN(p) case p: hipLaunchKernelGGL((k_ln_fwd<T, p>), dim3(grid), dim3(LN_THREADS), 0, st, a); break
  switch (P) { FAST_LN(1); FAST_LN(2); FAST_LN(3); FAST_LN(4); FAST_LN(6); FAST_LN(8); }
#undef FAST_LN
}
template <typename T>
static void launch_ln_bwd(const LnBwdArgs& a, int P, uint32_t grid, size_t lds, hipStream_t st) {
#define FAST_LN(p) case p: hipLaunchKernelGGL((k_ln_bwd<T, p>), dim3(grid), dim3(LN_THREADS), lds, st, a); break
  switch (P) { FAST_LN(1); FAST_LN(2); FAST_LN(3); FAST_LN(4); FAST_LN(6); FAST_LN(8); }
#undef FAST_LN
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
  if (n == 0) return ok();
  if (!x || !y) return fail(FAST_ERR_INVALID_ARG, "%s: NULL x/y", fn);
  const size_t es = elem_size(dtype);
  if (!aligned(x, es) || !aligned(res, es) || !aligned(y, es) || !aligned(sum, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: gamma/beta/mean/rstd not 4-byte aligned", fn);
  const LnPlan L = ln_plan(n, D, 16 / int(es));
  const LnArgs a = {n, D, L.G, x, res, gamma, beta, eps, y, sum, mean, rstd};
  const int64_t per = LN_THREADS / L.G;
  const uint32_t grid = uint32_t((n + per - 1) / per);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32) launch_ln_fwd<float>(a, L.P, grid, st);
  else launch_ln_fwd<uint16_t>(a, L.P, grid, st);
  return check_launch(fn);
}

extern "C" size_t fast_layer_norm_bwd_workspace(int64_t n, int D) {
  if (n < 0 || n >= (int64_t(1) << 31) || D <= 0 || D > LN_MAX_D) return 0;
  const LnPlan a = ln_plan(n, D, 4), b = ln_plan(n, D, 8);
  const int64_t nb = a.nb > b.nb ? a.nb : b.nb;
  return size_t(nb > 0 ? nb : 1) * 2 * D * sizeof(double);
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
  if (sums) {
    if (!ws || ws_bytes < fast_layer_norm_bwd_workspace(n, D))
      return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0,
                  fast_layer_norm_bwd_workspace(n, D));
    if (!aligned(ws, 8)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 8-byte aligned", fn);
  }
  if (n == 0 && !sums) return ok();
  const LnPlan L = ln_plan(n, D, 16 / int(es));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n > 0) {
    const LnBwdArgs a = {n, D, L.G, L.rows, h, gamma, mean, rstd, dy, dsum, dx,
                         sums ? static_cast<double*>(ws) : nullptr};
    const size_t lds = sums && L.G < LN_THREADS ? size_t(D) * sizeof(double) : 0;
    if (dtype == FAST_F32) launch_ln_bwd<float>(a, L.P, uint32_t(L.nb), lds, st);
    else launch_ln_bwd<uint16_t>(a, L.P, uint32_t(L.nb), lds, st);
  }
  if (sums)
    hipLaunchKernelGGL(k_ln_bwd_sum, dim3((2 * D + LN_SUM_COLS - 1) / LN_SUM_COLS), dim3(LN_THREADS), 0, st,
                       static_cast<const double*>(ws), n > 0 ? L.nb : 0, D, dgamma, dbeta);
  return check_launch(fn);
}
