// rotary.hip -- rotary positions with several axes, forward and backward.
//   theta[i,p] = pos[i, axis[p]] * omega[p]
//   (a, b) -> (a cos theta - b sin theta, a sin theta + b cos theta)
// for the element pairs p < pairs of every head of row i; the head's other
// elements are copied.  The map is orthogonal, so the backward turns the
// gradient by -theta.
//
// Bound by HBM: each element is read and written once.  The angles belong to a
// row, not to its heads: a workgroup first forms the sines and cosines of its
// rows in LDS, then streams the rows in pieces of 16 bytes.
//
// Positions may be event times far from zero, where an fp32 angle has no correct
// digit left: the product of the two fp32 factors is exact in fp64, it is reduced
// in revolutions to the nearest quarter there, and only the rest, at most an
// eighth of a revolution, is rounded to fp32 (2e-8 rad) and evaluated.
#include "rows.h"

namespace fast {

constexpr int ROT_THREADS = 256;
constexpr int ROT_LDS_PAIRS = 2048;     // (cos, sin) pairs per workgroup: 16 KB
constexpr int ROT_MAX_ROWS = 64;

struct RotArgs {
  int64_t n, ldx, ldy;
  int H, dh, pairs, axes;
  int rows;                             // rows per workgroup
  int units, upr;                       // pieces per head (rotated, copied), per row
  int crot;                             // rotated pieces of a head
  uint32_t mag_pairs, mag_upr, mag_units;
  const void* x;
  void* y;
  const float* pos;
  const int32_t* axis;
  const float* omega;
  float sign;
};

template <typename T, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS) k_rotary(RotArgs a) {
  constexpr int VE = CHUNK<T>;
  __shared__ float2 s_cs[ROT_LDS_PAIRS];
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows);
  const int P = a.pairs;
  for (int t = threadIdx.x; t < rows * P; t += ROT_THREADS) {
    const int r = int(div_small(t, a.mag_pairs)), p = t - r * P;
    int ax = a.axis ? a.axis[p] : 0;
    ax = ax < 0 ? 0 : (ax < a.axes ? ax : a.axes - 1);
    const double th = double(a.pos[(row0 + r) * a.axes + ax]) * double(a.omega[p]);   // exact
    const double rev = th * 0.15915494309189535;       // 1 / (2 pi)
    const double q = rint(rev * 4.0);
    const float f = float(rev - q * 0.25);             // |f| <= 1/8; NaN of an infinite angle
    float s, c;
    sincospif(2.f * f, &s, &c);
    const int k = int(q - 4.0 * floor(q * 0.25));      // quarter turns, 0..3
    const float s1 = (k & 1) ? c : s, c1 = (k & 1) ? s : c;
    s_cs[t] = make_float2((k == 1 || k == 2) ? -c1 : c1, (k >= 2 ? -s1 : s1) * a.sign);
  }
  __syncthreads();
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  for (int t = threadIdx.x; t < rows * a.upr; t += ROT_THREADS) {
    const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
    const int h = int(div_small(u, a.mag_units)), c = u - h * a.units;
    const T* xp = x + (row0 + r) * a.ldx + h * a.dh;
    T* yp = y + (row0 + r) * a.ldy + h * a.dh;
    if (c >= a.crot) {                                  // past the pairs: copied
      const int e = 2 * P + (c - a.crot) * VE;
      float v[VE];
      load_chunk(xp + e, a.dh - e, v);
      store_chunk(yp + e, a.dh - e, v);
    } else if constexpr (INTER) {                       // pairs (2p, 2p + 1)
      const int e = c * VE;
      float v[VE];
      load_chunk(xp + e, 2 * P - e, v);
#pragma unroll
      for (int j = 0; j < VE / 2; ++j) {
        const int p = e / 2 + j < P ? e / 2 + j : P - 1;
        const float2 cs = s_cs[r * P + p];
        const float va = v[2 * j], vb = v[2 * j + 1];
        v[2 * j] = fmaf(va, cs.x, -(vb * cs.y));
        v[2 * j + 1] = fmaf(va, cs.y, vb * cs.x);
      }
      store_chunk(yp + e, 2 * P - e, v);
    } else {                                            // pairs (p, pairs + p)
      const int e = c * VE;
      float va[VE], vb[VE];
      load_chunk(xp + e, P - e, va);
      load_chunk(xp + P + e, P - e, vb);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const int p = e + j < P ? e + j : P - 1;
        const float2 cs = s_cs[r * P + p];
        const float t0 = va[j];
        va[j] = fmaf(t0, cs.x, -(vb[j] * cs.y));
        vb[j] = fmaf(t0, cs.y, vb[j] * cs.x);
      }
      store_chunk(yp + e, P - e, va);
      store_chunk(yp + P + e, P - e, vb);
    }
  }
}

// Do the elements of rows of F elements, ldx and ldy apart, overlap other than
// element on element?
static bool rows_collide(const char* x, int64_t ldx, const char* y, int64_t ldy, int64_t n, int64_t F,
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

static fast_status_t rotary(const char* fn, int64_t n, int H, int dh, fast_dtype_t dtype, const void* x,
                            int64_t ldx, const float* pos, int axes, const int32_t* axis,
                            const float* omega, int pairs, int interleaved, void* y, int64_t ldy,
                            float sign, fast_stream_t stream) {
  if (n < 0) return fail(FAST_ERR_INVALID_ARG, "%s: n = %lld < 0", fn, (long long)n);
  if (H <= 0 || dh <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: H = %d, dh = %d", fn, H, dh);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (H > 64 || dh > 256)
    return fail(FAST_ERR_UNSUPPORTED, "%s: H = %d > 64 or dh = %d > 256", fn, H, dh);
  if (pairs < 0 || 2 * int64_t(pairs) > dh)
    return fail(FAST_ERR_INVALID_ARG, "%s: %d pairs in heads of %d", fn, pairs, dh);
  if (axes <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: axes = %d <= 0", fn, axes);
  const int64_t F = int64_t(H) * dh, es = elem_size(dtype);
  if (ldx < F || ldy < F)
    return fail(FAST_ERR_INVALID_ARG, "%s: rows of %lld elements, %lld and %lld apart", fn, (long long)F,
                (long long)ldx, (long long)ldy);
  if (n >= (int64_t(1) << 31)) return fail(FAST_ERR_UNSUPPORTED, "%s: n >= 2^31", fn);
  if (ldx >= (int64_t(1) << 31) || ldy >= (int64_t(1) << 31))
    return fail(FAST_ERR_UNSUPPORTED, "%s: row stride >= 2^31", fn);
  if (n == 0) return ok();
  if (!x || !y || (pairs > 0 && (!pos || !omega)))
    return fail(FAST_ERR_INVALID_ARG, "%s: NULL rows/pos/omega", fn);
  if (!aligned(x, es) || !aligned(y, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(pos, 4) || !aligned(omega, 4) || !aligned(axis, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: pos/axis/omega not 4-byte aligned", fn);
  if (rows_collide(static_cast<const char*>(x), ldx, static_cast<const char*>(y), ldy, n, F, es))
    return fail(FAST_ERR_INVALID_ARG, "%s: output rows overlap input rows", fn);
  RotArgs a = {};
  const int ve = 16 / int(es);
  a.n = n;
  a.ldx = ldx;
  a.ldy = ldy;
  a.H = H;
  a.dh = dh;
  a.pairs = pairs;
  a.axes = axes;
  a.crot = interleaved ? (2 * pairs + ve - 1) / ve : (pairs + ve - 1) / ve;
  const bool in_place = x == y;                        // the other elements are there already
  a.units = a.crot + (in_place ? 0 : (dh - 2 * pairs + ve - 1) / ve);
  if (a.units == 0) return ok();
  a.upr = a.units * H;
  int rows = pairs > 0 ? ROT_LDS_PAIRS / pairs : ROT_MAX_ROWS;
  a.rows = rows < ROT_MAX_ROWS ? rows : ROT_MAX_ROWS;
  a.mag_pairs = div_magic(pairs > 0 ? pairs : 1);
  a.mag_upr = div_magic(a.upr);
  a.mag_units = div_magic(a.units);
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.axis = axis;
  a.omega = omega;
  a.sign = sign;
  const uint32_t grid = uint32_t((n + a.rows - 1) / a.rows);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define FAST_ROT(T, I) hipLaunchKernelGGL((k_rotary<T, I>), dim3(grid), dim3(ROT_THREADS), 0, st, a)
  if (dtype == FAST_F32) {
    if (interleaved) FAST_ROT(float, true);
    else FAST_ROT(float, false);
  } else {
    if (interleaved) FAST_ROT(uint16_t, true);
    else FAST_ROT(uint16_t, false);
  }
#undef FAST_ROT
  return check_launch(fn);
}

}  // namespace fast

using namespace fast;

extern "C" fast_status_t fast_rotary_fwd(int64_t n, int H, int dh, fast_dtype_t dtype, const void* x,
                                         int64_t ldx, const float* pos, int axes,
                                         const int32_t* axis, const float* omega, int pairs,
                                         int interleaved, void* y, int64_t ldy,
                                         fast_stream_t stream) {
  return rotary("fast_rotary_fwd", n, H, dh, dtype, x, ldx, pos, axes, axis, omega, pairs, interleaved, y,
                ldy, 1.f, stream);
}

extern "C" fast_status_t fast_rotary_bwd(int64_t n, int H, int dh, fast_dtype_t dtype, const void* dy,
                                         int64_t lddy, const float* pos, int axes,
                                         const int32_t* axis, const float* omega, int pairs,
                                         int interleaved, void* dx, int64_t lddx,
                                         fast_stream_t stream) {
  return rotary("fast_rotary_bwd", n, H, dh, dtype, dy, lddy, pos, axes, axis, omega, pairs, interleaved, dx,
                lddx, -1.f, stream);
}
