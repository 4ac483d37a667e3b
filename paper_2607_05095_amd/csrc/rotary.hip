// rotary.hip -- rotary positions with several axes, forward and backward.
//   theta[i,p] = pos[i, axis[p]] * omega[p]
//   (a, b) -> (a cos theta - b sin theta, a sin theta + b cos theta)
// for the element pairs p < pairs of every head of row i; the head's other
// elements are copied.  The map is orthogonal, so the backward turns the
// gradient by -theta.
//
// Bound by HBM: each element is read and written once (500,000 rows of 8 x 128 bf16 342 us =
// 6.0 TB/s; 528,000 of 2 x 50 fp32, whose 400 bytes share lines, 92 = 4.6, a plain copy 78).  The angles belong to a
// row, not to its heads: a workgroup first forms the sines and cosines of its
// rows in LDS while the rows' pieces of 16 bytes are on their way to its registers.
//
// Positions may be event times far from zero, where an fp32 angle has no correct
// digit left: the product of the two fp32 factors is exact in fp64, it is reduced
// in revolutions to the nearest quarter there, and only the rest, at most an
// eighth of a revolution, is rounded to fp32 (2e-8 rad) and evaluated.
#include "rows.h"

namespace fast {

constexpr int ROT_THREADS = 256;
// Pieces per thread: 2 where a piece is 16 bytes, 1 where it is 16 of either half
// (528,000 rows of 2 x 50 fp32: 102 / 115 us with 2 / 1, by halves 108 / 101).
template <bool INTER> constexpr int ROT_UNROLL = INTER ? 2 : 1;
constexpr int ROT_PAIRS = 1024;         // (cos, sin) pairs per workgroup
constexpr int ROT_LDS_PAIRS = ROT_PAIRS + 8;

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

// (cos, sin) of a position times a frequency: the angle in quarter turns, its nearest whole number
// and the rest g, |g| <= 1/2, then the Taylor sums of sin and cos(g pi/2) through g^9 and
// g^10 (the next terms are below 2e-9); 1.5e-7 in all with their fp32 roundings.  The
// angle, a product of two fp32 factors, is exact in fp64; 2 / pi takes two terms, as the
// rounding of the first alone is 2e-7 rad at an angle of 2e9.  From 2^44 quarter turns
// on they are not enough, and the turns are reduced in integers as Payne and Hanek (1983)
// do: of the angle M 2^e, M < 2^64, times 2 / pi only the bits of 2 / pi behind whole
// revolutions count, a window of 96 of them, and of the product the 32 bits behind
// the point (5e-9 rad).  (sincos in fp64 there took 109.8 us instead of 92.8 for
// 528,000 rows of 2 x 50 fp32, in registers: 78 against 36.)
__constant__ const uint32_t ROT_TWO_OVER_PI[10] = {     // 32 zeros, then its bits behind the point
    0x00000000u, 0xa2f9836eu, 0x4e441529u, 0xfc2757d1u, 0xf534ddc0u,
    0xdb629599u, 0x3c439041u, 0xfe5163abu, 0xdebbc561u, 0xb7246e3au};
__device__ __forceinline__ float2 rot_turn(float pos, float omega, float sign) {
  constexpr double HI = 0.6366197723675814, LO = -3.935735335036497e-17;   // 2 / pi
  const double angle = double(pos) * double(omega), q = rint(angle * HI);
  float g;
  int k;                                             // q mod 4
  if (fabs(q) < 0x1p44) {
    g = float(fma(angle, LO, fma(angle, HI, -q)));
    k = int(__builtin_amdgcn_fract(q * 0.25) * 4.0);
  } else {
    const uint64_t bits = uint64_t(__double_as_longlong(angle));
    const int e = int(bits >> 52) & 2047;
    const bool number = e < 2047;                    // not infinite, not NaN
    const uint32_t at = number ? e - 1056 : 0;       // 11 (2^44) to 222 (2^255): words 0 to 9
    const uint64_t M = bits << 11 | uint64_t(1) << 63;
    const uint32_t m1 = uint32_t(M >> 32), m0 = uint32_t(M);
    const uint32_t* w = ROT_TWO_OVER_PI + (at >> 5);
    const uint32_t w0 = __funnelshift_l(w[1], w[0], at & 31), w1 = __funnelshift_l(w[2], w[1], at & 31),
                   w2 = __funnelshift_l(w[3], w[2], at & 31);
    uint32_t turn = m0 * w0 + m1 * w1 + __umulhi(m0, w1) + __umulhi(m1, w2);   // of a revolution, times 2^32
    if (bits >> 63) turn = 0u - turn;
    k = int((turn + (1u << 29)) >> 30);
    g = float(int32_t(turn - (uint32_t(k) << 30))) * 0x1p-30f;
    k &= 3;
    if (!number) g = NAN;
  }
  const float t = g * g;
  float s = fmaf(t, 1.604411847e-4f, -4.681754135e-3f);
  s = fmaf(s, t, 7.969262624e-2f);
  s = fmaf(s, t, -6.459640975e-1f);
  s = fmaf(s, t, 1.570796327f) * g;
  float c = fmaf(t, -2.520204237e-5f, 9.192602748e-4f);
  c = fmaf(c, t, -2.086348077e-2f);
  c = fmaf(c, t, 2.536695079e-1f);
  c = fmaf(c, t, -1.233700550f);
  c = fmaf(c, t, 1.f);
  const float s1 = (k & 1) ? c : s, c1 = (k & 1) ? s : c;
  return make_float2((k == 1 || k == 2) ? -c1 : c1, (k >= 2 ? -s1 : s1) * sign);
}

// A piece of a head: 16 bytes of it, or (pairs (p, pairs + p)) 16 bytes of either half.
template <int VE, bool INTER>
struct RotPiece {
  int64_t x, y;                         // element offsets of the head's first element
  int e, n, cs;                         // first element, elements left, first pair's place in LDS
  bool rot;
  float a[VE], b[INTER ? 1 : VE];
};

template <typename T, bool INTER, bool NT>
__global__ void __launch_bounds__(ROT_THREADS) k_rotary(RotArgs a) {
  constexpr int VE = CHUNK<T>, UN = ROT_UNROLL<INTER>;
  __shared__ float2 s_cs[ROT_LDS_PAIRS];
  const int64_t row0 = int64_t(blockIdx.x) * a.rows;
  const int rows = int(a.n - row0 < a.rows ? a.n - row0 : a.rows);
  const int P = a.pairs, total = rows * a.upr;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  // the rows' loads are in flight while the angles are formed
  RotPiece<VE, INTER> w[UN];
#pragma unroll
  for (int k = 0; k < UN; ++k) {
    const int t = threadIdx.x + (blockIdx.y * UN + k) * ROT_THREADS;
    if (t < total) {
      const int r = int(div_small(t, a.mag_upr)), u = t - r * a.upr;
      const int h = int(div_small(u, a.mag_units)), c = u - h * a.units;
      RotPiece<VE, INTER>& q = w[k];
      q.x = (row0 + r) * a.ldx + h * a.dh;
      q.y = (row0 + r) * a.ldy + h * a.dh;
      q.rot = c < a.crot;
      q.e = q.rot ? c * VE : 2 * P + (c - a.crot) * VE;        // past the pairs: copied
      q.n = (q.rot ? (INTER ? 2 * P : P) : a.dh) - q.e;
      q.cs = r * P + (INTER ? q.e / 2 : q.e);
      load_chunk(x + q.x + q.e, q.n, q.a);
      if constexpr (!INTER)
        if (q.rot) load_chunk(x + q.x + P + q.e, q.n, q.b);
    }
  }
  for (int t = threadIdx.x; t < rows * P; t += ROT_THREADS) {
    const int r = int(div_small(t, a.mag_pairs)), p = t - r * P;
    int ax = a.axis ? a.axis[p] : 0;
    ax = ax < 0 ? 0 : (ax < a.axes ? ax : a.axes - 1);
    s_cs[t] = rot_turn(a.pos[(row0 + r) * a.axes + ax], a.omega[p], a.sign);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < UN; ++k) {
    if (int(threadIdx.x + (blockIdx.y * UN + k) * ROT_THREADS) < total) {
      RotPiece<VE, INTER>& q = w[k];
      if (q.rot) {
        // s_cs is read past the head's last pair where the piece is partial: within the
        // array (ROT_LDS_PAIRS has CHUNK places more than pairs in use), and not used
        if constexpr (INTER) {
#pragma unroll
          for (int j = 0; j < VE / 2; ++j) {
            const float2 cs = s_cs[q.cs + j];
            const float va = q.a[2 * j], vb = q.a[2 * j + 1];
            q.a[2 * j] = fmaf(va, cs.x, -(vb * cs.y));
            q.a[2 * j + 1] = fmaf(va, cs.y, vb * cs.x);
          }
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            const float2 cs = s_cs[q.cs + j];
            const float va = q.a[j];
            q.a[j] = fmaf(va, cs.x, -(q.b[j] * cs.y));
            q.b[j] = fmaf(va, cs.y, q.b[j] * cs.x);
          }
          store_chunk(y + q.y + P + q.e, q.n, q.b);
        }
      }
      store_chunk<T, NT>(y + q.y + q.e, q.n, q.a);
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
  // (n and the strides are below 2^31 each: the products fit, their bytes might not)
  if ((n - 1) * (ldx > ldy ? ldx : ldy) >= (int64_t(1) << 56))
    return fail(FAST_ERR_UNSUPPORTED, "%s: %lld rows, %lld and %lld elements apart", fn, (long long)n,
                (long long)ldx, (long long)ldy);
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
  // whole rows, the kernel's pieces per thread; a row of more pieces is shared by workgroups
  // (blockIdx.y), each forming its angles
  const int tile = (interleaved ? ROT_UNROLL<true> : ROT_UNROLL<false>) * ROT_THREADS;
  a.rows = a.upr < tile ? tile / a.upr : 1;
  if (pairs > 0 && a.rows > ROT_PAIRS / pairs) a.rows = ROT_PAIRS / pairs;
  a.mag_pairs = div_magic(pairs > 0 ? pairs : 1);
  a.mag_upr = div_magic(a.upr);
  a.mag_units = div_magic(a.units);
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.axis = axis;
  a.omega = omega;
  a.sign = sign;
  const dim3 grid(uint32_t((n + a.rows - 1) / a.rows), uint32_t((a.rows * a.upr + tile - 1) / tile));
  if (!grid_fits(grid.x, ROT_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  // Rows of whole cache lines that go out in one stream (pairs side by side) bypass the
  // cache when rows and results are more than its last level holds: 1,000,000 rows
  // of 4 x 32 bf16, 102 -> 76 us; pairs by halves 105 -> 114, so they do not.
  const bool nt = interleaved && ldy * es % CACHE_LINE == 0 && F == ldy && aligned(y, CACHE_LINE) &&
                  2 * n * F * es > (int64_t(256) << 20);
#define FAST_ROT(T, I, N) hipLaunchKernelGGL((k_rotary<T, I, N>), grid, dim3(ROT_THREADS), 0, st, a)
  if (dtype == FAST_F32) {
    if (nt) FAST_ROT(float, true, true);
    else if (interleaved) FAST_ROT(float, true, false);
    else FAST_ROT(float, false, false);
  } else {
    if (nt) FAST_ROT(uint16_t, true, true);
    else if (interleaved) FAST_ROT(uint16_t, true, false);
    else FAST_ROT(uint16_t, false, false);
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
