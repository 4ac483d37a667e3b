// adamw.hip -- the AdamW step over many tensors, and the norm of their gradients.
//   g = scale grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   w = w - lr (decay w + (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps))
//
// Bound by HBM: 28 bytes an element with fp32 states and gradients, 16 (and an eighth) with
// states in 8 bits.  A launch takes the descriptors of up to AW_TENSORS tensors as
// arguments and cuts them into chunks of AW_UNIT elements, a workgroup each; a thread
// moves 4 of them, so 8 neighbouring lanes hold the 32 elements that
// share a scale in 8 bits and find its largest magnitude by DPP.
//
// States in 8 bits: a step changes v by a thousandth of itself or less, far below the
// eighth between neighbouring codes; rounded to the nearest, v would stand still.  So codes
// are rounded at random with the chance that keeps the mean, from a hash of the
// element's place and the step: repeated steps give the same bits.  The moments are
// formed in fp64 there: a code is then a function of the inputs and not of how
// products happen to be contracted.
//
// 100 M elements fp32 462 us (6.1 TB/s); 60 M in 61 tensors with bf16 gradients in 8 bits 215
// (two launches, 4.5 TB/s) and the norm of them 32 + 5; 400,000 elements in 24 tensors 6, 5 and 2.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int AW_THREADS = 256, AW_VEC = 4;
constexpr int AW_UNIT = AW_THREADS * AW_VEC;   // elements of a workgroup
constexpr int AW_TENSORS = 40;                 // descriptors of a launch: its arguments hold 4 KB
constexpr int AW_COUNT = 1024;                 // tensors of a call
constexpr int64_t AW_MAX_N = int64_t(1) << 40;

struct AwTensor {
  float* w;
  const void* g;
  void* m;
  void* v;
  uint8_t* ms;
  uint8_t* vs;
  uint16_t* copy;
  int64_t n;
  float decay;
  uint32_t id;
};
struct AwArgs {
  AwTensor t[AW_TENSORS];
  uint32_t first[AW_TENSORS + 1];     // chunks before the tensor
  int count;
  double b1, b2, eps;
  double lr;
  int64_t step;
  float bc1, bc2;                     // bias corrections of `step`
  uint32_t seed;
  const float* lr_dev;
  const int64_t* step_dev;
  const float* scale;
};
static_assert(sizeof(AwArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ uint32_t aw_mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// 4 elements at the element type's own alignment; FULL: all there, else n of them, one by one
// where there are fewer, zeros past them.  NT: streamed.
template <bool FULL, bool NT>
__device__ __forceinline__ void aw_load(const float* p, int n, float* x) { load_chunk_of<NT>(p, FULL ? 4 : n, x); }
template <bool FULL, bool NT>
__device__ __forceinline__ void aw_load(const uint16_t* p, int n, float* x) {
  if (FULL || n >= 4) {
    const u32x2_e w = ld_stream<u32x2_e, NT>(p);
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = j < n ? bf16_at(p + j) : 0.f;
}
template <bool FULL, bool NT>
__device__ __forceinline__ void aw_store(float* p, int n, const float* x) { store_chunk_of<NT>(p, FULL ? 4 : n, x); }
template <bool FULL, bool NT>
__device__ __forceinline__ void aw_store(uint16_t* p, int n, const float* x) {
  if (FULL || n >= 4) {
    st_stream<u32x2_e, NT>(p, u32x2_e{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3])});
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n) p[j] = uint16_t(bf16_rne(x[j]));
}
typedef uint32_t u32_b __attribute__((aligned(1)));
template <bool FULL, bool NT>
__device__ __forceinline__ uint32_t aw_load8(const uint8_t* p, int n) {
  if (FULL || n >= 4) return ld_stream<u32_b, NT>(p);
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n) w |= uint32_t(p[j]) << (8 * j);
  return w;
}
template <bool FULL, bool NT>
__device__ __forceinline__ void aw_store8(uint8_t* p, int n, uint32_t w) {
  if (FULL || n >= 4) {
    st_stream<u32_b, NT>(p, w);
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n) p[j] = uint8_t(w >> (8 * j));
}
// The values of 4 codes: code times 2^(byte - 127).
__device__ __forceinline__ void aw_values(uint32_t codes, uint32_t byte, float* x) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, mx_scale(byte), false);
  const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, mx_scale(byte), true);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

// x's code under the group's scale byte, the upper of two neighbours where the fraction
// above the lower is more than r / 65536.  root: what is not 0 does not become 0.
// s = x 2^-k: from 2^-6 on a code is the upper bits of the float (exponents 120 apart, 3 bits of
// mantissa, the fraction in the 20 below); codes below are multiples of 2^-9.
__device__ __forceinline__ uint32_t aw_code(float x, uint32_t byte, uint32_t r, bool root) {
  const float a = fabsf(x), s = ldexpf(a, 127 - int(byte));
  const uint32_t w = __float_as_uint(s);
  uint32_t code = (w >> 20) - (120u << 3) + ((w & 0xfffffu) > (r << 4) ? 1u : 0u);
  const float t = s * 512.f, low = floorf(t);
  // (next to 0 the fraction may be too small for fp32; it is above 0 all the same)
  const bool up = r != 0u ? t - low > float(r) * 0x1p-16f : (t < 1.f ? a > 0.f : t > low);
  uint32_t c = uint32_t(low) + (up ? 1u : 0u);
  if (root) c = a > 0.f && c == 0u ? 1u : c;
  code = s < 0x1p-6f ? c : code;
  // 2^128 is no fp32 number: from 256 2^120 (code 0x78 under byte 247) on, one step down
  if (byte >= MX_TOP_BYTE<FAST_MXFP8> && int(code >> 3) - 7 + int(byte) - 127 >= 128) --code;
  code |= x < 0.f ? 0x80u : 0u;
  return byte == 255u ? 0u : code;
}

// sqrt of a double, rounded to fp32: the reciprocal root and a Newton step, which leaves 2^-50.
__device__ __forceinline__ float aw_root(double v) {
  const double q = __builtin_amdgcn_rsq(v), r = v * q;
  const float x = float(fma(fma(-r, r, v), 0.5 * q, r));
  return v > 0.0 && v < double(INFINITY) ? x : float(v);   // 0, an infinity, no number
}

__device__ __forceinline__ float max8(float x) {          // the largest of 8 neighbouring lanes
  x = fmaxf(x, dpp_quad_xor1(x));
  x = fmaxf(x, dpp_quad_xor2(x));
  return fmaxf(x, dpp_row_half_mirror(x));
}
// The largest magnitude of the lanes' 4 elements over 8 lanes; infinite where one is not finite.
__device__ __forceinline__ float aw_top(const float* x) {
  float t = 0.f;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    t = fmaxf(t, fabsf(x[j]));
    bad |= !(fabsf(x[j]) < INFINITY);
  }
  return max8(bad ? INFINITY : t);
}

// A thread's 4 elements i .. i + 3 of a tensor, n of them there.  (Everything by value: a
// reference into the arguments makes the compiler copy all 4 KB of them into scratch memory.)
struct AwRule {
  double b1, b2;
  float eps, sc, lr, bc1, bc2;
  uint32_t key;
};
template <typename G, bool LOW, bool FULL, bool NT>
__device__ __forceinline__ void aw_step(const AwTensor p, const AwRule a, int64_t i, int n) {
  float w[4], g[4], m[4], root[4];
  const bool some = FULL || n > 0;
  if (some) {
    aw_load<FULL, NT>(p.w + i, n, w);
    aw_load<FULL, NT>(static_cast<const G*>(p.g) + i, n, g);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = g[q] = 0.f;
  }
  if constexpr (LOW) {
    float om[4], ov[4];
    uint32_t cm = 0, cv = 0, sm = 0, sv = 0;
    if (some) {
      cm = aw_load8<FULL, NT>(static_cast<const uint8_t*>(p.m) + i, n);
      cv = aw_load8<FULL, NT>(static_cast<const uint8_t*>(p.v) + i, n);
      sm = p.ms[i >> 5];
      sv = p.vs[i >> 5];
    }
    aw_values(cm, sm, om);
    aw_values(cv, sv, ov);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const double gd = double(g[q]) * double(a.sc), u = ov[q];
      m[q] = float(fma(a.b1, double(om[q]), (1.0 - a.b1) * gd));
      root[q] = aw_root(fma(a.b2, u * u, (1.0 - a.b2) * gd * gd));
      if (!FULL && q >= n) m[q] = root[q] = 0.f;          // past the end: no part in the scale
    }
    const uint32_t bm = mx_scale_byte<FAST_MXFP8>(aw_top(m)), bv = mx_scale_byte<FAST_MXFP8>(aw_top(root));
    const uint32_t hi = aw_mix(a.key + uint32_t(uint64_t(i) >> 32) * 0x9E3779B9u);
    cm = cv = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t rnd = aw_mix(hi ^ (uint32_t(i) + q));
      cm |= aw_code(m[q], bm, rnd & 0xffffu, false) << (8 * q);
      cv |= aw_code(root[q], bv, rnd >> 16, true) << (8 * q);
    }
    if (some) {
      aw_store8<FULL, NT>(static_cast<uint8_t*>(p.m) + i, n, cm);
      aw_store8<FULL, NT>(static_cast<uint8_t*>(p.v) + i, n, cv);
      if ((i & 31) == 0) {
        p.ms[i >> 5] = uint8_t(bm);
        p.vs[i >> 5] = uint8_t(bv);
      }
    }
  } else if (some) {
    const float b1 = float(a.b1), c1 = float(1.0 - a.b1), b2 = float(a.b2), c2 = float(1.0 - a.b2);
    float v[4];
    aw_load<FULL, NT>(static_cast<const float*>(p.m) + i, n, m);
    aw_load<FULL, NT>(static_cast<const float*>(p.v) + i, n, v);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float gs = g[q] * a.sc;
      m[q] = fmaf(b1, m[q], c1 * gs);
      v[q] = fmaf(b2, v[q], c2 * gs * gs);
      root[q] = sqrtf(v[q]);
    }
    aw_store<FULL, NT>(static_cast<float*>(p.m) + i, n, m);
    aw_store<FULL, NT>(static_cast<float*>(p.v) + i, n, v);
  }
  if (some) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float s = (m[q] * a.bc1) / fmaf(root[q], a.bc2, a.eps);
      w[q] = fmaf(-a.lr, fmaf(p.decay, w[q], s), w[q]);
    }
    aw_store<FULL, NT>(p.w + i, n, w);
    if (p.copy) aw_store<FULL, NT>(p.copy + i, n, w);
  }
}

// 1 / (1 - b1^t) and 1 / sqrt(1 - b2^t): from the host, or, for a captured step, of the number
// that the device holds, by one thread.
__device__ __forceinline__ void aw_correct(double b1, double b2, int64_t t, float* bc) {
  bc[0] = float(1.0 / (1.0 - pow(b1, double(t))));
  bc[1] = float(1.0 / sqrt(1.0 - pow(b2, double(t))));
}

template <typename G, bool LOW, bool NT>
__global__ void __launch_bounds__(AW_THREADS) k_adamw(AwArgs a) {
  __shared__ float s_bc[2];
  const float sc = a.scale ? *a.scale : 1.f;
  if (!(fabsf(sc) < INFINITY)) return;                    // the step is left out
  int64_t t = a.step;
  float bc1 = a.bc1, bc2 = a.bc2;
  if (a.step_dev) {
    t = *a.step_dev;
    t = t < 1 ? 1 : t;
    if (threadIdx.x == 0) aw_correct(a.b1, a.b2, t, s_bc);
    __syncthreads();
    bc1 = s_bc[0];
    bc2 = s_bc[1];
  }
  const float lr = a.lr_dev ? *a.lr_dev : float(a.lr);
  int j = 0;
  for (int h = 32; h > 0; h /= 2)                         // the last tensor that starts at or before the block
    if (j + h < a.count && a.first[j + h] <= blockIdx.x) j += h;
  const AwTensor p = a.t[j];
  const int64_t base = int64_t(blockIdx.x - a.first[j]) * AW_UNIT, i = base + threadIdx.x * AW_VEC;
  uint32_t key = 0;
  if constexpr (LOW) key = aw_mix(aw_mix(a.seed ^ uint32_t(t) * 0x9E3779B9u) ^ p.id);
  const AwRule rule = {a.b1, a.b2, float(a.eps), sc, lr, bc1, bc2, key};
  if (base + AW_UNIT <= p.n) {
    aw_step<G, LOW, true, NT>(p, rule, i, 4);
  } else {
    const int64_t left = p.n - i;
    aw_step<G, LOW, false, NT>(p, rule, i, left >= 4 ? 4 : (left > 0 ? int(left) : 0));
  }
}

// ------------------------------------------------------------------ the norm
// Squares and sums in fp64: a thread's in order, then the workgroup's by halves, then the
// workgroups' in order.
// A workgroup's elements: short lists in shorter chunks (400,000 elements 5.0 -> 3 us).
constexpr int GN_THREADS = 256, GN_CHUNK = 8192, GN_CHUNK_SHORT = 2048;
constexpr int64_t GN_SHORT = 1 << 22;
constexpr int GN_TENSORS = 128;
struct GnArgs {
  const void* g[GN_TENSORS];
  int64_t n[GN_TENSORS];
  uint32_t first[GN_TENSORS + 1];
  int count, chunk;
  double* part;
};
static_assert(sizeof(GnArgs) <= 4096, "kernel arguments");

template <int THREADS>
__device__ __forceinline__ double sum_group(double x, double* s) {
  s[threadIdx.x] = x;
  __syncthreads();
  for (int h = THREADS / 2; h > 0; h /= 2) {
    if (int(threadIdx.x) < h) s[threadIdx.x] += s[threadIdx.x + h];
    __syncthreads();
  }
  return s[0];
}

template <typename G>
__global__ void __launch_bounds__(GN_THREADS) k_grad_norm(GnArgs a) {
  __shared__ double s[GN_THREADS];
  int j = 0;
  for (int h = 64; h > 0; h /= 2)
    if (j + h < a.count && a.first[j + h] <= blockIdx.x) j += h;
  const G* g = static_cast<const G*>(a.g[j]);
  const int64_t base = int64_t(blockIdx.x - a.first[j]) * a.chunk, n = a.n[j];
  double t = 0.0;
#pragma unroll 4
  for (int r = 0; r < a.chunk; r += GN_THREADS * 4) {
    const int64_t i = base + r + threadIdx.x * 4;
    if (i >= n) break;
    float x[4];
    aw_load<false, false>(g + i, n - i >= 4 ? 4 : int(n - i), x);
#pragma unroll
    for (int q = 0; q < 4; ++q) t = fma(double(x[q]), double(x[q]), t);
  }
  t = sum_group<GN_THREADS>(t, s);
  if (threadIdx.x == 0) a.part[blockIdx.x] = t;
}
constexpr int GN_LAST = 1024;
__global__ void __launch_bounds__(GN_LAST) k_grad_norm_last(const double* __restrict__ part, int64_t n,
                                                            float max_norm, float* __restrict__ norm,
                                                            float* __restrict__ scale) {
  __shared__ double s[GN_LAST];
  double t = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += GN_LAST) t += part[i];
  t = sum_group<GN_LAST>(t, s);
  if (threadIdx.x == 0) {
    const float x = float(sqrt(t));
    *norm = x;
    if (scale) *scale = !(x < INFINITY) ? NAN : (x > max_norm ? max_norm / x : 1.f);
  }
}

// ------------------------------------------------------------------ host side
struct AwRange {
  uintptr_t at;
  uint64_t bytes : 63;
  uint64_t written : 1;
};
static int aw_add(AwRange* r, int k, const void* p, int64_t bytes, bool written) {
  if (!p || bytes <= 0) return k;
  r[k].at = reinterpret_cast<uintptr_t>(p);
  r[k].bytes = uint64_t(bytes);
  r[k].written = written;
  return k + 1;
}
// Does an array that is written overlap another?
static bool aw_overlap(AwRange* r, int k) {
  std::sort(r, r + k, [](const AwRange& x, const AwRange& y) { return x.at < y.at; });
  uintptr_t end = 0, wend = 0;                  // of all arrays before, of the written ones
  for (int i = 0; i < k; ++i) {
    if (r[i].at < (r[i].written ? end : wend)) return true;
    const uintptr_t e = r[i].at + r[i].bytes;
    if (e > end) end = e;
    if (r[i].written && e > wend) wend = e;
  }
  return false;
}

static fast_status_t aw_list(const char* fn, const fast_adamw_tensor_t* t, int count, fast_dtype_t gt) {
  if (count < 0) return fail(FAST_ERR_INVALID_ARG, "%s: count = %d < 0", fn, count);
  if (gt != FAST_F32 && gt != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (count > AW_COUNT) return fail(FAST_ERR_UNSUPPORTED, "%s: %d tensors, at most %d", fn, count, AW_COUNT);
  if (count > 0 && !t) return fail(FAST_ERR_INVALID_ARG, "%s: NULL tensors", fn);
  for (int j = 0; j < count; ++j) {
    if (t[j].n < 0) return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: n = %lld < 0", fn, j, (long long)t[j].n);
    if (t[j].n >= AW_MAX_N) return fail(FAST_ERR_UNSUPPORTED, "%s: tensor %d: n >= 2^40", fn, j);
    if (t[j].n > 0 && !t[j].grad) return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: NULL grad", fn, j);
    if (!aligned(t[j].grad, elem_size(gt)))
      return fail(FAST_ERR_UNSUPPORTED, "%s: tensor %d: grad not %d-byte aligned", fn, j, elem_size(gt));
  }
  return FAST_OK;
}

}  // namespace fast

using namespace fast;

extern "C" fast_status_t fast_adamw(const fast_adamw_tensor_t* tensors, int count, fast_dtype_t grad_dtype,
                                    fast_state_format_t format, double lr, double beta1, double beta2,
                                    double eps, int64_t step, uint32_t seed, const float* lr_dev,
                                    const int64_t* step_dev, const float* scale, fast_stream_t stream) {
  const char* fn = "fast_adamw";
  const fast_status_t s = aw_list(fn, tensors, count, grad_dtype);
  if (s != FAST_OK) return s;
  if (format != FAST_STATE_F32 && format != FAST_STATE_MXFP8)
    return fail(FAST_ERR_INVALID_ARG, "%s: bad state format", fn);
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
    return fail(FAST_ERR_INVALID_ARG, "%s: beta1 or beta2 outside [0, 1)", fn);
  if (!(eps >= 0.0) || !std::isfinite(eps) || !std::isfinite(lr))
    return fail(FAST_ERR_INVALID_ARG, "%s: lr or eps", fn);
  if (!step_dev && step < 1) return fail(FAST_ERR_INVALID_ARG, "%s: step = %lld < 1", fn, (long long)step);
  if (!aligned(lr_dev, 4) || !aligned(step_dev, 8) || !aligned(scale, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: lr_dev/step_dev/scale misaligned", fn);
  const bool low = format == FAST_STATE_MXFP8;
  const int64_t es = low ? 1 : 4, gs = elem_size(grad_dtype);
  // (on the heap: 115 KB of them are too much for the stack of a small thread)
  const std::unique_ptr<AwRange[]> ranges(new (std::nothrow) AwRange[count * 7 + 3]);
  if (!ranges) return fail(FAST_ERR_WORKSPACE, "%s: no host memory for %d tensors", fn, count);
  AwRange* r = ranges.get();
  int k = aw_add(r, 0, lr_dev, 4, false);
  k = aw_add(r, k, step_dev, 8, false);
  k = aw_add(r, k, scale, 4, false);
  int64_t total = 0;
  for (int j = 0; j < count; ++j) {
    const fast_adamw_tensor_t& t = tensors[j];
    if (!low && (t.m_scale || t.v_scale))
      return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: scales of fp32 states", fn, j);
    if (!std::isfinite(t.decay)) return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: decay", fn, j);
    if (t.n == 0) continue;
    if (!t.w || !t.m || !t.v || (low && (!t.m_scale || !t.v_scale)))
      return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: NULL w/m/v or scales", fn, j);
    if (!aligned(t.w, 4) || !aligned(t.m, es) || !aligned(t.v, es) || !aligned(t.copy, 2))
      return fail(FAST_ERR_UNSUPPORTED, "%s: tensor %d: an array not aligned to its elements", fn, j);
    k = aw_add(r, k, t.w, 4 * t.n, true);
    k = aw_add(r, k, t.m, es * t.n, true);
    k = aw_add(r, k, t.v, es * t.n, true);
    k = aw_add(r, k, t.copy, 2 * t.n, true);
    k = aw_add(r, k, t.grad, gs * t.n, false);
    if (low) {
      k = aw_add(r, k, t.m_scale, (t.n + 31) / 32, true);
      k = aw_add(r, k, t.v_scale, (t.n + 31) / 32, true);
    }
    total += t.n;
  }
  if (aw_overlap(r, k)) return fail(FAST_ERR_INVALID_ARG, "%s: an array that is written overlaps another", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  AwArgs a = {};
  a.b1 = beta1;
  a.b2 = beta2;
  a.eps = eps > 0.0 ? std::max(eps, 0x1p-149) : 0.0;   // (an fp32 number: above 0 where eps is, so that 0 / eps is 0)
  a.lr = lr;
  a.step = step;
  if (!step_dev) {
    a.bc1 = float(1.0 / (1.0 - std::pow(beta1, double(step))));
    a.bc2 = float(1.0 / std::sqrt(1.0 - std::pow(beta2, double(step))));
  }
  a.seed = seed;
  a.lr_dev = lr_dev;
  a.step_dev = step_dev;
  a.scale = scale;
  const int64_t chunk = AW_UNIT;
  // more than the 256 MB last-level cache holds is streamed: 1e8 elements with fp32 states 520 -> 489 us
  const bool nt = total * (low ? 16 : 28) > (int64_t(256) << 20);
  // launches fewer than 2^32 threads; larger lists are refused before the first of them
  int64_t blocks = 0;
  for (int j = 0; j < count; ++j) blocks += (tensors[j].n + chunk - 1) / chunk;
  if (!grid_fits(blocks, AW_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  if (blocks == 0) return ok();
  auto launch = [&] {
    if (a.count == 0) return;
    const dim3 grid(a.first[a.count]);
#define FAST_AW(G, L) \
  if (nt) hipLaunchKernelGGL((k_adamw<G, L, true>), grid, dim3(AW_THREADS), 0, st, a); \
  else hipLaunchKernelGGL((k_adamw<G, L, false>), grid, dim3(AW_THREADS), 0, st, a)
    if (grad_dtype == FAST_F32) {
      if (low) { FAST_AW(float, true); } else { FAST_AW(float, false); }
    } else {
      if (low) { FAST_AW(uint16_t, true); } else { FAST_AW(uint16_t, false); }
    }
#undef FAST_AW
    a.count = 0;
  };
  for (int j = 0; j < count; ++j) {
    const fast_adamw_tensor_t& t = tensors[j];
    if (t.n == 0) continue;
    a.t[a.count] = {t.w, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, t.decay, uint32_t(j)};
    a.first[a.count + 1] = a.first[a.count] + uint32_t((t.n + chunk - 1) / chunk);
    if (++a.count == AW_TENSORS) launch();
  }
  launch();
  return check_launch(fn);
}

extern "C" size_t fast_grad_norm_workspace(int64_t total, int count) {
  if (total < 0 || count < 0 || count > AW_COUNT || total >= int64_t(AW_COUNT) * AW_MAX_N) return 0;
  return size_t(std::max(total / GN_CHUNK, std::min(total, GN_SHORT) / GN_CHUNK_SHORT) + count + 1) * sizeof(double);
}

extern "C" fast_status_t fast_grad_norm(const fast_adamw_tensor_t* tensors, int count,
                                        fast_dtype_t grad_dtype, float max_norm, float* norm, float* scale,
                                        void* ws, size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_grad_norm";
  const fast_status_t s = aw_list(fn, tensors, count, grad_dtype);
  if (s != FAST_OK) return s;
  if (!(max_norm > 0.f)) return fail(FAST_ERR_INVALID_ARG, "%s: max_norm is not above 0", fn);
  if (!norm) return fail(FAST_ERR_INVALID_ARG, "%s: NULL norm", fn);
  if (norm == scale) return fail(FAST_ERR_INVALID_ARG, "%s: norm and scale are one place", fn);
  if (!aligned(norm, 4) || !aligned(scale, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: norm/scale not 4-byte aligned", fn);
  int64_t total = 0, blocks = 0;
  for (int j = 0; j < count; ++j) {
    const int64_t bytes = elem_size(grad_dtype) * tensors[j].n;
    if (meet(norm, 4, tensors[j].grad, bytes) || meet(scale, 4, tensors[j].grad, bytes))
      return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: norm or scale lies in grad", fn, j);
    total += tensors[j].n;
  }
  const int chunk = total <= GN_SHORT ? GN_CHUNK_SHORT : GN_CHUNK;
  for (int j = 0; j < count; ++j) blocks += (tensors[j].n + chunk - 1) / chunk;
  const size_t need = fast_grad_norm_workspace(total, count);
  if (!ws || ws_bytes < need)
    return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0, need);
  if (!aligned(ws, 8)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 8-byte aligned", fn);
  if (meet(norm, 4, ws, int64_t(need)) || meet(scale, 4, ws, int64_t(need)))
    return fail(FAST_ERR_INVALID_ARG, "%s: norm or scale lies in the workspace", fn);
  for (int j = 0; j < count; ++j)
    if (meet(ws, int64_t(need), tensors[j].grad, elem_size(grad_dtype) * tensors[j].n))
      return fail(FAST_ERR_INVALID_ARG, "%s: tensor %d: the workspace overlaps grad", fn, j);
  if (!grid_fits(blocks, GN_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  GnArgs a = {};
  a.part = static_cast<double*>(ws);
  a.chunk = chunk;
  auto launch = [&] {
    if (a.count == 0) return;
    const dim3 grid(a.first[a.count]);
    if (grad_dtype == FAST_F32) hipLaunchKernelGGL(k_grad_norm<float>, grid, dim3(GN_THREADS), 0, st, a);
    else hipLaunchKernelGGL(k_grad_norm<uint16_t>, grid, dim3(GN_THREADS), 0, st, a);
    a.part += a.first[a.count];
    a.count = 0;
  };
  for (int j = 0; j < count; ++j) {
    if (tensors[j].n == 0) continue;
    a.g[a.count] = tensors[j].grad;
    a.n[a.count] = tensors[j].n;
    a.first[a.count + 1] = a.first[a.count] + uint32_t((tensors[j].n + chunk - 1) / chunk);
    if (++a.count == GN_TENSORS) launch();
  }
  launch();
  hipLaunchKernelGGL(k_grad_norm_last, dim3(1), dim3(GN_LAST), 0, st, static_cast<const double*>(ws), blocks,
                     max_norm, norm, scale);
  return check_launch(fn);
}
