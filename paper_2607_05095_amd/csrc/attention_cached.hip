// attention_cached.hip -- edge softmax + aggregation fused (Sec. 4.3), K|V rows
// read from a cache in 8 or 4 bits through ids and a slot map.
//   t[e,h] = LReLU(scale <Q[v,h], K[slot e,h]>),  out[v,h] = sum softmax(t)[e,h] V[slot e,h]
// over the segment's edges that have a slot; lse = log sum exp t.
//
// Bound by HBM: per edge an id, a slot and a record of about H*dh*(2 or 1) bytes
// at a random place, against two fused multiply-adds per element.  A wave owns a
// segment, or a piece of a long one.  L lanes hold a record's heads, 8 codes of K
// and of V each, so 64 / L records are read at a time, CA_ROWS of them per lane in
// flight; each group of L lanes keeps its own running maximum, sum and
// accumulators (one pass, base 2), which are joined across the groups at the
// end.  The ids and slots of a round are read by one lane each and handed round.
//
// Segments longer than `cap` edges are cut at the multiples of cap (a power of
// two) in the block's edge order: a wave per multiple finds its segment with a
// 64-way search of the offsets and leaves at once unless that is a long one.
// Pieces write (maximum, sum, accumulators) to the workspace, and a second launch
// joins a segment's pieces in their order.
#include "attention.h"
#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int CA_THREADS = 256;
constexpr int CA_ROWS = 4;           // records in flight per lane

struct CaArgs {
  int64_t N, E;
  const int32_t* off;
  int H, dh, L;                      // L: lanes per record (a power of two up to 64)
  int shift;                         // cap = 1 << shift
  int64_t cells;                     // multiples of cap that may cut a segment
  const int64_t* ids;
  int64_t id_bound;
  const int32_t* slot_map;
  int64_t cache_rows;
  MxRecord rec;
  const uint8_t* cache;
  const void* Q;
  float scale, slope;
  void* out;
  float* lse;
  float* part;                       // [2 per multiple of cap][H][dh + 2]
};

__device__ __forceinline__ void ca_segment(const CaArgs& a, int64_t v, int64_t& s, int64_t& t) {
  s = clamp64(a.off[v], 0, a.E);
  t = clamp64(a.off[v + 1], s, a.E);
}

// Last v with off[v] <= x (off[0] is taken as 0): every round the lanes try 64
// equally spaced offsets.
__device__ __forceinline__ int64_t ca_find(const CaArgs& a, int64_t x) {
  const int lane = threadIdx.x & 63;
  int64_t lo = 0, hi = a.N;
  while (hi - lo > 1) {
    const int64_t step = (hi - lo + 63) >> 6, i = lo + lane * step;
    const bool le = lane == 0 || (i < hi && a.off[i] <= x);
    const int last = 63 - __builtin_clzll(__ballot(le));
    lo += last * step;
    hi = hi < lo + step ? hi : lo + step;
  }
  return lo;
}

__device__ __forceinline__ float ca_pow2(float x, float m) {   // 2^(x - m), 0 for x = -inf
  return __builtin_amdgcn_exp2f(x - (m == -INFINITY ? 0.f : m));
}

template <typename T, int FMT, int LPH>
__global__ void __launch_bounds__(CA_THREADS) k_attn_cached(CaArgs a) {
  constexpr int PB = FMT == FAST_MXFP4 ? MX_PIECE / 2 : MX_PIECE;
  const int lane = threadIdx.x & 63;
  int64_t item = int64_t(blockIdx.x) * (CA_THREADS / 64) + (threadIdx.x >> 6);
  const int64_t cuts = a.cells;      // items [0, cuts): the pieces that start at a multiple of cap
  int64_t v, s, t, e0, e1, slot = -1;
  if (item < cuts) {
    const int64_t m = item + 1, x = m << a.shift;
    v = ca_find(a, x);
    ca_segment(a, v, s, t);
    if (!(s < x && x < t) || t - s <= (int64_t(1) << a.shift)) return;
    e0 = x;
    e1 = t < x + (int64_t(1) << a.shift) ? t : x + (int64_t(1) << a.shift);
    slot = 2 * m;
  } else {
    v = item - cuts;
    if (v >= a.N) return;
    ca_segment(a, v, s, t);
    e0 = s;
    e1 = t;
    if (t - s > (int64_t(1) << a.shift)) {
      const int64_t m = s >> a.shift;
      e1 = (m + 1) << a.shift;
      slot = 2 * m + 1;
    }
  }
  const int L = a.L, GR = 64 / L, gi = lane / L;
  const int h = blockIdx.y * (L / LPH) + (lane & (L - 1)) / LPH, l = lane & (LPH - 1);
  const bool mine = h < a.H && l * MX_PIECE < a.dh;
  const int H = a.H, dh = a.dh;

  float q[8];
#pragma unroll
  for (int j = 0; j < 8; j += CHUNK<T>)
    load_chunk(static_cast<const T*>(a.Q) + (v * H + (h < H ? h : 0)) * dh + l * 8 + j,
               mine ? dh - l * 8 - j : 0, q + j);
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] *= a.scale * LOG2E;

  const int koff = h * a.rec.code_bytes + l * PB, voff = koff + H * a.rec.code_bytes;
  const int ksc = a.rec.scale_off + h * a.rec.groups + (l >> 2), vsc = ksc + H * a.rec.groups;
  float mx = -INFINITY, Z = 0.f, acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  const int per = GR * CA_ROWS < 64 ? GR * CA_ROWS : 64;       // edges per round
  for (int64_t base = e0; base < e1; base += per) {
    int my = -1;
    if (lane < per && base + lane < e1)
      my = int(mx_slot(a.ids[base + lane], a.id_bound, a.slot_map, a.cache_rows));
    MxPiece<FMT> kc[CA_ROWS], vc[CA_ROWS];
    uint32_t kb[CA_ROWS], vb[CA_ROWS];
    bool ok[CA_ROWS];
#pragma unroll
    for (int i = 0; i < CA_ROWS; ++i) {
      const int r = i * GR + gi;
      const int sl = __shfl(my, r & 63);
      ok[i] = r < per && sl >= 0;
      kc[i].zero();
      vc[i].zero();
      kb[i] = vb[i] = 127u;
      if (ok[i] && mine) {
        const uint8_t* rec = a.cache + sl * a.rec.stride;
        kc[i].load(rec + koff);
        vc[i].load(rec + voff);
        kb[i] = rec[ksc];
        vb[i] = rec[vsc];
      }
    }
    float tt[CA_ROWS], mn = mx;
#pragma unroll
    for (int i = 0; i < CA_ROWS; ++i) {
      float k[8], d = 0.f;
      kc[i].unpack(mx_scale(kb[i]), k);
#pragma unroll
      for (int j = 0; j < 8; ++j) d = fmaf(q[j], k[j], d);
      d = group_sum_ct<LPH>(d);
      tt[i] = ok[i] ? (d > 0.f ? d : a.slope * d) : -INFINITY;
      mn = fmaxf(mn, tt[i]);
    }
    const float corr = ca_pow2(mx, mn);
    mx = mn;
    Z *= corr;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] *= corr;
#pragma unroll
    for (int i = 0; i < CA_ROWS; ++i) {
      const float w = ca_pow2(tt[i], mx);
      float x[8];
      vc[i].unpack(mx_scale(vb[i]), x);
      Z += w;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = fmaf(w, x[j], acc[j]);
    }
  }
  // join the groups
  for (int o = L; o < 64; o *= 2) {
    const float om = __shfl_xor(mx, o), oz = __shfl_xor(Z, o);
    const float mn = fmaxf(mx, om);
    const float c0 = ca_pow2(mx, mn), c1 = ca_pow2(om, mn);
    Z = Z * c0 + oz * c1;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = acc[j] * c0 + __shfl_xor(acc[j], o) * c1;
    mx = mn;
  }
  if (gi != 0 || !mine) return;
  if (slot >= 0) {
    float* p = a.part + (slot * H + h) * (dh + 2);
    if (l == 0) {
      p[0] = mx;
      p[1] = Z;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (l * 8 + j < dh) p[2 + l * 8 + j] = acc[j];
    return;
  }
  const bool some = !(Z == 0.f);       // also of a NaN
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = some ? acc[j] / Z : 0.f;
  T* out = static_cast<T*>(a.out) + (v * H + h) * dh + l * 8;
#pragma unroll
  for (int j = 0; j < 8; j += CHUNK<T>) store_chunk(out + j, dh - l * 8 - j, acc + j);
  if (a.lse && l == 0) a.lse[v * H + h] = some ? (mx + log2f(Z)) * LN2 : -INFINITY;
}

// The pieces of the long segment that starts between multiples m and m + 1 of
// cap, if there is one: a workgroup per (m, head), threads over the pieces for
// the maximum and the sum, then over (element, every CJ_SLICES-th piece).
constexpr int CJ_THREADS = 256, CJ_COLS = 32, CJ_SLICES = CJ_THREADS / CJ_COLS;
template <typename T>
__global__ void __launch_bounds__(CJ_THREADS) k_attn_cached_join(CaArgs a) {
  __shared__ float s_red[CJ_THREADS / 64];
  __shared__ float s_acc[CJ_SLICES][CJ_COLS];
  const int64_t m = blockIdx.x, x = (m + 1) << a.shift, cap = int64_t(1) << a.shift;
  const int h = blockIdx.y, H = a.H, dh = a.dh;
  const int64_t v = ca_find(a, x);
  int64_t s, t;
  ca_segment(a, v, s, t);
  if (!(s < x && x < t) || t - s <= cap || (s >> a.shift) != m) return;
  const int64_t n = ((t - 1) >> a.shift) - m + 1;      // pieces; the first is slot 2m + 1, then 2(m + k)
  auto piece = [&](int64_t k) {
    return a.part + ((k == 0 ? 2 * m + 1 : 2 * (m + k)) * H + h) * (dh + 2);
  };
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float mx = -INFINITY;
  for (int64_t k = threadIdx.x; k < n; k += CJ_THREADS) mx = fmaxf(mx, piece(k)[0]);
  for (int o = 1; o < 64; o *= 2) mx = fmaxf(mx, __shfl_xor(mx, o));
  if (lane == 0) s_red[wave] = mx;
  __syncthreads();
  for (int w = 0; w < CJ_THREADS / 64; ++w) mx = fmaxf(mx, s_red[w]);
  __syncthreads();
  float Z = 0.f;
  for (int64_t k = threadIdx.x; k < n; k += CJ_THREADS) Z += piece(k)[1] * ca_pow2(piece(k)[0], mx);
  Z = group_sum(Z, 64);
  if (lane == 0) s_red[wave] = Z;
  __syncthreads();
  Z = 0.f;
  for (int w = 0; w < CJ_THREADS / 64; ++w) Z += s_red[w];
  const bool some = !(Z == 0.f);
  const int col = threadIdx.x % CJ_COLS, sl = threadIdx.x / CJ_COLS;
  T* out = static_cast<T*>(a.out) + (v * H + h) * dh;
  for (int c0 = 0; c0 < dh; c0 += CJ_COLS) {
    float acc = 0.f;
    if (c0 + col < dh)
      for (int64_t k = sl; k < n; k += CJ_SLICES)
        acc += piece(k)[2 + c0 + col] * ca_pow2(piece(k)[0], mx);
    s_acc[sl][col] = acc;
    __syncthreads();
    if (sl == 0 && c0 + col < dh) {
      for (int k = 1; k < CJ_SLICES; ++k) acc += s_acc[k][col];
      const float o = some ? acc / Z : 0.f;
      VecIO<T, 1>::store(out + c0 + col, &o);
    }
    __syncthreads();
  }
  if (a.lse && threadIdx.x == 0) a.lse[v * H + h] = some ? (mx + log2f(Z)) * LN2 : -INFINITY;
}

// Piece length of long segments: short enough that E / cap pieces fill the
// chip, long enough that a piece's partial result is small beside its records.
static int ca_shift(int64_t E) {
  int s = 6;
  while (s < 8 && (E >> (s + 1)) >= 2048) ++s;
  return s;
}

static int pow2_at_least(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

template <typename T, int FMT>
static void launch_ca(const CaArgs& a, int lph, dim3 grid, hipStream_t st) {
#define FAST_CA(n) case n: hipLaunchKernelGGL((k_attn_cached<T, FMT, n>), grid, dim3(CA_THREADS), 0, st, a); break
  switch (lph) { FAST_CA(1); FAST_CA(2); FAST_CA(4); FAST_CA(8); FAST_CA(16); FAST_CA(32); }
#undef FAST_CA
}

}  // namespace fast

using namespace fast;

extern "C" size_t fast_edge_attention_cached_workspace(int64_t num_dst, int64_t num_edges, int H,
                                                       int dh) {
  if (num_dst < 0 || num_edges < 0 || num_edges >= (int64_t(1) << 31) || H <= 0 || dh <= 0 || H > 64 ||
      dh > 256 || H * dh > 1024)
    return 0;
  const int64_t slots = 2 * ((num_edges >> ca_shift(num_edges)) + 1);
  return align_up(size_t(slots) * H * (dh + 2) * sizeof(float), 16);
}

extern "C" fast_status_t fast_edge_attention_fwd_cached(
    const fast_tcsr_t* g, int H, int dh, fast_dtype_t dtype, const void* Q, const int64_t* ids,
    int64_t id_bound, const int32_t* slot_map, fast_cache_format_t format, const void* cache,
    int64_t cache_rows, float scale, float neg_slope, void* out, float* lse, void* ws,
    size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_edge_attention_fwd_cached";
  if (!g) return fail(FAST_ERR_INVALID_ARG, "%s: graph is NULL", fn);
  const int64_t N = g->num_dst, E = g->num_edges;
  if (N < 0 || E < 0 || id_bound < 0 || cache_rows < 0)
    return fail(FAST_ERR_INVALID_ARG, "%s: negative size", fn);
  if (H <= 0 || dh <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: H = %d, dh = %d", fn, H, dh);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (format != FAST_MXFP8 && format != FAST_MXFP4)
    return fail(FAST_ERR_INVALID_ARG, "%s: bad cache format", fn);
  if (H > 64 || dh > 256 || H * dh > 1024)
    return fail(FAST_ERR_UNSUPPORTED, "%s: H = %d, dh = %d (at most 64, 256, 1024 together)", fn, H, dh);
  if (E >= (int64_t(1) << 31) || N >= (int64_t(1) << 31) || cache_rows >= (int64_t(1) << 31))
    return fail(FAST_ERR_UNSUPPORTED, "%s: N, E or cache_rows >= 2^31", fn);
  if (N == 0 && E > 0) return fail(FAST_ERR_INVALID_ARG, "%s: E > 0 edges but no destination", fn);
  if (N == 0) return ok();
  if (!g->dst_offsets || !Q || !out) return fail(FAST_ERR_INVALID_ARG, "%s: NULL dst_offsets/Q/out", fn);
  if (E > 0 && (!ids || (cache_rows > 0 && !cache)))
    return fail(FAST_ERR_INVALID_ARG, "%s: NULL ids/cache", fn);
  const size_t es = elem_size(dtype);
  if (!aligned(Q, es) || !aligned(out, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(cache, 16) || !aligned(ids, 8) || !aligned(lse, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: cache, ids or lse misaligned", fn);
  const size_t need = fast_edge_attention_cached_workspace(N, E, H, dh);
  if (!ws || ws_bytes < need)
    return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0, need);
  if (!aligned(ws, 16)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 16-byte aligned", fn);
  CaArgs a = {};
  a.N = N;
  a.E = E;
  a.off = g->dst_offsets;
  a.H = H;
  a.dh = dh;
  a.shift = ca_shift(E);
  a.cells = E > 0 ? (E - 1) >> a.shift : 0;
  a.ids = ids;
  a.id_bound = id_bound;
  a.slot_map = slot_map;
  a.cache_rows = cache_rows;
  a.rec = mx_record(2 * H, dh, format);
  a.cache = static_cast<const uint8_t*>(cache);
  a.Q = Q;
  a.scale = scale;
  a.slope = neg_slope;
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  const int lph = pow2_at_least((dh + MX_PIECE - 1) / MX_PIECE);
  int hpw = pow2_at_least(H);
  if (hpw > 64 / lph) hpw = 64 / lph;
  a.L = lph * hpw;
  const int waves = CA_THREADS / 64;
  const dim3 grid(uint32_t((a.cells + N + waves - 1) / waves), uint32_t((H + hpw - 1) / hpw));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32) {
    if (format == FAST_MXFP8) launch_ca<float, FAST_MXFP8>(a, lph, grid, st);
    else launch_ca<float, FAST_MXFP4>(a, lph, grid, st);
  } else {
    if (format == FAST_MXFP8) launch_ca<uint16_t, FAST_MXFP8>(a, lph, grid, st);
    else launch_ca<uint16_t, FAST_MXFP4>(a, lph, grid, st);
  }
  if (a.cells > 0) {
    const dim3 jg(uint32_t(a.cells), uint32_t(H));
    if (dtype == FAST_F32) hipLaunchKernelGGL((k_attn_cached_join<float>), jg, dim3(CJ_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_attn_cached_join<uint16_t>), jg, dim3(CJ_THREADS), 0, st, a);
  }
  return check_launch(fn);
}
