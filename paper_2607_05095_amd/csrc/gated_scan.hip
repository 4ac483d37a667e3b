// gated_scan.hip -- the gated linear recurrence over the events of each segment.
//   rate = log(1 + e^gate), a = e^(-rate dt), u = 1 - a;  s = a s + u x, h = s
//   back: d = dh + (a d of the event behind);  dx = u d,
//         dgate = d (x - s before) a dt sigmoid(gate)
//
// Bound by HBM: forward three arrays of rows, backward five.  A lane owns GS_VE columns of a
// segment and walks its events in order, the rows of GS_AHEAD events loaded ahead;
// lanes are dealt over (segment, columns) without gaps.  The backward walks windows of
// GS_WIN events from the last to the first: a window's states are formed again in
// registers from its first one, which the forward left in `states`, then its events
// are taken in reverse.
//
// A segment of `cut` events or more (of `cut` only where many lanes are busy with
// others) would keep few lanes busy for long.  It is cut into pieces of `piece` events, the last
// up to twice as long: a launch forms every piece's (product of a, result from zero), while
// other workgroups walk the short segments; a second chains them, a third walks the
// pieces from their known starts.  Piece j of a segment starts at b + j * piece; the
// starts of two pieces never share a slot of `piece` positions, so slot = start / piece
// numbers them.
#include <algorithm>

#include "rows.h"

namespace fast {

constexpr int GS_THREADS = 256;
constexpr int GS_AHEAD = 8;          // events whose rows are loaded together
constexpr int GS_WIN = 16;           // events of a backward window
constexpr int64_t GS_MAX_D = 8192;
constexpr int GS_CARRY = 16;         // pieces whose sums are loaded together

// ------------------------------------------------------------------ the gate
struct Gate {
  float a, u, k;                     // k: the slope of u over the gate, a dt sigmoid(gate)
};

// e^-x 2^up for x >= 0 within 2 ulp: the product with log2(e) in two parts.
__device__ __forceinline__ float exp_neg(float x, float up = 0.f) {
  const float h = -x * 0x1.715476p+0f;
  const float l = fmaf(-x, 0x1.715476p+0f, -h) - x * 0x1.4ae0cp-26f;
  const float e = __builtin_amdgcn_exp2f(h + up);
  return h + up < -126.f ? e : fmaf(e, l * 0x1.62e43p-1f, e);
}

// 1 / x, x >= 1 (or not a number).
__device__ __forceinline__ float rcp(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.f), r, r);
}

// u = 1 - a keeps its relative accuracy for slow gates and a for fast ones.
template <bool SPAN>
__device__ __forceinline__ Gate gate_of(float g, float dt) {
  Gate q;
  const float t = exp_neg(fabsf(g));                       // sigmoid(|g|) = 1 / (1 + t)
  const float r = rcp(1.f + t), big = r, small = t * r;
  const float sig = g >= 0.f ? big : small;
  if constexpr (!SPAN) {
    q.u = g >= 0.f ? big : small;
    q.a = g >= 0.f ? small : big;
    q.k = q.a * sig;
    return q;
  }
  // log(1 + t) = 2 artanh(z), z = t / (2 + t) <= 1/3: odd powers up to z^15 (2^-26)
  const float z = t * rcp(2.f + t), z2 = z * z;
  float p = 1.f / 15.f;
  p = fmaf(p, z2, 1.f / 13.f);
  p = fmaf(p, z2, 1.f / 11.f);
  p = fmaf(p, z2, 1.f / 9.f);
  p = fmaf(p, z2, 1.f / 7.f);
  p = fmaf(p, z2, 1.f / 5.f);
  p = fmaf(p, z2, 1.f / 3.f);
  const float rate = fmaf(2.f * z * z2, p, 2.f * z) + (g > 0.f ? g : 0.f);
  dt = dt < 0.f ? 0.f : dt;
  float y = rate * dt;
  const bool far = g < -86.f;                              // a rate below what fp32 holds, e^gate
  if (far) y = exp_neg(-g, 120.f) * (dt * 0x1p-120f);
  // 1 - e^-y: its series up to y^10 below log 2 (2^-26), the difference above
  const float e = exp_neg(y);
  float s = -1.f / 3628800.f;
  s = fmaf(s, y, 1.f / 362880.f);
  s = fmaf(s, y, -1.f / 40320.f);
  s = fmaf(s, y, 1.f / 5040.f);
  s = fmaf(s, y, -1.f / 720.f);
  s = fmaf(s, y, 1.f / 120.f);
  s = fmaf(s, y, -1.f / 24.f);
  s = fmaf(s, y, 1.f / 6.f);
  s = fmaf(s, y, -0.5f);
  s = fmaf(s * y, y, y);
  const bool slow = y < 0.693f;
  q.u = slow ? s : 1.f - e;
  q.a = e;
  q.k = far ? e * y : e * dt * sig;
  return q;
}

// ------------------------------------------------------------------ rows
struct GsArgs {
  const int32_t* off;
  int64_t N, E;
  int D, C;                          // columns; lanes of a row
  const void* x;
  const void* gate;
  int64_t ldx;
  const float* dt;
  const float* h0;                   // forward: start, backward: the same
  void* h;
  float* h_last;
  float* states;
  // backward
  const void* dh;
  const float* dh_last;
  void* dx;
  void* dgate;
  int64_t lddx;
  float* dh0;
  // long segments
  int64_t cut;                       // events of a segment that is cut (E + 1 and more: none is)
  int piece;
  int64_t slots;
  int32_t* owner;                    // the segment that has a piece in the slot, or -1
  float* pa;                         // [slots][D]: products of a, then the pieces' starts
  float* pb;                         // [slots][D]: results from zero
  uint32_t direct;                   // workgroups of the short segments, before those of the pieces
};

// VE columns at p, n of them in the row
template <typename T, int VE>
__device__ __forceinline__ void gs_load(const T* p, int n, float* x) {
  if (n >= VE) {
    if constexpr (VE == 4 && sizeof(T) == 4) {
      load_chunk_of(p, 4, x);
    } else if constexpr (VE == 4) {
      const u32x2_e w = *reinterpret_cast<const u32x2_e*>(p);
      x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    } else if constexpr (VE == 2 && sizeof(T) == 4) {
      const f32x2_e w = *reinterpret_cast<const f32x2_e*>(p);
      x[0] = w.x; x[1] = w.y;
    } else if constexpr (VE == 2) {
      const uint32_t w = *reinterpret_cast<const u32_e*>(p);
      x[0] = bf16_lo(w); x[1] = bf16_hi(w);
    } else if constexpr (sizeof(T) == 4) {
      x[0] = p[0];
    } else {
      x[0] = bf16_at(p);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    x[j] = 0.f;
    if (j < n) {
      if constexpr (sizeof(T) == 4) x[j] = p[j];
      else x[j] = bf16_at(p + j);
    }
  }
}
template <typename T, int VE>
__device__ __forceinline__ void gs_store(T* p, int n, const float* x) {
  if (n >= VE) {
    if constexpr (VE == 4 && sizeof(T) == 4) store_chunk_of(p, 4, x);
    else if constexpr (VE == 4) *reinterpret_cast<u32x2_e*>(p) = u32x2_e{bf16_pack(x[0], x[1]), bf16_pack(x[2], x[3])};
    else if constexpr (VE == 2 && sizeof(T) == 4) *reinterpret_cast<f32x2_e*>(p) = f32x2_e{x[0], x[1]};
    else if constexpr (VE == 2) *reinterpret_cast<u32_e*>(p) = bf16_pack(x[0], x[1]);
    else if constexpr (sizeof(T) == 4) p[0] = x[0];
    else p[0] = uint16_t(bf16_rne(x[0]));
    return;
  }
#pragma unroll
  for (int j = 0; j < VE; ++j)
    if (j < n) {
      if constexpr (sizeof(T) == 4) p[j] = x[j];
      else p[j] = uint16_t(bf16_rne(x[j]));
    }
}
template <int VE>
__device__ __forceinline__ void gs_start(const float* rows, int64_t row, int D, int c, int n, float* s) {
  if (rows) {
    gs_load<float, VE>(rows + row * D + c, n, s);
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) s[j] = 0.f;
  }
}

// Events [p, t) of a segment that starts at b, from the state s.
template <typename T, int VE, bool SPAN>
__device__ __forceinline__ void fwd_range(const GsArgs& a, int64_t b, int64_t p, int64_t t, int c, int n, float* s) {
  const T* x = static_cast<const T*>(a.x) + c;
  const T* g = static_cast<const T*>(a.gate) + c;
  for (int64_t e = p; e < t; e += GS_AHEAD) {
    float xs[GS_AHEAD][VE], gs[GS_AHEAD][VE], dt[GS_AHEAD];
    const int m = t - e < GS_AHEAD ? int(t - e) : GS_AHEAD;
#pragma unroll
    for (int j = 0; j < GS_AHEAD; ++j)
      if (j < m) {
        gs_load<T, VE>(x + (e + j) * a.ldx, n, xs[j]);
        gs_load<T, VE>(g + (e + j) * a.ldx, n, gs[j]);
        dt[j] = SPAN ? a.dt[e + j] : 1.f;
      }
    if (a.states && e > b && ((e - b) & (GS_WIN - 1)) == 0)
      gs_store<float, VE>(a.states + e / GS_WIN * a.D + c, n, s);
#pragma unroll
    for (int j = 0; j < GS_AHEAD; ++j)
      if (j < m) {
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          const Gate k = gate_of<SPAN>(gs[j][q], dt[j]);
          s[q] = fmaf(k.a, s[q], k.u * xs[j][q]);
        }
        if (a.h) gs_store<T, VE>(static_cast<T*>(a.h) + (e + j) * a.D + c, n, s);
      }
  }
}

// Events [p, t) in reverse, d: what reaches the last of them from behind; returns what reaches
// the event before p.  v: the segment, for its start.
template <typename T, int VE, bool SPAN>
__device__ __forceinline__ void bwd_range(const GsArgs& a, int64_t v, int64_t b, int64_t p, int64_t t, int c, int n,
                                          float* d) {
  if (t <= p) return;
  const T* x = static_cast<const T*>(a.x) + c;
  const T* g = static_cast<const T*>(a.gate) + c;
  const T* dh = static_cast<const T*>(a.dh) + c;
  for (int64_t e = p + (t - p - 1) / GS_WIN * GS_WIN; e >= p; e -= GS_WIN) {
    float u[GS_WIN][VE], w[GS_WIN][VE], k[GS_WIN][VE];     // (w: x, then a)
    const int m = t - e < GS_WIN ? int(t - e) : GS_WIN;
    float s[VE];
    if (e == b) gs_start<VE>(a.h0, v, a.D, c, n, s);
    else gs_load<float, VE>(a.states + e / GS_WIN * a.D + c, n, s);
#pragma unroll
    for (int j = 0; j < GS_WIN; ++j)
      if (j < m) {
        gs_load<T, VE>(x + (e + j) * a.ldx, n, w[j]);
        gs_load<T, VE>(g + (e + j) * a.ldx, n, k[j]);
      }
#pragma unroll
    for (int j = 0; j < GS_WIN; ++j)
      if (j < m) {
        const float dt = SPAN ? a.dt[e + j] : 1.f;
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          const Gate y = gate_of<SPAN>(k[j][q], dt);
          const float xv = w[j][q];
          k[j][q] = y.k * (xv - s[q]);
          s[q] = fmaf(y.a, s[q], y.u * xv);
          u[j][q] = y.u;
          w[j][q] = y.a;
        }
      }
#pragma unroll
    for (int j = GS_WIN - 1; j >= 0; --j)
      if (j < m) {
        float y[VE], o[VE];
        if (a.dh) {
          gs_load<T, VE>(dh + (e + j) * a.D, n, y);
        } else {
#pragma unroll
          for (int q = 0; q < VE; ++q) y[q] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          d[q] += y[q];
          y[q] = u[j][q] * d[q];
          o[q] = k[j][q] * d[q];
          d[q] *= w[j][q];
        }
        gs_store<T, VE>(static_cast<T*>(a.dx) + (e + j) * a.lddx + c, n, y);
        gs_store<T, VE>(static_cast<T*>(a.dgate) + (e + j) * a.lddx + c, n, o);
      }
  }
}

// ------------------------------------------------------------------ pieces
// Segments that start at or before a position, by a wave: 64 probes a round.
__device__ __forceinline__ int64_t starts_upto(const int32_t* __restrict__ off, int64_t N, int64_t pos) {
  int64_t lo = 0, hi = N;
  const int lane = threadIdx.x & 63;
  while (hi > lo) {
    const int64_t step = (hi - lo + 63) >> 6, i = lo + lane * step;
    const bool in = i < hi && off[i < hi ? i : hi - 1] <= pos;
    const int c = __popcll(__ballot(in));
    if (c == 0) break;
    hi = min(hi, lo + c * step);
    lo = lo + (c - 1) * step + 1;
  }
  return lo;
}
// The piece [p, t) of segment [b, e) that starts in slot k, if there is one.
struct Piece {
  int64_t p, t;
};
__device__ __forceinline__ bool piece_in(const GsArgs& a, int64_t b, int64_t e, int64_t k, Piece& r) {
  if (e - b < a.cut) return false;
  const int64_t q = k * a.piece, j = b >= q ? 0 : (q - b + a.piece - 1) / a.piece;
  r.p = b + j * a.piece;
  if (r.p >= q + a.piece || r.p + a.piece > e) return false;
  r.t = e - r.p < 2 * int64_t(a.piece) ? e : r.p + a.piece;
  return true;
}
__device__ __forceinline__ void segment_of(const GsArgs& a, int64_t v, int64_t& b, int64_t& e) {
  b = clamp64(a.off[v], 0, a.E);
  e = clamp64(a.off[v + 1], 0, a.E);
}
// The segment with a piece in slot k: that of the slot's first position, or of its last.
__device__ __forceinline__ int64_t find_owner(const GsArgs& a, int64_t k) {
  const int64_t q = k * a.piece;
  int64_t b, e;
  Piece r;
  const int64_t v = starts_upto(a.off, a.N, q) - 1;
  if (v >= 0) {
    segment_of(a, v, b, e);
    if (piece_in(a, b, e, k, r)) return v;
  }
  const int64_t w = starts_upto(a.off, a.N, q + a.piece - 1) - 1;
  if (w > v) {
    segment_of(a, w, b, e);
    if (piece_in(a, b, e, k, r)) return w;
  }
  return -1;
}

// A workgroup per slot: threads over the columns of its piece.
template <typename T, int VE, bool SPAN, bool BACK>
__device__ __forceinline__ void piece_sums(const GsArgs& a, int64_t k) {
  const int64_t v = find_owner(a, k);
  if (threadIdx.x == 0) a.owner[k] = int32_t(v);
  if (v < 0) return;
  int64_t b, e;
  Piece r;
  segment_of(a, v, b, e);
  piece_in(a, b, e, k, r);
  // nothing reads the sums of the piece that the chain ends with
  if (BACK ? r.p == b : r.t == e) return;
  for (int i = threadIdx.x; i < a.C; i += GS_THREADS) {
    const int c = i * VE, n = a.D - c;
    float pa[VE], pb[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      pa[q] = 1.f;
      pb[q] = 0.f;
    }
    const T* x = (BACK ? static_cast<const T*>(a.dh) : static_cast<const T*>(a.x)) + c;
    const int64_t ld = BACK ? a.D : a.ldx;
    const T* g = static_cast<const T*>(a.gate) + c;
    const int64_t len = r.t - r.p;
    for (int64_t o = 0; o < len; o += GS_AHEAD) {
      float xs[GS_AHEAD][VE], gs[GS_AHEAD][VE], dt[GS_AHEAD];
      const int m = len - o < GS_AHEAD ? int(len - o) : GS_AHEAD;
#pragma unroll
      for (int j = 0; j < GS_AHEAD; ++j)
        if (j < m) {
          const int64_t i = BACK ? r.t - 1 - o - j : r.p + o + j;
          gs_load<T, VE>(g + i * a.ldx, n, gs[j]);
          if (!BACK || a.dh) {
            gs_load<T, VE>(x + i * ld, n, xs[j]);
          } else {
#pragma unroll
            for (int q = 0; q < VE; ++q) xs[j][q] = 0.f;
          }
          dt[j] = SPAN ? a.dt[i] : 1.f;
        }
#pragma unroll
      for (int j = 0; j < GS_AHEAD; ++j)
        if (j < m) {
#pragma unroll
          for (int q = 0; q < VE; ++q) {
            const Gate y = gate_of<SPAN>(gs[j][q], dt[j]);
            pa[q] *= y.a;
            pb[q] = BACK ? y.a * (pb[q] + xs[j][q]) : fmaf(y.a, pb[q], y.u * xs[j][q]);
          }
        }
    }
    gs_store<float, VE>(a.pa + k * a.D + c, n, pa);
    gs_store<float, VE>(a.pb + k * a.D + c, n, pb);
  }
}

// ------------------------------------------------------------------ kernels
template <typename T, int VE, bool SPAN, bool BACK>
__global__ void __launch_bounds__(GS_THREADS) k_scan(GsArgs a) {
  if (blockIdx.x >= a.direct) {
    piece_sums<T, VE, SPAN, BACK>(a, blockIdx.x - a.direct);
    return;
  }
  const uint32_t i = blockIdx.x * GS_THREADS + threadIdx.x;
  const int64_t v = i / uint32_t(a.C);
  if (v >= a.N) return;
  const int c = int(i - uint32_t(v) * uint32_t(a.C)) * VE, n = a.D - c;
  int64_t b, e;
  segment_of(a, v, b, e);
  if (e - b >= a.cut) return;
  float s[VE];
  if constexpr (BACK) {
    gs_start<VE>(a.dh_last, v, a.D, c, n, s);
    bwd_range<T, VE, SPAN>(a, v, b, b, e, c, n, s);
    if (a.dh0) gs_store<float, VE>(a.dh0 + v * a.D + c, n, s);
  } else {
    gs_start<VE>(a.h0, v, a.D, c, n, s);
    fwd_range<T, VE, SPAN>(a, b, b, e, c, n, s);
    if (a.h_last) gs_store<float, VE>(a.h_last + v * a.D + c, n, s);
  }
}

// The pieces' starts: from the workgroup of the slot that holds a long segment's first piece
// (backward: from the last piece on).  The start of slot k takes pa's place.
template <bool BACK>
__global__ void __launch_bounds__(GS_THREADS) k_scan_chain(GsArgs a) {
  const int64_t k = blockIdx.x;
  const int64_t v = a.owner[k];
  if (v < 0) return;
  int64_t b, e;
  Piece r;
  segment_of(a, v, b, e);
  if (!piece_in(a, b, e, k, r) || r.p != b) return;
  const int64_t pieces = (e - b) / a.piece;
  for (int c = threadIdx.x; c < a.D; c += GS_THREADS) {
    const float* first = BACK ? a.dh_last : a.h0;
    float s = first ? first[v * a.D + c] : 0.f;
    for (int64_t j = 0; j < pieces; j += GS_CARRY) {
      float pa[GS_CARRY], pb[GS_CARRY];
      const int m = pieces - j < GS_CARRY ? int(pieces - j) : GS_CARRY;
#pragma unroll
      for (int q = 0; q < GS_CARRY; ++q)
        if (q < m && j + q + 1 < pieces) {                 // the chain's last piece has no sums
          const int64_t at = (b + (BACK ? pieces - 1 - j - q : j + q) * a.piece) / a.piece * a.D + c;
          pa[q] = a.pa[at];
          pb[q] = a.pb[at];
        }
#pragma unroll
      for (int q = 0; q < GS_CARRY; ++q)
        if (q < m) {
          const int64_t at = (b + (BACK ? pieces - 1 - j - q : j + q) * a.piece) / a.piece * a.D + c;
          a.pa[at] = s;
          if (j + q + 1 < pieces) s = fmaf(pa[q], s, pb[q]);
        }
    }
  }
}

template <typename T, int VE, bool SPAN, bool BACK>
__global__ void __launch_bounds__(GS_THREADS) k_scan_pieces(GsArgs a) {
  const int64_t k = blockIdx.x;
  const int64_t v = a.owner[k];
  if (v < 0) return;
  int64_t b, e;
  Piece r;
  segment_of(a, v, b, e);
  if (!piece_in(a, b, e, k, r)) return;
  for (int i = threadIdx.x; i < a.C; i += GS_THREADS) {
    const int c = i * VE, n = a.D - c;
    float s[VE];
    gs_load<float, VE>(a.pa + k * a.D + c, n, s);
    if constexpr (BACK) {
      bwd_range<T, VE, SPAN>(a, v, b, r.p, r.t, c, n, s);
      if (r.p == b && a.dh0) gs_store<float, VE>(a.dh0 + v * a.D + c, n, s);
    } else {
      fwd_range<T, VE, SPAN>(a, b, r.p, r.t, c, n, s);
      if (r.t == e && a.h_last) gs_store<float, VE>(a.h_last + v * a.D + c, n, s);
    }
  }
}

// ------------------------------------------------------------------ host side
constexpr int GS_PIECE = 64;         // a multiple of GS_WIN
struct GsPlan {
  int64_t cut, slots;
  int piece;
};
static GsPlan gs_plan(int64_t N, int64_t E, int D, int64_t es, int64_t longest) {
  GsPlan p = {};
  p.piece = GS_PIECE;
  // a walk of `cut` events should not outlast half of the whole: an event takes about
  // 0.13 us, the rows of all events their bytes at 6 TB/s
  const int64_t events = 3 * E * D * es / 1600000;
  p.cut = std::max<int64_t>(2 * GS_PIECE, std::min<int64_t>(events, 4096));
  p.slots = (E + p.piece - 1) / p.piece;
  if (E < p.cut || (longest > 0 && longest < p.cut)) {
    p.cut = int64_t(1) << 40;
    p.slots = 0;
  }
  return p;
}

static size_t gs_layout(int64_t slots, int D, char* ws, GsArgs* a) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = ws ? ws + at : nullptr;
    at += align_up(bytes, 256);
    return p;
  };
  char* o = take(size_t(slots) * 4);
  char* pa = take(size_t(slots) * D * 4);
  char* pb = take(size_t(slots) * D * 4);
  if (a) {
    a->owner = reinterpret_cast<int32_t*>(o);
    a->pa = reinterpret_cast<float*>(pa);
    a->pb = reinterpret_cast<float*>(pb);
  }
  return at;
}

static fast_status_t gs_check(const char* fn, const fast_tcsr_t* g, int D, fast_dtype_t dtype, int64_t ldx,
                              const char* ld_name) {
  if (!g) return fail(FAST_ERR_INVALID_ARG, "%s: NULL graph", fn);
  if (g->num_dst < 0 || g->num_edges < 0)
    return fail(FAST_ERR_INVALID_ARG, "%s: N = %lld, E = %lld", fn, (long long)g->num_dst, (long long)g->num_edges);
  if (D <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: D = %d <= 0", fn, D);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (ldx < D) return fail(FAST_ERR_INVALID_ARG, "%s: rows of %d elements, %s = %lld apart", fn, D, ld_name, (long long)ldx);
  if (D > GS_MAX_D) return fail(FAST_ERR_UNSUPPORTED, "%s: D = %d > %lld", fn, D, (long long)GS_MAX_D);
  const int64_t big = int64_t(1) << 31;
  if (g->num_dst >= big || g->num_edges >= big) return fail(FAST_ERR_UNSUPPORTED, "%s: N or E >= 2^31", fn);
  if (ldx >= big) return fail(FAST_ERR_UNSUPPORTED, "%s: %s >= 2^31", fn, ld_name);
  if (g->num_edges * ldx >= (int64_t(1) << 56))
    return fail(FAST_ERR_UNSUPPORTED, "%s: %lld rows, %lld elements apart", fn, (long long)g->num_edges, (long long)ldx);
  if (g->num_dst > 0 && !g->dst_offsets) return fail(FAST_ERR_INVALID_ARG, "%s: NULL dst_offsets", fn);
  if (!aligned(g->dst_offsets, 4)) return fail(FAST_ERR_UNSUPPORTED, "%s: dst_offsets not 4-byte aligned", fn);
  return FAST_OK;
}

template <bool BACK, typename T, int VE, bool SPAN>
static void gs_launch(const GsArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_scan<T, VE, SPAN, BACK>), dim3(uint32_t(a.direct + a.slots)), dim3(GS_THREADS), 0, st, a);
  if (a.slots == 0) return;
  hipLaunchKernelGGL((k_scan_chain<BACK>), dim3(uint32_t(a.slots)), dim3(GS_THREADS), 0, st, a);
  hipLaunchKernelGGL((k_scan_pieces<T, VE, SPAN, BACK>), dim3(uint32_t(a.slots)), dim3(GS_THREADS), 0, st, a);
}

template <bool BACK>
static fast_status_t gs_run(const char* fn, GsArgs& a, fast_dtype_t dtype, int64_t longest, void* ws,
                            hipStream_t st) {
  const int ve = 2;
  a.C = (a.D + ve - 1) / ve;
  const GsPlan p = gs_plan(a.N, a.E, a.D, elem_size(dtype), longest);
  a.cut = p.cut;
  a.piece = p.piece;
  a.slots = p.slots;
  gs_layout(p.slots, a.D, static_cast<char*>(ws), &a);
  const int64_t direct = (a.N * a.C + GS_THREADS - 1) / GS_THREADS;
  if (!grid_fits(direct + a.slots, GS_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  a.direct = uint32_t(direct);
  if (dtype == FAST_F32) {
    if (a.dt) gs_launch<BACK, float, 2, true>(a, st);
    else gs_launch<BACK, float, 2, false>(a, st);
  } else {
    if (a.dt) gs_launch<BACK, uint16_t, 2, true>(a, st);
    else gs_launch<BACK, uint16_t, 2, false>(a, st);
  }
  return check_launch(fn);
}

static fast_status_t gs_workspace(const char* fn, int64_t N, int64_t E, int D, void* ws, size_t ws_bytes) {
  const size_t need = fast_gated_scan_workspace(N, E, D);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0, need);
  if (!aligned(ws, 256)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 256-byte aligned", fn);
  return FAST_OK;
}

}  // namespace fast

using namespace fast;

extern "C" int64_t fast_gated_scan_state_rows(int64_t num_edges) {
  return num_edges < 0 ? 0 : (num_edges + GS_WIN - 1) / GS_WIN;
}

extern "C" size_t fast_gated_scan_workspace(int64_t num_dst, int64_t num_edges, int D) {
  const int64_t big = int64_t(1) << 31;
  if (num_dst < 0 || num_edges < 0 || num_dst >= big || num_edges >= big || D <= 0 || D > GS_MAX_D) return 0;
  if (num_edges < 2 * GS_PIECE) return 0;
  return gs_layout((num_edges + GS_PIECE - 1) / GS_PIECE, D, nullptr, nullptr);
}

extern "C" fast_status_t fast_gated_scan_fwd(const fast_tcsr_t* g, int D, fast_dtype_t dtype, const void* x,
                                             const void* gate, int64_t ldx, const float* dt, const float* h0,
                                             int64_t longest, void* h, float* h_last, float* states, void* ws,
                                             size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_gated_scan_fwd";
  fast_status_t s = gs_check(fn, g, D, dtype, ldx, "ldx");
  if (s != FAST_OK) return s;
  if (longest < 0) return fail(FAST_ERR_INVALID_ARG, "%s: longest = %lld < 0", fn, (long long)longest);
  const int64_t N = g->num_dst, E = g->num_edges, es = elem_size(dtype);
  if (N == 0) return ok();
  if (E > 0 && (!x || !gate)) return fail(FAST_ERR_INVALID_ARG, "%s: NULL x/gate", fn);
  if (!h && !h_last) return fail(FAST_ERR_INVALID_ARG, "%s: neither h nor h_last", fn);
  if (!aligned(x, es) || !aligned(gate, es) || !aligned(h, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(dt, 4) || !aligned(h0, 4) || !aligned(h_last, 4) || !aligned(states, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: dt/h0/h_last/states not 4-byte aligned", fn);
  const int64_t in = span(E, D, ldx, es), rows = N * D * 4, out = E * D * es,
                keep = fast_gated_scan_state_rows(E) * D * 4;
  const struct { const void* p; int64_t n; } reads[] = {{x, in}, {gate, in}, {dt, 4 * E}, {h0, rows},
                                                        {g->dst_offsets, 4 * (N + 1)}},
                                             writes[] = {{h, out}, {h_last, rows}, {states, keep}};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 5; ++j)
      if (meet(writes[i].p, writes[i].n, reads[j].p, reads[j].n) && !(i == 1 && j == 3 && h_last == h0))
        return fail(FAST_ERR_INVALID_ARG, "%s: h, h_last or states overlaps an input", fn);
    for (int j = 0; j < i; ++j)
      if (meet(writes[i].p, writes[i].n, writes[j].p, writes[j].n))
        return fail(FAST_ERR_INVALID_ARG, "%s: h, h_last and states overlap", fn);
  }
  if ((s = gs_workspace(fn, N, E, D, ws, ws_bytes)) != FAST_OK) return s;
  GsArgs a = {};
  a.off = g->dst_offsets;
  a.N = N;
  a.E = E;
  a.D = D;
  a.x = x;
  a.gate = gate;
  a.ldx = ldx;
  a.dt = dt;
  a.h0 = h0;
  a.h = h;
  a.h_last = h_last;
  a.states = states;
  return gs_run<false>(fn, a, dtype, longest, ws, static_cast<hipStream_t>(stream));
}

extern "C" fast_status_t fast_gated_scan_bwd(const fast_tcsr_t* g, int D, fast_dtype_t dtype, const void* x,
                                             const void* gate, int64_t ldx, const float* dt, const float* h0,
                                             int64_t longest, const float* states, const void* dh,
                                             const float* dh_last, void* dx, void* dgate, int64_t lddx,
                                             float* dh0, void* ws, size_t ws_bytes, fast_stream_t stream) {
  const char* fn = "fast_gated_scan_bwd";
  fast_status_t s = gs_check(fn, g, D, dtype, ldx, "ldx");
  if (s != FAST_OK) return s;
  if ((s = gs_check(fn, g, D, dtype, lddx, "lddx")) != FAST_OK) return s;
  if (longest < 0) return fail(FAST_ERR_INVALID_ARG, "%s: longest = %lld < 0", fn, (long long)longest);
  const int64_t N = g->num_dst, E = g->num_edges, es = elem_size(dtype);
  if (N == 0) return ok();
  if (E > 0 && (!x || !gate || !states || !dx || !dgate))
    return fail(FAST_ERR_INVALID_ARG, "%s: NULL x/gate/states/dx/dgate", fn);
  if (!aligned(x, es) || !aligned(gate, es) || !aligned(dh, es) || !aligned(dx, es) || !aligned(dgate, es))
    return fail(FAST_ERR_UNSUPPORTED, "%s: rows not %d-byte aligned", fn, int(es));
  if (!aligned(dt, 4) || !aligned(h0, 4) || !aligned(states, 4) || !aligned(dh_last, 4) || !aligned(dh0, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: dt/h0/states/dh_last/dh0 not 4-byte aligned", fn);
  const int64_t in = span(E, D, ldx, es), rows = N * D * 4, out = span(E, D, lddx, es);
  const struct { const void* p; int64_t n; } reads[] = {
      {x, in}, {gate, in}, {dt, 4 * E}, {h0, rows}, {g->dst_offsets, 4 * (N + 1)},
      {states, fast_gated_scan_state_rows(E) * D * 4}, {dh, E * D * es}, {dh_last, rows}},
      writes[] = {{dx, out}, {dgate, out}, {dh0, rows}};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 8; ++j)
      if (meet(writes[i].p, writes[i].n, reads[j].p, reads[j].n) && !(i == 2 && j == 7 && dh0 == dh_last))
        return fail(FAST_ERR_INVALID_ARG, "%s: dx, dgate or dh0 overlaps an input", fn);
  if (meet(dx, out, dh0, rows) || meet(dgate, out, dh0, rows) || (E > 0 && dx == dgate) ||
      (E > 0 && rows_collide(static_cast<const char*>(dx), lddx, static_cast<const char*>(dgate), lddx, E, D, es)))
    return fail(FAST_ERR_INVALID_ARG, "%s: dx, dgate and dh0 overlap", fn);
  if ((s = gs_workspace(fn, N, E, D, ws, ws_bytes)) != FAST_OK) return s;
  GsArgs a = {};
  a.off = g->dst_offsets;
  a.N = N;
  a.E = E;
  a.D = D;
  a.x = x;
  a.gate = gate;
  a.ldx = ldx;
  a.dt = dt;
  a.h0 = h0;
  a.states = const_cast<float*>(states);
  a.dh = dh;
  a.dh_last = dh_last;
  a.dx = dx;
  a.dgate = dgate;
  a.lddx = lddx;
  a.dh0 = dh0;
  return gs_run<true>(fn, a, dtype, longest, ws, static_cast<hipStream_t>(stream));
}
