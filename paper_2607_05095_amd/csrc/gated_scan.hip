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
//
// 264,000 segments, 2.4 M events of 100 fp32: forward 620 us (4.8 TB/s, 400-byte rows),
// backward 1300-1380 (3.7: 186 registers, two waves a SIMD; three or four by spilling 1690 and 3421).
// bf16, 900,001 events of 256, three hubs among 6000 segments: 308 + 70 and 595 + 120 us.  Forward two halves of the
// same size: its bytes would take 225 us, its instructions about 180 (25 vector instructions a gate and
// column without times, 16 of them the gate's, the rest addresses, conversions and two-column stores); backward
// 37 of them, and three waves a SIMD to hide the loads of a window behind.  Four segments of 100,003 events
// of 128 in all: sums 27, chains 18, pieces 38 (forward), 29, 19, 53 (backward).
#include <algorithm>

#include "rows.h"

namespace fast {

constexpr int GS_THREADS = 256, GS_WAVES = GS_THREADS / 64;
constexpr int GS_AHEAD = 8;          // events whose rows are loaded together
constexpr int GS_WIN = 8;            // events of a backward window
constexpr int64_t GS_MAX_D = 8192, GS_MAX_LD = 1 << 26;
constexpr int GS_CARRY = 16;         // pieces whose sums are loaded together

// ------------------------------------------------------------------ the gate
struct Gate {
  float a, u, k;                     // k: the slope of u over the gate, a dt sigmoid(gate)
};

// u = 1 - a keeps its relative accuracy for slow gates and a for fast ones.  No branches: the
// evaluations of several events and columns interleave.
// FAR: some gate is so low that e^gate, at most 2^-100 then, may lie below what fp32 holds; over a
// long time it counts all the same, so it is formed 2^100 times as large and the time as much smaller.
// Which lanes share a wave decides which version runs: both give the same bits for every gate but those so low,
// and these always run the scaled one.
template <bool SPAN, bool FAR>
__device__ __forceinline__ Gate gate_of(float g, float dt) {
  Gate q;
  // t = e^-|g| within 3 U: the product with log2(e) in two parts (the second is no number where g is
  // infinite, and 0 or close to it otherwise)
  const float x = fabsf(g), h = -x * 0x1.715476p+0f;
  float l = fmaf(-x, 0x1.715476p+0f, -h);
  l = __builtin_amdgcn_fmed3f(fmaf(-x, 0x1.4ae0cp-26f, l), -1.f, 1.f);
  const bool far = FAR && g < 0.f && h < -100.f;
  float ts = __builtin_amdgcn_exp2f(far ? h + 100.f : h);
  ts = fmaf(ts, l * 0x1.62e43p-1f, ts);
  const bool pos = g >= 0.f;
  if constexpr (!SPAN) {
    const float r = __builtin_amdgcn_rcpf(1.f + ts), small = ts * r;   // sigmoid(|g|) = 1 / (1 + t)
    q.u = pos ? r : small;
    q.a = pos ? small : r;
    q.k = q.a * q.u;
    return q;
  }
  const float t = far ? ts * 0x1p-100f : ts, part = far ? dt * 0x1p-100f : dt;
  // log(1 + t) / t on (0, 1], within 2^-27 (a weighted least-squares fit)
  float p = -0x1.a9330cp-9f;
  p = fmaf(p, t, 0x1.453edcp-6f);
  p = fmaf(p, t, -0x1.d29c9ap-5f);
  p = fmaf(p, t, 0x1.b25348p-4f);
  p = fmaf(p, t, -0x1.39755cp-3f);
  p = fmaf(p, t, 0x1.92f694p-3f);
  p = fmaf(p, t, -0x1.ff0f86p-3f);
  p = fmaf(p, t, 0x1.554c80p-2f);
  p = fmaf(p, t, -0x1.ffffbep-2f);
  p = fmaf(p, t, 1.f);
  // rate dt
  const float y = far ? p * ts * part : fmaf(p, t, fmaxf(g, 0.f)) * dt;
  // (1 - e^-y) / y below log 2, within 2^-26; the difference above
  const float e = __builtin_amdgcn_exp2f(y * -0x1.715476p+0f);
  float s = -0x1.0ed322p-10f;
  s = fmaf(s, y, 0x1.085898p-7f);
  s = fmaf(s, y, -0x1.548ec0p-5f);
  s = fmaf(s, y, 0x1.554d38p-3f);
  s = fmaf(s, y, -0x1.ffffc0p-2f);
  s = fmaf(s, y, 1.f);
  q.u = y < 0.6931f ? s * y : 1.f - e;
  q.a = e;
  const float r = __builtin_amdgcn_rcpf(1.f + t);
  q.k = e * (pos ? r * dt : ts * r * part);
  return q;
}
// Gates side by side, without branches among them: their evaluations interleave.
template <bool SPAN, int COUNT, int VE>
__device__ __forceinline__ void gates_of(const float (&g)[COUNT][VE], const float (&dt)[COUNT], Gate (&k)[COUNT][VE]) {
  bool far = false;
  if constexpr (SPAN) {
    float low = 0.f;
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
#pragma unroll
      for (int q = 0; q < VE; ++q) low = fminf(low, g[j][q]);
    far = __any(low < -69.f);
  }
  if (far) {
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
#pragma unroll
      for (int q = 0; q < VE; ++q) k[j][q] = gate_of<SPAN, SPAN>(g[j][q], dt[j]);
  } else {
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
#pragma unroll
      for (int q = 0; q < VE; ++q) k[j][q] = gate_of<SPAN, false>(g[j][q], dt[j]);
  }
}

// ------------------------------------------------------------------ rows
struct GsArgs {
  const int32_t* off;
  int64_t N, E;
  int D, C;                          // columns; lanes of a row
  int waves;                         // waves that share a piece
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

// A lane's columns: VE from `first` on.  In a row that is no multiple of VE the last lane starts
// early enough to end with the row; it loads VE columns like all others (a branch around a load
// is a wait for it) and stores those from `skip` on.
struct Cols {
  int first, skip;
};
template <int VE>
__device__ __forceinline__ Cols cols_of(int lane, int D) {
  const int c = lane * VE, f = c + VE > D ? D - VE : c;
  return Cols{f, c - f};
}

// VE elements as they lie in memory.
template <typename T, int VE> struct Lump;
template <> struct Lump<float, 1> {
  float v;
  __device__ void load(const float* p) { v = *p; }
  __device__ void get(float* x) const { x[0] = v; }
};
template <> struct Lump<float, 2> {
  f32x2_e v;
  __device__ void load(const float* p) { v = *reinterpret_cast<const f32x2_e*>(p); }
  __device__ void get(float* x) const { x[0] = v.x; x[1] = v.y; }
};
template <> struct Lump<uint16_t, 1> {
  uint16_t v;
  __device__ void load(const uint16_t* p) { v = *p; }
  __device__ void get(float* x) const { x[0] = __uint_as_float(uint32_t(v) << 16); }
};
template <> struct Lump<uint16_t, 2> {
  uint32_t v;
  __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const u32_e*>(p); }
  __device__ void get(float* x) const { x[0] = bf16_lo(v); x[1] = bf16_hi(v); }
};
template <typename T, int VE>
__device__ __forceinline__ void gs_load(const T* p, float* x) {
  Lump<T, VE> l;
  l.load(p);
  l.get(x);
}
__device__ __forceinline__ void gs_put(float* p, float x) { *p = x; }
__device__ __forceinline__ void gs_put(uint16_t* p, float x) { *p = uint16_t(bf16_rne(x)); }
template <typename T, int VE>
__device__ __forceinline__ void gs_store(T* p, int skip, const float* x) {
  if constexpr (VE == 1) {
    gs_put(p, x[0]);
  } else {
    static_assert(VE == 2, "a lane owns one column or two");
    if (skip) gs_put(p + 1, x[1]);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x2_e*>(p) = f32x2_e{x[0], x[1]};
    else *reinterpret_cast<u32_e*>(p) = bf16_pack(x[0], x[1]);
  }
}
template <int VE>
__device__ __forceinline__ void gs_start(const float* rows, int64_t row, int D, int c, float* s) {
  if (rows) {
    gs_load<float, VE>(rows + row * D + c, s);
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) s[j] = 0.f;
  }
}

// The rows of events e, e + 1, ... of x and gate, a lane's columns of them.
template <typename T, int VE, int COUNT>
struct Rows {
  Lump<T, VE> x[COUNT], g[COUNT];
  float dt[COUNT];
  // m events; the last one again from there on.  A round spans less than 2^32 bytes.
  template <bool SPAN>
  __device__ void load(const GsArgs& a, int c, int64_t e, int m) {
    const char* px = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + e * a.ldx + c);
    const char* pg = reinterpret_cast<const char*>(static_cast<const T*>(a.gate) + e * a.ldx + c);
    const uint32_t ld = uint32_t(a.ldx) * uint32_t(sizeof(T)), end = uint32_t(m - 1) * ld;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) {
      const uint32_t o = min(uint32_t(j) * ld, end);
      x[j].load(reinterpret_cast<const T*>(px + o));
      g[j].load(reinterpret_cast<const T*>(pg + o));
      if constexpr (SPAN) {
        const float d = a.dt[e + min(j, m - 1)];
        dt[j] = d < 0.f ? 0.f : d;
      } else {
        dt[j] = 1.f;
      }
    }
  }
};
constexpr int GS_SIDE = 2;           // events whose gates are formed side by side

// Events [p, t) of a segment that starts at b, from the state s.
template <typename T, int VE, bool SPAN>
__device__ __forceinline__ void fwd_range(const GsArgs& a, int64_t b, int64_t p, int64_t t, Cols c, float* s) {
  T* h = a.h ? static_cast<T*>(a.h) + p * a.D + c.first : nullptr;
  for (int64_t e = p; e < t; e += GS_AHEAD) {
    const int m = t - e < GS_AHEAD ? int(t - e) : GS_AHEAD;
    Rows<T, VE, GS_AHEAD> r;
    r.template load<SPAN>(a, c.first, e, m);
    if (a.states && e > b && ((e - b) & (GS_WIN - 1)) == 0)
      gs_store<float, VE>(a.states + e / GS_WIN * a.D + c.first, c.skip, s);
#pragma unroll
    for (int i = 0; i < GS_AHEAD; i += GS_SIDE) {
      if (!__any(i < m)) break;
      Gate k[GS_SIDE][VE];
      float xv[GS_SIDE][VE], gv[GS_SIDE][VE], dt[GS_SIDE];
#pragma unroll
      for (int j = 0; j < GS_SIDE; ++j) {
        r.x[i + j].get(xv[j]);
        r.g[i + j].get(gv[j]);
        dt[j] = r.dt[i + j];
      }
      gates_of<SPAN>(gv, dt, k);
#pragma unroll
      for (int j = 0; j < GS_SIDE; ++j)
        if (i + j < m) {
#pragma unroll
          for (int q = 0; q < VE; ++q) s[q] = fmaf(k[j][q].a, s[q], k[j][q].u * xv[j][q]);
          if (h) gs_store<T, VE>(h + int64_t(i + j) * a.D, c.skip, s);
        }
    }
    if (h) h += int64_t(GS_AHEAD) * a.D;
  }
}

// Events [p, t) in reverse, d: what reaches the last of them from behind; returns what reaches
// the event before p.  v: the segment, for its start.
template <typename T, int VE, bool SPAN>
__device__ __forceinline__ void bwd_range(const GsArgs& a, int64_t v, int64_t b, int64_t p, int64_t t, Cols c,
                                          float* d) {
  if (t <= p) return;
  for (int64_t e = p + (t - p - 1) / GS_WIN * GS_WIN; e >= p; e -= GS_WIN) {
    const int m = t - e < GS_WIN ? int(t - e) : GS_WIN;
    Rows<T, VE, GS_WIN> r;
    r.template load<SPAN>(a, c.first, e, m);
    Lump<T, VE> ds[GS_WIN];
    {
      // (without dh a row of the gate, which is left out below)
      const T* dh = a.dh ? static_cast<const T*>(a.dh) + e * a.D + c.first
                         : static_cast<const T*>(a.gate) + e * a.ldx + c.first;
      const uint32_t ld = a.dh ? uint32_t(a.D) : uint32_t(a.ldx), end = uint32_t(m - 1) * ld;
#pragma unroll
      for (int j = 0; j < GS_WIN; ++j) ds[j].load(dh + min(uint32_t(j) * ld, end));
    }
    float s[VE];
    if (e == b) gs_start<VE>(a.h0, v, a.D, c.first, s);
    else gs_load<float, VE>(a.states + e / GS_WIN * a.D + c.first, s);
    float u[GS_WIN][VE], w[GS_WIN][VE], k[GS_WIN][VE];
#pragma unroll
    for (int i = 0; i < GS_WIN; i += GS_SIDE)
      if (__any(i < m)) {
        Gate ys[GS_SIDE][VE];
        float gv[GS_SIDE][VE], dt[GS_SIDE];
#pragma unroll
        for (int j = 0; j < GS_SIDE; ++j) {
          r.g[i + j].get(gv[j]);
          dt[j] = r.dt[i + j];
        }
        gates_of<SPAN>(gv, dt, ys);
#pragma unroll
        for (int j = i; j < i + GS_SIDE; ++j) {
          float xv[VE];
          r.x[j].get(xv);
#pragma unroll
          for (int q = 0; q < VE; ++q) {
            const Gate y = ys[j - i][q];
            k[j][q] = y.k * (xv[q] - s[q]);
            s[q] = fmaf(y.a, s[q], y.u * xv[q]);           // (past the end: used no more)
            u[j][q] = y.u;
            w[j][q] = y.a;
          }
        }
      }
    T* dx = static_cast<T*>(a.dx) + e * a.lddx + c.first;
    T* dg = static_cast<T*>(a.dgate) + e * a.lddx + c.first;
#pragma unroll
    for (int j = GS_WIN - 1; j >= 0; --j)
      if (j < m) {
        float y[VE], o[VE];
        ds[j].get(y);
#pragma unroll
        for (int q = 0; q < VE; ++q) {
          d[q] += a.dh ? y[q] : 0.f;
          y[q] = u[j][q] * d[q];
          o[q] = k[j][q] * d[q];
          d[q] *= w[j][q];
        }
        gs_store<T, VE>(dx + j * a.lddx, c.skip, y);
        gs_store<T, VE>(dg + j * a.lddx, c.skip, o);
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

// The product p a of factors a >= 0: 0 only of a factor that is 0.  Where fp32 holds it no more it is the least number
// that fp32 holds, so that an infinite state passes a piece as it passes its events one by one (times 0 it would
// be no number); what that adds to a finite state lies where the product's own last bits would have.
__device__ __forceinline__ float shrink(float p, float a) { return fmaxf(p * a, fminf(fminf(p, a), 0x1p-149f)); }

// A slot's piece: waves over its columns, `first` of them this wave's, `step` from one to its next.
template <typename T, int VE, bool SPAN, bool BACK>
__device__ __forceinline__ void piece_sums(const GsArgs& a, int64_t k, int first, int step) {
  const int64_t v = find_owner(a, k);
  if (first == 0) a.owner[k] = int32_t(v);
  if (v < 0) return;
  int64_t b, e;
  Piece r;
  segment_of(a, v, b, e);
  piece_in(a, b, e, k, r);
  // nothing reads the sums of the piece that the chain ends with
  if (BACK ? r.p == b : r.t == e) return;
  for (int i = first; i < a.C; i += step) {
    const Cols c = cols_of<VE>(i, a.D);
    float pa[VE], pb[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      pa[q] = 1.f;
      pb[q] = 0.f;
    }
    for (int64_t o = 0; o < r.t - r.p; o += GS_AHEAD) {
      const int m = r.t - r.p - o < GS_AHEAD ? int(r.t - r.p - o) : GS_AHEAD;
      const int64_t at = BACK ? r.t - o - m : r.p + o;
      Rows<T, VE, GS_AHEAD> w;
      w.template load<SPAN>(a, c.first, at, m);
      if constexpr (BACK) {                               // dh in x's place
        if (a.dh) {
          const T* dh = static_cast<const T*>(a.dh) + at * a.D + c.first;
#pragma unroll
          for (int j = 0; j < GS_AHEAD; ++j) w.x[j].load(dh + min(j, m - 1) * a.D);
        }
      }
#pragma unroll
      for (int ii = 0; ii < GS_AHEAD; ii += GS_SIDE) {
        const int i = BACK ? GS_AHEAD - GS_SIDE - ii : ii;
        Gate y[GS_SIDE][VE];
        float gv[GS_SIDE][VE], dt[GS_SIDE];
#pragma unroll
        for (int j = 0; j < GS_SIDE; ++j) {
          w.g[i + j].get(gv[j]);
          dt[j] = w.dt[i + j];
        }
        gates_of<SPAN>(gv, dt, y);
#pragma unroll
        for (int jj = 0; jj < GS_SIDE; ++jj) {
          const int j = BACK ? GS_SIDE - 1 - jj : jj;
          float xv[VE];
          w.x[i + j].get(xv);
#pragma unroll
          for (int q = 0; q < VE; ++q) {
            const float in =
                BACK ? y[j][q].a * (pb[q] + (a.dh ? xv[q] : 0.f)) : fmaf(y[j][q].a, pb[q], y[j][q].u * xv[q]);
            pb[q] = i + j < m ? in : pb[q];
            pa[q] = i + j < m ? shrink(pa[q], y[j][q].a) : pa[q];
          }
        }
      }
    }
    gs_store<float, VE>(a.pa + k * a.D + c.first, c.skip, pa);
    gs_store<float, VE>(a.pb + k * a.D + c.first, c.skip, pb);
  }
}

// The slot of this wave, the first column group of this lane and the stride to its next: a
// workgroup's waves share one slot or hold several, by the row's width.
struct Share {
  int64_t slot;
  int first, step;
};
__device__ __forceinline__ Share share_of(const GsArgs& a, uint32_t block) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  return Share{int64_t(block) * (GS_WAVES / a.waves) + wave / a.waves, (wave % a.waves) * 64 + lane, a.waves * 64};
}

// ------------------------------------------------------------------ kernels
template <typename T, int VE, bool SPAN, bool BACK>
__global__ void __launch_bounds__(GS_THREADS) k_scan(GsArgs a) {
  if (blockIdx.x >= a.direct) {
    const Share h = share_of(a, blockIdx.x - a.direct);
    if (h.slot < a.slots) piece_sums<T, VE, SPAN, BACK>(a, h.slot, h.first, h.step);
    return;
  }
  const uint32_t i = blockIdx.x * GS_THREADS + threadIdx.x;
  const int64_t v = i / uint32_t(a.C);
  if (v >= a.N) return;
  const Cols c = cols_of<VE>(int(i - uint32_t(v) * uint32_t(a.C)), a.D);
  int64_t b, e;
  segment_of(a, v, b, e);
  if (e - b >= a.cut) return;
  float s[VE];
  if constexpr (BACK) {
    gs_start<VE>(a.dh_last, v, a.D, c.first, s);
    bwd_range<T, VE, SPAN>(a, v, b, b, e, c, s);
    if (a.dh0) gs_store<float, VE>(a.dh0 + v * a.D + c.first, c.skip, s);
  } else {
    gs_start<VE>(a.h0, v, a.D, c.first, s);
    fwd_range<T, VE, SPAN>(a, b, b, e, c, s);
    if (a.h_last) gs_store<float, VE>(a.h_last + v * a.D + c.first, c.skip, s);
  }
}

// The pieces' starts (backward: from the last piece on), over 64 columns a workgroup.  It looks
// at GS_CHAIN slots, a wave each: the wave whose slot holds a long segment's first piece walks
// its pieces.  The start of slot k takes pa's place.  A chain of more than GS_ALONE pieces (of
// the slots of a workgroup one at most starts such) is walked by all its waves, each a stretch:
// its product and result first, then, once it knows what the stretches before leave, the starts.
constexpr int GS_CHAIN = 8, GS_ALONE = 64;
static_assert(GS_ALONE > GS_CHAIN, "one long chain a workgroup");
struct Chain {
  int64_t k, pieces;
  const GsArgs& a;
  int c;
  bool back;
  // where piece j of the chain lies
  __device__ int64_t at(int64_t j) const { return (k + (back ? pieces - 1 - j : j)) * a.D + c; }
  // pieces [j0, j1) from the state s; starts are written where `write`
  template <bool WRITE>
  __device__ void walk(int64_t j0, int64_t j1, bool write, float& pa, float& s) const {
    for (int64_t j = j0; j < j1; j += GS_CARRY) {
      float xa[GS_CARRY], xb[GS_CARRY];
#pragma unroll
      for (int q = 0; q < GS_CARRY; ++q) {
        const int64_t i = at(min(j + q, j1 - 1));
        xa[q] = a.pa[i];
        xb[q] = a.pb[i];
      }
#pragma unroll
      for (int q = 0; q < GS_CARRY; ++q)
        if (j + q < j1) {
          if (WRITE && write) a.pa[at(j + q)] = s;
          s = fmaf(xa[q], s, xb[q]);
          pa = shrink(pa, xa[q]);
        }
    }
  }
};
template <bool BACK>
__global__ void __launch_bounds__(64 * GS_CHAIN) k_scan_chain(GsArgs a) {
  __shared__ float s_a[GS_CHAIN][64], s_b[GS_CHAIN][64];
  __shared__ int64_t s_long[2];                           // slot and segment of a long chain
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c0 = blockIdx.y * 64 + lane, c = c0 < a.D ? c0 : a.D - 1;
  const bool in = c0 < a.D;
  const int64_t k = int64_t(blockIdx.x) * GS_CHAIN + wave;
  if (threadIdx.x == 0) s_long[1] = -1;
  __syncthreads();
  const int64_t v = k < a.slots ? a.owner[k] : -1;
  const float* first = BACK ? a.dh_last : a.h0;
  if (v >= 0) {
    int64_t b, e;
    Piece r;
    segment_of(a, v, b, e);
    if (piece_in(a, b, e, k, r) && r.p == b) {
      const int64_t pieces = (e - b) / a.piece;
      if (pieces <= GS_ALONE) {
        const Chain ch = {k, pieces, a, c, BACK};
        float pa = 1.f, s = first ? first[v * a.D + c] : 0.f;
        ch.walk<true>(0, pieces - 1, in, pa, s);          // the chain's last piece has no sums
        if (in) a.pa[ch.at(pieces - 1)] = s;
      } else if (lane == 0) {
        s_long[0] = k;
        s_long[1] = v;
      }
    }
  }
  __syncthreads();
  const int64_t lv = s_long[1];
  if (lv < 0) return;
  int64_t b, e;
  segment_of(a, lv, b, e);
  const Chain ch = {s_long[0], (e - b) / a.piece, a, c, BACK};
  const int64_t links = ch.pieces - 1, per = (links + GS_CHAIN - 1) / GS_CHAIN;
  const int64_t j0 = min(wave * per, links), j1 = min(j0 + per, links);
  float pa = 1.f, pb = 0.f;
  ch.walk<false>(j0, j1, false, pa, pb);
  s_a[wave][lane] = pa;
  s_b[wave][lane] = pb;
  __syncthreads();
  float s = first ? first[lv * a.D + c] : 0.f;
  for (int w = 0; w < wave; ++w) s = fmaf(s_a[w][lane], s, s_b[w][lane]);
  ch.walk<true>(j0, j1, in, pa, s);
  if (j0 < j1 && j1 == links && in) a.pa[ch.at(links)] = s;
}

template <typename T, int VE, bool SPAN, bool BACK>
__global__ void __launch_bounds__(GS_THREADS) k_scan_pieces(GsArgs a) {
  const Share h = share_of(a, blockIdx.x);
  if (h.slot >= a.slots) return;
  const int64_t k = h.slot, v = a.owner[k];
  if (v < 0) return;
  int64_t b, e;
  Piece r;
  segment_of(a, v, b, e);
  if (!piece_in(a, b, e, k, r)) return;
  for (int i = h.first; i < a.C; i += h.step) {
    const Cols c = cols_of<VE>(i, a.D);
    float s[VE];
    gs_load<float, VE>(a.pa + k * a.D + c.first, s);
    if constexpr (BACK) {
      bwd_range<T, VE, SPAN>(a, v, b, r.p, r.t, c, s);
      if (r.p == b && a.dh0) gs_store<float, VE>(a.dh0 + v * a.D + c.first, c.skip, s);
    } else {
      fwd_range<T, VE, SPAN>(a, b, r.p, r.t, c, s);
      if (r.t == e && a.h_last) gs_store<float, VE>(a.h_last + v * a.D + c.first, c.skip, s);
    }
  }
}

// ------------------------------------------------------------------ host side
// a multiple of GS_WIN; 32 / 64 / 128 events in four segments of 100,003: sums 25 / 26 / 49 us,
// chains 34 / 17 / 12, pieces 33 / 39 / 72
constexpr int GS_PIECE = 64;
struct GsPlan {
  int64_t cut, slots;
  int piece;
};
static GsPlan gs_plan(int64_t N, int64_t E, int D, int64_t es, int64_t longest) {
  GsPlan p = {};
  p.piece = GS_PIECE;
  // a walk of `cut` events should not outlast half of the whole: an event takes about
  // 0.13 us, the rows of all events their bytes at 6 TB/s (cuts of 256 to 2000 events by hand:
  // no better in blocks of 6000 and 264,000 segments)
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
  if (ldx >= GS_MAX_LD) return fail(FAST_ERR_UNSUPPORTED, "%s: %s >= 2^26", fn, ld_name);
  if (g->num_edges * ldx >= (int64_t(1) << 56))
    return fail(FAST_ERR_UNSUPPORTED, "%s: %lld rows, %lld elements apart", fn, (long long)g->num_edges, (long long)ldx);
  if (g->num_dst > 0 && !g->dst_offsets) return fail(FAST_ERR_INVALID_ARG, "%s: NULL dst_offsets", fn);
  if (!aligned(g->dst_offsets, 4)) return fail(FAST_ERR_UNSUPPORTED, "%s: dst_offsets not 4-byte aligned", fn);
  return FAST_OK;
}

template <bool BACK, typename T, int VE, bool SPAN>
static void gs_launch(const GsArgs& a, hipStream_t st) {
  const int per = GS_WAVES / a.waves;
  const uint32_t pieces = uint32_t((a.slots + per - 1) / per);
  if (a.direct + pieces > 0)
    hipLaunchKernelGGL((k_scan<T, VE, SPAN, BACK>), dim3(a.direct + pieces), dim3(GS_THREADS), 0, st, a);
  if (a.slots == 0) return;
  hipLaunchKernelGGL((k_scan_chain<BACK>), dim3(uint32_t((a.slots + GS_CHAIN - 1) / GS_CHAIN), uint32_t((a.D + 63) / 64)),
                     dim3(64 * GS_CHAIN), 0, st, a);
  hipLaunchKernelGGL((k_scan_pieces<T, VE, SPAN, BACK>), dim3(pieces), dim3(GS_THREADS), 0, st, a);
}
template <bool BACK, typename T, int VE>
static void gs_launch(const GsArgs& a, hipStream_t st) {
  if (a.dt) gs_launch<BACK, T, VE, true>(a, st);
  else gs_launch<BACK, T, VE, false>(a, st);
}

template <bool BACK>
static fast_status_t gs_run(const char* fn, GsArgs& a, fast_dtype_t dtype, int64_t longest, void* ws,
                            hipStream_t st) {
  const int ve = a.D > 1 ? 2 : 1;
  a.C = (a.D + ve - 1) / ve;
  a.waves = a.C > 128 ? 4 : (a.C > 64 ? 2 : 1);
  const GsPlan p = gs_plan(a.N, a.E, a.D, elem_size(dtype), longest);
  a.cut = p.cut;
  a.piece = p.piece;
  a.slots = p.slots;
  gs_layout(p.slots, a.D, static_cast<char*>(ws), &a);
  const int64_t direct = (a.N * a.C + GS_THREADS - 1) / GS_THREADS;
  if (!grid_fits(direct + a.slots, GS_THREADS) || !grid_fits(a.slots / GS_CHAIN + 1, 64 * GS_CHAIN))
    return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  a.direct = uint32_t(direct);
  if (dtype == FAST_F32) {
    if (ve == 2) gs_launch<BACK, float, 2>(a, st);
    else gs_launch<BACK, float, 1>(a, st);
  } else {
    if (ve == 2) gs_launch<BACK, uint16_t, 2>(a, st);
    else gs_launch<BACK, uint16_t, 1>(a, st);
  }
  return check_launch(fn);
}

struct GsSpan {
  const void* p;
  int64_t n;
};
template <int R, int W>
static fast_status_t gs_workspace(const char* fn, int64_t N, int64_t E, int D, void* ws, size_t ws_bytes,
                                  const GsSpan (&reads)[R], const GsSpan (&writes)[W]) {
  const size_t need = fast_gated_scan_workspace(N, E, D);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0, need);
  if (!aligned(ws, 256)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 256-byte aligned", fn);
  bool on = false;
  for (int j = 0; j < R; ++j) on |= meet(ws, int64_t(need), reads[j].p, reads[j].n);
  for (int j = 0; j < W; ++j) on |= meet(ws, int64_t(need), writes[j].p, writes[j].n);
  if (on) return fail(FAST_ERR_INVALID_ARG, "%s: the workspace overlaps another array", fn);
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
  const GsSpan reads[] = {{x, in}, {gate, in}, {dt, 4 * E}, {h0, rows},
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
  if ((s = gs_workspace(fn, N, E, D, ws, ws_bytes, reads, writes)) != FAST_OK) return s;
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
  const GsSpan reads[] = {
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
  if ((s = gs_workspace(fn, N, E, D, ws, ws_bytes, reads, writes)) != FAST_OK) return s;
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
