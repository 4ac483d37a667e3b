// attention_cached.hip -- edge softmax + aggregation fused (Sec. 4.3), K|V rows
// read from a cache in 8 or 4 bits through ids and a slot map.
//   t[e,h] = LReLU(scale <Q[v,h], K[slot e,h]>),  out[v,h] = sum softmax(t)[e,h] V[slot e,h]
// over the segment's edges that have a slot; lse = log sum exp t.
//
// Bound by HBM: per edge an id, a slot and a record of about H*dh*(2 or 1) bytes
// at a random place, against two fused multiply-adds per element.  L lanes
// hold a record's heads, 16 (or 8) codes of K and of V each; CA_ROWS records per lane
// are in flight.  A running maximum, sum and accumulators in base 2 make one pass.
// 264,000 segments of 2.4 M edges, 8 bits, 2 x 50 fp32: 153 us for the first launch, 6.9 TB/s of the
// lines it touches (a record of a 272 MB cache two, a slot of an 8 MB map one), 162 with the other
// two; 226 on a cache of 4.3 GB with a map of 800 MB, 176 without a map.
//
// Where there are many short segments, L lanes own one and walk its edges: no
// joins.  Where segments are longer, or too few to fill the chip that way, a wave
// owns one, its 64 / L groups of lanes take the edges in turn, and their
// results are joined by lane exchanges at the end; where they are longer and
// fewer still, a workgroup's 4 waves share one and join in LDS.
//
// Segments longer than `cap` edges (a power of two) are left to a second launch, which
// cuts them at the multiples of cap in the block's edge order.  Every multiple belongs
// to one segment, whose lanes note in the first launch whether it is a long one.  A
// workgroup of the second launch takes the piece between two multiples of the long
// segment that comes in from the left, then of the one that goes out to the
// right: its waves split the piece, join in LDS and write (maximum, sum,
// accumulators) to the workspace.  A third launch joins a segment's pieces in their
// order.  (Joining in the workgroup that finishes a segment's last piece needs an
// agent-wide fence per piece, which writes the L2 back: 72 us against 20 for
// four histories of 100,003 edges.  Looking for the long segments with a search of the
// offsets, in the first launch, cost 30 us of 190 in registers and waves for a
// block of 264,000 short segments.)
#include <algorithm>

#include "attention.h"
#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int CA_THREADS = 256, CA_WAVES = CA_THREADS / 64;
constexpr int CA_ROWS = 4;           // records in flight per lane
constexpr int CA_AHEAD = 2;          // places that a lane looks up at once
constexpr int CA_SHIFT = 6, CA_SHIFT_MAX = 11;   // cap = 64 .. 2048 (4096: see ca_plan)
constexpr int CA_BLOCKS = 2048;      // segments that get a workgroup each, at most: 8 per CU
constexpr int CA_CELLS = 1024;       // workgroups of the second launch, at most: 4 per CU (a power of two)

constexpr int64_t CA_LANES_N = 4096; // segments above which a few lanes may own one
constexpr int64_t CA_SHORT_E = 8191, CA_MEDIUM_E = 131071;   // edges up to which cap is 64 and 128 there

struct CaArgs {
  int64_t N, E;
  const int32_t* off;
  int H, dh;
  int lph, L;                        // lanes per head, per record (powers of two up to 64)
  int shift;                         // cap = 1 << shift
  int64_t cells;                     // cells between multiples of cap, 0 where no segment can be long
  int64_t rounds;                    // cells per workgroup of the other launches: b, b + CA_CELLS, ...
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
  float* part;                       // [2 per cell][H][dh + 2]
  int32_t* mark;                     // at ca_mark_at(m): the long segment that holds edge m cap, or -1
};

__device__ __forceinline__ void ca_segment(const CaArgs& a, int64_t v, int64_t& s, int64_t& t) {
  s = clamp64(a.off[v], 0, a.E);
  t = clamp64(a.off[v + 1], s, a.E);
}

__device__ __forceinline__ float ca_pow2(float x, float m) {   // 2^(x - m), 0 for x = -inf
  return __builtin_amdgcn_exp2f(x - (m == -INFINITY ? 0.f : m));
}

// A lane's place: head h, its codes [first, first + VE) of which those from `own` on
// are its own (the last piece of a head of 8 (2 k + 1) codes starts 8 earlier
// and shares them with its neighbour); the running softmax.  Its scale is that of its own
// codes; where the 8 others are of the group before, they may not be finite under it,
// and their products with q = 0 are dropped (`keep`).
template <int VE>
struct CaLane {
  int h, l, first, own;
  bool mine;                         // the lane holds codes
  uint32_t code, scale;              // its K codes and their scale within a record
  uint32_t keep;                     // 0 where the first 8 codes are of another group, else all bits
  float q[VE], mx, Z, acc[VE];
};

// lanes per head: known to the compiler, or (LPH = 0) read from the arguments; negative where a
// last piece may begin in another group than its own codes (heads of 1 to 8 elements past
// a multiple of 32): their test in the others took 3 to 5 per cent
template <int LPH>
__device__ __forceinline__ int ca_lph(const CaArgs& a) { return LPH > 0 ? LPH : LPH < 0 ? -LPH : a.lph; }

template <typename T, int FMT, int VE, int LPH>
__device__ __forceinline__ void ca_init(const CaArgs& a, int64_t v, CaLane<VE>& c) {
  const int lane = threadIdx.x & 63, lph = ca_lph<LPH>(a);
  c.h = blockIdx.y * (a.L / lph) + (lane & (a.L - 1)) / lph;
  c.l = lane & (lph - 1);
  c.mine = c.h < a.H && c.l * VE < a.dh;
  const int last = (a.dh + MX_PIECE - 1) / MX_PIECE * MX_PIECE - VE;   // >= 0 for the VE in use
  c.own = c.l * VE;
  c.first = c.own < last ? c.own : last;
  const T* q = static_cast<const T*>(a.Q) + (v * a.H + c.h) * a.dh + c.first;
#pragma unroll
  for (int j = 0; j < VE; j += CHUNK<T>)
    load_chunk(q + j, c.mine && c.first + j >= c.own ? a.dh - c.first - j : 0, c.q + j);
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    c.q[j] *= a.scale * LOG2E;
    c.acc[j] = 0.f;
  }
  c.mx = -INFINITY;
  c.Z = 0.f;
  c.code = uint32_t(c.h * a.rec.code_bytes + (FMT == FAST_MXFP4 ? c.first / 2 : c.first));
  c.scale = uint32_t(a.rec.scale_off + c.h * a.rec.groups + c.own / MX_GROUP);
  c.keep = c.first / MX_GROUP == c.own / MX_GROUP ? ~0u : 0u;
}

// No record.
constexpr uint32_t CA_NONE = 0xffffffffu;

// The codes in flight.  They are zeroed once, for the lanes that hold none; a record
// that is not there leaves its place as it was, and nothing uses it.
template <int FMT, int VE>
struct CaCodes {
  MxPiece<FMT, VE> k[CA_ROWS], v[CA_ROWS];
  uint32_t ks[CA_ROWS], vs[CA_ROWS];
  __device__ void zero() {
#pragma unroll
    for (int i = 0; i < CA_ROWS; ++i) {
      k[i].zero();
      v[i].zero();
      ks[i] = vs[i] = 127u;
    }
  }
};

// CA_ROWS records at rec[] (CA_NONE: none) folded into the running softmax.
// rec[] is the record's byte in a cache of less than 4 GiB, so that an address is a
// base that all lanes share plus 32 bits, or (BIG) its slot.
template <int FMT, int VE, int LPH, bool BIG>
__device__ __forceinline__ void ca_fold(const CaArgs& a, const uint32_t (&rec)[CA_ROWS], CaLane<VE>& c,
                                        CaCodes<FMT, VE>& r) {
  const uint8_t* kbase = a.cache;
  const uint8_t* vbase = a.cache + a.H * a.rec.code_bytes;
  const uint8_t* sbase = a.cache + a.H * a.rec.groups;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    if (rec[i] != CA_NONE && c.mine) {
      if constexpr (BIG) {
        const uint64_t o = uint64_t(rec[i]) * uint32_t(a.rec.stride);
        r.k[i].load(kbase + (o + c.code));
        r.v[i].load(vbase + (o + c.code));
        r.ks[i] = kbase[o + c.scale];
        r.vs[i] = sbase[o + c.scale];
      } else {
        const uint32_t o = rec[i] + c.code, s = rec[i] + c.scale;
        r.k[i].load(kbase + o);
        r.v[i].load(vbase + o);
        r.ks[i] = kbase[s];
        r.vs[i] = sbase[s];
      }
    }
  }
  float t[CA_ROWS], mn = c.mx;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    t[i] = -INFINITY;
    if (rec[i] != CA_NONE) {           // all lanes of a record alike
      float k[VE], d = 0.f;
      r.k[i].unpack(mx_scale(r.ks[i]), k);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        if (VE == 16 && LPH <= 0 && j == MX_PIECE) d = __uint_as_float(__float_as_uint(d) & c.keep);
        d = fmaf(c.q[j], k[j], d);
      }
      if constexpr (LPH != 0) d = group_sum_ct<(LPH > 0 ? LPH : -LPH)>(d);
      else d = group_sum(d, a.lph);
      t[i] = d * (d > 0.f ? 1.f : a.slope);
    }
    mn = fmaxf(mn, t[i]);
  }
  const float corr = ca_pow2(c.mx, mn), ref = mn == -INFINITY ? 0.f : mn;
  c.mx = mn;
  c.Z *= corr;
#pragma unroll
  for (int j = 0; j < VE; ++j) c.acc[j] *= corr;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    if (rec[i] != CA_NONE) {
      const float w = __builtin_amdgcn_exp2f(t[i] - ref);
      float x[VE];
      r.v[i].unpack(mx_scale(r.vs[i]), x);
      c.Z += w;
#pragma unroll
      for (int j = 0; j < VE; ++j) c.acc[j] = fmaf(w, x[j], c.acc[j]);
    }
  }
}

// Where edge e's record is, as ca_fold takes it.
template <bool BIG>
__device__ __forceinline__ uint32_t ca_rec(const CaArgs& a, int64_t e, int64_t e1) {
  if (e >= e1) return CA_NONE;
  const int64_t s = mx_slot(a.ids[e], a.id_bound, a.slot_map, a.cache_rows);
  if (s < 0) return CA_NONE;
  return BIG ? uint32_t(s) : uint32_t(s) * uint32_t(a.rec.stride);
}

// Edges [e0, e1) by the whole wave: 64 records' places at a time, one per lane, then the
// groups of lanes take every (64 / L)-th of them; the groups joined at the end.
template <int FMT, int VE, int LPH, bool BIG>
__device__ __forceinline__ void ca_wave(const CaArgs& a, int64_t e0, int64_t e1, CaLane<VE>& c) {
  const int lane = threadIdx.x & 63, L = a.L, GR = 64 / L, gi = lane / L;
  CaCodes<FMT, VE> codes;
  codes.zero();
  for (int64_t base = e0; base < e1; base += 64) {
    const uint32_t my = ca_rec<BIG>(a, base + lane, e1);
    const int n = int(e1 - base < 64 ? e1 - base : 64);
    for (int r0 = 0; r0 < n; r0 += GR * CA_ROWS) {
      uint32_t rec[CA_ROWS];
#pragma unroll
      for (int i = 0; i < CA_ROWS; ++i) {
        const int r = r0 + i * GR + gi;
        const uint32_t o = __shfl(my, r & 63);
        rec[i] = r < 64 ? o : CA_NONE;
      }
      ca_fold<FMT, VE, LPH, BIG>(a, rec, c, codes);
    }
  }
  for (int o = L; o < 64; o *= 2) {
    const float om = __shfl_xor(c.mx, o), oz = __shfl_xor(c.Z, o);
    const float mn = fmaxf(c.mx, om);
    const float c0 = ca_pow2(c.mx, mn), c1 = ca_pow2(om, mn);
    c.Z = c.Z * c0 + oz * c1;
#pragma unroll
    for (int j = 0; j < VE; ++j) c.acc[j] = c.acc[j] * c0 + __shfl_xor(c.acc[j], o) * c1;
    c.mx = mn;
  }
}

template <typename T, int VE>
__device__ __forceinline__ void ca_store(const CaArgs& a, int64_t v, CaLane<VE>& c) {
  if (!c.mine) return;
  const bool some = !(c.Z == 0.f);     // also of a NaN
  const float inv = some ? 1.f / c.Z : 0.f;
#pragma unroll
  for (int j = 0; j < VE; ++j) c.acc[j] = some ? c.acc[j] * inv : 0.f;
  T* out = static_cast<T*>(a.out) + (v * a.H + c.h) * a.dh + c.first;
#pragma unroll
  for (int j = 0; j < VE; j += CHUNK<T>)
    if (c.first + j >= c.own) store_chunk(out + j, a.dh - c.first - j, c.acc + j);
  if (a.lse && c.l == 0) a.lse[v * a.H + c.h] = some ? (c.mx + log2f(c.Z)) * LN2 : -INFINITY;
}

// Edges [e0, e1) of segment v by a workgroup, into partial result `slot` (-1: they are the segment).
// The waves' results meet in LDS, where a thread per element adds its weighted
// accumulators: 4 segments, 100,003 edges in all, H 4, dh 32, 15.3 us with one result
// per wave, 18.0 with one per group of lanes, which spares the lane exchanges.
constexpr int CA_PAD = 65;             // odd: a column of LDS in as many banks
template <typename T, int FMT, int VE, int LPH, bool BIG>
__device__ __forceinline__ void ca_piece(const CaArgs& a, int64_t v, int64_t e0, int64_t e1, int64_t slot,
                                         float (*s_acc)[VE + 2][CA_PAD]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, L = a.L;
  CaLane<VE> c;
  ca_init<T, FMT, VE, LPH>(a, v, c);
  const int64_t each = (e1 - e0 + CA_WAVES - 1) / CA_WAVES;
  const int64_t w0 = e0 + wave * each, w1 = w0 + each < e1 ? w0 + each : e1;
  ca_wave<FMT, VE, LPH, BIG>(a, w0, w1, c);
  s_acc[wave][VE][lane] = c.mx;
  s_acc[wave][VE + 1][lane] = c.Z;
#pragma unroll
  for (int j = 0; j < VE; ++j) s_acc[wave][j][lane] = c.acc[j];
  __syncthreads();
  const int lph = ca_lph<LPH>(a), last = (a.dh + MX_PIECE - 1) / MX_PIECE * MX_PIECE - VE;
  for (int t = threadIdx.x; t < VE * L; t += CA_THREADS) {
    const int j = t % VE, p = t / VE;          // element j of lane p
    const int h = blockIdx.y * (L / lph) + p / lph, own = (p & (lph - 1)) * VE;
    const int e = (own < last ? own : last) + j;
    if (h >= a.H || e < own || e >= a.dh) continue;
    float mx = -INFINITY, Z = 0.f, acc = 0.f;
    for (int w = 0; w < CA_WAVES; ++w) mx = fmaxf(mx, s_acc[w][VE][p]);
    for (int w = 0; w < CA_WAVES; ++w) {
      const float k = ca_pow2(s_acc[w][VE][p], mx);
      Z = fmaf(s_acc[w][VE + 1][p], k, Z);
      acc = fmaf(s_acc[w][j][p], k, acc);
    }
    if (slot < 0) {
      const bool some = !(Z == 0.f);           // also of a NaN
      const float o = some ? acc / Z : 0.f;
      VecIO<T, 1>::store(static_cast<T*>(a.out) + (v * a.H + h) * a.dh + e, &o);
      if (a.lse && e == 0) a.lse[v * a.H + h] = some ? (mx + log2f(Z)) * LN2 : -INFINITY;
    } else {
      float* q = a.part + (slot * a.H + h) * (a.dh + 2);
      if (e == 0) {
        q[0] = mx;
        q[1] = Z;
      }
      q[2 + e] = acc;
    }
  }
  __syncthreads();                     // before the next piece of this workgroup
}

// Where the mark of cell m is: the cells of a workgroup lie side by side.
__device__ __forceinline__ int64_t ca_mark_at(const CaArgs& a, int64_t m) {
  return (m & (CA_CELLS - 1)) * a.rounds + m / CA_CELLS;
}

// What the other launches read: for every multiple of cap inside segment v, whether
// it is long.  The `n` lanes of the segment share the work.
__device__ __forceinline__ void ca_mark(const CaArgs& a, int64_t v, int64_t s, int64_t t, int lane, int n) {
  if (s == t || blockIdx.y != 0) return;
  const int64_t cap = int64_t(1) << a.shift;
  const int64_t first = (s + cap - 1) >> a.shift, last = (t - 1) >> a.shift;
  for (int64_t m = first + lane; m <= last; m += n) a.mark[ca_mark_at(a, m)] = t - s > cap ? int32_t(v) : -1;
}

// Who owns a segment: L lanes, a wave, or a workgroup.
enum CaOwner { CA_GROUP, CA_WAVE, CA_BLOCK };
template <typename T, int FMT, int VE, int LPH, bool BIG, CaOwner OWNER>
__global__ void __launch_bounds__(CA_THREADS) k_attn_cached(CaArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t cap = int64_t(1) << a.shift;
  CaLane<VE> c;
  int64_t s, t;
  if constexpr (OWNER == CA_BLOCK) {
    __shared__ float s_acc[CA_WAVES][VE + 2][CA_PAD];
    const int64_t v = blockIdx.x;
    ca_segment(a, v, s, t);
    if (a.cells > 0) ca_mark(a, v, s, t, threadIdx.x, CA_THREADS);
    if (t - s > cap) return;           // in pieces
    ca_piece<T, FMT, VE, LPH, BIG>(a, v, s, t, -1, s_acc);
  } else if constexpr (OWNER == CA_WAVE) {
    const int64_t v = int64_t(blockIdx.x) * CA_WAVES + wave;
    if (v >= a.N) return;
    ca_segment(a, v, s, t);
    if (a.cells > 0) ca_mark(a, v, s, t, lane, 64);
    if (t - s > cap) return;
    ca_init<T, FMT, VE, LPH>(a, v, c);
    ca_wave<FMT, VE, LPH, BIG>(a, s, t, c);
    if (lane < a.L) ca_store<T, VE>(a, v, c);
  } else {
    const int L = a.L, gl = lane & (L - 1), g0 = lane - gl;
    const int64_t v = int64_t(blockIdx.x) * (CA_THREADS / L) + threadIdx.x / L;
    if (v >= a.N) return;
    ca_segment(a, v, s, t);
    if (a.cells > 0) ca_mark(a, v, s, t, gl, L);
    if (t - s > cap) return;
    ca_init<T, FMT, VE, LPH>(a, v, c);
    CaCodes<FMT, VE> codes;
    codes.zero();
    for (int64_t base = s; base < t; base += CA_AHEAD * L) {   // CA_AHEAD places per lane at a time
      uint32_t my[CA_AHEAD];
#pragma unroll
      for (int k = 0; k < CA_AHEAD; ++k) my[k] = ca_rec<BIG>(a, base + k * L + gl, t);
#pragma unroll
      for (int k = 0; k < CA_AHEAD; ++k) {
        const int n = int(t - base - k * L < L ? t - base - k * L : L);
        for (int r0 = 0; r0 < n; r0 += CA_ROWS) {
          uint32_t rec[CA_ROWS];
#pragma unroll
          for (int i = 0; i < CA_ROWS; ++i) {
            const uint32_t o = __shfl(my[k], g0 + ((r0 + i) & (L - 1)));
            rec[i] = r0 + i < n ? o : CA_NONE;
          }
          ca_fold<FMT, VE, LPH, BIG>(a, rec, c, codes);
        }
      }
    }
    ca_store<T, VE>(a, v, c);
  }
}

// Joins the n pieces of segment v, which starts in cell m, for head h.  A chunk of pieces at a
// time: a thread loads its element of CJ_AHEAD of them, and (another role of the
// same threads) a piece's maximum and sum, all in flight together; the weights go
// through LDS.
constexpr int CJ_THREADS = 512, CJ_AHEAD = 8;
template <typename T>
__device__ __forceinline__ void ca_join(const CaArgs& a, int64_t v, int64_t m, int64_t n, int h) {
  __shared__ float s_w[CJ_THREADS], s_sum[CJ_THREADS], s_red[2][CJ_THREADS / 64];
  const int H = a.H, dh = a.dh, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int cols = 1;                        // the elements of a head, padded to a power of two
  while (cols < dh) cols *= 2;
  const int slices = CJ_THREADS / cols, col = tid & (cols - 1), sl = tid / cols;
  const int chunk = CJ_AHEAD * slices < CJ_THREADS ? CJ_AHEAD * slices : CJ_THREADS;
  const int64_t step = int64_t(H) * (dh + 2);
  const float* first = a.part + (2 * m + 1) * step + h * (dh + 2);   // slot 2m + 1, then 2(m + k)
  const float* rest = a.part + 2 * m * step + h * (dh + 2);
  const int64_t ahead = 2 * step * slices;
  float mx = -INFINITY, Z = 0.f, acc = 0.f;
  for (int64_t k0 = 0; k0 < n; k0 += chunk) {
    const int c = int(n - k0 < chunk ? n - k0 : chunk);
    float pa[CJ_AHEAD], pm = -INFINITY, pz = 0.f;
    const float* q = rest + 2 * (k0 + sl) * step + 2 + col;
#pragma unroll
    for (int i = 0; i < CJ_AHEAD; ++i, q += ahead) {
      pa[i] = 0.f;
      if (sl + i * slices < c && col < dh) pa[i] = *(i == 0 && k0 + sl == 0 ? first + 2 + col : q);
    }
    if (tid < c) {
      const float* p = k0 + tid == 0 ? first : rest + 2 * (k0 + tid) * step;
      pm = p[0];
      pz = p[1];
    }
    float mn = pm;
    for (int o = 1; o < 64; o *= 2) mn = fmaxf(mn, __shfl_xor(mn, o));
    if (lane == 0) s_red[0][wave] = mn;
    __syncthreads();
    mn = mx;
    for (int w = 0; w < CJ_THREADS / 64; ++w) mn = fmaxf(mn, s_red[0][w]);
    const float corr = ca_pow2(mx, mn), weight = ca_pow2(pm, mn);
    mx = mn;
    Z = fmaf(pz, weight, Z * corr);
    s_w[tid] = weight;
    __syncthreads();
    acc *= corr;
#pragma unroll
    for (int i = 0; i < CJ_AHEAD; ++i) {
      const int k = sl + i * slices;
      if (k < c) acc = fmaf(pa[i], s_w[k], acc);
    }
    __syncthreads();                   // before the next weights
  }
  Z = group_sum(Z, 64);
  if (lane == 0) s_red[1][wave] = Z;
  s_sum[tid] = acc;
  __syncthreads();
  Z = 0.f;
  for (int w = 0; w < CJ_THREADS / 64; ++w) Z += s_red[1][w];
  const bool some = !(Z == 0.f);
  if (sl == 0 && col < dh) {
    for (int k = 1; k < slices; ++k) acc += s_sum[k * cols + col];
    const float o = some ? acc / Z : 0.f;
    VecIO<T, 1>::store(static_cast<T*>(a.out) + (v * H + h) * dh + col, &o);
  }
  if (a.lse && tid == 0) a.lse[v * H + h] = some ? (mx + log2f(Z)) * LN2 : -INFINITY;
  __syncthreads();                     // before the next segment's sums
}

// The marks of a lane's cell m (-1: none) and of the cell behind it, one round trip for the
// wave.  Returns the lanes that have one.
__device__ __forceinline__ uint64_t ca_marks(const CaArgs& a, int64_t m, int32_t& here, int32_t& next) {
  here = m >= 0 && m < a.cells ? a.mark[ca_mark_at(a, m)] : -1;
  next = m >= 0 && m + 1 < a.cells ? a.mark[ca_mark_at(a, m + 1)] : -1;
  // marks of malformed offsets may be anything
  if (here >= a.N) here = -1;
  if (next >= a.N) next = -1;
  return __ballot(here >= 0 || next >= 0);
}

// The pieces of long segments in cells b, b + CA_CELLS, ... (so that a long history is
// spread over the workgroups).
template <typename T, int FMT, int VE, int LPH, bool BIG>
__global__ void __launch_bounds__(CA_THREADS) k_attn_cached_long(CaArgs a) {
  __shared__ float s_acc[CA_WAVES][VE + 2][CA_PAD];
  const int64_t cap = int64_t(1) << a.shift;
  for (int64_t base = 0; base < a.rounds; base += 64) {
    const int64_t k = base + (threadIdx.x & 63);
    int32_t here, next;
    for (uint64_t set = ca_marks(a, k < a.rounds ? blockIdx.x + k * CA_CELLS : -1, here, next); set;
         set &= set - 1) {             // the same in every wave
      const int i = __builtin_ctzll(set);
      const int64_t x = (blockIdx.x + (base + i) * CA_CELLS) << a.shift, y = x + cap;
      int32_t seg[2] = {__builtin_amdgcn_readlane(here, i), __builtin_amdgcn_readlane(next, i)};
      for (int k = 0; k < 2; ++k) {
        const int32_t v = seg[k];
        if (v < 0 || (k == 1 && v == seg[0])) continue;
        int64_t s, t;
        ca_segment(a, v, s, t);
        const int64_t e0 = s > x ? s : x, e1 = t < y ? t : y;
        if (t - s > cap && e0 < e1)
          ca_piece<T, FMT, VE, LPH, BIG>(a, v, e0, e1, 2 * (x >> a.shift) + (s >= x ? 1 : 0), s_acc);
      }
    }
  }
}

// Joins the long segments that start in cells b, b + CA_CELLS, ... for b = blockIdx.x, blockIdx.x +
// gridDim.x, ..., head blockIdx.y: those that hold the next cell's first edge.
template <typename T>
__global__ void __launch_bounds__(CJ_THREADS) k_attn_cached_join(CaArgs a) {
  // the cells of all b, CA_CELLS apart, in one list: 64 of them at a time
  const uint32_t rounds = uint32_t(a.rounds), lists = (CA_CELLS - blockIdx.x + gridDim.x - 1) / gridDim.x;
  for (uint32_t base = 0; base < lists * rounds; base += 64) {
    const uint32_t q = base + (threadIdx.x & 63), l = q / rounds;
    const int64_t m = l < lists ? blockIdx.x + l * gridDim.x + int64_t(q - l * rounds) * CA_CELLS : -1;
    int32_t here, next;
    for (uint64_t set = ca_marks(a, m, here, next); set; set &= set - 1) {
      const int i = __builtin_ctzll(set);
      const int32_t v = __builtin_amdgcn_readlane(next, i);
      if (v < 0) continue;
      const int64_t at = __builtin_amdgcn_readlane(int32_t(m), i);    // at most 2^23 cells
      int64_t s, t;
      ca_segment(a, v, s, t);
      if (t - s > (int64_t(1) << a.shift) && s >> a.shift == at)
        ca_join<T>(a, v, at, ((t - 1) >> a.shift) - at + 1, blockIdx.y);
    }
  }
}

// Fewer than 64 segments: every wave holds all offsets, so that pieces and whole segments go
// in one launch, without marks.  Workgroups [0, cells) take the pieces of their cell, the
// others a short segment each.
constexpr int CA_FEW = 64;
template <typename T, int FMT, int VE, int LPH, bool BIG>
__global__ void __launch_bounds__(CA_THREADS) k_attn_cached_few(CaArgs a) {
  __shared__ float s_acc[CA_WAVES][VE + 2][CA_PAD];
  const int lane = threadIdx.x & 63;
  const int64_t cap = int64_t(1) << a.shift, m = blockIdx.x;
  if (m < a.cells) {
    const int64_t x = m << a.shift, y = x + cap;
    const int o = lane <= a.N ? int(clamp64(a.off[lane], 0, a.E)) : int(a.E);
    int e = __shfl_down(o, 1);
    e = e > o ? e : o;
    const bool mine = lane < a.N && e - o > cap && o < y && e > x;
    for (uint64_t set = __ballot(mine); set; set &= set - 1) {
      const int v = __builtin_ctzll(set);
      const int64_t s = __builtin_amdgcn_readlane(o, v), t = __builtin_amdgcn_readlane(e, v);
      ca_piece<T, FMT, VE, LPH, BIG>(a, v, s > x ? s : x, t < y ? t : y, 2 * m + (s >= x ? 1 : 0), s_acc);
    }
    return;
  }
  const int64_t v = m - a.cells;
  int64_t s, t;
  ca_segment(a, v, s, t);
  if (t - s <= cap) ca_piece<T, FMT, VE, LPH, BIG>(a, v, s, t, -1, s_acc);
}
template <typename T>
__global__ void __launch_bounds__(CJ_THREADS) k_attn_cached_few_join(CaArgs a) {
  int64_t s, t;
  ca_segment(a, blockIdx.x, s, t);
  if (t - s > int64_t(1) << a.shift)
    ca_join<T>(a, blockIdx.x, s >> a.shift, ((t - 1) >> a.shift) - (s >> a.shift) + 1, blockIdx.y);
}

static int pow2_at_least(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

// Pieces are taken twice as long while at least this many of them are left: more where a wave
// has only one or two records of a kind in flight, fewer of the shortest.
constexpr int64_t CA_PIECES = 640;
static int64_t ca_pieces(int groups, int shift) { return groups <= 2 ? CA_PIECES : shift < 8 ? 320 : 480; }

// How a call is carried out.
struct CaPlan {
  int ve, lph, L;
  bool cross;                          // a last piece may begin in another group than its own codes
  CaOwner owner;
  bool few;                            // k_attn_cached_few
  int shift;
  int64_t cells;
};
static CaPlan ca_plan(int64_t N, int64_t E, int H, int dh) {
  CaPlan p = {};
  // 16 codes a lane: half the lanes and fewer instructions per record
  p.ve = dh > 8 ? 16 : 8;
  p.cross = dh % MX_GROUP >= 1 && dh % MX_GROUP <= MX_PIECE;
  p.lph = pow2_at_least((dh + p.ve - 1) / p.ve);
  int hpw = pow2_at_least(H);
  if (hpw > 64 / p.lph) hpw = 64 / p.lph;
  p.L = p.lph * hpw;
  // A wave per segment where they are few or longer than two rounds of its lanes, else L lanes;
  // a workgroup where workgroups are few and the mean segment gives each wave work.
  // L lanes / wave / workgroup, us, 4 x 32 bf16: 20,000 segments of 10 edges 31 / 39 / 109, 5000 of
  // 10 16 / 16 / 33, 3000 of 100 74 / 33 / 34, 400 of 250 162 / 30 / 19, 600 of 10 12 / 9 / 11.
  const int64_t mean = N > 0 ? E / N : 0;
  if (mean >= 64 && N <= CA_BLOCKS) p.owner = CA_BLOCK;
  else if (N <= CA_LANES_N || mean >= 2 * CA_ROWS * (64 / p.L)) p.owner = CA_WAVE;
  else p.owner = CA_GROUP;
  // Where a wave or a workgroup owns a segment, a piece of cap edges takes cap / (16 * 64 / L)
  // rounds, each about 1 us of dependent loads, so pieces are short, 64 edges, and
  // longer only as their number grows past what the chip runs at once: 64 / 256 / 1024
  // edges, us, one segment of 1000, 8 x 128 14 / 28 / 70, 4 x 32 9.9 / 11.3 / 13.8; 60 of
  // 60,000 in all, 4 x 32, 19 / 17 / 31; four of 100,003 28 / 21 / 32; one of 1,000,000
  // 284 / 113 / 86.
  //   - Not cut at all where the block is no more than a workgroup gets through while
  //     the pieces' results are joined: four segments of 1000 in all, 4 x 32, 12.8 / 8.2 us.
  //   - Not where 64 or more segments are about that long (fewer take one launch less), if
  //     the rounds of an uncut one are few or pass while the block's bytes do: 379
  //     segments of 139,715, cut at 128 / not cut, 4 x 32 52 / 22, 2 x 100 51 / 50 and with
  //     three hubs 51 / 112, 8 x 128 105 / 72 and 107 / 199 (these two are cut); 1500 of
  //     500,000, 8 x 128, not cut: 337 / 188 and 364 / 315.
  // Where a few lanes own a segment, one of 256 takes 45 us, so there are shorter pieces in a block
  // that takes less, 64 / 128 / 256: 6600 segments of 2200 edges in all, three hubs,
  // 14.1 / 17.2 / 53.0 us; 20,000 of 20,000 with hubs 17.0 / 17.3 / 17.6; 50,000 of 100,000
  // with hubs 35.3 / 31.5 / 31.9; 100,000 of 1,000,000 with hubs 130.6 / 111.6 / 100.6.
  const int groups = 64 / p.L;
  if (p.owner == CA_GROUP) {
    p.shift = E <= CA_SHORT_E ? 6 : E <= CA_MEDIUM_E ? 7 : 8;
  } else {
    p.shift = CA_SHIFT;
    while (p.shift < CA_SHIFT_MAX && (E >> (p.shift + 1)) >= ca_pieces(groups, p.shift)) ++p.shift;
    if (E <= std::min(1024, 128 * groups) && std::min(E, 2 * mean) <= 80 * groups) {
      p.shift = 10;
    } else if (N >= CA_FEW && mean <= 2048) {
      int whole = p.shift;
      while ((int64_t(1) << whole) < 2 * mean) ++whole;
      const int64_t round = groups * CA_ROWS * (p.owner == CA_BLOCK ? CA_WAVES : 1);
      if ((int64_t(1) << whole) <= round * (12 + (3 * E * H * dh >> 23))) p.shift = whole;
    }
  }
  // cells of cap edges; none where no segment can be long
  p.cells = E > (int64_t(1) << p.shift) ? ((E - 1) >> p.shift) + 1 : 0;
  p.few = N < CA_FEW && p.cells > 0;
  return p;
}
// The most cells that ca_plan takes for up to N segments and up to E edges: the workspace grows
// with both, so that one for the largest block serves all.
static int64_t ca_cells_most(int64_t N, int64_t E, int H, int dh) {
  const CaPlan p = ca_plan(N, E, H, dh);
  auto cells = [](int64_t e, int shift) { return (e >> shift) + 1; };
  // pieces of 64 up to twice CA_PIECES of them, then longer ones up to CA_SHIFT_MAX
  int64_t most = std::max({p.cells, std::min(cells(E, CA_SHIFT), 2 * CA_PIECES + 1),
                           cells(E, CA_SHIFT_MAX)});
  if (N > CA_LANES_N) {                // a few lanes may own a segment, at this many edges or fewer
    const int64_t e = std::min(E, 2 * CA_ROWS * (64 / p.L) * N);
    most = std::max({most, cells(std::min(e, CA_SHORT_E), 6), cells(std::min(e, CA_MEDIUM_E), 7),
                     cells(e, 8)});
  }
  return most;
}
static size_t ca_part_bytes(int64_t cells, int H, int dh) {
  return align_up(size_t(2 * cells) * H * (dh + 2) * sizeof(float), 16);
}

// Lanes per head known to the compiler and 32-bit record addresses where a cache is below 4 GiB
// and heads have 17 to 128 elements; else one kernel that reads the lanes from the arguments and
// addresses records in 64 bits.  The former / the latter on a cache just below 4 GiB, with a map of
// 200,000,000 ids, 264,000 segments of 2.4 M edges: 2 x 50 fp32 8 bits 226 / 252 us, 4 x 32
// bf16 4 bits 208 / 235 (5.4 GB, by the latter: 253 and 236); without a map 176 / 204, 156 / 188.
template <typename T, int FMT>
static void launch_ca(const CaArgs& a, const CaPlan& p, bool big, dim3 grid, dim3 long_grid, hipStream_t st) {
#define FAST_CAK(K, g) hipLaunchKernelGGL(K, g, dim3(CA_THREADS), 0, st, a)
#define FAST_CA(V, N, B)                                                                       \
  do {                                                                                         \
    if (p.few) FAST_CAK((k_attn_cached_few<T, FMT, V, N, B>), grid);                           \
    else if (p.owner == CA_BLOCK) FAST_CAK((k_attn_cached<T, FMT, V, N, B, CA_BLOCK>), grid);  \
    else if (p.owner == CA_WAVE) FAST_CAK((k_attn_cached<T, FMT, V, N, B, CA_WAVE>), grid);    \
    else FAST_CAK((k_attn_cached<T, FMT, V, N, B, CA_GROUP>), grid);                           \
    if (a.cells > 0 && !p.few) FAST_CAK((k_attn_cached_long<T, FMT, V, N, B>), long_grid);     \
  } while (0)
  if (p.ve == 8) FAST_CA(8, 0, true);
  else if (big) FAST_CA(16, 0, true);
  else if (a.lph == 2) FAST_CA(16, 2, false);
  else if (a.lph == 4 && !p.cross) FAST_CA(16, 4, false);
  else if (a.lph == 4) FAST_CA(16, -4, false);
  else if (a.lph == 8 && !p.cross) FAST_CA(16, 8, false);
  else if (a.lph == 8) FAST_CA(16, -8, false);
  else FAST_CA(16, 0, true);
#undef FAST_CA
#undef FAST_CAK
}

}  // namespace fast

using namespace fast;

extern "C" size_t fast_edge_attention_cached_workspace(int64_t num_dst, int64_t num_edges, int H,
                                                       int dh) {
  if (num_dst < 0 || num_edges < 0 || num_dst >= (int64_t(1) << 31) ||
      num_edges >= (int64_t(1) << 31) || H <= 0 || dh <= 0 || H > 64 ||
      dh > 256 || H * dh > 1024)
    return 0;
  // never 0; partial results, then a mark per cell
  const int64_t cells = ca_cells_most(num_dst, num_edges, H, dh);
  return ca_part_bytes(cells, H, dh) + align_up(size_t(cells + CA_CELLS) * sizeof(int32_t), 16);
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
  if (!aligned(cache, 16) || !aligned(ids, 8) || !aligned(slot_map, 4) || !aligned(g->dst_offsets, 4) ||
      !aligned(lse, 4))
    return fail(FAST_ERR_UNSUPPORTED, "%s: cache, ids, slot_map, dst_offsets or lse misaligned", fn);
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
  const CaPlan p = ca_plan(N, E, H, dh);
  a.lph = p.lph;
  a.L = p.L;
  a.shift = p.shift;
  a.cells = p.cells;
  a.rounds = (a.cells + CA_CELLS - 1) / CA_CELLS;
  a.mark = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + ca_part_bytes(a.cells, H, dh));
  const bool big = a.rec.stride * cache_rows >= (int64_t(1) << 32);
  const int hpw = p.L / p.lph;
  const uint32_t heads = uint32_t((H + hpw - 1) / hpw);
  const int64_t per = p.few || p.owner == CA_BLOCK ? 1 : p.owner == CA_WAVE ? CA_WAVES : CA_THREADS / a.L;
  const dim3 grid(uint32_t((p.few ? a.cells : 0) + (N + per - 1) / per), heads);
  const uint32_t cells = uint32_t(a.cells < CA_CELLS ? a.cells : CA_CELLS);
  if (!grid_fits(grid.x, CA_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  const dim3 long_grid(cells, heads);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32) {
    if (format == FAST_MXFP8) launch_ca<float, FAST_MXFP8>(a, p, big, grid, long_grid, st);
    else launch_ca<float, FAST_MXFP4>(a, p, big, grid, long_grid, st);
  } else {
    if (format == FAST_MXFP8) launch_ca<uint16_t, FAST_MXFP8>(a, p, big, grid, long_grid, st);
    else launch_ca<uint16_t, FAST_MXFP4>(a, p, big, grid, long_grid, st);
  }
  if (p.few) {
    const dim3 join_grid = dim3(uint32_t(N), uint32_t(H));
    if (dtype == FAST_F32)
      hipLaunchKernelGGL((k_attn_cached_few_join<float>), join_grid, dim3(CJ_THREADS), 0, st, a);
    else
      hipLaunchKernelGGL((k_attn_cached_few_join<uint16_t>), join_grid, dim3(CJ_THREADS), 0, st, a);
  } else if (a.cells > 0) {
    const uint32_t lists = 512 / uint32_t(H);        // about 512 workgroups in all
    const dim3 join_grid(cells < lists ? cells : lists, uint32_t(H));
    if (dtype == FAST_F32)
      hipLaunchKernelGGL((k_attn_cached_join<float>), join_grid, dim3(CJ_THREADS), 0, st, a);
    else
      hipLaunchKernelGGL((k_attn_cached_join<uint16_t>), join_grid, dim3(CJ_THREADS), 0, st, a);
  }
  return check_launch(fn);
}
