// attention_cached.hip -- edge softmax + aggregation fused (Sec. 4.3), K|V rows
// read from a cache in 8 or 4 bits through ids and a slot map.
//   t[e,h] = LReLU(scale <Q[v,h], K[slot e,h]>),  out[v,h] = sum softmax(t)[e,h] V[slot e,h]
// over the segment's edges that have a slot; lse = log sum exp t.
//
// Bound by HBM: per edge an id, a slot and a record of about H*dh*(2 or 1) bytes
// at a random place, against two fused multiply-adds per element.  L lanes
// hold a record's heads, 8 codes of K and of V each; CA_ROWS records per lane
// are in flight.  A running maximum, sum and accumulators in base 2 make one pass.
//
// Where there are many short segments, L lanes own one and walk its edges: no
// joins.  Where segments are longer, or too few to fill the chip that way, a wave
// owns one, its 64 / L groups of lanes take the edges in turn, and their
// results are joined by lane exchanges at the end.
//
// Segments longer than `cap` edges (a power of two) are cut at the multiples of cap in
// the block's edge order.  A workgroup per cell between two multiples looks up the
// long segment that comes in from the left and the one that goes out to
// the right with a 64-way search of the offsets, and leaves at once where there is
// none.  Its waves split the piece, join in LDS and write (maximum, sum,
// accumulators) to the workspace; a second launch joins a segment's pieces in order.
#include "attention.h"
#include "mx.h"
#include "rows.h"

namespace fast {

constexpr int CA_THREADS = 256, CA_WAVES = CA_THREADS / 64;
constexpr int CA_ROWS = 4;           // records in flight per lane
constexpr int CA_AHEAD = 2;          // places that a lane looks up at once

struct CaArgs {
  int64_t N, E;
  const int32_t* off;
  int H, dh;
  int lph, L;                        // lanes per head, per record (powers of two up to 64)
  int shift;                         // cap = 1 << shift
  int64_t cells, cell_blocks;        // cells of cap edges (0 where no segment can be long), their workgroups
  int cells_per_block;               // 1 or CA_WAVES: cells b, b + cell_blocks, ...
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
  int32_t* starts;                   // [cells] the long segment that starts in a cell, or -1
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

// A lane's place: head h, its codes [first, first + VE) of which those from `own` on
// are its own (the last piece of a head of 8 (2 k + 1) codes starts 8 earlier
// and shares them with its neighbour); the running softmax.
template <int VE>
struct CaLane {
  int h, l, first, own;
  bool mine;                         // the lane holds codes
  uint32_t code, scale;              // its K codes and their scale within a record
  float q[VE], mx, Z, acc[VE];
};

// lanes per head: known to the compiler, or (LPH = 0) read from the arguments
template <int LPH>
__device__ __forceinline__ int ca_lph(const CaArgs& a) { return LPH > 0 ? LPH : a.lph; }

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
  c.scale = uint32_t(a.rec.scale_off + c.h * a.rec.groups + c.first / MX_GROUP);
}

// CA_ROWS records at rec[] (CA_NONE: none) folded into the running softmax.
// rec[] is the record's byte in a cache of less than 4 GiB, so that an address is a
// base that all lanes share plus 32 bits, or (BIG) its slot.
constexpr uint32_t CA_NONE = 0xffffffffu;
template <int FMT, int VE, int LPH, bool BIG>
__device__ __forceinline__ void ca_fold(const CaArgs& a, const uint32_t (&rec)[CA_ROWS], CaLane<VE>& c) {
  MxPiece<FMT, VE> kc[CA_ROWS], vc[CA_ROWS];
  uint32_t kb[CA_ROWS], vb[CA_ROWS];
  const uint8_t* kbase = a.cache;
  const uint8_t* vbase = a.cache + a.H * a.rec.code_bytes;
  const uint8_t* sbase = a.cache + a.H * a.rec.groups;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    kc[i].zero();
    vc[i].zero();
    kb[i] = vb[i] = 127u;
    if (rec[i] != CA_NONE && c.mine) {
      if constexpr (BIG) {
        const uint64_t o = uint64_t(rec[i]) * uint32_t(a.rec.stride);
        kc[i].load(kbase + (o + c.code));
        vc[i].load(vbase + (o + c.code));
        kb[i] = kbase[o + c.scale];
        vb[i] = sbase[o + c.scale];
      } else {
        const uint32_t o = rec[i] + c.code, s = rec[i] + c.scale;
        kc[i].load(kbase + o);
        vc[i].load(vbase + o);
        kb[i] = kbase[s];
        vb[i] = sbase[s];
      }
    }
  }
  float t[CA_ROWS], mn = c.mx;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    t[i] = -INFINITY;
    if (i > 0 && !__any(rec[i] != CA_NONE)) continue;    // no lane has a record here
    float k[VE], d = 0.f;
    kc[i].unpack(mx_scale(kb[i]), k);
#pragma unroll
    for (int j = 0; j < VE; ++j) d = fmaf(c.q[j], k[j], d);
    if constexpr (LPH > 0) d = group_sum_ct<LPH>(d);
    else d = group_sum(d, a.lph);
    d *= d > 0.f ? 1.f : a.slope;
    t[i] = rec[i] != CA_NONE ? d : -INFINITY;
    mn = fmaxf(mn, t[i]);
  }
  const float corr = ca_pow2(c.mx, mn), ref = mn == -INFINITY ? 0.f : mn;
  c.mx = mn;
  c.Z *= corr;
#pragma unroll
  for (int j = 0; j < VE; ++j) c.acc[j] *= corr;
#pragma unroll
  for (int i = 0; i < CA_ROWS; ++i) {
    if (i > 0 && !__any(rec[i] != CA_NONE)) continue;
    const float w = __builtin_amdgcn_exp2f(t[i] - ref);
    float x[VE];
    vc[i].unpack(mx_scale(vb[i]), x);
    c.Z += w;
#pragma unroll
    for (int j = 0; j < VE; ++j) c.acc[j] = fmaf(w, x[j], c.acc[j]);
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
      ca_fold<FMT, VE, LPH, BIG>(a, rec, c);
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

// Edges [e0, e1) of segment v by a workgroup, into partial result `slot`.
template <typename T, int FMT, int VE, int LPH, bool BIG>
__device__ __forceinline__ void ca_piece(const CaArgs& a, int64_t v, int64_t e0, int64_t e1, int64_t slot,
                                         float (*s_acc)[VE + 2][64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
  if (wave == 0 && lane < a.L && c.mine) {
    float mx = -INFINITY, Z = 0.f;
    for (int w = 0; w < CA_WAVES; ++w) mx = fmaxf(mx, s_acc[w][VE][lane]);
#pragma unroll
    for (int j = 0; j < VE; ++j) c.acc[j] = 0.f;
    for (int w = 0; w < CA_WAVES; ++w) {
      const float k = ca_pow2(s_acc[w][VE][lane], mx);
      Z = fmaf(s_acc[w][VE + 1][lane], k, Z);
#pragma unroll
      for (int j = 0; j < VE; ++j) c.acc[j] = fmaf(s_acc[w][j][lane], k, c.acc[j]);
    }
    float* p = a.part + (slot * a.H + c.h) * (a.dh + 2);
    if (c.l == 0) {
      p[0] = mx;
      p[1] = Z;
    }
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (c.first + j >= c.own && c.first + j < a.dh) p[2 + c.first + j] = c.acc[j];
  }
  __syncthreads();                     // before the next piece of this workgroup
}

struct CaFound {
  int64_t v, e0, e1, slot;             // slot < 0: no piece
};

// WAVE: a wave per segment, else L lanes per segment.
template <typename T, int FMT, int VE, int LPH, bool BIG, bool WAVE>
__global__ void __launch_bounds__(CA_THREADS) k_attn_cached(CaArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t cap = int64_t(1) << a.shift;
  if (int64_t(blockIdx.x) < a.cell_blocks) {
    __shared__ float s_acc[CA_WAVES][VE + 2][64];
    __shared__ CaFound s_found[2 * CA_WAVES];
    // each wave looks into one of this workgroup's cells
    const int64_t m = blockIdx.x + wave * a.cell_blocks, x = m << a.shift, y = x + cap;
    const bool look = wave < a.cells_per_block && m < a.cells;
    CaFound l = {0, 0, 0, -1}, r = l;
    if (look) {
      int64_t s, t, start = -1;
      l.v = ca_find(a, x);             // comes in from the left, or starts at x
      ca_segment(a, l.v, s, t);
      if (s <= x && x < t && t - s > cap) {
        l = {l.v, x, t < y ? t : y, s == x ? 2 * m + 1 : 2 * m};
        if (s == x) start = l.v;
      }
      if (y < a.E) {
        r.v = ca_find(a, y);           // goes out to the right
        ca_segment(a, r.v, s, t);
        if (x < s && s < y && y < t && t - s > cap) {
          r = {r.v, s, y, 2 * m + 1};
          start = r.v;
        }
      }
      if (lane == 0 && blockIdx.y == 0) a.starts[m] = int32_t(start);
    }
    if (lane == 0) {
      s_found[2 * wave] = l;
      s_found[2 * wave + 1] = r;
    }
    __syncthreads();
    for (int k = 0; k < 2 * a.cells_per_block; ++k) {
      const CaFound f = s_found[k];
      if (f.slot >= 0) ca_piece<T, FMT, VE, LPH, BIG>(a, f.v, f.e0, f.e1, f.slot, s_acc);
    }
    return;
  }
  const int64_t block = int64_t(blockIdx.x) - a.cell_blocks;
  CaLane<VE> c;
  int64_t s, t;
  if constexpr (WAVE) {
    const int64_t v = block * CA_WAVES + wave;
    if (v >= a.N) return;
    ca_segment(a, v, s, t);
    if (t - s > cap) return;           // in pieces
    ca_init<T, FMT, VE, LPH>(a, v, c);
    ca_wave<FMT, VE, LPH, BIG>(a, s, t, c);
    if (lane < a.L) ca_store<T, VE>(a, v, c);
  } else {
    const int L = a.L, gl = lane & (L - 1), g0 = lane - gl;
    const int64_t v = block * (CA_THREADS / L) + threadIdx.x / L;
    if (v >= a.N) return;
    ca_segment(a, v, s, t);
    if (t - s > cap) return;
    ca_init<T, FMT, VE, LPH>(a, v, c);
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
          ca_fold<FMT, VE, LPH, BIG>(a, rec, c);
        }
      }
    }
    ca_store<T, VE>(a, v, c);
  }
}

// Joins the pieces of the long segments that start in cells b, b + gridDim.x, ...,
// head blockIdx.y.  Threads over a segment's pieces find the maximum; then,
// CJ_THREADS pieces at a time, one thread per piece forms its weight, and threads
// (element, every slices-th piece) add the weighted accumulators.
constexpr int CJ_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(CJ_THREADS) k_attn_cached_join(CaArgs a) {
  __shared__ float s_red[2][CJ_THREADS / 64];
  __shared__ float s_w[CJ_THREADS];
  __shared__ float s_acc[CJ_THREADS];
  const int h = blockIdx.y, H = a.H, dh = a.dh;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int cols = 1;                        // the elements of a head, padded to a power of two
  while (cols < dh) cols *= 2;
  const int slices = CJ_THREADS / cols, col = threadIdx.x & (cols - 1), sl = threadIdx.x / cols;
  for (int64_t m = blockIdx.x; m < a.cells; m += gridDim.x) {
    const int64_t v = a.starts[m];
    if (v < 0) continue;
    int64_t s, t;
    ca_segment(a, v, s, t);
    const int64_t n = ((t - 1) >> a.shift) - m + 1;    // pieces; the first is slot 2m + 1, then 2(m + k)
    const int64_t step = int64_t(H) * (dh + 2);
    const float* first = a.part + (2 * m + 1) * step + h * (dh + 2);
    const float* rest = a.part + 2 * m * step + h * (dh + 2);
    auto piece = [&](int64_t k) { return k == 0 ? first : rest + 2 * k * step; };
    float mx = -INFINITY;
    for (int64_t k = threadIdx.x; k < n; k += CJ_THREADS) mx = fmaxf(mx, piece(k)[0]);
    for (int o = 1; o < 64; o *= 2) mx = fmaxf(mx, __shfl_xor(mx, o));
    if (lane == 0) s_red[0][wave] = mx;
    __syncthreads();
    for (int w = 0; w < CJ_THREADS / 64; ++w) mx = fmaxf(mx, s_red[0][w]);
    float Z = 0.f, acc = 0.f;
    for (int64_t k0 = 0; k0 < n; k0 += CJ_THREADS) {
      const int c = int(n - k0 < CJ_THREADS ? n - k0 : CJ_THREADS);
      if (int(threadIdx.x) < c) {
        const float* p = piece(k0 + threadIdx.x);
        const float w = ca_pow2(p[0], mx);
        s_w[threadIdx.x] = w;
        Z = fmaf(p[1], w, Z);
      }
      __syncthreads();
      if (col < dh) {
#pragma unroll 8
        for (int k = sl; k < c; k += slices) acc = fmaf(piece(k0 + k)[2 + col], s_w[k], acc);
      }
      __syncthreads();                 // before the next weights
    }
    Z = group_sum(Z, 64);
    if (lane == 0) s_red[1][wave] = Z;
    s_acc[threadIdx.x] = acc;
    __syncthreads();
    Z = 0.f;
    for (int w = 0; w < CJ_THREADS / 64; ++w) Z += s_red[1][w];
    const bool some = !(Z == 0.f);
    if (sl == 0 && col < dh) {
      for (int k = 1; k < slices; ++k) acc += s_acc[k * cols + col];
      const float o = some ? acc / Z : 0.f;
      VecIO<T, 1>::store(static_cast<T*>(a.out) + (v * H + h) * dh + col, &o);
    }
    if (a.lse && threadIdx.x == 0) a.lse[v * H + h] = some ? (mx + log2f(Z)) * LN2 : -INFINITY;
    __syncthreads();                   // before the next segment's sums
  }
}

// Piece length of long segments: a workgroup's 4 waves take 64 edges each, and more
// where there are pieces enough to fill the chip.
static int ca_shift(int64_t E) {
  int s = 8;
  while (s < 10 && (E >> (s + 1)) >= 8192) ++s;
  return s;
}

static int pow2_at_least(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

template <typename T, int FMT, bool WAVE>
static void launch_ca(const CaArgs& a, int ve, bool big, dim3 grid, hipStream_t st) {
#define FAST_CA(V, N, B) \
  hipLaunchKernelGGL((k_attn_cached<T, FMT, V, N, B, WAVE>), grid, dim3(CA_THREADS), 0, st, a)
  if (ve == 8) FAST_CA(8, 0, true);
  else if (big) FAST_CA(16, 0, true);
  else if (a.lph == 2) FAST_CA(16, 2, false);
  else if (a.lph == 4) FAST_CA(16, 4, false);
  else if (a.lph == 8) FAST_CA(16, 8, false);
  else FAST_CA(16, 0, true);
#undef FAST_CA
}

static int64_t ca_cells(int64_t E) {
  const int s = ca_shift(E);
  return E > (int64_t(1) << s) ? ((E - 1) >> s) + 1 : 0;
}
static size_t ca_part_bytes(int64_t E, int H, int dh) {
  return align_up(size_t(2 * ca_cells(E)) * H * (dh + 2) * sizeof(float), 16);
}

}  // namespace fast

using namespace fast;

extern "C" size_t fast_edge_attention_cached_workspace(int64_t num_dst, int64_t num_edges, int H,
                                                       int dh) {
  if (num_dst < 0 || num_edges < 0 || num_edges >= (int64_t(1) << 31) || H <= 0 || dh <= 0 || H > 64 ||
      dh > 256 || H * dh > 1024)
    return 0;
  return ca_part_bytes(num_edges, H, dh) + align_up(size_t(ca_cells(num_edges) + 1) * sizeof(int32_t), 16);
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
  a.cells = ca_cells(E);
  // Cells are looked at CA_WAVES to a workgroup where there are many, so that the
  // looking costs little; a workgroup each where they may be all the work.
  a.cells_per_block = a.cells > 2048 ? CA_WAVES : 1;
  a.cell_blocks = (a.cells + a.cells_per_block - 1) / a.cells_per_block;
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
  a.starts = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + ca_part_bytes(E, H, dh));
  // 16 codes a lane (fewer instructions per record) where every lane's codes lie in
  // one group: a head's last piece may start 8 codes early, which crosses a
  // group's border where 1 to 8 elements are left past one.
  const int ve = dh > 8 && (dh % MX_GROUP == 0 || dh % MX_GROUP > 8) ? 16 : 8;
  a.lph = pow2_at_least((dh + ve - 1) / ve);
  int hpw = pow2_at_least(H);
  if (hpw > 64 / a.lph) hpw = 64 / a.lph;
  a.L = a.lph * hpw;
  const bool big = a.rec.stride * cache_rows >= (int64_t(1) << 32);
  // Few segments, or long ones: a wave each.
  const bool wave = N <= 4096 || E / N >= 2 * CA_ROWS * (64 / a.L);
  const int64_t per = wave ? CA_WAVES : CA_THREADS / a.L;
  const dim3 grid(uint32_t(a.cell_blocks + (N + per - 1) / per), uint32_t((H + hpw - 1) / hpw));
  hipStream_t st = static_cast<hipStream_t>(stream);
#define FAST_CAL(T, F)                            \
  do {                                            \
    if (wave) launch_ca<T, F, true>(a, ve, big, grid, st);  \
    else launch_ca<T, F, false>(a, ve, big, grid, st); \
  } while (0)
  if (dtype == FAST_F32) {
    if (format == FAST_MXFP8) FAST_CAL(float, FAST_MXFP8);
    else FAST_CAL(float, FAST_MXFP4);
  } else {
    if (format == FAST_MXFP8) FAST_CAL(uint16_t, FAST_MXFP8);
    else FAST_CAL(uint16_t, FAST_MXFP4);
  }
#undef FAST_CAL
  if (a.cells > 0) {
    const dim3 jg(uint32_t(a.cells > 2048 ? (a.cells + 15) / 16 : a.cells), uint32_t(H));
    if (dtype == FAST_F32) hipLaunchKernelGGL((k_attn_cached_join<float>), jg, dim3(CJ_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_attn_cached_join<uint16_t>), jg, dim3(CJ_THREADS), 0, st, a);
  }
  return check_launch(fn);
}
