// linear.hip -- products of rows with weights, with an epilogue, and their backward.
//   z = x w^T + bias,  y = act(z) + res;   dz = dy act'(pre),  dx = dz w,  dw = dz^T x
//
// All products run as one shape, C[r, c] = sum_k A[r, k] B[c, k], with k side by side in
// both operands: forward A = x, B = w; dx A = dz, B = w^T (transposed first, it is small);
// dw A = dz^T, B = x^T, transposed on their way into LDS.  A 16-byte chunk of k is what a
// lane feeds to the matrix unit: 8 bf16 values to one 32x32x16 instruction, 4 fp32 values
// to four 32x32x2 instructions (which k a lane holds is free as long as both operands
// agree).  B's rows go into the instruction's rows and A's into its columns, so a lane
// ends with 4 neighbouring columns of C in a row of its own.
//
// Bound by HBM for narrow rows (n (in + out) elements), by the matrix units from a few
// hundred columns on.  264,000 rows bf16 272 -> 256: 76 us, dx 78-88, dw 96 + 11; fp32 372 -> 200 with
// gelu and its pre 470-550, dx 380-475, dw 310-375 (the clock falls over repeated passes), dz 122; 40,000 rows bf16
// 2048 -> 2048 with silu and residual 480-560, dx of dz in two parts 780-880 (850 TFLOP/s; of one part, as
// without an activation or with relu, 400), dw in three parts 1040-1240 (970), dz 220.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace fast {

constexpr int64_t LIN_MAX = 16384;        // columns
constexpr int64_t LIN_MAX_LD = 1 << 22;   // elements from row to row: a tile's rows within 2^32 bytes
constexpr int LIN_THREADS = 256;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void lin_mma(uint16_t, const u32x4& a, const u32x4& b, f32x16_t& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                              0, 0);
}
__device__ __forceinline__ void lin_mma(float, const u32x4& a, const u32x4& b, f32x16_t& c) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
}

// p[i] where p is the same for the whole wave and i elements are less than 2^32 bytes: the form that a
// load takes as a scalar base and a 32-bit offset.
template <typename T>
__device__ __forceinline__ const T* at_offset(const T* p, uint32_t i) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) + size_t(i * uint32_t(sizeof(T))));
}

// A row's end.  A chunk of k that reaches past it is loaded from far enough back to end with the
// row, like all others in one instruction (a branch around a load is a wait for it), and its
// first `skip` elements, which belong to the chunk before, are cleared in both operands.
// Rows of less than a chunk are loaded element by element.
template <typename T>
__device__ __forceinline__ u32x4 lin_load(const T* p) {
  const u32x4_e w = *reinterpret_cast<const u32x4_e*>(p);
  return u32x4{w.x, w.y, w.z, w.w};
}
template <typename T>
__device__ __forceinline__ u32x4 lin_load_short(const T* p, int n) {
  u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < CHUNK<T> - 1; ++j)
    if (j < n) {
      if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(p[j]);
      else w[j / 2] |= uint32_t(p[j]) << (16 * (j & 1));
    }
  return w;
}
__device__ __forceinline__ void lin_unpack(float, const u32x4& w, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void lin_unpack(uint16_t, const u32x4& w, float* x) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
// bf16: elements skip, skip + 1, ... of a chunk moved to its start, zeros behind them (0 <= skip < 8)
__device__ __forceinline__ u32x4 lin_shift(const u32x4& w, int skip) {
  uint64_t lo = uint64_t(w[1]) << 32 | w[0], hi = uint64_t(w[3]) << 32 | w[2];
  if (skip >= 4) {
    lo = hi;
    hi = 0;
    skip -= 4;
  }
  if (skip > 0) {
    lo = lo >> (16 * skip) | hi << (64 - 16 * skip);
    hi >>= 16 * skip;
  }
  return u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
}
template <typename T>
__device__ __forceinline__ u32x4 lin_mask(int skip) {
  u32x4 m;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    if constexpr (sizeof(T) == 4) m[d] = d >= skip ? ~0u : 0u;
    else m[d] = 2 * d >= skip ? ~0u : (2 * d + 1 >= skip ? 0xffff0000u : 0u);
  }
  return m;
}

// ------------------------------------------------------------------ fp32 in three parts
// An fp32 value is the sum of three bf16 values: rounded to nearest, subtracted (exactly), rounded again; the
// rest has 8 bits or fewer.  The second is at most 2^-8 of the value, the third 2^-16.  A product of two is then
// six products of parts; the three that are left out are at most 2^-23 of it together, of either sign (cut off
// instead of rounded, the parts would all have the value's sign and twice the size: 2^-21, and sums of products
// short by the mean of it).  Six bf16 instructions take 2.7
// times less than the fp32 ones of the same product.  An infinity has no such parts (and a part
// of 0 times an infinity is no number), and what rounds to one neither: a workgroup that meets such a value does
// its tile again with fp32 instructions.
struct LinParts {
  u32x4 p[3];                        // 8 values: their first, second and third parts
};
// cut: accumulates what is not a number once a value was not finite, or rounded to an infinity.
__device__ __forceinline__ LinParts lin_split(const float* x, float& cut) {
  LinParts r;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    float y[2], z[2];
    r.p[0][d] = bf16_pack(x[2 * d], x[2 * d + 1]);
    y[0] = x[2 * d] - bf16_lo(r.p[0][d]);
    y[1] = x[2 * d + 1] - bf16_hi(r.p[0][d]);
    r.p[1][d] = bf16_pack(y[0], y[1]);
    z[0] = y[0] - bf16_lo(r.p[1][d]);
    z[1] = y[1] - bf16_hi(r.p[1][d]);
    cut = fmaf(y[0], 0.f, fmaf(y[1], 0.f, cut));
    r.p[2][d] = __builtin_amdgcn_perm(__float_as_uint(z[1]), __float_as_uint(z[0]), 0x07060302u);
  }
  return r;
}
template <typename T> constexpr int LIN_PARTS = sizeof(T) == 4 ? 3 : 1;

// ------------------------------------------------------------------ activations
// e^-h, h >= 0, within (1.3 h + 2) U of itself, U half a step of fp32: one rounded product, where a second one would
// keep 2 U.  What is that far out is e^-h beside the row's other values, and its error h U of that.
__device__ __forceinline__ float exp_down(float h) {
  return __builtin_amdgcn_exp2f(h * -0x1.715476p+0f);
}
// Phi(-|z|) and phi(z) sqrt(2 pi): e^(-z^2 / 2) times half of e^(x^2) erfc(x) at x = |z| / sqrt 2, which is
// t times a polynomial in t = 1 / (1 + 0.48 x), within 2^-21.5 (a weighted least-squares fit).
__device__ __forceinline__ float2 gauss(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0x1.5b8ea0p-2f, 1.f)), e = exp_down(0.5f * z * z);
  float p = -0x1.908a46p-5f;
  p = fmaf(p, t, 0x1.0ed562p-2f);
  p = fmaf(p, t, -0x1.0aae58p-1f);
  p = fmaf(p, t, 0x1.853468p-2f);
  p = fmaf(p, t, -0x1.2be910p-4f);
  p = fmaf(p, t, 0x1.cbc510p-3f);
  p = fmaf(p, t, 0x1.da3e00p-3f);
  p = fmaf(p, t, 0x1.16153cp-2f);
  p = fmaf(p, t, 0x1.1547b2p-2f);
  return make_float2(0.5f * p * t * e, e);
}
__device__ __forceinline__ float act_of(int act, float z) {
  if (act == FAST_ACT_RELU) return z > 0.f ? z : (z == z ? 0.f : z);
  if (act == FAST_ACT_GELU) {
    const float q = gauss(z).x;
    return z * (z > 0.f ? 1.f - q : q);
  }
  if (act == FAST_ACT_SILU) {
    const float r = __builtin_amdgcn_rcpf(1.f + exp_down(fabsf(z)));
    // (far out e^z lies below the normal numbers, z e^z not yet: 2^100 times as much of it)
    const float h = z * 0x1.715476p+0f;
    const bool far = h < -100.f;
    const float t = __builtin_amdgcn_exp2f(far ? h + 100.f : h);
    return z > 0.f ? z * r : z * r * t * (far ? 0x1p-100f : 1.f);
  }
  return z;
}
__device__ __forceinline__ float slope_of(int act, float z) {
  if (act == FAST_ACT_RELU) return z > 0.f ? 1.f : (z == z ? 0.f : z);
  if (act == FAST_ACT_GELU) {
    const float2 g = gauss(z);
    return fmaf(z * 0x1.988454p-2f, g.y, z > 0.f ? 1.f - g.x : g.x);
  }
  if (act == FAST_ACT_SILU) {
    const float t = exp_down(fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + t), p = z > 0.f ? r : t * r;
    return fmaf(z * p, z > 0.f ? t * r : r, p);            // p (1 + z (1 - p))
  }
  return 1.f;
}

// ------------------------------------------------------------------ the products
struct LinArgs {
  const void* a;                     // [n, K], lda apart
  int64_t lda;
  const void* b;                     // [M, K], ldb apart
  int64_t ldb;
  int64_t n;
  int M;
  int64_t K;
  const float* bias;
  int act;
  const void* res;
  int64_t ldres;
  void* y;
  int64_t ldy;
  void* pre;                         // rows of M elements
  int tiles_c;                       // tiles along c
  // weight gradients: K is cut into splits of `rows`, each with a result of its own
  int64_t rows;
  float* part;
  float* sums;
};

// f(integral_constant) for 0 .. N-1: an array of accumulators stays in registers only if every
// index is a constant.
template <int N, typename F>
__device__ __forceinline__ void lin_each(F f) {
  if constexpr (N > 0) {
    lin_each<N - 1>(f);
    f(std::integral_constant<int, N - 1>());
  }
}

// The epilogue of a lane: VE neighbouring columns, the same in every row that it finishes.
template <typename T, int VE>
struct LinEnd {
  static constexpr bool CHUNKS = VE == CHUNK<T>;
  const LinArgs& p;
  int c, n;                          // first column, columns in the row
  float bias[VE];
  __device__ LinEnd(const LinArgs& p_, int c_) : p(p_), c(c_), n(p_.M - c_) {
#pragma unroll
    for (int j = 0; j < VE; ++j) bias[j] = p.bias && j < n ? p.bias[c + j] : 0.f;
  }
  // row r's chunk of res, ahead of its use (the row's last chunk, if it is not whole, and rows past
  // the end load something else)
  __device__ u32x4 ahead(int64_t r) const {
    static_assert(CHUNKS, "whole chunks");
    if (!p.res || p.M < VE) return u32x4{0u, 0u, 0u, 0u};
    return lin_load(static_cast<const T*>(p.res) + min(r, p.n - 1) * p.ldres + (n >= VE ? c : 0));
  }
  __device__ void finish(int64_t r, float* z, u32x4 raw = u32x4{0u, 0u, 0u, 0u}) const {
    if (r >= p.n || n <= 0) return;
    float t[VE];
    const T* res = p.res ? static_cast<const T*>(p.res) + r * p.ldres + c : nullptr;
    T* pre = p.pre ? static_cast<T*>(p.pre) + r * p.M + c : nullptr;
    T* y = static_cast<T*>(p.y) + r * p.ldy + c;
    if constexpr (CHUNKS) {
      if (n >= VE) lin_unpack(T(), raw, t);
      else if (res) load_chunk(res, n, t);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        t[j] = 0.f;
        if (res && j < n) VecIO<T, 1>::load(res + j, &t[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) z[j] += bias[j];
    if (pre) put(pre, z);
    if (p.act != FAST_ACT_NONE) {
#pragma unroll
      for (int j = 0; j < VE; ++j) z[j] = act_of(p.act, z[j]);
    }
    if (res) {
#pragma unroll
      for (int j = 0; j < VE; ++j) z[j] += t[j];
    }
    put(y, z);
  }
  __device__ void put(T* o, const float* z) const {
    if constexpr (CHUNKS) {
      store_chunk(o, n, z);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (j < n) VecIO<T, 1>::store(o + j, &z[j]);
    }
  }
};

// The tiles of a workgroup: WR x WC waves of TR x TC blocks of 32 x 32 each, KB bytes of k.
template <int WR_, int WC_, int TR_, int TC_, int KB_>
struct LinTile {
  static constexpr int WR = WR_, WC = WC_, TR = TR_, TC = TC_, KB = KB_;
  static constexpr int THREADS = 64 * WR * WC, BR = 32 * WR * TR, BC = 32 * WC * TC;
  static constexpr int CHUNKS = KB / 16;                       // of a row of LDS
  static constexpr int ROW = KB + 16;                          // 16 lanes' chunks fall into different banks
  static constexpr int BUF = (BR + BC) * ROW;                  // a tile of k of both operands
  // (the epilogue takes 32 rows of every wave's block through it)
  static constexpr int LDS = 2 * BUF > WR * WC * 32 * (TC * 32 + 4) * 4 ? 2 * BUF : WR * WC * 32 * (TC * 32 + 4) * 4;
};
typedef LinTile<4, 2, 2, 2, 64> LinBig;    // 256 x 128
typedef LinTile<2, 2, 2, 2, 64> LinMid;    // 128 x 128
typedef LinTile<2, 2, 2, 2, 128> LinGrad;  // 128 x 128 of weight gradients
typedef LinTile<2, 4, 2, 2, 64> LinWide;   // 128 x 256

// A wave's part of a tile: TR x TC blocks of 32 x 32 over a tile of k in LDS.
template <typename T, typename Tile>
__device__ __forceinline__ void lin_step(const char* la, const char* lb, f32x16_t (&acc)[Tile::TR][Tile::TC]) {
  constexpr int TR = Tile::TR, TC = Tile::TC, ROW = Tile::ROW;
  const int lane = threadIdx.x & 63;
  la += (lane & 31) * ROW + (lane >> 5) * 16;
  lb += (lane & 31) * ROW + (lane >> 5) * 16;
#pragma unroll
  for (int k = 0; k < Tile::KB; k += 32) {
    u32x4 fa[TR], fb[TC];
#pragma unroll
    for (int i = 0; i < TR; ++i) fa[i] = *reinterpret_cast<const u32x4*>(la + i * 32 * ROW + k);
#pragma unroll
    for (int j = 0; j < TC; ++j) fb[j] = *reinterpret_cast<const u32x4*>(lb + j * 32 * ROW + k);
#pragma unroll
    for (int i = 0; i < TR; ++i)
#pragma unroll
      for (int j = 0; j < TC; ++j) lin_mma(T(), fb[j], fa[i], acc[i][j]);
  }
}

// The same with PA and PB parts of the operands, their tiles one behind the other.
template <typename Tile, int PA, int PB>
__device__ __forceinline__ void lin_step_parts(const char* la, const char* lb,
                                               f32x16_t (&acc)[Tile::TR][Tile::TC]) {
  constexpr int TR = Tile::TR, TC = Tile::TC, ROW = Tile::ROW;
  const int lane = threadIdx.x & 63;
  la += (lane & 31) * ROW + (lane >> 5) * 16;
  lb += (lane & 31) * ROW + (lane >> 5) * 16;
#pragma unroll
  for (int k = 0; k < Tile::KB; k += 32) {
    u32x4 fa[TR][PA], fb[TC][PB];
#pragma unroll
    for (int i = 0; i < TR; ++i)
#pragma unroll
      for (int s = 0; s < PA; ++s) fa[i][s] = *reinterpret_cast<const u32x4*>(la + (s * Tile::BR + i * 32) * ROW + k);
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int s = 0; s < PB; ++s) fb[j][s] = *reinterpret_cast<const u32x4*>(lb + (s * Tile::BC + j * 32) * ROW + k);
    // the small products first
#pragma unroll
    for (int s = PA + PB - 2 < 2 ? PA + PB - 2 : 2; s >= 0; --s)
#pragma unroll
      for (int q = 0; q < PA; ++q)
        if (s - q >= 0 && s - q < PB) {
#pragma unroll
          for (int i = 0; i < TR; ++i)
#pragma unroll
            for (int j = 0; j < TC; ++j) lin_mma(uint16_t(), fb[j][s - q], fa[i][q], acc[i][j]);
        }
  }
}
template <int TR, int TC>
__device__ __forceinline__ void lin_clear(f32x16_t (&acc)[TR][TC]) {
#pragma unroll
  for (int i = 0; i < TR; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
}

// The wave's block through LDS, 32 rows at a time, so that rows leave in whole chunks.
// ahead(row of the wave's block): what out will want, on its way before the block is turned;
// out(row, values, that): of VE columns from (lane % (TC * 32 / VE)) * VE on.
template <int VE, int TR, int TC, typename G, typename F>
__device__ __forceinline__ void lin_out(char* lds, const f32x16_t (&acc)[TR][TC], G ahead, F out) {
  constexpr int W = TC * 32, LD = W + 4, PER = W / VE, ROWS = 64 / PER, COUNT = 32 / ROWS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* buf = reinterpret_cast<float*>(lds) + wave * 32 * LD;
  lin_each<TR>([&](auto I) {
    constexpr int i = decltype(I)::value;
    u32x4 raw[COUNT];
#pragma unroll
    for (int q = 0; q < COUNT; ++q) raw[q] = ahead(i * 32 + q * ROWS + lane / PER);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(buf + (lane & 31) * LD + j * 32 + q * 8 + (lane >> 5) * 4) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
#pragma unroll
    for (int q = 0; q < COUNT; ++q) {
      const int r = q * ROWS + lane / PER, c = lane % PER * VE;
      float z[VE];
#pragma unroll
      for (int v = 0; v < VE; v += 4) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(buf + r * LD + c + v);
        z[v] = w.x; z[v + 1] = w.y; z[v + 2] = w.z; z[v + 3] = w.w;
      }
      out(i * 32 + r, z, raw[q]);
    }
  });
}

// Tiles of BR rows and BC columns; the next tile of k is on its way into registers while this
// one is multiplied from LDS.  SHORT: rows of less than a chunk.
template <typename T, typename Tile, bool SHORT>
__global__ void __launch_bounds__(Tile::THREADS) k_linear(LinArgs p) {
  constexpr int TR = Tile::TR, TC = Tile::TC, BR = Tile::BR, BC = Tile::BC, BUF = Tile::BUF;
  constexpr int VE = CHUNK<T>, BK = Tile::KB / int(sizeof(T)), STEP = Tile::THREADS / Tile::CHUNKS;
  constexpr int NA = BR / STEP, NB = BC / STEP;
  __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t r0 = int64_t(id / uint32_t(p.tiles_c)) * BR;
  const int c0 = int(id % uint32_t(p.tiles_c)) * BC;
  const int row = threadIdx.x / Tile::CHUNKS, chunk = threadIdx.x % Tile::CHUNKS;
  // places as 32-bit offsets from the tile's corner, which is the same for the whole workgroup
  const T* A = static_cast<const T*>(p.a) + r0 * p.lda;
  const T* B = static_cast<const T*>(p.b) + int64_t(c0) * p.ldb;
  uint32_t oa[NA], ob[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
    oa[i] = uint32_t(min(int64_t(i * STEP + row), p.n - 1 - r0)) * uint32_t(p.lda);
#pragma unroll
  for (int i = 0; i < NB; ++i) ob[i] = uint32_t(min(i * STEP + row, p.M - 1 - c0)) * uint32_t(p.ldb);
  const int K = int(p.K), full = K / BK, tiles = (K + BK - 1) / BK;
  // this thread's chunk of the last tile, where that is not full
  const int last = full * BK + chunk * VE, back = min(last, K - VE);
  const u32x4 mask = lin_mask<T>(last - back);
  u32x4 ra[NA], rb[NB];
  auto load = [&](int t) {
    if constexpr (SHORT) {
#pragma unroll
      for (int i = 0; i < NA; ++i) ra[i] = lin_load_short(A + oa[i], chunk == 0 ? K : 0);
#pragma unroll
      for (int i = 0; i < NB; ++i) rb[i] = lin_load_short(B + ob[i], chunk == 0 ? K : 0);
    } else {
      const uint32_t k = t < full ? chunk * VE : back;
      const T* pa = A + (t < full ? t * BK : 0);
      const T* pb = B + (t < full ? t * BK : 0);
#pragma unroll
      for (int i = 0; i < NA; ++i) ra[i] = lin_load(at_offset(pa, oa[i] + k));
#pragma unroll
      for (int i = 0; i < NB; ++i) rb[i] = lin_load(at_offset(pb, ob[i] + k));
    }
  };
  auto put = [&](int t, char* buf) {
    char* at = buf + row * Tile::ROW + chunk * 16;
    if (!SHORT && t >= full) {
#pragma unroll
      for (int i = 0; i < NA; ++i) ra[i] &= mask;
#pragma unroll
      for (int i = 0; i < NB; ++i) rb[i] &= mask;
    }
#pragma unroll
    for (int i = 0; i < NA; ++i) *reinterpret_cast<u32x4*>(at + i * STEP * Tile::ROW) = ra[i];
#pragma unroll
    for (int i = 0; i < NB; ++i) *reinterpret_cast<u32x4*>(at + (BR + i * STEP) * Tile::ROW) = rb[i];
  };
  f32x16_t acc[TR][TC];
#pragma unroll
  for (int i = 0; i < TR; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  const int wave = threadIdx.x >> 6, wr = wave / Tile::WC, wc = wave % Tile::WC;
  load(0);
  put(0, lds);
  __syncthreads();
  int cur = 0;
  for (int t = 0; t < tiles; ++t) {
    const bool more = t + 1 < tiles;
    if (more) load(t + 1);
    const char* buf = lds + cur * BUF;
    lin_step<T, Tile>(buf + wr * TR * 32 * Tile::ROW, buf + (BR + wc * TC * 32) * Tile::ROW, acc);
    cur ^= 1;
    if (more) put(t + 1, lds + cur * BUF);
    __syncthreads();
  }
  const LinEnd<T, VE> end(p, c0 + wc * TC * 32 + (threadIdx.x & 63) % (TC * 32 / VE) * VE);
  const int64_t rw = r0 + wr * TR * 32;
  lin_out<VE>(lds, acc, [&](int r) { return end.ahead(rw + r); },
              [&](int r, float* z, u32x4 raw) { end.finish(rw + r, z, raw); });
}

// k_linear of fp32 rows in parts; K >= 8.  One buffer in LDS, so that two workgroups share a CU:
// one multiplies while the other cuts its next tile of k up.
template <typename Tile>
__global__ void __launch_bounds__(Tile::THREADS) k_linear_parts(LinArgs p) {
  constexpr int TR = Tile::TR, TC = Tile::TC, BR = Tile::BR, BC = Tile::BC, ROW = Tile::ROW;
  constexpr int VE = 8, BK = Tile::KB / 2, STEP = Tile::THREADS / Tile::CHUNKS, NA = BR / STEP, NB = BC / STEP;
  __shared__ __attribute__((aligned(16))) char lds[3 * (BR + BC) * ROW];
  static_assert(sizeof(lds) >= Tile::WR * Tile::WC * 32 * (TC * 32 + 4) * 4, "the epilogue's buffer");
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t r0 = int64_t(id / uint32_t(p.tiles_c)) * BR;
  const int c0 = int(id % uint32_t(p.tiles_c)) * BC;
  const int row = threadIdx.x / Tile::CHUNKS, chunk = threadIdx.x % Tile::CHUNKS;
  const float* A = static_cast<const float*>(p.a) + r0 * p.lda;
  const float* B = static_cast<const float*>(p.b) + int64_t(c0) * p.ldb;
  uint32_t oa[NA], ob[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i)
    oa[i] = uint32_t(min(int64_t(i * STEP + row), p.n - 1 - r0)) * uint32_t(p.lda);
#pragma unroll
  for (int i = 0; i < NB; ++i) ob[i] = uint32_t(min(i * STEP + row, p.M - 1 - c0)) * uint32_t(p.ldb);
  const int K = int(p.K), full = K / BK, tiles = (K + BK - 1) / BK;
  const int last = full * BK + chunk * VE, back = min(last, K - VE), skip = last - back;
  u32x4 ra[NA][2], rb[NB][2];
  auto load = [&](int t) {
    const uint32_t k = t < full ? chunk * VE : back;
    const float* pa = A + (t < full ? t * BK : 0);
    const float* pb = B + (t < full ? t * BK : 0);
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      ra[i][0] = lin_load(at_offset(pa, oa[i] + k));
      ra[i][1] = lin_load(at_offset(pa, oa[i] + k + 4));
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      rb[i][0] = lin_load(at_offset(pb, ob[i] + k));
      rb[i][1] = lin_load(at_offset(pb, ob[i] + k + 4));
    }
  };
  float cut = 0.f;
  auto part = [&](const u32x4 (&w)[2], bool end, char* at, int rows) {
    float x[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) x[j] = __uint_as_float(w[j / 4][j % 4]);
    if (end) {
#pragma unroll
      for (int j = 0; j < VE; ++j) x[j] = j >= skip ? x[j] : 0.f;
    }
    const LinParts s = lin_split(x, cut);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4*>(at + q * rows * ROW) = s.p[q];
  };
  auto put = [&](int t) {
    char* at = lds + row * ROW + chunk * 16;
#pragma unroll
    for (int i = 0; i < NA; ++i) part(ra[i], t >= full, at + i * STEP * ROW, BR);
#pragma unroll
    for (int i = 0; i < NB; ++i) part(rb[i], t >= full, at + (3 * BR + i * STEP) * ROW, BC);
  };
  f32x16_t acc[TR][TC];
  lin_clear(acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / Tile::WC, wc = wave % Tile::WC;
  load(0);
  for (int t = 0; t < tiles; ++t) {
    put(t);
    __syncthreads();
    if (t + 1 < tiles) load(t + 1);
    lin_step_parts<Tile, 3, 3>(lds + wr * TR * 32 * ROW, lds + (3 * BR + wc * TC * 32) * ROW, acc);
    __syncthreads();
  }
  if (__syncthreads_or(cut != cut)) {                     // not finite: from memory, in fp32
    lin_clear(acc);
    const int half = lane >> 5;
    for (int k = half * 4; k - half * 4 < K; k += 8) {
      const int at = min(k, K - 4);
      const u32x4 m = lin_mask<float>(k - at);
      u32x4 fa[TR], fb[TC];
#pragma unroll
      for (int i = 0; i < TR; ++i) {
        const int64_t r = min(int64_t(wr * TR * 32 + i * 32 + (lane & 31)), p.n - 1 - r0);
        fa[i] = lin_load(A + r * p.lda + at) & m;
      }
#pragma unroll
      for (int j = 0; j < TC; ++j) {
        const int64_t c = min(wc * TC * 32 + j * 32 + (lane & 31), p.M - 1 - c0);
        fb[j] = lin_load(B + c * p.ldb + at) & m;
      }
#pragma unroll
      for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < TC; ++j) lin_mma(float(), fb[j], fa[i], acc[i][j]);
    }
  }
  const LinEnd<float, 4> end(p, c0 + wc * TC * 32 + lane % (TC * 8) * 4);
  const int64_t rw = r0 + wr * TR * 32;
  lin_out<4>(lds, acc, [&](int r) { return end.ahead(rw + r); },
             [&](int r, float* z, u32x4 raw) { end.finish(rw + r, z, raw); });
}

// Few rows: 32 x 32 results a workgroup, its waves share k, each feeding the matrix unit from
// global memory; their sums are added in order in LDS.
template <typename T, int WAVES, bool SHORT>
__global__ void __launch_bounds__(64 * WAVES) k_linear_few(LinArgs p) {
  constexpr int VE = CHUNK<T>, STEP = 2 * VE, LD = 36, AHEAD = 4, ROUND = AHEAD * WAVES * STEP;
  __shared__ float buf[WAVES][32 * LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int64_t r0 = int64_t(blockIdx.x / uint32_t(p.tiles_c)) * 32;
  const int c0 = int(blockIdx.x % uint32_t(p.tiles_c)) * 32, K = int(p.K);
  const int64_t r = min(r0 + (lane & 31), p.n - 1);
  const int c = min(c0 + (lane & 31), p.M - 1);
  const T* ga = static_cast<const T*>(p.a) + r * p.lda;
  const T* gb = static_cast<const T*>(p.b) + int64_t(c) * p.ldb;
  constexpr int VO = 16 / WAVES;                          // results of a thread
  const int t = threadIdx.x * VO;
  const LinEnd<T, VO> end(p, c0 + t % 32);
  u32x4 raw = {0u, 0u, 0u, 0u};
  if constexpr (LinEnd<T, VO>::CHUNKS) raw = end.ahead(r0 + t / 32);
  f32x16_t acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = 0.f;
  if constexpr (SHORT) {
    if (wave == 0) lin_mma(T(), lin_load_short(gb, half ? 0 : K), lin_load_short(ga, half ? 0 : K), acc);
  } else {
    for (int k = wave * STEP + half * VE; k - half * VE < K; k += ROUND) {
      u32x4 fa[AHEAD], fb[AHEAD];
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) {
        const int at = min(k + s * WAVES * STEP, K - VE);
        fa[s] = lin_load(ga + at);
        fb[s] = lin_load(gb + at);
      }
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) {
        const int at = k + s * WAVES * STEP;
        if (at - half * VE + STEP > K) {                   // (the same for the whole wave)
          const u32x4 m = lin_mask<T>(at - min(at, K - VE));
          fa[s] &= m;
          fb[s] &= m;
        }
        lin_mma(T(), fb[s], fa[s], acc);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<f32x4*>(&buf[wave][(lane & 31) * LD + q * 8 + half * 4]) =
        f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  __syncthreads();
  float z[VO];
#pragma unroll
  for (int v = 0; v < VO; ++v) z[v] = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
#pragma unroll
    for (int v = 0; v < VO; ++v) z[v] += buf[w][t / 32 * LD + t % 32 + v];
  end.finish(r0 + t / 32, z, raw);
}

// A handful of rows (a request's, one token's): a wave per column takes w's row and up to R rows of x
// a chunk a lane, and adds up over its lanes.  K >= a chunk.  Bound by w's bytes,
// below them by the launch: one row past 2048 x 8192 weights in fp32 11 us, past 100 x 272 3.8.
template <typename T, int R>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_row(LinArgs p) {
  constexpr int VE = CHUNK<T>, AHEAD = 4, STEP = 64 * VE;
  const int lane = threadIdx.x & 63, c = int(blockIdx.x) * (LIN_THREADS / 64) + (threadIdx.x >> 6), K = int(p.K);
  const int64_t r0 = int64_t(blockIdx.y) * R;
  const T* w = static_cast<const T*>(p.b) + int64_t(min(c, p.M - 1)) * p.ldb;
  const T* x[R];
#pragma unroll
  for (int r = 0; r < R; ++r) x[r] = static_cast<const T*>(p.a) + min(r0 + r, p.n - 1) * p.lda;
  const LinEnd<T, 1> end(p, c);
  float sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) sum[r] = 0.f;
  auto add = [&](const u32x4& wv, const u32x4& xv, float& s) {
    float a[VE], b[VE];
    lin_unpack(T(), wv, a);
    lin_unpack(T(), xv, b);
#pragma unroll
    for (int j = 0; j < VE; ++j) s = fmaf(a[j], b[j], s);
  };
  for (int k0 = 0; k0 < K; k0 += AHEAD * STEP) {
    u32x4 wv[AHEAD], xv[R][AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int at = min(k0 + s * STEP + lane * VE, K - VE);
      wv[s] = lin_load(w + at);
#pragma unroll
      for (int r = 0; r < R; ++r) xv[r][s] = lin_load(x[r] + at);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int first = k0 + s * STEP, at = first + lane * VE;
      if (first + STEP > K) {                            // (the same for the whole wave)
        const u32x4 m = lin_mask<T>(at - min(at, K - VE));
        wv[s] &= m;
#pragma unroll
        for (int r = 0; r < R; ++r) xv[r][s] &= m;
      }
#pragma unroll
      for (int r = 0; r < R; ++r) add(wv[s], xv[r][s], sum[r]);
    }
  }
  float z = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float v = sum[r];
    v += dpp_quad_xor1(v);
    v += dpp_quad_xor2(v);
    v += dpp_row_half_mirror(v);
    v += dpp_row_mirror(v);
    v = sum_halves32(sum_rows16(v));
    z = lane == r ? v : z;
  }
  if (lane < R) end.finish(r0 + lane, &z);
}

// Many narrow bf16 rows: the weights stay in LDS, a wave holds 32 whole rows as the matrix unit's
// operand in registers, loads the next 32 while it multiplies the last columns, and waits for no
// other wave.  Columns lie in LDS in the order in which a lane's results are 8 neighbours of one
// row: 16 bytes to store, 64 a row and instruction (8 bytes, 16 a row: 95 us for 77 at 264000 rows of
// 272 x 256).  3.6 TB/s there, 5.1 at 100 x 64; 12 waves take 81 us, 16 spill.  STEPS: 32-element steps
// of k.  C = A B^T + bias.
constexpr int LS_WAVES = 8, LS_LDS = 156 * 1024, LS_STEPS = 9;
template <int STEPS>
__global__ void __launch_bounds__(64 * LS_WAVES) k_linear_stream(LinArgs p) {
  constexpr int ROW = STEPS * 64 + 16, C = STEPS * 4;
  __shared__ __attribute__((aligned(16))) char s_w[LS_LDS];    // [groups of 32][ROW], then the bias
  const int K = int(p.K), groups = (p.M + 31) / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15;
  const uint16_t* A = static_cast<const uint16_t*>(p.a);
  const uint16_t* B = static_cast<const uint16_t*>(p.b);
  float* s_bias = reinterpret_cast<float*>(s_w + groups * 32 * ROW);
  for (int t = threadIdx.x; t < groups * 32 * C; t += 64 * LS_WAVES) {
    const int m = t / C, c = t % C * 8, at = min(c, K - 8);
    const int slot = (m & ~31) | (m & 4) << 2 | (m & 24) >> 1 | (m & 3);
    u32x4 v = lin_load(B + int64_t(min(m, p.M - 1)) * p.ldb + at);
    if (c != at) v = c < K ? lin_shift(v, c - at) : u32x4{0u, 0u, 0u, 0u};
    *reinterpret_cast<u32x4*>(s_w + slot * ROW + c * 2) = v;
  }
  for (int t = threadIdx.x; t < groups * 32; t += 64 * LS_WAVES)
    s_bias[t] = p.bias && t < p.M ? p.bias[t] : 0.f;
  __syncthreads();
  const uint32_t wg = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t tiles = (p.n + 31) / 32, t0 = tiles * wg / gridDim.x, t1 = tiles * (wg + 1) / gridDim.x;
  u32x4 a[2][STEPS];
  auto load = [&](int64_t tile) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint16_t* x = A + min(tile * 32 + r * 16 + i, p.n - 1) * p.lda;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) a[r][s] = lin_load(x + min(s * 32 + g * 8, K - 8));
    }
  };
  // a chunk that passes K was loaded moved back to end there
  const int last = K / 8, skip = K % 8 ? 8 - K % 8 : 0;
  const char* wl = s_w + i * ROW + g * 16;
  int64_t tile = t0 + wave;
  if (tile < t1) load(tile);
  for (; tile < t1; tile += LS_WAVES) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = 4 * s + g;
      if (c >= last)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          a[r][s] = c == last && skip ? lin_shift(a[r][s], skip) : u32x4{0u, 0u, 0u, 0u};
    }
    for (int b = 0; b < groups; ++b) {
      f32x4_t acc[2][2];
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[q & 1][q >> 1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const char* w = wl + b * 32 * ROW;
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8_t wf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(w + h * 16 * ROW + s * 64));
#pragma unroll
          for (int r = 0; r < 2; ++r)
            acc[r][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, __builtin_bit_cast(bf16x8_t, a[r][s]), acc[r][h], 0, 0, 0);
        }
      if (b + 1 == groups && tile + LS_WAVES < t1) load(tile + LS_WAVES);
      const int c = b * 32 + g * 8, left = p.M - c;
      const f32x4 b0 = *reinterpret_cast<const f32x4*>(s_bias + c), b1 = *reinterpret_cast<const f32x4*>(s_bias + c + 4);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int64_t row = tile * 32 + r * 16 + i;
        if (row >= p.n) continue;
        uint16_t* y = static_cast<uint16_t*>(p.y) + row * p.ldy + c;
        const u32x4 v{bf16_pack(acc[r][0][0] + b0.x, acc[r][0][1] + b0.y), bf16_pack(acc[r][0][2] + b0.z, acc[r][0][3] + b0.w),
                      bf16_pack(acc[r][1][0] + b1.x, acc[r][1][1] + b1.y), bf16_pack(acc[r][1][2] + b1.z, acc[r][1][3] + b1.w)};
        if (left >= 8) {
          *reinterpret_cast<u32x4_e*>(y) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 7; ++e)
            if (e < left) y[e] = uint16_t(v[e >> 1] >> (16 * (e & 1)));
        }
      }
    }
  }
}

// ------------------------------------------------------------------ weight gradients
// Rows of A and B side by side in memory are k here: 64 rows of bf16 (32 of fp32) are read a
// few columns per thread, turned in registers and put into LDS as in k_linear.
template <typename T> struct LinTurn;
template <> struct LinTurn<uint16_t> {        // 2 columns of 8 rows
  static constexpr int COLS = 2, ROWS = 8;
  uint32_t w[8];
  // Of an odd width the last column is loaded with the one before; width 1: alone.
  uint32_t at;
  int shift;
  __device__ void place(int col, int width) {
    const int c = min(col, width - 1);
    shift = c + 1 < width || width == 1 ? 0 : 16;
    at = uint32_t(c - (shift ? 1 : 0));
  }
  // rows row, row + 1, ... of p; END: row `last` again from there on; ONE: width 1
  template <bool END, bool ONE>
  __device__ void load(const uint16_t* p, uint32_t ld, int row, int last) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t* q = END ? at_offset(p, at + uint32_t(min(row + j, last)) * ld) : at_offset(p + j * size_t(ld), at + row * ld);
      if constexpr (ONE) w[j] = *q;
      else w[j] = *reinterpret_cast<const u32_e*>(q);
    }
  }
  // rows past the end count nothing
  __device__ void trim(int64_t rows) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = j < rows ? w[j] >> shift : 0u;
  }
  template <int ROW>
  __device__ void put(char* o) const {
    u32x4 lo, hi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x05040100u);
      hi[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
    }
    *reinterpret_cast<u32x4*>(o) = lo;
    *reinterpret_cast<u32x4*>(o + ROW) = hi;
  }
  __device__ void add(float* s) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[0] += bf16_lo(w[j]);
      s[1] += bf16_hi(w[j]);
    }
  }
};
// p.a: dz [K, n] (n columns, lda apart), p.b: x [K, M]; PRODUCT: part[split][n][M]; sums (NULL for
// none): from the workgroups of the first tile of columns, sums[split][n] of dz's columns.
// ONE: n or M is 1.
template <typename T, typename Tile, bool PRODUCT, bool ONE>
__global__ void __launch_bounds__(Tile::THREADS) k_linear_wgrad(LinArgs p) {
  constexpr int TR = Tile::TR, TC = Tile::TC, BR = Tile::BR, BC = Tile::BC, BUF = Tile::BUF;
  constexpr int BK = Tile::KB / int(sizeof(T));
  typedef LinTurn<T> Turn;
    // an operand's tile: column groups, pieces per thread, chunks between a thread's pieces
  constexpr int GA = BR / Turn::COLS, NTA = GA * Tile::CHUNKS / Tile::THREADS, NEXTA = Tile::THREADS / GA;
  constexpr int GB = BC / Turn::COLS, NTB = GB * Tile::CHUNKS / Tile::THREADS, NEXTB = Tile::THREADS / GB;
  static_assert(NTA * NEXTA == Tile::CHUNKS && NTB * NEXTB == Tile::CHUNKS, "whole pieces");
  __shared__ __attribute__((aligned(16))) char lds[Tile::LDS];
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const uint32_t tiles_r = uint32_t((p.n + BR - 1) / BR), tiles = tiles_r * uint32_t(p.tiles_c);
  const uint32_t split = id / tiles, tile = id % tiles;
  const int r0 = int(tile / uint32_t(p.tiles_c)) * BR, c0 = int(tile % uint32_t(p.tiles_c)) * BC;
  const T* A = static_cast<const T*>(p.a);
  const T* B = static_cast<const T*>(p.b);
  const int64_t k0 = int64_t(split) * p.rows, k1 = min(k0 + p.rows, p.K);
  const int grpa = threadIdx.x % GA, firsta = threadIdx.x / GA, grpb = threadIdx.x % GB, firstb = threadIdx.x / GB;
  const bool sums = p.sums && c0 == 0;
  Turn ta[NTA], tb[NTB];
#pragma unroll
  for (int i = 0; i < NTA; ++i) ta[i].place(r0 + grpa * Turn::COLS, int(p.n));
  if (PRODUCT) {
#pragma unroll
    for (int i = 0; i < NTB; ++i) tb[i].place(c0 + grpb * Turn::COLS, p.M);
  }
  // END: the tile that the split ends in
  auto load = [&](int64_t k, auto end) {
    constexpr bool END = decltype(end)::value;
    const int last = int(k1 - 1 - k);
    const T* a = A + k * p.lda;
    const T* b = PRODUCT ? B + k * p.ldb : nullptr;
#pragma unroll
    for (int i = 0; i < NTA; ++i) {
      const int row = (firsta + i * NEXTA) * Turn::ROWS;
      if (ONE && p.n == 1) ta[i].template load<END, true>(a, uint32_t(p.lda), row, last);
      else ta[i].template load<END, false>(a, uint32_t(p.lda), row, last);
    }
    if constexpr (PRODUCT) {
#pragma unroll
      for (int i = 0; i < NTB; ++i) {
        const int row = (firstb + i * NEXTB) * Turn::ROWS;
        if (ONE && p.M == 1) tb[i].template load<END, true>(b, uint32_t(p.ldb), row, last);
        else tb[i].template load<END, false>(b, uint32_t(p.ldb), row, last);
      }
    }
  };
  double sum[Turn::COLS];                               // (a tile's in fp32)
#pragma unroll
  for (int j = 0; j < Turn::COLS; ++j) sum[j] = 0.0;
  const bool odd = sizeof(T) == 2 && ((p.n | p.M) & 1);  // a last column to be shifted into place
  auto put = [&](int64_t k, char* buf) {
    if (odd || k + BK > k1) {
#pragma unroll
      for (int i = 0; i < NTA; ++i) ta[i].trim(k1 - k - (firsta + i * NEXTA) * Turn::ROWS);
      if (PRODUCT) {
#pragma unroll
        for (int i = 0; i < NTB; ++i) tb[i].trim(k1 - k - (firstb + i * NEXTB) * Turn::ROWS);
      }
    }
    if (sums) {
      float s[Turn::COLS];
#pragma unroll
      for (int j = 0; j < Turn::COLS; ++j) s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < NTA; ++i) ta[i].add(s);
#pragma unroll
      for (int j = 0; j < Turn::COLS; ++j) sum[j] += s[j];
    }
    if constexpr (PRODUCT) {
#pragma unroll
      for (int i = 0; i < NTA; ++i)
        ta[i].template put<Tile::ROW>(buf + grpa * Turn::COLS * Tile::ROW + (firsta + i * NEXTA) * 16);
#pragma unroll
      for (int i = 0; i < NTB; ++i)
        tb[i].template put<Tile::ROW>(buf + (BR + grpb * Turn::COLS) * Tile::ROW + (firstb + i * NEXTB) * 16);
    }
  };
  f32x16_t acc[TR][TC];
#pragma unroll
  for (int i = 0; i < TR; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  const int wave = threadIdx.x >> 6, wr = wave / Tile::WC, wc = wave % Tile::WC;
  auto multiply = [&](const char* buf) {
    if constexpr (PRODUCT)
      lin_step<T, Tile>(buf + wr * TR * 32 * Tile::ROW, buf + (BR + wc * TC * 32) * Tile::ROW, acc);
  };
  typedef std::integral_constant<bool, false> Whole;
  typedef std::integral_constant<bool, true> End;
  const int64_t full = k1 > k0 ? (k1 - k0) / BK : 0;    // (a split past the end adds zeros)
  int64_t k = k0;
  int cur = 0;
  if (full > 0) {
    load(k, Whole());
    put(k, lds);
    __syncthreads();
    for (int64_t t = 0; t < full; ++t, k += BK) {
      const bool more = t + 1 < full;
      if (more) load(k + BK, Whole());
      multiply(lds + cur * BUF);
      cur ^= 1;
      if (more) put(k + BK, lds + cur * BUF);
      __syncthreads();
    }
  }
  if (k < k1) {
    load(k, End());
    put(k, lds + cur * BUF);
    __syncthreads();
    multiply(lds + cur * BUF);
    __syncthreads();
  }
  if constexpr (PRODUCT) {
    float* part = p.part + int64_t(split) * p.n * p.M;
    const int col = c0 + wc * TC * 32 + (threadIdx.x & 63) % (TC * 8) * 4;
    lin_out<4>(lds, acc, [](int) { return u32x4{0u, 0u, 0u, 0u}; }, [&](int r, float* z, u32x4) {
      const int64_t row = r0 + wr * TR * 32 + r;
      if (row < p.n && col < p.M) store_chunk_of(part + row * p.M + col, p.M - col, z);
    });
  }
  if (sums) {                                           // the threads of a column group, in order
    __syncthreads();
    double* s = reinterpret_cast<double*>(lds);
#pragma unroll
    for (int j = 0; j < Turn::COLS; ++j) s[firsta * BR + grpa * Turn::COLS + j] = sum[j];
    __syncthreads();
    for (int c = threadIdx.x; c < BR && r0 + c < p.n; c += Tile::THREADS) {
      double x = 0.0;
      for (int f = 0; f < NEXTA; ++f) x += s[f * BR + c];
      p.sums[int64_t(split) * p.n + r0 + c] = float(x);
    }
  }
}

// k_linear_wgrad of fp32 dz (and x of fp32 or bf16) in parts.
template <typename T> struct LinCols;           // 8 rows of LinCols::COLS columns
template <> struct LinCols<float> {
  static constexpr int COLS = 1;
  float w[8];
  uint32_t at;
  __device__ void place(int col, int width) { at = uint32_t(min(col, width - 1)); }
  template <bool END, bool ONE>
  __device__ void load(const float* p, uint32_t ld, int row, int last) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      w[j] = END ? *at_offset(p, at + uint32_t(min(row + j, last)) * ld) : *at_offset(p + j * size_t(ld), at + row * ld);
  }
  __device__ void trim(int64_t rows) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = j < rows ? w[j] : 0.f;
  }
  // (`rows`: of a part's tile)
  template <int ROW>
  __device__ void put(char* o, int rows, float& cut) const {
    const LinParts s = lin_split(w, cut);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4*>(o + q * rows * ROW) = s.p[q];
  }
};
template <> struct LinCols<uint16_t> : LinTurn<uint16_t> {
  template <int ROW>
  __device__ void put(char* o, int, float& cut) const {
    LinTurn<uint16_t>::template put<ROW>(o);
#pragma unroll
    for (int j = 0; j < 8; ++j) cut = fmaf(bf16_lo(w[j]), 0.f, fmaf(bf16_hi(w[j]), 0.f, cut));
  }
};
__device__ __forceinline__ float lin_value(float x) { return x; }
__device__ __forceinline__ float lin_value(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }

// As k_linear_wgrad; ONE: p.M is 1.
// Eight waves: 128 registers, so that two workgroups share a CU and one multiplies while the other cuts
// up (144 and one workgroup: 1150 us for 1050 at 40,000 rows of 2048 x 2048 bf16).  The bound spills 6 registers
// there (28 bytes of scratch a lane, bf16 rows).
template <typename T, typename Tile, bool PRODUCT, bool ONE>
__global__ void __launch_bounds__(Tile::THREADS, Tile::THREADS == 512 ? 4 : 1) k_linear_wgrad_parts(LinArgs p) {
  constexpr int TR = Tile::TR, TC = Tile::TC, BR = Tile::BR, BC = Tile::BC, ROW = Tile::ROW, PB = LIN_PARTS<T>;
  constexpr int BK = Tile::KB / 2;
  typedef LinCols<float> ColsA;
  typedef LinCols<T> ColsB;
  constexpr int GA = BR, NTA = GA * Tile::CHUNKS / Tile::THREADS, NEXTA = Tile::THREADS / GA;
  constexpr int GB = BC / ColsB::COLS, NTB = GB * Tile::CHUNKS / Tile::THREADS, NEXTB = Tile::THREADS / GB;
  static_assert(NTA * NEXTA == Tile::CHUNKS && NTB * NEXTB == Tile::CHUNKS, "whole pieces");
  constexpr int OUT = Tile::WR * Tile::WC * 32 * (TC * 32 + 4) * 4, BUF = (3 * BR + PB * BC) * ROW;
  __shared__ __attribute__((aligned(16))) char lds[PRODUCT ? (BUF > OUT ? BUF : OUT) : NEXTA * BR * 8];
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const uint32_t tiles_r = uint32_t((p.n + BR - 1) / BR), tiles = tiles_r * uint32_t(p.tiles_c);
  const uint32_t split = id / tiles, tile = id % tiles;
  const int r0 = int(tile / uint32_t(p.tiles_c)) * BR, c0 = int(tile % uint32_t(p.tiles_c)) * BC;
  const float* A = static_cast<const float*>(p.a);
  const T* B = static_cast<const T*>(p.b);
  const int64_t k0 = int64_t(split) * p.rows, k1 = min(k0 + p.rows, p.K);
  const int ga = threadIdx.x % GA, fa0 = threadIdx.x / GA, gb = threadIdx.x % GB, fb0 = threadIdx.x / GB;
  const bool sums = p.sums && c0 == 0;
  ColsA ta[NTA];
  ColsB tb[NTB];
#pragma unroll
  for (int i = 0; i < NTA; ++i) ta[i].place(r0 + ga, int(p.n));
#pragma unroll
  for (int i = 0; i < NTB; ++i) tb[i].place(c0 + gb * ColsB::COLS, PRODUCT ? p.M : 1);
  auto load = [&](int64_t k, auto end) {
    constexpr bool END = decltype(end)::value;
    const int last = int(k1 - 1 - k);
#pragma unroll
    for (int i = 0; i < NTA; ++i)
      ta[i].template load<END, false>(A + k * p.lda, uint32_t(p.lda), (fa0 + i * NEXTA) * 8, last);
    if constexpr (PRODUCT) {
#pragma unroll
      for (int i = 0; i < NTB; ++i)
        tb[i].template load<END, ONE>(B + k * p.ldb, uint32_t(p.ldb), (fb0 + i * NEXTB) * 8, last);
    }
  };
  float cut = 0.f;
  double sum = 0.0;                                     // (a tile's in fp32)
  const bool odd = sizeof(T) == 2 && (p.M & 1);
  auto put = [&](int64_t k) {
    if (k + BK > k1) {
#pragma unroll
      for (int i = 0; i < NTA; ++i) ta[i].trim(k1 - k - (fa0 + i * NEXTA) * 8);
    }
    if (PRODUCT && (odd || k + BK > k1)) {
#pragma unroll
      for (int i = 0; i < NTB; ++i) tb[i].trim(k1 - k - (fb0 + i * NEXTB) * 8);
    }
    if (sums) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NTA; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += ta[i].w[j];
      sum += s;
    }
    if constexpr (PRODUCT) {
#pragma unroll
      for (int i = 0; i < NTA; ++i) ta[i].template put<ROW>(lds + ga * ROW + (fa0 + i * NEXTA) * 16, BR, cut);
#pragma unroll
      for (int i = 0; i < NTB; ++i)
        tb[i].template put<ROW>(lds + (3 * BR + gb * ColsB::COLS) * ROW + (fb0 + i * NEXTB) * 16, BC, cut);
    }
  };
  f32x16_t acc[TR][TC];
  lin_clear(acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / Tile::WC, wc = wave % Tile::WC;
  auto multiply = [&] {
    if constexpr (PRODUCT)
      lin_step_parts<Tile, 3, PB>(lds + wr * TR * 32 * ROW, lds + (3 * BR + wc * TC * 32) * ROW, acc);
  };
  typedef std::integral_constant<bool, false> Whole;
  typedef std::integral_constant<bool, true> End;
  const int64_t full = k1 > k0 ? (k1 - k0) / BK : 0;
  int64_t k = k0;
  if (full > 0) load(k, Whole());
  for (int64_t t = 0; t < full; ++t, k += BK) {
    put(k);
    __syncthreads();
    if (t + 1 < full) load(k + BK, Whole());
    multiply();
    __syncthreads();
  }
  if (k < k1) {
    load(k, End());
    put(k);
    __syncthreads();
    multiply();
    __syncthreads();
  }
  if (PRODUCT && __syncthreads_or(cut != cut)) {          // not finite: from memory, in fp32
    lin_clear(acc);
    for (int64_t q = k0; q < k1; q += 8) {
      u32x4 fa[TR], fb[TC];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t r = q + (lane >> 5) * 4 + j, rr = min(r, k1 - 1);
#pragma unroll
        for (int i = 0; i < TR; ++i) {
          const float v = A[rr * p.lda + min(r0 + wr * TR * 32 + i * 32 + (lane & 31), int(p.n) - 1)];
          fa[i][j] = r < k1 ? __float_as_uint(v) : 0u;
        }
#pragma unroll
        for (int i = 0; i < TC; ++i) {
          const float v = lin_value(B[rr * p.ldb + min(c0 + wc * TC * 32 + i * 32 + (lane & 31), p.M - 1)]);
          fb[i][j] = r < k1 ? __float_as_uint(v) : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int j = 0; j < TC; ++j) lin_mma(float(), fb[j], fa[i], acc[i][j]);
    }
  }
  if constexpr (PRODUCT) {
    float* part = p.part + int64_t(split) * p.n * p.M;
    const int col = c0 + wc * TC * 32 + lane % (TC * 8) * 4;
    lin_out<4>(lds, acc, [](int) { return u32x4{0u, 0u, 0u, 0u}; }, [&](int r, float* z, u32x4) {
      const int64_t row = r0 + wr * TR * 32 + r;
      if (row < p.n && col < p.M) store_chunk_of(part + row * p.M + col, p.M - col, z);
    });
  }
  if (sums) {
    __syncthreads();
    double* s = reinterpret_cast<double*>(lds);
    s[fa0 * BR + ga] = sum;
    __syncthreads();
    for (int c = threadIdx.x; c < BR && r0 + c < p.n; c += Tile::THREADS) {
      double x = 0.0;
      for (int f = 0; f < NEXTA; ++f) x += s[f * BR + c];
      p.sums[int64_t(split) * p.n + r0 + c] = float(x);
    }
  }
}

// A value as two bf16 parts, each rounded to nearest: together within 2^-16 of it.  What the first would
// round to an infinity is cut off instead; an infinity and what is no number have no second part.
__device__ __forceinline__ void lin_two(float x, float& hi, float& lo) {
  const bool finite = fabsf(x) < INFINITY;
  hi = __uint_as_float(bf16_rne(x) << 16);
  if (finite && fabsf(hi) == INFINITY) hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  lo = finite ? x - hi : 0.f;
}

// dz = dy act'(pre) in fp32 (and, for dx of bf16 rows, in two bf16 parts side by side: rounded to one it would
// move dx by as much as dx's own rounding does; a slope of 0 or 1 leaves a bf16 number, one part) and its
// columns' sums: a workgroup takes DZ_ROWS rows and up to 256 chunks of columns, a thread one chunk
// of every `groups`-th row, DZ_AHEAD of them loaded together.  A row's last chunk starts early
// enough to end with it (both writers of an element write the same value; one counts it).
// SHORT: rows of less than a chunk.
constexpr int DZ_AHEAD = 4, DZ_ROWS = 64;
struct DzArgs {
  int64_t n, lddy;
  int M, act;
  int chunks, lanes;                                    // of a row; of them in a workgroup
  const void* dy;
  const void* pre;
  float* dz;                                            // NULL where only near is needed
  uint16_t* near;                                       // NULL: none
  int parts;                                            // of near: M of them in a row, or M and M
  float* sums;                                          // [row blocks][M], or NULL
};
template <typename T, bool SHORT>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_dz(DzArgs p) {
  constexpr int VE = CHUNK<T>;
  __shared__ float s[LIN_THREADS * VE];
  const int groups = LIN_THREADS / p.lanes, lane = threadIdx.x % p.lanes, g = threadIdx.x / p.lanes;
  const int chunk = blockIdx.y * p.lanes + lane;
  const bool in = g < groups && chunk < p.chunks;
  const int c = SHORT ? 0 : min(chunk * VE, p.M - VE), skip = SHORT ? 0 : chunk * VE - c, n = SHORT ? p.M : VE;
  const int64_t r0 = int64_t(blockIdx.x) * DZ_ROWS, r1 = min(r0 + DZ_ROWS, p.n);
  float sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.f;
  if (in) {
    const T* dy = static_cast<const T*>(p.dy) + r0 * p.lddy + c;
    const T* pre = static_cast<const T*>(p.pre) + r0 * p.M + c;
    const int64_t o0 = r0 * p.M + c;
    const int rows = int(r1 - r0);
    for (int r = g; r < rows; r += DZ_AHEAD * groups) {
      u32x4 d[DZ_AHEAD], z[DZ_AHEAD];
#pragma unroll
      for (int i = 0; i < DZ_AHEAD; ++i) {
        const int64_t q = min(r + i * groups, rows - 1);
        if constexpr (SHORT) {
          d[i] = lin_load_short(dy + q * p.lddy, n);
          z[i] = lin_load_short(pre + q * p.M, n);
        } else {
          d[i] = lin_load(dy + q * p.lddy);
          z[i] = lin_load(pre + q * p.M);
        }
      }
#pragma unroll
      for (int i = 0; i < DZ_AHEAD; ++i)
        if (r + i * groups < rows) {
          const int64_t o = o0 + int64_t(r + i * groups) * p.M;
          float x[VE], y[VE];
          lin_unpack(T(), d[i], x);
          lin_unpack(T(), z[i], y);
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            x[j] *= slope_of(p.act, y[j]);
            sum[j] += x[j];
          }
          if (p.dz) {
#pragma unroll
            for (int j = 0; j < VE; j += 4) store_chunk(p.dz + o + j, SHORT ? n - j : 4, x + j);
          }
          if constexpr (sizeof(T) == 2) {
            if (p.near && p.parts == 1) {
              store_chunk(p.near + o, n, x);
            } else if (p.near) {
              uint16_t* q = p.near + 2 * (o - c) + c;
#pragma unroll
              for (int j = 0; j < VE; ++j) lin_two(x[j], x[j], y[j]);
              store_chunk(q, n, x);
              store_chunk(q + p.M, n, y);
            }
          }
        }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int j = 0; j < VE; ++j) s[threadIdx.x * VE + j] = sum[j];
  __syncthreads();
  if (in && g == 0) {
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (j >= skip && j < n) {
        double x = 0.0;
        for (int q = 0; q < groups; ++q) x += s[(q * p.lanes + lane) * VE + j];
        p.sums[int64_t(blockIdx.x) * p.M + c + j] = float(x);
      }
  }
}

// out[i] = the sum over the parts in fp64, in an order of their own: a workgroup takes COLS elements, its
// THREADS / COLS groups every so many-th part.
template <int COLS, int THREADS>
__global__ void __launch_bounds__(THREADS) k_linear_join(const float* __restrict__ part, int64_t parts,
                                                             int64_t size, float* __restrict__ out) {
  constexpr int PARTS = THREADS / COLS;
  __shared__ double s[PARTS][COLS];
  const int col = threadIdx.x % COLS, q = threadIdx.x / COLS;
  const int64_t i = int64_t(blockIdx.x) * COLS + col;
  double t = 0.0;
  if (i < size) {
#pragma unroll 8
    for (int64_t b = q; b < parts; b += PARTS) t += part[b * size + i];
  }
  if constexpr (PARTS > 1) {
    s[q][col] = t;
    __syncthreads();
  }
  if (q == 0 && i < size) {
    for (int k = 1; k < PARTS; ++k) t += s[k][col];
    out[i] = float(t);
  }
}

// w [M, K] -> wt [K, ld], zeros behind its M columns; PARTS 2: its M columns twice, for dz in two parts.  In the
// second ones what is not finite is 0: the first part has carried it, and the second, of either sign or 0,
// would make it no number.
template <typename T, int PARTS>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_turn(const T* __restrict__ w, int M, int K, T* __restrict__ wt,
                                                             int ld) {
  __shared__ T s[32][33];
  const int k0 = blockIdx.x * 32, m0 = blockIdx.y * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
  for (int i = y; i < 32; i += 8) {
    const int c = m0 + i, m = PARTS == 2 && c >= M ? c - M : c;
    T v = m < M && k0 + x < K ? w[int64_t(m) * K + k0 + x] : T(0);
    if constexpr (PARTS == 2) {
      if (c >= M && (v & 0x7f80) == 0x7f80) v = T(0);
    }
    s[i][x] = v;
  }
  __syncthreads();
  for (int i = y; i < 32; i += 8)
    if (k0 + i < K && m0 + x < ld) wt[int64_t(k0 + i) * ld + m0 + x] = s[x][i];
}

// ------------------------------------------------------------------ host side
// Long products into wide rows take 256 x 128, which reads a quarter less from L2 than 128 x 128
// (40,000 x 2048 x 2048 bf16 485 against 548 us, 8192^3 1178 / 1697; the library 349 / 728;
// 256 x 256 leaves one workgroup per CU, whose epilogue nothing hides).  Otherwise more workgroups per
// CU count for more: 128 x 128.  Both at 40,000 rows, k x columns: 1024 x 1024 107 / 124, 2048 x 512 119 / 120,
// 1024 x 512 67 / 65, 2048 x 256 68 / 64, 512 x 512 42 / 41 (512 x 2048 126 / 139: left to 128 x 128); 16,384 rows
// (256 tiles of 256 x 256) 1024 x 1024 46 / 57; 8192 (128 of them) 2048 x 1024 53 / 49.
static bool lin_big(int64_t n, int M, int64_t K) {
  return K >= 1024 && M >= 512 && ((n + 255) / 256) * ((M + 255) / 256) >= 256;
}
constexpr int LS_GRID = 256;                // workgroups: one per CU
// The streaming kernel's rule: rows that a wave's registers and weights that LDS hold, and enough of
// them to pay for bringing the weights to every CU.  At 264000 rows, in x out, against 128 x 128 tiles:
// 272 x 256 77 us and 111, 256 x 256 74 and 80, 200 x 200 49 and 73, 100 x 64 17 and 31; at 16384 rows
// 12.6 and 12.2, 11.1 and 11.3, 100 x 64 6.6 and 6.9; at 4096 11.9 and 8.1.  As wide as LDS holds, 264000 rows: 64 x 960
// 145 and 189, 128 x 480 91 and 131; 16384: 20.5 and 18.2, 13.6 and 12.6.  LS_STEPS covers k <= 288; a step
// more would take 320 x 200 from 93 to 79, two 352 x 200 nowhere (117).
constexpr int64_t LS_ROWS = 16384;
static int ls_steps(int64_t K) { return K <= 64 ? 2 : K <= 128 ? 4 : K <= 192 ? 6 : int((K + 31) / 32); }
static bool ls_use(const LinArgs& a) {
  return a.act == FAST_ACT_NONE && !a.res && a.K >= 8 && a.K <= 32 * LS_STEPS && a.n >= LS_ROWS &&
         (a.M + 31) / 32 * 32 * (ls_steps(a.K) * 64 + 20) <= LS_LDS;
}
template <typename T, typename Tile>
static void lin_tiled(LinArgs& a, hipStream_t st) {
  a.tiles_c = (a.M + Tile::BC - 1) / Tile::BC;
  const dim3 grid(uint32_t((a.n + Tile::BR - 1) / Tile::BR * a.tiles_c));
  if constexpr (std::is_same<Tile, LinMid>::value) {
    if (a.K < CHUNK<T>) {
      hipLaunchKernelGGL((k_linear<T, Tile, true>), grid, dim3(Tile::THREADS), 0, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((k_linear<T, Tile, false>), grid, dim3(Tile::THREADS), 0, st, a);
}
// Tiles of 128 x 128 from as many of them on (columns counted in 32s); below, 32 x 32 a workgroup
// gives more workgroups and shorter walks.  Tiles against 32 x 32 at `tiles` x 256 columns, us: bf16,
// k = 64 / 1024, 64 tiles 7.3 and 7.7 / 18.6 and 21.7, 32 tiles 7.4 and 5.6 / 18.4 and 11.3; fp32 128
// tiles 13.5 and 14.0 / 69 and 82, 96 tiles 13.2 and 11.1 / 68 and 63.
template <typename T>
static bool lin_many(int64_t n, int M) {
  return n * ((M + 31) / 32 * 32) >= (sizeof(T) == 4 ? 128 : 64) * 16384;
}
// Products of fp32 rows in parts from this length on: 264,000 rows into 200 columns in parts against
// fp32 instructions, k = 200 252 us and 288, 100 183 / 187, 64 126 / 130, 48 119 / 109, 16 95 / 68.
constexpr int64_t LIN_PARTS_K = 64;
// A wave per column for a few rows, as long as waves are few for the bytes of a row: against 32 x 32 a
// workgroup, one row into 2048 columns fp32 k = 272 4.2 us and 5.6, 2048 3.7 / 14.1, 8192 11 / 49; bf16
// 1024 3.8 / 4.4, 8192 4.7 / 20; 16 rows bf16 1024 7.8 / 5.1, 2048 7.3 / 7.9; 32 rows into 256 fp32
// 272 3.9 / 5.7, bf16 512 4.1 / 4.4.
constexpr int64_t LR_ROWS = 32;
static bool lr_use(int64_t n, int M, int64_t bytes) {
  const int64_t waves = M * ((n + 3) / 4);
  return n <= LR_ROWS && bytes >= 1024 && waves <= std::min<int64_t>(3 * bytes, 8192);
}
template <typename T>
static void lin_product(LinArgs a, hipStream_t st) {
  if constexpr (sizeof(T) == 4) {
    if (lin_many<T>(a.n, a.M) && a.K >= LIN_PARTS_K) {
      a.tiles_c = (a.M + 127) / 128;
      hipLaunchKernelGGL((k_linear_parts<LinMid>), dim3(uint32_t((a.n + 127) / 128 * a.tiles_c)), dim3(LinMid::THREADS), 0, st, a);
      return;
    }
  }
  if constexpr (sizeof(T) == 2) {
    if (ls_use(a)) {
      const dim3 grid(LS_GRID), block(64 * LS_WAVES);
      const int steps = ls_steps(a.K);
      if (steps == 2) hipLaunchKernelGGL((k_linear_stream<2>), grid, block, 0, st, a);
      else if (steps == 4) hipLaunchKernelGGL((k_linear_stream<4>), grid, block, 0, st, a);
      else if (steps == 6) hipLaunchKernelGGL((k_linear_stream<6>), grid, block, 0, st, a);
      else if (steps == 7) hipLaunchKernelGGL((k_linear_stream<7>), grid, block, 0, st, a);
      else if (steps == 8) hipLaunchKernelGGL((k_linear_stream<8>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((k_linear_stream<9>), grid, block, 0, st, a);
      return;
    }
    if (lin_big(a.n, a.M, a.K)) {
      lin_tiled<T, LinBig>(a, st);
      return;
    }
  }
  if (lin_many<T>(a.n, a.M)) {
    lin_tiled<T, LinMid>(a, st);
    return;
  }
  if (lr_use(a.n, a.M, a.K * int64_t(sizeof(T)))) {
    const uint32_t cols = uint32_t((a.M + 3) / 4);
    if (a.n == 1) hipLaunchKernelGGL((k_linear_row<T, 1>), dim3(cols), dim3(LIN_THREADS), 0, st, a);
    else if (a.n == 2) hipLaunchKernelGGL((k_linear_row<T, 2>), dim3(cols), dim3(LIN_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_linear_row<T, 4>), dim3(cols, uint32_t((a.n + 3) / 4)), dim3(LIN_THREADS), 0, st, a);
    return;
  }
  // Waves that share k: 4 up to 1024 bytes of it, and where there are more workgroups than CUs; 8 otherwise.  4 / 8
  // waves into 256 columns, us: 504 workgroups, fp32 k = 256 6.6 / 8.1, 272 7.6 / 8.3, 384 8.7 / 11.9, 512 10.9 / 11.9,
  // 1024 21.2 / 21.4; 152, fp32 256 5.1 / 4.6, 272 5.4 / 4.8, 384 6.1 / 6.7, 512 6.9 / 6.4, 1024 10.4 / 10.1; 16, bf16
  // 272 3.7 / 3.4, 544 4.4 / 3.8, 768 5.4 / 6.0, 1024 6.2 / 5.9.
  a.tiles_c = (a.M + 31) / 32;
  const dim3 grid(uint32_t((a.n + 31) / 32 * a.tiles_c));
  if (a.K < CHUNK<T>) hipLaunchKernelGGL((k_linear_few<T, 4, true>), grid, dim3(256), 0, st, a);
  else if (a.K * int64_t(sizeof(T)) <= 1024 || grid.x > 256)
    hipLaunchKernelGGL((k_linear_few<T, 4, false>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_linear_few<T, 8, false>), grid, dim3(512), 0, st, a);
}
// Few elements: many groups share their parts (4125 parts of 200 13 us, with 256 threads 21); few parts: a
// thread takes all of an element's (4 of 2048 x 2048 19 us, 64-byte pieces 110).
constexpr int64_t LJ_MANY = 16384, LJ_PARTS = 16;
static void lin_join(const float* part, int64_t parts, int64_t size, float* out, hipStream_t st) {
  auto launch = [&](auto kernel, int cols, int threads) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t((size + cols - 1) / cols)), dim3(threads), 0, st, part, parts, size, out);
  };
  if (size < LJ_MANY) launch(k_linear_join<16, 1024>, 16, 1024);
  else if (parts > LJ_PARTS) launch(k_linear_join<64, 256>, 64, 256);
  else launch(k_linear_join<256, 256>, 256, 256);
}
// Workgroups of lin_product times its threads, at most
static bool lin_fits(int64_t n, int M) {
  return grid_fits((n + 127) / 128 * ((M + 127) / 128), LIN_THREADS);
}

struct LinPlan {
  int64_t rows;                      // k of a split
  int splits;
  bool parts, wide;                  // fp32 operands in parts; tiles of 128 x 256
  int64_t tiles;                     // of a split's result
  int64_t dz_blocks;
};
constexpr int64_t LIN_SPLIT_MAX = 16384;     // rows whose products are added in fp32, at most
static LinPlan lin_plan(int64_t n, int K, int M, fast_dtype_t dtype, fast_act_t act) {
  LinPlan p = {};
  const bool acts = act != FAST_ACT_NONE;
  p.parts = dtype == FAST_F32 || acts;
  p.dz_blocks = (n + DZ_ROWS - 1) / DZ_ROWS;
  // 128 x 256 / 128 x 128 at 40,000 rows, columns of x x of dz, us: 372 x 200 61 / 59, 512 x 512 120 / 120, 768 x 768
  // 224 / 236, 1024 x 1024 328 / 368
  p.wide = acts && dtype == FAST_BF16 && K >= 512;
  p.tiles = int64_t((M + 127) / 128) * (p.wide ? (K + 255) / 256 : (K + 127) / 128);
  // 512 workgroups, two a CU (256 / 512 / 1024, us: 264,000 rows 272 x 256 bf16 117 / 93 / 103, 372 x 200 fp32 391 / 304 /
  // 334; 40,000 rows 2048 x 2048 bf16 with silu 1234 / 1090 / 1124)
  int64_t s = std::max<int64_t>(1, 512 / p.tiles);
  s = std::min<int64_t>(s, (n + 255) / 256);
  s = std::max<int64_t>({s, (n + LIN_SPLIT_MAX - 1) / LIN_SPLIT_MAX, 1});
  p.rows = ((n + s - 1) / s + 63) / 64 * 64;
  p.splits = int(s);                 // (trailing ones may be empty)
  return p;
}

struct LinWork {
  char* wt;
  float* dz;
  uint16_t* near;
  float* part;
  float* sums;
};
// bf16 parts that dx reads dz in: with a slope other than 0 and 1 dz is no bf16 number
static int lin_dx_parts(fast_dtype_t dtype, fast_act_t act) {
  return dtype == FAST_BF16 && act != FAST_ACT_NONE && act != FAST_ACT_RELU ? 2 : 1;
}
static int lin_wt_ld(int M, int64_t es) { return int((M * es + 15) / 16 * 16 / es); }
static size_t lin_layout(int64_t n, int K, int M, fast_dtype_t dtype, fast_act_t act, char* ws, LinWork* w) {
  const LinPlan p = lin_plan(n, K, M, dtype, act);
  const int64_t es = elem_size(dtype);
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    char* q = ws ? ws + at : nullptr;
    at += align_up(size_t(bytes), 256);
    return q;
  };
  LinWork t;
  t.wt = take(int64_t(K) * lin_wt_ld(lin_dx_parts(dtype, act) * M, es) * es);
  const bool acts = act != FAST_ACT_NONE;
  t.dz = acts ? reinterpret_cast<float*>(take(n * M * 4)) : nullptr;
  t.near = acts && dtype == FAST_BF16 ? reinterpret_cast<uint16_t*>(take(lin_dx_parts(dtype, act) * n * M * 2)) : nullptr;
  t.part = reinterpret_cast<float*>(take(int64_t(p.splits) * M * K * 4));
  t.sums = reinterpret_cast<float*>(take((act != FAST_ACT_NONE ? p.dz_blocks : p.splits) * M * 4));
  if (w) *w = t;
  return at;
}

static fast_status_t lin_check(const char* fn, int64_t n, int K, int M, fast_dtype_t dtype, fast_act_t act) {
  if (n < 0) return fail(FAST_ERR_INVALID_ARG, "%s: n = %lld < 0", fn, (long long)n);
  if (K <= 0 || M <= 0) return fail(FAST_ERR_INVALID_ARG, "%s: in = %d, out = %d", fn, K, M);
  if (dtype != FAST_F32 && dtype != FAST_BF16) return fail(FAST_ERR_INVALID_ARG, "%s: bad dtype", fn);
  if (act != FAST_ACT_NONE && act != FAST_ACT_RELU && act != FAST_ACT_GELU && act != FAST_ACT_SILU)
    return fail(FAST_ERR_INVALID_ARG, "%s: bad activation", fn);
  if (K > LIN_MAX || M > LIN_MAX)
    return fail(FAST_ERR_UNSUPPORTED, "%s: in = %d or out = %d > %lld", fn, K, M, (long long)LIN_MAX);
  if (n >= (int64_t(1) << 31)) return fail(FAST_ERR_UNSUPPORTED, "%s: n >= 2^31", fn);
  return FAST_OK;
}
static fast_status_t lin_rows(const char* fn, const char* name, const void* p, int64_t n, int F, int64_t ld,
                              int64_t es) {
  if (ld < F) return fail(FAST_ERR_INVALID_ARG, "%s: %s: rows of %d elements, %lld apart", fn, name, F, (long long)ld);
  if (ld >= LIN_MAX_LD) return fail(FAST_ERR_UNSUPPORTED, "%s: %s: row stride >= 2^22", fn, name);
  if (n > 0 && !p) return fail(FAST_ERR_INVALID_ARG, "%s: NULL %s", fn, name);
  if (!aligned(p, es)) return fail(FAST_ERR_UNSUPPORTED, "%s: %s not %d-byte aligned", fn, name, int(es));
  return FAST_OK;
}

template <typename T>
static void lin_bwd(int64_t n, int K, int M, fast_dtype_t dtype, const void* x, int64_t ldx, const void* w,
                    fast_act_t act, const void* pre, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dw,
                    float* dbias, char* ws, hipStream_t st) {
  const LinPlan p = lin_plan(n, K, M, dtype, act);
  LinWork m;
  lin_layout(n, K, M, dtype, act, ws, &m);
  const bool acts = act != FAST_ACT_NONE;
  if (n > 0 && acts) {
    DzArgs d = {n, lddy, M, act, (M + CHUNK<T> - 1) / CHUNK<T>, 0, dy, pre, dw || sizeof(T) == 4 ? m.dz : nullptr,
                dx ? m.near : nullptr, lin_dx_parts(dtype, act), dbias ? m.sums : nullptr};
    d.lanes = std::min(d.chunks, LIN_THREADS);
    const dim3 grid(uint32_t(p.dz_blocks), uint32_t((d.chunks + d.lanes - 1) / d.lanes));
    if (M < CHUNK<T>) hipLaunchKernelGGL((k_linear_dz<T, true>), grid, dim3(LIN_THREADS), 0, st, d);
    else hipLaunchKernelGGL((k_linear_dz<T, false>), grid, dim3(LIN_THREADS), 0, st, d);
  }
  const int64_t lddz = acts ? M : lddy;
  if (dx && n > 0) {
    // dz in two parts is one product of twice the length, so all its kernels serve it
    const int parts = lin_dx_parts(dtype, act), ld = lin_wt_ld(parts * M, sizeof(T));
    const dim3 grid(uint32_t((K + 31) / 32), uint32_t((ld + 31) / 32));
    auto turn = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(LIN_THREADS), 0, st, static_cast<const T*>(w), M, K, reinterpret_cast<T*>(m.wt), ld);
    };
    if constexpr (sizeof(T) == 2) {
      if (parts == 2) turn(k_linear_turn<T, 2>);
    }
    if (parts == 1) turn(k_linear_turn<T, 1>);
    LinArgs a = {};
    a.a = !acts ? dy : (sizeof(T) == 4 ? static_cast<const void*>(m.dz) : m.near);
    a.lda = parts * lddz;
    a.b = m.wt;
    a.ldb = ld;
    a.n = n;
    a.M = K;
    a.K = parts * M;
    a.y = dx;
    a.ldy = lddx;
    lin_product<T>(a, st);
  }
  auto join = [&](const float* part, int64_t parts, int64_t size, float* out) {
    if (parts != 1) lin_join(part, parts, size, out, st);
  };
  const int64_t parts = n > 0 ? int64_t(p.splits) : 0;
  if (n > 0 && (dw || (dbias && !acts))) {
    LinArgs a = {};
    a.a = acts ? m.dz : dy;
    a.lda = lddz;
    a.b = x;
    a.ldb = ldx;
    a.n = M;
    a.M = dw ? K : 1;                                   // (dbias alone: one tile of columns)
    a.K = n;
    a.rows = p.rows;
    a.part = parts == 1 ? dw : m.part;
    a.sums = !dbias || acts ? nullptr : (parts == 1 ? dbias : m.sums);
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    auto launch = [&](auto tile, auto product, auto one) {
      typedef decltype(tile) Tile;
      constexpr bool PRODUCT = decltype(product)::value, ONE = decltype(one)::value;
      a.tiles_c = (a.M + Tile::BC - 1) / Tile::BC;
      const dim3 grid(uint32_t(parts * ((M + Tile::BR - 1) / Tile::BR) * a.tiles_c));
      if constexpr (std::is_same<Tile, LinGrad>::value)
        hipLaunchKernelGGL((k_linear_wgrad<uint16_t, Tile, PRODUCT, ONE>), grid, dim3(Tile::THREADS), 0, st, a);
      else
        hipLaunchKernelGGL((k_linear_wgrad_parts<T, Tile, PRODUCT, ONE>), grid, dim3(Tile::THREADS), 0, st, a);
    };
    if constexpr (sizeof(T) == 4) {
      if (dw) launch(LinMid(), yes, no);
      else launch(LinMid(), no, no);
    } else if (acts) {
      if (p.wide) launch(LinWide(), yes, no);
      else if (K > 1) launch(LinMid(), yes, no);
      else launch(LinMid(), yes, yes);
    } else {
      if (dw && M > 1 && K > 1) launch(LinGrad(), yes, no);
      else if (dw) launch(LinGrad(), yes, yes);
      else if (M > 1) launch(LinGrad(), no, no);
      else launch(LinGrad(), no, yes);
    }
  }
  if (dw) join(m.part, parts, int64_t(M) * K, dw);
  if (dbias && acts) {                                  // a part per block of rows
    lin_join(m.sums, p.dz_blocks, M, dbias, st);
  } else if (dbias) {
    join(m.sums, parts, M, dbias);
  }
}

}  // namespace fast

using namespace fast;

extern "C" fast_status_t fast_linear_fwd(int64_t n, int in, int out, fast_dtype_t dtype, const void* x, int64_t ldx,
                                         const void* w, const float* bias, fast_act_t act, const void* res,
                                         int64_t ldres, void* y, int64_t ldy, void* pre, fast_stream_t stream) {
  const char* fn = "fast_linear_fwd";
  fast_status_t s = lin_check(fn, n, in, out, dtype, act);
  if (s != FAST_OK) return s;
  const int64_t es = elem_size(dtype);
  if (pre && act == FAST_ACT_NONE) return fail(FAST_ERR_INVALID_ARG, "%s: pre without an activation", fn);
  if ((s = lin_rows(fn, "x", x, n, in, ldx, es)) != FAST_OK) return s;
  if ((s = lin_rows(fn, "y", y, n, out, ldy, es)) != FAST_OK) return s;
  if (res && (s = lin_rows(fn, "res", res, n, out, ldres, es)) != FAST_OK) return s;
  if (n == 0) return ok();
  if (!w) return fail(FAST_ERR_INVALID_ARG, "%s: NULL w", fn);
  if (!aligned(w, es) || !aligned(pre, es)) return fail(FAST_ERR_UNSUPPORTED, "%s: w/pre not %d-byte aligned", fn, int(es));
  if (!aligned(bias, 4)) return fail(FAST_ERR_UNSUPPORTED, "%s: bias not 4-byte aligned", fn);
  if (!lin_fits(n, out)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  const int64_t sx = span(n, in, ldx, es), sr = span(n, out, ldres, es), sy = span(n, out, ldy, es),
                sw = int64_t(in) * out * es, sp = n * out * es;
  if (meet(y, sy, x, sx) || meet(y, sy, w, sw) || meet(y, sy, bias, 4 * int64_t(out)) ||
      (meet(y, sy, res, sr) && !(y == res && ldy == ldres)))
    return fail(FAST_ERR_INVALID_ARG, "%s: y overlaps an input", fn);
  if (meet(pre, sp, x, sx) || meet(pre, sp, w, sw) || meet(pre, sp, bias, 4 * int64_t(out)) || meet(pre, sp, res, sr) ||
      meet(pre, sp, y, sy))
    return fail(FAST_ERR_INVALID_ARG, "%s: pre overlaps another array", fn);
  LinArgs a = {};
  a.a = x;
  a.lda = ldx;
  a.b = w;
  a.ldb = in;
  a.n = n;
  a.M = out;
  a.K = in;
  a.bias = bias;
  a.act = act;
  a.res = res;
  a.ldres = ldres;
  a.y = y;
  a.ldy = ldy;
  a.pre = pre;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32) lin_product<float>(a, st);
  else lin_product<uint16_t>(a, st);
  return check_launch(fn);
}

extern "C" size_t fast_linear_bwd_workspace(int64_t n, int in, int out, fast_dtype_t dtype, fast_act_t act) {
  if (n < 0 || n >= (int64_t(1) << 31) || in <= 0 || out <= 0 || in > LIN_MAX || out > LIN_MAX) return 0;
  if (dtype != FAST_F32 && dtype != FAST_BF16) return 0;
  return lin_layout(n, in, out, dtype, act, nullptr, nullptr);
}

extern "C" fast_status_t fast_linear_bwd(int64_t n, int in, int out, fast_dtype_t dtype, const void* x, int64_t ldx,
                                         const void* w, fast_act_t act, const void* pre, const void* dy, int64_t lddy,
                                         void* dx, int64_t lddx, float* dw, float* dbias, void* ws, size_t ws_bytes,
                                         fast_stream_t stream) {
  const char* fn = "fast_linear_bwd";
  fast_status_t s = lin_check(fn, n, in, out, dtype, act);
  if (s != FAST_OK) return s;
  const int64_t es = elem_size(dtype);
  if ((pre != nullptr) != (act != FAST_ACT_NONE) && (n > 0 || pre))
    return fail(FAST_ERR_INVALID_ARG, "%s: pre goes with an activation", fn);
  if ((s = lin_rows(fn, "dy", dy, n, out, lddy, es)) != FAST_OK) return s;
  if (dw && (s = lin_rows(fn, "x", x, n, in, ldx, es)) != FAST_OK) return s;
  if (dx && (s = lin_rows(fn, "dx", dx, n, in, lddx, es)) != FAST_OK) return s;
  if (!dx && !dw && !dbias) return ok();
  if (dx && n > 0 && !w) return fail(FAST_ERR_INVALID_ARG, "%s: NULL w", fn);
  if (!aligned(w, es) || !aligned(pre, es)) return fail(FAST_ERR_UNSUPPORTED, "%s: w/pre not %d-byte aligned", fn, int(es));
  if (!aligned(dw, 4) || !aligned(dbias, 4)) return fail(FAST_ERR_UNSUPPORTED, "%s: dw/dbias not 4-byte aligned", fn);
  const size_t need = fast_linear_bwd_workspace(n, in, out, dtype, act);
  if (!ws || ws_bytes < need)
    return fail(FAST_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws ? ws_bytes : 0, need);
  if (!aligned(ws, 256)) return fail(FAST_ERR_UNSUPPORTED, "%s: workspace not 256-byte aligned", fn);
  const LinPlan plan = lin_plan(n, in, out, dtype, act);
  if (!lin_fits(n, in) || !grid_fits((int64_t(in) * out + 63) / 64, LIN_THREADS) ||
      (act != FAST_ACT_NONE && !grid_fits(plan.dz_blocks, LIN_THREADS)) ||
      ((dw || dbias) && !grid_fits(plan.splits * plan.tiles, plan.wide ? LinWide::THREADS : LIN_THREADS)))
    return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
  const int64_t sw = int64_t(in) * out;
  const struct { const void* p; int64_t n; } reads[] = {{dw ? x : nullptr, span(n, in, ldx, es)},
                                                        {dx ? w : nullptr, sw * es},
                                                        {pre, n * out * es},
                                                        {dy, span(n, out, lddy, es)}},
                                             writes[] = {{dx, dx ? span(n, in, lddx, es) : 0},
                                                         {dw, 4 * sw}, {dbias, 4 * int64_t(out)}};
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < 4; ++j)
      if (meet(writes[i].p, writes[i].n, reads[j].p, reads[j].n))
        return fail(FAST_ERR_INVALID_ARG, "%s: dx, dw or dbias overlaps an input", fn);
    for (int j = 0; j < i; ++j)
      if (meet(writes[i].p, writes[i].n, writes[j].p, writes[j].n))
        return fail(FAST_ERR_INVALID_ARG, "%s: dx, dw and dbias overlap", fn);
    if (meet(ws, int64_t(need), writes[i].p, writes[i].n))
      return fail(FAST_ERR_INVALID_ARG, "%s: the workspace overlaps dx, dw or dbias", fn);
  }
  for (int j = 0; j < 4; ++j)
    if (meet(ws, int64_t(need), reads[j].p, reads[j].n))
      return fail(FAST_ERR_INVALID_ARG, "%s: the workspace overlaps an input", fn);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32)
    lin_bwd<float>(n, in, out, dtype, x, ldx, w, act, pre, dy, lddy, dx, lddx, dw, dbias, static_cast<char*>(ws), st);
  else
    lin_bwd<uint16_t>(n, in, out, dtype, x, ldx, w, act, pre, dy, lddy, dx, lddx, dw, dbias, static_cast<char*>(ws), st);
  return check_launch(fn);
}
