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
// hundred columns on.
#include <algorithm>

#include "rows.h"

namespace fast {

constexpr int64_t LIN_MAX = 16384;        // columns
constexpr int LIN_THREADS = 256;
constexpr int LIN_KB = 128;               // bytes of k in a tile
constexpr int LIN_ROW = LIN_KB + 16;      // LDS row: 16 lanes' chunks fall into different banks

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
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

// 16 bytes at p, of which n elements are in the row (zeros past them)
template <typename T>
__device__ __forceinline__ u32x4 lin_load(const T* p, int64_t n) {
  if (n >= CHUNK<T>) {
    const u32x4_e w = *reinterpret_cast<const u32x4_e*>(p);
    return u32x4{w.x, w.y, w.z, w.w};
  }
  u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < CHUNK<T>; ++j)
    if (j < n) {
      if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(p[j]);
      else w[j / 2] |= uint32_t(p[j]) << (16 * (j & 1));
    }
  return w;
}

// ------------------------------------------------------------------ activations
__device__ __forceinline__ float act_of(int act, float z) {
  if (act == FAST_ACT_RELU) return z > 0.f ? z : (z == z ? 0.f : z);
  if (act == FAST_ACT_GELU) return 0.5f * z * erfcf(z * -0x1.6a09e6p-1f);
  if (act == FAST_ACT_SILU) return z / (1.f + expf(-z));
  return z;
}
__device__ __forceinline__ float slope_of(int act, float z) {
  if (act == FAST_ACT_RELU) return z > 0.f ? 1.f : (z == z ? 0.f : z);
  if (act == FAST_ACT_GELU)
    return fmaf(0.5f, erfcf(z * -0x1.6a09e6p-1f), z * expf(-0.5f * z * z) * 0x1.988454p-2f);
  if (act == FAST_ACT_SILU) {
    const float p = 1.f / (1.f + expf(-z));
    return p * fmaf(z, 1.f - p, 1.f);
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
  int splits;                        // of one operand a; the same number behind them reads a2
  const void* a2;
  float* part;
};

// The epilogue of VE neighbouring columns from c on of row r.
template <typename T, int VE>
__device__ __forceinline__ void lin_finish(const LinArgs& p, int64_t r, int c, float* z) {
  const int n = p.M - c;
  if (r >= p.n || n <= 0) return;
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (j < n) z[j] += p.bias[c + j];
  }
  T* pre = p.pre ? static_cast<T*>(p.pre) + r * p.M + c : nullptr;
  const T* res = p.res ? static_cast<const T*>(p.res) + r * p.ldres + c : nullptr;
  T* y = static_cast<T*>(p.y) + r * p.ldy + c;
  if constexpr (VE == CHUNK<T>) {
    if (pre) store_chunk(pre, n, z);
#pragma unroll
    for (int j = 0; j < VE; ++j) z[j] = act_of(p.act, z[j]);
    if (res) {
      float t[VE];
      load_chunk(res, n, t);
#pragma unroll
      for (int j = 0; j < VE; ++j) z[j] += t[j];
    }
    store_chunk(y, n, z);
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (j < n) {
        float t;
        if (pre) VecIO<T, 1>::store(pre + j, &z[j]);
        z[j] = act_of(p.act, z[j]);
        if (res) {
          VecIO<T, 1>::load(res + j, &t);
          z[j] += t;
        }
        VecIO<T, 1>::store(y + j, &z[j]);
      }
  }
}

// A wave's part of a tile: TR x TC blocks of 32 x 32 over a tile of k in LDS.
template <typename T, int TR, int TC>
__device__ __forceinline__ void lin_step(const char* la, const char* lb, f32x16_t (&acc)[TR][TC]) {
  const int lane = threadIdx.x & 63;
  la += (lane & 31) * LIN_ROW + (lane >> 5) * 16;
  lb += (lane & 31) * LIN_ROW + (lane >> 5) * 16;
#pragma unroll
  for (int k = 0; k < LIN_KB; k += 32) {
    u32x4 fa[TR], fb[TC];
#pragma unroll
    for (int i = 0; i < TR; ++i) fa[i] = *reinterpret_cast<const u32x4*>(la + i * 32 * LIN_ROW + k);
#pragma unroll
    for (int j = 0; j < TC; ++j) fb[j] = *reinterpret_cast<const u32x4*>(lb + j * 32 * LIN_ROW + k);
#pragma unroll
    for (int i = 0; i < TR; ++i)
#pragma unroll
      for (int j = 0; j < TC; ++j) lin_mma(T(), fb[j], fa[i], acc[i][j]);
  }
}

// The wave's block through LDS, 32 rows at a time, so that rows leave in whole chunks.
// out(row of the wave's block, column, values).
template <int VE, int TR, int TC, typename F>
__device__ __forceinline__ void lin_out(char* lds, const f32x16_t (&acc)[TR][TC], F out) {
  constexpr int W = TC * 32, LD = W + 4, PER = W / VE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* buf = reinterpret_cast<float*>(lds) + wave * 32 * LD;
#pragma unroll
  for (int i = 0; i < TR; ++i) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(buf + (lane & 31) * LD + j * 32 + q * 8 + (lane >> 5) * 4) =
            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
#pragma unroll
    for (int t = lane; t < 32 * PER; t += 64) {
      const int r = t / PER, c = t % PER * VE;
      float z[VE];
#pragma unroll
      for (int v = 0; v < VE; v += 4) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(buf + r * LD + c + v);
        z[v] = w.x; z[v + 1] = w.y; z[v + 2] = w.z; z[v + 3] = w.w;
      }
      out(i * 32 + r, c, z);
    }
  }
}

// Tiles of BR rows and BC columns, four waves of 2 x 2; the next tile of k is on its way
// into registers while this one is multiplied from LDS.
template <typename T, int TR, int TC>
__global__ void __launch_bounds__(LIN_THREADS) k_linear(LinArgs p) {
  constexpr int BR = TR * 64, BC = TC * 64, VE = CHUNK<T>, BK = LIN_KB / int(sizeof(T));
  constexpr int NA = BR / 32, NB = BC / 32, BUF = (BR + BC) * LIN_ROW;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUF];
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t r0 = int64_t(id / uint32_t(p.tiles_c)) * BR;
  const int c0 = int(id % uint32_t(p.tiles_c)) * BC;
  const int row = threadIdx.x >> 3, chunk = threadIdx.x & 7;
  const T* ga[NA];
  const T* gb[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int64_t r = r0 + i * 32 + row;
    ga[i] = static_cast<const T*>(p.a) + (r < p.n ? r : p.n - 1) * p.lda + chunk * VE;
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int c = c0 + i * 32 + row;
    gb[i] = static_cast<const T*>(p.b) + int64_t(c < p.M ? c : p.M - 1) * p.ldb + chunk * VE;
  }
  u32x4 ra[NA], rb[NB];
  auto load = [&](int64_t k) {
    if (k + BK <= p.K) {
#pragma unroll
      for (int i = 0; i < NA; ++i) ra[i] = lin_load(ga[i] + k, VE);
#pragma unroll
      for (int i = 0; i < NB; ++i) rb[i] = lin_load(gb[i] + k, VE);
    } else {
      const int64_t left = p.K - k - chunk * VE;
#pragma unroll
      for (int i = 0; i < NA; ++i) ra[i] = lin_load(ga[i] + k, left);
#pragma unroll
      for (int i = 0; i < NB; ++i) rb[i] = lin_load(gb[i] + k, left);
    }
  };
  auto put = [&](char* buf) {
    char* at = buf + row * LIN_ROW + chunk * 16;
#pragma unroll
    for (int i = 0; i < NA; ++i) *reinterpret_cast<u32x4*>(at + i * 32 * LIN_ROW) = ra[i];
#pragma unroll
    for (int i = 0; i < NB; ++i) *reinterpret_cast<u32x4*>(at + (BR + i * 32) * LIN_ROW) = rb[i];
  };
  f32x16_t acc[TR][TC];
#pragma unroll
  for (int i = 0; i < TR; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  const int wave = threadIdx.x >> 6, wr = wave >> 1, wc = wave & 1;
  load(0);
  put(lds);
  __syncthreads();
  int cur = 0;
  for (int64_t k = 0; k < p.K; k += BK) {
    const bool more = k + BK < p.K;
    if (more) load(k + BK);
    const char* buf = lds + cur * BUF;
    lin_step<T, TR, TC>(buf + wr * TR * 32 * LIN_ROW, buf + (BR + wc * TC * 32) * LIN_ROW, acc);
    cur ^= 1;
    if (more) put(lds + cur * BUF);
    __syncthreads();
  }
  lin_out<VE>(lds, acc, [&](int r, int c, float* z) {
    lin_finish<T, VE>(p, r0 + wr * TR * 32 + r, c0 + wc * TC * 32 + c, z);
  });
}

// Few rows: 32 x 32 results a workgroup, its waves share k, each feeding the matrix unit from
// global memory; their sums are added in order in LDS.
template <typename T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) k_linear_few(LinArgs p) {
  constexpr int VE = CHUNK<T>, STEP = 2 * VE, LD = 36, AHEAD = 4;
  __shared__ float buf[WAVES][32 * LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r0 = int64_t(blockIdx.x / uint32_t(p.tiles_c)) * 32;
  const int c0 = int(blockIdx.x % uint32_t(p.tiles_c)) * 32;
  const int64_t r = min(r0 + (lane & 31), p.n - 1);
  const int c = min(c0 + (lane & 31), p.M - 1);
  const T* ga = static_cast<const T*>(p.a) + r * p.lda + (lane >> 5) * VE;
  const T* gb = static_cast<const T*>(p.b) + int64_t(c) * p.ldb + (lane >> 5) * VE;
  f32x16_t acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = 0.f;
  for (int64_t k = int64_t(wave) * STEP; k < p.K; k += int64_t(AHEAD) * WAVES * STEP) {
    u32x4 fa[AHEAD], fb[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int64_t at = k + int64_t(s) * WAVES * STEP, left = p.K - at - (lane >> 5) * VE;
      fa[s] = lin_load(ga + at, left);
      fb[s] = lin_load(gb + at, left);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) lin_mma(T(), fb[s], fa[s], acc);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *reinterpret_cast<f32x4*>(&buf[wave][(lane & 31) * LD + q * 8 + (lane >> 5) * 4]) =
        f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  __syncthreads();
  constexpr int VO = 16 / WAVES;
  const int t = threadIdx.x * VO;
  float z[VO];
#pragma unroll
  for (int v = 0; v < VO; ++v) z[v] = 0.f;
  for (int w = 0; w < WAVES; ++w)
#pragma unroll
    for (int v = 0; v < VO; ++v) z[v] += buf[w][t / 32 * LD + t % 32 + v];
  lin_finish<T, VO>(p, r0 + t / 32, c0 + t % 32, z);
}

// ------------------------------------------------------------------ weight gradients
// Rows of A and B side by side in memory are k here: 64 rows of bf16 (32 of fp32) are read a
// few columns per thread, turned in registers and put into LDS as in k_linear.
template <typename T> struct LinTurn;
template <> struct LinTurn<uint16_t> {        // 2 columns of 8 rows
  static constexpr int COLS = 2, ROWS = 8;
  uint32_t w[8];
  __device__ void load(const uint16_t* p, int64_t ld, bool pair, int64_t rows) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = 0u;
      if (j < rows) w[j] = pair ? *reinterpret_cast<const u32_e*>(p + j * ld) : uint32_t(p[j * ld]);
    }
  }
  __device__ void put(char* at) const {
    u32x4 lo, hi;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x05040100u);
      hi[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
    }
    *reinterpret_cast<u32x4*>(at) = lo;
    *reinterpret_cast<u32x4*>(at + LIN_ROW) = hi;
  }
};
template <> struct LinTurn<float> {           // a column of 4 rows
  static constexpr int COLS = 1, ROWS = 4;
  uint32_t w[4];
  __device__ void load(const float* p, int64_t ld, bool, int64_t rows) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = j < rows ? __float_as_uint(p[j * ld]) : 0u;
  }
  __device__ void put(char* at) const { *reinterpret_cast<u32x4*>(at) = u32x4{w[0], w[1], w[2], w[3]}; }
};

// p.a: dz [K, n] (n columns, lda apart), p.b: x [K, M]; part[split][n][M].
template <typename T>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_wgrad(LinArgs p) {
  constexpr int TR = 2, TC = 2, BR = TR * 64, BC = TC * 64, BK = LIN_KB / int(sizeof(T));
  typedef LinTurn<T> Turn;
  constexpr int GRP = BR / Turn::COLS;                  // column groups of an operand's tile
  constexpr int NT = GRP * 8 / LIN_THREADS;             // pieces per thread and operand
  constexpr int BUF = (BR + BC) * LIN_ROW;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUF];
  const uint32_t id = xcd_tile(blockIdx.x, gridDim.x);
  const uint32_t tiles_r = uint32_t((p.n + BR - 1) / BR), tiles = tiles_r * uint32_t(p.tiles_c);
  const uint32_t split = id / tiles, tile = id % tiles;
  const int r0 = int(tile / uint32_t(p.tiles_c)) * BR, c0 = int(tile % uint32_t(p.tiles_c)) * BC;
  const bool second = split >= uint32_t(p.splits);
  const T* A = static_cast<const T*>(second ? p.a2 : p.a);
  const T* B = static_cast<const T*>(p.b);
  const int64_t k0 = int64_t(second ? split - p.splits : split) * p.rows, k1 = min(k0 + p.rows, p.K);
  const int grp = threadIdx.x % GRP, first = threadIdx.x / GRP;
  constexpr int NEXT = LIN_THREADS / GRP;               // chunks between a thread's pieces
  const int width = int(p.n);
  const int ca = min(r0 + grp * Turn::COLS, width - 1), cb = min(c0 + grp * Turn::COLS, p.M - 1);
  const bool pa = ca + 1 < width, pb = cb + 1 < p.M;
  Turn ta[NT], tb[NT];
  auto load = [&](int64_t k) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int64_t at = k + (first + i * NEXT) * Turn::ROWS;
      ta[i].load(A + at * p.lda + ca, p.lda, pa, k1 - at);
      tb[i].load(B + at * p.ldb + cb, p.ldb, pb, k1 - at);
    }
  };
  auto put = [&](char* buf) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      char* at = buf + grp * Turn::COLS * LIN_ROW + (first + i * NEXT) * 16;
      ta[i].put(at);
      tb[i].put(at + BR * LIN_ROW);
    }
  };
  f32x16_t acc[TR][TC];
#pragma unroll
  for (int i = 0; i < TR; ++i)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  const int wave = threadIdx.x >> 6, wr = wave >> 1, wc = wave & 1;
  load(k0);
  put(lds);
  __syncthreads();
  int cur = 0;
  for (int64_t k = k0; k < k1; k += BK) {
    const bool more = k + BK < k1;
    if (more) load(k + BK);
    const char* buf = lds + cur * BUF;
    lin_step<T, TR, TC>(buf + wr * TR * 32 * LIN_ROW, buf + (BR + wc * TC * 32) * LIN_ROW, acc);
    cur ^= 1;
    if (more) put(lds + cur * BUF);
    __syncthreads();
  }
  float* part = p.part + int64_t(split) * p.n * p.M;
  lin_out<4>(lds, acc, [&](int r, int c, float* z) {
    const int64_t row = r0 + wr * TR * 32 + r;
    const int col = c0 + wc * TC * 32 + c;
    if (row < p.n && col < p.M) store_chunk_of(part + row * p.M + col, p.M - col, z);
  });
}

// dz = dy act'(pre) (bf16: the nearest value and what is left, 16 bits of it together),
// and the sums of its columns over the workgroup's rows.
constexpr int DZ_ROWS = 256, DZ_COLS = 64;             // rows and 16-byte chunks of a workgroup
struct DzArgs {
  int64_t n, lddy;
  int M, act;
  const void* dy;
  const void* pre;
  void* dz;
  void* rest;
  float* sums;                                          // [row blocks][M], or NULL
};
template <typename T>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_dz(DzArgs p) {
  constexpr int VE = CHUNK<T>, WAVES = LIN_THREADS / 64;
  __shared__ float s[WAVES][DZ_COLS * VE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = (blockIdx.y * DZ_COLS + lane) * VE, n = p.M - c;
  const int64_t r0 = int64_t(blockIdx.x) * DZ_ROWS, r1 = min(r0 + DZ_ROWS, p.n);
  float sum[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) sum[j] = 0.f;
  if (n > 0) {
#pragma unroll 4
    for (int64_t r = r0 + wave; r < r1; r += WAVES) {
      float d[VE];
      load_chunk(static_cast<const T*>(p.dy) + r * p.lddy + c, n, d);
      if (p.act != FAST_ACT_NONE) {
        float z[VE], t[VE];
        load_chunk(static_cast<const T*>(p.pre) + r * p.M + c, n, z);
#pragma unroll
        for (int j = 0; j < VE; ++j) d[j] *= slope_of(p.act, z[j]);
        store_chunk(static_cast<T*>(p.dz) + r * p.M + c, n, d);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int j = 0; j < VE; ++j) {
            const float near = __uint_as_float(bf16_rne(d[j]) << 16);
            t[j] = fabsf(near) < INFINITY ? d[j] - near : 0.f;
          }
          store_chunk(static_cast<T*>(p.rest) + r * p.M + c, n, t);
        }
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) sum[j] += d[j];
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int j = 0; j < VE; ++j) s[wave][lane * VE + j] = sum[j];
  __syncthreads();
  for (int t = threadIdx.x; t < DZ_COLS * VE; t += LIN_THREADS) {
    const int col = blockIdx.y * DZ_COLS * VE + t;
    if (col < p.M) {
      double x = 0.0;
      for (int w = 0; w < WAVES; ++w) x += s[w][t];
      p.sums[int64_t(blockIdx.x) * p.M + col] = float(x);
    }
  }
}

// out[i] = the sum over the parts, in order, in fp64: 64 threads per 16 elements.
constexpr int LJ_COLS = 16, LJ_PARTS = LIN_THREADS / LJ_COLS;
__global__ void __launch_bounds__(LIN_THREADS) k_linear_join(const float* __restrict__ part, int64_t parts,
                                                             int64_t size, float* __restrict__ out) {
  __shared__ double s[LJ_PARTS][LJ_COLS];
  const int col = threadIdx.x % LJ_COLS, q = threadIdx.x / LJ_COLS;
  const int64_t i = int64_t(blockIdx.x) * LJ_COLS + col;
  double t = 0.0;
  if (i < size) {
#pragma unroll 4
    for (int64_t b = q; b < parts; b += LJ_PARTS) t += part[b * size + i];
  }
  s[q][col] = t;
  __syncthreads();
  if (q == 0 && i < size) {
    for (int k = 1; k < LJ_PARTS; ++k) t += s[k][col];
    out[i] = float(t);
  }
}

// w [M, K] -> wt [K, ld], its columns from M on zeros
template <typename T>
__global__ void __launch_bounds__(LIN_THREADS) k_linear_turn(const T* __restrict__ w, int M, int K, T* __restrict__ wt,
                                                             int ld) {
  __shared__ T s[32][33];
  const int k0 = blockIdx.x * 32, m0 = blockIdx.y * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
  for (int i = y; i < 32; i += 8) s[i][x] = m0 + i < M && k0 + x < K ? w[int64_t(m0 + i) * K + k0 + x] : T(0);
  __syncthreads();
  for (int i = y; i < 32; i += 8)
    if (k0 + i < K && m0 + x < ld) wt[int64_t(k0 + i) * ld + m0 + x] = s[x][i];
}

// ------------------------------------------------------------------ host side
template <typename T>
static void lin_product(LinArgs a, hipStream_t st) {
  const int64_t tr = (a.n + 127) / 128, tc = (a.M + 127) / 128;
  if (tr * tc >= 256) {
    a.tiles_c = int(tc);
    hipLaunchKernelGGL((k_linear<T, 2, 2>), dim3(uint32_t(tr * tc)), dim3(LIN_THREADS), 0, st, a);
    return;
  }
  a.tiles_c = (a.M + 31) / 32;
  const dim3 grid(uint32_t((a.n + 31) / 32 * a.tiles_c));
  if (a.K * int64_t(sizeof(T)) <= 1024) hipLaunchKernelGGL((k_linear_few<T, 4>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_linear_few<T, 16>), grid, dim3(1024), 0, st, a);
}
// Workgroups of lin_product times its threads, at most
static bool lin_fits(int64_t n, int M) {
  return grid_fits((n + 127) / 128 * ((M + 127) / 128), LIN_THREADS);
}

struct LinPlan {
  int64_t rows;                      // k of a split
  int splits, planes;
  int64_t dz_blocks;
};
constexpr int64_t LIN_SPLIT_MAX = 16384;     // rows whose products are added in fp32, at most
static LinPlan lin_plan(int64_t n, int K, int M, fast_dtype_t dtype, fast_act_t act) {
  LinPlan p = {};
  const int64_t tiles = int64_t((M + 127) / 128) * ((K + 127) / 128);
  int64_t s = std::max<int64_t>(1, 512 / tiles);
  s = std::min<int64_t>(s, (n + 255) / 256);
  s = std::max<int64_t>({s, (n + LIN_SPLIT_MAX - 1) / LIN_SPLIT_MAX, 1});
  p.rows = ((n + s - 1) / s + 63) / 64 * 64;
  p.splits = int(s);                 // (trailing ones may be empty)
  p.planes = dtype == FAST_BF16 && act != FAST_ACT_NONE ? 2 : 1;
  p.dz_blocks = (n + DZ_ROWS - 1) / DZ_ROWS;
  return p;
}

struct LinWork {
  char* wt;
  char* dz;
  char* rest;
  float* part;
  float* sums;
};
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
  t.wt = take(int64_t(K) * lin_wt_ld(M, es) * es);
  t.dz = act != FAST_ACT_NONE ? take(n * M * es) : nullptr;
  t.rest = p.planes == 2 ? take(n * M * es) : nullptr;
  t.part = reinterpret_cast<float*>(take(int64_t(p.splits) * p.planes * M * K * 4));
  t.sums = reinterpret_cast<float*>(take(p.dz_blocks * M * 4));
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
  if (ld >= (int64_t(1) << 31)) return fail(FAST_ERR_UNSUPPORTED, "%s: %s: row stride >= 2^31", fn, name);
  if (n * ld >= (int64_t(1) << 56))
    return fail(FAST_ERR_UNSUPPORTED, "%s: %s: %lld rows, %lld elements apart", fn, name, (long long)n, (long long)ld);
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
  if (n > 0 && (dbias || acts)) {
    const DzArgs d = {n, lddy, M, act, dy, pre, m.dz, m.rest, dbias ? m.sums : nullptr};
    const int per = DZ_COLS * CHUNK<T>;
    hipLaunchKernelGGL(k_linear_dz<T>, dim3(uint32_t(p.dz_blocks), uint32_t((M + per - 1) / per)), dim3(LIN_THREADS), 0,
                       st, d);
  }
  if (dbias)
    hipLaunchKernelGGL(k_linear_join, dim3(uint32_t((M + LJ_COLS - 1) / LJ_COLS)), dim3(LIN_THREADS), 0, st, m.sums,
                       p.dz_blocks, int64_t(M), dbias);
  const void* dz = acts ? m.dz : dy;
  const int64_t lddz = acts ? M : lddy;
  if (dx && n > 0) {
    const int ld = lin_wt_ld(M, sizeof(T));
    hipLaunchKernelGGL(k_linear_turn<T>, dim3(uint32_t((K + 31) / 32), uint32_t((ld + 31) / 32)), dim3(LIN_THREADS), 0,
                       st, static_cast<const T*>(w), M, K, reinterpret_cast<T*>(m.wt), ld);
    LinArgs a = {};
    a.a = dz;
    a.lda = lddz;
    a.b = m.wt;
    a.ldb = ld;
    a.n = n;
    a.M = K;
    a.K = M;
    a.y = dx;
    a.ldy = lddx;
    lin_product<T>(a, st);
  }
  if (dw) {
    LinArgs a = {};
    a.a = dz;
    a.a2 = m.rest;
    a.lda = lddz;
    a.b = x;
    a.ldb = ldx;
    a.n = M;
    a.M = K;
    a.K = n;
    a.rows = p.rows;
    a.splits = p.splits;
    a.tiles_c = (K + 127) / 128;
    const int64_t parts = n > 0 ? int64_t(p.splits) * p.planes : 0;
    a.part = parts == 1 ? dw : m.part;
    if (parts > 0)
      hipLaunchKernelGGL(k_linear_wgrad<T>, dim3(uint32_t(parts * ((M + 127) / 128) * a.tiles_c)), dim3(LIN_THREADS),
                         0, st, a);
    if (parts != 1) {
      const int64_t size = int64_t(M) * K;
      hipLaunchKernelGGL(k_linear_join, dim3(uint32_t((size + LJ_COLS - 1) / LJ_COLS)), dim3(LIN_THREADS), 0, st, m.part,
                         parts, size, dw);
    }
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
  if (!lin_fits(n, in) || !grid_fits((int64_t(in) * out + LJ_COLS - 1) / LJ_COLS, LIN_THREADS)) return fail(FAST_ERR_UNSUPPORTED, "%s: 2^32 threads or more", fn);
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
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == FAST_F32)
    lin_bwd<float>(n, in, out, dtype, x, ldx, w, act, pre, dy, lddy, dx, lddx, dw, dbias, static_cast<char*>(ws), st);
  else
    lin_bwd<uint16_t>(n, in, out, dtype, x, ldx, w, act, pre, dy, lddy, dx, lddx, dw, dbias, static_cast<char*>(ws), st);
  return check_launch(fn);
}
