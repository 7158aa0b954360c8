// Rows kept in 4 bits (OCP's MXFP4) and their product: blocks of 32 columns of a row share a power of two.
//
//   a = max |x| over the block, e = the least whole number with a <= 7 * 2^e, held within [-120, 125]
//   q = the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 to |x| / 2^e (of two as near the one whose code is even), with x's sign;  the value is then q * 2^e
//
// A value is off by at most half the distance of its neighbours, 2^e in the largest binade.  (7 instead of 6 as the border: what lies between is as
// near to 6 as a value can be to 5, and a whole block keeps one more bit.)  The factor is kept as the byte e + 127; 255 is a block with an
// infinity or a NaN among its values, all of which is NaN.
//
// Products are those of exactly the stored values: two codes multiply to at most 7 bits, the matrix cores add them up in fp32 with their blocks' factors.
#include <hip/hip_runtime.h>
#include "guard.h"

#include <algorithm>
#include <string>

#include "../../include/gnnstage.h"
#include "common.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// rows start anywhere: the memory system takes vectors at any address of their elements
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef bf16_t bf16x8_u __attribute__((ext_vector_type(8), aligned(2)));
typedef uint32_t u32x4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_u __attribute__((aligned(1)));

typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Eight columns c .. c + 7 of a row, zeros from d on (the row's last eight are loaded where it ends: one vector load for every thread): their largest magnitude as the bits of a float (infinities and NaNs are above every number), and
// their codes of x / 2^e, two an instruction, rounded to the nearest, to the even of two as near.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float *row, int c, int d) {
    if (d < 8) {
#pragma unroll
      for (int t = 0; t < 8; ++t) v[t] = c + t < d ? row[c + t] : 0.f;
      return;
    }
    const int at = min(c, d - 8);
    const f32x4_u x = *reinterpret_cast<const f32x4_u *>(row + at), y = *reinterpret_cast<const f32x4_u *>(row + at + 4);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v[t] = x[t];
      v[4 + t] = y[t];
    }
  }
  // moves what was loaded from further to the left, where the row ends, to its place
  __device__ __forceinline__ void settle(int c, int d) {
    const int n = c - (d - 8);
    if (d < 8 || n <= 0) return;
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = n & 1 ? (t < 7 ? v[t + (t < 7)] : 0.f) : v[t];
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = n & 2 ? (t < 6 ? v[t + 2 * (t < 6)] : 0.f) : v[t];
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = n & 4 ? (t < 4 ? v[t + 4 * (t < 4)] : 0.f) : v[t];
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = n >= 8 ? 0.f : v[t];
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t a = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) a = max(a, __builtin_bit_cast(uint32_t, v[t]) & 0x7fffffffu);
    return a;
  }
  __device__ __forceinline__ uint32_t codes(float factor) const {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], factor, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], factor, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], factor, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], factor, 3);
  }
};
template <>
struct Eight<bf16_t> {
  uint32_t v[4];
  __device__ __forceinline__ void load(const bf16_t *row, int c, int d) {
    if (d < 8) {
      const uint16_t *x = reinterpret_cast<const uint16_t *>(row);
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = (c + 2 * t < d ? (uint32_t)x[c + 2 * t] : 0u) | (c + 2 * t + 1 < d ? (uint32_t)x[c + 2 * t + 1] << 16 : 0u);
      return;
    }
    const u32x4_u x = *reinterpret_cast<const u32x4_u *>(row + min(c, d - 8));
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = x[t];
  }
  __device__ __forceinline__ void settle(int c, int d) {
    const int n = c - (d - 8);
    if (d < 8 || n <= 0) return;
    const uint32_t half = n & 1 ? 16 : 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = __builtin_amdgcn_alignbit(t < 3 ? v[t + (t < 3)] : 0u, v[t], half);
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = n & 2 ? (t < 3 ? v[t + (t < 3)] : 0u) : v[t];
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = n & 4 ? (t < 2 ? v[t + 2 * (t < 2)] : 0u) : v[t];
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = n >= 8 ? 0u : v[t];
  }
  __device__ __forceinline__ uint32_t largest() const {
    u16x2 a = {0, 0};
#pragma unroll
    for (int t = 0; t < 4; ++t) a = __builtin_elementwise_max(a, __builtin_bit_cast(u16x2, v[t] & 0x7fff7fffu));
    return (uint32_t)max(a[0], a[1]) << 16;
  }
  __device__ __forceinline__ uint32_t codes(float factor) const {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v[0]), factor, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v[1]), factor, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v[2]), factor, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v[3]), factor, 3);
  }
};

// The byte of the factor of a block whose largest magnitude has the bits a; 255: not finite
__device__ __forceinline__ uint32_t byte_of(uint32_t a) {
  // a = f 2^(E - 127) <= 7 2^e = 1.75 2^(2 + e): e = E - 129 up to f = 1.75, one more beyond
  const int e = min(max((int)(a >> 23) - 129 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), -120), 125);
  return a >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
}
__device__ __forceinline__ float factor_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }  // 255: infinity

// Where a thread works: `across` threads (a row's, 256 of them at most) side by side, the rows below one another.  magic: thread / across as a product.
struct Grid {
  uint32_t across, down, magic;
};
Grid grid_of(int per_row) {
  Grid g;
  g.across = (uint32_t)std::min(per_row, 256);
  g.down = 256 / g.across;
  g.magic = 65536 / g.across + 1;  // (exact below 256)
  return g;
}

// A thread per eight columns of kStoreRows rows, whose loads are on their way together; four neighbouring lanes per block (quads never straddle rows: a row has
// whole blocks).
constexpr int kStoreRows = 4;  // 700,001 x 100 bf16, 187 MB: one row 57 us, four 38 (4.9 TB/s)
template <typename T>
__global__ __launch_bounds__(256) void rows4_store_kernel(const T *x, int64_t ld, int64_t rows, int d, int per_row, Grid at, uint8_t *q, int64_t ld_q, uint8_t *scale,
                                                          int64_t ld_s) {
  const uint32_t y = threadIdx.x * at.magic >> 16;
  const int64_t r0 = (int64_t)blockIdx.x * at.down * kStoreRows + y;
  const int g = (int)(blockIdx.y * 256 + threadIdx.x - y * at.across);
  if (y >= at.down || r0 >= rows || g >= per_row) return;  // whole quads
  Eight<T> v[kStoreRows];
#pragma unroll
  for (int i = 0; i < kStoreRows; ++i) v[i].load(x + (size_t)(min(r0 + i * at.down, rows - 1) * ld), g * 8, d);
#pragma unroll
  for (int i = 0; i < kStoreRows; ++i) {
    const int64_t r = r0 + i * at.down;
    v[i].settle(g * 8, d);
    uint32_t a = v[i].largest();
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2 of the quad
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
    if (r >= rows) break;  // whole quads
    const uint32_t byte = byte_of(a);
    *reinterpret_cast<uint32_t *>(q + (size_t)(r * ld_q) + g * 4) = byte == 255 ? 0u : v[i].codes(factor_of(byte));
    if ((g & 3) == 0) scale[(size_t)(r * ld_s) + (g >> 2)] = (uint8_t)byte;
  }
}

// The columns of x (d x rows) as rows: a thread per block, 64 columns and four blocks down a workgroup.  256 x 100,003 fp32 25 us (4.7 TB/s), bf16 29 us (2.3 TB/s: an instruction's loads are 128
// bytes of a row); 256 x 400,009 106 and 97 us.
template <typename T>
__global__ __launch_bounds__(256) void rows4_store_columns_kernel(const T *x, int64_t ld, int64_t rows, int d, int blocks, uint8_t *q, int64_t ld_q, uint8_t *scale,
                                                                  int64_t ld_s) {
  const int64_t r = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int block = (int)blockIdx.y * 4 + (threadIdx.x >> 6);
  if (r >= rows || block >= blocks) return;
  Eight<float> v[4];
  uint32_t a = 0;
#pragma unroll
  for (int t = 0; t < 32; ++t) {
    const int k = block * 32 + t;
    v[t >> 3].v[t & 7] = k < d ? (float)x[(size_t)(k * ld) + r] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) a = max(a, v[i].largest());
  const uint32_t byte = byte_of(a);
  const float factor = factor_of(byte);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = byte == 255 ? 0u : v[i].codes(factor);
  *reinterpret_cast<u32x4 *>(q + (size_t)(r * ld_q) + block * 16) = w;
  scale[(size_t)(r * ld_s) + block] = (uint8_t)byte;
}

// A thread per eight columns.  Bound by memory: 700,001 x 100 to bf16, 187 MB in 31 us, 6.0 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void rows4_load_kernel(const uint8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, int64_t rows, int d, int per_row, Grid at,
                                                         T *x, int64_t ld) {
  const uint32_t y = threadIdx.x * at.magic >> 16;
  const int64_t r = (int64_t)blockIdx.x * at.down + y;
  const int g = (int)(blockIdx.y * 256 + threadIdx.x - y * at.across), c = g * 8;
  if (y >= at.down || r >= rows || g >= per_row) return;
  const uint32_t w = *reinterpret_cast<const uint32_t *>(q + (size_t)(r * ld_q) + g * 4);
  const uint32_t byte = scale[(size_t)(r * ld_s) + (g >> 2)];
  const float f = byte == 255 ? NAN : factor_of(byte);
  T *row = x + (size_t)(r * ld) + c;
  const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 1), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 2),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, f, 3)};
  if (c + 8 <= d) {
    if constexpr (sizeof(T) == 2) {
      bf16x8_u o;
#pragma unroll
      for (int t = 0; t < 8; ++t) o[t] = (bf16_t)v[t >> 1][t & 1];
      *reinterpret_cast<bf16x8_u *>(row) = o;
    } else {
      f32x4_u lo, hi;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        lo[t] = v[t >> 1][t & 1];
        hi[t] = v[2 + (t >> 1)][t & 1];
      }
      *reinterpret_cast<f32x4_u *>(row) = lo;
      *reinterpret_cast<f32x4_u *>(row + 4) = hi;
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (c + t < d) row[t] = (T)v[t >> 1][t & 1];
  }
}
// launch(first row, rows, workgroups down, workgroups across) for as many rows as a launch takes
template <typename F>
int for_grid_slabs(int64_t rows, int per_row, int64_t down, F launch) {
  const int64_t gy = (per_row + 255) / 256, most = kMostBlocks / gy * down;
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t m = std::min(most, rows - r);
    launch(r, m, dim3((unsigned)((m + down - 1) / down), (unsigned)gy));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
  }
  return hipSuccess;
}

// ---- the product ----------------------------------------------------------------------------------------------------
struct ProductArgs {
  const uint8_t *a, *a_scale, *b, *b_scale;
  int64_t ld_a, ld_as, ld_b, ld_bs;
  int64_t M, N;
  int32_t blocks;     // of 32 columns
  const float *bias;  // by column of the result, or NULL
  void *out;
  int64_t ld_out;
  int32_t per;         // tiles of 32 rows a wave
  int32_t side;        // waves of a workgroup side by side, all or one; the others are below one another
  uint32_t split_cols, xcd_cols, xcd_rows;  // an XCD's workgroups, and whether XCDs have columns of their own or rows
};
// Operands of a row: 256 columns at a time, eight blocks.  Matrix instructions take 64 columns, 32 from each half of the wave; here the lower half has the blocks
// 0 .. 3, the upper one 4 .. 7, one per instruction: a lane's are 64 bytes side by side, and their factors one word, a byte for each instruction.
struct Operand {
  u32x4 q[4];
  uint32_t scale;
  __device__ __forceinline__ void load(const uint8_t *row, const uint8_t *scales, int block, int blocks) {
    const int left = blocks - block;
    if (left >= 4) {
#pragma unroll
      for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const u32x4 *>(row + (size_t)(block + s) * 16);
      scale = *reinterpret_cast<const u32_u *>(scales + block);
    } else {
      scale = 0x7f7f7f7fu;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        q[s] = u32x4{0, 0, 0, 0};
        if (s < left) {
          q[s] = *reinterpret_cast<const u32x4 *>(row + (size_t)(block + s) * 16);
          scale = (scale & ~(0xffu << (8 * s))) | (uint32_t)scales[block + s] << (8 * s);
        }
      }
    }
  }
  __device__ __forceinline__ i32x8 operator()(int s) const { return i32x8{(int)q[s][0], (int)q[s][1], (int)q[s][2], (int)q[s][3], 0, 0, 0, 0}; }
};
template <int S>
__device__ __forceinline__ f32x16 multiply(const Operand &a, const Operand &b, f32x16 c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a(S), b(S), c, 4, 4, S, (int)a.scale, S, (int)b.scale);  // 4: e2m1
}

// A wave owns 32 kAcross columns and goes down `per` tiles of 32 rows.  A lane's columns are side by side (column kAcross l + t is the t-th instruction's l-th), so that
// rows are written 256 (fp32: 512) bytes at a time from the registers.  Register i of lane l: row 8 (i / 4) + 4 (l / 32) + i % 4.
// Bound by the results' writes: 8,191 x 100,003 x 256 to bf16 365 us, 4.5 TB/s (rows of 200,006 bytes: two workgroups share a line; at whole lines 5.4 - 5.9), matrix cores 0.2 of
// the time; 3 x 400,009 x 256 by the other operands, 54 MB in 15.5 us: 784 workgroups, 512 of which are there at a time.  Beyond 256 columns operands are loaded for every tile when it needs
// them: 8,191 x 100,003 x 512 1,340 us, x 602 1,640.
// ONE: up to 256 columns of operands, those of the wave's columns stay in registers and the next rows' are on their way.
constexpr int kAcross = 4;
constexpr int kGroup = 4;  // waves of a workgroup (2 / 4 / 8: 441 / 371 / 399 - 476 us)
template <typename O, bool ONE>
__global__ __launch_bounds__(64 * kGroup, 2) void rows4_product_kernel(const ProductArgs p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31, h = lane >> 5;
  // An XCD has a share of the columns (or rows) and goes through it along the rows: what is side by side in memory is written at about the same time, so
  // that the lines that two workgroups share are whole when they leave the L2, and the columns' operands stay there.
  const uint32_t xcd = blockIdx.x & 7, local = blockIdx.x >> 3, lr = local / p.xcd_cols, lc = local - lr * p.xcd_cols;
  const uint32_t gc = p.split_cols ? xcd * p.xcd_cols + lc : lc, gr = p.split_cols ? lr : xcd * p.xcd_rows + lr;
  const int64_t col_tile = (int64_t)gc * p.side + wave % p.side, tile0 = ((int64_t)gr * (kGroup / p.side) + wave / p.side) * p.per;
  const int64_t n0 = col_tile * (32 * kAcross), tile1 = min(tile0 + p.per, (p.M + 31) / 32);
  if (n0 >= p.N || tile0 >= tile1) return;
  // (past the last row or column: that one once more, whatever it gives is not written)
  auto load_a = [&](Operand &x, int64_t tile, int block) {
    const int64_t m = min(tile * 32 + l, p.M - 1);
    x.load(p.a + (size_t)(m * p.ld_a), p.a_scale + (size_t)(m * p.ld_as), block + 4 * h, p.blocks);
  };
  auto load_b = [&](Operand (&x)[kAcross], int block) {
#pragma unroll
    for (int t = 0; t < kAcross; ++t) {
      const int64_t n = min(n0 + kAcross * l + t, p.N - 1);
      x[t].load(p.b + (size_t)(n * p.ld_b), p.b_scale + (size_t)(n * p.ld_bs), block + 4 * h, p.blocks);
    }
  };
  Operand b[kAcross], a, next;
  if constexpr (ONE) {
    load_a(next, tile0, 0);
    load_b(b, 0);
  }
  const int64_t n = n0 + kAcross * l;
  const bool whole = n + kAcross <= p.N;
  float bias[kAcross];
#pragma unroll
  for (int t = 0; t < kAcross; ++t) bias[t] = p.bias && n + t < p.N ? p.bias[n + t] : 0.f;
  for (int64_t tile = tile0; tile < tile1; ++tile) {
    // (waves side by side have the same tiles, and stay in step: 391 -> 371 us at 8,191 x 100,003 x 256)
    if (p.side == kGroup) __builtin_amdgcn_s_barrier();
    f32x16 sum[kAcross];
#pragma unroll
    for (int t = 0; t < kAcross; ++t)
#pragma unroll
      for (int k = 0; k < 16; ++k) sum[t][k] = 0.f;
    if constexpr (ONE) {
      a = next;
      if (tile + 1 < tile1) load_a(next, tile + 1, 0);
#pragma unroll
      for (int t = 0; t < kAcross; ++t) sum[t] = multiply<3>(a, b[t], multiply<2>(a, b[t], multiply<1>(a, b[t], multiply<0>(a, b[t], sum[t]))));
    } else {
      for (int block = 0; block < p.blocks; block += 8) {
        load_a(a, tile, block);
        load_b(b, block);
#pragma unroll
        for (int t = 0; t < kAcross; ++t) sum[t] = multiply<3>(a, b[t], multiply<2>(a, b[t], multiply<1>(a, b[t], multiply<0>(a, b[t], sum[t]))));
      }
    }
    const int64_t m0 = tile * 32 + 4 * h;
    O *row = static_cast<O *>(p.out) + (size_t)(m0 * p.ld_out) + n;
    const bool all = tile * 32 + 32 <= p.M;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int down = 8 * (k >> 2) + (k & 3);
      if (!all && m0 + down >= p.M) continue;
      O *out = row + (size_t)(down * p.ld_out);
      if (whole) {
        typedef O vector __attribute__((ext_vector_type(kAcross), aligned(sizeof(O))));
        vector v;
#pragma unroll
        for (int t = 0; t < kAcross; ++t) v[t] = (O)(sum[t][k] + bias[t]);
        *reinterpret_cast<vector *>(out) = v;
      } else {
#pragma unroll
        for (int t = 0; t < kAcross; ++t)
          if (n + t < p.N) out[t] = (O)(sum[t][k] + bias[t]);
      }
    }
  }
}

bool sizes_ok(int64_t rows, int d, std::string &err) {
  if (rows < 0 || rows > ((int64_t)1 << 40)) { err = "rows must not be negative (nor beyond 2^40)"; return false; }
  if (d < 1 || d > 65536) { err = "a width must be in [1, 65536]"; return false; }
  return true;
}
bool stored_ok(const void *q, int64_t ld_q, const void *scale, int64_t ld_s, int d, std::string &err) {
  if (!q || !scale) { err = "q and scale must not be NULL"; return false; }
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || ld_q % 16 != 0) { err = "q must be 16-byte aligned, its leading dimension a multiple of 16"; return false; }
  if (ld_q < round_up(d, 32) / 2 || ld_s < (d + 31) / 32) { err = "q rows need 16 bytes per 32 columns, scale rows a byte"; return false; }
  return true;
}
bool matrix_ok(const void *x, int dtype, std::string &err) {
  if (!x) { err = "a matrix must not be NULL"; return false; }
  if (reinterpret_cast<uintptr_t>(x) & (dtype == GNNSTAGE_BF16 ? 1u : 3u)) { err = "a matrix is not aligned to its elements"; return false; }
  return true;
}

template <typename T>
int run_store(const T *x, int64_t ld, int64_t rows, int d, bool columns, uint8_t *q, int64_t ld_q, uint8_t *scale, int64_t ld_s, hipStream_t s) {
  const int blocks = (d + 31) / 32;
  const Grid at = grid_of(blocks * 4);
  if (!columns)
    return for_grid_slabs(rows, blocks * 4, at.down * kStoreRows, [&](int64_t r, int64_t m, dim3 groups) {
      hipLaunchKernelGGL(rows4_store_kernel<T>, groups, dim3(256), 0, s, x + (size_t)(r * ld), ld, m, d, blocks * 4, at, q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s),
                         ld_s);
    });
  const int gy = (blocks + 3) / 4;
  const int64_t most = kMostBlocks / gy * 64;
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t m = std::min(most, rows - r);
    hipLaunchKernelGGL(rows4_store_columns_kernel<T>, dim3((unsigned)((m + 63) / 64), (unsigned)gy), dim3(256), 0, s, x + r, ld, m, d, blocks, q + (size_t)(r * ld_q), ld_q,
                       scale + (size_t)(r * ld_s), ld_s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
  }
  return hipSuccess;
}

constexpr int64_t kWaves = 8192;  // that a launch should have before they take more than a tile each: four rounds of two per SIMD
// (8,191 x 100,003 x 256, 4 / 6 / 8 / 10 / 16 tiles a wave: 409 / 379 / 371 / 376 / 407 us: fewer load the columns' operands more often, more get out of step)
constexpr int64_t kMostTiles = 8;
template <typename O>
int run_product(ProductArgs p, hipStream_t s) {
  const int64_t col_tiles = (p.N + 32 * kAcross - 1) / (32 * kAcross), rows = p.M;
  p.side = col_tiles >= kGroup ? kGroup : 1;
  const int64_t col_groups = (col_tiles + p.side - 1) / p.side;
  // as many rows as a launch takes workgroups for
  const int64_t most = std::max<int64_t>(1, kMostBlocks / 2 / col_groups) * 32;
  const uint8_t *a = p.a, *a_scale = p.a_scale;
  O *out = static_cast<O *>(p.out);
  for (int64_t r = 0; r < rows; r += most) {
    p.M = std::min(most, rows - r);
    p.a = a + (size_t)(r * p.ld_a);
    p.a_scale = a_scale + (size_t)(r * p.ld_as);
    p.out = out + (size_t)(r * p.ld_out);
    const int64_t row_tiles = (p.M + 31) / 32;
    p.per = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kMostTiles, row_tiles * col_tiles / kWaves));
    const int64_t row_groups = (row_tiles + (int64_t)p.per * (kGroup / p.side) - 1) / ((int64_t)p.per * (kGroup / p.side));
    p.split_cols = col_groups >= 16;
    p.xcd_cols = (uint32_t)(p.split_cols ? (col_groups + 7) / 8 : col_groups);
    p.xcd_rows = (uint32_t)(p.split_cols ? row_groups : (row_groups + 7) / 8);
    hipLaunchKernelGGL((p.blocks <= 8 ? rows4_product_kernel<O, true> : rows4_product_kernel<O, false>),
                       dim3(p.xcd_cols * p.xcd_rows * 8), dim3(64 * kGroup), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
  }
  return hipSuccess;
}

int store(const char *name, bool columns, const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t d, uint8_t *q, int64_t ld_q, uint8_t *scale, int64_t ld_s,
          void *hip_stream) {
  const std::string me = std::string(name) + ": ";
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, me + "unknown dtype");
  if (!sizes_ok(rows, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  if (ld_x < (columns ? rows : d)) return stage_error(GNNSTAGE_EINVAL, me + (columns ? "ld_x is below rows" : "ld_x is below d"));
  if (rows == 0) return GNNSTAGE_OK;
  if (!matrix_ok(x, dtype, err) || !stored_ok(q, ld_q, scale, ld_s, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int e = dtype == GNNSTAGE_BF16 ? run_store(static_cast<const bf16_t *>(x), ld_x, rows, d, columns, q, ld_q, scale, ld_s, s)
                                       : run_store(static_cast<const float *>(x), ld_x, rows, d, columns, q, ld_q, scale, ld_s, s);
  if (e != hipSuccess) return stage_error(GNNSTAGE_EHIP, me + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}

}  // namespace

extern "C" int gnnstage_rows4_store(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t d, uint8_t *q, int64_t ld_q, uint8_t *scale, int64_t ld_s,
                                    void *hip_stream) try {
  return store("gnnstage_rows4_store", false, x, dtype, ld_x, rows, d, q, ld_q, scale, ld_s, hip_stream);
}
GNNSTAGE_GUARD_INT

extern "C" int gnnstage_rows4_store_columns(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t d, uint8_t *q, int64_t ld_q, uint8_t *scale,
                                            int64_t ld_s, void *hip_stream) try {
  return store("gnnstage_rows4_store_columns", true, x, dtype, ld_x, rows, d, q, ld_q, scale, ld_s, hip_stream);
}
GNNSTAGE_GUARD_INT

extern "C" int gnnstage_rows4_load(const uint8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, int64_t rows, int32_t d, void *x, int32_t dtype, int64_t ld_x,
                                   void *hip_stream) try {
  const std::string me = "gnnstage_rows4_load: ";
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, me + "unknown dtype");
  if (!sizes_ok(rows, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  if (ld_x < d) return stage_error(GNNSTAGE_EINVAL, me + "ld_x is below d");
  if (rows == 0) return GNNSTAGE_OK;
  if (!matrix_ok(x, dtype, err) || !stored_ok(q, ld_q, scale, ld_s, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  const int per_row = (d + 7) / 8;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const Grid at = grid_of(per_row);
  const int e = for_grid_slabs(rows, per_row, at.down, [&](int64_t r, int64_t m, dim3 groups) {
    if (dtype == GNNSTAGE_BF16)
      hipLaunchKernelGGL(rows4_load_kernel<bf16_t>, groups, dim3(256), 0, s, q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s, m, d, per_row, at,
                         static_cast<bf16_t *>(x) + (size_t)(r * ld_x), ld_x);
    else
      hipLaunchKernelGGL(rows4_load_kernel<float>, groups, dim3(256), 0, s, q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s, m, d, per_row, at,
                         static_cast<float *>(x) + (size_t)(r * ld_x), ld_x);
  });
  if (e != hipSuccess) return stage_error(GNNSTAGE_EHIP, me + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT

extern "C" int gnnstage_rows4_product(const uint8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, int64_t rows, const uint8_t *other_q, int64_t ld_oq,
                                      const uint8_t *other_scale, int64_t ld_os, int64_t others, int32_t d, const float *bias, void *out, int32_t dtype, int64_t ld_out,
                                      void *hip_stream) try {
  const std::string me = "gnnstage_rows4_product: ";
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, me + "unknown dtype");
  if (!sizes_ok(rows, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  if (others < 0 || others > ((int64_t)1 << 29)) return stage_error(GNNSTAGE_EINVAL, me + "others must be in [0, 2^29]");
  if (ld_out < others) return stage_error(GNNSTAGE_EINVAL, me + "ld_out is below others");
  if (rows == 0 || others == 0) return GNNSTAGE_OK;
  if (!matrix_ok(out, dtype, err) || !stored_ok(q, ld_q, scale, ld_s, d, err) || !stored_ok(other_q, ld_oq, other_scale, ld_os, d, err))
    return stage_error(GNNSTAGE_EINVAL, me + err);
  ProductArgs p{};
  p.a = q;
  p.a_scale = scale;
  p.ld_a = ld_q;
  p.ld_as = ld_s;
  p.b = other_q;
  p.b_scale = other_scale;
  p.ld_b = ld_oq;
  p.ld_bs = ld_os;
  p.M = rows;
  p.N = others;
  p.blocks = (d + 31) / 32;
  p.bias = bias;
  p.out = out;
  p.ld_out = ld_out;
  const int e = dtype == GNNSTAGE_BF16 ? run_product<bf16_t>(p, static_cast<hipStream_t>(hip_stream)) : run_product<float>(p, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return stage_error(GNNSTAGE_EHIP, me + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
