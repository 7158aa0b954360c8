// Rows kept in 8 bits between a forward and a backward pass: blocks of 32 columns of a row share a power of two.
//
//   a = max |x| over the block, e = the least whole number with a <= 127 * 2^e, held within [-120, 121]
//   q = x / 2^e rounded to the nearest whole number, ties to even, in [-127, 127];  the row's value is then q * 2^e
//
// A value is off by at most half a step, 2^(e-1) <= a / 127 (blocks whose largest value is above 127 * 2^121: by a step).  A power of two rather
// than a / 127 as the factor: q * 2^e is then exact in bf16 and fp32 both, so the matrix cores multiply exactly what was
// stored, and the products need no factor of their own.  Below 2^-121 everything is zero (q * 2^e has to stay a normal bf16
// number).  The factor is kept as the byte e + 127, the exponent field of 2^e in fp32; 255 is a block with an infinity or a NaN
// among its values, which restores to NaN (q = 0 times the infinity that 255 stands for in an exponent field).
#include <hip/hip_runtime.h>
#include "guard.h"

#include <algorithm>
#include <string>

#include "../../include/gnnstage.h"
#include "common.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// rows start anywhere: the memory system takes vectors at any address of their elements
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef bf16_t bf16x8_u __attribute__((ext_vector_type(8), aligned(2)));

// columns c .. c + 7 of a row; zeros from d on
template <typename T>
__device__ inline void load8(const T *row, int c, int d, float (&v)[8]) {
  if (c + 8 <= d) {
    if constexpr (sizeof(T) == 2) {
      const bf16x8_u x = *reinterpret_cast<const bf16x8_u *>(row + c);
#pragma unroll
      for (int t = 0; t < 8; ++t) v[t] = (float)x[t];
    } else {
      const f32x4_u x = *reinterpret_cast<const f32x4_u *>(row + c), y = *reinterpret_cast<const f32x4_u *>(row + c + 4);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v[t] = x[t];
        v[4 + t] = y[t];
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t] = c + t < d ? (float)row[c + t] : 0.f;
  }
}

// A thread per eight columns, four neighbouring lanes per block (quads never straddle rows: a row has whole blocks).
template <typename T>
__global__ __launch_bounds__(256) void rows8_store_kernel(const T *x, int64_t ld, int64_t rows, int d, int blocks, int8_t *q, int64_t ld_q,
                                                          uint8_t *scale, int64_t ld_s) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_row = blocks * 4;
  const int64_t r = i / per_row;
  if (r >= rows) return;
  const int g = (int)(i - r * per_row), c = g * 8;
  float v[8];
  load8<T>(x + (size_t)(r * ld), c, d, v);
  // the largest magnitude, compared as bits: infinities and NaNs are above every number
  uint32_t a = 0;
#pragma unroll
  for (int t = 0; t < 8; ++t) a = max(a, __builtin_bit_cast(uint32_t, v[t]) & 0x7fffffffu);
  a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2 of the quad
  a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
  // a = 1.f * 2^(E - 127) <= 127 * 2^e: e = E - 127 - 6 up to 1.f = 127 / 64, one more beyond
  int e = (int)(a >> 23) - 133 + ((a & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  e = min(max(e, -120), 121);
  const bool finite = a < 0x7f800000u;
  const float inv = finite ? __builtin_bit_cast(float, (uint32_t)(127 - e) << 23) : 0.f;
  uint32_t w[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    // added to 1.5 * 2^23 the product is rounded to a whole number, whose low byte is the result (x * inv is exact)
    const float y = finite ? fminf(fmaxf(v[t] * inv, -127.f), 127.f) : 0.f;
    w[t] = __builtin_bit_cast(uint32_t, y + 12582912.f) & 0xffu;
  }
  const u32x2 out = {w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24};
  *reinterpret_cast<u32x2 *>(q + (size_t)(r * ld_q) + c) = out;
  if ((g & 3) == 0) scale[(size_t)(r * ld_s) + (g >> 2)] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
}

template <typename T>
__global__ __launch_bounds__(256) void rows8_load_kernel(const int8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, int64_t rows, int d,
                                                         int per_row, T *x, int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = i / per_row;
  if (r >= rows) return;
  const int c = (int)(i - r * per_row) * 8;
  const u32x2 w = *reinterpret_cast<const u32x2 *>(q + (size_t)(r * ld_q) + c);
  const float f = __builtin_bit_cast(float, (uint32_t)scale[(size_t)(r * ld_s) + (c >> 5)] << 23);
  float v[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) v[t] = (float)(int8_t)(w[t >> 2] >> (8 * (t & 3))) * f;
  T *row = x + (size_t)(r * ld) + c;
  if (c + 8 <= d) {
    if constexpr (sizeof(T) == 2) {
      bf16x8_u o;
#pragma unroll
      for (int t = 0; t < 8; ++t) o[t] = (bf16_t)v[t];
      *reinterpret_cast<bf16x8_u *>(row) = o;
    } else {
      f32x4_u lo, hi;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        lo[t] = v[t];
        hi[t] = v[4 + t];
      }
      *reinterpret_cast<f32x4_u *>(row) = lo;
      *reinterpret_cast<f32x4_u *>(row + 4) = hi;
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (c + t < d) row[t] = (T)v[t];
  }
}

// Splits of a weight gradient: as many as launch_gemm_tn takes at most for these sizes.
constexpr int kMaxSplits = 256;
int splits_for(int d, int d_out) {
  const int64_t tiles = (int64_t)((d + 63) / 64) * ((d_out + 63) / 64);
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, 2048 / tiles));
}
struct Layout {
  size_t partial = 0, bias_partial = 0, dy = 0, total = 0;
  int64_t dy_rows = 0;
  int splits = 0, ld_dy = 0;
};
constexpr int64_t kMostRows = (int64_t)1 << 30;  // of one product; more are several
Layout layout(int64_t rows, int d, int d_out, int dtype) {
  Layout l;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~(size_t)255;
    return at;
  };
  l.splits = splits_for(d, d_out);
  l.ld_dy = round_up(d_out, 8);
  l.partial = take(sizeof(float) * (size_t)l.splits * d * d_out);
  l.bias_partial = take(sizeof(float) * (size_t)l.splits * d_out);
  // gradient rows whose vectors of eight are not aligned are copied, some at a time (bf16; fp32 rows are read as they are)
  l.dy_rows = std::max<int64_t>(1, std::min<int64_t>(rows, 262144));
  l.dy = take(dtype == GNNSTAGE_BF16 ? 2 * (size_t)l.dy_rows * l.ld_dy : 0);
  l.total = off;
  return l;
}

bool sizes_ok(int64_t rows, int d, std::string &err) {
  if (rows < 0 || rows > ((int64_t)1 << 40)) { err = "rows must not be negative (nor beyond 2^40)"; return false; }
  if (d < 1 || d > 65536) { err = "a width must be in [1, 65536]"; return false; }
  return true;
}
// Of a weight gradient: what adds up the row splits has four threads per element of dW and dbias in one launch, below 2^32.
bool outputs_ok(int d, int d_out, std::string &err) {
  if ((int64_t)d * d_out > ((int64_t)1 << 30) - ((int64_t)1 << 17)) { err = "d * d_out must be at most 2^30 - 2^17"; return false; }
  return true;
}
bool stored_ok(const void *q, int64_t ld_q, const void *scale, int64_t ld_s, int d, std::string &err) {
  if (!q || !scale) { err = "q and scale must not be NULL"; return false; }
  if ((reinterpret_cast<uintptr_t>(q) & 15u) || ld_q % 16 != 0) { err = "q must be 16-byte aligned, its leading dimension a multiple of 16"; return false; }
  if (ld_q < round_up(d, 32) || ld_s < (d + 31) / 32) { err = "q rows need d rounded up to 32 bytes, scale rows a byte per 32 columns"; return false; }
  return true;
}

}  // namespace

int launch_rows8_store(const void *x, int dtype, int64_t ld, int64_t rows, int d, int8_t *q, int64_t ld_q, uint8_t *scale, int64_t ld_s,
                       hipStream_t s) {
  const int blocks = (d + 31) / 32;
  return for_row_slabs(rows, blocks * 4, [&](int64_t r, int64_t m, unsigned gx) {
    if (dtype == DT_BF16)
      hipLaunchKernelGGL(rows8_store_kernel<bf16_t>, dim3(gx), dim3(256), 0, s, static_cast<const bf16_t *>(x) + (size_t)(r * ld), ld, m, d, blocks,
                         q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s);
    else
      hipLaunchKernelGGL(rows8_store_kernel<float>, dim3(gx), dim3(256), 0, s, static_cast<const float *>(x) + (size_t)(r * ld), ld, m, d, blocks,
                         q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s);
  });
}

extern "C" int gnnstage_rows8_store(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t d, int8_t *q, int64_t ld_q, uint8_t *scale,
                                    int64_t ld_s, void *hip_stream) try {
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_store: unknown dtype");
  if (!sizes_ok(rows, d, err)) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_store: " + err);
  if (ld_x < d) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_store: ld_x is below d");
  if (rows == 0) return GNNSTAGE_OK;
  if (!x) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_store: x must not be NULL");
  if (!stored_ok(q, ld_q, scale, ld_s, d, err)) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_store: " + err);
  const int e = launch_rows8_store(x, dtype, ld_x, rows, d, q, ld_q, scale, ld_s, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return stage_error(GNNSTAGE_EHIP, std::string("gnnstage_rows8_store: ") + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT

extern "C" int gnnstage_rows8_load(const int8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, int64_t rows, int32_t d, void *x,
                                   int32_t dtype, int64_t ld_x, void *hip_stream) try {
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_load: unknown dtype");
  if (!sizes_ok(rows, d, err)) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_load: " + err);
  if (ld_x < d) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_load: ld_x is below d");
  if (rows == 0) return GNNSTAGE_OK;
  if (!x) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_load: x must not be NULL");
  if (!stored_ok(q, ld_q, scale, ld_s, d, err)) return stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_load: " + err);
  const int per_row = (d + 7) / 8;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int e = for_row_slabs(rows, per_row, [&](int64_t r, int64_t m, unsigned gx) {
    if (dtype == GNNSTAGE_BF16)
      hipLaunchKernelGGL(rows8_load_kernel<bf16_t>, dim3(gx), dim3(256), 0, s, q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s, m, d,
                         per_row, static_cast<bf16_t *>(x) + (size_t)(r * ld_x), ld_x);
    else
      hipLaunchKernelGGL(rows8_load_kernel<float>, dim3(gx), dim3(256), 0, s, q + (size_t)(r * ld_q), ld_q, scale + (size_t)(r * ld_s), ld_s, m, d,
                         per_row, static_cast<float *>(x) + (size_t)(r * ld_x), ld_x);
  });
  if (e != hipSuccess) return stage_error(GNNSTAGE_EHIP, std::string("gnnstage_rows8_load: ") + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT

extern "C" size_t gnnstage_rows8_weight_grad_workspace_size(int64_t rows, int32_t d, int32_t d_out, int32_t dtype) try {
  std::string err;
  if (!sizes_ok(rows, d, err) || !sizes_ok(rows, d_out, err) || !outputs_ok(d, d_out, err)) {
    stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_weight_grad: " + err);
    return 0;
  }
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) {
    stage_error(GNNSTAGE_EINVAL, "gnnstage_rows8_weight_grad: unknown dtype");
    return 0;
  }
  return layout(rows, d, d_out, dtype).total;
}
GNNSTAGE_GUARD_SIZE

extern "C" int gnnstage_rows8_weight_grad(const int8_t *q, int64_t ld_q, const uint8_t *scale, int64_t ld_s, const void *dY, int32_t dtype,
                                          int64_t ld_dy, int64_t rows, int32_t d, int32_t d_out, float *dW, float *dbias, void *workspace,
                                          size_t workspace_bytes, void *hip_stream) try {
  const char *const me = "gnnstage_rows8_weight_grad: ";
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return stage_error(GNNSTAGE_EINVAL, std::string(me) + "unknown dtype");
  if (!sizes_ok(rows, d, err) || !sizes_ok(rows, d_out, err) || !outputs_ok(d, d_out, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  if (ld_dy < d_out || ld_dy > INT32_MAX || ld_q >= 1 << 24 || ld_s >= 1 << 24)
    return stage_error(GNNSTAGE_EINVAL, std::string(me) + "ld_dy is below d_out or beyond 2^31 - 1, or ld_q or ld_s beyond 2^24 - 1");
  if (rows == 0) return GNNSTAGE_OK;
  if (!dY || !dW) return stage_error(GNNSTAGE_EINVAL, std::string(me) + "dY and dW must not be NULL");
  if (!stored_ok(q, ld_q, scale, ld_s, d, err)) return stage_error(GNNSTAGE_EINVAL, me + err);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return stage_error(GNNSTAGE_EINVAL, std::string(me) + "workspace must be 256-byte aligned");
  const Layout l = layout(rows, d, d_out, dtype);
  if (workspace_bytes < l.total)
    return stage_error(GNNSTAGE_ENOMEM, std::string(me) + "workspace smaller than gnnstage_rows8_weight_grad_workspace_size()");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(workspace);
  const bool copy = dtype == GNNSTAGE_BF16 && ((reinterpret_cast<uintptr_t>(dY) & 15u) || ld_dy % 8 != 0 || d_out % 8 != 0 || ld_dy >= 1 << 24);
  const int64_t step = copy ? l.dy_rows : kMostRows;
  const int elt = dtype == GNNSTAGE_BF16 ? 2 : 4;
  for (int64_t r = 0; r < rows; r += step) {
    const int64_t m = std::min(step, rows - r);
    const char *dy = static_cast<const char *>(dY) + (size_t)(r * ld_dy) * elt;
    int e = 0;
    if (copy) {
      e = launch_copy_rows(dy, (int)ld_dy, ws + l.dy, l.ld_dy, m, d_out, dtype, s);
      dy = ws + l.dy;
    }
    GemmTnArgs t{};
    t.A = q + (size_t)(r * ld_q);
    t.a_dtype = DT_ROWS8;
    t.lda = (int)ld_q;
    t.a_scale = scale + (size_t)(r * ld_s);
    t.ld_scale = (int)ld_s;
    t.B = dy;
    t.ldb = copy ? l.ld_dy : (int)ld_dy;
    t.b_cols = copy ? l.ld_dy : d_out;  // (behind the last row's d_out columns there may be nothing)
    t.M = (int)m;
    t.I = d;
    t.O = d_out;
    t.scale = 1.f;
    t.dW = dW;
    t.partial = reinterpret_cast<float *>(ws + l.partial);
    t.max_splits = l.splits;
    t.dbias = dbias;
    t.bias_partial = dbias ? reinterpret_cast<float *>(ws + l.bias_partial) : nullptr;
    if (e == 0) e = launch_gemm_tn(t, dtype, s);
    if (e != 0) return stage_error(GNNSTAGE_EHIP, me + std::string(hipGetErrorString((hipError_t)e)));
  }
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
