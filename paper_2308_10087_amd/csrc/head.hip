// The loss head over many classes without logits: row losses of a linear softmax cross-entropy head and the gradients of its
// rows, weights and biases.
//
//   z_ic = h_i . W_c + b_c,  m_i = max_c z_ic,  o_i = sum_{c != y_i} exp(z_ic - m_i),  e_i = exp(z_iy - m_i),  l_i = o_i + e_i
//   loss_i = log l_i - (z_iy - m_i)                     (log1p(o_i / e_i) where the label holds more than half of l_i)
//   g_ic   = inv_n exp(z_ic - m_i) / l_i, c != y_i;     g_iy = -inv_n o_i / l_i
//   dh_i   = sum_c g_ic W_c,   dW_c += sum_i g_ic h_i,   db_c += sum_i g_ic
//
// The label's own term is kept apart from the others: softmax_y - 1 = -o / l has no cancellation, so a row that is sure of its
// class has a gradient and a loss with as many digits as any other.
#include <hip/hip_runtime.h>
#include "guard.h"

#include <algorithm>
#include <string>

#include "../../include/gnntrain.h"
#include "common.h"
#include "lds_tile.h"

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

__device__ inline float load_elt(const void *p, int dtype, size_t i) {
  return dtype == DT_BF16 ? (float)static_cast<const bf16_t *>(p)[i] : static_cast<const float *>(p)[i];
}
__device__ inline void store_elt(void *p, int dtype, size_t i, float v) {
  if (dtype == DT_BF16)
    static_cast<bf16_t *>(p)[i] = (bf16_t)v;
  else
    static_cast<float *>(p)[i] = v;
}
__device__ inline bool is_labelled(const int32_t *labels, const uint8_t *mask, int64_t r, int C) {
  return (mask == nullptr || mask[r] != 0) && (uint32_t)labels[r] < (uint32_t)C;
}
__device__ inline float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// ---- in pieces of rows and classes -------------------------------------------------------------------------------
// A slab of rows goes through the classes in pieces: the logits of a piece are a library product into scratch memory, then the
// rows' running maximum and sum.  A second sweep computes each piece's logits again, turns them into gradients in place and
// multiplies these with the weights and the rows.  Rows without a label are zeros that go through all of it: how many there are is known to the
// device only, and the products are sized on the host (60,000 x 100 x 2,000 in fp32: 1,310 us with 2 % of the rows labelled, 1,410 with all).

// What a row of the slab has seen so far.
struct RowState {
  float max, others, own, unused;  // own: the label's logit
};

// A slab's rows, packed: padded with zeros to ld columns; rows without a label are zeros altogether (what they hold must
// reach no sum, not even as a factor of zero), have loss 0 and label -1.
__global__ __launch_bounds__(256) void pack_rows_kernel(const void *h, int dtype, int64_t ld_h, const int32_t *labels, const uint8_t *mask,
                                                        int64_t rows, int d, int C, void *out, int ld, int32_t *label, RowState *state,
                                                        float *row_loss) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const bool on = is_labelled(labels, mask, r, C);
  for (int c = lane; c < ld; c += 64) store_elt(out, dtype, (size_t)r * ld + c, on && c < d ? load_elt(h, dtype, (size_t)(r * ld_h) + c) : 0.f);
  if (lane == 0) {
    label[r] = on ? labels[r] : -1;
    state[r] = RowState{-INFINITY, 0.f, 0.f, 0.f};
    if (!on) row_loss[r] = 0.f;
  }
}

// Rows of a piece's logits: a wave per row, four rows per workgroup, or (WAVES = 16) a workgroup per row where the classes are many, so that few rows occupy
// more of the card and a lane's chain of exponentials is short: from 2,048 classes on where the rows are few, else from 4,096.  The kernel alone, 100 x 50,021:
// 647 us with a wave per row, 46 with a workgroup; calls of width 64 in fp32, waves / workgroups: 1,000 x 600 49 / 51, 1,000 x 2,100 78 / 69, 5,000 x 2,100
// 138 / 148, 20,000 x 2,100 377 / 447, 5,000 x 8,000 399 / 373, 20,000 x 8,000 1,584 / 1,415.
constexpr int kWideRow = 2048;

template <int WAVES>
constexpr int row_threads = WAVES == 1 ? 256 : 64 * WAVES;

template <int WAVES>
__device__ __forceinline__ int64_t my_row() {
  return WAVES == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x;
}

// over the lanes that share a row; every lane gets the result
template <int WAVES, bool MAX>
__device__ __forceinline__ float row_join(float v) {
  v = MAX ? wave_max(v) : wave_sum(v);
  if constexpr (WAVES > 1) {
    __shared__ float part[WAVES];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = MAX ? fmaxf(v, part[w]) : v + part[w];
  }
  return v;
}

// The classes [c0, c0 + n) of a slab's rows.
template <int WAVES>
__global__ __launch_bounds__(row_threads<WAVES>) void piece_state_kernel(const float *logits, int ld, const float *bias, const int32_t *label, int64_t rows,
                                                          int c0, int n, int last, RowState *state, float *row_loss) {
  constexpr int kStep = 64 * WAVES;
  const int lane = threadIdx.x & (kStep - 1);
  const int64_t r = my_row<WAVES>();
  if (r >= rows) return;
  const int y = label[r] - c0;
  if (label[r] < 0) return;
  const float *z = logits + (size_t)r * ld;
  RowState s = state[r];
  float mx = s.max;
#pragma unroll 4
  for (int c = lane; c < n; c += kStep) mx = fmaxf(mx, z[c] + (bias ? bias[c0 + c] : 0.f));
  mx = row_join<WAVES, true>(mx);
  float others = 0.f;
#pragma unroll 4
  for (int c = lane; c < n; c += kStep)
    if (c != y) others += expf(z[c] + (bias ? bias[c0 + c] : 0.f) - mx);
  others = row_join<WAVES, false>(others);
  // nothing but logits of minus infinity so far: there is no sum yet (their differences are no numbers)
  if (mx == -INFINITY)
    others = 0.f;
  else
    others += s.others * (s.max == -INFINITY ? 0.f : expf(s.max - mx));
  if (lane != 0) return;
  s.max = mx;
  s.others = others;
  if (y >= 0 && y < n) s.own = z[y] + (bias ? bias[c0 + y] : 0.f);
  state[r] = s;
  if (last) {
    const float zl = s.own - mx, own = expf(zl), sum = others + own;
    row_loss[r] = own > 0.5f * sum ? log1pf(others / own) : logf(sum) - zl;
  }
}

// The gradients of a piece's logits: fp32 in place, or as the sum of three bf16 numbers, which is all of their bits: the weight
// gradient is fp32.  Columns [n, ld) are written as zeros.
template <int WAVES>
__global__ __launch_bounds__(row_threads<WAVES>) void piece_grad_kernel(float *logits, int ld, const float *bias, const int32_t *label, int64_t rows, int c0,
                                                         int n, float inv_n, const RowState *state, bf16_t *high, bf16_t *low, bf16_t *lowest) {
  constexpr int kStep = 64 * WAVES;
  const int lane = threadIdx.x & (kStep - 1);
  const int64_t r = my_row<WAVES>();
  if (r >= rows) return;
  float *z = logits + (size_t)r * ld;
  const bool on = label[r] >= 0;
  const int y = label[r] - c0;
  const RowState s = state[r];
  const float inv_sum = 1.f / (s.others + expf(s.own - s.max));
  for (int c = lane; c < ld; c += kStep) {
    float g = 0.f;
    if (on && c < n) g = (c == y ? -s.others : expf(z[c] + (bias ? bias[c0 + c] : 0.f) - s.max)) * inv_sum * inv_n;
    if (high != nullptr) {
      const bf16_t x = (bf16_t)g;
      const float rest = g - (float)x;
      const bf16_t y2 = (bf16_t)rest;
      high[(size_t)r * ld + c] = x;
      low[(size_t)r * ld + c] = y2;
      lowest[(size_t)r * ld + c] = (bf16_t)(rest - (float)y2);
    } else {
      z[c] = g;
    }
  }
}

// Both at once where the classes are one piece: loss and gradients of a row.
template <int WAVES>
__global__ __launch_bounds__(row_threads<WAVES>) void whole_grad_kernel(float *logits, int ld, const float *bias, const int32_t *label, int64_t rows, int n,
                                                         float inv_n, float *row_loss, bf16_t *high, bf16_t *low, bf16_t *lowest) {
  constexpr int kStep = 64 * WAVES;
  const int lane = threadIdx.x & (kStep - 1);
  const int64_t r = my_row<WAVES>();
  if (r >= rows) return;
  float *z = logits + (size_t)r * ld;
  const int y = label[r];
  const bool on = y >= 0;
  const float zy = on ? z[y] + (bias ? bias[y] : 0.f) : 0.f;  // read before the joins below: in fp32 the gradients overwrite it
  float mx = -INFINITY, others = 0.f;
#pragma unroll 4
  for (int c = lane; c < n; c += kStep) mx = fmaxf(mx, z[c] + (bias ? bias[c] : 0.f));
  mx = row_join<WAVES, true>(mx);
#pragma unroll 4
  for (int c = lane; c < n; c += kStep)
    if (c != y) others += expf(z[c] + (bias ? bias[c] : 0.f) - mx);
  others = row_join<WAVES, false>(others);
  const float zl = on ? zy - mx : 0.f, own = expf(zl), sum = others + own, inv_sum = 1.f / sum;
  for (int c = lane; c < ld; c += kStep) {
    float g = 0.f;
    if (on && c < n) g = (c == y ? -others : expf(z[c] + (bias ? bias[c] : 0.f) - mx)) * inv_sum * inv_n;
    if (high != nullptr) {
      const bf16_t x = (bf16_t)g;
      const float rest = g - (float)x;
      const bf16_t y2 = (bf16_t)rest;
      high[(size_t)r * ld + c] = x;
      low[(size_t)r * ld + c] = y2;
      lowest[(size_t)r * ld + c] = (bf16_t)(rest - (float)y2);
    } else {
      z[c] = g;
    }
  }
  if (lane == 0 && on) row_loss[r] = own > 0.5f * sum ? log1pf(others / own) : logf(sum) - zl;
}

// dh = what the pieces have added up, in the rows' type; zeros for rows without a label
__global__ __launch_bounds__(256) void finish_rows_kernel(const float *acc, const int32_t *label, int64_t rows, int d, void *dh, int dtype,
                                                          int64_t ld_dh) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * d) return;
  const int64_t r = i / d;
  store_elt(dh, dtype, (size_t)(r * ld_dh + i % d), label[r] >= 0 ? acc[i] : 0.f);
}

// out[c][r] = in[r][c], r < rows, c < n: 32 x 32 at a time
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(const T *in, int64_t ld, int rows, int n, T *out, int64_t ld_out) {
  __shared__ T tile[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    if (r0 + y + i < rows && c0 + x < n) tile[y + i][x] = in[(size_t)(r0 + y + i) * ld + c0 + x];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    if (c0 + y + i < n && r0 + x < rows) out[(size_t)(c0 + y + i) * ld_out + r0 + x] = tile[x][y + i];
}

// dW[k][c0 + c] += piece[k][c], c < n
__global__ __launch_bounds__(256) void add_piece_kernel(const float *piece, int d, int n, float *dW, int C, int c0) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)d * n) return;
  dW[(size_t)(i / n) * C + c0 + i % n] += piece[i];
}

constexpr int kPieceClasses = 8192;  // at least, where rows are many; few rows' logits are one piece
constexpr int64_t kPieceElements = 1 << 26;  // logits of a slab's piece
constexpr int64_t kSlabRows = 131072;

// Which fp32 products serve.  rows x width x classes, in us, on the products of the stages' layers / on the head's own (head32.hip, tiles of 128 rows):
// 2,000 x 256 x 1,000 85 / 112, 34,493 x 256 x 172 209 / 278, 34,493 x 256 x 1,000 733 / 742, 100,000 x 64 x 1,000 901 / 1,176;
// 5,000 x 500 x 1,500 364 / 333, 5,000 x 1,000 x 700 332 / 295, 5,196 x 1,000 x 2,003 840 / 725.
constexpr int kOwnWidth = 384;
constexpr double kOwnWork = 3e9;  // rows * classes * width
// Few rows against many classes: dh = g W^T is a sum over the classes with few outputs, which the products above give to as few workgroups.  With the gradients
// turned it is one over the rows of its operands, which is cut into many.  rows x width x classes, fp32, in us, as they are / turned: 100 x 256 x 50,021 686 / 359,
// 2,000 x 128 x 20,000 1,414 / 851; 1,000 x 600 x 2,000 169 / 174, 4,096 x 256 x 4,096 367 / 383, 300 x 64 x 800 46 / 55.
constexpr int64_t kFewRows = 4096;
constexpr int kManyClasses = 8192;
struct Plan {
  int64_t rows = 0, slab = 0;
  int d = 0, C = 0, dtype = 0, elt = 4, Kp = 0, Cp = 0, piece = 0, ld = 0, max_splits = 0, max_splits_turned = 0;
  bool grads = false;
  bool own32 = false;   // fp32 products on the head's own kernels
  bool turned = false;  // dh from the turned gradients
  int ld_turned = 0;
  size_t Wt = 0, Wn = 0, rows_at = 0, label = 0, state = 0, logits = 0, high = 0, low = 0, lowest = 0, acc = 0, zeros = 0, tmp = 0, turn = 0, partial = 0,
         bias_partial = 0, total = 0;
};

bool make_plan(int64_t rows, int d, int C, int dtype, bool grads, Plan &p, std::string &err) {
  if (rows < 0 || rows > ((int64_t)1 << 40)) { err = "rows must not be negative (nor beyond 2^40)"; return false; }
  if (d < 1 || d > 65534) { err = "the rows' width must be in [1, 65534]"; return false; }
  if (C < 1 || C > (1 << 24)) { err = "n_classes must be in [1, 2^24]"; return false; }
  if ((int64_t)C * d > (int64_t)1 << 33) { err = "the weights must be 2^33 elements at most"; return false; }  // (a launch lays them out, 2^32 threads at most)
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) { err = "unknown dtype"; return false; }
  p.rows = rows;
  p.d = d;
  p.C = C;
  p.dtype = dtype;
  p.elt = dtype == GNNSTAGE_BF16 ? 2 : 4;
  p.grads = grads;
  p.Kp = round_up(d, 8);
  p.Cp = round_up(C, 8);
  const int64_t few = std::max<int64_t>(1, std::min(rows, kSlabRows));
  p.piece = (int)std::min<int64_t>(p.Cp, std::max<int64_t>(kPieceClasses, kPieceElements / std::max<int64_t>(few, d) / 8 * 8));
  p.ld = p.piece;
  p.slab = std::max<int64_t>(128, std::min(kSlabRows, kPieceElements / std::max(p.ld, p.d)));
  p.slab = std::min(p.slab, std::max<int64_t>(rows, 1));
  const int64_t tiles = (int64_t)((d + 127) / 128) * ((p.piece + 127) / 128);
  p.turned = grads && p.slab <= kFewRows && C >= kManyClasses;
  p.own32 = dtype == GNNSTAGE_F32 && d >= kOwnWidth && (double)p.slab * C * d >= kOwnWork;
  p.ld_turned = round_up((int)p.slab, 8);
  p.max_splits = p.own32 ? tn32_splits(p.slab, d, p.piece) : (int)std::max<int64_t>(1, std::min<int64_t>(256, 1024 / tiles));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align256(off + bytes);
    return at;
  };
  const size_t m = (size_t)p.slab;
  // as many as the room for the weight gradients' partial sums holds
  p.max_splits_turned = (int)std::max<int64_t>(1, std::min<int64_t>(256, (int64_t)p.max_splits * std::max<int64_t>(p.piece, p.slab) / p.slab));
  p.Wt = take((size_t)p.elt * C * p.Kp);
  p.Wn = take((size_t)p.elt * d * p.Cp);
  p.rows_at = take((size_t)p.elt * m * p.Kp);
  p.label = take(sizeof(int32_t) * m);
  p.state = take(sizeof(RowState) * m);
  p.logits = take(sizeof(float) * m * p.ld);
  if (grads) {
    p.high = take(dtype == GNNSTAGE_BF16 ? 2 * m * p.ld : 0);
    p.low = take(dtype == GNNSTAGE_BF16 ? 2 * m * p.ld : 0);
    p.lowest = take(dtype == GNNSTAGE_BF16 ? 2 * m * p.ld : 0);
    p.acc = take(sizeof(float) * m * d);
    p.zeros = take(p.own32 ? 0 : sizeof(float) * (size_t)round_up(d, 64));
    p.tmp = take(p.own32 ? 0 : sizeof(float) * (size_t)d * p.piece);
    p.turn = take(p.turned ? (size_t)p.elt * p.piece * p.ld_turned : 0);
    p.partial = take(sizeof(float) * (size_t)p.max_splits * d * std::max<size_t>(p.piece, p.turned ? m : 0));
    p.bias_partial = take(sizeof(float) * (size_t)p.max_splits * p.piece);
  }
  p.total = off;
  return true;
}

struct Call {
  const void *h;
  int64_t ld_h;
  const void *W;
  const float *bias;
  const int32_t *labels;
  const uint8_t *mask;
  float inv_n;
  float *row_loss;
  void *dh;
  int64_t ld_dh;
  float *dW, *db;
  char *ws;
};

#define HEAD_TRY(expr)                \
  do {                                \
    const int e_ = (int)(expr);       \
    if (e_ != 0) return e_;           \
  } while (0)

// a hipError_t
int run_in_pieces(const Plan &p, const Call &c, hipStream_t s) {
  auto at = [&](size_t off) { return c.ws + off; };
  const StageWeightsArgs w{c.W, p.d, p.C, at(p.Wt), p.Kp, at(p.Wn), p.Cp};
  HEAD_TRY(launch_stage_weights(&w, 1, p.dtype, nullptr, s));
  const bool one = p.piece >= p.C, own32 = p.own32;
  if (c.dh && (!one || p.dtype == GNNSTAGE_BF16) && !own32 && !p.turned) HEAD_TRY(launch_fill_zero(at(p.zeros), sizeof(float) * (size_t)round_up(p.d, 64), s));
  float *logits = reinterpret_cast<float *>(at(p.logits)), *acc = reinterpret_cast<float *>(at(p.acc));
  int32_t *label = reinterpret_cast<int32_t *>(at(p.label));
  RowState *state = reinterpret_cast<RowState *>(at(p.state));
  bf16_t *high = p.dtype == GNNSTAGE_BF16 ? reinterpret_cast<bf16_t *>(at(p.high)) : nullptr;
  bf16_t *low = p.dtype == GNNSTAGE_BF16 ? reinterpret_cast<bf16_t *>(at(p.low)) : nullptr;
  bf16_t *lowest = p.dtype == GNNSTAGE_BF16 ? reinterpret_cast<bf16_t *>(at(p.lowest)) : nullptr;
  // Without gradients, rows in whole 16-byte pieces are read where they are: those without a label, which may hold anything, meet no other row.
  // (450,061 x 600 x 103 classes, fp32: 1,681 us from a packed copy, 1,067 without.)
  const bool in_place = !p.grads && p.d % 8 == 0 && c.ld_h * p.elt % 16 == 0 && (reinterpret_cast<uintptr_t>(c.h) & 15u) == 0 && c.ld_h <= INT32_MAX;
  for (int64_t row0 = 0; row0 < p.rows; row0 += p.slab) {
    const int64_t M = std::min(p.slab, p.rows - row0);
    const char *h = static_cast<const char *>(c.h) + (size_t)(row0 * c.ld_h) * p.elt;
    const char *rows_at = in_place ? h : at(p.rows_at);
    const int64_t ld_rows = in_place ? c.ld_h : p.Kp;
    const unsigned waves = (unsigned)((M + 3) / 4);
    const bool wide = p.piece >= (M <= kFewRows ? kWideRow : 2 * kWideRow);
    hipLaunchKernelGGL(pack_rows_kernel, dim3(waves), dim3(256), 0, s, h, p.dtype, c.ld_h, c.labels + row0, c.mask ? c.mask + row0 : nullptr, M, p.d, p.C,
                       (void *)at(p.rows_at), in_place ? 0 : p.Kp, label, state, c.row_loss + row0);
    HEAD_TRY(hipGetLastError());
    auto piece_logits = [&](int c0, int n) {
      if (own32)
        return launch_nt32(reinterpret_cast<const float *>(rows_at), ld_rows, reinterpret_cast<const float *>(at(p.Wt)) + (size_t)c0 * p.Kp, p.Kp, (int)M,
                           n, p.Kp, logits, p.ld, false, s);
      GemmNtArgs g{};
      g.A = rows_at;
      g.a_dtype = p.dtype;
      g.lda = ld_rows;
      g.Bt = at(p.Wt) + (size_t)c0 * p.Kp * p.elt;
      g.ldb = p.Kp;
      g.M = (int)M;
      g.N = n;
      g.K = p.d;
      g.Kp = p.Kp;
      g.epilogue = EPI_PLAIN;
      g.blocks = p.dtype == GNNSTAGE_F32;
      g.out = logits;
      g.out_dtype = DT_F32;
      g.out_ld = p.ld;
      return launch_gemm_nt(g, p.dtype, s);
    };
    for (int c0 = 0; c0 < p.C; c0 += p.piece) {
      const int n = std::min(p.piece, p.C - c0);
      HEAD_TRY(piece_logits(c0, n));
      if (one && p.grads) {
        if (wide)
          hipLaunchKernelGGL(whole_grad_kernel<16>, dim3((unsigned)M), dim3(1024), 0, s, logits, p.ld, c.bias, label, M, n, c.inv_n, c.row_loss + row0, high, low, lowest);
        else
          hipLaunchKernelGGL(whole_grad_kernel<1>, dim3(waves), dim3(256), 0, s, logits, p.ld, c.bias, label, M, n, c.inv_n, c.row_loss + row0, high, low, lowest);
        HEAD_TRY(hipGetLastError());
        continue;
      }
      if (wide)
        hipLaunchKernelGGL(piece_state_kernel<16>, dim3((unsigned)M), dim3(1024), 0, s, logits, p.ld, c.bias, label, M, c0, n, (int)(c0 + n == p.C),
                           state, c.row_loss + row0);
      else
        hipLaunchKernelGGL(piece_state_kernel<1>, dim3(waves), dim3(256), 0, s, logits, p.ld, c.bias, label, M, c0, n, (int)(c0 + n == p.C), state,
                           c.row_loss + row0);
      HEAD_TRY(hipGetLastError());
    }
    if (!p.grads) continue;
    for (int c0 = 0; c0 < p.C; c0 += p.piece) {
      const int n = std::min(p.piece, p.C - c0);
      if (!one) {
        HEAD_TRY(piece_logits(c0, n));
        if (wide)
          hipLaunchKernelGGL(piece_grad_kernel<16>, dim3((unsigned)M), dim3(1024), 0, s, logits, p.ld, c.bias, label, M, c0, n, c.inv_n, state, high, low, lowest);
        else
          hipLaunchKernelGGL(piece_grad_kernel<1>, dim3(waves), dim3(256), 0, s, logits, p.ld, c.bias, label, M, c0, n, c.inv_n, state, high, low, lowest);
        HEAD_TRY(hipGetLastError());
      }
      // bf16: dh from the first two of the gradients' numbers, 2^-16 of each.  (From the first alone, 2^-8 of the label's too: 2,000 x 500 x 41 classes, relative error
      // 2.2e-3 against 1.66e-3 with both, bf16's own, and 2.4e-2 where all classes share a column of 16 times what tells them apart; a sixth product costs
      // 20,000 x 500 x 2,000 785 -> 944 us, 3,000 x 1,000 x 9,000 3,335 -> 3,670.)
      const int parts = high ? 2 : 1;
      if (c.dh && p.turned) {
        if (c0 == 0) HEAD_TRY(launch_fill_zero(acc, sizeof(float) * (size_t)M * p.d, s));
        const dim3 grid((unsigned)((n + 31) / 32), (unsigned)((M + 31) / 32));
        for (int part = 0; part < parts; ++part) {
          if (high)
            hipLaunchKernelGGL(turn_kernel<bf16_t>, grid, dim3(256), 0, s, part == 0 ? high : low, p.ld, (int)M, n, reinterpret_cast<bf16_t *>(at(p.turn)),
                               p.ld_turned);
          else
            hipLaunchKernelGGL(turn_kernel<float>, grid, dim3(256), 0, s, logits, p.ld, (int)M, n, reinterpret_cast<float *>(at(p.turn)), p.ld_turned);
          HEAD_TRY(hipGetLastError());
          if (own32) {
            HEAD_TRY(launch_tn32(reinterpret_cast<const float *>(at(p.turn)), p.ld_turned, reinterpret_cast<const float *>(at(p.Wt)) + (size_t)c0 * p.Kp, p.Kp,
                                 n, (int)M, p.d, acc, p.d, nullptr, reinterpret_cast<float *>(at(p.partial)), nullptr, p.max_splits_turned, s));
            continue;
          }
          GemmTnArgs t{};
          t.A = at(p.turn);
          t.a_dtype = p.dtype;
          t.lda = p.ld_turned;
          t.B = at(p.Wt) + (size_t)c0 * p.Kp * p.elt;
          t.ldb = p.Kp;
          t.M = n;
          t.I = (int)M;
          t.O = p.d;
          t.scale = 1.f;
          t.dW = acc;
          t.partial = reinterpret_cast<float *>(at(p.partial));
          t.max_splits = p.max_splits_turned;
          HEAD_TRY(launch_gemm_tn(t, p.dtype, s));
        }
      }
      if (own32) {  // (columns of the gradients from n up to a multiple of 8 are zeros, and so are the weights')
        if (c.dh && !p.turned)
          HEAD_TRY(launch_nt32(logits, p.ld, reinterpret_cast<const float *>(at(p.Wn)) + c0, p.Cp, (int)M, p.d, round_up(n, 8), acc, p.d, c0 > 0, s));
        if (c.dW || c.db)
          HEAD_TRY(launch_tn32(reinterpret_cast<const float *>(at(p.rows_at)), p.Kp, logits, p.ld, (int)M, p.d, n, c.dW ? c.dW + c0 : nullptr, p.C,
                               c.db ? c.db + c0 : nullptr, reinterpret_cast<float *>(at(p.partial)), reinterpret_cast<float *>(at(p.bias_partial)),
                               p.max_splits, s));
        continue;
      }
      if (c.dh && !p.turned) {
        for (int part = 0; part < parts; ++part) {
          GemmNtArgs g{};
          g.A = !high ? (const void *)logits : part == 0 ? high : low;
          g.a_dtype = p.dtype;
          g.lda = p.ld;
          g.Bt = at(p.Wn) + (size_t)c0 * p.elt;
          g.ldb = p.Cp;
          g.M = (int)M;
          g.N = p.d;
          g.K = n;
          g.Kp = round_up(n, 8);
          g.epilogue = c0 == 0 && part == 0 ? EPI_PLAIN : EPI_RES;
          g.blocks = p.dtype == GNNSTAGE_F32;
          g.bias = reinterpret_cast<const float *>(at(p.zeros));
          g.aux = acc;
          g.aux_dtype = DT_F32;
          g.aux_ld = p.d;
          g.out = acc;
          g.out_dtype = DT_F32;
          g.out_ld = p.d;
          HEAD_TRY(launch_gemm_nt(g, p.dtype, s));
        }
      }
      if (c.dW || c.db) {
        const bool whole = one && c.dW;
        float *tmp = whole ? c.dW : reinterpret_cast<float *>(at(p.tmp));
        if (!whole) HEAD_TRY(launch_fill_zero(tmp, sizeof(float) * (size_t)p.d * n, s));
        for (int part = 0; part < (high ? 3 : 1); ++part) {
          GemmTnArgs t{};
          t.A = at(p.rows_at);
          t.a_dtype = p.dtype;
          t.lda = p.Kp;
          t.B = high ? (const void *)(part == 0 ? high : part == 1 ? low : lowest) : logits;
          t.ldb = p.ld;
          t.M = (int)M;
          t.I = p.d;
          t.O = n;
          t.scale = 1.f;
          t.dW = tmp;
          t.partial = reinterpret_cast<float *>(at(p.partial));
          t.max_splits = p.max_splits;
          t.dbias = c.db ? c.db + c0 : nullptr;
          t.bias_partial = c.db ? reinterpret_cast<float *>(at(p.bias_partial)) : nullptr;
          HEAD_TRY(launch_gemm_tn(t, p.dtype, s));
        }
        if (!whole && c.dW) {
          hipLaunchKernelGGL(add_piece_kernel, dim3((unsigned)(((int64_t)p.d * n + 255) / 256)), dim3(256), 0, s, tmp, p.d, n, c.dW, p.C, c0);
          HEAD_TRY(hipGetLastError());
        }
      }
    }
    if (c.dh) {
      hipLaunchKernelGGL(finish_rows_kernel, dim3((unsigned)((M * p.d + 255) / 256)), dim3(256), 0, s, acc, label, M, p.d,
                         (void *)(static_cast<char *>(c.dh) + (size_t)(row0 * c.ld_dh) * p.elt), p.dtype, c.ld_dh);
      HEAD_TRY(hipGetLastError());
    }
  }
  return hipSuccess;
}

// ---- bf16 rows of up to 256 columns: the logits never leave the registers -----------------------------------------------------
// Two kernels of one shape.  A wave OWNS 32 vectors (rows, or classes) whose products' sums it keeps, and the other side is
// STREAMED past it in tiles of 32 vectors:
//
//   rows kernel     owns rows, streams classes:  z[c][i] = W_c . h_i;  p = exp(z - running max);  sum_c p W_c, sum_c p
//   classes kernel  owns classes, streams rows:  z[i][c] = h_i . W_c;  g = exp(z - log l_i) (label: -o_i / l_i);  sum_i g h_i, sum_i g
//
// The first product's result has the streamed index in its registers and the owned one in its lanes (32 x 32 x 16 matrix
// instructions: register i of lane l is streamed vector 8 (i / 4) + 4 (l / 32) + i % 4, owned vector l % 32), which is the layout of
// the second product's right operand if its reduction index runs in the order 8 (j / 4) + 4 (l / 32) + j % 4: p goes from one
// product to the next without leaving its lane.  The left operand of the second product is the streamed tile turned by the LDS
// transpose reads, four rows of one column per lane at a time, in that same order.  So one LDS copy of a tile, loaded by the
// direct-to-LDS path, serves both products.
// Bound by the matrix cores: per owned and streamed vector 4 d operations (rows kernel), 6 d (classes kernel: g enters as the sum
// of two bf16 numbers, since dW is fp32), per wave and tile 32 (48) matrix instructions at d = 256 and half the LDS bandwidth; tiles with large
// factors take 16 (48) more, see mean_scale and kExactPerClass.
// Two workgroups of four waves per compute unit at width 256 (three at 128, four at 64): one's exponentials run under the other's products.

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896f;
constexpr float kExactFrom = 1.f / 64;  // of g times the number of rows that inv_n stands for (1 / 2 takes as long)
constexpr int kExactRows = 16384;
constexpr int kExactPerClass = 128;
constexpr float kCoarseTo = 1.f / 32;  // see mean_scale
constexpr float kNoMax = -3.4028234663852886e38f;  // the least number: of a row that has seen no more than minus infinity
// exp(z - m): the difference first, so that it is exact for the logits that count, however large they are
__device__ __forceinline__ float exp_diff(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }
constexpr int kTile = 32;           // streamed vectors of a step
constexpr int kOwned = 128;         // owned vectors of a workgroup, 32 per wave
// Workgroups that run at once: per compute unit two (width 256: a wave's sums are half of the registers), three or four.
template <int DP>
constexpr int kPerUnit = DP == 256 ? 2 : DP == 128 ? 3 : 4;
int round_of(int DP) { return 256 * (DP == 256 ? kPerUnit<256> : DP == 128 ? kPerUnit<128> : kPerUnit<64>); }
constexpr int kRowItems = 1536;     // most (row tile, class range) pairs that leave partial sums
constexpr int kMetaBlock = 2048;    // rows of a counting workgroup

// What depends on the number of labelled rows, which the host does not know.
struct Meta {
  int32_t n;               // labelled rows
  int32_t row_tiles;       // of kOwned
  int32_t splits;          // class ranges of the rows kernel
  int32_t tiles_per;       // class tiles of a range
  int32_t row_steps;       // tiles of kTile rows: what a class tile of the classes kernel streams
  int32_t groups;          // workgroups of the classes kernel that have work
  int32_t unused[2];
};

template <int DP>
struct Geometry {
  static constexpr int row_bytes = DP * 2, chunks = DP / 8, rows_per_load = 64 / chunks, loads = kTile / (4 * rows_per_load);
  static constexpr int tile_bytes = kTile * row_bytes;
};
// A lane's places in a tile: of what it loads, of its rows in the first product, of its columns in the second.
template <int DP>
struct Places {
  uint32_t load, first, second;
  __device__ Places(int wave, int lane) {
    typedef Geometry<DP> G;
    const int row = wave * G::rows_per_load + lane / G::chunks;
    load = lds_piece<DP>(row, lane % G::chunks);
    first = lds_piece<DP>(lane & 31, lane >> 5);
    second = lds_turn_place<DP>(lane);
  }
  // the addresses below are these with constant bits turned over; made anew in every step, or the compiler keeps them all in
  // registers and spills
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(first), "+v"(second)); }
};
template <int DP>
__device__ __forceinline__ void load_tile(const bf16_t *src, lds_char *dst, int wave, uint32_t place) {
  typedef Geometry<DP> G;
#pragma unroll
  for (int q = 0; q < G::loads; ++q) {
    constexpr int step = 4 * G::rows_per_load;
    // (the q-th load's row is step rows on: its swizzle differs where step / 4 is odd)
    const uint32_t turn = (lds_swizzle<DP>(q * step) ^ lds_swizzle<DP>(0)) << 4;
    load_lds16(reinterpret_cast<const char *>(src) + (place ^ turn) + q * step * G::row_bytes, dst + q * step * G::row_bytes + wave * 1024);
  }
}
template <int DP>
__device__ __forceinline__ bf16x8 first_operand(const lds_char *tile, uint32_t place, int ks) {
  return *reinterpret_cast<const LDS_AS bf16x8 *>(tile + (place ^ ((32 * ks) & (Geometry<DP>::row_bytes - 1) & 255)) + ((32 * ks) & ~255));
}
// The owned vectors as right operands of the first product: most in registers; the rest, where the registers do not reach, in LDS.
template <int DP, int IN_REGS>
struct Owned {
  static constexpr int steps = DP / 16, in_lds = steps - IN_REGS;
  bf16x8 reg[IN_REGS];
  lds_char *lds;
  // vector: this lane's (lane % 32 of the wave's 32)
  __device__ __forceinline__ Owned(const bf16_t *vector, int wave, int lane, char *shared) {
    lds = (lds_char *)shared + wave * in_lds * 1024 + lane * 16;
    const bf16_t *v = vector + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < steps; ++i) {
      const bf16x8 x = *reinterpret_cast<const bf16x8 *>(v + 16 * i);
      if (i < IN_REGS)
        reg[i] = x;
      else
        *reinterpret_cast<LDS_AS bf16x8 *>(lds + (i - IN_REGS) * 1024) = x;  // read by this lane alone
    }
  }
  __device__ __forceinline__ bf16x8 operator()(int ks) const {
    return ks < IN_REGS ? reg[ks < IN_REGS ? ks : 0] : *reinterpret_cast<const LDS_AS bf16x8 *>(lds + (ks - IN_REGS) * 1024);
  }
};
template <int DP>
__device__ __forceinline__ void clear(f32x16 (&o)[DP / 32]) {
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int t = 0; t < 16; ++t) o[i][t] = 0.f;
}
__device__ __forceinline__ void wait_tile() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // this wave's loads to LDS are there (vmcnt 0) ...
  __syncthreads();                     // ... and everybody's; what the other buffer held is done with
}

struct RowsArgs {
  const Meta *meta;
  const bf16_t *rows, *W;   // DIRECT: the caller's rows, which the list picks; else packed [.][DP].  W: [.][DP]
  int64_t ld_rows;
  const float *bias;        // padded to whole tiles with minus infinity
  const int32_t *label;     // of the labelled rows, side by side
  const int32_t *list;      // labelled row -> row
  int32_t C, d;
  float inv_n;
  float *row_loss;          // by row
  bf16_t *dh;               // by row, or NULL
  int64_t ld_dh;
  float *max, *log, *t;     // of the labelled rows: the row's maximum, -log2 of its sum, o / l
  float *part;              // [item][wave][DP][32]: sum p W
  float *part_stat;         // [item][4][kOwned]: maximum, others, the label's logit, the sum of the factors that part was made with
  // workgroups from items on write the zeros of the other rows' dh: memory's work, next to the matrix cores'
  int32_t items, fills;
  const int32_t *labels;    // by row
  const uint8_t *mask;
  int64_t all_rows;
};

template <int DP>
__device__ void fill_rows(const RowsArgs &a) {
  constexpr int per_row = DP / 8;
  const bool wide = (a.ld_dh & 7) == 0 && (reinterpret_cast<uintptr_t>(a.dh) & 15u) == 0;
  const int64_t all = a.all_rows * per_row;
  // (eight pieces' labels are asked for at a time: no read passes the writes in front of it)
  for (int64_t i0 = ((int64_t)blockIdx.x - a.items) * 2048 + threadIdx.x; i0 < all; i0 += (int64_t)a.fills * 2048) {
    bool zero[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t row = min(i0 + u * 256, all - 1) / per_row;
      zero[u] = (a.mask != nullptr && a.mask[row] == 0) | ((uint32_t)a.labels[row] >= (uint32_t)a.C);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = i0 + u * 256;
      const int k = (int)(i % per_row) * 8;
      if (i >= all || k >= a.d || !zero[u]) continue;
      bf16_t *dst = a.dh + (size_t)(i / per_row * a.ld_dh) + k;
      if (wide && k + 8 <= a.d) {
        // (past the caches: 179 MB of zeros went through them in 64 us, 28 so)
        __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, reinterpret_cast<u32x4 *>(dst));
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (k + t < a.d) dst[t] = (bf16_t)0.f;
      }
    }
  }
}

// The end of a row, from its maximum, the others' sum and the label's logit.
struct RowEnd {
  float t, loss, log;
};
__device__ inline RowEnd end_row(float m, float others, float zl) {
  const float y = zl - m, own = exp_diff(zl, m), sum = others + own;
  RowEnd e;
  e.t = others / sum;
  e.loss = own > 0.5f * sum ? log1pf(others / own) : logf(sum) - y;
  e.log = -log2f(sum);  // (apart from the maximum, which may be so large that a sum of the two has lost it)
  return e;
}

// dh = inv_n t (sum_c p W_c / sum_c p - W_y), t = o / l: the mean of the other classes' weights less the label's.  What all classes' weights have in common is in
// both and has to cancel, so the mean's factors p are added up as the product takes them, rounded (held), not as they were.  A factor of one bf16 number is
// then off by 2^-8 of itself times its weights' distance from the mean; tiles with a factor above kCoarseTo of what the row has added up so far go around once
// more with what the first number has left (2^-16).  The factors that stay coarse cost at most 1.6e-3 sqrt(kCoarseTo) = 2.9e-4 of dh beside its own rounding's 1.65e-3.
// Relative error of dh, 2,000 rows of 256 columns, 41 classes whose weights share a column of 0 / 4 / 16 times what tells them apart: 1.69 / 2.03 / 4.82e-3 with
// coarse factors against the sum of the unrounded ones, 1.66e-3 throughout so; it differs from fp32 factors' by 3e-5 to 8e-5 (before 1e-3 to 5e-3).
// Calls in us with coarse factors / kCoarseTo 1/32 / 1/64 / 1/256: 46,657 x 100 x 10,007 (half labelled) 364 / 389 / 403 / 427, 517 x 256 x 50,021 170 / 180 / 184 / 187,
// 20,011 x 256 x 100,003 3,990 / 4,050 / 4,080 / 4,275, 232,965 x 256 x 41 132 / 135 / 135 / 135.
__device__ inline float mean_scale(float t, float held) { return held > 0.f ? t / held : 0.f; }

typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
// the sum of a lane's 16 factors
__device__ __forceinline__ float sum_of(const bf16x8 (&p)[2]) {
  const bf16x2 one = {(bf16_t)1.f, (bf16_t)1.f};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[i], p[i], 0, 1), one, s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[i], p[i], 2, 3), one, s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[i], p[i], 4, 5), one, s, false);
    s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p[i], p[i], 6, 7), one, s, false);
  }
  return s;
}

template <int DP, bool GRAD, bool DIRECT, int IN_REGS>
__global__ __launch_bounds__(256, kPerUnit<DP>) void head_rows_kernel(const RowsArgs a) {
  typedef Geometry<DP> G;
  typedef Owned<DP, IN_REGS> Own;
  __shared__ __attribute__((aligned(1024))) char tile0[G::tile_bytes];
  __shared__ __attribute__((aligned(1024))) char tile1[G::tile_bytes];
  __shared__ __attribute__((aligned(16))) float bias0[kTile];
  __shared__ __attribute__((aligned(16))) float bias1[kTile];
  __shared__ __attribute__((aligned(16))) char shared[Own::in_lds > 0 ? 4 * Own::in_lds * 1024 : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  if (GRAD && (int)blockIdx.x >= a.items) {
    fill_rows<DP>(a);
    return;
  }
  const Meta &meta = *a.meta;
  const int splits = meta.splits, item = blockIdx.x, row_tile = item / splits, split = item - row_tile * splits;
  if (row_tile >= meta.row_tiles) return;
  const int first = row_tile * kOwned + wave * 32;
  // (past the last labelled row: that row once more, whatever it gives is not written)
  f32x16 sum[DP / 32];
  clear<DP>(sum);
  float m = kNoMax, others = 0.f, zl = -INFINITY, held = 0.f;
  Places<DP> at(wave, lane);
  const int tiles = (a.C + kTile - 1) / kTile, begin = split * meta.tiles_per, end = min(tiles, begin + meta.tiles_per);
  auto load = [&](int tile, lds_char *dst, float *bias) {
    load_tile<DP>(a.W + (size_t)tile * kTile * DP, dst, wave, at.load);
    if (threadIdx.x < kTile / 4) load_lds16(a.bias + (size_t)tile * kTile + threadIdx.x * 4, (lds_char *)bias);
  };
  if (begin < end) load(begin, (lds_char *)tile0, bias0);
  // (past the last labelled row: that row once more, whatever it gives is not written)
  const Own own(DIRECT ? a.rows + (size_t)(a.list[min(first + (lane & 31), meta.n - 1)] * a.ld_rows) : a.rows + (size_t)(first + (lane & 31)) * DP,
                wave, lane, shared);
  const int label = a.label[first + (lane & 31)];
  auto step = [&](int tile, const lds_char *now, const float *bias, lds_char *next, float *next_bias) {
    wait_tile();
    if (tile + 1 < end) load(tile + 1, next, next_bias);
    at.renew();
    f32x16 z;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 b = *reinterpret_cast<const f32x4 *>(bias + 8 * q + 4 * h);
#pragma unroll
      for (int r = 0; r < 4; ++r) z[4 * q + r] = b[r];
    }
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(first_operand<DP>(now, at.first, ks), own(ks), z, 0, 0, 0);
    float most = z[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, z[i]);
    // The maximum follows only where a logit is more than 5 above it: p then stays below e^5, and the sums are rarely rescaled.
    if (__any(most > m + 5.f)) {
      const float up = fmaxf(m, fmaxf(most, __shfl_xor(most, 32))), f = exp_diff(m, up);
      m = up;
      others *= f;
      if constexpr (GRAD) {
        held *= f;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
#pragma unroll
          for (int t = 0; t < 16; ++t) sum[i][t] *= f;
      }
    }
    const int rel = label - tile * kTile;
    if (__any((uint32_t)rel < (uint32_t)kTile)) {  // the label's own term is kept out of the sums
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (rel == 8 * (i >> 2) + 4 * h + (i & 3)) {
          zl = z[i];
          z[i] = -INFINITY;
        }
      most = z[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, z[i]);
    }
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      z[i] = exp_diff(z[i], m);
      part += z[i];
    }
    others += part;
    if constexpr (GRAD) {
      // once, and where factors are large once more for what the first number has left of them
      bool again = __any(exp_diff(most, m) > kCoarseTo * others);
#pragma unroll 1
      for (;;) {
        bf16x8 p[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i >> 3][i & 7] = (bf16_t)z[i];
        held += sum_of(p);
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
          for (int t = 0; t < 2; ++t)
            sum[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_turned<DP>(now, at.second, dt, t), p[t], sum[dt], 0, 0, 0);
        if (!again) break;
        again = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] -= (float)p[i >> 3][i & 7];
      }
    }
  };
  for (int tile = begin; tile < end; tile += 2) {
    step(tile, (const lds_char *)tile0, bias0, (lds_char *)tile1, bias1);
    if (tile + 1 < end) step(tile + 1, (const lds_char *)tile1, bias1, (lds_char *)tile0, bias0);
  }
  others += __shfl_xor(others, 32);
  if constexpr (GRAD) held += __shfl_xor(held, 32);
  zl = __shfl(zl, (lane & 31) + 32 * ((label >> 2) & 1));  // from the half that had the label
  const int i = first + (lane & 31);
  if (splits > 1) {
    float *stat = a.part_stat + (size_t)item * 4 * kOwned + wave * 32 + (lane & 31);
    if (h == 0) {
      stat[0] = m;
      stat[kOwned] = others;
      stat[2 * kOwned] = zl;
      if constexpr (GRAD) stat[3 * kOwned] = held;
    }
    if constexpr (GRAD) {
      float *out = a.part + ((size_t)item * 4 + wave) * DP * 32 + (lane & 31);
#pragma unroll
      for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int t = 0; t < 16; ++t) out[(32 * dt + 8 * (t >> 2) + 4 * h + (t & 3)) * 32] = sum[dt][t];
    }
    return;
  }
  const bool on = i < meta.n;
  const RowEnd e = end_row(m, others, zl);
  const int row = on ? a.list[i] : -1;
  if (on && h == 0) {
    a.row_loss[row] = e.loss;
    a.max[i] = m;
    a.log[i] = e.log;
    a.t[i] = e.t;
  }
  if constexpr (GRAD) {
    const float scale = mean_scale(e.t, held);
    // A lane has four columns side by side of its row at a time; through LDS (the tiles are done with) a row's pieces come together: half of
    // the columns in a pass, 16-byte pieces permuted by the row.
    const bf16_t *wy = a.W + (size_t)max(label, 0) * DP;
    const bool wide = (a.ld_dh & 7) == 0 && (reinterpret_cast<uintptr_t>(a.dh) & 15u) == 0;
    constexpr int half = DP / 2, pieces = half / 8, rows_at_once = 64 / pieces;
    __syncthreads();
    lds_char *const room = (wave & 2 ? (lds_char *)tile1 : (lds_char *)tile0) + (wave & 1) * (G::tile_bytes / 2);
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      bf16x4 w[DP / 64][4];
#pragma unroll
      for (int dt = 0; dt < DP / 64; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) w[dt][q] = *reinterpret_cast<const bf16x4 *>(wy + pass * half + 32 * dt + 8 * q + 4 * h);
#pragma unroll
      for (int dt = 0; dt < DP / 64; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          bf16x4 o;
#pragma unroll
          for (int r = 0; r < 4; ++r) o[r] = (bf16_t)((sum[pass * (DP / 64) + dt][4 * q + r] * scale - e.t * (float)w[dt][q][r]) * a.inv_n);
          const int piece = 4 * dt + q, at_row = lane & 31;
          *reinterpret_cast<LDS_AS bf16x4 *>(room + at_row * DP + ((piece ^ (at_row & (pieces - 1))) << 4) + 8 * h) = o;
        }
      // (read by the wave that wrote it)
#pragma unroll
      for (int k = 0; k < 32 / rows_at_once; ++k) {
        const int at_row = k * rows_at_once + lane / pieces, piece = lane % pieces, c = pass * half + piece * 8;
        const bf16x8 o = *reinterpret_cast<const LDS_AS bf16x8 *>(room + at_row * DP + ((piece ^ (at_row & (pieces - 1))) << 4));
        const int to = __shfl(row, at_row);
        if (to < 0) continue;
        bf16_t *dst = a.dh + (size_t)((int64_t)to * a.ld_dh) + c;
        if (wide && c + 8 <= a.d) {
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), reinterpret_cast<u32x4 *>(dst));  // (41 classes: 156 us through the caches, 144 so)
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (c + t < a.d) dst[t] = o[t];
        }
      }
    }
  }
}

// Joins the class ranges of 32 rows and 16 columns (a workgroup): each range has its own maximum.
constexpr int kMaxSplits = 64;
constexpr int kJoinColumns = 16;
template <int DP, bool GRAD>
__global__ __launch_bounds__(256) void head_join_kernel(const RowsArgs a) {
  const Meta &meta = *a.meta;
  const int splits = meta.splits, row_tile = blockIdx.x >> 2, wave = blockIdx.x & 3, d0 = blockIdx.y * kJoinColumns;
  if (splits == 1 || row_tile >= meta.row_tiles) return;
  __shared__ float stat[GRAD ? 4 : 3][kMaxSplits][32], red[8][32];
  __shared__ float turned[32][kJoinColumns + 1];
  __shared__ float scale[32], ts[32];
  __shared__ int label[32], row[32];
  const int n = threadIdx.x & 31, g = threadIdx.x >> 5, i = row_tile * kOwned + wave * 32 + n;
  const int64_t item0 = (int64_t)row_tile * splits;
  const int lab = a.label[i];
  float m = kNoMax;
  for (int s = g; s < splits; s += 8) {
    const float *p = a.part_stat + (size_t)(item0 + s) * 4 * kOwned + wave * 32 + n;
    stat[0][s][n] = p[0];
    stat[1][s][n] = p[kOwned];
    stat[2][s][n] = p[2 * kOwned];
    if constexpr (GRAD) stat[3][s][n] = p[3 * kOwned];
    m = fmaxf(m, p[0]);
  }
  red[g][n] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) m = fmaxf(m, red[k][n]);
  __syncthreads();
  for (int s = g; s < splits; s += 8) {  // from maxima to factors
    const float f = exp_diff(stat[0][s][n], m);
    stat[0][s][n] = f;
    stat[1][s][n] *= f;
  }
  __syncthreads();
  if (g == 0) {
    float others = 0.f, held = 0.f;
    for (int s = 0; s < splits; ++s) {
      others += stat[1][s][n];
      if constexpr (GRAD) held += stat[0][s][n] * stat[3][s][n];
    }
    const float zl = lab >= 0 ? stat[2][lab / kTile / meta.tiles_per][n] : -INFINITY;
    const RowEnd e = end_row(m, others, zl);
    const bool on = i < meta.n;
    scale[n] = mean_scale(e.t, held);
    ts[n] = e.t;
    label[n] = on ? lab : -1;
    row[n] = on ? a.list[i] : -1;
    if (on && d0 == 0) {
      a.row_loss[a.list[i]] = e.loss;
      a.max[i] = m;
      a.log[i] = e.log;
      a.t[i] = e.t;
    }
  }
  if (!GRAD || a.dh == nullptr) return;
  const float *part = a.part + (((size_t)item0 * 4 + wave) * DP + d0 + g) * 32 + n;
  float x = 0.f, y = 0.f;
#pragma unroll 8
  for (int s = 0; s < splits; ++s) {
    const float f = stat[0][s][n];
    x = fmaf(part[(size_t)s * 4 * DP * 32], f, x);
    y = fmaf(part[(size_t)s * 4 * DP * 32 + 8 * 32], f, y);
  }
  turned[n][g] = x;
  turned[n][g + 8] = y;
  __syncthreads();
  for (int k = threadIdx.x; k < 32 * kJoinColumns; k += 256) {
    const int r = k / kJoinColumns, c = k % kJoinColumns;
    if (label[r] >= 0 && d0 + c < a.d)
      a.dh[(size_t)((int64_t)row[r] * a.ld_dh) + d0 + c] =
          (bf16_t)((turned[r][c] * scale[r] - ts[r] * (float)a.W[(size_t)label[r] * DP + d0 + c]) * a.inv_n);
  }
}

struct ClassesArgs {
  const Meta *meta;
  const bf16_t *rows, *W;  // as in RowsArgs
  int64_t ld_rows;
  const int32_t *list;
  const float *bias;
  const float *stats;      // of the labelled rows, padded_rows each: maximum, -log2 sum, label (int), o / l
  int64_t padded_rows;
  int32_t C, d, class_tiles;
  float inv_n;
  float *dW, *db;          // "+=", either may be NULL
  float *part;             // [slot][DP][part_cols]
  float *part_db;          // [slot][kOwned]
  int32_t part_cols;       // kOwned, or a single class tile's columns in whole waves
  int32_t by_tile;         // which slots, see slot_of
};
// The classes kernel's work, (class tile, row step) pairs in that order, is cut into one run per workgroup (group g: from pair
// total g / groups on), so that all of them end together: with a workgroup per class tile, 782 class tiles in rounds of 512 took 2.88 ms.  A run's
// class tiles that are whole are added to dW and db by the kernel; of one that is cut, a group writes its share.
__device__ inline int64_t run_begin(int64_t total, int groups, int g) { return total * g / groups; }
// Where: a run has two cut tiles at most, the one that it begins in and the one that it ends in.  And from share to share group or tile go up by one, never down, so
// that their sum is a place of its own too: with few class tiles that is half the room (232,965 rows x 256, 41 classes: 34 MB, 134 MB with two slots a group
// of 128 columns each).
__device__ inline int64_t slot_of(const ClassesArgs &a, int group, int class_tile, bool begins) {
  return a.by_tile ? (int64_t)group + class_tile : 2 * (int64_t)group + (begins ? 0 : 1);
}

//
// EXACT: 16 bits of g are up to 2^-16 of a single term of dW.  Added up over many labelled rows of a class that is less than what an fp32 product's own sum is off by;
// over few it is not.  So where a slab's labelled rows are kExactRows at most, or fewer than kExactPerClass a class, the tiles with large g (a label's, a sure
// row's: what a column of dW consists of where rows have its class) go around once more for the third bf16 number, which is all of a g's bits; g in tiles
// without a large one keep 16.  Relative error of dW (norm / worst column), 16 bits, all, the fp32 products of the plain form:
//   370 rows of 96 classes              1.6e-6          2.3e-7          2.3e-7
//   17,000 of 1,000   (17 a class)      1.2e-6 / 4.3e-6 3.0e-7 / 0.6e-6 7.6e-7 / 1.9e-6     calls at width 256: 138 / 152 us
//   40,000 of 1,000   (40)              1.0e-6 / 3.7e-6 4.4e-7 / 1.0e-6 1.0e-6 / 2.2e-6                         180 / 236
//   17,000 of 172     (99)              7.0e-7 / 2.2e-6 3.3e-7 / 0.7e-6 1.4e-6 / 2.0e-6     width 128:           59 / 65
//   400,000 of 1,000  (400)             5.5e-7 / 2.2e-6 4.6e-7 / 1.4e-6 1.4e-6 / 3.0e-6                         1,023 / 1,477
//   120,000 of 41     (2,900)           2.8e-7 / 1.0e-6 2.2e-7 / 0.6e-6 1.4e-6 / 1.7e-6                         108 / 128
// (18,010 of 100,003, width 256: 4,000 / 4,110 us; 23,300 of 10,007, width 100: 385 / 422.)
template <int DP, bool DIRECT, bool EXACT, int IN_REGS>
__global__ __launch_bounds__(256, kPerUnit<DP>) void head_classes_kernel(const ClassesArgs a) {
  typedef Geometry<DP> G;
  typedef Owned<DP, IN_REGS> Own;
  struct Stats {
    float max[kTile];
    float log[kTile];
    int32_t label[kTile];
    float t[kTile];
  };
  __shared__ __attribute__((aligned(1024))) char tile0[G::tile_bytes];
  __shared__ __attribute__((aligned(1024))) char tile1[G::tile_bytes];
  __shared__ __attribute__((aligned(16))) Stats stats0;
  __shared__ __attribute__((aligned(16))) Stats stats1;
  __shared__ __attribute__((aligned(16))) char shared[Own::in_lds > 0 ? 4 * Own::in_lds * 1024 : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int row_steps = a.meta->row_steps, groups = a.meta->groups, n = a.meta->n, group = blockIdx.x;
  if (group >= groups || EXACT != (n <= kExactRows || n < (int64_t)kExactPerClass * a.C)) return;
  const int64_t total = (int64_t)a.class_tiles * row_steps, run0 = run_begin(total, groups, group), run1 = run_begin(total, groups, group + 1);
  Places<DP> at(wave, lane);
  int32_t index[DIRECT ? G::loads : 1];  // of the rows that this lane loads next
  auto look_up = [&](int tile) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int q = 0; q < G::loads; ++q) index[q] = a.list[min(tile * kTile + q * 4 * G::rows_per_load + wave * G::rows_per_load + lane / G::chunks, n - 1)];
    }
  };
  auto load = [&](int tile, lds_char *dst, Stats *st) {
    if constexpr (DIRECT) {
      // (rows past the last labelled one: that one again, times g = 0)
#pragma unroll
      for (int q = 0; q < G::loads; ++q) {
        constexpr int step = 4 * G::rows_per_load;
        const uint32_t turn = (lds_swizzle<DP>(q * step) ^ lds_swizzle<DP>(0)) << 4;
        load_lds16(reinterpret_cast<const char *>(a.rows + (size_t)(index[q] * a.ld_rows)) + ((at.load ^ turn) & (G::row_bytes - 1)),
                   dst + q * step * G::row_bytes + wave * 1024);
      }
    } else {
      load_tile<DP>(a.rows + (size_t)tile * kTile * DP, dst, wave, at.load);
    }
    if (threadIdx.x < kTile)
      load_lds16(a.stats + (size_t)(threadIdx.x >> 3) * a.padded_rows + (size_t)tile * kTile + (threadIdx.x & 7) * 4, (lds_char *)st);
  };
  for (int64_t pair = run0; pair < run1;) {
    const int class_tile = (int)(pair / row_steps), begin = (int)(pair - (int64_t)class_tile * row_steps);
    const int end = (int)min((int64_t)row_steps, begin + (run1 - pair));
    const int first = class_tile * kOwned + wave * 32, c = first + (lane & 31);
    const bool idle = first >= a.C;  // this wave has no classes; it still loads
    __syncthreads();  // the last class tile's streamed rows are done with
    look_up(begin);
    const Own own(a.W + (size_t)c * DP, wave, lane, shared);
    const float bias = a.bias[c];
    f32x16 sum[DP / 32];
    clear<DP>(sum);
    float g_sum = 0.f, g_low = 0.f;
    load(begin, (lds_char *)tile0, &stats0);
    look_up(begin + 1);
    auto step = [&](int tile, const lds_char *now, const Stats *st, lds_char *next, Stats *next_st) {
      wait_tile();
      if (tile + 1 < end) {
        load(tile + 1, next, next_st);
        look_up(tile + 2);
      }
      if (idle) return;
      // Once, and where EXACT once more for the last bits of tiles that have large g: they are made again, since keeping them takes registers that are not there.
      bool again = false;
#pragma unroll 1
      for (;;) {
        at.renew();
        // (the bias first, as in the rows kernel: the same logits to the last bit, so that large ones meet their own maximum)
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = bias;
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(first_operand<DP>(now, at.first, ks), own(ks), z, 0, 0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 m = *reinterpret_cast<const f32x4 *>(st->max + 8 * q + 4 * h), l = *reinterpret_cast<const f32x4 *>(st->log + 8 * q + 4 * h);
#pragma unroll
          for (int r = 0; r < 4; ++r) z[4 * q + r] = __builtin_amdgcn_exp2f(fmaf(z[4 * q + r] - m[r], kLog2e, l[r]));
        }
        if (__any((uint32_t)(st->label[lane & 31] - first) < 32u)) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const i32x4 y = *reinterpret_cast<const i32x4 *>(st->label + 8 * q + 4 * h);
            const f32x4 t = *reinterpret_cast<const f32x4 *>(st->t + 8 * q + 4 * h);
#pragma unroll
            for (int r = 0; r < 4; ++r) z[4 * q + r] = y[r] == c ? -t[r] : z[4 * q + r];
          }
        }
        float largest = 0.f;
        if (!again) {
          // db takes g as it is; its long sum is compensated
          float part = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            part += z[i];
            if constexpr (EXACT) largest = fmaxf(largest, fabsf(z[i]));
          }
          const float y = part - g_low, s = g_sum + y;
          g_low = (s - g_sum) - y;
          g_sum = s;
        }
        const bool more = EXACT && __any(largest > kExactFrom);
        bf16x8 high[2], low[2];  // g = high + low to 16 bits, + a third to all of them
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          high[i >> 3][i & 7] = (bf16_t)z[i];
          z[i] -= (float)high[i >> 3][i & 7];
          low[i >> 3][i & 7] = (bf16_t)z[i];
        }
        if (again) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            high[i >> 3][i & 7] = (bf16_t)(z[i] - (float)low[i >> 3][i & 7]);
            low[i >> 3][i & 7] = (bf16_t)0.f;
          }
        }
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const bf16x8 x = lds_turned<DP>(now, at.second, dt, t);
            sum[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, high[t], sum[dt], 0, 0, 0);
            sum[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, low[t], sum[dt], 0, 0, 0);
          }
        if (!more) break;
        again = true;
      }
    };
    for (int tile = begin; tile < end; tile += 2) {
      step(tile, (const lds_char *)tile0, &stats0, (lds_char *)tile1, &stats1);
      if (tile + 1 < end) step(tile + 1, (const lds_char *)tile1, &stats1, (lds_char *)tile0, &stats0);
    }
    const bool whole = begin == 0 && end == row_steps;
    const int64_t slot = slot_of(a, group, class_tile, pair == run0);
    pair += end - begin;
    if (c >= a.C) continue;
    g_sum += __shfl_xor(g_sum, 32);
    if (a.db != nullptr && h == 0) {
      if (whole)
        a.db[c] += g_sum * a.inv_n;
      else
        a.part_db[slot * kOwned + wave * 32 + (lane & 31)] = g_sum;
    }
    if (a.dW == nullptr) continue;
    float *to = whole ? a.dW + c : a.part + slot * DP * a.part_cols + wave * 32 + (lane & 31);
    int64_t stride = whole ? a.C : a.part_cols;
    const int d = DIRECT ? DP : a.d;
    asm volatile("" : "+s"(stride));  // (or the compiler makes all addresses ahead of the loop, and spills)
    to += 4 * h * stride;
    if (whole) {
      // (16 at a time: what is added to has to be read, and no read passes the writes in front of it)
#pragma unroll
      for (int dt = 0; dt < DP / 32; ++dt) {
        float old[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const int k = 32 * dt + 8 * (t >> 2) + (t & 3);
          old[t] = k + 4 * h < d ? to[k * stride] : 0.f;
        }
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const int k = 32 * dt + 8 * (t >> 2) + (t & 3);
          if (k + 4 * h < d) to[k * stride] = old[t] + sum[dt][t] * a.inv_n;
        }
      }
    } else {
#pragma unroll
      for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          const int k = 32 * dt + 8 * (t >> 2) + (t & 3);
          if (k + 4 * h < d) to[k * stride] = sum[dt][t];
        }
    }
  }
}

// The shares of the class tiles that were cut, in the order of their rows.  A workgroup: 64 classes, four rows k of dW (row d is db) side
// by side, or one row whose shares are added up in four runs where there are many.
template <int DP>
__global__ __launch_bounds__(256) void head_reduce_kernel(const ClassesArgs a) {
  __shared__ float red[4][64];
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6, row_steps = a.meta->row_steps, groups = a.meta->groups;
  const int class_tile = blockIdx.x >> 1, in_tile = (blockIdx.x & 1) * 64 + tx, c = class_tile * kOwned + in_tile;
  if (groups == 0) return;
  const int64_t total = (int64_t)a.class_tiles * row_steps, from = (int64_t)class_tile * row_steps, to = from + row_steps;
  // the groups that have the tile's first and last pair
  auto owner = [&](int64_t pair) {
    int g = (int)min((int64_t)groups - 1, (pair * groups + groups - 1) / total);
    while (run_begin(total, groups, g) > pair) --g;
    while (g + 1 < groups && run_begin(total, groups, g + 1) <= pair) ++g;
    return g;
  };
  const int g0 = owner(from), g1 = owner(to - 1);
  if (g0 == g1) return;  // whole workgroup: nothing was cut
  const bool begins = run_begin(total, groups, g0) >= from;  // the first of them, in this tile
  auto share = [&](int k, int g) {
    const int64_t slot = slot_of(a, g, class_tile, g != g0 || begins);
    return k == a.d ? a.part_db[slot * kOwned + in_tile] : a.part[(slot * DP + k) * a.part_cols + in_tile];
  };
  auto wanted = [&](int k) { return k < a.d ? a.dW != nullptr : k == a.d && a.db != nullptr; };
  auto add = [&](int k, float x) {
    float *dst = k == a.d ? a.db + c : a.dW + (size_t)k * a.C + c;
    *dst += a.inv_n * x;
  };
  const int shares = g1 - g0 + 1;
  if (shares <= 8) {
    for (int k = blockIdx.y * 4 + ty; k <= a.d; k += gridDim.y * 4)
      if (wanted(k) && c < a.C) {
        float x = 0.f;
        for (int g = g0; g <= g1; ++g) x += share(k, g);
        add(k, x);
      }
    return;
  }
  for (int k = blockIdx.y; k <= a.d; k += gridDim.y) {
    if (!wanted(k)) continue;  // whole workgroup
    const int per = (shares + 3) / 4, r0 = g0 + ty * per, r1 = min(g1 + 1, r0 + per);
    float x = 0.f;
    if (c < a.C) {
      int g = r0;
      for (; g + 8 <= r1; g += 8) {
        float v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = share(k, g + t);
        x += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
      }
      for (; g < r1; ++g) x += share(k, g);
    }
    red[ty][tx] = x;
    __syncthreads();
    if (ty == 0 && c < a.C) add(k, (red[0][tx] + red[1][tx]) + (red[2][tx] + red[3][tx]));
    __syncthreads();
  }
}

struct PrepareArgs {
  const bf16_t *h, *W;
  int64_t ld_h;
  const float *bias_in;
  const int32_t *labels;
  const uint8_t *mask;
  int64_t rows;
  int32_t d, C, DP, padded_classes;
  int32_t *counts;        // labelled rows of every kMetaBlock
  int32_t n_counts;
  Meta *meta;
  int32_t *list;
  int64_t padded_rows;
  bf16_t *packed, *Wt;
  float *bias;
  float *stats;           // maximum, -log2 sum, label, t
  float *row_loss;
  int32_t max_splits, round;
};

// Workgroups [0, n_counts) count labelled rows; the others turn the weights, 64 x 64 at a time, and pad the biases.
__global__ __launch_bounds__(256) void head_count_kernel(const PrepareArgs a) {
  __shared__ bf16_t turned[64][66];
  __shared__ int total;
  if ((int)blockIdx.x < a.n_counts) {
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    const int64_t r0 = (int64_t)blockIdx.x * kMetaBlock;
    int count = 0;
    for (int i = threadIdx.x; i < kMetaBlock; i += 256) {
      const bool on = r0 + i < a.rows && is_labelled(a.labels, a.mask, r0 + i, a.C);
      count += __popcll(__ballot(on));  // the wave's
    }
    if ((threadIdx.x & 63) == 0) atomicAdd(&total, count);
    __syncthreads();
    if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
    return;
  }
  const int tk = a.DP / 64, block = blockIdx.x - a.n_counts, k0 = block % tk * 64, c0 = block / tk * 64;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  if (k0 == 0 && threadIdx.x < 64) {
    const int c = c0 + threadIdx.x;
    float b = -INFINITY;
    if (c < a.C) b = a.bias_in == nullptr ? 0.f : a.bias_in[c];
    a.bias[c] = b;
  }
#pragma unroll
  for (int i = 0; i < 64; i += 4) {
    const int k = k0 + y + i, c = c0 + x;
    turned[x][y + i] = k < a.d && c < a.C ? a.W[(size_t)k * a.C + c] : (bf16_t)0.f;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 4) a.Wt[(size_t)(c0 + y + i) * a.DP + k0 + x] = turned[y + i][x];
}

// The list of labelled rows, in their order; what hangs on their number.
__global__ __launch_bounds__(256) void head_list_kernel(const PrepareArgs a) {
  __shared__ int before, in_wave[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) before = 0;
  __syncthreads();
  int mine = 0;
  for (int i = threadIdx.x; i < (int)blockIdx.x; i += 256) mine += a.counts[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
  if (lane == 0) atomicAdd(&before, mine);
  __syncthreads();
  int at = before;
  const int64_t r0 = (int64_t)blockIdx.x * kMetaBlock;
  int32_t *label = reinterpret_cast<int32_t *>(a.stats + 2 * a.padded_rows);
  for (int i = 0; i < kMetaBlock; i += 256) {
    const int64_t r = r0 + i + threadIdx.x;
    const bool in = r < a.rows, on = in && is_labelled(a.labels, a.mask, r, a.C);
    const uint64_t votes = __ballot(on);
    if (lane == 0) in_wave[wave] = __popcll(votes);
    __syncthreads();
    int pos = at + __popcll(votes & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) pos += in_wave[w];
    if (on) {
      a.list[pos] = (int32_t)r;
      label[pos] = a.labels[r];
    } else if (in) {
      a.row_loss[r] = 0.f;
    }
    at += in_wave[0] + in_wave[1] + in_wave[2] + in_wave[3];
    __syncthreads();
  }
  if ((int)blockIdx.x == a.n_counts - 1 && wave == 0) {
    Meta m{};
    m.n = at;
    m.row_tiles = (at + kOwned - 1) / kOwned;
    // class ranges: as many as make the last round of workgroups a full one.  A range costs its tiles and about eight more (its
    // rows, its partial sums and their reading).  Every lane weighs one number of ranges.
    static_assert(kMaxSplits == 64, "a lane each");
    const int tiles = (a.C + kTile - 1) / kTile, tried = lane + 1;
    int per = (tiles + tried - 1) / tried;
    const int real = (tiles + per - 1) / per;
    const int64_t items = (int64_t)m.row_tiles * real;
    const bool may = tried <= a.max_splits && (real == 1 || items <= kRowItems);
    uint64_t cost = may ? (uint64_t)(((items + a.round - 1) / a.round * (per + (real > 1 ? 8 : 4))) << 6 | lane) : ~0ull;  // the fewest of equals
    uint64_t least = cost;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) least = min(least, (uint64_t)__shfl_xor((unsigned long long)least, o));
    m.splits = __shfl(real, (int)(least & 63));
    m.tiles_per = __shfl(per, (int)(least & 63));
    m.row_steps = (at + kTile - 1) / kTile;
    // Equal runs (of four steps at least) where that is faster than whole class tiles in rounds: the shares of cut tiles take as long to write and
    // to add up as about 24 steps.  517 rows x 50,021 classes (17 steps, 391 class tiles): 67 + 75 us in equal runs, 79 in whole tiles.
    const int64_t class_tiles = a.padded_classes / kOwned, pairs = class_tiles * m.row_steps;
    const int64_t whole = (class_tiles + a.round - 1) / a.round * (m.row_steps + 2), equal = pairs / a.round + 24;
    m.groups = m.row_steps == 0 ? 0 : whole <= equal ? (int32_t)class_tiles : (int32_t)min((int64_t)a.round, (pairs + 3) / 4);
    if (lane == 0) *a.meta = m;
    // what stands behind the last labelled row, up to a whole workgroup's
    for (int i = at + lane; i < m.row_tiles * kOwned; i += 64) {
      a.stats[i] = INFINITY;
      a.stats[a.padded_rows + i] = a.stats[3 * a.padded_rows + i] = 0.f;
      label[i] = -1;
    }
  }
}

// The labelled rows side by side, zeros from d to DP and behind the last of them up to whole workgroups.  A thread per eight columns.
__global__ __launch_bounds__(256) void head_pack_kernel(const PrepareArgs a) {
  const int per_row = a.DP / 8;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / per_row;
  const int k = (threadIdx.x % per_row) * 8, n = a.meta->n;
  if (i >= (int64_t)(n + kOwned - 1) / kOwned * kOwned) return;
  bf16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
  if (i < n) {
    const bf16_t *src = a.h + (size_t)(a.list[i] * a.ld_h) + k;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (k + t < a.d) v[t] = src[t];
  }
  *reinterpret_cast<bf16x8 *>(a.packed + (size_t)i * a.DP + k) = v;
}

struct FusedPlan {
  int64_t rows = 0, padded_rows = 0, max_items = 0;
  int d = 0, C = 0, DP = 0, padded_classes = 0, n_counts = 0, max_splits = 1, class_tiles = 0, part_cols = kOwned;
  bool by_tile = false;
  size_t counts = 0, meta = 0, list = 0, stats = 0, packed = 0, Wt = 0, bias = 0, part = 0, part_stat = 0, part_dW = 0, part_db = 0, total = 0;
};
constexpr int64_t kFusedRows = (int64_t)1 << 20;  // of a slab: their packed copy is half a gigabyte at most

bool fused_takes(int d, int dtype) { return dtype == GNNSTAGE_BF16 && d <= 256; }

// Rows of the very width in whole 16-byte pieces are read where they are, others from a packed copy.
bool read_in_place(const void *h, int64_t ld_h, int d) {
  return (d == 64 || d == 128 || d == 256) && ld_h % 8 == 0 && (reinterpret_cast<uintptr_t>(h) & 15u) == 0;
}

FusedPlan fused_plan(int64_t all_rows, int d, int C, bool grads, bool in_place) {
  FusedPlan p;
  const int64_t rows = std::min(all_rows, kFusedRows);
  p.rows = rows;
  p.d = d;
  p.C = C;
  p.DP = d <= 64 ? 64 : d <= 128 ? 128 : 256;
  const int64_t row_tiles = std::max<int64_t>(1, (rows + kOwned - 1) / kOwned);
  p.padded_rows = row_tiles * kOwned;
  p.class_tiles = (C + kOwned - 1) / kOwned;
  p.padded_classes = p.class_tiles * kOwned;
  p.n_counts = (int)std::max<int64_t>(1, (rows + kMetaBlock - 1) / kMetaBlock);
  // class ranges of eight tiles at least
  p.max_splits = std::max(1, std::min(kMaxSplits, (C + 8 * kTile - 1) / (8 * kTile)));
  p.max_items = std::min(row_tiles * p.max_splits, std::max<int64_t>(row_tiles, kRowItems));
  size_t off = 0;
  auto take = [&](size_t b) {
    const size_t at = off;
    off = align256(off + b);
    return at;
  };
  p.counts = take(sizeof(int32_t) * (size_t)p.n_counts);
  p.meta = take(sizeof(Meta));
  p.list = take(sizeof(int32_t) * (size_t)p.padded_rows);
  p.stats = take(4 * sizeof(float) * (size_t)p.padded_rows);
  p.Wt = take(2 * (size_t)p.padded_classes * p.DP);
  p.bias = take(sizeof(float) * (size_t)p.padded_classes);
  const int64_t part_items = p.max_splits > 1 ? std::min<int64_t>(p.max_items, kRowItems) : 0;
  p.part_stat = take(sizeof(float) * 4 * kOwned * (size_t)part_items);
  p.part = take(grads ? sizeof(float) * (size_t)kOwned * p.DP * (size_t)part_items : 0);
  const int64_t groups = grads ? std::min<int64_t>(round_of(p.DP), ((int64_t)p.class_tiles * ((rows + kTile - 1) / kTile) + 3) / 4) : 0;
  p.by_tile = p.class_tiles < groups;
  p.part_cols = p.class_tiles == 1 ? round_up(C, 32) : kOwned;
  const int64_t slots = p.by_tile ? groups + p.class_tiles : 2 * groups;
  p.part_dW = take(sizeof(float) * (size_t)slots * p.DP * p.part_cols);
  p.part_db = take(sizeof(float) * (size_t)slots * kOwned);
  // last, so that a call whose rows need no copy can do without
  p.packed = off;
  p.total = align256(off + (in_place ? 0 : 2 * (size_t)p.padded_rows * p.DP));
  return p;
}

// Owned operands in registers, of d / 16 (the others in LDS): as many as the registers reach for.  Width 256, 18 k rows x 100 k classes: rows kernel
// 8 / 12 / 16 4.30 / 4.26 / 4.24 ms (all of them, then), classes kernel 4 / 8 / 10 / 12 5.07 / 4.24 / 4.24 / 4.25 ms.
template <int DP>
constexpr int kClassesInRegs = DP == 256 ? 10 : DP == 128 ? 6 : 4;

// a slab of at most p.rows rows; first: the weights are not there yet
template <int DP, bool DIRECT>
int run_fused(const FusedPlan &p, const Call &c, int64_t rows, bool first, hipStream_t s) {
  auto at = [&](size_t off) { return c.ws + off; };
  PrepareArgs a{};
  a.h = static_cast<const bf16_t *>(c.h);
  a.W = static_cast<const bf16_t *>(c.W);
  a.ld_h = c.ld_h;
  a.bias_in = c.bias;
  a.labels = c.labels;
  a.mask = c.mask;
  a.rows = rows;
  a.d = p.d;
  a.C = p.C;
  a.DP = DP;
  a.padded_classes = p.padded_classes;
  a.counts = reinterpret_cast<int32_t *>(at(p.counts));
  a.n_counts = (int)((rows + kMetaBlock - 1) / kMetaBlock);
  a.meta = reinterpret_cast<Meta *>(at(p.meta));
  a.list = reinterpret_cast<int32_t *>(at(p.list));
  a.padded_rows = p.padded_rows;
  a.packed = reinterpret_cast<bf16_t *>(at(p.packed));
  a.Wt = reinterpret_cast<bf16_t *>(at(p.Wt));
  a.bias = reinterpret_cast<float *>(at(p.bias));
  a.stats = reinterpret_cast<float *>(at(p.stats));
  a.row_loss = c.row_loss;
  a.max_splits = p.max_splits;
  a.round = round_of(DP);
  const unsigned turn_blocks = first ? (unsigned)(p.padded_classes / 64 * (DP / 64)) : 0;
  hipLaunchKernelGGL(head_count_kernel, dim3((unsigned)a.n_counts + turn_blocks), dim3(256), 0, s, a);
  HEAD_TRY(hipGetLastError());
  hipLaunchKernelGGL(head_list_kernel, dim3((unsigned)a.n_counts), dim3(256), 0, s, a);
  HEAD_TRY(hipGetLastError());
  const int64_t row_tiles = (rows + kOwned - 1) / kOwned;
  if (!DIRECT) {
    hipLaunchKernelGGL(head_pack_kernel, dim3((unsigned)(row_tiles * kOwned * (DP / 8) / 256)), dim3(256), 0, s, a);
    HEAD_TRY(hipGetLastError());
  }

  RowsArgs r{};
  r.meta = a.meta;
  r.rows = DIRECT ? a.h : a.packed;
  r.ld_rows = c.ld_h;
  r.W = a.Wt;
  r.bias = a.bias;
  r.label = reinterpret_cast<const int32_t *>(a.stats + 2 * p.padded_rows);
  r.list = a.list;
  r.C = p.C;
  r.d = p.d;
  r.inv_n = c.inv_n;
  r.row_loss = c.row_loss;
  r.dh = static_cast<bf16_t *>(c.dh);
  r.ld_dh = c.ld_dh;
  r.max = a.stats;
  r.log = a.stats + p.padded_rows;
  r.t = a.stats + 3 * p.padded_rows;
  r.part = reinterpret_cast<float *>(at(p.part));
  r.part_stat = reinterpret_cast<float *>(at(p.part_stat));
  constexpr int kAll = DP / 16;
  const bool sums = c.dh != nullptr;
  r.items = (int32_t)std::min(row_tiles * p.max_splits, std::max<int64_t>(row_tiles, kRowItems));
  r.fills = sums ? (int32_t)std::min<int64_t>(8192, (rows * (DP / 8) + 2047) / 2048) : 0;
  r.labels = c.labels;
  r.mask = c.mask;
  r.all_rows = rows;
  hipLaunchKernelGGL((sums ? head_rows_kernel<DP, true, DIRECT, kAll> : head_rows_kernel<DP, false, DIRECT, kAll>),
                     dim3((unsigned)(r.items + r.fills)), dim3(256), 0, s, r);
  HEAD_TRY(hipGetLastError());
  if (p.max_splits > 1) {
    const unsigned blocks = 4u * (unsigned)std::min<int64_t>(row_tiles, kRowItems);
    hipLaunchKernelGGL((sums ? head_join_kernel<DP, true> : head_join_kernel<DP, false>), dim3(blocks, sums ? (unsigned)((p.d + kJoinColumns - 1) / kJoinColumns) : 1u),
                       dim3(256), 0, s, r);
    HEAD_TRY(hipGetLastError());
  }
  if (!c.dW && !c.db) return hipSuccess;
  ClassesArgs k{};
  k.meta = a.meta;
  k.rows = r.rows;
  k.ld_rows = c.ld_h;
  k.list = a.list;
  k.W = a.Wt;
  k.bias = a.bias;
  k.stats = a.stats;
  k.padded_rows = p.padded_rows;
  k.C = p.C;
  k.d = p.d;
  k.class_tiles = p.class_tiles;
  k.inv_n = c.inv_n;
  k.dW = c.dW;
  k.db = c.db;
  k.part = reinterpret_cast<float *>(at(p.part_dW));
  k.part_db = reinterpret_cast<float *>(at(p.part_db));
  k.part_cols = p.part_cols;
  k.by_tile = p.by_tile;
  const int64_t groups = std::max<int64_t>(round_of(p.DP), p.class_tiles);  // at most
  hipLaunchKernelGGL((head_classes_kernel<DP, DIRECT, true, kClassesInRegs<DP>>), dim3((unsigned)groups), dim3(256), 0, s, k);
  HEAD_TRY(hipGetLastError());
  if (rows > kExactRows && rows >= (int64_t)kExactPerClass * p.C) {  // how many have labels is known to the device: one of the two returns at once
    hipLaunchKernelGGL((head_classes_kernel<DP, DIRECT, false, kClassesInRegs<DP>>), dim3((unsigned)groups), dim3(256), 0, s, k);
    HEAD_TRY(hipGetLastError());
  }
  // many shares of few class tiles: a workgroup per row of dW; few shares of many: some rows each
  const unsigned gy = p.class_tiles < 64 ? (unsigned)p.d + 1 : 8u;
  hipLaunchKernelGGL(head_reduce_kernel<DP>, dim3(2u * (unsigned)p.class_tiles, gy), dim3(256), 0, s, k);
  return (int)hipGetLastError();
}
template <int DP>
int run_fused(const FusedPlan &p, const Call &c, int64_t rows, bool first, hipStream_t s) {
  return read_in_place(c.h, c.ld_h, p.d) ? run_fused<DP, true>(p, c, rows, first, s) : run_fused<DP, false>(p, c, rows, first, s);
}

size_t workspace_bytes_of(const Plan &p, bool in_place) {
  return fused_takes(p.d, p.dtype) ? fused_plan(p.rows, p.d, p.C, p.grads, in_place).total : p.total;
}

}  // namespace

size_t head_workspace_bytes(const void *h, int64_t ld_h, int64_t rows, int d, int n_classes, int dtype) {
  Plan p;
  std::string err;
  if (!make_plan(rows, d, n_classes, dtype, true, p, err)) {
    train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: " + err);
    return 0;
  }
  return workspace_bytes_of(p, read_in_place(h, ld_h, d));
}

extern "C" size_t gnntrain_head_xent_workspace_size(int64_t rows, int32_t d, int32_t n_classes, int32_t dtype, int32_t want_grads) try {
  Plan p;
  std::string err;
  if (!make_plan(rows, d, n_classes, dtype, want_grads != 0, p, err)) {
    train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: " + err);
    return 0;
  }
  return workspace_bytes_of(p, false);  // whether rows can be read in place is not known from their sizes
}
GNNSTAGE_GUARD_SIZE

extern "C" int gnntrain_head_xent(const void *h, int64_t ld_h, const void *W, int32_t dtype, const float *bias, const int32_t *labels,
                                  const uint8_t *mask, int64_t rows, int32_t d, int32_t n_classes, float inv_n_train, float *row_loss, void *dh,
                                  int64_t ld_dh, float *dW, float *db, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  const bool grads = dh != nullptr || dW != nullptr || db != nullptr;
  Plan p;
  std::string err;
  if (!make_plan(rows, d, n_classes, dtype, grads, p, err)) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: " + err);
  if (ld_h < d || (dh != nullptr && ld_dh < d)) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: a leading dimension is below d");
  if (rows == 0) return GNNSTAGE_OK;
  if (!h || !W || !labels || !row_loss) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: h, W, labels and row_loss must not be NULL");
  if (dh == h) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: dh must not be h, which is read after dh is written");
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: workspace must be 256-byte aligned");
  if (workspace_bytes < workspace_bytes_of(p, read_in_place(h, ld_h, d))) return train_error(GNNSTAGE_ENOMEM, "gnntrain_head_xent: workspace smaller than gnntrain_head_xent_workspace_size()");
  const Call c{h, ld_h, W, bias, labels, mask, inv_n_train, row_loss, dh, ld_dh, dW, db, static_cast<char *>(workspace)};
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  int e = hipSuccess;
  if (fused_takes(d, dtype)) {
    const FusedPlan f = fused_plan(rows, d, n_classes, grads, read_in_place(h, ld_h, d));
    for (int64_t r = 0; r < rows && e == hipSuccess; r += f.rows) {
      Call slab = c;
      slab.h = static_cast<const bf16_t *>(h) + (size_t)(r * ld_h);
      slab.labels = labels + r;
      slab.mask = mask ? mask + r : nullptr;
      slab.row_loss = row_loss + r;
      slab.dh = dh ? static_cast<bf16_t *>(dh) + (size_t)(r * ld_dh) : nullptr;
      const int64_t m = std::min(f.rows, rows - r);
      e = f.DP == 64 ? run_fused<64>(f, slab, m, r == 0, s) : f.DP == 128 ? run_fused<128>(f, slab, m, r == 0, s) : run_fused<256>(f, slab, m, r == 0, s);
    }
  } else {
    e = run_in_pieces(p, c, s);
  }
  if (e != hipSuccess) return train_error(GNNSTAGE_EHIP, std::string("gnntrain_head_xent: ") + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
