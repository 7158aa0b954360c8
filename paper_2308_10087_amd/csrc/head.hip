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
// multiplies these with the weights and the rows.

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

// The classes [c0, c0 + n) of a slab's rows; a wave per row.
__global__ __launch_bounds__(256) void piece_state_kernel(const float *logits, int ld, const float *bias, const int32_t *label, int64_t rows,
                                                          int c0, int n, int last, RowState *state, float *row_loss) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int y = label[r] - c0;
  if (label[r] < 0) return;
  const float *z = logits + (size_t)r * ld;
  RowState s = state[r];
  float mx = s.max;
  for (int c = lane; c < n; c += 64) mx = fmaxf(mx, z[c] + (bias ? bias[c0 + c] : 0.f));
  mx = wave_max(mx);
  float others = 0.f;
  for (int c = lane; c < n; c += 64)
    if (c != y) others += expf(z[c] + (bias ? bias[c0 + c] : 0.f) - mx);
  others = wave_sum(others);
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

// The gradients of a piece's logits: fp32 in place, or as the sum of two bf16 numbers (16 bits of significand: the weight
// gradient is fp32 and keeps more than one bf16 number holds).  Columns [n, ld) are written as zeros.
__global__ __launch_bounds__(256) void piece_grad_kernel(float *logits, int ld, const float *bias, const int32_t *label, int64_t rows, int c0,
                                                         int n, float inv_n, const RowState *state, bf16_t *high, bf16_t *low) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  float *z = logits + (size_t)r * ld;
  const bool on = label[r] >= 0;
  const int y = label[r] - c0;
  const RowState s = state[r];
  const float inv_sum = 1.f / (s.others + expf(s.own - s.max));
  for (int c = lane; c < ld; c += 64) {
    float g = 0.f;
    if (on && c < n) g = (c == y ? -s.others : expf(z[c] + (bias ? bias[c0 + c] : 0.f) - s.max)) * inv_sum * inv_n;
    if (high != nullptr) {
      const bf16_t x = (bf16_t)g;
      high[(size_t)r * ld + c] = x;
      low[(size_t)r * ld + c] = (bf16_t)(g - (float)x);
    } else {
      z[c] = g;
    }
  }
}

// dh = what the pieces have added up, in the rows' type; zeros for rows without a label
__global__ __launch_bounds__(256) void finish_rows_kernel(const float *acc, const int32_t *label, int64_t rows, int d, void *dh, int dtype,
                                                          int64_t ld_dh) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * d) return;
  const int64_t r = i / d;
  store_elt(dh, dtype, (size_t)(r * ld_dh + i % d), label[r] >= 0 ? acc[i] : 0.f);
}

// dW[k][c0 + c] += piece[k][c], c < n
__global__ __launch_bounds__(256) void add_piece_kernel(const float *piece, int d, int n, float *dW, int C, int c0) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)d * n) return;
  dW[(size_t)(i / n) * C + c0 + i % n] += piece[i];
}

constexpr int kPieceClasses = 8192;
constexpr int64_t kPieceElements = 1 << 26;  // logits of a slab's piece
constexpr int64_t kSlabRows = 131072;

struct Plan {
  int64_t rows = 0, slab = 0;
  int d = 0, C = 0, dtype = 0, elt = 4, Kp = 0, Cp = 0, piece = 0, ld = 0, max_splits = 0;
  bool grads = false;
  size_t Wt = 0, Wn = 0, rows_at = 0, label = 0, state = 0, logits = 0, high = 0, low = 0, acc = 0, zeros = 0, tmp = 0, partial = 0,
         bias_partial = 0, total = 0;
};

bool make_plan(int64_t rows, int d, int C, int dtype, bool grads, Plan &p, std::string &err) {
  if (rows < 0 || rows > ((int64_t)1 << 40)) { err = "rows must not be negative (nor beyond 2^40)"; return false; }
  if (d < 1 || d > 65536) { err = "the rows' width must be in [1, 65536]"; return false; }
  if (C < 1 || C > (1 << 24)) { err = "n_classes must be in [1, 2^24]"; return false; }
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) { err = "unknown dtype"; return false; }
  p.rows = rows;
  p.d = d;
  p.C = C;
  p.dtype = dtype;
  p.elt = dtype == GNNSTAGE_BF16 ? 2 : 4;
  p.grads = grads;
  p.Kp = round_up(d, 8);
  p.Cp = round_up(C, 8);
  p.piece = std::min(p.Cp, kPieceClasses);
  p.ld = p.piece;
  p.slab = std::max<int64_t>(128, std::min(kSlabRows, kPieceElements / std::max(p.ld, p.d)));
  p.slab = std::min(p.slab, std::max<int64_t>(rows, 1));
  const int tiles = (d + 127) / 128 * ((p.piece + 127) / 128);
  p.max_splits = std::max(1, std::min(256, 1024 / tiles));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = align256(off + bytes);
    return at;
  };
  const size_t m = (size_t)p.slab;
  p.Wt = take((size_t)p.elt * C * p.Kp);
  p.Wn = take((size_t)p.elt * d * p.Cp);
  p.rows_at = take((size_t)p.elt * m * p.Kp);
  p.label = take(sizeof(int32_t) * m);
  p.state = take(sizeof(RowState) * m);
  p.logits = take(sizeof(float) * m * p.ld);
  if (grads) {
    p.high = take(dtype == GNNSTAGE_BF16 ? 2 * m * p.ld : 0);
    p.low = take(dtype == GNNSTAGE_BF16 ? 2 * m * p.ld : 0);
    p.acc = take(sizeof(float) * m * d);
    p.zeros = take(sizeof(float) * (size_t)round_up(d, 64));
    p.tmp = take(sizeof(float) * (size_t)d * p.piece);
    p.partial = take(sizeof(float) * (size_t)p.max_splits * d * p.piece);
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
  if (p.grads) HEAD_TRY(launch_fill_zero(at(p.zeros), sizeof(float) * (size_t)round_up(p.d, 64), s));
  float *logits = reinterpret_cast<float *>(at(p.logits)), *acc = reinterpret_cast<float *>(at(p.acc));
  int32_t *label = reinterpret_cast<int32_t *>(at(p.label));
  RowState *state = reinterpret_cast<RowState *>(at(p.state));
  bf16_t *high = p.dtype == GNNSTAGE_BF16 ? reinterpret_cast<bf16_t *>(at(p.high)) : nullptr;
  bf16_t *low = p.dtype == GNNSTAGE_BF16 ? reinterpret_cast<bf16_t *>(at(p.low)) : nullptr;
  for (int64_t row0 = 0; row0 < p.rows; row0 += p.slab) {
    const int64_t M = std::min(p.slab, p.rows - row0);
    const unsigned waves = (unsigned)((M + 3) / 4);
    hipLaunchKernelGGL(pack_rows_kernel, dim3(waves), dim3(256), 0, s, static_cast<const char *>(c.h) + (size_t)(row0 * c.ld_h) * p.elt, p.dtype,
                       c.ld_h, c.labels + row0, c.mask ? c.mask + row0 : nullptr, M, p.d, p.C, (void *)at(p.rows_at), p.Kp, label, state,
                       c.row_loss + row0);
    HEAD_TRY(hipGetLastError());
    auto piece_logits = [&](int c0, int n) {
      GemmNtArgs g{};
      g.A = at(p.rows_at);
      g.a_dtype = p.dtype;
      g.lda = p.Kp;
      g.Bt = at(p.Wt) + (size_t)c0 * p.Kp * p.elt;
      g.ldb = p.Kp;
      g.M = (int)M;
      g.N = n;
      g.K = p.d;
      g.Kp = p.Kp;
      g.epilogue = EPI_PLAIN;
      g.out = logits;
      g.out_dtype = DT_F32;
      g.out_ld = p.ld;
      return launch_gemm_nt(g, p.dtype, s);
    };
    for (int c0 = 0; c0 < p.C; c0 += p.piece) {
      const int n = std::min(p.piece, p.C - c0);
      HEAD_TRY(piece_logits(c0, n));
      hipLaunchKernelGGL(piece_state_kernel, dim3(waves), dim3(256), 0, s, logits, p.ld, c.bias, label, M, c0, n, (int)(c0 + n == p.C), state,
                         c.row_loss + row0);
      HEAD_TRY(hipGetLastError());
    }
    if (!p.grads) continue;
    for (int c0 = 0; c0 < p.C; c0 += p.piece) {
      const int n = std::min(p.piece, p.C - c0);
      if (p.piece < p.C) HEAD_TRY(piece_logits(c0, n));  // the only piece's are still there
      hipLaunchKernelGGL(piece_grad_kernel, dim3(waves), dim3(256), 0, s, logits, p.ld, c.bias, label, M, c0, n, c.inv_n, state, high, low);
      HEAD_TRY(hipGetLastError());
      if (c.dh) {
        GemmNtArgs g{};
        g.A = high ? (const void *)high : logits;  // dh is of the rows' type: the rounding of its factors to bf16 is below its own
        g.a_dtype = p.dtype;
        g.lda = p.ld;
        g.Bt = at(p.Wn) + (size_t)c0 * p.elt;
        g.ldb = p.Cp;
        g.M = (int)M;
        g.N = p.d;
        g.K = n;
        g.Kp = round_up(n, 8);
        g.epilogue = c0 == 0 ? EPI_PLAIN : EPI_RES;
        g.bias = reinterpret_cast<const float *>(at(p.zeros));
        g.aux = acc;
        g.aux_dtype = DT_F32;
        g.aux_ld = p.d;
        g.out = acc;
        g.out_dtype = DT_F32;
        g.out_ld = p.d;
        HEAD_TRY(launch_gemm_nt(g, p.dtype, s));
      }
      if (c.dW || c.db) {
        const bool whole = p.piece >= p.C && c.dW;
        float *tmp = whole ? c.dW : reinterpret_cast<float *>(at(p.tmp));
        if (!whole) HEAD_TRY(launch_fill_zero(tmp, sizeof(float) * (size_t)p.d * n, s));
        for (int part = 0; part < (high ? 2 : 1); ++part) {
          GemmTnArgs t{};
          t.A = at(p.rows_at);
          t.a_dtype = p.dtype;
          t.lda = p.Kp;
          t.B = high ? (const void *)(part ? low : high) : logits;
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

}  // namespace

extern "C" size_t gnntrain_head_xent_workspace_size(int64_t rows, int32_t d, int32_t n_classes, int32_t dtype, int32_t want_grads) try {
  Plan p;
  std::string err;
  if (!make_plan(rows, d, n_classes, dtype, want_grads != 0, p, err)) {
    train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: " + err);
    return 0;
  }
  return p.total;
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
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return train_error(GNNSTAGE_EINVAL, "gnntrain_head_xent: workspace must be 256-byte aligned");
  if (workspace_bytes < p.total) return train_error(GNNSTAGE_ENOMEM, "gnntrain_head_xent: workspace smaller than gnntrain_head_xent_workspace_size()");
  const Call c{h, ld_h, W, bias, labels, mask, inv_n_train, row_loss, dh, ld_dh, dW, db, static_cast<char *>(workspace)};
  const int e = run_in_pieces(p, c, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return train_error(GNNSTAGE_EHIP, std::string("gnntrain_head_xent: ") + hipGetErrorString((hipError_t)e));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
