// What logits answer: the log probability of a row's given class, the entropy, the best classes; and the gradient of the logits from those of
// log probability and entropy.
//
//   z_c = l_c + b_c,  M = max z,  s = sum_c exp(z_c - M),  t = sum_c exp(z_c - M) (z_c - M)
//   logp = z_id - M - log s,   H = log s - t / s,   best classes in the order of (z, lower class first)
//   dz_c = g_logp ([c = id] - p_c) - g_H p_c (log p_c + H),   p_c = exp(z_c - M - log s)
//
// One pass over a row.  A lane keeps its sums against a reference of its own, which follows its largest logit only where that is more than 8 above it;
// references meet at the end.  The given class stays out of the sums: -log1p(others / own) and, where it is the largest, log s = log1p(others)
// have no cancellation in rows that are sure of it.  A probability of zero contributes nothing to t (0 times minus infinity is no number).
//
// Best classes: a wave keeps the 64 best of what it has seen in its lanes, in order, as 64-bit keys (the logit's bits in the numbers' order, then the
// class turned over, so that of equals the lower class is the larger key).  A logit has to be above the n_top-th of them to be looked at: one
// comparison per vector.  Those that are wait in LDS until there are 64, which are sorted and merged in: a row of n logits in random order
// has about 64 + n_top ln(n / 64) of them, two or three mergers.
#include <hip/hip_runtime.h>
#include "guard.h"

#include <algorithm>
#include <string>

#include "../../include/gnntrain.h"
#include "common.h"

namespace {

constexpr float kLog2e = 1.44269504088896f;
constexpr float kNoMax = -3.4028234663852886e38f;  // the least number: a reference that has seen nothing but minus infinity
constexpr float kFollow = 8.f;
__device__ __forceinline__ float exp_diff(float z, float m) { return __builtin_amdgcn_exp2f((z - m) * kLog2e); }

template <typename T>
constexpr int kVec = 16 / sizeof(T);
template <typename T, int N>
struct Vec {
  typedef T aligned_type __attribute__((ext_vector_type(N)));
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// ---- a row's sums ---------------------------------------------------------------------------------------------------
struct Sums {
  float m, s, t, top;  // reference, sum exp(z - m), sum exp(z - m) (z - m), the largest z
};
__device__ __forceinline__ Sums no_sums() { return Sums{kNoMax, 0.f, 0.f, -INFINITY}; }
// sums against another reference, which is not below theirs
__device__ __forceinline__ void refer(Sums &x, float m) {
  const float f = exp_diff(x.m, m);
  x.t = f > 0.f ? f * (x.t + x.s * (x.m - m)) : 0.f;
  x.s *= f;
  x.m = m;
}
__device__ __forceinline__ void join(Sums &x, Sums y) {
  const float m = fmaxf(x.m, y.m);
  refer(x, m);
  refer(y, m);
  x.s += y.s;
  x.t += y.t;
  x.top = fmaxf(x.top, y.top);
}
template <int LANES>
__device__ __forceinline__ void join_lanes(Sums &x) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) join(x, Sums{__shfl_xor(x.m, o), __shfl_xor(x.s, o), __shfl_xor(x.t, o), __shfl_xor(x.top, o)});
}

struct Answer {
  float M, log_s, logp, H;
};
// x: without the given class; zl: its logit, if there is one
__device__ __forceinline__ Answer end_row(Sums x, bool given, float zl) {
  refer(x, x.top);  // (not a number where every logit is minus infinity, or one is infinity: so is all that follows)
  const float M = x.top, own = given ? exp_diff(zl, M) : 0.f, total = x.s + own, d = zl - M;
  const float t = x.t + (own > 0.f ? own * d : own);
  const bool sure = own > 0.5f * total;
  const float ratio = x.s / own;
  Answer a;
  a.M = M;
  a.log_s = sure ? log1pf(ratio) + d : logf(total);
  a.logp = !given ? 0.f : sure ? -log1pf(ratio) : d - a.log_s;
  const float H = a.log_s - t / total;
  a.H = H < 0.f ? 0.f : H;
  return a;
}

// ---- the best classes -----------------------------------------------------------------------------------------------
typedef uint64_t Key;  // 0: none
__device__ __forceinline__ Key key_of(float z, int c) {
  if (!(z == z)) return 0;  // no number is no alternative
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);  // (minus zero is zero)
  return (Key)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~c;
}
__device__ __forceinline__ float logit_of(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int class_of(Key k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ Key lanes_xor(Key k, int o) {
  return (Key)(uint32_t)__shfl_xor((int)(k >> 32), o) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)k, o);
}
__device__ __forceinline__ Key lanes_at(Key k, int lane) {
  return (Key)(uint32_t)__shfl((int)(k >> 32), lane) << 32 | (uint32_t)__shfl((int)(uint32_t)k, lane);
}
// one step of a bitonic network: the larger of two lanes o apart goes to the lower one where `down`
__device__ __forceinline__ Key exchange(Key k, int o, bool down) {
  const Key other = lanes_xor(k, o);
  const bool lower = ((threadIdx.x & o) == 0) == down;
  return (k > other) == lower ? k : other;
}
__device__ __forceinline__ Key sort_lanes(Key k) {
#pragma unroll
  for (int n = 2; n <= 64; n <<= 1)
#pragma unroll
    for (int o = n >> 1; o > 0; o >>= 1) k = exchange(k, o, (threadIdx.x & n & 63) == 0);
  return k;
}
// the 64 best of two ordered lists, in order; turned: the second one, from its last to its first
__device__ __forceinline__ Key merge_lanes(Key list, Key turned) {
  Key k = list > turned ? list : turned;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) k = exchange(k, o, true);
  return k;
}

constexpr int kWaiting = 128;  // room for keys that wait, per wave
struct Best {
  Key list;      // lane i: the i-th best
  Key *waiting;  // LDS
  int n, n_top;  // waiting; asked for
  bool open;     // there are not n_top yet
  float least;   // the n_top-th's logit
  __device__ __forceinline__ Best(Key *room, int n_top) : list(0), waiting(room), n(0), n_top(n_top), open(true), least(-INFINITY) {}
  __device__ __forceinline__ void merge() {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_wave_barrier();
    Key k = lane < n ? waiting[lane] : 0;
    const Key rest = lane + 64 < n ? waiting[lane + 64] : 0;
    __builtin_amdgcn_wave_barrier();
    waiting[lane] = rest;
    __builtin_amdgcn_wave_barrier();
    n = max(n - 64, 0);
    k = sort_lanes(k);
    list = merge_lanes(list, lanes_at(k, 63 - lane));
    const Key last = lanes_at(list, n_top - 1);
    open = last == 0;
    least = open ? -INFINITY : logit_of(last);
  }
  // a key per lane (0: none)
  __device__ __forceinline__ void wait(Key k) {
    const uint64_t votes = __ballot(k != 0);
    if (votes == 0) return;
    if (k != 0) waiting[n + __popcll(votes & ((1ull << (threadIdx.x & 63)) - 1))] = k;
    n += __popcll(votes);
    if (n >= 64) merge();
  }
};

// ---- a wave's part of a row -----------------------------------------------------------------------------------------
// Classes [c0, c1): what lies in front of the first 16-byte border a class per lane, whole vectors, what is left a class per lane.
template <typename T, bool TOP>
__device__ __forceinline__ void scan(const T *row, const float *bias, int c0, int c1, int id, Sums &x, Best &best) {
  constexpr int N = kVec<T>;
  typedef typename Vec<T, N>::aligned_type TV;
  typedef typename Vec<float, 4>::type BV;
  const int lane = threadIdx.x & 63;
  const int head = min(c1 - c0, (int)((-(reinterpret_cast<uintptr_t>(row + c0) / sizeof(T))) & (N - 1)));
  const int a0 = c0 + head, vectors = (c1 - a0) / N, tail = c1 - a0 - vectors * N;
  auto take = [&](float (&z)[N], int c, bool in) {  // in: whether this lane's are classes at all (else all minus infinity)
    float most = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, z[i]);
    if constexpr (TOP) {
      if (best.open || __any(most > best.least)) {
#pragma unroll
        for (int i = 0; i < N; ++i) best.wait(in && (best.open || z[i] >= best.least) ? key_of(z[i], c + i) : 0);
      }
    }
    x.top = fmaxf(x.top, most);
    if (__any(most > x.m + kFollow)) refer(x, fmaxf(x.m, most));
    const int rel = id - c;
    if (__any((uint32_t)rel < (uint32_t)N && in)) {
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = rel == i ? -INFINITY : z[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = z[i] - x.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
      x.s += e;
      x.t = fmaf(e, fmaxf(d, -200.f), x.t);
    }
  };
  auto single = [&](int c, bool in) {  // a class per lane
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = -INFINITY;
    if (in) z[0] = (float)row[c] + (bias ? bias[c] : 0.f);
    if constexpr (TOP) best.wait(in && (best.open || z[0] >= best.least) ? key_of(z[0], c) : 0);
    x.top = fmaxf(x.top, z[0]);
    if (__any(z[0] > x.m + kFollow)) refer(x, fmaxf(x.m, z[0]));
    if (c == id) z[0] = -INFINITY;
    const float d = z[0] - x.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    x.s += e;
    x.t = fmaf(e, fmaxf(d, -200.f), x.t);
  };
  if (head > 0) single(c0 + lane, lane < head);
  TV next;
  BV next_bias[N / 4];
  auto load = [&](int v) {
    if (v < vectors) {
      next = *reinterpret_cast<const TV *>(row + a0 + v * N);
      if (bias) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) next_bias[q] = *reinterpret_cast<const BV *>(bias + a0 + v * N + 4 * q);
      }
    }
  };
  load(lane);
  for (int v0 = 0; v0 < vectors; v0 += 64) {
    const int v = v0 + lane;
    const bool in = v < vectors;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      z[i] = in ? (float)next[i] : -INFINITY;
      if (bias) z[i] = in ? z[i] + next_bias[i / 4][i % 4] : -INFINITY;
    }
    load(v + 64);
    take(z, a0 + v * N, in);
  }
  if (tail > 0) single(a0 + vectors * N + lane, lane < tail);
}

struct AnswerArgs {
  const void *logits;
  int64_t ld;
  const float *bias;
  const int32_t *ids;
  const uint8_t *mask;
  int64_t rows;
  int32_t C, n_top;
  float *logp, *entropy, *norm;
  int32_t *top_ids;
  float *top_logp;
  int32_t splits, part;  // a row's parts and their classes
  Sums *part_sums;       // [row][split]
  Key *part_keys;        // [row][n_top][split]
};
__device__ __forceinline__ void write_row(const AnswerArgs &a, int64_t r, const Answer &w) {
  if (a.logp) a.logp[r] = w.logp;
  if (a.entropy) a.entropy[r] = w.H;
  if (a.norm) {
    a.norm[2 * r] = w.M;
    a.norm[2 * r + 1] = w.log_s;
  }
}
__device__ __forceinline__ void write_best(const AnswerArgs &a, int64_t r, int i, Key k, const Answer &w) {
  a.top_ids[r * a.n_top + i] = k ? class_of(k) : -1;
  a.top_logp[r * a.n_top + i] = (k ? logit_of(k) : NAN) - w.M - w.log_s;  // (none only where there are not as many numbers)
}
// a row that takes no part
__device__ __forceinline__ void write_none(const AnswerArgs &a, int64_t r, int lane, int lanes) {
  if (lane == 0) write_row(a, r, Answer{0.f, 0.f, 0.f, 0.f});
  for (int i = lane; i < a.n_top; i += lanes) {
    a.top_ids[r * a.n_top + i] = -1;
    a.top_logp[r * a.n_top + i] = -INFINITY;
  }
}
template <typename T>
__device__ __forceinline__ float given_logit(const AnswerArgs &a, const T *row, int id) {
  return id < 0 ? -INFINITY : (float)row[id] + (a.bias ? a.bias[id] : 0.f);
}
__device__ __forceinline__ int given_class(const AnswerArgs &a, int64_t r) {
  const int id = a.ids ? a.ids[r] : -1;
  return (uint32_t)id < (uint32_t)a.C ? id : -1;
}

// Rows of at most 4 LANES classes: LANES lanes each, four classes a lane.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void answer_short_kernel(const AnswerArgs a) {
  const int lane = threadIdx.x & (LANES - 1);
  const int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (r >= a.rows) return;  // all lanes of the row
  if (a.mask && a.mask[r] == 0) {
    write_none(a, r, lane, LANES);
    return;
  }
  const T *row = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
  const int id = given_class(a, r);
  float z[4], zl = -INFINITY;
  Sums x = no_sums();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = lane + i * LANES;
    z[i] = -INFINITY;
    if (c < a.C) z[i] = (float)row[c] + (a.bias ? a.bias[c] : 0.f);
    x.top = fmaxf(x.top, z[i]);
    if (c == id) zl = z[i];
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) x.top = fmaxf(x.top, __shfl_xor(x.top, o, LANES));
  zl = __shfl(zl, max(id, 0) & (LANES - 1), LANES);
  x.m = fmaxf(x.top, kNoMax);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (lane + i * LANES == id) continue;
    const float d = z[i] - x.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    x.s += e;
    x.t = fmaf(e, fmaxf(d, -200.f), x.t);
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    x.s += __shfl_xor(x.s, o, LANES);
    x.t += __shfl_xor(x.t, o, LANES);
  }
  const Answer w = end_row(x, id >= 0, zl);
  if (lane == 0) write_row(a, r, w);
  if (a.n_top == 0) return;
  Key key[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) key[i] = lane + i * LANES < a.C ? key_of(z[i], lane + i * LANES) : 0;
  for (int n = 0; n < a.n_top; ++n) {
    Key k = key[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) k = k > key[i] ? k : key[i];
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
      const Key other = lanes_xor(k, o);
      k = k > other ? k : other;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (key[i] == k) key[i] = 0;
    if (lane == 0) write_best(a, r, n, k, w);
  }
}

// A wave per row (WAVES 1: four rows per workgroup), or a workgroup of four waves per row or part of one.
template <typename T, bool TOP, int WAVES>
__global__ __launch_bounds__(256) void answer_kernel(const AnswerArgs a) {
  __shared__ Key room[TOP ? 4 * kWaiting : 1];
  __shared__ Sums met[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (r >= a.rows) return;  // the whole wave (WAVES 1), nobody else's
  if (a.mask && a.mask[r] == 0) {
    if (WAVES == 1 || (wave == 0 && blockIdx.y == 0)) write_none(a, r, lane, 64);
    return;
  }
  const T *row = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
  const int id = given_class(a, r);
  Sums x = no_sums();
  Best best(room + (TOP ? wave * kWaiting : 0), a.n_top);
  int c0 = 0, c1 = a.C;
  if constexpr (WAVES > 1) {
    const int begin = (int)blockIdx.y * a.part, end = min(a.C, begin + a.part), each = ((end - begin + 3) / 4 + 63) / 64 * 64;
    c0 = min(end, begin + wave * each);
    c1 = min(end, c0 + each);
  }
  scan<T, TOP>(row, a.bias, c0, c1, id, x, best);
  if constexpr (TOP)
    if (best.n > 0) best.merge();
  join_lanes<64>(x);
  if constexpr (WAVES > 1) {
    if constexpr (TOP) room[wave * kWaiting + lane] = best.list;
    if (lane == 0) met[wave] = x;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      join(x, met[w]);
      if constexpr (TOP) best.list = merge_lanes(best.list, room[w * kWaiting + 63 - lane]);
    }
    if (a.splits > 1) {
      if (lane == 0) a.part_sums[r * a.splits + blockIdx.y] = x;
      if constexpr (TOP)
        if (lane < a.n_top) a.part_keys[(r * a.n_top + lane) * a.splits + blockIdx.y] = best.list;
      return;
    }
  }
  const Answer w = end_row(x, id >= 0, given_logit(a, row, id));
  if (lane == 0) write_row(a, r, w);
  if constexpr (TOP)
    if (lane < a.n_top) write_best(a, r, lane, best.list, w);
}

// The parts of a row, a wave per row.  First all parts' best, then their second: what comes later is hardly ever looked at.
template <typename T, bool TOP>
__global__ __launch_bounds__(64) void answer_join_kernel(const AnswerArgs a) {
  __shared__ Key room[TOP ? kWaiting : 1];
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  if (a.mask && a.mask[r] == 0) return;  // written
  const int id = given_class(a, r);
  Sums x = no_sums();
  for (int i = lane; i < a.splits; i += 64) join(x, a.part_sums[r * a.splits + i]);
  join_lanes<64>(x);
  const T *row = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
  const Answer w = end_row(x, id >= 0, given_logit(a, row, id));
  if (lane == 0) write_row(a, r, w);
  if constexpr (TOP) {
    Best best(room, a.n_top);
    const int n = a.n_top * a.splits;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Key k = i0 + lane < n ? a.part_keys[r * n + i0 + lane] : 0;
      // (of equal logits the lower class may come later here)
      best.wait(k != 0 && (best.open || logit_of(k) >= best.least) ? k : 0);
    }
    if (best.n > 0) best.merge();
    if (lane < a.n_top) write_best(a, r, lane, best.list, w);
  }
}

constexpr int kMostTop = 64;
// Classes of a row that four lanes more or less take at a time (answer_short_kernel); beyond 64 with few best classes only, whose rounds go over all of a
// row's lanes.
constexpr int kShort = 256, kShortTop = 8;
constexpr int kLong = 4096;         // classes from which a row is a workgroup's
constexpr int kWorkgroups = 512;    // that a launch should have: fewer rows are cut
constexpr int kLeastPart = 2048;    // classes of a part

struct AnswerPlan {
  int splits = 1, part = 0;
  size_t sums = 0, keys = 0, total = 256;
};
AnswerPlan answer_plan(int64_t rows, int C, int n_top) {
  AnswerPlan p;
  p.part = C;
  if (C >= kLong && rows > 0 && rows < kWorkgroups) {
    const int64_t want = std::min<int64_t>((kWorkgroups + rows - 1) / rows, C / kLeastPart);
    p.part = (int)(((C + want - 1) / want + 255) / 256 * 256);
    p.splits = (C + p.part - 1) / p.part;
  }
  if (p.splits > 1) {
    p.keys = (sizeof(Sums) * (size_t)rows * p.splits + 255) & ~(size_t)255;
    p.total = p.keys + ((sizeof(Key) * (size_t)rows * p.splits * n_top + 255) & ~(size_t)255);
  }
  return p;
}

template <typename T, bool TOP>
int run_answer(const AnswerArgs &a, const AnswerPlan &p, hipStream_t s) {
  auto slabs = [&](auto kernel, int threads_per_row) {
    return for_row_slabs(a.rows, threads_per_row, [&](int64_t r, int64_t m, unsigned gx) {
      AnswerArgs b = a;
      b.logits = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
      b.rows = m;
      b.ids = a.ids ? a.ids + r : nullptr;
      b.mask = a.mask ? a.mask + r : nullptr;
      b.logp = a.logp ? a.logp + r : nullptr;
      b.entropy = a.entropy ? a.entropy + r : nullptr;
      b.norm = a.norm ? a.norm + 2 * r : nullptr;
      b.top_ids = a.top_ids ? a.top_ids + r * a.n_top : nullptr;
      b.top_logp = a.top_logp ? a.top_logp + r * a.n_top : nullptr;
      hipLaunchKernelGGL(kernel, dim3(gx, (unsigned)p.splits), dim3(256), 0, s, b);
    });
  };
  if (a.C <= kShort && (a.C <= 64 || a.n_top <= kShortTop)) {
    if (a.C <= 16) return slabs(answer_short_kernel<T, 4>, 4);
    if (a.C <= 32) return slabs(answer_short_kernel<T, 8>, 8);
    if (a.C <= 64) return slabs(answer_short_kernel<T, 16>, 16);
    if (a.C <= 128) return slabs(answer_short_kernel<T, 32>, 32);
    return slabs(answer_short_kernel<T, 64>, 64);
  }
  if (a.C < kLong) return slabs(answer_kernel<T, TOP, 1>, 64);
  const int e = slabs(answer_kernel<T, TOP, 4>, 256);
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((answer_join_kernel<T, TOP>), dim3((unsigned)a.rows), dim3(64), 0, s, a);
  return (int)hipGetLastError();
}

// ---- the gradient ---------------------------------------------------------------------------------------------------
struct GradArgs {
  const void *logits;
  int64_t ld;
  const float *bias;
  const int32_t *ids;
  const uint8_t *mask;
  int64_t rows;
  int32_t C;
  const float *logp, *entropy, *norm, *g_logp, *g_entropy;
  void *dlogits;
  int64_t ld_dl;
  float *dbias, *part;   // part: [group][C], NULL where there is one group
  int32_t across;        // threads along a row; 256 / across rows at a time
  int64_t rows_per;      // rows of a group (grid.y)
};
struct RowGrad {
  float M, log_s, gl, gh;
  float H, own;  // own: g_logp (1 - p_id)
  int32_t id, on;
};
constexpr int kRowsAhead = 64;  // whose numbers are in LDS at a time: chains of that many additions (fewer by the rows at a time) in dbias, then one of their sums

// Workgroups own columns and go down their group's rows: the bias is read once per group, its gradient stays in registers.
template <typename T, typename O, bool SUMS>
__global__ __launch_bounds__(256) void grad_kernel(const GradArgs a) {
  constexpr int N = 16 / (sizeof(T) < sizeof(O) ? sizeof(O) : sizeof(T));
  typedef typename Vec<T, N>::type TV;
  typedef typename Vec<O, N>::type OV;
  __shared__ RowGrad of[kRowsAhead];
  __shared__ float columns[SUMS ? 256 * N : 1];
  const int down = 256 / a.across, ty = threadIdx.x / a.across, tx = threadIdx.x - ty * a.across;
  const int c = ((int)blockIdx.x * a.across + tx) * N;
  const bool mine = ty < down && c < a.C, whole = c + N <= a.C;
  float b[N], sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    b[i] = a.bias && mine && c + i < a.C ? a.bias[c + i] : 0.f;
    sum[i] = 0.f;
  }
  const int64_t r_end = min(a.rows, ((int64_t)blockIdx.y + 1) * a.rows_per);
  for (int64_t r0 = (int64_t)blockIdx.y * a.rows_per; r0 < r_end; r0 += kRowsAhead) {
    const int n = (int)min((int64_t)kRowsAhead, r_end - r0);
    __syncthreads();
    if ((int)threadIdx.x < n) {
      const int64_t r = r0 + threadIdx.x;
      RowGrad w{};
      w.on = a.mask == nullptr || a.mask[r] != 0;
      w.id = -1;
      if (w.on) {
        const int id = a.ids ? a.ids[r] : -1;
        w.M = a.norm[2 * r];
        w.log_s = a.norm[2 * r + 1];
        if (a.g_logp && (uint32_t)id < (uint32_t)a.C) {
          w.id = id;
          w.gl = a.g_logp[r];
          w.own = -expm1f(a.logp[r]) * w.gl;
        }
        if (a.g_entropy) {
          w.gh = a.g_entropy[r];
          w.H = a.entropy[r];
        }
      }
      of[threadIdx.x] = w;
    }
    __syncthreads();
    if (!mine) continue;
    float chain[N];
#pragma unroll
    for (int i = 0; i < N; ++i) chain[i] = 0.f;
    for (int k = ty; k < n; k += down) {
      const RowGrad w = of[k];
      const T *src = static_cast<const T *>(a.logits) + (size_t)((r0 + k) * a.ld) + c;
      O *dst = static_cast<O *>(a.dlogits) + (size_t)((r0 + k) * a.ld_dl) + c;
      float z[N], g[N];
      if (w.on) {
        if (whole) {
          const TV v = *reinterpret_cast<const TV *>(src);
#pragma unroll
          for (int i = 0; i < N; ++i) z[i] = (float)v[i];
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) z[i] = c + i < a.C ? (float)src[i] : -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float log_p = z[i] + b[i] - w.M - w.log_s, p = __builtin_amdgcn_exp2f(log_p * kLog2e);
        const float of_H = w.gh * p * (fmaxf(log_p, -200.f) + w.H);
        g[i] = w.on ? (c + i == w.id ? w.own : -p * w.gl) - of_H : 0.f;
        chain[i] += g[i];
      }
      if (whole) {
        OV v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (O)g[i];
        *reinterpret_cast<OV *>(dst) = v;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (c + i < a.C) dst[i] = (O)g[i];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += chain[i];
  }
  if constexpr (SUMS) {
    // the rows side by side, one after the other
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) columns[threadIdx.x * N + i] = sum[i];
    __syncthreads();
    for (int i = threadIdx.x; i < a.across * N; i += 256) {
      const int col = (int)blockIdx.x * a.across * N + i;
      if (col >= a.C) continue;
      float s = 0.f;
      for (int y = 0; y < down; ++y) s += columns[y * a.across * N + i];
      if (a.part)
        a.part[(size_t)blockIdx.y * a.C + col] = s;
      else
        a.dbias[col] += s;
    }
  }
}

// dbias += the groups' sums: 64 columns a workgroup, every sixteenth group a thread
__global__ __launch_bounds__(1024) void grad_bias_kernel(const float *part, int groups, int C, float *dbias) {
  __shared__ float of[16][64];
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6, c = blockIdx.x * 64 + x;
  float s = 0.f;
  if (c < C)
    for (int g = y; g < groups; g += 16) s += part[(size_t)g * C + c];
  of[y][x] = s;
  __syncthreads();
  for (int w = 8; w > 0; w >>= 1) {
    if (y < w) of[y][x] += of[y + w][x];
    __syncthreads();
  }
  if (y == 0 && c < C) dbias[c] += of[0][x];
}

struct GradPlan {
  int across = 0, blocks = 0;
  int64_t groups = 1, rows_per = 0;
  size_t total = 256;
};
constexpr int64_t kPartElements = (int64_t)1 << 25;  // of the groups' sums
GradPlan grad_plan(int64_t rows, int C, int n) {
  GradPlan p;
  p.across = std::min(256, (C + n - 1) / n);
  p.blocks = (C + p.across * n - 1) / (p.across * n);
  const int64_t down = 256 / p.across;
  const int64_t want = (2048 + p.blocks - 1) / p.blocks;
  const int64_t most = std::max<int64_t>(1, kPartElements / C);
  p.groups = std::max<int64_t>(1, std::min({want, most, (rows + 4 * down - 1) / (4 * down)}));
  p.rows_per = std::max<int64_t>(1, (rows + p.groups - 1) / p.groups);
  p.groups = std::max<int64_t>(1, (rows + p.rows_per - 1) / p.rows_per);
  p.total = p.groups > 1 ? (sizeof(float) * (size_t)p.groups * C + 255) & ~(size_t)255 : 256;
  return p;
}

bool sizes_ok(int64_t rows, int C, std::string &err) {
  if (rows < 0 || rows > ((int64_t)1 << 40)) { err = "rows must not be negative (nor beyond 2^40)"; return false; }
  if (C < 1 || C > (1 << 24)) { err = "n_classes must be in [1, 2^24]"; return false; }
  return true;
}
bool top_ok(int n_top, int C, std::string &err) {
  if (n_top < 0 || n_top > kMostTop || n_top > C) { err = "n_top must be in [0, 64] and n_classes at most"; return false; }
  return true;
}

}  // namespace

extern "C" size_t gnntrain_logprobs_workspace_size(int64_t rows, int32_t n_classes, int32_t n_top) try {
  std::string err;
  if (!sizes_ok(rows, n_classes, err) || !top_ok(n_top, n_classes, err)) {
    train_error(GNNSTAGE_EINVAL, "gnntrain_logprobs: " + err);
    return 0;
  }
  return answer_plan(rows, n_classes, n_top).total;
}
GNNSTAGE_GUARD_SIZE

extern "C" int gnntrain_logprobs(const void *logits, int32_t dtype, int64_t ld, const float *bias, const int32_t *ids, const uint8_t *mask, int64_t rows,
                                 int32_t n_classes, int32_t n_top, float *logp, float *entropy, float *norm, int32_t *top_ids, float *top_logp, void *workspace,
                                 size_t workspace_bytes, void *hip_stream) try {
  const char *const me = "gnntrain_logprobs: ";
  std::string err;
  if (dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) return train_error(GNNSTAGE_EINVAL, std::string(me) + "unknown dtype");
  if (!sizes_ok(rows, n_classes, err) || !top_ok(n_top, n_classes, err)) return train_error(GNNSTAGE_EINVAL, me + err);
  if (ld < n_classes) return train_error(GNNSTAGE_EINVAL, std::string(me) + "ld is below n_classes");
  if (rows == 0) return GNNSTAGE_OK;
  if (!logits) return train_error(GNNSTAGE_EINVAL, std::string(me) + "logits must not be NULL");
  if (reinterpret_cast<uintptr_t>(logits) & (dtype == GNNSTAGE_BF16 ? 1u : 3u)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "logits are not aligned to their elements");
  if (logp && !ids) return train_error(GNNSTAGE_EINVAL, std::string(me) + "logp needs ids");
  if (n_top > 0 && (!top_ids || !top_logp)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "n_top needs top_ids and top_logp");
  const AnswerPlan p = answer_plan(rows, n_classes, n_top);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "workspace must be 256-byte aligned");
  if (workspace_bytes < p.total) return train_error(GNNSTAGE_ENOMEM, std::string(me) + "workspace smaller than gnntrain_logprobs_workspace_size()");
  AnswerArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.bias = bias;
  a.ids = ids;
  a.mask = mask;
  a.rows = rows;
  a.C = n_classes;
  a.n_top = n_top;
  a.logp = logp;
  a.entropy = entropy;
  a.norm = norm;
  a.top_ids = n_top > 0 ? top_ids : nullptr;
  a.top_logp = n_top > 0 ? top_logp : nullptr;
  a.splits = p.splits;
  a.part = p.part;
  a.part_sums = reinterpret_cast<Sums *>(static_cast<char *>(workspace) + p.sums);
  a.part_keys = reinterpret_cast<Key *>(static_cast<char *>(workspace) + p.keys);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int e = dtype == GNNSTAGE_BF16 ? (n_top > 0 ? run_answer<bf16_t, true>(a, p, s) : run_answer<bf16_t, false>(a, p, s))
                                       : (n_top > 0 ? run_answer<float, true>(a, p, s) : run_answer<float, false>(a, p, s));
  if (e != hipSuccess) return train_error(GNNSTAGE_EHIP, me + std::string(hipGetErrorString((hipError_t)e)));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT

extern "C" size_t gnntrain_logprobs_grad_workspace_size(int64_t rows, int32_t n_classes) try {
  std::string err;
  if (!sizes_ok(rows, n_classes, err)) {
    train_error(GNNSTAGE_EINVAL, "gnntrain_logprobs_grad: " + err);
    return 0;
  }
  return std::max(grad_plan(rows, n_classes, 4).total, grad_plan(rows, n_classes, 8).total);
}
GNNSTAGE_GUARD_SIZE

namespace {
template <typename T, typename O>
int run_grad(GradArgs a, float *room, hipStream_t s) {
  constexpr int N = 16 / (sizeof(T) < sizeof(O) ? sizeof(O) : sizeof(T));
  const GradPlan p = grad_plan(a.rows, a.C, N);
  a.across = p.across;
  a.rows_per = p.rows_per;
  a.part = p.groups > 1 ? room : nullptr;
  // (a grid's y axis takes 65,535; a launch 2^32 work-items)
  hipLaunchKernelGGL((a.dbias ? grad_kernel<T, O, true> : grad_kernel<T, O, false>), dim3((unsigned)p.blocks, (unsigned)p.groups), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias || p.groups == 1) return (int)e;
  hipLaunchKernelGGL(grad_bias_kernel, dim3((unsigned)((a.C + 63) / 64)), dim3(1024), 0, s, room, (int)p.groups, a.C, a.dbias);
  return (int)hipGetLastError();
}
}  // namespace

extern "C" int gnntrain_logprobs_grad(const void *logits, int32_t dtype, int64_t ld, const float *bias, const int32_t *ids, const uint8_t *mask, int64_t rows,
                                      int32_t n_classes, const float *logp, const float *entropy, const float *norm, const float *g_logp, const float *g_entropy,
                                      void *dlogits, int32_t dl_dtype, int64_t ld_dl, float *dbias, void *workspace, size_t workspace_bytes, void *hip_stream) try {
  const char *const me = "gnntrain_logprobs_grad: ";
  std::string err;
  if ((dtype != GNNSTAGE_F32 && dtype != GNNSTAGE_BF16) || (dl_dtype != GNNSTAGE_F32 && dl_dtype != GNNSTAGE_BF16))
    return train_error(GNNSTAGE_EINVAL, std::string(me) + "unknown dtype");
  if (!sizes_ok(rows, n_classes, err)) return train_error(GNNSTAGE_EINVAL, me + err);
  if (ld < n_classes || ld_dl < n_classes) return train_error(GNNSTAGE_EINVAL, std::string(me) + "a leading dimension is below n_classes");
  if (rows == 0) return GNNSTAGE_OK;
  if (!logits || !dlogits || !norm) return train_error(GNNSTAGE_EINVAL, std::string(me) + "logits, norm and dlogits must not be NULL");
  if ((reinterpret_cast<uintptr_t>(logits) & (dtype == GNNSTAGE_BF16 ? 1u : 3u)) || (reinterpret_cast<uintptr_t>(dlogits) & (dl_dtype == GNNSTAGE_BF16 ? 1u : 3u)))
    return train_error(GNNSTAGE_EINVAL, std::string(me) + "logits or dlogits are not aligned to their elements");
  if (g_logp && (!ids || !logp)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "g_logp needs ids and logp");
  if (g_entropy && !entropy) return train_error(GNNSTAGE_EINVAL, std::string(me) + "g_entropy needs entropy");
  if (dlogits == logits && (dtype != dl_dtype || ld != ld_dl)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "dlogits may be logits only with their type and leading dimension");
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "workspace must be 256-byte aligned");
  if (workspace_bytes < gnntrain_logprobs_grad_workspace_size(rows, n_classes))
    return train_error(GNNSTAGE_ENOMEM, std::string(me) + "workspace smaller than gnntrain_logprobs_grad_workspace_size()");
  GradArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.bias = bias;
  a.ids = ids;
  a.mask = mask;
  a.rows = rows;
  a.C = n_classes;
  a.logp = logp;
  a.entropy = entropy;
  a.norm = norm;
  a.g_logp = g_logp;
  a.g_entropy = g_entropy;
  a.dlogits = dlogits;
  a.ld_dl = ld_dl;
  a.dbias = dbias;
  float *room = static_cast<float *>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int e = dtype == GNNSTAGE_BF16 ? (dl_dtype == GNNSTAGE_BF16 ? run_grad<bf16_t, bf16_t>(a, room, s) : run_grad<bf16_t, float>(a, room, s))
                                       : (dl_dtype == GNNSTAGE_BF16 ? run_grad<float, bf16_t>(a, room, s) : run_grad<float, float>(a, room, s));
  if (e != hipSuccess) return train_error(GNNSTAGE_EHIP, me + std::string(hipGetErrorString((hipError_t)e)));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
