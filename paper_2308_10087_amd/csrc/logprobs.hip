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
// class turned over, so that of equals the lower class is the larger key).  A logit has to be above a border to be looked at: one comparison per vector.  The border is what is
// known to be below n_top others: the n_top-th of the first whole step's lanes' largest, then of the wave's list, or what another wave of the row has found.  Those that are above
// wait in LDS until there are 16 (of more than 16 best: 64), which are sorted and merged in.  (8,191 x 100,003 bf16 with ten best: 170 M vector
// instructions, 429 us; without the first step's border 436, merged 64 at a time 434, both 182 M and 443; without any best classes 407.)
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

// Between what lanes of a wave write to LDS and what others of them read there.  LDS does a wave's instructions in their order; that the compiler keeps to it takes fences: a barrier
// of the wave alone orders no accesses, and a lane that wrote nothing might go on with what it read before.  (No instructions of their own.)
__device__ __forceinline__ void lds_written() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
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
// a lane's value of the lane O further (its number's bit O turned over): within 16 lanes by the data path's own moves, beyond by swaps of rows
template <int O>
__device__ __forceinline__ uint32_t lanes_xor(uint32_t x) {
  if constexpr (O == 1)
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);  // lanes 1 0 3 2 of the quad
  else if constexpr (O == 2)
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);  // lanes 2 3 0 1
  else if constexpr (O == 4)  // quads 0 and 2 from the left, 1 and 3 from the right
    return (uint32_t)__builtin_amdgcn_update_dpp(__builtin_amdgcn_mov_dpp((int)x, 0x104, 0xf, 0xf, true), (int)x, 0x114, 0xf, 0xa, false);
  else if constexpr (O == 8)
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true);  // around by eight
  else if constexpr (O == 16) {
    const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? y[0] : y[1];
  } else {
    const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? y[0] : y[1];
  }
}
template <int O>
__device__ __forceinline__ float lanes_xor(float x) { return __builtin_bit_cast(float, lanes_xor<O>(__builtin_bit_cast(uint32_t, x))); }
__device__ __forceinline__ Key lanes_at(Key k, int lane) {
  return (Key)(uint32_t)__shfl((int)(k >> 32), lane) << 32 | (uint32_t)__shfl((int)(uint32_t)k, lane);
}
// one step of a bitonic network: the larger of two lanes O apart goes to the lower one where `down`
template <int O>
__device__ __forceinline__ Key exchange(Key k, bool down) {
  const Key other = (Key)lanes_xor<O>((uint32_t)(k >> 32)) << 32 | lanes_xor<O>((uint32_t)k);
  const bool lower = ((threadIdx.x & O) == 0) == down;
  return (k > other) == lower ? k : other;
}
template <int N>
__device__ __forceinline__ Key sort_step(Key k) {  // blocks of N lanes, ordered in turn down and up
  const bool down = (threadIdx.x & N & 63) == 0;
  if constexpr (N >= 64) k = exchange<32>(k, down);
  if constexpr (N >= 32) k = exchange<16>(k, down);
  if constexpr (N >= 16) k = exchange<8>(k, down);
  if constexpr (N >= 8) k = exchange<4>(k, down);
  if constexpr (N >= 4) k = exchange<2>(k, down);
  return exchange<1>(k, down);
}
__device__ __forceinline__ Key sort_lanes(Key k) { return sort_step<64>(sort_step<32>(sort_step<16>(sort_step<8>(sort_step<4>(sort_step<2>(k)))))); }
// 16 lanes whose eights are ordered down and up: all of them up
__device__ __forceinline__ Key sort_sixteen_up(Key k) { return exchange<1>(exchange<2>(exchange<4>(exchange<8>(k, false), false), false), false); }
// the 64 best of two ordered lists, in order; turned: the second one, from its last to its first
__device__ __forceinline__ Key merge_lanes(Key list, Key turned) {
  Key k = exchange<32>(list > turned ? list : turned, true);
  k = exchange<8>(exchange<16>(k, true), true);
  return exchange<1>(exchange<2>(exchange<4>(k, true), true), true);
}

template <int O>
__device__ __forceinline__ void join_across(Sums &x) { join(x, Sums{lanes_xor<O>(x.m), lanes_xor<O>(x.s), lanes_xor<O>(x.t), lanes_xor<O>(x.top)}); }
__device__ __forceinline__ void join_lanes(Sums &x) {
  join_across<1>(x);
  join_across<2>(x);
  join_across<4>(x);
  join_across<8>(x);
  join_across<16>(x);
  join_across<32>(x);
}

// the next number below; of minus infinity (and of NaN) there is none: NaN
__device__ __forceinline__ float below(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const uint32_t n = x > 0.f ? b - 1 : x < 0.f ? b + 1 : 0x80000001u;
  return x > -INFINITY ? __builtin_bit_cast(float, n) : NAN;
}

#define LDS_AS __attribute__((address_space(3)))
constexpr int kWaiting = 64 * 9;  // room for keys that wait, per wave: 63 and a step's
// A logit is looked at unless it is at most the border: nothing is at most NaN.  Between two steps of a wave the border is the n_top-th best itself, since what comes
// later and is equal is a higher class; within a step, and to the other waves of the row, the number below it.
struct Best {
  Key list;        // lane i: the i-th best
  LDS_AS Key *waiting;
  volatile LDS_AS float *borders;  // of the row's waves, where they share it (LDS has no NULL)
  bool share;
  int n, n_top;    // waiting; asked for
  float least;     // the n_top-th's logit, NaN while there is none
  float others, within;
  float floor;     // a number that is below n_top others at least (and not one of them), NaN while none is known
  __device__ __forceinline__ Best(Key *room, float *row_borders, bool share, int n_top)
      : list(0), waiting((LDS_AS Key *)room), borders((LDS_AS float *)row_borders), share(share), n(0), n_top(n_top), least(NAN), others(NAN), within(NAN), floor(NAN) {}
  // The border before a step, with what the row's other waves have found (whenever that was: what one of them has found is right for all)
  __device__ __forceinline__ float border() {
    if (share) others = fmaxf(fmaxf(borders[0], borders[1]), fmaxf(borders[2], borders[3]));
    return fmaxf(fmaxf(least, floor), others);
  }
  // and within it
  __device__ __forceinline__ void enter() { within = fmaxf(fmaxf(below(least), floor), others); }
  // The first whole step: of the lanes' largest logits the n_top-th is a number that n_top classes reach, so that not all of the step waits.
  __device__ __forceinline__ void start(float most) {
    if (n_top < 64) {
      const Key kth = lanes_at(sort_lanes(key_of(most, threadIdx.x & 63)), n_top - 1);
      floor = kth == 0 ? NAN : below(logit_of(kth));
      tell(floor);
    }
  }
  __device__ __forceinline__ void tell(float x) {
    if (share && (threadIdx.x & 63) == 0) borders[threadIdx.x >> 6] = x;
  }
  // this lane's class c, where `in`
  __device__ __forceinline__ void look(bool in, float z, int c) {
    const bool mine = in && !(z <= within);
    if (__ballot(mine) != 0) wait(mine ? key_of(z, c) : 0);
  }
  // a key per lane (0: none), 64 fewer than kWaiting before settle()
  __device__ __forceinline__ void wait(Key k) {
    const uint64_t votes = __ballot(k != 0);
    if (k != 0) waiting[n + __popcll(votes & ((1ull << (threadIdx.x & 63)) - 1))] = k;
    n += __popcll(votes);
  }
  // as many as are merged in at once: few best are settled by few merges, but soon
  __device__ __forceinline__ bool full() const { return n >= (n_top <= 16 ? 16 : 64); }
  // merges all that waits in
  __device__ __forceinline__ void settle() {
    const int lane = threadIdx.x & 63;
    lds_written();
#pragma unroll 1
    while (n > 0) {
      Key last = lanes_at(list, n_top - 1);
      if (n <= 16) {  // in the last lanes, from the least to the best
        const int at = lane - 48;
        Key k = at >= 0 && at < n ? waiting[at] : 0;
        k = sort_step<8>(sort_step<4>(sort_step<2>(k)));
        k = sort_sixteen_up(k);
        n = 0;
        list = merge_lanes(list, k);
      } else {
        const int at = n - 64 + lane;
        const Key k = at >= 0 ? waiting[at] : 0;
        n = max(n - 64, 0);
        if (!__any(k > last)) continue;
        list = merge_lanes(list, lanes_at(sort_lanes(k), 63 - lane));
      }
      last = lanes_at(list, n_top - 1);
      least = last == 0 ? NAN : logit_of(last);
      tell(fmaxf(below(least), floor));
    }
    lds_written();
  }
};

// ---- a wave's part of a row -----------------------------------------------------------------------------------------
// Classes [c0, c1), the same for all lanes: what lies in front of the first 16-byte border a class per lane, whole vectors, what is left a class per lane.
template <typename T, bool TOP, bool BIAS>
__device__ __forceinline__ void scan(const T *row, const float *bias, int c0, int c1, int id, Sums &x, Best &best) {
  constexpr int N = kVec<T>;
  typedef typename Vec<T, N>::aligned_type TV;
  typedef typename Vec<float, 4>::type BV;
  const int lane = threadIdx.x & 63;
  const int head = min(c1 - c0, (int)((-(reinterpret_cast<uintptr_t>(row + c0) / sizeof(T))) & (N - 1)));
  const int a0 = c0 + head, vectors = (c1 - a0) / N, tail = c1 - a0 - vectors * N;
  auto add = [&](float z) {
    const float d = z - x.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    x.s += e;
    x.t = fmaf(e, fmaxf(d, -200.f), x.t);  // (e is what says that d is no number)
  };
  // c: this lane's first class; first: the first lane's.  in: whether this lane's are classes at all (else all minus infinity)
  auto take = [&](float (&z)[N], int c, int first, bool in) {
    float most = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, z[i]);
    if constexpr (TOP) {
      if (__any(!(most <= best.border()))) {
        if (!(best.least == best.least) && !(best.floor == best.floor)) best.start(most);
        best.enter();
#pragma unroll
        for (int i = 0; i < N; ++i) best.look(in, z[i], c + i);
        if (best.full()) best.settle();
      }
    }
    x.top = fmaxf(x.top, most);
    if (__any(most > x.m + kFollow)) refer(x, fmaxf(x.m, most));
    if ((uint32_t)(id - first) < 64u * N) {
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = c + i == id ? -INFINITY : z[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) add(z[i]);
  };
  auto single = [&](int c, bool in) {  // a class per lane
    float z = -INFINITY;
    if (in) z = (float)row[c] + (BIAS ? bias[c] : 0.f);
    if constexpr (TOP) {
      best.border();
      best.enter();
      best.look(in, z, c);
    }
    x.top = fmaxf(x.top, z);
    if (__any(z > x.m + kFollow)) refer(x, fmaxf(x.m, z));
    add(c == id ? -INFINITY : z);
  };
  if (head > 0) single(c0 + lane, lane < head);
  struct Loaded {
    TV v;
    BV b[N / 4];
  };
  const T *src = row + a0 + lane * N;
  const float *bsrc = bias + a0 + lane * N;
  auto load = [&](Loaded &l, int step) {
    l.v = *reinterpret_cast<const TV *>(src + step * (64 * N));
    if constexpr (BIAS) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) l.b[q] = *reinterpret_cast<const BV *>(bsrc + step * (64 * N) + 4 * q);
    }
  };
  auto open = [&](float (&z)[N], const Loaded &l) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = BIAS ? (float)l.v[i] + l.b[i / 4][i % 4] : (float)l.v[i];
  };
  // Whole steps of all lanes, in pairs; the next pair is on its way, without a branch (an access is waited for together with all in front of it): behind the last
  // step that one again.
  const int steps = vectors / 64;
  if (steps > 0) {
    Loaded next[2];
    load(next[0], 0);
    load(next[1], min(1, steps - 1));
    for (int step = 0; step < steps; step += 2) {
      const Loaded now[2] = {next[0], next[1]};
      load(next[0], min(step + 2, steps - 1));
      load(next[1], min(step + 3, steps - 1));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (step + i >= steps) break;
        float z[N];
        open(z, now[i]);
        take(z, a0 + ((step + i) * 64 + lane) * N, a0 + (step + i) * 64 * N, true);
      }
    }
  }
  if (steps * 64 < vectors) {
    const int v = steps * 64 + lane;
    const bool in = v < vectors;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = -INFINITY;
    if (in) {
      Loaded l;
      load(l, steps);
      open(z, l);
    }
    take(z, a0 + v * N, a0 + steps * 64 * N, in);
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

// Rows of few classes, at most N LANES: LANES (2 or 4) lanes each, with their logits in registers, so that what a row costs is its classes and not the lanes'
// meetings.  Bound by the chain of a wave's life: loads in four round trips, LDS, a search per best class (232,965 x 41 fp32, 3 best, 66 % of the rows: 18 us, the bytes alone 6), and by where it
// begins: 6,400 bytes of LDS let 25 waves onto a CU, 28.4 of which are its share there.  Rows that take no part are loaded as well: 17, 18, 18, 16 us with all, 66, 30 and 2 % of them.  A
// wave's rows go through LDS, kPitch floats apart: LANES times an odd number, in which lanes meet in no bank.
template <typename T, int LANES, int N>
__global__ __launch_bounds__(64) void answer_short_kernel(const AnswerArgs a) {
  constexpr int kRows = 64 / LANES, kPitch = LANES * (N + 1);
  __shared__ float at[kRows * kPitch];
  const int lane = threadIdx.x, mine = lane / LANES, sub = lane & (LANES - 1), C = a.C;
  const int64_t r0 = (int64_t)blockIdx.x * kRows, r = r0 + mine;
  const int rows = (int)min((int64_t)kRows, a.rows - r0);
  const bool on = mine < rows && (a.mask == nullptr || a.mask[r] != 0);
  const T *src = static_cast<const T *>(a.logits) + (size_t)(r0 * a.ld);
  // Rows (of up to 32 classes: two or four of them) an instruction, a class per lane, without a branch: past the last row that one once more, which writes what is there; past
  // the last class minus infinity, no class.  (Rows that take no part come along.)
  {
    constexpr int W = N * LANES, kWide = W <= 16 ? 16 : W <= 32 ? 32 : 64, kOnce = 64 / kWide, kPieces = (W + 63) / 64, kBatch = kPieces == 1 ? 8 : 4;
    static_assert(kRows % (kOnce * kBatch) == 0, "whole batches");
    const int c = lane & (kWide - 1), y = lane / kWide;
    float b[kPieces];
#pragma unroll
    for (int q = 0; q < kPieces; ++q) b[q] = a.bias ? a.bias[min(c + 64 * q, C - 1)] : 0.f;
#pragma unroll 1
    for (int row0 = y; row0 < kRows; row0 += kOnce * kBatch) {
      T v[kBatch][kPieces];
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
#pragma unroll
        for (int q = 0; q < kPieces; ++q) v[i][q] = src[(uint32_t)(min(row0 + i * kOnce, rows - 1) * (int)a.ld) + (uint32_t)min(c + 64 * q, C - 1)];
      if (c < W) {  // (of 48 classes' lanes the last 16 have no place)
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
          for (int q = 0; q < kPieces; ++q)
            at[min(row0 + i * kOnce, rows - 1) * kPitch + c + 64 * q] = c + 64 * q < C ? (float)v[i][q] + b[q] + 0.f : -INFINITY;  // (minus zero is zero)
      }
    }
  }
  __syncthreads();
  if (mine >= rows) return;  // all lanes of the row
  if (!on) {
    write_none(a, r, sub, LANES);
    return;
  }
  const int id = given_class(a, r);
  float *const mine_at = at + mine * kPitch;
  const float zl = mine_at[max(id, 0)];
  float z[N];
  auto read = [&]() {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = mine_at[sub + i * LANES];
  };
  // (the row's lanes are of one wave, whose LDS instructions are done in their order)
  if (id >= 0 && sub == 0) mine_at[id] = -INFINITY;
  lds_written();
  read();
  Sums x = no_sums();
  x.top = id >= 0 ? zl : -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) x.top = fmaxf(x.top, z[i]);
  auto most_of = [&](float v) {
    if constexpr (LANES >= 2) v = fmaxf(v, lanes_xor<1>(v));
    if constexpr (LANES >= 4) v = fmaxf(v, lanes_xor<2>(v));
    return v;
  };
  auto sum_of = [&](float v) {
    if constexpr (LANES >= 2) v += lanes_xor<1>(v);
    if constexpr (LANES >= 4) v += lanes_xor<2>(v);
    return v;
  };
  x.top = most_of(x.top);
  x.m = fmaxf(x.top, kNoMax);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = z[i] - x.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    x.s += e;
    x.t = fmaf(e, fmaxf(d, -200.f), x.t);
  }
  x.s = sum_of(x.s);
  x.t = sum_of(x.t);
  const Answer w = end_row(x, id >= 0, zl);
  if (sub == 0) write_row(a, r, w);
  if (a.n_top == 0) return;
  // The best, the lowest class that has it, which then is no number any more, and so on.
  if (id >= 0 && sub == 0) mine_at[id] = zl;
  for (int n = 0; n < a.n_top; ++n) {
    lds_written();
    read();
    float v = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) v = fmaxf(v, z[i]);
    v = most_of(v);
    int c = N * LANES;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) c = z[i] == v ? sub + i * LANES : c;
    if constexpr (LANES >= 2) c = min(c, (int)lanes_xor<1>((uint32_t)c));
    if constexpr (LANES >= 4) c = min(c, (int)lanes_xor<2>((uint32_t)c));
    if (sub == 0) {
      if (c < C) mine_at[c] = NAN;
      write_best(a, r, n, c < C ? key_of(v, c) : 0, w);
    }
  }
}

// A wave per row (WAVES 1: four rows per workgroup), or a workgroup of four waves per row or part of one.  Bound by the vector units next to memory: 64 logits take 13
// vector instructions, one of them the exponential (8,191 x 100,003 bf16 with bias, ten best: 170 M of them, 400 us, 4.1 TB/s; reads alone would take 268).
template <typename T, bool TOP, bool BIAS, int WAVES>
__global__ __launch_bounds__(256) void answer_kernel(const AnswerArgs a) {
  __shared__ Key room[TOP ? 4 * kWaiting : 1];
  __shared__ Sums met[4];
  __shared__ float borders[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (r >= a.rows) return;  // the whole wave (WAVES 1), nobody else's
  if (a.mask && a.mask[r] == 0) {
    if (WAVES == 1 || (wave == 0 && blockIdx.y == 0)) write_none(a, r, lane, 64);
    return;
  }
  const T *row = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
  const int id = given_class(a, r);
  Sums x = no_sums();
  Best best(room + (TOP ? wave * kWaiting : 0), borders, WAVES > 1, a.n_top);
  int c0 = 0, c1 = a.C;
  if constexpr (WAVES > 1) {
    if constexpr (TOP) {
      if (lane == 0) borders[wave] = NAN;
      __syncthreads();
    }
    const int begin = (int)blockIdx.y * a.part, end = min(a.C, begin + a.part), each = ((end - begin + 3) / 4 + 63) / 64 * 64;
    c0 = min(end, begin + wave * each);
    c1 = min(end, c0 + each);
  }
  scan<T, TOP, BIAS>(row, a.bias, c0, c1, id, x, best);
  if constexpr (TOP) best.settle();
  join_lanes(x);
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
  __shared__ float unused[1];
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  if (a.mask && a.mask[r] == 0) return;  // written
  const int id = given_class(a, r);
  Sums x = no_sums();
  for (int i = lane; i < a.splits; i += 64) join(x, a.part_sums[r * a.splits + i]);
  join_lanes(x);
  const T *row = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
  const Answer w = end_row(x, id >= 0, given_logit(a, row, id));
  if (lane == 0) write_row(a, r, w);
  if constexpr (TOP) {
    Best best(room, unused, false, a.n_top);
    const int n = a.n_top * a.splits;
    for (int i0 = 0; i0 < n; i0 += 64) {
      const Key k = i0 + lane < n ? a.part_keys[r * n + i0 + lane] : 0;
      // (of equal logits the lower class may come later here)
      best.wait(k != 0 && !(logit_of(k) < best.least) ? k : 0);
      if (best.full()) best.settle();
    }
    best.settle();
    if (lane < a.n_top) write_best(a, r, lane, best.list, w);
  }
}

constexpr int kMostTop = 64;
// Rows of at most kShort classes go through LDS (answer_short_kernel), beyond 64 with at most kShortTop best classes, each of which goes over all of the row.  fp32, in us,
// through LDS / a wave per row: 50,000 x 41, 3 best 13 / 58; x 64, 60 best 52 / 62; x 200, 8 best 31 / 54, 20 best 52 / 60, 32 best 75 / 65, 64 best 129 / 90.
constexpr int kShort = 256, kShortTop = 24;
constexpr int kLanes = 2;  // of a row of at most 64 classes (232,965 x 41, 3 best, 66 % of the rows: 1, 2, 4 lanes 25, 22, 25 us, with a place worked out per element)
// Others take a wave per row, or a workgroup where the classes are many and the rows few.  fp32, 5 best, in us, a wave / a workgroup: 600 x 4,000 14 / 13, 600 x 8,000
// 19 / 13, 1,000 x 20,000 33 / 24, 1,000 x 100,003 125 / 75, 2,000 x 20,000 36 / 38, 2,000 x 100,003 151 / 149, 5,000 x 1,000 14 / 27, 5,000 x 8,000 34 / 48, 8,191 x 100,003 587 / 562 (bf16,
// ten best, with bias 400 / 417).
constexpr int kLong = 4096;
constexpr int64_t kManyRows = 2048;
constexpr int kWorkgroups = 512;    // that a launch of them should have: fewer rows are cut
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
  // as many rows at a time as a launch takes workgroups for: launch(arguments, workgroups)
  auto slabs = [&](int64_t rows_each, int64_t threads, auto launch) {
    const int64_t most = kMostBlocks * 256 / threads * rows_each;
    for (int64_t r = 0; r < a.rows; r += most) {
      AnswerArgs b = a;
      b.logits = static_cast<const T *>(a.logits) + (size_t)(r * a.ld);
      b.rows = std::min(most, a.rows - r);
      b.ids = a.ids ? a.ids + r : nullptr;
      b.mask = a.mask ? a.mask + r : nullptr;
      b.logp = a.logp ? a.logp + r : nullptr;
      b.entropy = a.entropy ? a.entropy + r : nullptr;
      b.norm = a.norm ? a.norm + 2 * r : nullptr;
      b.top_ids = a.top_ids ? a.top_ids + r * a.n_top : nullptr;
      b.top_logp = a.top_logp ? a.top_logp + r * a.n_top : nullptr;
      launch(b, (unsigned)((b.rows + rows_each - 1) / rows_each));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return (int)e;
    }
    return (int)hipSuccess;
  };
  if (a.C <= kShort && (a.C <= 64 || a.n_top <= kShortTop) && a.ld < 1 << 24) {  // (64 rows' places fit 32 bits)
    return slabs(a.C <= 64 ? 64 / kLanes : 16, 64, [&](const AnswerArgs &b, unsigned gx) {
      auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(gx), dim3(64), 0, s, b); };
      if (a.C <= 16) run(answer_short_kernel<T, kLanes, 16 / kLanes>);
      else if (a.C <= 32) run(answer_short_kernel<T, kLanes, 32 / kLanes>);
      else if (a.C <= 48) run(answer_short_kernel<T, kLanes, 48 / kLanes>);
      else if (a.C <= 64) run(answer_short_kernel<T, kLanes, 64 / kLanes>);
      else if (a.C <= 128) run(answer_short_kernel<T, 4, 32>);
      else run(answer_short_kernel<T, 4, 64>);
    });
  }
  if (a.C < kLong || a.rows >= kManyRows) return slabs(4, 256, [&](const AnswerArgs &b, unsigned gx) { hipLaunchKernelGGL((a.bias ? answer_kernel<T, TOP, true, 1> : answer_kernel<T, TOP, false, 1>), dim3(gx), dim3(256), 0, s, b); });
  const int e = slabs(1, 256, [&](const AnswerArgs &b, unsigned gx) { hipLaunchKernelGGL((a.bias ? answer_kernel<T, TOP, true, 4> : answer_kernel<T, TOP, false, 4>), dim3(gx, (unsigned)p.splits), dim3(256), 0, s, b); });
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
  int64_t rows_per;      // rows of a group
  uint32_t blocks, groups, per_xcd;  // workgroups along a row, groups of rows, workgroups of an XCD
};
struct RowGrad {
  float M, log_s;
  float a, b, b_own, own;  // dz = p (a log p + b), of the given class own + p (a log p + b_own), own = g_logp (1 - p) without the cancellation
  int32_t id, on;
};
constexpr int kAhead = 4;       // rows of a thread on their way
constexpr int kChain = 32;      // rows of a thread that dbias adds up in one chain, of which there is then one of their sums
constexpr int kRowsAhead = 256;  // at most whose numbers are in LDS at a time

// Workgroups own columns and go down their group's rows: the bias is read once per group, its gradient stays in registers.  Bound by memory: 8,191 x 100,003 bf16 3.28 GB in 690 us,
// 4.8 TB/s (rows of 200,006 bytes, whose lines two workgroups share; at whole lines a copy of this shape has 5.4).
template <typename T, typename O, bool SUMS>
__global__ __launch_bounds__(256) void grad_kernel(const GradArgs a) {
  constexpr int N = 16 / (sizeof(T) < sizeof(O) ? sizeof(O) : sizeof(T));
  typedef typename Vec<T, N>::type TV;
  typedef typename Vec<O, N>::type OV;
  __shared__ RowGrad of[kRowsAhead];
  __shared__ float columns[SUMS ? 256 * N : 1];
  // an XCD's workgroups follow one another along the rows: the lines that two of them share are written at about the same time
  const uint32_t at = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3), group = at / a.blocks, block = at - group * a.blocks;
  if (group >= a.groups) return;
  const int down = 256 / a.across, ty = threadIdx.x / a.across, tx = threadIdx.x - ty * a.across;
  const int c = ((int)block * a.across + tx) * N;
  const bool mine = ty < down && c < a.C, whole = c + N <= a.C;
  float b[N], sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    b[i] = a.bias && mine && c + i < a.C ? a.bias[c + i] : 0.f;
    sum[i] = 0.f;
  }
  const int chunk = min(kRowsAhead, kChain * down);
  const int64_t r_end = min(a.rows, ((int64_t)group + 1) * a.rows_per);
  for (int64_t r0 = (int64_t)group * a.rows_per; r0 < r_end; r0 += chunk) {
    const int n = (int)min((int64_t)chunk, r_end - r0);
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
        if (a.g_entropy) {
          w.a = -a.g_entropy[r];
          w.b_own = w.a * a.entropy[r];
        }
        w.b = w.b_own;
        if (a.g_logp && (uint32_t)id < (uint32_t)a.C) {
          const float gl = a.g_logp[r];
          w.id = id;
          w.b -= gl;
          w.own = -expm1f(a.logp[r]) * gl;
        }
      }
      of[threadIdx.x] = w;
    }
    __syncthreads();
    if (!mine) continue;
    float chain[N];
#pragma unroll
    for (int i = 0; i < N; ++i) chain[i] = 0.f;
    auto row_of = [&](int k) { return static_cast<const T *>(a.logits) + (size_t)((r0 + k) * a.ld) + c; };
    auto grad = [&](const RowGrad &w, const float (&z)[N], float (&g)[N]) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float log_p = z[i] + b[i] - w.M - w.log_s, p = __builtin_amdgcn_exp2f(log_p * kLog2e);
        g[i] = p * fmaf(w.a, fmaxf(log_p, -200.f), w.b);
      }
      if ((uint32_t)(w.id - c) < (uint32_t)N) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float log_p = z[i] + b[i] - w.M - w.log_s;
          const float own = w.own + __builtin_amdgcn_exp2f(log_p * kLog2e) * fmaf(w.a, fmaxf(log_p, -200.f), w.b_own);
          g[i] = c + i == w.id ? own : g[i];
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        g[i] = w.on ? g[i] : 0.f;
        chain[i] += g[i];
      }
    };
    auto vector_row = [&](int k, const TV &v) {
      float z[N], g[N];
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = (float)v[i];
      grad(of[k], z, g);
      OV o;
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = (O)g[i];
      *reinterpret_cast<OV *>(static_cast<O *>(a.dlogits) + (size_t)((r0 + k) * a.ld_dl) + c) = o;
    };
    if (__all(whole)) {
      // kAhead rows at a time; the next ones' loads go ahead of the stores of these, without a branch between: an access is waited for together with all in front
      // of it, of whatever kind.  (What a row's store may overwrite is that row.)
      const int batches = (n - ty + kAhead * down - 1) / (kAhead * down);
      TV next[kAhead];
      auto load = [&](int k0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) next[j] = *reinterpret_cast<const TV *>(row_of(min(k0 + j * down, n - 1)));
      };
      load(ty);
      int k0 = ty;
      for (int i = 0; i + 1 < batches; ++i, k0 += kAhead * down) {
        TV v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = next[j];
        load(k0 + kAhead * down);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) vector_row(k0 + j * down, v[j]);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (k0 + j * down < n) vector_row(k0 + j * down, next[j]);
    } else {
      for (int k = ty; k < n; k += down) {
        if (whole) {
          vector_row(k, *reinterpret_cast<const TV *>(row_of(k)));
          continue;
        }
        float z[N], g[N];
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = c + i < a.C ? (float)row_of(k)[i] : -INFINITY;
        grad(of[k], z, g);
        O *dst = static_cast<O *>(a.dlogits) + (size_t)((r0 + k) * a.ld_dl) + c;
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
      const int col = (int)block * a.across * N + i;
      if (col >= a.C) continue;
      float s = 0.f;
      for (int y = 0; y < down; ++y) s += columns[y * a.across * N + i];
      if (a.part)
        a.part[(size_t)group * a.C + col] = s;
      else
        a.dbias[col] += s;
    }
  }
}

// dbias += the groups' sums: WIDE columns a workgroup, the groups among its 1024 / WIDE rows of threads
template <int WIDE>
__global__ __launch_bounds__(1024) void grad_bias_kernel(const float *part, int groups, int C, float *dbias) {
  constexpr int kDown = 1024 / WIDE;
  __shared__ float of[kDown][WIDE];
  const int x = threadIdx.x % WIDE, y = threadIdx.x / WIDE, c = blockIdx.x * WIDE + x;
  float s = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int g = y; g < groups; g += kDown) s += part[(size_t)g * C + c];
  }
  of[y][x] = s;
  __syncthreads();
  for (int w = kDown / 2; w > 0; w >>= 1) {
    if (y < w) of[y][x] += of[y + w][x];
    __syncthreads();
  }
  if (y == 0 && c < C) dbias[c] += of[0][x];
}

constexpr int kNarrow = 4096;  // classes up to which a workgroup adds up 16 of them, else 128 (wide pieces of the groups' rows)
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
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kPartElements / C, kMostBlocks / 2 / p.blocks));
  // Workgroups that end soon keep in step with those beside them (rows of 200 KB at odd places, copied: 32 rows each 5.2 TB/s, 195 4.5), 2,048 of them at least.  In us, with 512 / 1,024 /
  // 2,048 / 4,096 at least, dbias among them: 232,965 x 41 fp32 34 / 25 / 28 / 27, 70,001 x 172 fp32 24.5 / 24.6 / 26.6 / 31.7, bf16 33 / 40 / 39 / 39, 20,000 x 1,000 fp32 35 / 35 / 36 / 42,
  // 8,191 x 100,003 bf16 716 with any.
  const int64_t few = std::max<int64_t>(kAhead * down, (rows * p.blocks + 2047) / 2048);
  p.rows_per = std::max<int64_t>(std::min<int64_t>(kChain * down, few), (rows + most - 1) / most);
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
  a.blocks = (uint32_t)p.blocks;
  a.groups = (uint32_t)p.groups;
  a.per_xcd = (a.blocks * a.groups + 7) / 8;
  hipLaunchKernelGGL((a.dbias ? grad_kernel<T, O, true> : grad_kernel<T, O, false>), dim3(a.per_xcd * 8), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias || p.groups == 1) return (int)e;
  if (a.C <= kNarrow)
    hipLaunchKernelGGL(grad_bias_kernel<16>, dim3((unsigned)((a.C + 15) / 16)), dim3(1024), 0, s, room, (int)p.groups, a.C, a.dbias);
  else
    hipLaunchKernelGGL(grad_bias_kernel<128>, dim3((unsigned)((a.C + 127) / 128)), dim3(1024), 0, s, room, (int)p.groups, a.C, a.dbias);
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
