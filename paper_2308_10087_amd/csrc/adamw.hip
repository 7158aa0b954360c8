// One AdamW step (Loshchilov & Hutter, ICLR 2019, Algorithm 2) over many tensors at once, the two running means in 32 or in 8 bits.
//
//   g = scale g;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  p = p (1 - lr wd) - lr c1 m / (sqrt(v c2) + eps),  c = 1 / (1 - b^t)
//
// In 8 bits a tensor keeps m and r = sqrt(v), whose range is the gradients' and not that of their squares, in blocks of 32 elements with a power
// of two each (the byte e + 127) and codes of 4 bits of exponent and 3 of mantissa (the finite numbers of OCP's e4m3; a block is one of its
// MXFP8 blocks):
//
//   a = max |x| over the block, e = the least whole number with a <= 1.75 2^8 2^e, held within [-117, 119]
//   y = |x| / 2^e, its spacing s = 2^(max(binade of y, -6) - 3), code of s floor(y / s + u),  u of 0 .. 65535 / 65536
//
// The rounding is a draw, up with the probability of y's place between its neighbours: v moves by a thousandth of itself per step, codes are
// 6 to 12 % apart, so that nearest rounding would leave it where it is for good; a draw keeps the mean of r.  That of v = r^2 then has the draws' variance in it: a step moves r by
// D = (1 - b2) |g^2 - v| / (2 r) off a code, of which a draw makes up to D s of variance, which decays by b2 a step: v is too large by up to E|g^2 - v| s / (2 r), whatever b2 is (less than 14 %
// of it down to 2^-14 of the block's largest root; 3 to 4 % for normal gradients, 6 % for such of one step in fifty).  r > 0 does not become 0 (that would
// divide by eps alone): it is rounded to the least code at least.  The draws are SplitMix64's (Steele, Lea, Flood 2014): elements 2 j and 2 j + 1
// of a tensor have the low and the high half of the output for state key + (j + 1) gamma, 16 bits for m and 16 above them for r; tensor k's key is
// the output for state output(seed + t gamma) + (k + 1) gamma.
//
// Every operation up to a code is one rounding of fp32 (no contraction), so that a program can say which code it will be.
#include <hip/hip_runtime.h>
#include "guard.h"

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "../../include/gnntrain.h"
#include "adamw.h"
#include "common.h"

#pragma clang fp contract(off)

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
// tensors start anywhere: the memory system takes vectors at any address of their elements
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
typedef bf16_t bf16x4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;
__host__ __device__ inline uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

constexpr int kTensors = 40;  // of a launch: its arguments stay below 4 KB
struct Tensor {
  float *p;
  const void *g;
  void *m, *v;
  uint8_t *m_scale, *v_scale;
  void *compute;
  int64_t n;
  uint64_t key;
  float keep;  // 1 - lr wd
  int8_t g_bf16, compute_bf16, unused[2];
};
struct Args {
  Tensor t[kTensors];
  int32_t first[kTensors];  // workgroup (negative: a tensor that the launch in front of this one began); past the last tensor: beyond every one
  const float *grad_scale;
  float b1, b2, a1, a2, rate, root_scale, eps;  // a = 1 - b, rate = lr c1, root_scale = sqrt(c2)
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

template <typename T, typename V>
__device__ __forceinline__ f32x4 load4(const T *x, int64_t i, int64_t n) {
  f32x4 r = {0.f, 0.f, 0.f, 0.f};
  if (i + 4 <= n) {
    const V v = *reinterpret_cast<const V *>(x + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = (float)v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) r[k] = (float)x[i + k];
  }
  return r;
}
template <typename T, typename V>
__device__ __forceinline__ void store4(T *x, int64_t i, int64_t n, f32x4 r) {
  if (i + 4 <= n) {
    V v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (T)r[k];
    *reinterpret_cast<V *>(x + i) = v;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) x[i + k] = (T)r[k];
  }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *x, int64_t i, int64_t n) {
  if (i + 4 <= n) return *reinterpret_cast<const uint32_t *>(x + i);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (i + k < n) w |= (uint32_t)x[i + k] << (8 * k);
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t *x, int64_t i, int64_t n, uint32_t w) {
  if (i + 4 <= n) {
    *reinterpret_cast<uint32_t *>(x + i) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) x[i + k] = (uint8_t)(w >> (8 * k));
  }
}
// the numbers of four codes and their block's byte (0: a block of zeros, as it is cleared; 255: infinity, which makes every NaN code NaN)
__device__ __forceinline__ f32x4 decode4(uint32_t w, uint32_t scale) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const float f = __builtin_bit_cast(float, scale << 23);
  return f32x4{lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f};
}
// Four elements of a block that eight neighbouring lanes share; u: a draw of 16 bits each.  POSITIVE: roots, which stay above zero.
template <bool POSITIVE>
__device__ __forceinline__ uint32_t encode4(f32x4 four, const uint32_t (&u)[4], uint32_t &scale) {
  const float x[4] = {four[0], four[1], four[2], four[3]};  // (a vector's element has no address that its bits could be taken from)
  uint32_t a = 0;  // the largest magnitude, compared as bits: infinities and NaNs are above every number
#pragma unroll
  for (int k = 0; k < 4; ++k) a = max(a, __builtin_bit_cast(uint32_t, x[k]) & 0x7fffffffu);
  a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2 of the quad
  a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
  a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x141, 0xf, 0xf, true));  // lanes 7 .. 0 of the eight
  if (a >= 0x7f000000u) {  // 2^127 and beyond, which a code may be rounded up out of
    scale = 255;
    return 0x7f7f7f7fu;
  }
  // a = f 2^(E - 127) <= 1.75 2^(8 + e): e = E - 127 - 8 up to f = 1.75, one more beyond
  const int e = max((int)(a >> 23) - 135 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), -117);
  scale = (uint32_t)(e + 127);
  const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float y = fabsf(x[k]) * inv;
    const uint32_t binade = max(__builtin_bit_cast(uint32_t, y) >> 23, 121u);
    const float t = y * __builtin_bit_cast(float, (257u - binade) << 23) + (float)u[k] * 0x1p-16f;
    uint32_t c = (binade - 121u) * 8u + (uint32_t)t;
    if (POSITIVE)
      c = x[k] > 0.f ? max(c, 1u) : c;
    else
      c |= (__builtin_bit_cast(uint32_t, x[k]) >> 24) & 0x80u;
    w |= c << (8 * k);
  }
  return w;
}

// Workgroups go through 1,024 ITER elements of one tensor each.  Bound by memory: 26.2 M elements with fp32 states and a bf16 copy (0.79 GB) 138 - 154 us, 5.1 - 5.7 TB/s; 102.7 M with
// states in 8 bits and bf16 gradients (1.66 GB) 307 us, 5.4 TB/s, next to about 100 vector instructions an element.
template <int BITS, int ITER>
__global__ __launch_bounds__(256) void adamw_kernel(const Args a) {
  // whose workgroup this is: a lane per tensor
  const int lane = threadIdx.x & 63;
  const int which = __popcll(__ballot(lane < kTensors && a.first[min(lane, kTensors - 1)] <= (int)blockIdx.x)) - 1;
  const Tensor &x = a.t[which];
  const int64_t n = x.n, i0 = ((int64_t)((int)blockIdx.x - a.first[which]) * ITER) * 1024 + threadIdx.x * 4;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  f32x4 p[ITER], g[ITER], m[ITER], v[ITER];
  uint32_t mc[ITER], vc[ITER], ms[ITER], vs[ITER];
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int64_t i = i0 + it * 1024;
    p[it] = load4<float, f32x4_u>(x.p, i, n);
    g[it] = x.g_bf16 ? load4<bf16_t, bf16x4_u>(static_cast<const bf16_t *>(x.g), i, n) : load4<float, f32x4_u>(static_cast<const float *>(x.g), i, n);
    if constexpr (BITS == 32) {
      m[it] = load4<float, f32x4_u>(static_cast<const float *>(x.m), i, n);
      v[it] = load4<float, f32x4_u>(static_cast<const float *>(x.v), i, n);
    } else {
      mc[it] = load_codes(static_cast<const uint8_t *>(x.m), i, n);
      vc[it] = load_codes(static_cast<const uint8_t *>(x.v), i, n);
      ms[it] = i < n ? x.m_scale[i >> 5] : 0u;
      vs[it] = i < n ? x.v_scale[i >> 5] : 0u;
    }
  }
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int64_t i = i0 + it * 1024;
    f32x4 root;
    if constexpr (BITS == 8) {
      m[it] = decode4(mc[it], ms[it]);
      v[it] = decode4(vc[it], vs[it]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float gk = g[it][k] * gs;
      m[it][k] = a.b1 * m[it][k] + a.a1 * gk;
      if constexpr (BITS == 8) v[it][k] = v[it][k] * v[it][k];
      v[it][k] = a.b2 * v[it][k] + a.a2 * gk * gk;
      root[k] = sqrtf(v[it][k]);
      p[it][k] = p[it][k] * x.keep - a.rate * m[it][k] / (root[k] * a.root_scale + a.eps);
    }
    store4<float, f32x4_u>(x.p, i, n, p[it]);
    if (x.compute) {
      if (x.compute_bf16)
        store4<bf16_t, bf16x4_u>(static_cast<bf16_t *>(x.compute), i, n, p[it]);
      else
        store4<float, f32x4_u>(static_cast<float *>(x.compute), i, n, p[it]);
    }
    if constexpr (BITS == 32) {
      store4<float, f32x4_u>(static_cast<float *>(x.m), i, n, m[it]);
      store4<float, f32x4_u>(static_cast<float *>(x.v), i, n, v[it]);
    } else {
      const uint64_t w0 = mix(x.key + (uint64_t)(i / 2 + 1) * kGolden), w1 = mix(x.key + (uint64_t)(i / 2 + 2) * kGolden);
      const uint32_t h[4] = {(uint32_t)w0, (uint32_t)(w0 >> 32), (uint32_t)w1, (uint32_t)(w1 >> 32)};
      uint32_t um[4], uv[4], m_scale, v_scale;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        um[k] = h[k] & 0xffffu;
        uv[k] = h[k] >> 16;
        if (i + k >= n) m[it][k] = root[k] = 0.f;  // (0 / eps + ... never reaches a neighbour's block)
      }
      const uint32_t cm = encode4<false>(m[it], um, m_scale), cv = encode4<true>(root, uv, v_scale);
      store_codes(static_cast<uint8_t *>(x.m), i, n, cm);
      store_codes(static_cast<uint8_t *>(x.v), i, n, cv);
      if ((lane & 7) == 0 && i < n) {
        x.m_scale[i >> 5] = (uint8_t)m_scale;
        x.v_scale[i >> 5] = (uint8_t)v_scale;
      }
    }
  }
}

// Elements from which fp32 states take four parts a workgroup, which have four times the loads in flight.  The kernel in us, one part / four, with a bf16 copy: one tensor of 2^18 elements 3.2 /
// 5.0, 2^20 5.5 / 6.7, 2^21 8.8 / 9.2, 2^22 21.0 / 19.3, 2^23 38.2 / 37.9, 2^26 369 / 371; 18 tensors of 2^18 in all 3.5 / 6.4, 2^21 9.6 / 11.0, 2^22 19.8 / 20.7, 2^23 39.3 / 38.8, 2^26 418 / 394.  8
// bits stay with one (2^26: 193 / 208).
constexpr int64_t kManyElements = 1 << 21;

}  // namespace

std::string adamw_check(const gnntrain_adamw_tensor *t, int n, int bits, const float *grad_scale) {
  struct Range {
    uintptr_t from, to;
    int tensor;  // -1: grad_scale
    bool written;
  };
  std::vector<Range> ranges;
  ranges.reserve((size_t)n * 7 + 1);
  for (int i = 0; i < n; ++i) {
    const gnntrain_adamw_tensor &x = t[i];
    auto bad = [&](const char *why) { return "tensor " + std::to_string(i) + ": " + why; };
    if (x.count < 0 || x.count > ((int64_t)1 << 35)) return bad("count must be in [0, 2^35]");
    if (x.count == 0) continue;
    if (!x.p || !x.g || !x.m || !x.v) return bad("p, g, m and v must not be NULL");
    if ((x.g_dtype != GNNSTAGE_F32 && x.g_dtype != GNNSTAGE_BF16) || (x.compute && x.compute_dtype != GNNSTAGE_F32 && x.compute_dtype != GNNSTAGE_BF16)) return bad("unknown dtype");
    const uintptr_t g_align = x.g_dtype == GNNSTAGE_BF16 ? 1 : 3, c_align = x.compute && x.compute_dtype == GNNSTAGE_BF16 ? 1 : 3;
    if (((reinterpret_cast<uintptr_t>(x.p) | reinterpret_cast<uintptr_t>(x.m) | reinterpret_cast<uintptr_t>(x.v)) & 3) || (reinterpret_cast<uintptr_t>(x.g) & g_align) ||
        (reinterpret_cast<uintptr_t>(x.compute) & c_align))
      return bad("a buffer is not aligned to its elements (codes: to four bytes)");
    if (bits == 8 && (!x.m_scale || !x.v_scale)) return bad("states in 8 bits need m_scale and v_scale");
    auto add = [&](const void *p, size_t bytes, bool written) {
      if (p) ranges.push_back(Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, i, written});
    };
    const size_t c = (size_t)x.count, state = bits == 32 ? 4 * c : c;
    add(x.p, 4 * c, true);
    add(x.g, (x.g_dtype == GNNSTAGE_BF16 ? 2 : 4) * c, false);
    add(x.m, state, true);
    add(x.v, state, true);
    if (bits == 8) {
      add(x.m_scale, (c + 31) / 32, true);
      add(x.v_scale, (c + 31) / 32, true);
    }
    if (x.compute != x.p) add(x.compute, (x.compute_dtype == GNNSTAGE_BF16 ? 2 : 4) * c, true);
    else if (x.compute_dtype != GNNSTAGE_F32) return bad("compute is p, but not of its type");
  }
  if (grad_scale) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(grad_scale);
    if (at & 3) return "grad_scale is not aligned to its element";
    ranges.push_back(Range{at, at + sizeof(float), -1, false});
  }
  // no written buffer meets another one (gradients may be shared): in the order of their beginnings, against what reaches furthest so far
  std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.from < b.from; });
  uintptr_t written_to = 0, read_to = 0;
  for (const Range &r : ranges) {
    if (r.from < written_to || (r.written && r.from < read_to)) {
      // (grad_scale may be the one that it meets)
      if (r.tensor < 0 || (grad_scale && r.from < reinterpret_cast<uintptr_t>(grad_scale + 1) && r.to > reinterpret_cast<uintptr_t>(grad_scale))) return "grad_scale lies in a buffer that the step writes";
      return "a buffer of tensor " + std::to_string(r.tensor) + " overlaps one that the step writes";
    }
    (r.written ? written_to : read_to) = std::max(r.written ? written_to : read_to, r.to);
  }
  return std::string();
}

int launch_adamw(const gnntrain_adamw_tensor *t, int n, int bits, const AdamwRates &r, const float *grad_scale, int64_t step, uint64_t seed, hipStream_t s) {
  Args a;
  a.grad_scale = grad_scale;
  a.b1 = r.beta1;
  a.b2 = r.beta2;
  a.a1 = 1.f - r.beta1;
  a.a2 = 1.f - r.beta2;
  // bias corrections 1 / (1 - beta^t), formed in double on the host
  a.rate = (float)((double)r.lr / (1.0 - std::pow((double)r.beta1, (double)step)));
  a.root_scale = (float)std::sqrt(1.0 / (1.0 - std::pow((double)r.beta2, (double)step)));
  a.eps = r.eps;
  const uint64_t base = mix(seed + (uint64_t)step * kGolden);
  int64_t all = 0;
  for (int i = 0; i < n; ++i) all += t[i].count;
  const bool many = bits == 32 && all >= kManyElements;
  const int64_t per = many ? 4096 : 1024;
  int64_t done = 0;  // workgroups of tensor i in earlier launches
  for (int i = 0; i < n;) {
    int k = 0;
    int64_t blocks = 0;
    while (i < n && k < kTensors && blocks < kMostBlocks) {
      const gnntrain_adamw_tensor &x = t[i];
      const int64_t left = (x.count + per - 1) / per - done, b = std::min(left, kMostBlocks - blocks);
      if (b > 0) {
        Tensor &y = a.t[k];
        y.p = x.p;
        y.g = x.g;
        y.m = x.m;
        y.v = x.v;
        y.m_scale = x.m_scale;
        y.v_scale = x.v_scale;
        y.compute = x.compute == x.p ? nullptr : x.compute;
        y.n = x.count;
        y.key = mix(base + (uint64_t)(i + 1) * kGolden);
        y.keep = (float)(1.0 - (double)r.lr * (double)x.weight_decay);
        y.g_bf16 = x.g_dtype == GNNSTAGE_BF16;
        y.compute_bf16 = x.compute_dtype == GNNSTAGE_BF16;
        a.first[k++] = (int32_t)(blocks - done);
        blocks += b;
      }
      if (b < left) {  // the others are the next launch's
        done += b;
        break;
      }
      done = 0;
      ++i;
    }
    if (k == 0) break;
    for (; k < kTensors; ++k) a.first[k] = INT32_MAX;
    hipLaunchKernelGGL((bits == 8 ? adamw_kernel<8, 1> : many ? adamw_kernel<32, 4> : adamw_kernel<32, 1>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (int)e;
  }
  return hipSuccess;
}

extern "C" int gnntrain_adamw_step(const gnntrain_adamw_tensor *tensors, int32_t n, int32_t state_bits, float lr, float beta1, float beta2, float eps,
                                   const float *grad_scale, int64_t t, uint64_t seed, void *hip_stream) try {
  const char *const me = "gnntrain_adamw_step: ";
  if (state_bits != 32 && state_bits != 8) return train_error(GNNSTAGE_EINVAL, std::string(me) + "state_bits must be 32 or 8");
  if (n < 0 || (n > 0 && !tensors)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "n must not be negative, nor tensors NULL");
  if (t < 1) return train_error(GNNSTAGE_EINVAL, std::string(me) + "t counts from 1");
  if (!(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f)) return train_error(GNNSTAGE_EINVAL, std::string(me) + "beta1 and beta2 must be in [0, 1)");
  const std::string err = adamw_check(tensors, n, state_bits, grad_scale);
  if (!err.empty()) return train_error(GNNSTAGE_EINVAL, me + err);
  const int e = launch_adamw(tensors, n, state_bits, AdamwRates{lr, beta1, beta2, eps}, grad_scale, t, seed, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return train_error(GNNSTAGE_EHIP, me + std::string(hipGetErrorString((hipError_t)e)));
  return GNNSTAGE_OK;
}
GNNSTAGE_GUARD_INT
