// fp32 products of the loss head in pieces (head.hip): logits and row gradients
//
//   NT:  C[M x N] (+)= A[M x K] . B[N x K]^T
//   TN:  D[I x O] += A[M x I]^T . B[M x O], column sums of B on the side
//
// on v_mfma_f32_32x32x2_f32.  Nothing hangs on the last bit of these sums (no ReLU decides on them), so unlike the products of the stages'
// fp32 layers, whose outputs are each one chain of additions in the order of k, they may be added up in blocks of 256 products, which is nearer to
// 64 bits, and use tiles that feed the matrix cores: 128 x 128 (or 64) outputs per workgroup, 32 steps of the reduction at a time in two LDS
// buffers filled by direct loads, two workgroups per compute unit.
// Bound by the fp32 matrix cores: the head of 5,196 rows of 1,000 columns and 2,003 classes, 62 GFLOP, takes 725 us with them, 86 TFLOP/s, and 840 us
// with the layers' products.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lds_tile.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int BK = 32;     // of the reduction, per LDS tile
constexpr int BLOCK = 8;   // tiles of one chain of additions
static __device__ __align__(16) float zeros32[4];

__device__ __forceinline__ void wait_tile() {
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt 0
  __syncthreads();
}

// ---- NT.  A tile row is 32 floats of k (eight 16-byte pieces, permuted by the row: 16 rows side by side meet no bank twice).  A lane reads four k at a
// time, half h of a wave the k 8 g + 4 h ..: the matrix instructions pair k with k + 4, in both operands alike.
struct Nt32Args {
  const float *A, *B;
  int64_t lda, ldb, ldc;
  int32_t M, N, K;  // K a multiple of 4; rows 16-byte aligned
  float *C;
  int32_t add;      // C += instead of C =
};
template <int BN>
__global__ __launch_bounds__(256, 2) void nt32_kernel(const Nt32Args a) {
  constexpr int JT = BN / 64;
  __shared__ __attribute__((aligned(1024))) char a0[128 * BK * 4];
  __shared__ __attribute__((aligned(1024))) char a1[128 * BK * 4];
  __shared__ __attribute__((aligned(1024))) char b0[BN * BK * 4];
  __shared__ __attribute__((aligned(1024))) char b1[BN * BK * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  // an XCD takes a run of tiles: those of the same rows of A share its L2
  const int work = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), nt = (a.N + BN - 1) / BN;
  const int m0 = work / nt * 128, n0 = work % nt * BN;
  if (m0 >= a.M) return;
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * (BN / 2);
  auto load = [&](int k0, lds_char *as, lds_char *bs) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = (q * 4 + wave) * 8 + (lane >> 3), k = k0 + (((lane & 7) ^ ((r >> 1) & 7)) << 2);
      load_lds16(k < a.K ? static_cast<const void *>(a.A + (size_t)min(m0 + r, a.M - 1) * a.lda + k) : zeros32, as + (q * 4 + wave) * 1024);
    }
#pragma unroll
    for (int q = 0; q < BN / 32; ++q) {
      const int r = (q * 4 + wave) * 8 + (lane >> 3), k = k0 + (((lane & 7) ^ ((r >> 1) & 7)) << 2);
      load_lds16(k < a.K ? static_cast<const void *>(a.B + (size_t)min(n0 + r, a.N - 1) * a.ldb + k) : zeros32, bs + (q * 4 + wave) * 1024);
    }
  };
  f32x16 acc[2][JT], sum[2][JT];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < 16; ++t) acc[i][j][t] = sum[i][j][t] = 0.f;
  auto close = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          sum[i][j][t] += acc[i][j][t];
          acc[i][j][t] = 0.f;
        }
  };
  const int row = lane & 31, turn = (row >> 1) & 7;
  auto step = [&](int k0, const lds_char *as, const lds_char *bs, lds_char *as_next, lds_char *bs_next) {
    wait_tile();
    if (k0 + BK < a.K) load(k0 + BK, as_next, bs_next);
#pragma unroll
    for (int g = 0; g < BK / 8; ++g) {
      f32x4 fa[2], fb[JT];
      const int at = ((2 * g + h) ^ turn) << 4;
#pragma unroll
      for (int i = 0; i < 2; ++i) fa[i] = *reinterpret_cast<const LDS_AS f32x4 *>(as + (wm + 32 * i + row) * (BK * 4) + at);
#pragma unroll
      for (int j = 0; j < JT; ++j) fb[j] = *reinterpret_cast<const LDS_AS f32x4 *>(bs + (wn + 32 * j + row) * (BK * 4) + at);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < JT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i][e], fb[j][e], acc[i][j], 0, 0, 0);
    }
    if (k0 / BK % BLOCK == BLOCK - 1) close();
  };
  load(0, (lds_char *)a0, (lds_char *)b0);
  for (int k0 = 0; k0 < a.K; k0 += 2 * BK) {
    step(k0, (const lds_char *)a0, (const lds_char *)b0, (lds_char *)a1, (lds_char *)b1);
    if (k0 + BK < a.K) step(k0 + BK, (const lds_char *)a1, (const lds_char *)b1, (lds_char *)a0, (lds_char *)b0);
  }
  close();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      float old[16];
      const int n = n0 + wn + 32 * j + row;
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int m = m0 + wm + 32 * i + 8 * (t >> 2) + 4 * h + (t & 3);
        old[t] = a.add && m < a.M && n < a.N ? a.C[(size_t)m * a.ldc + n] : 0.f;
      }
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int m = m0 + wm + 32 * i + 8 * (t >> 2) + 4 * h + (t & 3);
        if (m < a.M && n < a.N) a.C[(size_t)m * a.ldc + n] = old[t] + sum[i][j][t];
      }
    }
}

// ---- TN.  A tile is 32 rows of 128 columns as they lie in memory; a lane reads one column of two neighbouring rows.
struct Tn32Args {
  const float *A, *B;
  int64_t lda, ldb;
  int32_t M, I, O;        // rows 16-byte aligned and readable up to I and O rounded up to 4
  int32_t splits, rows_per;
  float *part, *part_sum;  // [split][I][O], [split][O] (NULL: no column sums)
};
__global__ __launch_bounds__(256, 2) void tn32_kernel(const Tn32Args a) {
  __shared__ __attribute__((aligned(1024))) char a0[BK * 512];
  __shared__ __attribute__((aligned(1024))) char a1[BK * 512];
  __shared__ __attribute__((aligned(1024))) char b0[BK * 512];
  __shared__ __attribute__((aligned(1024))) char b1[BK * 512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int work = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), ti = (a.I + 127) / 128, tiles = ti * ((a.O + 127) / 128);
  const int tile = work % tiles, split = work / tiles;
  if (split >= a.splits) return;
  const int i0 = tile % ti * 128, o0 = tile / ti * 128, r_begin = split * a.rows_per, r_end = min(a.M, r_begin + a.rows_per);
  const int wi = (wave >> 1) * 64, wo = (wave & 1) * 64;
  auto load = [&](int r0, lds_char *as, lds_char *bs) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = r0 + (q * 4 + wave) * 2 + (lane >> 5), c = (lane & 31) * 4;
      load_lds16(r < r_end && i0 + c < a.I ? static_cast<const void *>(a.A + (size_t)r * a.lda + i0 + c) : zeros32, as + (q * 4 + wave) * 1024);
      load_lds16(r < r_end && o0 + c < a.O ? static_cast<const void *>(a.B + (size_t)r * a.ldb + o0 + c) : zeros32, bs + (q * 4 + wave) * 1024);
    }
  };
  f32x16 acc[2][2], sum[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < 16; ++t) acc[i][j][t] = sum[i][j][t] = 0.f;
  auto close = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          sum[i][j][t] += acc[i][j][t];
          acc[i][j][t] = 0.f;
        }
  };
  const bool sums = a.part_sum != nullptr && i0 == 0 && threadIdx.x < 128;
  float column = 0.f;
  auto step = [&](int r0, const lds_char *as, const lds_char *bs, lds_char *as_next, lds_char *bs_next) {
    wait_tile();
    if (r0 + BK < r_end) load(r0 + BK, as_next, bs_next);
#pragma unroll
    for (int k = 0; k < BK; k += 2) {
      float fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) fa[i] = *reinterpret_cast<const LDS_AS float *>(as + (k + h) * 512 + (wi + 32 * i + (lane & 31)) * 4);
#pragma unroll
      for (int j = 0; j < 2; ++j) fb[j] = *reinterpret_cast<const LDS_AS float *>(bs + (k + h) * 512 + (wo + 32 * j + (lane & 31)) * 4);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
    if (sums) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < BK; ++k) x += *reinterpret_cast<const LDS_AS float *>(bs + k * 512 + threadIdx.x * 4);
      column += x;
    }
    if ((r0 - r_begin) / BK % BLOCK == BLOCK - 1) close();
  };
  if (r_begin < r_end) load(r_begin, (lds_char *)a0, (lds_char *)b0);
  for (int r0 = r_begin; r0 < r_end; r0 += 2 * BK) {
    step(r0, (const lds_char *)a0, (const lds_char *)b0, (lds_char *)a1, (lds_char *)b1);
    if (r0 + BK < r_end) step(r0 + BK, (const lds_char *)a1, (const lds_char *)b1, (lds_char *)a0, (lds_char *)b0);
  }
  close();
  if (sums && o0 + (int)threadIdx.x < a.O) a.part_sum[(size_t)split * a.O + o0 + threadIdx.x] = column;
  float *P = a.part + (size_t)split * a.I * a.O;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int ii = i0 + wi + 32 * i + 8 * (t >> 2) + 4 * h + (t & 3), oo = o0 + wo + 32 * j + (lane & 31);
        if (ii < a.I && oo < a.O) P[(size_t)ii * a.O + oo] = sum[i][j][t];
      }
}
// D[i][o] += sum over the splits, in their order; row I is the column sums
__global__ __launch_bounds__(256) void tn32_reduce_kernel(const float *part, const float *part_sum, int splits, int I, int O, float *D, int64_t ldd,
                                                          float *sums) {
  const int o = blockIdx.x * 256 + threadIdx.x, i = blockIdx.y;
  if (o >= O) return;
  const bool column = i == I;
  float *dst = column ? sums : D == nullptr ? nullptr : D + (size_t)i * ldd;
  if (dst == nullptr) return;
  const float *src = column ? part_sum + o : part + (size_t)i * O + o;
  const size_t stride = column ? (size_t)O : (size_t)I * O;
  float x = 0.f;
  int s = 0;
  for (; s + 4 <= splits; s += 4) x += (src[s * stride] + src[(s + 1) * stride]) + (src[(s + 2) * stride] + src[(s + 3) * stride]);
  for (; s < splits; ++s) x += src[s * stride];
  dst[o] += x;
}

}  // namespace

int launch_nt32(const float *A, int64_t lda, const float *B, int64_t ldb, int M, int N, int K, float *C, int64_t ldc, bool add, hipStream_t s) {
  if (M <= 0 || N <= 0) return hipSuccess;
  const Nt32Args a{A, B, lda, ldb, ldc, M, N, K, C, add};
  // narrower tiles where 128 x 128 ones leave compute units without work: 41 x 8 tiles of a 5,196 x 1,000 product are one round
  // of 328 workgroups for 256 compute units
  const int64_t mt = (M + 127) / 128, wide = mt * ((N + 127) / 128), narrow = mt * ((N + 63) / 64);
  if (wide >= 512)
    hipLaunchKernelGGL(nt32_kernel<128>, dim3((unsigned)((wide + 7) / 8 * 8)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(nt32_kernel<64>, dim3((unsigned)((narrow + 7) / 8 * 8)), dim3(256), 0, s, a);
  return (int)hipGetLastError();
}

int tn32_splits(int64_t M, int I, int O) {
  const int64_t tiles = (int64_t)((I + 127) / 128) * ((O + 127) / 128);
  // three workgroups per compute unit in all, of four LDS tiles at least
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(256, (768 + tiles - 1) / tiles), (M + 127) / 128));
}

int launch_tn32(const float *A, int64_t lda, const float *B, int64_t ldb, int M, int I, int O, float *D, int64_t ldd, float *sums, float *part,
                float *part_sum, int max_splits, hipStream_t s) {
  if (M <= 0 || I <= 0 || O <= 0) return hipSuccess;
  int splits = std::min(max_splits, tn32_splits(M, I, O));
  const int rows_per = ((M + splits - 1) / splits + BK - 1) / BK * BK;
  splits = (M + rows_per - 1) / rows_per;
  const Tn32Args a{A, B, lda, ldb, M, I, O, splits, rows_per, part, sums ? part_sum : nullptr};
  const int64_t blocks = (int64_t)((I + 127) / 128) * ((O + 127) / 128) * splits;
  hipLaunchKernelGGL(tn32_kernel, dim3((unsigned)((blocks + 7) / 8 * 8)), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  // (rows of D are planes of the grid, 65,535 at most: d is within them)
  hipLaunchKernelGGL(tn32_reduce_kernel, dim3((unsigned)((O + 255) / 256), (unsigned)I + 1), dim3(256), 0, s, part, part_sum, splits, I, O, D, ldd, sums);
  return (int)hipGetLastError();
}
