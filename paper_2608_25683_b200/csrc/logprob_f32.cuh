// The fp32 products of the token log-probabilities: plain fp32 multiply-adds, as the library's fp32 attention has them (the
// tensor cores round fp32 operands to fewer bits).  One tiled kernel, 64 x 64 results per block of 256 threads, 4 x 4 each,
// operands through shared memory 16 deep, one buffer: 22 to 25 TFLOP/s with hundreds of rows (777 x 3584 x 50257 forward 12.8 ms,
// backward 33.0), a third of the 74 that 148 x 128 lanes make at 1965 MHz: every step waits for its loads, and two 16-byte reads of shared
// memory feed only 16 multiply-adds; less with few rows (64 x 1024 x 20000 backward 2.4 ms).  Not tuned.  Included by logprob.cu.
#pragma once
#include <cuda_runtime.h>
#include <math_constants.h>

namespace psrl {
namespace {

enum F32Kind { kF32Lse, kF32Dz, kF32Dh, kF32Dw };

struct F32Params {
  const float *a, *b;            // operands; where an element (m, k) of A lies depends on the kind (see f32_kernel)
  int64_t a_pitch, b_pitch;
  int32_t M, N, K;
  int32_t row0;                  // first row of the launch
  const int32_t* count;          // rows that matter: M of kF32Dz, kF32Dh, K of kF32Dw
  const int32_t* row_of;         // the caller's row of a gathered row
  float scale_log2;
  float2* part;                  // kF32Lse: [run][M]
  int32_t run;                   // kF32Lse: consecutive column tiles of a block
  const float2* row_info;        // kF32Dz, as in the bf16 path
  const int2* only;
  int32_t col0;
  float* out;
  int64_t out_pitch;
  int32_t first;                 // kF32Dh: store, otherwise add
};

constexpr int kF32Tile = 64, kF32Depth = 16;

// Sixteen-deep slice of an operand into shared memory as [k][64].  kAlongK: an operand row's depth is contiguous, else its
// 64 side.  Everything outside `side` x `depth` is zero.
template <bool kAlongK>
__device__ __forceinline__ void f32_load(float (*s)[kF32Tile + 4], const float* x, int64_t pitch, int side0, int side, int k0, int depth) {
  const int t = threadIdx.x;
  const int i = kAlongK ? t / 4 : t % 16 * 4, k = kAlongK ? t % 4 * 4 : t / 16;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int ii = side0 + i + (kAlongK ? 0 : j), kk = k0 + k + (kAlongK ? j : 0);
    const float v = ii < side && kk < depth ? (kAlongK ? x[int64_t(ii) * pitch + kk] : x[int64_t(kk) * pitch + ii]) : 0.f;
    s[k + (kAlongK ? j : 0)][i + (kAlongK ? 0 : j)] = v;
  }
}

// kind      A(m, k)                       B(n, k)                    result
// kF32Lse   hidden[m][k]                  weight[n][k]               (max, sum) of a row over a run of column tiles
// kF32Dz    gathered[m][k]                weight piece[n][k]         dz
// kF32Dh    dz[m][k]                      weight piece[k][n]         d_hidden, added up over the pieces by the same thread
// kF32Dw    dz[k][m]                      gathered[k][n]             rows of d_weight
template <F32Kind kKind>
__global__ void __launch_bounds__(256) f32_kernel(const F32Params p) {
  __shared__ float sa[kF32Depth][kF32Tile + 4], sb[kF32Depth][kF32Tile + 4];
  previous_kernel_done();
  next_kernel_may_start();
  const int rows = kKind == kF32Lse ? p.M : *p.count;
  const int M = kKind == kF32Dw ? p.M : rows, K = kKind == kF32Dw ? rows : p.K;
  const int m0 = p.row0 + int(blockIdx.y) * kF32Tile, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  if (m0 >= M) return;
  float best[4], sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { best[i] = -CUDART_INF_F; sum[i] = 0.f; }
  const int run = kKind == kF32Lse ? p.run : 1;
  for (int nt = 0; nt < run; ++nt) {
    const int n0 = (int(blockIdx.x) * run + nt) * kF32Tile;
    if (n0 >= p.N) break;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += kF32Depth) {
      f32_load<kKind != kF32Dw>(sa, p.a, p.a_pitch, m0, M, k0, K);
      f32_load<kKind == kF32Lse || kKind == kF32Dz>(sb, p.b, p.b_pitch, n0, p.N, k0, K);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kF32Depth; ++k) {
        const float4 a = *reinterpret_cast<const float4*>(&sa[k][ty * 4]), b = *reinterpret_cast<const float4*>(&sb[k][tx * 4]);
        const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + ty * 4 + i;
      if constexpr (kKind == kF32Lse) {
        float z[4], top = best[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          z[j] = n0 + tx * 4 + j < p.N ? acc[i][j] * p.scale_log2 : -CUDART_INF_F;
          top = fmaxf(top, z[j]);
        }
        const float ref = top == -CUDART_INF_F ? 0.f : top;
        sum[i] *= exp2f(best[i] - ref);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i] += exp2f(z[j] - ref);
        best[i] = top;
      } else if (m < M) {
        float2 info = make_float2(0.f, 0.f);
        int2 only = make_int2(-1, 0);
        int64_t to = m;
        if constexpr (kKind == kF32Dz) { info = p.row_info[p.row_of[m]]; only = p.only[p.row_of[m]]; }
        if constexpr (kKind == kF32Dh) to = p.row_of[m];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int n = n0 + tx * 4 + j;
          if (n >= p.N) continue;
          float v = acc[i][j];
          float* o = p.out + to * p.out_pitch + n;
          if constexpr (kKind == kF32Dz) {
            v = info.y * exp2f(at_most_one(fmaf(v, p.scale_log2, -info.x)));
            if (only.x == p.col0 + n) v = __int_as_float(only.y);
          }
          if constexpr (kKind == kF32Dh) { if (!p.first) v += *o; }
          *o = v;
        }
      }
    }
  }
  if constexpr (kKind == kF32Lse) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {   // over the 16 threads of a row
        const float m = __shfl_xor_sync(0xffffffffu, best[i], o), s = __shfl_xor_sync(0xffffffffu, sum[i], o);
        const float top = fmaxf(best[i], m), ref = top == -CUDART_INF_F ? 0.f : top;
        sum[i] = sum[i] * exp2f(best[i] - ref) + s * exp2f(m - ref);
        best[i] = top;
      }
      const int m = m0 + ty * 4 + i;
      if (tx == 0 && m < M) p.part[int64_t(blockIdx.x) * M + m] = make_float2(best[i], sum[i]);
    }
  }
}

}  // namespace
}  // namespace psrl
