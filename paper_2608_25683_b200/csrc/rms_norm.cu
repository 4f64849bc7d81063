// Root-mean-square norm of the residual stream, its gradients, and rows in 8 bits.
//
//   h = x + residual (rounded as it is stored),  y = h r w,  r = (mean(h^2) + eps)^-1/2
//   8 bits: codes = e4m3(y / s), s = max(amax |y| / 448, 2^-126) for each row
//   g = d_y w:  d_x = d_summed + r (g - h r^2 mean(g h)),  d_weight = sum over the rows of d_y h r
//
// Memory bound: each element is read once and written once.  A row stays in the registers of a group of threads between the
// loads, the sum over it and the stores, so nothing is read twice; up to 32 lanes the sum is made by shuffles, beyond that with one
// barrier.  Blocks are persistent, keep the weight in registers and, in the backward, their share of d_weight's sums, which a
// second kernel adds up in the blocks' order: no atomics, the same bits every time.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math_constants.h>

#include <algorithm>

#include "../../include/psrl.h"
#include "kernels.h"
#include "sm100_pair.cuh"

namespace psrl {
namespace {
using sm100::next_kernel_may_start;
using sm100::previous_kernel_done;

constexpr int kMaxDim = 32768;
constexpr float kCodeMax = 448.f;          // the largest e4m3 number
constexpr float kLeastScale = 0x1p-126f;   // a row of zeros, or nearly: its codes are zeros, or nearly

struct FwdParams {
  const void *x, *residual, *weight;
  void *summed, *y;
  uint8_t* codes;
  float* scales;
  int64_t x_pitch, residual_pitch, summed_pitch, y_pitch, codes_pitch;
  int64_t rows;       // times heads
  int32_t heads, vecs;
  float inv_dim, eps;
  int32_t norm;       // 0: only the 8-bit output of x itself
};

struct BwdParams {
  const void *h, *weight, *d_y, *d_summed;
  void* d_x;
  float* part;        // [blocks][dim], or NULL
  int* status;
  int64_t h_pitch, d_y_pitch, d_summed_pitch, d_x_pitch;
  int64_t rows;
  int32_t heads, vecs;
  float inv_dim, eps;
};

template <class T> constexpr int kElems = 16 / int(sizeof(T));

// a 16-byte vector of bf16 or fp32 numbers
template <class T>
__device__ __forceinline__ void widen(const uint4& v, float (&o)[kElems<T>]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      o[i] = __uint_as_float(w[i]);
    } else {
      o[2 * i] = __uint_as_float(w[i] << 16);
      o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <class T>
__device__ __forceinline__ uint4 narrow(const float (&o)[kElems<T>]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(o[i]);
    } else {
      const __nv_bfloat162 p = __floats2bfloat162_rn(o[2 * i], o[2 * i + 1]);   // the only rounding of an output
      w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// max that a NaN survives
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

struct Add {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct MaxNan {
  __device__ __forceinline__ float operator()(float a, float b) const { return max_nan(a, b); }
};

// The values of a group of kGroup threads joined, for all of them, in a fixed order.  Beyond a warp: `s` holds a value for each warp.
// Every row has one barrier at least, so a warp that writes for the row after next knows that all have read this row's: two
// rows in a row use two `s`.
template <int kGroup, class Op>
__device__ __forceinline__ float join(float v, Op op, float* s) {
#pragma unroll
  for (int o = (kGroup < 32 ? kGroup : 32) / 2; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  if constexpr (kGroup > 32) {
    constexpr int kWarps = kGroup / 32;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < kWarps ? s[threadIdx.x & 31] : 0.f;   // sums and sizes: zero changes nothing
#pragma unroll
    for (int o = kWarps > 16 ? 16 : kWarps > 8 ? 8 : kWarps > 4 ? 4 : 2; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    v = __shfl_sync(0xffffffffu, v, 0);
  }
  return v;
}
template <int kGroup>
__device__ __forceinline__ float2 join_sums(float2 v, float2* s) {
#pragma unroll
  for (int o = (kGroup < 32 ? kGroup : 32) / 2; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if constexpr (kGroup > 32) {
    constexpr int kWarps = kGroup / 32;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < kWarps ? s[threadIdx.x & 31] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = kWarps > 16 ? 16 : kWarps > 8 ? 8 : kWarps > 4 ? 4 : 2; o > 0; o >>= 1) {
      v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
      v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    v.x = __shfl_sync(0xffffffffu, v.x, 0);
    v.y = __shfl_sync(0xffffffffu, v.y, 0);
  }
  return v;
}

// Squares of numbers beyond 2^56 may pass fp32's range: the sum is then made again of h 2^-110, whose squares do not, and whose
// roundings are the same.  (eps is nothing beside such a row.  NaN and infinities come this way, too, and stay.)  So with the backward's sum of
// g h, which may pass the range where its mean along the unit row does not: h 2^-110 keeps it in as long as no g h is beyond 2^220.
constexpr float kSmall = 0x1p-110f;
__device__ __forceinline__ bool too_large(float sum) { return !(sum <= FLT_MAX); }

constexpr int threads_of(int group) { return group > 32 ? group : 256; }

// Row i of rows x heads, in vectors of the matrix at `pitch` elements a row.
template <class T>
__device__ __forceinline__ int64_t vec_at(int64_t row, int head, int64_t pitch, int vecs) {
  return row * (pitch / kElems<T>) + int64_t(head) * vecs;
}

// A row's vectors of one matrix, zeros where there are none.
template <class T, int kGroup, int kVecs>
__device__ __forceinline__ void load_row(uint4 (&v)[kVecs], const void* base, int64_t pitch, int64_t row, int head, int vecs, bool live) {
  const uint4* at = static_cast<const uint4*>(base) + vec_at<T>(row, head, pitch, vecs);
  const int lane = threadIdx.x % kGroup;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    v[k] = make_uint4(0, 0, 0, 0);
    if (live && lane + k * kGroup < vecs) v[k] = at[lane + k * kGroup];
  }
}

template <class T, int kGroup, int kVecs, bool kCodes>
__global__ void __launch_bounds__(threads_of(kGroup)) rms_fwd_kernel(const __grid_constant__ FwdParams p) {
  constexpr int kE = kElems<T>, kPerBlock = threads_of(kGroup) / kGroup;
  __shared__ float s_sum[2][3][32];   // two rows in a row use two
  const int lane = threadIdx.x % kGroup, group = threadIdx.x / kGroup;
  previous_kernel_done();
  next_kernel_may_start();
  uint4 w[kVecs];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int v = lane + k * kGroup;
    w[k] = make_uint4(0, 0, 0, 0);
    if (p.weight && v < p.vecs) w[k] = static_cast<const uint4*>(p.weight)[v];
  }
  int turn = 0;
  const int64_t stride = int64_t(gridDim.x) * kPerBlock;
  int64_t i = int64_t(blockIdx.x) * kPerBlock + group, row = 0;
  int head = 0;
  uint4 xv[kVecs], rv[kVecs];
  auto load = [&](int64_t at) {
    const bool live = at < p.rows;
    row = p.heads == 1 ? at : at / p.heads;
    head = p.heads == 1 ? 0 : int(at - row * p.heads);
    load_row<T, kGroup, kVecs>(xv, p.x, p.x_pitch, row, head, p.vecs, live);
    if (p.residual) load_row<T, kGroup, kVecs>(rv, p.residual, p.residual_pitch, row, head, p.vecs, live);
  };
  constexpr bool kAhead = kGroup < 1024;   // beyond that registers are short
  if (kAhead) load(i);
  // all threads of a warp take part in its shuffles: a group without a row of its own goes along with the others
  for (; i - group < p.rows; i += stride, turn ^= 1) {
    if (!kAhead) load(i);
    const bool live = i < p.rows;
    const int64_t this_row = row;
    const int this_head = head;
    uint4 hv[kVecs];
    if (p.residual) {
      uint4* to = static_cast<uint4*>(p.summed) + vec_at<T>(this_row, this_head, p.summed_pitch, p.vecs);
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        float a[kE], b[kE];
        widen<T>(xv[k], a);
        widen<T>(rv[k], b);
#pragma unroll
        for (int e = 0; e < kE; ++e) a[e] += b[e];
        hv[k] = narrow<T>(a);
        const int v = lane + k * kGroup;
        if (p.summed && live && v < p.vecs) to[v] = hv[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) hv[k] = xv[k];
    }
    if (kAhead) load(i + stride);   // the next row is on its way while this one is summed and stored
    float r = 1.f;
    if (p.norm) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        float h[kE];
        widen<T>(hv[k], h);
#pragma unroll
        for (int e = 0; e < kE; ++e) sum = fmaf(h[e], h[e], sum);
      }
      sum = join<kGroup>(sum, Add(), s_sum[turn][0]);
      r = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
      if (kGroup > 32 ? too_large(sum) : __any_sync(0xffffffffu, too_large(sum))) {   // uniform in a warp, or in the block
        float small = 0.f;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
          float h[kE];
          widen<T>(hv[k], h);
#pragma unroll
          for (int e = 0; e < kE; ++e) small = fmaf(h[e] * kSmall, h[e] * kSmall, small);
        }
        small = join<kGroup>(small, Add(), s_sum[turn][1]);
        if (too_large(sum)) r = rsqrtf(small * p.inv_dim) * kSmall;
      }
    }
    auto normed = [&](int k, float (&o)[kE]) {
      float g[kE];
      widen<T>(hv[k], o);
      widen<T>(w[k], g);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        o[e] *= r;
        if (p.weight) o[e] *= g[e];
      }
    };
    uint4* y = static_cast<uint4*>(p.y) + vec_at<T>(this_row, this_head, p.y_pitch, p.vecs);
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float o[kE];
      normed(k, o);
      const int v = lane + k * kGroup;
      if (v < p.vecs) {
        if (p.y && live) y[v] = narrow<T>(o);
        if constexpr (kCodes) {
#pragma unroll
          for (int e = 0; e < kE; ++e) amax = max_nan(amax, fabsf(o[e]));
        }
      }
    }
    if constexpr (kCodes) {
      amax = join<kGroup>(amax, MaxNan(), s_sum[turn][2]);
      const float scale = too_large(amax) ? CUDART_NAN_F : max_nan(amax / kCodeMax, kLeastScale);   // an infinity has no code
      const float inv = 1.f / scale;
      uint8_t* c = p.codes + this_row * p.codes_pitch + int64_t(this_head) * p.vecs * kE;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        float o[kE];
        normed(k, o);
        uint32_t b[kE / 4];
#pragma unroll
        for (int e = 0; e < kE; e += 4) {   // rounded to the nearest code, ties to even; what passes the largest by a rounding is held there
          const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(o[e] * inv, o[e + 1] * inv), __NV_SATFINITE, __NV_E4M3);
          const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(o[e + 2] * inv, o[e + 3] * inv), __NV_SATFINITE, __NV_E4M3);
          b[e / 4] = lo | hi << 16;
        }
        const int v = lane + k * kGroup;
        if (live && v < p.vecs) {
          if constexpr (kE == 8) reinterpret_cast<uint2*>(c)[v] = make_uint2(b[0], b[1]);
          else reinterpret_cast<uint32_t*>(c)[v] = b[0];
        }
      }
      if (live && lane == 0) p.scales[i] = scale;
    }
  }
}

// Groups of 320 and 384 threads with two vectors each are alone on an SM and take all the registers that they can use (145 a thread for 117; 8192
// bf16 rows of 6144: 79.4 -> 76.0 us).  Groups of 384 to 768 with one vector, in fp32, take no more than leave room for bwd_per_sm() blocks.
constexpr int least_blocks(int group, int vecs, bool f32) {
  if (vecs == 2 && (group == 320 || group == 384)) return 1;
  return f32 && vecs == 1 && group >= 384 && group <= 768 ? (1024 + group - 1) / group : 0;
}
template <class T, int kGroup, int kVecs>
__global__ void __launch_bounds__(threads_of(kGroup), least_blocks(kGroup, kVecs, sizeof(T) == 4)) rms_bwd_kernel(const __grid_constant__ BwdParams p) {
  constexpr int kE = kElems<T>, kThreads = threads_of(kGroup), kPerBlock = kThreads / kGroup;
  __shared__ float2 s_sum[2][2][32];
  __shared__ float s_part[kGroup > 32 ? 1 : kThreads * kVecs * kE];
  previous_kernel_done();
  next_kernel_may_start();
  if (p.status && blockIdx.x == 0 && threadIdx.x == 0) *p.status = int(PSRL_OK);
  const int lane = threadIdx.x % kGroup, group = threadIdx.x / kGroup;
  uint4 w[kVecs];
  float dw[kVecs][kE];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int v = lane + k * kGroup;
    w[k] = make_uint4(0, 0, 0, 0);
    if (p.weight && v < p.vecs) w[k] = static_cast<const uint4*>(p.weight)[v];
#pragma unroll
    for (int e = 0; e < kE; ++e) dw[k][e] = 0.f;
  }
  int turn = 0;
  constexpr bool kAhead = kVecs == 1 || (kVecs == 2 && kGroup < 1024);   // beyond that registers are short
  const int64_t stride = int64_t(gridDim.x) * kPerBlock;
  int64_t i = int64_t(blockIdx.x) * kPerBlock + group, row = 0;
  int head = 0;
  uint4 next_h[kVecs], next_g[kVecs], next_s[kVecs];
  auto load = [&](int64_t at) {
    const bool live = at < p.rows;
    row = p.heads == 1 ? at : at / p.heads;
    head = p.heads == 1 ? 0 : int(at - row * p.heads);
    load_row<T, kGroup, kVecs>(next_h, p.h, p.h_pitch, row, head, p.vecs, live);
    load_row<T, kGroup, kVecs>(next_g, p.d_y, p.d_y_pitch, row, head, p.vecs, live);
    load_row<T, kGroup, kVecs>(next_s, p.d_summed, p.d_summed_pitch, row, head, p.vecs, live && p.d_summed);
  };
  if (kAhead) load(i);
  for (; i - group < p.rows; i += stride, turn ^= 1) {
    if (!kAhead) load(i);
    const bool live = i < p.rows;
    uint4* dx = static_cast<uint4*>(p.d_x) + vec_at<T>(row, head, p.d_x_pitch, p.vecs);
    uint4 hv[kVecs], gv[kVecs], sv[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) { hv[k] = next_h[k]; gv[k] = next_g[k]; sv[k] = next_s[k]; }
    if (kAhead) load(i + stride);   // the next row is on its way while this one is summed and stored
    auto sums = [&](float small) {
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        float a[kE], g[kE], c[kE];
        widen<T>(hv[k], a);
        widen<T>(gv[k], g);
        widen<T>(w[k], c);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          a[e] *= small;
          if (p.weight) g[e] *= c[e];
          s.x = fmaf(a[e], a[e], s.x);
          s.y = fmaf(a[e], g[e], s.y);
        }
      }
      return s;
    };
    float2 s = join_sums<kGroup>(sums(1.f), s_sum[turn][0]);
    float r = rsqrtf(fmaf(s.x, p.inv_dim, p.eps)), along = s.y * p.inv_dim * r;   // mean of g times the unit row h r
    const bool far = too_large(s.x), again = far || too_large(fabsf(s.y));
    if (kGroup > 32 ? again : __any_sync(0xffffffffu, again)) {
      const float2 t = join_sums<kGroup>(sums(kSmall), s_sum[turn][1]);
      if (again) {
        const float near = far ? rsqrtf(t.x * p.inv_dim) : r * (1.f / kSmall);
        along = t.y * p.inv_dim * near;
        if (far) r = near * kSmall;
      }
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float a[kE], g[kE], c[kE], o[kE];
      widen<T>(hv[k], a);
      widen<T>(gv[k], g);
      widen<T>(w[k], c);
      widen<T>(sv[k], o);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float unit = a[e] * r;
        if (live) dw[k][e] = fmaf(g[e], unit, dw[k][e]);
        const float gw = p.weight ? g[e] * c[e] : g[e];
        o[e] = fmaf(r, fmaf(-unit, along, gw), o[e]);
      }
      const int v = lane + k * kGroup;
      if (p.d_x && live && v < p.vecs) dx[v] = narrow<T>(o);
    }
  }
  if (!p.part) return;
  float* part = p.part + int64_t(blockIdx.x) * p.vecs * kE;
  if constexpr (kGroup > 32) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int v = lane + k * kGroup;
      if (v < p.vecs)
#pragma unroll
        for (int e = 0; e < kE; e += 4) *reinterpret_cast<float4*>(part + v * kE + e) = make_float4(dw[k][e], dw[k][e + 1], dw[k][e + 2], dw[k][e + 3]);
    }
  } else {
    constexpr int kRow = kGroup * kVecs * kE;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
#pragma unroll
      for (int e = 0; e < kE; ++e) s_part[group * kRow + (lane + k * kGroup) * kE + e] = dw[k][e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.vecs * kE; c += kThreads) {
      float s = 0.f;
      for (int g = 0; g < kPerBlock; ++g) s += s_part[g * kRow + c];
      part[c] = s;
    }
  }
}

// d_weight: the blocks' sums, added in a fixed order.  A block takes 32 columns, 32 threads share the parts of each.
template <class T>
__global__ void __launch_bounds__(1024) rms_weight_kernel(const float* part, int parts, int dim, T* d_weight) {
  previous_kernel_done();
  next_kernel_may_start();
  __shared__ float s[32][33];
  const int c = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  float sum = 0.f;
  if (col < dim)
    for (int i = slice; i < parts; i += 32) sum += part[int64_t(i) * dim + col];
  s[slice][c] = sum;
  __syncthreads();
  sum = s[c][slice];   // thread (slice, c) now has part c of column `slice`
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (c == 0 && blockIdx.x * 32 + slice < dim) {
    if constexpr (sizeof(T) == 4) d_weight[blockIdx.x * 32 + slice] = sum;
    else d_weight[blockIdx.x * 32 + slice] = __float2bfloat16_rn(sum);
  }
}

// Threads of a row's group and the vectors of each.
struct Shape {
  int group, vecs;
};
// Few vectors to a thread hide the latency of a row with many threads where rows are few; with many rows more vectors in flight
// a thread and fewer barriers a byte are better.  The backward, with three loads and d_weight's sums to hold, takes two vectors a
// thread, so that there are registers for the next row (8192 bf16 rows of 5120: three vectors and no row ahead 111 us, two 69); in
// fp32, where a vector is half the values, one a thread and twice the threads (8192 rows of 2560: 100 -> 55 us, of 4096: 122 -> 88;
// in bf16 that takes 100 us for 89 at 8192 wide).  Longer rows have three vectors a thread or four, each as it comes (4096 bf16 rows of
// 12288: three 85 us, four 122).
Shape shape_of(int vecs, int64_t rows, bool backward, bool f32) {
  if (vecs <= 8) return {8, 1};
  if (vecs <= 16) return {16, 1};
  if (vecs <= 32) return {32, 1};
  if (rows <= 2 * resident_ctas()) {
    if (vecs <= 128) return {128, 1};
    if (vecs <= 256) return {256, 1};
    if (vecs <= 512) return {512, 1};
    if (vecs <= 1024) return {1024, 1};
    if (vecs <= 2048) return {1024, 2};
    return vecs <= 4096 ? Shape{1024, 4} : Shape{1024, 8};
  }
  if (vecs <= 64) return {32, 2};
  if (backward) {
    if (vecs <= 128) return {128, 1};
    if (vecs <= 256) return f32 ? Shape{256, 1} : Shape{128, 2};
    if (vecs <= 384) return f32 ? Shape{384, 1} : Shape{192, 2};
    if (vecs <= 512) return f32 ? Shape{512, 1} : Shape{256, 2};
    if (vecs <= 640) return f32 ? Shape{640, 1} : Shape{320, 2};
    if (vecs <= 768) return f32 ? Shape{768, 1} : Shape{384, 2};
    if (vecs <= 1024) return f32 ? Shape{1024, 1} : Shape{512, 2};
    if (vecs <= 1536) return {512, 3};
  } else {
    if (vecs <= 128) return {32, 4};
    if (vecs <= 256) return {128, 2};
    if (vecs <= 512) return {256, 2};
    if (vecs <= 768) return {256, 3};
    if (vecs <= 1024) return {256, 4};
  }
  if (vecs <= 2048) return {512, 4};
  return vecs <= 4096 ? Shape{1024, 4} : Shape{1024, 8};
}

// Blocks of an SM in the backward, which the workspace goes by as each leaves a row of sums: as many as the registers hold.  With
// room to spare the blocks gather on the SMs that the launch before left first (8192 fp32 rows of 3000, one block of 768 threads to
// an SM 118 us, two 67).
int bwd_per_sm(const Shape& s, bool f32) {
  if (f32 && s.vecs == 1) return (1024 + threads_of(s.group) - 1) / threads_of(s.group);
  return std::max(1, (s.vecs == 1 ? 768 : 512) / threads_of(s.group));
}

// Blocks of a launch: as many as the SMs hold, and no more than there are rows for.
int64_t blocks_of(const Shape& s, int64_t rows, int per_sm) {
  const int per_block = threads_of(s.group) / s.group;
  return std::min<int64_t>(int64_t(resident_ctas()) * per_sm, (rows + per_block - 1) / per_block);
}

// Every kernel here may start before the one before it on the stream has ended, and touches memory behind previous_kernel_done() only.  What it
// reads may be written while it is here: no pointer is __restrict__, as the compiler may move loads through those in front of the wait.
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), unsigned blocks, unsigned threads, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

template <class Kernel>
cudaError_t launch_fwd(Kernel kernel, const Shape& s, const FwdParams& p, cudaStream_t stream, int (&per_sm)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  int n = dev >= 0 && dev < 64 ? per_sm[dev] : 0;
  if (n == 0) {
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads_of(s.group), 0);
    if (e != cudaSuccess) return e;
    n = std::max(1, n);
    if (dev >= 0 && dev < 64) per_sm[dev] = n;
  }
  return launch_early(kernel, unsigned(blocks_of(s, p.rows, n)), unsigned(threads_of(s.group)), stream, p);
}

template <class T, int kGroup, int kVecs, class P>
cudaError_t launch_one(const P& p, cudaStream_t stream) {
  const Shape s{kGroup, kVecs};
  if constexpr (std::is_same_v<P, FwdParams>) {
    static int per_sm[2][64] = {};
    if (p.codes) return launch_fwd(rms_fwd_kernel<T, kGroup, kVecs, true>, s, p, stream, per_sm[0]);
    return launch_fwd(rms_fwd_kernel<T, kGroup, kVecs, false>, s, p, stream, per_sm[1]);
  } else {
    return launch_early(rms_bwd_kernel<T, kGroup, kVecs>, unsigned(blocks_of(s, p.rows, bwd_per_sm(s, sizeof(T) == 4))), unsigned(threads_of(kGroup)), stream, p);
  }
}

template <class T, class P>
cudaError_t launch(const P& p, cudaStream_t stream) {
  constexpr bool kBackward = std::is_same_v<P, BwdParams>;
  const Shape s = shape_of(p.vecs, p.rows, kBackward, sizeof(T) == 4);
  switch (s.group * 16 + s.vecs) {
    case 8 * 16 + 1: return launch_one<T, 8, 1>(p, stream);
    case 16 * 16 + 1: return launch_one<T, 16, 1>(p, stream);
    case 32 * 16 + 1: return launch_one<T, 32, 1>(p, stream);
    case 32 * 16 + 2: return launch_one<T, 32, 2>(p, stream);
    case 128 * 16 + 1: return launch_one<T, 128, 1>(p, stream);
    case 256 * 16 + 1: return launch_one<T, 256, 1>(p, stream);
    case 512 * 16 + 1: return launch_one<T, 512, 1>(p, stream);
    case 512 * 16 + 4: return launch_one<T, 512, 4>(p, stream);
    case 1024 * 16 + 1: return launch_one<T, 1024, 1>(p, stream);
    case 1024 * 16 + 2: return launch_one<T, 1024, 2>(p, stream);
    case 1024 * 16 + 4: return launch_one<T, 1024, 4>(p, stream);
  }
  if constexpr (!kBackward || sizeof(T) == 2) {
    if (s.group * 16 + s.vecs == 128 * 16 + 2) return launch_one<T, 128, 2>(p, stream);
    if (s.group * 16 + s.vecs == 256 * 16 + 2) return launch_one<T, 256, 2>(p, stream);
  }
  if constexpr (kBackward) {
    if (s.group == 512 && s.vecs == 3) return launch_one<T, 512, 3>(p, stream);
    if constexpr (sizeof(T) == 4) {
      if (s.group == 384) return launch_one<T, 384, 1>(p, stream);
      if (s.group == 640) return launch_one<T, 640, 1>(p, stream);
      if (s.group == 768) return launch_one<T, 768, 1>(p, stream);
    } else {
      if (s.group == 192) return launch_one<T, 192, 2>(p, stream);
      if (s.group == 320) return launch_one<T, 320, 2>(p, stream);
      if (s.group == 384) return launch_one<T, 384, 2>(p, stream);
      if (s.group == 512) return launch_one<T, 512, 2>(p, stream);
    }
  } else {
    switch (s.group * 16 + s.vecs) {
      case 32 * 16 + 4: return launch_one<T, 32, 4>(p, stream);
      case 256 * 16 + 3: return launch_one<T, 256, 3>(p, stream);
      case 256 * 16 + 4: return launch_one<T, 256, 4>(p, stream);
    }
  }
  // 8 vectors a thread: only fp32 rows of more than 16384 get here
  if constexpr (sizeof(T) == 4) return launch_one<T, 1024, 8>(p, stream);
  else return cudaErrorInvalidValue;
}

int vec_elems(psrl_dtype_t t) { return t == PSRL_BF16 ? 8 : 4; }
bool known(psrl_dtype_t t) { return t == PSRL_F32 || t == PSRL_BF16; }
bool pitch_ok(int64_t pitch, int64_t least, int64_t unit) { return pitch >= least && pitch % unit == 0 && pitch <= (int64_t(1) << 40); }
// a tensor that may be left out, with its pitch; in place of another one only with the same pitch
bool tensor_ok(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool same_rows(const void* out, int64_t out_pitch, const void* in, int64_t in_pitch, int64_t rows) {
  return !out || out != in || out_pitch == in_pitch || rows <= 1;
}
// A row's codes are fewer bytes than the row: over an input they have to lie at the beginning of the row that they are made of, which is read before
// they are stored; those of a second head would lie over the first one's elements.
bool codes_apart(const void* codes, int64_t codes_pitch, const void* in, int64_t in_pitch, psrl_dtype_t dtype, int64_t rows, int32_t heads) {
  return !codes || codes != in || (heads == 1 && (rows <= 1 || codes_pitch == in_pitch * (dtype == PSRL_BF16 ? 2 : 4)));
}
constexpr int64_t kMostRows = int64_t(1) << 32;

psrl_status_t check(psrl_dtype_t dtype, int64_t rows, int32_t heads, int32_t dim, float eps) {
  if (!known(dtype)) return PSRL_ERR_UNSUPPORTED;
  if (rows < 0 || heads < 1 || heads > 65535 || rows > kMostRows || !(eps > 0.f) || !(eps <= FLT_MAX)) return PSRL_ERR_INVALID_ARG;
  if (dim < 8 || dim % 8 || dim > kMaxDim) return PSRL_ERR_SHAPE;
  return PSRL_OK;
}

psrl_status_t done(cudaError_t e) {
  if (e == cudaSuccess) return PSRL_OK;
  set_last_cuda_error(e);
  return PSRL_ERR_CUDA;
}

}  // namespace
}  // namespace psrl

extern "C" {

psrl_status_t psrl_rms_norm_fwd(psrl_dtype_t dtype, int64_t n_rows, int32_t n_heads, int32_t dim, const void* x, int64_t x_pitch,
                                const void* residual, int64_t residual_pitch, const void* weight, float eps, void* summed,
                                int64_t summed_pitch, void* y, int64_t y_pitch, void* codes, int64_t codes_pitch, float* scales,
                                void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, n_heads, dim, eps);
  if (st != PSRL_OK) return st;
  const int64_t least = int64_t(n_heads) * dim, unit = vec_elems(dtype);
  if (!pitch_ok(x_pitch, least, unit) || (residual && !pitch_ok(residual_pitch, least, unit)) || (residual && summed && !pitch_ok(summed_pitch, least, unit)) ||
      (y && !pitch_ok(y_pitch, least, unit)) || (codes && !pitch_ok(codes_pitch, least, 16)))
    return PSRL_ERR_SHAPE;
  if (n_rows == 0) return PSRL_OK;
  if (!residual) summed = nullptr;   // x itself is the stream
  if (!x || !tensor_ok(x) || !tensor_ok(residual) || !tensor_ok(weight) || !tensor_ok(summed) || !tensor_ok(y) || !tensor_ok(codes) ||
      (!codes) != (!scales) || (scales && !ptr_aligned(scales, 4)) || (y && y == summed) || (codes && (codes == y || codes == summed)) ||
      !codes_apart(codes, codes_pitch, x, x_pitch, dtype, n_rows, n_heads) || !codes_apart(codes, codes_pitch, residual, residual_pitch, dtype, n_rows, n_heads) ||
      !same_rows(summed, summed_pitch, x, x_pitch, n_rows) || !same_rows(summed, summed_pitch, residual, residual_pitch, n_rows) ||
      !same_rows(y, y_pitch, x, x_pitch, n_rows) || !same_rows(y, y_pitch, residual, residual_pitch, n_rows))
    return PSRL_ERR_INVALID_ARG;
  if (!summed && !y && !codes) return PSRL_OK;
  FwdParams p{x, residual, weight, summed, y, static_cast<uint8_t*>(codes), scales, x_pitch, residual_pitch, summed_pitch, y_pitch, codes_pitch,
              n_rows * n_heads, n_heads, int32_t(dim / unit), 1.f / float(dim), eps, 1};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return done(dtype == PSRL_BF16 ? launch<__nv_bfloat16>(p, s) : launch<float>(p, s));
}

psrl_status_t psrl_quantize_rows(psrl_dtype_t dtype, int64_t n_rows, int32_t dim, const void* x, int64_t x_pitch, void* codes,
                                 int64_t codes_pitch, float* scales, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, 1, dim, 1.f);
  if (st != PSRL_OK) return st;
  const int64_t unit = vec_elems(dtype);
  if (!pitch_ok(x_pitch, dim, unit) || !pitch_ok(codes_pitch, dim, 16)) return PSRL_ERR_SHAPE;
  if (n_rows == 0) return PSRL_OK;
  if (!ptr_aligned(x, 16) || !ptr_aligned(codes, 16) || !ptr_aligned(scales, 4) || !codes_apart(codes, codes_pitch, x, x_pitch, dtype, n_rows, 1)) return PSRL_ERR_INVALID_ARG;
  FwdParams p{x, nullptr, nullptr, nullptr, nullptr, static_cast<uint8_t*>(codes), scales, x_pitch, 0, 0, 0, codes_pitch,
              n_rows, 1, int32_t(dim / unit), 1.f / float(dim), 0.f, 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return done(dtype == PSRL_BF16 ? launch<__nv_bfloat16>(p, s) : launch<float>(p, s));
}

size_t psrl_rms_norm_workspace_bytes(psrl_dtype_t dtype, int64_t n_rows, int32_t n_heads, int32_t dim) {
  using namespace psrl;
  if (check(dtype, n_rows, n_heads, dim, 1.f) != PSRL_OK) return 0;
  if (n_rows == 0) return kWsHeaderBytes;
  const int64_t rows = n_rows * n_heads;
  const bool f32 = dtype == PSRL_F32;
  const Shape s = shape_of(dim / vec_elems(dtype), rows, true, f32);
  return kWsHeaderBytes + size_t(blocks_of(s, rows, bwd_per_sm(s, f32))) * size_t(dim) * sizeof(float);
}

psrl_status_t psrl_rms_norm_bwd(psrl_dtype_t dtype, int64_t n_rows, int32_t n_heads, int32_t dim, const void* summed, int64_t summed_pitch,
                                const void* weight, float eps, const void* d_y, int64_t d_y_pitch, const void* d_summed,
                                int64_t d_summed_pitch, void* d_x, int64_t d_x_pitch, void* d_weight, void* workspace,
                                size_t workspace_bytes, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, n_heads, dim, eps);
  if (st != PSRL_OK) return st;
  const int64_t least = int64_t(n_heads) * dim, unit = vec_elems(dtype);
  if (!pitch_ok(summed_pitch, least, unit) || !pitch_ok(d_y_pitch, least, unit) || (d_summed && !pitch_ok(d_summed_pitch, least, unit)) ||
      (d_x && !pitch_ok(d_x_pitch, least, unit)))
    return PSRL_ERR_SHAPE;
  const size_t need = d_weight ? psrl_rms_norm_workspace_bytes(dtype, n_rows, n_heads, dim) : kWsHeaderBytes;
  if ((d_weight && (!weight || !tensor_ok(d_weight))) || (workspace ? !ptr_aligned(workspace, 256) : need > kWsHeaderBytes)) return PSRL_ERR_INVALID_ARG;
  if (workspace && workspace_bytes < need) return PSRL_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t es = dtype == PSRL_BF16 ? 2 : 4;
  if (n_rows == 0) {
    cudaError_t e = workspace ? cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s) : cudaSuccess;
    if (e == cudaSuccess && d_weight) e = cudaMemsetAsync(d_weight, 0, size_t(dim) * es, s);
    return done(e);
  }
  if (!summed || !d_y || !tensor_ok(summed) || !tensor_ok(weight) || !tensor_ok(d_y) || !tensor_ok(d_summed) || !tensor_ok(d_x) ||
      !same_rows(d_x, d_x_pitch, summed, summed_pitch, n_rows) || !same_rows(d_x, d_x_pitch, d_y, d_y_pitch, n_rows) ||
      !same_rows(d_x, d_x_pitch, d_summed, d_summed_pitch, n_rows))
    return PSRL_ERR_INVALID_ARG;
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kWsHeaderBytes);
  BwdParams p{summed, weight, d_y, d_summed, d_x, d_weight ? part : nullptr, static_cast<int*>(workspace), summed_pitch, d_y_pitch, d_summed_pitch,
              d_x_pitch, n_rows * n_heads, n_heads, int32_t(dim / unit), 1.f / float(dim), eps};
  cudaError_t e = dtype == PSRL_BF16 ? launch<__nv_bfloat16>(p, s) : launch<float>(p, s);
  if (e == cudaSuccess && d_weight) {
    const bool f32 = dtype == PSRL_F32;
    const Shape shape = shape_of(p.vecs, p.rows, true, f32);
    const int parts = int(blocks_of(shape, p.rows, bwd_per_sm(shape, f32)));
    const unsigned grid = unsigned((dim + 31) / 32);
    e = dtype == PSRL_BF16 ? launch_early(rms_weight_kernel<__nv_bfloat16>, grid, 1024, s, part, parts, dim, static_cast<__nv_bfloat16*>(d_weight))
                           : launch_early(rms_weight_kernel<float>, grid, 1024, s, part, parts, dim, static_cast<float*>(d_weight));
  }
  return done(e);
}

}  // extern "C"
