// The products in fp32 arithmetic, as in the library's other fp32 paths: out [M, N] = A [M, depth] B [N, depth]^T, each operand with its
// depth contiguous (K-major) or the other side (MN-major).
//
// Bound by the fp32 pipes: a thread holds 8 x 8 sums (4 x 4 in the small tile) and makes two multiply-adds an instruction; the next
// slice of the depth is on its way to registers while one is multiplied.  Where there are fewer tiles than SMs the depth is cut, and the
// parts' sums are added in order by a second kernel, with the epilogue.
#pragma once
#include "linear_act.cuh"
#include "sm100_pair.cuh"

namespace psrl {
namespace {

// Every kernel here may start before the one before it on the stream has ended, and touches memory behind previous_kernel_done() only: its
// barriers and tensor memory are laid out meanwhile (1 row x 1024 x 1024 5.7 -> 4.2 us, 4096 x 4096 10.7 -> 9.0).
// What it reads may be written while it is here, so no pointer is __restrict__ and no load is of the read-only kind: the compiler may move
// those in front of the wait.
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

struct F32Operand {
  const float* at;
  int64_t pitch;
};
struct F32Epilogue {
  const float *bias, *mul, *residual;
  float *y, *z;
  int64_t mul_pitch, residual_pitch, y_pitch, z_pitch;
  int32_t act;
};
struct F32Params {
  F32Operand a, b;
  int32_t M, N, depth, slice;   // depth of a part, a multiple of 32
  float* part;                  // [parts][M][part_pitch], or NULL: the epilogue here
  int64_t part_pitch;           // N in whole fours
  int32_t m_tiles;
  F32Epilogue e;
  int32_t clear;                // the call's first kernel: it clears the status
  int* status;                  // NULL: a call without a workspace, whose depth is not cut
};

// Depth of a slice in shared memory: the small tile's few products would not cover the way of shorter ones from memory.
constexpr int f32_depth(int tile) { return tile == 64 ? 32 : 16; }

// The epilogue of four numbers from a multiple of four columns, or of the `left` that there are.  z may lie over mul or residual, so
// both are read first.
__device__ __forceinline__ void f32_read(const float* at, int left, float (&o)[4]) {
  if (left >= 4) {
    const float4 v = *reinterpret_cast<const float4*>(at);
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i < left ? at[i] : 0.f;
  }
}
__device__ __forceinline__ void f32_write(float* at, int left, const float (&o)[4]) {
  if (left >= 4) {
    *reinterpret_cast<float4*>(at) = make_float4(o[0], o[1], o[2], o[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) at[i] = o[i];
  }
}
__device__ __forceinline__ void f32_finish(const F32Epilogue& e, int64_t m, int64_t n, int left, float (&v)[4]) {
  float mul[4], res[4], bias[4];
  if (e.mul) f32_read(e.mul + m * e.mul_pitch + n, left, mul);
  if (e.residual) f32_read(e.residual + m * e.residual_pitch + n, left, res);
  if (e.bias) {
    f32_read(e.bias + n, left, bias);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += bias[i];
  }
  if (e.z) f32_write(e.z + m * e.z_pitch + n, left, v);
  activate<true>(v, e.act);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (e.mul) v[i] *= mul[i];
    if (e.residual) v[i] += res[i];
  }
  f32_write(e.y + m * e.y_pitch + n, left, v);
}

// A thread's vectors of a slice of kTile rows: along the depth (K-major) or along the tile.
template <int kTile, bool kMn>
struct F32Slice {
  static constexpr int kF32Depth = f32_depth(kTile), kVecs = kTile * kF32Depth / 4 / 256;
  float4 v[kVecs];

  __device__ __forceinline__ static void place(int i, int& row, int& k) {
    const int id = int(threadIdx.x) + i * 256;
    if (kMn) {
      row = id % (kTile / 4) * 4;
      k = id / (kTile / 4);
    } else {
      row = id / (kF32Depth / 4);
      k = id % (kF32Depth / 4) * 4;
    }
  }
  __device__ __forceinline__ void load(const F32Operand& o, int row0, int rows, int k0, int k_end) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      int r, k;
      place(i, r, k);
      r += row0;
      k += k0;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r >= rows || k >= k_end) continue;
      const float* at = kMn ? o.at + int64_t(k) * o.pitch + r : o.at + int64_t(r) * o.pitch + k;
      const int left = kMn ? rows - r : k_end - k;
      if (left >= 4) {
        v[i] = *reinterpret_cast<const float4*>(at);
      } else {
        v[i].x = at[0];
        if (left > 1) v[i].y = at[1];
        if (left > 2) v[i].z = at[2];
      }
    }
  }
  __device__ __forceinline__ void store(float (&s)[kF32Depth][kTile + 4]) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      int r, k;
      place(i, r, k);
      if (kMn) {
        *reinterpret_cast<float4*>(&s[k][r]) = v[i];
      } else {
        s[k][r] = v[i].x;
        s[k + 1][r] = v[i].y;
        s[k + 2][r] = v[i].z;
        s[k + 3][r] = v[i].w;
      }
    }
  }
};

// kTile x kTile, 256 threads.  A thread's rows and columns lie in runs of four, kTile / 2 apart where it has eight.
template <int kTile, bool kAMn, bool kBMn>
__global__ void __launch_bounds__(256) linear_f32_kernel(const __grid_constant__ F32Params p) {
  using namespace sm100;
  constexpr int kRuns = kTile / 64, kF32Depth = f32_depth(kTile);
  previous_kernel_done();
  next_kernel_may_start();
  __shared__ __align__(16) float sa[2][kF32Depth][kTile + 4], sb[2][kF32Depth][kTile + 4];
  if (p.clear && p.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = int(PSRL_OK);
  const int mt = int(blockIdx.x) % p.m_tiles, nt = int(blockIdx.x) / p.m_tiles;
  const int m0 = mt * kTile, n0 = nt * kTile;
  const int k0 = int(blockIdx.y) * p.slice, k_end = min(p.depth, k0 + p.slice);
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  f32x2 acc[kRuns * 4][kRuns * 2];
#pragma unroll
  for (int i = 0; i < kRuns * 4; ++i)
#pragma unroll
    for (int j = 0; j < kRuns * 2; ++j) acc[i][j] = make_f32x2(0.f, 0.f);
  F32Slice<kTile, kAMn> a;
  F32Slice<kTile, kBMn> b;
  a.load(p.a, m0, p.M, k0, k_end);
  b.load(p.b, n0, p.N, k0, k_end);
  a.store(sa[0]);
  b.store(sb[0]);
  __syncthreads();
  int at = 0;
  for (int k = k0; k < k_end; k += kF32Depth, at ^= 1) {
    const bool more = k + kF32Depth < k_end;
    if (more) {
      a.load(p.a, m0, p.M, k + kF32Depth, k_end);
      b.load(p.b, n0, p.N, k + kF32Depth, k_end);
    }
#pragma unroll
    for (int d = 0; d < kF32Depth; ++d) {
      float4 x[kRuns], y[kRuns];
#pragma unroll
      for (int r = 0; r < kRuns; ++r) {
        x[r] = *reinterpret_cast<const float4*>(&sa[at][d][r * (kTile / 2) + ty * 4]);
        y[r] = *reinterpret_cast<const float4*>(&sb[at][d][r * (kTile / 2) + tx * 4]);
      }
#pragma unroll
      for (int r = 0; r < kRuns; ++r) {
        const float xv[4] = {x[r].x, x[r].y, x[r].z, x[r].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 xx = make_f32x2(xv[i], xv[i]);
#pragma unroll
          for (int c = 0; c < kRuns; ++c) {
            acc[r * 4 + i][c * 2] = fma2(xx, make_f32x2(y[c].x, y[c].y), acc[r * 4 + i][c * 2]);
            acc[r * 4 + i][c * 2 + 1] = fma2(xx, make_f32x2(y[c].z, y[c].w), acc[r * 4 + i][c * 2 + 1]);
          }
        }
      }
    }
    if (more) {
      a.store(sa[at ^ 1]);
      b.store(sb[at ^ 1]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kRuns; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + r * (kTile / 2) + ty * 4 + i;
      if (m >= p.M) continue;
#pragma unroll
      for (int c = 0; c < kRuns; ++c) {
        const int n = n0 + c * (kTile / 2) + tx * 4;
        float v[4];
        split_f32x2(acc[r * 4 + i][c * 2], v[0], v[1]);
        split_f32x2(acc[r * 4 + i][c * 2 + 1], v[2], v[3]);
        const int left = p.N - n;
        if (left <= 0) continue;
        if (p.part) f32_write(p.part + (int64_t(blockIdx.y) * p.M + m) * p.part_pitch + n, left, v);
        else f32_finish(p.e, m, n, left, v);
      }
    }
}

// The parts' sums added in order, and the epilogue: one thread for four numbers.
__global__ void __launch_bounds__(256) linear_f32_join_kernel(const float* part, int parts, int M, int N, const __grid_constant__ F32Epilogue e) {
  sm100::previous_kernel_done();
  sm100::next_kernel_may_start();
  const int fours = (N + 3) / 4;
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, all = int64_t(M) * fours;
  if (at >= all) return;
  float v[4] = {};
  for (int i = 0; i < parts; ++i) {
    const float4 x = reinterpret_cast<const float4*>(part)[i * all + at];
    v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
  }
  const int64_t m = at / fours, n = (at - m * fours) * 4;
  f32_finish(e, m, n, int(N - n < 4 ? N - n : 4), v);
}

// The tile and the parts of the depth that a product is cut into.
struct F32Shape {
  int tile, parts;
  int64_t slice;
};
inline F32Shape f32_shape(int64_t M, int64_t N, int64_t depth) {
  const int64_t sms = resident_ctas();
  F32Shape s{};
  auto tiles = [&](int64_t t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
  // 1000 x 2048 x 2048: large tiles 224 us, small ones 299; 253 x 1568 x 1202, the depth cut in seven, 41 and 81; 381 x 416 x 830 32 and 29
  s.tile = tiles(128) >= sms || (depth >= 1024 && double(M) * double(N) * double(depth) >= 4e8) ? 128 : 64;
  // two blocks for every SM, of at least 64 deep each
  const int64_t want = std::max<int64_t>(1, 2 * sms / tiles(s.tile)), most = std::max<int64_t>(1, depth / 64);
  const int64_t parts = std::min(want, most);
  s.slice = ((depth + parts - 1) / parts + 31) / 32 * 32;
  s.parts = int((depth + s.slice - 1) / s.slice);
  return s;
}
inline size_t f32_part_bytes(int64_t M, int64_t N, int64_t depth) {
  const F32Shape s = f32_shape(M, N, depth);
  return s.parts > 1 ? size_t(s.parts) * M * ((N + 3) / 4 * 4) * sizeof(float) : 0;
}

template <bool kAMn, bool kBMn>
cudaError_t f32_product(F32Params p, float* part, cudaStream_t stream) {
  const F32Shape s = f32_shape(p.M, p.N, p.depth);
  p.slice = int32_t(s.slice);
  p.part = s.parts > 1 ? part : nullptr;
  p.part_pitch = (int64_t(p.N) + 3) / 4 * 4;
  p.m_tiles = (p.M + s.tile - 1) / s.tile;
  const int64_t tiles = int64_t(p.m_tiles) * ((p.N + s.tile - 1) / s.tile);
  if (tiles > INT32_MAX) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(tiles), unsigned(s.parts));
  cudaError_t e = launch(s.tile == 128 ? linear_f32_kernel<128, kAMn, kBMn> : linear_f32_kernel<64, kAMn, kBMn>, grid, 256, 0, stream, p);
  if (e == cudaSuccess && s.parts > 1)
    e = launch(linear_f32_join_kernel, dim3(unsigned((int64_t(p.M) * (p.part_pitch / 4) + 255) / 256)), 256, 0, stream, part, s.parts, p.M, p.N, p.e);
  return e;
}

}  // namespace
}  // namespace psrl
