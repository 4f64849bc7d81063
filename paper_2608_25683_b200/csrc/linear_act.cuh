// Activations of the products' epilogue and their slopes, in fp32.
#pragma once
#include <cuda_runtime.h>

#include "../../include/psrl.h"

namespace psrl {
namespace {

constexpr float kGeluIn = 0.7978845608028654f, kGeluCubic = 0.044715f;   // sqrt(2 / pi); the tanh form's factor
constexpr float kRootHalf = 0.7071067811865476f, kNormal = 0.3989422804014327f;   // sqrt(1 / 2), 1 / sqrt(2 pi)

// 1 / (1 + e^-z).  The quick exponential and division are a few steps of 2^-23 off, below a rounding to bf16 by far.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
// The tanh form of the gelu: z (1 + tanh(u)) / 2 = z sigmoid(2 u), which loses nothing where the tanh nears -1.
__device__ __forceinline__ float gelu_u2(float z) { return 2.f * kGeluIn * fmaf(kGeluCubic * z * z, z, z); }

template <int kN>
__device__ __forceinline__ void activate(float (&v)[kN], int act) {
  if (act == PSRL_ACT_NONE) return;
  if (act == PSRL_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];   // NaN stays
  } else if (act == PSRL_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= sigmoid(v[i]);
  } else if (act == PSRL_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= 0.5f * (1.f + erff(v[i] * kRootHalf));
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= sigmoid(gelu_u2(v[i]));
  }
}

// Values of the activation at z, and its slopes in z's place.
template <int kN>
__device__ __forceinline__ void act_and_slope(float (&z)[kN], int act, float (&value)[kN]) {
  if (act == PSRL_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      value[i] = z[i];
      z[i] = 1.f;
    }
  } else if (act == PSRL_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      value[i] = z[i] < 0.f ? 0.f : z[i];
      z[i] = z[i] > 0.f ? 1.f : z[i] <= 0.f ? 0.f : z[i];   // NaN stays
    }
  } else if (act == PSRL_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float s = sigmoid(z[i]);
      value[i] = z[i] * s;
      z[i] = fmaf(value[i], 1.f - s, s);
    }
  } else if (act == PSRL_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float c = 0.5f * (1.f + erff(z[i] * kRootHalf));
      value[i] = z[i] * c;
      z[i] = fmaf(z[i] * kNormal, __expf(-0.5f * z[i] * z[i]), c);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float s = sigmoid(gelu_u2(z[i])), near = fminf(fmaxf(z[i], -64.f), 64.f);   // beyond, 1 - s is nothing, and z^2 may be infinite
      value[i] = z[i] * s;
      z[i] = fmaf(value[i] * (1.f - s), 2.f * kGeluIn * fmaf(3.f * kGeluCubic * near, near, 1.f), s);
    }
  }
}

}  // namespace
}  // namespace psrl
