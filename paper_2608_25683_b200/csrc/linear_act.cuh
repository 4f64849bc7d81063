// Activations of the products' epilogue and their slopes, in fp32.
#pragma once
#include <cuda_runtime.h>

#include "../../include/psrl.h"

namespace psrl {
namespace {

constexpr float kGeluIn = 0.7978845608028654f, kGeluCubic = 0.044715f;   // sqrt(2 / pi); the tanh form's factor
constexpr float kRootHalf = 0.7071067811865476f, kNormal = 0.3989422804014327f;   // sqrt(1 / 2), 1 / sqrt(2 pi)

constexpr float kLog2e = 1.4426950408889634f, kUp = 0x1p24f;

// kF32: results are kept in fp32, with CUDA's exponential, division and error function, a few steps of 2^-23 off.  For results in bf16 the
// approximate exponential and reciprocal of the hardware do: within 2^-19 near 0 and 2^-16 at |x| = 100, for a half step of 2^-8.
// 2^x.  The callers' x = 24 + log2(e) u: the 24 keeps e^u among the normal numbers as long as u e^u is a number of bf16 at all, so smaller
// ones may be taken for 0.
__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / (1 + e^-u), as e / (1 + e) with e = e^u where u may be far below 0: e^-u passes fp32's range there.  From u = 40 on it is 1.  A NaN stays in the
// product with z.
__device__ __forceinline__ float sigmoid_up(float x) {   // of u with x = 24 + log2(e) u
  const float e = exp2_of(fminf(x, 24.f + 40.f * kLog2e));
  return e * reciprocal(kUp + e);
}
template <bool kF32>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (kF32) {
    const float e = expf(-fabsf(z));
    return (z < 0.f ? e : 1.f) / (1.f + e);
  } else {
    return sigmoid_up(fmaf(z, kLog2e, 24.f));
  }
}
// `rest`: 1 minus that, in fp32 as exact as its size.
template <bool kF32>
__device__ __forceinline__ float sigmoid(float z, float& rest) {
  if constexpr (kF32) {
    const float e = expf(-fabsf(z)), r = 1.f / (1.f + e), s = e * r;
    rest = z < 0.f ? r : s;
    return z < 0.f ? s : r;
  } else {
    const float s = sigmoid<false>(z);
    rest = 1.f - s;
    return s;
  }
}
// The share of the normal distribution below z, (1 + erf(z / sqrt 2)) / 2, and its density.  For negative z that sum cancels (at z = -5 4 % were
// off), so for z = -x it is made as e^(-x^2 / 2) R(x): R falls smoothly from 1/2 to 1 / (x sqrt(2 pi)), here a polynomial in t = 1 / (1 + 0.3 x), fitted
// to its values (linear program, least largest relative error for x up to 14) and within 2^-18.8 of them, for results in bf16.  In fp32 the
// complementary error function; in the products' epilogue it took 1.3 to 1.6 times the kernel's time.
template <bool kF32>
__device__ __forceinline__ float normal_below(float z, float& density) {
  if constexpr (kF32) {
    density = kNormal * expf(-0.5f * z * z);
    return 0.5f * erfcf(-z * kRootHalf);
  } else {
    const float e = exp2_of(fmaf(-0.5f * kLog2e * z, z, 24.f)), t = reciprocal(fmaf(0.3f, fabsf(z), 1.f));
    density = kNormal / kUp * e;
    float r = fmaf(-0.084582456f / kUp, t, 0.240540715f / kUp);
    r = fmaf(r, t, -0.0486076733f / kUp);
    r = fmaf(r, t, 0.164743758f / kUp);
    r = fmaf(r, t, 0.106710682f / kUp);
    r = fmaf(r, t, 0.12127377f / kUp);
    r = fmaf(r, t, -7.97300737e-05f / kUp);
    const float tail = e * r;
    return z < 0.f ? tail : 1.f - tail;
  }
}
// The tanh form of the gelu: z (1 + tanh(u)) / 2 = z sigmoid(2 u), which loses nothing where the tanh nears -1; in bf16 the exponent at once, for
// log2(e) 2 sqrt(2 / pi) (z + 0.044715 z^3).
__device__ __forceinline__ float gelu_u2(float z) { return 2.f * kGeluIn * fmaf(kGeluCubic * z * z, z, z); }
template <bool kF32>
__device__ __forceinline__ float gelu_share(float z) {
  if constexpr (kF32) return sigmoid<true>(gelu_u2(z));
  else return sigmoid_up(fmaf(z, fmaf(2.f * kGeluIn * kLog2e * kGeluCubic, z * z, 2.f * kGeluIn * kLog2e), 24.f));
}
template <bool kF32>
__device__ __forceinline__ float gelu_share(float z, float& rest) {
  if constexpr (kF32) return sigmoid<true>(gelu_u2(z), rest);
  const float s = gelu_share<false>(z);
  rest = 1.f - s;
  return s;
}

template <bool kF32, int kN>
__device__ __forceinline__ void activate(float (&v)[kN], int act) {
  if (act == PSRL_ACT_NONE) return;
  if (act == PSRL_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];   // NaN stays
  } else if (act == PSRL_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= sigmoid<kF32>(v[i]);
  } else if (act == PSRL_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float density;
      v[i] *= normal_below<kF32>(v[i], density);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] *= gelu_share<kF32>(v[i]);
  }
}

// Values of the activation at z, and its slopes in z's place.
template <bool kF32, int kN>
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
      float rest;
      const float s = sigmoid<kF32>(z[i], rest);
      value[i] = z[i] * s;
      z[i] = fmaf(value[i], rest, s);
    }
  } else if (act == PSRL_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float density;
      const float c = normal_below<kF32>(z[i], density);
      value[i] = z[i] * c;
      z[i] = fmaf(z[i], density, c);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float rest;
      const float s = gelu_share<kF32>(z[i], rest), near = fminf(fmaxf(z[i], -64.f), 64.f);   // beyond, `rest` or s is nothing, and z^2 may be infinite
      value[i] = z[i] * s;
      z[i] = fmaf(value[i] * rest, 2.f * kGeluIn * fmaf(3.f * kGeluCubic * near, near, 1.f), s);
    }
  }
}

}  // namespace
}  // namespace psrl
