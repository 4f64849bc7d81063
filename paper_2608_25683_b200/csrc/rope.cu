// Rotary positions of the tree's query rows, fused with the way of K and V into the paged pools and back.
//
// Pair i of a row's head is turned by the angle pos * f_i.  The angle is only needed modulo a full turn, so f_i is
// kept as a 64-bit fixed-point fraction of a turn: pos * f_i wraps around exactly in integer arithmetic, and an angle
// at position 10^6 is as good as one at position 1 (a product in fp32 would be off by 0.06 radians there).
//
// Memory bound: every element is read once and written once.  A warp takes a row: the row's cos / sin serve all its
// Hq + Hkv heads, which stream by in 16-byte vectors.  A lane handles the two vectors that rotate into each other, so each
// element is loaded and stored by the same thread and the rotation may run in place.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "../../include/psrl.h"
#include "kernels.h"
#include "plan.h"

struct psrl_rope {
  psrl_rope_desc_t desc;
  std::vector<double> freq;      // radians per position
  std::vector<uint64_t> turns;   // the same as a fraction of a turn, in units of 2^-64
  double scale = 1.0;
};

namespace psrl {
namespace {

constexpr int kMaxPairs = 128;

struct Frequencies {
  uint64_t turns[kMaxPairs];
};

// One operand of the launch: heads [head0, head0 + heads) of the block's work.  Row r of the source is at
// (by_slot ? slot[r] : r) * src_row, head h at h * src_head, in elements; the destination likewise.
struct Part {
  const void* src;
  void* dst;
  int64_t src_row, src_head, dst_row, dst_head;
  int32_t src_by_slot, dst_by_slot, heads, rotate;
};

struct RopeParams {
  Part part[3];
  const int32_t* pos;
  const int32_t* slot;
  int64_t rows;
  int32_t heads;        // sum over the parts
  int32_t shares;       // warps of a row
  int32_t pairs;        // rotary_dim / 2
  int32_t units;        // two-vector units per head: d / (2 * kElems)
  int32_t interleaved;
  float scale, sign;
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }  // the only rounding below fp32

// cos and sin (times the factor, sin with the direction's sign) of pair x at position pos
__device__ __forceinline__ float2 turn_at(const RopeParams& p, const Frequencies& f, int32_t pos, int x) {
  const uint64_t turn = uint64_t(int64_t(pos)) * f.turns[x];
  // signed fraction of a turn in [-1/2, 1/2); sincospi takes half turns
  const float half_turns = float(int32_t(turn >> 32)) * 0x1p-31f;
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c * p.scale, s * p.scale * p.sign);
}

template <class T>
__device__ __forceinline__ void rotate(T& a, T& b, float2 t) {
  const float x1 = to_f(a), x2 = to_f(b);
  from_f(a, x1 * t.x - x2 * t.y);
  from_f(b, x2 * t.x + x1 * t.y);
}

// Two 16-byte vectors of one head, rotated in place.  bf16 is widened by shifts and packed two at a time.
template <bool kBf16, bool kInterleaved, int kTurns>
__device__ __forceinline__ void rotate_vectors(uint4& xv, uint4& yv, const float2 (&t)[kTurns]) {
  uint32_t x[4] = {xv.x, xv.y, xv.z, xv.w}, y[4] = {yv.x, yv.y, yv.z, yv.w};
  auto low = [](uint32_t w) { return __uint_as_float(w << 16); };
  auto high = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
  auto pack = [](float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);   // the only rounding below fp32
    return *reinterpret_cast<const uint32_t*>(&v);
  };
  auto turn = [](float& a, float& b, float2 c) {
    const float p = a * c.x - b * c.y, q = b * c.x + a * c.y;
    a = p;
    b = q;
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kBf16 && !kInterleaved) {        // x holds the first members of eight pairs, y the second
      float a0 = low(x[i]), a1 = high(x[i]), b0 = low(y[i]), b1 = high(y[i]);
      turn(a0, b0, t[2 * i]);
      turn(a1, b1, t[2 * i + 1]);
      x[i] = pack(a0, a1);
      y[i] = pack(b0, b1);
    } else if constexpr (kBf16) {                  // a word is a pair
      float a = low(x[i]), b = high(x[i]), c = low(y[i]), d = high(y[i]);
      turn(a, b, t[i]);
      turn(c, d, t[4 + i]);
      x[i] = pack(a, b);
      y[i] = pack(c, d);
    } else if constexpr (!kInterleaved) {
      float a = __uint_as_float(x[i]), b = __uint_as_float(y[i]);
      turn(a, b, t[i]);
      x[i] = __float_as_uint(a);
      y[i] = __float_as_uint(b);
    } else if (i % 2 == 0) {
      float a = __uint_as_float(x[i]), b = __uint_as_float(x[i + 1]), c = __uint_as_float(y[i]), d = __uint_as_float(y[i + 1]);
      turn(a, b, t[i / 2]);
      turn(c, d, t[2 + i / 2]);
      x[i] = __float_as_uint(a); x[i + 1] = __float_as_uint(b);
      y[i] = __float_as_uint(c); y[i + 1] = __float_as_uint(d);
    }
  }
  xv = make_uint4(x[0], x[1], x[2], x[3]);
  yv = make_uint4(y[0], y[1], y[2], y[3]);
}

// A warp takes a row, or a share of its heads where there are few rows.  It computes the row's cos / sin once, every lane
// keeps those of its two vectors in registers, and streams the heads, two vectors of a head per lane and step.  No
// barrier, no index arithmetic per head but an addition.
//
// Two heads in flight per lane, 64 registers: the gradients of 195,923 rows of 80 heads, 8.03 GB,
// take 1206 us, what a plain copy of as much takes; one head 1260, three 1275, four (80 registers) 1224.  Blocks of
// four warps: 8,758 rows of 48 heads 43.1 us, of eight warps 45.0.
constexpr int kWarps = 4, kBatch = 2;

template <bool kBf16, bool kInterleaved>
__global__ void __launch_bounds__(kWarps * 32, 32 / kWarps) rope_kernel(const __grid_constant__ RopeParams p,
                                                              const __grid_constant__ Frequencies f) {
  constexpr int kElems = kBf16 ? 8 : 4, kBytes = kBf16 ? 2 : 4;
  __shared__ float2 cs[kWarps][kMaxPairs];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t task = int64_t(blockIdx.x) * kWarps + warp;
  if (task >= p.rows * p.shares) return;
  const int64_t row = p.shares == 1 ? task : task / p.shares;
  const int share = int(task - row * p.shares);
  const int64_t slot = p.slot ? int64_t(p.slot[row]) : 0;
  const int32_t pos = p.pos[row];
  for (int x = lane; x < p.pairs; x += 32) cs[warp][x] = turn_at(p, f, pos, x);
  __syncwarp();
  const int u = lane % p.units, at = lane / p.units, step = 32 / p.units;
  if (at >= step) return;
  const bool rotated = u < p.pairs / kElems;
  // byte offsets of the lane's two vectors inside a head, and their pairs
  const int a = (kInterleaved || !rotated ? 2 * u : u) * 16;
  const int b = kInterleaved || !rotated ? a + 16 : a + p.pairs * kBytes;
  float2 t[kElems];
#pragma unroll
  for (int e = 0; e < kElems; ++e) t[e] = rotated ? cs[warp][u * kElems + e] : make_float2(1.f, 0.f);
  int first = p.heads * share / p.shares, last = p.heads * (share + 1) / p.shares;   // of all parts' heads in a row
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const Part& q = p.part[k];
    const int h0 = max(first, 0) + at, h_end = min(last, q.heads);
    const int64_t src_step = q.src_head * (step * kBytes), dst_step = q.dst_head * (step * kBytes);
    const char* src = static_cast<const char*>(q.src) + ((q.src_by_slot ? slot : row) * q.src_row + h0 * q.src_head) * kBytes;
    char* dst = static_cast<char*>(q.dst) + ((q.dst_by_slot ? slot : row) * q.dst_row + h0 * q.dst_head) * kBytes;
    const bool turn = q.rotate && rotated;
#pragma unroll 1
    for (int h = h0; h < h_end; h += kBatch * step) {
      uint4 x[kBatch], y[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (h + i * step < h_end) {
          x[i] = *reinterpret_cast<const uint4*>(src + i * src_step + a);
          y[i] = *reinterpret_cast<const uint4*>(src + i * src_step + b);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (h + i * step < h_end) {
          if (turn) rotate_vectors<kBf16, kInterleaved>(x[i], y[i], t);
          *reinterpret_cast<uint4*>(dst + i * dst_step + a) = x[i];
          *reinterpret_cast<uint4*>(dst + i * dst_step + b) = y[i];
        }
      }
      src += kBatch * src_step;
      dst += kBatch * dst_step;
    }
    first -= q.heads;
    last -= q.heads;
  }
}

// The same element by element, where rotary_dim does not divide into pairs of 16-byte vectors: one thread per pair of
// elements, a block per few rows.  Uncommon sizes; bound by instructions, not by HBM.
template <class T>
__global__ void __launch_bounds__(256) rope_scalar_kernel(const __grid_constant__ RopeParams p, const __grid_constant__ Frequencies f) {
  __shared__ float2 cs[kMaxPairs];
  const int64_t row = blockIdx.x;
  const int64_t slot = p.slot ? int64_t(p.slot[row]) : 0;
  for (int x = threadIdx.x; x < p.pairs; x += 256) cs[x] = turn_at(p, f, p.pos[row], x);
  __syncthreads();
  for (int w = threadIdx.x; w < p.heads * p.units; w += 256) {
    const int u = w % p.units;
    int h = w / p.units, k = 0;
    while (h >= p.part[k].heads) { h -= p.part[k].heads; ++k; }
    const Part& q = p.part[k];
    const T* src = static_cast<const T*>(q.src) + (q.src_by_slot ? slot : row) * q.src_row + h * q.src_head;
    T* dst = static_cast<T*>(q.dst) + (q.dst_by_slot ? slot : row) * q.dst_row + h * q.dst_head;
    const bool rotated = u < p.pairs;
    const int a = p.interleaved || !rotated ? 2 * u : u, b = p.interleaved || !rotated ? a + 1 : a + p.pairs;
    T x = src[a], y = src[b];
    if (rotated && q.rotate) rotate(x, y, cs[u]);
    dst[a] = x;
    dst[b] = y;
  }
}

psrl_status_t launch(const psrl_rope& rope, RopeParams& p, psrl_dtype_t dtype, bool inverse, cudaStream_t stream) {
  const int d = rope.desc.head_dim, rot = rope.desc.rotary_dim;
  const int full = dtype == PSRL_BF16 ? 8 : 4;
  p.heads = 0;
  for (Part& q : p.part) {
    if (!q.src) q.heads = 0;
    p.heads += q.heads;
  }
  if (p.rows == 0 || p.heads == 0) return PSRL_OK;
  // Whole vectors need both halves of the rotated part, and the rest of the head, to be pairs of 16-byte vectors.
  const bool wide = rot % (2 * full) == 0 && d % (2 * full) == 0;   // then at most 32 units a head
  const int elems = wide ? full : 1;
  p.pairs = rot / 2;
  p.units = d / (2 * elems);
  p.interleaved = rope.desc.layout == PSRL_ROPE_INTERLEAVED;
  p.scale = float(rope.scale);
  p.sign = inverse ? -1.f : 1.f;
  // A warp per row; with fewer rows than twelve warps on every SM, the heads of a row are shared out as far as there are
  // four for each warp.
  const int64_t warps = int64_t(resident_ctas()) * 12;
  p.shares = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(warps / p.rows, p.heads / 4)));
  const int64_t grid = wide ? (p.rows * p.shares + kWarps - 1) / kWarps : p.rows;
  if (grid > INT32_MAX) return PSRL_ERR_SHAPE;
  Frequencies f{};
  for (size_t i = 0; i < rope.turns.size(); ++i) f.turns[i] = rope.turns[i];
  if (wide) {
    auto kernel = dtype == PSRL_BF16 ? (p.interleaved ? rope_kernel<true, true> : rope_kernel<true, false>)
                                     : (p.interleaved ? rope_kernel<false, true> : rope_kernel<false, false>);
    kernel<<<unsigned(grid), kWarps * 32, 0, stream>>>(p, f);
  } else {
    if (dtype == PSRL_BF16) rope_scalar_kernel<__nv_bfloat16><<<unsigned(grid), 256, 0, stream>>>(p, f);
    else rope_scalar_kernel<float><<<unsigned(grid), 256, 0, stream>>>(p, f);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { set_last_cuda_error(e); return PSRL_ERR_CUDA; }
  return PSRL_OK;
}

bool finite_pos(double x) { return std::isfinite(x) && x > 0.0; }

// NULL is "skip"; else aligned, and the pitch at least a row and a whole number of 16-byte vectors
bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool pitch_ok(int64_t pitch, int64_t heads, int d, psrl_dtype_t t) {
  const int64_t es = t == PSRL_BF16 ? 2 : 4;
  return pitch >= heads * d && pitch <= (int64_t(1) << 40) && (pitch * es) % 16 == 0;
}

// In place, but with rows at other distances: a row would be written over one that has yet to be read.
bool two_pitches(const void* x, int64_t x_pitch, const void* y, int64_t y_pitch, int64_t rows) {
  return x && x == y && x_pitch != y_pitch && rows > 1;
}

// The pairs' frequencies; false if the description's scaling arguments make no sense.
bool frequencies(const psrl_rope_desc_t& d, std::vector<double>& freq, double& scale) {
  const double r = d.rotary_dim, two_pi = 6.283185307179586476925286766559;
  const int n = d.rotary_dim / 2;
  if (!std::isfinite(d.base) || d.base <= 1.0) return false;
  if (d.scaling != PSRL_ROPE_UNSCALED && !finite_pos(d.factor)) return false;
  if (!std::isfinite(d.attention_scale) || d.attention_scale < 0.0) return false;
  double base = d.base;
  if (d.scaling == PSRL_ROPE_NTK) {
    if (d.rotary_dim == 2) return false;
    base *= std::pow(d.factor, r / (r - 2.0));
    if (!std::isfinite(base) || base <= 0.0) return false;
  }
  freq.resize(n);
  for (int i = 0; i < n; ++i) freq[i] = std::pow(base, -2.0 * i / r);
  scale = 1.0;
  if (d.scaling == PSRL_ROPE_LINEAR)
    for (double& x : freq) x /= d.factor;
  if (d.scaling == PSRL_ROPE_YARN || d.scaling == PSRL_ROPE_BANDED) {
    const double low = d.low == 0.0 ? 1.0 : d.low;
    const double high = d.high == 0.0 ? (d.scaling == PSRL_ROPE_YARN ? 32.0 : 4.0) : d.high;
    if (d.factor < 1.0 || d.original_positions < 1 || !finite_pos(low) || !finite_pos(high) || low >= high) return false;
    const double orig = d.original_positions;
    auto edge = [&](double turns) { return r * std::log(orig / (turns * two_pi)) / (2.0 * std::log(base)); };
    const double first = std::fmax(std::floor(edge(high)), 0.0), last = std::fmin(std::ceil(edge(low)), r - 1.0);
    for (int i = 0; i < n; ++i) {
      double keep;
      if (d.scaling == PSRL_ROPE_YARN) keep = 1.0 - (i - first) / std::fmax(last - first, 0.001);
      else keep = (orig * freq[i] / two_pi - low) / (high - low);
      keep = std::fmin(std::fmax(keep, 0.0), 1.0);
      freq[i] = freq[i] * keep + freq[i] / d.factor * (1.0 - keep);
    }
    if (d.scaling == PSRL_ROPE_YARN) scale = 0.1 * std::log(d.factor) + 1.0;
  }
  if (d.attention_scale > 0.0) scale = d.attention_scale;
  for (double x : freq)
    if (!std::isfinite(x) || x < 0.0 || x > 1e6) return false;
  return true;
}

}  // namespace
}  // namespace psrl

extern "C" {

psrl_status_t psrl_rope_create(const psrl_rope_desc_t* desc, psrl_rope_t** out) {
  if (out) *out = nullptr;
  if (!desc || !out) return PSRL_ERR_INVALID_ARG;
  if (desc->head_dim < 8 || desc->head_dim > 2 * psrl::kMaxPairs || desc->head_dim % 8 || desc->rotary_dim < 2 ||
      desc->rotary_dim > desc->head_dim || desc->rotary_dim % 2)
    return PSRL_ERR_SHAPE;
  if (desc->layout < PSRL_ROPE_HALF || desc->layout > PSRL_ROPE_INTERLEAVED || desc->scaling < PSRL_ROPE_UNSCALED ||
      desc->scaling > PSRL_ROPE_BANDED)
    return PSRL_ERR_INVALID_ARG;
  psrl_rope* r = new (std::nothrow) psrl_rope;
  if (!r) return PSRL_ERR_HOST_OOM;
  try {
    r->desc = *desc;
    if (!psrl::frequencies(*desc, r->freq, r->scale)) {
      delete r;
      return PSRL_ERR_INVALID_ARG;
    }
    for (double f : r->freq) {
      const long double turn = static_cast<long double>(f) / 6.283185307179586476925286766559L;
      const long double frac = turn - std::floor(turn);
      r->turns.push_back(static_cast<uint64_t>(frac * 18446744073709551616.0L));
    }
  } catch (const std::bad_alloc&) {
    delete r;
    return PSRL_ERR_HOST_OOM;
  }
  *out = r;
  return PSRL_OK;
}

psrl_status_t psrl_rope_frequencies(const psrl_rope_t* rope, const double** freq, int32_t* n, double* scale) {
  if (!rope || !freq || !n || !scale) return PSRL_ERR_INVALID_ARG;
  *freq = rope->freq.data();
  *n = static_cast<int32_t>(rope->freq.size());
  *scale = rope->scale;
  return PSRL_OK;
}

void psrl_rope_destroy(psrl_rope_t* rope) { delete rope; }

psrl_status_t psrl_rope_qkv_fwd(const psrl_plan_t* plan, const psrl_rope_t* rope, const void* q, int64_t q_pitch,
                                const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out,
                                void* k_pool, void* v_pool, int64_t pool_capacity, void* stream) {
  using namespace psrl;
  if (!plan || !plan->p || !rope) return PSRL_ERR_INVALID_ARG;
  const Plan& P = *plan->p;
  if ((q && !q_out) || (k && !k_pool) || (v && !v_pool) || !ok16(q) || !ok16(k) || !ok16(v) || !ok16(q_out) ||
      !ok16(k_pool) || !ok16(v_pool))
    return PSRL_ERR_INVALID_ARG;
  if (rope->desc.head_dim != P.d || (q && !pitch_ok(q_pitch, P.Hq, P.d, P.dtype)) ||
      (k && !pitch_ok(k_pitch, P.Hkv, P.d, P.dtype)) || (v && !pitch_ok(v_pitch, P.Hkv, P.d, P.dtype)) ||
      ((k || v) && pool_capacity < P.pool_slots))
    return PSRL_ERR_SHAPE;
  if (two_pitches(q, q_pitch, q_out, int64_t(P.Hq) * P.d, P.T_q)) return PSRL_ERR_INVALID_ARG;
  if (!P.dev) return PSRL_ERR_WORKSPACE;
  RopeParams p{};
  const int64_t d = P.d;
  p.part[0] = {q, q_out, q_pitch, d, P.Hq * d, d, 0, 0, P.Hq, 1};
  p.part[1] = {k, k_pool, k_pitch, d, d, pool_capacity * d, 0, 1, P.Hkv, 1};
  p.part[2] = {v, v_pool, v_pitch, d, d, pool_capacity * d, 0, 1, P.Hkv, 0};
  p.pos = P.dev + P.hdr.off_qrow_pos;
  p.slot = P.dev + P.hdr.off_qrow_slot;
  p.rows = P.T_q;
  return launch(*rope, p, P.dtype, false, static_cast<cudaStream_t>(stream));
}

psrl_status_t psrl_rope_qkv_bwd(const psrl_plan_t* plan, const psrl_rope_t* rope, const void* d_q, const void* dk_pool,
                                const void* dv_pool, int64_t pool_capacity, void* dq_out, int64_t dq_pitch,
                                void* dk_out, int64_t dk_pitch, void* dv_out, int64_t dv_pitch, void* stream) {
  using namespace psrl;
  if (!plan || !plan->p || !rope) return PSRL_ERR_INVALID_ARG;
  const Plan& P = *plan->p;
  if ((d_q && !dq_out) || (dk_pool && !dk_out) || (dv_pool && !dv_out) || !ok16(d_q) || !ok16(dk_pool) ||
      !ok16(dv_pool) || !ok16(dq_out) || !ok16(dk_out) || !ok16(dv_out))
    return PSRL_ERR_INVALID_ARG;
  if (rope->desc.head_dim != P.d || (d_q && !pitch_ok(dq_pitch, P.Hq, P.d, P.dtype)) ||
      (dk_pool && !pitch_ok(dk_pitch, P.Hkv, P.d, P.dtype)) || (dv_pool && !pitch_ok(dv_pitch, P.Hkv, P.d, P.dtype)) ||
      ((dk_pool || dv_pool) && pool_capacity < P.pool_slots))
    return PSRL_ERR_SHAPE;
  if (two_pitches(d_q, int64_t(P.Hq) * P.d, dq_out, dq_pitch, P.T_q)) return PSRL_ERR_INVALID_ARG;
  if (!P.dev) return PSRL_ERR_WORKSPACE;
  RopeParams p{};
  const int64_t d = P.d;
  p.part[0] = {d_q, dq_out, P.Hq * d, d, dq_pitch, d, 0, 0, P.Hq, 1};
  p.part[1] = {dk_pool, dk_out, d, pool_capacity * d, dk_pitch, d, 1, 0, P.Hkv, 1};
  p.part[2] = {dv_pool, dv_out, d, pool_capacity * d, dv_pitch, d, 1, 0, P.Hkv, 0};
  p.pos = P.dev + P.hdr.off_qrow_pos;
  p.slot = P.dev + P.hdr.off_qrow_slot;
  p.rows = P.T_q;
  return launch(*rope, p, P.dtype, true, static_cast<cudaStream_t>(stream));
}

psrl_status_t psrl_rope_rows(const psrl_rope_t* rope, psrl_dtype_t dtype, const void* x, int64_t x_pitch,
                             const int32_t* positions, int64_t n_rows, int32_t n_heads, void* y, int64_t y_pitch,
                             int inverse, void* stream) {
  using namespace psrl;
  if (!rope || n_rows < 0 || n_heads < 1 || n_heads > 65535) return PSRL_ERR_INVALID_ARG;
  if (dtype != PSRL_F32 && dtype != PSRL_BF16) return PSRL_ERR_UNSUPPORTED;
  const int64_t d = rope->desc.head_dim;
  if (!pitch_ok(x_pitch, n_heads, int(d), dtype) || !pitch_ok(y_pitch, n_heads, int(d), dtype)) return PSRL_ERR_SHAPE;
  if (n_rows == 0) return PSRL_OK;
  if (!ptr_aligned(x, 16) || !ptr_aligned(y, 16) || !ptr_aligned(positions, 4) || two_pitches(x, x_pitch, y, y_pitch, n_rows))
    return PSRL_ERR_INVALID_ARG;
  RopeParams p{};
  p.part[0] = {x, y, x_pitch, d, y_pitch, d, 0, 0, n_heads, 1};
  p.pos = positions;
  p.rows = n_rows;
  return launch(*rope, p, dtype, inverse != 0, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
