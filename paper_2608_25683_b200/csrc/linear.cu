// Matrix products of a layer with what follows them in the same kernel, and their gradients.
//
//   z = sx[m] sw[n] sum_k x[m, k] w[n, k] + bias[n],   y = act(z) * mul + residual         (forward)
//   dz = d_y * mul * act'(z),  d_mul = d_y * act(z),  d_bias = sum_m dz                     (one elementwise pass)
//   d_x = dz w,  d_weight = dz^T x                                                          (one launch for both)
//
// The products run on one matrix kernel: tile 256 x 256 (or 128 wide) of a CTA pair (cta_group::2: each CTA holds 128 rows of A and
// half of B's columns, so a 128-byte deep step brings 32 KB into each SM for 512 tensor cycles), 32 KB stages filled by TMA, two
// accumulators in tensor memory so that the epilogue of one tile runs under the products of the next, persistent CTAs.
// Operands lie K-major in the forward; in the gradients the weights, x and, for d_weight, dz lie with the other side contiguous
// (MN-major), which the descriptors of shared memory take as they are: nothing is transposed in memory.
// The epilogue's own operands (residual, mul) come through TMA into the buffers that its results leave from.
//
// dz is rounded to bf16 before the gradients' products, as the tensor cores take their operands in pairs of a type: d_x and d_weight are 2.3e-3 from 64
// bits in the 2-norm, of which 1.7e-3 are their own rounding.  A second bf16 part of it would double the products, which are the call's time.
#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "../../include/psrl.h"
#include "attn_bf16_common.cuh"
#include "kernels.h"
#include "linear_act.cuh"
#include "linear_f32.cuh"
#include "sm100_pair.cuh"
#include "tma.h"

namespace psrl {
namespace {
using namespace sm100;

constexpr int kRowBytes = 128;                 // of an operand in a stage: 64 bf16 or 128 e4m3 deep
constexpr int kOperandBytes = 128 * kRowBytes; // one CTA's share of A or B in a stage
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kOutBytes = 128 * 128;           // what an epilogue group loads or stores at a time: 128 rows of 128 bytes
// Three warps issue the copies, a step each in turn.  A look at a stage's barrier takes a thread up to 350 cycles while the tensor
// cores use the shared memory, and a copy some 50, of the 512 that a step takes: one thread for all, 4 copies a step of the gradients, left
// the tensor pipe busy for 67 % of 4096 x 4096 x 8192.  A 13th warp would cost each thread 40 registers, which the epilogue needs.
constexpr int kGroups = 2, kEpilogueWarps = 4 * kGroups, kTmaWarps = 3, kTmaWarp = kEpilogueWarps, kMmaWarp = kTmaWarp + kTmaWarps;
constexpr int kGemmThreads = (kMmaWarp + 1) * 32;

// kPlain: results leave through two buffers a group.  kFull: with mul, residual or z, three: one holds mul and then z, one the
// residual and then y, and one is loaded ahead (mul's, where there are both).
enum Epilogue { kPlain, kFull };
constexpr int stages(Epilogue e) { return e == kPlain ? 5 : 4; }
constexpr int buffers(Epilogue e) { return e == kPlain ? 2 : 3; }
constexpr size_t gemm_smem(Epilogue e) { return size_t(stages(e)) * kStageBytes + size_t(kGroups) * buffers(e) * kOutBytes + 1024; }

struct Maps {
  CUtensorMap a[2], b[2], out[2];   // of the products of the launch
  CUtensorMap mul, residual, z;
};
// out [M, N] = A [M, depth] B [N, depth]^T
struct Product {
  int32_t M, N, steps;          // steps: of 128 bytes of depth (64 rows of an MN-major operand)
  int32_t m_tiles, n_tiles, tile_n;
  int32_t a_mn, b_mn;           // MN-major
  int32_t group;                // row tiles that are walked together
};
struct Params {
  Product product[2];           // the second one: fewer steps a tile, or empty
  int32_t ratio;                // tiles of the second that cost one of the first
  const __nv_bfloat16* bias;
  const float *x_scale, *w_scale;
  __nv_bfloat16 *y, *z;         // of the first product, for the columns behind the last whole 16 bytes of a row
  int64_t y_pitch, z_pitch;
  int32_t act, has_mul, has_residual, has_z;
  int32_t share;                // no pair has more than one tile
  int32_t clear;                // the call's first kernel: it clears the status, the later ones leave what those before them recorded
  int* status;
};

template <bool kFp8>
__device__ __forceinline__ void mma_step(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kFp8) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(kDescHi), "r"(idesc), "r"(accumulate)
        : "memory");
  } else {
    mma_pair(d, a_lo, b_lo, idesc, accumulate);
  }
}
// e4m3 x e4m3 (format 0 of both operands) -> fp32, both K-major
__host__ __device__ constexpr uint32_t make_idesc_fp8(int M, int N) { return (1u << 4) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24); }

// Tile `unit` of a product: groups of row tiles, inside a group the row tile moves fastest, so that the CTAs at work share column
// tiles and a group's rows stay in the L2.
__device__ __forceinline__ void tile_of(const Product& p, int unit, int& mt, int& nt) {
  const int per = p.group * p.n_tiles;
  const int g = unit / per, r = unit - g * per;
  const int gm = min(p.group, p.m_tiles - g * p.group);
  nt = r / gm;
  mt = g * p.group + r - nt * gm;
}

// What a pair of CTAs does: pair c of C takes the tiles c, c + C, ... of the first product.  The first r pairs then have one more
// than the others, who make up for it with the first tiles of the second; the rest of those go round.  No counter, no order
// that could vary.
struct Schedule {
  int n_first, n_second, mine, ahead, light;
  bool lighter;
  __device__ __forceinline__ Schedule(const Params& p, int c, int C) {
    n_first = p.product[0].m_tiles * p.product[0].n_tiles;
    n_second = p.product[1].m_tiles * p.product[1].n_tiles;
    const int q = n_first / C, r = n_first - q * C;
    mine = q + (c < r ? 1 : 0);
    light = C - r;
    lighter = c >= r;
    ahead = r > 0 ? min(p.ratio, n_second / light) : 0;
  }
  __device__ __forceinline__ bool get(const Params& p, int c, int C, int i, int& which, int& mt, int& nt) const {
    if (i < mine) {
      which = 0;
      tile_of(p.product[0], c + i * C, mt, nt);
      return true;
    }
    const int j = i - mine;
    int at = ahead * light;
    if (lighter && j < ahead) at = j * light + c - (C - light);
    else at += (lighter ? j - ahead : j) * C + c;
    if (at >= n_second) return false;
    which = 1;
    tile_of(p.product[1], at, mt, nt);
    return true;
  }
};

template <int kStages>
struct __align__(8) Barriers {
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], in[kGroups][3];
};

// The buffers of an epilogue group.  Use n of them is buffer n % count; thread 0 of the group sees to it that a buffer's last store
// has been read out before it is loaded or written again.
constexpr uint32_t kBarGroup = 1, kGroupThreads = 128;   // named barrier 1 + group

__device__ __forceinline__ void put16(uint8_t* b, int row, int chunk, uint4 v) {
  *reinterpret_cast<uint4*>(b + row * 128 + ((chunk ^ (row & 7)) << 4)) = v;
}
__device__ __forceinline__ uint4 get16(const uint8_t* b, int row, int chunk) {
  return *reinterpret_cast<const uint4*>(b + row * 128 + ((chunk ^ (row & 7)) << 4));
}

// eight bf16 of a vector that ends at `n`, from column `col`; the same for all threads
__device__ __forceinline__ uint4 load_bias(const __nv_bfloat16* bias, int col, int n) {
  if (col + 8 <= n) return *reinterpret_cast<const uint4*>(bias + col);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = col + 2 * i < n ? __bfloat162float(bias[col + 2 * i]) : 0.f, hi = col + 2 * i + 1 < n ? __bfloat162float(bias[col + 2 * i + 1]) : 0.f;
    w[i] = pack_bf16(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// four fp32 of such a vector
__device__ __forceinline__ float4 load_scale(const float* scale, int col, int n) {
  if (col + 4 <= n && (reinterpret_cast<uintptr_t>(scale) & 15) == 0) return *reinterpret_cast<const float4*>(scale + col);
  float o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = col + i < n ? scale[col + i] : 0.f;
  return make_float4(o[0], o[1], o[2], o[3]);
}
// eight numbers and a vector of eight bf16
__device__ __forceinline__ void add8(float* v, const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] += __uint_as_float(w[i] << 16);
    v[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void mul8(float* v, const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] *= __uint_as_float(w[i] << 16);
    v[2 * i + 1] *= __uint_as_float(w[i] & 0xffff0000u);
  }
}
// the first `count` of eight bf16
__device__ __forceinline__ void store_few(__nv_bfloat16* at, const uint4& x, int count) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < count) at[i] = __ushort_as_bfloat16(static_cast<unsigned short>(w[i / 2] >> (i % 2 * 16)));
}
__device__ __forceinline__ uint4 narrow8(const float* v) {
  return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// Looks at the barrier of a tile's products before the wait for them gives up: a step takes 0.3 us, or 1.5 where all SMs wait for memory, a look with
// its sleep some 0.1; the tile before may have to be waited for as well.  steps <= 2^24.
__device__ __forceinline__ uint32_t looks(int steps) { return kSpinLimit + 64u * uint32_t(steps); }

// kRagged: a row of the result ends inside 16 bytes.  (In every call the columns behind its last whole ones would cost 1 to 2 % of a shallow product.)
template <bool kFp8, Epilogue kEpilogue, bool kRagged>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
linear_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kStages = stages(kEpilogue), kBuffers = buffers(kEpilogue);
  constexpr int kDepth = kFp8 ? 128 : 64;
  __shared__ Barriers<kStages> bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_go[kGroups][2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int cluster = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;

  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < kStages; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&bar.acc_full[i], 1); mbar_init(&bar.acc_empty[i], 8); }   // four warps in either CTA
    for (int g = 0; g < kGroups; ++g)
      for (int i = 0; i < 3; ++i) mbar_init(&bar.in[g][i], 1);
    fence_mbar_init();
    tma_prefetch_desc(&maps.a[0]);
    tma_prefetch_desc(&maps.b[0]);
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();   // the peer's barriers exist before anything arrives on them
  tc_fence_after();
  previous_kernel_done();
  next_kernel_may_start();
  if (p.clear && p.status && blockIdx.x == 0 && tid == 0) *p.status = int(PSRL_OK);

  const Schedule plan(p, cluster, n_clusters);
  const uint32_t tmem = s_tmem;
  volatile int* abortp = &s_abort;
  int which, mt, nt;

  if (warp >= kTmaWarp && warp < kTmaWarp + kTmaWarps) {
    // ======================= TMA producers (both CTAs) =======================
    if (lane == 0) {
      uint32_t turn = uint32_t(kTmaWarps - (warp - kTmaWarp)) % kTmaWarps;   // 0: this warp's step
      uint32_t it = 0;
      bool ok = true;
      for (int i = 0; ok && plan.get(p, cluster, n_clusters, i, which, mt, nt); ++i) {
        const Product& q = p.product[which];
        const CUtensorMap *ma = &maps.a[which], *mb = &maps.b[which];
        const int m0 = mt * 256 + int(rank) * 128, half = q.tile_n / 2, n0 = nt * q.tile_n + int(rank) * half;
        const uint32_t stage_tx = 2 * (kOperandBytes + uint32_t(half) * kRowBytes);   // of both CTAs
        for (int kb = 0; kb < q.steps; ++kb, ++it) {
          const bool mine = turn == 0;
          turn = turn + 1 == kTmaWarps ? 0 : turn + 1;
          if (!mine) continue;
          const uint32_t s = it % kStages, round = it / kStages;
          if (round > 0 && !mbar_wait(&bar.empty[s], (round + 1) & 1, abortp, p.status)) { ok = false; break; }
          // the second CTA's copies count on the first one's barrier as well
          if (rank == 0) mbar_expect_tx(&bar.full[s], stage_tx);
          const uint32_t full = in_leader(&bar.full[s]);
          uint8_t* sa = smem + s * kStageBytes;
          uint8_t* sb = sa + kOperandBytes;
          if (q.a_mn) {
            tma_load_pair(sa, ma, full, m0, kb * kDepth);
            tma_load_pair(sa + kOperandBytes / 2, ma, full, m0 + 64, kb * kDepth);
          } else {
            tma_load_pair(sa, ma, full, kb * kDepth, m0);
          }
          if (q.b_mn) {
            tma_load_pair(sb, mb, full, n0, kb * kDepth);
            if (half > 64) tma_load_pair(sb + kOperandBytes / 2, mb, full, n0 + 64, kb * kDepth);
          } else {
            tma_load_pair(sb, mb, full, kb * kDepth, n0);
          }
        }
      }
      // the last arrivals on the stages' barriers come from the pair's products: this CTA stays until they are here
      for (uint32_t i = 0; i < kStages && ok; ++i) {
        const uint32_t uses = it / kStages + (i < it % kStages ? 1 : 0);
        if (uses > 0) ok = mbar_wait(&bar.empty[i], (uses + 1) & 1, abortp, p.status);
      }
    }
  } else if (warp == kMmaWarp) {
    // ======================= MMA issuer (first CTA of the pair) =======================
    if (rank == 0) {
      // An MN-major operand's 64-wide blocks are kLbo bytes apart and a 16-deep step is 16 rows of 128 bytes; K-major, a step is 32
      // bytes (16 bf16 or 32 e4m3).
      constexpr uint32_t kLbo = kOperandBytes / 2, kStepK = 32 >> 4, kStepMn = 2048 >> 4;
      const bool elected = elect_one();
      uint32_t it = 0, tile = 0;
      bool ok = true;
      for (int i = 0; ok && plan.get(p, cluster, n_clusters, i, which, mt, nt); ++i, ++tile) {
        const Product& q = p.product[which];
        const uint32_t idesc = kFp8 ? make_idesc_fp8(256, q.tile_n) : make_idesc(256, q.tile_n, q.a_mn, q.b_mn);
        const uint32_t step_a = q.a_mn ? kStepMn : kStepK, lbo_a = q.a_mn ? kLbo : 0;
        const uint32_t step_b = q.b_mn ? kStepMn : kStepK, lbo_b = q.b_mn ? kLbo : 0;
        const uint32_t a = tile & 1, use = tile >> 1;
        if (use > 0) ok = __all_sync(0xffffffffu, mbar_wait(&bar.acc_empty[a], (use + 1) & 1, abortp, p.status));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + a * 256;
        for (int kb = 0; kb < q.steps; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (!mbar_wait_all1(&bar.full[s], (it / kStages) & 1, abortp, p.status)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_u32(smem) + s * kStageBytes, sb = sa + kOperandBytes;
          const uint32_t da = desc_lo(sa, lbo_a), db = desc_lo(sb, lbo_b);
          if (elected) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) mma_step<kFp8>(d, da + k * step_a, db + k * step_b, idesc, (kb > 0 || k > 0) ? 1u : 0u);
            commit_pair(&bar.empty[s]);
          }
          __syncwarp();
        }
        if (ok && elected) commit_pair(&bar.acc_full[a]);
        __syncwarp();
      }
    }
  } else {
    // ======================= epilogue: one thread per row, a group for every other tile =======================
    // Where no pair has a second tile, the groups share the one: every other 64 columns of it.
    const int group = warp >> 2, gt = tid & 127;
    const uint32_t bar_id = kBarGroup + group;
    const uint32_t lane_addr = tmem + (uint32_t(warp & 3) << 21) + (p.share ? 0 : group * 256);   // lane 32 * (warp % 4)
    const uint32_t acc_empty = in_leader(&bar.acc_empty[group]);
    uint8_t* buf = smem + kStages * kStageBytes + group * kBuffers * kOutBytes;
    const bool has_second = kEpilogue == kFull && (p.has_mul || p.has_z);
    const int per = has_second ? 2 : 1;          // buffers a chunk takes: mul -> z if there is one of them, then residual -> y
    uint32_t base = 0, go = 0;                   // uses of buffers before this tile; hand-overs between the group's warps
    uint32_t phases = 0;                         // parity that the next load into each buffer completes
    uint32_t tile = 0;
    bool ok = true;
    for (int i = 0; ok && plan.get(p, cluster, n_clusters, i, which, mt, nt); ++i, ++tile) {
      if (!p.share && (tile & 1) != uint32_t(group)) continue;
      const Product& q = p.product[which];
      const int row0 = mt * 256 + int(rank) * 128, n0 = nt * q.tile_n, n_end = min(n0 + q.tile_n, q.N);
      [[maybe_unused]] const int whole = q.N & ~7;
      const int chunk0 = p.share ? group : 0, stride = p.share ? 128 : 64;   // columns from one of this group's chunks to the next
      const int all = row0 < q.M ? (n_end - n0 + 63) / 64 : 0, chunks = p.share ? (all + 1 - group) / 2 : all;
      int issued = 0;
      // thread 0: loads into the buffers of uses up to `until` of this tile, which are free
      auto issue = [&](int until) {
        until = min(until, chunks * per);
        for (; issued < until; ++issued) {
          const bool of_mul = per == 2 && !(issued & 1);
          if (kEpilogue == kPlain || !(of_mul ? p.has_mul : p.has_residual)) continue;
          const int b = int((base + issued) % kBuffers);
          mbar_expect_tx(&bar.in[group][b], kOutBytes);
          tma_load_2d(buf + b * kOutBytes, of_mul ? &maps.mul : &maps.residual, &bar.in[group][b], n0 + chunk0 * 64 + issued / per * stride, row0);
        }
      };
      if (kEpilogue == kFull && gt == 0) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        issue(kBuffers);
      }
      // one warp waits for its group: the four leave together if the wait gives up, so none is missed at their barrier
      if ((warp & 3) == 0) {
        ok = mbar_wait(&bar.acc_full[p.share ? 0 : group], (tile >> 1) & 1, abortp, p.status, looks(p.product[0].steps));   // the deeper one
        if (lane == 0) s_go[group][go & 1] = ok;
      }
      named_sync(bar_id, kGroupThreads);
      ok = s_go[group][go++ & 1];
      if (!ok) break;
      tc_fence_after();
      const float sx = kFp8 && row0 + gt < q.M ? p.x_scale[row0 + gt] : 1.f;
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        const int at_col = chunk0 * 64 + c * stride, col = n0 + at_col;
        const uint32_t n = base + uint32_t(c * per);
        uint32_t r[2][32];
        tmem_ld32(lane_addr + at_col, r[0]);
        tmem_ld32(lane_addr + at_col + 32, r[1]);
        if ((warp & 3) == 0) {
          if (gt == 0) {
            // the buffers of this chunk: free, and with their loads under way
            if (kEpilogue == kPlain) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            else if (issued < (c + 1) * per) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            issue((c + 1) * per);
          }
          __syncwarp();
          if (kEpilogue == kFull) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              if (u >= per || !(per == 2 && u == 0 ? p.has_mul : p.has_residual)) continue;
              const int b = int((n + u) % kBuffers);
              ok = ok && mbar_wait(&bar.in[group][b], (phases >> b) & 1, abortp, p.status);
            }
            ok = __all_sync(0xffffffffu, ok);
            if (lane == 0) s_go[group][go & 1] = ok;
          }
        }
        tmem_wait_ld();
        named_sync(bar_id, kGroupThreads);
        if (kEpilogue == kFull) {
          ok = s_go[group][go++ & 1];
          if (!ok) break;
        }
        const int of_z = int(n % kBuffers), of_y = int((n + uint32_t(per) - 1) % kBuffers);
        uint8_t* first = buf + of_y * kOutBytes;
        uint8_t* second = buf + of_z * kOutBytes;   // with per == 2 only
        if (kEpilogue == kFull) {
          // complete already; this thread's own look at the barrier orders its reads behind the copies
          if (p.has_mul) {
            mbar_wait(&bar.in[group][of_z], (phases >> of_z) & 1, abortp, p.status);
            phases ^= 1u << of_z;
          }
          if (p.has_residual) {
            mbar_wait(&bar.in[group][of_y], (phases >> of_y) & 1, abortp, p.status);
            phases ^= 1u << of_y;
          }
        }
        // 32 columns at a time, all that they read first, and every choice once for all of them: with reads and branches for each 8 columns a
        // chunk of 64 took 1300 cycles, with bias 2300 and with mul, z and silu 5900; so 620, 1550 and 5000
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = col + h * 32;
          if (kEpilogue == kFull && h == 1 && gt == 0) {
            // the stores of the chunks before this one have been read out by now: the buffers they left are loaded ahead
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            issue(c * per + kBuffers);
          }
          uint4 bias[4], mul[4], res[4];
          float4 scale[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (p.bias) bias[j] = load_bias(p.bias, at + j * 8, q.N);
            if constexpr (kFp8) {
              scale[2 * j] = load_scale(p.w_scale, at + j * 8, q.N);
              scale[2 * j + 1] = load_scale(p.w_scale, at + j * 8 + 4, q.N);
            }
            if constexpr (kEpilogue == kFull) {
              if (p.has_mul) mul[j] = get16(second, gt, h * 4 + j);
              if (p.has_residual) res[j] = get16(first, gt, h * 4 + j);
            }
          }
          float v[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[h][e]);
          if constexpr (kFp8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              v[4 * j] *= sx * scale[j].x; v[4 * j + 1] *= sx * scale[j].y;
              v[4 * j + 2] *= sx * scale[j].z; v[4 * j + 3] *= sx * scale[j].w;
            }
          }
          if (p.bias) {
#pragma unroll
            for (int j = 0; j < 4; ++j) add8(&v[j * 8], bias[j]);
          }
          if (kEpilogue == kFull && p.has_z) {
#pragma unroll
            for (int j = 0; j < 4; ++j) put16(second, gt, h * 4 + j, narrow8(&v[j * 8]));
          }
          activate<false>(v, p.act);
          if (kEpilogue == kFull && p.has_mul) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mul8(&v[j * 8], mul[j]);
          }
          if (kEpilogue == kFull && p.has_residual) {
#pragma unroll
            for (int j = 0; j < 4; ++j) add8(&v[j * 8], res[j]);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) put16(first, gt, h * 4 + j, narrow8(&v[j * 8]));
        }
        fence_proxy_async();
        named_sync(bar_id, kGroupThreads);
        if (gt == 0) {
          if (!kRagged || col < whole) {
            tma_store_2d(&maps.out[which], first, col, row0);
            if (kEpilogue == kFull && p.has_z) tma_store_2d(&maps.z, second, col, row0);
          }
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      }
      if (!ok) break;
      // A copy to memory ends with whole 16 bytes whatever the tensor's extent: what lies behind a row's last whole ones, in the last chunk
      // of the last column tile, is stored by its thread.
      if (kRagged && whole < n_end && chunks > 0) {
        const int col = n0 + chunk0 * 64 + (chunks - 1) * stride;
        const uint32_t n = base + uint32_t((chunks - 1) * per);
        if (col <= whole && whole < col + 64) {
          if (row0 + gt < q.M) {
            store_few(p.y + (row0 + gt) * p.y_pitch + whole, get16(buf + int((n + uint32_t(per) - 1) % kBuffers) * kOutBytes, gt, (whole - col) / 8), q.N - whole);
            if (kEpilogue == kFull && p.has_z) store_few(p.z + (row0 + gt) * p.z_pitch + whole, get16(buf + int(n % kBuffers) * kOutBytes, gt, (whole - col) / 8), q.N - whole);
          }
          named_sync(bar_id, kGroupThreads);   // before the buffers are loaded again
        }
      }
      base += uint32_t(chunks * per);
      // the accumulator may be overwritten
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_leader(acc_empty);
    }
    if (gt == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  // ---- teardown ----
  __syncthreads();
  if (s_abort) {
    // a wait gave up: let copies and products in flight come to rest before the memory they use is given back
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  cluster_sync();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------------------- few rows

// Few rows (the next tokens of rollouts): bound by the weights' bytes, which have to come in on all SMs at once.  The operands change
// places: 128 columns of the result (rows of the weight) are the tile's rows, up to kFewRows rows of x its columns, so that the tensor
// cores' work is no more than the rows need; and the depth is shared by a cluster of CTAs, which add their sums through one
// another's shared memory in the order of their ranks: one launch, no sums in memory, no atomics.
constexpr int kFewRows = 128;                  // rows of x in a tile at most
constexpr int kFewThreads = 6 * 32, kFewTma = 4, kFewMma = 5;
constexpr int kFewMaxStages = 12, kFewMaxSplit = 8;

struct FewMaps {
  CUtensorMap a, b;
};
struct FewParams {
  int32_t rows, cols;          // of the result
  int32_t steps, col_tiles, tile_rows;   // tile_rows: rows of x in a tile, a multiple of 16
  int32_t a_mn;                // the weight lies with the result's columns contiguous (d_x)
  int32_t stages, splits, tmem_cols;
  const __nv_bfloat16 *bias, *mul, *residual;
  const float *x_scale, *w_scale;
  __nv_bfloat16 *y, *z;
  int64_t mul_pitch, residual_pitch, y_pitch, z_pitch;
  int32_t act;
  int32_t clear;               // as above
  int* status;
};

__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// four bf16 at a multiple of four columns, or the `left` ones that there are
__device__ __forceinline__ void load4(const __nv_bfloat16* at, int left, float (&o)[4]) {
  if (left >= 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(at);
    o[0] = __uint_as_float(v.x << 16); o[1] = __uint_as_float(v.x & 0xffff0000u);
    o[2] = __uint_as_float(v.y << 16); o[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = e < left ? __bfloat162float(at[e]) : 0.f;
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* at, int left, const float (&v)[4]) {
  if (left >= 4) {
    *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) at[e] = __float2bfloat16_rn(v[e]);
  }
}
__device__ __forceinline__ uint32_t in_rank(uint32_t addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
template <bool kFp8>
__device__ __forceinline__ void mma_few(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kFp8) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(kDescHi), "r"(idesc), "r"(accumulate)
        : "memory");
  } else {
    mma_ss_lo(d, a_lo, b_lo, idesc, accumulate);
  }
}

template <bool kFp8>
__global__ void __launch_bounds__(kFewThreads) linear_few_kernel(const __grid_constant__ FewMaps maps, const __grid_constant__ FewParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kDepth = kFp8 ? 128 : 64;
  __shared__ __align__(8) uint64_t full[kFewMaxStages], empty[kFewMaxStages], acc_full;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = p.splits > 1 ? cluster_rank() : 0;
  const int tile = int(blockIdx.x) / p.splits;
  const int row_tile = tile / p.col_tiles, col0 = (tile - row_tile * p.col_tiles) * 128, row0 = row_tile * p.tile_rows;
  const int kb0 = int(int64_t(p.steps) * rank / p.splits), kb1 = int(int64_t(p.steps) * (rank + 1) / p.splits);
  const uint32_t b_bytes = uint32_t(p.tile_rows) * kRowBytes, stage_bytes = kOperandBytes + b_bytes;

  volatile int* abortp = &s_abort;
  if (warp == kFewMma) {
    tmem_alloc(&s_tmem, uint32_t(p.tmem_cols));
    tmem_relinquish();
  } else if (warp == kFewTma && lane == 0) {
    tma_prefetch_desc(&maps.a);
    tma_prefetch_desc(&maps.b);
    s_abort = 0;
    for (int i = 0; i < p.stages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    mbar_init(&acc_full, 1);
    fence_mbar_init();
  }
  previous_kernel_done();
  if (p.clear && p.status && blockIdx.x == 0 && threadIdx.x == 0) *p.status = int(PSRL_OK);
  // the first loads need nothing of the other warps: they are on their way while tensor memory is handed out
  auto load = [&](int kb, int s) {
    uint8_t* sa = smem + s * stage_bytes;
    mbar_expect_tx(&full[s], stage_bytes);
    if (p.a_mn) {
      tma_load_2d(sa, &maps.a, &full[s], col0, kb * kDepth);
      tma_load_2d(sa + kOperandBytes / 2, &maps.a, &full[s], col0 + 64, kb * kDepth);
    } else {
      tma_load_2d(sa, &maps.a, &full[s], kb * kDepth, col0);
    }
    tma_load_2d(sa + kOperandBytes, &maps.b, &full[s], kb * kDepth, row0);
  };
  if (warp == kFewTma && lane == 0)
    for (int s = 0; s < p.stages && kb0 + s < kb1; ++s) load(kb0 + s, s);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  next_kernel_may_start();   // not before this one has its tensor memory
  const uint32_t tmem = s_tmem;

  if (warp == kFewTma) {
    if (lane == 0) {
      for (int kb = kb0 + p.stages, s = 0, round = 1; kb < kb1; ++kb) {
        if (!mbar_wait(&empty[s], (round + 1) & 1, abortp, p.status)) break;
        load(kb, s);
        if (++s == p.stages) { s = 0; ++round; }
      }
    }
  } else if (warp == kFewMma) {
    constexpr uint32_t kLbo = kOperandBytes / 2, kStepK = 32 >> 4, kStepMn = 2048 >> 4;
    const bool elected = elect_one();
    const uint32_t idesc = kFp8 ? make_idesc_fp8(128, p.tile_rows) : make_idesc(128, p.tile_rows, p.a_mn, 0);
    const uint32_t step_a = p.a_mn ? kStepMn : kStepK, lbo_a = p.a_mn ? kLbo : 0;
    bool ok = true;
    for (int kb = kb0, s = 0, round = 0; kb < kb1; ++kb) {
      if (!mbar_wait_all1(&full[s], round & 1, abortp, p.status)) { ok = false; break; }
      tc_fence_after();
      const uint32_t sa = smem_u32(smem) + s * stage_bytes;
      const uint32_t da = desc_lo(sa, lbo_a), db = desc_lo(sa + kOperandBytes, 0);
      if (elected) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) mma_few<kFp8>(tmem, da + k * step_a, db + k * kStepK, idesc, (kb > kb0 || k > 0) ? 1u : 0u);
        mma_commit(&empty[s]);
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; ++round; }
    }
    if (ok && elected) mma_commit(&acc_full);
    __syncwarp();
    // all products are done before the stages' memory takes the sums (and before this CTA leaves)
    if (ok) mbar_wait(&acc_full, 0, abortp, p.status);
  } else {
    mbar_wait(&acc_full, 0, abortp, p.status, looks(kb1 - kb0));
    tc_fence_after();
  }
  __syncthreads();
  const int rows = min(p.tile_rows, p.rows - row0);
  float* sums = reinterpret_cast<float*>(smem);   // [tile_rows][128]
  if (warp < 4) {
    const uint32_t lane_addr = tmem + (uint32_t(warp) << 21);
    for (int c0 = 0; c0 < rows; c0 += 16) {
      uint32_t r[16];
      tmem_ld16(lane_addr + c0, r);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[(c0 + i) * 128 + threadIdx.x] = __uint_as_float(r[i]);
    }
  }
  if (p.splits > 1) cluster_sync();
  else __syncthreads();
  // Row r belongs to rank r % splits: a warp takes several of the rank's rows at a time, a lane four columns of each.
  const int col = col0 + lane * 4, left = p.cols - col;
  if (left > 0 && !s_abort) {
    float bias[4] = {}, scale[4] = {1.f, 1.f, 1.f, 1.f};
    if (p.bias) load4(p.bias + col, left, bias);
    if constexpr (kFp8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) scale[e] = e < left ? p.w_scale[col + e] : 0.f;
    }
    // with many parts to add there are few rows for each rank, and the other way round
    auto rows_of_rank = [&](auto rows_at_once, auto most_parts) {
      constexpr int kRows = decltype(rows_at_once)::value, kParts = decltype(most_parts)::value, kWarps = kFewThreads / 32;
      for (int r0 = int(rank) + p.splits * warp; r0 < rows; r0 += p.splits * kWarps * kRows) {
        float v[kRows][4], mul[kRows][4], res[kRows][4];
        [[maybe_unused]] float sx[kRows];
        float4 part[kRows][kParts];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const int r = r0 + i * p.splits * kWarps;
          if (r >= rows) break;
          const int64_t row = row0 + r;
          if (p.mul) load4(p.mul + row * p.mul_pitch + col, left, mul[i]);
          if (p.residual) load4(p.residual + row * p.residual_pitch + col, left, res[i]);
          if constexpr (kFp8) sx[i] = p.x_scale[row];
          const uint32_t at = smem_u32(sums + r * 128 + lane * 4);
#pragma unroll
          for (int k = 0; k < kParts; ++k)
            if (k < p.splits) part[i][k] = p.splits > 1 ? load_cluster(in_rank(at, uint32_t(k))) : *reinterpret_cast<const float4*>(sums + r * 128 + lane * 4);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const int r = r0 + i * p.splits * kWarps;
          if (r >= rows) break;
          const int64_t row = row0 + r;
          v[i][0] = part[i][0].x; v[i][1] = part[i][0].y; v[i][2] = part[i][0].z; v[i][3] = part[i][0].w;
#pragma unroll
          for (int k = 1; k < kParts; ++k)
            if (k < p.splits) { v[i][0] += part[i][k].x; v[i][1] += part[i][k].y; v[i][2] += part[i][k].z; v[i][3] += part[i][k].w; }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (kFp8) v[i][e] *= sx[i] * scale[e];
            if (p.bias) v[i][e] += bias[e];
          }
          if (p.z) store4(p.z + row * p.z_pitch + col, left, v[i]);
          activate<false>(v[i], p.act);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (p.mul) v[i][e] *= mul[i][e];
            if (p.residual) v[i][e] += res[i][e];
          }
          store4(p.y + row * p.y_pitch + col, left, v[i]);
        }
      }
    };
    if (p.splits <= 2) rows_of_rank(std::integral_constant<int, 6>(), std::integral_constant<int, 2>());
    else rows_of_rank(std::integral_constant<int, 2>(), std::integral_constant<int, kFewMaxSplit>());
  }
  if (p.splits > 1) cluster_sync();   // the others are done with this CTA's sums
  tc_fence_before();
  __syncthreads();
  if (s_abort) {
    // a wait gave up: let copies and products in flight come to rest before the memory they use is given back
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  if (warp == kFewMma) {
    tc_fence_after();
    tmem_dealloc(tmem, uint32_t(p.tmem_cols));
  }
}

// ------------------------------------------------------------------------------------------------- elementwise backward

// dz = d_y * mul * act'(z), d_mul = d_y * act(z), and sums over the rows of dz: a block takes 32 vectors of columns and 64 rows (more
// where there are millions), and leaves its column sums for bias_kernel, which adds them in order.  Memory bound: every element once, so
// a thread has the vectors of four rows on their way at a time, as they lie in memory: 4096 x 14336 with mul 92 us (5.1 TB/s); widened
// and two at a time 220 us.  Blocks of 128 vectors, two rows side by side, 102 us, and 23 where 777 rows of 3584 take 8.
constexpr int kDzRows = 64, kDzVecs = 32, kDzLanes = 8, kDzThreads = kDzVecs * kDzLanes;
template <class T> constexpr int kVec = 16 / int(sizeof(T));

template <class T>
struct DzParams {
  const T *d_y, *mul, *z;
  T *dz, *d_mul;               // NULL: not wanted
  float* part;                 // [row blocks][N], or NULL
  int64_t d_y_pitch, mul_pitch, z_pitch, dz_pitch, d_mul_pitch;
  int32_t M, N, act, rows;     // rows of a block
  int* status;
};

// a vector, or the `left` numbers that there are
template <class T>
__device__ __forceinline__ uint4 load_vec(const T* at, int left) {
  if (left >= kVec<T>) return *reinterpret_cast<const uint4*>(at);
  uint32_t w[4] = {};
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) {
    if (i >= left) break;
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(at[i]);
    else w[i / 2] |= uint32_t(__bfloat16_as_ushort(at[i])) << (i % 2 * 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <class T>
__device__ __forceinline__ void widen_vec(const uint4& v, float (&o)[kVec<T>]) {
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
__device__ __forceinline__ void store_vec(T* at, int left, const float (&o)[kVec<T>]) {
  if (left >= kVec<T>) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(o[i]);
      else w[i] = pack_bf16(o[2 * i], o[2 * i + 1]);
    }
    *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
      if (i < left) at[i] = T(o[i]);
  }
}

template <class T>
__global__ void __launch_bounds__(kDzThreads, 2) dz_kernel(const __grid_constant__ DzParams<T> p) {
  constexpr int kE = kVec<T>, kBatch = 4;
  previous_kernel_done();
  next_kernel_may_start();
  __shared__ float s_sum[kDzThreads][kE + 1];
  if (p.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = int(PSRL_OK);
  const int tx = threadIdx.x % kDzVecs, ty = threadIdx.x / kDzVecs;
  const int64_t col = (int64_t(blockIdx.x) * kDzVecs + tx) * kE;
  const int left = int(p.N - col < kE ? p.N - col : kE);
  float sum[kE] = {};
  if (left > 0) {
    const int64_t end = min(int64_t(p.M), (int64_t(blockIdx.y) + 1) * p.rows);
    for (int64_t row0 = int64_t(blockIdx.y) * p.rows + ty; row0 < end; row0 += kDzLanes * kBatch) {
      uint4 g4[kBatch], m4[kBatch], z4[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int64_t row = min(row0 + b * kDzLanes, end - 1);   // behind the end the last row again, for nothing
        g4[b] = load_vec(p.d_y + row * p.d_y_pitch + col, left);
        if (p.mul) m4[b] = load_vec(p.mul + row * p.mul_pitch + col, left);
        if (p.z) z4[b] = load_vec(p.z + row * p.z_pitch + col, left);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int64_t row = row0 + b * kDzLanes;
        if (row >= end) break;
        float g[kE], m[kE];
        widen_vec<T>(g4[b], g);
        if (p.mul) widen_vec<T>(m4[b], m);
        if (p.z) {
          float z[kE], d[kE];
          widen_vec<T>(z4[b], z);
          act_and_slope<sizeof(T) == 4>(z, p.act, d);   // d: values, z: slopes
#pragma unroll
          for (int e = 0; e < kE; ++e) {
            d[e] *= g[e];
            if (p.mul) g[e] *= m[e];
            g[e] *= z[e];
          }
          if (p.d_mul) store_vec(p.d_mul + row * p.d_mul_pitch + col, left, d);
        } else if (p.mul) {
#pragma unroll
          for (int e = 0; e < kE; ++e) g[e] *= m[e];
        }
        if (p.dz) store_vec(p.dz + row * p.dz_pitch + col, left, g);
#pragma unroll
        for (int e = 0; e < kE; ++e) sum[e] += g[e];
      }
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < kE; ++e) s_sum[threadIdx.x][e] = sum[e];
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * kDzVecs * kE;
  for (int i = threadIdx.x; i < kDzVecs * kE; i += kDzThreads) {
    if (first + i >= p.N) break;
    float s = 0.f;
    for (int y = 0; y < kDzLanes; ++y) s += s_sum[y * kDzVecs + i / kE][i % kE];
    p.part[int64_t(blockIdx.y) * p.N + first + i] = s;
  }
}

// d_bias from the blocks' sums: a block takes 32 columns, 32 threads share the parts of each, in a fixed order.
template <class T>
__global__ void __launch_bounds__(1024) bias_kernel(const float* part, int parts, int N, T* d_bias) {
  previous_kernel_done();
  next_kernel_may_start();
  __shared__ float s[32][33];
  const int c = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t col = int64_t(blockIdx.x) * 32 + c;
  float sum = 0.f;
  if (col < N)
    for (int i = slice; i < parts; i += 32) sum += part[int64_t(i) * N + col];
  s[slice][c] = sum;
  __syncthreads();
  sum = s[c][slice];   // thread (slice, c) now has part c of column `slice`
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (c == 0 && int64_t(blockIdx.x) * 32 + slice < N) d_bias[int64_t(blockIdx.x) * 32 + slice] = T(sum);
}

// ------------------------------------------------------------------------------------------------------------------- host

int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t dz_rows(int64_t M) { return std::max<int64_t>(kDzRows, div_up(M, 65535)); }   // at most 65,535 blocks of rows

template <bool kFp8, Epilogue kEpilogue, bool kRagged>
cudaError_t launch_gemm_as(const Maps& maps, const Params& p, int clusters, cudaStream_t stream) {
  static bool done[64] = {};
  const cudaError_t e = ensure_dynamic_smem(linear_kernel<kFp8, kEpilogue, kRagged>, gemm_smem(kEpilogue), done);
  if (e != cudaSuccess) return e;
  return launch(linear_kernel<kFp8, kEpilogue, kRagged>, dim3(2 * clusters), kGemmThreads, gemm_smem(kEpilogue), stream, maps, p);
}
template <bool kFp8, Epilogue kEpilogue>
cudaError_t launch_gemm(const Maps& maps, Params& p, cudaStream_t stream) {
  int64_t tiles = 0;
  for (const Product& q : p.product) tiles += int64_t(q.m_tiles) * q.n_tiles;
  if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int clusters = static_cast<int>(std::min<int64_t>(tiles, resident_ctas() / 2));
  p.share = tiles <= clusters;
  if (p.product[0].N % 8) return launch_gemm_as<kFp8, kEpilogue, true>(maps, p, clusters, stream);
  return launch_gemm_as<kFp8, kEpilogue, false>(maps, p, clusters, stream);
}

Product product_of(int64_t M, int64_t N, int64_t depth, int64_t step, int tile_n, int a_mn, int b_mn, int64_t group_bytes) {
  Product q{};
  q.M = int32_t(M); q.N = int32_t(N); q.steps = int32_t(div_up(depth, step));
  q.tile_n = tile_n;
  q.m_tiles = int32_t(div_up(M, 256)); q.n_tiles = int32_t(div_up(N, tile_n));
  q.a_mn = a_mn; q.b_mn = b_mn;
  // even groups of at most group_bytes (a row tile is 256 rows of 128 bytes for each step)
  const int64_t most = std::max<int64_t>(1, group_bytes / (int64_t(q.steps) * 256 * kRowBytes));
  const int64_t groups = div_up(q.m_tiles, most);
  q.group = int32_t(div_up(q.m_tiles, groups));
  return q;
}

// Rounds of tiles that the pairs of CTAs make, in 256-wide ones; a 128-wide tile takes 0.85 of the time of one while loads are waited for
// (4096 deep 22.5 and 26.1 us), and no less than three quarters, by its bytes.
double rounds_of(int64_t M, int64_t N, int tile_n) {
  const int64_t pairs = std::max(1, resident_ctas() / 2), tiles = div_up(M, 256) * div_up(N, tile_n);
  return double(div_up(tiles, pairs)) * (tile_n == 256 ? 1.0 : 0.85);
}
int tile_of(int64_t M, int64_t N) { return rounds_of(M, N, 128) < rounds_of(M, N, 256) ? 128 : 256; }

// How a product of few rows is shared out: the CTAs of a cluster that split its depth, and stages of memory.
struct FewShape {
  int tile_rows, stages, splits;
  int64_t col_tiles, row_tiles;
  size_t smem;
};
FewShape few_shape(int64_t rows, int64_t cols, int64_t steps) {
  FewShape f{};
  f.row_tiles = div_up(rows, kFewRows);
  f.tile_rows = int(round_up(div_up(rows, f.row_tiles), 16));
  f.col_tiles = div_up(cols, 128);
  const int64_t tiles = f.row_tiles * f.col_tiles, sms = resident_ctas();
  // two CTAs an SM, so that one's loads run under the other's beginning and end
  const size_t room = 111 * 1024;
  f.stages = int(std::min<size_t>(kFewMaxStages, room / (kOperandBytes + size_t(f.tile_rows) * kRowBytes)));
  f.splits = 1;
  while (f.splits < kFewMaxSplit && tiles * f.splits * 2 <= 2 * sms && steps / (f.splits * 2) >= 4) f.splits *= 2;
  // shallow and narrow products: rows in smaller tiles, for the epilogue's sake
  while (f.tile_rows > 16 && f.row_tiles * f.col_tiles * f.splits * 2 <= sms) {
    f.tile_rows = int(round_up(f.tile_rows / 2, 16));
    f.row_tiles = div_up(rows, f.tile_rows);
    f.stages = int(std::min<size_t>(kFewMaxStages, room / (kOperandBytes + size_t(f.tile_rows) * kRowBytes)));
  }
  const size_t stage = kOperandBytes + size_t(f.tile_rows) * kRowBytes;
  f.smem = std::max(size_t(f.stages) * stage, size_t(f.tile_rows) * 128 * sizeof(float)) + 1024;
  return f;
}
// Estimates of times in us that decide which kernel a product goes to, from 28 products of 192 to 1024 rows, 512 to 14336 deep and 512 to
// 8192 wide: they pick the quicker one but for the last 10 % in two.  The pairs of CTAs make one round of tiles after the other, a step of
// 128 bytes takes them 0.33 us (128 wide tiles 0.28).  The few-rows kernel shares the depth out; its weights come at 5.5 TB/s from memory,
// its 32 KB a step and CTA at 15 TB/s from the L2, in rounds of two CTAs for each SM.  (4096 deep and wide: 384 rows 23.1 us with this
// one, 26.8 with that; 768 rows 36.3 and 26.8.)
constexpr double kStepUs[2] = {0.28, 0.33};   // of a 128 wide tile, of a 256 wide one
double few_time(int64_t rows, int64_t cols, int64_t steps) {
  const FewShape f = few_shape(rows, cols, steps);
  const int64_t tiles = f.row_tiles * f.col_tiles, ctas = tiles * f.splits, places = 2 * int64_t(resident_ctas());
  double l2 = double(tiles) * double(steps) * double(kOperandBytes + f.tile_rows * kRowBytes) / 15e6;
  if (ctas > places) l2 *= double(div_up(ctas, places) * places) / double(ctas);
  return (rows <= kFewRows / 2 ? 5.0 : 8.5) + std::max(l2, double(cols) * double(steps) * kRowBytes / 5.5e6);
}
bool few_better(int64_t rows, int64_t cols, int64_t steps) {
  if (rows <= kFewRows) return true;
  const int tile_n = tile_of(rows, cols);
  const int64_t pairs = std::max(1, resident_ctas() / 2);
  return few_time(rows, cols, steps) < 6.0 + double(div_up(div_up(rows, 256) * div_up(cols, tile_n), pairs) * steps) * kStepUs[tile_n == 256];
}
// The gradients' products (rows 0: not that one) of `cols` columns: the tiles' width, and the time of both in one launch.
struct GradShape {
  int tile_n;
  double time;
};
GradShape grad_shape(int64_t rows_x, int64_t steps_x, int64_t rows_w, int64_t steps_w, int64_t cols) {
  const int64_t pairs = std::max(1, resident_ctas() / 2);
  GradShape best{256, 1e30};
  for (int tile_n : {256, 128}) {
    const int64_t n = div_up(cols, tile_n), x = div_up(rows_x, 256) * n, w = div_up(rows_w, 256) * n;
    const int64_t deepest = std::max(x ? steps_x : 0, w ? steps_w : 0);
    const double time = 6.0 + std::max(double(deepest), double(x * steps_x + w * steps_w) / double(pairs) + 0.5 * double(deepest)) * kStepUs[tile_n == 256];
    if (time < best.time) best = {tile_n, time};
  }
  return best;
}

template <bool kFp8>
cudaError_t launch_few(const FewMaps& maps, FewParams& p, const FewShape& f, cudaStream_t stream) {
  static bool done[64] = {};
  cudaError_t e = ensure_dynamic_smem(linear_few_kernel<kFp8>, 113 * 1024, done);
  if (e != cudaSuccess) return e;
  p.col_tiles = int32_t(f.col_tiles);
  p.tile_rows = f.tile_rows; p.stages = f.stages; p.splits = f.splits;
  p.tmem_cols = f.tile_rows <= 32 ? 32 : f.tile_rows <= 64 ? 64 : 128;
  const int64_t blocks = f.row_tiles * f.col_tiles * f.splits;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(blocks));
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = f.smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(f.splits);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, linear_few_kernel<kFp8>, maps, p);
}

constexpr int64_t kGroupBytes = int64_t(36) << 20, kGradGroupBytes = int64_t(16) << 20;

bool al16(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool opt16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool al4(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool pitch16(int64_t pitch, int64_t cols, int64_t unit) { return pitch >= cols && pitch % unit == 0 && pitch <= (int64_t(1) << 36); }
bool same_rows(const void* out, int64_t out_pitch, const void* in, int64_t in_pitch, int64_t rows) {
  return !out || out != in || out_pitch == in_pitch || rows <= 1;
}
constexpr int64_t kMost = int64_t(1) << 30;
// elements of 16 bytes
int64_t unit_of(psrl_dtype_t t) { return t == PSRL_F32 ? 4 : t == PSRL_BF16 ? 8 : 16; }

psrl_status_t cuda_failed(cudaError_t e) {
  set_last_cuda_error(e);
  return PSRL_ERR_CUDA;
}

psrl_status_t check(psrl_dtype_t t, int64_t M, int32_t K, int32_t N, psrl_activation_t act, const void* x, int64_t xp, const void* weight, int64_t wp) {
  if (t != PSRL_F32 && t != PSRL_BF16 && t != PSRL_E4M3) return PSRL_ERR_UNSUPPORTED;
  if (M < 0 || M > kMost || act < PSRL_ACT_NONE || act > PSRL_ACT_GELU_TANH) return PSRL_ERR_INVALID_ARG;
  if (K < 8 || K % 8 || K > kMost || N < 1 || N > kMost || !pitch16(xp, K, unit_of(t)) || !pitch16(wp, K, unit_of(t))) return PSRL_ERR_SHAPE;
  if (M > 0 && (!al16(x) || !al16(weight))) return PSRL_ERR_INVALID_ARG;
  return PSRL_OK;
}

// Where the backward's workspace holds what: dz unless it is d_y itself, and the column sums' parts.
struct Layout {
  size_t dz = 0, part = 0, f32 = 0, total = 0;
  int64_t dz_pitch = 0;
};
Layout layout(psrl_dtype_t t, int64_t M, int64_t K, int64_t N, bool with_dz, bool with_bias) {
  Layout L;
  size_t at = kWsHeaderBytes;
  auto take = [&](size_t bytes) {
    const size_t a = at;
    at += (bytes + 255) / 256 * 256;
    return a;
  };
  L.dz_pitch = round_up(N, 8);
  if (with_dz) L.dz = take(size_t(M) * L.dz_pitch * (t == PSRL_F32 ? 4 : 2));
  if (with_bias) L.part = take(size_t(div_up(M, dz_rows(M))) * N * sizeof(float));
  if (t == PSRL_F32) L.f32 = take(std::max(f32_part_bytes(M, K, N), f32_part_bytes(N, K, M)));
  L.total = at;
  return L;
}

template <class T>
cudaError_t run_dz(const DzParams<T>& p, T* d_bias, cudaStream_t s) {
  const dim3 grid(unsigned(div_up(p.N, kDzVecs * kVec<T>)), unsigned(div_up(p.M, p.rows)));
  cudaError_t e = launch(dz_kernel<T>, grid, kDzThreads, 0, s, p);
  if (e == cudaSuccess && d_bias)
    e = launch(bias_kernel<T>, dim3(unsigned(div_up(p.N, 32))), 1024, 0, s, p.part, int(grid.y), p.N, d_bias);
  return e;
}

}  // namespace
}  // namespace psrl

extern "C" {

size_t psrl_linear_workspace_bytes(psrl_dtype_t dtype, int64_t n_rows, int32_t in_dim, int32_t out_dim, int backward) {
  using namespace psrl;
  if (n_rows < 0 || n_rows > kMost || in_dim < 1 || out_dim < 1) return 0;
  if (n_rows == 0) return kWsHeaderBytes;
  if (backward) return layout(dtype, n_rows, in_dim, out_dim, true, true).total;
  return kWsHeaderBytes + (dtype == PSRL_F32 ? f32_part_bytes(n_rows, out_dim, in_dim) : 0);
}

psrl_status_t psrl_linear_fwd(psrl_dtype_t dtype, int64_t n_rows, int32_t in_dim, int32_t out_dim, const void* x, int64_t x_pitch,
                              const float* x_scale, const void* weight, int64_t weight_pitch, const float* weight_scale, const void* bias,
                              psrl_activation_t activation, const void* mul, int64_t mul_pitch, const void* residual,
                              int64_t residual_pitch, void* y, int64_t y_pitch, void* z, int64_t z_pitch, void* workspace,
                              size_t workspace_bytes, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, in_dim, out_dim, activation, x, x_pitch, weight, weight_pitch);
  if (st != PSRL_OK) return st;
  const int64_t M = n_rows, N = out_dim, unit = dtype == PSRL_F32 ? 4 : 8;
  const bool fp8 = dtype == PSRL_E4M3;
  if ((mul && !pitch16(mul_pitch, N, unit)) || (residual && !pitch16(residual_pitch, N, unit)) || !pitch16(y_pitch, N, unit) || (z && !pitch16(z_pitch, N, unit)))
    return PSRL_ERR_SHAPE;
  const size_t need = psrl_linear_workspace_bytes(dtype, n_rows, in_dim, out_dim, 0);
  if (workspace ? !ptr_aligned(workspace, 256) : need > kWsHeaderBytes) return PSRL_ERR_INVALID_ARG;
  if (workspace && workspace_bytes < need) return PSRL_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (M == 0) {
    if (!workspace) return PSRL_OK;
    const cudaError_t e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);   // otherwise the first kernel clears the status
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  if (!al16(y) || !opt16(bias) || !opt16(mul) || !opt16(residual) || !opt16(z) || (z && z == y) || fp8 != (x_scale != nullptr) || fp8 != (weight_scale != nullptr) ||
      (fp8 && (!al4(x_scale) || !al4(weight_scale))))
    return PSRL_ERR_INVALID_ARG;
  for (const void* out : {static_cast<const void*>(y), static_cast<const void*>(z)}) {
    const int64_t pitch = out == y ? y_pitch : z_pitch;
    if (!same_rows(out, pitch, mul, mul_pitch, M) || !same_rows(out, pitch, residual, residual_pitch, M)) return PSRL_ERR_INVALID_ARG;
  }
  int* status = static_cast<int*>(workspace);
  if (dtype == PSRL_F32) {
    F32Params q{};
    q.a = {static_cast<const float*>(x), x_pitch};
    q.b = {static_cast<const float*>(weight), weight_pitch};
    q.M = int32_t(M); q.N = int32_t(N); q.depth = in_dim; q.clear = 1; q.status = status;
    q.e = {static_cast<const float*>(bias), static_cast<const float*>(mul), static_cast<const float*>(residual), static_cast<float*>(y), static_cast<float*>(z),
           mul_pitch, residual_pitch, y_pitch, z_pitch, activation};
    const cudaError_t e = f32_product<false, false>(q, reinterpret_cast<float*>(static_cast<char*>(workspace) + kWsHeaderBytes), s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  const int64_t step = fp8 ? 128 : 64;
  using Bf = __nv_bfloat16;
  if (few_better(M, N, div_up(in_dim, step))) {
    const FewShape f = few_shape(M, N, div_up(in_dim, step));
    FewMaps maps;
    const bool made = fp8 ? make_map_u8_2d(&maps.a, weight, in_dim, N, weight_pitch, 128) && make_map_u8_2d(&maps.b, x, in_dim, M, x_pitch, f.tile_rows)
                          : make_map_bf16_2d(&maps.a, weight, in_dim, N, weight_pitch * 2, 128) && make_map_bf16_2d(&maps.b, x, in_dim, M, x_pitch * 2, f.tile_rows);
    if (!made) return PSRL_ERR_CUDA;
    FewParams q{};
    q.rows = int32_t(M); q.cols = int32_t(N); q.steps = int32_t(div_up(in_dim, step));
    q.bias = static_cast<const Bf*>(bias); q.mul = static_cast<const Bf*>(mul); q.residual = static_cast<const Bf*>(residual);
    q.x_scale = x_scale; q.w_scale = weight_scale;
    q.y = static_cast<Bf*>(y); q.z = static_cast<Bf*>(z);
    q.mul_pitch = mul_pitch; q.residual_pitch = residual_pitch; q.y_pitch = y_pitch; q.z_pitch = z_pitch;
    q.act = activation; q.clear = 1; q.status = status;
    const cudaError_t e = fp8 ? launch_few<true>(maps, q, f, s) : launch_few<false>(maps, q, f, s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  Maps maps{};
  Params p{};
  p.product[0] = product_of(M, N, in_dim, step, tile_of(M, N), 0, 0, kGroupBytes);
  const uint32_t half = uint32_t(p.product[0].tile_n / 2);
  const bool full = mul || residual || z;
  bool made = fp8 ? make_map_u8_2d(&maps.a[0], x, in_dim, M, x_pitch, 128) && make_map_u8_2d(&maps.b[0], weight, in_dim, N, weight_pitch, half)
                  : make_map_bf16_2d(&maps.a[0], x, in_dim, M, x_pitch * 2, 128) && make_map_bf16_2d(&maps.b[0], weight, in_dim, N, weight_pitch * 2, half);
  const int64_t whole = N >= 8 ? N / 8 * 8 : N;   // columns that leave by copies; fewer than eight leave without
  made = made && make_map_bf16_2d(&maps.out[0], y, whole, M, y_pitch * 2, 128);
  if (mul) made = made && make_map_bf16_2d(&maps.mul, mul, N, M, mul_pitch * 2, 128);
  if (residual) made = made && make_map_bf16_2d(&maps.residual, residual, N, M, residual_pitch * 2, 128);
  if (z) made = made && make_map_bf16_2d(&maps.z, z, whole, M, z_pitch * 2, 128);
  if (!made) return PSRL_ERR_CUDA;
  p.bias = static_cast<const __nv_bfloat16*>(bias);
  p.y = static_cast<__nv_bfloat16*>(y); p.y_pitch = y_pitch;
  p.z = static_cast<__nv_bfloat16*>(z); p.z_pitch = z_pitch;
  p.x_scale = x_scale; p.w_scale = weight_scale;
  p.act = activation;
  p.has_mul = mul != nullptr; p.has_residual = residual != nullptr; p.has_z = z != nullptr;
  p.clear = 1; p.status = status;
  const cudaError_t e = fp8 ? (full ? launch_gemm<true, kFull>(maps, p, s) : launch_gemm<true, kPlain>(maps, p, s))
                            : (full ? launch_gemm<false, kFull>(maps, p, s) : launch_gemm<false, kPlain>(maps, p, s));
  return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
}

psrl_status_t psrl_linear_bwd(psrl_dtype_t dtype, int64_t n_rows, int32_t in_dim, int32_t out_dim, const void* x, int64_t x_pitch,
                              const void* weight, int64_t weight_pitch, const void* z, int64_t z_pitch, psrl_activation_t activation,
                              const void* mul, int64_t mul_pitch, const void* d_y, int64_t d_y_pitch, void* d_x, int64_t d_x_pitch,
                              void* d_weight, int64_t d_weight_pitch, void* d_bias, void* d_mul, int64_t d_mul_pitch, void* workspace,
                              size_t workspace_bytes, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, in_dim, out_dim, activation, x, x_pitch, weight, weight_pitch);
  if (st != PSRL_OK) return st;
  if (dtype == PSRL_E4M3) return PSRL_ERR_UNSUPPORTED;
  const int64_t M = n_rows, N = out_dim, K = in_dim, unit = unit_of(dtype);
  const size_t es = dtype == PSRL_F32 ? 4 : 2;
  if (!pitch16(d_y_pitch, N, unit) || (z && !pitch16(z_pitch, N, unit)) || (mul && !pitch16(mul_pitch, N, unit)) || (d_mul && !pitch16(d_mul_pitch, N, unit)) ||
      (d_x && !pitch16(d_x_pitch, K, unit)) || (d_weight && !pitch16(d_weight_pitch, K, unit)))
    return PSRL_ERR_SHAPE;
  if (!opt16(d_x) || !opt16(d_weight) || !opt16(d_bias)) return PSRL_ERR_INVALID_ARG;
  const bool elementwise = activation != PSRL_ACT_NONE || mul;
  Layout L;
  L.total = kWsHeaderBytes;
  if (M > 0) L = layout(dtype, M, K, N, elementwise, d_bias != nullptr);
  if (workspace ? !ptr_aligned(workspace, 256) : L.total > kWsHeaderBytes) return PSRL_ERR_INVALID_ARG;
  if (workspace && workspace_bytes < L.total) return PSRL_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  char* ws = static_cast<char*>(workspace);
  if (M == 0) {
    if (workspace) e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);
    if (e == cudaSuccess && d_weight) e = cudaMemset2DAsync(d_weight, size_t(d_weight_pitch) * es, 0, size_t(K) * es, size_t(N), s);
    if (e == cudaSuccess && d_bias) e = cudaMemsetAsync(d_bias, 0, size_t(N) * es, s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  if (!al16(d_y) || !opt16(z) || !opt16(mul) || !opt16(d_mul) || (activation != PSRL_ACT_NONE && !z) || (d_mul && (!mul || !z)) ||
      !same_rows(d_mul, d_mul_pitch, d_y, d_y_pitch, M) || !same_rows(d_mul, d_mul_pitch, mul, mul_pitch, M) || !same_rows(d_mul, d_mul_pitch, z, z_pitch, M))
    return PSRL_ERR_INVALID_ARG;
  int* status = static_cast<int*>(workspace);
  int32_t first = 1;   // no kernel of this call has been launched yet
  const void* dz = d_y;
  int64_t dz_pitch = d_y_pitch;
  if (elementwise || d_bias) {
    if (elementwise && (d_x || d_weight)) { dz = ws + L.dz; dz_pitch = L.dz_pitch; }
    auto run = [&](auto zero) {
      using T = decltype(zero);
      DzParams<T> q{};
      q.d_y = static_cast<const T*>(d_y); q.d_y_pitch = d_y_pitch;
      q.mul = static_cast<const T*>(mul); q.mul_pitch = mul_pitch;
      q.z = activation != PSRL_ACT_NONE || d_mul ? static_cast<const T*>(z) : nullptr; q.z_pitch = z_pitch;
      q.d_mul = static_cast<T*>(d_mul); q.d_mul_pitch = d_mul_pitch;
      q.dz = dz == d_y ? nullptr : reinterpret_cast<T*>(ws + L.dz); q.dz_pitch = dz_pitch;
      q.part = d_bias ? reinterpret_cast<float*>(ws + L.part) : nullptr;
      q.M = int32_t(M); q.N = int32_t(N); q.act = activation; q.rows = int32_t(dz_rows(M)); q.status = status;
      return run_dz(q, static_cast<T*>(d_bias), s);
    };
    e = dtype == PSRL_F32 ? run(float()) : run(__nv_bfloat16());
    if (e != cudaSuccess) return cuda_failed(e);
    first = 0;   // dz_kernel has cleared the status
  }
  if (!d_x && !d_weight) {
    if (first && workspace) e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  if (dtype == PSRL_F32) {
    const F32Operand z_at{static_cast<const float*>(dz), dz_pitch}, x_at{static_cast<const float*>(x), x_pitch}, w_at{static_cast<const float*>(weight), weight_pitch};
    float* part = reinterpret_cast<float*>(ws + L.f32);
    auto params = [&](F32Operand a, F32Operand b, int64_t rows, int64_t depth, void* out, int64_t pitch) {
      F32Params q{};
      q.a = a; q.b = b;
      q.M = int32_t(rows); q.N = int32_t(K); q.depth = int32_t(depth); q.clear = first; q.status = status;
      first = 0;
      q.e.y = static_cast<float*>(out); q.e.y_pitch = pitch;
      return q;
    };
    if (d_x) e = f32_product<false, true>(params(z_at, w_at, M, N, d_x, d_x_pitch), part, s);
    if (e == cudaSuccess && d_weight) e = f32_product<true, true>(params(z_at, x_at, N, M, d_weight, d_weight_pitch), part, s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  // Both in one launch, or d_x shared out over its depth first, as the times of the few-rows kernel and of the pairs' rounds go; by the
  // sizes alone, so that a gradient has the same bits whether or not the other is wanted.
  const int64_t steps_x = div_up(N, 64), steps_w = div_up(M, 64);
  const GradShape both = grad_shape(M, steps_x, N, steps_w, K), of_weight = grad_shape(0, 0, N, steps_w, K);
  if (d_x && few_time(M, K, steps_x) + of_weight.time < both.time) {
    const FewShape f = few_shape(M, K, div_up(N, 64));
    FewMaps maps;
    if (!make_map_bf16_2d(&maps.a, weight, K, N, weight_pitch * 2, 64) || !make_map_bf16_2d(&maps.b, dz, N, M, dz_pitch * 2, f.tile_rows)) return PSRL_ERR_CUDA;
    FewParams q{};
    q.rows = int32_t(M); q.cols = int32_t(K); q.steps = int32_t(div_up(N, 64)); q.a_mn = 1;
    q.y = static_cast<__nv_bfloat16*>(d_x); q.y_pitch = d_x_pitch; q.clear = first; q.status = status;
    first = 0;
    e = launch_few<false>(maps, q, f, s);
    if (e != cudaSuccess) return cuda_failed(e);
    if (!d_weight) return PSRL_OK;
    d_x = nullptr;
  }
  // the deeper product first: its tiles cost more
  const int tile_n = d_x ? both.tile_n : of_weight.tile_n;
  Product px = product_of(M, K, N, 64, tile_n, 0, 1, kGradGroupBytes), pw = product_of(N, K, M, 64, tile_n, 1, 1, kGradGroupBytes);
  if (!d_x) px.m_tiles = 0;
  if (!d_weight) pw.m_tiles = 0;
  const int ix = !d_x || (d_weight && pw.steps > px.steps) ? 1 : 0, iw = 1 - ix;
  Maps maps{};
  Params p{};
  p.product[ix] = px;
  p.product[iw] = pw;
  p.ratio = (p.product[0].steps + 6) / std::max(p.product[1].steps + 6, 1);
  p.clear = first; p.status = status;
  bool made = true;
  if (d_x)
    made = make_map_bf16_2d(&maps.a[ix], dz, N, M, dz_pitch * 2, 128) && make_map_bf16_2d(&maps.b[ix], weight, K, N, weight_pitch * 2, 64) &&
           make_map_bf16_2d(&maps.out[ix], d_x, K, M, d_x_pitch * 2, 128);
  if (made && d_weight)
    made = make_map_bf16_2d(&maps.a[iw], dz, N, M, dz_pitch * 2, 64) && make_map_bf16_2d(&maps.b[iw], x, K, M, x_pitch * 2, 64) &&
           make_map_bf16_2d(&maps.out[iw], d_weight, K, N, d_weight_pitch * 2, 128);
  if (!made) return PSRL_ERR_CUDA;
  e = launch_gemm<false, kPlain>(maps, p, s);
  return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
}

}  // extern "C"
