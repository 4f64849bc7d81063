// Log-probabilities of target tokens under softmax(scale * hidden * weight^T) over a large vocabulary, and their
// gradients, without ever holding the logits: the last step of a policy's forward pass and the first of its backward.
//
// All four contractions (logits, logits again in the backward, d_hidden, d_weight) run on one matrix kernel:
//   tile 256 x 256 of a CTA pair (cta_group::2: each CTA holds 128 rows of A and 128 of the 256 columns of B, so a
//   64-deep step brings 32 KB into each SM for 512 tensor cycles; a lone CTA with a 128 x 256 tile would need 48 KB),
//   five or six 32 KB stages filled by TMA, two 256-column accumulators in tensor memory so that the epilogue of one tile
//   runs under the products of the next, persistent CTAs.
// What differs is how the operands lie (K-major or MN-major in shared memory) and the epilogue:
//   kLse   running maximum and sum of exponentials of a row over a run of vocabulary tiles   -> partial (max, sum)
//   kDz    dz = -scale G softmax, with the entries of the row's targets put in afterwards    -> bf16, one piece of the
//          vocabulary at a time in the workspace (the softmax part is rounded to bf16 as the tensor cores need it)
//   kGrad  both gradients of a piece in one launch: d_hidden += dz W, added to fp32 sums over the pieces by the TMA unit
//          and rounded once at the end, and d_weight = dz^T hidden, the whole sum in tensor memory, rounded once.
//          The few deep tiles of d_hidden come first, the many shallow ones of d_weight even out what they leave (GradPlan);
//          with few rows the depth of d_hidden is split as well, into partial sums that a last kernel adds in order.
// The pieces make dz as large as the caller's hidden states, not as the logits.
//
// The backward works on the rows that matter alone: a row without a target, or whose d_logprob are all zero (prompts,
// padding, samples without advantage), has dz = 0 whatever its hidden state holds.  The other rows are gathered first -
// one copy of their hidden states, against three products of the vocabulary's depth saved for every row left out - and
// their number stays on the device, where the products read it.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "../../include/psrl.h"
#include "attn_bf16_common.cuh"
#include "kernels.h"
#include "tma.h"

namespace psrl {
namespace {
using namespace sm100;

constexpr int kBK = 64;                      // K per stage
constexpr int kOperandBytes = 128 * kBK * 2; // one CTA's share of A or B in a stage
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kOutBytes = 128 * 128;         // what an epilogue group stores at a time: 128 rows of 128 bytes
// Two epilogue groups of four warps, one for each accumulator, so that where tiles are shallow the latencies of one tile's
// way out (products, hand-over, stores) pass under the other's; a TMA warp, an MMA warp.  d_weight of 64 rows, 1.07 GB:
// one group 335 us, two with half of every tile each 298, with every other tile each 218.
constexpr int kGroups = 2, kEpilogueWarps = 4 * kGroups, kTmaWarp = kEpilogueWarps, kMmaWarp = kTmaWarp + 1;
constexpr int kGemmThreads = (kEpilogueWarps + 2) * 32;
constexpr int kMaxRun = 8;                   // vocabulary tiles whose maximum and sum stay in registers

enum Kind { kLse, kDz, kGrad };

// Up to kTwiceRows rows, half of a tile's rows are free and everything is bound by the weights' bytes.  dz is then kept
// twice, rounded to bf16 and what that leaves, in rows r and 128 + r: the second CTA of a pair computes the same logits as the
// first, and both products add the two.  With more rows dz's roundings average out in d_weight's sums.
constexpr int kTwiceRows = 128;

// 32 KB stages of operands; the kinds that store tiles give one of them to their output buffers, two per group
constexpr int stages(Kind k) { return k == kLse ? 6 : 5; }
constexpr size_t gemm_smem(Kind k) { return size_t(stages(k)) * kStageBytes + (k == kLse ? 0 : size_t(kGroups) * 2 * kOutBytes) + 1024; }

struct GemmMaps {
  CUtensorMap a, b;     // kGrad: of d_hidden
  CUtensorMap a2, b2;   // kGrad: of d_weight
  CUtensorMap out;      // kDz: dz; kGrad: the fp32 sums of d_hidden.  Boxes of 128 rows
  CUtensorMap out2;     // kGrad: the piece's rows of d_weight
};

struct GemmParams {
  int32_t M, N;                 // valid rows and columns of the product
  int32_t n_tiles, k_blocks;
  int32_t twice;                // kDz, kGrad: rows 128 ... hold the rest of dz below bf16 (see kTwiceRows)
  const int32_t* count;         // kDz, kGrad: rows that matter, on the device (kLse: NULL, all M)
  const int32_t* row_of;        // kDz: the caller's row of a gathered row
  int32_t group;                // kLse, kDz: row tiles that are walked together
  int32_t tile_n;               // columns of a tile: 256, or fewer in the logits (a multiple of 64)
  int32_t run;                  // kLse: consecutive column tiles of one work unit
  float scale_log2;             // logits in powers of two: scale * log2(e)
  float2* part;                 // kLse: [unit column][group][M] (max, sum), powers of two
  int32_t* part_at;             // kLse: the vocabulary entry of the maximum
  const float2* row_info;       // kDz: per row (lse * log2(e), -scale * G)
  const int2* only;             // kDz: per row its target and the bits of dz there, if it has exactly one; else (-1, 0)
  int32_t col0;                 // kDz: first vocabulary entry of the piece
  int32_t vocab;                // kGrad: entries of the piece
  int32_t splits;               // kGrad: parts of d_hidden's sum over them
  int32_t acc_rows;             // kGrad: rows of one part's sums
  int32_t want_hidden, want_weight;   // kGrad
  int32_t first;                // kGrad: the first piece: the sums are stored, later they are added to
  uint32_t* pace;               // kLse: what all pairs have begun, zero at the start (see keep_pace); NULL: each at its own pace
  uint32_t pace_shift;          // in units of 1 << pace_shift steps
  int* status;
};

// The kernels of a call are launched so that each may start while the one before it runs out: what a kernel needs of the
// call's earlier kernels it reads after previous_kernel_done().
__device__ __forceinline__ void previous_kernel_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void next_kernel_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ------------------------------------------------------------------------------------------- pair-of-CTAs wrappers
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// shared::cluster address of the first CTA's copy of a shared-memory variable
__device__ __forceinline__ uint32_t in_leader(const void* p) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
  return a;
}
__device__ __forceinline__ void arrive_leader(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* m, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(kDescHi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// arrives on the barrier of both CTAs when the products issued so far are done
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
      "h"(uint16_t(3))
      : "memory");
}
// A box from shared memory to a tiled tensor map, or added to what is there (fp32).  Parts outside the tensor are dropped.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, const void* smem_src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(smem_src)), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void tma_add_2d(const CUtensorMap* m, const void* smem_src, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(smem_src)), "r"(x), "r"(y)
               : "memory");
}

// Work unit -> row tile and first column tile: groups of row tiles, inside a group the row tile moves fastest, so that the
// CTAs at work share column tiles and a group's rows stay in the L2.  For logits (tiles as deep as the hidden dimension) a
// group is as many row tiles as fit kGroupBytes: 8192 x 4096 x 131072 forward in 6.2 ms, with 72 MB or 18 MB 6.8 to 7.4;
// 16384 x 2048 x 131072 5.8 to 6.1, a tenth less than with 16 tiles; at a hidden size of 8192 18 to 144 MB are within the
// noise.  For gradients, whose tiles are as deep as the rows or the vocabulary and walk it in step, the operands of the CTAs
// at work count and not the group's: kGradGroup tiles, 8192 x 4096 x 131072 backward in 20.1 ms, with 4 20.5, 16 20.6, 32 21.5.
constexpr int64_t kGroupBytes = int64_t(36) << 20;
constexpr int kGradGroup = 8;
__device__ __forceinline__ void unit_tile(int group, int m_tiles, int unit, int n_units, int& mt, int& nu) {
  const int per = group * n_units;
  const int g = unit / per, r = unit - g * per;
  const int gm = min(group, m_tiles - g * group);
  nu = r / gm;
  mt = g * group + r - nu * gm;
}

// Pace.  The pairs at work share what they read of the rows and of the weights only while they are about as far along the
// depth: left to themselves they drift apart by whole tiles, and what one of them has fetched has left the L2 when the others
// come by (8192 x 8192 x 65536: 18.4 GB read from DRAM, 10.4 with pace, 4.4 if each group of rows reads the weights once).
// So each pair counts every few steps that it begins, and goes on only when all pairs' sum is that of pairs one such unit
// behind.  It is a help and no barrier: a pair that has waited in vain (kPaceTries, about 0.2 ms; other work may hold some
// SMs) waits no more, and one that is through counts kPaceDone, which frees the others.  Forward, TFLOP/s with a pause
// between the calls: 16384 x 8192 in units of 8 steps 1480 to 1535, without pace 1236 to 1500; 2048 x 16384 x 65536 1460, 1350; 1024 x 8192
// 1440, 1270 to 1400; 8192 x 4096 in units of 16 1530 to 1580, 1450 to 1555 (units of 8 cost 3 % there back to back).  At a
// hidden size of 2048 it loses up to 3 %, with 512 to 700 rows 1 %, with less than four rounds of tiles up to 13 %.  In between:
// 3584 deep 8192 rows 1600 with pace, 1558 without, 16384 rows 1628, 1565, 2048 rows the same; 2560 deep 8192 rows 1610, 1589, 2048
// rows 1430, 1470.  So the depth could be a little lower; it is where the gain is beyond doubt at every number of rows.  The
// gradients lose 1 to 2 %: few pairs at work share an operand there.
constexpr int kPaceTries = 200;
constexpr size_t kPaceAt = 128;            // in the header of the workspace
constexpr int kPaceRows = 1024, kPaceDepth = 4096;
constexpr uint32_t kPaceDone = 1u << 24;   // 74 pairs' stay below 2^31
__device__ __forceinline__ void count_pace(uint32_t* pace, uint32_t n) {
  asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(pace), "r"(n) : "memory");
}
__device__ __forceinline__ uint32_t read_pace(const uint32_t* pace) {
  uint32_t n;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(n) : "l"(pace) : "memory");
  return n;
}
__device__ __forceinline__ bool keep_pace(const uint32_t* pace, uint32_t want) {
  for (int i = 0; i < kPaceTries; ++i) {
    if (int32_t(read_pace(pace) - want) >= 0) return true;
    __nanosleep(100);
  }
  return false;
}

// The targets of a row, kept inside the array whatever the offsets say.
__device__ __forceinline__ void target_range(const int32_t* off, int64_t row, int n_targets, int& b, int& e) {
  b = off ? min(max(off[row], 0), n_targets) : int(row);
  e = off ? min(max(off[row + 1], b), n_targets) : int(row) + 1;
}

// What a pair of CTAs does next in kGrad: a tile of d_hidden (over part of its depth) or of d_weight.
struct GradWork {
  int weight;       // 1: d_weight
  int mt, nt;
  int kb0, kb1;     // steps of its sum
  int split;
};
// Pair c of C takes the units c, c + C, ... of d_hidden.  The first r pairs then have one more than the others, who make up
// for it with the first tiles of d_weight; the rest of those go round.  No counter, no order that could vary.
struct GradPlan {
  int m_tiles, v_tiles, per, n_hidden, mine, n_weight, ahead, light, steps, row_steps;
  bool lighter;

  __device__ __forceinline__ GradPlan(const GemmParams& p, int rows, int c, int C) {
    m_tiles = p.want_hidden ? (rows + 255) / 256 : 0;   // twice: rows <= 128, one tile as well
    v_tiles = p.want_weight ? (p.vocab + 255) / 256 : 0;
    per = m_tiles * p.n_tiles;
    n_hidden = per * p.splits;
    steps = (p.vocab + kBK - 1) / kBK;
    row_steps = (rows + kBK - 1) / kBK << p.twice;
    const int q = n_hidden / C, r = n_hidden - q * C;
    mine = q + (c < r ? 1 : 0);
    n_weight = v_tiles * p.n_tiles;
    light = C - r;
    lighter = c >= r;
    // cost of a unit in steps; a tile of few steps is bound by its epilogue, worth about six
    ahead = r > 0 ? min((steps / p.splits + 6) / max(row_steps, 6), n_weight / light) : 0;
  }
  __device__ __forceinline__ bool get(const GemmParams& p, int c, int C, int i, GradWork& w) const {
    if (i < mine) {
      const int u = c + i * C;
      w.weight = 0;
      w.split = u / per;
      unit_tile(kGradGroup, m_tiles, u - w.split * per, p.n_tiles, w.mt, w.nt);
      w.kb0 = part_of(steps, w.split, p.splits);
      w.kb1 = part_of(steps, w.split + 1, p.splits);
      return true;
    }
    const int j = i - mine;
    int at = ahead * light;
    if (lighter && j < ahead) at = j * light + c - (C - light);
    else at += (lighter ? j - ahead : j) * C + c;
    if (at >= n_weight) return false;
    w.weight = 1;
    w.split = 0;
    w.kb0 = 0;
    w.kb1 = row_steps;
    unit_tile(kGradGroup, v_tiles, at, p.n_tiles, w.mt, w.nt);
    return true;
  }
  // where part k of n begins; n <= 16 parts of fewer than 2^25 steps
  __device__ __forceinline__ static int part_of(int steps, int k, int n) { return int(unsigned(steps) * unsigned(k) / unsigned(n)); }
};

template <int kStages>
struct __align__(8) PairBarriers {
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
};

// How results leave: the CTA's 128 rows, 128 bytes of each at a time, through two buffers in shared memory (the 128-byte
// swizzle of the tensor map makes the row-per-thread writes free of bank conflicts) and one TMA store per buffer.  With 32
// bytes per thread and row straight to global memory, or a store for each warp's 32 rows, d_weight of 64 rows (1.07 GB) took
// 335 us: the first is bound by scattered sectors, the second by the TMA unit's time per box.
// The four warps of a group take every step together; the named barrier is theirs.
constexpr uint32_t kBarOut = 1, kOutThreads = 128;   // barrier 1 + group
struct TileOut {
  uint8_t* buf;      // two times kOutBytes
  uint32_t bar;
  int row;           // the thread's row of the tile
  uint32_t n = 0;    // stores so far

  // the buffer to write to next: once the store before last has been read out
  __device__ __forceinline__ uint8_t* next() {
    if (n >= 2 && row == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
    named_sync(bar, kOutThreads);
    return buf + (n & 1) * kOutBytes;
  }
  __device__ __forceinline__ void put(uint8_t* b, int chunk, uint4 v) const {
    *reinterpret_cast<uint4*>(b + row * 128 + ((chunk ^ (row & 7)) << 4)) = v;
  }
  __device__ __forceinline__ void send(const CUtensorMap* m, int x, int y, bool add) {
    fence_proxy_async();
    named_sync(bar, kOutThreads);
    if (row == 0) {
      if (add) tma_add_2d(m, buf + (n & 1) * kOutBytes, x, y);
      else tma_store_2d(m, buf + (n & 1) * kOutBytes, x, y);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    ++n;
  }
  __device__ __forceinline__ void finish() {
    if (row == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
};

// Exponent of a probability: z - lse, both in powers of two, each with its own rounding.  With logits of 10^8 that alone is some
// hundred, and the probability infinite, so it is held at one.  NaN stays.
__device__ __forceinline__ float at_most_one(float exponent) {
  float y;
  asm("min.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(exponent));
  return y;
}

// dz rounded to bf16, or the rest below that
__device__ __forceinline__ __nv_bfloat16 dz_part(float v, bool rest) {
  const __nv_bfloat16 y = __float2bfloat16_rn(v);
  return rest ? __float2bfloat16_rn(v - __bfloat162float(y)) : y;
}

template <Kind kKind>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmMaps maps, const GemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int kStages = stages(kKind);
  __shared__ PairBarriers<kStages> bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_go[kGroups][2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int cluster = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;
  const int n_units = (p.n_tiles + p.run - 1) / p.run;
  const int tile_n = kKind == kGrad ? 256 : p.tile_n;

  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < kStages; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&bar.acc_full[i], 1); mbar_init(&bar.acc_empty[i], 8); }   // four warps in either CTA
    fence_mbar_init();
    tma_prefetch_desc(&maps.a);
    tma_prefetch_desc(&maps.b);
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
  if (kKind == kLse && blockIdx.x == 0 && tid == 0) *p.status = int(PSRL_OK);

  const int rows = kKind == kLse ? p.M : *p.count;
  const int m_tiles = (rows + 255) / 256;

  const GradPlan plan(p, rows, cluster, n_clusters);   // kGrad

  // The i-th work unit of this pair: a row tile and consecutive column tiles, all over steps kb0 .. kb1.
  auto work = [&](int i, GradWork& w, int& nt_end) -> bool {
    if constexpr (kKind == kGrad) {
      if (!plan.get(p, cluster, n_clusters, i, w)) return false;
      nt_end = w.nt + 1;
    } else {
      const int unit = cluster + i * n_clusters;
      if (unit >= m_tiles * n_units) return false;
      int nu;
      unit_tile(p.group, m_tiles, unit, n_units, w.mt, nu);
      w.weight = 0;
      w.kb0 = 0;
      w.kb1 = p.k_blocks;
      w.split = nu;
      w.nt = nu * p.run;
      nt_end = min(w.nt + p.run, p.n_tiles);
    }
    return true;
  };

  const uint32_t tmem = s_tmem;
  volatile int* abortp = &s_abort;
  GradWork w;
  int nt_end;

  if (warp == kTmaWarp) {
    // ======================= TMA producer (both CTAs) =======================
    if (lane == 0) {
      const uint32_t stage_tx = 2 * (kOperandBytes + uint32_t(tile_n) * kBK);   // of both CTAs
      uint32_t it = 0;
      bool ok = true, wait_pace = true;
      const bool paced = kKind == kLse && p.pace && rank == 0;   // the second CTA keeps step through the stages
      for (int i = 0; ok && work(i, w, nt_end); ++i) {
        const bool a_mn = kKind == kGrad && w.weight;
        const CUtensorMap* ma = a_mn ? &maps.a2 : &maps.a;
        const CUtensorMap* mb = a_mn ? &maps.b2 : &maps.b;
        const int m0 = w.mt * 256 + int(rank) * 128;
        for (int nt = w.nt; nt < nt_end && ok; ++nt) {
          const int n0 = nt * tile_n + int(rank) * (tile_n / 2);
          // twice: the second half of d_weight's steps are the rows from 128 on
          const int skip = kKind == kGrad && w.weight && p.twice ? 128 / kBK - w.kb1 / 2 : 0;
          for (int step = w.kb0; step < w.kb1; ++step, ++it) {
            const int kb = step + (skip && step >= w.kb1 / 2 ? skip : 0);
            if (paced && (it & ((1u << p.pace_shift) - 1)) == 0) {
              count_pace(p.pace, 1);
              const uint32_t n = it >> p.pace_shift;
              if (wait_pace && n > 1) wait_pace = keep_pace(p.pace, (n - 1) * uint32_t(n_clusters));
            }
            const uint32_t s = it % kStages, round = it / kStages;
            if (round > 0 && !mbar_wait(&bar.empty[s], (round + 1) & 1, abortp, p.status)) { ok = false; break; }
            // the second CTA's copies count on the first one's barrier as well
            if (rank == 0) mbar_expect_tx(&bar.full[s], stage_tx);
            const uint32_t full = in_leader(&bar.full[s]);
            uint8_t* sa = smem + s * kStageBytes;
            uint8_t* sb = sa + kOperandBytes;
            if (a_mn) {
              tma_load_pair(sa, ma, full, m0, kb * kBK);
              tma_load_pair(sa + kOperandBytes / 2, ma, full, m0 + 64, kb * kBK);
            } else {
              tma_load_pair(sa, ma, full, kb * kBK, m0);
            }
            if (kKind == kGrad) {
              tma_load_pair(sb, mb, full, n0, kb * kBK);
              tma_load_pair(sb + kOperandBytes / 2, mb, full, n0 + 64, kb * kBK);
            } else {
              tma_load_pair(sb, mb, full, kb * kBK, n0);
            }
          }
        }
      }
      if (paced) count_pace(p.pace, kPaceDone);
      // the last arrivals on the stages' barriers come from the pair's products: this CTA stays until they are here
      for (uint32_t i = 0; i < kStages && ok; ++i) {
        const uint32_t uses = it / kStages + (i < it % kStages ? 1 : 0);
        if (uses > 0) ok = mbar_wait(&bar.empty[i], (uses + 1) & 1, abortp, p.status);
      }
    }
  } else if (warp == kMmaWarp) {
    // ======================= MMA issuer (first CTA of the pair) =======================
    if (rank == 0) {
      // Operands: hidden, weight and dz with the depth contiguous (K-major) in the logits; in the gradients both lie with
      // the other side contiguous (MN-major), but for dz in d_hidden.  An MN-major operand's 64-wide blocks are kLbo bytes
      // apart and a 16-deep step is 16 rows of 128 bytes; K-major, a step is 32 bytes.
      constexpr uint32_t kLbo = kOperandBytes / 2, kStepK = 32 >> 4, kStepMn = 2048 >> 4;
      constexpr uint32_t kStepB = kKind == kGrad ? kStepMn : kStepK;
      const bool elected = elect_one();
      uint32_t it = 0, tile = 0;
      bool ok = true;
      for (int i = 0; ok && work(i, w, nt_end); ++i) {
        const bool a_mn = kKind == kGrad && w.weight;
        const uint32_t idesc = make_idesc(256, tile_n, a_mn ? 1 : 0, kKind == kGrad ? 1 : 0);
        const uint32_t step_a = a_mn ? kStepMn : kStepK, lbo_a = a_mn ? kLbo : 0;
        for (int nt = w.nt; nt < nt_end && ok; ++nt, ++tile) {
          const uint32_t a = tile & 1, use = tile >> 1;
          if (use > 0) ok = __all_sync(0xffffffffu, mbar_wait(&bar.acc_empty[a], (use + 1) & 1, abortp, p.status));
          if (!ok) break;
          tc_fence_after();
          const uint32_t d = tmem + a * 256;
          for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
            const uint32_t s = it % kStages;
            if (!mbar_wait_all1(&bar.full[s], (it / kStages) & 1, abortp, p.status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sa = smem_u32(smem) + s * kStageBytes, sb = sa + kOperandBytes;
            const uint32_t da = desc_lo(sa, lbo_a), db = desc_lo(sb, kKind == kGrad ? kLbo : 0);
            if (elected) {
#pragma unroll
              for (uint32_t k = 0; k < kBK / 16; ++k)
                mma_pair(d, da + k * step_a, db + k * kStepB, idesc, (kb > w.kb0 || k > 0) ? 1u : 0u);
              commit_pair(&bar.empty[s]);
            }
            __syncwarp();
          }
          if (ok && elected) commit_pair(&bar.acc_full[a]);
          __syncwarp();
        }
      }
    }
  } else {
    // ======================= epilogue: one thread per row, a group for every other tile =======================
    const int group = warp >> 2, gt = tid & 127;
    const uint32_t bar_id = kBarOut + group;
    const uint32_t lane_addr = tmem + (uint32_t(warp & 3) << 21) + group * 256;   // lane 32 * (warp % 4)
    const uint32_t acc_empty = in_leader(&bar.acc_empty[group]);
    TileOut out;
    out.buf = smem + kStages * kStageBytes + group * 2 * kOutBytes;
    out.bar = bar_id;
    out.row = gt;
    uint32_t tile = 0;
    bool ok = true;
    for (int i = 0; ok && work(i, w, nt_end); ++i) {
      const int row0 = w.mt * 256 + int(rank) * 128, row = row0 + gt;
      const bool rest = kKind == kDz && p.twice && rank == 1;
      const int of_row = rest ? gt : row;
      const bool live = of_row < rows;
      float best = -CUDART_INF_F, sum = 0.f;                       // kLse
      int best_at = 0;
      float lse2 = 0.f, coef = 0.f;                                // kDz
      int2 only = make_int2(-1, 0);
      if (kKind == kDz && live) {
        const int user_row = p.row_of[of_row];
        const float2 ri = p.row_info[user_row];
        lse2 = ri.x; coef = ri.y;
        only = p.only[user_row];
      }
      for (int nt = w.nt; nt < nt_end; ++nt, ++tile) {
        if ((tile & 1) != uint32_t(group)) continue;
        // one warp waits for its group: the four leave together if the wait gives up, so none is missed at their barrier
        if ((warp & 3) == 0) {
          ok = mbar_wait(&bar.acc_full[group], (tile >> 1) & 1, abortp, p.status);
          if (lane == 0) s_go[group][(tile >> 1) & 1] = ok;
        }
        named_sync(bar_id, kOutThreads);
        ok = s_go[group][(tile >> 1) & 1];
        if (!ok) break;
        tc_fence_after();
        const int n0 = nt * tile_n, n_end = min(n0 + tile_n, p.N);
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const int col = n0 + c * 64;
          if (col >= n_end) break;   // uniform in the group
          uint32_t r[2][32];
          tmem_ld32(lane_addr + c * 64, r[0]);
          tmem_ld32(lane_addr + c * 64 + 32, r[1]);
          tmem_wait_ld();
          if constexpr (kKind == kLse) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (col + 32 * h + 32 > p.N) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (col + 32 * h + i >= p.N) r[h][i] = __float_as_uint(p.scale_log2 > 0.f ? -CUDART_INF_F : CUDART_INF_F);
              }
              float top = -CUDART_INF_F;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float z = __uint_as_float(r[h][i]) * p.scale_log2;
                r[h][i] = __float_as_uint(z);
                top = fmaxf(top, z);
              }
              if (top > best) {   // seldom after the first columns
                sum *= ex2(best - top);
                best = top;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (__uint_as_float(r[h][i]) == top) best_at = col + 32 * h + i;
              }
              const float ref = best == -CUDART_INF_F ? 0.f : best;   // nothing finite yet: every term is zero
              float s0 = 0.f, s1 = 0.f;
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                s0 += ex2(__uint_as_float(r[h][i]) - ref);
                s1 += ex2(__uint_as_float(r[h][i + 1]) - ref);
              }
              sum += s0 + s1;
            }
          } else if (kKind == kGrad && !w.weight) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (col + 32 * h >= p.N) break;
              uint8_t* b = out.next();
#pragma unroll
              for (int j = 0; j < 8; ++j)
                out.put(b, j, w.kb1 > w.kb0 ? make_uint4(r[h][4 * j], r[h][4 * j + 1], r[h][4 * j + 2], r[h][4 * j + 3])
                                            : make_uint4(0, 0, 0, 0));   // an empty sum writes no accumulator
              // the parts' sums follow one another; rows behind the last one are sums nobody reads, but not another part's
              if (row0 < p.acc_rows) out.send(&maps.out, col + 32 * h, w.split * p.acc_rows + row0, !p.first);
            }
          } else {
            uint8_t* b = out.next();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t o[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float lo = __uint_as_float(r[j / 4][j % 4 * 8 + 2 * i]), hi = __uint_as_float(r[j / 4][j % 4 * 8 + 2 * i + 1]);
                if constexpr (kKind == kDz) {
                  lo = coef * ex2(at_most_one(fmaf(lo, p.scale_log2, -lse2)));
                  hi = coef * ex2(at_most_one(fmaf(hi, p.scale_log2, -lse2)));
                }
                o[i] = pack_bf16(lo, hi);
                if (kKind == kDz && rest) o[i] = pack_bf16(lo - __uint_as_float(o[i] << 16), hi - __uint_as_float(o[i] & 0xffff0000u));
              }
              // kDz: rows behind the last one are zero, as the product for d_weight reads dz in steps of kBK rows
              const bool any = kKind == kDz ? live : w.kb1 > w.kb0;
              out.put(b, j, any ? make_uint4(o[0], o[1], o[2], o[3]) : make_uint4(0, 0, 0, 0));
            }
            if constexpr (kKind == kDz) {
              // the row's target, where it is in these columns, over what this thread has just written (patch_kernel does it for
              // rows with several: their number has no limit, and a tile would wait for its longest row)
              const uint32_t x = uint32_t(only.x) - uint32_t(p.col0 + col);
              if (x < uint32_t(min(64, p.N - col)))
                *reinterpret_cast<__nv_bfloat16*>(b + gt * 128 + (((x >> 3) ^ (gt & 7)) << 4) + (x & 7) * 2) =
                    dz_part(__int_as_float(only.y), rest);
            }
            out.send(kKind == kGrad ? &maps.out2 : &maps.out, col, row0, false);
          }
        }
        // the accumulator may be overwritten
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_leader(acc_empty);
      }
      if (kKind == kLse && ok && live) {
        const int64_t at = (int64_t(w.split) * kGroups + group) * rows + row;
        p.part[at] = make_float2(best, sum);
        p.part_at[at] = best_at;
      }
    }
    if (kKind != kLse) out.finish();
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

// ------------------------------------------------------------------------------------------------- small kernels

// Few rows (the next tokens of a rollout): the weights are read once whatever the rows, so the products are bound by HBM
// and ordinary fp32 arithmetic keeps up, two multiply-adds an instruction.  A warp takes four vocabulary entries at a time
// and holds their products with all kRows hidden rows, which lie in shared memory; running maximum and sum per row.
constexpr int kFewThreads = 256, kFewV = 4;
// Blocks of an SM, and of the launch for each SM: one wave, as every block gets the same share of the vocabulary (4096 x 131072,
// 4 rows: 185 us; twice as many blocks are no quicker and leave twice the partial sums).
__host__ __device__ constexpr int few_blocks(int rows) { return rows == 1 ? 4 : rows == 2 ? 3 : 2; }
constexpr size_t kFewSmem = 128 * 1024;   // hidden rows at most

// eight bf16 as four pairs of fp32
__device__ __forceinline__ void widen(const uint4& x, f32x2 (&o)[4]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = make_f32x2(w[j] << 16, w[j] & 0xffff0000u);
}

template <int kRows>
__global__ void __launch_bounds__(kFewThreads, few_blocks(kRows)) few_rows_kernel(int M, int vecs, int vocab, const uint4* __restrict__ hidden,
                                                               int64_t h_pitch_vecs, const uint4* __restrict__ weight,
                                                               int64_t w_pitch_vecs, float scale_log2, float2* __restrict__ part, int* __restrict__ status) {
  next_kernel_may_start();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = int(PSRL_OK);
  extern __shared__ uint4 s_h[];   // [kRows][vecs]
  __shared__ float2 s_best[kFewThreads / 32][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kRows * vecs; i += kFewThreads) {
    const int r = i / vecs;
    s_h[i] = r < M ? hidden[r * h_pitch_vecs + (i - r * vecs)] : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  float best[kRows], sum[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) { best[r] = -CUDART_INF_F; sum[r] = 0.f; }
  const int stride = gridDim.x * (kFewThreads / 32) * kFewV;
  for (int v0 = (blockIdx.x * (kFewThreads / 32) + warp) * kFewV; v0 < vocab; v0 += stride) {
    f32x2 acc[kRows][kFewV];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int k = 0; k < kFewV; ++k) acc[r][k] = make_f32x2(0.f, 0.f);
    const uint4* wp[kFewV];
#pragma unroll
    for (int k = 0; k < kFewV; ++k) wp[k] = weight + int64_t(min(v0 + k, vocab - 1)) * w_pitch_vecs;
#pragma unroll 2
    for (int i = lane; i < vecs; i += 32) {
      f32x2 w[kFewV][4];
#pragma unroll
      for (int k = 0; k < kFewV; ++k) widen(__ldcs(wp[k] + i), w[k]);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        f32x2 h[4];
        widen(s_h[r * vecs + i], h);
#pragma unroll
        for (int k = 0; k < kFewV; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[r][k] = fma2(h[j], w[k][j], acc[r][k]);
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      float z[kFewV], top = best[r];
#pragma unroll
      for (int k = 0; k < kFewV; ++k) {
        float x, y;
        split_f32x2(acc[r][k], x, y);
        x += y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        z[k] = v0 + k < vocab ? x * scale_log2 : -CUDART_INF_F;
        top = fmaxf(top, z[k]);
      }
      const float ref = top == -CUDART_INF_F ? 0.f : top;
      sum[r] *= ex2(best[r] - ref);
#pragma unroll
      for (int k = 0; k < kFewV; ++k) sum[r] += ex2(z[k] - ref);
      best[r] = top;
    }
  }
  if (lane == 0)
    for (int r = 0; r < kRows; ++r) s_best[warp][r] = make_float2(best[r], sum[r]);
  __syncthreads();
  if (threadIdx.x < kRows && threadIdx.x < M) {
    const int r = threadIdx.x;
    float top = -CUDART_INF_F, s = 0.f;
    for (int i = 0; i < kFewThreads / 32; ++i) top = fmaxf(top, s_best[i][r].x);
    const float ref = top == -CUDART_INF_F ? 0.f : top;
    for (int i = 0; i < kFewThreads / 32; ++i) s += s_best[i][r].y * ex2(s_best[i][r].x - ref);
    part[int64_t(blockIdx.x) * M + r] = make_float2(top, s);
  }
}

// lse of kRows rows from their partial (max, sum), then the log-probabilities of the rows' targets: the target's logit is a
// dot product of its own (two rows read per target, against a whole pass over the weights for the lse).
// The tensor cores cut off what a step of 16 adds below the sum's last bit, always towards zero: after 256 steps a logit of
// 20 is about 3e-5 short.  That matters where one entry carries the sum - a confident row, whose log-probability is the
// small difference of two such numbers - so the largest entry's logit is computed again, in fp32, and its term replaced:
// lse of 8192 rows of 4096 deep products 3.0e-6 -> 6.3e-7 relative to 64 bits.
__device__ __forceinline__ float warp_sum(f32x2 acc) {
  float z, z1;
  split_f32x2(acc, z, z1);
  z += z1;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
  return z;
}
// dot product of two rows of `vecs` 16-byte vectors, for the whole warp
__device__ __forceinline__ float warp_dot(const float* x, const float* y, int vecs) {
  const float4 *xv = reinterpret_cast<const float4*>(x), *yv = reinterpret_cast<const float4*>(y);
  f32x2 acc = make_f32x2(0.f, 0.f);
#pragma unroll 4
  for (int i = threadIdx.x & 31; i < vecs; i += 32) {
    const float4 a = xv[i], b = yv[i];
    acc = fma2(make_f32x2(a.x, a.y), make_f32x2(b.x, b.y), acc);
    acc = fma2(make_f32x2(a.z, a.w), make_f32x2(b.z, b.w), acc);
  }
  return warp_sum(acc);
}
__device__ __forceinline__ float warp_dot(const __nv_bfloat16* x, const __nv_bfloat16* y, int vecs) {
  const uint4 *xv = reinterpret_cast<const uint4*>(x), *yv = reinterpret_cast<const uint4*>(y);
  f32x2 acc = make_f32x2(0.f, 0.f);
#pragma unroll 4
  for (int i = threadIdx.x & 31; i < vecs; i += 32) {
    f32x2 a[4], b[4];
    widen(xv[i], a);
    widen(yv[i], b);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = fma2(a[j], b[j], acc);
  }
  return warp_sum(acc);
}

constexpr int kFinalThreads = 256;
template <int kRows, class T>
__global__ void __launch_bounds__(kFinalThreads) final_kernel(const float2* __restrict__ part, const int32_t* __restrict__ part_at, int n_parts, int M, int hidden_dim,
                                                              int vocab, const T* __restrict__ hidden, int64_t h_pitch,
                                                              const T* __restrict__ weight, int64_t w_pitch,
                                                              const int32_t* __restrict__ targets, const int32_t* __restrict__ off,
                                                              int n_targets, float scale, float* __restrict__ logprob,
                                                              float* __restrict__ lse) {
  constexpr int kSlices = kFinalThreads / kRows, kWarps = kFinalThreads / 32;
  __shared__ float2 s_part[kSlices][kRows];
  __shared__ int32_t s_at[kSlices][kRows];
  __shared__ float s_lse[kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row0 = blockIdx.x * kRows, mine = threadIdx.x % kRows, slice = threadIdx.x / kRows, row = row0 + mine;
  // The targets' logits need nothing of the kernel before: they are computed while it runs out.  Target number `at` of the
  // block's rows is warp at % kWarps's.
  const int vecs = hidden_dim / int(16 / sizeof(T));
  int at = 0;
  for (int r = 0; r < kRows && row0 + r < M; ++r) {
    int b, e;
    target_range(off, row0 + r, n_targets, b, e);
    for (int t = b; t < e; ++t, ++at) {
      if (at % kWarps != warp) continue;
      const int y = targets[t];
      if (y < 0 || y >= vocab) continue;
      const float z = warp_dot(hidden + int64_t(row0 + r) * h_pitch, weight + int64_t(y) * w_pitch, vecs);
      if (lane == 0) logprob[t] = scale * z;   // the same thread subtracts the lse below
    }
  }
  previous_kernel_done();
  float m = -CUDART_INF_F, s = 0.f;
  int m_at = 0;
  if (row < M) {
    for (int i = slice; i < n_parts; i += kSlices) {
      const float2 x = part[int64_t(i) * M + row];
      if (part_at && x.x > m) m_at = part_at[int64_t(i) * M + row];
      const float top = fmaxf(m, x.x);
      const float ref = top == -CUDART_INF_F ? 0.f : top;
      s = s * exp2f(m - ref) + x.y * exp2f(x.x - ref);
      m = top;
    }
  }
  s_part[slice][mine] = make_float2(m, s);
  s_at[slice][mine] = m_at;
  for (int half = kSlices / 2; half > 0; half /= 2) {
    __syncthreads();
    if (slice < half) {
      const float2 x = s_part[slice][mine], y = s_part[slice + half][mine];
      const float top = fmaxf(x.x, y.x), ref = top == -CUDART_INF_F ? 0.f : top;
      s_part[slice][mine] = make_float2(top, x.y * exp2f(x.x - ref) + y.y * exp2f(y.x - ref));
      if (y.x > x.x) s_at[slice][mine] = s_at[slice + half][mine];
    }
  }
  __syncthreads();
  for (int r = warp; r < kRows && row0 + r < M; r += kWarps) {
    float2 x = s_part[0][r];
    if (part_at && fabsf(x.x) <= 1e30f) {   // not for infinities and NaN
      const float z = warp_dot(hidden + int64_t(row0 + r) * h_pitch, weight + int64_t(s_at[0][r]) * w_pitch, vecs) * (scale * kLog2e);
      const float d = z - x.x, rest = x.y - 1.f;   // the maximum's term of the sum is one
      if (fabsf(d) < 64.f) x.y = rest + exp2f(d);
      // logits so large that the two sums are far apart: the smaller of the largest term and the rest does not count
      else if (d < 0.f && rest > 0.f) x.y = rest;
      else x = make_float2(z, rest == rest ? 1.f : rest);   // NaN stays
    }
    if (lane == 0) {
      const float l = ((x.x == -CUDART_INF_F ? 0.f : x.x) + log2f(x.y)) * kLn2;
      s_lse[r] = l;
      lse[row0 + r] = l;
    }
  }
  __syncthreads();
  at = 0;
  for (int r = 0; r < kRows && row0 + r < M; ++r) {
    int b, e;
    target_range(off, row0 + r, n_targets, b, e);
    if (lane == 0) {
      for (int t = b + (warp - at % kWarps + kWarps) % kWarps; t < e; t += kWarps) {
        const int y = targets[t];
        // a log-probability is not positive; the two sums are rounded apart.  (fminf would turn NaN into a certainty.)
        const float x = logprob[t] - s_lse[r];
        logprob[t] = y >= 0 && y < vocab ? (x > 0.f ? 0.f : x) : 0.f;
      }
    }
    at += e - b;
  }
}

// Per row the sum G of its targets' gradients, and dz at every target: scale (g_t - G p_t), g_t = the sum over the row's
// targets with the same token.  Written as (g_t - G) - G (e^lp - 1): for a row with one token the first difference is
// zero and nothing cancels as its probability nears one.  A warp per row; one bit per row says whether any gradient is not
// zero.
// Equal tokens: 32 targets at a time are compared across the warp; a row with more than that keeps its tokens' sums in a
// hash table of twice as many places, and the warp adds one batch after the other, so the order of every sum is fixed.
constexpr int kRowsPerByte = 8;
struct TokenSum {
  int32_t token;
  float sum;
};
// the place of `token` in a table of `places` that has room; -1 is free
__device__ __forceinline__ int place_of(volatile TokenSum* table, int places, int token, bool insert) {
  uint32_t at = (uint32_t(token) * 2654435761u) % uint32_t(places);
  for (int i = 0; i < places; ++i) {
    const int seen = insert ? atomicCAS(const_cast<int32_t*>(&table[at].token), -1, token) : table[at].token;
    if (seen == token || seen == -1) break;
    at = at + 1 == uint32_t(places) ? 0 : at + 1;
  }
  return int(at);
}

__global__ void __launch_bounds__(kRowsPerByte * 32) rows_kernel(int M, int vocab, const int32_t* __restrict__ targets,
                                                                 const int32_t* __restrict__ off, int n_targets,
                                                                 const float* __restrict__ logprob, const float* __restrict__ lse,
                                                                 const float* __restrict__ d_logprob, float scale,
                                                                 float2* __restrict__ row_info, int2* __restrict__ only,
                                                                 float* __restrict__ entry, TokenSum* table,
                                                                 uint8_t* __restrict__ matters, int* __restrict__ status) {
  next_kernel_may_start();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = int(PSRL_OK);
  __shared__ uint32_t s_bits;
  if (threadIdx.x == 0) s_bits = 0;
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * kRowsPerByte + warp;
  if (row < M) {
    int b, e;
    target_range(off, row, n_targets, b, e);
    float total = 0.f;
    bool any = false;
    for (int t = b + lane; t < e; t += 32) {
      const int y = targets[t];
      if (y < 0 || y >= vocab) continue;
      const float g = d_logprob[t];
      total += g;
      any |= g != 0.f;   // NaN counts
    }
    any = __any_sync(0xffffffffu, any);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    int2 one = make_int2(-1, 0);
    if (any) {
      volatile TokenSum* mine = table + 2 * int64_t(b);   // read past the L1, which atomics do not update
      const int places = 2 * (e - b);
      const bool hashed = e - b > 32;
      if (hashed) {
        for (int i = lane; i < places; i += 32) { mine[i].token = -1; mine[i].sum = 0.f; }
        __syncwarp();
      }
      for (int t0 = b; t0 < e; t0 += 32) {
        const int t = t0 + lane;
        const int y = t < e ? targets[t] : -1;
        const bool valid = y >= 0 && y < vocab;
        const float g = valid ? d_logprob[t] : 0.f;
        const uint32_t same = __match_any_sync(0xffffffffu, valid ? y : -1 - lane);
        float sum = 0.f;
        for (int j = 0; j < 32; ++j) {
          const float x = __shfl_sync(0xffffffffu, g, j);
          if (same >> j & 1) sum += x;
        }
        if (!hashed) {
          if (valid) {
            const float v = scale * ((sum - total) - total * expm1f(logprob[t]));
            entry[t] = v;
            if (e - b == 1) one = make_int2(y, __float_as_int(v));
          }
        } else if (valid && lane == __ffs(same) - 1) {
          volatile TokenSum& at = mine[place_of(mine, places, y, true)];   // one lane per token
          at.sum = at.sum + sum;
        }
        __syncwarp();
      }
      if (hashed) {
        __threadfence_block();
        for (int t = b + lane; t < e; t += 32) {
          const int y = targets[t];
          if (y >= 0 && y < vocab)
            entry[t] = scale * ((mine[place_of(mine, places, y, false)].sum - total) - total * expm1f(logprob[t]));
        }
      }
    }
    if (lane == 0) {
      row_info[row] = make_float2(lse[row] * kLog2e, -scale * total);
      only[row] = one;
      if (any) atomicOr(&s_bits, 1u << warp);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) matters[blockIdx.x] = uint8_t(s_bits);
}

// dz at the targets of the rows that have several, over what the product's epilogue has stored: one thread per target.
template <class T>
__global__ void __launch_bounds__(256) patch_kernel(int n_targets, const int32_t* __restrict__ targets, const int32_t* __restrict__ row_at,
                                                    const float* __restrict__ entry, const int32_t* __restrict__ count, int col0, int nv,
                                                    int twice, T* __restrict__ dz, int64_t pitch) {
  previous_kernel_done();
  next_kernel_may_start();
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= n_targets) return;
  const uint32_t x = uint32_t(targets[t]) - uint32_t(col0), row = uint32_t(row_at[t]);
  if (x >= uint32_t(nv) || row >= uint32_t(*count)) return;
  if constexpr (sizeof(T) == 4) {
    dz[int64_t(row) * pitch + x] = entry[t];
  } else {
    dz[int64_t(row) * pitch + x] = dz_part(entry[t], false);
    if (twice) dz[int64_t(row + 128) * pitch + x] = dz_part(entry[t], true);
  }
}

// d_hidden from the parts of its sum, in order.
__global__ void __launch_bounds__(256) sum_kernel(const float4* __restrict__ acc, int splits, int64_t split_vecs, int twice, int pitch_vecs, int vecs,
                                                  const int32_t* __restrict__ count, const int32_t* __restrict__ row_of,
                                                  uint2* __restrict__ d_hidden, int64_t dh_pitch_vecs) {
  previous_kernel_done();
  const int row = blockIdx.x, i = blockIdx.y * 256 + threadIdx.x;
  if (row >= *count || i >= vecs) return;
  acc += int64_t(row) * pitch_vecs + i;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < splits << twice; ++k) {
    const float4 x = acc[(k >> twice) * split_vecs + (k & twice) * int64_t(128) * pitch_vecs];
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  d_hidden[row_of[row] * dh_pitch_vecs + i] = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
}

// Gathers the hidden states of the rows that matter, in order, and zeroes the others' d_hidden.  A warp per row; a block
// counts the rows before its own itself: one bit per row is little to read.
__global__ void __launch_bounds__(kRowsPerByte * 32) gather_kernel(int M, int twice, const uint8_t* __restrict__ matters, const uint4* __restrict__ hidden,
                                                                   int64_t h_pitch_vecs, int vecs, uint4* __restrict__ gathered,
                                                                   int32_t* __restrict__ row_of, int32_t* __restrict__ count,
                                                                   const int32_t* __restrict__ off, int n_targets, int32_t* __restrict__ row_at,
                                                                   uint4* __restrict__ d_hidden, int64_t dh_pitch_vecs) {
  __shared__ int s_before;
  if (threadIdx.x == 0) s_before = 0;
  __syncthreads();
  previous_kernel_done();
  next_kernel_may_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, byte = blockIdx.x;
  int before = 0;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(matters);
  for (int i = threadIdx.x; i <= byte / 4; i += kRowsPerByte * 32)
    before += __popc(words[i] & (i < byte / 4 ? ~0u : (1u << byte % 4 * 8) - 1));
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0 && before) atomicAdd(&s_before, before);
  __syncthreads();
  const uint32_t bits = matters[byte];
  const int at0 = s_before, row = byte * kRowsPerByte + warp;
  if (row < M) {
    const bool mine = bits >> warp & 1;
    const int at = at0 + __popc(bits & ((1u << warp) - 1));
    if (off) {
      // where the targets of a row with several of them are gathered to; -1: nothing for patch_kernel to do
      int b, e;
      target_range(off, row, n_targets, b, e);
      for (int t = b + lane; t < e; t += 32) row_at[t] = mine && e - b > 1 ? at : -1;
    }
    if (mine) {
      if (lane == 0) row_of[at] = row;
#pragma unroll 8
      for (int i = lane; i < vecs; i += 32) {
        const uint4 x = hidden[row * h_pitch_vecs + i];
        gathered[int64_t(at) * vecs + i] = x;
        if (twice) gathered[int64_t(at + 128) * vecs + i] = x;
      }
    } else if (d_hidden) {
      for (int i = lane; i < vecs; i += 32) d_hidden[row * dh_pitch_vecs + i] = make_uint4(0, 0, 0, 0);
    }
  }
  if (blockIdx.x == gridDim.x - 1) {
    const int n = at0 + __popc(bits);
    if (threadIdx.x == 0) *count = n;
    // the rows behind the last one, up to a whole step of the product that sums over rows
    const int64_t end = int64_t((n + kBK - 1) / kBK * kBK) * vecs;
    for (int64_t i = int64_t(n) * vecs + threadIdx.x; i < end; i += kRowsPerByte * 32) {
      gathered[i] = make_uint4(0, 0, 0, 0);
      if (twice) gathered[i + int64_t(128) * vecs] = make_uint4(0, 0, 0, 0);
    }
  }
}

}  // namespace
}  // namespace psrl

#include "logprob_f32.cuh"

namespace psrl {
namespace {

// ------------------------------------------------------------------------------------------------- host side

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Up to kFewRows rows the forward takes few_rows_kernel: 1, 2, 4 rows of 4096 x 131072 weights 164, 176, 185 us, by the
// matrix kernel, whose sums are less exact, 257, 220, 222 (64 rows 205); 8 rows by this kernel were 415 us (fp32 arithmetic).
constexpr int kFewRows = 4;

struct Layout {
  int32_t tile_n, n_tiles, run, n_parts;
  int32_t few;                   // rows that few_rows_kernel is built for, 0: the matrix kernel
  int64_t piece;                 // vocabulary entries of one piece of the backward
  int64_t rows, acc_rows;        // rows that the backward's gathered buffers and the sums of d_hidden hold
  int32_t splits;                // parts of d_hidden's sums
  int32_t twice;                 // dz in two bf16 parts
  size_t part, part_at, row_info, only, entry, table, row_at, matters, row_of, count, gathered, dz, acc, total;
};

// Columns of a tile of the logits.  Wide tiles use the tensor cores and the L2 best; with few tiles the rounds of the 74 pairs
// of CTAs come out uneven, and narrower ones even them (79 tiles of 256 columns take two rounds, so do 105 of 192).
int tile_columns(int64_t m_tiles, int64_t v, int64_t k_blocks, int pairs) {
  if (m_tiles * ((v + 255) / 256) >= 4 * pairs) return 256;
  int best = 256;
  int64_t least = INT64_MAX;
  for (int w = 256; w >= 64; w -= 64) {
    const int64_t tiles = m_tiles * ((v + w - 1) / w), cost = (tiles + pairs - 1) / pairs * (2 * w * k_blocks + 1500);
    if (cost < least) { least = cost; best = w; }
  }
  return best;
}

Layout layout(psrl_dtype_t dtype, int64_t n, int64_t h, int64_t v, int64_t n_targets, bool backward) {
  const bool f32 = dtype == PSRL_F32;
  Layout L{};
  const int64_t m_tiles = (n + 255) / 256;
  // the forward's tiles; the backward's of the logits too while all rows are one tile (how many of them matter is not known here)
  const int pairs = resident_ctas() / 2;
  L.tile_n = !backward || m_tiles == 1 ? tile_columns(m_tiles, v, (h + kBK - 1) / kBK, pairs) : 256;
  L.n_tiles = static_cast<int32_t>((v + L.tile_n - 1) / L.tile_n);
  size_t at = kWsHeaderBytes;
  auto take = [&](size_t bytes) { const size_t a = at; at += (bytes + 255) / 256 * 256; return a; };
  if (!backward && f32) {
    const int64_t blocks = ((n + kF32Tile - 1) / kF32Tile) * ((v + kF32Tile - 1) / kF32Tile);
    L.run = static_cast<int32_t>(std::min<int64_t>(16, std::max<int64_t>(1, blocks / (8 * resident_ctas()))));
    L.n_parts = static_cast<int32_t>((v + int64_t(kF32Tile) * L.run - 1) / (int64_t(kF32Tile) * L.run));
    L.part = take(size_t(L.n_parts) * n * sizeof(float2));
  } else if (!backward) {
    // short runs while there are few tiles (they balance the pairs of CTAs), long ones to keep the partials small
    const int64_t tiles = m_tiles * L.n_tiles;
    L.run = static_cast<int32_t>(std::min<int64_t>(kMaxRun, std::max<int64_t>(1, tiles / (pairs * 16))));
    L.n_parts = (L.n_tiles + L.run - 1) / L.run * kGroups;
    if (n <= kFewRows) {
      for (L.few = 1; L.few < n;) L.few *= 2;
      if (size_t(L.few) * h * 2 > kFewSmem) L.few = 0;
      const int64_t per_block = kFewThreads / 32 * kFewV;
      if (L.few) L.n_parts = static_cast<int32_t>(std::min<int64_t>(few_blocks(L.few) * resident_ctas(), (v + per_block - 1) / per_block));
    }
    L.part = take(size_t(L.n_parts) * n * sizeof(float2));
    if (!L.few) L.part_at = take(size_t(L.n_parts) * n * sizeof(int32_t));
  } else {
    L.twice = !f32 && n <= kTwiceRows;
    L.rows = L.twice ? 256 : round_up(n, kBK);
    L.acc_rows = L.twice ? 256 : round_up(n, 128);
    // a piece of dz is 64 Mi numbers (in bf16 it then partly stays in the L2 for the two products that read it) but at least
    // 8192 entries wide: below that the fp32 sums of d_hidden cost more traffic than the products hide
    const int64_t most_wide = std::max<int64_t>(8192, (int64_t(64) << 20) / L.rows / 256 * 256);
    const int64_t pieces = (v + most_wide - 1) / most_wide;
    L.piece = round_up((v + pieces - 1) / pieces, 256);
    L.row_info = take(size_t(n) * sizeof(float2));
    L.only = take(size_t(n) * sizeof(int2));
    L.entry = take(size_t(n_targets) * sizeof(float));
    L.table = take(2 * size_t(n_targets) * sizeof(TokenSum));
    L.row_at = take(size_t(n_targets) * sizeof(int32_t));
    L.matters = take(size_t(n + 7) / 8 + 3);
    L.row_of = take(size_t(n) * sizeof(int32_t));
    L.count = take(sizeof(int32_t));
    const size_t es = f32 ? 4 : 2;
    L.gathered = take(size_t(L.rows) * h * es);
    L.dz = take(size_t(L.rows) * L.piece * es);
    // Parts of d_hidden's sum: with few rows there are fewer of its tiles than pairs of CTAs, and each is as deep as the
    // piece; two units for every pair, of at least 16 steps, share that out (777 rows, half of them without targets, one unit
    // for every pair 441 us, two 416, four 425: 30 calls after a pause; in long runs the power cap makes the 416 us 466).
    const int64_t tiles = m_tiles * ((h + 255) / 256), most = std::min<int64_t>(16, L.piece / kBK / 16);
    L.splits = tiles >= pairs ? 1 : static_cast<int32_t>(std::max<int64_t>(1, std::min(most, (2 * pairs + tiles - 1) / tiles)));
    if (!f32) L.acc = take(size_t(L.splits) * L.acc_rows * round_up(h, 32) * sizeof(float));
  }
  L.total = at;
  return L;
}

// A kernel of a call; all but the first may start before the one before has ended (see previous_kernel_done).
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream, bool first, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = first ? 0 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

template <Kind kKind>
cudaError_t launch_gemm(const GemmMaps& maps, GemmParams& p, bool first, cudaStream_t stream) {
  static bool done[64] = {};
  cudaError_t e = ensure_dynamic_smem(gemm_kernel<kKind>, gemm_smem(kKind), done);
  if (e != cudaSuccess) return e;
  if (p.tile_n == 0) p.tile_n = 256;
  // even groups of at most kGroupBytes (a row tile is 256 rows of 2 bytes)
  const int64_t row_tiles = std::max<int64_t>(1, (int64_t(p.M) + 255) / 256);
  const int64_t most = std::max<int64_t>(1, kGroupBytes / (int64_t(std::max(p.k_blocks, 1)) * kBK * 512));
  const int64_t groups = (row_tiles + most - 1) / most;
  p.group = int32_t((row_tiles + groups - 1) / groups);
  p.n_tiles = (p.N + p.tile_n - 1) / p.tile_n;
  if (p.run < 1) p.run = 1;
  int64_t units = (int64_t(p.M) + 255) / 256 * ((p.n_tiles + p.run - 1) / p.run);
  if (kKind == kGrad) units = units * p.splits + (int64_t(p.vocab) + 255) / 256 * p.n_tiles;
  if (units > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int clusters = static_cast<int>(std::min<int64_t>(units, resident_ctas() / 2));
  return launch(gemm_kernel<kKind>, dim3(2 * clusters), kGemmThreads, gemm_smem(kKind), stream, first, maps, p);
}

template <int kRows>
cudaError_t launch_few(const Layout& L, int32_t M, int32_t h, int32_t v, const void* hidden, int64_t hp, const void* weight, int64_t wp,
                       float scale, float2* part, int* status, cudaStream_t stream) {
  static bool done[64] = {};
  const size_t smem = size_t(kRows) * h * 2;
  cudaError_t e = ensure_dynamic_smem(few_rows_kernel<kRows>, kFewSmem, done);
  if (e != cudaSuccess) return e;
  return launch(few_rows_kernel<kRows>, dim3(unsigned(L.n_parts)), kFewThreads, smem, stream, true, M, h / 8, v, static_cast<const uint4*>(hidden),
                hp / 8, static_cast<const uint4*>(weight), wp / 8, scale * kLog2e, part, status);
}

// One launch counts 65,535 blocks of rows; further rows take further launches.
template <F32Kind kKind>
cudaError_t launch_f32(F32Params p, int64_t col_blocks, int64_t rows, bool first, cudaStream_t stream) {
  constexpr int64_t kMost = 65535;
  const int64_t row_blocks = (rows + kF32Tile - 1) / kF32Tile;
  if (col_blocks > INT32_MAX) return cudaErrorInvalidValue;
  cudaError_t e = cudaSuccess;
  for (int64_t at = 0; e == cudaSuccess && at < row_blocks; at += kMost) {
    p.row0 = static_cast<int32_t>(at * kF32Tile);
    e = launch(f32_kernel<kKind>, dim3(unsigned(col_blocks), unsigned(std::min(kMost, row_blocks - at))), 256, 0, stream, first && at == 0, p);
  }
  return e;
}

psrl_status_t cuda_failed(cudaError_t e) {
  set_last_cuda_error(e);
  return PSRL_ERR_CUDA;
}

bool al16(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool al4(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
constexpr int64_t kMostEntries = int64_t(1) << 30;   // rows, targets, vocabulary: indices and twice as many stay in 32 bits
// elements of a 16-byte vector
int64_t vec_of(psrl_dtype_t t) { return t == PSRL_BF16 ? 8 : 4; }
bool pitch16(psrl_dtype_t t, int64_t pitch, int64_t cols) { return pitch >= cols && pitch % vec_of(t) == 0 && pitch <= (int64_t(1) << 36); }

// Shared checks of both directions; PSRL_OK with n_rows == 0 means there is nothing to do.
psrl_status_t check(psrl_dtype_t t, int64_t n, int32_t h, int32_t v, const void* hidden, int64_t hp, const void* weight, int64_t wp,
                    const int32_t* targets, int64_t n_targets, const int32_t* off, float scale) {
  if (t != PSRL_BF16 && t != PSRL_F32) return PSRL_ERR_UNSUPPORTED;
  if (n < 0 || n_targets < 0 || n > kMostEntries || n_targets > kMostEntries) return PSRL_ERR_INVALID_ARG;
  if (h < 8 || h % 8 || v < 1 || v > kMostEntries || !pitch16(t, hp, h) || !pitch16(t, wp, h)) return PSRL_ERR_SHAPE;
  if (!off && n_targets != n) return PSRL_ERR_SHAPE;
  if (!(scale == scale) || scale == 0.f || scale > 1e30f || scale < -1e30f) return PSRL_ERR_INVALID_ARG;
  if (n == 0) return PSRL_OK;
  if (!al16(hidden) || !al16(weight) || (n_targets && !al4(targets)) || (off && !al4(off))) return PSRL_ERR_INVALID_ARG;
  return PSRL_OK;
}

}  // namespace
}  // namespace psrl

extern "C" {

size_t psrl_token_logprob_workspace_bytes(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab, int64_t n_targets,
                                          int backward) {
  if (n_rows < 0 || hidden_dim < 1 || vocab < 1 || n_targets < 0) return 0;
  if (n_rows == 0) return psrl::kWsHeaderBytes;
  return psrl::layout(dtype, n_rows, hidden_dim, vocab, n_targets, backward != 0).total;
}

psrl_status_t psrl_token_logprob_fwd(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab, const void* hidden,
                                     int64_t hidden_pitch, const void* weight, int64_t weight_pitch,
                                     const int32_t* targets, int64_t n_targets, const int32_t* target_off, float scale,
                                     float* logprob, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, hidden_dim, vocab, hidden, hidden_pitch, weight, weight_pitch, targets, n_targets, target_off, scale);
  if (st != PSRL_OK) return st;
  if (!ptr_aligned(workspace, 256)) return PSRL_ERR_INVALID_ARG;
  if (workspace_bytes < psrl_token_logprob_workspace_bytes(dtype, n_rows, hidden_dim, vocab, n_targets, 0)) return PSRL_ERR_WORKSPACE;
  if (n_rows && (!al4(lse) || (n_targets && !al4(logprob)))) return PSRL_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (n_rows == 0) {
    e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);   // otherwise the first kernel clears the status
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  const Layout L = layout(dtype, n_rows, hidden_dim, vocab, n_targets, false);
  char* ws = static_cast<char*>(workspace);
  float2* part = reinterpret_cast<float2*>(ws + L.part);
  int32_t* part_at = reinterpret_cast<int32_t*>(ws + L.part_at);
  int* status = reinterpret_cast<int*>(ws);
  const int32_t M = static_cast<int32_t>(n_rows);
  if (dtype == PSRL_F32) {
    e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);
    if (e != cudaSuccess) return cuda_failed(e);
    F32Params p{};
    p.a = static_cast<const float*>(hidden); p.a_pitch = hidden_pitch; p.b = static_cast<const float*>(weight); p.b_pitch = weight_pitch;
    p.M = M; p.N = vocab; p.K = hidden_dim; p.scale_log2 = scale * kLog2e; p.part = part; p.run = L.run;
    e = launch_f32<kF32Lse>(p, L.n_parts, n_rows, true, s);
  } else if (L.few) {
    e = L.few == 1 ? launch_few<1>(L, M, hidden_dim, vocab, hidden, hidden_pitch, weight, weight_pitch, scale, part, status, s)
      : L.few == 2 ? launch_few<2>(L, M, hidden_dim, vocab, hidden, hidden_pitch, weight, weight_pitch, scale, part, status, s)
                   : launch_few<4>(L, M, hidden_dim, vocab, hidden, hidden_pitch, weight, weight_pitch, scale, part, status, s);
  } else {
    GemmMaps maps;
    if (!make_map_bf16_2d(&maps.a, hidden, hidden_dim, n_rows, hidden_pitch * 2, 128) ||
        !make_map_bf16_2d(&maps.b, weight, hidden_dim, vocab, weight_pitch * 2, L.tile_n / 2))
      return PSRL_ERR_CUDA;
    GemmParams p{};
    p.M = M;
    p.N = vocab;
    p.k_blocks = (hidden_dim + kBK - 1) / kBK;
    p.tile_n = L.tile_n;
    p.run = L.run;
    p.scale_log2 = scale * kLog2e;
    p.part = part;
    p.part_at = part_at;
    p.status = status;
    // where depth and rows are such that the pairs' operands fill the L2, and over several rounds of tiles (see keep_pace)
    const bool paced = hidden_dim >= kPaceDepth && n_rows >= kPaceRows && (n_rows + 255) / 256 * ((vocab + 255) / 256) >= 4 * (resident_ctas() / 2);
    if (paced) {
      e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);
      if (e != cudaSuccess) return cuda_failed(e);
      p.pace = reinterpret_cast<uint32_t*>(ws + kPaceAt);
      p.pace_shift = p.k_blocks > 64 ? 3 : 4;
    }
    e = launch_gemm<kLse>(maps, p, true, s);
  }
  if (e != cudaSuccess) return cuda_failed(e);
  // rows of a block: 32 read the partials in whole lines; with few rows more threads to each of them finish sooner
  const int rows = M >= 4096 ? 32 : M >= 256 ? 4 : 1;
  const dim3 grid(unsigned((M + rows - 1) / rows));
  if (dtype == PSRL_F32) {
    auto final = rows == 32 ? final_kernel<32, float> : rows == 4 ? final_kernel<4, float> : final_kernel<1, float>;
    e = launch(final, grid, kFinalThreads, 0, s, false, part, nullptr, L.n_parts, M, hidden_dim, vocab, static_cast<const float*>(hidden),
               hidden_pitch, static_cast<const float*>(weight), weight_pitch, targets, target_off, static_cast<int>(n_targets), scale,
               logprob, lse);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  using Bf = __nv_bfloat16;
  auto final = rows == 32 ? final_kernel<32, Bf> : rows == 4 ? final_kernel<4, Bf> : final_kernel<1, Bf>;
  e = launch(final, grid, kFinalThreads, 0, s, false, part, L.few ? nullptr : part_at, L.n_parts, M, hidden_dim, vocab,
             static_cast<const __nv_bfloat16*>(hidden), hidden_pitch, static_cast<const __nv_bfloat16*>(weight), weight_pitch, targets,
             target_off, static_cast<int>(n_targets), scale, logprob, lse);
  return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
}

psrl_status_t psrl_token_logprob_bwd(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab, const void* hidden,
                                     int64_t hidden_pitch, const void* weight, int64_t weight_pitch,
                                     const int32_t* targets, int64_t n_targets, const int32_t* target_off, float scale,
                                     const float* logprob, const float* lse, const float* d_logprob, void* d_hidden,
                                     int64_t d_hidden_pitch, void* d_weight, int64_t d_weight_pitch, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  using namespace psrl;
  psrl_status_t st = check(dtype, n_rows, hidden_dim, vocab, hidden, hidden_pitch, weight, weight_pitch, targets, n_targets, target_off, scale);
  if (st != PSRL_OK) return st;
  if (!ptr_aligned(workspace, 256) || (d_hidden && !al16(d_hidden)) || (d_weight && !al16(d_weight))) return PSRL_ERR_INVALID_ARG;
  if ((d_hidden && !pitch16(dtype, d_hidden_pitch, hidden_dim)) || (d_weight && !pitch16(dtype, d_weight_pitch, hidden_dim))) return PSRL_ERR_SHAPE;
  if (workspace_bytes < psrl_token_logprob_workspace_bytes(dtype, n_rows, hidden_dim, vocab, n_targets, 1)) return PSRL_ERR_WORKSPACE;
  if (n_rows && (!al4(lse) || (n_targets && (!al4(logprob) || !al4(d_logprob))))) return PSRL_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (n_rows == 0 || (!d_hidden && !d_weight)) e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);   // otherwise the first kernel clears the status
  if (e != cudaSuccess) return cuda_failed(e);
  const size_t es = dtype == PSRL_F32 ? 4 : 2;
  const int64_t vec = vec_of(dtype);
  if (n_rows == 0) {
    if (d_weight) e = cudaMemset2DAsync(d_weight, size_t(d_weight_pitch) * es, 0, size_t(hidden_dim) * es, vocab, s);
    return e == cudaSuccess ? PSRL_OK : cuda_failed(e);
  }
  if (!d_hidden && !d_weight) return PSRL_OK;
  const Layout L = layout(dtype, n_rows, hidden_dim, vocab, n_targets, true);
  char* ws = static_cast<char*>(workspace);
  GemmParams base{};
  base.status = reinterpret_cast<int*>(ws);
  base.scale_log2 = scale * kLog2e;
  base.twice = L.twice;
  float2* row_info = reinterpret_cast<float2*>(ws + L.row_info);
  int2* only = reinterpret_cast<int2*>(ws + L.only);
  float* entry = reinterpret_cast<float*>(ws + L.entry);
  int32_t* row_at = reinterpret_cast<int32_t*>(ws + L.row_at);
  __nv_bfloat16* dz = reinterpret_cast<__nv_bfloat16*>(ws + L.dz);
  float* acc = reinterpret_cast<float*>(ws + L.acc);
  const int64_t acc_pitch = round_up(hidden_dim, 32);
  const int32_t M = static_cast<int32_t>(n_rows);
  e = launch(rows_kernel, dim3(unsigned((n_rows + kRowsPerByte - 1) / kRowsPerByte)), kRowsPerByte * 32, 0, s, true, M, vocab, targets,
             target_off, static_cast<int>(n_targets), logprob, lse, d_logprob, scale, row_info, only, entry,
             reinterpret_cast<TokenSum*>(ws + L.table), reinterpret_cast<uint8_t*>(ws + L.matters), base.status);
  if (e != cudaSuccess) return cuda_failed(e);
  __nv_bfloat16* gathered = reinterpret_cast<__nv_bfloat16*>(ws + L.gathered);
  base.count = reinterpret_cast<int32_t*>(ws + L.count);
  base.row_of = reinterpret_cast<int32_t*>(ws + L.row_of);
  e = launch(gather_kernel, dim3(unsigned((n_rows + kRowsPerByte - 1) / kRowsPerByte)), kRowsPerByte * 32, 0, s, false, M, L.twice,
             reinterpret_cast<uint8_t*>(ws + L.matters), static_cast<const uint4*>(hidden), hidden_pitch / vec, static_cast<int>(hidden_dim / vec),
             reinterpret_cast<uint4*>(gathered), reinterpret_cast<int32_t*>(ws + L.row_of), reinterpret_cast<int32_t*>(ws + L.count),
             target_off, static_cast<int>(n_targets), row_at, static_cast<uint4*>(d_hidden), d_hidden_pitch / vec);
  if (e != cudaSuccess) return cuda_failed(e);
  if (dtype == PSRL_F32) {
    const float *hf = reinterpret_cast<const float*>(ws + L.gathered), *wf = static_cast<const float*>(weight);
    float* zf = reinterpret_cast<float*>(ws + L.dz);
    for (int64_t v0 = 0; v0 < vocab; v0 += L.piece) {
      const int32_t nv = static_cast<int32_t>(std::min<int64_t>(L.piece, vocab - v0));
      F32Params p{};
      p.count = base.count; p.row_of = base.row_of; p.scale_log2 = base.scale_log2; p.row_info = row_info; p.only = only;
      p.col0 = static_cast<int32_t>(v0); p.first = v0 == 0;
      F32Params z = p;
      z.a = hf; z.a_pitch = hidden_dim; z.b = wf + v0 * weight_pitch; z.b_pitch = weight_pitch;
      z.M = M; z.N = nv; z.K = hidden_dim; z.out = zf; z.out_pitch = L.piece;
      e = launch_f32<kF32Dz>(z, (nv + kF32Tile - 1) / kF32Tile, n_rows, false, s);
      if (e == cudaSuccess && target_off && n_targets)
        e = launch(patch_kernel<float>, dim3(unsigned((n_targets + 255) / 256)), 256, 0, s, false, static_cast<int>(n_targets), targets, row_at,
                   entry, base.count, p.col0, static_cast<int>(nv), 0, zf, L.piece);
      if (e == cudaSuccess && d_hidden) {
        F32Params g = p;
        g.a = zf; g.a_pitch = L.piece; g.b = wf + v0 * weight_pitch; g.b_pitch = weight_pitch;
        g.M = M; g.N = hidden_dim; g.K = nv; g.out = static_cast<float*>(d_hidden); g.out_pitch = d_hidden_pitch;
        e = launch_f32<kF32Dh>(g, (hidden_dim + kF32Tile - 1) / kF32Tile, n_rows, false, s);
      }
      if (e == cudaSuccess && d_weight) {
        F32Params g = p;
        g.a = zf; g.a_pitch = L.piece; g.b = hf; g.b_pitch = hidden_dim;
        g.M = nv; g.N = hidden_dim; g.out = static_cast<float*>(d_weight) + v0 * d_weight_pitch; g.out_pitch = d_weight_pitch;
        e = launch_f32<kF32Dw>(g, (hidden_dim + kF32Tile - 1) / kF32Tile, nv, false, s);
      }
      if (e != cudaSuccess) return cuda_failed(e);
    }
    return PSRL_OK;
  }
  const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(weight);
  for (int64_t v0 = 0; v0 < vocab; v0 += L.piece) {
    const int64_t nv = std::min<int64_t>(L.piece, vocab - v0);
    const __nv_bfloat16* wv = w + v0 * weight_pitch;
    GemmMaps mz, mg;
    if (!make_map_bf16_2d(&mz.a, gathered, hidden_dim, L.rows, int64_t(hidden_dim) * 2, 128) ||
        !make_map_bf16_2d(&mz.b, wv, hidden_dim, nv, weight_pitch * 2, L.tile_n / 2) ||
        !make_map_bf16_2d(&mg.a, dz, nv, L.rows, L.piece * 2, 128) ||
        !make_map_bf16_2d(&mg.b, wv, hidden_dim, nv, weight_pitch * 2, 64) ||
        !make_map_bf16_2d(&mg.a2, dz, nv, L.rows, L.piece * 2, 64) ||
        !make_map_bf16_2d(&mg.b2, gathered, hidden_dim, L.rows, int64_t(hidden_dim) * 2, 64) ||
        !make_map_bf16_2d(&mz.out, dz, nv, L.rows, L.piece * 2, 128) ||
        !make_map_f32_2d(&mg.out, acc, hidden_dim, L.splits * L.acc_rows, acc_pitch * 4, 128) ||
        (d_weight && !make_map_bf16_2d(&mg.out2, static_cast<__nv_bfloat16*>(d_weight) + v0 * d_weight_pitch, hidden_dim, nv,
                                       d_weight_pitch * 2, 128)))
      return PSRL_ERR_CUDA;
    GemmParams z = base;
    z.M = M; z.N = static_cast<int32_t>(nv); z.k_blocks = (hidden_dim + kBK - 1) / kBK;
    z.row_info = row_info; z.only = only; z.col0 = static_cast<int32_t>(v0);
    z.tile_n = L.tile_n;
    e = launch_gemm<kDz>(mz, z, false, s);
    if (e != cudaSuccess) return cuda_failed(e);
    if (target_off && n_targets) {
      e = launch(patch_kernel<__nv_bfloat16>, dim3(unsigned((n_targets + 255) / 256)), 256, 0, s, false, static_cast<int>(n_targets), targets, row_at, entry,
                 base.count, z.col0, static_cast<int>(nv), L.twice, dz, L.piece);
      if (e != cudaSuccess) return cuda_failed(e);
    }
    GemmParams g = base;
    g.M = M; g.N = hidden_dim; g.vocab = static_cast<int32_t>(nv);
    g.want_hidden = d_hidden != nullptr; g.want_weight = d_weight != nullptr;
    g.splits = L.splits;
    g.acc_rows = static_cast<int32_t>(L.acc_rows);
    g.first = v0 == 0;
    e = launch_gemm<kGrad>(mg, g, false, s);
    if (e != cudaSuccess) return cuda_failed(e);
  }
  if (d_hidden) {
    e = launch(sum_kernel, dim3(unsigned(n_rows), unsigned((hidden_dim / 4 + 255) / 256)), 256, 0, s, false, reinterpret_cast<const float4*>(acc),
               L.splits, L.acc_rows * acc_pitch / 4, L.twice, static_cast<int>(acc_pitch / 4), hidden_dim / 4, base.count, base.row_of,
               static_cast<uint2*>(d_hidden), d_hidden_pitch / 4);
    if (e != cudaSuccess) return cuda_failed(e);
  }
  return PSRL_OK;
}

}  // extern "C"
