// Copying and compacting blocks of the paged K/V pools: the data movement behind the cache manager's decisions
// (paper Sec. 5.2: blocks are evicted, restored and released as micro-batches come and go).
//
// psrl_kv_copy moves extents between pools that do not overlap.  psrl_kv_move slides extents down inside a pool, where
// an extent's destination may overlap its own source or an earlier extent's: a memmove over a whole arena in one pass.
//
// Both are bound by HBM (every byte read once, written once).  The extent list is host data and travels in the kernel's
// parameters, so a call needs no device copy of it, may be captured into a graph, and leaves nothing behind.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/psrl_cache.h"
#include "kernels.h"
#include "move_order.h"
#include "sm100.cuh"

namespace psrl {
namespace {

struct Pools {
  const uint4 *k_src, *v_src;
  uint4 *k_dst, *v_dst;
  int64_t src_cap, dst_cap;
  int32_t heads;
  int32_t vecs;  // 16-byte vectors per slot and head
};

// ------------------------------------------------------------------------------------------------ disjoint copies

constexpr int kShortList = 64, kLongList = 1000;   // extents that travel in a launch's parameters
constexpr int kCopyThreads = 256, kCopyPiece = 1024;  // vectors of one block: 16 KB, four per thread

template <int kMax>
struct CopyList {
  int32_t n;
  int32_t piece_slots;
  int32_t src[kMax], dst[kMax], slots[kMax];
  int32_t first_piece[kMax + 1];
};

template <int kMax>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyList<kMax> list, const Pools p) {
  const int piece = blockIdx.x, head = blockIdx.y;
  int lo = 0, hi = list.n;  // the last extent whose first piece is <= piece
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list.first_piece[mid] <= piece) lo = mid; else hi = mid;
  }
  const int at = (piece - list.first_piece[lo]) * list.piece_slots;
  const int n = min(list.piece_slots, list.slots[lo] - at) * p.vecs;
  const uint4* src = blockIdx.z ? p.v_src : p.k_src;
  uint4* dst = blockIdx.z ? p.v_dst : p.k_dst;
  if (!src) return;
  src += (int64_t(head) * p.src_cap + list.src[lo] + at) * p.vecs;
  dst += (int64_t(head) * p.dst_cap + list.dst[lo] + at) * p.vecs;
  uint4 r[kCopyPiece / kCopyThreads];
#pragma unroll
  for (int i = 0; i < kCopyPiece / kCopyThreads; ++i)
    if (threadIdx.x + i * kCopyThreads < n) r[i] = src[threadIdx.x + i * kCopyThreads];
#pragma unroll
  for (int i = 0; i < kCopyPiece / kCopyThreads; ++i)
    if (threadIdx.x + i * kCopyThreads < n) dst[threadIdx.x + i * kCopyThreads] = r[i];
}

template <int kMax>
psrl_status_t launch_copies(const psrl_kv_extent_t* ext, int32_t n, const Pools& p, cudaStream_t stream) {
  CopyList<kMax> list;
  list.piece_slots = std::max(1, kCopyPiece / p.vecs);
  for (int32_t at = 0; at < n; at += kMax) {
    list.n = std::min(kMax, n - at);
    int64_t pieces = 0;
    for (int32_t i = 0; i < list.n; ++i) {
      const psrl_kv_extent_t& e = ext[at + i];
      list.src[i] = e.src_slot; list.dst[i] = e.dst_slot; list.slots[i] = e.n_slots;
      list.first_piece[i] = static_cast<int32_t>(pieces);
      pieces += (int64_t(e.n_slots) + list.piece_slots - 1) / list.piece_slots;
      if (pieces > INT32_MAX) return PSRL_ERR_SHAPE;
    }
    list.first_piece[list.n] = static_cast<int32_t>(pieces);
    copy_kernel<kMax><<<dim3(unsigned(pieces), unsigned(p.heads), 2), kCopyThreads, 0, stream>>>(list, p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_last_cuda_error(e); return PSRL_ERR_CUDA; }
  }
  return PSRL_OK;
}

psrl_status_t copy_extents(const psrl_kv_extent_t* ext, int32_t n, const Pools& p, cudaStream_t stream) {
  // a short list costs a launch less parameter traffic
  return n <= kShortList ? launch_copies<kShortList>(ext, n, p, stream) : launch_copies<kLongList>(ext, n, p, stream);
}

// ------------------------------------------------------------------------------------------------ moves in place
//
// The slots of all extents, in ascending order, of every (pool, head) are one long sequence of 16-byte vectors, cut into
// chunks of one load per thread slot of the whole grid.  Vectors only move down, and a chunk's sources lie above every
// destination of the chunks before it, so
//   - a chunk may be loaded while earlier chunks are still being stored, and
//   - a chunk may be stored once it and the chunks before it have been loaded by EVERY block,
// which is the only synchronisation.
//   large moves   one block per SM (cooperative launch, all resident).  The sequence is cut into 64 KB parts, handed out
//                 in order; a warp takes a part, loads it into its own share of shared memory with bulk copies, counts it
//                 as loaded, waits until the parts whose sources it overwrites are, and stores it.  Every part handed out
//                 gets loaded whatever the others do, and the parts waited for are no later ones, so the waits end
//                 (move_order.h has the arithmetic and why the counts of 32 groups are enough).
//                 169,632 slots of 4 KB:
//                 239 us, 5.8 TB/s; the same copied to other pools, where nothing waits, 209 us.  (Chunks of the whole
//                 grid, stored once every block had loaded its share of them, took 270 us in registers and 296 us through
//                 six stages of shared memory: all blocks ran at the pace of the slowest.)
//   small moves   one cluster of up to eight blocks and its hardware barrier: an ordinary launch, nothing to zero first;
//                 a chunk is one load per thread slot, the next one in flight while a block waits

constexpr int kMoveThreads = 512, kMoveRegs = 8;           // small moves: 64 KB per block and chunk
constexpr int kWarpVecs = 32 * kMoveRegs;                  // a warp's part of a chunk: 4 KB of consecutive vectors
constexpr int kClusterMax = 8;

template <int kMax>
struct MoveList {
  int32_t n;
  int32_t slots;              // sum of the extents
  int32_t src[kMax], dst[kMax];
  int32_t first[kMax + 1];    // slots before the extent
};

// A warp's part of a chunk: its vectors, and in lane i where its row i (slot of one pool and head) goes.
struct Held {
  uint4 v[kMoveRegs];
  int64_t dst_at;   // in vectors from the pool's start, -1 past the end
  int32_t pool;
};

template <class List>
__device__ __forceinline__ void load_part(const List& list, const Pools& p, uint32_t warp_part, uint32_t total_rows, Held& h) {
  const int lane = threadIdx.x & 31;
  const uint32_t rows = kWarpVecs / p.vecs;
  const uint64_t row0 = uint64_t(warp_part) * rows;
  int64_t src_at = -1;
  h.dst_at = -1;
  h.pool = 0;
  if (lane < int(rows) && row0 + lane < total_rows) {
    const uint32_t row = uint32_t(row0) + lane;
    const uint32_t ph = row / uint32_t(list.slots);
    const int s = int(row - ph * uint32_t(list.slots));
    h.pool = ph >= uint32_t(p.heads);
    const int head = int(ph) - h.pool * p.heads;
    int lo = 0, hi = list.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (list.first[mid] <= s) lo = mid; else hi = mid;
    }
    const int in = s - list.first[lo];
    src_at = (int64_t(head) * p.src_cap + list.src[lo] + in) * p.vecs;
    h.dst_at = (int64_t(head) * p.src_cap + list.dst[lo] + in) * p.vecs;
  }
  const int shift = 31 - __clz(p.vecs);
#pragma unroll
  for (int j = 0; j < kMoveRegs; ++j) {
    const int vec = j * 32 + lane, r = vec >> shift, x = vec & (p.vecs - 1);
    const int64_t at = __shfl_sync(0xffffffffu, src_at, r);
    const int z = __shfl_sync(0xffffffffu, h.pool, r);
    h.v[j] = make_uint4(0, 0, 0, 0);
    if (at >= 0) h.v[j] = __ldcg((z ? p.v_src : p.k_src) + at + x);
  }
}

// True once every thread of the block HOLDS its loads: the barrier's predicate is computed from their values, so no later
// store, of this or another block, can be seen by them.  (A fence would order them too, but also wait for the stores of
// the chunk before.)
__device__ __forceinline__ void settle(const Held& h) {
  uint32_t x = 0;
#pragma unroll
  for (int j = 0; j < kMoveRegs; ++j) x |= h.v[j].x ^ h.v[j].y ^ h.v[j].z ^ h.v[j].w;
  __syncthreads_or(x != 0);
}

__device__ __forceinline__ void store_part(const Pools& p, const Held& h) {
  const int lane = threadIdx.x & 31;
  const int shift = 31 - __clz(p.vecs);
#pragma unroll
  for (int j = 0; j < kMoveRegs; ++j) {
    const int vec = j * 32 + lane, r = vec >> shift, x = vec & (p.vecs - 1);
    const int64_t at = __shfl_sync(0xffffffffu, h.dst_at, r);
    const int z = __shfl_sync(0xffffffffu, h.pool, r);
    if (at >= 0) (z ? p.v_dst : p.k_dst)[at + x] = h.v[j];
  }
}

template <int kMax>
__global__ void __launch_bounds__(kMoveThreads, 1) move_cluster_kernel(const __grid_constant__ MoveList<kMax> list, const Pools p,
                                                                       int* ws, uint32_t n_chunks, uint32_t total_rows, bool first) {
  const uint32_t warps = gridDim.x * (kMoveThreads / 32);
  const uint32_t mine = blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5);
  Held h[2];
  load_part(list, p, mine, total_rows, h[0]);
  if (first && blockIdx.x == 0 && threadIdx.x == 0) ws[0] = int(PSRL_OK);
  auto step = [&](uint32_t c, Held& now, Held& next) {
    settle(now);
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    if (c + 1 < n_chunks) load_part(list, p, (c + 1) * warps + mine, total_rows, next);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    store_part(p, now);
  };
  for (uint32_t c = 0; c < n_chunks; c += 2) {
    step(c, h[0], h[1]);
    if (c + 1 < n_chunks) step(c + 1, h[1], h[0]);
  }
}

// Three warps with 64 KB each; twelve with 16 KB take 328 us instead of 239: the counters, one line of the L2, bound them.
constexpr int kBulkWarps = 3, kBulkBytes = 64 * 1024, kBulkLanes = 8;   // a lane's share of a part: 8 KB
constexpr size_t kBulkSmem = size_t(kBulkWarps) * kBulkBytes;

// The contiguous pieces of rows [row, end) of the sequence: calls f(pool, first source vector, first destination vector,
// rows, rows before).
template <class List, class F>
__device__ __forceinline__ void for_pieces(const List& list, const Pools& p, uint32_t row, uint32_t end, F f) {
  if (row >= end) return;
  uint32_t ph = row / uint32_t(list.slots);
  int s = int(row - ph * uint32_t(list.slots));
  int lo = extent_of(list.first, list.n, s);
  uint32_t done = 0;
  while (row < end) {
    const int in = s - list.first[lo];
    const uint32_t n = min(end - row, uint32_t(list.first[lo + 1] - s));
    const int pool = ph >= uint32_t(p.heads), head = int(ph) - pool * p.heads;
    const int64_t base = int64_t(head) * p.src_cap + in;
    f(pool, (base + list.src[lo]) * p.vecs, (base + list.dst[lo]) * p.vecs, n, done);
    row += n;
    done += n;
    s += int(n);
    if (++lo == list.n) { lo = 0; s = 0; ++ph; }
  }
}

// ws[0] status, ws[8] the next part, ws[16 + g % kRing] parts of group g that have been loaded (never reset)
template <int kMax>
__global__ void __launch_bounds__(kBulkWarps * 32, 1) move_bulk_kernel(const __grid_constant__ MoveList<kMax> list, const Pools p, int* ws,
                                                                       uint32_t n_parts, uint32_t total_rows) {
  extern __shared__ __align__(128) uint8_t part_mem[];
  __shared__ uint64_t landed[kBulkWarps];
  __shared__ int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t row_bytes = uint32_t(p.vecs) * 16, part_rows = kBulkBytes / row_bytes, lane_rows = part_rows / kBulkLanes;
  uint8_t* mine = part_mem + warp * kBulkBytes + lane * lane_rows * row_bytes;
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kBulkWarps; ++i) sm100::mbar_init(&landed[i], 1);
    sm100::fence_mbar_init();
  }
  __syncthreads();
  volatile int* abortp = &s_abort;
  uint32_t phase = 0, next_group = 0;   // groups below next_group are known to be loaded
  while (true) {
    uint32_t part = 0;
    if (lane == 0) part = uint32_t(atomicAdd(ws + 8, 1));
    part = __shfl_sync(0xffffffffu, part, 0);
    if (part >= n_parts) break;
    const uint32_t begin = part * part_rows, end = min(begin + part_rows, total_rows);
    const uint32_t my_row = lane < kBulkLanes ? min(begin + lane * lane_rows, end) : end;
    if (lane == 0) sm100::mbar_expect_tx(&landed[warp], (end - begin) * row_bytes);
    __syncwarp();
    for_pieces(list, p, my_row, min(my_row + lane_rows, end), [&](int pool, int64_t src, int64_t, uint32_t n, uint32_t done) {
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                       sm100::smem_u32(mine + done * row_bytes)),
                   "l"((pool ? p.v_src : p.k_src) + src), "r"(n * row_bytes), "r"(sm100::smem_u32(&landed[warp]))
                   : "memory");
    });
    if (!__all_sync(0xffffffffu, sm100::mbar_wait(&landed[warp], phase, abortp, ws))) break;
    phase ^= 1;
    const uint32_t group = part / kGroup, until = wait_until(list, part, end, part_rows);
    // The copies have landed: nothing reads this part's sources any more.  Their values are here, so no store that follows can
    // change them, and the count needs no release (which waits for the part before to be stored as well: 270 us, not 238).
    if (lane == 0) asm volatile("red.relaxed.gpu.global.add.s32 [%0], 1;" ::"l"(ws + 16 + group % kRing) : "memory");
    const uint32_t g = poll_from(next_group, group) + lane;
    const int want = int(full_count(g, n_parts));
    bool ok = false;
    for (uint32_t it = 0; it < (1u << 22) && !ok; ++it) {
      int seen = want;
      if (g <= until) asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(ws + 16 + g % kRing) : "memory");
      ok = __all_sync(0xffffffffu, seen >= want);
      if (it > 4096) __nanosleep(64);
      if (__any_sync(0xffffffffu, *abortp)) break;
    }
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) {
      if (lane == 0) { s_abort = 1; atomicExch(ws, int(PSRL_ERR_TIMEOUT)); }
      break;
    }
    next_group = max(next_group, until + 1);
    __syncwarp();   // what any lane has seen loaded orders every lane's stores
    asm volatile("fence.proxy.async;" ::: "memory");
    for_pieces(list, p, my_row, min(my_row + lane_rows, end), [&](int pool, int64_t, int64_t dst, uint32_t n, uint32_t done) {
      asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"((pool ? p.v_dst : p.k_dst) + dst),
                   "r"(sm100::smem_u32(mine + done * row_bytes)), "r"(n * row_bytes)
                   : "memory");
    });
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // the stores themselves may still be on their way
    __syncwarp();
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncthreads();
  if (s_abort)
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // copies in flight come to rest before the block's memory is given back
}

template <int kMax>
psrl_status_t move_extents(const psrl_kv_extent_t* ext, int32_t n, Pools p, int* ws, bool first, cudaStream_t stream) {
  MoveList<kMax> list;
  list.n = n;
  int64_t slots = 0;
  for (int32_t i = 0; i < n; ++i) {
    list.src[i] = ext[i].src_slot; list.dst[i] = ext[i].dst_slot; list.first[i] = static_cast<int32_t>(slots);
    slots += ext[i].n_slots;
  }
  list.first[n] = static_cast<int32_t>(slots);
  list.slots = static_cast<int32_t>(slots);
  if (!p.k_src) { p.k_src = p.v_src; p.k_dst = p.v_dst; p.v_src = nullptr; }
  const int64_t rows = slots * p.heads * (p.v_src ? 2 : 1);
  if (rows > INT32_MAX) return PSRL_ERR_SHAPE;
  uint32_t total = static_cast<uint32_t>(rows);
  cudaLaunchConfig_t cfg{};
  cfg.stream = stream;
  cudaLaunchAttribute attr{};
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaSuccess;
  // A cluster moves 0.5 MB a chunk; past kClusterChunks of them the whole GPU is quicker in spite of its dearer launch.
  constexpr int64_t kClusterChunks = 4;
  const int64_t block_rows = int64_t(kMoveThreads) * kMoveRegs / p.vecs, blocks = (rows + block_rows - 1) / block_rows;
  if (blocks <= kClusterMax * kClusterChunks) {
    unsigned grid = 1;
    while (grid < std::min<int64_t>(blocks, kClusterMax)) grid *= 2;
    const uint32_t n_chunks = static_cast<uint32_t>((blocks + grid - 1) / grid);
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kMoveThreads);
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = grid;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    e = cudaLaunchKernelEx(&cfg, move_cluster_kernel<kMax>, list, p, ws, n_chunks, total, first);
  } else {
    static bool done[64] = {};
    e = ensure_dynamic_smem(move_bulk_kernel<kMax>, kBulkSmem, done);
    const int64_t part_rows = kBulkBytes / (int64_t(p.vecs) * 16), parts = (rows + part_rows - 1) / part_rows;
    const int64_t grid = std::min<int64_t>(std::min(resident_ctas(), int(kSpan * kGroup / kBulkWarps)), (parts + kBulkWarps - 1) / kBulkWarps);
    // a group has to be at work as a whole: a device with fewer warps than that would wait for parts that nobody has taken
    if (grid * kBulkWarps < std::min<int64_t>(int64_t(kGroup), parts)) return PSRL_ERR_UNSUPPORTED;
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(kBulkWarps * 32);
    cfg.dynamicSmemBytes = kBulkSmem;
    attr.id = cudaLaunchAttributeCooperative;
    attr.val.cooperative = 1;
    // a later part of a long list keeps the status of the parts before
    const size_t keep = first ? 0 : 8 * sizeof(int);
    if (e == cudaSuccess) e = cudaMemsetAsync(reinterpret_cast<char*>(ws) + keep, 0, kWsHeaderBytes - keep, stream);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, move_bulk_kernel<kMax>, list, p, ws, static_cast<uint32_t>(parts), total);
  }
  if (e != cudaSuccess) { set_last_cuda_error(e); return PSRL_ERR_CUDA; }
  return PSRL_OK;
}

// ------------------------------------------------------------------------------------------------ argument checks

bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool in_range(const psrl_kv_extent_t& e, int64_t src_cap, int64_t dst_cap) {
  return e.n_slots >= 0 && e.src_slot >= 0 && e.dst_slot >= 0 && int64_t(e.src_slot) + e.n_slots <= src_cap &&
         int64_t(e.dst_slot) + e.n_slots <= dst_cap;
}

bool row_ok(int32_t row_bytes) { return row_bytes == 128 || row_bytes == 256 || row_bytes == 512; }

// bytes of the two tensors overlap
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + uintptr_t(b_bytes) && y < x + uintptr_t(a_bytes);
}

struct Range {
  int64_t at, end;
};
bool disjoint(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.at < b.at; });
  for (size_t i = 1; i < r.size(); ++i)
    if (r[i].at < r[i - 1].end) return false;
  return true;
}

}  // namespace
}  // namespace psrl

extern "C" {

psrl_status_t psrl_kv_copy(const psrl_kv_extent_t* extents, int32_t n_extents, int32_t n_kv_heads, int32_t row_bytes,
                           const void* k_src, const void* v_src, int64_t src_capacity, void* k_dst, void* v_dst,
                           int64_t dst_capacity, void* stream) {
  using namespace psrl;
  if (n_extents < 0 || (n_extents && !extents) || (k_src && !k_dst) || (v_src && !v_dst) || !ok16(k_src) ||
      !ok16(v_src) || !ok16(k_dst) || !ok16(v_dst))
    return PSRL_ERR_INVALID_ARG;
  if (n_kv_heads < 1 || n_kv_heads > 65535 || !row_ok(row_bytes) || src_capacity < 0 || dst_capacity < 0 ||
      src_capacity > INT32_MAX || dst_capacity > INT32_MAX)
    return PSRL_ERR_SHAPE;
  const int64_t src_bytes = src_capacity * n_kv_heads * row_bytes, dst_bytes = dst_capacity * n_kv_heads * row_bytes;
  if (!k_src) k_dst = nullptr;
  if (!v_src) v_dst = nullptr;
  // a pool copied onto itself is fine as long as no extent is written that another (or itself) reads
  const bool same = (k_src && k_src == k_dst) || (v_src && v_src == v_dst);
  if ((k_src != k_dst && overlap(k_src, src_bytes, k_dst, dst_bytes)) ||
      (v_src != v_dst && overlap(v_src, src_bytes, v_dst, dst_bytes)) || overlap(k_src, src_bytes, v_dst, dst_bytes) ||
      overlap(v_src, src_bytes, k_dst, dst_bytes) || overlap(k_dst, dst_bytes, v_dst, dst_bytes) ||
      (same && src_capacity != dst_capacity))
    return PSRL_ERR_INVALID_ARG;
  try {
    std::vector<psrl_kv_extent_t> list;
    std::vector<Range> written, all;
    list.reserve(n_extents);
    for (int32_t i = 0; i < n_extents; ++i) {
      const psrl_kv_extent_t& e = extents[i];
      if (!in_range(e, src_capacity, dst_capacity)) return PSRL_ERR_SHAPE;
      if (e.n_slots == 0) continue;
      list.push_back(e);
      written.push_back({e.dst_slot, int64_t(e.dst_slot) + e.n_slots});
    }
    if (!disjoint(written)) return PSRL_ERR_INVALID_ARG;
    if (same) {
      for (const psrl_kv_extent_t& e : list) {
        // written ranges are sorted and disjoint: the first one that ends behind the source's start decides
        auto it = std::lower_bound(written.begin(), written.end(), int64_t(e.src_slot),
                                   [](const Range& r, int64_t at) { return r.end <= at; });
        if (it != written.end() && it->at < int64_t(e.src_slot) + e.n_slots) return PSRL_ERR_INVALID_ARG;
      }
    }
    if (list.empty() || (!k_src && !v_src)) return PSRL_OK;
    const Pools p{static_cast<const uint4*>(k_src), static_cast<const uint4*>(v_src), static_cast<uint4*>(k_dst),
                  static_cast<uint4*>(v_dst), src_capacity, dst_capacity, n_kv_heads, row_bytes / 16};
    return copy_extents(list.data(), static_cast<int32_t>(list.size()), p, static_cast<cudaStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return PSRL_ERR_HOST_OOM;
  }
}

psrl_status_t psrl_kv_move(const psrl_kv_extent_t* extents, int32_t n_extents, int32_t n_kv_heads, int32_t row_bytes,
                           void* k_pool, void* v_pool, int64_t pool_capacity, void* workspace, size_t workspace_bytes,
                           void* stream) {
  using namespace psrl;
  if (n_extents < 0 || (n_extents && !extents) || !ok16(k_pool) || !ok16(v_pool) || !ptr_aligned(workspace, 256))
    return PSRL_ERR_INVALID_ARG;
  if (n_kv_heads < 1 || n_kv_heads > 65535 || !row_ok(row_bytes) || pool_capacity < 0 || pool_capacity > INT32_MAX)
    return PSRL_ERR_SHAPE;
  if (workspace_bytes < kWsHeaderBytes) return PSRL_ERR_WORKSPACE;
  const int64_t bytes = pool_capacity * n_kv_heads * row_bytes;
  if (overlap(k_pool, bytes, v_pool, bytes)) return PSRL_ERR_INVALID_ARG;
  try {
    std::vector<psrl_kv_extent_t> list;
    int64_t src_end = 0, dst_end = 0;
    for (int32_t i = 0; i < n_extents; ++i) {
      const psrl_kv_extent_t& e = extents[i];
      if (!in_range(e, pool_capacity, pool_capacity)) return PSRL_ERR_SHAPE;
      if (e.n_slots == 0) continue;
      if (e.dst_slot > e.src_slot || e.src_slot < src_end || e.dst_slot < dst_end) return PSRL_ERR_INVALID_ARG;
      src_end = int64_t(e.src_slot) + e.n_slots;
      dst_end = int64_t(e.dst_slot) + e.n_slots;
      if (e.dst_slot != e.src_slot) list.push_back(e);
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (list.empty() || (!k_pool && !v_pool)) {
      const cudaError_t e = cudaMemsetAsync(workspace, 0, kWsHeaderBytes, s);
      if (e == cudaSuccess) return PSRL_OK;
      set_last_cuda_error(e);
      return PSRL_ERR_CUDA;
    }
    const Pools p{static_cast<const uint4*>(k_pool), static_cast<const uint4*>(v_pool), static_cast<uint4*>(k_pool),
                  static_cast<uint4*>(v_pool), pool_capacity, pool_capacity, n_kv_heads, row_bytes / 16};
    // a short list costs a launch less parameter traffic
    const bool few = list.size() <= kShortList;
    for (size_t at = 0; at < list.size(); at += kLongList) {
      const int32_t n = static_cast<int32_t>(std::min(list.size() - at, size_t(kLongList)));
      int* ws = static_cast<int*>(workspace);
      const psrl_status_t st = few ? move_extents<kShortList>(list.data() + at, n, p, ws, at == 0, s)
                                   : move_extents<kLongList>(list.data() + at, n, p, ws, at == 0, s);
      if (st != PSRL_OK) return st;
    }
  } catch (const std::bad_alloc&) {
    return PSRL_ERR_HOST_OOM;
  }
  return PSRL_OK;
}

}  // extern "C"
