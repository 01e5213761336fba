// Routes: the entries of a CSR matrix R (few entries a row, few columns) in the order of their columns, stable.
//
//   offsets[e]  first place of column e (e = E: entries whose column is outside [0, E), behind all others)
//   rows[p], order[p]   row and index of the entry at place p;   pos[q] the place of entry q
//
// A counting sort in one launch: a cluster of up to 8 blocks shares the entries, every warp a run of consecutive ones with counters of its
// own in shared memory (so that places do not depend on the order in which anything runs), the blocks' sums go through
// distributed shared memory.  Bound by latency: two walks over the entries and three cluster barriers.
#pragma once
#include <cooperative_groups.h>

#include "gm_common.cuh"

namespace gm {

constexpr int kRouteMaxCols = 2048;
constexpr int kRouteThreads = 1024;
constexpr int kRouteBlocks = 8;
constexpr int kRouteCounterBytes = 200 * 1024;

// The row of entry q: rows of a router's matrix are mostly equally long, so the proportional one is tried first.
__device__ __forceinline__ int route_row(const i64* __restrict__ row_ptr, int n_rows, i64 nnz, i64 q) {
  int g = static_cast<int>(static_cast<float>(q) * static_cast<float>(n_rows) / static_cast<float>(nnz));
  g = max(0, min(n_rows - 1, g));
  const i64 a = row_ptr[g], b = row_ptr[g + 1];
  if (a <= q && q < b) return g;
  return static_cast<int>(q < a ? last_le(row_ptr, 0, max(0, g - 1), q) : last_le(row_ptr, min(n_rows - 1, g + 1), n_rows - 1, q));
}

__host__ __device__ inline int route_warps(int cols) {
  const int w = kRouteCounterBytes / ((cols + 1) * 4);
  return w < 1 ? 1 : (w > 32 ? 32 : w);
}
inline size_t route_smem(int cols, int warps) { return static_cast<size_t>(warps + 2) * (cols + 1) * 4; }

__global__ void __launch_bounds__(kRouteThreads) k_route_plan(const i64* __restrict__ row_ptr, const int32_t* __restrict__ col,
                                                              int n_rows, i64 nnz, int E, i64* __restrict__ offsets,
                                                              int32_t* __restrict__ rows, int32_t* __restrict__ order,
                                                              int32_t* __restrict__ pos) {
  namespace cg = cooperative_groups;
  extern __shared__ u32 route_sm[];
  __shared__ u32 scan_tmp[33];
  cg::cluster_group cluster = cg::this_cluster();
  const int bins = E + 1, warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  u32* cnt = route_sm + static_cast<size_t>(warp) * bins;   // this warp's entries per column, then its next places
  u32* sum = route_sm + static_cast<size_t>(warps) * bins;  // this block's entries per column: read by the others
  u32* base = sum + bins;                                   // first place of this block's entries of a column
  for (int e = lane; e < bins; e += 32) cnt[e] = 0;
  const i64 n_warps = static_cast<i64>(gridDim.x) * warps, per = (nnz + n_warps - 1) / n_warps;
  const i64 q0 = min(nnz, (static_cast<i64>(blockIdx.x) * warps + warp) * per), q1 = min(nnz, q0 + per);
  __syncwarp();
  for (i64 q = q0 + lane; q < q1; q += 32) {
    const int c = col[q];
    atomicAdd(&cnt[static_cast<u32>(c) < static_cast<u32>(E) ? c : E], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < bins; e += blockDim.x) {
    u32 s = 0;
    for (int w = 0; w < warps; ++w) {
      u32* at = route_sm + static_cast<size_t>(w) * bins + e;
      const u32 v = *at;
      *at = s;
      s += v;
    }
    sum[e] = s;
  }
  cluster.sync();
  u32 before = 0;
  for (int e0 = 0; e0 < bins; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    u32 all = 0, mine = 0;
    if (e < bins) {
      for (unsigned b = 0; b < gridDim.x; ++b) {
        const u32 v = cluster.map_shared_rank(sum, b)[e];
        if (b < blockIdx.x) mine += v;
        all += v;
      }
    }
    u32 total;
    const u32 first = before + block_exclusive_scan(all, scan_tmp, &total);
    before += total;
    if (e < bins) {
      base[e] = first + mine;
      if (blockIdx.x == 0) offsets[e] = first;
    }
    __syncthreads();
  }
  cluster.sync();  // (no block leaves while another still reads its sums)
  for (i64 qb = q0; qb < q1; qb += 32) {
    const i64 q = qb + lane;
    const bool in = q < q1;
    int e = -1;
    if (in) {
      const int c = col[q];
      e = static_cast<u32>(c) < static_cast<u32>(E) ? c : E;
    }
    const u32 peers = __match_any_sync(0xffffffffu, e);
    u32 place = 0;
    if (in) place = base[e] + cnt[e] + __popc(peers & lanemask_lt());
    __syncwarp();
    if (in && (peers & lanemask_lt()) == 0) cnt[e] += __popc(peers);
    __syncwarp();
    if (in) {
      pos[q] = static_cast<int32_t>(place);
      order[place] = static_cast<int32_t>(q);
      rows[place] = route_row(row_ptr, n_rows, nnz, q);
    }
  }
}

}  // namespace gm
