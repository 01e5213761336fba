// Routes: the entries of a CSR matrix R (few entries a row, few columns) in the order of their columns, stable.
//
//   offsets[e]  first place of column e (e = E: entries whose column is outside [0, E), behind all others)
//   rows[p], order[p]   row and index of the entry at place p;   pos[q] the place of entry q
//
// A counting sort, in one launch where there are few entries: a cluster of up to 16 blocks shares them, every warp a run of consecutive ones with counters of its
// own in shared memory (so that places do not depend on the order in which anything runs), the blocks' sums go through
// distributed shared memory.  Bound by latency, and with few entries by its own instructions, which every launch fetches anew: the walks are loops
// that are not unrolled (a few entries 3.9 us, 4.7 with them unrolled by eight).
#pragma once
#include <cooperative_groups.h>

#include "gm_t5.cuh"

namespace gm {

constexpr int kRouteMaxCols = 2048;
constexpr int kRouteThreads = 1024;
constexpr int kRouteBlocks = 16;     // where a cluster of so many fits the device, else 8
// With more than kRouteWide entries in at most kRouteWideCols columns: as many blocks, which need a launch for their sums (131072 entries in 64
// columns: 15.7 us, 21.6 by the cluster; 32768 entries: 10.1 against 8.8; 240000 in 2000 columns: 154 against
// 52, for every block reads all blocks' sums; the border between 64 and 2000 columns is not measured closer).
constexpr int kRouteWideBlocks = 128;
constexpr int kRouteWideThreads = 256;
constexpr i64 kRouteWide = 65536;
constexpr int kRouteWideCols = 128;
constexpr int kRouteCounterBytes = 200 * 1024;

// The end of row r + lane, as an int (there are fewer than 2^31 entries); what lies behind the last row ends nowhere.
__device__ __forceinline__ int route_end(const i64* __restrict__ row_ptr, int n_rows, int r) {
  const int i = r + static_cast<int>(threadIdx.x & 31);
  return i < n_rows ? static_cast<int>(min(row_ptr[i + 1], static_cast<i64>(INT_MAX))) : INT_MAX;
}
// The row of an entry that the window of ends does not reach (many rows without entries).
__device__ __noinline__ int route_far(const i64* __restrict__ row_ptr, int n_rows, int q) {
  return static_cast<int>(last_le(row_ptr, 0, n_rows - 1, q));
}
// Rows of a warp's 32 consecutive entries, q this lane's, from a row r that does not lie behind the first one's and the ends of the 32 rows from
// there on.
__device__ __forceinline__ int route_rows(const i64* __restrict__ row_ptr, int n_rows, int q, int r, int end) {
  int k = 0;  // ends that are not behind q
#pragma unroll
  for (int step = 16; step > 0; step >>= 1)
    if (__shfl_sync(0xffffffffu, end, k + step - 1) <= q) k += step;
  return __shfl_sync(0xffffffffu, end, k) > q ? min(n_rows - 1, r + k) : route_far(row_ptr, n_rows, q);
}

// The last row that starts at or before entry q: looked for where it would be if all rows were equally long, then by bisection.
__device__ __forceinline__ int route_first_row(const i64* __restrict__ row_ptr, int n_rows, i64 nnz, i64 q) {
  const int lane = threadIdx.x & 31;
  const int g = max(0, min(n_rows - 32, static_cast<int>(static_cast<float>(q) * static_cast<float>(n_rows) / static_cast<float>(nnz)) - 15));
  const i64 start = g + lane <= n_rows ? row_ptr[g + lane] : LLONG_MAX;
  const u32 before = __ballot_sync(0xffffffffu, start <= q);  // (starts ascend: a run of low bits)
  const int k = __popc(before);
  return k > 0 && (k < 32 || g + 32 >= n_rows) ? min(n_rows - 1, g + k - 1) : route_far(row_ptr, n_rows, static_cast<int>(q));
}

__host__ __device__ inline int route_warps(int cols) {
  const int w = kRouteCounterBytes / ((cols + 1) * 4);
  return w < 1 ? 1 : (w > 32 ? 32 : w);
}
inline size_t route_smem(int cols, int warps) { return static_cast<size_t>(warps + 2) * (cols + 1) * 4; }

// Each block's entries per column, for k_route_plan<false> with as many blocks and warps: sums[column * blocks + block].
__global__ void __launch_bounds__(kRouteThreads, 1) k_route_count(const int32_t* __restrict__ col, i64 nnz, int E, u32* __restrict__ sums) {
  extern __shared__ u32 route_sm[];
  const int bins = E + 1, warps = blockDim.x >> 5;
  grid_launch_next();
  for (int e = threadIdx.x; e < bins; e += blockDim.x) route_sm[e] = 0;
  __syncthreads();
  grid_wait();
  const i64 n_warps = static_cast<i64>(gridDim.x) * warps, per = (nnz + n_warps - 1) / n_warps;  // (the same shares as there)
  const int q0 = static_cast<int>(min(nnz, static_cast<i64>(blockIdx.x) * warps * per)), q1 = static_cast<int>(min(nnz, q0 + warps * per));
#pragma unroll 4
  for (int q = q0 + static_cast<int>(threadIdx.x); q < q1; q += blockDim.x) {
    const int c = col[q];
    atomicAdd(&route_sm[static_cast<u32>(c) < static_cast<u32>(E) ? c : E], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < bins; e += blockDim.x) sums[static_cast<i64>(e) * gridDim.x + blockIdx.x] = route_sm[e];
}

// kCluster: the blocks are one cluster and tell each other their sums; else these come from k_route_count.
template <bool kCluster>
__global__ void __launch_bounds__(kRouteThreads, 1) k_route_plan(const i64* __restrict__ row_ptr, const int32_t* __restrict__ col,
                                                              int n_rows, i64 nnz, int E, const u32* __restrict__ sums, i64* __restrict__ offsets,
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
  grid_launch_next();
  for (int e = lane; e < bins; e += 32) cnt[e] = 0;
  grid_wait();
  const i64 n_warps = static_cast<i64>(gridDim.x) * warps, per = (nnz + n_warps - 1) / n_warps;
  const int q0 = static_cast<int>(min(nnz, (static_cast<i64>(blockIdx.x) * warps + warp) * per)), q1 = static_cast<int>(min(nnz, q0 + per));
  __syncwarp();
#pragma unroll 4
  for (int q = q0 + lane; q < q1; q += 32) {
    const int c = col[q];
    atomicAdd(&cnt[static_cast<u32>(c) < static_cast<u32>(E) ? c : E], 1u);
  }
  // on their way while the blocks add up: this warp's first columns and rows
  int c = q0 + lane < q1 ? col[q0 + lane] : 0;
  int r = q0 < q1 ? route_first_row(row_ptr, n_rows, nnz, q0) : 0;
  int end = route_end(row_ptr, n_rows, r);
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
  if (kCluster) {
    cluster.sync();
  } else {  // a warp adds up a column's blocks
    __syncthreads();
    const int blocks = static_cast<int>(gridDim.x), mine = static_cast<int>(blockIdx.x);
#pragma unroll 4
    for (int e = warp; e < bins; e += warps) {
      u32 before = 0, all = 0;
      for (int i = lane; i < blocks; i += 32) {
        const u32 v = sums[static_cast<i64>(e) * blocks + i];
        all += v;
        if (i < mine) before += v;
      }
      all = warp_sum(all);
      before = warp_sum(before);
      if (lane == 0) { sum[e] = all; base[e] = before; }
    }
    __syncthreads();
  }
  u32 before = 0;
  for (int e0 = 0; e0 < bins; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    u32 all = 0, mine = 0;
    if (e < bins) {
      if (kCluster) {
        for (unsigned b0 = 0; b0 < gridDim.x; b0 += 4) {  // (1, 2 or a multiple of four blocks)
          u32 v[4];
#pragma unroll
          for (unsigned i = 0; i < 4; ++i) v[i] = cluster.map_shared_rank(sum, min(b0 + i, gridDim.x - 1))[e];
#pragma unroll
          for (unsigned i = 0; i < 4; ++i)
            if (b0 + i < gridDim.x) {
              if (b0 + i < blockIdx.x) mine += v[i];
              all += v[i];
            }
        }
      } else {
        all = sum[e];
        mine = base[e];
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
  if (kCluster) cluster.sync();  // (no block leaves while another still reads its sums)
#pragma unroll 1
  for (int qb = q0; qb < q1; qb += 32) {
    const int q = qb + lane;
    const bool in = q < q1;
    const int e = in ? (static_cast<u32>(c) < static_cast<u32>(E) ? c : E) : -1;
    c = q + 32 < q1 ? col[q + 32] : 0;
    const int row = route_rows(row_ptr, n_rows, min(q, q1 - 1), r, end);
    r = __shfl_sync(0xffffffffu, row, 31);
    end = route_end(row_ptr, n_rows, r);
    const u32 peers = __match_any_sync(0xffffffffu, e), below = peers & lanemask_lt();
    u32 place = 0;
    if (in) place = base[e] + cnt[e] + __popc(below);
    __syncwarp();
    if (in && below == 0) cnt[e] += __popc(peers);
    __syncwarp();
    if (in) {
      pos[q] = static_cast<int32_t>(place);
      order[place] = q;
      rows[place] = row;
    }
  }
}

}  // namespace gm
