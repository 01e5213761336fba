// Routes: the entries of a CSR matrix R (few entries a row, few columns) in the order of their columns, stable.
//
//   offsets[e]  first place of column e (e = E: entries whose column is outside [0, E), behind all others)
//   rows[p], order[p]   row and index of the entry at place p;   pos[q] the place of entry q
//
// A counting sort in one launch: a cluster of up to 16 blocks shares the entries, every warp a run of consecutive ones with counters of its
// own in shared memory (so that places do not depend on the order in which anything runs), the blocks' sums go through
// distributed shared memory.  Bound by latency: two walks over the entries and three cluster barriers.
#pragma once
#include <cooperative_groups.h>

#include "gm_t5.cuh"

namespace gm {

constexpr int kRouteMaxCols = 2048;
constexpr int kRouteThreads = 1024;
constexpr int kRouteBlocks = 16;     // where a cluster of so many fits the device, else 8
constexpr int kRouteAhead = 8;  // loads of columns under way
constexpr int kRouteCounterBytes = 200 * 1024;

// Rows of a warp's 32 consecutive entries qb + lane (those below q1), given a row r that does not lie behind the first one's; returns the last
// one's.  The next rows' starts are looked at 32 at a time; where rows without entries follow in large numbers, by bisection.
__device__ __forceinline__ int route_rows(const i64* __restrict__ row_ptr, int n_rows, i64 q1, i64 qb, int r, int* row) {
  const int lane = threadIdx.x & 31;
  const i64 q = qb + lane;
  bool open = q < q1;
  *row = r;
  for (int round = 0; round < 2 && __any_sync(0xffffffffu, open); ++round) {
    const int base = r + 32 * round;  // rows base .. base + 31: their ends
    const i64 end = base + 1 + lane <= n_rows ? row_ptr[base + 1 + lane] : LLONG_MAX;
    int k = 0;  // ends that are not behind q
#pragma unroll
    for (int step = 16; step > 0; step >>= 1)
      if (__shfl_sync(0xffffffffu, end, k + step - 1) <= q) k += step;
    const i64 at = __shfl_sync(0xffffffffu, end, k);
    if (open && (k < 31 || at > q)) {
      *row = min(n_rows - 1, base + k);
      open = false;
    }
  }
  if (open) *row = static_cast<int>(last_le(row_ptr, min(n_rows - 1, r + 64), n_rows - 1, q));
  return __shfl_sync(0xffffffffu, *row, static_cast<int>(min(static_cast<i64>(31), q1 - qb - 1)));
}

// The last row that starts at or before entry q: looked for where it would be if all rows were equally long, then by bisection.
__device__ __forceinline__ int route_first_row(const i64* __restrict__ row_ptr, int n_rows, i64 nnz, i64 q) {
  const int lane = threadIdx.x & 31;
  const int g = max(0, min(n_rows - 32, static_cast<int>(static_cast<float>(q) * static_cast<float>(n_rows) / static_cast<float>(nnz)) - 15));
  const i64 start = g + lane <= n_rows ? row_ptr[g + lane] : LLONG_MAX;
  const u32 before = __ballot_sync(0xffffffffu, start <= q);  // (starts ascend: a run of low bits)
  const int k = __popc(before);
  if (k > 0 && (k < 32 || g + 32 >= n_rows)) return min(n_rows - 1, g + k - 1);
  return static_cast<int>(last_le(row_ptr, 0, n_rows - 1, q));
}

__host__ __device__ inline int route_warps(int cols) {
  const int w = kRouteCounterBytes / ((cols + 1) * 4);
  return w < 1 ? 1 : (w > 32 ? 32 : w);
}
inline size_t route_smem(int cols, int warps) { return static_cast<size_t>(warps + 2) * (cols + 1) * 4; }

__global__ void __launch_bounds__(kRouteThreads, 1) k_route_plan(const i64* __restrict__ row_ptr, const int32_t* __restrict__ col,
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
  grid_launch_next();
  for (int e = lane; e < bins; e += 32) cnt[e] = 0;
  grid_wait();
  const i64 n_warps = static_cast<i64>(gridDim.x) * warps, per = (nnz + n_warps - 1) / n_warps;
  const i64 q0 = min(nnz, (static_cast<i64>(blockIdx.x) * warps + warp) * per), q1 = min(nnz, q0 + per);
  // the first columns and their rows stay in registers for the second walk
  int c0[kRouteAhead], row0[kRouteAhead];
#pragma unroll
  for (int j = 0; j < kRouteAhead; ++j) c0[j] = q0 + 32 * j + lane < q1 ? col[q0 + 32 * j + lane] : 0;
  int r = q0 < q1 ? route_first_row(row_ptr, n_rows, nnz, q0) : 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kRouteAhead; ++j)
    if (q0 + 32 * j + lane < q1) atomicAdd(&cnt[static_cast<u32>(c0[j]) < static_cast<u32>(E) ? c0[j] : E], 1u);
#pragma unroll
  for (int j = 0; j < kRouteAhead; ++j)
    if (q0 + 32 * j < q1) r = route_rows(row_ptr, n_rows, q1, q0 + 32 * j, r, &row0[j]);
  for (i64 qb = q0 + 32 * kRouteAhead; qb < q1; qb += 32 * kRouteAhead) {
    int c[kRouteAhead];
#pragma unroll
    for (int j = 0; j < kRouteAhead; ++j) c[j] = qb + 32 * j + lane < q1 ? col[qb + 32 * j + lane] : 0;
#pragma unroll
    for (int j = 0; j < kRouteAhead; ++j)
      if (qb + 32 * j + lane < q1) atomicAdd(&cnt[static_cast<u32>(c[j]) < static_cast<u32>(E) ? c[j] : E], 1u);
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
  for (i64 qa = q0; qa < q1; qa += 32 * kRouteAhead) {
    if (qa > q0) {
#pragma unroll
      for (int j = 0; j < kRouteAhead; ++j) c0[j] = qa + 32 * j + lane < q1 ? col[qa + 32 * j + lane] : 0;
#pragma unroll
      for (int j = 0; j < kRouteAhead; ++j)
        if (qa + 32 * j < q1) r = route_rows(row_ptr, n_rows, q1, qa + 32 * j, r, &row0[j]);
    }
#pragma unroll
    for (int j = 0; j < kRouteAhead; ++j) {
      const i64 q = qa + 32 * j + lane;
      if (qa + 32 * j < q1) {
        const bool in = q < q1;
        const int e = in ? (static_cast<u32>(c0[j]) < static_cast<u32>(E) ? c0[j] : E) : -1;
        const u32 peers = __match_any_sync(0xffffffffu, e);
        u32 place = 0;
        if (in) place = base[e] + cnt[e] + __popc(peers & lanemask_lt());
        __syncwarp();
        if (in && (peers & lanemask_lt()) == 0) cnt[e] += __popc(peers);
        __syncwarp();
        if (in) {
          pos[q] = static_cast<int32_t>(place);
          order[place] = static_cast<int32_t>(q);
          rows[place] = row0[j];
        }
      }
    }
  }
}

}  // namespace gm
