// Routed products on the 5th-generation tensor cores (tcgen05, sums in tensor memory).
//
//   k_route_product    out[p, m] = sum_k  W[e(p)][m, k] * X[row(p), k]      p: place in the order of the columns of R
//   k_route_product8   the same with e4m3 operands and a scale per 128 values of k
//   k_route_dw         dW[e][m, j] = sum over the places p of column e of dP[p, m] * X[row(p), j]
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gm_t5.cuh"

namespace gm {

constexpr int kTileM = 128;        // rows of a block of W (or of dW) per tile: the lanes of tensor memory
constexpr int kTileN = 256;        // places (or columns of dW) per tile: columns of tensor memory, twice
constexpr int kRowBytes = 128;     // of one operand row in a stage: 64 values of 16 bits, 128 of 8
constexpr int kStages = 4;
constexpr int kStageA = kTileM * kRowBytes, kStageB = kTileN * kRowBytes, kStage = kStageA + kStageB;
constexpr u32 kTmemColumns = 512;

struct ProductArgs {
  const i64* offsets;
  const int32_t* rows;
  int E, n_m, n_k;      // columns of R, rows of a block of W, length of the sums
  int x_rows;           // rows of X: the index that reads as zeros
  i64 places;           // entries of R
  void* out;
  i64 out_stride;
  u32 type;             // of the operands in the instruction descriptor
  const float* xs;      // 8 bits: scales of X (rows x blocks of k) ...
  i64 xs_stride;
  const float* ws;      // ... and of W (E x groups of rows x blocks of k)
  i64 ws_block, ws_row;
  int* err;
};

struct DwArgs {
  const i64* offsets;
  const int32_t* rows;  // nullptr: X has a row per place
  int E, n_m, n_j;
  int x_rows;
  i64 places;
  void* out;
  i64 out_block, out_stride;
  u32 type;
  int* err;
};

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// The barriers and the place in tensor memory of a block, behind its stages.
struct T5Block {
  u64 full[kStages], empty[kStages];
  u64 sums_full[2], sums_empty[2], drain;
  u32 tmem;
  u32 scan_tmp[34];
};

// Places of each column, cut into parts of at most kTileN places that differ by less than 16 in size.
struct Part { int e, first, n; };
__device__ __forceinline__ int part_count(int places) { return (places + kTileN - 1) / kTileN; }
__device__ __forceinline__ int part_size(int places, int parts) { return ((places + parts - 1) / parts + 15) & ~15; }

// off[e]: first place of column e; part[e]: parts of the columns before it.  All threads of the block.
__device__ __forceinline__ void list_parts(const i64* __restrict__ offsets, int E, int* off, int* part, u32* scan_tmp) {
  u32 before = 0;
  for (int e0 = 0; e0 <= E; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    int a = 0, n = 0;
    if (e <= E) a = static_cast<int>(offsets[e]);
    if (e < E) n = part_count(static_cast<int>(offsets[e + 1]) - a);
    u32 total;
    const u32 first = before + block_exclusive_scan(static_cast<u32>(n), scan_tmp, &total);
    before += total;
    if (e <= E) { off[e] = a; part[e] = static_cast<int>(first); }
    __syncthreads();
  }
}
__device__ __forceinline__ Part part_at(const int* off, const int* part, int E, int id) {
  int lo = 0, hi = E - 1;  // the last e with part[e] <= id (columns without places have no part)
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (part[mid] <= id) lo = mid; else hi = mid - 1;
  }
  Part t;
  t.e = lo;
  const int places = off[lo + 1] - off[lo], parts = part[lo + 1] - part[lo], size = part_size(places, parts), j = id - part[lo];
  t.first = off[lo] + j * size;
  t.n = min(size, off[lo + 1] - t.first);
  return t;
}

__device__ __forceinline__ char* t5_align(char* p) {
  return p + ((1024 - (smem_u32(p) & 1023)) & 1023);
}

__device__ __forceinline__ void t5_begin(T5Block* b, int epilogue_warps) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&b->full[i], 1); mbar_init(&b->empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&b->sums_full[i], 1); mbar_init(&b->sums_empty[i], epilogue_warps); }
    mbar_init(&b->drain, 1);
    mbar_fence_init();
  }
  __syncwarp();
  if (threadIdx.x < 32) tmem_alloc(&b->tmem, kTmemColumns);
  t5_fence_before();
  __syncthreads();
  t5_fence_after();
}

// A role that gave up waiting says so; copies in flight are waited for (with a limit) before the block leaves.
__device__ __forceinline__ void t5_drain_copies(T5Block* b, u32 issued) {
  for (u32 i = issued > kStages ? issued - kStages : 0; i < issued; ++i) t5_wait(&b->full[i % kStages], (i / kStages) & 1);
}

// Rows of the result behind the last routed place are zero.
template <typename TO>
__device__ __forceinline__ void zero_rows(TO* out, i64 stride, i64 p0, i64 p1, int width) {
  for (i64 p = p0 + blockIdx.x; p < p1; p += gridDim.x)
    for (int m = threadIdx.x; m < width; m += blockDim.x) out[p * stride + m] = from_float<TO>(0.f);
}

// Lane = row m of the tile, v[j] = place j of a run of 32: out[(p + j) * stride + m].
template <typename TO>
__device__ __forceinline__ void store_places(TO* __restrict__ out, i64 stride, i64 p, int n, int m, int n_m, const u32 (&v)[32]) {
  if (m < n_m) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < n) out[(p + j) * stride + m] = from_float<TO>(__uint_as_float(v[j]));
  }
}

// kAmn: W is contiguous along its own rows m, not along k (the product with W itself instead of its transpose).
// kGather: X has a row per row of R, fetched four at a time by index; else a row per place.
template <bool kAmn, bool kGather, typename TO>
__global__ void __launch_bounds__(192, 1) k_route_product(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                          const ProductArgs a) {
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  T5Block* b = reinterpret_cast<T5Block*>(stages + kStages * kStage);
  int* off = reinterpret_cast<int*>(b + 1);
  int* part = off + a.E + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  t5_begin(b, 4);
  list_parts(a.offsets, a.E, off, part, b->scan_tmp);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_kb = (a.n_k + 63) / 64;
  const i64 n_tiles = static_cast<i64>(part[a.E]) * n_mt;
  const u32 stage0 = smem_u32(stages), tmem = b->tmem;
  zero_rows(static_cast<TO*>(a.out), a.out_stride, off[a.E], a.places, a.n_m);

  if (warp == 0) {  // copies
    u32 it = 0;
    bool ok = true;
    for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
      const int m0 = static_cast<int>(id % n_mt) * kTileM, n16 = (t.n + 15) & ~15;
      int4 r[2];
      if (kGather) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int g = (lane + 32 * h) * 4;
          r[h].x = g + 0 < t.n ? a.rows[t.first + g + 0] : a.x_rows;
          r[h].y = g + 1 < t.n ? a.rows[t.first + g + 1] : a.x_rows;
          r[h].z = g + 2 < t.n ? a.rows[t.first + g + 2] : a.x_rows;
          r[h].w = g + 3 < t.n ? a.rows[t.first + g + 3] : a.x_rows;
        }
      }
      const u32 bytes = kStageA + (kGather ? n16 : (n16 + 31) / 32 * 32) * kRowBytes;
      for (int kb = 0; kb < n_kb; ++kb, ++it) {
        const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA;
        ok = t5_wait(&b->empty[s], ((it / kStages) & 1) ^ 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&b->full[s], bytes);
          if (kAmn) {
            tma_load_3d(sa, &map_w, m0, kb * 64, t.e, &b->full[s]);
            tma_load_3d(sa + kStageA / 2, &map_w, m0 + 64, kb * 64, t.e, &b->full[s]);
          } else {
            tma_load_3d(sa, &map_w, kb * 64, m0, t.e, &b->full[s]);
          }
        }
        __syncwarp();
        if (kGather) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if ((lane + 32 * h) * 4 < n16) tma_gather4(sb + (lane + 32 * h) * 4 * kRowBytes, &map_x, kb * 64, r[h], &b->full[s]);
        } else if (lane * 32 < n16) {
          tma_load_2d(sb + lane * 32 * kRowBytes, &map_x, kb * 64, t.first + lane * 32, &b->full[s]);
        }
      }
    }
    if (!ok) {
      if (lane == 0) dev_set_error(a.err, kDevTimeout);
      t5_drain_copies(b, it);
    }
  } else if (warp == 1) {  // matrix instructions
    if (lane == 0) {
      u32 it = 0, n_done = 0;
      bool ok = true;
      for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x, ++n_done) {
        const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
        const u32 idesc = t5_idesc(a.type, kAmn, false, kTileM, (t.n + 15) & ~15), buf = n_done & 1, d = tmem + buf * kTileN;
        ok = t5_wait(&b->sums_empty[buf], ((n_done >> 1) & 1) ^ 1);
        if (!ok) break;
        t5_fence_after();
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA;
          ok = t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u64 da = kAmn ? t5_desc_mn(sa + j * 16 * kRowBytes, kStageA / 2) : t5_desc_k(sa + j * 32);
            t5_mma_f16(d, da, t5_desc_k(sb + j * 32), idesc, kb > 0 || j > 0);
          }
          t5_commit(&b->empty[s]);
        }
        if (ok) t5_commit(&b->sums_full[buf]);
      }
      if (!ok) {
        dev_set_error(a.err, kDevTimeout);
        t5_commit(&b->drain);
        t5_wait(&b->drain, 0);
      }
    }
    __syncwarp();
  } else {  // results
    const int quad = warp & 3;
    u32 n_done = 0;
    bool ok = true;
    for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x, ++n_done) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
      const int m = static_cast<int>(id % n_mt) * kTileM + quad * 32 + lane;
      const u32 buf = n_done & 1;
      ok = __all_sync(0xffffffffu, t5_wait(&b->sums_full[buf], (n_done >> 1) & 1));
      if (!ok) break;
      t5_fence_after();
      for (int c = 0; c < t.n; c += 32) {
        u32 v[32];
        t5_ld32(v, tmem + buf * kTileN + c + (static_cast<u32>(quad * 32) << 16));
        t5_wait_ld();
        store_places(static_cast<TO*>(a.out), a.out_stride, static_cast<i64>(t.first) + c, t.n - c, m, a.n_m, v);
      }
      t5_fence_before();
      if (lane == 0) mbar_arrive(&b->sums_empty[buf]);
    }
    if (!ok && lane == 0) dev_set_error(a.err, kDevTimeout);
  }
  t5_fence_before();
  __syncthreads();
  t5_fence_after();
  if (warp == 0) tmem_free(tmem, kTmemColumns);
}

// 8 bits.  The sums of 128 values of k go to a buffer of their own in tensor memory; eight warps take them out, multiply by both
// scales and add them up in registers (a thread: one row of W, half the places of the tile).
// kRowScales: W has scales for each row and 128 values; else for each 128 rows, so that a tile has one.
template <bool kGather, bool kRowScales, typename TO>
__global__ void __launch_bounds__(320, 1) k_route_product8(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                                                           const ProductArgs a) {
  constexpr int kAhead = 4;  // blocks of k whose scales are brought in together
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  T5Block* b = reinterpret_cast<T5Block*>(stages + kStages * kStage);
  float* scale = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(b + 1) + 15) & ~static_cast<uintptr_t>(15));  // [2][kAhead][kTileN]
  int* off = reinterpret_cast<int*>(scale + 2 * kAhead * kTileN);
  int* part = off + a.E + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  t5_begin(b, 8);
  list_parts(a.offsets, a.E, off, part, b->scan_tmp);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_kb = (a.n_k + 127) / 128;
  const i64 n_tiles = static_cast<i64>(part[a.E]) * n_mt;
  const u32 stage0 = smem_u32(stages), tmem = b->tmem;
  zero_rows(static_cast<TO*>(a.out), a.out_stride, off[a.E], a.places, a.n_m);

  if (warp == 0) {
    u32 it = 0;
    bool ok = true;
    for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
      const int m0 = static_cast<int>(id % n_mt) * kTileM, n16 = (t.n + 15) & ~15;
      int4 r[2];
      if (kGather) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int g = (lane + 32 * h) * 4;
          r[h].x = g + 0 < t.n ? a.rows[t.first + g + 0] : a.x_rows;
          r[h].y = g + 1 < t.n ? a.rows[t.first + g + 1] : a.x_rows;
          r[h].z = g + 2 < t.n ? a.rows[t.first + g + 2] : a.x_rows;
          r[h].w = g + 3 < t.n ? a.rows[t.first + g + 3] : a.x_rows;
        }
      }
      const u32 bytes = kStageA + (kGather ? n16 : (n16 + 31) / 32 * 32) * kRowBytes;
      for (int kb = 0; kb < n_kb; ++kb, ++it) {
        const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA;
        ok = t5_wait(&b->empty[s], ((it / kStages) & 1) ^ 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(&b->full[s], bytes);
          tma_load_3d(sa, &map_w, kb * 128, m0, t.e, &b->full[s]);
        }
        __syncwarp();
        if (kGather) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if ((lane + 32 * h) * 4 < n16) tma_gather4(sb + (lane + 32 * h) * 4 * kRowBytes, &map_x, kb * 128, r[h], &b->full[s]);
        } else if (lane * 32 < n16) {
          tma_load_2d(sb + lane * 32 * kRowBytes, &map_x, kb * 128, t.first + lane * 32, &b->full[s]);
        }
      }
    }
    if (!ok) {
      if (lane == 0) dev_set_error(a.err, kDevTimeout);
      t5_drain_copies(b, it);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      u32 it = 0;
      bool ok = true;
      for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
        const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
        const u32 idesc = t5_idesc(a.type, false, false, kTileM, (t.n + 15) & ~15);
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA, buf = it & 1, d = tmem + buf * kTileN;
          ok = t5_wait(&b->sums_empty[buf], ((it >> 1) & 1) ^ 1) && t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) t5_mma_f8(d, t5_desc_k(sa + j * 32), t5_desc_k(sb + j * 32), idesc, j > 0);
          t5_commit(&b->empty[s]);
          t5_commit(&b->sums_full[buf]);
        }
      }
      if (!ok) {
        dev_set_error(a.err, kDevTimeout);
        t5_commit(&b->drain);
        t5_wait(&b->drain, 0);
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2, tid = threadIdx.x - 64;
    u32 it = 0;
    bool ok = true;
    // (a wait that gave up skips the work from there on, not the barriers among these warps)
    for (i64 id = blockIdx.x; id < n_tiles; id += gridDim.x) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / n_mt));
      const int m0 = static_cast<int>(id % n_mt) * kTileM, m = m0 + quad * 32 + lane;
      float acc[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[c][j] = 0.f;
      // this thread brings in the scales of place `tid` of the tile
      const float* xs = nullptr;
      if (tid < t.n) xs = a.xs + static_cast<i64>(kGather ? a.rows[t.first + tid] : t.first + tid) * a.xs_stride;
      const float* ws = a.ws + static_cast<i64>(t.e) * a.ws_block + (kRowScales ? static_cast<i64>(min(m, a.n_m - 1)) : static_cast<i64>(m0 / 128)) * a.ws_row;
      float next[kAhead], wnext[kAhead];
      auto fetch = [&](int kb) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          wnext[i] = kb + i < n_kb ? ws[kb + i] : 0.f;
          next[i] = xs && kb + i < n_kb ? xs[kb + i] : 0.f;
        }
      };
      fetch(0);
      for (int kb0 = 0; kb0 < n_kb; kb0 += kAhead) {
        float* sc = scale + ((kb0 / kAhead) & 1) * kAhead * kTileN;
        float w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          w[i] = wnext[i];
          sc[i * kTileN + tid] = kRowScales ? next[i] : next[i] * wnext[i];
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (kb0 + kAhead < n_kb) fetch(kb0 + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (kb0 + i < n_kb && ok) {
            const u32 buf = it & 1;
            ok = __all_sync(0xffffffffu, t5_wait(&b->sums_full[buf], (it >> 1) & 1));
            if (ok) {
              t5_fence_after();
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                if (half * 128 + c * 32 < t.n) {
                  u32 v[32];
                  t5_ld32(v, tmem + buf * kTileN + half * 128 + c * 32 + (static_cast<u32>(quad * 32) << 16));
                  t5_wait_ld();
                  const float4* s4 = reinterpret_cast<const float4*>(sc + i * kTileN + half * 128 + c * 32);
#pragma unroll
                  for (int j = 0; j < 8; ++j) {
                    const float4 s = s4[j];
                    acc[c][4 * j + 0] += __uint_as_float(v[4 * j + 0]) * (kRowScales ? s.x * w[i] : s.x);
                    acc[c][4 * j + 1] += __uint_as_float(v[4 * j + 1]) * (kRowScales ? s.y * w[i] : s.y);
                    acc[c][4 * j + 2] += __uint_as_float(v[4 * j + 2]) * (kRowScales ? s.z * w[i] : s.z);
                    acc[c][4 * j + 3] += __uint_as_float(v[4 * j + 3]) * (kRowScales ? s.w * w[i] : s.w);
                  }
                }
              }
              t5_fence_before();
              if (lane == 0) mbar_arrive(&b->sums_empty[buf]);
              ++it;
            }
          }
        }
      }
      if (ok) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int at = half * 128 + c * 32;
          u32 v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(acc[c][j]);
          if (at < t.n) store_places(static_cast<TO*>(a.out), a.out_stride, static_cast<i64>(t.first) + at, t.n - at, m, a.n_m, v);
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");  // (the scales' buffers go round again)
    }
    if (!ok && lane == 0) dev_set_error(a.err, kDevTimeout);
  }
  t5_fence_before();
  __syncthreads();
  t5_fence_after();
  if (warp == 0) tmem_free(tmem, kTmemColumns);
}

// Both operands lie with the reduction across their rows; rows come four at a time by index, and an index behind the last row reads
// as zeros, which ends a column's sum inside a stage whatever lies behind it.
template <bool kGather, typename TO>
__global__ void __launch_bounds__(192, 1) k_route_dw(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_x,
                                                     const DwArgs a) {
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  T5Block* b = reinterpret_cast<T5Block*>(stages + kStages * kStage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  t5_begin(b, 4);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_jt = (a.n_j + kTileN - 1) / kTileN;
  const i64 n_tiles = static_cast<i64>(a.E) * n_mt * n_jt;
  const u32 stage0 = smem_u32(stages), tmem = b->tmem;
  constexpr u32 kBlock = 64 * kRowBytes;  // 64 places of 64 values

  if (warp == 0) {
    u32 it = 0;
    bool ok = true;
    const int g = lane & 15, hi = lane >> 4;
    for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
      const int e = static_cast<int>(id / (n_mt * n_jt)), rest = static_cast<int>(id % (n_mt * n_jt));
      const int m0 = rest % n_mt * kTileM, j0 = rest / n_mt * kTileN, n_cb = min(4, (a.n_j - j0 + 63) / 64);
      const int p0 = static_cast<int>(a.offsets[e]), p1 = static_cast<int>(a.offsets[e + 1]);
      const u32 bytes = (2 + n_cb) * kBlock;
      const int none = static_cast<int>(a.places);
      auto row = [&](int p) { return p < p1 ? (kGather ? a.rows[p] : p) : a.x_rows; };
      int4 next = make_int4(row(p0 + 4 * g), row(p0 + 4 * g + 1), row(p0 + 4 * g + 2), row(p0 + 4 * g + 3));
      for (int p = p0; p < p1; p += 64, ++it) {
        const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA;
        const int q = p + 4 * g;
        const int4 rx = next, rp = make_int4(q < p1 ? q : none, q + 1 < p1 ? q + 1 : none, q + 2 < p1 ? q + 2 : none, q + 3 < p1 ? q + 3 : none);
        next = make_int4(row(q + 64), row(q + 65), row(q + 66), row(q + 67));
        ok = t5_wait(&b->empty[s], ((it / kStages) & 1) ^ 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&b->full[s], bytes);
        __syncwarp();
        tma_gather4(sa + hi * kBlock + g * 4 * kRowBytes, &map_p, m0 + hi * 64, rp, &b->full[s]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int cb = 2 * h + hi;
          if (cb < n_cb) tma_gather4(sb + cb * kBlock + g * 4 * kRowBytes, &map_x, j0 + cb * 64, rx, &b->full[s]);
        }
      }
    }
    if (!ok) {
      if (lane == 0) dev_set_error(a.err, kDevTimeout);
      t5_drain_copies(b, it);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      u32 it = 0, n_done = 0;
      bool ok = true;
      for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
        const int e = static_cast<int>(id / (n_mt * n_jt)), rest = static_cast<int>(id % (n_mt * n_jt)), j0 = rest / n_mt * kTileN;
        const int p0 = static_cast<int>(a.offsets[e]), p1 = static_cast<int>(a.offsets[e + 1]);
        if (p0 >= p1) continue;
        const u32 idesc = t5_idesc(a.type, true, true, kTileM, (min(kTileN, a.n_j - j0) + 15) & ~15), buf = n_done & 1, d = tmem + buf * kTileN;
        ok = t5_wait(&b->sums_empty[buf], ((n_done >> 1) & 1) ^ 1);
        if (!ok) break;
        t5_fence_after();
        for (int p = p0; p < p1; p += 64, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kStageA;
          ok = t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            t5_mma_f16(d, t5_desc_mn(sa + j * 16 * kRowBytes, kBlock), t5_desc_mn(sb + j * 16 * kRowBytes, kBlock), idesc, p > p0 || j > 0);
          t5_commit(&b->empty[s]);
        }
        if (ok) t5_commit(&b->sums_full[buf]);
        ++n_done;
      }
      if (!ok) {
        dev_set_error(a.err, kDevTimeout);
        t5_commit(&b->drain);
        t5_wait(&b->drain, 0);
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3;
    u32 n_done = 0;
    bool ok = true;
    for (i64 id = blockIdx.x; ok && id < n_tiles; id += gridDim.x) {
      const int e = static_cast<int>(id / (n_mt * n_jt)), rest = static_cast<int>(id % (n_mt * n_jt));
      const int m = rest % n_mt * kTileM + quad * 32 + lane, j0 = rest / n_mt * kTileN, n = min(kTileN, a.n_j - j0);
      const bool some = a.offsets[e] < a.offsets[e + 1];
      TO* out = static_cast<TO*>(a.out) + static_cast<i64>(e) * a.out_block + static_cast<i64>(m) * a.out_stride + j0;
      const u32 buf = n_done & 1;
      if (some) {
        ok = __all_sync(0xffffffffu, t5_wait(&b->sums_full[buf], (n_done >> 1) & 1));
        if (!ok) break;
        t5_fence_after();
      }
      for (int c = 0; c < n; c += 32) {
        u32 v[32];
        if (some) {
          t5_ld32(v, tmem + buf * kTileN + c + (static_cast<u32>(quad * 32) << 16));
          t5_wait_ld();
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0;
        }
        if (m < a.n_m) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (c + j < n) out[c + j] = from_float<TO>(__uint_as_float(v[j]));
        }
      }
      if (some) {
        t5_fence_before();
        if (lane == 0) mbar_arrive(&b->sums_empty[buf]);
        ++n_done;
      }
    }
    if (!ok && lane == 0) dev_set_error(a.err, kDevTimeout);
  }
  t5_fence_before();
  __syncthreads();
  t5_fence_after();
  if (warp == 0) tmem_free(tmem, kTmemColumns);
}

// Copies into an aligned layout for the tensor maps: dst (blocks x rows x padded columns), the padding zero.
template <typename T>
__global__ void k_route_pack(const T* __restrict__ src, i64 block_stride, i64 row_stride, i64 col_stride, i64 n_blocks, i64 n_rows,
                             i64 n_cols, i64 padded, T* __restrict__ dst) {
  const i64 total = n_blocks * n_rows * padded;
  for (i64 i = static_cast<i64>(blockIdx.x) * blockDim.x + threadIdx.x; i < total; i += static_cast<i64>(gridDim.x) * blockDim.x) {
    const i64 c = i % padded, br = i / padded, r = br % n_rows, blk = br / n_rows;
    dst[i] = c < n_cols ? src[blk * block_stride + r * row_stride + c * col_stride] : T(0);
  }
}

}  // namespace gm
