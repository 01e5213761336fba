// Routed products on the 5th-generation tensor cores (tcgen05, sums in tensor memory).
//
//   k_route_product         out[p, m] = sum_k  W[e(p)][m, k] * X[row(p), k]      p: place in the order of the columns of R
//   k_route_product_scaled  the same with e4m3 operands and a scale per 128 values of k
//   k_route_dw              dW[e][m, j] = sum over the places p of column e of dP[p, m] * X[row(p), j]
//
// All three work on tiles of 256 x 256 sums, a pair of blocks (of neighbouring SMs) each: either block brings in half of both
// operands and keeps half of the sums, 256 columns by 128 lanes of its tensor memory.  A single block per 128 x 256 tile moves 1.5
// times the bytes through shared memory per product, which then bounds it (268 against 227 us at 32768 places x 2048 x 2048).
// What bounds the pairs is the way from L2 to the SMs: 32 KB a stage and block, at 85 GB/s per SM 380 ns, which is the library's matrix
// product's pace (1.62 PFLOP/s), too; these reach 1.46 PFLOP/s with 256 places a tile (16384 places x 2048 x 4096, a row per place), 1.31 with
// rows by index, 1.15 with the 205 places that a tile holds on average at 32768 places in 64 columns of skewed popularity.
// The places are the instruction's N: a column's places are cut into as few parts as there can be, and a part of 33 places costs matrix time for 64.
// The sums have two buffers, so that the results of one tile are taken out while the next one is summed up.  Every role of a block finds its
// tiles by itself; that costs each of them a fraction of a microsecond a tile, and took up to 0.9 with divisions in 64 bits.
//
// Rows of X are fetched by index with 16-byte asynchronous copies of four warps.  (Tensor-map loads of four rows by index took
// about 50 cycles each however many warps issued them, four times what the matrix instructions take for those rows.)
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gm_route_words.h"
#include "gm_t5.cuh"

namespace gm {

constexpr int kTileM = 256;        // rows of a block of W (or of dW) per tile, half of them per block of threads
constexpr int kTileN = 256;        // places (or columns of dW) per tile
constexpr int kFewN = 64;          // the same where columns of R have few places
constexpr int kRowBytes = 128;     // of one operand row in a stage: 64 values of 16 bits, 128 of 8
constexpr int kHalf = 128 * kRowBytes;  // one block's share of 256 rows of an operand in a stage
constexpr u32 kTmemColumns = 512;
constexpr int kMostStages = 10;

// How a block's memory is used with kN places per tile.  Few places leave room for more stages, and tensor memory for more buffers:
// then the weights alone bound the products, and what counts is how much of them is on its way.
template <int kN>
struct Shape {
  static constexpr int kStages = kN == kTileN ? 6 : 10;
  static constexpr int kStage = kHalf + kN / 2 * kRowBytes;
  static constexpr int kBuffers = kTmemColumns / kN;  // of sums
  static_assert(kStages <= kMostStages, "barriers");
};
constexpr int kStages = Shape<kTileN>::kStages, kStage = Shape<kTileN>::kStage;
constexpr int kMostBuffers = Shape<kFewN>::kBuffers;

struct ProductArgs {
  const i64* offsets;
  const int32_t* rows;
  int E, n_m, n_k;      // columns of R, rows of a block of W, length of the sums
  i64 places;           // entries of R
  const char* x;        // rows by index: base, bytes from row to row
  i64 x_stride;
  void* out;
  i64 out_stride;
  int out_align;        // bytes that the rows' addresses are multiples of
  u32 type;             // of the operands in the instruction descriptor
  const float* xs;      // 8 bits: scales of X (rows x blocks of k) ...
  i64 xs_stride;
  const float* ws;      // ... and of W (E x groups of rows x blocks of k)
  i64 ws_block, ws_row;
  RouteWord word;
};

struct DwArgs {
  const i64* offsets;
  const int32_t* rows;
  int E, n_m, n_j;
  const char* dp;
  i64 dp_stride;
  const char* x;
  i64 x_stride;
  void* out;
  i64 out_block, out_stride;
  int out_align;        // bytes that the rows' addresses are multiples of
  u32 type;
  RouteWord word;
};

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Which rows of X a tile needs is itself copied into shared memory, during the tile before and by the warp that needs it.
constexpr int kIndexSlot = 128;  // one block's rows of a tile

// two values in a word, the first one in the low half
template <typename T> __device__ __forceinline__ u32 pack_floats(float lo, float hi);
template <> __device__ __forceinline__ u32 pack_floats<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const u32*>(&v);
}
template <> __device__ __forceinline__ u32 pack_floats<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const u32*>(&v);
}

// The barriers and the place in tensor memory of a block, behind its stages.
struct T5Block {
  u64 full[kMostStages], empty[kMostStages], copied[kMostStages];
  u64 sums_full[kMostBuffers], sums_empty[kMostBuffers], drain;
  u32 tmem;
  u32 scan_tmp[34];
  int index[2 * kIndexSlot];
};

// Places of each column, cut into as few parts of at most kN places as there can be: all of one size, a multiple of 32, but for the last one, which has
// what is left (257 places are 160 and 97, and 1793 seven times 256 and one).
struct Part { int e, first, n; };
__device__ __forceinline__ int round32(int n) { return (n + 31) & ~31; }
template <int kN> __device__ __forceinline__ int part_count(int places) { return (places + kN - 1) / kN; }
__device__ __forceinline__ int part_size(int places, int parts) { return round32((places + parts - 1) / parts); }

// off[e]: first place of column e; part[e]: parts of the columns before it.  All threads of the block.
template <int kN>
__device__ __forceinline__ void list_parts(const i64* __restrict__ offsets, int E, int* off, int* part, u32* scan_tmp) {
  u32 before = 0;
  for (int e0 = 0; e0 <= E; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    int a = 0, n = 0;
    if (e <= E) a = static_cast<int>(offsets[e]);
    if (e < E) n = part_count<kN>(static_cast<int>(offsets[e + 1]) - a);
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

__device__ __forceinline__ char* t5_align(char* p) { return p + ((1024 - (smem_u32(p) & 1023)) & 1023); }

// full_arrivals: on the leader's barrier of a stage, by both blocks;  result_warps: of one block.
__device__ __forceinline__ void t5_begin(T5Block* b, int full_arrivals, int result_warps, int copy_threads) {
  grid_launch_next();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMostStages; ++i) { mbar_init(&b->full[i], full_arrivals); mbar_init(&b->empty[i], 1); mbar_init(&b->copied[i], copy_threads); }
    for (int i = 0; i < kMostBuffers; ++i) { mbar_init(&b->sums_full[i], 1); mbar_init(&b->sums_empty[i], 2 * result_warps); }
    mbar_init(&b->drain, 1);
    mbar_fence_init();
  }
  __syncwarp();
  if (threadIdx.x < 32) tmem_alloc(&b->tmem, kTmemColumns);
  t5_fence_before();
  __syncthreads();
  cluster_sync_all();
  t5_fence_after();
}
// Both blocks leave together: neither's memory is gone while the other's instructions read it or arrive in it.
__device__ __forceinline__ void t5_end(u32 tmem) {
  t5_fence_before();
  __syncthreads();
  cluster_sync_all();
  t5_fence_after();
  if (threadIdx.x < 32) tmem_free(tmem, kTmemColumns);
}
// After a wait that gave up: the copies in flight are waited for (with a limit) before the blocks leave.
template <int kStages = gm::kStages>
__device__ __forceinline__ void t5_drain_copies(T5Block* b, u32 issued) {
  for (u32 i = issued > kStages ? issued - kStages : 0; i < issued; ++i) t5_wait(&b->full[i % kStages], (i / kStages) & 1);
}
__device__ __forceinline__ void t5_drain_matrix(T5Block* b) {
  t5_commit(&b->drain);
  t5_wait(&b->drain, 0);
}

// Rows by index: the copying threads go as far ahead as there are stages.  Their copies arrive on the stage's own barrier of the block;
// one thread that has no copies under way itself makes them visible to the matrix instructions and tells the leader (614 us for
// 32768 places x 2048 x 2048, 742 with a fence by every copying thread, which waits for all its copies; both before the arrivals at the
// leader's barrier were left at the default scope: releasing at cluster scope takes 0.6 us a stage, 614 -> 250 us.  What has to be seen across
// blocks is the barrier alone: each block's matrix unit reads that block's own memory).
template <int kStages = gm::kStages>
struct CopyQueue {
  T5Block* b;
  u32 issued = 0;
  __device__ __forceinline__ explicit CopyQueue(T5Block* block) : b(block) {}
  __device__ __forceinline__ bool slot_free() {
    return __all_sync(0xffffffffu, t5_wait(&b->empty[issued % kStages], ((issued / kStages) & 1) ^ 1));
  }
  __device__ __forceinline__ void done() {  // the stage's copies are all issued
    copy_arrive(&b->copied[issued % kStages]);
    copy_commit();
    ++issued;
  }
};

template <int kStages = gm::kStages>
__device__ __forceinline__ bool hand_over(T5Block* b, u32 stage) {
  if (!t5_wait(&b->copied[stage % kStages], (stage / kStages) & 1)) return false;
  fence_to_matrix();
  mbar_arrive_at(leader_bar(&b->full[stage % kStages]));
  return true;
}

// The rows of X of one block's half of the places, for every tile and stage: eight lanes have a row of a stage.
// kFixed: the first 128 of the tile's places (or the others), else half of them.
template <int kN, int kValueBytes, bool kFixed>
__device__ __forceinline__ void gather_rows(const ProductArgs& a, T5Block* b, u32 stage0, int* index, const int* off, const int* part, u32 n_tiles,
                                            int n_mt, int thread) {
  using S = Shape<kN>;
  CopyQueue<S::kStages> queue(b);
  constexpr int kStep = kRowBytes / kValueBytes;
  const int n_kb = (a.n_k + kStep - 1) / kStep, c = thread & 7, r0 = thread >> 3, lane = thread & 31;
  const u32 at = kHalf + r0 * kRowBytes + ((c ^ (r0 & 7)) << 4);  // (rows r0 + 16 i: the same swizzle)
  constexpr int kApart = 16, kRows = kN / 2 / kApart;  // a thread's rows: r0 + 16 i
  const int my_row = (thread >> 5) * 4 + (lane & 3) + kApart * (lane >> 2);  // the one whose index this lane brings in for its warp
  const i64 width = static_cast<i64>(a.n_k) * kValueBytes;
  const u32 rank = cluster_rank();
  const u32 pairs = gridDim.x >> 1;
  const auto bring_rows = [&](u32 id, int slot) {
    if (id >= n_tiles || lane >= 4 * kRows) return;
    const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
    const int half = kFixed ? 128 : round32(t.n) / 2, p = rank * half + my_row;
    int* to = index + slot * kIndexSlot + my_row;
    if (my_row < half && p < t.n) copy4(smem_u32(to), a.rows + t.first + p);
    else *to = -1;
  };
  bool ok = true;
  int slot = 0;
  bring_rows(blockIdx.x >> 1, 0);
  copy_commit();
  for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += pairs, slot ^= 1) {
    const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
    const int half = kFixed ? 128 : round32(t.n) / 2;
    // this tile's rows came with the last tile's first stage
    if (n_kb > S::kStages && id >= pairs) copy_wait<S::kStages>();
    else copy_wait_all();
    __syncwarp();
    const char* src[kRows];
    u32 there = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = index[slot * kIndexSlot + r0 + kApart * i];
      src[i] = a.x;
      if (r >= 0) {
        src[i] += r * a.x_stride;
        there |= 1u << i;
      }
    }
    __syncwarp();
    bring_rows(id + pairs, slot ^ 1);
    for (int kb = 0; kb < n_kb; ++kb) {
      ok = queue.slot_free();
      if (!ok) break;
      const u32 dst = stage0 + queue.issued % S::kStages * S::kStage + at;
      const i64 x = static_cast<i64>(kb) * kRowBytes + c * 16;
      const u32 bytes = static_cast<u32>(max(static_cast<i64>(0), min(static_cast<i64>(16), width - x)));
      const i64 from = bytes ? x : 0;
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (r0 + kApart * i < half && (!kFixed || (there >> i & 1))) copy16(dst + i * kApart * kRowBytes, src[i] + from, there >> i & 1 ? bytes : 0);
      queue.done();
    }
  }
  copy_wait_all();
  if (!ok && (thread & 31) == 0) route_word_report(a.word);
}

template <int kN>
__device__ __forceinline__ void hand_over_rows(const ProductArgs& a, T5Block* b, u32 n_tiles, int n_kb) {
  const i64 pairs = gridDim.x >> 1, mine = (static_cast<i64>(n_tiles) - (blockIdx.x >> 1) + pairs - 1) / pairs * n_kb;
  bool ok = true;
  for (i64 it = 0; ok && it < mine; ++it) ok = hand_over<Shape<kN>::kStages>(b, static_cast<u32>(it));
  if (!ok) route_word_report(a.word);
}

// Tiles of W (and of X with a row per place) by tensor map.  One warp; lane 0 has W, lane i 32 rows of X.
template <int kN, int kValueBytes, bool kAmn, bool kGather, bool kFixed>
__device__ __forceinline__ void copy_tiles(const ProductArgs& a, const CUtensorMap* map_w, const CUtensorMap* map_x, T5Block* b, u32 stage0,
                                           const int* off, const int* part, u32 n_tiles, int n_mt) {
  using S = Shape<kN>;
  constexpr int kStages = S::kStages, kStage = S::kStage;
  constexpr int kStep = kRowBytes / kValueBytes;
  const int lane = threadIdx.x & 31, n_kb = (a.n_k + kStep - 1) / kStep;
  const u32 rank = cluster_rank();
  u32 it = 0;
  bool ok = true;
  for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
    const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
    const int m0 = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM + rank * 128, half = kFixed ? 128 : round32(t.n) / 2;
    const u32 bytes = 2 * (kHalf + (kGather ? 0 : round32(half) * kRowBytes));
    for (int kb = 0; kb < n_kb; ++kb, ++it) {
      const u32 s = it % kStages, sa = stage0 + s * kStage;
      ok = __all_sync(0xffffffffu, t5_wait(&b->empty[s], ((it / kStages) & 1) ^ 1));
      if (!ok) break;
      const u32 bar = leader_bar(&b->full[s]);
      if (lane == 0) {
        if (rank == 0) mbar_arrive_expect_tx(&b->full[s], bytes);
        if (kAmn) {
          tma_load_3d(sa, map_w, m0, kb * kStep, t.e, bar);
          tma_load_3d(sa + kHalf / 2, map_w, m0 + 64, kb * kStep, t.e, bar);
        } else {
          tma_load_3d(sa, map_w, kb * kStep, m0, t.e, bar);
        }
      }
      if (!kGather && lane * 32 < half) tma_load_2d(sa + kHalf + lane * 32 * kRowBytes, map_x, kb * kStep, t.first + rank * half + lane * 32, bar);
    }
  }
  if (!ok) {
    if (lane == 0) route_word_report(a.word);
    if (rank == 0) t5_drain_copies<kStages>(b, it);
  }
}

// Rows of the result behind the last routed place are zero.
template <typename TO>
__device__ __forceinline__ void zero_rows(TO* out, i64 stride, i64 p0, i64 p1, int width) {
  for (i64 p = p0 + blockIdx.x; p < p1; p += gridDim.x)
    for (int m = threadIdx.x; m < width; m += blockDim.x) out[p * stride + m] = from_float<TO>(0.f);
}

// Lane = row m of the tile, v[j] = place j of a run of 16: out[(p + j) * stride + m].
template <typename TO>
__device__ __forceinline__ void store_places(TO* __restrict__ out, i64 stride, i64 p, int n, int m, int n_m, const u32 (&v)[16]) {
  if (m < n_m) {
    TO* to = out + p * stride + m;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (j < n) *to = from_float<TO>(__uint_as_float(v[j]));
      to += stride;
    }
  }
}

// 32 sums as results, two to a word where these have 16 bits.
template <typename TO>
__device__ __forceinline__ void result_words(const u32 (&v)[32], u32 (&w)[8 * sizeof(TO)]) {
  if constexpr (sizeof(TO) == 4) {
#pragma unroll
    for (int j = 0; j < 32; ++j) w[j] = v[j];
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_floats<TO>(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
  }
}
// 32 consecutive results at an address that is a multiple of `align` bytes, 16 at least.
template <typename TO>
__device__ __forceinline__ void store_run(TO* __restrict__ out, int align, const u32 (&v)[32]) {
  constexpr int kWords = 8 * sizeof(TO);
  u32 w[kWords];
  result_words<TO>(v, w);
  u32* to = reinterpret_cast<u32*>(out);
  if (align >= 32) {  // whole sectors of 32 bytes
#pragma unroll
    for (int j = 0; j < kWords; j += 8)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to + j), "r"(w[j]), "r"(w[j + 1]), "r"(w[j + 2]), "r"(w[j + 3]),
                   "r"(w[j + 4]), "r"(w[j + 5]), "r"(w[j + 6]), "r"(w[j + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4*>(to + j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
  }
}
// A warp's 32 rows (a lane each) by kOutRun results: laid down in shared memory (32 rows of 128 bytes, swizzled as the tensor map wants it), from
// where one copy writes whole lines.  With 32 bytes of its own row per lane and store, a tile of 256 x 256 took 2.8 us instead of 2.05, more than a
// short sum's products.
constexpr int kOutBytes = 32 * kRowBytes;
template <typename TO> constexpr int kOutRun = kRowBytes / sizeof(TO);
template <typename TO, int kFirst>  // 32 sums that are the values kFirst .. kFirst + 31 of the rows
__device__ __forceinline__ void lay_down(u32 to, const u32 (&v)[32]) {
  constexpr int kWords = 8 * sizeof(TO);
  const int lane = threadIdx.x & 31;
  u32 w[kWords];
  result_words<TO>(v, w);
#pragma unroll
  for (int j = 0; j < kWords; j += 4) {
    const u32 at = to + lane * kRowBytes + (((kFirst * sizeof(TO) / 16 + j / 4) ^ (lane & 7)) << 4);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[j]), "r"(w[j + 1]), "r"(w[j + 2]), "r"(w[j + 3]) : "memory");
  }
}

// A warp's rows (a lane each) by up to 32 consecutive results, rows that start anywhere: sixteen words of sixteen rows change places among sixteen
// lanes, then half a warp stores 64 consecutive bytes of a row (a lane's own row would be a sector per value: 100 us instead of 44 for 2631
// rows of 1829 values).  All lanes call.
template <typename TO>
__device__ __forceinline__ void store_turned(TO* __restrict__ out, i64 stride, int rows, int n, int align, const u32 (&v)[32]) {
  constexpr int kWords = 8 * sizeof(TO), kPer = 4 / sizeof(TO);  // values in a word
  const int lane = threadIdx.x & 31;
  u32 w[kWords];
  result_words<TO>(v, w);
#pragma unroll
  for (int set = 0; set < kWords; set += 16) {
#pragma unroll
    for (int s = 8; s > 0; s >>= 1)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if ((j & s) == 0) {
          const bool upper = lane & s;
          const u32 got = __shfl_xor_sync(0xffffffffu, upper ? w[set + j] : w[set + j + s], s);
          if (upper) w[set + j] = got; else w[set + j + s] = got;
        }
    const int c = (set + (lane & 15)) * kPer;
    TO* to = out + (lane & 16) * stride + c;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if ((lane & 16) + j < rows && c < n) {
        if constexpr (kPer == 1) {
          *reinterpret_cast<u32*>(to) = w[set + j];
        } else if (align >= 4 && c + 1 < n) {
          *reinterpret_cast<u32*>(to) = w[set + j];
        } else {
          *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(w[set + j]);
          if (c + 1 < n) *reinterpret_cast<uint16_t*>(to + 1) = static_cast<uint16_t>(w[set + j] >> 16);
        }
      }
      to += stride;
    }
  }
}

// kAmn: W is contiguous along its own rows m, not along k (the product with W itself instead of its transpose).
// kGather: X has a row per row of R, fetched by index; else a row per place.
// Warps: 0 copies by tensor map, 1 matrix instructions, 2-5 results, 6-9 copies by index, 10 hands those over.
template <int kN, bool kAmn, bool kGather, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGather ? 352 : 192, 1)
    k_route_product(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const ProductArgs a) {
  using S = Shape<kN>;
  constexpr int kStages = S::kStages, kStage = S::kStage, kBuffers = S::kBuffers;
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  T5Block* b = reinterpret_cast<T5Block*>(stages + kStages * kStage);
  int* off = reinterpret_cast<int*>(b + 1);
  int* part = off + a.E + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const u32 rank = cluster_rank();
  t5_begin(b, kGather ? 3 : 1, 4, 128);
  grid_wait();
  list_parts<kN>(a.offsets, a.E, off, part, b->scan_tmp);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_kb = (a.n_k + 63) / 64;
  const u32 n_tiles = static_cast<u32>(part[a.E]) * n_mt;
  const u32 stage0 = smem_u32(stages), tmem = b->tmem;
  zero_rows(static_cast<TO*>(a.out), a.out_stride, off[a.E], a.places, a.n_m);

  if (warp == 0) {
    copy_tiles<kN, 2, kAmn, kGather, false>(a, &map_w, &map_x, b, stage0, off, part, n_tiles, n_mt);
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      u32 it = 0, n_done = 0;
      bool ok = true;
      for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1, ++n_done) {
        const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
        const u32 idesc = t5_idesc(a.type, kAmn, false, kTileM, round32(t.n)), buf = n_done % kBuffers, d = tmem + buf * kN;
        ok = t5_wait(&b->sums_empty[buf], ((n_done / kBuffers) & 1) ^ 1);
        if (!ok) break;
        t5_fence_after();
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kHalf;
          ok = t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u64 da = kAmn ? t5_desc_mn(sa + j * 16 * kRowBytes, kHalf / 2) : t5_desc_k(sa + j * 32);
            t5_mma_f16(d, da, t5_desc_k(sb + j * 32), idesc, kb > 0 || j > 0);
          }
          t5_commit(&b->empty[s]);
        }
        if (ok) t5_commit(&b->sums_full[buf]);
      }
      if (!ok) {
        route_word_report(a.word);
        t5_drain_matrix(b);
      }
    }
    __syncwarp();
  } else if (warp < 6) {
    const int quad = warp & 3;
    u32 n_done = 0;
    bool ok = true;
    for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1, ++n_done) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
      const int m = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM + rank * 128 + quad * 32 + lane;
      const u32 buf = n_done % kBuffers;
      ok = __all_sync(0xffffffffu, t5_wait_sum(&b->sums_full[buf], (n_done / kBuffers) & 1, n_kb));
      if (!ok) break;
      t5_fence_after();
      for (int c = 0; c < t.n; c += 16) {
        u32 v[16];
        t5_ld16(v, tmem + buf * kN + c + (static_cast<u32>(quad * 32) << 16));
        t5_wait_ld16(v);
        store_places(static_cast<TO*>(a.out), a.out_stride, static_cast<i64>(t.first) + c, t.n - c, m, a.n_m, v);
      }
      t5_fence_before();
      if (lane == 0) mbar_arrive_at(leader_bar(&b->sums_empty[buf]));
    }
    if (!ok && lane == 0) route_word_report(a.word);
  } else if (warp < 10) {
    gather_rows<kN, 2, false>(a, b, stage0, b->index, off, part, n_tiles, n_mt, threadIdx.x - 192);
  } else {
    if (lane == 0) hand_over_rows<kN>(a, b, n_tiles, n_kb);
    __syncwarp();
  }
  t5_end(tmem);
}

// 8 bits.  The sums of 128 values of k go to a buffer of their own in tensor memory; eight warps take them out, multiply by both scales
// and add them up in registers.  The scales come through a ring in shared memory, a slot per block of k.
//
// Here the places are the lanes (the instruction's M) and the rows of W the columns, so that a thread has one place: its scale times
// that of the 128 rows of W is one number per thread and block of k, and the rows of the result are stored in whole runs.  (With the rows of W
// as lanes a scale per column has to be read from shared memory for every sum: 547 against 457 us at 32768 places x 4096 x 2048, 397 by now.)
// What bounds it is the way of the sums out of tensor memory and through the FP32 units: 0.69 us per block of k and tile, of which the matrix
// instructions need 0.28; without either's work 0.55 us remain, the way from one buffer's last product to its next one.
// kRowScales: W has scales for each row and 128 values, which are read from shared memory, else for each 128 rows.
// Warps: 0 copies by tensor map, 1 matrix instructions, 2 hands over what 12-15 copy by index, 3 scales, 4-11 results.  The results' registers
// are what the others give up: 512 threads begin with 128 each.
constexpr int kScaleSlots = 8;
constexpr int kScaleSlot = 128 + kTileM;  // floats: of a block's places, of the rows of W (or two for 128 of them each)
struct ScaleBlock { u64 full[kScaleSlots], empty[kScaleSlots]; };

// Brings in the scales of `rows` (of X, per lane, -1: none) and of W.  One warp.
template <int kPlaces, bool kRowScales>
__device__ __forceinline__ void copy_scales(const ProductArgs& a, u32 to, const int (&row)[kPlaces / 32], const float* ws, int m0, int n_w, int kb) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kPlaces / 32; ++i)
    if (row[i] >= 0) copy4(to + (lane + 32 * i) * 4, a.xs + row[i] * a.xs_stride + kb);
  to += kPlaces * 4;
  if (kRowScales) {
    for (int i = lane; i < n_w; i += 32)
      if (m0 + i < a.n_m) copy4(to + i * 4, ws + static_cast<i64>(m0 + i) * a.ws_row + kb);
  } else if (lane * 128 < n_w && m0 + lane * 128 < a.n_m) {
    copy4(to + lane * 4, ws + static_cast<i64>(m0 / 128 + lane) * a.ws_row + kb);
  }
}

template <bool kGather, bool kRowScales, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(512, 1)
    k_route_product_scaled(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const ProductArgs a) {
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  float* scales = reinterpret_cast<float*>(stages + kStages * kStage);
  T5Block* b = reinterpret_cast<T5Block*>(scales + kScaleSlots * kScaleSlot);
  ScaleBlock* sb = reinterpret_cast<ScaleBlock*>(b + 1);
  int* off = reinterpret_cast<int*>(sb + 1);
  int* part = off + a.E + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const u32 rank = cluster_rank();
  if (threadIdx.x == 32)
    for (int i = 0; i < kScaleSlots; ++i) { mbar_init(&sb->full[i], 32); mbar_init(&sb->empty[i], 8); }
  t5_begin(b, kGather ? 3 : 1, 8, 128);
  grid_wait();
  list_parts<kTileN>(a.offsets, a.E, off, part, b->scan_tmp);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_kb = (a.n_k + 127) / 128;
  const u32 n_tiles = static_cast<u32>(part[a.E]) * n_mt;
  const u32 stage0 = smem_u32(stages), scale0 = smem_u32(scales), tmem = b->tmem;
  zero_rows(static_cast<TO*>(a.out), a.out_stride, off[a.E], a.places, a.n_m);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(48));
    if (warp == 0) {
      copy_tiles<kTileN, 1, false, kGather, true>(a, &map_w, &map_x, b, stage0, off, part, n_tiles, n_mt);
    } else if (warp == 1 && lane == 0 && rank == 0) {
      u32 it = 0;
      bool ok = true;
      const u32 idesc = t5_idesc(a.type, false, false, 256, 256);
      for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kStages, sw = stage0 + s * kStage, sx = sw + kHalf, buf = it & 1, d = tmem + buf * 256;
          ok = t5_wait(&b->sums_empty[buf], ((it >> 1) & 1) ^ 1) && t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) t5_mma_f8(d, t5_desc_k(sx + j * 32), t5_desc_k(sw + j * 32), idesc, j > 0);
          t5_commit(&b->empty[s]);
          t5_commit(&b->sums_full[buf]);
        }
      }
      if (!ok) {
        route_word_report(a.word);
        t5_drain_matrix(b);
      }
    } else if (kGather && warp == 2 && lane == 0) {
      hand_over_rows<kTileN>(a, b, n_tiles, n_kb);
    } else if (warp == 3) {
      u32 it = 0;
      bool ok = true;
      for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
        const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
        const int m0 = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM;
        const float* ws = a.ws + static_cast<i64>(t.e) * a.ws_block;
        int row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = rank * 128 + lane + 32 * i;
          row[i] = p < t.n ? (kGather ? a.rows[t.first + p] : t.first + p) : -1;
        }
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kScaleSlots;
          ok = __all_sync(0xffffffffu, t5_wait(&sb->empty[s], ((it / kScaleSlots) & 1) ^ 1));
          if (!ok) break;
          copy_scales<128, kRowScales>(a, scale0 + s * kScaleSlot * 4, row, ws, m0, kTileM, kb);
          copy_arrive(&sb->full[s]);
        }
      }
      copy_wait_all();
      if (!ok && lane == 0) route_word_report(a.word);
    }
    __syncwarp();
  } else if (warp < 12) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(208));
    const int quad = warp & 3, half = (warp - 4) >> 2, place = rank * 128 + quad * 32 + lane;
    u32 it = 0;
    bool ok = true;
    for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
      const int m = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM + half * 128;  // this warp's first row of W
      const bool some = place - lane < t.n;                              // whether this warp has places at all
      u64 acc[64];                                                       // two rows of W each
#pragma unroll
      for (int j = 0; j < 64; ++j) acc[j] = 0;
#pragma unroll 1
      for (int kb = 0; kb < n_kb; ++kb, ++it) {
        const u32 buf = it & 1, s = it % kScaleSlots;
        ok = __all_sync(0xffffffffu, t5_wait(&sb->full[s], (it / kScaleSlots) & 1) && t5_wait(&b->sums_full[buf], (it >> 1) & 1));
        if (!ok) break;
        t5_fence_after();
        if (some) {
          const float* slot = scales + s * kScaleSlot;
          const float x = slot[quad * 32 + lane] * (kRowScales ? 1.f : slot[128 + half]);
          const u64 x2 = pair_of(__float_as_uint(x), __float_as_uint(x));
          const u32 from = tmem + buf * 256 + half * 128 + (static_cast<u32>(quad * 32) << 16);
          const u32 sw = smem_u32(slot + 128 + half * 128);
          u32 v[2][16];
          t5_ld16(v[0], from);
#pragma unroll
          for (int c = 0; c < 8; ++c) {  // sixteen rows of W: the next ones are on their way while these are added up
            u64 w[8];
            if (kRowScales) {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(w[2 * j]), "=l"(w[2 * j + 1]) : "r"(sw + (c * 16 + j * 4) * 4));
            }
            t5_wait_ld16(v[c & 1]);
            if (c + 1 < 8) {
              t5_ld16(v[(c + 1) & 1], from + (c + 1) * 16);
            } else {  // all out: the buffer is free
              t5_fence_before();
              if (lane == 0) mbar_arrive_at(leader_bar(&b->sums_empty[buf]));
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
              fma2(acc[c * 8 + j], pair_of(v[c & 1][2 * j], v[c & 1][2 * j + 1]), kRowScales ? mul2(w[j], x2) : x2);
          }
        } else {
          t5_fence_before();
          if (lane == 0) mbar_arrive_at(leader_bar(&b->sums_empty[buf]));
        }
        __syncwarp();  // every lane has read its scales: lane 0's arrival speaks for all of them
        if (lane == 0) mbar_arrive(&sb->empty[s]);
      }
      if (ok && some) {
        TO* out = static_cast<TO*>(a.out) + (static_cast<i64>(t.first) + place - lane) * a.out_stride + m;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u32 v[32];
#pragma unroll
          for (int j = 0; j < 16; ++j) asm("mov.b64 {%0, %1}, %2;" : "=r"(v[2 * j]), "=r"(v[2 * j + 1]) : "l"(acc[c * 16 + j]));
          if (a.out_align >= 16 && a.n_m - m - c * 32 >= 32) {
            if (place < t.n) store_run(out + lane * a.out_stride + c * 32, a.out_align, v);
          } else if (m + c * 32 < a.n_m) {
            store_turned(out + c * 32, a.out_stride, t.n - (place - lane), a.n_m - m - c * 32, a.out_align, v);
          }
        }
      }
    }
    if (!ok && lane == 0) route_word_report(a.word);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(48));
    if (kGather) gather_rows<kTileN, 1, true>(a, b, stage0, b->index, off, part, n_tiles, n_mt, threadIdx.x - 384);
  }
  t5_end(tmem);
}

// The same for columns of R with few places: they are the columns again (the instruction's N, 32 or 64), eight buffers of sums and ten stages
// keep W on its way, and a thread has one row of W and up to 32 places, whose scales it reads from shared memory.  512 places in 128 columns of
// 1536 x 4096: 154 us (5.2 TB/s of weights); in 64 columns 98, 125 with tiles of 256 places.
// Warps: 0 copies by tensor map, 1 matrix instructions, 2 hands over what 12-15 copy by index, 3 scales, 4-11 results.
constexpr int kFewSlot = kFewN + 128;
template <bool kGather, bool kRowScales, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGather ? 512 : 384, 1)
    k_route_product_scaled_few(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const ProductArgs a) {
  using S = Shape<kFewN>;
  constexpr int kStages = S::kStages, kStage = S::kStage, kBuffers = S::kBuffers;
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  float* scales = reinterpret_cast<float*>(stages + kStages * kStage);
  T5Block* b = reinterpret_cast<T5Block*>(scales + kScaleSlots * kFewSlot);
  ScaleBlock* sb = reinterpret_cast<ScaleBlock*>(b + 1);
  int* off = reinterpret_cast<int*>(sb + 1);
  int* part = off + a.E + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const u32 rank = cluster_rank();
  if (threadIdx.x == 32)
    for (int i = 0; i < kScaleSlots; ++i) { mbar_init(&sb->full[i], 32); mbar_init(&sb->empty[i], 8); }
  t5_begin(b, kGather ? 3 : 1, 8, 128);
  grid_wait();
  list_parts<kFewN>(a.offsets, a.E, off, part, b->scan_tmp);
  const int n_mt = (a.n_m + kTileM - 1) / kTileM, n_kb = (a.n_k + 127) / 128;
  const u32 n_tiles = static_cast<u32>(part[a.E]) * n_mt;
  const u32 stage0 = smem_u32(stages), scale0 = smem_u32(scales), tmem = b->tmem;
  zero_rows(static_cast<TO*>(a.out), a.out_stride, off[a.E], a.places, a.n_m);

  if (warp == 0) {
    copy_tiles<kFewN, 1, false, kGather, false>(a, &map_w, &map_x, b, stage0, off, part, n_tiles, n_mt);
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      u32 it = 0;
      bool ok = true;
      for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
        const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
        const u32 idesc = t5_idesc(a.type, false, false, kTileM, round32(t.n));
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const u32 s = it % kStages, sw = stage0 + s * kStage, sx = sw + kHalf, buf = it % kBuffers, d = tmem + buf * kFewN;
          ok = t5_wait(&b->sums_empty[buf], ((it / kBuffers) & 1) ^ 1) && t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) t5_mma_f8(d, t5_desc_k(sw + j * 32), t5_desc_k(sx + j * 32), idesc, j > 0);
          t5_commit(&b->empty[s]);
          t5_commit(&b->sums_full[buf]);
        }
      }
      if (!ok) {
        route_word_report(a.word);
        t5_drain_matrix(b);
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    if (kGather && lane == 0) hand_over_rows<kFewN>(a, b, n_tiles, n_kb);
    __syncwarp();
  } else if (warp == 3) {
    u32 it = 0;
    bool ok = true;
    for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
      const int m0 = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM + rank * 128;
      const float* ws = a.ws + static_cast<i64>(t.e) * a.ws_block;
      int row[kFewN / 32];
#pragma unroll
      for (int i = 0; i < kFewN / 32; ++i) {
        const int p = lane + 32 * i;
        row[i] = p < t.n ? (kGather ? a.rows[t.first + p] : t.first + p) : -1;
      }
      for (int kb = 0; kb < n_kb; ++kb, ++it) {
        const u32 s = it % kScaleSlots;
        ok = __all_sync(0xffffffffu, t5_wait(&sb->empty[s], ((it / kScaleSlots) & 1) ^ 1));
        if (!ok) break;
        copy_scales<kFewN, kRowScales>(a, scale0 + s * kFewSlot * 4, row, ws, m0, 128, kb);
        copy_arrive(&sb->full[s]);
      }
    }
    copy_wait_all();
    if (!ok && lane == 0) route_word_report(a.word);
  } else if (warp < 12) {
    const int quad = warp & 3, half = (warp - 4) >> 2;
    u32 it = 0;
    bool ok = true;
    for (u32 id = blockIdx.x >> 1; ok && id < n_tiles; id += gridDim.x >> 1) {
      const Part t = part_at(off, part, a.E, static_cast<int>(id / static_cast<u32>(n_mt)));
      const int m = static_cast<int>(id % static_cast<u32>(n_mt)) * kTileM + rank * 128 + quad * 32 + lane;
      const int each = round32(t.n) / 2, mine = min(each, t.n - half * each);  // places of this warp's half of the columns
      float acc[2][16] = {};
#pragma unroll 1
      for (int kb = 0; kb < n_kb; ++kb, ++it) {
        const u32 buf = it % kBuffers, s = it % kScaleSlots;
        ok = __all_sync(0xffffffffu, t5_wait(&sb->full[s], (it / kScaleSlots) & 1) && t5_wait(&b->sums_full[buf], (it / kBuffers) & 1));
        if (!ok) break;
        t5_fence_after();
        const float* slot = scales + s * kFewSlot;
        const float w = slot[kFewN + (kRowScales ? quad * 32 + lane : 0)];
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (c * 16 < mine) {
            u32 v[16];
            t5_ld16(v, tmem + buf * kFewN + half * each + c * 16 + (static_cast<u32>(quad * 32) << 16));
            t5_wait_ld16(v);
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[c][j] = fmaf(__uint_as_float(v[j]), slot[half * each + c * 16 + j] * w, acc[c][j]);
          }
        t5_fence_before();
        __syncwarp();  // every lane has read its scales: lane 0's arrivals speak for all of them
        if (lane == 0) {
          mbar_arrive_at(leader_bar(&b->sums_empty[buf]));
          mbar_arrive(&sb->empty[s]);
        }
      }
      if (ok) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32 v[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(acc[c][j]);
          if (c * 16 < mine)
            store_places(static_cast<TO*>(a.out), a.out_stride, static_cast<i64>(t.first) + half * each + c * 16, mine - c * 16, m, a.n_m, v);
        }
      }
    }
    if (!ok && lane == 0) route_word_report(a.word);
  } else {
    gather_rows<kFewN, 1, false>(a, b, stage0, b->index, off, part, n_tiles, n_mt, threadIdx.x - 384);
  }
  t5_end(tmem);
}

// Both operands lie with the reduction (64 places a stage) across their rows.  Stages of 64 places of one column come by tensor map (dP, and X
// with a row per place); rows by index, and a column's last places, 16 bytes at a time by eight warps: what lies behind the last place is
// not read but zero, so that a sum ends inside a stage whatever its neighbour holds.
// 16384 places in 8 columns, 4096 x 2048: 217 us (1.27 PFLOP/s), 190 with X by place; 8188 in 32 columns, 1408 x 1024, four stages a sum: 52 us.
// Warps: 0 copies by tensor map, 1 matrix instructions, 2-5 results, 6-13 copies, 14 hands those over.
constexpr int kDwStages = 5;

// A walk over a pair of blocks' tiles of dW, every role's own.  (No division by the tiles of a column on the way: with one, in 64 bits, walking took a role
// 0.9 us a tile.)
struct DwWalk {
  const DwArgs& a;
  const int* off;
  u32 n_mt, n_per, step_e, step_rest;  // tiles along m, tiles of a column, what the pairs' number is in these
  u32 e, rest;
  int p0, p1, m0, j0, half;            // places, first row and column, columns of X per block (128 or 64)
  __device__ __forceinline__ DwWalk(const DwArgs& args, const int* offsets) : a(args), off(offsets) {
    const u32 pairs = gridDim.x >> 1, first = blockIdx.x >> 1;
    n_mt = (a.n_m + kTileM - 1) / kTileM;
    n_per = n_mt * ((a.n_j + kTileN - 1) / kTileN);
    step_e = pairs / n_per;
    step_rest = pairs - step_e * n_per;
    e = first / n_per;
    rest = first - e * n_per;
    look();
  }
  __device__ __forceinline__ bool more() const { return e < static_cast<u32>(a.E); }
  __device__ __forceinline__ void look() {
    if (!more()) return;
    const u32 j = rest / n_mt;
    p0 = off[e];
    p1 = off[e + 1];
    m0 = static_cast<int>(rest - j * n_mt) * kTileM;
    j0 = static_cast<int>(j) * kTileN;
    half = a.n_j - j0 > 128 ? 128 : 64;
  }
  __device__ __forceinline__ void next() {
    e += step_e;
    rest += step_rest;
    if (rest >= n_per) { rest -= n_per; ++e; }
    look();
  }
};

template <bool kGather, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(480, 1)
    k_route_dw(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_out, const DwArgs a) {
  constexpr int kStages = kDwStages;
  extern __shared__ char t5_sm[];
  char* stages = t5_align(t5_sm);
  char* results = stages + kStages * kStage;  // two for each result warp
  T5Block* b = reinterpret_cast<T5Block*>(results + 8 * kOutBytes);
  int* off = reinterpret_cast<int*>(b + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const u32 rank = cluster_rank();
  t5_begin(b, 3, 4, 256);
  grid_wait();
  for (int e = threadIdx.x; e <= a.E; e += blockDim.x) off[e] = static_cast<int>(a.offsets[e]);
  __syncthreads();
  const u32 stage0 = smem_u32(stages), tmem = b->tmem;
  constexpr u32 kBlock = 64 * kRowBytes;  // 64 places of 64 values

  if (warp == 0) {
    if (lane == 0) {
      u32 it = 0;
      bool ok = true;
      for (DwWalk t(a, off); ok && t.more(); t.next()) {
        const int m = t.m0 + rank * 128, j = t.j0 + rank * t.half;
        for (int p = t.p0; p < t.p1; p += 64, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kHalf;
          ok = t5_wait(&b->empty[s], ((it / kStages) & 1) ^ 1);
          if (!ok) break;
          const bool whole = p + 64 <= t.p1;
          if (rank == 0) mbar_arrive_expect_tx(&b->full[s], whole ? 2 * (2 + (kGather ? 0 : t.half / 64)) * kBlock : 0);
          if (whole) {
            const u32 bar = leader_bar(&b->full[s]);
            tma_load_2d(sa, &map_p, m, p, bar);
            tma_load_2d(sa + kBlock, &map_p, m + 64, p, bar);
            if (!kGather) {
              tma_load_2d(sb, &map_x, j, p, bar);
              if (t.half > 64) tma_load_2d(sb + kBlock, &map_x, j + 64, p, bar);
            }
          }
        }
      }
      if (!ok) {
        route_word_report(a.word);
        if (rank == 0) t5_drain_copies<kStages>(b, it);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      u32 it = 0, n_done = 0;
      bool ok = true;
      for (DwWalk t(a, off); ok && t.more(); t.next()) {
        if (t.p0 >= t.p1) continue;
        const u32 idesc = t5_idesc(a.type, true, true, kTileM, 2 * t.half), buf = n_done & 1, d = tmem + buf * kTileN;
        ok = t5_wait(&b->sums_empty[buf], ((n_done >> 1) & 1) ^ 1);
        if (!ok) break;
        t5_fence_after();
        for (int p = t.p0; p < t.p1; p += 64, ++it) {
          const u32 s = it % kStages, sa = stage0 + s * kStage, sb = sa + kHalf;
          ok = t5_wait(&b->full[s], (it / kStages) & 1);
          if (!ok) break;
          t5_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            t5_mma_f16(d, t5_desc_mn(sa + j * 16 * kRowBytes, kBlock), t5_desc_mn(sb + j * 16 * kRowBytes, kBlock), idesc, p > t.p0 || j > 0);
          t5_commit(&b->empty[s]);
        }
        if (ok) t5_commit(&b->sums_full[buf]);
        ++n_done;
      }
      if (!ok) {
        route_word_report(a.word);
        t5_drain_matrix(b);
      }
    }
    __syncwarp();
  } else if (warp == 14) {
    if (lane == 0) {
      u32 it = 0;
      bool ok = true;
      for (DwWalk t(a, off); ok && t.more(); t.next())
        for (int p = t.p0; ok && p < t.p1; p += 64, ++it) ok = hand_over<kStages>(b, it);
      if (!ok) route_word_report(a.word);
    }
    __syncwarp();
  } else if (warp >= 6) {
    // sixteen lanes have a row: 256 bytes of dP, 256 (or 128) of X; a thread the rows r0 + 16 i of a stage
    const int thread = threadIdx.x - 192, c = thread & 15, r0 = thread >> 4;
    const u32 at = (c >> 3) * kBlock + r0 * kRowBytes + (((c & 7) ^ (r0 & 7)) << 4);  // (rows r0 + 16 i: the same swizzle)
    CopyQueue<kStages> queue(b);
    bool ok = true;
    for (DwWalk t(a, off); ok && t.more(); t.next()) {
      const int m = t.m0 + rank * 128 + c * 8, j = t.j0 + rank * t.half + c * 8;
      const u32 m_bytes = 2 * max(0, min(8, a.n_m - m)), j_bytes = 2 * max(0, min(8, a.n_j - j));
      const char* dp = a.dp + (m_bytes ? 2 * static_cast<i64>(m) : 0);
      const char* x = a.x + (j_bytes ? 2 * static_cast<i64>(j) : 0);
      int next[4], after[4];  // rows of X of the next stage and the one behind it
      const auto rows_at = [&](int p, int (&to)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = p + r0 + 16 * i;
          to[i] = q < t.p1 ? (kGather ? a.rows[q] : q) : -1;
        }
      };
      rows_at(t.p0, next);
      rows_at(t.p0 + 64, after);
      for (int p = t.p0; p < t.p1; p += 64) {
        ok = queue.slot_free();
        if (!ok) break;
        const u32 dst = stage0 + queue.issued % kStages * kStage + at;
        const bool whole = p + 64 <= t.p1;
        if ((kGather || !whole) && c * 8 < t.half) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            copy16(dst + kHalf + i * 16 * kRowBytes, next[i] >= 0 ? x + next[i] * a.x_stride : x, next[i] >= 0 ? j_bytes : 0);
        }
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int q = p + r0 + 16 * i;
            copy16(dst + i * 16 * kRowBytes, q < t.p1 ? dp + q * a.dp_stride : dp, q < t.p1 ? m_bytes : 0);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) next[i] = after[i];
        rows_at(p + 128, after);
        queue.done();
      }
    }
    copy_wait_all();
    if (!ok && lane == 0) route_word_report(a.word);
  } else if (warp >= 2) {
    const int quad = warp & 3;
    u32 n_done = 0, run = 0;
    bool ok = true;
    for (DwWalk t(a, off); ok && t.more(); t.next()) {
      const int e = static_cast<int>(t.e), m = t.m0 + rank * 128 + quad * 32 + lane, n = min(kTileN, a.n_j - t.j0);
      TO* out = static_cast<TO*>(a.out) + static_cast<i64>(e) * a.out_block + static_cast<i64>(m - lane) * a.out_stride + t.j0;
      const u32 buf = n_done & 1;
      if (t.p0 < t.p1) {
        ok = __all_sync(0xffffffffu, t5_wait_sum(&b->sums_full[buf], (n_done >> 1) & 1, (t.p1 - t.p0 + 63) / 64));
        if (!ok) break;
        t5_fence_after();
        const u32 sums = tmem + buf * kTileN + (static_cast<u32>(quad * 32) << 16);
        if (a.out_align >= 16) {
          for (int c = 0; c < n; c += kOutRun<TO>) {
            const u32 slot = smem_u32(results) + (quad * 2 + (run & 1)) * kOutBytes;
            if (lane == 0) tma_store_read<1>();
            __syncwarp();
            u32 v[32];
            t5_ld32(v, sums + c);
            t5_wait_ld();
            lay_down<TO, 0>(slot, v);
            if constexpr (sizeof(TO) == 2) {
              t5_ld32(v, sums + c + 32);
              t5_wait_ld();
              lay_down<TO, 32>(slot, v);
            }
            fence_to_matrix();
            __syncwarp();
            if (lane == 0) tma_store_3d(&map_out, t.j0 + c, m - lane, e, slot);
            ++run;
          }
        } else {
          for (int c = 0; c < n; c += 32) {
            u32 v[32];
            t5_ld32(v, sums + c);
            t5_wait_ld();
            store_turned(out + c, a.out_stride, a.n_m - (m - lane), n - c, a.out_align, v);
          }
        }
        t5_fence_before();
        if (lane == 0) mbar_arrive_at(leader_bar(&b->sums_empty[buf]));
        ++n_done;
      } else {  // a column without entries
        for (int r = 0; r < 32 && m - lane + r < a.n_m; ++r)
          if (a.out_align >= 16) {
            for (int c = lane * 8; c < n; c += 256)
              for (int j = 0; j < 8 * static_cast<int>(sizeof(TO)) / 16; ++j)
                if (c + 8 <= n) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(out + r * a.out_stride + c) + 16 * j) = make_uint4(0, 0, 0, 0);
            for (int c = n / 8 * 8 + lane; c < n; c += 32) out[r * a.out_stride + c] = from_float<TO>(0.f);
          } else {
            for (int c = lane; c < n; c += 32) out[r * a.out_stride + c] = from_float<TO>(0.f);
          }
      }
    }
    if (lane == 0) tma_store_done();
    if (!ok && lane == 0) route_word_report(a.word);
  }
  __syncwarp();
  t5_end(tmem);
}

// Copies rows of whole units (of 1 to 8 bytes) into rows that start on 16 bytes, the padding zero.  A warp has a row, four units of a lane in flight.
template <typename T>
__global__ void __launch_bounds__(256) k_route_pack_rows(const T* __restrict__ src, i64 block_stride, i64 row_stride, i64 n_blocks, i64 n_rows, int n_units,
                                                         int padded, T* __restrict__ dst) {
  const int lane = threadIdx.x & 31;
  const i64 step = static_cast<i64>(gridDim.x) * 8;
  grid_launch_next();
  grid_wait();
  for (i64 r = static_cast<i64>(blockIdx.x) * 8 + (threadIdx.x >> 5); r < n_blocks * n_rows; r += step) {
    const i64 blk = r / n_rows;
    const T* from = src + blk * block_stride + (r - blk * n_rows) * row_stride;
    T* to = dst + r * padded;
    for (int c = lane; c < padded; c += 128) {
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = c + 32 * i < n_units ? from[c + 32 * i] : T(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + 32 * i < padded) to[c + 32 * i] = v[i];
    }
  }
}

// The same for any strides: dst (blocks x rows x padded columns).
template <typename T>
__global__ void k_route_pack(const T* __restrict__ src, i64 block_stride, i64 row_stride, i64 col_stride, i64 n_blocks, i64 n_rows,
                             i64 n_cols, i64 padded, T* __restrict__ dst) {
  const i64 total = n_blocks * n_rows * padded;
  grid_launch_next();
  grid_wait();
  for (i64 i = static_cast<i64>(blockIdx.x) * blockDim.x + threadIdx.x; i < total; i += static_cast<i64>(gridDim.x) * blockDim.x) {
    const i64 c = i % padded, br = i / padded, r = br % n_rows, blk = br / n_rows;
    dst[i] = c < n_cols ? src[blk * block_stride + r * row_stride + c * col_stride] : T(0);
  }
}

}  // namespace gm
