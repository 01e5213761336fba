// Sums over the entries of a row of R, and their gradients (R times dense rows, and the product sampled at R's entries).
//
//   k_route_sum        Y[i,:] = sum over the entries q of row i of r_q * P[pos[q],:]
//   k_route_sum_grads  dP[pos[q],:] = r_q * dY[i,:],   dr_q = <dY[i,:], P[pos[q],:]>
//
// Both are bound by memory: P is read once (and dP written once), a row of Y or dY serves all entries of its row of R.  Sums are kept
// in 32 bits, in the order of the row's entries, and rounded once.
#pragma once
#include "gm_route_product.cuh"

namespace gm {

template <typename T> struct Vec8;  // eight consecutive values as floats
template <> struct Vec8<float> {
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <> struct Vec8<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const u32 w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint4 a;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&a);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = a;
  }
};
template <> struct Vec8<__half> {
  static __device__ __forceinline__ void load(const __half* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const __half2* h = reinterpret_cast<const __half2*>(&a);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(h[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(__half* p, const float (&v)[8]) {
    uint4 a;
    __half2* h = reinterpret_cast<__half2*>(&a);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = a;
  }
};

// kVec: rows are 16-byte aligned and a multiple of eight wide; a thread then has 16 bytes of columns at a time, else one column.
template <typename T, bool kVec>
__device__ __forceinline__ void store_cols(T* p, const float (&v)[8]) {
  if (kVec) Vec8<T>::store(p, v);
  else *p = from_float<T>(v[0]);
}

// A thread's columns as they lie in memory, so that many loads can be under way in few registers.
template <typename T, bool kVec> struct Raw {
  using type = T;
  static __device__ __forceinline__ type load(const T* p) { return *p; }
  static __device__ __forceinline__ void values(const type& r, float (&v)[8]) { v[0] = static_cast<float>(r); }
};
template <typename T> struct Raw<T, true> {  // 16 bytes
  struct alignas(16) type { T v[16 / sizeof(T)]; };
  static __device__ __forceinline__ type load(const T* p) {
    type r;
    *reinterpret_cast<uint4*>(&r) = __ldcs(reinterpret_cast<const uint4*>(p));
    return r;
  }
  static __device__ __forceinline__ void values(const type& r, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = r.v[i];
    } else {
      Vec8<T>::load(r.v, v);
    }
  }
};
template <typename T> __device__ __forceinline__ void store4(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    struct alignas(8) { T t[4]; } w = {{from_float<T>(v[0]), from_float<T>(v[1]), from_float<T>(v[2]), from_float<T>(v[3])}};
    *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(&w);
  }
}

struct SumArgs {
  const i64* row_ptr;
  const float* val;       // nullptr: every entry counts once
  const i64* offsets;
  const int32_t* rows;    // by place
  const int32_t* pos;     // by entry
  int E;
  i64 entries;
  int width;
  const void* p;
  i64 p_stride;
  void* y;
  i64 y_stride;
};

// A thread has sixteen columns: two runs of eight 16-bit values, or four of four floats, whatever the rows' length.  65536 entries of 2048 bf16 values in
// rows of 1, 2, 8 entries: 140, 84, 56 us; with eight columns 301, 158, 61, with 32 columns 172, 100, 66.  Floats: 190, 127, 98 us; with eight columns 267,
// 172, 100, with 32 columns 209, 148, 105.
template <typename TI, bool kVec> constexpr int kSumUnits = kVec ? sizeof(TI) : 8;

// kUnits: runs of columns per thread, a block's threads apart; eight loads of 16 bytes (or sixteen of one value) are in flight, for as many
// entries as that leaves.
template <typename TI, typename TO, bool kVec, int kUnits, int kThreads>
__global__ void __launch_bounds__(kThreads) k_route_sum(const SumArgs a, int n_chunks) {
  constexpr int kCols = kVec ? 16 / sizeof(TI) : 1, kEntries = (kVec ? 8 : 16) / kUnits, step = kThreads * kCols;
  const i64 i = blockIdx.x / n_chunks;
  const int c = static_cast<int>(blockIdx.x % n_chunks) * kUnits * step + threadIdx.x * kCols;
  grid_launch_next();
  if (c >= a.width) return;
  grid_wait();
  const i64 q0 = max(static_cast<i64>(0), a.row_ptr[i]), q1 = min(a.entries, a.row_ptr[i + 1]);
  const int routed = static_cast<int>(a.offsets[a.E]);
  const TI* p = static_cast<const TI*>(a.p) + c;
  float acc[kUnits][8] = {};
  for (i64 q = q0; q < q1; q += kEntries) {  // places first, then values, then sums
    int at[kEntries];
    float r[kEntries];
#pragma unroll
    for (int j = 0; j < kEntries; ++j) {
      const bool in = q + j < q1;
      at[j] = in ? a.pos[q + j] : INT_MAX;
      r[j] = in && a.val ? a.val[q + j] : 1.f;
    }
    typename Raw<TI, kVec>::type v[kEntries][kUnits];
#pragma unroll
    for (int j = 0; j < kEntries; ++j)
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        if (at[j] < routed && c + u * step < a.width) v[j][u] = Raw<TI, kVec>::load(p + at[j] * a.p_stride + u * step);
#pragma unroll
    for (int j = 0; j < kEntries; ++j)
      if (at[j] < routed) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          float f[8];
          Raw<TI, kVec>::values(v[j][u], f);
#pragma unroll
          for (int x = 0; x < kCols; ++x) acc[u][x] = fmaf(r[j], f[x], acc[u][x]);
        }
      }
  }
  TO* y = static_cast<TO*>(a.y) + i * a.y_stride + c;
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
    if (c + u * step < a.width) {
      if constexpr (kCols == 4) store4(y + u * step, acc[u]);
      else store_cols<TO, kVec>(y + u * step, acc[u]);
    }
}

// A warp per entry, in the order of the rows of R (so that a row's entries share its row of dY in cache).
template <typename T, typename TD, bool kVec>
__global__ void __launch_bounds__(256) k_route_sum_grads(const SumArgs a, TD* __restrict__ dp, i64 dp_stride, float* __restrict__ dval) {
  const int lane = threadIdx.x & 31;
  const i64 q = static_cast<i64>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
  grid_launch_next();
  if (q >= a.entries) return;
  grid_wait();
  const int at = a.pos[q];
  TD* out = dp + at * dp_stride;
  if (at >= a.offsets[a.E]) {  // routed nowhere
    for (int c = lane; c < a.width; c += 32) out[c] = from_float<TD>(0.f);
    if (lane == 0) dval[q] = 0.f;
    return;
  }
  const float r = a.val[q];
  const T* dy = static_cast<const T*>(a.y) + a.rows[at] * a.y_stride;
  const T* p = static_cast<const T*>(a.p) + at * a.p_stride;
  // four runs of columns of both rows in flight (110 us without, 96 us with them, at 44231 x 2880)
  using R = Raw<T, kVec>;
  constexpr int kCols = kVec ? 16 / sizeof(T) : 1, step = 32 * kCols, kRuns = 4;
  float dot = 0.f;
  for (int c = lane * kCols; c < a.width; c += step * kRuns) {
    typename R::type graw[kRuns], vraw[kRuns];
#pragma unroll
    for (int u = 0; u < kRuns; ++u)
      if (c + u * step < a.width) {
        graw[u] = *reinterpret_cast<const typename R::type*>(dy + c + u * step);  // (other entries of the row read it too)
        vraw[u] = R::load(p + c + u * step);
      }
#pragma unroll
    for (int u = 0; u < kRuns; ++u)
      if (c + u * step < a.width) {
        float g[8], v[8];
        R::values(graw[u], g);
        R::values(vraw[u], v);
#pragma unroll
        for (int x = 0; x < kCols; ++x) {
          dot = fmaf(g[x], v[x], dot);
          g[x] *= r;
        }
        if constexpr (kCols == 4) store4(out + c + u * step, g);
        else store_cols<TD, kVec>(out + c + u * step, g);
      }
  }
  dot = warp_sum(dot);
  if (lane == 0) dval[q] = dot;
}

}  // namespace gm
