// Blocks of 1 x 128 or 128 x 128 values to e4m3 with a scale each.
//
//   s = max(largest finite |x|, 2^-100) / 448,   q = x / s, rounded to the nearest value of e4m3 (ties to the even one)
//
// A value that is not finite becomes NaN (e4m3 has no infinity) and leaves its block's scale alone.  Bound by memory: 16-bit values
// are read once and wait in registers, as they came, between the maximum and the rounding.  The maximum is one of 16-bit integers (the
// magnitudes' bit patterns are in their order, what is not finite above all that is), two at a time: with floats, 16 x 2048 x 4096 values in tiles
// took 211 us, 73 so (5.5 TB/s; 0.84 of what a copy reaches); in rows 75.
#pragma once
#include <cuda_fp8.h>

#include "gm_route_sum.cuh"

namespace gm {

constexpr float kQuantLeast = 7.888609052210118e-31f;  // 2^-100: 448 over it is finite

template <typename T> struct Half16;  // bit pattern of the smallest magnitude that is not finite, two values to floats
template <> struct Half16<__nv_bfloat16> {
  static constexpr u32 kInf = 0x7f80;
  static __device__ __forceinline__ float2 floats(u32 w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
};
template <> struct Half16<__half> {
  static constexpr u32 kInf = 0x7c00;
  static __device__ __forceinline__ float2 floats(u32 w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
};

// x / s for 16-bit x with inv = 448 / largest: the product is within 2 units of 2^-23 of the quotient.  x and the largest have at most 11
// significant bits, so a quotient that is no border between two values of e4m3 (5 bits) is at least 2^-16 away from one, and one that
// is a border has at most 5 significant bits itself: rounded to 20 bits, neither ends up on a wrong side, and the rounding to e4m3
// gives what the exact quotient would, ties included.
__device__ __forceinline__ float quant_ratio(float x, float inv) {
  return __uint_as_float((__float_as_uint(x * inv) + 8u) & ~15u);
}
__device__ __forceinline__ u32 quant_pack2(float2 v) { return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3); }

// Eight values, two in a word.  kMixed: some may not be finite.
template <typename T, bool kMixed>
__device__ __forceinline__ uint2 quant_eight(const uint4& x, float inv) {
  const u32 w[4] = {x.x, x.y, x.z, x.w};
  u32 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = Half16<T>::floats(w[i]);
    float2 r = make_float2(quant_ratio(f.x, inv), quant_ratio(f.y, inv));
    if (kMixed) {
      const float nan = __uint_as_float(0x7fffffffu);
      if ((w[i] & 0x7fffu) >= Half16<T>::kInf) r.x = nan;
      if (((w[i] >> 16) & 0x7fffu) >= Half16<T>::kInf) r.y = nan;
    }
    q[i] = quant_pack2(r);
  }
  return make_uint2(q[0] | (q[1] << 16), q[2] | (q[3] << 16));
}
// the larger magnitudes' bit patterns, in either half of the word
__device__ __forceinline__ u32 quant_most(const uint4& x, u32 most) {
  constexpr u32 kAbs = 0x7fff7fffu;
  most = __vmaxu2(most, __vmaxu2(x.x & kAbs, x.y & kAbs));
  return __vmaxu2(most, __vmaxu2(x.z & kAbs, x.w & kAbs));
}
// the same of the finite ones alone
template <typename T>
__device__ __forceinline__ u32 quant_most_finite(const uint4& x, u32 most) {
  const u32 w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32 lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    most = __vmaxu2(most, (lo < Half16<T>::kInf ? lo : 0u) | (hi < Half16<T>::kInf ? hi << 16 : 0u));
  }
  return most;
}
__device__ __forceinline__ u32 quant_larger_half(u32 most) { return max(most & 0xffffu, most >> 16); }
template <typename T>
__device__ __forceinline__ float quant_largest(u32 bits) { return fmaxf(Half16<T>::floats(bits).x, kQuantLeast); }

struct QuantArgs {
  const void* x;
  i64 x_block, x_row, x_col;   // strides in elements
  i64 n_blocks, n_rows;
  int n_cols, col_groups;
  unsigned char* q;            // contiguous
  float* s;
};

// kVec: rows of x start on 16 bytes, are contiguous, and a multiple of eight wide.
template <typename T, bool kVec>
__device__ __forceinline__ uint4 quant_load(const T* row, i64 col_stride, int c, int n_cols) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (kVec) {
    if (c < n_cols) v = __ldcs(reinterpret_cast<const uint4*>(row + c));
  } else {
    const uint16_t* x = reinterpret_cast<const uint16_t*>(row);
    u32 w[4] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n_cols) w[i >> 1] |= static_cast<u32>(x[(c + i) * col_stride]) << (16 * (i & 1));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}
template <bool kVec>
__device__ __forceinline__ void quant_store(unsigned char* row, int c, int n_cols, uint2 q) {
  if (kVec) {
    if (c < n_cols) *reinterpret_cast<uint2*>(row + c) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n_cols) row[c + i] = static_cast<unsigned char>((i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) & 0xff);
  }
}

// Rows: sixteen lanes have a block of 128 values, and four such blocks in flight.
// kFlat: rows are a multiple of 128 wide and follow each other without gaps, so that a block's number is its address.
constexpr int kQuantAhead = 4;
template <typename T, bool kVec, bool kFlat>
__global__ void __launch_bounds__(256) k_quantize_rows(const QuantArgs a) {
  const int l = threadIdx.x & 15;
  const i64 units = a.n_blocks * a.n_rows * a.col_groups, first = static_cast<i64>(blockIdx.x) * 16 * kQuantAhead + (threadIdx.x >> 4);
  uint4 x[kQuantAhead];
  unsigned char* to[kQuantAhead];
  int col[kQuantAhead];
  grid_launch_next();
  grid_wait();
#pragma unroll
  for (int j = 0; j < kQuantAhead; ++j) {
    const i64 unit = first + 16 * j;
    if (kFlat) {
      col[j] = unit < units ? 0 : a.n_cols;
      to[j] = a.q + unit * 128 + l * 8;
      x[j] = quant_load<T, kVec>(static_cast<const T*>(a.x) + unit * 128 + l * 8, 1, col[j], a.n_cols);
    } else {
      const i64 row = unit < units ? unit / a.col_groups : 0;
      col[j] = unit < units ? static_cast<int>(unit - row * a.col_groups) * 128 + l * 8 : a.n_cols;
      to[j] = a.q + row * a.n_cols;
      x[j] = quant_load<T, kVec>(static_cast<const T*>(a.x) + row / a.n_rows * a.x_block + row % a.n_rows * a.x_row, a.x_col, col[j], a.n_cols);
    }
  }
#pragma unroll
  for (int j = 0; j < kQuantAhead; ++j) {
    u32 most = quant_most(x[j], 0);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, o));
    most = quant_larger_half(most);
    const bool mixed = most >= Half16<T>::kInf;
    if (__any_sync(0xffffffffu, mixed)) {
      u32 fin = quant_most_finite<T>(x[j], 0);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) fin = __vmaxu2(fin, __shfl_xor_sync(0xffffffffu, fin, o));
      if (mixed) most = quant_larger_half(fin);
    }
    const float largest = quant_largest<T>(most), inv = 448.f / largest;
    const uint2 q = mixed ? quant_eight<T, true>(x[j], inv) : quant_eight<T, false>(x[j], inv);
    quant_store<kVec>(to[j], col[j], a.n_cols, q);
    const i64 unit = first + 16 * j;
    if (l == 0 && unit < units) a.s[unit] = largest / 448.f;
  }
}

// Tiles of 128 x 128: a thread has eight columns of eight rows.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) k_quantize_tiles(const QuantArgs a, int row_groups) {
  __shared__ u32 warp_most[2][8];
  const u32 unit = blockIdx.x, cg = unit % a.col_groups, br = unit / a.col_groups;
  const i64 blk = br / row_groups, r0 = static_cast<i64>(br % row_groups) * 128;
  const int c = cg * 128 + (threadIdx.x & 15) * 8, r = threadIdx.x >> 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* x = static_cast<const T*>(a.x) + blk * a.x_block;
  uint4 v[8];
  grid_launch_next();
  grid_wait();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const i64 row = r0 + r + 16 * j;
    v[j] = quant_load<T, kVec>(x + (row < a.n_rows ? row : 0) * a.x_row, a.x_col, row < a.n_rows ? c : a.n_cols, a.n_cols);
  }
  u32 most = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) most = quant_most(v[j], most);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (lane == 0) warp_most[0][warp] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) most = __vmaxu2(most, warp_most[0][i]);
  most = quant_larger_half(most);
  const bool mixed = most >= Half16<T>::kInf;  // the same for all threads
  if (mixed) {
    u32 fin = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) fin = quant_most_finite<T>(v[j], fin);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) fin = __vmaxu2(fin, __shfl_xor_sync(0xffffffffu, fin, o));
    if (lane == 0) warp_most[1][warp] = fin;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) fin = __vmaxu2(fin, warp_most[1][i]);
    most = quant_larger_half(fin);
  }
  const float largest = quant_largest<T>(most), inv = 448.f / largest;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const i64 row = r0 + r + 16 * j;
    if (row < a.n_rows)
      quant_store<kVec>(a.q + (blk * a.n_rows + row) * a.n_cols, c, a.n_cols, mixed ? quant_eight<T, true>(v[j], inv) : quant_eight<T, false>(v[j], inv));
  }
  if (threadIdx.x == 0) a.s[unit] = largest / 448.f;
}

}  // namespace gm
