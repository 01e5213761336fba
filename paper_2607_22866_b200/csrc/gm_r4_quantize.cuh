// Blocks of 1 x 128 or 128 x 128 values to e4m3 with a scale each.
//
//   s = max(largest finite |x|, 2^-100) / 448,   q = x / s, rounded to the nearest value of e4m3 (ties to the even one)
//
// A value that is not finite becomes NaN (e4m3 has no infinity) and leaves its block's scale alone.  Bound by memory: 16-bit values
// are read once and kept in registers between the maximum and the rounding.
#pragma once
#include <cuda_fp8.h>

#include "gm_r3_sum.cuh"

namespace gm {

constexpr float kQuantLeast = 7.888609052210118e-31f;  // 2^-100: 448 over it is finite

// x / s for 16-bit x with inv = 448 / largest: the product is within 2 units of 2^-23 of the quotient.  x and the largest have at most 11
// significant bits, so a quotient that is no border between two values of e4m3 (5 bits) is at least 2^-16 away from one, and one that
// is a border has at most 5 significant bits itself: rounded to 20 bits, neither ends up on a wrong side, and the rounding to e4m3
// gives what the exact quotient would, ties included.
__device__ __forceinline__ float quant_ratio(float x, float inv) {
  return __uint_as_float((__float_as_uint(x * inv) + 8u) & ~15u);
}
__device__ __forceinline__ u32 quant_pack4(float a, float b, float c, float d) {
  const u32 lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const u32 hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
// |x| where it is finite, else 0
__device__ __forceinline__ float quant_abs(float x) {
  const float v = fabsf(x);
  return v <= 3.4028234663852886e38f ? v : 0.f;
}
// not finite -> NaN, which the conversion keeps (an infinity times the inverse scale would saturate)
__device__ __forceinline__ float quant_value(float x, float inv) {
  const float v = fabsf(x);
  return v <= 3.4028234663852886e38f ? quant_ratio(x, inv) : __uint_as_float(0x7fffffffu);
}

struct QuantArgs {
  const void* x;
  i64 x_block, x_row, x_col;   // strides in elements
  i64 n_blocks, n_rows;
  int n_cols, col_groups;
  u32* q;                      // contiguous; bytes when the width is no multiple of eight
  float* s;
};

// kVec: rows of x are 16-byte aligned, contiguous, and a multiple of eight wide.
template <typename T, bool kVec>
__device__ __forceinline__ void quant_load(const T* row, i64 col_stride, int c, int n_cols, float (&v)[8]) {
  if (kVec) {
    if (c < n_cols) Vec8<T>::load(row + c, v);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n_cols ? static_cast<float>(row[(c + i) * col_stride]) : 0.f;
  }
}
template <bool kVec>
__device__ __forceinline__ void quant_store(unsigned char* row, int c, int n_cols, const float (&v)[8], float inv) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = quant_value(v[i], inv);
  const uint2 q = make_uint2(quant_pack4(w[0], w[1], w[2], w[3]), quant_pack4(w[4], w[5], w[6], w[7]));
  if (kVec) {
    if (c < n_cols) *reinterpret_cast<uint2*>(row + c) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n_cols) row[c + i] = static_cast<unsigned char>((i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) & 0xff);
  }
}

// Rows: sixteen lanes have a block of 128 values.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) k_quantize_rows(const QuantArgs a) {
  const i64 unit = static_cast<i64>(blockIdx.x) * 16 + (threadIdx.x >> 4);
  const int l = threadIdx.x & 15;
  const i64 rows = a.n_blocks * a.n_rows;
  const bool in = unit < rows * a.col_groups;
  const i64 row = in ? unit / a.col_groups : 0;
  const int c = in ? static_cast<int>(unit % a.col_groups) * 128 + l * 8 : a.n_cols;
  const T* x = static_cast<const T*>(a.x) + (row / a.n_rows) * a.x_block + (row % a.n_rows) * a.x_row;
  float v[8];
  quant_load<T, kVec>(x, a.x_col, c, a.n_cols, v);
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = fmaxf(most, quant_abs(v[i]));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  most = fmaxf(most, kQuantLeast);
  if (!in) return;
  quant_store<kVec>(reinterpret_cast<unsigned char*>(a.q) + row * a.n_cols, c, a.n_cols, v, 448.f / most);
  if (l == 0) a.s[unit] = most / 448.f;
}

// Tiles of 128 x 128: a thread has eight columns of eight rows.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256) k_quantize_tiles(const QuantArgs a, int row_groups) {
  __shared__ float warp_most[8];
  const i64 unit = blockIdx.x;
  const int cg = static_cast<int>(unit % a.col_groups);
  const i64 br = unit / a.col_groups;
  const i64 blk = br / row_groups, r0 = br % row_groups * 128;
  const int c = cg * 128 + (threadIdx.x & 15) * 8, r = threadIdx.x >> 4;
  const T* x = static_cast<const T*>(a.x) + blk * a.x_block;
  float v[8][8];
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const i64 row = r0 + r + 16 * j;
    quant_load<T, kVec>(x + (row < a.n_rows ? row : 0) * a.x_row, a.x_col, row < a.n_rows ? c : a.n_cols, a.n_cols, v[j]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, quant_abs(v[j][i]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if ((threadIdx.x & 31) == 0) warp_most[threadIdx.x >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) most = fmaxf(most, warp_most[i]);
  most = fmaxf(most, kQuantLeast);
  const float inv = 448.f / most;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const i64 row = r0 + r + 16 * j;
    if (row < a.n_rows)
      quant_store<kVec>(reinterpret_cast<unsigned char*>(a.q) + (blk * a.n_rows + row) * a.n_cols, c, a.n_cols, v[j], inv);
  }
  if (threadIdx.x == 0) a.s[unit] = most / 448.f;
}

}  // namespace gm
