// The 8-bit cache format: OCP e4m3 codes with a power-of-two scale byte E
// (value = code * 2^(E - 127)) for each block of scale_rows rows and kv head.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ltd_device.hpp"

namespace ltd {

constexpr float kQ8Max = 448.f;             // largest code
constexpr int kQ8MinByte = 27;              // 2^-100: every value of a block is exact in bf16 ...
constexpr int kQ8MaxByte = 214;             // 2^87: ... and sums under softmax weights stay finite in fp32
constexpr uint32_t kQ8Mantissa448 = 0x600000u;  // fraction bits of 448 = 1.75 * 2^8

// 2^(byte - 127) for a byte in [1, 254].
__device__ __forceinline__ float q8_scale(int byte) {
  return __uint_as_float(static_cast<uint32_t>(byte) << 23);
}

// The smallest scale byte in range under which `amax` (>= 0) is at most 448:
// amax = 1.m * 2^x needs 2^(x - 8), and twice that when 1.m > 1.75.
__device__ __forceinline__ int q8_needed_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7FFFFFu) > kQ8Mantissa448 ? 1 : 0);
  return min(max(e, kQ8MinByte), kQ8MaxByte);
}

// Two codes' values (kHigh picks the upper or the lower half of the word).
typedef float q8_f32x2 __attribute__((ext_vector_type(2)));
template <bool kHigh>
__device__ __forceinline__ q8_f32x2 q8_decode2(uint32_t codes) {
  return __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), kHigh);
}

// x limited to the codes' range; NaN stays NaN.
__device__ __forceinline__ float q8_limit(float x) {
  return x != x ? x : fminf(fmaxf(x, -kQ8Max), kQ8Max);
}

// Four values as codes, rounded to nearest even.
__device__ __forceinline__ uint32_t q8_encode4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(q8_limit(a), q8_limit(b), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(q8_limit(c), q8_limit(d), r, true);
  return static_cast<uint32_t>(r);
}

// Four codes of scale byte `from` as codes of scale byte `to` >= from, given
// shift = 2^(from - to) (0 where that is below float32's normal range: every
// code then rounds to zero).
__device__ __forceinline__ float q8_shift(int from, int to) {
  return __uint_as_float(static_cast<uint32_t>(max(127 + from - to, 0)) << 23);
}
__device__ __forceinline__ uint32_t q8_rescale4(uint32_t codes, float shift) {
  const q8_f32x2 lo = q8_decode2<false>(codes), hi = q8_decode2<true>(codes);
  return q8_encode4(lo.x * shift, lo.y * shift, hi.x * shift, hi.y * shift);
}

// Physical page, row in the page and scale index of a logical cache row.
struct Q8Row {
  int64_t page;  // sequence (contiguous) or block id (paged)
  int row;       // row within it
};
__device__ __forceinline__ Q8Row q8_row(const int32_t* __restrict__ block_table, int b, int row,
                                        int kv_rows, int max_blocks) {
  if (block_table == nullptr) return Q8Row{b, row};
  return Q8Row{block_table[static_cast<int64_t>(b) * max_blocks + row / kv_rows], row % kv_rows};
}

}  // namespace ltd
