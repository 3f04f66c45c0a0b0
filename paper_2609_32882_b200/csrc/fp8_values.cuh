// Values and scales of the 8-bit form that the quantisation (fp8_quantize.cu) and the norm of the residual stream (residual_norm.cu) write.
#pragma once
#include "common.cuh"

namespace vsa2 {

constexpr uint32_t kInf = 0x7f800000u;
// exponent + 127 from the bits of max|x|: 448 = 1.75 * 2^8, so a fraction above 0.75 carries (at most 254 - 8 + 1)
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) { return (uint32_t)max((int)((top + 0x1fffffu) >> 23) - 8, 0); }
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ uint32_t scale_of(float inverse) { return 254u - (__float_as_uint(inverse) >> 23); }
__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// Blocks where something is not finite are rare: only they look at every value (CHECK).  (An infinity becomes NaN; the conversion alone would make it 448.)
template <bool CHECK>
__device__ __forceinline__ float scaled(float x, float inv) { return !CHECK || finite_bits(x) ? x * inv : __uint_as_float(0x7fffffffu); }
// bytes i .. i+7 of a row of `cols` values (its start 16-byte aligned, i a multiple of 8)
__device__ __forceinline__ void put8(unsigned char* row, int i, int cols, uint32_t lo, uint32_t hi) {
  if (i + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + i) = make_uint2(lo, hi);
  } else {
    for (int j = 0; i + j < cols; ++j) row[i + j] = (unsigned char)((j < 4 ? lo >> 8 * j : hi >> 8 * (j - 4)) & 0xffu);
  }
}
// scale of block kb of row `row` (of a form with `rows` rows and `blocks` blocks a row); the last block clears what is left of its word
__device__ __forceinline__ void put_scale(unsigned char* scales, int rows, int row, int kb, int blocks, uint32_t byte) {
  unsigned char* word = scales + ((size_t)(kb >> 2) * rows + row) * 4;
  word[kb & 3] = (unsigned char)byte;
  if (kb == blocks - 1)
    for (int j = (kb & 3) + 1; j < 4; ++j) word[j] = 0;
}

}  // namespace vsa2
