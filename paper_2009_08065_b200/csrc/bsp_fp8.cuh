// What the 8-bit calls share: the format of values and scales, and operands of a matrix product in that form.
//
// A value is e4m3 or e5m2 (bsp_fp8_format); the scale of a block is a power of two, held as its exponent plus 127 in a byte: the
// smallest that brings the block's largest magnitude to at most 448 = 1.75 * 2^8 (e4m3) or 57344 = 1.75 * 2^15 (e5m2).  Powers
// of two: dividing by one is exact, so a value is rounded once, the same on every route, and a value that is brought to 8
// bits again stays as it is; floating-point values lose no precision by it (only range at the lower end, 2^17 below the
// block's largest); and the tensor core takes such scales beside its operands.
#pragma once

#include "bsp_common.cuh"

namespace bsp {
namespace fp8 {

constexpr int kBlock = 128;                  // values that share a scale along the contraction
constexpr uint32_t kNan = 0x7fu;             // NaN in both formats

// An operand of out[i, j] = sum_k A(i, k) B(j, k): `rows` rows i, values along k next to each other or (mn) ld bytes apart;
// scale of (i, k) at s[(i >> s_shift) * s_row + (k / 128) * s_k].
struct Operand {
  const uint8_t* q;
  int rows, ld, mn, fmt;
  const uint8_t* s;
  long long s_row, s_k;
  int s_shift;
};

__host__ __device__ constexpr int blocks_of(int n) { return (n - 1) / kBlock + 1; }      // n >= 1 (up to the largest int)
// Largest size in any direction: the kernels count up to a tile beyond it.
constexpr int kMostSize = 0x7ffffe00;
inline bool known_format(int fmt) { return fmt == BSP_FP8_E4M3 || fmt == BSP_FP8_E5M2; }

#ifdef __CUDACC__
// Scale byte for a largest magnitude given as float32 bits (finite).
__device__ __forceinline__ int scale_byte(uint32_t amax_bits, int top) {
  const int e = static_cast<int>(amax_bits >> 23) - top + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, 0);
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte != 0u ? byte << 23 : 0x400000u); }
// 1 / scale, for bytes that scale_byte gives (at most 254 - 8 + 1).
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float(static_cast<uint32_t>(254 - byte) << 23); }
__host__ __device__ constexpr int top_of(int fmt) { return fmt == BSP_FP8_E4M3 ? 8 : 15; }

// The two values of the lower half, the first in the lower byte.
template <int FMT>
__device__ __forceinline__ void from_fp8x2(uint32_t two, float& lo, float& hi) {
  uint32_t h;
  if (FMT == BSP_FP8_E4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  else asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
}
// Four values, the first in the lowest byte.
template <int FMT>
__device__ __forceinline__ uint32_t to_fp8x4(float x0, float x1, float x2, float x3) {
  uint32_t r;
  if (FMT == BSP_FP8_E4M3)
    asm("{\n\t.reg .b16 l, u;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 u, %4, %3;\n\tmov.b32 %0, {l, u};\n\t}"
        : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  else
    asm("{\n\t.reg .b16 l, u;\n\tcvt.rn.satfinite.e5m2x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e5m2x2.f32 u, %4, %3;\n\tmov.b32 %0, {l, u};\n\t}"
        : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  return r;
}
// The larger magnitudes of two pairs of bf16 values, NaN where there is one (signs are left undefined).
__device__ __forceinline__ uint32_t abs_max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The larger magnitude of a pair, as 16 bits.
__device__ __forceinline__ uint32_t abs_max_of(uint32_t a) { return max((a >> 16) & 0x7fffu, a & 0x7fffu); }
// Scale byte and multiplier of a block whose largest magnitude has these 16 bits.  A block with an infinity or a NaN gets scale 1 and
// the multiplier NaN, which makes every value the NaN code.
template <int FMT>
__device__ __forceinline__ uint32_t block_scale(uint32_t amax16, float& inv) {
  const bool bad = amax16 >= 0x7f80u;
  const int byte = bad ? 127 : scale_byte(amax16 << 16, top_of(FMT));
  inv = bad ? __uint_as_float(0x7fffffffu) : scale_inverse(byte);
  return static_cast<uint32_t>(byte);
}
// Four values times their multipliers as 8 bits.
template <int FMT>
__device__ __forceinline__ uint32_t four_to_fp8(uint32_t x0, uint32_t x1, float i0, float i1, float i2, float i3) {
  return to_fp8x4<FMT>(__uint_as_float(x0 << 16) * i0, __uint_as_float(x0 & 0xffff0000u) * i1, __uint_as_float(x1 << 16) * i2,
                       __uint_as_float(x1 & 0xffff0000u) * i3);
}
#endif

}  // namespace fp8
}  // namespace bsp
