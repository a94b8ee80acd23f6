// Number formats of the low-precision operators.
//
// 8-bit operands: float8 e4m3 codes with a power-of-two scale (one E8M0 byte b, 2^(b - 127)) for
// 128 consecutive columns of a row.  A power of two because the tensor core then applies the
// scales itself (kind::mxf8f6f4) and because scaling by it rounds nothing: a code is the e4m3
// rounding of the element.  Cache rows: integer codes with a bf16 scale, whose uniform steps lose
// a third of e4m3's error on Gaussian data (0.7 % against 2.6 %) where no tensor core reads them.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace bag {

constexpr int kScaleBlock = 128;        // columns of one scale of an 8-bit operand
constexpr uint32_t kInfBits = 0x7f800000u;

BAG_DEV uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Largest |x| of a group of W neighbouring lanes, as bits (an infinity or NaN is >= kInfBits).
template <int W>
BAG_DEV uint32_t group_max(uint32_t m) {
  if constexpr (W == 32) {
    return __reduce_max_sync(0xffffffffu, m);
  } else {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
  }
}

// Scale byte of a block with the largest magnitude `amax` (bits): the least b >= 0 with
// amax <= 448 * 2^(b - 127).  448 = 1.75 * 2^8, so b is amax's exponent - 8, one more where its
// significand is above 1.75: there the sum carries into the exponent.
BAG_DEV uint32_t e8m0_of(uint32_t amax) {
  const uint32_t b = max((amax + 0x1fffffu) >> 23, 8u) - 8u;
  return amax >= kInfBits ? 255u : b;
}

// 1 / scale of byte b <= 247 (exact); NaN for 255, which makes every code of the block NaN.
BAG_DEV float e8m0_inverse(uint32_t b) { return b == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float((254u - b) << 23); }

// Four e4m3 codes, the first in the lowest byte (nearest, ties to even).
BAG_DEV uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// n <= 4 bytes of `v`, the lowest first, to p (4-byte aligned).
BAG_DEV void store_bytes(uint8_t* p, uint32_t v, int n) {
  if (n >= 4) {
    *reinterpret_cast<uint32_t*>(p) = v;
  } else {
    for (int i = 0; i < n; ++i) p[i] = (uint8_t)(v >> (8 * i));
  }
}

// Two fp32 operations in one instruction.
BAG_DEV float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
BAG_DEV float2 sum2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
BAG_DEV float2 muladd2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

// GELU (tanh form) of two values: y / (1 + exp(-2u)), u = sqrt(2/pi) (y + 0.044715 y^3), the same
// function as 0.5 y (1 + tanh u).  exp2 and the reciprocal of the special-function unit: relative
// error up to 2^-20, and for negative y what the rounding of the exponent x adds, up to |x| 1.75 2^-23
// (2^-17 at y = -6, where the value is -8e-11 and 1 + tanh u in fp32 has no bit left): below the
// roundings to 16 and 8 bits that follow, and below fp32's own at the sums this is applied to.  (A power
// that overflows gives 1 / inf = 0.)
BAG_DEV float2 gelu2(float2 y) {
  const float k = -2.0f * 0.7978845608028654f * 1.4426950408889634f;  // exp(-2u) = 2^(y (k + k' y^2))
  float2 e = mul2(y, muladd2(mul2(y, y), make_float2(k * 0.044715f, k * 0.044715f), make_float2(k, k)));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
  e = sum2(e, make_float2(1.f, 1.f));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.x));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.y));
  return mul2(y, e);
}

// Largest magnitude of three values (a NaN if there is one).
BAG_DEV float max3_abs(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

}  // namespace bag
