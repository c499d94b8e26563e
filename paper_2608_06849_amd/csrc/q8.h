// The 8-bit caches: layout of a unit and the conversions of its codes.
//
// A unit is (page, retrieval KV head) of the paged cache or (sequence, streaming
// KV head, block of 16 slots) of the ring: 16 rows (tokens) of width D.
//   K codes     16 D bytes, [row][D]
//   V codes     16 D bytes, [D / 4][row / 4][4 dims][4 rows]: 4 x 4 tiles
//   scale bytes 32, [row][2] (K, V)
// A row's value is code * 2^(byte - 127); byte 255 with codes 0 is a row of NaN.
//
// The layout is made for 16-byte loads that a wave of the decode pass feeds to
// v_mfma_f32_16x16x32_bf16 without moving anything between lanes: 64
// consecutive bytes of each of 16 K rows a load, and 64 consecutive V tiles,
// of which each gives its lane four dimensions' codes of four tokens.  Codes of
// either format are exact in bf16, and a power-of-two scale multiplies a score or a
// probability without rounding it, so only probabilities and sums are rounded, to fp32.
#pragma once
#include "aoh_device.h"

namespace aoh {

constexpr int kScaleBytes = 2 * kPage;  // of a unit

// 2^(b - 127) of the scale byte b in byte BYTE of w; infinite for 255.  One
// instruction, where the compiler shifts and masks.
template <int BYTE>
__device__ __forceinline__ float scale_of(uint32_t w) {
  static_assert(BYTE >= 0 && BYTE < 4, "byte of a word");
  uint32_t r;
  const uint32_t sh = 23;
  if constexpr (BYTE == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "s"(sh), "v"(w));
  else if constexpr (BYTE == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "s"(sh), "v"(w));
  else if constexpr (BYTE == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "s"(sh), "v"(w));
  else
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "s"(sh), "v"(w));
  return __builtin_bit_cast(float, r);
}

// Offset of the V code of dimension d, row r in its unit.
__device__ __forceinline__ int v_offset(int d, int r) { return ((d >> 2) * 4 + (r >> 2)) * 16 + (d & 3) * 4 + (r & 3); }

// Four codes to bf16, exactly.
template <bool I8>
__device__ __forceinline__ void codes_to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (I8) {
    const uint32_t f0 = __builtin_bit_cast(uint32_t, (float)(int8_t)w);
    const uint32_t f1 = __builtin_bit_cast(uint32_t, (float)(int8_t)(w >> 8));
    const uint32_t f2 = __builtin_bit_cast(uint32_t, (float)(int8_t)(w >> 16));
    const uint32_t f3 = __builtin_bit_cast(uint32_t, (float)(int8_t)(w >> 24));
    // at most 7 bits each: the upper halves of the floats
    lo = __builtin_amdgcn_perm(f1, f0, 0x07060302u);
    hi = __builtin_amdgcn_perm(f3, f2, 0x07060302u);
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
  }
}

// Eight codes as an operand of a matrix instruction.
template <bool I8>
__device__ __forceinline__ bf16x8 codes_operand(uint32_t w0, uint32_t w1) {
  u32x4 r;
  uint32_t lo, hi;
  codes_to_bf16<I8>(w0, lo, hi);
  r[0] = lo;
  r[1] = hi;
  codes_to_bf16<I8>(w1, lo, hi);
  r[2] = lo;
  r[3] = hi;
  return __builtin_bit_cast(bf16x8, r);
}

// Four codes to fp32, exactly.
template <bool I8>
__device__ __forceinline__ f32x4 codes_to_f32(uint32_t w) {
  if constexpr (I8) {
    return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
  } else {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return f32x4{a[0], a[1], b[0], b[1]};
  }
}

// Scale byte of a row whose largest magnitude has the float bits `amax` (NaN and
// infinity have the largest ones): the least E with amax <= c 2^E, c = 448
// (1.75 2^8) or 127 (1.984375 2^6), from -100 on, as E + 127; 255 from 2^127 on.
template <bool I8>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  const int e = (int)(amax >> 23);
  const uint32_t c = I8 ? 0x7e0000u : 0x600000u;  // fraction of c
  const int b = e - (I8 ? 6 : 8) + ((amax & 0x7fffffu) > c ? 1 : 0);
  return e >= 254 ? 255u : (uint32_t)max(b, 27);
}

// The factor 2^-E of a scale byte; 0 for a row of NaN.
__device__ __forceinline__ float inverse_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 255u ? 0u : (254u - byte) << 23);
}

// Four values times 2^-E to codes, to nearest with ties to even.  The scaled
// values do not exceed the largest code, so nothing saturates; rows of NaN give
// codes 0 (`zero`).
template <bool I8>
__device__ __forceinline__ uint32_t to_codes(const float* x, float inv, bool zero) {
  uint32_t w;
  if constexpr (I8) {
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = (uint32_t)(int)rintf(zero ? 0.f : x[i] * inv) & 0xffu;
    w = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = zero ? 0.f : x[i] * inv;
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
    w = (uint32_t)p;
  }
  return w;
}

}  // namespace aoh
