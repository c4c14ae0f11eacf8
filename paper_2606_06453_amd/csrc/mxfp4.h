// The 4-bit cache type (VX_KV_MXFP4): E2M1 codes (magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6), one E8M0
// scale 2^(E - 127) per group of 32 channels of a token, E = 255 for a NaN group.
//
// A (page, KV head) slice is ps * D / 2 bytes of codes, then ps * D / 32 bytes of scales.  The order
// inside a slice is that of the attention's matrix operands:
//   K  codes [token][D / 2], the even channel in the low nibble; scales [token][D / 32].  An operand
//      of S^T = K Q^T is D / 4 consecutive channels of one token: one load of 16 bytes (D = 128) and
//      one scale.
//   V  codes [token / 4][16 pieces][token % 4][D / 32]; scales [token / 4][D / 32][token % 4].  An
//      operand of O^T = V^T P^T is a piece, D / 16 channels, of four consecutive tokens: with the
//      four tokens side by side that is one load of 16 bytes (D = 128) and one of the four scales.
//      Tokens share no byte, so rows of one slice can be written at the same time.
#pragma once
#include "vx_device.h"

namespace vx {
namespace mx {

constexpr int kGroup = 32;
constexpr int kMinScale = 8;      // smallest stored value 2^-120: normal in bf16 and fp32
constexpr int kMaxScale = 252;    // 6 * 2^125 is finite
constexpr int kNanScale = 255;

__host__ __device__ constexpr int64_t slice_bytes(int ps, int D) { return (int64_t)ps * (D / 2 + D / kGroup); }
__host__ __device__ constexpr int codes_bytes(int ps, int D) { return ps * (D / 2); }

// Offsets inside a slice of the 8 channels 8 c8 .. of token t.  V: of their first piece; with 4 channels
// per piece (D = 64) the next one follows 8 bytes later.
__device__ __forceinline__ int k_code(int t, int c8, int D) { return t * (D / 2) + 4 * c8; }
__device__ __forceinline__ int v_code(int t, int c8, int D) {
  return D == 128 ? (((t >> 2) * 16 + c8) * 4 + (t & 3)) * 4 : (((t >> 2) * 16 + 2 * c8) * 4 + (t & 3)) * 2;
}
__device__ __forceinline__ int k_scale(int t, int grp, int D) { return t * (D / kGroup) + grp; }
__device__ __forceinline__ int v_scale(int t, int grp, int D) { return ((t >> 2) * (D / kGroup) + grp) * 4 + (t & 3); }

// The conversions' scale operand of scale byte E.  They take its exponent field alone, 255 as NaN, and
// neither its sign nor its mantissa.
__device__ __forceinline__ float scale_operand(uint32_t e) { return __uint_as_float(e << 23); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// Byte B of w, two codes, as a bf16 pair or two floats times the scale: exact.
template <int B>
__device__ __forceinline__ uint32_t pair_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
template <int B>
__device__ __forceinline__ float2_t pair_f32(uint32_t w, float scale) {
  return __builtin_bit_cast(float2_t, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, B));
}

// Largest magnitude of 8 bf16 values as its bit pattern (ordered as the magnitudes are, infinities and
// NaN above every finite value).
__device__ __forceinline__ uint32_t amax_bits(const uint4& w) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  uint32_t m = 0;
#pragma unroll
  for (int x = 0; x < 4; x++) m = max(m, max(ws[x] & 0x7fffu, (ws[x] >> 16) & 0x7fffu));
  return m;
}

// The scale of a group from its largest magnitude's bits: the exponent of the magnitude rounded to one
// mantissa bit, two binades up, so that it rounds to at most 6 as any other value of its binade does.
__device__ __forceinline__ uint32_t group_scale(uint32_t amax) {
  const int e = (int)((amax + 0x20u) >> 7) - 2;
  return amax >= 0x7f80u ? (uint32_t)kNanScale : (uint32_t)min(max(e, kMinScale), kMaxScale);
}

// 8 bf16 values as codes: value / 2^(E - 127) to the nearest, ties to the even code, at most 6 (codes 0
// in a NaN group).
__device__ __forceinline__ uint32_t encode8(const uint4& w, uint32_t e) {
  const float s = __uint_as_float(e << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w.x), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w.y), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w.z), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, w.w), s, 3);
  return e == (uint32_t)kNanScale ? 0u : c;
}

// 8 channels of codes at 8 c8 of a V row.
__device__ __forceinline__ void put_v_codes(uint8_t* slice, int t, int c8, int D, uint32_t codes) {
  uint8_t* p = slice + v_code(t, c8, D);
  if (D == 128) {
    *reinterpret_cast<uint32_t*>(p) = codes;
  } else {
    *reinterpret_cast<uint16_t*>(p) = (uint16_t)codes;
    *reinterpret_cast<uint16_t*>(p + 8) = (uint16_t)(codes >> 16);
  }
}
__device__ __forceinline__ uint32_t get_v_codes(const uint8_t* slice, int t, int c8, int D) {
  const uint8_t* p = slice + v_code(t, c8, D);
  if (D == 128) return *reinterpret_cast<const uint32_t*>(p);
  return (uint32_t)*reinterpret_cast<const uint16_t*>(p) | ((uint32_t)*reinterpret_cast<const uint16_t*>(p + 8) << 16);
}

}  // namespace mx
}  // namespace vx
