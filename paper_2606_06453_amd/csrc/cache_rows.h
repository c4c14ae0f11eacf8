// Rounding of 8 channels of a row to the cache's types, and back, shared by the kernels that write or read
// rows by slot.
#pragma once
#include "vx_device.h"
#include "vx_internal.h"

namespace vx {

// 8 fp32 quotients value / scale as fp8 codes: the nearest even code, finite values and infinities at most
// the format's largest, NaN stays NaN.
template <int KT>
__device__ __forceinline__ uint2 fp8_codes(float (&x)[8]) {
  constexpr float kTop = KT == kKvFp8E4M3 ? 448.f : 57344.f;
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = x[e] != x[e] ? x[e] : fminf(fmaxf(x[e], -kTop), kTop);
  int lo = 0, hi = 0;
  if constexpr (KT == kKvFp8E4M3) {
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
  } else {
    lo = __builtin_amdgcn_cvt_pk_bf8_f32(x[0], x[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_bf8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_bf8_f32(x[4], x[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_bf8_f32(x[6], x[7], hi, true);
  }
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// 8 bf16 values as fp8 codes of value / scale.
template <int KT>
__device__ __forceinline__ uint2 encode_fp8(const uint4& w, float scale) {
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    x[2 * e] = bf16lo(ws[e]) / scale;
    x[2 * e + 1] = bf16hi(ws[e]) / scale;
  }
  return fp8_codes<KT>(x);
}

template <int KT>
__device__ __forceinline__ uint4 decode_fp8(const uint2& w, float scale) {
  const int ws[2] = {(int)w.x, (int)w.y};
  uint32_t o[4];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    float2_t lo, hi;
    if constexpr (KT == kKvFp8E4M3) {
      lo = __builtin_amdgcn_cvt_pk_f32_fp8(ws[h], false);
      hi = __builtin_amdgcn_cvt_pk_f32_fp8(ws[h], true);
    } else {
      lo = __builtin_amdgcn_cvt_pk_f32_bf8(ws[h], false);
      hi = __builtin_amdgcn_cvt_pk_f32_bf8(ws[h], true);
    }
    o[2 * h] = f32_to_bf16_rne(lo[0] * scale) | (f32_to_bf16_rne(lo[1] * scale) << 16);
    o[2 * h + 1] = f32_to_bf16_rne(hi[0] * scale) | (f32_to_bf16_rne(hi[1] * scale) << 16);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Largest of the four adjacent lanes that hold a group.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, false));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, false));
}

}  // namespace vx
