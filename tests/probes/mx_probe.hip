// Test-only probe: the E2M1 conversions of gfx950, one element per thread.
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float f32x2v __attribute__((ext_vector_type(2)));

// out[n] = {bf16 pair of byte 0, of byte 3, fp32 pair of byte 1} of codes[n] at scale[n]
__global__ void from_e2m1(const uint32_t* codes, const float* scale, uint32_t* pairs, float* values, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  const uint32_t w = codes[i];
  const float s = scale[i];
  pairs[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
  pairs[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  const f32x2v f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
  values[2 * i] = f[0];
  values[2 * i + 1] = f[1];
}

// codes[n]: the bf16 pair of pairs[n] at scale[n] in byte 2, 0x11 in the other bytes
__global__ void to_e2m1(const uint32_t* pairs, const float* scale, uint32_t* codes, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  codes[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0x11111111u, __builtin_bit_cast(bf16x2v, pairs[i]), scale[i], 2);
}

extern "C" int vxt_from_e2m1(const void* codes, const void* scale, void* pairs, void* values, int n, void* stream) {
  hipLaunchKernelGGL(from_e2m1, dim3((n + 255) / 256), dim3(256), 0, (hipStream_t)stream, (const uint32_t*)codes,
                     (const float*)scale, (uint32_t*)pairs, (float*)values, n);
  return (int)hipGetLastError();
}

extern "C" int vxt_to_e2m1(const void* pairs, const void* scale, void* codes, int n, void* stream) {
  hipLaunchKernelGGL(to_e2m1, dim3((n + 255) / 256), dim3(256), 0, (hipStream_t)stream, (const uint32_t*)pairs,
                     (const float*)scale, (uint32_t*)codes, n);
  return (int)hipGetLastError();
}
