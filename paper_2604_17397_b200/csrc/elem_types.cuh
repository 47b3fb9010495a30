// Elements of the three types the dense operators take (SDVG_BF16, SDVG_F16, SDVG_F32) as fp32 values.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "sdvg.h"

namespace sdvg {

inline bool elem_type_ok(int type) { return type == SDVG_BF16 || type == SDVG_F16 || type == SDVG_F32; }
__host__ __device__ inline int elem_bytes(int type) { return type == SDVG_F32 ? 4 : 2; }

__device__ __forceinline__ float load_elem(const void* base, long long i, int type) {
  if (type == SDVG_F32) return static_cast<const float*>(base)[i];
  if (type == SDVG_F16) return __half2float(static_cast<const __half*>(base)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[i]);
}

// One rounding, to nearest even; a finite value above a type's range becomes an infinity.
__device__ __forceinline__ void store_elem(void* base, long long i, int type, float v) {
  if (type == SDVG_F32) static_cast<float*>(base)[i] = v;
  else if (type == SDVG_F16) static_cast<__half*>(base)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(base)[i] = __float2bfloat16_rn(v);
}

}  // namespace sdvg
