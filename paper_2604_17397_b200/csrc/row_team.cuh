// Parts of kernels that walk rows of 16-byte vectors: packed fp32 pairs, a per-thread ring of rows on their way into shared
// memory, warp sums.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "sdvg.h"

namespace rows {

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Eight columns as four packed pairs of fp32.
typedef unsigned long long Pair;
struct Vec8 {
  Pair p[4];
};
__device__ __forceinline__ Pair pair_of(float lo, float hi) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 floats_of(Pair a) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(a));
  return f;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

__device__ __forceinline__ void unpack8(const uint4& a, int type, Vec8& v) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  if (type == SDVG_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = pair_of(bf16_lo(w[j]), bf16_hi(w[j]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      v.p[j] = pair_of(f.x, f.y);
    }
  }
}

__device__ __forceinline__ void store8(char* at, int type, const Vec8& v) {
  float2 f[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = floats_of(v.p[j]);
  if (type == SDVG_F32) {
    float4* o = reinterpret_cast<float4*>(at);
    __stcs(o, make_float4(f[0].x, f[0].y, f[1].x, f[1].y));
    __stcs(o + 1, make_float4(f[2].x, f[2].y, f[3].x, f[3].y));
    return;
  }
  uint32_t w[4];
  if (type == SDVG_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[j].x, f[j].y);
      w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __half2 h = __floats2half2_rn(f[j].x, f[j].y);
      w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  __stcs(reinterpret_cast<uint4*>(at), make_uint4(w[0], w[1], w[2], w[3]));
}

__device__ __forceinline__ void copy16(void* smem, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(src)
               : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's pieces of a tensor's next rows, W bytes per element (0: no such tensor): piece i of ring slot s is W / 2
// vectors of 16 bytes, the warp's 32 threads side by side.
template <int W, int NI>
struct Ring {
  static constexpr int kVecs = W / 2;
  static constexpr int kBytes = NI * kVecs * 16;       // per thread and slot
  uint4* mine;                                         // this thread's first vector
  __device__ __forceinline__ uint4* at(int slot, int i, int h) const { return mine + ((slot * NI + i) * kVecs + h) * 32; }
  __device__ __forceinline__ void request(int slot, int i, const char* row) const {
#pragma unroll
    for (int h = 0; h < kVecs; ++h) copy16(at(slot, i, h), row + (i * 256 * W + 16 * h));
  }
  __device__ __forceinline__ void values(int slot, int i, int type, Vec8& v) const {
    if constexpr (W == 2) {
      unpack8(*at(slot, i, 0), type, v);
    } else if constexpr (W == 4) {
      const float4 a = *reinterpret_cast<const float4*>(at(slot, i, 0)), b = *reinterpret_cast<const float4*>(at(slot, i, 1));
      v.p[0] = pair_of(a.x, a.y);
      v.p[1] = pair_of(a.z, a.w);
      v.p[2] = pair_of(b.x, b.y);
      v.p[3] = pair_of(b.z, b.w);
    }
  }
};

}  // namespace rows
