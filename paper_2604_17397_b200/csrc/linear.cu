// Linear layer with its epilogue for sm_100a: out = residual + gate * act(x W^T + bias).
//
// The product runs on the 5th-generation tensor cores (tcgen05.mma, 16-bit operands, fp32 accumulators in tensor
// memory) with the WEIGHTS as the M-side operand: a tile's 128 accumulator lanes are output features and its columns are
// tokens.  A thread of the epilogue then owns one feature, whose bias stays in a register and whose gate changes only
// with the token group, and the 32 lanes of a warp read and write 32 neighbouring features of a token: 64 or 128
// contiguous bytes without a detour through shared memory and without any demand on strides or alignment.  It also
// makes few tokens cheap: the token side of the instruction goes down to 16 columns, so that one row costs one pass
// over the weights.
//
// Operand tiles (64 elements of `inner` = one 128-byte swizzled row) are staged by TMA, which fills what lies past the
// ends of either matrix with zeros.
#include <cuda.h>
#include <math.h>

#include <mutex>

#include "bounded_wait.cuh"
#include "elem_types.cuh"
#include "sdvg_internal.h"
#include "sm100_ptx.cuh"
#include "tensor_map.h"

namespace {

using namespace sm100;

constexpr int kTileF = 128;                          // features per tile: the instruction's M
constexpr int kTileK = 64;                           // elements of `inner` per stage: one 128-byte swizzled row
constexpr int kMaxTileT = 256;                       // tokens per tile: the instruction's N, a multiple of 16
constexpr uint64_t kWaitLimitNs = 2000000000ull;     // 2 s per wait
constexpr int kWorkspaceBytes = 256;
constexpr int kMaxDevices = 64;

struct alignas(64) LinearParams {
  CUtensorMap w_map;                                 // box 64 x 128 features
  CUtensorMap x_map;                                 // box 64 x tile_t tokens
  void* out;
  const void* residual;
  const float* bias;
  const float* gate;
  long long ld_out, ld_res, ld_gate;
  int gate_rows;
  int rows, cols;
  int act;
  int tile_t, tiles_f, k_iters, stages;
  uint32_t idesc;
  unsigned int* status;
};

template <int OutType> struct OutElem;
template <> struct OutElem<SDVG_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float get(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct OutElem<SDVG_F16> {
  using T = __half;
  static __device__ __forceinline__ float get(T v) { return __half2float(v); }
  static __device__ __forceinline__ T put(float v) { return __float2half_rn(v); }
};
template <> struct OutElem<SDVG_F32> {
  using T = float;
  static __device__ __forceinline__ float get(T v) { return v; }
  static __device__ __forceinline__ T put(float v) { return v; }
};

// Both exponential forms keep their relative accuracy where the value vanishes: v / (1 + e^-z) tends to -0 for z -> -inf
// (the exponential overflows to infinity), and GELU uses erfc, which has no 1 + erf cancellation.
__device__ __forceinline__ float activate(float v, int act) {
  if (act == SDVG_ACT_SILU) return __fdividef(v, 1.f + __expf(-v));
  if (act == SDVG_ACT_GELU_TANH) return __fdividef(v, 1.f + __expf(-1.5957691216057308f * fmaf(0.044715f * v * v, v, v)));
  if (act == SDVG_ACT_GELU) return 0.5f * v * erfcf(-0.70710678118654752f * v);
  return v;
}

// Epilogue of 32 tokens m0 .. of one feature n: `acc` holds the sums; tokens from `m_end` on are not touched.
template <int OutType>
__device__ __forceinline__ void epilogue32(const LinearParams& p, const uint32_t (&acc)[32], int n, int m0, int m_end) {
  using E = OutElem<OutType>;
  using T = typename E::T;
  if (n >= p.cols || m0 >= m_end) return;
  const int count = min(32, m_end - m0);
  T res[32];
  if (p.residual) {
    const T* r = static_cast<const T*>(p.residual) + (long long)m0 * p.ld_res + n;
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < count) res[j] = r[j * p.ld_res];
  }
  float g[32];
  if (p.gate) {
    const int g0 = m0 / p.gate_rows, g1 = (m0 + count - 1) / p.gate_rows;
    const float* gp = p.gate + g0 * p.ld_gate + n;
    const float first = gp[0];
    if (g0 == g1) {
#pragma unroll
      for (int j = 0; j < 32; ++j) g[j] = first;
    } else {
      long long next = (long long)(g0 + 1) * p.gate_rows;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (j < count) {
          if (m0 + j == next) {
            gp += p.ld_gate;
            next += p.gate_rows;
          }
          g[j] = gp[0];
        }
      }
    }
  }
  const float b = p.bias ? p.bias[n] : 0.f;
  T* o = static_cast<T*>(p.out) + (long long)m0 * p.ld_out + n;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    if (j < count) {
      float v = activate(__uint_as_float(acc[j]) + b, p.act);
      if (p.gate) v *= g[j];
      if (p.residual) v += E::get(res[j]);
      o[j * p.ld_out] = E::put(v);
    }
  }
}

struct TileSmem {
  uint64_t full[8], empty[8], done;
  uint32_t tmem;
};

// One CTA per tile of 128 features x tile_t tokens: warp 0 fetches, warp 1 issues the products, then all four warps
// run the epilogue (32 features each).
template <int OutType>
__global__ void __launch_bounds__(128) linear_tile_kernel(const __grid_constant__ LinearParams p) {
  extern __shared__ uint8_t raw[];
  __shared__ TileSmem sm;
  uint8_t* buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int n0 = (blockIdx.x % p.tiles_f) * kTileF;
  const int m0 = (blockIdx.x / p.tiles_f) * p.tile_t;
  const int w_bytes = kTileF * 128, stage_bytes = w_bytes + p.tile_t * 128;
  uint32_t tmem_cols = 32;
  while (tmem_cols < (uint32_t)p.tile_t) tmem_cols *= 2;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    mbar_init(&sm.done, 1);
    fence_mbar_init();
    prefetch_tmap(&p.w_map);
    prefetch_tmap(&p.x_map);
  }
  if (warp == 0) {
    tmem_alloc(&sm.tmem, tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;

  if (warp == 0) {
    if (elect_one()) {
      int i = 0;
      for (; i < p.k_iters; ++i) {
        const int s = i % p.stages;
        if (!wait_for(&sm.empty[s], ((i / p.stages) & 1) ^ 1, p.status, kWaitLimitNs)) break;
        uint8_t* st = buf + s * stage_bytes;
        mbar_expect_tx(&sm.full[s], stage_bytes);
        tma_load_2d(st, &p.w_map, &sm.full[s], i * kTileK, n0);
        tma_load_2d(st + w_bytes, &p.x_map, &sm.full[s], i * kTileK, m0);
      }
      if (i < p.k_iters)                             // gave up: see the copies in flight land before the CTA may leave
        for (int j = max(0, i - p.stages); j < i; ++j)
          wait_for(&sm.full[j % p.stages], (j / p.stages) & 1, p.status, kWaitLimitNs);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      bool ok = true;
      for (int i = 0; i < p.k_iters; ++i) {
        const int s = i % p.stages;
        if (!(ok = wait_for(&sm.full[s], (i / p.stages) & 1, p.status, kWaitLimitNs))) break;
        tc_fence_after();
        const uint32_t st = smem_u32(buf + s * stage_bytes);
        const uint64_t a = smem_desc_sw128(st, 16, 1024), b = smem_desc_sw128(st + w_bytes, 16, 1024);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ss(tmem, a + 2 * kk, b + 2 * kk, p.idesc, i > 0 || kk > 0);
        mma_commit(&sm.empty[s]);
      }
      if (ok) mma_commit(&sm.done);
    }
  }
  __syncwarp();
  if (__all_sync(0xffffffffu, wait_for(&sm.done, 0, p.status, kWaitLimitNs))) {
    tc_fence_after();
    const int m_end = min(p.rows, m0 + p.tile_t);
    for (int c = 0; m0 + c < m_end; c += 32) {
      uint32_t acc[32];
      tmem_ld32(tmem + ((uint32_t)(warp * 32) << 16) + c, acc);
      tmem_wait_ld();
      epilogue32<OutType>(p, acc, n0 + warp * 32 + lane, m0 + c, m_end);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(tmem, tmem_cols);
}

// ---- host side -------------------------------------------------------------------------------

// 16-bit matrix [rows, inner] with a row stride, as (inner, row): box = 64 elements x box_rows, 128-byte swizzle; what lies
// past either end reads as zero.
int make_map(CUtensorMap* m, const void* base, int type, int inner, int rows, int64_t ld, int box_rows) {
  const sdvg::EncodeTiledFn fn = sdvg::encode_tiled_fn();
  if (!fn) return SDVG_ERR_CUDA;
  if (rows == 1) ld = ((int64_t)inner + 7) / 8 * 8;              // not read, but the map wants a legal one
  cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  cuuint32_t box[2] = {(cuuint32_t)kTileK, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  const CUresult r = fn(m, type == SDVG_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                        const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SDVG_OK : SDVG_ERR_CUDA;
}

std::mutex g_setup_mu;

constexpr int kTileDynamic = 4 * (kTileF + kMaxTileT) * 128 + 1024;

template <int OutType>
int launch_tile(const LinearParams& p, long long tiles, cudaStream_t stream) {
  static bool ready[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return sdvg::cuda_status(e);
  if (dev < 0 || dev >= kMaxDevices) return SDVG_ERR_INVALID_ARG;
  {
    std::lock_guard<std::mutex> lock(g_setup_mu);
    if (!ready[dev]) {
      e = cudaFuncSetAttribute(linear_tile_kernel<OutType>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileDynamic);
      if (e != cudaSuccess) return sdvg::cuda_status(e);
      ready[dev] = true;
    }
  }
  const int dynamic = p.stages * (kTileF + p.tile_t) * 128 + 1024;
  linear_tile_kernel<OutType><<<(unsigned)tiles, 128, dynamic, stream>>>(p);
  return sdvg::cuda_status(cudaGetLastError());
}

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int sdvg_linear(const void* x, int64_t ld_x, const void* w, int64_t ld_w, const float* bias, int act, const float* gate,
                int64_t ld_gate, int gate_rows, const void* residual, int64_t ld_residual, void* out, int64_t ld_out,
                int rows, int cols, int inner, int in_type, int out_type, void* workspace, size_t workspace_bytes,
                void* stream) {
  SDVG_RANGE();
  constexpr int kMaxExtent = 0x7fffffff - 1024;                  // a tile's end past the matrix's is still an int
  if (rows < 0 || cols < 0 || inner < 1 || rows > kMaxExtent || cols > kMaxExtent || inner > kMaxExtent)
    return SDVG_ERR_BAD_SHAPE;
  if ((in_type != SDVG_BF16 && in_type != SDVG_F16) || !sdvg::elem_type_ok(out_type)) return SDVG_ERR_INVALID_ARG;
  if (act < SDVG_ACT_NONE || act > SDVG_ACT_GELU || (gate && gate_rows < 1)) return SDVG_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return SDVG_OK;
  if (!x || !w || !out || !workspace || workspace_bytes < (size_t)kWorkspaceBytes) return SDVG_ERR_INVALID_ARG;
  if ((rows > 1 && (ld_x < inner || ld_out < cols)) || (cols > 1 && ld_w < inner)) return SDVG_ERR_BAD_SHAPE;
  if (residual && rows > 1 && ld_residual != 0 && ld_residual < cols) return SDVG_ERR_BAD_SHAPE;
  if (gate && rows > gate_rows && ld_gate < cols) return SDVG_ERR_BAD_SHAPE;
  // the tensor map's stride is a 40-bit byte count
  if ((rows > 1 && ld_x >= (int64_t)1 << 39) || (cols > 1 && ld_w >= (int64_t)1 << 39)) return SDVG_ERR_BAD_SHAPE;
  if (!sdvg::aligned16(x) || !sdvg::aligned16(w) || (rows > 1 && (ld_x & 7)) || (cols > 1 && (ld_w & 7)))
    return SDVG_ERR_MISALIGNED;
  if (!aligned_to(out, sdvg::elem_bytes(out_type)) || !aligned_to(residual, sdvg::elem_bytes(out_type)) ||
      !aligned_to(bias, 4) || !aligned_to(gate, 4) || !aligned_to(workspace, 256))
    return SDVG_ERR_MISALIGNED;
  int st = sdvg::require_sm100();
  if (st != SDVG_OK) return st;
  LinearParams p = {};
  p.out = out;
  p.residual = residual;
  p.bias = bias;
  p.gate = gate;
  p.ld_out = ld_out;
  p.ld_res = ld_residual;
  p.ld_gate = ld_gate;
  p.gate_rows = gate_rows;
  p.rows = rows;
  p.cols = cols;
  p.act = act;
  p.tile_t = rows >= kMaxTileT ? kMaxTileT : (rows + 15) / 16 * 16;
  p.tiles_f = (cols + kTileF - 1) / kTileF;
  p.k_iters = (inner + kTileK - 1) / kTileK;
  p.stages = 4;
  p.idesc = idesc_16bit_f32(kTileF, p.tile_t, in_type == SDVG_BF16);
  p.status = (unsigned int*)workspace + 1;
  const long long tiles = (long long)p.tiles_f * ((rows + p.tile_t - 1) / p.tile_t);
  if (tiles >= 1ll << 31) return SDVG_ERR_BAD_SHAPE;
  if ((st = make_map(&p.w_map, w, in_type, inner, cols, ld_w, kTileF)) != SDVG_OK) return st;
  if ((st = make_map(&p.x_map, x, in_type, inner, rows, ld_x, p.tile_t)) != SDVG_OK) return st;
  if (out_type == SDVG_F32) return launch_tile<SDVG_F32>(p, tiles, (cudaStream_t)stream);
  if (out_type == SDVG_F16) return launch_tile<SDVG_F16>(p, tiles, (cudaStream_t)stream);
  return launch_tile<SDVG_BF16>(p, tiles, (cudaStream_t)stream);
}

}  // extern "C"
