// A matrix to E4M3 codes with one power-of-two scale per 128 columns of a row, or per 128 x 128 block, and back.
//
// A CTA owns a tile of 128 x 128 elements: 16 threads side by side hold a row's 128 columns, 8 each, and 4 rows 32 apart, in registers
// between the two passes that a data-dependent scale needs (largest magnitude, then quantise).  With a scale per row its
// maximum is among 16 lanes; with one per block it goes through shared memory.  Bound by HBM: 2 or 4 bytes read and 1 written
// per element.
#include "e4m3_scale.cuh"
#include "elem_types.cuh"
#include "overlap.cuh"
#include "row_team.cuh"
#include "sdvg_internal.h"
#include "sm100_ptx.cuh"

namespace {

using namespace rows;

constexpr int kThreads = 512;
constexpr int kRows = 4;                               // of a thread, 32 apart

struct BlockParams {
  const void* x;
  void* out;
  uint8_t* scale;                                      // exponent byte of (row or row block, column block) at row * ld_scale + block
  long long ld_x, ld_out, ld_scale;
  int x_type, out_type;
  int block_rows;                                      // 1 or 128
  int rows, cols, col_blocks;
};

// Eight columns from c on, zeros past the row's end.
template <bool VEC>
__device__ __forceinline__ void load8(float (&v)[8], const BlockParams& p, long long row, int c) {
  const long long at = row * p.ld_x + c;
  if (VEC && c + 8 <= p.cols) {
    if (p.x_type == SDVG_F32) {
      const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + at);
      const float4 a = s[0], b = s[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
      Vec8 u;
      unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.x) + at), p.x_type, u);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = floats_of(u.p[j]);
        v[2 * j] = f.x;
        v[2 * j + 1] = f.y;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < p.cols ? sdvg::load_elem(p.x, at + j, p.x_type) : 0.f;
  }
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads) quant_blocks_kernel(const __grid_constant__ BlockParams p) {
  __shared__ float s_top[kThreads / 32];
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const int tile = blockIdx.x / p.col_blocks, block = blockIdx.x % p.col_blocks;
  const int lane = threadIdx.x % 16, c = block * 128 + lane * 8;
  const long long r0 = (long long)tile * 128 + threadIdx.x / 16;
  float v[kRows][8];
  float top[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (r0 + 32 * i < p.rows) {
      load8<VEC>(v[i], p, r0 + 32 * i, c);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    top[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; j += 2) top[i] = sdvg::larger(top[i], v[i][j], v[i][j + 1]);
  }
  if (p.block_rows == 1) {
#pragma unroll
    for (int i = 0; i < kRows; ++i)
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
  } else {
    float m = sdvg::warp_largest(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
    if (threadIdx.x % 32 == 0) s_top[threadIdx.x / 32] = m;
    __syncthreads();
    m = sdvg::warp_largest(s_top[threadIdx.x % (kThreads / 32)]);
#pragma unroll
    for (int i = 0; i < kRows; ++i) top[i] = m;
    if (threadIdx.x == 0) p.scale[tile * p.ld_scale + block] = (uint8_t)(sdvg::scale_exponent(m) + 127);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const long long r = r0 + 32 * i;
    if (r >= p.rows) break;
    const int e = sdvg::scale_exponent(top[i]);
    const float f = sdvg::power_of_two(-e);
    if (p.block_rows == 1 && lane == 0) p.scale[r * p.ld_scale + block] = (uint8_t)(e + 127);
    const uint2 o = make_uint2(sm100::pack_e4m3x4(v[i][0] * f, v[i][1] * f, v[i][2] * f, v[i][3] * f),
                               sm100::pack_e4m3x4(v[i][4] * f, v[i][5] * f, v[i][6] * f, v[i][7] * f));
    uint8_t* to = static_cast<uint8_t*>(p.out) + r * p.ld_out + c;
    if (VEC && c + 8 <= p.cols) {
      *reinterpret_cast<uint2*>(to) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < p.cols) to[j] = (uint8_t)((j < 4 ? o.x : o.y) >> (8 * (j % 4)));
    }
  }
}

// Codes times their scales, rounded once.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) dequant_blocks_kernel(const __grid_constant__ BlockParams p) {
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const int tile = blockIdx.x / p.col_blocks, block = blockIdx.x % p.col_blocks;
  const int c = block * 128 + threadIdx.x % 16 * 8;
  const long long r0 = (long long)tile * 128 + threadIdx.x / 16;
  const int out_bytes = sdvg::elem_bytes(p.out_type);
  uint2 w[kRows];
  uint8_t s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const long long r = r0 + 32 * i;
    w[i] = make_uint2(0, 0);
    s[i] = 0;
    if (r >= p.rows || c >= p.cols) continue;
    s[i] = p.scale[(p.block_rows == 1 ? r : tile) * p.ld_scale + block];
    const uint8_t* from = static_cast<const uint8_t*>(p.x) + r * p.ld_x + c;
    if (VEC && c + 8 <= p.cols) {
      w[i] = *reinterpret_cast<const uint2*>(from);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < p.cols) (j < 4 ? w[i].x : w[i].y) |= (uint32_t)from[j] << (8 * (j % 4));
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const long long r = r0 + 32 * i;
    if (r >= p.rows || c >= p.cols) continue;
    Vec8 v;
    const float f = sdvg::scale_of_byte(s[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a = sm100::unpack_e4m3x2((uint16_t)((j < 2 ? w[i].x : w[i].y) >> (16 * (j % 2))));
      v.p[j] = pair_of(a.x * f, a.y * f);
    }
    if (VEC && c + 8 <= p.cols) {
      store8(static_cast<char*>(p.out) + (r * p.ld_out + c) * out_bytes, p.out_type, v);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 a = floats_of(v.p[j]);
        if (c + 2 * j < p.cols) sdvg::store_elem(p.out, r * p.ld_out + c + 2 * j, p.out_type, a.x);
        if (c + 2 * j + 1 < p.cols) sdvg::store_elem(p.out, r * p.ld_out + c + 2 * j + 1, p.out_type, a.y);
      }
    }
  }
}

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

// The checks that both directions share; `type` and `values` are those of the 16- or 32-bit side.  0 rows: nothing to do (-1).
int check(const void* values, int64_t ld_values, int type, const void* codes, int64_t ld_codes, const void* scale, int64_t ld_scale,
          int block_rows, int rows, int cols, bool* vec) {
  constexpr int kMaxExtent = 0x7fffffff - 1024;
  if (rows < 0 || cols < 0 || rows > kMaxExtent || cols > kMaxExtent) return SDVG_ERR_BAD_SHAPE;
  if (!sdvg::elem_type_ok(type) || (block_rows != 1 && block_rows != 128)) return SDVG_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return -1;
  if (!values || !codes || !scale) return SDVG_ERR_INVALID_ARG;
  if (rows > 1 && (ld_values < cols || ld_codes < cols)) return SDVG_ERR_BAD_SHAPE;
  const long long blocks = (cols + 127) / 128, tiles = (rows + 127) / 128;
  if (rows > block_rows && ld_scale < blocks) return SDVG_ERR_BAD_SHAPE;
  if (blocks * tiles > 0x7fffffff) return SDVG_ERR_BAD_SHAPE;
  const int bytes = sdvg::elem_bytes(type);
  if (!aligned_to(values, bytes)) return SDVG_ERR_MISALIGNED;
  *vec = sdvg::aligned16(values) && aligned_to(codes, 8) &&
         (rows == 1 || (ld_values * bytes % 16 == 0 && ld_codes % 8 == 0));
  return sdvg::require_sm100();
}

}  // namespace

extern "C" {

int sdvg_quant_e4m3_blocks(const void* x, int64_t ld_x, int x_type, void* out8, int64_t ld_out, void* scale, int64_t ld_scale,
                           int block_rows, int rows, int cols, void* stream) {
  SDVG_RANGE();
  bool vec = false;
  const int st = check(x, ld_x, x_type, out8, ld_out, scale, ld_scale, block_rows, rows, cols, &vec);
  if (st != SDVG_OK) return st < 0 ? SDVG_OK : st;
  BlockParams p = {x, out8, (uint8_t*)scale, ld_x, ld_out, ld_scale, x_type, 0, block_rows, rows, cols, (cols + 127) / 128};
  const unsigned grid = (unsigned)(p.col_blocks * (long long)((rows + 127) / 128));
  return sdvg::cuda_status(sdvg::launch_overlapped(vec ? quant_blocks_kernel<true> : quant_blocks_kernel<false>, grid, kThreads, 0, 0,
                                                   (cudaStream_t)stream, p));
}

int sdvg_dequant_e4m3_blocks(const void* x8, int64_t ld_x, const void* scale, int64_t ld_scale, int block_rows, void* out,
                             int64_t ld_out, int out_type, int rows, int cols, void* stream) {
  SDVG_RANGE();
  bool vec = false;
  const int st = check(out, ld_out, out_type, x8, ld_x, scale, ld_scale, block_rows, rows, cols, &vec);
  if (st != SDVG_OK) return st < 0 ? SDVG_OK : st;
  BlockParams p = {x8, out, (uint8_t*)scale, ld_x, ld_out, ld_scale, 0, out_type, block_rows, rows, cols, (cols + 127) / 128};
  const unsigned grid = (unsigned)(p.col_blocks * (long long)((rows + 127) / 128));
  return sdvg::cuda_status(sdvg::launch_overlapped(vec ? dequant_blocks_kernel<true> : dequant_blocks_kernel<false>, grid, kThreads,
                                                   0, 0, (cudaStream_t)stream, p));
}

}  // extern "C"
