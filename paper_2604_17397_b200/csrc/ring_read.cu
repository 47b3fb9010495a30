// A slot of an 8-bit ring as bf16 tensors: code times scale in fp32, rounded to bf16.  A thread turns 16 codes of a (token, head) row (one 16-byte
// load) into two 16-byte stores.  Bound by HBM: 1 byte read and 2 written per element.
#include <cuda_bf16.h>

#include "overlap.cuh"
#include "sdvg_internal.h"
#include "sm100_ptx.cuh"

namespace {

constexpr int kThreads = 256;

struct ReadJob {
  const uint4* src;          // (head 0, token 0) of the slot
  uint4* dst;                // [tokens, heads, dim]
  const float* scale;        // of (head, tile) at head * scale_head_stride + tile
};
struct ReadParams {
  ReadJob job[2];
  int tokens, heads;
  long long head_stride;     // 16-byte vectors of the ring
  long long scale_head_stride;
  int tile_shift;            // tile of token t: t >> tile_shift
};

__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float scale) {      // of the two low bytes
  const float2 f = sm100::unpack_e4m3x2((uint16_t)codes);
  const __nv_bfloat162 h = __floats2bfloat162_rn(f.x * scale, f.y * scale);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__global__ void __launch_bounds__(kThreads) ring_read_e4m3_kernel(const __grid_constant__ ReadParams p) {
  constexpr int kVecs = 8;                                     // 16-byte vectors of a (token, head) row of 128 codes
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const ReadJob job = p.job[blockIdx.y];
  const long long total = (long long)p.tokens * p.heads * kVecs;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < total; i += (long long)gridDim.x * kThreads) {
    const int j = (int)(i % kVecs);
    const long long row = i / kVecs;
    const int h = (int)(row % p.heads);
    const long long t = row / p.heads;
    const uint4 c = job.src[h * p.head_stride + t * kVecs + j];
    const float s = job.scale[h * p.scale_head_stride + (t >> p.tile_shift)];
    __stcs(job.dst + 2 * i, make_uint4(bf16_pair(c.x, s), bf16_pair(c.x >> 16, s), bf16_pair(c.y, s), bf16_pair(c.y >> 16, s)));
    __stcs(job.dst + 2 * i + 1, make_uint4(bf16_pair(c.z, s), bf16_pair(c.z >> 16, s), bf16_pair(c.w, s), bf16_pair(c.w >> 16, s)));
  }
}

}  // namespace

extern "C" {

int sdvg_cache_read_block_e4m3(const sdvg_cache* c, int slot, const float* k_descale, const float* v_descale, void* k_out,
                               void* v_out, void* stream) {
  SDVG_RANGE();
  if (!c || (!k_out && !v_out)) return SDVG_ERR_INVALID_ARG;
  if (c->elem_bytes != 1) return SDVG_ERR_BAD_SHAPE;
  if (slot < 0 || slot >= c->slots) return SDVG_ERR_INVALID_ARG;
  const bool tiled = !k_descale && !v_descale;                 // the ring's own scales
  if (tiled ? !c->k_tile_scale || !c->v_tile_scale : (k_out && !k_descale) || (v_out && !v_descale))
    return tiled ? SDVG_ERR_BAD_STATE : SDVG_ERR_INVALID_ARG;
  if (!sdvg::aligned16(k_out) || !sdvg::aligned16(v_out) ||
      ((reinterpret_cast<uintptr_t>(k_descale) | reinterpret_cast<uintptr_t>(v_descale)) & 3))
    return SDVG_ERR_MISALIGNED;
  const int st = sdvg::require_sm100();
  if (st != SDVG_OK) return st;
  ReadParams p = {};
  const int tiles = sdvg::scale_tiles(c->block_tokens);
  p.tokens = c->block_tokens;
  p.heads = c->heads;
  p.head_stride = (long long)c->slots * c->block_tokens * 8;
  p.scale_head_stride = tiled ? (long long)c->slots * tiles : 1;
  p.tile_shift = tiled ? 7 : 31;                               // 31: one scale for every token
  const void* bufs[2] = {c->k_buf, c->v_buf};
  void* outs[2] = {k_out, v_out};
  const float* scales[2] = {tiled ? c->k_tile_scale + (size_t)slot * tiles : k_descale,
                            tiled ? c->v_tile_scale + (size_t)slot * tiles : v_descale};
  int jobs = 0;
  for (int i = 0; i < 2; ++i)
    if (outs[i]) p.job[jobs++] = ReadJob{(const uint4*)bufs[i] + sdvg::slot_offset(c, 0, slot) / 16, (uint4*)outs[i], scales[i]};
  const long long total = (long long)p.tokens * p.heads * 8, want = (total + kThreads - 1) / kThreads;
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const dim3 grid((unsigned)(want < sms * 32ll ? want : sms * 32ll), jobs);
  return sdvg::cuda_status(sdvg::launch_overlapped(ring_read_e4m3_kernel, grid, kThreads, 0, 0, (cudaStream_t)stream, p));
}

}  // extern "C"
