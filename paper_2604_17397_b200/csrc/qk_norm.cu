// RMS norm of q and k, 3D rotary embedding and the ring write of k' and v, one pass over the rows of a QKV product.
#include <cuda_bf16.h>
#include <math.h>

#include "rope_args.h"
#include "sdvg_internal.h"

namespace {

struct QkJob {
  const __nv_bfloat16* src;      // token t at src + t * ld
  long long ld;
  const float* weight;           // null: 1
  __nv_bfloat16* dst;            // contiguous [tokens, heads, dim], or null
  __nv_bfloat16* slot;           // (head 0, slot, token 0) of the ring, or null
  int norm;                      // q, k; v is copied
};

struct QkParams {
  QkJob job[3];
  int tokens, heads, dim;
  int scope;
  float eps;
  long long slot_head_stride;
  // rotary fields
  int grid_hw, grid_w, frame_offset, pairs_f, pairs_h, tab_h_off, tab_w_off;
  const float2* tab;
};

constexpr int kThreads = 256;

// (cos, sin) of pair `pr` of the token at frame f, row y, column x.
__device__ __forceinline__ float2 pair_cs(const QkParams& p, int t, int pr) {
  const int f = t / p.grid_hw, rem = t - f * p.grid_hw, y = rem / p.grid_w, x = rem - y * p.grid_w;
  const int pairs_w = p.dim / 2 - p.pairs_f - p.pairs_h;
  int idx;
  if (pr < p.pairs_f) idx = (p.frame_offset + f) * p.pairs_f + pr;
  else if (pr < p.pairs_f + p.pairs_h) idx = p.tab_h_off + y * p.pairs_h + (pr - p.pairs_f);
  else idx = p.tab_w_off + x * pairs_w + (pr - p.pairs_f - p.pairs_h);
  return __ldg(p.tab + idx);
}

// One CTA per (token, tensor); a warp takes the heads in turn.
__global__ void __launch_bounds__(kThreads) qk_norm_kernel(const __grid_constant__ QkParams p) {
  __shared__ float buf[kThreads / 32];
  const QkJob& job = p.job[blockIdx.y];
  const int t = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const __nv_bfloat16* src = job.src + t * job.ld;
  const int c_total = p.heads * p.dim;
  float rstd = 1.f;
  if (job.norm && p.scope == SDVG_SCOPE_ROW) {
    float q = 0.f;
    for (int c = threadIdx.x; c < c_total; c += kThreads) {
      const float v = __bfloat162float(src[c]);
      q = fmaf(v, v, q);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
    if (lane == 0) buf[warp] = q;
    __syncthreads();
    q = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) q += buf[w];
    rstd = 1.f / sqrtf(q / (float)c_total + p.eps);
  }
  for (int h = warp; h < p.heads; h += kThreads / 32) {
    const __nv_bfloat16* row = src + h * p.dim;
    if (job.norm && p.scope == SDVG_SCOPE_HEAD) {
      float q = 0.f;
      for (int d = lane; d < p.dim; d += 32) {
        const float v = __bfloat162float(row[d]);
        q = fmaf(v, v, q);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
      rstd = 1.f / sqrtf(q / (float)p.dim + p.eps);
    }
    for (int pr = lane; pr < p.dim / 2; pr += 32) {
      __nv_bfloat162 w = *reinterpret_cast<const __nv_bfloat162*>(row + 2 * pr);
      if (job.norm) {
        float re = __bfloat162float(w.x) * rstd, im = __bfloat162float(w.y) * rstd;
        if (job.weight) {
          const float* g = job.weight + (p.scope == SDVG_SCOPE_ROW ? h * p.dim : 0) + 2 * pr;
          re *= g[0];
          im *= g[1];
        }
        const float2 cs = pair_cs(p, t, pr);
        w = __floats2bfloat162_rn(re * cs.x - im * cs.y, re * cs.y + im * cs.x);
      }
      if (job.dst) *reinterpret_cast<__nv_bfloat162*>(job.dst + (long long)t * c_total + h * p.dim + 2 * pr) = w;
      if (job.slot)
        *reinterpret_cast<__nv_bfloat162*>(job.slot + h * p.slot_head_stride + (long long)t * p.dim + 2 * pr) = w;
    }
  }
}

}  // namespace

extern "C" {

int sdvg_qk_norm_rope3d_commit(sdvg_cache* c, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                               int64_t ld_v, const float* q_weight, const float* k_weight, int scope, float eps,
                               void* q_out, void* k_out, int frames, int grid_h, int grid_w, int frame_offset,
                               const float* cos_sin_tab, int tab_frames, int64_t block_index, int flags,
                               int64_t* evicted_block, void* stream) {
  SDVG_RANGE();
  if (!c || !k || !v) return SDVG_ERR_INVALID_ARG;
  if (c->elem_bytes != 2) return SDVG_ERR_BAD_SHAPE;
  if ((q == nullptr) != (q_out == nullptr)) return SDVG_ERR_INVALID_ARG;
  if (scope != SDVG_SCOPE_ROW && scope != SDVG_SCOPE_HEAD) return SDVG_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !isfinite(eps)) return SDVG_ERR_INVALID_ARG;
  const int64_t width = (int64_t)c->heads * c->head_dim;
  if (width > 16384) return SDVG_ERR_BAD_SHAPE;
  if ((q && ld_q < width) || ld_k < width || ld_v < width) return SDVG_ERR_BAD_SHAPE;
  if (((q ? ld_q : 0) | ld_k | ld_v) & 7) return SDVG_ERR_MISALIGNED;
  if (!sdvg::aligned16(q) || !sdvg::aligned16(k) || !sdvg::aligned16(v) || !sdvg::aligned16(q_out) ||
      !sdvg::aligned16(k_out) || !sdvg::aligned16(q_weight) || !sdvg::aligned16(k_weight))
    return SDVG_ERR_MISALIGNED;
  QkParams p = {};
  int st = sdvg::fill_rope(p, c->head_dim, c->block_tokens,
                           sdvg::RopeArgs{frames, grid_h, grid_w, frame_offset, tab_frames, cos_sin_tab});
  if (st != SDVG_OK) return st;
  int slot = 0;
  if ((st = sdvg::ring_begin_commit(c, block_index, flags, &slot)) != SDVG_OK) return st;
  if ((st = sdvg::require_sm100()) != SDVG_OK) return st;
  p.tokens = c->block_tokens;
  p.heads = c->heads;
  p.dim = c->head_dim;
  p.scope = scope;
  p.eps = eps;
  p.slot_head_stride = (long long)c->slots * c->block_tokens * c->head_dim;
  __nv_bfloat16* kslot = (__nv_bfloat16*)c->k_buf + sdvg::slot_offset(c, 0, slot);
  __nv_bfloat16* vslot = (__nv_bfloat16*)c->v_buf + sdvg::slot_offset(c, 0, slot);
  int n = 0;
  if (q) p.job[n++] = QkJob{(const __nv_bfloat16*)q, ld_q, q_weight, (__nv_bfloat16*)q_out, nullptr, 1};
  p.job[n++] = QkJob{(const __nv_bfloat16*)k, ld_k, k_weight, (__nv_bfloat16*)k_out, kslot, 1};
  p.job[n++] = QkJob{(const __nv_bfloat16*)v, ld_v, nullptr, nullptr, vslot, 0};
  qk_norm_kernel<<<dim3(p.tokens, n), kThreads, 0, (cudaStream_t)stream>>>(p);
  if ((st = sdvg::cuda_status(cudaGetLastError())) != SDVG_OK) return st;
  sdvg::ring_end_commit(c, block_index, flags, slot, evicted_block);
  return SDVG_OK;
}

}  // extern "C"
