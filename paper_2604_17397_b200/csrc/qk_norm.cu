// RMS norm of q and k, 3D rotary embedding and the ring write of k' and v, one pass over the rows of a QKV product.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "rope_args.h"
#include "row_team.cuh"
#include "sdvg_internal.h"

namespace {

using namespace rows;

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
  int tokens, heads;
  int scope;
  float eps;
  long long slot_head_stride;
  // rotary fields
  int grid_hw, grid_w, frame_offset, pairs_f, pairs_h, tab_h_off, tab_w_off;
  const float2* tab;
};

constexpr int kSlots = 2;                              // rows on their way per team
constexpr int kTeamThreads = 640;                      // most threads of a CTA team with two pieces each; leaves a thread 96 registers

// A row (token) of q, k or v is split over a team: a CTA, or one warp where two pieces per lane hold the row.  A thread
// holds NI pieces of 8 columns, 256 columns apart, which is a whole number of heads: its pieces sit at the same place of
// their heads and share the four (cos, sin) pairs of the token, and their ring addresses are a constant step apart.  The
// next rows are on their way into shared memory meanwhile.  Bound by HBM: three reads and three writes of a block tensor.
template <int D, int NI, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : NI == 2 ? kTeamThreads : 512) qk_norm_kernel(const __grid_constant__ QkParams p) {
  constexpr int kGroup = D / 8;                        // lanes of a head
  extern __shared__ uint4 s_ring[];
  __shared__ float s_part[2][32];
  const QkJob& job = p.job[blockIdx.y];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int width = p.heads * D;
  const int c0 = ((WARP ? 0 : warp * 32 * NI) + lane) * 8;             // first piece; piece i: c0 + 256 i
  auto valid = [&](int i) { return c0 + 256 * i < width; };
  const int teams = WARP ? gridDim.x * (blockDim.x / 32) : gridDim.x, me = WARP ? blockIdx.x * (blockDim.x / 32) + warp : blockIdx.x;
  const int share = p.tokens / teams, rest = p.tokens % teams;
  const int begin = me * share + min(me, rest), total = share + (me < rest ? 1 : 0);

  const Ring<2, NI> ring{s_ring + warp * 32 * (kSlots * Ring<2, NI>::kBytes / 16) + lane};
  const char* src = reinterpret_cast<const char*>(job.src + begin * job.ld + c0);
  int asked = 0;
  auto request = [&](int slot) {
    if (asked < total) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (valid(i)) ring.request(slot, i, src);
    }
    copy_commit();                                     // an empty group where there is no such row
    ++asked;
    src += job.ld * 2;
  };
#pragma unroll
  for (int k = 0; k < kSlots; ++k) request(k);

  // this thread's four pairs: where the axis' sub-table has them, and which position of the token they turn by
  int pair_at[4], pair_step[4], axis[4];
  const int pairs_w = D / 2 - p.pairs_f - p.pairs_h;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int pr = lane % kGroup * 4 + e;
    if (pr < p.pairs_f) pair_at[e] = pr, pair_step[e] = p.pairs_f, axis[e] = 0;
    else if (pr < p.pairs_f + p.pairs_h) pair_at[e] = p.tab_h_off + pr - p.pairs_f, pair_step[e] = p.pairs_h, axis[e] = 1;
    else pair_at[e] = p.tab_w_off + pr - p.pairs_f - p.pairs_h, pair_step[e] = pairs_w, axis[e] = 2;
  }
  Vec8 w[NI];
  if (job.norm) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const float* at = job.weight + (p.scope == SDVG_SCOPE_ROW ? c0 + 256 * i : c0 % D);
      float4 a = make_float4(1.f, 1.f, 1.f, 1.f), b = a;
      if (job.weight && valid(i)) a = __ldg(reinterpret_cast<const float4*>(at)), b = __ldg(reinterpret_cast<const float4*>(at) + 1);
      w[i].p[0] = pair_of(a.x, a.y);
      w[i].p[1] = pair_of(a.z, a.w);
      w[i].p[2] = pair_of(b.x, b.y);
      w[i].p[3] = pair_of(b.z, b.w);
    }
  }
  char* dst = reinterpret_cast<char*>(job.dst + (long long)begin * width + c0);
  char* to_ring = reinterpret_cast<char*>(job.slot + c0 / D * p.slot_head_stride + (long long)begin * D + c0 % D);
  const long long ring_step = 256 / D * p.slot_head_stride * 2;        // bytes between the ring addresses of two pieces
  int f = begin / p.grid_hw, y = (begin - f * p.grid_hw) / p.grid_w, x = begin % p.grid_w;   // the token's position
  const float inv_n = 1.f / (float)(p.scope == SDVG_SCOPE_ROW ? width : D);
  int slot = 0, turn = 0;
  for (int r = 0; r < total; ++r, slot = slot + 1 == kSlots ? 0 : slot + 1) {                // uniform over the team
    float2 cs[4];
    if (job.norm) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = axis[e] == 0 ? p.frame_offset + f : axis[e] == 1 ? y : x;
        cs[e] = __ldg(p.tab + pair_at[e] + pos * pair_step[e]);
      }
    }
    if (++x == p.grid_w) {
      x = 0;
      if (++y == p.grid_hw / p.grid_w) {
        y = 0;
        ++f;
      }
    }
    copy_wait<kSlots - 1>();                           // this thread's own copies: nobody else reads them
    uint4 v[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = *ring.at(slot, i, 0);
    if (job.norm) {
      Vec8 s[NI];
      float rstd[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        unpack8(v[i], SDVG_BF16, s[i]);
        Pair a = 0, b = 0;
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          a = fma2(s[i].p[j], s[i].p[j], a);
          b = fma2(s[i].p[j + 1], s[i].p[j + 1], b);
        }
        const float2 q = floats_of(add2(a, b));
        rstd[i] = valid(i) ? q.x + q.y : 0.f;
      }
      if (p.scope == SDVG_SCOPE_ROW) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) q += rstd[i];
        q = warp_sum(q);
        if (!WARP) {
          // a buffer is written again only two rows later, after a barrier that its readers have reached
          if (lane == 0) s_part[turn][warp] = q;
          __syncthreads();
          q = warp_sum(lane < blockDim.x / 32 ? s_part[turn][lane] : 0.f);
          turn ^= 1;
        }
        q = rsqrtf(fmaf(q, inv_n, p.eps));
#pragma unroll
        for (int i = 0; i < NI; ++i) rstd[i] = q;
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
#pragma unroll
          for (int o = kGroup / 2; o > 0; o >>= 1) rstd[i] += __shfl_xor_sync(0xffffffffu, rstd[i], o);
          rstd[i] = rsqrtf(fmaf(rstd[i], inv_n, p.eps));
        }
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const Pair r2 = pair_of(rstd[i], rstd[i]);
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 n = floats_of(mul2(mul2(s[i].p[e], r2), w[i].p[e]));
          const __nv_bfloat162 h = __floats2bfloat162_rn(fmaf(n.x, cs[e].x, -n.y * cs[e].y), fmaf(n.x, cs[e].y, n.y * cs[e].x));
          o[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        v[i] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
    request(slot);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (valid(i)) {
        if (job.dst) __stcs(reinterpret_cast<uint4*>(dst + 512 * i), v[i]);
        if (job.slot) *reinterpret_cast<uint4*>(to_ring + ring_step * i) = v[i];
      }
    dst += 2 * width;
    to_ring += 2 * D;
  }
  copy_wait<0>();
}

template <int D, int NI, bool WARP>
int launch_team(const QkParams& p, int jobs, int threads, cudaStream_t stream) {
  const int dynamic = threads * kSlots * Ring<2, NI>::kBytes;
  static_assert((WARP ? 128 : NI == 2 ? kTeamThreads : 512) * kSlots * Ring<2, NI>::kBytes <= 64 * 1024, "ring size");
  // a grid that the device holds at once: teams walk rows of equal number.  Asked again when the shape changes.
  static thread_local int known_dev = -1, known_dynamic = -1, resident = 0, sms = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return sdvg::cuda_status(e);
  if (dev != known_dev || dynamic != known_dynamic) {
    auto kernel = qk_norm_kernel<D, NI, WARP>;
    known_dev = -1;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, dynamic);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    known_dev = dev;
    known_dynamic = dynamic;                           // a multiple of the thread count for each instance
  }
  const int rows_per_cta = WARP ? threads / 32 : 1;
  const int want = (p.tokens + rows_per_cta - 1) / rows_per_cta, most = std::max(1, sms * std::max(resident, 1) / jobs);
  qk_norm_kernel<D, NI, WARP><<<dim3(std::min(want, most), jobs), threads, dynamic, stream>>>(p);
  return sdvg::cuda_status(cudaGetLastError());
}

template <int D>
int launch(const QkParams& p, int jobs, cudaStream_t stream) {
  const int vecs = p.heads * D / 8;
  if (vecs <= 32) return launch_team<D, 1, true>(p, jobs, 128, stream);
  if (vecs <= 64) return launch_team<D, 2, true>(p, jobs, 128, stream);
  if (vecs <= 2 * kTeamThreads) return launch_team<D, 2, false>(p, jobs, (vecs + 63) / 64 * 32, stream);
  return launch_team<D, 4, false>(p, jobs, (vecs + 127) / 128 * 32, stream);       // at most 2048 vectors: 512 threads
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
  p.scope = scope;
  p.eps = eps;
  p.slot_head_stride = (long long)c->slots * c->block_tokens * c->head_dim;
  __nv_bfloat16* kslot = (__nv_bfloat16*)c->k_buf + sdvg::slot_offset(c, 0, slot);
  __nv_bfloat16* vslot = (__nv_bfloat16*)c->v_buf + sdvg::slot_offset(c, 0, slot);
  int n = 0;
  if (q) p.job[n++] = QkJob{(const __nv_bfloat16*)q, ld_q, q_weight, (__nv_bfloat16*)q_out, nullptr, 1};
  p.job[n++] = QkJob{(const __nv_bfloat16*)k, ld_k, k_weight, (__nv_bfloat16*)k_out, kslot, 1};
  p.job[n++] = QkJob{(const __nv_bfloat16*)v, ld_v, nullptr, nullptr, vslot, 0};
  st = c->head_dim == 128 ? launch<128>(p, n, (cudaStream_t)stream) : launch<64>(p, n, (cudaStream_t)stream);
  if (st != SDVG_OK) return st;
  sdvg::ring_end_commit(c, block_index, flags, slot, evicted_block);
  return SDVG_OK;
}

}  // extern "C"
