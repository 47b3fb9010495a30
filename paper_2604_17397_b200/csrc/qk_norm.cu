// RMS norm of q and k, 3D rotary embedding and the ring write of k' and v, one pass over the rows of a QKV product.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "overlap.cuh"
#include "rope_args.h"
#include "row_team.cuh"
#include "sdvg_internal.h"

namespace {

using namespace rows;

struct QkParams {
  // token t at q + t * ld_q; q and q_out null for none
  const __nv_bfloat16 *q, *k, *v;
  long long ld_q, ld_k, ld_v;
  const float *q_weight, *k_weight;                    // null: 1
  __nv_bfloat16 *q_out, *k_out;                        // contiguous [tokens, heads, dim]; k_out may be null
  __nv_bfloat16 *k_slot, *v_slot;                      // (head 0, slot, token 0) of the ring
  long long slot_head_stride;
  int tokens, heads;
  int scope;
  float eps;
  // rotary fields
  int grid_hw, grid_w, frame_offset, pairs_f, pairs_h, tab_h_off, tab_w_off;
  const float2* tab;
};

constexpr int kSlots = 2;                              // tokens on their way per team
constexpr int kTeamThreads = 640;                      // most threads of a CTA team with two pieces each; leaves a thread 96 registers

// This thread's part of the sums of squares of one row, per piece.
template <int NI>
__device__ __forceinline__ void squares(const Ring<2, NI>& ring, int slot, float (&q)[NI]) {
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    Vec8 s;
    ring.values(slot, i, SDVG_BF16, s);
    Pair a = 0, b = 0;
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      a = fma2(s.p[j], s.p[j], a);
      b = fma2(s.p[j + 1], s.p[j + 1], b);
    }
    const float2 f = floats_of(add2(a, b));
    q[i] = f.x + f.y;
  }
}

template <int NI>
__device__ __forceinline__ void load_weights(Vec8 (&w)[NI], const float* weight, bool per_head, int c0, int dim, int width) {
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int c = c0 + 256 * i;
    float4 a = make_float4(1.f, 1.f, 1.f, 1.f), b = a;
    if (weight && c < width) {
      const float4* at = reinterpret_cast<const float4*>(weight + (per_head ? c % dim : c));
      a = at[0];
      b = at[1];
    }
    w[i].p[0] = pair_of(a.x, a.y);
    w[i].p[1] = pair_of(a.z, a.w);
    w[i].p[2] = pair_of(b.x, b.y);
    w[i].p[3] = pair_of(b.z, b.w);
  }
}

// rotate(v * rstd * w), rounded once.
__device__ __forceinline__ uint4 norm_rotate(const Vec8& v, float rstd, const Vec8& w, const float2 (&cs)[4]) {
  const Pair r = pair_of(rstd, rstd);
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 n = floats_of(mul2(mul2(v.p[e], r), w.p[e]));
    const __nv_bfloat162 h = __floats2bfloat162_rn(fmaf(n.x, cs[e].x, -n.y * cs[e].y), fmaf(n.x, cs[e].y, n.y * cs[e].x));
    o[e] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A token's rows of q, k and v are split over a team: a CTA, or one warp where two pieces per lane hold a row.  A thread
// holds NI pieces of 8 columns of each, 256 columns apart, which is a whole number of heads: its pieces sit at the same
// place of their heads and share the token's four (cos, sin) pairs, fetched once for q and k, and their ring addresses are a
// constant step apart.  q and k are reduced together, with one barrier per token.  The next tokens are on their way into
// shared memory meanwhile, every thread fetching what it will read itself.  Bound by HBM: three reads and three writes of a
// block tensor.  With q, k and v as separate rows of the grid it took 63 us at 40 heads x 128 x 4680 tokens (287.5 MB).
template <int D, int NI, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : NI == 2 ? kTeamThreads : 512) qk_norm_kernel(const __grid_constant__ QkParams p) {
  constexpr int kGroup = D / 8;                        // lanes of a head
  extern __shared__ uint4 s_ring[];
  __shared__ float2 s_part[2][32];
  sdvg::overlap_wait();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int width = p.heads * D;
  const int c0 = ((WARP ? 0 : warp * 32 * NI) + lane) * 8;             // first piece; piece i: c0 + 256 i
  auto valid = [&](int i) { return c0 + 256 * i < width; };
  const int teams = WARP ? gridDim.x * (blockDim.x / 32) : gridDim.x, me = WARP ? blockIdx.x * (blockDim.x / 32) + warp : blockIdx.x;
  const int share = p.tokens / teams, rest = p.tokens % teams;
  const int begin = me * share + min(me, rest), total = share + (me < rest ? 1 : 0);

  constexpr int kRingVecs = kSlots * Ring<2, NI>::kBytes / 16 * 32;    // of a warp
  uint4* base = s_ring + warp * 3 * kRingVecs + lane;
  const Ring<2, NI> rq{base}, rk{base + kRingVecs}, rv{base + 2 * kRingVecs};
  const bool has_q = p.q != nullptr;
  const char* q = reinterpret_cast<const char*>(p.q + begin * p.ld_q + c0);
  const char* k = reinterpret_cast<const char*>(p.k + begin * p.ld_k + c0);
  const char* v = reinterpret_cast<const char*>(p.v + begin * p.ld_v + c0);
  int asked = 0;
  auto request = [&](int slot) {
    if (asked < total) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (valid(i)) {
          if (has_q) rq.request(slot, i, q);
          rk.request(slot, i, k);
          rv.request(slot, i, v);
        }
    }
    copy_commit();                                     // an empty group where there is no such token
    ++asked;
    q += p.ld_q * 2;
    k += p.ld_k * 2;
    v += p.ld_v * 2;
  };
#pragma unroll
  for (int s = 0; s < kSlots; ++s) request(s);

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
  const bool per_head = p.scope == SDVG_SCOPE_HEAD;
  Vec8 wq[NI], wk[NI];
  load_weights<NI>(wq, p.q_weight, per_head, c0, D, width);
  load_weights<NI>(wk, p.k_weight, per_head, c0, D, width);
  char* q_out = reinterpret_cast<char*>(p.q_out + (long long)begin * width + c0);
  char* k_out = reinterpret_cast<char*>(p.k_out + (long long)begin * width + c0);
  long long to_ring = (c0 / D * p.slot_head_stride + (long long)begin * D + c0 % D) * 2;
  const long long ring_step = 256 / D * p.slot_head_stride * 2;        // bytes between the ring addresses of two pieces
  int f = begin / p.grid_hw, y = (begin - f * p.grid_hw) / p.grid_w, x = begin % p.grid_w;   // the token's position
  const int grid_h = p.grid_hw / p.grid_w;
  const float inv_n = 1.f / (float)(per_head ? D : width);
  int slot = 0, turn = 0;
  for (int r = 0; r < total; ++r, slot = slot + 1 == kSlots ? 0 : slot + 1) {                // uniform over the team
    float2 cs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int pos = axis[e] == 0 ? p.frame_offset + f : axis[e] == 1 ? y : x;
      cs[e] = p.tab[pair_at[e] + pos * pair_step[e]];
    }
    if (++x == p.grid_w) {
      x = 0;
      if (++y == grid_h) {
        y = 0;
        ++f;
      }
    }
    copy_wait<kSlots - 1>();                           // this thread's own copies: nobody else reads them
    float sq[NI], sk[NI];
    squares<NI>(rk, slot, sk);
    if (has_q) squares<NI>(rq, slot, sq);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (!valid(i)) sk[i] = 0.f;                      // what the ring holds there was never fetched
      if (!valid(i) || !has_q) sq[i] = 0.f;
    }
    if (per_head) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int o = kGroup / 2; o > 0; o >>= 1) {
          sq[i] += __shfl_xor_sync(0xffffffffu, sq[i], o);
          sk[i] += __shfl_xor_sync(0xffffffffu, sk[i], o);
        }
        sq[i] = rsqrtf(fmaf(sq[i], inv_n, p.eps));
        sk[i] = rsqrtf(fmaf(sk[i], inv_n, p.eps));
      }
    } else {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NI; ++i) sum.x += sq[i], sum.y += sk[i];
      sum = make_float2(warp_sum(sum.x), warp_sum(sum.y));
      if (!WARP) {
        // a buffer is written again only two tokens later, after a barrier that its readers have reached
        if (lane == 0) s_part[turn][warp] = sum;
        __syncthreads();
        sum = lane < blockDim.x / 32 ? s_part[turn][lane] : make_float2(0.f, 0.f);
        sum = make_float2(warp_sum(sum.x), warp_sum(sum.y));
        turn ^= 1;
      }
      const float a = rsqrtf(fmaf(sum.x, inv_n, p.eps)), b = rsqrtf(fmaf(sum.y, inv_n, p.eps));
#pragma unroll
      for (int i = 0; i < NI; ++i) sq[i] = a, sk[i] = b;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (valid(i)) {
        Vec8 s;
        if (has_q) {
          rq.values(slot, i, SDVG_BF16, s);
          __stcs(reinterpret_cast<uint4*>(q_out + 512 * i), norm_rotate(s, sq[i], wq[i], cs));
        }
        rk.values(slot, i, SDVG_BF16, s);
        const uint4 o = norm_rotate(s, sk[i], wk[i], cs);
        if (p.k_out) __stcs(reinterpret_cast<uint4*>(k_out + 512 * i), o);
        *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p.k_slot) + to_ring + ring_step * i) = o;
        *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p.v_slot) + to_ring + ring_step * i) = *rv.at(slot, i, 0);
      }
    request(slot);
    q_out += 2 * width;
    k_out += 2 * width;
    to_ring += 2 * D;
  }
  copy_wait<0>();
  // not earlier: a next grid's teams that take over an SM one by one run out of step with the others (target block: 56.1 us
  // back to back when begun at the start, 53.8 here)
  sdvg::overlap_begin();
}

template <int D, int NI, bool WARP>
int launch_team(const QkParams& p, int threads, cudaStream_t stream) {
  const int dynamic = threads * 3 * kSlots * Ring<2, NI>::kBytes;
  constexpr int kMostDynamic = (WARP ? 128 : NI == 2 ? kTeamThreads : 512) * 3 * kSlots * Ring<2, NI>::kBytes;
  static_assert(kMostDynamic <= 200 * 1024, "ring size");
  // a grid that the device holds at once: teams walk rows of equal number.  Asked again when the shape changes.
  static thread_local int known_dev = -1, known_dynamic = -1, resident = 0, sms = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return sdvg::cuda_status(e);
  if (dev != known_dev || dynamic != known_dynamic) {
    auto kernel = qk_norm_kernel<D, NI, WARP>;
    known_dev = -1;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostDynamic);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, dynamic);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    known_dev = dev;
    known_dynamic = dynamic;                           // a multiple of the thread count for each instance
  }
  const int rows_per_cta = WARP ? threads / 32 : 1;
  const int want = (p.tokens + rows_per_cta - 1) / rows_per_cta;
  return sdvg::cuda_status(sdvg::launch_overlapped(qk_norm_kernel<D, NI, WARP>, std::min(want, sms * std::max(resident, 1)),
                                                   threads, dynamic, 0, stream, p));
}

template <int D>
int launch(const QkParams& p, cudaStream_t stream) {
  const int vecs = p.heads * D / 8;
  if (vecs <= 32) return launch_team<D, 1, true>(p, 128, stream);
  if (vecs <= 64) return launch_team<D, 2, true>(p, 128, stream);
  if (vecs <= 2 * kTeamThreads) return launch_team<D, 2, false>(p, (vecs + 63) / 64 * 32, stream);
  return launch_team<D, 4, false>(p, (vecs + 127) / 128 * 32, stream);       // at most 2048 vectors: 512 threads
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
  p.q = (const __nv_bfloat16*)q;
  p.k = (const __nv_bfloat16*)k;
  p.v = (const __nv_bfloat16*)v;
  p.ld_q = ld_q;
  p.ld_k = ld_k;
  p.ld_v = ld_v;
  p.q_weight = q_weight;
  p.k_weight = k_weight;
  p.q_out = (__nv_bfloat16*)q_out;
  p.k_out = (__nv_bfloat16*)k_out;
  p.k_slot = (__nv_bfloat16*)c->k_buf + sdvg::slot_offset(c, 0, slot);
  p.v_slot = (__nv_bfloat16*)c->v_buf + sdvg::slot_offset(c, 0, slot);
  st = c->head_dim == 128 ? launch<128>(p, (cudaStream_t)stream) : launch<64>(p, (cudaStream_t)stream);
  if (st != SDVG_OK) return st;
  sdvg::ring_end_commit(c, block_index, flags, slot, evicted_block);
  return SDVG_OK;
}

}  // extern "C"
