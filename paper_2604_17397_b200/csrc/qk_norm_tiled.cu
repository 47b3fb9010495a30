// RMS norm of q and k, 3D rotary embedding and the quantising write into an 8-bit ring whose scales are chosen from the data, one power
// of two per 128 tokens and head.
//
// A scale needs the largest magnitude of 128 tokens of a head, and a norm over a whole token needs all its heads: two
// reductions across each other.  So a norm over the token gets a pass of its own first, which leaves one factor per token of q
// and k; q and k, read from HBM then, are still in L2 for the second pass where they fit.  The second pass does the rest in
// one reading: a group of 256 threads holds a (tile, head) in registers between its largest magnitude and its codes.
//
// A CTA keeps one tile of 128 tokens and walks heads of q, k and v with it, so that the tokens' rotary factors are looked up
// once, into shared memory.  Its two groups take (tensor, head) items in turn, each with a barrier of its own, so that one group's
// arithmetic runs under the other's waits; what they will read next is on its way into shared memory meanwhile (cp.async,
// every thread fetching just what it will read itself).
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "e4m3_scale.cuh"
#include "overlap.cuh"
#include "rope_args.h"
#include "row_team.cuh"
#include "sdvg_internal.h"
#include "sm100_ptx.cuh"

namespace {

using namespace rows;

constexpr int kTile = sdvg::kScaleTileTokens;          // 128 tokens
constexpr int kDim = 128;
constexpr int kGroupThreads = 256, kGroups = 2, kThreads = kGroups * kGroupThreads;
constexpr int kStep = kGroupThreads / 16;              // 16 threads side by side hold a row of a head: rows 16 apart
constexpr int kRows = kTile / kStep;                   // 8 per thread
constexpr int kSlots = 2;                              // items on their way per group
constexpr int kItemVecs = kTile * 16;                  // 16-byte vectors of a (tile, head)
constexpr int kTurnBytes = kTile * 64 * (int)sizeof(float2);
constexpr int kDynamic = kTurnBytes + kGroups * kSlots * kItemVecs * 16;
static_assert(kDynamic + 4 * 1024 <= 227 * 1024);

struct TileJob {
  const __nv_bfloat16* src;                            // token t, head h at src + t * ld + h * 128
  long long ld;
  uint2* dst;                                          // codes; 8-byte units
  long long token_stride, head_stride;
  float* scale;                                        // of (head, tile) at scale[head * scale_head_stride + tile]
  long long scale_head_stride;
  const float* weight;                                 // null: 1
  const float* rstd;                                   // per token (norm over the token), null: 1, or per head
  bool turned;                                         // q or k: normed and rotated
};

struct TiledParams {
  TileJob job[3];                                      // q, k, v
  int jobs;
  int tokens, heads, groups;                           // head groups of a tile: a CTA each
  float eps;
  // rotary fields
  int grid_hw, grid_w, frame_offset, pairs_f, pairs_h, tab_h_off, tab_w_off;
  const float2* tab;
};

struct StatParams {
  const __nv_bfloat16* src[2];
  long long ld[2];
  float* rstd;                                         // [tensor][tokens]
  int tokens, vecs;
  float eps, inv_width;
};

// One warp per row of q or k.
constexpr int kStatThreads = 256;
__global__ void __launch_bounds__(kStatThreads) row_rstd_kernel(const __grid_constant__ StatParams p) {
  sdvg::overlap_wait();
  sdvg::overlap_begin();                               // not before the wait: the kernel after this one counts on it
  const int lane = threadIdx.x % 32, t = blockIdx.x * (kStatThreads / 32) + threadIdx.x / 32, which = blockIdx.y;
  if (t >= p.tokens) return;
  const uint4* row = reinterpret_cast<const uint4*>(p.src[which] + t * p.ld[which]);
  Pair a = 0, b = 0;
  auto add = [&](const uint4& v) {
    Vec8 s;
    unpack8(v, SDVG_BF16, s);
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      a = fma2(s.p[j], s.p[j], a);
      b = fma2(s.p[j + 1], s.p[j + 1], b);
    }
  };
  int i = lane;
  for (; i + 128 <= p.vecs + 31; i += 128) {           // four vectors of the warp at a time while the first three are whole
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + 32 * k < p.vecs ? row[i + 32 * k] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) add(v[k]);
  }
  for (; i < p.vecs; i += 32) add(row[i]);
  const float2 f = floats_of(add2(a, b));
  const float sum = warp_sum(f.x + f.y);
  if (lane == 0) p.rstd[(long long)which * p.tokens + t] = rsqrtf(fmaf(sum, p.inv_width, p.eps));
}

// Where a group's walk over its (tensor, head) items stands: every second item of the CTA's.
struct Walk {
  int which, head;                                     // head of the CTA's; which == jobs: past the end
  __device__ __forceinline__ void next(int heads) {
    head += kGroups;
    while (head >= heads) {
      head -= heads;
      ++which;
    }
  }
};

// Smallest scale (its exponent) whose inverse makes one finite number with any factor of a norm, which is at most 2^75: the inverse
// square root of the smallest float.  In tiles of smaller scales, those of zeros above all, the values take the norm's factor first.
constexpr int kFoldedScale = -52;

// HEAD: a norm per head.  A token's factor of the norm meets a value only where it is quantised, as one factor with the scale's
// inverse (a power of two, so that this rounds as the product with the norm's factor alone), and the largest magnitude of its row
// before that: rounding keeps the order of magnitudes.  A row's values meet their weights before either, in fp32's range for weights from
// 2^-60 to 2^60.
template <bool HEAD>
__global__ void __launch_bounds__(kThreads, 1) qk_tiled_kernel(const __grid_constant__ TiledParams p) {
  extern __shared__ uint4 s_dynamic[];
  __shared__ float s_top[kGroups][2][kGroupThreads / 32];
  __shared__ float s_rstd[3][kTile];
  __shared__ int s_place[3][kTile];
  // (cos, sin) of [token][which two of a thread's four pairs][thread of the row]: 16 bytes side by side
  float4* s_turn = reinterpret_cast<float4*>(s_dynamic);
  const int tile = blockIdx.x / p.groups, part = blockIdx.x % p.groups;
  const int share = p.heads / p.groups, rest = p.heads % p.groups;
  const int h0 = part * share + min(part, rest), heads = share + (part < rest ? 1 : 0);
  const int t0 = tile * kTile, count = min(kTile, p.tokens - t0);
  const int group = threadIdx.x / kGroupThreads, id = threadIdx.x % kGroupThreads, j = id % 16, r0 = id / 16;
  uint4* ring = s_dynamic + kTurnBytes / 16 + group * kSlots * kItemVecs + id;
  // The pass over the rows lets this kernel begin when all before it in the stream is done and written: only its own factors are
  // still to come.  What is read before they are goes past the L1 cache.
  if (HEAD) sdvg::overlap_wait();

  Walk asked{0, group};
  while (asked.head >= heads) {                        // a CTA of one head: the second group begins with the second tensor
    asked.head -= heads;
    ++asked.which;
  }
  Walk at = asked;
  auto request = [&](int slot) {
    if (asked.which < p.jobs) {
      const TileJob& job = p.job[asked.which];
      const __nv_bfloat16* src = job.src + (t0 + r0) * job.ld + (h0 + asked.head) * kDim + 8 * j;
      const long long step = kStep * job.ld;
      uint4* const to = ring + slot * kItemVecs;
      if (count == kTile) {
#pragma unroll
        for (int i = 0; i < kRows; ++i, src += step) copy16(to + i * kGroupThreads, src);
      } else {
        for (int i = 0; r0 + kStep * i < count; ++i, src += step) copy16(to + i * kGroupThreads, src);
      }
      asked.next(heads);
    }
    copy_commit();                                     // an empty group where there is no such item
  };
#pragma unroll
  for (int s = 0; s < kSlots; ++s) request(s);
  // rows past the last token are never fetched: zeros in this thread's places for them
  for (int i = 0; i < kRows; ++i)
    if (r0 + kStep * i >= count) ring[i * kGroupThreads] = ring[kItemVecs + i * kGroupThreads] = make_uint4(0, 0, 0, 0);
  static_assert(kSlots == 2);

  // the tile's rotary factors and norms: a thread looks up one pair, whose axis it settles once, for every eighth token
  if (threadIdx.x < kTile) {
    const int t = min(t0 + (int)threadIdx.x, p.tokens - 1), f = t / p.grid_hw, rem = t - f * p.grid_hw, y = rem / p.grid_w;
    s_place[0][threadIdx.x] = p.frame_offset + f;
    s_place[1][threadIdx.x] = y;
    s_place[2][threadIdx.x] = rem - y * p.grid_w;
  }
  __syncthreads();
  const int pr = threadIdx.x % 64, pairs_w = kDim / 2 - p.pairs_f - p.pairs_h;
  const int axis = pr < p.pairs_f ? 0 : pr < p.pairs_f + p.pairs_h ? 1 : 2;
  const float2* const of_pair = p.tab + pr + (axis == 0 ? 0 : axis == 1 ? p.tab_h_off - p.pairs_f : p.tab_w_off - p.pairs_f - p.pairs_h);
  const int per_place = axis == 0 ? p.pairs_f : axis == 1 ? p.pairs_h : pairs_w;
#pragma unroll
  for (int t = threadIdx.x / 64; t < kTile; t += kThreads / 64)
    reinterpret_cast<float2*>(s_turn)[t * 64 + pr % 4 / 2 * 32 + pr / 4 * 2 + pr % 2] = __ldcg(of_pair + (long long)s_place[axis][t] * per_place);
  if (!HEAD) sdvg::overlap_wait();
  for (int i = threadIdx.x; i < p.jobs * kTile; i += kThreads) {
    const TileJob& job = p.job[i / kTile];
    s_rstd[i / kTile][i % kTile] = job.rstd && i % kTile < count ? job.rstd[t0 + i % kTile] : 1.f;
  }
  __syncthreads();

  int slot = 0, turn = 0;
  for (; at.which < p.jobs; at.next(heads), slot = slot + 1 == kSlots ? 0 : slot + 1) {      // uniform over the group
    const int h = h0 + at.head;
    const TileJob& job = p.job[at.which];
    const float* const rstd = s_rstd[at.which] + r0;
    const bool turned = job.turned;
    copy_wait<kSlots - 1>();                           // this thread's own copies: nobody else reads them
    float v[kRows][8], of_row[HEAD ? kRows : 1] = {};
    float top = 0.f;
    if (turned) {
      Pair w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pair_of(1.f, 1.f);
      if (job.weight) {
        const float4* from = reinterpret_cast<const float4*>(job.weight + (HEAD ? 0 : h * kDim) + 8 * j);
        const float4 a = from[0], b = from[1];
        w[0] = pair_of(a.x, a.y), w[1] = pair_of(a.z, a.w), w[2] = pair_of(b.x, b.y), w[3] = pair_of(b.z, b.w);
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int r = r0 + kStep * i;
        Vec8 s;
        unpack8(ring[slot * kItemVecs + i * kGroupThreads], SDVG_BF16, s);
        float factor;
        if constexpr (HEAD) {
          const Pair a = fma2(s.p[0], s.p[0], mul2(s.p[1], s.p[1])), b = fma2(s.p[2], s.p[2], mul2(s.p[3], s.p[3]));
          const float2 f = floats_of(add2(a, b));
          float sum = f.x + f.y;
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          factor = of_row[i] = rsqrtf(fmaf(sum, 1.f / kDim, p.eps));
        } else {
          factor = rstd[kStep * i];
        }
        const float4 c0 = s_turn[r * 32 + j], c1 = s_turn[r * 32 + 16 + j];
        const float2 cs[4] = {{c0.x, c0.y}, {c0.z, c0.w}, {c1.x, c1.y}, {c1.z, c1.w}};
        float largest = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 n = floats_of(mul2(s.p[e], w[e]));
          v[i][2 * e] = fmaf(n.x, cs[e].x, -n.y * cs[e].y);
          v[i][2 * e + 1] = fmaf(n.x, cs[e].y, n.y * cs[e].x);
          largest = sdvg::larger(largest, v[i][2 * e], v[i][2 * e + 1]);
        }
        top = fmaxf(top, largest * factor);            // rows past the last token are zeros, or NaN
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        Vec8 s;
        unpack8(ring[slot * kItemVecs + i * kGroupThreads], SDVG_BF16, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = floats_of(s.p[e]);
          v[i][2 * e] = f.x;
          v[i][2 * e + 1] = f.y;
          top = sdvg::larger(top, f.x, f.y);
        }
        if constexpr (HEAD) of_row[i] = 1.f;
      }
    }
    request(slot);
    top = sdvg::warp_largest(top);
    // a buffer is written again only two items later, after a barrier that its readers have reached
    if (id % 32 == 0) s_top[group][turn][id / 32] = top;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(kGroupThreads) : "memory");
    top = sdvg::warp_largest(s_top[group][turn][id % (kGroupThreads / 32)]);
    turn ^= 1;
    const int e = sdvg::scale_exponent(top);
    const float inv = sdvg::power_of_two(-e);
    const bool apart = e < kFoldedScale;                // the same for the group
    if (apart) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float n = HEAD ? of_row[HEAD ? i : 0] : rstd[kStep * i];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] *= n;
        if constexpr (HEAD) of_row[i] = 1.f;
      }
    }
    if (id == 0) job.scale[h * job.scale_head_stride + tile] = sdvg::power_of_two(e);
    uint2* dst = job.dst + (t0 + r0) * job.token_stride + h * job.head_stride + j;
    const long long step = kStep * job.token_stride;
    auto codes = [&](int i) {
      const float f = (HEAD ? of_row[HEAD ? i : 0] : apart ? 1.f : rstd[kStep * i]) * inv;
      const float(&a)[8] = v[i];
      return make_uint2(sm100::pack_e4m3x4(a[0] * f, a[1] * f, a[2] * f, a[3] * f), sm100::pack_e4m3x4(a[4] * f, a[5] * f, a[6] * f, a[7] * f));
    };
    if (count == kTile) {
#pragma unroll
      for (int i = 0; i < kRows; ++i, dst += step) __stcs(dst, codes(i));
    } else {
#pragma unroll
      for (int i = 0; i < kRows; ++i, dst += step)
        if (r0 + kStep * i < count) __stcs(dst, codes(i));
    }
  }
  copy_wait<0>();
  sdvg::overlap_begin();
}

constexpr size_t kStatusBytes = 256;                   // in front of the factors: the layout of every other workspace

int device_sms(int* sms) {
  static thread_local int cached_dev = -1, cached = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev != cached_dev) {
    e = cudaDeviceGetAttribute(&cached, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(qk_tiled_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynamic);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(qk_tiled_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynamic);
    if (e == cudaSuccess) cached_dev = dev;
  }
  *sms = cached;
  return sdvg::cuda_status(e);
}

// Head groups of a tile: the number whose waves of CTAs (one per SM) cost least, a CTA's own start being worth about two heads.
int head_groups(int tiles, int heads, int sms) {
  int best = 1;
  long long best_cost = 0;
  for (int g = 1; g <= heads; ++g) {
    const long long cost = ((long long)tiles * g + sms - 1) / sms * ((heads + g - 1) / g + 2);
    if (!best_cost || cost < best_cost) {
      best = g;
      best_cost = cost;
    }
  }
  return best;
}

}  // namespace

extern "C" {

size_t sdvg_qk_norm_workspace_bytes(int block_tokens) {
  return block_tokens < 1 ? 0 : kStatusBytes + (size_t)block_tokens * 2 * sizeof(float);
}

int sdvg_qk_norm_rope3d_commit_e4m3_tiled(sdvg_cache* c, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v,
                                          int64_t ld_v, const float* q_weight, const float* k_weight, int scope, float eps,
                                          void* q8_out, float* q_tile_scale, int frames, int grid_h, int grid_w,
                                          int frame_offset, const float* cos_sin_tab, int tab_frames, int64_t block_index,
                                          int flags, int64_t* evicted_block, void* workspace, size_t workspace_bytes,
                                          void* stream) {
  SDVG_RANGE();
  if (!c || !k || !v) return SDVG_ERR_INVALID_ARG;
  if (c->elem_bytes != 1) return SDVG_ERR_BAD_SHAPE;
  if (!c->k_tile_scale || !c->v_tile_scale) return SDVG_ERR_BAD_STATE;
  if ((q == nullptr) != (q8_out == nullptr) || (q && !q_tile_scale)) return SDVG_ERR_INVALID_ARG;
  if (scope != SDVG_SCOPE_ROW && scope != SDVG_SCOPE_HEAD) return SDVG_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !isfinite(eps)) return SDVG_ERR_INVALID_ARG;
  const int64_t width = (int64_t)c->heads * kDim;
  if (width > 16384) return SDVG_ERR_BAD_SHAPE;
  if ((q && ld_q < width) || ld_k < width || ld_v < width) return SDVG_ERR_BAD_SHAPE;
  if (scope == SDVG_SCOPE_ROW && (!workspace || workspace_bytes < sdvg_qk_norm_workspace_bytes(c->block_tokens)))
    return SDVG_ERR_INVALID_ARG;
  if (((q ? ld_q : 0) | ld_k | ld_v) & 7) return SDVG_ERR_MISALIGNED;
  if (!sdvg::aligned16(q) || !sdvg::aligned16(k) || !sdvg::aligned16(v) || !sdvg::aligned16(q8_out) ||
      !sdvg::aligned16(q_weight) || !sdvg::aligned16(k_weight) || (reinterpret_cast<uintptr_t>(q_tile_scale) & 3) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255))
    return SDVG_ERR_MISALIGNED;
  TiledParams p = {};
  int st = sdvg::fill_rope(p, kDim, c->block_tokens, sdvg::RopeArgs{frames, grid_h, grid_w, frame_offset, tab_frames, cos_sin_tab});
  if (st != SDVG_OK) return st;
  int slot = 0;
  if ((st = sdvg::ring_begin_commit(c, block_index, flags, &slot)) != SDVG_OK) return st;
  if ((st = sdvg::require_sm100()) != SDVG_OK) return st;
  int sms = 0;
  if ((st = device_sms(&sms)) != SDVG_OK) return st;
  const cudaStream_t s = (cudaStream_t)stream;
  const int tiles = sdvg::scale_tiles(c->block_tokens);
  p.tokens = c->block_tokens;
  p.heads = c->heads;
  p.eps = eps;
  float* const rstd = scope == SDVG_SCOPE_ROW ? (float*)((char*)workspace + kStatusBytes) : nullptr;
  const long long head_stride = (long long)c->slots * c->block_tokens * (kDim / 8), slot_scale = (long long)slot * tiles;
  auto ring = [&](void* buf) { return (uint2*)buf + sdvg::slot_offset(c, 0, slot) / 8; };
  auto add = [&](const void* src, int64_t ld, uint2* dst, long long token_stride, long long heads_at, float* scale,
                 long long scale_stride, const float* weight, const float* factors, bool turned) {
    p.job[p.jobs++] =
        TileJob{(const __nv_bfloat16*)src, ld, dst, token_stride, heads_at, scale, scale_stride, weight, factors, turned};
  };
  // q was read last by the pass before, and is first to be found in L2
  if (q)
    add(q, ld_q, (uint2*)q8_out, (long long)c->heads * (kDim / 8), kDim / 8, q_tile_scale, tiles, q_weight,
        rstd ? rstd + c->block_tokens : nullptr, true);
  add(k, ld_k, ring(c->k_buf), kDim / 8, head_stride, c->k_tile_scale + slot_scale, (long long)c->slots * tiles, k_weight, rstd, true);
  add(v, ld_v, ring(c->v_buf), kDim / 8, head_stride, c->v_tile_scale + slot_scale, (long long)c->slots * tiles, nullptr, nullptr, false);
  p.groups = head_groups(tiles, c->heads, sms);
  const long long grid = (long long)tiles * p.groups;
  if (grid > 0x7fffffff) return SDVG_ERR_BAD_SHAPE;
  if (scope == SDVG_SCOPE_ROW) {
    StatParams r = {};
    r.src[0] = (const __nv_bfloat16*)k;
    r.src[1] = (const __nv_bfloat16*)q;
    r.ld[0] = ld_k;
    r.ld[1] = ld_q;
    r.rstd = rstd;
    r.tokens = c->block_tokens;
    r.vecs = (int)(width / 8);
    r.eps = eps;
    r.inv_width = 1.f / (float)width;
    constexpr int kPer = kStatThreads / 32;
    st = sdvg::cuda_status(sdvg::launch_overlapped(row_rstd_kernel, dim3((r.tokens + kPer - 1) / kPer, q ? 2 : 1), kStatThreads, 0, 0, s, r));
    if (st != SDVG_OK) return st;
  }
  st = sdvg::cuda_status(sdvg::launch_overlapped(rstd ? qk_tiled_kernel<false> : qk_tiled_kernel<true>, (unsigned)grid, kThreads, kDynamic, 0, s, p));
  if (st != SDVG_OK) return st;
  sdvg::ring_end_commit(c, block_index, flags, slot, evicted_block);
  return SDVG_OK;
}

}  // extern "C"
