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

#include <algorithm>
#include <mutex>

#include "bounded_wait.cuh"
#include "elem_types.cuh"
#include "overlap.cuh"
#include "sdvg_internal.h"
#include "sm100_ptx.cuh"
#include "tensor_map.h"

namespace {

using namespace sm100;

constexpr int kTileF = 128;                          // features per tile: the instruction's M
constexpr int kTileK = 64;                           // elements of `inner` per stage: one 128-byte swizzled row
constexpr int kMaxTileT = 256;                       // tokens per tile: the instruction's N, a multiple of 16
constexpr uint64_t kWaitLimitNs = 2000000000ull;     // 2 s per wait
constexpr int kMaxStages = 8;
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
  int tile_t, tiles_f, tiles_t, k_iters, stages;
  int split;                                         // CTAs (a cluster) that share a tile's sum; tiles only
  int group;                                         // feature tiles of a group of the tile order (pairs)
  long long tiles;
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

// The exponential forms keep their relative accuracy where the value vanishes: v / (1 + e^-z) tends to -0 for z -> -inf
// (the exponential overflows to infinity; a denominator past 2^126 gives 0 already, for a value of 1e-36).
//
// GELU: v Phi(v) with the lower tail h = erfc(z) / 2, z = |v| / sqrt 2, taken directly, without the cancellation of 1 + erf:
// erfc(z) e^(z^2) / t with t = 1 / (1 + 0.45 z) is smooth on 0 < t <= 1, and a polynomial of degree 9 in t, fitted by
// least squares with weights driven towards an even relative error, is within 3.3e-8 of it (relative, in exact arithmetic;
// 6.2e-7 in fp32 for |v| < 3, 4.1e-6 at |v| = 12, where the rounding of v^2 counts).  The library's erfcf, 16 at a time,
// took so many registers that others spilled.  For v > 0 the tail is taken off with a bounded factor: past 15 it is 0 in fp32 and
// the result is v itself, at infinity too, where v h would be infinity times 0.
__device__ __forceinline__ float gelu_erf(float v) {
  const float z = fabsf(v);
  const float t = __fdividef(1.f, fmaf(0.31819805f, z, 1.f));
  float q = -0.02069617911700f;
  q = fmaf(q, t, 0.09534660188561f);
  q = fmaf(q, t, -0.15029583590903f);
  q = fmaf(q, t, 0.07120466716636f);
  q = fmaf(q, t, -0.01118113013510f);
  q = fmaf(q, t, 0.05997585263270f);
  q = fmaf(q, t, 0.08762596187607f);
  q = fmaf(q, t, 0.11413582878705f);
  q = fmaf(q, t, 0.12694158118874f);
  q = fmaf(q, t, 0.12694266037636f);
  const float h = q * t * __expf(-0.5f * v * v);
  return v > 0.f ? fmaf(-fminf(v, 1e4f), h, v) : v * h;
}

// The choice is made once for the 16 values, and the epilogue is instantiated once per kernel: unrolled over a tile with
// the choice inside, its code outgrew the instruction caches and the fetches took ten times the arithmetic.
__device__ __forceinline__ void activate16(float (&v)[16], int act) {
  if (act == SDVG_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __fdividef(v[j], 1.f + __expf(-v[j]));
  } else if (act == SDVG_ACT_GELU_TANH) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      v[j] = __fdividef(v[j], 1.f + __expf(-1.5957691216057308f * fmaf(0.044715f * v[j] * v[j], v[j], v[j])));
  } else if (act == SDVG_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = gelu_erf(v[j]);
  }
}

// A row stride whose multiples the compiler must form where they are used: hoisted out of the epilogue's loop, 16 of them
// for each of two matrices cost 64 registers and spilled others into its loop.
__device__ __forceinline__ long long stride_here(long long ld) {
  asm volatile("" : "+l"(ld));
  return ld;
}

// Residual of 16 tokens m0 .. of one feature n, requested a block ahead of its use: the epilogue would otherwise spend
// most of its time waiting for these loads.
template <int OutType>
__device__ __forceinline__ void load_residual16(const LinearParams& p, typename OutElem<OutType>::T (&res)[16], int n,
                                                int m0, int m_end) {
  using T = typename OutElem<OutType>::T;
  if (!p.residual || n >= p.cols) return;
  const long long ld = stride_here(p.ld_res);
  const T* r = static_cast<const T*>(p.residual) + m0 * ld + n;
  if (m0 + 16 <= m_end) {
#pragma unroll
    for (int j = 0; j < 16; ++j, r += ld) res[j] = *r;
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j, r += ld)
      if (m0 + j < m_end) res[j] = *r;
  }
}

// The gate of one feature over a tile's tokens m0 .. m_end: nearly always one or two groups, whose values are fetched once per
// tile; `border` is the first token of the second.
struct TileGate {
  float first, second;
  int border;
  bool few;                                            // at most two groups
};
__device__ __forceinline__ TileGate tile_gate(const LinearParams& p, int n, int m0, int m_end) {
  TileGate g{1.f, 1.f, 0x7fffffff, true};
  if (!p.gate || n >= p.cols || m0 >= m_end) return g;
  const int group = m0 / p.gate_rows;
  const long long border = (long long)(group + 1) * p.gate_rows;
  const float* at = p.gate + group * p.ld_gate + n;
  g.first = at[0];
  if (border < m_end) {
    g.border = (int)border;
    g.second = at[p.ld_gate];
    g.few = border + p.gate_rows >= m_end;
  }
  return g;
}

// Epilogue of these tokens: `acc` holds the sums; tokens from `m_end` on are not touched.
template <int OutType>
__device__ __forceinline__ void epilogue16(const LinearParams& p, float (&acc)[16], typename OutElem<OutType>::T (&res)[16],
                                           int n, int m0, int m_end, float b, const TileGate& gate) {
  using E = OutElem<OutType>;
  using T = typename E::T;
  if (n >= p.cols || m0 >= m_end) return;
  const int count = min(16, m_end - m0);
  const long long ld = stride_here(p.ld_out);
  T* o = static_cast<T*>(p.out) + m0 * ld + n;
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[j] += b;
  activate16(acc, p.act);
  if (p.gate) {
    if (gate.few) {
#pragma unroll
      for (int j = 0; j < 16; ++j) acc[j] *= m0 + j < gate.border ? gate.first : gate.second;
    } else {
      const int group = m0 / p.gate_rows;
      const float* gp = p.gate + group * p.ld_gate + n;
      long long next = (long long)(group + 1) * p.gate_rows;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (j < count) {
          if (m0 + j == next) {
            gp += p.ld_gate;
            next += p.gate_rows;
          }
          acc[j] *= *gp;
        }
      }
    }
  }
  if (p.residual) {
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] += E::get(res[j]);
  }
  if (count == 16) {
#pragma unroll
    for (int j = 0; j < 16; ++j, o += ld) *o = E::put(acc[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j, o += ld)
      if (j < count) *o = E::put(acc[j]);
  }
}

// Position in the ring of operand stages: the stage and the parity of its current use.
struct RingPos {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) {
      stage = 0;
      phase ^= 1;
    }
  }
  __device__ __forceinline__ void back(int stages) {
    if (--stage < 0) {
      stage = stages - 1;
      phase ^= 1;
    }
  }
};

// fp32 outputs: the tensor core adds a product to the accumulator by truncation, so a sum over `inner` drifts in one
// direction by about 2^-26 of its magnitude per 16 products (measured 3.7e-6 relative for inner = 5120, fp32's own
// rounding giving 1e-7).  That is far below the rounding of a 16-bit output but not of an fp32 one, so there the sum is
// cut into chunks: each chunk gets a fresh accumulator, and the epilogue warps add the chunks with round-to-nearest.
// Relative errors at 300 x 6144 x 512: 1.0e-6 with chunks of 1024, 7.3e-7 with 768, 6.1e-7 with 640, 4.8e-7 with 512.  For many
// tokens short chunks cost time, since tensor memory is read slowly under products (4680 x 6144 x 1536 with gate and
// residual: 93, 96 and 100 us with 768, 640 and 512; a whole sum 89); for few they do not (3 x 5120 x 30720: 50 us and 4.8e-7
// with 512, 50 and 2.4e-7 with 256, 51 and 1.7e-7 with 128).
constexpr int kPairChunkIters = 640 / kTileK;
constexpr int kTileChunkIters = 256 / kTileK;

// ---- few tokens: a cluster per tile, which splits `inner` ---------------------------------------
//
// One tile is 128 features x tile_t tokens.  With few tokens there are few tiles and each is a long sum, bound by how fast
// the weights arrive: the CTAs of a cluster each take a part of `inner`, leave their sums in shared memory, and after a
// cluster barrier every CTA adds up its share of the tokens from all of them (distributed shared memory, always in the
// order of the ranks) and runs the epilogue on it.  No workspace, no atomics, equal calls give equal bits.
constexpr int kTileThreads = 192;                    // four epilogue warps, producer, issuer
constexpr int kMaxTileFew = 64;                      // tokens per tile
constexpr int kMaxSplit = 8;                         // portable cluster size

struct TileSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full, acc_empty;
  uint32_t tmem;
};

// Tensor memory columns: the accumulator, and the total if there are several chunks; a power of two.
__host__ __device__ constexpr uint32_t tile_tmem_cols(int tile_t, bool with_total) {
  uint32_t cols = 32;
  while (cols < (uint32_t)tile_t * (with_total ? 2 : 1)) cols *= 2;
  return cols;
}

// Adds the accumulators of all chunks (BUFFERS of them in turn) and leaves the total in the tensor memory columns behind them:
// a warp's 32 features, SETS sets of 16 columns below `cols`, set i from column_of(i) on.  Between chunks the total is in
// registers.  Returns false when a wait gave up.  `release` tells the issuer that an accumulator is free
// again, as soon as it is read: the products two chunks on wait for it, and those of the next tile would otherwise wait
// for the epilogue.
template <int BUFFERS, int SETS, class Column, class Release>
__device__ __forceinline__ bool add_chunks(int chunks, uint32_t lanes, int acc_stride, Column column_of, int cols, RingPos& r,
                                           uint64_t* acc_full, unsigned int* status, Release release) {
  float sum[SETS][16];
#pragma unroll
  for (int i = 0; i < SETS; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[i][j] = 0.f;
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    if (!__all_sync(0xffffffffu, wait_for(&acc_full[r.stage], r.phase, status, kWaitLimitNs))) return false;
    tc_fence_after();
    const uint32_t part = lanes + r.stage * acc_stride;
#pragma unroll
    for (int i = 0; i < SETS; ++i)
      if (column_of(i) < cols) {
        float v[16];
        tmem_ld16(part + column_of(i), reinterpret_cast<uint32_t(&)[16]>(v));
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[i][j] += v[j];
      }
    tc_fence_before();
    __syncwarp();
    release(r.stage);
    r.next(BUFFERS);
  }
#pragma unroll
  for (int i = 0; i < SETS; ++i)
    if (column_of(i) < cols) tmem_st16(lanes + BUFFERS * acc_stride + column_of(i), reinterpret_cast<uint32_t(&)[16]>(sum[i]));
  tmem_wait_st();
  return true;
}

template <int OutType>
__global__ void __launch_bounds__(kTileThreads) linear_tile_kernel(const __grid_constant__ LinearParams p) {
  constexpr bool kChunked = OutType == SDVG_F32;
  using T = typename OutElem<OutType>::T;
  extern __shared__ uint8_t raw[];
  __shared__ TileSmem sm;
  uint8_t* buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0, tile = blockIdx.x / p.split;
  const int n0 = (tile % p.tiles_f) * kTileF;
  const int m0 = (tile / p.tiles_f) * p.tile_t, m_end = min(p.rows, m0 + p.tile_t);
  const int w_bytes = kTileF * 128, stage_bytes = w_bytes + p.tile_t * 128;
  // this CTA's part of `inner`: never empty
  const int share = p.k_iters / p.split, rest = p.k_iters % p.split;
  const int k0 = rank * share + min(rank, rest), iters = share + (rank < rest ? 1 : 0);
  const int chunks = kChunked ? (iters + kTileChunkIters - 1) / kTileChunkIters : 1;
  const uint32_t tmem_cols = tile_tmem_cols(p.tile_t, kChunked && p.k_iters > kTileChunkIters);
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    mbar_init(&sm.acc_full, 1);
    mbar_init(&sm.acc_empty, 4);
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
  sdvg::overlap_wait();

  if (warp == 4) {
    if (elect_one()) {
      int i = 0;
      RingPos r;
      for (; i < iters; ++i, r.next(p.stages)) {
        const int s = r.stage;
        if (!wait_for(&sm.empty[s], r.phase ^ 1, p.status, kWaitLimitNs)) break;
        uint8_t* st = buf + s * stage_bytes;
        mbar_expect_tx(&sm.full[s], stage_bytes);
        tma_load_2d(st, &p.w_map, &sm.full[s], (k0 + i) * kTileK, n0);
        tma_load_2d(st + w_bytes, &p.x_map, &sm.full[s], (k0 + i) * kTileK, m0);
      }
      // only now: SMs hold several of these CTAs, and a next grid that starts while they still hold them lands on the SMs
      // with room, which are not the ones that will be idle (3 x 5120 x 30720 back to back: 62 us when begun at the start, 51 here)
      sdvg::overlap_begin();
      if (i < iters)                                   // gave up: see the copies in flight land before the CTA may leave
        for (int j = min(i, p.stages); j > 0; --j) {
          r.back(p.stages);
          wait_for(&sm.full[r.stage], r.phase, p.status, kWaitLimitNs);
        }
    }
    __syncwarp();
  } else if (warp == 5) {
    if (elect_one()) {
      bool ok = true;
      RingPos r, acc;
      for (int c = 0; ok && c < chunks; ++c, acc.next(1)) {
        if (!(ok = wait_for(&sm.acc_empty, acc.phase ^ 1, p.status, kWaitLimitNs))) break;
        tc_fence_after();
        const int i0 = c * kTileChunkIters, i1 = kChunked ? min(iters, i0 + kTileChunkIters) : iters;
        for (int i = i0; i < i1; ++i, r.next(p.stages)) {
          const int s = r.stage;
          if (!(ok = wait_for(&sm.full[s], r.phase, p.status, kWaitLimitNs))) break;
          tc_fence_after();
          const uint32_t st = smem_u32(buf + s * stage_bytes);
          const uint64_t a = smem_desc_sw128(st, 16, 1024), b = smem_desc_sw128(st + w_bytes, 16, 1024);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ss(tmem, a + 2 * kk, b + 2 * kk, p.idesc, i > i0 || kk > 0);
          mma_commit(&sm.empty[s]);
        }
        if (ok) mma_commit(&sm.acc_full);
      }
    }
    __syncwarp();
  } else {
    const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
    const int n = n0 + warp * 32 + lane;
    const float b = p.bias && n < p.cols ? p.bias[n] : 0.f;
    RingPos r;
    const bool summed = kChunked && chunks > 1;
    bool ok;
    if (summed)
      ok = add_chunks<1, kMaxTileFew / 16>(chunks, lanes, p.tile_t, [](int i) { return 16 * i; }, m_end - m0, r, &sm.acc_full, p.status, [&](int) {
        if (lane == 0) mbar_arrive(&sm.acc_empty);
      });
    else
      ok = __all_sync(0xffffffffu, wait_for(&sm.acc_full, r.phase, p.status, kWaitLimitNs));
    if (ok) {
      tc_fence_after();
      const uint32_t sums = lanes + (summed ? p.tile_t : 0);
      const TileGate gate = tile_gate(p, n, m0, m_end);
      float* mine = reinterpret_cast<float*>(buf) + warp * 32 + lane;      // [token][128 features]: the ring is read and free
#pragma unroll 1
      for (int c = 0; m0 + c < m_end; c += 16) {
        float acc[16];
        T res[16];
        if (p.split == 1) load_residual16<OutType>(p, res, n, m0 + c, m_end);
        tmem_ld16(sums + c, reinterpret_cast<uint32_t(&)[16]>(acc));
        tmem_wait_ld();
        if (p.split == 1) {
          epilogue16<OutType>(p, acc, res, n, m0 + c, m_end, b, gate);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) mine[(c + j) * kTileF] = acc[j];
        }
      }
    }
  }
  if (p.split > 1) {
    // a CTA that gave up joins the barriers as well; the status word says that the outputs are undefined
    cluster_arrive();
    cluster_wait();
    if (warp < 4) {
      const int per = (m_end - m0 + p.split - 1) / p.split, first = rank * per, last = min(m_end - m0, first + per);
      const int n = n0 + warp * 32 + lane;
      const float b = p.bias && n < p.cols ? p.bias[n] : 0.f;
      const uint32_t mine = smem_u32(buf) + (warp * 32 + lane) * 4;
      const TileGate gate = tile_gate(p, n, m0 + first, m0 + last);
#pragma unroll 1
      for (int c = first; c < last; c += 16) {
        T res[16];
        load_residual16<OutType>(p, res, n, m0 + c, m0 + last);
        float acc[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[j] = 0.f;
#pragma unroll 1
        for (int s = 0; s < p.split; ++s) {
          const uint32_t from = map_to_rank(mine, s);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (c + j < last) acc[j] += ld_cluster_f32(from + (c + j) * kTileF * 4);
        }
        epilogue16<OutType>(p, acc, res, n, m0 + c, m0 + last, b, gate);
      }
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();                                    // nobody leaves while its sums may still be read
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(tmem, tmem_cols);
}

// ---- many tokens: CTA pairs, persistent ---------------------------------------------------------
//
// A pair of CTAs (two SMs) works on one tile of 256 features x tile_t tokens: each CTA holds 128 of the features (its
// accumulator lanes) and fetches half of the token tile, and one tcgen05.mma of the even CTA reads both halves, so that a
// token tile crosses into shared memory once per pair.  Accumulators are double-buffered in tensor memory (2 x 256
// columns): the epilogue of one tile runs under the products of the next.
//
// What bounds it: per stage of 64 elements a CTA's tensor core takes 2 tile_t clocks, and its shared memory 256 + tile_t
// (16 KB of weights and 64 tile_t bytes of tokens, written once and read once, at 128 bytes a clock; measured over `inner`:
// 167, 190, 240 and 340 ns a stage for 64, 128, 176 and 256 tokens).  So tiles of 256 tokens are balanced and smaller ones
// wait for shared memory; on long runs the power cap holds both back.  4680 x 5120 x 5120 with gate and residual: tensor
// pipe active 89% of the time.  Under the power cap, back to back, over several boxes: 4680 x 5120 x 15360 552 to 595 us (1334 to
// 1237 TFLOP/s; a library product alone 542 to 560), x 20480 with GELU 737 to 780 (706 to 733).
constexpr int kEpiWarps = 8;
constexpr int kPairThreads = 32 * (kEpiWarps + 2);
constexpr int kPairSmem = 227 * 1024 - 512;          // dynamic shared memory of a CTA; the barriers are static
// Tokens per tile of a chunked sum: a thread holds half of them between chunks.
constexpr int kMaxTileChunked = 128;
// Accumulators in tensor memory and their columns.  A chunked sum has three (and its total behind them): reading one takes about
// as long as the products of a chunk, and with two the products waited for it (chunks of 512: 105 against 100 us).
template <int OutType>
constexpr int kAccs = OutType == SDVG_F32 ? 3 : 2;
template <int OutType>
constexpr int kAccStride = OutType == SDVG_F32 ? kMaxTileChunked : kMaxTileT;
static_assert((kAccs<SDVG_F32> + 1) * kAccStride<SDVG_F32> <= 512 && kAccs<SDVG_BF16> * kAccStride<SDVG_BF16> <= 512);

struct PairSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], acc_full[3], acc_empty[3];
  uint32_t tmem;
};

// Tile t of the list: groups of `group` neighbouring feature tiles, token tiles within a group, features innermost, so
// that the pairs that run at the same time share operand tiles in L2 on both sides.
__device__ __forceinline__ void tile_of(const LinearParams& p, long long t, int* f, int* tok) {
  const long long per_group = (long long)p.group * p.tiles_t;
  const int g = (int)(t / per_group);
  const int r = (int)(t - g * per_group);
  const int width = min(p.group, p.tiles_f - g * p.group);
  *tok = r / width;
  *f = g * p.group + r % width;
}

template <int OutType>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    linear_pair_kernel(const __grid_constant__ LinearParams p) {
  constexpr bool kChunked = OutType == SDVG_F32;
  using T = typename OutElem<OutType>::T;
  extern __shared__ uint8_t raw[];
  __shared__ PairSmem sm;
  uint8_t* buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const int w_bytes = kTileF * 128, stage_bytes = w_bytes + p.tile_t * 64;
  const int chunks = kChunked ? (p.k_iters + kPairChunkIters - 1) / kPairChunkIters : 1;
  sdvg::overlap_begin();
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&sm.full[s], 1);                     // the even CTA's counts the bytes of both
      mbar_init(&sm.empty[s], 1);
    }
    for (int b = 0; b < kAccs<OutType>; ++b) {
      mbar_init(&sm.acc_full[b], 1);
      mbar_init(&sm.acc_empty[b], 2 * kEpiWarps);    // the even CTA's: the epilogue warps of both
    }
    fence_mbar_init();
    prefetch_tmap(&p.w_map);
    prefetch_tmap(&p.x_map);
  }
  if (warp == 0) {
    tmem_alloc_pair(&sm.tmem, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                                    // the other CTA's barriers are initialised as well
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  sdvg::overlap_wait();

  if (warp == kEpiWarps) {
    // ================= producer: this CTA's features and its half of the token tile =================
    if (elect_one()) {
      RingPos r;
      int issued = 0;                                // up to the number of stages
      bool ok = true;
      for (long long t = pair; ok && t < p.tiles; t += pairs) {
        int ft, tt;
        tile_of(p, t, &ft, &tt);
        const int n0 = (2 * ft + (int)rank) * kTileF, m0 = tt * p.tile_t + (int)rank * (p.tile_t / 2);
        for (int i = 0; i < p.k_iters; ++i, r.next(p.stages)) {
          const int s = r.stage;
          if (!(ok = wait_for(&sm.empty[s], r.phase ^ 1, p.status, kWaitLimitNs))) break;
          issued = min(issued + 1, p.stages);
          uint8_t* st = buf + s * stage_bytes;
          const uint32_t full = map_to_rank(smem_u32(&sm.full[s]), 0);
          if (rank == 0) mbar_expect_tx(&sm.full[s], 2 * stage_bytes);
          tma_load_2d_pair(st, &p.w_map, full, i * kTileK, n0);
          tma_load_2d_pair(st + w_bytes, &p.x_map, full, i * kTileK, m0);
        }
      }
      // every stage is read (on a give-up: landed, as far as this CTA can tell) before the CTA may leave
      for (; issued > 0; --issued) {
        r.back(p.stages);
        if (ok) ok = wait_for(&sm.empty[r.stage], r.phase, p.status, kWaitLimitNs);
        else if (rank == 0) wait_for(&sm.full[r.stage], r.phase, p.status, kWaitLimitNs);
      }
    }
  } else if (warp == kEpiWarps + 1) {
    // ================= issuer: the even CTA, for both ==============================================
    if (rank == 0 && elect_one()) {
      RingPos r, acc;
      bool ok = true;
      for (long long t = pair; ok && t < p.tiles; t += pairs) {
        for (int c = 0; ok && c < chunks; ++c, acc.next(kAccs<OutType>)) {
          const int b = acc.stage;
          if (!(ok = wait_for(&sm.acc_empty[b], acc.phase ^ 1, p.status, kWaitLimitNs))) break;
          tc_fence_after();
          const int i0 = c * kPairChunkIters, i1 = kChunked ? min(p.k_iters, i0 + kPairChunkIters) : p.k_iters;
          for (int i = i0; i < i1; ++i, r.next(p.stages)) {
            const int s = r.stage;
            if (!(ok = wait_for(&sm.full[s], r.phase, p.status, kWaitLimitNs))) break;
            tc_fence_after();
            const uint32_t st = smem_u32(buf + s * stage_bytes);
            const uint64_t da = smem_desc_sw128(st, 16, 1024), db = smem_desc_sw128(st + w_bytes, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ss_pair(tmem + b * kAccStride<OutType>, da + 2 * kk, db + 2 * kk, p.idesc, i > i0 || kk > 0);
            mma_commit_pair(&sm.empty[s]);
          }
          if (ok) mma_commit_pair(&sm.acc_full[b]);
        }
      }
    }
  } else if (warp < kEpiWarps) {
    // ================= epilogue: warps w and w + 4 share 32 features and take 32-token column blocks in turn ==========
    const int quad = warp % 4, half = warp / 4;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t empty = map_to_rank(smem_u32(sm.acc_empty), 0);
    RingPos r;
    bool ok = true;
    for (long long t = pair; ok && t < p.tiles; t += pairs) {
      int ft, tt;
      tile_of(p, t, &ft, &tt);
      const int n = (2 * ft + (int)rank) * kTileF + quad * 32 + lane;
      const int m0 = tt * p.tile_t, m_end = min(p.rows, m0 + p.tile_t);
      const float bias = p.bias && n < p.cols ? p.bias[n] : 0.f;
      // this warp's columns: blocks of 32 from 32 half on, 64 apart, handled as two halves of 16
      const TileGate gate = tile_gate(p, n, m0, m_end);
      T ahead0[16], ahead1[16];
      load_residual16<OutType>(p, ahead0, n, m0 + half * 32, m_end);
      load_residual16<OutType>(p, ahead1, n, m0 + half * 32 + 16, m_end);
      auto release = [&](int stage) {
        if (lane == 0) mbar_arrive_cluster(empty + 8 * stage);
      };
      const bool summed = kChunked && chunks > 1;
      if (summed)
        ok = add_chunks<kAccs<OutType>, kMaxTileChunked / 32>(
            chunks, lanes, kAccStride<OutType>, [&](int i) { return (i / 2 * 2 + half) * 32 + (i & 1) * 16; }, m_end - m0, r,
            sm.acc_full, p.status, release);
      else
        ok = __all_sync(0xffffffffu, wait_for(&sm.acc_full[r.stage], r.phase, p.status, kWaitLimitNs));
      if (!ok) break;
      tc_fence_after();
      const uint32_t sums = lanes + (summed ? kAccs<OutType> : r.stage) * kAccStride<OutType>;
#pragma unroll 1
      for (int col = half * 32; m0 + col < m_end; col += 64) {
        float acc0[16], acc1[16];
        tmem_ld16(sums + col, reinterpret_cast<uint32_t(&)[16]>(acc0));
        tmem_ld16(sums + col + 16, reinterpret_cast<uint32_t(&)[16]>(acc1));
        tmem_wait_ld();
        epilogue16<OutType>(p, acc0, ahead0, n, m0 + col, m_end, bias, gate);
        load_residual16<OutType>(p, ahead0, n, m0 + col + 64, m_end);
        epilogue16<OutType>(p, acc1, ahead1, n, m0 + col + 16, m_end, bias, gate);
        load_residual16<OutType>(p, ahead1, n, m0 + col + 80, m_end);
      }
      if (!summed) {
        tc_fence_before();
        __syncwarp();
        release(r.stage);
        r.next(kAccs<OutType>);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();                                    // neither CTA leaves while the other may still reach into it
  tc_fence_after();
  if (warp == 0) tmem_dealloc_pair(tmem, 512);
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

// More tokens than this go to the pairs.  At 5120 x 5120: 64 tokens 17.7 us (clusters of four) against 19.5, 128 tokens 20.6
// (clusters of two) against 19.4.
constexpr int kPairRows = kMaxTileFew;

// Tokens per tile of the pairs: the size whose waves of tiles cost least.  A tile's time grows linearly with its tokens on
// top of a part that does not depend on them (the features' operand tiles come in whatever the token count), worth about
// kFixedTokens: at 4680 x 5120 x 15360 a wave of tiles took 13.9, 18.9, 24.8 and 32.3 us for 64, 128, 192 and 256 tokens.
// Small tiles lose to that part, large ones to the last, partly filled wave (5120 features: 6 waves either way, 179 us at
// 224 tokens and 190 us at 256; 194 us in 10 full waves of 128).
constexpr int kFixedTokens = 80;
int pair_tile(int rows, int tiles_f, int pairs, int largest) {
  int best = largest;
  long long best_cost = 0;
  for (int nt = largest; nt >= 64; nt -= 16) {
    const long long tiles = (long long)tiles_f * ((rows + nt - 1) / nt);
    const long long cost = (tiles + pairs - 1) / pairs * (nt + kFixedTokens);
    if (!best_cost || cost < best_cost) {
      best = nt;
      best_cost = cost;
    }
  }
  return best;
}

constexpr int kTileStages = 4;
constexpr int kTileDynamic = kTileStages * (kTileF + kMaxTileFew) * 128 + 1024;

// The CTAs that an SM can hold find their tensor memory columns at once, because no tile takes a larger share of an SM's
// columns than of its shared memory.  That matters for a cluster: its CTAs wait for each other, and if one of them could
// wait for columns that a CTA of another waiting cluster holds, two clusters could wait for each other for good.
constexpr bool columns_within_share(int tile_t) {
  return tile_tmem_cols(tile_t, true) * (228 * 1024 / 512) <= (uint32_t)(kTileStages * (kTileF + tile_t) * 128 + 1024);
}
static_assert(columns_within_share(16) && columns_within_share(32) && columns_within_share(48) && columns_within_share(64));
static_assert(kMaxTileFew == 64, "the sizes checked above");

// CTAs per tile: as many as it takes to give every SM work, while all of them run at once and each keeps four stages of the sum,
// or eight where the SMs have more than one CTA then (a second CTA per SM brings less).  Measured in graphs, times in us for
// 1, 2, 4 and 8 parts: one row, 1536 x 1536 5.9, 5.6, 5.2, 6.1; 3 rows, 5120 x 5120 24.3, 16.2, 13.7, 15.3 and 1536 x 9216 9.7, 9.2,
// 10.2, 17.2; 5 rows, 700 x 12000 5.8, 7.1, 8.2, 18.6; 64 rows, 6144 x 1536 27.2, 18.2, 12.7, 11.9.
int tile_split(long long tiles, int k_iters, int tile_t, int sms) {
  const int per_sm = 228 * 1024 / (kTileStages * (kTileF + tile_t) * 128 + 3 * 1024);
  int split = 1;
  while (split < kMaxSplit && tiles * split < sms && tiles * 2 * split <= (long long)sms * per_sm &&
         k_iters >= (tiles * 2 * split <= sms ? 8 : 16) * split)
    split *= 2;
  return split;
}

// One-time set-up per device and output type: the opt-in to the kernels' dynamic shared memory, and how many CTA pairs
// the device runs at once.
template <int OutType>
int set_up(int* pairs) {
  static int pairs_of_device[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return sdvg::cuda_status(e);
  if (dev < 0 || dev >= kMaxDevices) return SDVG_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lock(g_setup_mu);
  if (!pairs_of_device[dev]) {
    e = cudaFuncSetAttribute(linear_tile_kernel<OutType>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileDynamic);
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    e = cudaFuncSetAttribute(linear_pair_kernel<OutType>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kPairSmem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, linear_pair_kernel<OutType>, &cfg);
    if (e != cudaSuccess || n < 1) return sdvg::cuda_status(e != cudaSuccess ? e : cudaErrorUnknown);
    pairs_of_device[dev] = n;
  }
  *pairs = pairs_of_device[dev];
  return SDVG_OK;
}

template <int OutType>
int launch(LinearParams& p, const void* x, int64_t ld_x, const void* w, int64_t ld_w, int inner, int in_type,
           cudaStream_t stream) {
  int pairs = 0;
  int st = set_up<OutType>(&pairs);
  if (st != SDVG_OK) return st;
  const bool by_pair = p.rows > kPairRows;
  const int feature_tile = by_pair ? 2 * kTileF : kTileF;
  p.tiles_f = (p.cols + feature_tile - 1) / feature_tile;
  if (by_pair) p.tile_t = pair_tile(p.rows, p.tiles_f, pairs, OutType == SDVG_F32 ? kMaxTileChunked : kMaxTileT);
  else p.tile_t = (std::min(p.rows, kMaxTileFew) + 15) / 16 * 16;
  p.tiles_t = (p.rows + p.tile_t - 1) / p.tile_t;
  p.tiles = (long long)p.tiles_f * p.tiles_t;
  if (p.tiles >= 1ll << 28) return SDVG_ERR_BAD_SHAPE;
  p.idesc = idesc_16bit_f32(feature_tile, p.tile_t, in_type == SDVG_BF16);
  if ((st = make_map(&p.w_map, w, in_type, inner, p.cols, ld_w, kTileF)) != SDVG_OK) return st;
  if ((st = make_map(&p.x_map, x, in_type, inner, p.rows, ld_x, by_pair ? p.tile_t / 2 : p.tile_t)) != SDVG_OK) return st;
  if (by_pair) {
    // anything from 2 to 16 is within 3% of the best: 565 to 582 us at 4680 x 5120 x 15360 (4 best), 98 to 101 at 4680 x 6144 x 1536
    // into fp32 (8 and up best); wider groups run out of L2, 64: 742 us there
    p.group = 8;
    p.stages = std::min(kMaxStages, (kPairSmem - 1024) / (kTileF * 128 + p.tile_t * 64));
    const int grid = 2 * (int)std::min((long long)pairs, p.tiles);
    return sdvg::cuda_status(
        sdvg::launch_overlapped(linear_pair_kernel<OutType>, grid, kPairThreads, kPairSmem, 0, stream, p));
  }
  p.split = tile_split(p.tiles, p.k_iters, p.tile_t, 2 * pairs);
  p.stages = kTileStages;
  return sdvg::cuda_status(sdvg::launch_overlapped(linear_tile_kernel<OutType>, (unsigned)p.tiles * p.split, kTileThreads,
                                                   p.stages * (kTileF + p.tile_t) * 128 + 1024, p.split > 1 ? p.split : 0,
                                                   stream, p));
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
  constexpr int kMaxInner = 1 << 26;                             // one sum stays far below the limit of a wait
  if (rows < 0 || cols < 0 || inner < 1 || rows > kMaxExtent || cols > kMaxExtent || inner > kMaxInner)
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
  p.k_iters = (inner + kTileK - 1) / kTileK;
  p.status = (unsigned int*)workspace + 1;
  const cudaStream_t s = (cudaStream_t)stream;
  if (out_type == SDVG_F32) return launch<SDVG_F32>(p, x, ld_x, w, ld_w, inner, in_type, s);
  if (out_type == SDVG_F16) return launch<SDVG_F16>(p, x, ld_x, w, ld_w, inner, in_type, s);
  return launch<SDVG_BF16>(p, x, ld_x, w, ld_w, inner, in_type, s);
}

}  // extern "C"
