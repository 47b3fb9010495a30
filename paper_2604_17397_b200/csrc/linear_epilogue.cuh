// Parts of the linear layers that do not depend on the operands' type: the epilogue, the ring of operand stages, the sum over
// several accumulators, and the order and the sizes of the tiles.  An accumulator lane is an output feature, a column a token.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>

#include "bounded_wait.cuh"
#include "sdvg.h"
#include "sm100_ptx.cuh"

namespace linear {

using namespace sm100;

constexpr int kTileF = 128;                          // features per tile: the instruction's M
constexpr uint64_t kWaitLimitNs = 2000000000ull;     // 2 s per wait

struct EpilogueParams {
  void* out;
  const void* residual;
  const float* bias;
  const float* gate;
  long long ld_out, ld_res, ld_gate;
  int gate_rows;
  int rows, cols;
  int act;
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
template <> struct OutElem<SDVG_E4M3> {
  using T = uint8_t;                                   // codes; what scales them is the layer's
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
__device__ __forceinline__ void load_residual16(const EpilogueParams& p, typename OutElem<OutType>::T (&res)[16], int n,
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
__device__ __forceinline__ TileGate tile_gate(const EpilogueParams& p, int n, int m0, int m_end) {
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

// gate * act(acc + bias) of the first `count` tokens from m0 on.
template <auto ACTIVATE = activate16>
__device__ __forceinline__ void gated16(const EpilogueParams& p, float (&acc)[16], int n, int m0, int count, float b,
                                        const TileGate& gate) {
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[j] += b;
  ACTIVATE(acc, p.act);
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
}

// Epilogue of these tokens: `acc` holds the sums; tokens from `m_end` on are not touched.
template <int OutType, auto ACTIVATE = activate16>
__device__ __forceinline__ void epilogue16(const EpilogueParams& p, float (&acc)[16], typename OutElem<OutType>::T (&res)[16],
                                           int n, int m0, int m_end, float b, const TileGate& gate) {
  using E = OutElem<OutType>;
  using T = typename E::T;
  if (n >= p.cols || m0 >= m_end) return;
  const int count = min(16, m_end - m0);
  const long long ld = stride_here(p.ld_out);
  T* o = static_cast<T*>(p.out) + m0 * ld + n;
  gated16<ACTIVATE>(p, acc, n, m0, count, b, gate);
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

// Adds the accumulators of all chunks (BUFFERS of them in turn) and leaves the total in the tensor memory columns from total_at on
// (behind them, or in place of the only one): a warp's 32 features, SETS sets of 16 columns below `cols`, set i from column_of(i) on.  Between chunks the total is in
// registers.  Returns false when a wait gave up.  `release` tells the issuer that an accumulator is free
// again, as soon as it is read: the products two chunks on wait for it, and those of the next tile would otherwise wait
// for the epilogue.
template <int BUFFERS, int SETS, class Column, class Release>
__device__ __forceinline__ bool add_chunks(int chunks, uint32_t lanes, int acc_stride, int total_at, Column column_of, int cols, RingPos& r,
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
    if (column_of(i) < cols) tmem_st16(lanes + total_at + column_of(i), reinterpret_cast<uint32_t(&)[16]>(sum[i]));
  tmem_wait_st();
  return true;
}

// Tile t of the list: groups of `group` neighbouring feature tiles, token tiles within a group, features innermost, so
// that the pairs that run at the same time share operand tiles in L2 on both sides.
template <class Params>
__device__ __forceinline__ void tile_of(const Params& p, long long t, int* f, int* tok) {
  const long long per_group = (long long)p.group * p.tiles_t;
  const int g = (int)(t / per_group);
  const int r = (int)(t - g * per_group);
  const int width = min(p.group, p.tiles_f - g * p.group);
  *tok = r / width;
  *f = g * p.group + r % width;
}

// Tokens per tile of the pairs: the size whose waves of tiles cost least.  A tile's time grows linearly with its tokens on
// top of a part that does not depend on them (the features' operand tiles come in whatever the token count), worth about
// kFixedTokens: at 4680 x 5120 x 15360 a wave of tiles took 13.9, 18.9, 24.8 and 32.3 us for 64, 128, 192 and 256 tokens.
// Small tiles lose to that part, large ones to the last, partly filled wave (5120 features: 6 waves either way, 179 us at
// 224 tokens and 190 us at 256; 194 us in 10 full waves of 128).
constexpr int kFixedTokens = 80;
inline int pair_tile(int rows, int tiles_f, int pairs, int largest) {
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

}  // namespace linear
