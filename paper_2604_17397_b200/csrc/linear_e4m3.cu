// Linear layer on E4M3 operands with power-of-two block scales: out = residual + gate * act(x W^T + bias), where a row of x has one
// scale per 128 elements of `inner`, and W one per 128 x 128 block (or per row and 128 elements).
//
// The scales never meet the sums in registers: the tensor core takes them itself (tcgen05.mma kind::mxf8f6f4.block_scale, one
// exponent byte per operand row and step of 32 elements).  Four instructions of 32 elements make a stage of 128, so all
// four take the same byte, and a 32-bit word of scales serves four stages.  As in linear.cu the weights are the M-side
// operand, accumulator lanes are features and columns tokens; a stage is the same 128-byte rows with twice the elements.
//
// A warp of its own brings the scales: it gathers the words of the tile's rows (row-major bytes, so that whoever made them
// needs to know no layout), puts them into shared memory in the order of the tensor core and hands them to the issuer, which
// copies them to tensor memory (tcgen05.cp) in order with its products.
#include <cuda.h>
#include <math.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "e4m3_scale.cuh"
#include "elem_types.cuh"
#include "linear_e4m3_cut.h"
#include "linear_epilogue.cuh"
#include "overlap.cuh"
#include "row_team.cuh"
#include "sdvg_internal.h"
#include "tensor_map.h"

namespace {

using namespace linear;
using namespace linear8;

static_assert(kTileFeatures == kTileF);

constexpr int kWordStages = 4;                       // stages that a 32-bit word of scales serves
constexpr int kMaxStages = 8;
constexpr int kWorkspaceBytes = 256;
constexpr int kMaxDevices = 64;

struct alignas(64) Linear8Params : EpilogueParams {
  CUtensorMap w_map;                                 // box 128 x the features of a CTA: 128, or 256 (pairs with SUBS = 2)
  CUtensorMap x_map;                                 // box 128 x tile_t tokens (tiles), or half of them (pairs)
  const uint8_t *x_scale, *w_scale;                  // exponent bytes: of row r and 128-element block b at scale[(r >> shift) * ld + b]
  long long ld_xs, ld_ws;
  int w_shift;                                       // 0 or 7
  bool x_vec, w_vec;                                 // rows of scales can be read 16 bytes at a time
  uint8_t* out_scale;                                // 8-bit outputs: exponent byte of row r and 128-column block b
  long long ld_os;
  int tile_t, tiles_f, tiles_t, k_iters, stages;
  int split;                                         // CTAs (a cluster) that share a tile's sum; tiles only
  int group;                                         // feature tiles of a group of the tile order (pairs)
  int whole;                                         // sums are not cut into chunks (pairs)
  long long tiles;
  uint32_t idesc;
  unsigned int* status;
};

// Word `word` (blocks 4 word .. 4 word + 3) of a row of `blocks` exponent bytes; bytes past the row's end are not read.
__device__ __forceinline__ uint32_t scale_word(const uint8_t* row, int word, int blocks) {
  const uint8_t* at = row + 4 * word;
  if (4 * word + 4 <= blocks) return *reinterpret_cast<const uint32_t*>(at);
  uint32_t v = 0;
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (4 * word + j < blocks) v |= (uint32_t)at[j] << (8 * j);
  return v;
}

// The scales of rows r0 + lane, + 32, .. (GROUPS * 128 of them; those from r_end on are 0), four words of each at a time: fetched
// word by word, a word took a way to memory and back, 2200 clocks for four stages that take 800 (333 x 5120 x 776: 17.4 us).
template <int GROUPS>
struct ScaleWords {
  uint32_t w[4 * GROUPS][4];
  // Words 4 v .. 4 v + 3 of `blocks` bytes.  vec: rows begin at multiples of 16 bytes, and are read 16 bytes at a time; of the last row, `last`,
  // whose stride may not be there, only what is whole.
  __device__ __forceinline__ void load(const uint8_t* scale, long long ld, int shift, int r0, int r_end, int last, int v, int blocks,
                                       bool vec) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int c = 0; c < 4 * GROUPS; ++c) {
      const int r = r0 + 32 * c + lane;
      const uint8_t* row = scale + (long long)(r >> shift) * ld;
      if (r >= r_end) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[c][j] = 0;
      } else if (vec && (16 * v + 16 <= blocks || r >> shift < last)) {
        const uint4 x = *reinterpret_cast<const uint4*>(row + 16 * v);
        w[c][0] = x.x, w[c][1] = x.y, w[c][2] = x.z, w[c][3] = x.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[c][j] = scale_word(row, 4 * v + j, blocks);
      }
    }
  }
  // Word j into GROUPS blocks of 512 bytes, [32 lanes][4 words] each: the order in which they are copied to tensor memory.
  __device__ __forceinline__ void store(uint4* to, int j) const {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) to[32 * g + lane] = make_uint4(w[4 * g][j], w[4 * g + 1][j], w[4 * g + 2][j], w[4 * g + 3][j]);
  }
};

// ---- 8-bit outputs ------------------------------------------------------------------------------
// The four warps that hold the 128 features of a block exchange their largest magnitudes per token through shared memory: 16 tokens
// at a time, two buffers in turn, one bounded wait.
struct Exchange {
  uint4 top[2][16];                                  // [turn][token] of the four warps
  uint64_t bar;                                      // a warp's arrival
};

// Rounds 16 tokens of the block (acc: this lane's feature n) to E4M3 and stores them with their scales.  Returns false when a wait gave up.
__device__ __forceinline__ bool quantise16(const Linear8Params& p, Exchange& x, int& turn, const float (&acc)[16], int n, int quad,
                                           int m0, int m_end) {
  const int lane = threadIdx.x % 32;
  const bool mine = n < p.cols;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float m = sdvg::warp_largest(mine ? sdvg::larger(0.f, acc[j]) : 0.f);
    if (lane == j) top = __float_as_uint(m);
  }
  const int buffer = turn & 1;
  if (lane < 16) reinterpret_cast<uint32_t*>(&x.top[buffer][lane])[quad] = top;
  __syncwarp();
  if (lane == 0) mbar_arrive(&x.bar);
  const bool ok = __all_sync(0xffffffffu, wait_for(&x.bar, (uint32_t)buffer, p.status, kWaitLimitNs));
  ++turn;
  if (!ok) return false;
  const uint4 t = x.top[buffer][lane % 16];
  const int e = sdvg::scale_exponent(max(max(t.x, t.y), max(t.z, t.w)));
  const int block = n / 128;                         // the same for the warp
  if (quad == 0 && lane < 16 && m0 + lane < m_end && block * 128 < p.cols)
    p.out_scale[(long long)(m0 + lane) * p.ld_os + block] = (uint8_t)(e + 127);
  const float inv = sdvg::power_of_two(-e);
  const long long ld = stride_here(p.ld_out);
  uint8_t* o = static_cast<uint8_t*>(p.out) + m0 * ld + n;
#pragma unroll
  for (int j = 0; j < 16; j += 4) {
    const float i0 = __shfl_sync(0xffffffffu, inv, j), i1 = __shfl_sync(0xffffffffu, inv, j + 1),
                i2 = __shfl_sync(0xffffffffu, inv, j + 2), i3 = __shfl_sync(0xffffffffu, inv, j + 3);
    const uint32_t c = pack_e4m3x4(acc[j] * i0, acc[j + 1] * i1, acc[j + 2] * i2, acc[j + 3] * i3);
#pragma unroll
    for (int i = 0; i < 4; ++i, o += ld)
      if (mine && m0 + j + i < m_end) *o = (uint8_t)(c >> (8 * i));
  }
  return true;
}

// ---- outputs by way of shared memory --------------------------------------------------------------
// Where rows of the output begin at multiples of 16 bytes and hold whole vectors, a warp takes its 32 features x 16 tokens from tensor
// memory as fragments (a lane then has features g, g + 8, g + 16 and g + 24, g = lane / 4, of tokens 2 q, 2 q + 1, 2 q + 8 and 2 q + 9, q =
// lane % 4), turns them in shared memory and stores 16 bytes per lane.  One store and one address per element and lane, as in the
// general epilogue, took as long as the products of a tile (4680 x 5120 x 20480 into bf16: 42 of 290 us, GELU another 43).
constexpr int kTurnBytes = 1024;                       // of a warp

// Values of a lane: v[4 f + k] is feature g + 8 f of the lane's k-th token.
struct Lane {
  int n, m, q;                                         // first feature, first token (of the warp's block), lane % 4
  __device__ __forceinline__ int token(int k) const { return m + 2 * q + (k & 1) + 8 * (k / 2); }
};

struct FragGate {
  TileGate of[4];
};

// activate16 in packed pairs, which is what an epilogue of 8-bit products has time for: the constants of an exponential's argument
// are multiplied out (z is -u log2 e), a quotient is one reciprocal, whose limits are those of activate16: past 2^126 it is 0.
__device__ __forceinline__ rows::Pair exp2_pair(rows::Pair z) {
  const float2 f = rows::floats_of(z);
  float2 e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(f.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(f.y));
  return rows::pair_of(e.x, e.y);
}
__device__ __forceinline__ rows::Pair reciprocal_pair(rows::Pair d) {
  const float2 f = rows::floats_of(d);
  float2 r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(f.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(f.y));
  return rows::pair_of(r.x, r.y);
}
__device__ __forceinline__ void activate_pairs(float (&v)[16], int act) {
  using namespace rows;
  constexpr float kLog2e = 1.4426950408889634f;
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float2 y = floats_of(f(pair_of(v[i], v[i + 1])));
      v[i] = y.x;
      v[i + 1] = y.y;
    }
  };
  const Pair one = pair_of(1.f, 1.f);
  if (act == SDVG_ACT_SILU) {
    const Pair c = pair_of(-kLog2e, -kLog2e);
    each([&](Pair a) { return mul2(a, reciprocal_pair(add2(exp2_pair(mul2(a, c)), one))); });
  } else if (act == SDVG_ACT_GELU_TANH) {
    constexpr float k = -1.5957691216057308f * kLog2e;
    const Pair c1 = pair_of(k, k), c3 = pair_of(k * 0.044715f, k * 0.044715f);
    each([&](Pair a) { return mul2(a, reciprocal_pair(add2(exp2_pair(mul2(a, fma2(mul2(a, a), c3, c1))), one))); });
  } else if (act == SDVG_ACT_GELU) {
    // gelu_erf: max(a, 0) - |a| h, with the tail h, the polynomial and the bounded factor that are described there; value by value
    // its code was twice as long, which a short launch waits for (333 x 1111 x 777: 2.0 us of 7.7, in pairs 0.8), and so do long ones
    // (4680 x 5120 x 20480 into bf16: 456 us against 422)
    constexpr float kPoly[10] = {-0.02069617911700f, 0.09534660188561f, -0.15029583590903f, 0.07120466716636f, -0.01118113013510f,
                                 0.05997585263270f, 0.08762596187607f, 0.11413582878705f, 0.12694158118874f, 0.12694266037636f};
    const Pair half = pair_of(-0.5f * kLog2e, -0.5f * kLog2e), slope = pair_of(0.31819805f, 0.31819805f);
    each([&](Pair a) {
      const float2 f = floats_of(a);
      const float2 z = make_float2(fabsf(f.x), fabsf(f.y));
      const Pair t = reciprocal_pair(fma2(pair_of(z.x, z.y), slope, one));
      Pair q = pair_of(kPoly[0], kPoly[0]);
#pragma unroll
      for (int k = 1; k < 10; ++k) q = fma2(q, t, pair_of(kPoly[k], kPoly[k]));
      const Pair h = mul2(mul2(q, t), exp2_pair(mul2(mul2(a, a), half)));
      return fma2(pair_of(-fminf(z.x, 1e4f), -fminf(z.y, 1e4f)), h, pair_of(fmaxf(f.x, 0.f), fmaxf(f.y, 0.f)));
    });
  }
}

// gate * act(acc + bias)
__device__ __forceinline__ void gated_frag(const Linear8Params& p, float (&v)[16], const Lane& l, int m_end, const float (&bias)[4],
                                           const FragGate& gate) {
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] += bias[i / 4];
  activate_pairs(v, p.act);
  if (!p.gate) return;
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const TileGate& g = gate.of[f];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int m = l.token(k);
      if (g.few) v[4 * f + k] *= m < g.border ? g.first : g.second;
      else if (m < m_end && l.n + 8 * f < p.cols) v[4 * f + k] *= p.gate[(m / p.gate_rows) * p.ld_gate + l.n + 8 * f];
    }
  }
}

template <int OutType>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (OutType == SDVG_BF16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
  } else {
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
}

// Residual of the 16 tokens, requested a block ahead of its use: lane i takes four features from 4 (i % 8) on of tokens i / 8, + 4, + 8 and
// + 12, as it will store them.
template <int OutType>
struct Residual {
  using Vec = typename std::conditional<OutType == SDVG_F32, uint4, uint2>::type;
  Vec v[4];
  __device__ __forceinline__ void load(const Linear8Params& p, int n0, int m, int m_end) {
    using T = typename OutElem<OutType>::T;
    if (!p.residual) return;
    const int lane = threadIdx.x % 32, n = n0 + lane % 8 * 4;
    const T* r = static_cast<const T*>(p.residual) + (m + lane / 8) * p.ld_res + n;
    const long long step = 4 * p.ld_res;
#pragma unroll
    for (int i = 0; i < 4; ++i, r += step)
      if (m + lane / 8 + 4 * i < m_end && n < p.cols) v[i] = *reinterpret_cast<const Vec*>(r);
  }
  __device__ __forceinline__ void add(int i, float (&f)[4]) const {
    if constexpr (OutType == SDVG_F32) {
      const uint4 x = v[i];
      f[0] += __uint_as_float(x.x), f[1] += __uint_as_float(x.y), f[2] += __uint_as_float(x.z), f[3] += __uint_as_float(x.w);
    } else {
      const uint32_t w[2] = {v[i].x, v[i].y};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float2 x;
        if constexpr (OutType == SDVG_BF16) x = make_float2(rows::bf16_lo(w[k]), rows::bf16_hi(w[k]));
        else x = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
        f[2 * k] += x.x;
        f[2 * k + 1] += x.y;
      }
    }
  }
};

// fp32 outputs, and 16-bit ones with a residual, which is added before they are rounded: 8 tokens at a time are turned as fp32.
template <int OutType>
__device__ __forceinline__ void store_frag32(const Linear8Params& p, const float (&v)[16], const Residual<OutType>& res, const Lane& l,
                                             int m_end, uint32_t turn) {
  using T = typename OutElem<OutType>::T;
  const int lane = threadIdx.x % 32, g = lane / 4, n = l.n - g + lane % 8 * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // token t of the eight: 128 bytes at 128 t, whose 16-byte pieces are moved round so that neither side meets a bank twice
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int t = 2 * l.q + k;
#pragma unroll
      for (int f = 0; f < 4; ++f)
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(turn + t * 128 + ((g / 4 + 2 * f) ^ t) * 16 + g % 4 * 4), "f"(v[4 * f + 2 * h + k])
                     : "memory");
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = lane / 8 + 4 * i, m = l.m + 8 * h + t;
      float f[4];
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3])
                   : "r"(turn + t * 128 + ((lane % 8) ^ t) * 16) : "memory");
      if (p.residual) res.add(2 * h + i, f);
      if (m < m_end && n < p.cols) {
        T* o = static_cast<T*>(p.out) + m * p.ld_out + n;
        if constexpr (OutType == SDVG_F32) {
          *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
        } else {
          *reinterpret_cast<uint2*>(o) = make_uint2(pack16<OutType>(f[0], f[1]), pack16<OutType>(f[2], f[3]));
        }
      }
    }
    __syncwarp();
  }
}

// 16-bit outputs without a residual.
template <int OutType>
__device__ __forceinline__ void store_frag(const Linear8Params& p, const float (&v)[16], const Lane& l, int m_end, uint32_t turn) {
  const int lane = threadIdx.x % 32;
  uint32_t h[8];                                       // of two neighbouring tokens: [feature block][tokens 0 and 1, or 8 and 9]
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    h[i] = pack16<OutType>(v[2 * i], v[2 * i + 1]);
  }
  // token t of the block: 64 bytes at 64 t, whose 16-byte pieces are moved round so that neither side meets a bank twice
  auto at = [&](int t, int piece) { return turn + t * 64 + (piece ^ (t / 2 % 4)) * 16; };
  st_frag_t4(at(lane % 8, lane / 8), h[0], h[2], h[4], h[6]);
  st_frag_t4(at(8 + lane % 8, lane / 8), h[1], h[3], h[5], h[7]);
  __syncwarp();
  const int n = l.n - lane / 4 + lane % 4 * 8;         // this lane's vector
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = lane / 4 + 8 * i;
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at(t, lane % 4)) : "memory");
    if (l.m + t < m_end && n < p.cols)
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + (l.m + t) * p.ld_out + n) = x;
  }
  __syncwarp();
}

// 8-bit outputs.  Returns false when a wait gave up.
__device__ __forceinline__ bool quantise_frag(const Linear8Params& p, Exchange& x, int& turns, const float (&v)[16], const Lane& l, int quad,
                                              int m_end, uint32_t turn) {
  const int lane = threadIdx.x % 32, g = lane / 4;
  float top[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float a[4];
#pragma unroll
    for (int f = 0; f < 4; ++f) a[f] = l.n + 8 * f < p.cols ? v[4 * f + k] : 0.f;
    top[k] = sdvg::larger(sdvg::larger(0.f, a[0], a[1]), a[2], a[3]);
#pragma unroll
    for (int o = 4; o < 32; o *= 2) top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], o));
  }
  const int buffer = turns & 1;
  if (lane < 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      reinterpret_cast<float*>(&x.top[buffer][2 * lane + (k & 1) + 8 * (k / 2)])[quad] = top[k];
  }
  __syncwarp();
  if (lane == 0) mbar_arrive(&x.bar);
  const bool ok = __all_sync(0xffffffffu, wait_for(&x.bar, (uint32_t)buffer, p.status, kWaitLimitNs));
  ++turns;
  if (!ok) return false;
  const uint4 t = x.top[buffer][lane % 16];
  const int e = sdvg::scale_exponent(max(max(t.x, t.y), max(t.z, t.w)));
  const int n0 = l.n - g, block = n0 / 128;            // the same for the warp
  if (quad == 0 && lane < 16 && l.m + lane < m_end && block * 128 < p.cols)
    p.out_scale[(long long)(l.m + lane) * p.ld_os + block] = (uint8_t)(e + 127);
  const float mine = sdvg::power_of_two(-e);           // of token lane % 16
  float inv[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) inv[k] = __shfl_sync(0xffffffffu, mine, 2 * l.q + (k & 1) + 8 * (k / 2));
  // codes of a feature's four tokens; then lanes of neighbouring features trade tokens, so that each has both features of two
  uint32_t c[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) c[f] = pack_e4m3x4(v[4 * f] * inv[0], v[4 * f + 1] * inv[1], v[4 * f + 2] * inv[2], v[4 * f + 3] * inv[3]);
  const bool odd = g & 1;
  const uint32_t keep = odd ? 0x7531 : 0x6420, give = odd ? 0x6420 : 0x7531, lo = odd ? 0x1504 : 0x5140, hi = odd ? 0x3726 : 0x7362;
  const int token = 2 * l.q + odd;                     // and 8 tokens on
  // token t of the block: 32 bytes at 32 t, whose halves change places every four tokens, for the banks' sake
  auto at = [&](int t, int half) { return turn + t * 32 + (half ^ (t / 4 % 2)) * 16; };
#pragma unroll
  for (int f = 0; f < 4; f += 2) {
    const uint32_t k = __byte_perm(c[f], c[f + 1], keep);
    const uint32_t r = __shfl_xor_sync(0xffffffffu, __byte_perm(c[f], c[f + 1], give), 4);
    const uint32_t a = __byte_perm(k, r, lo), b = __byte_perm(k, r, hi);       // feature blocks f and f + 1: (token, token + 8)
    const uint32_t to = at(token, f / 2) + g / 2 * 2, to8 = at(token + 8, f / 2) + g / 2 * 2;
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"((uint16_t)a) : "memory");
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to8), "h"((uint16_t)(a >> 16)) : "memory");
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + 8), "h"((uint16_t)b) : "memory");
    asm volatile("st.shared.u16 [%0], %1;" ::"r"(to8 + 8), "h"((uint16_t)(b >> 16)) : "memory");
  }
  __syncwarp();
  const int row = lane / 2, n = n0 + lane % 2 * 16;
  uint4 w;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at(row, lane % 2)) : "memory");
  if (l.m + row < m_end && n < p.cols) *reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + (l.m + row) * p.ld_out + n) = w;
  __syncwarp();
  return true;
}

// ---- small tiles: 128 features x 16 to 64 tokens, by a cluster that splits `inner` ------------------
//
// For few tokens, whose time is that of the weights' way from memory, and for small products of many, which would not give every
// pair a tile (choose_cut).  Two CTAs share an SM: one multiplies while the other begins or ends.
constexpr int kTileThreads = 224;                    // four epilogue warps, producer, issuer, scales
constexpr int kTileScaleCols = 8;                    // and its columns in tensor memory

struct TileSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], sf_full[kScaleSlots], sf_empty[kScaleSlots], acc_full, acc_empty;
  Exchange exchange;
  uint32_t tmem;
};

// Tensor memory columns: the accumulator (whose place the total of several chunks takes) and two words of scales.
__host__ __device__ constexpr uint32_t tile_tmem_cols(int tile_t) {
  uint32_t cols = 32;
  while (cols < (uint32_t)tile_t + 2 * kTileScaleCols) cols *= 2;
  return cols;
}

template <int OutType>
__global__ void __launch_bounds__(kTileThreads) linear8_tile_kernel(const __grid_constant__ Linear8Params p) {
  constexpr bool kChunked = OutType == SDVG_F32, kOut8 = OutType == SDVG_E4M3;
  using T = typename OutElem<OutType>::T;
  extern __shared__ uint8_t raw[];
  __shared__ TileSmem sm;
  uint8_t* buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0, tile = blockIdx.x / p.split;
  const int n0 = (tile % p.tiles_f) * kTileF;
  const int m0 = (tile / p.tiles_f) * p.tile_t, m_end = min(p.rows, m0 + p.tile_t);
  const int w_bytes = kTileF * 128, stage_bytes = w_bytes + p.tile_t * 128;
  uint8_t* slots = buf + p.stages * stage_bytes;
  // this CTA's part of `inner`: never empty
  const int share = p.k_iters / p.split, rest = p.k_iters % p.split;
  const int k0 = rank * share + min(rank, rest), iters = share + (rank < rest ? 1 : 0);
  const int word0 = k0 / kWordStages, words = (k0 + iters - 1) / kWordStages - word0 + 1;
  const int chunks = kChunked ? (iters + kTileChunkIters - 1) / kTileChunkIters : 1;
  const uint32_t tmem_cols = tile_tmem_cols(p.tile_t);
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      mbar_init(&sm.sf_full[s], 1);
      mbar_init(&sm.sf_empty[s], 1);
    }
    mbar_init(&sm.acc_full, 1);
    mbar_init(&sm.acc_empty, 4);
    mbar_init(&sm.exchange.bar, 4);
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
      // only now, as in linear.cu: a next grid that starts while SMs still hold several of these CTAs lands on the wrong SMs
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
      RingPos r, acc, sf;
      int word = -1;                                   // none yet
      uint32_t scales = 0;
      for (int c = 0; ok && c < chunks; ++c, acc.next(1)) {
        if (!(ok = wait_for(&sm.acc_empty, acc.phase ^ 1, p.status, kWaitLimitNs))) break;
        tc_fence_after();
        const int i0 = c * kTileChunkIters, i1 = kChunked ? min(iters, i0 + kTileChunkIters) : iters;
        for (int i = i0; i < i1; ++i, r.next(p.stages)) {
          const int s = r.stage, k = k0 + i;
          if (k / kWordStages != word) {
            word = k / kWordStages;
            if (!(ok = wait_for(&sm.sf_full[sf.stage], sf.phase, p.status, kWaitLimitNs))) break;
            tc_fence_after();
            // two places in turn: the products of the word before may still read theirs
            scales = tmem + p.tile_t + (word & 1) * kTileScaleCols;
            const uint32_t from = smem_u32(slots + sf.stage * kTileSlotBytes);
            tmem_cp_scales(scales, from);
            tmem_cp_scales(scales + 4, from + 512);
            mma_commit(&sm.sf_empty[sf.stage]);
            sf.next(kScaleSlots);
          }
          if (!(ok = wait_for(&sm.full[s], r.phase, p.status, kWaitLimitNs))) break;
          tc_fence_after();
          const uint32_t st = smem_u32(buf + s * stage_bytes);
          const uint64_t a = smem_desc_sw128(st, 16, 1024), b = smem_desc_sw128(st + w_bytes, 16, 1024);
          const uint32_t idesc = p.idesc | idesc_scale_step(k % kWordStages);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ss_mx(tmem, a + 2 * kk, b + 2 * kk, idesc, scales, scales + 4, i > i0 || kk > 0);
          mma_commit(&sm.empty[s]);
        }
        if (ok) mma_commit(&sm.acc_full);
      }
    }
    __syncwarp();
  } else if (warp == 6) {
    RingPos sf;
    bool ok = true;
    for (int v = word0 / 4; ok && 4 * v < word0 + words; ++v) {
      ScaleWords<1> fw, fx;
      fw.load(p.w_scale, p.ld_ws, p.w_shift, n0, min(p.cols, n0 + kTileF), (p.cols - 1) >> p.w_shift, v, p.k_iters, p.w_vec);
      fx.load(p.x_scale, p.ld_xs, 0, m0, m_end, p.rows - 1, v, p.k_iters, p.x_vec);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!ok || 4 * v + j < word0 || 4 * v + j >= word0 + words) continue;
        if (!(ok = __all_sync(0xffffffffu, wait_for(&sm.sf_empty[sf.stage], sf.phase ^ 1, p.status, kWaitLimitNs)))) continue;
        uint4* to = reinterpret_cast<uint4*>(slots + sf.stage * kTileSlotBytes);
        fw.store(to, j);
        fx.store(to + 32, j);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.sf_full[sf.stage]);
        sf.next(kScaleSlots);
      }
    }
  } else {
    const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
    const int n = n0 + warp * 32 + lane;
    const float b = p.bias && n < p.cols ? p.bias[n] : 0.f;
    RingPos r;
    const bool summed = kChunked && chunks > 1;
    bool ok;
    if (summed)
      ok = add_chunks<1, kMaxTileFew / 16>(chunks, lanes, p.tile_t, 0, [](int i) { return 16 * i; }, m_end - m0, r, &sm.acc_full,
                                           p.status, [&](int) {
        if (lane == 0) mbar_arrive(&sm.acc_empty);
      });
    else
      ok = __all_sync(0xffffffffu, wait_for(&sm.acc_full, r.phase, p.status, kWaitLimitNs));
    if (ok) {
      tc_fence_after();
      const TileGate gate = tile_gate(p, n, m0, m_end);
      float* mine = reinterpret_cast<float*>(buf) + warp * 32 + lane;      // [token][128 features]: the ring is read and free
      int turn = 0;
#pragma unroll 1
      for (int c = 0; ok && m0 + c < m_end; c += 16) {
        float acc[16];
        T res[16];
        if (!kOut8 && p.split == 1) load_residual16<OutType>(p, res, n, m0 + c, m_end);
        tmem_ld16(lanes + c, reinterpret_cast<uint32_t(&)[16]>(acc));
        tmem_wait_ld();
        if (p.split > 1) {
#pragma unroll
          for (int j = 0; j < 16; ++j) mine[(c + j) * kTileF] = acc[j];
        } else if constexpr (kOut8) {
          if (n < p.cols) gated16<activate_pairs>(p, acc, n, m0 + c, min(16, m_end - m0 - c), b, gate);
          ok = quantise16(p, sm.exchange, turn, acc, n, warp, m0 + c, m_end);
        } else {
          epilogue16<OutType, activate_pairs>(p, acc, res, n, m0 + c, m_end, b, gate);
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
      int turn = 0;
#pragma unroll 1
      for (int c = first; c < last; c += 16) {
        T res[16];
        if (!kOut8) load_residual16<OutType>(p, res, n, m0 + c, m0 + last);
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
        if constexpr (kOut8) {
          if (n < p.cols) gated16<activate_pairs>(p, acc, n, m0 + c, min(16, last - c), b, gate);
          if (!quantise16(p, sm.exchange, turn, acc, n, warp, m0 + c, m0 + last)) break;
        } else {
          epilogue16<OutType, activate_pairs>(p, acc, res, n, m0 + c, m0 + last, b, gate);
        }
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

// ---- large tiles: CTA pairs, persistent ---------------------------------------------------------
//
// A pair of CTAs (two SMs) works on a tile of SUBS x 256 features x tile_t tokens: each CTA holds SUBS x 128 of the features and fetches half
// of the token tile, and one tcgen05.mma of the even CTA reads the operands of both.  Each CTA's tensor memory holds the
// scales of its own features and of all the tile's tokens; the even CTA's copy moves both CTAs' words at once.
//
// What bounds it is how fast operand tiles come from L2: an SM gets 41 to 46 bytes a clock (measured with the products left out),
// while its tensor core, twice as fast on a byte as on a half, would take 66 with tiles of 256 x 240.  So where there are
// features enough a CTA takes 256 of them (SUBS = 2), which share each token tile: 50 bytes a clock.  The two accumulators
// of 240 columns then belong to one tile, and the next tile cannot run under its epilogue.  What hides most of that: at
// a tile's end the first half's last kSkew stages are multiplied before the second half's, and at its begin again, so that
// one half's epilogue runs under the other's products; and operands of the next tile arrive meanwhile.
// With SUBS = 1 the two accumulators belong to neighbouring tiles, and the epilogue of one runs under the products of the next.
// The last 32 columns of tensor memory are the scales' (two words in turn).
constexpr int kEpiWarps = 16;
constexpr int kPairThreads = 32 * (kEpiWarps + 3);
constexpr int kPairSmem = 224 * 1024;                // dynamic shared memory of a CTA; the barriers and exchanges are static
constexpr int kScaleCol = 480, kPairScaleCols = 16;
constexpr int kAccs = 2;
constexpr int kSkew = 3;
static_assert(kAccs * kMaxTileT <= kScaleCol);
static_assert(kScaleCol + 2 * kPairScaleCols <= 512);

// A word of scales of the CTA's features, and of the tile's tokens.
template <int SUBS>
constexpr int kPairSlotBytes = SUBS * 512 + 1024;
template <int SUBS>
__host__ __device__ constexpr int pair_stage_bytes(int tile_t) { return SUBS * kTileF * 128 + tile_t * 64; }

// What is not operand stages: the alignment, the scales, the space in which the epilogue warps turn outputs.
template <int SUBS, bool TURNED>
constexpr int pair_fixed_bytes = 1024 + kScaleSlots * kPairSlotBytes<SUBS> + (TURNED ? kEpiWarps * kTurnBytes : 0);

struct PairSmem {
  uint64_t full[kMaxStages], empty[kMaxStages], sf_full[kScaleSlots], sf_empty[kScaleSlots], acc_full[kAccs], acc_empty[kAccs];
  Exchange exchange[kEpiWarps / 4];
  uint32_t tmem;
};
static_assert(sizeof(PairSmem) + kPairSmem <= 227 * 1024 - 512);

// Adds the chunks of a sum in registers, round-to-nearest, 16 columns from `col`, col + 64, .. each, and leaves the total in the accumulator
// of the last, which stays the caller's to release.  (A place of its own for the total left room for tiles of 160 tokens:
// 4680 x 20480 x 5120 with gate and residual 638 us against 516, 4680 x 8192 x 5120 274 against 230, both in chunks of 2560.)
template <class Release>
__device__ __forceinline__ bool total_in_last(int chunks, uint32_t lanes, int col, int cols, RingPos& r, uint64_t* acc_full,
                                              unsigned int* status, Release release) {
  constexpr int kStep = 16 * kEpiWarps / 4, kSets = (kMaxTileT + kStep - 1) / kStep;
  float sum[kSets][16];
#pragma unroll
  for (int i = 0; i < kSets; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[i][j] = 0.f;
#pragma unroll 1
  for (int c = 0;; ++c) {
    if (!__all_sync(0xffffffffu, wait_for(&acc_full[r.stage], r.phase, status, kWaitLimitNs))) return false;
    tc_fence_after();
    const uint32_t part = lanes + r.stage * kMaxTileT + col;
#pragma unroll
    for (int i = 0; i < kSets; ++i)
      if (col + i * kStep < cols) {
        float v[16];
        tmem_ld16(part + i * kStep, reinterpret_cast<uint32_t(&)[16]>(v));
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[i][j] += v[j];
      }
    if (c == chunks - 1) break;
    tc_fence_before();
    __syncwarp();
    release(r.stage);
    r.next(kAccs);
  }
#pragma unroll
  for (int i = 0; i < kSets; ++i)
    if (col + i * kStep < cols)
      tmem_st16(lanes + r.stage * kMaxTileT + col + i * kStep, reinterpret_cast<uint32_t(&)[16]>(sum[i]));
  tmem_wait_st();
  return true;
}

// TURNED: the outputs go by way of shared memory.
template <int OutType, int SUBS, bool TURNED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    linear8_pair_kernel(const __grid_constant__ Linear8Params p) {
  constexpr bool kChunked = OutType == SDVG_F32 && SUBS == 1, kOut8 = OutType == SDVG_E4M3;
  using T = typename OutElem<OutType>::T;
  extern __shared__ uint8_t raw[];
  __shared__ PairSmem sm;
  uint8_t* buf = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  constexpr int kFeatures = SUBS * kTileF, w_bytes = kFeatures * 128;  // of a CTA
  const int stage_bytes = pair_stage_bytes<SUBS>(p.tile_t);
  uint8_t* slots = buf + p.stages * stage_bytes;
  const uint32_t turn_space = smem_u32(slots + kScaleSlots * kPairSlotBytes<SUBS>) + (TURNED ? warp % kEpiWarps * kTurnBytes : 0);
  const int chunks = p.whole ? 1 : (p.k_iters + kPairChunkIters - 1) / kPairChunkIters;
  const int words = (p.k_iters + kWordStages - 1) / kWordStages;
  sdvg::overlap_begin();
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(&sm.full[s], 1);                     // the even CTA's counts the bytes of both
      mbar_init(&sm.empty[s], 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      mbar_init(&sm.sf_full[s], 2);                  // the even CTA's: the scale warps of both
      mbar_init(&sm.sf_empty[s], 1);
    }
    for (int b = 0; b < kAccs; ++b) {
      mbar_init(&sm.acc_full[b], 1);
      mbar_init(&sm.acc_empty[b], 2 * kEpiWarps);    // the even CTA's: the epilogue warps of both
    }
    for (int g = 0; g < kEpiWarps / 4; ++g) mbar_init(&sm.exchange[g].bar, 4);
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
        const int n0 = (2 * ft + (int)rank) * kFeatures, m0 = tt * p.tile_t + (int)rank * (p.tile_t / 2);
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
      RingPos sf;
      int word_slot = 0;                             // words copied so far: two places of tensor memory in turn
      // a stage's operands are there, and its scales, whose word is copied when its first stage comes
      auto arrived = [&](int i, const RingPos& r) {
        if (i % kWordStages == 0) {
          if (!wait_for(&sm.sf_full[sf.stage], sf.phase, p.status, kWaitLimitNs)) return false;
          tc_fence_after();
          const uint32_t to = tmem + kScaleCol + (word_slot & 1) * kPairScaleCols;
          const uint32_t from = smem_u32(slots + sf.stage * kPairSlotBytes<SUBS>);
#pragma unroll
          for (int g = 0; g < SUBS; ++g) tmem_cp_scales_pair(to + 4 * g, from + 512 * g);
          tmem_cp_scales_pair(to + 4 * SUBS, from + 512 * SUBS);
          if (p.tile_t > 128) tmem_cp_scales_pair(to + 4 * SUBS + 4, from + 512 * SUBS + 512);
          mma_commit_pair(&sm.sf_empty[sf.stage]);
          sf.next(kScaleSlots);
          ++word_slot;
        }
        if (!wait_for(&sm.full[r.stage], r.phase, p.status, kWaitLimitNs)) return false;
        tc_fence_after();
        return true;
      };
      // the products of stage i of half `sub` into accumulator b; `behind`: words copied after this stage's
      auto multiply = [&](int i, const RingPos& r, int sub, int b, bool onto, int behind) {
        const uint32_t st = smem_u32(buf + r.stage * stage_bytes);
        const uint64_t da = smem_desc_sw128(st + sub * kTileF * 128, 16, 1024), db = smem_desc_sw128(st + w_bytes, 16, 1024);
        const uint32_t idesc = p.idesc | idesc_scale_step(i % kWordStages);
        const uint32_t scales = tmem + kScaleCol + ((word_slot - 1 - behind) & 1) * kPairScaleCols;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          mma_ss_mx_pair(tmem + b * kMaxTileT, da + 2 * kk, db + 2 * kk, idesc, scales + 4 * sub, scales + 4 * SUBS, onto || kk > 0);
      };
      RingPos r, acc;
      bool ok = true;
      for (long long t = pair; ok && t < p.tiles; t += pairs) {
        if constexpr (SUBS == 1) {
          for (int c = 0; ok && c < chunks; ++c, acc.next(kAccs)) {
            if (!(ok = wait_for(&sm.acc_empty[acc.stage], acc.phase ^ 1, p.status, kWaitLimitNs))) break;
            const int i0 = c * kPairChunkIters, i1 = p.whole ? p.k_iters : min(p.k_iters, i0 + kPairChunkIters);
            for (int i = i0; i < i1; ++i, r.next(p.stages)) {
              if (!(ok = arrived(i, r))) break;
              multiply(i, r, 0, acc.stage, i > i0, 0);
              mma_commit_pair(&sm.empty[r.stage]);
            }
            if (ok) mma_commit_pair(&sm.acc_full[acc.stage]);
          }
        } else {
          // stages [0, head) and [tail, k_iters) go first through the first half and then through the second
          const int head = min(kSkew, p.k_iters), tail = max(head, p.k_iters - kSkew);
          int i = 0;
          while (ok && i < p.k_iters) {
            const int run = i == 0 ? head : i < tail ? 1 : p.k_iters - tail;
            RingPos second = r;
            if (i == 0 && !(ok = wait_for(&sm.acc_empty[0], acc.phase ^ 1, p.status, kWaitLimitNs))) break;
            const int words_before = word_slot;
            for (int k = i; ok && k < i + run; ++k, r.next(p.stages)) {
              if (!(ok = arrived(k, r))) break;
              multiply(k, r, 0, 0, k > 0, 0);
            }
            if (!ok) break;
            if (i + run == p.k_iters) mma_commit_pair(&sm.acc_full[0]);
            if (i == 0 && !(ok = wait_for(&sm.acc_empty[1], acc.phase ^ 1, p.status, kWaitLimitNs))) break;
            tc_fence_after();
            // the first stage that begins a word within the run: those before it use the word before
            const int turn = (i + kWordStages - 1) / kWordStages * kWordStages;
            for (int k = i; k < i + run; ++k, second.next(p.stages)) {
              multiply(k, second, 1, 1, k > 0, word_slot != words_before && k < turn ? 1 : 0);
              mma_commit_pair(&sm.empty[second.stage]);
            }
            if (i + run == p.k_iters) mma_commit_pair(&sm.acc_full[1]);
            i += run;
          }
          acc.phase ^= 1;
        }
      }
    }
  } else if (warp == kEpiWarps + 2) {
    // ================= scales: of this CTA's features and of all the tile's tokens =================
    RingPos sf;
    int issued = 0;
    bool ok = true;
    for (long long t = pair; ok && t < p.tiles; t += pairs) {
      int ft, tt;
      tile_of(p, t, &ft, &tt);
      const int n0 = (2 * ft + (int)rank) * kFeatures, m0 = tt * p.tile_t, m_end = min(p.rows, m0 + p.tile_t);
      for (int v = 0; ok && 4 * v < words; ++v) {
        ScaleWords<SUBS> fw;
        ScaleWords<2> fx;
        fw.load(p.w_scale, p.ld_ws, p.w_shift, n0, min(p.cols, n0 + kFeatures), (p.cols - 1) >> p.w_shift, v, p.k_iters, p.w_vec);
        fx.load(p.x_scale, p.ld_xs, 0, m0, m_end, p.rows - 1, v, p.k_iters, p.x_vec);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!ok || 4 * v + j >= words) continue;
          if (!(ok = __all_sync(0xffffffffu, wait_for(&sm.sf_empty[sf.stage], sf.phase ^ 1, p.status, kWaitLimitNs)))) continue;
          issued = min(issued + 1, kScaleSlots);
          uint4* to = reinterpret_cast<uint4*>(slots + sf.stage * kPairSlotBytes<SUBS>);
          fw.store(to, j);
          fx.store(to + 32 * SUBS, j);
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_to_rank(smem_u32(&sm.sf_full[sf.stage]), 0));
          sf.next(kScaleSlots);
        }
      }
    }
    // every word is copied before the CTA may leave
    for (; ok && issued > 0; --issued) {
      sf.back(kScaleSlots);
      ok = __all_sync(0xffffffffu, wait_for(&sm.sf_empty[sf.stage], sf.phase, p.status, kWaitLimitNs));
    }
  } else {
    // ================= epilogue: warps w, w + 4, .. share 32 features and take 16-token column blocks in turn ==========
    const int quad = warp % 4, part = warp / 4;
    constexpr int kParts = kEpiWarps / 4;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t empty = map_to_rank(smem_u32(sm.acc_empty), 0);
    RingPos r;
    bool ok = true;
    int turn = 0;
    for (long long t = pair; ok && t < p.tiles; t += pairs) {
      int ft, tt;
      tile_of(p, t, &ft, &tt);
      const int m0 = tt * p.tile_t, m_end = min(p.rows, m0 + p.tile_t);
#pragma unroll 1
      for (int sub = 0; sub < SUBS; ++sub) {
        const int n0 = (2 * ft + (int)rank) * kFeatures + sub * kTileF + quad * 32, n = n0 + lane;
        float bias[TURNED ? 4 : 1];
        FragGate gate;
        T ahead[16];
        Residual<OutType> vectors;
        Lane at{n0 + lane / 4, m0 + part * 16, lane % 4};
        auto request = [&] {
          if constexpr (TURNED) {
#pragma unroll
            for (int f = 0; f < 4; ++f) {
              bias[f] = p.bias && at.n + 8 * f < p.cols ? p.bias[at.n + 8 * f] : 0.f;
              gate.of[f] = tile_gate(p, at.n + 8 * f, m0, m_end);
            }
            if constexpr (!kOut8) vectors.load(p, n0, at.m, m_end);
          } else {
            bias[0] = p.bias && n < p.cols ? p.bias[n] : 0.f;
            gate.of[0] = tile_gate(p, n, m0, m_end);
            if constexpr (!kOut8) load_residual16<OutType>(p, ahead, n, m0 + part * 16, m_end);
          }
        };
        if constexpr (!kChunked) request();          // a chunked sum needs the registers until its total is back in tensor memory
        auto release = [&](int stage) {
          if (lane == 0) mbar_arrive_cluster(empty + 8 * stage);
        };
        if (kChunked && chunks > 1)
          ok = total_in_last(chunks, lanes, part * 16, m_end - m0, r, sm.acc_full, p.status, release);
        else
          ok = __all_sync(0xffffffffu, wait_for(&sm.acc_full[r.stage], r.phase, p.status, kWaitLimitNs));
        if (!ok) break;
        tc_fence_after();
        if constexpr (kChunked) request();
        const uint32_t sums = lanes + r.stage * kMaxTileT;
#pragma unroll 1
        for (int col = part * 16; m0 + col < m_end; col += 16 * kParts) {
          float acc[16];
          if constexpr (TURNED) {
            float lo[8], hi[8];
            tmem_ld_frag16(sums + col, lo);
            tmem_ld_frag16(sums + col + (16u << 16), hi);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) {              // register i: feature block i / 2 % 2, token i % 2 + 2 (i / 4)
              acc[4 * (i / 2 % 2) + i % 2 + 2 * (i / 4)] = lo[i];
              acc[4 * (2 + i / 2 % 2) + i % 2 + 2 * (i / 4)] = hi[i];
            }
            at.m = m0 + col;
            gated_frag(p, acc, at, m_end, bias, gate);
            if constexpr (kOut8) {
              if (!(ok = quantise_frag(p, sm.exchange[part], turn, acc, at, quad, m_end, turn_space))) break;
            } else {
              if (OutType == SDVG_F32 || p.residual) {
                store_frag32<OutType>(p, acc, vectors, at, m_end, turn_space);
                vectors.load(p, n0, m0 + col + 16 * kParts, m_end);
              } else if constexpr (OutType != SDVG_F32) {
                store_frag<OutType>(p, acc, at, m_end, turn_space);
              }
            }
          } else {
            tmem_ld16(sums + col, reinterpret_cast<uint32_t(&)[16]>(acc));
            tmem_wait_ld();
            if constexpr (kOut8) {
              if (n < p.cols) gated16<activate_pairs>(p, acc, n, m0 + col, min(16, m_end - m0 - col), bias[0], gate.of[0]);
              if (!(ok = quantise16(p, sm.exchange[part], turn, acc, n, quad, m0 + col, m_end))) break;
            } else {
              epilogue16<OutType, activate_pairs>(p, acc, ahead, n, m0 + col, m_end, bias[0], gate.of[0]);
              load_residual16<OutType>(p, ahead, n, m0 + col + 16 * kParts, m_end);
            }
          }
        }
        if (!ok) break;
        tc_fence_before();
        __syncwarp();
        release(r.stage);
        r.next(kAccs);
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

// Matrix of codes [rows, inner] with a row stride, as (inner, row): box = 128 elements x box_rows, 128-byte swizzle; what lies
// past either end reads as zero.
int make_map(CUtensorMap* m, const void* base, int inner, int rows, int64_t ld, int box_rows) {
  const sdvg::EncodeTiledFn fn = sdvg::encode_tiled_fn();
  if (!fn) return SDVG_ERR_CUDA;
  if (rows == 1) ld = ((int64_t)inner + 15) / 16 * 16;           // not read, but the map wants a legal one
  cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {(cuuint32_t)kTileK, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? SDVG_OK : SDVG_ERR_CUDA;
}

std::mutex g_setup_mu;

static_assert(2 * (tile_dynamic(32) + 3 * 1024) <= 228 * 1024 && 2 * (tile_dynamic(64) + 3 * 1024) <= 228 * 1024);

// As in linear.cu: no tile takes a larger share of an SM's tensor memory columns than of its shared memory, so that a CTA that an
// SM can hold finds its columns at once, and clusters never wait for each other's.
constexpr bool columns_within_share(int tile_t) {
  return tile_tmem_cols(tile_t) * (228 * 1024 / 512) <= (uint32_t)tile_dynamic(tile_t);
}
static_assert(columns_within_share(16) && columns_within_share(32) && columns_within_share(48) && columns_within_share(64));
static_assert(kMaxTileFew == 64, "the sizes checked above");

// One-time set-up per device and output type: the opt-in to the kernels' dynamic shared memory, and how many CTA pairs
// the device runs at once.
template <int OutType, int SUBS, bool TURNED>
cudaError_t set_up_pair(int* pairs) {
  cudaError_t e = cudaFuncSetAttribute(linear8_pair_kernel<OutType, SUBS, TURNED>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
  if (e != cudaSuccess) return e;
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
  e = cudaOccupancyMaxActiveClusters(&n, linear8_pair_kernel<OutType, SUBS, TURNED>, &cfg);
  *pairs = std::min(*pairs, n);
  return e;
}

template <int OutType>
int set_up(int* pairs) {
  static int pairs_of_device[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return sdvg::cuda_status(e);
  if (dev < 0 || dev >= kMaxDevices) return SDVG_ERR_INVALID_ARG;
  std::lock_guard<std::mutex> lock(g_setup_mu);
  if (!pairs_of_device[dev]) {
    e = cudaFuncSetAttribute(linear8_tile_kernel<OutType>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             std::max(tile_dynamic(32), tile_dynamic(kMaxTileFew)));
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    int n = 0x7fffffff;
    e = set_up_pair<OutType, 1, false>(&n);
    if (e == cudaSuccess) e = set_up_pair<OutType, 2, false>(&n);
    if (e == cudaSuccess) e = set_up_pair<OutType, 1, true>(&n);
    if (e == cudaSuccess) e = set_up_pair<OutType, 2, true>(&n);
    if (e != cudaSuccess || n < 1) return sdvg::cuda_status(e != cudaSuccess ? e : cudaErrorUnknown);
    pairs_of_device[dev] = n;
  }
  *pairs = pairs_of_device[dev];
  return SDVG_OK;
}

template <int OutType, int SUBS, bool TURNED>
int launch_pair(Linear8Params& p, const void* x, int64_t ld_x, const void* w, int64_t ld_w, int inner, int pairs, cudaStream_t stream) {
  p.tiles_f = (p.cols + 2 * SUBS * kTileF - 1) / (2 * SUBS * kTileF);
  p.tiles_t = (p.rows + p.tile_t - 1) / p.tile_t;
  p.tiles = (long long)p.tiles_f * p.tiles_t;
  if (p.tiles >= 1ll << 28) return SDVG_ERR_BAD_SHAPE;
  p.idesc = idesc_mx_e4m3(2 * kTileF, p.tile_t);
  int st = make_map(&p.w_map, w, inner, p.cols, ld_w, SUBS * kTileF);
  if (st != SDVG_OK) return st;
  if ((st = make_map(&p.x_map, x, inner, p.rows, ld_x, p.tile_t / 2)) != SDVG_OK) return st;
  p.group = 8 / SUBS;
  p.stages = std::min(kMaxStages, (kPairSmem - pair_fixed_bytes<SUBS, TURNED>) / pair_stage_bytes<SUBS>(p.tile_t));
  const int grid = 2 * (int)std::min((long long)pairs, p.tiles);
  return sdvg::cuda_status(
      sdvg::launch_overlapped(linear8_pair_kernel<OutType, SUBS, TURNED>, grid, kPairThreads, kPairSmem, 0, stream, p));
}
// The skewed stages of both ends are all in the ring at once.
static_assert((kPairSmem - pair_fixed_bytes<2, true>) / pair_stage_bytes<2>(kMaxTileT) > kSkew);

template <int OutType>
int launch(Linear8Params& p, const void* x, int64_t ld_x, const void* w, int64_t ld_w, int inner, cudaStream_t stream) {
  int pairs = 0;
  int st = set_up<OutType>(&pairs);
  if (st != SDVG_OK) return st;
  p.whole = whole_sums(p.k_iters, OutType == SDVG_F32);
  const Cut cut = choose_cut(p.rows, p.cols, p.k_iters, pairs, !p.whole);             // 80 ns where pairs are considered, else 10
  p.tile_t = cut.tile_t;
  if (cut.subs) {
    constexpr int kVec = OutType == SDVG_E4M3 ? 16 : OutType == SDVG_F32 ? 4 : 8;          // elements of 16 bytes
    constexpr uintptr_t kResBytes = OutType == SDVG_F32 ? 16 : 8;                           // four of the residual's
    const bool turned = sdvg::aligned16(p.out) && p.cols % kVec == 0 && p.ld_out % kVec == 0 &&
                        (!p.residual || (reinterpret_cast<uintptr_t>(p.residual) % kResBytes == 0 && p.ld_res % 4 == 0));
    if (cut.subs == 2)
      return turned ? launch_pair<OutType, 2, true>(p, x, ld_x, w, ld_w, inner, pairs, stream)
                    : launch_pair<OutType, 2, false>(p, x, ld_x, w, ld_w, inner, pairs, stream);
    return turned ? launch_pair<OutType, 1, true>(p, x, ld_x, w, ld_w, inner, pairs, stream)
                  : launch_pair<OutType, 1, false>(p, x, ld_x, w, ld_w, inner, pairs, stream);
  }
  p.tiles_f = (p.cols + kTileF - 1) / kTileF;
  p.tiles_t = (p.rows + p.tile_t - 1) / p.tile_t;
  p.tiles = (long long)p.tiles_f * p.tiles_t;
  if (p.tiles >= 1ll << 28) return SDVG_ERR_BAD_SHAPE;
  p.idesc = idesc_mx_e4m3(kTileF, p.tile_t);
  if ((st = make_map(&p.w_map, w, inner, p.cols, ld_w, kTileF)) != SDVG_OK) return st;
  if ((st = make_map(&p.x_map, x, inner, p.rows, ld_x, p.tile_t)) != SDVG_OK) return st;
  p.split = cut.split;
  p.stages = tile_stages(p.tile_t);
  return sdvg::cuda_status(sdvg::launch_overlapped(linear8_tile_kernel<OutType>, (unsigned)p.tiles * p.split, kTileThreads,
                                                   tile_dynamic(p.tile_t), p.split > 1 ? p.split : 0, stream, p));
}

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int sdvg_linear_e4m3(const void* x8, int64_t ld_x, const void* x_scale, int64_t ld_x_scale, const void* w8, int64_t ld_w,
                     const void* w_scale, int64_t ld_w_scale, int w_scale_rows, const float* bias, int act, const float* gate,
                     int64_t ld_gate, int gate_rows, const void* residual, int64_t ld_residual, void* out, int64_t ld_out,
                     void* out_scale, int64_t ld_out_scale, int rows, int cols, int inner, int out_type, void* workspace,
                     size_t workspace_bytes, void* stream) {
  SDVG_RANGE();
  constexpr int kMaxExtent = 0x7fffffff - 1024;                  // a tile's end past the matrix's is still an int
  constexpr int kMaxInner = 1 << 26;                             // one sum stays far below the limit of a wait
  if (rows < 0 || cols < 0 || inner < 1 || rows > kMaxExtent || cols > kMaxExtent || inner > kMaxInner)
    return SDVG_ERR_BAD_SHAPE;
  const bool out8 = out_type == SDVG_E4M3;
  if (!out8 && !sdvg::elem_type_ok(out_type)) return SDVG_ERR_INVALID_ARG;
  if (act < SDVG_ACT_NONE || act > SDVG_ACT_GELU || (gate && gate_rows < 1)) return SDVG_ERR_INVALID_ARG;
  if (w_scale_rows != 1 && w_scale_rows != 128) return SDVG_ERR_INVALID_ARG;
  if (out8 ? residual != nullptr : out_scale != nullptr) return SDVG_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return SDVG_OK;
  if (!x8 || !x_scale || !w8 || !w_scale || !out || (out8 && !out_scale) || !workspace ||
      workspace_bytes < (size_t)kWorkspaceBytes)
    return SDVG_ERR_INVALID_ARG;
  const int blocks = (inner + 127) / 128, out_blocks = (cols + 127) / 128;
  const bool w_scales = cols > w_scale_rows;                     // more than one row of them
  if ((rows > 1 && (ld_x < inner || ld_out < cols || ld_x_scale < blocks)) || (cols > 1 && ld_w < inner) ||
      (w_scales && ld_w_scale < blocks) || (out8 && rows > 1 && ld_out_scale < out_blocks))
    return SDVG_ERR_BAD_SHAPE;
  if (residual && rows > 1 && ld_residual != 0 && ld_residual < cols) return SDVG_ERR_BAD_SHAPE;
  if (gate && rows > gate_rows && ld_gate < cols) return SDVG_ERR_BAD_SHAPE;
  // the tensor map's stride is a 40-bit byte count
  if ((rows > 1 && ld_x >= (int64_t)1 << 40) || (cols > 1 && ld_w >= (int64_t)1 << 40)) return SDVG_ERR_BAD_SHAPE;
  if (!sdvg::aligned16(x8) || !sdvg::aligned16(w8) || (rows > 1 && (ld_x & 15)) || (cols > 1 && (ld_w & 15)) ||
      !aligned_to(x_scale, 4) || !aligned_to(w_scale, 4) || (rows > 1 && (ld_x_scale & 3)) || (w_scales && (ld_w_scale & 3)))
    return SDVG_ERR_MISALIGNED;
  const int out_bytes = out8 ? 1 : sdvg::elem_bytes(out_type);
  if (!aligned_to(out, out_bytes) || !aligned_to(residual, out_bytes) || !aligned_to(bias, 4) || !aligned_to(gate, 4) ||
      !aligned_to(workspace, 256))
    return SDVG_ERR_MISALIGNED;
  int st = sdvg::require_sm100();
  if (st != SDVG_OK) return st;
  Linear8Params p = {};
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
  p.x_scale = (const uint8_t*)x_scale;
  p.w_scale = (const uint8_t*)w_scale;
  p.ld_xs = ld_x_scale;
  p.ld_ws = ld_w_scale;
  p.w_shift = w_scale_rows == 128 ? 7 : 0;
  p.x_vec = sdvg::aligned16(x_scale) && (rows == 1 || ld_x_scale % 16 == 0);
  p.w_vec = sdvg::aligned16(w_scale) && (!w_scales || ld_w_scale % 16 == 0);
  p.out_scale = (uint8_t*)out_scale;
  p.ld_os = ld_out_scale;
  p.k_iters = blocks;
  p.status = (unsigned int*)workspace + 1;
  const cudaStream_t s = (cudaStream_t)stream;
  if (out8) return launch<SDVG_E4M3>(p, x8, ld_x, w8, ld_w, inner, s);
  if (out_type == SDVG_F32) return launch<SDVG_F32>(p, x8, ld_x, w8, ld_w, inner, s);
  if (out_type == SDVG_F16) return launch<SDVG_F16>(p, x8, ld_x, w8, ld_w, inner, s);
  return launch<SDVG_BF16>(p, x8, ld_x, w8, ld_w, inner, s);
}

}  // extern "C"
