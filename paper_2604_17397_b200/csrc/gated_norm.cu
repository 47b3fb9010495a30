// Residual add of a sublayer's output (with its own norm and gate) and the modulated norm that opens the next sublayer,
// one pass over the rows.
//
// Bound by HBM: every row of x and y is read once and every row of x_out and out written once.  A row is split over a team
// (a CTA, or one warp where a warp can hold the row) and stays in registers between its statistics and its outputs.
// A thread keeps the same columns for all rows it walks, and with them the vectors, combined to three:
//   s = x + G * post(y),  out = norm(s) * A + B,   G = gate * post_weight,  A = weight * (1 + scale),  B = bias * (1 + scale) + shift
// which change only with the row group; read per row instead, they were 60 KB through L1 for 40 KB of row (5120 columns).
// The next rows are on their way into shared memory meanwhile (cp.async, every thread fetching just what it will read
// itself, so that no barrier is needed): held in registers they cost the occupancy that hides the reductions.
// The arithmetic is in packed pairs (fma.rn.f32x2).
#include <math.h>

#include <algorithm>

#include "elem_types.cuh"
#include "overlap.cuh"
#include "row_team.cuh"
#include "sdvg_internal.h"

namespace {

using sdvg::load_elem;
using sdvg::store_elem;
using namespace rows;

struct NormParams {
  const void* x;
  const void* y;               // null: no sublayer output
  void* x_out;                 // null: not wanted
  void* out;                   // null: not wanted
  const float* post_weight;
  const float* gate;
  const float* weight;
  const float* bias;
  const float* scale;
  const float* shift;
  long long ld_x, ld_y, ld_x_out, ld_out, ld_gate, ld_mod;
  int x_type, y_type, out_type;
  int post, norm;
  int gate_rows, mod_rows;
  int rows, cols;
  float eps, inv_cols, num_cols;
};

// Sum and centred sum of squares of a part of a row: parts combine without the cancellation of a difference of squares.
struct Moments {
  float sum, m2;
};

constexpr int kSlots = 2;                              // rows on their way per team
constexpr int kTeamThreads = 640;                      // most threads of a CTA team; leaves a thread 96 registers

// Ordinary loads, here and wherever these kernels read: the read-only path is for data that no one writes during the kernel's
// whole life, which begins under the end of the kernel before it, and that may be the one which writes these vectors.
__device__ __forceinline__ void load_vector(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *(reinterpret_cast<const float4*>(p) + 1);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// Joins the warps' moments of a row to its mean and 1 / deviation: warp w has the sum and the centred sum of squares of
// counts[w] columns.  With one warp per row there is nothing to join.
template <bool WARP>
struct Team {
  Moments (*part)[32];                                 // two exchange buffers
  const float* counts;
  int turn = 0;

  __device__ __forceinline__ void join(const NormParams& p, int kind, Moments m, float* mean, float* rstd) {
    if (!WARP) {
      // a buffer is written again only two exchanges later, after a barrier that its readers have reached
      const int lane = threadIdx.x % 32;
      if (lane == 0) part[turn][threadIdx.x / 32] = m;
      __syncthreads();
      const bool mine = lane < blockDim.x / 32;
      const Moments other = mine ? part[turn][lane] : Moments{0.f, 0.f};
      if (kind == SDVG_NORM_LAYER) {
        m.sum = warp_sum(other.sum);
        const float n = mine ? counts[lane] : 0.f;
        const float off = n > 0.f ? __fdividef(other.sum, n) - m.sum * p.inv_cols : 0.f;
        m.m2 = warp_sum(fmaf(n * off, off, other.m2));
      } else {
        m.m2 = warp_sum(other.m2);
      }
      turn ^= 1;
    }
    *mean = m.sum / p.num_cols;                        // a division: a constant row's mean is that constant
    *rstd = rsqrtf(fmaf(m.m2, p.inv_cols, p.eps));
  }
};

// This warp's moments of a row of vectors held in v.
template <int NI, class Valid>
__device__ __forceinline__ Moments warp_moments(const Vec8 (&v)[NI], int kind, float inv_count, Valid valid) {
  Moments m{0.f, 0.f};
  if (kind == SDVG_NORM_LAYER) {
    Pair a = 0, b = 0;                                 // 0.0f pairs
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (valid(i)) {
        a = add2(a, add2(v[i].p[0], v[i].p[1]));
        b = add2(b, add2(v[i].p[2], v[i].p[3]));
      }
    const float2 f = floats_of(add2(a, b));
    m.sum = warp_sum(f.x + f.y);
  }
  const float mid = -m.sum * inv_count;
  const Pair mid2 = pair_of(mid, mid);
  Pair a = 0, b = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (valid(i)) {
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const Pair d = add2(v[i].p[j], mid2), e = add2(v[i].p[j + 1], mid2);
        a = fma2(d, d, a);
        b = fma2(e, e, b);
      }
    }
  const float2 f = floats_of(add2(a, b));
  m.m2 = warp_sum(f.x + f.y);
  return m;
}

// (v - mean) * rstd
template <int NI>
__device__ __forceinline__ void apply_norm(Vec8 (&v)[NI], float mean, float rstd) {
  const Pair r = pair_of(rstd, rstd), c = pair_of(-mean, -mean);
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) v[i].p[j] = mul2(add2(v[i].p[j], c), r);
}

// Rows of aligned vectors.  XW and YW: bytes of x's and y's elements (YW = 0: no y).  A thread holds NI pieces of 8 columns; the
// pieces of a warp are 32 vectors apart, so that they are a constant distance from one address per row, which moves on by the
// row stride.  FULL: the team's pieces are all inside the row.
template <int XW, int YW, int NI, bool WARP, bool FULL>
__global__ void __launch_bounds__(WARP ? 128 : kTeamThreads) gated_norm_kernel(const __grid_constant__ NormParams p) {
  extern __shared__ uint4 s_ring[];
  __shared__ Moments s_part[2][32];
  __shared__ float s_count[32];
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int c0 = ((WARP ? 0 : warp * 32 * NI) + lane) * 8;             // first piece; piece i: c0 + 256 i
  auto valid = [&](int i) { return FULL || c0 + 256 * i < p.cols; };
  // neighbouring rows per team: they share their group's vectors
  const int teams = WARP ? gridDim.x * (blockDim.x / 32) : gridDim.x, me = WARP ? blockIdx.x * (blockDim.x / 32) + warp : blockIdx.x;
  const int share = p.rows / teams, rest = p.rows % teams;
  const long long begin = (long long)me * share + min(me, rest), end = begin + share + (me < rest ? 1 : 0);
  float own = 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) own += valid(i) ? 8.f : 0.f;
  const float count = warp_sum(own), inv_count = count > 0.f ? 1.f / count : 0.f;
  if (!WARP && lane == 0) s_count[warp] = count;
  Team<WARP> team{s_part, s_count};

  uint4* ring = s_ring + warp * 32 * (kSlots * (Ring<XW, NI>::kBytes + Ring<YW, NI>::kBytes) / 16) + lane;
  const Ring<XW, NI> rx{ring};
  const Ring<YW, NI> ry{ring + kSlots * Ring<XW, NI>::kBytes / 16 * 32};
  const int out_bytes = p.out_type == SDVG_F32 ? 4 : 2;
  const char* x = static_cast<const char*>(p.x) + (begin * p.ld_x + c0) * XW;
  const char* y = static_cast<const char*>(p.y) + (begin * p.ld_y + c0) * YW;
  char* x_out = static_cast<char*>(p.x_out) + (begin * p.ld_x_out + c0) * XW;
  char* out = static_cast<char*>(p.out) + (begin * p.ld_out + c0) * out_bytes;
  const long long step_x = p.ld_x * XW, step_y = p.ld_y * YW, step_x_out = p.ld_x_out * XW, step_out = p.ld_out * out_bytes;
  int asked = 0;                                       // rows requested so far; x and y point at the next one
  const int total = (int)(end - begin);
  auto request = [&](int slot) {
    if (asked < total) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (valid(i)) {
          rx.request(slot, i, x);
          if (YW) ry.request(slot, i, y);
        }
    }
    copy_commit();                                     // an empty group where there is no such row
    ++asked;
    x += step_x;
    y += step_y;
  };
#pragma unroll
  for (int k = 0; k < kSlots; ++k) request(k);

  Vec8 G[YW ? NI : 1], A[NI], B[NI];
  long long new_gate = begin, new_mod = begin;         // rows at which the vectors change
  int slot = 0;
  for (long long r = begin; r < end; ++r, slot = slot + 1 == kSlots ? 0 : slot + 1) {      // uniform over the team
    if (YW && r == new_gate) {
      const unsigned group = p.gate ? (unsigned)r / (unsigned)p.gate_rows : 0;
      new_gate = p.gate ? (long long)(group + 1) * p.gate_rows : end;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, w[8];
        if (valid(i)) {
          if (p.gate) load_vector(p.gate + group * p.ld_gate + c0 + 256 * i, g);
          if (p.post_weight) {
            load_vector(p.post_weight + c0 + 256 * i, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] *= w[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) G[i].p[j] = pair_of(g[2 * j], g[2 * j + 1]);
      }
    }
    if (p.out && r == new_mod) {
      const bool mod = p.scale || p.shift;
      const unsigned group = mod ? (unsigned)r / (unsigned)p.mod_rows : 0;
      new_mod = mod ? (long long)(group + 1) * p.mod_rows : end;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float a[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, b[8] = {}, f[8];
        if (valid(i)) {
          const int c = c0 + 256 * i;
          if (p.weight) load_vector(p.weight + c, a);
          if (p.bias) load_vector(p.bias + c, b);
          if (p.scale) {
            load_vector(p.scale + group * p.ld_mod + c, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              a[j] = fmaf(a[j], f[j], a[j]);
              // not 0 times a scale that may be infinite.  In this form it costs the kernel, whose 96 registers are all taken, 1 us
              // of 36 at 4680 x 5120; as a branch on p.bias, or in functions of its own, 2 to 9
              b[j] = fmaf(b[j], b[j] != 0.f ? f[j] : 0.f, b[j]);
            }
          }
          if (p.shift) {
            load_vector(p.shift + group * p.ld_mod + c, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] += f[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          A[i].p[j] = pair_of(a[2 * j], a[2 * j + 1]);
          B[i].p[j] = pair_of(b[2 * j], b[2 * j + 1]);
        }
      }
    }
    copy_wait<kSlots - 1>();                           // this thread's own copies: nobody else reads them
    Vec8 s[NI];
    float mean = 0.f, rstd = 1.f;
    if constexpr (YW != 0) {
      Vec8 v[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) ry.values(slot, i, p.y_type, v[i]);
      if (p.post != SDVG_NORM_NONE) {
        team.join(p, p.post, warp_moments<NI>(v, p.post, inv_count, valid), &mean, &rstd);
        apply_norm<NI>(v, mean, rstd);
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        rx.values(slot, i, p.x_type, s[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i].p[j] = fma2(G[i].p[j], v[i].p[j], s[i].p[j]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) rx.values(slot, i, p.x_type, s[i]);
    }
    request(slot);
    if (p.x_out) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (valid(i)) store8(x_out + 256 * XW * i, p.x_type, s[i]);
      x_out += step_x_out;
    }
    if (!p.out) continue;
    if (p.norm != SDVG_NORM_NONE) {
      team.join(p, p.norm, warp_moments<NI>(s, p.norm, inv_count, valid), &mean, &rstd);
      apply_norm<NI>(s, mean, rstd);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i].p[j] = fma2(s[i].p[j], A[i].p[j], B[i].p[j]);
      if (valid(i)) store8(out + 256 * out_bytes * i, p.out_type, s[i]);
    }
    out += step_out;
  }
  copy_wait<0>();
}

// Single columns of a row, 32 apart, of any type: the type is looked at once per row, not per element.
template <int NI, class Valid>
__device__ __forceinline__ void load_singles(float (&v)[NI], const void* base, long long at, int type, Valid valid) {
  if (type == SDVG_F32) {
    const float* s = static_cast<const float*>(base) + at;
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = valid(i) ? s[32 * i] : 0.f;
  } else {
    const uint16_t* s = static_cast<const uint16_t*>(base) + at;
    uint16_t h[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) h[i] = valid(i) ? s[32 * i] : 0;
    if (type == SDVG_BF16) {
#pragma unroll
      for (int i = 0; i < NI; ++i) v[i] = __uint_as_float((uint32_t)h[i] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) v[i] = __half2float(__ushort_as_half(h[i]));
    }
  }
}
template <int NI, class Valid>
__device__ __forceinline__ void store_singles(const float (&v)[NI], void* base, long long at, int type, Valid valid) {
  if (type == SDVG_F32) {
    float* o = static_cast<float*>(base) + at;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (valid(i)) o[32 * i] = v[i];
  } else {
    uint16_t* o = static_cast<uint16_t*>(base) + at;
    uint16_t h[NI];
    if (type == SDVG_BF16) {
#pragma unroll
      for (int i = 0; i < NI; ++i) h[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) h[i] = __half_as_ushort(__float2half_rn(v[i]));
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (valid(i)) o[32 * i] = h[i];
  }
}

// Rows that are not made of aligned vectors: one CTA per row, NI single columns per thread; what is in flight comes from the
// CTAs of an SM.
template <int NI>
__global__ void __launch_bounds__(NI == 16 ? 512 : 256) gated_norm_single_kernel(const __grid_constant__ NormParams p) {
  __shared__ Moments s_part[2][32];
  __shared__ float s_count[32];
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int c0 = warp * 32 * NI + lane;                // first column; piece i: c0 + 32 i
  const long long r = blockIdx.x;
  auto valid = [&](int i) { return c0 + 32 * i < p.cols; };
  float s[NI], y[NI];
  load_singles<NI>(s, p.x, r * p.ld_x + c0, p.x_type, valid);
  if (p.y) load_singles<NI>(y, p.y, r * p.ld_y + c0, p.y_type, valid);
  const int left = p.cols - warp * 32 * NI;
  const float count = (float)max(0, min(left, 32 * NI)), inv_count = count > 0.f ? 1.f / count : 0.f;
  if (lane == 0) s_count[warp] = count;
  Team<false> team{s_part, s_count};
  auto moments = [&](const float (&v)[NI], int kind) {
    Moments m{0.f, 0.f};
    if (kind == SDVG_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < NI; ++i) m.sum += valid(i) ? v[i] : 0.f;
      m.sum = warp_sum(m.sum);
    }
    const float mid = m.sum * inv_count;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const float d = valid(i) ? v[i] - mid : 0.f;
      m.m2 = fmaf(d, d, m.m2);
    }
    m.m2 = warp_sum(m.m2);
    return m;
  };
  // f(i, element of the vector at this piece)
  auto with_vector = [&](const float* vec, auto f) {
    if (!vec) return;
#pragma unroll
    for (int i = 0; i < NI; ++i) f(i, valid(i) ? vec[c0 + 32 * i] : 0.f);
  };
  float mean = 0.f, rstd = 1.f;
  if (p.y) {
    if (p.post != SDVG_NORM_NONE) {
      team.join(p, p.post, moments(y, p.post), &mean, &rstd);
#pragma unroll
      for (int i = 0; i < NI; ++i) y[i] = (y[i] - mean) * rstd;
    }
    with_vector(p.post_weight, [&](int i, float w) { y[i] *= w; });
    if (p.gate) {
      with_vector(p.gate + ((unsigned)r / (unsigned)p.gate_rows) * p.ld_gate, [&](int i, float g) { s[i] = fmaf(g, y[i], s[i]); });
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) s[i] += y[i];
    }
  }
  if (p.x_out) store_singles<NI>(s, p.x_out, r * p.ld_x_out + c0, p.x_type, valid);
  if (!p.out) return;
  if (p.norm != SDVG_NORM_NONE) {
    team.join(p, p.norm, moments(s, p.norm), &mean, &rstd);
#pragma unroll
    for (int i = 0; i < NI; ++i) s[i] = (s[i] - mean) * rstd;
  }
  const long long group = p.scale || p.shift ? (unsigned)r / (unsigned)p.mod_rows : 0;
  with_vector(p.weight, [&](int i, float f) { s[i] *= f; });
  with_vector(p.bias, [&](int i, float f) { s[i] += f; });
  with_vector(p.scale ? p.scale + group * p.ld_mod : nullptr, [&](int i, float f) { s[i] = fmaf(s[i], f, s[i]); });
  with_vector(p.shift ? p.shift + group * p.ld_mod : nullptr, [&](int i, float f) { s[i] += f; });
  store_singles<NI>(s, p.out, r * p.ld_out + c0, p.out_type, valid);
}

// ---- rows that no team can hold: one CTA per row, which reads it once per statistic -----------------------------

constexpr int kLongThreads = 512;

// Sum over the CTA; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* buf) {
  v = warp_sum(v);
  __syncthreads();                                     // the last sum's readers are done with buf
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(threadIdx.x % 32 < kLongThreads / 32 ? buf[threadIdx.x % 32] : 0.f);
}

// `value(c)` gives the row's column c; the mean is subtracted for a layer norm, and the variance is
// taken from the centred values.
template <class Value>
__device__ __forceinline__ void row_stats(const NormParams& p, int kind, Value value, float* buf, float* mean, float* rstd) {
  *mean = 0.f;
  *rstd = 1.f;
  if (kind == SDVG_NORM_NONE) return;
  if (kind == SDVG_NORM_LAYER) {
    float s = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kLongThreads) s += value(c);
    *mean = block_sum(s, buf) / p.num_cols;
  }
  float q = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += kLongThreads) {
    const float d = value(c) - *mean;
    q = fmaf(d, d, q);
  }
  *rstd = 1.f / sqrtf(block_sum(q, buf) * p.inv_cols + p.eps);
}

__global__ void __launch_bounds__(kLongThreads) gated_norm_long_kernel(const __grid_constant__ NormParams p) {
  __shared__ float buf[kLongThreads / 32];
  sdvg::overlap_begin();
  sdvg::overlap_wait();
  const long long r = blockIdx.x;
  const float* gate = p.gate ? p.gate + (r / p.gate_rows) * p.ld_gate : nullptr;
  const float* scale = p.scale ? p.scale + (r / p.mod_rows) * p.ld_mod : nullptr;
  const float* shift = p.shift ? p.shift + (r / p.mod_rows) * p.ld_mod : nullptr;
  float y_mean = 0.f, y_rstd = 1.f;
  if (p.y) row_stats(p, p.post, [&](int c) { return load_elem(p.y, r * p.ld_y + c, p.y_type); }, buf, &y_mean, &y_rstd);
  auto sum = [&](int c) {
    float v = load_elem(p.x, r * p.ld_x + c, p.x_type);
    if (p.y) {
      float y = (load_elem(p.y, r * p.ld_y + c, p.y_type) - y_mean) * y_rstd;
      if (p.post_weight) y *= p.post_weight[c];
      v = gate ? fmaf(gate[c], y, v) : v + y;
    }
    return v;
  };
  float mean = 0.f, rstd = 1.f;
  if (p.out) row_stats(p, p.norm, sum, buf, &mean, &rstd);
  for (int c = threadIdx.x; c < p.cols; c += kLongThreads) {
    const float s = sum(c);                          // read before either output is written: both may be in place
    if (p.x_out) store_elem(p.x_out, r * p.ld_x_out + c, p.x_type, s);
    if (!p.out) continue;
    float o = (s - mean) * rstd;
    if (p.weight) o *= p.weight[c];
    if (p.bias) o += p.bias[c];
    if (scale) o *= 1.f + scale[c];
    if (shift) o += shift[c];
    store_elem(p.out, r * p.ld_out + c, p.out_type, o);
  }
}

// ---- host side -------------------------------------------------------------------------------

int device_sms(int* sms) {
  static thread_local int cached_dev = -1, cached = 0;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev != cached_dev) {
    e = cudaDeviceGetAttribute(&cached, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) cached_dev = dev;
  }
  *sms = cached;
  return sdvg::cuda_status(e);
}

constexpr int kMostDynamic = 200 * 1024;
constexpr int kFreeDynamic = 40 * 1024;                // needs no opt-in, with what the kernel has statically: 48 KB in all

template <int XW, int YW, int NI, bool WARP, bool FULL>
int launch_team_as(const NormParams& p, int threads, int sms, cudaStream_t stream) {
  const int rows_per_cta = WARP ? threads / 32 : 1;
  const int want = (p.rows + rows_per_cta - 1) / rows_per_cta;
  const int dynamic = threads * kSlots * (Ring<XW, NI>::kBytes + Ring<YW, NI>::kBytes);
  static_assert((WARP ? 128 : kTeamThreads) * kSlots * (Ring<XW, NI>::kBytes + Ring<YW, NI>::kBytes) <= kMostDynamic, "ring size");
  int grid = want;
  if (want > sms || dynamic > kFreeDynamic) {
    // a grid that the device holds at once: teams walk rows of equal number.  Asked again when the shape changes.
    static thread_local int known_dev = -1, known_dynamic = -1, resident = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return sdvg::cuda_status(e);
    if (dev != known_dev || dynamic != known_dynamic) {
      auto kernel = gated_norm_kernel<XW, YW, NI, WARP, FULL>;
      known_dev = -1;
      if (dynamic > kFreeDynamic) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostDynamic);
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, dynamic);
      if (e != cudaSuccess) return sdvg::cuda_status(e);
      known_dev = dev;
      known_dynamic = dynamic;                         // a multiple of the thread count for each instance
    }
    grid = std::min(want, sms * std::max(resident, 1));
  }
  return sdvg::cuda_status(sdvg::launch_overlapped(gated_norm_kernel<XW, YW, NI, WARP, FULL>, grid, threads, dynamic, 0, stream, p));
}

template <int XW, int YW, int NI, bool WARP>
int launch_team(const NormParams& p, int threads, int sms, cudaStream_t stream) {
  return p.cols == (WARP ? 32 : threads) * NI * 8 ? launch_team_as<XW, YW, NI, WARP, true>(p, threads, sms, stream)
                                                  : launch_team_as<XW, YW, NI, WARP, false>(p, threads, sms, stream);
}

template <int XW, int YW>
int launch_vec(const NormParams& p, int sms, cudaStream_t stream) {
  const int vecs = p.cols / 8;
  if (vecs <= 32) return launch_team<XW, YW, 1, true>(p, 128, sms, stream);
  if (vecs <= 64) return launch_team<XW, YW, 2, true>(p, 128, sms, stream);
  if (vecs <= 2 * kTeamThreads) return launch_team<XW, YW, 2, false>(p, (vecs + 63) / 64 * 32, sms, stream);
  return -1;
}

int launch(const NormParams& p, bool vec, cudaStream_t stream) {
  int sms = 0;
  int st = device_sms(&sms);
  if (st != SDVG_OK) return st;
  st = -1;                                             // -1: a row does not fit the team
  if (vec) {
    const bool x4 = p.x_type == SDVG_F32, y4 = p.y && p.y_type == SDVG_F32;
    if (!p.y) st = x4 ? launch_vec<4, 0>(p, sms, stream) : launch_vec<2, 0>(p, sms, stream);
    else if (y4) st = x4 ? launch_vec<4, 4>(p, sms, stream) : launch_vec<2, 4>(p, sms, stream);
    else st = x4 ? launch_vec<4, 2>(p, sms, stream) : launch_vec<2, 2>(p, sms, stream);
    if (st != -1) return st;
  } else if (p.cols <= 512 * 16) {
    auto single = [&](void (*kernel)(NormParams), int pieces) {
      const int threads = ((p.cols + pieces - 1) / pieces + 31) / 32 * 32;
      return sdvg::cuda_status(sdvg::launch_overlapped(kernel, p.rows, threads, 0, 0, stream, p));
    };
    if (p.cols <= 256) return single(gated_norm_single_kernel<1>, 1);
    if (p.cols <= 1024) return single(gated_norm_single_kernel<4>, 4);
    if (p.cols <= 2048) return single(gated_norm_single_kernel<8>, 8);
    return single(gated_norm_single_kernel<16>, 16);
  }
  return sdvg::cuda_status(sdvg::launch_overlapped(gated_norm_long_kernel, p.rows, kLongThreads, 0, 0, stream, p));
}

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int sdvg_gated_norm(const void* x, int64_t ld_x, int x_type, const void* y, int64_t ld_y, int y_type, int post_norm,
                    const float* post_weight, const float* gate, int64_t ld_gate, int gate_rows, void* x_out,
                    int64_t ld_x_out, int norm, const float* weight, const float* bias, const float* scale,
                    const float* shift, int64_t ld_mod, int mod_rows, float eps, void* out, int64_t ld_out, int out_type,
                    int rows, int cols, void* stream) {
  SDVG_RANGE();
  constexpr int kMaxExtent = 0x7fffffff - 1024;                  // a column one step of a CTA further on is still an int
  if (rows < 0 || cols < 1 || rows > kMaxExtent || cols > kMaxExtent) return SDVG_ERR_BAD_SHAPE;
  if (post_norm < SDVG_NORM_NONE || post_norm > SDVG_NORM_LAYER || norm < SDVG_NORM_NONE || norm > SDVG_NORM_LAYER)
    return SDVG_ERR_INVALID_ARG;
  if (!sdvg::elem_type_ok(x_type) || (y && !sdvg::elem_type_ok(y_type)) || (out && !sdvg::elem_type_ok(out_type)))
    return SDVG_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !isfinite(eps)) return SDVG_ERR_INVALID_ARG;
  if (!y && (post_norm != SDVG_NORM_NONE || post_weight || gate)) return SDVG_ERR_INVALID_ARG;
  if ((gate && gate_rows < 1) || ((scale || shift) && mod_rows < 1)) return SDVG_ERR_INVALID_ARG;
  if (rows == 0) return SDVG_OK;
  if (!x || (!x_out && !out)) return SDVG_ERR_INVALID_ARG;
  if (rows > 1 && (ld_x < cols || (y && ld_y < cols) || (x_out && ld_x_out < cols) || (out && ld_out < cols)))
    return SDVG_ERR_BAD_SHAPE;
  if ((gate && rows > gate_rows && ld_gate < cols) || ((scale || shift) && rows > mod_rows && ld_mod < cols))
    return SDVG_ERR_BAD_SHAPE;
  if (!aligned_to(x, sdvg::elem_bytes(x_type)) || (y && !aligned_to(y, sdvg::elem_bytes(y_type))) ||
      !aligned_to(x_out, sdvg::elem_bytes(x_type)) || (out && !aligned_to(out, sdvg::elem_bytes(out_type))) ||
      !aligned_to(post_weight, 4) || !aligned_to(gate, 4) || !aligned_to(weight, 4) || !aligned_to(bias, 4) ||
      !aligned_to(scale, 4) || !aligned_to(shift, 4))
    return SDVG_ERR_MISALIGNED;
  const int st = sdvg::require_sm100();
  if (st != SDVG_OK) return st;
  NormParams p = {};
  p.x = x;
  p.y = y;
  p.x_out = x_out;
  p.out = out;
  p.post_weight = post_weight;
  p.gate = gate;
  p.weight = weight;
  p.bias = bias;
  p.scale = scale;
  p.shift = shift;
  p.ld_x = ld_x;
  p.ld_y = ld_y;
  p.ld_x_out = ld_x_out;
  p.ld_out = ld_out;
  p.ld_gate = ld_gate;
  p.ld_mod = ld_mod;
  p.x_type = x_type;
  p.y_type = y_type;
  p.out_type = out_type;
  p.post = post_norm;
  p.norm = norm;
  p.gate_rows = gate_rows;
  p.mod_rows = mod_rows;
  p.rows = rows;
  p.cols = cols;
  p.eps = eps;
  p.inv_cols = 1.f / (float)cols;
  p.num_cols = (float)cols;
  // whole vectors: every address a row or a vector is read or written at is a multiple of 16 bytes
  auto rows_ok = [&](const void* base, int64_t ld, int type) {
    return !base || (sdvg::aligned16(base) && (rows == 1 || ld * sdvg::elem_bytes(type) % 16 == 0));
  };
  auto groups_ok = [&](const float* base, int64_t ld, int group_rows) {
    return !base || (sdvg::aligned16(base) && (rows <= group_rows || ld % 4 == 0));
  };
  const bool vec = cols % 8 == 0 && rows_ok(x, ld_x, x_type) && rows_ok(y, ld_y, y_type) && rows_ok(x_out, ld_x_out, x_type) &&
                   rows_ok(out, ld_out, out_type) && groups_ok(gate, ld_gate, gate_rows) && groups_ok(scale, ld_mod, mod_rows) &&
                   groups_ok(shift, ld_mod, mod_rows) && sdvg::aligned16(post_weight) && sdvg::aligned16(weight) &&
                   sdvg::aligned16(bias);
  return launch(p, vec, (cudaStream_t)stream);
}

}  // extern "C"
