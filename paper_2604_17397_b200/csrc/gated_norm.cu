// Residual add of a sublayer's output (with its own norm and gate) and the modulated norm that opens the next sublayer,
// one pass over the rows.
#include <math.h>

#include "elem_types.cuh"
#include "sdvg_internal.h"

namespace {

using sdvg::load_elem;
using sdvg::store_elem;

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
  float eps, inv_cols;
};

constexpr int kThreads = 256;

// Sum over the CTA; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();                                   // the last sum's readers are done with buf
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = threadIdx.x % 32 < kThreads / 32 ? buf[threadIdx.x % 32] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One CTA per row.  `value(c)` gives the row's column c; the mean is subtracted for a layer norm, and the variance is
// taken from the centred values.
template <class Value>
__device__ __forceinline__ void row_stats(const NormParams& p, int kind, Value value, float* buf, float* mean, float* rstd) {
  *mean = 0.f;
  *rstd = 1.f;
  if (kind == SDVG_NORM_NONE) return;
  if (kind == SDVG_NORM_LAYER) {
    float s = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += kThreads) s += value(c);
    *mean = block_sum(s, buf) * p.inv_cols;
  }
  float q = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += kThreads) {
    const float d = value(c) - *mean;
    q = fmaf(d, d, q);
  }
  *rstd = 1.f / sqrtf(block_sum(q, buf) * p.inv_cols + p.eps);
}

__global__ void __launch_bounds__(kThreads) gated_norm_kernel(const NormParams p) {
  __shared__ float buf[kThreads / 32];
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
  for (int c = threadIdx.x; c < p.cols; c += kThreads) {
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

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace

extern "C" {

int sdvg_gated_norm(const void* x, int64_t ld_x, int x_type, const void* y, int64_t ld_y, int y_type, int post_norm,
                    const float* post_weight, const float* gate, int64_t ld_gate, int gate_rows, void* x_out,
                    int64_t ld_x_out, int norm, const float* weight, const float* bias, const float* scale,
                    const float* shift, int64_t ld_mod, int mod_rows, float eps, void* out, int64_t ld_out, int out_type,
                    int rows, int cols, void* stream) {
  SDVG_RANGE();
  if (rows < 0 || cols < 1) return SDVG_ERR_BAD_SHAPE;
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
  gated_norm_kernel<<<rows, kThreads, 0, (cudaStream_t)stream>>>(p);
  return sdvg::cuda_status(cudaGetLastError());
}

}  // extern "C"
