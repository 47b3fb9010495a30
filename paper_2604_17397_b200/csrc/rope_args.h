// Checks of the rotary arguments (block grid, frame range, table) and the fields a kernel needs of them.
#pragma once

#include "sdvg_internal.h"

namespace sdvg {

struct RopeArgs {
  int frames, grid_h, grid_w, frame_offset, tab_frames;
  const float* tab;
};

template <class Params>
int fill_rope(Params& p, int head_dim, int tokens, const RopeArgs& r) {
  if (r.frames <= 0 || r.grid_h <= 0 || r.grid_w <= 0) return SDVG_ERR_BAD_SHAPE;
  if ((long long)r.frames * r.grid_h * r.grid_w != tokens) return SDVG_ERR_BAD_SHAPE;
  if (!r.tab) return SDVG_ERR_INVALID_ARG;
  if (!sdvg::aligned16(r.tab)) return SDVG_ERR_MISALIGNED;
  if (r.tab_frames <= 0) return SDVG_ERR_BAD_SHAPE;
  int pf, ph, pw;
  sdvg_rope3d_pairs(head_dim, &pf, &ph, &pw);
  // the kernels' offsets into the table are ints
  if ((long long)r.tab_frames * pf + (long long)r.grid_h * ph + (long long)r.grid_w * pw > 0x7fffffff) return SDVG_ERR_BAD_SHAPE;
  if (r.frame_offset < 0 || (long long)r.frame_offset + r.frames > r.tab_frames) return SDVG_ERR_BAD_STATE;
  p.grid_hw = r.grid_h * r.grid_w;
  p.grid_w = r.grid_w;
  p.frame_offset = r.frame_offset;
  p.pairs_f = pf;
  p.pairs_h = ph;
  p.tab_h_off = r.tab_frames * pf;                 // in (cos, sin) pairs
  p.tab_w_off = p.tab_h_off + r.grid_h * ph;
  p.tab = reinterpret_cast<const float2*>(r.tab);
  return SDVG_OK;
}

}  // namespace sdvg
