"""Per-block speculative schedule (Sec. 3 "Inference flow", Fig. 2) on the device.

Host glue only: it strings the library's entry points together in the order the
paper gives and takes the accept/reject branch on the host.  For every block b

  1. the drafter takes ``steps`` denoise steps; each step is one fused
     rope + stage call and one attention call against the drafter ring K^D;
  2. the drafter's final K/V of the block are committed to K^D unconditionally
     (the drafter always conditions on its own earlier outputs);
  3. the router scores the block (worst frame against tau, global block 0 is
     always rejected);
  4. accepted: the target-shaped K/V of the draft block are committed to the
     target ring K^T.  Rejected: the target takes ``steps`` steps of its own
     against K^T and commits the K/V of the regenerated block.

K^D and K^T are independent rings with their own shapes and window sizes.
The tensors of every call come from a ``provider`` callback, so the same
function drives synthetic traces and a real model.
"""
from __future__ import annotations

import functools
from dataclasses import dataclass, field
from typing import Callable, Optional

import numpy as np
import torch

from . import api


def _on_the_models_device(method):
    """The method of a ModelState or a TransformerLayer with the model's device current.  Some library calls launch on the current
    device and its stream, others go by their tensors: here all of them go to one stream."""
    @functools.wraps(method)
    def run(self, *args, **kw):
        dev = getattr(self, "m", self).table.device
        if dev.type != "cuda" or dev.index is None or dev.index == torch.cuda.current_device():
            return method(self, *args, **kw)
        with torch.cuda.device(dev):
            return method(self, *args, **kw)
    return run


@dataclass
class ModelState:
    """Everything one model (drafter or target) needs for its steps."""
    cache: api.Cache
    grid: tuple                    # (latent frames per block, grid rows, grid columns)
    table: torch.Tensor            # device (cos, sin) table built for tab_frames frame positions
    tab_frames: int
    scale: float
    workspace: torch.Tensor = None
    # 8-bit ring (cache.e4m3): static inverse scales per head, device fp32 [heads]; a ring with tile scales
    # (cache.tile_scales) chooses its scales itself and takes none
    q_inv_scale: torch.Tensor = None
    k_inv_scale: torch.Tensor = None
    v_inv_scale: torch.Tensor = None

    def __post_init__(self):
        if self.workspace is None:
            self.workspace = api.attn_workspace(device=self.table.device)
        shape = (self.cache.block_tokens, self.cache.heads, self.cache.head_dim)
        dev = self.table.device
        self.e4m3 = bool(getattr(self.cache, "e4m3", False))
        self.tiled = bool(getattr(self.cache, "tile_scales", False))
        if self.tiled:
            # scales of the roped queries of the current step, [heads][tiles], written by the fused prologue
            self.q_tile_scale = torch.ones((self.cache.heads, self.cache.tiles), dtype=torch.float32, device=dev)
        elif self.e4m3:
            if self.q_inv_scale is None or self.k_inv_scale is None or self.v_inv_scale is None:
                raise ValueError("an 8-bit ring with static scales needs q, k and v inverse scales")
            self.qk_descale = 1.0 / (self.q_inv_scale * self.k_inv_scale)
            self.v_descale = 1.0 / self.v_inv_scale
        # the roped queries of the current step: bf16, or E4M3 codes for an 8-bit ring
        self.q_roped = torch.empty(shape, dtype=torch.uint8 if self.e4m3 else torch.bfloat16, device=dev)
        self.out = torch.empty(shape, dtype=torch.bfloat16, device=dev)

    @property
    def frames(self) -> int:
        return self.grid[0]

    def new_q_roped(self) -> torch.Tensor:
        return torch.zeros_like(self.q_roped)

    def stage_and_attend(self, q, k, v, block: int, q_roped, out) -> None:
        """One denoise step of `block`: fused rope (+ quantise) + stage, then attention against the ring."""
        if self.tiled:
            api.sdvg_rope3d_qk_commit_e4m3_tiled(self.cache, q, k, v, q_roped, self.q_tile_scale, self.grid,
                                                 block * self.frames, self.table, self.tab_frames, block, api.SDVG_STAGE)
        elif self.e4m3:
            api.sdvg_rope3d_qk_commit_e4m3(self.cache, q, k, v, q_roped, self.q_inv_scale, self.k_inv_scale,
                                           self.v_inv_scale, self.grid, block * self.frames, self.table,
                                           self.tab_frames, block, api.SDVG_STAGE)
        else:
            api.sdvg_rope3d_qk_commit(self.cache, q, k, v, q_roped, None, self.grid, block * self.frames, self.table,
                                      self.tab_frames, block, api.SDVG_STAGE)
        self.attend(q_roped, block, out)

    def attend(self, q_roped, block: int, out) -> None:
        """Attention of the staged `block` against the ring; q_roped holds what the prologue of this ring wrote."""
        if self.tiled:
            api.sdvg_block_attn_fwd_e4m3_tiled(q_roped, self.q_tile_scale, self.cache, block, out, None, self.scale,
                                               self.workspace)
        elif self.e4m3:
            api.sdvg_block_attn_fwd_e4m3(q_roped, None, None, self.cache, block, self.qk_descale, self.v_descale, out,
                                         None, self.scale, self.workspace)
        else:
            api.sdvg_block_attn_fwd(q_roped, None, None, self.cache, block, out, None, self.scale, self.workspace)

    def block_steps(self, qs, ks, vs, block: int, q_ropeds, outs) -> None:
        """All denoise steps of `block` in ONE library call (per step: fused rope (+ quantise) + stage, attention)."""
        if self.tiled:
            if getattr(self, "_step_scales", None) is None or len(self._step_scales) != len(qs):
                self._step_scales = [torch.ones_like(self.q_tile_scale) for _ in qs]
            api.sdvg_block_steps_e4m3_tiled(self.cache, qs, ks, vs, q_ropeds, self._step_scales, outs, self.grid,
                                            block * self.frames, self.table, self.tab_frames, block, self.scale,
                                            self.workspace)
        elif self.e4m3:
            api.sdvg_block_steps_e4m3(self.cache, qs, ks, vs, q_ropeds, outs, self.q_inv_scale, self.k_inv_scale,
                                      self.v_inv_scale, self.qk_descale, self.v_descale, self.grid, block * self.frames,
                                      self.table, self.tab_frames, block, self.scale, self.workspace)
        else:
            api.sdvg_block_steps(self.cache, qs, ks, vs, q_ropeds, outs, self.grid, block * self.frames, self.table,
                                 self.tab_frames, block, self.scale, self.workspace)

    @_on_the_models_device
    def check_status(self, where: str) -> None:
        """Raise if a kernel of this model gave up on a bounded wait since the workspace was last reset
        (the status word is sticky, so one check covers every launch since then); synchronises the stream."""
        st = api.sdvg_block_attn_status(self.workspace)
        if st != api.SDVG_OK:
            raise api.SdvgError(st, where)

    def commit_final(self, k, v, block: int) -> int:
        """Rope the block's final K and write it with V into the ring (SDVG_FINAL); returns the evicted block."""
        if self.tiled:
            return api.sdvg_rope3d_qk_commit_e4m3_tiled(self.cache, None, k, v, None, None, self.grid,
                                                        block * self.frames, self.table, self.tab_frames, block,
                                                        api.SDVG_FINAL)
        if self.e4m3:
            return api.sdvg_rope3d_qk_commit_e4m3(self.cache, None, k, v, None, None, self.k_inv_scale, self.v_inv_scale,
                                                  self.grid, block * self.frames, self.table, self.tab_frames, block,
                                                  api.SDVG_FINAL)
        return api.sdvg_rope3d_qk_commit(self.cache, None, k, v, None, None, self.grid, block * self.frames, self.table,
                                         self.tab_frames, block, api.SDVG_FINAL)


@dataclass
class LayerWeights:
    """A transformer layer around the block attention: matrices as stored ([out features, in features], bf16), vectors
    fp32.  width = heads * head_dim of the model's ring."""
    w_qkv: torch.Tensor                    # [3 * width, width]: q, k, v stacked
    w_out: torch.Tensor                    # [width, width]
    w_up: torch.Tensor                     # [hidden, width]
    w_down: torch.Tensor                   # [width, hidden]
    b_qkv: torch.Tensor = None
    b_out: torch.Tensor = None
    b_up: torch.Tensor = None
    b_down: torch.Tensor = None
    q_norm: torch.Tensor = None            # RMS norm weights of q and k: [width], or [head_dim] with SDVG_SCOPE_HEAD
    k_norm: torch.Tensor = None
    scope: int = api.SDVG_SCOPE_ROW
    post_attn: torch.Tensor = None         # weight of an RMS norm after the attention projection; None: no such norm
    post_ff: torch.Tensor = None           # and after the feed-forward pair
    act: int = api.SDVG_ACT_GELU_TANH
    eps: float = 1e-6


class TransformerLayer:
    """One layer of a model (Sec. 4.1 "Models") in library calls: modulated norm, QKV projection, norm of q and k with
    rotary and stage, block attention, output projection onto the residual stream, modulated norm, feed-forward pair.

    ``x`` is the residual stream [block_tokens, width] (bf16 or fp32), ``mod`` the modulation of the step, fp32
    [groups, 6 * width]: shift, scale, gate of the attention half, then of the feed-forward half; token t uses row
    t // ceil(block_tokens / groups) (one row per latent frame, or one for the block).  The buffers between the calls
    belong to the layer: steps of one layer must not overlap on the device.
    """

    def __init__(self, weights: LayerWeights, m: ModelState, x_dtype: torch.dtype = torch.bfloat16):
        c = m.cache
        self.w, self.m, self.width, self.tokens = weights, m, c.heads * c.head_dim, c.block_tokens
        hidden, dev = weights.w_up.shape[0], m.table.device
        new = lambda cols, dtype=torch.bfloat16: torch.empty((self.tokens, cols), dtype=dtype, device=dev)
        self.h, self.qkv, self.ff = new(self.width), new(3 * self.width), new(hidden)
        self.x1 = new(self.width, x_dtype)                       # the stream between the two halves
        post = weights.post_attn is not None or weights.post_ff is not None
        self.y = new(self.width) if post else None
        self.q8 = [new(self.width) for _ in range(3)] if m.e4m3 else None

    def _mod(self, mod: torch.Tensor):
        rows = -(-self.tokens // mod.shape[0])
        mod = mod[:-(-self.tokens // rows)]                      # rows that a token reaches: all, where they divide evenly
        return [mod[:, i * self.width:(i + 1) * self.width] for i in range(6)], rows

    def _heads(self, t: torch.Tensor) -> torch.Tensor:
        return t.unflatten(1, (self.m.cache.heads, self.m.cache.head_dim))

    def _qkv(self, x, mod, with_q: bool = True):
        """q (or None), k, v of the stream x as column ranges of one product."""
        w, n = self.w, self.width
        (shift, scale, *_), rows = self._mod(mod)
        api.sdvg_gated_norm(x, self.h, scale=scale, shift=shift, modulate_rows=rows, eps=w.eps)
        first = 0 if with_q else n
        out = self.qkv[:, first:]
        api.sdvg_linear(self.h, w.w_qkv[first:], out, self.m.workspace, bias=None if w.b_qkv is None else w.b_qkv[first:])
        parts = [out[:, i:i + n] for i in range(0, 3 * n - first, n)]
        return parts if with_q else [None] + parts

    def _rms(self, t, weight, out) -> torch.Tensor:
        """RMS norm of a column range into a contiguous [tokens, heads, dim] tensor (an 8-bit ring takes such tensors).  Rounded to
        bf16 before the rotation, which over a bf16 ring is one pass with the norm and rounds once."""
        if self.w.scope == api.SDVG_SCOPE_ROW:
            api.sdvg_gated_norm(t, out, norm=api.SDVG_NORM_RMS, weight=weight, eps=self.w.eps)
        else:
            dim = self.m.cache.head_dim
            api.sdvg_gated_norm(t, out, norm=api.SDVG_NORM_NONE)           # columns of the product to contiguous rows
            rows = out.view(-1, dim)
            api.sdvg_gated_norm(rows, rows, norm=api.SDVG_NORM_RMS, weight=weight, eps=self.w.eps)
        return self._heads(out)

    def _write_kv(self, q, k, v, block: int, flags: int, q_roped=None) -> int:
        """Norm, rotary and ring write; returns the evicted block."""
        m, w = self.m, self.w
        if not m.e4m3:
            q, k, v = (None if t is None else self._heads(t) for t in (q, k, v))
            return api.sdvg_qk_norm_rope3d_commit(m.cache, q, k, v, w.q_norm, w.k_norm, w.scope, w.eps, q_roped, None, m.grid,
                                                  block * m.frames, m.table, m.tab_frames, block, flags)
        q = None if q is None else self._rms(q, w.q_norm, self.q8[0])
        k = self._rms(k, w.k_norm, self.q8[1])
        api.sdvg_gated_norm(v, self.q8[2], norm=api.SDVG_NORM_NONE)
        v = self._heads(self.q8[2])
        if m.tiled:
            return api.sdvg_rope3d_qk_commit_e4m3_tiled(m.cache, q, k, v, q_roped, None if q is None else m.q_tile_scale,
                                                        m.grid, block * m.frames, m.table, m.tab_frames, block, flags)
        return api.sdvg_rope3d_qk_commit_e4m3(m.cache, q, k, v, q_roped, None if q is None else m.q_inv_scale, m.k_inv_scale,
                                              m.v_inv_scale, m.grid, block * m.frames, m.table, m.tab_frames, block, flags)

    @_on_the_models_device
    def step(self, x, mod, block: int, x_out) -> None:
        """One denoise step of `block`: the ring's slot of the block is staged, x_out (may be x) receives the stream."""
        m, w = self.m, self.w
        q, k, v = self._qkv(x, mod)
        self._write_kv(q, k, v, block, api.SDVG_STAGE, m.q_roped)
        m.attend(m.q_roped, block, m.out)
        (_, _, gate1, shift2, scale2, gate2), rows = self._mod(mod)
        attn = m.out.view(self.tokens, self.width)
        if w.post_attn is None:
            api.sdvg_linear(attn, w.w_out, self.x1, m.workspace, bias=w.b_out, gate=gate1, gate_rows=rows, residual=x)
            api.sdvg_gated_norm(self.x1, self.h, scale=scale2, shift=shift2, modulate_rows=rows, eps=w.eps)
        else:
            api.sdvg_linear(attn, w.w_out, self.y, m.workspace, bias=w.b_out)
            api.sdvg_gated_norm(x, self.h, y=self.y, gate=gate1, gate_rows=rows, post_norm=api.SDVG_NORM_RMS,
                                post_weight=w.post_attn, x_out=self.x1, scale=scale2, shift=shift2, modulate_rows=rows,
                                eps=w.eps)
        api.sdvg_linear(self.h, w.w_up, self.ff, m.workspace, bias=w.b_up, act=w.act)
        if w.post_ff is None:
            api.sdvg_linear(self.ff, w.w_down, x_out, m.workspace, bias=w.b_down, gate=gate2, gate_rows=rows, residual=self.x1)
        else:
            api.sdvg_linear(self.ff, w.w_down, self.y, m.workspace, bias=w.b_down)
            api.sdvg_gated_norm(self.x1, None, y=self.y, gate=gate2, gate_rows=rows, post_norm=api.SDVG_NORM_RMS,
                                post_weight=w.post_ff, x_out=x_out, eps=w.eps)

    @_on_the_models_device
    def commit(self, x, mod, block: int, check: bool = False) -> int:
        """The block's final K/V from its final stream into the ring (SDVG_FINAL); returns the evicted block.  K and V come from
        a product with bounded waits; ``check`` reads the status word (and so synchronises) before the ring is written, and
        raises if a kernel of this model gave up."""
        _, k, v = self._qkv(x, mod, with_q=False)
        if check:
            self.m.check_status(f"final K/V of block {block}")
        return self._write_kv(None, k, v, block, api.SDVG_FINAL)


@dataclass
class TimeModulation:
    """The modulation of a step from its time features (Sec. 4.1: the sampler's time steps): fp32 [groups, 6 * width] =
    offsets + W_mod silu(W2 silu(W1 features + b1) + b2) + b_mod, features bf16 [groups, ...]."""
    w1: torch.Tensor
    w2: torch.Tensor
    w_mod: torch.Tensor
    b1: torch.Tensor = None
    b2: torch.Tensor = None
    b_mod: torch.Tensor = None
    offsets: torch.Tensor = None           # learned, fp32 [1, 6 * width]

    def __call__(self, features, workspace, out=None) -> torch.Tensor:
        rows, dev = features.shape[0], features.device
        new = lambda cols, dtype=torch.bfloat16: torch.empty((rows, cols), dtype=dtype, device=dev)
        a, e = new(self.w1.shape[0]), new(self.w2.shape[0])
        out = new(self.w_mod.shape[0], torch.float32) if out is None else out
        api.sdvg_linear(features, self.w1, a, workspace, bias=self.b1, act=api.SDVG_ACT_SILU)
        api.sdvg_linear(a, self.w2, e, workspace, bias=self.b2, act=api.SDVG_ACT_SILU)
        api.sdvg_linear(e, self.w_mod, out, workspace, bias=self.b_mod,
                        residual=None if self.offsets is None else self.offsets.expand(rows, -1))
        return out


@dataclass
class TraceResult:
    accept: np.ndarray
    q_min: np.ndarray
    drafter_evicted: list = field(default_factory=list)
    target_evicted: list = field(default_factory=list)
    drafter_attn_calls: int = 0
    target_attn_calls: int = 0
    target_source: list = field(default_factory=list)     # per block: "accepted" or "regenerated"


def _denoise(model: str, m: ModelState, block: int, steps: int, provider, on_attention, layer) -> int:
    for s in range(steps):
        if layer is not None:
            x, mod, x_out = provider(model, block, "step", s)
            layer.step(x, mod, block, x_out)
        else:
            q, k, v = provider(model, block, "step", s)
            m.stage_and_attend(q, k, v, block, m.q_roped, m.out)
        if on_attention is not None:
            on_attention(model, block, s, m.q_roped, m.out)
    return steps


def _commit_clean(m: ModelState, block: int, layer, given) -> int:
    if layer is not None:
        x, mod, _ = given
        return layer.commit(x, mod, block, check=True)
    _, k, v = given
    return m.commit_final(k, v, block)


def run_schedule(num_blocks: int, steps: int, scores: torch.Tensor, tau: float,
                 drafter: ModelState, target: ModelState,
                 provider: Callable, first_block_index: int = 0,
                 on_attention: Optional[Callable] = None,
                 drafter_layer: Optional[TransformerLayer] = None,
                 target_layer: Optional[TransformerLayer] = None) -> TraceResult:
    """Generate ``num_blocks`` blocks with the drafter/router/target flow.

    scores    device fp32 [num_blocks, frames]: the per-frame reward of every draft block
              (in a real system they appear one block at a time; routing here is also
              done one block at a time, with the block's global index)
    provider  ``provider(model, block, kind, step)`` -> (q, k, v) device bf16 tensors of the
              model's shape; kind is "step" (one denoise step), "clean" (the model's final
              K/V, q is None) or "accepted" (target-shaped K/V of an accepted draft block)
    on_attention  optional ``f(model, block, step, q_roped, out)`` called after each
              attention launch (the tensors are reused by the next step; q_roped holds E4M3
              codes when the model's ring is an 8-bit one)
    drafter_layer, target_layer   optional layers around the models' attention: for such a model the provider gives
              (x, mod, x_out), the residual stream, the step's modulation and where the step's stream goes, in
              place of (q, k, v); for "clean" and "accepted" x_out is not used
    A model whose ``cache`` is an 8-bit ring takes every step through the _e4m3 entry points.
    The flow synchronises where it reads something back: the accept decision of a block, the status word after each
    model's steps, and with a layer once more between a commit's projection of K and V and its ring write.
    """
    if scores.dtype != torch.float32 or scores.dim() != 2 or scores.shape[0] != num_blocks:
        raise ValueError("scores must be float32 [num_blocks, frames]")
    frames = scores.shape[1]
    dev = scores.device
    accept_d = torch.zeros(num_blocks, dtype=torch.uint8, device=dev)
    qmin_d = torch.zeros(num_blocks, dtype=torch.float32, device=dev)
    res = TraceResult(accept=np.zeros(num_blocks, dtype=np.uint8), q_min=np.zeros(num_blocks, dtype=np.float32))
    flat = scores.reshape(-1)
    for i in range(num_blocks):
        b = first_block_index + i
        res.drafter_attn_calls += _denoise("drafter", drafter, b, steps, provider, on_attention, drafter_layer)
        api.sdvg_route(flat[i * frames:(i + 1) * frames], None, 1, frames, b, tau, accept_d[i:i + 1],
                       qmin_d[i:i + 1], None)
        accepted = bool(accept_d[i].item())               # synchronises
        # a kernel that gave up leaves undefined outputs: stop before anything derived from them enters a ring
        drafter.check_status(f"drafter steps of block {b}")
        res.drafter_evicted.append(_commit_clean(drafter, b, drafter_layer, provider("drafter", b, "clean", 0)))
        if accepted:
            given = provider("target", b, "accepted", 0)
            res.target_source.append("accepted")
        else:
            res.target_attn_calls += _denoise("target", target, b, steps, provider, on_attention, target_layer)
            target.check_status(f"target steps of block {b}")
            given = provider("target", b, "clean", 0)
            res.target_source.append("regenerated")
        res.target_evicted.append(_commit_clean(target, b, target_layer, given))
    res.accept = accept_d.cpu().numpy()
    res.q_min = qmin_d.cpu().numpy()
    return res


class BlockStepGraph:
    """The S denoising steps of ONE block captured into a CUDA graph (Sec. 4.1: 4 steps per block).

    The capture holds ONE library call (sdvg_block_steps: per step the fused rope + stage kernel followed
    by the attention kernel), reading q, k, v from fixed input tensors (``self.q[s]``, ``self.k[s]``,
    ``self.v[s]``: fill them before ``replay``) and writing ``self.out[s]``.  The ring state does not change inside the loop (SDVG_STAGE leaves it
    alone), so the captured launches stay valid until the block's final commit; a new block needs a
    new capture because its ring slot, frame offset and key segments differ.  One eager pass runs
    first: the library's one-time set-up (kernel attributes, device queries) must not happen during
    capture.
    """

    def __init__(self, m: ModelState, block: int, steps: int):
        shape = (m.cache.block_tokens, m.cache.heads, m.cache.head_dim)
        dev = m.table.device
        new = lambda: torch.zeros(shape, dtype=torch.bfloat16, device=dev)
        self.q, self.k, self.v = ([new() for _ in range(steps)] for _ in range(3))
        self.q_roped = [m.new_q_roped() for _ in range(steps)]
        self.out = [new() for _ in range(steps)]
        self.m, self.block, self.steps = m, block, steps
        self._run()                                   # warm-up, eager
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._run()

    def _run(self):
        self.m.block_steps(self.q, self.k, self.v, self.block, self.q_roped, self.out)

    def replay(self):
        self.graph.replay()
