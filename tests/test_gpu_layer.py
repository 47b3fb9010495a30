"""A transformer layer around the block attention in library calls: against the separate calls, against fp64, captured,
and driving the speculative schedule."""
import numpy as np
import pytest
import torch

from dense_utils import f64
from gpu_utils import to_bits
from oracle import dense_oracle as D
from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api, schedule, synth

pytestmark = pytest.mark.gpu

SH = synth.Shape("layer", heads=3, head_dim=64, frames=2, grid_h=5, grid_w=7, slots=2)
WIDE = synth.Shape("layer128", heads=2, head_dim=128, frames=3, grid_h=4, grid_w=12, slots=3)


def randn(gen, *shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda") * std + mean


def weights(sh, seed, scope="row", post=False, hidden=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c = sh.heads * sh.head_dim
    f = hidden or 4 * c
    mat = lambda n, k: randn(gen, n, k, std=k ** -0.5).bfloat16()
    vec = lambda n, std=0.2, mean=0.0: randn(gen, n, std=std, mean=mean)
    width = c if scope == "row" else sh.head_dim
    return schedule.LayerWeights(mat(3 * c, c), mat(c, c), mat(f, c), mat(c, f), vec(3 * c), vec(c), vec(f), vec(c),
                                 vec(width, mean=1.0), vec(width, mean=1.0),
                                 api.SDVG_SCOPE_ROW if scope == "row" else api.SDVG_SCOPE_HEAD,
                                 vec(c, mean=1.0) if post else None, vec(c, mean=1.0) if post else None)


def model(sh, blocks=4, **cache):
    tab = api.sdvg_rope3d_table(sh.head_dim, blocks * sh.frames, sh.grid_h, sh.grid_w).cuda()
    kw = {}
    if cache.get("e4m3") and not cache.get("tile_scales"):
        kw = {k: torch.full((sh.heads,), 448.0 / 8.0, device="cuda") for k in ("q_inv_scale", "k_inv_scale", "v_inv_scale")}
    return schedule.ModelState(api.Cache(sh.slots, sh.heads, sh.block_tokens, sh.head_dim, **cache),
                               (sh.frames, sh.grid_h, sh.grid_w), tab, blocks * sh.frames, sh.scale, **kw)


def stream(sh, seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c = sh.heads * sh.head_dim
    return randn(gen, sh.block_tokens, c, std=1.5).to(dtype), randn(gen, sh.frames, 6 * c, std=0.3)


def layer_ref(sh, w, x, mod, ring_k, ring_v, block, tab, tab_frames):
    """fp64; ring_k, ring_v: [keys, heads, dim] of the visible committed blocks.  Returns (stream, k of the block, v)."""
    t, c, rows = sh.block_tokens, sh.heads * sh.head_dim, sh.block_tokens // sh.frames
    v64 = lambda a: None if a is None else f64(a)
    scope = "row" if w.scope == api.SDVG_SCOPE_ROW else "head"
    m = [mod[:, i * c:(i + 1) * c] for i in range(6)]
    _, h = D.gated_norm_ref(x, scale=m[1], shift=m[0], mod_rows=rows)
    qkv = D.linear_ref(h, f64(w.w_qkv), v64(w.b_qkv))
    q, k, v = (qkv[:, i * c:(i + 1) * c].reshape(t, sh.heads, sh.head_dim) for i in range(3))
    grid = (sh.frames, sh.grid_h, sh.grid_w)
    q, k = (D.qk_norm_rope_ref(a, v64(n), scope, w.eps, grid, block * sh.frames, tab, tab_frames)
            for a, n in ((q, w.q_norm), (k, w.k_norm)))
    keys, vals = np.concatenate([ring_k, k]), np.concatenate([ring_v, v])
    a = np.empty((t, c))
    for i in range(sh.heads):
        s = q[:, i] @ keys[:, i].T * sh.scale
        e = np.exp(s - s.max(-1, keepdims=True))
        a[:, i * sh.head_dim:(i + 1) * sh.head_dim] = e / e.sum(-1, keepdims=True) @ vals[:, i]
    p = D.linear_ref(a, f64(w.w_out), v64(w.b_out))
    post = "none" if w.post_attn is None else "rms"
    x1, h = D.gated_norm_ref(x, p, post, v64(w.post_attn), m[2], rows, "layer", None, None, m[4], m[3], rows)
    f = D.linear_ref(D.linear_ref(h, f64(w.w_up), v64(w.b_up), "gelu_tanh"), f64(w.w_down), v64(w.b_down))
    out, _ = D.gated_norm_ref(x1, f, post, v64(w.post_ff), m[5], rows)
    return out, k, v


@pytest.mark.parametrize("sh,scope,post,dtype", [(SH, "row", False, torch.bfloat16), (SH, "head", True, torch.bfloat16),
                                                 (WIDE, "row", True, torch.float32), (WIDE, "head", False, torch.float32)])
def test_layer_over_blocks_against_fp64(sh, scope, post, dtype):
    w, m = weights(sh, 1, scope, post), model(sh)
    layer = schedule.TransformerLayer(w, m, dtype)
    tab, held = m.table.cpu().numpy(), []
    none = np.empty((0, sh.heads, sh.head_dim))
    for b in range(4):                                           # one more than the larger ring: the last evicts
        x, mod = stream(sh, 10 + b, dtype)
        x_out = torch.full_like(x, float("nan"))
        layer.step(x, mod, b, x_out)
        m.check_status("layer")
        visible = held[-(sh.slots - 1):]
        ref, k, v = layer_ref(sh, w, f64(x), f64(mod), np.concatenate([none] + [a for a, _ in visible]),
                              np.concatenate([none] + [a for _, a in visible]), b, tab, m.tab_frames)
        got = f64(x_out)
        # eight intermediate results are rounded to bf16 (each off by at most 2^-8 relative) on a path of gain about one
        rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert rel <= 8 * 2.0 ** -8, (b, rel)
        assert np.abs(got - ref).max() <= 0.1 * np.abs(ref).max()
        assert layer.commit(x, mod, b) == (b - sh.slots if b >= sh.slots else -1)
        got_k, got_v = m.cache.read_block(b % sh.slots)
        for g, r in ((got_k, k), (got_v, v)):
            assert np.linalg.norm(f64(g) - r) <= 4 * 2.0 ** -8 * np.linalg.norm(r)
        held.append((f64(got_k), f64(got_v)))


def test_layer_equals_the_separate_calls_in_place_and_in_a_graph():
    sh, b = WIDE, 0
    w, m, m2 = weights(sh, 2), model(sh), model(sh)
    layer = schedule.TransformerLayer(w, m)
    x, mod = stream(sh, 20)
    x_out = torch.empty_like(x)
    layer.step(x, mod, b, x_out)
    # the same calls one by one, on buffers of their own
    t, c, rows = sh.block_tokens, sh.heads * sh.head_dim, sh.block_tokens // sh.frames
    new = lambda cols: torch.empty((t, cols), device="cuda", dtype=torch.bfloat16)
    part = [mod[:, i * c:(i + 1) * c] for i in range(6)]
    h, qkv, x1, h2, ff, y = new(c), new(3 * c), new(c), new(c), new(4 * c), new(c)
    ws = m2.workspace
    api.sdvg_gated_norm(x, h, scale=part[1], shift=part[0], modulate_rows=rows)
    api.sdvg_linear(h, w.w_qkv, qkv, ws, bias=w.b_qkv)
    q, k, v = (qkv[:, i * c:(i + 1) * c].view(t, sh.heads, sh.head_dim) for i in range(3))
    q_r, k_r = torch.empty_like(m2.q_roped), torch.empty_like(m2.q_roped)
    api.sdvg_qk_norm_rope3d_commit(m2.cache, q, k, v, w.q_norm, w.k_norm, api.SDVG_SCOPE_ROW, 1e-6, q_r, k_r, m2.grid, 0, m2.table,
                                   m2.tab_frames, b, api.SDVG_STAGE)
    attn = torch.empty_like(m2.out)
    api.sdvg_block_attn_fwd(q_r, k_r, v.contiguous(), m2.cache, b, attn, None, sh.scale, ws)
    api.sdvg_linear(attn.view(t, c), w.w_out, x1, ws, bias=w.b_out, gate=part[2], gate_rows=rows, residual=x)
    api.sdvg_gated_norm(x1, h2, scale=part[4], shift=part[3], modulate_rows=rows)
    api.sdvg_linear(h2, w.w_up, ff, ws, bias=w.b_up, act=api.SDVG_ACT_GELU_TANH)
    api.sdvg_linear(ff, w.w_down, y, ws, bias=w.b_down, gate=part[5], gate_rows=rows, residual=x1)
    assert np.array_equal(to_bits(m.q_roped), to_bits(q_r)) and np.array_equal(to_bits(m.out), to_bits(attn))
    assert np.array_equal(to_bits(x_out), to_bits(y))
    # in place, and captured and replayed on other inputs and back
    same = x.clone()
    layer.step(same, mod, b, same)
    assert torch.equal(same, x_out)
    replayed = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, mod, b, replayed)
    keep = x.clone()
    x.copy_(torch.flip(keep, (0,)))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(replayed, x_out)
    x.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(replayed, x_out)
    m.check_status("layer")


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_layer_over_8_bit_rings(tiled, scope):
    """The same layer over an 8-bit ring stays within the format's step (2^-4) of the bf16 ring's."""
    sh = WIDE
    w = weights(sh, 3, scope)
    m, m8 = model(sh), model(sh, e4m3=True, tile_scales=tiled)
    one, eight = schedule.TransformerLayer(w, m), schedule.TransformerLayer(w, m8)
    for b in range(4):
        x, mod = stream(sh, 30 + b)
        a, c = torch.empty_like(x), torch.empty_like(x)
        one.step(x, mod, b, a)
        eight.step(x, mod, b, c)
        m.check_status("bf16")
        m8.check_status("e4m3")
        rel = float((a.float() - c.float()).norm() / a.float().norm())
        assert rel <= 2.0 ** -4, (b, rel)
        assert one.commit(x, mod, b) == eight.commit(x, mod, b)


def test_schedule_with_layers_runs_both_branches():
    """The drafter/router/target flow on layers: accept pattern and evictions are the oracle's, and each ring ends with the K/V of
    the stream that the branch taken committed."""
    sh, blocks, steps = SH, 5, 2
    scores = np.array([[1.0, 1.0], [1.0, 0.5], [-2.0, 1.0], [0.9, 0.8], [1.0, -3.0]], dtype=np.float32)
    d, t = model(sh, blocks), model(sh, blocks)
    dl, tl = schedule.TransformerLayer(weights(sh, 5), d), schedule.TransformerLayer(weights(sh, 6), t)
    sink = torch.empty((sh.block_tokens, sh.heads * sh.head_dim), device="cuda", dtype=torch.bfloat16)
    seeds = {"step": 0, "clean": 50, "accepted": 70}
    given = lambda who, b, kind, s: stream(sh, 1000 * (who == "target") + 100 * b + seeds[kind] + s) + (sink,)
    res = schedule.run_schedule(blocks, steps, torch.from_numpy(scores).cuda(), 0.0, d, t, given, drafter_layer=dl, target_layer=tl)
    accept, _, _ = O.route_ref(scores.reshape(-1), None, blocks, 2, 0, 0.0)
    assert res.accept.tolist() == accept.tolist() == [0, 1, 0, 1, 0]
    assert res.drafter_attn_calls == steps * blocks and res.target_attn_calls == steps * 3
    assert res.target_source == ["regenerated", "accepted", "regenerated", "accepted", "regenerated"]
    assert res.drafter_evicted == res.target_evicted == [-1, -1, 0, 1, 2]
    check = model(sh, blocks)
    again = schedule.TransformerLayer(weights(sh, 6), check)
    for b in range(blocks):
        x, mod, _ = given("target", b, "accepted" if accept[b] else "clean", 0)
        again.commit(x, mod, b)
    for s in range(sh.slots):
        for a, c in zip(t.cache.read_block(s), check.cache.read_block(s)):
            assert torch.equal(a, c)


def test_time_modulation_against_fp64():
    gen = torch.Generator(device="cuda").manual_seed(7)
    mat = lambda n, k: randn(gen, n, k, std=k ** -0.5).bfloat16()
    vec = lambda n: randn(gen, n, std=0.2)
    tm = schedule.TimeModulation(mat(192, 256), mat(192, 192), mat(6 * 192, 192), vec(192), vec(192), vec(6 * 192),
                                 randn(gen, 1, 6 * 192))
    feats = randn(gen, 3, 256).bfloat16()
    ws = api.attn_workspace()
    got = tm(feats, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK and got.dtype == torch.float32 and got.shape == (3, 6 * 192)
    e = D.linear_ref(D.linear_ref(f64(feats), f64(tm.w1), f64(tm.b1), "silu"), f64(tm.w2), f64(tm.b2), "silu")
    ref = D.linear_ref(e, f64(tm.w_mod), f64(tm.b_mod)) + f64(tm.offsets)
    # two intermediate results rounded to bf16
    assert np.linalg.norm(f64(got) - ref) <= 2 * 2.0 ** -8 * np.linalg.norm(ref)


@pytest.mark.parametrize("cols", [64, 1536, 1537, 10248])
@pytest.mark.parametrize("groups", [3, 100])
def test_norms_see_the_modulation_that_the_call_before_them_wrote(cols, groups):
    """One modulation buffer rewritten in place by a linear layer, each time just before the norm that reads it as gate, scale and
    shift; launches overlap, results are those of calls with a wait between them."""
    gen = torch.Generator(device="cuda").manual_seed(41)
    rows, ws = 300, api.attn_workspace()
    feats = [randn(gen, groups, 64).bfloat16() for _ in range(4)]
    w = randn(gen, 3 * cols, 64, std=1 / 8).bfloat16()
    x, y = (randn(gen, rows, cols).bfloat16() for _ in range(2))
    mod = torch.zeros((groups, 3 * cols), device="cuda")
    gate, scale, shift = (mod[:, i * cols:(i + 1) * cols] for i in range(3))

    def chain(sync):
        outs = torch.full((24, rows, cols), float("nan"), device="cuda", dtype=torch.bfloat16)
        torch.cuda.synchronize()
        for i, out in enumerate(outs):
            api.sdvg_linear(feats[i % 4], w, mod, ws)
            if sync:
                torch.cuda.synchronize()
            api.sdvg_gated_norm(x, out, y=y, gate=gate, gate_rows=rows // groups, scale=scale, shift=shift, modulate_rows=rows // groups)
            if sync:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs

    want = chain(True)
    assert not torch.equal(want[0], want[1]) and torch.equal(want[0], want[4])
    assert all(torch.equal(chain(False), want) for _ in range(5))


@pytest.mark.parametrize("heads,dim", [(2, 64), (25, 128)])
def test_the_prologue_sees_the_norm_weights_that_the_call_before_it_wrote(heads, dim):
    gen = torch.Generator(device="cuda").manual_seed(42)
    grid, c, ws = (2, 10, 15), heads * dim, api.attn_workspace()
    tokens = 300
    q, k, v = (randn(gen, tokens, heads, dim).bfloat16() for _ in range(3))
    feats = [randn(gen, 1, 64).bfloat16() for _ in range(4)]
    w = randn(gen, c, 64, std=1 / 8).bfloat16()
    weight = torch.zeros((1, c), device="cuda")
    tab = api.sdvg_rope3d_table(dim, 2, 10, 15).cuda()
    cache = api.Cache(2, heads, tokens, dim)

    def chain(sync):
        outs = torch.zeros((24, tokens, heads, dim), device="cuda", dtype=torch.bfloat16)
        torch.cuda.synchronize()
        for i, out in enumerate(outs):
            api.sdvg_linear(feats[i % 4], w, weight, ws)
            if sync:
                torch.cuda.synchronize()
            api.sdvg_qk_norm_rope3d_commit(cache, q, k, v, weight[0], weight[0], api.SDVG_SCOPE_ROW, 1e-6, out, None, grid, 0, tab, 2, 0,
                                           api.SDVG_STAGE)
            if sync:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return outs, cache.read_block(0)[0]

    want, ring = chain(True)
    assert not torch.equal(want[0], want[1]) and torch.equal(want[0], want[4])
    for _ in range(5):
        got, got_ring = chain(False)
        assert torch.equal(got, want) and torch.equal(got_ring, ring)
