"""The transformer layer with 8-bit matrices and rows in library calls: against the separate calls, against the 16-bit layer, captured,
and driving the speculative schedule."""
import numpy as np
import pytest
import torch

from dense_utils import f64
from gpu_utils import to_bits
from oracle import dense_oracle as D
from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api, schedule, synth
from test_gpu_layer import SH, WIDE, model, randn, stream, weights

pytestmark = pytest.mark.gpu

ODD = synth.Shape("layer128x5", heads=5, head_dim=128, frames=2, grid_h=9, grid_w=11, slots=2)
RINGS = {"bf16": {}, "static": dict(e4m3=True), "tiled": dict(e4m3=True, tile_scales=True)}


@pytest.mark.parametrize("sh,ring", [(SH, "bf16"), (WIDE, "bf16"), (WIDE, "static"), (WIDE, "tiled"), (ODD, "tiled")])
@pytest.mark.parametrize("scope,post", [("row", False), ("head", True)])
def test_layer_stays_near_the_16_bit_one(sh, ring, scope, post):
    w, m, m8 = weights(sh, 1, scope, post), model(sh), model(sh, **RINGS[ring])
    one, eight = schedule.TransformerLayer(w, m), schedule.TransformerLayerE4M3(w, m8)
    for b in range(4):
        x, mod = stream(sh, 10 + b)
        a, c = torch.empty_like(x), torch.full_like(x, float("nan"))
        one.step(x, mod, b, a)
        eight.step(x, mod, b, c)
        m8.check_status("8-bit layer")
        # each of the four products has two operands off by at most 2^-4 of a value; the stream they are added to is exact
        change = (a.float() - x.float()).norm()
        assert float((a.float() - c.float()).norm()) <= 8 * 2.0 ** -4 * float(change), b
        assert one.commit(x, mod, b) == eight.commit(x, mod, b)
        if ring == "bf16":
            for g, r in zip(m8.cache.read_block(b % sh.slots), m.cache.read_block(b % sh.slots)):
                assert float((g.float() - r.float()).norm()) <= 2 * 2.0 ** -4 * float(r.float().norm())


@pytest.mark.parametrize("ring", list(RINGS))
def test_layer_equals_the_separate_calls_in_place_and_in_a_graph(ring):
    sh, b = ODD, 0
    w, m, m2 = weights(sh, 2), model(sh, **RINGS[ring]), model(sh, **RINGS[ring])
    layer = schedule.TransformerLayerE4M3(w, m)
    x, mod = stream(sh, 20)
    x_out = torch.empty_like(x)
    layer.step(x, mod, b, x_out)
    t, c, rows = sh.block_tokens, sh.heads * sh.head_dim, sh.block_tokens // sh.frames
    part, ws = [mod[:, i * c:(i + 1) * c] for i in range(6)], m2.workspace
    quant = lambda a, block: (lambda q: (api.sdvg_quant_e4m3_blocks(a, *q), q)[1])(api.e4m3_matrix(*a.shape, block))
    w_qkv, w_out, w_up, w_down = (quant(a, 128) for a in (w.w_qkv, w.w_out, w.w_up, w.w_down))
    h, attn8, h2, ff = (api.e4m3_matrix(t, n) for n in (c, c, c, 4 * c))
    new = lambda n: torch.empty((t, n), device="cuda", dtype=torch.bfloat16)
    qkv, x1, y = new(3 * c), new(c), new(c)
    api.sdvg_gated_norm_e4m3(x, *h, scale=part[1], shift=part[0], modulate_rows=rows)
    api.sdvg_linear_e4m3(*h, *w_qkv, qkv, ws, bias=w.b_qkv)
    q, k, v = (qkv[:, i * c:(i + 1) * c].view(t, sh.heads, sh.head_dim) for i in range(3))
    args = (m2.cache, q, k, v, w.q_norm, w.k_norm, api.SDVG_SCOPE_ROW, 1e-6, m2.q_roped)
    at = (m2.grid, 0, m2.table, m2.tab_frames, b, api.SDVG_STAGE)
    if ring == "bf16":
        api.sdvg_qk_norm_rope3d_commit(*args, None, *at)
    elif ring == "static":
        api.sdvg_qk_norm_rope3d_commit_e4m3(*args, m2.q_inv_scale, m2.k_inv_scale, m2.v_inv_scale, *at)
    else:
        api.sdvg_qk_norm_rope3d_commit_e4m3_tiled(*args, m2.q_tile_scale, *at, api.qk_norm_workspace(t))
    m2.attend(m2.q_roped, b, m2.out)
    api.sdvg_quant_e4m3_blocks(m2.out.view(t, c), *attn8)
    api.sdvg_linear_e4m3(*attn8, *w_out, x1, ws, bias=w.b_out, gate=part[2], gate_rows=rows, residual=x)
    api.sdvg_gated_norm_e4m3(x1, *h2, scale=part[4], shift=part[3], modulate_rows=rows)
    api.sdvg_linear_e4m3(*h2, *w_up, ff[0], ws, bias=w.b_up, act=api.SDVG_ACT_GELU_TANH, out_scale=ff[1])
    api.sdvg_linear_e4m3(*ff, *w_down, y, ws, bias=w.b_down, gate=part[5], gate_rows=rows, residual=x1)
    assert torch.equal(m.q_roped, m2.q_roped) and np.array_equal(to_bits(m.out), to_bits(m2.out))
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


@pytest.mark.parametrize("ring", ["static", "tiled"])
def test_schedule_with_8_bit_layers_runs_both_branches(ring):
    sh, blocks, steps = WIDE, 5, 2
    scores = np.array([[1.0, 1.0], [1.0, 0.5], [-2.0, 1.0], [0.9, 0.8], [1.0, -3.0]], dtype=np.float32)
    d, t = model(sh, blocks, **RINGS[ring]), model(sh, blocks, **RINGS[ring])
    dl, tl = schedule.TransformerLayerE4M3(weights(sh, 5), d), schedule.TransformerLayerE4M3(weights(sh, 6), t)
    sink = torch.empty((sh.block_tokens, sh.heads * sh.head_dim), device="cuda", dtype=torch.bfloat16)
    seeds = {"step": 0, "clean": 50, "accepted": 70}
    given = lambda who, b, kind, s: stream(sh, 1000 * (who == "target") + 100 * b + seeds[kind] + s) + (sink,)
    res = schedule.run_schedule(blocks, steps, torch.from_numpy(scores).cuda(), 0.0, d, t, given, drafter_layer=dl, target_layer=tl)
    accept, _, _ = O.route_ref(scores.reshape(-1), None, blocks, 2, 0, 0.0)
    assert res.accept.tolist() == accept.tolist() == [0, 1, 0, 1, 0]
    assert res.drafter_evicted == res.target_evicted == [-1, -1, -1, 0, 1]
    check = model(sh, blocks, **RINGS[ring])
    again = schedule.TransformerLayerE4M3(weights(sh, 6), check)
    for b in range(blocks):
        x, mod, _ = given("target", b, "accepted" if accept[b] else "clean", 0)
        again.commit(x, mod, b)
    for s in range(sh.slots):
        for a, c in zip(t.cache.read_block(s), check.cache.read_block(s)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("rows", [1, 3])
def test_time_modulation_in_8_bits(rows):
    gen = torch.Generator(device="cuda").manual_seed(7)
    mat = lambda n, k: randn(gen, n, k, std=k ** -0.5).bfloat16()
    vec = lambda n: randn(gen, n, std=0.2)
    tm = schedule.TimeModulation(mat(192, 256), mat(192, 192), mat(6 * 192, 192), vec(192), vec(192), vec(6 * 192),
                                 randn(gen, 1, 6 * 192))
    feats, ws = randn(gen, rows, 256).bfloat16(), api.attn_workspace()
    got = schedule.TimeModulationE4M3(tm)(feats, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK and got.dtype == torch.float32 and got.shape == (rows, 6 * 192)
    e = D.linear_ref(D.linear_ref(f64(feats), f64(tm.w1), f64(tm.b1), "silu"), f64(tm.w2), f64(tm.b2), "silu")
    ref = D.linear_ref(e, f64(tm.w_mod), f64(tm.b_mod))
    # three products of two operands each, off by at most 2^-4 of a value, on a path of gain about one; the offsets are exact
    assert np.linalg.norm(f64(got) - f64(tm.offsets) - ref) <= 6 * 2.0 ** -4 * np.linalg.norm(ref)


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_the_ring_write_sees_what_the_calls_before_it_wrote(tiled, scope):
    """Rows, norm weights and rotary table rewritten in place just before each call; launches overlap, results are those of calls with a
    wait between them."""
    gen = torch.Generator(device="cuda").manual_seed(42)
    heads, grid, ws = 6, (2, 10, 15), api.attn_workspace()
    tokens, c = 300, 6 * 128
    width = c if scope == "row" else 128
    h, hs = api.e4m3_matrix(tokens, 256)
    rows = [randn(gen, tokens, 256).bfloat16() for _ in range(4)]
    w, wsc = api.e4m3_matrix(3 * c, 256, 128)
    api.sdvg_quant_e4m3_blocks(randn(gen, 3 * c, 256, std=1 / 16), w, wsc)
    feats, u = [randn(gen, 1, 64).bfloat16() for _ in range(4)], randn(gen, width, 64, std=1 / 8).bfloat16()
    qkv, weight = torch.zeros((tokens, 3 * c), device="cuda", dtype=torch.bfloat16), torch.zeros((1, width), device="cuda")
    q, k, v = (qkv[:, i * c:(i + 1) * c].view(tokens, heads, 128) for i in range(3))
    tables = [api.sdvg_rope3d_table(128, n, 10, 15).cuda()[:api.lib().sdvg_rope3d_table_floats(128, 2, 10, 15)] for n in (2, 3, 4, 5)]
    table = torch.zeros_like(tables[0])
    cache = api.Cache(2, heads, tokens, 128, e4m3=True, tile_scales=tiled)
    inv, space = torch.full((heads,), 30.0, device="cuda"), api.qk_norm_workspace(tokens)
    sc = api.SDVG_SCOPE_ROW if scope == "row" else api.SDVG_SCOPE_HEAD

    def chain(sync):
        outs = torch.zeros((24, tokens, heads, 128), device="cuda", dtype=torch.uint8)
        scales = torch.zeros((24, heads, 3), device="cuda")
        pause = torch.cuda.synchronize if sync else lambda: None
        pause()
        for i, out in enumerate(outs):
            table.copy_(tables[i % 4])
            pause()
            api.sdvg_linear(feats[i % 4], u, weight, ws)
            pause()
            api.sdvg_gated_norm_e4m3(rows[i % 4], h, hs, norm=api.SDVG_NORM_RMS)
            pause()
            api.sdvg_linear_e4m3(h, hs, w, wsc, qkv, ws)
            pause()
            args = (cache, q, k, v, weight[0], weight[0], sc, 1e-6, out)
            at = (grid, 0, table, 2, 0, api.SDVG_STAGE)
            if tiled:
                api.sdvg_qk_norm_rope3d_commit_e4m3_tiled(*args, scales[i], *at, space)
            else:
                api.sdvg_qk_norm_rope3d_commit_e4m3(*args, inv, inv, inv, *at)
            pause()
        torch.cuda.synchronize()
        return outs, scales, *cache.read_block(0)

    want = chain(True)
    assert not torch.equal(want[0][0], want[0][1]) and torch.equal(want[0][0], want[0][4])
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(chain(False), want))


def test_two_streams_with_workspaces_of_their_own():
    """The same ring shapes written at once from two streams, each with its own cache and workspaces."""
    made = []
    for seed in (1, 2):
        m = model(ODD, **RINGS["tiled"])
        made.append((schedule.TransformerLayerE4M3(weights(ODD, seed), m), m, *stream(ODD, 40 + seed), torch.cuda.Stream()))
    want = []
    for layer, m, x, mod, _ in made:
        out = torch.empty_like(x)
        layer.step(x, mod, 0, out)
        torch.cuda.synchronize()
        want.append((out.clone(), m.q_roped.clone()))
    for _ in range(10):
        outs = []
        for layer, m, x, mod, s in made:
            with torch.cuda.stream(s):
                out = torch.empty_like(x)
                layer.step(x, mod, 0, out)
                outs.append(out)
        torch.cuda.synchronize()
        for (o, q), got, (_, m, *_) in zip(want, outs, made):
            assert torch.equal(got, o) and torch.equal(m.q_roped, q)
