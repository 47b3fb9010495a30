"""sdvg_qk_norm_rope3d_commit against fp64, against the unfused calls, and its ring semantics."""
import numpy as np
import pytest
import torch

from dense_utils import U, assert_close, f64, norm_error, rounding
from gpu_utils import Canaries, to_bits
from oracle import dense_oracle as O
from paper_2604_17397_b200 import api

pytestmark = pytest.mark.gpu

SCOPES = {"row": api.SDVG_SCOPE_ROW, "head": api.SDVG_SCOPE_HEAD}
EPS = 1e-6


def make(heads, dim, grid, slots, scope="row", fused=True, weights=True, seed=0, block=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, c = grid[0] * grid[1] * grid[2], heads * dim
    r = lambda *shape, std=1.0, mean=0.0: torch.randn(shape, generator=gen, device="cuda") * std + mean
    if fused:
        wide = r(t, 3 * c + 8, std=1.7).bfloat16()
        wide[:, 3 * c:] = float("nan")
        q, k, v = (wide[:, i * c:(i + 1) * c].view(t, heads, dim) for i in range(3))
    else:
        q, k, v = (r(t, heads, dim, std=1.7).bfloat16() for _ in range(3))
    width = c if scope == "row" else dim
    tab_frames = (block + 1) * grid[0]
    return dict(q=q, k=k, v=v, qw=r(width, std=0.3, mean=1.0) if weights else None, kw=r(width, std=0.3, mean=1.0) if weights else None,
                scope=scope, grid=grid, tab=api.sdvg_rope3d_table(dim, tab_frames, grid[1], grid[2]).cuda(), tab_frames=tab_frames)


def call(cache, s, q_out, k_out, block, flags=api.SDVG_STAGE, stream=None, q=True):
    return api.sdvg_qk_norm_rope3d_commit(cache, s["q"] if q else None, s["k"], s["v"], s["qw"], s["kw"], SCOPES[s["scope"]], EPS,
                                          q_out, k_out, s["grid"], block * s["grid"][0], s["tab"], s["tab_frames"], block, flags,
                                          stream=stream)


def expected(s, block):
    got = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x, w = f64(x), f64(w)
        ref = O.qk_norm_rope_ref(x, w, s["scope"], EPS, s["grid"], block * s["grid"][0], s["tab"].cpu().numpy(), s["tab_frames"])
        flat = x.reshape(x.shape[0], -1) if s["scope"] == "row" else x
        o, e = norm_error(flat, np.zeros_like(flat), "rms", EPS)
        f = 1.0 if w is None else np.abs(w)
        e, o = ((e + 4 * U * np.abs(o)) * f).reshape(x.shape), (np.abs(o) * f).reshape(x.shape)
        pair = lambda a: np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1)         # |cos|, |sin| <= 1
        e = pair(e) + 4 * U * pair(o)
        got.append((ref, e + rounding(np.abs(ref) + e, torch.bfloat16)))
    return got


GRIDS = [(1, 1, 1), (2, 4, 8), (1, 7, 23), (3, 5, 11)]


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("heads,dim", [(1, 64), (2, 64), (3, 128), (12, 128), (13, 64), (40, 128)])
@pytest.mark.parametrize("scope,fused,weights", [("row", True, True), ("head", False, True), ("row", False, False), ("head", True, False)])
def test_parity(grid, heads, dim, scope, fused, weights):
    s = make(heads, dim, grid, 3, scope, fused, weights, seed=heads + dim)
    t = s["q"].shape[0]
    cache = api.Cache(3, heads, t, dim)
    guard = Canaries()
    guard.watch_cache(cache)
    q_out, k_out = (guard.new((t, heads, dim), torch.bfloat16) for _ in range(2))
    assert call(cache, s, q_out, k_out, 0) == -1
    (q_ref, q_tol), (k_ref, k_tol) = expected(s, 0)
    assert_close(q_out, q_ref, q_tol, "q")
    assert_close(k_out, k_ref, k_tol, "k")
    ring_k, ring_v = cache.read_block(0)
    assert np.array_equal(to_bits(ring_k), to_bits(k_out)) and np.array_equal(to_bits(ring_v), to_bits(s["v"]))
    guard.check()
    assert cache.state() == (0, [-1, -1, -1], 0)


def test_frame_positions_past_the_first_block():
    s = make(4, 128, (2, 3, 5), 4, block=2, seed=5)
    cache = api.Cache(4, 4, 30, 128)
    for b in range(2):
        call(cache, s, None, None, b, api.SDVG_FINAL, q=False)
    q_out = torch.empty((30, 4, 128), device="cuda", dtype=torch.bfloat16)
    call(cache, s, q_out, None, 2)
    (q_ref, q_tol), (k_ref, k_tol) = expected(s, 2)
    assert_close(q_out, q_ref, q_tol)
    assert_close(cache.read_block(2)[0], k_ref, k_tol)


def test_ring_order_eviction_and_untouched_slots():
    grid, slots = (1, 3, 5), 2
    cache = api.Cache(slots, 2, 15, 64)
    held = {}
    for b in range(5):
        s = make(2, 64, grid, slots, seed=b, block=b)
        call(cache, s, None, None, b, api.SDVG_STAGE, q=False)
        other = held.get(b - 1)
        if other:                                  # the neighbour's slot is left as it was
            k, v = cache.read_block((b - 1) % slots)
            assert torch.equal(k, other[0]) and torch.equal(v, other[1])
        assert call(cache, s, None, None, b, api.SDVG_FINAL, q=False) == (b - slots if b >= slots else -1)
        held[b] = cache.read_block(b % slots)
        _, (k_ref, k_tol) = expected(s, b)
        assert_close(held[b][0], k_ref, k_tol)
        assert torch.equal(held[b][1], s["v"])
    with pytest.raises(api.SdvgError) as e:
        call(cache, make(2, 64, grid, slots, block=7), None, None, 7, q=False)
    assert e.value.status == api.SDVG_ERR_BAD_STATE


@pytest.mark.parametrize("scope", ["row", "head"])
def test_in_place_and_graph_replay(scope):
    s = make(5, 128, (2, 6, 7), 3, scope, fused=False, seed=11)
    cache = api.Cache(3, 5, 84, 128)
    q_out, k_out = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    call(cache, s, q_out, k_out, 0)
    k_ring, v_ring = cache.read_block(0)
    again_q, again_k = torch.zeros_like(q_out), torch.zeros_like(k_out)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(cache, s, again_q, again_k, 0, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(again_q, q_out) and torch.equal(again_k, k_out)
    graph = torch.cuda.CUDAGraph()
    again_q.zero_()
    with torch.cuda.graph(graph):
        call(cache, s, again_q, again_k, 0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again_q, q_out)
    call(cache, s, s["q"], s["k"], 0)
    assert torch.equal(s["q"], q_out) and torch.equal(s["k"], k_out)
    k2, v2 = cache.read_block(0)
    assert torch.equal(k2, k_ring) and torch.equal(v2, v_ring)


def test_nan_and_infinity_stay_in_their_token_and_head():
    s = make(3, 64, (1, 4, 4), 2, "head", seed=3)
    s["q"][2, 1, 5] = float("nan")
    s["k"][7, 0, 9] = float("inf")
    s["v"][1, 1, 1] = float("nan")
    cache = api.Cache(2, 3, 16, 64)
    q_out, k_out = (torch.empty((16, 3, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    call(cache, s, q_out, k_out, 0)
    bad_q, bad_k = (torch.isnan(t.float()).any(-1).nonzero().tolist() for t in (q_out, k_out))
    assert bad_q == [[2, 1]] and bad_k == [[7, 0]]
    assert np.array_equal(to_bits(cache.read_block(0)[1]), to_bits(s["v"]))


def test_model_sized_row_scope():
    s = make(40, 128, (3, 30, 52), 2, seed=17)
    cache = api.Cache(2, 40, 4680, 128)
    q_out = torch.full((4680, 40, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    call(cache, s, q_out, None, 0)
    # fp64 on the device; the rotation as a complex product with the table
    pf, ph, pw = api.sdvg_rope3d_pairs(128)
    z = torch.view_as_complex(s["tab"].double().view(-1, 2))
    f, y, x = z[:3 * pf].view(3, pf), z[3 * pf:3 * pf + 30 * ph].view(30, ph), z[3 * pf + 30 * ph:].view(52, pw)
    turn = torch.cat([f[:, None, None].expand(3, 30, 52, pf), y[None, :, None].expand(3, 30, 52, ph),
                      x[None, None].expand(3, 30, 52, pw)], -1).reshape(4680, 1, 64)
    for src, w, got in ((s["q"], s["qw"], q_out), (s["k"], s["kw"], cache.read_block(0)[0])):
        v = src.double().reshape(4680, -1)
        v = (v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w.double()).view(4680, 40, 64, 2)
        ref = torch.view_as_real(torch.view_as_complex(v) * turn).reshape(4680, 40, 128)
        room = v.abs().sum(-1, keepdim=True).expand(-1, -1, -1, 2).reshape(ref.shape)
        # the fp32 arithmetic (a sum of 5120 squares, a root, four products) stays below 2^-16 of the pair
        assert bool(((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -15 * room).all())
    assert torch.equal(cache.read_block(0)[1], s["v"])


def test_binding_refuses_mismatched_tensors():
    s = make(2, 64, (1, 4, 4), 2)
    cache = api.Cache(2, 2, 16, 64)
    q_out = torch.empty((16, 2, 64), device="cuda", dtype=torch.bfloat16)
    for change in (dict(q=s["q"][:15]), dict(k=s["k"].half()), dict(qw=s["qw"][:64]), dict(kw=s["kw"].bfloat16()),
                   dict(v=s["v"].transpose(0, 1)), dict(q=s["q"].cpu())):
        with pytest.raises((ValueError, api.SdvgError)):
            call(cache, {**s, **change}, q_out, None, 0)
    with pytest.raises(ValueError):
        call(cache, s, torch.empty((16, 2, 128), device="cuda", dtype=torch.bfloat16)[..., :64], None, 0)
    assert cache.state()[2] == -1                  # nothing was staged


@pytest.mark.parametrize("heads,dim", [(80, 128), (81, 128), (96, 128), (128, 128), (160, 64), (161, 64), (255, 64), (256, 64)])
@pytest.mark.parametrize("scope,fused,weights", [("row", True, True), ("head", False, True), ("head", True, False)])
def test_parity_of_the_widest_tokens(heads, dim, scope, fused, weights):
    """Around 10240 elements, where a thread goes from two pieces to four, with whole and partly filled last warps, up to 16384."""
    grid = (2, 3, 5)
    s = make(heads, dim, grid, 3, scope, fused, weights, seed=heads)
    cache = api.Cache(3, heads, 30, dim)
    guard = Canaries()
    guard.watch_cache(cache)
    q_out, k_out = (guard.new((30, heads, dim), torch.bfloat16) for _ in range(2))
    assert call(cache, s, q_out, k_out, 0) == -1
    (q_ref, q_tol), (k_ref, k_tol) = expected(s, 0)
    assert_close(q_out, q_ref, q_tol, "q")
    assert_close(k_out, k_ref, k_tol, "k")
    ring_k, ring_v = cache.read_block(0)
    assert np.array_equal(to_bits(ring_k), to_bits(k_out)) and np.array_equal(to_bits(ring_v), to_bits(s["v"]))
    guard.check()


def test_more_tokens_than_teams_at_the_widest():
    """Every team walks several tokens, so that its ring wraps."""
    s = make(128, 128, (3, 20, 20), 2, seed=8)
    cache = api.Cache(2, 128, 1200, 128)
    q_out = torch.full((1200, 128, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    call(cache, s, q_out, None, 0)
    (q_ref, q_tol), (k_ref, k_tol) = expected(s, 0)
    assert_close(q_out, q_ref, q_tol, "q")
    assert_close(cache.read_block(0)[0], k_ref, k_tol, "k")
    assert torch.equal(cache.read_block(0)[1], s["v"])


@pytest.mark.parametrize("heads,dim", [(129, 128), (257, 64)])
def test_tokens_past_the_widest_are_refused(heads, dim):
    s = make(heads, dim, (1, 2, 2), 2, "head")
    cache = api.Cache(2, heads, 4, dim)
    with pytest.raises(api.SdvgError) as e:
        call(cache, s, torch.empty((4, heads, dim), device="cuda", dtype=torch.bfloat16), None, 0)
    assert e.value.status == api.SDVG_ERR_BAD_SHAPE and cache.state()[2] == -1
