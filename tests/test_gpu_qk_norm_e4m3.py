"""Norm, rotary and the quantising write into an 8-bit ring (static and tile scales), and the read-back, against fp64."""
import numpy as np
import pytest
import torch

from dense_utils import U, assert_close, f64, norm_error
from e4m3_utils import half_step_tiles
from gpu_utils import Canaries
from oracle import dense_oracle as D
from oracle import e4m3_blocks_oracle as B
from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api
from test_gpu_qk_norm import EPS, SCOPES, make

pytestmark = pytest.mark.gpu


def problem(heads, grid, slots, tiled, scope="row", fused=True, weights=True, seed=0, block=0, gain=None):
    s = make(heads, 128, grid, slots, scope, fused, weights, seed, block)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    if gain is not None:                                       # heads and stretches of tokens of different magnitude
        t = s["v"].shape[0]
        f = torch.exp2(torch.randint(-gain, gain, (t // 50 + 1, heads, 1), generator=gen, device="cuda").float())
        s["v"].mul_(f.repeat_interleave(50, 0)[:t].bfloat16())
        for w in (s["qw"], s["kw"]):
            w.mul_(torch.exp2(torch.randint(-gain, gain, w.shape, generator=gen, device="cuda").float()))
    s["tiled"] = tiled
    if not tiled:
        # sized for 5 to 20: some values saturate
        s["inv"] = [448 / (5 + 15 * torch.rand(heads, generator=gen, device="cuda")) for _ in range(3)]
    return s


def ring(s, slots):
    t, heads = s["k"].shape[:2]
    return api.Cache(slots, heads, t, 128, e4m3=True, tile_scales=s["tiled"])


def call(cache, s, q8, q_scale=None, block=0, flags=api.SDVG_STAGE, q=True, stream=None, workspace=None):
    args = (cache, s["q"] if q else None, s["k"], s["v"], s["qw"], s["kw"], SCOPES[s["scope"]], EPS, q8 if q else None)
    pos = (s["grid"], block * s["grid"][0], s["tab"], s["tab_frames"], block, flags)
    if s["tiled"]:
        if workspace is None and s["scope"] == "row":
            workspace = s.setdefault("space", api.qk_norm_workspace(s["k"].shape[0]))
        return api.sdvg_qk_norm_rope3d_commit_e4m3_tiled(*args, q_scale if q else None, *pos, workspace, stream=stream)
    return api.sdvg_qk_norm_rope3d_commit_e4m3(*args, s["inv"][0] if q else None, *s["inv"][1:], *pos, stream=stream)


def expected(s, block):
    """[(value, bound)] of q, k, v before they are quantised."""
    got = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x, w = f64(x), f64(w)
        ref = D.qk_norm_rope_ref(x, w, s["scope"], EPS, s["grid"], block * s["grid"][0], s["tab"].cpu().numpy(), s["tab_frames"])
        flat = x.reshape(x.shape[0], -1) if s["scope"] == "row" else x
        o, e = norm_error(flat, np.zeros_like(flat), "rms", EPS)
        f = 1.0 if w is None else np.abs(w)
        e, o = ((e + 4 * U * np.abs(o)) * f).reshape(x.shape), (np.abs(o) * f).reshape(x.shape)
        pair = lambda a: np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1)         # |cos|, |sin| <= 1
        got.append((ref, pair(e) + 4 * U * pair(o)))
    v = f64(s["v"])
    return got + [(v, np.zeros_like(v))]


def check_static(codes, ref, err, inv):
    inv = f64(inv)[None, :, None]
    want, err = ref * inv, err * inv + U * np.abs(ref * inv)
    tol = np.minimum(err + B.half_step(np.abs(want) + err, 1.0), np.abs(want) + 448)
    clipped = np.clip(want, -448, 448)
    assert_close(O.e4m3_decode(codes.cpu().numpy()), clipped, np.broadcast_to(tol, clipped.shape))


def scales_of(cache, slot):
    return cache.k_scale[:, slot].cpu().numpy(), cache.v_scale[:, slot].cpu().numpy()


def check_slot(cache, s, slot, refs):
    codes = cache.read_block(slot)
    if s["tiled"]:
        for c, sc, (ref, err) in zip(codes, scales_of(cache, slot), refs[1:]):
            half_step_tiles(c, sc, ref, err)
    else:
        for c, (ref, err), inv in zip(codes, refs[1:], s["inv"][1:]):
            check_static(c, ref, err, inv)


GRIDS = [(1, 1, 1), (2, 4, 8), (1, 8, 16), (1, 7, 23), (3, 5, 11), (3, 10, 13)]


@pytest.mark.parametrize("grid", GRIDS)
@pytest.mark.parametrize("heads", [1, 2, 3, 12, 40, 81])
@pytest.mark.parametrize("scope,fused,weights", [("row", True, True), ("head", False, True), ("row", False, False), ("head", True, False)])
@pytest.mark.parametrize("tiled", [False, True])
def test_parity(grid, heads, scope, fused, weights, tiled):
    s = problem(heads, grid, 3, tiled, scope, fused, weights, seed=heads)
    t = s["q"].shape[0]
    cache, guard = ring(s, 3), Canaries()
    guard.watch_cache(cache)
    q8 = guard.new((t, heads, 128), torch.uint8)
    q_scale = guard.new((heads, -(-t // 128)), torch.float32) if tiled else None
    assert call(cache, s, q8, q_scale) == -1
    refs = expected(s, 0)
    if tiled:
        half_step_tiles(q8, q_scale.cpu().numpy(), *refs[0])
        assert bool((cache.k_scale[:, 1:] == 1).all()) and bool((cache.v_scale[:, 1:] == 1).all())
    else:
        check_static(q8, *refs[0], s["inv"][0])
    check_slot(cache, s, 0, refs)
    guard.check()
    assert cache.state() == (0, [-1, -1, -1], 0)


@pytest.mark.parametrize("scope", ["row", "head"])
def test_tiles_of_different_magnitude(scope):
    s = problem(5, (2, 13, 17), 2, True, scope, seed=3, gain=20)
    cache = ring(s, 2)
    q8, q_scale = torch.empty(s["q"].shape, device="cuda", dtype=torch.uint8), torch.empty((5, cache.tiles), device="cuda")
    call(cache, s, q8, q_scale)
    refs = expected(s, 0)
    half_step_tiles(q8, q_scale.cpu().numpy(), *refs[0])
    check_slot(cache, s, 0, refs)


@pytest.mark.parametrize("tiled", [False, True])
def test_equal_to_the_quantiser_where_nothing_is_normed(tiled):
    """v is quantised as the commit without a norm does it, bit for bit, also infinities, NaN and a block of zeros."""
    s = problem(3, (1, 20, 15), 2, tiled, fused=False, seed=5)
    v = s["v"]
    v[3, 0, 5], v[200, 1, 6], v[130:200, 2] = float("nan"), float("inf"), 0
    v[128:256, 0] = 0
    cache, other = ring(s, 2), ring(s, 2)
    call(cache, s, None, q=False)
    if tiled:
        api.sdvg_kv_commit_e4m3_tiled(other, s["k"].contiguous(), v, 0, api.SDVG_STAGE)
        assert torch.equal(cache.v_scale[:, 0], other.v_scale[:, 0])
    else:
        api.sdvg_kv_commit_e4m3(other, s["k"].contiguous(), v, *s["inv"][1:], 0, api.SDVG_STAGE)
    assert torch.equal(cache.read_block(0)[1] & 0x7F, other.read_block(0)[1] & 0x7F)


@pytest.mark.parametrize("tiled", [False, True])
def test_ring_order_eviction_and_untouched_slots(tiled):
    grid, slots = (1, 3, 50), 2
    held, cache = {}, None
    for b in range(5):
        s = problem(2, grid, slots, tiled, seed=b, block=b)
        cache = cache or ring(s, slots)
        call(cache, s, None, block=b, q=False)
        if b:
            for got, was in zip(cache.read_block((b - 1) % slots), held[b - 1]):
                assert torch.equal(got, was)
        assert call(cache, s, None, block=b, flags=api.SDVG_FINAL, q=False) == (b - slots if b >= slots else -1)
        held[b] = cache.read_block(b % slots)
        check_slot(cache, s, b % slots, expected(s, b))
    with pytest.raises(api.SdvgError) as e:
        call(cache, problem(2, grid, slots, tiled, block=7), None, block=7, q=False)
    assert e.value.status == api.SDVG_ERR_BAD_STATE


@pytest.mark.parametrize("scope", ["row", "head"])
@pytest.mark.parametrize("tiled", [False, True])
def test_streams_graphs_and_equal_bits(scope, tiled):
    s = problem(12, (2, 11, 13), 3, tiled, scope, seed=11)
    cache = ring(s, 3)
    new = lambda: (torch.zeros(s["q"].shape, device="cuda", dtype=torch.uint8),
                   torch.zeros((12, cache.tiles), device="cuda") if tiled else None)
    first, second, third = new(), new(), new()
    call(cache, s, *first)
    held = [t.clone() for t in cache.read_block(0)]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(cache, s, *second, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(cache, s, *third)
    keep = s["k"].clone()
    s["k"].copy_(torch.flip(keep, (0,)))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(cache.read_block(0)[0], held[0])
    s["k"].copy_(keep)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for other in (second, third):
        assert torch.equal(other[0], first[0]) and (not tiled or torch.equal(other[1], first[1]))
    assert all(torch.equal(a, b) for a, b in zip(cache.read_block(0), held))


def test_the_whole_block_of_the_target():
    """40 heads, 4680 tokens: sampled heads against fp64, and the per-token norm under every head group of a tile."""
    s = problem(40, (3, 30, 52), 2, True, seed=13)
    cache = ring(s, 2)
    q8, q_scale = torch.empty(s["q"].shape, device="cuda", dtype=torch.uint8), torch.empty((40, cache.tiles), device="cuda")
    for _ in range(3):
        call(cache, s, q8, q_scale)
    refs = expected(s, 0)
    for h in (0, 9, 10, 21, 39):
        one = slice(h, h + 1)
        half_step_tiles(q8[:, one], q_scale[one].cpu().numpy(), *(a[:, one] for a in refs[0]))
        for c, sc, ref in zip(cache.read_block(0), scales_of(cache, 0), refs[1:]):
            half_step_tiles(c[:, one], sc[one], *(a[:, one] for a in ref))


def test_more_tiles_than_sms():
    s = problem(2, (5, 64, 80), 1, True, seed=17)
    cache = ring(s, 1)
    q8, q_scale = torch.empty(s["q"].shape, device="cuda", dtype=torch.uint8), torch.empty((2, cache.tiles), device="cuda")
    call(cache, s, q8, q_scale)
    refs = expected(s, 0)
    half_step_tiles(q8, q_scale.cpu().numpy(), *refs[0])
    check_slot(cache, s, 0, refs)


# ---- reading back ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,tokens,slots,slot", [(1, 1, 1, 0), (3, 127, 2, 1), (2, 129, 3, 2), (12, 1000, 2, 0), (40, 4680, 2, 1)])
@pytest.mark.parametrize("tiled", [False, True])
def test_read_back(heads, tokens, slots, slot, tiled):
    cache = api.Cache(slots, heads, tokens, 128, e4m3=True, tile_scales=tiled)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    for raw in (cache._k_raw, cache._v_raw):
        raw.copy_(torch.randint(0, 256, raw.shape, generator=gen, device="cuda", dtype=torch.uint8))      # NaN codes among them
    if tiled:
        for sc in (cache.k_scale, cache.v_scale):
            sc.copy_(torch.exp2(torch.randint(-126, 100, sc.shape, generator=gen, device="cuda").float()))
        scales = [sc[:, slot].repeat_interleave(128, 1)[:, :tokens].T[:, :, None].cpu().numpy() for sc in (cache.k_scale, cache.v_scale)]
        given = ()
    else:
        given = tuple(torch.rand(heads, generator=gen, device="cuda") * 3 for _ in range(2))
        scales = [g.cpu().numpy()[None, :, None] for g in given]
    guard = Canaries()
    outs = [guard.new((tokens, heads, 128), torch.bfloat16) for _ in range(2)]
    api.sdvg_cache_read_block_e4m3(cache, slot, *outs, *given)
    guard.check()
    for codes, f, got in zip(cache.read_block(slot), scales, outs):
        # the product in fp32 and its rounding to bf16
        want = torch.from_numpy(O.e4m3_decode(codes.cpu().numpy()).astype(np.float32) * f.astype(np.float32)).bfloat16()
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    one = guard.new((tokens, heads, 128), torch.bfloat16)
    api.sdvg_cache_read_block_e4m3(cache, slot, None, one, *((None, given[1]) if given else ()))
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(one), torch.nan_to_num(outs[1]))


@pytest.mark.parametrize("tiled", [False, True])
def test_what_was_written_is_read_back(tiled):
    s = problem(6, (2, 9, 16), 2, tiled, "head", seed=19)
    cache = ring(s, 2)
    if not tiled:
        s["inv"] = [torch.full((6,), 16.0, device="cuda")] * 3
    call(cache, s, None, q=False)
    k, v = (torch.empty(s["k"].shape, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    given = () if tiled else (1 / s["inv"][1], 1 / s["inv"][2])
    api.sdvg_cache_read_block_e4m3(cache, 0, k, v, *given)
    for got, (ref, _) in zip((k, v), expected(s, 0)[1:]):
        assert np.linalg.norm(f64(got) - ref) <= (2 ** -4 + 2 ** -8) * np.linalg.norm(ref)
