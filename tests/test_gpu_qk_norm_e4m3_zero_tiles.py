"""The tile-scaled ring write where a tile's values vanish or are tiny: scales at the low end, against fp64 and the quantiser's rule."""
import numpy as np
import pytest
import torch

from e4m3_utils import half_step_tiles
from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api
from test_gpu_qk_norm_e4m3 import call, check_slot, expected, problem, ring, scales_of

pytestmark = pytest.mark.gpu

LOWEST = 2.0 ** O.E4M3_SCALE_EXP_MIN


def written(s, slots=1):
    """(codes, scales [heads, tiles]) of q, k and v, and the cache."""
    cache = ring(s, slots)
    q8 = torch.full(s["q"].shape, 0x55, device="cuda", dtype=torch.uint8)
    q_scale = torch.full((s["q"].shape[1], cache.tiles), 3.0, device="cuda")
    call(cache, s, q8, q_scale)
    k8, v8 = cache.read_block(0)
    return [(q8, q_scale.cpu().numpy()), *zip((k8, v8), scales_of(cache, 0))], cache


def check(s):
    got, cache = written(s)
    refs = expected(s, 0)
    half_step_tiles(*got[0], *refs[0])
    check_slot(cache, s, 0, refs)
    return got


def assert_zeros(codes, scales, heads, first, last):
    """Tokens first .. last of these heads, whole tiles or what there is of them."""
    assert bool((codes[first:last, heads] & 0x7F == 0).all())
    assert (scales[heads, first // 128:-(-last // 128)] == LOWEST).all()


# one token; a tile that is not full; whole tiles and a rest
@pytest.mark.parametrize("grid", [(1, 1, 1), (1, 5, 9), (2, 8, 16), (1, 20, 15)])
@pytest.mark.parametrize("scope", ["row", "head"])
@pytest.mark.parametrize("weights", [True, False])
def test_a_block_of_zeros(grid, scope, weights):
    s = problem(3, grid, 1, True, scope, fused=False, weights=weights, seed=1)
    for what in "qkv":
        s[what].zero_()
    for codes, scales in check(s):
        assert_zeros(codes, scales, slice(0, 3), 0, codes.shape[0])


@pytest.mark.parametrize("size", [1.0, 2.0 ** -3, 2.0 ** -7, 2.0 ** -14])
@pytest.mark.parametrize("tile", [0, 1, 2])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_a_tile_of_one_head(scope, tile, size):
    """The other heads of its tokens are not zero: their rms sets the factor of a norm over the token."""
    s = problem(3, (1, 20, 15), 1, True, scope, seed=2)
    first, last = 128 * tile, min(128 * tile + 128, 300)
    for what in "qkv":
        s[what].mul_(size)
        s[what][first:last, 1] = 0
    for codes, scales in check(s):
        assert_zeros(codes, scales, slice(1, 2), first, last)
        assert (scales[[0, 2]] > LOWEST).all()


@pytest.mark.parametrize("size", [1.0, 2.0 ** -7])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_weights_of_zero(scope, size):
    s = problem(3, (1, 11, 13), 1, True, scope, seed=3)
    heads = slice(1, 2) if scope == "row" else slice(0, 3)
    for what in ("qw", "kw"):
        s[what].view(-1, 128)[heads if scope == "row" else slice(None)] = 0
    for what in "qkv":
        s[what].mul_(size)
    got = check(s)
    for codes, scales in got[:2]:
        assert_zeros(codes, scales, heads, 0, 143)


@pytest.mark.parametrize("scope", ["row", "head"])
def test_a_zero_row_next_to_others(scope):
    """Rows of zeros whose tile has a scale of its own, next to tiny and ordinary rows."""
    s = problem(2, (1, 10, 13), 1, True, scope, seed=4)
    for what in "qk":
        s[what][5] = 0
        s[what][6:9] *= 2.0 ** -20
        s[what][129] = 0
    for codes, _ in check(s)[:2]:
        assert bool((codes[[5, 129]] & 0x7F == 0).all())


# powers of two in the weights scale every step exactly, as long as nothing leaves fp32's normal range: equal codes
@pytest.mark.parametrize("size", [2.0 ** -7, 1.0, 2.0 ** 10])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_scales_move_with_the_weights(scope, size):
    s = problem(3, (1, 20, 15), 1, True, scope, weights=True, seed=5)
    for what in "qk":
        s[what].mul_(size)
    s["qw"], s["kw"] = torch.ones_like(s["qw"]), torch.ones_like(s["kw"])
    base = check(s)
    for power in (-104, -70, -50, -49, -48, -47, -46, -45, -44, -20, 30, 55, 70, 100):
        s["qw"].fill_(2.0 ** power)
        s["kw"].fill_(2.0 ** power)
        got = check(s)
        for (codes, scales), (was, was_scales) in zip(got[:2], base):
            assert torch.equal(codes, was), power
            assert (scales == was_scales * 2.0 ** power).all()


@pytest.mark.parametrize("power", [-112, -116, -118, -120, -124, -126, -130, -140])
@pytest.mark.parametrize("size", [2.0 ** -7, 1.0])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_values_near_the_lowest_scale(scope, size, power):
    """The scale stops at 2^-126; below, values turn subnormal in fp32 and vanish in the codes."""
    s = problem(2, (1, 12, 13), 1, True, scope, seed=6)
    for what in "qk":
        s[what].mul_(size)
    s["qw"].fill_(2.0 ** power)
    s["kw"].fill_(2.0 ** power)
    got, _ = written(s)
    for (codes, scales), (ref, err) in zip(got[:2], expected(s, 0)):
        # a product or a sum that is subnormal is off by up to half of 2^-149, times a factor of at most 1000 if before the norm's;
        # three of them make a value
        half_step_tiles(codes, scales, ref, err + 3 * 1000 * 2.0 ** -150)


def test_equal_to_the_quantiser_with_signs():
    """v, which no norm changes, as the commit without a norm writes it: whole bytes, but for the sign of NaN."""
    s = problem(3, (1, 20, 15), 1, True, fused=False, seed=7)
    v = s["v"]
    v[3, 0, 5], v[200, 1, 6], v[201, 1, 7], v[130:200, 2] = float("nan"), float("inf"), -float("inf"), 0
    v[128:256, 0] = 0
    cache, other = ring(s, 1), ring(s, 1)
    call(cache, s, None, q=False)
    api.sdvg_kv_commit_e4m3_tiled(other, s["k"].contiguous(), v, 0, api.SDVG_STAGE)
    assert torch.equal(cache.v_scale, other.v_scale)
    a, b = (c.read_block(0)[1] for c in (cache, other))
    nan = a & 0x7F == 0x7F
    assert torch.equal(nan, b & 0x7F == 0x7F) and torch.equal(a[~nan], b[~nan])
    assert int((a[~nan] >= 0x80).sum()) > 1000


def test_static_codes_equal_the_quantisers_with_signs():
    s = problem(3, (1, 20, 15), 1, False, fused=False, seed=8)
    v = s["v"]
    v[3, 0, 5], v[200, 1, 6], v[201, 1, 7], v[130:200, 2] = float("nan"), float("inf"), -float("inf"), 0
    cache, other = ring(s, 1), ring(s, 1)
    call(cache, s, None, q=False)
    api.sdvg_kv_commit_e4m3(other, s["k"].contiguous(), v, *s["inv"][1:], 0, api.SDVG_STAGE)
    a, b = (c.read_block(0)[1] for c in (cache, other))
    nan = a & 0x7F == 0x7F
    assert torch.equal(nan, b & 0x7F == 0x7F) and torch.equal(a[~nan], b[~nan])


@pytest.mark.parametrize("scope", ["row", "head"])
def test_attention_over_a_block_with_zero_keys(scope):
    """What the codes are for: a head whose keys of a tile are zero attends to them like to any others."""
    t, heads = 300, 3
    s = problem(heads, (1, 20, 15), 1, True, scope, seed=9)
    for what in "qk":
        s[what].mul_(2.0 ** -5)
    s["k"][128:256, 1] = 0
    got, cache = written(s)
    out = torch.empty((t, heads, 128), device="cuda", dtype=torch.bfloat16)
    (q8, q_scale), (k8, ks), (v8, vs) = got
    ws = api.attn_workspace()
    api.sdvg_block_attn_fwd_e4m3_tiled(q8, torch.from_numpy(q_scale).cuda(), cache, 0, out, None, 128 ** -0.5, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    tiles = np.arange(t) // 128
    q, k, v = (O.e4m3_decode(c.cpu().numpy()) * f.T[tiles][..., None] for c, f in ((q8, q_scale), (k8, ks), (v8, vs)))
    for h in range(heads):
        z = q[:, h] @ k[:, h].T * 128 ** -0.5
        e = np.exp(z - z.max(1, keepdims=True))
        total = e.sum(1, keepdims=True)
        want = e / total @ v[:, h]
        # the exponentials, of which the largest is at least 1, are rounded to 8 bits: 2^-4 of each or 2^-10; the result to bf16
        tol = (2.0 ** -4 + t * 2.0 ** -10 / total + 2.0 ** -8) * np.abs(v[:, h]).max()
        assert (np.abs(out[:, h].double().cpu().numpy() - want) <= tol).all()
