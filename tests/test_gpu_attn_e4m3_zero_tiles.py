"""The attention over a ring with tile scales where tiles of q, k or v are zero or tiny: scales down to 2^-126 multiply to less than
fp32 holds, and keys past the last token must stay masked all the same."""
import numpy as np
import pytest
import torch

from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api

pytestmark = pytest.mark.gpu

HEADS = 3


def attend(q, k, v, blocks=1):
    """q, k, v bf16 [tokens, heads, 128]: committed as `blocks` equal blocks, the last of them the staged one; (out, reference, bound)."""
    t = q.shape[0]
    cache, ws = api.Cache(blocks, HEADS, t, 128, e4m3=True, tile_scales=True), api.attn_workspace()
    for b in range(blocks):
        api.sdvg_kv_commit_e4m3_tiled(cache, k, v, b, api.SDVG_STAGE if b == blocks - 1 else api.SDVG_FINAL)
    q8 = torch.empty(q.shape, device="cuda", dtype=torch.uint8)
    qs = torch.empty((HEADS, cache.tiles), device="cuda")
    api.sdvg_quant_e4m3_tiled(q, q8, qs)
    out = torch.full(q.shape, float("nan"), device="cuda", dtype=torch.bfloat16)
    api.sdvg_block_attn_fwd_e4m3_tiled(q8, qs, cache, blocks - 1, out, None, 128 ** -0.5, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    (k8, v8), tile = cache.read_block(0), np.arange(t) // 128
    value = lambda c, f: O.e4m3_decode(c.cpu().numpy()) * f.cpu().numpy().astype(np.float64).T[tile][..., None]
    qv, kv, vv = value(q8, qs), value(k8, cache.k_scale[:, 0]), value(v8, cache.v_scale[:, 0])
    ref, tol = np.empty(qv.shape), np.empty(qv.shape)
    for h in range(HEADS):
        z = qv[:, h] @ kv[:, h].T * 128 ** -0.5
        e = np.exp(z - z.max(1, keepdims=True))
        total = e.sum(1, keepdims=True)
        ref[:, h] = e / total @ vv[:, h]
        # the exponentials, of which the largest is at least 1, are rounded to 8 bits: 2^-4 of each or 2^-10; the result to bf16.  Equal
        # blocks double both sums
        tol[:, h] = (2.0 ** -4 + t * 2.0 ** -10 / total + 2.0 ** -8) * np.abs(vv[:, h]).max()
    return out.double().cpu().numpy(), ref, tol


def tensors(t, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((t, HEADS, 128), generator=gen, device="cuda").bfloat16() for _ in range(3)]


@pytest.mark.parametrize("tokens", [1, 100, 128, 300, 513])
@pytest.mark.parametrize("blocks", [1, 3])
@pytest.mark.parametrize("zeros", ["q", "k", "v", "qk", "qkv"])
def test_zeros(tokens, blocks, zeros):
    given = dict(zip("qkv", tensors(tokens, tokens)))
    for what in zeros:
        given[what].zero_()
    out, ref, tol = attend(**given, blocks=blocks)
    assert (np.abs(out - ref) <= tol + 2.0 ** -133).all()


@pytest.mark.parametrize("tokens", [300, 513])
@pytest.mark.parametrize("zeros", ["q", "k", "v", "qk", "kv", "qkv"])
@pytest.mark.parametrize("tile", [0, 1, -1])
def test_a_tile_of_zeros(tokens, zeros, tile):
    given = dict(zip("qkv", tensors(tokens, tokens)))
    tiles = -(-tokens // 128)
    first = 128 * (tile % tiles)
    for what in zeros:
        given[what][first:first + 128, 1] = 0
    out, ref, tol = attend(**given)
    assert (np.abs(out - ref) <= tol).all()


@pytest.mark.parametrize("power", [-100, -70, -40])
@pytest.mark.parametrize("tiny", ["q", "k", "qk"])
def test_tiny_values(tiny, power):
    given = dict(zip("qkv", tensors(300, 1)))
    for what in tiny:
        given[what].mul_(2.0 ** power)
    out, ref, tol = attend(**given)
    assert (np.abs(out - ref) <= tol).all()
