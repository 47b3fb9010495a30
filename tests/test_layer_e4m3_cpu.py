"""Host glue of the 8-bit layer with the library's calls replaced by a record; no GPU."""
import types

import pytest
import torch

from paper_2604_17397_b200 import api, schedule
from test_layer_cpu import GRID, lib  # noqa: F401 (the fixture builds the library)

TOKENS = 12


def model(name, heads, dim, e4m3=False, tiled=False):
    cache = types.SimpleNamespace(name=name, heads=heads, head_dim=dim, block_tokens=TOKENS, slots=3, e4m3=e4m3, tile_scales=tiled, tiles=1)
    kw = {} if not e4m3 or tiled else {k: torch.ones(heads) for k in ("q_inv_scale", "k_inv_scale", "v_inv_scale")}
    return schedule.ModelState(cache, GRID, torch.zeros(8), 16, 1.0, torch.zeros(256, dtype=torch.uint8), **kw)


@pytest.fixture
def record(monkeypatch):
    calls = []
    for name in ("sdvg_gated_norm", "sdvg_gated_norm_e4m3", "sdvg_quant_e4m3_blocks", "sdvg_linear_e4m3", "sdvg_linear",
                 "sdvg_qk_norm_rope3d_commit", "sdvg_qk_norm_rope3d_commit_e4m3", "sdvg_qk_norm_rope3d_commit_e4m3_tiled",
                 "sdvg_block_attn_fwd", "sdvg_block_attn_fwd_e4m3", "sdvg_block_attn_fwd_e4m3_tiled"):
        monkeypatch.setattr(api, name, lambda *a, _n=name[5:], **kw: calls.append((_n, a, kw)))
    return calls


def weights(width, **kw):
    mat = lambda n, k: torch.zeros((n, k), dtype=torch.bfloat16)
    return schedule.LayerWeights(mat(3 * width, width), mat(width, width), mat(4 * width, width), mat(width, 4 * width), **kw)


RING = {"bf16": ("qk_norm_rope3d_commit", "block_attn_fwd"), "static": ("qk_norm_rope3d_commit_e4m3", "block_attn_fwd_e4m3"),
        "tiled": ("qk_norm_rope3d_commit_e4m3_tiled", "block_attn_fwd_e4m3_tiled")}


@pytest.mark.parametrize("ring", list(RING))
@pytest.mark.parametrize("post", [False, True])
def test_calls_of_a_step_and_a_commit(record, ring, post):
    heads, dim = (3, 64) if ring == "bf16" else (2, 128)
    width = heads * dim
    vec = torch.ones(width) if post else None
    m = model("m", heads, dim, ring != "bf16", ring == "tiled")
    layer = schedule.TransformerLayerE4M3(weights(width, post_attn=vec, post_ff=vec), m)
    assert [c[0] for c in record] == ["quant_e4m3_blocks"] * 4
    # a product's rows of k begin with a scale's, whatever the width
    assert layer.w_qkv.scale.shape[0] == (3 * width if width % 128 else 3 * width // 128)
    assert layer.w_qkv.rows_from(width).scale.shape[0] == 2 * width // (1 if width % 128 else 128)
    record.clear()
    x, mod = torch.zeros((TOKENS, width), dtype=torch.bfloat16), torch.zeros((2, 6 * width))
    layer.step(x, mod, 0, x)
    norm, lin = "gated_norm_e4m3", "linear_e4m3"
    tail = [lin, "gated_norm"] if post else [lin]
    assert [c[0] for c in record] == [norm, lin, *RING[ring], norm, lin, norm, lin, *tail]
    hidden = [c for c in record if c[0] == lin][2]
    assert hidden[2]["out_scale"] is not None and hidden[1][4].dtype == torch.uint8
    record.clear()
    layer.commit(x, mod, 0)
    assert [c[0] for c in record] == [norm, lin, RING[ring][0]]
    assert record[1][1][4].shape == (TOKENS, 2 * width) and record[2][1][1] is None


def test_rows_of_a_scale_are_not_cut():
    m = schedule.E4M3Matrix(torch.zeros((300, 128), dtype=torch.uint8), torch.zeros((3, 1), dtype=torch.uint8))
    assert m.rows_from(0) is m and m.rows_from(128).codes.shape[0] == 172 and m.rows_from(256).scale.shape[0] == 1
    with pytest.raises(ValueError):
        m.rows_from(100)
