"""The 8-bit operators on matrices and rings of more than 2^31 elements, and on single rows of any stride."""
import pytest
import torch

from paper_2604_17397_b200 import api
from test_gpu_linear_e4m3_pairs import OUTS, largest, operand, randn, values

pytestmark = pytest.mark.gpu

ROWS = [0, 1, 33333, 65535, 69998, 69999]


def coded(rows, cols, block_rows=1):
    return (torch.empty((rows, cols), device="cuda", dtype=torch.uint8),
            torch.empty((-(-rows // block_rows), -(-cols // 128)), device="cuda", dtype=torch.uint8))


def far(t, rows):
    """Far rows of a tensor."""
    return torch.stack([t[r] for r in rows])


@pytest.mark.parametrize("cols", [32768, 32761])
@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_outputs_of_a_product(cols, out):
    rows, inner = 70000, 400
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = operand(randn(gen, rows, inner), 1), operand(randn(gen, cols, inner, std=inner ** -0.5), 128)
    o = torch.empty((rows, cols), device="cuda", dtype=OUTS[out])
    scale = torch.empty((rows, -(-cols // 128)), device="cuda", dtype=torch.uint8) if out == "e4m3" else None
    ws = api.attn_workspace()
    api.sdvg_linear_e4m3(*x, *w, o, ws, act=api.SDVG_ACT_SILU, out_scale=scale)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    xv, wv = values(far(x[0], ROWS), far(x[1], ROWS), 1), values(*w, 128)
    v = xv @ wv.t()
    ref = v * torch.sigmoid(v)
    err = 1.13 * (inner + 2) * 2.0 ** -23 * (xv.abs() @ wv.abs().t()) + 2.0 ** -14 * ref.abs() + 1e-36
    got = far(o, ROWS)
    if out == "bf16":
        assert bool(((got.double() - ref).abs() <= err + (ref.abs() + err) * 2.0 ** -8).all())
    else:
        f = torch.exp2(far(scale, ROWS).double() - 127)
        assert bool((largest((ref.abs() - err).clamp(min=0)) <= 448 * f).all()) and bool((largest(ref.abs() + err) > 224 * f).all())
        each = f.repeat_interleave(128, 1)[:, :cols]
        got = got.view(torch.float8_e4m3fn).double() * each
        assert bool(((got - ref).abs() <= err + torch.maximum((ref.abs() + err) / 16, each / 1024)).all())


@pytest.mark.parametrize("rows,cols", [(70000, 32768), (70000, 32761)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantised_matrices(rows, cols, block_rows):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16)
    for i in range(0, rows, 10000):
        x[i:i + 10000] = randn(gen, min(10000, rows - i), cols)
    codes, scale = coded(rows, cols, block_rows)
    api.sdvg_quant_e4m3_blocks(x, codes, scale)
    small, small_scale = coded(256, cols, block_rows)
    first = 69632                                              # two whole tiles near the end
    api.sdvg_quant_e4m3_blocks(x[first:first + 256], small, small_scale)
    assert torch.equal(codes[first:first + 256], small)
    assert torch.equal(scale[first // block_rows:(first + 256) // block_rows], small_scale)
    back = torch.empty_like(x)
    api.sdvg_dequant_e4m3_blocks(codes, scale, back)
    want = torch.empty((256, cols), device="cuda", dtype=torch.bfloat16)
    api.sdvg_dequant_e4m3_blocks(small, small_scale, want)
    assert torch.equal(back[first:first + 256], want)
    assert bool(((back[-8:].double() - x[-8:].double()).abs() <= x[-8:].double().abs().amax() / 14).all())


@pytest.mark.parametrize("cols,rows", [(32768, 70000), (10240, 220000), (4099, 530000)])
def test_normed_rows(cols, rows):
    """Rows that no team holds, whole vectors, single columns."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16)
    for i in range(0, rows, 20000):
        x[i:i + 20000] = randn(gen, min(20000, rows - i), cols)
    codes, scale = coded(rows, cols)
    api.sdvg_gated_norm_e4m3(x, codes, scale, norm=api.SDVG_NORM_RMS)
    some, some_scale = coded(64, cols)
    api.sdvg_gated_norm_e4m3(x[-64:], some, some_scale, norm=api.SDVG_NORM_RMS)
    assert torch.equal(codes[-64:], some) and torch.equal(scale[-64:], some_scale)


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("scope", ["row", "head"])
def test_a_ring_of_many_slots(tiled, scope):
    """The last slot of a ring of 2.4e9 codes is written and read back as the only slot of a small one."""
    heads, grid, slots = 128, (3, 30, 52), 31
    t, c = 4680, 128 * 128
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (randn(gen, t, heads, 128).bfloat16() for _ in range(3))
    wide = c if scope == "row" else 128
    w = torch.rand(wide, generator=gen, device="cuda") + 0.5
    tab = api.sdvg_rope3d_table(128, 3 * slots, 30, 52).cuda()
    inv = torch.full((heads,), 40.0, device="cuda")
    kind = api.SDVG_SCOPE_ROW if scope == "row" else api.SDVG_SCOPE_HEAD
    space = api.qk_norm_workspace(t)
    got = []
    for n in (slots, 1):
        cache = api.Cache(n, heads, t, 128, e4m3=True, tile_scales=tiled)
        q8 = torch.empty((t, heads, 128), device="cuda", dtype=torch.uint8)
        q_scale = torch.empty((heads, cache.tiles), device="cuda") if tiled else None
        for b in range(n):
            last = b == n - 1
            args = (cache, q if last else None, k, v, w, w, kind, 1e-6, q8 if last else None)
            # the last block stands at the same place of both rings' tables
            pos = (grid, 3 * (slots - 1) if last else 0, tab, 3 * slots, b, api.SDVG_STAGE if last else api.SDVG_FINAL)
            if tiled:
                api.sdvg_qk_norm_rope3d_commit_e4m3_tiled(*args, q_scale if last else None, *pos, space)
            else:
                api.sdvg_qk_norm_rope3d_commit_e4m3(*args, inv if last else None, inv, inv, *pos)
        out = [torch.empty((t, heads, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        api.sdvg_cache_read_block_e4m3(cache, n - 1, *out, *(() if tiled else (1 / inv, 1 / inv)))
        got.append((q8, *out, *cache.read_block(n - 1)))
        cache.close()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_single_rows_of_any_stride(out):
    """The stride of a single row is not read: one of a matrix whose rows are an odd number of bytes apart."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    inner, cols = 300, 515
    x, w = operand(randn(gen, 1, inner), 1), operand(randn(gen, cols, inner), 128)
    row = lambda t, ld: torch.as_strided(t, t.shape, (ld, 1))
    ws, res = api.attn_workspace(), []
    for strange in (False, True):
        a = (row(x[0], 301), row(x[1], 1)) if strange else x
        o = torch.empty((1, cols), device="cuda", dtype=OUTS[out])
        sc = torch.empty((1, -(-cols // 128)), device="cuda", dtype=torch.uint8) if out == "e4m3" else None
        api.sdvg_linear_e4m3(*a, *w, row(o, 7) if strange else o, ws, out_scale=sc)
        res.append((o, sc))
    assert torch.equal(res[0][0], res[1][0]) and (out != "e4m3" or torch.equal(res[0][1], res[1][1]))
