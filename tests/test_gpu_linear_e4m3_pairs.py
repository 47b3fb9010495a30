"""sdvg_linear_e4m3 by pairs of CTAs, with tiles of 256 and of 512 features, against 64 bits on the GPU.

Which kernel a size takes is an estimate's choice; tests/test_linear_e4m3_cut.py holds it to what is assumed here.
"""
import math

import pytest
import torch

from dense_utils import DTYPES, U
from paper_2604_17397_b200 import api, schedule, synth

pytestmark = pytest.mark.gpu

ACTS = {"none": api.SDVG_ACT_NONE, "silu": api.SDVG_ACT_SILU, "gelu_tanh": api.SDVG_ACT_GELU_TANH, "gelu": api.SDVG_ACT_GELU}
OUTS = {**DTYPES, "e4m3": torch.uint8}

# features of a tile -> (rows, cols, inner): whole vectors of every output type, and columns that are none
SIZES = {256: (777, 3008, 1200), 512: (289, 16144, 768)}
ODD = {256: (777, 3013, 1200), 512: (289, 16141, 768)}
# sums of few stages, whole or with a rest, up to the first that fill the ring twice
SHORT = {256: [(1889, 13888, 512), (1035, 11200, 513), (5793, 1155, 768), (5793, 1155, 780), (4756, 408, 1024)],
         512: [(2377, 10944, 384), (2377, 10944, 260), (596, 11696, 512), (781, 8902, 500), (5671, 1155, 640), (289, 16141, 700),
               (261, 15125, 896), (198, 19062, 1024), (198, 19062, 1030)]}
BLOCK = (4680, 5120, 5120)                                   # 512
LONG = [(777, 3008, 6400), (777, 3013, 7700)]                # 256: fp32 sums in chunks


def randn(gen, *shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda") * std


def matrix(rows, cols, ld, lead, fill):
    """uint8 [rows, cols] with row stride ld, `lead` bytes into a buffer of `fill`."""
    buf = torch.full((lead + rows * ld,), fill, device="cuda", dtype=torch.uint8)
    return buf[lead:].view(rows, ld)[:, :cols]


# row strides and first addresses of the scales: whole vectors of 16 bytes, or words only
LAYOUTS = {"vectors": (16, 0), "stride": (4, 0), "address": (16, 4)}


def operand(v, block_rows, layout="vectors", more=0):
    """Codes and scales of v; what lies between the rows is NaN."""
    rows, cols = v.shape
    pad, lead = LAYOUTS[layout]
    blocks = -(-cols // 128)
    ld = -(-blocks // pad) * pad
    if pad == 4 and ld % 16 == 0:
        ld += 4
    codes = matrix(rows, cols, -(-cols // 16) * 16 + 16 * more, 0, 0x7F)
    scale = matrix(-(-rows // block_rows), blocks, ld, lead, 255)
    api.sdvg_quant_e4m3_blocks(v, codes, scale)
    return codes, scale


def make(size, out="bf16", act="none", bias=True, gate_rows=0, residual="", seed=0, w_rows=128, spread=6.0, layout="vectors", more=0):
    rows, cols, inner = size
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sized = lambda n: torch.exp2(spread * torch.rand((n, -(-inner // 128)), generator=gen, device="cuda") - spread / 2
                                 ).repeat_interleave(128, 1)[:, :inner]
    x = randn(gen, rows, inner) * sized(rows)
    w = randn(gen, cols, inner, std=1 / math.sqrt(inner)) * (sized(cols) if w_rows == 1 else sized(-(-cols // 128)).repeat_interleave(128, 0)[:cols])
    s = dict(x=operand(x, 1, layout, more), w=operand(w, w_rows, layout, more), act=act, gate_rows=gate_rows, out=out, w_rows=w_rows)
    s["bias"] = randn(gen, cols) if bias else None
    s["gate"] = randn(gen, -(-rows // gate_rows), cols) if gate_rows else None
    s["residual"] = randn(gen, rows if residual == "rows" else 1, cols, std=2.0).to(OUTS[out]).expand(rows, cols) if residual else None
    return s


def call(s, out, ws, out_scale=None, stream=None):
    api.sdvg_linear_e4m3(*s["x"], *s["w"], out, ws, bias=s["bias"], act=ACTS[s["act"]], residual=s["residual"], gate=s["gate"],
                         gate_rows=s["gate_rows"], out_scale=out_scale, stream=stream)


def values(codes, scale, block_rows):
    """In 64 bits; the scale byte 255 is NaN."""
    rows, cols = codes.shape
    f = torch.exp2(scale.double() - 127).masked_fill_(scale == 255, float("nan"))
    return codes.contiguous().view(torch.float8_e4m3fn).double() * f.repeat_interleave(128, 1)[:, :cols].repeat_interleave(block_rows, 0)[:rows]


def activation(v, act):
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu_tanh":
        return v * torch.sigmoid(math.sqrt(8 / math.pi) * (v + 0.044715 * v ** 3))
    return v * torch.special.erfc(-v / math.sqrt(2)) / 2 if act == "gelu" else v


def expected(s):
    """(reference, bound) before the rounding to the output's type: linear_tolerance in torch."""
    x, w = values(*s["x"], 1), values(*s["w"], s["w_rows"])
    b = 0.0 if s["bias"] is None else s["bias"].double()
    v = x @ w.t() + b
    err = (x.shape[1] + 2) * 2 * U * (x.abs() @ w.abs().t() + abs(b))
    a = activation(v, s["act"])
    if s["act"] != "none":
        err = 1.13 * err + 2.0 ** -14 * a.abs() + 1e-36
    g = torch.ones_like(a[:1]) if s["gate"] is None else s["gate"].double().repeat_interleave(s["gate_rows"], 0)[:x.shape[0]]
    r = torch.zeros_like(a[:1]) if s["residual"] is None else s["residual"].double()
    return g * a + r, g.abs() * err + 4 * U * ((g * a).abs() + r.abs())


def largest(a):
    """Per row and 128 columns; NaN left out."""
    return torch.nn.functional.pad(a.nan_to_num(0.0, math.inf, math.inf), (0, -a.shape[1] % 128)).unflatten(1, (-1, 128)).amax(2)


def assert_within(got, ref, tol):
    assert torch.equal(got.isnan(), ref.isnan())
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf])
    fine = ~(inf | ref.isnan())
    assert bool(((got - ref).abs() <= tol)[fine].all()), float(((got - ref).abs() - tol)[fine].max())


def check(s, more=0, in_place=False):
    """The call, its outputs and what lies around them; returns outputs (and scales)."""
    rows, cols = s["x"][0].shape[0], s["w"][0].shape[0]
    ws, dtype = api.attn_workspace(), OUTS[s["out"]]
    ref, err = expected(s)
    buf = torch.full((rows + 2, cols + more), 77, device="cuda", dtype=dtype)
    out = buf[1:-1, :cols]
    scale = None
    if s["out"] == "e4m3":
        blocks = -(-cols // 128)
        sbuf = torch.full((rows + 2, blocks + 1), 33, device="cuda", dtype=torch.uint8)
        scale = sbuf[1:-1, :-1]
    if in_place:
        out.copy_(s["residual"])
        s["residual"] = out
    call(s, out, ws, scale)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    if s["out"] == "e4m3":
        f = torch.exp2(scale.double() - 127)
        # the smallest power of two for a largest magnitude that is known up to err; 2^-126 is the least, 2^120 the greatest
        assert bool(((largest((ref.abs() - err).clamp(min=0)) <= 448 * f) | (scale == 247)).all())
        assert bool(((largest(ref.abs() + err) > 224 * f) | (scale == 1)).all())
        each = f.repeat_interleave(128, 1)[:, :cols]
        got, top = out.contiguous().view(torch.float8_e4m3fn).double() * each, 448 * each
        assert_within(got, torch.where(ref.isnan(), ref, ref.clamp(-top, top)), err + torch.maximum((ref.abs() + err) / 16, each / 1024))
        assert bool((sbuf[0] == 33).all()) and bool((sbuf[-1] == 33).all()) and bool((sbuf[:, -1] == 33).all())
    else:
        assert_within(out.double(), ref, err + (ref.abs() + err) * torch.finfo(dtype).eps / 2 + {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25, "fp32": 2.0 ** -126}[s["out"]])
    assert bool((buf[0] == 77).all()) and bool((buf[-1] == 77).all()) and bool((buf[:, cols:] == 77).all())
    return out, scale


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("sizes", [SIZES, ODD], ids=["vectors", "odd"])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("out", list(OUTS))
def test_activations(tile, sizes, act, out):
    rows = sizes[tile][0]
    check(make(sizes[tile], out, act, gate_rows=-(-rows // 3), residual="" if out == "e4m3" else "broadcast", seed=tile))


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("sizes,more", [(SIZES, 0), (SIZES, 16), (ODD, 0)], ids=["vectors", "wide", "odd"])
@pytest.mark.parametrize("gate_rows", [0, 1, 7, 100])
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
def test_residuals_and_gates(tile, sizes, more, gate_rows, out):
    """Gates that change within a block of tokens; the residual apart, and the outputs over it."""
    for residual, in_place in (("rows", False), ("rows", True), ("broadcast", False)):
        check(make(sizes[tile], out, "silu", gate_rows=gate_rows, residual=residual, seed=tile + gate_rows), more, in_place)


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("gate_rows", [1, 7, 100])
@pytest.mark.parametrize("sizes,more", [(SIZES, 0), (SIZES, 16), (ODD, 3)], ids=["vectors", "wide", "odd"])
def test_gates_of_8_bit_rows(tile, gate_rows, sizes, more):
    check(make(sizes[tile], "e4m3", "gelu_tanh", gate_rows=gate_rows, seed=tile + gate_rows), more)


def test_a_block_onto_its_stream():
    s = make(BLOCK, "fp32", gate_rows=1560, residual="rows", seed=1)
    check(s)
    check(s, in_place=True)
    check(make(BLOCK, "bf16", "gelu", gate_rows=1560, residual="rows", seed=2), in_place=True)


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("w_rows", [1, 128])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("out", ["fp32", "e4m3"])
def test_scales_and_strides(tile, w_rows, layout, out):
    """Scales per row of the weights, scale rows that cannot be read 16 bytes at a time, rows of codes further apart."""
    for sizes in (SIZES, ODD):
        check(make(sizes[tile], out, w_rows=w_rows, layout=layout, spread=20.0 if w_rows == 1 else 6.0, more=w_rows % 2, seed=3))


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
def test_few_stages(tile, out):
    for size in SHORT[tile]:
        check(make(size, out, bias=False, seed=size[2], residual="" if out == "e4m3" else "broadcast"))


@pytest.mark.parametrize("size", LONG)
@pytest.mark.parametrize("w_rows,layout", [(128, "vectors"), (1, "stride")])
def test_long_sums(size, w_rows, layout):
    check(make(size, "fp32", "gelu", gate_rows=50, residual="rows", seed=5, w_rows=w_rows, layout=layout), in_place=True)


@pytest.mark.parametrize("rows,cols,inner", [(1560, 5120, 1792), (1560, 5120, 1793), (777, 3008, 2560), (1560, 5120, 5120), (777, 3013, 6144)])
def test_fp32_sums_keep_their_digits(rows, cols, inner):
    """Terms of one sign, whose truncations add up: a chunk of 1792 has 56 steps of 32 products, each off by half a step (2^-24 of the sum
    so far) on average, the sum so far being half the chunk's on average; the chunks are added to nearest."""
    gen = torch.Generator(device="cuda").manual_seed(inner)
    x, w = operand(randn(gen, rows, inner).abs(), 1), operand(randn(gen, cols, inner, std=inner ** -0.5).abs(), 128)
    out, ws = torch.full((rows, cols), math.nan, device="cuda"), api.attn_workspace()
    api.sdvg_linear_e4m3(*x, *w, out, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    ref = values(*x, 1) @ values(*w, 128).t()
    chunks = -(-inner // 1792)
    assert float((out.double() - ref).norm() / ref.norm()) <= 56 * 2.0 ** -25 + chunks * 2.0 ** -24


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("sizes", [SIZES, ODD], ids=["vectors", "odd"])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
def test_extreme_scales_and_special_codes(tile, sizes, out):
    """Exponents at the ends of the quantiser's range cancel; all-zero blocks (scale 2^-126) add nothing; NaN codes and the NaN scale
    reach just the elements that they belong to."""
    s = make(sizes[tile], out, bias=False, seed=23, spread=0.0)
    (x, xs), (w, ws) = s["x"], s["w"]
    rows, cols = x.shape[0], w.shape[0]
    xs[:, 0], ws[:, 0] = 247, 10                           # 2^120 * 2^-117
    x[:, 128:256], xs[:, 1] = 0, 1
    w[:, 256:384], ws[:, 2] = 0, 1
    xs[1, 2] = 254                                         # 0 times anything finite
    check(s)
    last_row, last_col = rows - 1, cols - 1
    x[0, 5], x[last_row, 700] = 0x7F, 0xFF
    w[7, 400], w[last_col, 1] = 0xFF, 0x7F
    xs[130, 3] = 255
    got, scale = check(s)
    nan = (got.contiguous().view(torch.float8_e4m3fn) if out == "e4m3" else got).float().isnan()
    want = torch.zeros_like(nan)
    want[[0, 130, last_row]] = True
    want[:, [7, last_col]] = True
    assert torch.equal(nan, want)
    if out == "e4m3":
        assert bool((scale[[0, 130, last_row]] == 1).all())        # nothing but NaN: as a block of zeros


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("sizes", [SIZES, ODD], ids=["vectors", "odd"])
def test_infinities(tile, sizes):
    rows, cols, _ = sizes[tile]
    for out in ("bf16", "fp32"):
        s = make(sizes[tile], out, "silu", gate_rows=1, residual="rows", seed=29)
        s["residual"] = s["residual"].clone()
        s["residual"][0, 3], s["residual"][rows - 1, cols - 1] = math.inf, -math.inf
        s["gate"][1, 4], s["gate"][5, 6] = -math.inf, math.nan
        check(s)
    s = make(sizes[tile], "e4m3", gate_rows=1, seed=29)
    s["gate"][1, 4], s["bias"][4] = math.inf, 1e30
    s["gate"][2, cols - 1] = math.nan
    got, scale = check(s)
    assert int(scale[1, 0]) == 247 and int(got[1, 4]) == 0x7E and int(got[1, :4].max() & 0x7F) == 0
    assert int(got[2, cols - 1]) & 0x7F == 0x7F


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("sizes", [SIZES, ODD], ids=["vectors", "odd"])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "gelu"])
@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
def test_infinite_sums_and_far_tails(tile, sizes, act, out):
    """Through the bias: infinities, NaN and values whose activation underflows, next to ordinary ones."""
    s = make(sizes[tile], out, act, seed=41)
    special = [math.inf, -math.inf, math.nan, -1e4, 1e4, -60.0, 60.0, 0.0, -1e30, 1e30]
    if out == "e4m3":
        s["bias"][:10:2] = torch.tensor([math.nan, -1e4, -60.0, 0.0, -1e30])       # what does not set the scale of its block
        check(s)
        return
    s["bias"][:10] = torch.tensor(special)
    rows, cols, _ = sizes[tile]
    got = torch.empty((rows, cols), device="cuda", dtype=OUTS[out])
    call(s, got, api.attn_workspace())
    got = got.double()
    ref, err = expected(s)
    assert bool(got[:, 0].isposinf().all()) and bool(got[:, 2].isnan().all())
    assert bool((got[:, 1].isnan() | (got[:, 1] == 0)).all())      # -inf times 0, or 0 by its limit
    rest = slice(3, None)
    assert_within(got[:, rest], ref[:, rest], (err + (ref.abs() + err) * torch.finfo(OUTS[out]).eps / 2 + 2.0 ** -126)[:, rest])


@pytest.mark.parametrize("tile", [256, 512])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
def test_equal_calls_give_equal_bits_on_streams_and_in_graphs(tile, out):
    s = make(ODD[tile] if out == "fp32" else SIZES[tile], out, "gelu_tanh", gate_rows=100, seed=31)
    rows, cols = s["x"][0].shape[0], s["w"][0].shape[0]
    ws = api.attn_workspace()
    new = lambda: (torch.zeros((rows, cols), device="cuda", dtype=OUTS[out]),
                   torch.zeros((rows, -(-cols // 128)), device="cuda", dtype=torch.uint8) if out == "e4m3" else None)
    a, b, c = new(), new(), new()
    call(s, a[0], ws, a[1])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    call(s, b[0], ws, b[1], stream=other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, c[0], ws, c[1])
        call(s, c[0], ws, c[1])
    keep = s["x"][0].clone()
    s["x"][0].copy_(keep.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(a[0], c[0])
    s["x"][0].copy_(keep)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for d in (b, c):
        assert torch.equal(a[0], d[0]) and (out != "e4m3" or torch.equal(a[1], d[1]))


def test_launches_that_overlap_with_the_operators_around_them():
    """Rows quantised, products of both kinds of tiles, a norm, a product of few rows: without waits and one by one."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows, inner, wide = 777, 1200, 3008
    x, ws = randn(gen, rows, inner).bfloat16(), api.attn_workspace()
    w1, w2, w3 = (operand(randn(gen, n, k, std=k ** -0.5), 128) for n, k in ((wide, inner), (9999, wide), (inner, wide)))
    results = []
    for wait in (False, True):
        pause = torch.cuda.synchronize if wait else lambda: None
        h, f = api.e4m3_matrix(rows, inner), api.e4m3_matrix(rows, wide)
        y, z = torch.empty((rows, 9999), device="cuda", dtype=torch.bfloat16), torch.empty((rows, inner), device="cuda", dtype=torch.bfloat16)
        few, o = torch.empty((3, wide), device="cuda"), torch.empty((rows, inner), device="cuda")
        z.copy_(x)
        for _ in range(6):
            for step in (lambda: api.sdvg_gated_norm_e4m3(z, *h),
                         lambda: api.sdvg_linear_e4m3(*h, *w1, f[0], ws, act=api.SDVG_ACT_GELU, out_scale=f[1]),
                         lambda: api.sdvg_linear_e4m3(*f, *w2, y, ws, act=api.SDVG_ACT_SILU),
                         lambda: api.sdvg_linear_e4m3(h[0][:3], h[1][:3], *w1, few, ws),
                         lambda: api.sdvg_linear_e4m3(*f, *w3, z, ws, residual=z),
                         lambda: api.sdvg_gated_norm(z, o)):
                step()
                pause()
        torch.cuda.synchronize()
        assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
        results.append((o, y, few, f[0]))
    for a, b in zip(*results):
        assert torch.equal(a, b) and bool(a.float().isfinite().all())


def test_a_layer_whose_products_are_those_of_pairs():
    """The drafter's block over a ring with tile scales: near the 16-bit layer, in place, captured, without waits and one by one."""
    from test_gpu_layer import model, stream, weights
    sh = synth.Shape("pairs128x12", heads=12, head_dim=128, frames=3, grid_h=30, grid_w=52, slots=2)
    kw = dict(e4m3=True, tile_scales=True)
    w, m, m8 = weights(sh, 1), model(sh), model(sh, **kw)
    one, eight = schedule.TransformerLayer(w, m), schedule.TransformerLayerE4M3(w, m8)
    x, mod = stream(sh, 10)
    a, c, d = torch.empty_like(x), torch.full_like(x, float("nan")), x.clone()
    one.step(x, mod, 0, a)
    eight.step(x, mod, 0, c)
    m8.check_status("8-bit layer")
    change = (a.float() - x.float()).norm()
    assert float((a.float() - c.float()).norm()) <= 8 * 2.0 ** -4 * float(change)
    eight.step(d, mod, 0, d)
    torch.cuda.synchronize()
    assert torch.equal(c, d)
    graph, e = torch.cuda.CUDAGraph(), torch.empty_like(x)
    with torch.cuda.graph(graph):
        for _ in range(2):
            eight.step(x, mod, 0, e)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    m8.check_status("8-bit layer")
    assert torch.equal(c, e)
