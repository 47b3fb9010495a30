"""sdvg_linear_e4m3 and the quantisation of its operands against fp64."""
import math

import numpy as np
import pytest
import torch

from dense_utils import DTYPES, assert_close, f64, linear_tolerance
from e4m3_utils import check_quantised
from oracle import dense_oracle as D
from oracle import e4m3_blocks_oracle as B
from paper_2604_17397_b200 import api

pytestmark = pytest.mark.gpu

ACTS = {"none": api.SDVG_ACT_NONE, "silu": api.SDVG_ACT_SILU, "gelu_tanh": api.SDVG_ACT_GELU_TANH, "gelu": api.SDVG_ACT_GELU}
OUTS = {**DTYPES, "e4m3": torch.uint8}


def randn(gen, *shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda") * std


def coded(x, block_rows, pad=16, more=0, fill=0x7F):
    """E4M3 codes and scales of x as the oracle quantises them; what lies between the rows is NaN."""
    codes, scale = B.quantise(f64(x), block_rows)
    got = []
    for a, p in ((codes, 16), (scale, 4)):
        ld = -(-a.shape[1] // p) * p + more * p
        buf = torch.full((a.shape[0], ld), fill if p == 16 else 255, device="cuda", dtype=torch.uint8)
        buf[:, :a.shape[1]] = torch.from_numpy(a).cuda()
        got.append(buf[:, :a.shape[1]])
    return got


def problem(rows, cols, inner, out="bf16", act="none", bias=True, gate_rows=0, residual="", seed=0, w_rows=128, spread=6.0, more=0):
    """spread: blocks differ in magnitude by up to 2^spread."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sized = lambda n: torch.exp2(spread * torch.rand((n, -(-inner // 128)), generator=gen, device="cuda") - spread / 2
                                 ).repeat_interleave(128, 1)[:, :inner]
    x = randn(gen, rows, inner) * sized(rows)
    w = randn(gen, cols, inner, std=1 / math.sqrt(inner)) * sized(-(-cols // 128)).repeat_interleave(128, 0)[:cols]
    s = dict(x=coded(x, 1, more=more), w=coded(w, w_rows, more=more), act=act, gate_rows=gate_rows, out=out, w_rows=w_rows)
    s["bias"] = randn(gen, cols) if bias else None
    s["gate"] = randn(gen, -(-rows // gate_rows), cols) if gate_rows else None
    s["residual"] = None
    if residual:
        s["residual"] = randn(gen, rows if residual == "rows" else 1, cols, std=2.0).to(OUTS[out]).expand(rows, cols)
    return s


def call(s, out, ws, out_scale=None, stream=None):
    api.sdvg_linear_e4m3(*s["x"], *s["w"], out, ws, bias=s["bias"], act=ACTS[s["act"]], residual=s["residual"], gate=s["gate"],
                         gate_rows=s["gate_rows"], out_scale=out_scale, stream=stream)


def expected(s, dtype):
    """(reference, bound) of the result rounded to dtype."""
    x, w = (B.values(c.cpu().numpy(), e.cpu().numpy(), n) for (c, e), n in ((s["x"], 1), (s["w"], s["w_rows"])))
    b, g, r = (f64(s[k]) for k in ("bias", "gate", "residual"))
    ref = D.linear_ref(x, w, b, s["act"], g, s["gate_rows"], r)
    per_row = None if g is None else D.of_rows(g, x.shape[0], s["gate_rows"])
    return ref, linear_tolerance(x, w, b, s["act"], per_row, r, ref, dtype)


def check(s, ld_out=None, in_place=False):
    ws = api.attn_workspace()
    rows, cols = s["x"][0].shape[0], s["w"][0].shape[0]
    dtype = OUTS[s["out"]]
    buf = torch.full((rows + 2, ld_out or cols), 77, device="cuda", dtype=dtype)         # a row before, a row after
    out = buf[1:rows + 1, :cols]
    if s["out"] == "e4m3":
        blocks = -(-cols // 128)
        sbuf = torch.full((rows + 2, blocks + 1), 33, device="cuda", dtype=torch.uint8)
        call(s, out, ws, sbuf[1:rows + 1, :blocks])
        assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
        check_quantised(out, sbuf[1:rows + 1, :blocks], *expected(s, torch.float32))
        assert bool((sbuf[0] == 33).all()) and bool((sbuf[-1] == 33).all()) and bool((sbuf[:, blocks:] == 33).all())
    else:
        ref, tol = expected(s, dtype)
        if in_place:
            out.copy_(s["residual"])
            s["residual"] = out
        call(s, out, ws)
        assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
        assert_close(out, ref, tol)
    assert bool((buf[0] == 77).all()) and bool((buf[rows + 1] == 77).all()) and bool((buf[:, cols:] == 77).all())
    return out


@pytest.mark.parametrize("rows,cols,inner", [(1, 128, 128), (64, 128, 512), (65, 256, 128), (256, 256, 512)])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
def test_plain_tiles(rows, cols, inner, out):
    check(problem(rows, cols, inner, out, bias=False, seed=1))


SHAPES = [(1, 1, 1), (1, 1536, 256), (2, 5, 7), (3, 130, 72), (15, 128, 640), (16, 127, 63), (17, 129, 129), (33, 100, 700),
          (64, 257, 1100), (127, 64, 640), (128, 300, 130), (129, 260, 515), (241, 129, 1281), (256, 256, 128), (257, 127, 1537),
          (300, 515, 2000), (513, 70, 64), (1000, 640, 72)]


@pytest.mark.parametrize("rows,cols,inner", SHAPES)
@pytest.mark.parametrize("out", ["bf16", "fp32", "fp16", "e4m3"])
def test_shapes(rows, cols, inner, out):
    check(problem(rows, cols, inner, out, gate_rows=max(1, rows // 3), residual="" if out == "e4m3" else "rows",
                  seed=rows + cols + inner))


@pytest.mark.parametrize("rows", [5, 100])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32", "e4m3"])
def test_activations(rows, act, out):
    for cols in (200, 201, 208):                               # whole vectors of 8, none, of 16
        check(problem(rows, cols, 300, out, act, residual="" if out == "e4m3" else "broadcast", gate_rows=rows, seed=7))


@pytest.mark.parametrize("out", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("cols,ld_out,gate_rows", [(192, 192, 1), (192, 200, 7), (320, 336, 40), (16, 16, 100), (48, 64, 3), (176, 192, 100)])
def test_outputs_of_whole_vectors(out, cols, ld_out, gate_rows):
    """Gates that change within a block of tokens, strides wider than the rows, features that end inside a warp's 32."""
    for rows in (65, 130, 333):
        s = problem(rows, cols, 260, out, "silu", gate_rows=gate_rows, residual="" if out == "e4m3" else "rows", seed=rows + cols)
        check(s, ld_out=ld_out)
        if out != "e4m3":
            check(s, ld_out=ld_out, in_place=True)


@pytest.mark.parametrize("rows", [64, 65])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "gelu"])
def test_infinite_sums_and_far_tails(rows, act):
    """Through the bias: infinities, NaN and values whose activation underflows, next to ordinary ones."""
    with np.errstate(invalid="ignore", over="ignore"):
        _infinite_sums_and_far_tails(rows, act)


def _infinite_sums_and_far_tails(rows, act):
    s = problem(rows, 128, 128, "bf16", act, seed=41)
    s["bias"][:8] = torch.tensor([float("inf"), float("-inf"), float("nan"), -1e4, 1e4, -60.0, 60.0, 0.0])
    out = torch.empty((rows, 128), device="cuda", dtype=torch.bfloat16)
    call(s, out, api.attn_workspace())
    torch.cuda.synchronize()
    got = f64(out)
    ref, tol = expected(s, torch.bfloat16)
    assert np.isposinf(got[:, 0]).all() and np.isnan(got[:, 2]).all()
    assert (np.isnan(got[:, 1]) | (got[:, 1] == 0)).all()      # -inf times 0, or 0 by its limit
    assert (np.abs(got[:, 3:] - ref[:, 3:]) <= tol[:, 3:]).all()


@pytest.mark.parametrize("rows,cols,inner", [(3, 300, 1400), (90, 300, 1400), (90, 1, 600)])
def test_scales_per_row_of_the_weights(rows, cols, inner):
    check(problem(rows, cols, inner, "fp32", seed=11, w_rows=1, spread=20.0, more=1))


@pytest.mark.parametrize("rows,cols,inner", [(3, 520, 9000), (40, 70, 5120), (70, 140, 9000), (80, 144, 6144), (80, 144, 6145), (200, 513, 12800)])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
def test_long_sums(rows, cols, inner, out):
    check(problem(rows, cols, inner, out, act="silu", seed=13, residual="" if out == "e4m3" else "rows"))


@pytest.mark.parametrize("rows", [6, 150])
def test_strides_and_in_place(rows):
    check(problem(rows, 150, 260, "bf16", residual="rows", seed=17, more=3), ld_out=157, in_place=True)
    check(problem(rows, 150, 260, "e4m3", seed=17, more=3), ld_out=153)


@pytest.mark.parametrize("rows", [2, 80])
def test_several_tiles_per_pair_and_wide_outputs(rows):
    check(problem(rows * 12, 5000, 200, "bf16", seed=19, gate_rows=7))
    check(problem(rows * 12, 5000, 200, "e4m3", act="gelu", seed=19, gate_rows=7))


@pytest.mark.parametrize("rows", [4, 70])
@pytest.mark.parametrize("out", ["fp32", "e4m3"])
def test_extreme_scales_and_special_codes(rows, out):
    """Exponents at the ends of the quantiser's range cancel; all-zero blocks (scale 2^-126) add nothing; NaN codes and the NaN scale
    reach just the elements that they belong to."""
    s = problem(rows, 256, 512, out, bias=False, seed=23, spread=0.0)
    (x, xs), (w, ws_) = s["x"], s["w"]
    xs[:, 0], ws_[:, 0] = 247, 10                          # 2^120 * 2^-117
    x[:, 128:256], xs[:, 1] = 0, 1
    w[:, 256:384], ws_[:, 2] = 0, 1
    xs[1, 2] = 254                                         # 0 times anything finite
    check(s)
    x[0, 5] = 0x7F
    w[7, 400] = 0xFF
    xs[2, 3] = 255
    out_t = torch.zeros((rows, 256), device="cuda", dtype=OUTS[out])
    scale = torch.zeros((rows, 2), device="cuda", dtype=torch.uint8) if out == "e4m3" else None
    call(s, out_t, api.attn_workspace(), scale)
    nan = torch.isnan(out_t.view(torch.float8_e4m3fn).float() if out == "e4m3" else out_t)
    want = torch.zeros_like(nan)
    want[0], want[2], want[:, 7] = True, True, True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("rows", [4, 200])
def test_infinities_of_gate_and_residual(rows):
    s = problem(rows, 130, 128, "bf16", act="silu", gate_rows=1, residual="rows", seed=29)
    s["residual"] = s["residual"].clone()
    s["residual"][0, 3] = float("inf")
    s["gate"][1, 4] = float("-inf")
    check(s)
    s = problem(rows, 130, 128, "e4m3", gate_rows=1, seed=29)
    s["gate"][1, 4], s["bias"][4] = float("inf"), 1e30
    out, scale = torch.empty((rows, 130), device="cuda", dtype=torch.uint8), torch.empty((rows, 2), device="cuda", dtype=torch.uint8)
    call(s, out, api.attn_workspace(), scale)
    assert int(scale[1, 0]) == 247 and int(out[1, 4]) == 0x7E and int(out[1, :4].max() & 0x7F) == 0


@pytest.mark.parametrize("rows", [1, 65])
def test_equal_calls_give_equal_bits_and_streams(rows):
    s = problem(rows, 700, 1300, "fp32", seed=31)
    ws = api.attn_workspace()
    a, b = (torch.empty((rows, 700), device="cuda") for _ in range(2))
    call(s, a, ws)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    call(s, b, ws, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    c = torch.empty_like(a)
    with torch.cuda.graph(graph):
        call(s, c, ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, c)


def test_nothing_to_do():
    ws = api.attn_workspace()
    x, xs = api.e4m3_matrix(4, 64)
    w, wscale = api.e4m3_matrix(8, 64, 128)
    api.sdvg_linear_e4m3(x[:0], xs[:0], w, wscale, torch.empty((0, 8), device="cuda"), ws)
    api.sdvg_linear_e4m3(x, xs, w[:0], wscale[:0], torch.empty((4, 0), device="cuda"), ws)


# ---- quantisation and back -------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (127, 40), (128, 128), (130, 300), (257, 1000)])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantised_matrices_equal_the_oracle(rows, cols, dtype, block_rows):
    gen = torch.Generator(device="cuda").manual_seed(rows * cols)
    for odd in (0, 1):
        size = torch.exp2(torch.randint(-40, 40, (rows, 1), generator=gen, device="cuda").float() / (4 if dtype == "fp16" else 1))
        x = torch.empty((rows, -(-cols // 8) * 8 + odd), device="cuda", dtype=DTYPES[dtype])[:, :cols]
        x.copy_((randn(gen, rows, cols) * size).to(DTYPES[dtype]))
        codes, scale = B.quantise(f64(x), block_rows)
        out = torch.full((rows + 2, -(-cols // 8) * 8 + 8 + odd), 77, device="cuda", dtype=torch.uint8)
        s = torch.full((scale.shape[0] + 2, scale.shape[1] + 1), 33, device="cuda", dtype=torch.uint8)
        o, so = out[1:-1, :cols], s[1:-1, :-1]
        api.sdvg_quant_e4m3_blocks(x, o, so)
        assert np.array_equal(so.cpu().numpy(), scale)
        assert np.array_equal(o.cpu().numpy(), codes)
        assert bool((out[0] == 77).all()) and bool((out[-1] == 77).all()) and bool((out[:, cols:] == 77).all())
        assert bool((s[0] == 33).all()) and bool((s[-1] == 33).all()) and bool((s[:, -1] == 33).all())
        for back in DTYPES.values():
            got = torch.full((rows, cols + 8 - cols % 8 + odd), 5.0, device="cuda", dtype=back)
            api.sdvg_dequant_e4m3_blocks(o, so, got[:, :cols])
            want = torch.from_numpy(B.values(codes, scale, block_rows)).to(back)
            assert torch.equal(got[:, :cols].cpu(), want) and bool((got[:, cols:] == 5).all())


@pytest.mark.parametrize("block_rows", [1, 128])
def test_special_values_are_quantised_as_written(block_rows):
    x = torch.zeros((130, 260), device="cuda")
    x[0, 0], x[0, 130], x[1, 3], x[129, 259] = float("nan"), float("inf"), 2.0 ** -140, -float("inf")
    x[2, 5], x[3, 6], x[128, 0] = 448.0, 450.0, 2.0 ** -149
    codes, scale = B.quantise(f64(x), block_rows)
    o, s = api.e4m3_matrix(130, 260, block_rows)
    api.sdvg_quant_e4m3_blocks(x, o, s)
    assert np.array_equal(s.cpu().numpy(), scale) and np.array_equal(o.cpu().numpy() & 0x7F, codes & 0x7F)
    s[0, 0], s[-1, -1] = 0, 255
    got = torch.empty((130, 260), device="cuda")
    api.sdvg_dequant_e4m3_blocks(o, s, got)
    want = torch.from_numpy(B.values(o.cpu().numpy(), s.cpu().numpy(), block_rows)).float()
    assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))


def test_the_quantised_operands_of_a_product():
    """Quantised by the library, multiplied, against the product of what the codes stand for, and near the unquantised one."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w = randn(gen, 150, 1000).bfloat16(), randn(gen, 270, 1000, std=1000 ** -0.5).bfloat16()
    xq, wq = api.e4m3_matrix(150, 1000), api.e4m3_matrix(270, 1000, 128)
    api.sdvg_quant_e4m3_blocks(x, *xq)
    api.sdvg_quant_e4m3_blocks(w, *wq)
    s = dict(x=xq, w=wq, act="none", gate_rows=0, out="fp32", w_rows=128, bias=None, gate=None, residual=None)
    got = f64(check(s))
    ref = f64(x) @ f64(w).T
    # each operand is off by at most 2^-4, 3.6% rms at worst evenly spread; both independent
    assert np.linalg.norm(got - ref) <= 0.06 * np.linalg.norm(ref)


def values_on_gpu(codes, scale, block_rows):
    f = torch.exp2(scale.double() - 127).repeat_interleave(128, 1)[:, :codes.shape[1]].repeat_interleave(block_rows, 0)[:codes.shape[0]]
    return codes.view(torch.float8_e4m3fn).double() * f


@pytest.mark.parametrize("rows,cols,inner", [(2500, 10000, 130), (2333, 9999, 1150), (4680, 5120, 512), (1111, 20480, 900), (4680, 1536, 2816)])
@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
def test_many_tiles(rows, cols, inner, out):
    """Rounds of tiles of every width, all outputs, in 64 bits on the GPU; the bound is that of linear_tolerance without an activation."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, w = api.e4m3_matrix(rows, inner), api.e4m3_matrix(cols, inner, 128)
    api.sdvg_quant_e4m3_blocks(randn(gen, rows, inner) * torch.exp2(4 * torch.rand((rows, 1), generator=gen, device="cuda")), *x)
    api.sdvg_quant_e4m3_blocks(randn(gen, cols, inner, std=inner ** -0.5), *w)
    gate, bias = randn(gen, 3, cols), randn(gen, cols)
    per = -(-rows // 3)
    o = torch.full((rows + 1, cols), 77, device="cuda", dtype=OUTS[out])
    scale = torch.zeros((rows, -(-cols // 128)), device="cuda", dtype=torch.uint8) if out == "e4m3" else None
    ws = api.attn_workspace()
    for _ in range(3):
        api.sdvg_linear_e4m3(*x, *w, o[:rows], ws, bias=bias, gate=gate, gate_rows=per, out_scale=scale)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    xv, wv = values_on_gpu(*x, 1), values_on_gpu(*w, 128)
    g = gate.double().repeat_interleave(per, 0)[:rows]
    v = xv @ wv.t() + bias.double()
    err = ((inner + 2) * 2 * 2.0 ** -24 * (xv.abs() @ wv.abs().t() + bias.double().abs()) + 4 * 2.0 ** -24 * v.abs()) * g.abs()
    ref = v * g
    if out == "e4m3":
        f = torch.exp2(scale.double() - 127).repeat_interleave(128, 1)[:, :cols]
        got = o[:rows].view(torch.float8_e4m3fn).double() * f
        tol = err + torch.maximum((ref.abs() + err) / 16, f / 1024)
        # the scale is the smallest for a block's largest magnitude, which is known up to err
        top = lambda a: torch.nn.functional.pad(a, (0, -cols % 128)).unflatten(1, (-1, 128)).amax(2)
        assert bool((top(ref.abs() - err) <= 448 * f[:, ::128]).all()) and bool((top(ref.abs() + err) > 224 * f[:, ::128]).all())
    else:
        got = o[:rows].double()
        tol = err + (ref.abs() + err) * torch.finfo(OUTS[out]).eps / 2
    assert bool(((got - ref).abs() <= tol).all())
    assert bool((o[rows] == 77).all())


def bound_on_gpu(x, w, bias, act, gate, residual, dtype):
    """linear_tolerance and the reference, in 64 bits on the GPU, for sizes that only pairs of CTAs take; gate per row or None."""
    u = 2.0 ** -24
    v = x @ w.t() + bias
    err = (x.shape[1] + 2) * 2 * u * (x.abs() @ w.abs().t() + bias.abs())
    a = v * torch.sigmoid(v) if act == "silu" else v
    if act == "silu":
        err = 1.13 * err + 2.0 ** -14 * a.abs() + 1e-36
    g = torch.ones_like(a[:1]) if gate is None else gate
    r = torch.zeros_like(a[:1]) if residual is None else residual
    ref = g * a + r
    err = g.abs() * err + 4 * u * ((g * a).abs() + r.abs())
    return ref, err if dtype is None else err + (ref.abs() + err) * torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32", "e4m3"])
@pytest.mark.parametrize("cols,more,gate_rows,residual", [(3008, 0, 1, "rows"), (3016, 8, 7, "rows"), (3012, 4, 100, "broadcast"), (3013, 0, 300, "rows"),
                                                          (3024, 16, 0, ""), (2990, 0, 777, "broadcast")])
def test_outputs_of_pairs(out, cols, more, gate_rows, residual):
    """Rows of whole vectors and not, strides wider than the rows, gates that change within a block of tokens, in place."""
    rows, inner = 777, 1200
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, w = api.e4m3_matrix(rows, inner), api.e4m3_matrix(cols, inner, 128)
    api.sdvg_quant_e4m3_blocks(randn(gen, rows, inner), *x)
    api.sdvg_quant_e4m3_blocks(randn(gen, cols, inner, std=inner ** -0.5), *w)
    bias, ws = randn(gen, cols), api.attn_workspace()
    gate = randn(gen, -(-rows // gate_rows), cols) if gate_rows else None
    per_row = None if gate is None else gate.double().repeat_interleave(gate_rows, 0)[:rows]
    act = "silu" if gate_rows % 2 else "none"
    dtype = OUTS[out]
    res = None
    if residual and out != "e4m3":
        res = randn(gen, rows if residual == "rows" else 1, cols, std=2.0).to(dtype).expand(rows, cols)
    buf = torch.full((rows + 2, cols + more), 77, device="cuda", dtype=dtype)
    o = buf[1:-1, :cols]
    ref, tol = bound_on_gpu(values_on_gpu(*x, 1), values_on_gpu(*w, 128), bias.double(), act, per_row, None if res is None else res.double(),
                            None if out == "e4m3" else dtype)
    for in_place in (False, residual == "rows" and res is not None):
        if in_place:
            o.copy_(res)
        scale = torch.zeros((rows, -(-cols // 128)), device="cuda", dtype=torch.uint8) if out == "e4m3" else None
        api.sdvg_linear_e4m3(*x, *w, o, ws, bias=bias, act=ACTS[act], gate=gate, gate_rows=gate_rows, residual=o if in_place else res,
                             out_scale=scale)
        assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
        if out == "e4m3":
            f = torch.exp2(scale.double() - 127).repeat_interleave(128, 1)[:, :cols]
            top = lambda a: torch.nn.functional.pad(a, (0, -cols % 128)).unflatten(1, (-1, 128)).amax(2)
            assert bool((top(ref.abs() - tol) <= 448 * f[:, ::128]).all()) and bool((top(ref.abs() + tol) > 224 * f[:, ::128]).all())
            got, within = o.view(torch.float8_e4m3fn).double() * f, tol + torch.maximum((ref.abs() + tol) / 16, f / 1024)
        else:
            got, within = o.double(), tol
        assert bool(((got - ref).abs() <= within).all())
        assert bool((buf[0] == 77).all()) and bool((buf[-1] == 77).all()) and bool((buf[:, cols:] == 77).all())


@pytest.mark.parametrize("cols", [3000, 3001])
@pytest.mark.parametrize("rows,inner", [(777, 6144), (777, 6272), (700, 7800), (2555, 6400)])
def test_long_fp32_sums_of_pairs(rows, inner, cols):
    gen = torch.Generator(device="cuda").manual_seed(inner)
    x, w = api.e4m3_matrix(rows, inner), api.e4m3_matrix(cols, inner, 128)
    api.sdvg_quant_e4m3_blocks(randn(gen, rows, inner).abs(), *x)                    # all terms of one sign: the drift adds up
    api.sdvg_quant_e4m3_blocks(randn(gen, cols, inner, std=inner ** -0.5).abs(), *w)
    res, bias, ws = randn(gen, rows, cols), randn(gen, cols), api.attn_workspace()
    o = torch.full((rows, cols), float("nan"), device="cuda")
    api.sdvg_linear_e4m3(*x, *w, o, ws, bias=bias, residual=res)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    ref, tol = bound_on_gpu(values_on_gpu(*x, 1), values_on_gpu(*w, 128), bias.double(), "none", None, res.double(), torch.float32)
    assert bool(((o.double() - ref).abs() <= tol).all())
    # the truncation of the tensor core, 32 products at a time, off by at most half a step of the sum each on average: 2^-25 per step
    # of a sum of up to 6144; later chunks are added to nearest
    assert float((o.double() - ref).norm() / ref.norm()) <= 6144 / 32 * 2.0 ** -25
