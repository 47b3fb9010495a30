"""sdvg_gated_norm_e4m3 against fp64: the gated residual add and the modulated norm after it, into E4M3 rows."""
import numpy as np
import pytest
import torch

from dense_utils import DTYPES, assert_close, f64
from e4m3_utils import check_quantised
from oracle import e4m3_blocks_oracle as B
from paper_2604_17397_b200 import api
from test_gpu_gated_norm import KINDS, expected, problem, randn

pytestmark = pytest.mark.gpu


def call(s, x_out, out, scale, stream=None):
    api.sdvg_gated_norm_e4m3(s["x"], out, scale, y=s["y"], gate=s["gate"], gate_rows=s["gate_rows"], post_norm=KINDS[s["post"]],
                             post_weight=s["post_weight"], x_out=x_out, norm=KINDS[s["norm"]], weight=s["weight"], bias=s["bias"],
                             scale=s["scale"], shift=s["shift"], modulate_rows=s["mod_rows"], eps=s["eps"], stream=stream)


def check(s, x_out=True, ld=None, in_place=False):
    """The codes' values known up to the bound of fp32 outputs."""
    s["o"] = torch.float32
    (x_ref, ref), (x_tol, tol) = expected(s)
    rows, cols = s["x"].shape
    blocks, ld = -(-cols // 128), ld or -(-cols // 8) * 8 + 8
    out = torch.full((rows + 2, ld), 77, device="cuda", dtype=torch.uint8)
    scale = torch.full((rows + 2, blocks + 1), 33, device="cuda", dtype=torch.uint8)
    xo = torch.full((rows + 2, cols + 8), 77.0, device="cuda", dtype=s["x"].dtype)
    if in_place:
        xo[1:-1, :cols].copy_(s["x"])
        s["x"] = xo[1:-1, :cols]
    call(s, xo[1:-1, :cols] if x_out else None, out[1:-1, :cols], scale[1:-1, :-1])
    torch.cuda.synchronize()
    check_quantised(out[1:-1, :cols], scale[1:-1, :-1], ref, tol)
    for buf, fill in ((out, 77), (scale, 33), (xo, 77)):
        assert bool((buf[0] == fill).all()) and bool((buf[-1] == fill).all())
    assert bool((out[:, cols:] == 77).all()) and bool((scale[:, -1] == 33).all()) and bool((xo[:, cols:] == 77).all())
    if x_out:
        assert_close(xo[1:-1, :cols], x_ref, x_tol, "x_out")


COLS = [1, 2, 7, 8, 31, 64, 100, 120, 127, 128, 129, 136, 255, 256, 264, 513, 1000, 1024, 1032, 1537, 2048, 4097, 5120, 8192, 8200, 10000, 16384,
        20001]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms"), ("none", "layer")])
def test_widths(cols, norm, post):
    # eps as large as the spread keeps rows of one or two columns well conditioned
    check(problem(9, cols, norm=norm, post=post, affine=True, mod_rows=4, gate_rows=5, seed=cols, eps=1e-2 if cols < 8 else 1e-6))


@pytest.mark.parametrize("x", list(DTYPES))
@pytest.mark.parametrize("y", ["", "bf16", "fp16", "fp32"])
@pytest.mark.parametrize("cols", [256, 261, 1536])
def test_types(x, y, cols):
    check(problem(7, cols, x, y, mod_rows=3, gate_rows=2 if y else 0, seed=5), x_out=bool(y))


@pytest.mark.parametrize("rows,cols", [(1, 1536), (700, 200), (1500, 1032), (333, 1999)])
def test_many_rows_and_odd_strides(rows, cols):
    check(problem(rows, cols, norm="rms", gate_rows=rows, mod_rows=97, seed=6))
    check(problem(rows, cols, "fp32", "", norm="layer", pad=3, seed=6), x_out=False, ld=cols + 1)


@pytest.mark.parametrize("cols", [136, 1537, 5120, 9000])
def test_in_place(cols):
    check(problem(20, cols, gate_rows=20, seed=8), in_place=True)


@pytest.mark.parametrize("cols", [64, 300, 1537, 5120, 10248, 9001])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_as_they_are_are_quantised_exactly(cols, dtype):
    """No norm and nothing to add: the codes of sdvg_quant_e4m3_blocks, and of the oracle."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = (randn(gen, 40, cols) * torch.exp2(torch.arange(40, device="cuda") % 13 - 6.0)[:, None]).to(DTYPES[dtype])
    x[3, 5], x[4, 6] = float("nan"), float("inf")
    x[5] = 0
    out, scale = api.e4m3_matrix(40, cols)
    api.sdvg_gated_norm_e4m3(x, out, scale, norm=api.SDVG_NORM_NONE)
    codes, bytes_ = B.quantise(f64(x), 1)
    assert np.array_equal(scale.cpu().numpy(), bytes_)
    assert np.array_equal(out.cpu().numpy() & 0x7F, codes & 0x7F)
    other, other_scale = api.e4m3_matrix(40, cols)
    api.sdvg_quant_e4m3_blocks(x, other, other_scale)
    finite = torch.isfinite(x)
    assert torch.equal(scale, other_scale) and torch.equal(out[finite], other[finite])


def test_streams_graphs_and_equal_bits():
    s = problem(200, 1536, gate_rows=50, mod_rows=40, seed=9)
    made = [api.e4m3_matrix(200, 1536) for _ in range(3)]
    call(s, None, *made[0])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    call(s, None, *made[1], stream=other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, None, *made[2])
    graph.replay()
    torch.cuda.synchronize()
    for o, sc in made[1:]:
        assert torch.equal(o, made[0][0]) and torch.equal(sc, made[0][1])


def test_a_product_of_normed_rows():
    """Norm into 8-bit rows, product, norm of the product: launches that overlap, against the same calls one by one."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = randn(gen, 300, 1024).bfloat16()
    w, ws = api.e4m3_matrix(512, 1024, 128)
    api.sdvg_quant_e4m3_blocks(randn(gen, 512, 1024, std=1 / 32), w, ws)
    space = api.attn_workspace()
    results = []
    for wait in (False, True):
        h, hs = api.e4m3_matrix(300, 1024)
        y, o = torch.empty((300, 512), device="cuda", dtype=torch.bfloat16), torch.empty((300, 512), device="cuda")
        pause = torch.cuda.synchronize if wait else lambda: None
        for _ in range(5):
            api.sdvg_gated_norm_e4m3(x, h, hs)
            pause()
            api.sdvg_linear_e4m3(h, hs, w, ws, y, space, act=api.SDVG_ACT_GELU)
            pause()
            api.sdvg_gated_norm(y, o)
            pause()
        torch.cuda.synchronize()
        results.append(o)
    assert torch.equal(*results)
