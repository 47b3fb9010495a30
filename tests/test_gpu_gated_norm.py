"""sdvg_gated_norm against fp64: the gated residual add and the modulated norm after it."""
import numpy as np
import pytest
import torch

from dense_utils import DTYPES, assert_close, f64, gated_norm_tolerance
from oracle import dense_oracle as O
from paper_2604_17397_b200 import api

pytestmark = pytest.mark.gpu

KINDS = {"none": api.SDVG_NORM_NONE, "rms": api.SDVG_NORM_RMS, "layer": api.SDVG_NORM_LAYER}


def randn(gen, *shape, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda") * std + mean


def rows_of(gen, rows, cols, dtype, pad=0, std=1.0, mean=0.0):
    buf = torch.full((rows, cols + pad), float("nan"), device="cuda", dtype=dtype)
    buf[:, :cols] = randn(gen, rows, cols, std=std, mean=mean).to(dtype)
    return buf[:, :cols]


def problem(rows, cols, x="bf16", y="bf16", out="bf16", norm="layer", post="none", affine=False, mod_rows=0, gate_rows=0,
            pad=0, seed=0, std=2.0, mean=0.5, eps=1e-6):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(x=rows_of(gen, rows, cols, DTYPES[x], pad, std, mean), y=rows_of(gen, rows, cols, DTYPES[y], pad) if y else None,
             norm=norm, post=post, mod_rows=mod_rows, gate_rows=gate_rows, eps=eps, o=DTYPES[out])
    s["gate"] = randn(gen, -(-rows // gate_rows), cols) if gate_rows else None
    # scale and shift as column ranges of one modulation matrix, as a model has them
    mod = randn(gen, -(-rows // mod_rows), 2 * cols, std=0.5) if mod_rows else None
    s["scale"], s["shift"] = (mod[:, :cols], mod[:, cols:]) if mod_rows else (None, None)
    s["weight"] = randn(gen, cols, std=0.3, mean=1.0) if affine else None
    s["bias"] = randn(gen, cols, std=0.3) if affine else None
    s["post_weight"] = randn(gen, cols, std=0.3, mean=1.0) if post != "none" and affine else None
    return s


def call(s, x_out, out, stream=None):
    api.sdvg_gated_norm(s["x"], out, y=s["y"], gate=s["gate"], gate_rows=s["gate_rows"], post_norm=KINDS[s["post"]],
                        post_weight=s["post_weight"], x_out=x_out, norm=KINDS[s["norm"]], weight=s["weight"], bias=s["bias"],
                        scale=s["scale"], shift=s["shift"], modulate_rows=s["mod_rows"], eps=s["eps"], stream=stream)


def expected(s):
    v = {k: f64(s[k]) for k in ("x", "y", "post_weight", "gate", "weight", "bias", "scale", "shift")}
    rows = v["x"].shape[0]
    refs = O.gated_norm_ref(v["x"], v["y"], s["post"], v["post_weight"], v["gate"], s["gate_rows"], s["norm"], v["weight"],
                            v["bias"], v["scale"], v["shift"], s["mod_rows"], s["eps"])
    per = lambda a, n: None if a is None else O.of_rows(a, rows, n)
    tols = gated_norm_tolerance(v["x"], v["y"], s["post"], v["post_weight"], per(v["gate"], s["gate_rows"]), s["norm"],
                                v["weight"], v["bias"], per(v["scale"], s["mod_rows"]), per(v["shift"], s["mod_rows"]),
                                s["eps"], refs, s["x"].dtype, s["o"])
    return refs, tols


def check(s, want=("x_out", "out"), in_place=""):
    refs, tols = expected(s)
    rows, cols = s["x"].shape
    bufs = {}
    for name, dtype in (("x_out", s["x"].dtype), ("out", s["o"])):
        buf = torch.full((rows + 2, cols + 8), 77.0, device="cuda", dtype=dtype)
        bufs[name] = (buf, buf[1:rows + 1, :cols])
    if in_place:                       # the named output takes the storage of x or y
        name, source = in_place.split("=")
        bufs[name][1].copy_(s[source])
        s[source] = bufs[name][1]
    call(s, *(bufs[n][1] if n in want else None for n in ("x_out", "out")))
    torch.cuda.synchronize()
    for (name, (buf, t)), ref, tol in zip(bufs.items(), refs, tols):
        if name in want:
            assert_close(t, ref, tol, name)
            assert bool((buf[0] == 77).all()) and bool((buf[rows + 1] == 77).all()) and bool((buf[:, cols:] == 77).all())
        elif not in_place:
            assert bool((buf == 77).all())


COLS = [1, 2, 7, 8, 31, 64, 100, 128, 255, 256, 513, 1024, 1032, 1537, 2048, 4097, 5120, 8192, 10000, 16384, 20001]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms"), ("layer", "layer"), ("none", "rms")])
def test_widths(cols, norm, post):
    # eps as large as the spread keeps rows of one or two columns well conditioned
    check(problem(9, cols, norm=norm, post=post, affine=True, mod_rows=4, gate_rows=5, seed=cols, eps=1e-2 if cols < 8 else 1e-6))


@pytest.mark.parametrize("rows", [3, 400])
@pytest.mark.parametrize("x,y", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "")])
def test_every_team_size(rows, x, y):
    """Widths that differ by a warp of the team, up to the widest: among them rings of just under, at and over 48 KB."""
    for cols in range(512, 10241, 512 if x == "bf16" else 256):
        for c in (cols - 8, cols):
            s = problem(rows, c, x, y, "bf16", gate_rows=rows if y else 0, seed=c)
            out = torch.full((rows, c), float("nan"), device="cuda", dtype=torch.bfloat16)
            call(s, None, out)
            v = s["x"].double() + (s["gate"].double() * s["y"].double() if y else 0)
            n = (v - v.mean(1, keepdim=True)) / torch.sqrt(v.var(1, keepdim=True, unbiased=False) + 1e-6)
            # half a step of bf16, and far less for the fp32 arithmetic
            assert bool(((out.double() - n).abs() <= 2.0 ** -8 * n.abs() + 2.0 ** -14 * (1 + n.abs())).all()), c


@pytest.mark.parametrize("x", list(DTYPES))
@pytest.mark.parametrize("y", ["", *DTYPES])
@pytest.mark.parametrize("out", list(DTYPES))
@pytest.mark.parametrize("cols", [96, 1536, 1541])
def test_types(x, y, out, cols):
    check(problem(13, cols, x, y, out, affine=cols != 96, mod_rows=13, gate_rows=3 if y else 0, post="rms" if y else "none", seed=cols))


@pytest.mark.parametrize("rows", [1, 2, 37, 700])
@pytest.mark.parametrize("mod_rows,gate_rows", [(1, 1), (7, 0), (0, 11), (64, 3), (1000, 1000)])
@pytest.mark.parametrize("cols", [64, 1280])
def test_row_groups(rows, mod_rows, gate_rows, cols):
    check(problem(rows, cols, mod_rows=mod_rows, gate_rows=gate_rows, seed=rows))


@pytest.mark.parametrize("pad", [1, 4, 8, 24])
@pytest.mark.parametrize("x,out", [("bf16", "bf16"), ("fp32", "bf16")])
def test_strided_rows(pad, x, out):
    check(problem(21, 520, x, "bf16", out, pad=pad, gate_rows=6, mod_rows=9, seed=pad))


@pytest.mark.parametrize("x,y,out,how", [("bf16", "bf16", "bf16", "x_out=x"), ("fp32", "bf16", "bf16", "x_out=x"),
                                         ("bf16", "fp16", "bf16", "out=x"), ("fp32", "bf16", "bf16", "out=y"),
                                         ("fp16", "fp16", "fp32", "x_out=y")])
@pytest.mark.parametrize("rows,cols", [(5, 72), (400, 1537), (400, 5120)])
def test_in_place(x, y, out, how, rows, cols):
    check(problem(rows, cols, x, y, out, gate_rows=100, mod_rows=100, post="rms", seed=cols), in_place=how)


@pytest.mark.parametrize("want", [("x_out",), ("out",)])
@pytest.mark.parametrize("cols", [72, 1537, 5120])
def test_either_output_alone(want, cols):
    check(problem(30, cols, gate_rows=7, post="layer", affine=True), want=want)


@pytest.mark.parametrize("cols", [100, 5120])
def test_large_mean_keeps_the_variance(cols):
    """A mean a thousand times the spread: sums of squares would lose the variance, centred values keep it."""
    check(problem(20, cols, "fp32", "", "fp32", mean=1000.0, std=1.0, seed=4))


@pytest.mark.parametrize("cols", [64, 1536, 1537, 9000])
def test_zero_rows_constant_rows_and_zero_eps(cols):
    s = problem(4, cols, "fp32", "", "fp32", norm="layer", eps=1e-6)
    s["x"][0] = 0.0
    s["x"][1] = 3.0
    out = torch.empty((4, cols), device="cuda")
    call(s, None, out)
    assert bool((out[:2] == 0).all()) and bool(torch.isfinite(out).all())
    s["eps"], s["norm"] = 0.0, "rms"
    call(s, None, out)
    assert bool(torch.isnan(out[0]).all()) and torch.allclose(out[1], torch.ones_like(out[1]), atol=1e-6)


@pytest.mark.parametrize("cols", [64, 1536, 1537])
def test_infinities_and_nan_stay_in_their_rows(cols):
    s = problem(6, cols, "bf16", "bf16", "fp32", norm="layer", post="rms", gate_rows=2)
    s["x"][1, 5] = float("inf")
    s["y"][3, 7] = float("nan")
    out = torch.empty((6, cols), device="cuda")
    x_out = torch.empty_like(s["x"], memory_format=torch.contiguous_format)
    call(s, x_out, out)
    bad = torch.isnan(out).any(1).cpu().tolist()
    assert bad == [False, True, False, True, False, False]
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(x_out[3].float()).all())
    assert bool(torch.isinf(x_out[1, 5])) and bool(torch.isfinite(x_out[[0, 2, 4, 5]].float()).all())
    assert bool(torch.isfinite(out[[0, 2, 4, 5]]).all())


def test_nothing_to_do_and_offsets_past_32_bits():
    s = problem(3, 64)
    api.sdvg_gated_norm(s["x"][:0], torch.empty((0, 64), device="cuda"))
    ld = (1 << 30) + 8
    far = torch.empty((3 * ld,), device="cuda", dtype=torch.bfloat16).view(3, ld)
    far[:, :64] = s["x"]
    out = torch.empty((3 * ld,), device="cuda", dtype=torch.bfloat16).view(3, ld)[:, :64]
    (_, ref), (_, tol) = expected(s)
    call({**s, "x": far[:, :64]}, None, out)
    assert_close(out, ref, tol)


@pytest.mark.parametrize("rows,cols", [(50, 256), (300, 1536), (4680, 5120)])
def test_equal_calls_give_equal_bits_on_streams_and_from_a_graph(rows, cols):
    s = problem(rows, cols, gate_rows=1560, mod_rows=1560, post="rms")
    first = [torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    call(s, *first)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(t) for t in first] for _ in range(3)]
    torch.cuda.synchronize()
    for st, o in zip(streams, outs):
        call(s, *o, stream=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, *outs[2])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, first))


def test_model_sized():
    rows, cols = 4680, 5120
    s = problem(rows, cols, gate_rows=1560, mod_rows=1560, seed=9)
    x_out, out = (torch.full((rows, cols), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    call(s, x_out, out)
    rep = lambda v: v.double().repeat_interleave(1560, 0)
    v = s["x"].double() + rep(s["gate"]) * s["y"].double()
    n = (v - v.mean(1, keepdim=True)) / torch.sqrt(v.var(1, keepdim=True, unbiased=False) + 1e-6)
    o = n * (1 + rep(s["scale"])) + rep(s["shift"])
    # fp32 arithmetic is far below the bf16 rounding: half a step plus 2^-14 of the terms for it
    assert bool(((x_out.double() - v).abs() <= 2.0 ** -8 * v.abs() + 2.0 ** -20 * (v.abs() + 10)).all())
    assert bool(((out.double() - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -14 * (n.abs() + 1) * (1 + rep(s["scale"]).abs())).all())


def test_binding_refuses_mismatched_tensors():
    s = problem(4, 24, gate_rows=2, mod_rows=2, affine=True)
    out = torch.empty((4, 24), device="cuda", dtype=torch.bfloat16)
    for change in (dict(y=s["y"][:3]), dict(gate=s["gate"][:1]), dict(weight=s["weight"].bfloat16()), dict(bias=s["bias"][1:]),
                   dict(scale=s["scale"][:1]), dict(mod_rows=0), dict(x=s["x"].int()), dict(x=s["x"].cpu()),
                   dict(shift=s["shift"].contiguous()), dict(y=None)):
        with pytest.raises((ValueError, api.SdvgError)):
            call({**s, **change}, None, out)
    with pytest.raises(api.SdvgError):
        api.sdvg_gated_norm(s["x"], None)


@pytest.mark.parametrize("cols", [64, 1536, 1537, 20001])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("affine", [False, True])
def test_infinite_scales_travel_as_in_the_formula(cols, norm, affine):
    """In every kernel (a warp per row, a CTA, single columns, long rows); without a bias, whose product with an infinite
    scale may cancel the other term's."""
    s = problem(6, cols, "bf16", "bf16", "fp32", norm=norm, affine=affine, mod_rows=3, gate_rows=2, seed=cols)
    s["bias"] = None
    s["scale"][0, 3], s["scale"][1, 5], s["scale"][1, 7], s["shift"][0, 9] = float("inf"), float("-inf"), float("nan"), float("inf")
    out = torch.empty((6, cols), device="cuda")
    for shift in (s["shift"], None):
        s["shift"] = shift
        (_, ref), _ = expected(s)
        call(s, None, out)
        got = f64(out)
        assert np.isinf(ref[:3, 3]).all() and np.isinf(ref[3:, 5]).all()
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]) and np.array_equal(np.isinf(got), np.isinf(ref))


@pytest.mark.parametrize("cols", [64, 1536, 1537, 20001])
def test_infinite_scales_with_a_bias_of_zero(cols):
    s = problem(6, cols, "bf16", "", "fp32", affine=True, mod_rows=3, seed=cols)
    s["scale"][0, 3], s["scale"][1, 5], s["bias"][3], s["bias"][5] = float("inf"), float("-inf"), 0.0, -0.0
    out = torch.empty((6, cols), device="cuda")
    (_, ref), _ = expected(s)
    call(s, None, out)
    got = f64(out)
    assert np.isinf(ref[:3, 3]).all() and np.isinf(ref[3:, 5]).all() and not np.isnan(ref).any()
    assert np.array_equal(np.isinf(got), np.isinf(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
