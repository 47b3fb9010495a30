"""sdvg_linear against fp64: out = residual + gate * act(x W^T + bias)."""
import math

import numpy as np
import pytest
import torch

from dense_utils import DTYPES, assert_close, f64, linear_tolerance, rounding
from oracle import dense_oracle as O
from paper_2604_17397_b200 import api

pytestmark = pytest.mark.gpu

ACTS = {"none": api.SDVG_ACT_NONE, "silu": api.SDVG_ACT_SILU, "gelu_tanh": api.SDVG_ACT_GELU_TANH, "gelu": api.SDVG_ACT_GELU}


def randn(gen, *shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda") * std


def strided(gen, rows, cols, dtype, std=1.0, ld=None, fill=None):
    """[rows, cols] view of a wider buffer; what lies between the rows is NaN."""
    ld = ld or -(-cols // 8) * 8
    buf = torch.full((rows, ld), float("nan"), device="cuda", dtype=dtype)
    buf[:, :cols] = randn(gen, rows, cols, std=std).to(dtype) if fill is None else fill
    return buf[:, :cols]


def problem(rows, cols, inner, dtype="bf16", out="", act="none", bias=True, gate_rows=0, residual="", seed=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, o = DTYPES[dtype], DTYPES[out or dtype]
    s = dict(x=strided(gen, rows, inner, t), w=strided(gen, cols, inner, t, std=std / math.sqrt(inner)), act=act,
             gate_rows=gate_rows, o=o)
    s["bias"] = randn(gen, cols) if bias else None
    s["gate"] = randn(gen, -(-rows // gate_rows), cols) if gate_rows else None
    s["residual"] = None
    if residual:
        s["residual"] = randn(gen, rows if residual == "rows" else 1, cols, std=2.0).to(o).expand(rows, cols)
    return s


def call(s, out, ws, stream=None):
    api.sdvg_linear(s["x"], s["w"], out, ws, bias=s["bias"], act=ACTS[s["act"]], residual=s["residual"], gate=s["gate"],
                    gate_rows=s["gate_rows"], stream=stream)


def expected(s):
    x, w, b, g, r = (f64(s[k]) for k in ("x", "w", "bias", "gate", "residual"))
    ref = O.linear_ref(x, w, b, s["act"], g, s["gate_rows"], r)
    per_row = None if g is None else O.of_rows(g, x.shape[0], s["gate_rows"])
    return ref, linear_tolerance(x, w, b, s["act"], per_row, r, ref, s["o"])


def check(s, ld_out=None, in_place=False):
    ws = api.attn_workspace()
    rows, cols = s["x"].shape[0], s["w"].shape[0]
    ref, tol = expected(s)
    ld = ld_out or cols
    buf = torch.full((rows + 2, ld), 77.0, device="cuda", dtype=s["o"])     # a row before, a row after
    out = buf[1:rows + 1, :cols]
    if in_place:
        out.copy_(s["residual"])
        s["residual"] = out
    call(s, out, ws)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK
    assert_close(out, ref, tol)
    assert bool((buf[0] == 77).all()) and bool((buf[rows + 1] == 77).all()) and bool((buf[:, cols:] == 77).all())
    return out


SHAPES = [(1, 1, 1), (1, 1536, 256), (2, 5, 7), (3, 130, 72), (15, 128, 64), (16, 127, 63), (17, 129, 65), (33, 100, 200),
          (64, 257, 100), (127, 64, 640), (128, 300, 130), (129, 260, 515), (255, 129, 257), (256, 256, 128),
          (257, 127, 191), (300, 515, 1000), (513, 70, 64), (1000, 640, 72)]


@pytest.mark.parametrize("rows,cols,inner", SHAPES)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp32")])
def test_shapes(rows, cols, inner, dtype, out):
    check(problem(rows, cols, inner, dtype, out, gate_rows=max(1, rows // 3), residual="rows", seed=rows + cols + inner))


@pytest.mark.parametrize("rows,cols,inner", [(1, 100, 9001), (2, 129, 1030), (16, 130, 2048), (31, 257, 4097), (33, 129, 5000),
                                             (48, 500, 1500), (64, 1000, 2050), (64, 128, 20000), (65, 130, 4000)])
@pytest.mark.parametrize("dtype,out", [("bf16", "fp32"), ("fp16", "fp16")])
def test_few_rows_share_long_sums(rows, cols, inner, dtype, out):
    """Up to 64 rows: clusters that split the inner axis unevenly, chunks of fp32 sums that end inside a part."""
    check(problem(rows, cols, inner, dtype, out, gate_rows=5, residual="rows", act="silu", seed=inner))


@pytest.mark.parametrize("rows,cols,inner", [(3, 1024, 5120), (64, 256, 6144), (300, 512, 6144), (257, 256, 20000)])
def test_fp32_outputs_keep_fp32_accuracy_over_long_sums(rows, cols, inner):
    """Accumulated in one go, the tensor core's truncation drifts: 3.7e-6 at inner 5120, and more beyond.  In chunks of at most 640 it stays
    at most 40 truncated additions of 2^-23 of a partial sum that is on average far below the full one: under 2^-20."""
    s = problem(rows, cols, inner, out="fp32", bias=False)
    out = torch.empty((rows, cols), device="cuda")
    call(s, out, api.attn_workspace())
    ref = s["x"].double() @ s["w"].double().t()
    assert float((out.double() - ref).norm() / ref.norm()) <= 2.0 ** -20


def test_two_graphs_that_share_a_workspace_replay_at_once():
    ws = api.attn_workspace()
    cases = []
    for rows, cols, inner in ((8, 512, 4096), (700, 512, 1024)):
        s = problem(rows, cols, inner, act="silu", seed=rows)
        out = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16)
        call(s, out, ws)
        want, graph, stream = out.clone(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(5):
                call(s, out, ws)
        out.zero_()
        cases.append((out, want, graph, stream))
    torch.cuda.synchronize()
    for _ in range(10):
        for _, _, graph, stream in cases:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out, want, _, _ in cases)
    assert api.sdvg_block_attn_status(ws) == api.SDVG_OK


def test_calls_from_two_threads():
    import threading
    results, failures = {}, []

    def work(i):
        try:
            torch.cuda.set_device(0)
            s = problem(40 + 300 * i, 200, 700, act="gelu", seed=i)
            stream = torch.cuda.Stream()
            ws = api.attn_workspace()
            out = torch.empty((s["x"].shape[0], 200), device="cuda", dtype=torch.bfloat16)
            torch.cuda.synchronize()
            for _ in range(50):
                call(s, out, ws, stream=stream)
            stream.synchronize()
            results[i] = (s, out)
        except Exception as e:                                # reported by the main thread
            failures.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for s, out in results.values():
        ref, tol = expected(s)
        assert_close(out, ref, tol)


def test_a_row_of_dependent_calls_sees_each_others_results():
    """Launches overlap the end of the one before; their reads must not."""
    gen = torch.Generator(device="cuda").manual_seed(31)
    ws = api.attn_workspace()
    w = [strided(gen, 256, 256, torch.bfloat16, std=1 / 16) for _ in range(3)]
    for rows in (3, 64, 500):
        x = strided(gen, rows, 256, torch.bfloat16)
        bufs = [torch.zeros((rows, 256), device="cuda", dtype=torch.bfloat16) for _ in range(3)]

        def chain(sync):
            cur = x
            for i in range(30):
                api.sdvg_linear(cur, w[i % 3], bufs[i % 3], ws, act=api.SDVG_ACT_SILU if i % 2 else api.SDVG_ACT_NONE, residual=cur)
                if sync:
                    torch.cuda.synchronize()
                api.sdvg_gated_norm(bufs[i % 3], bufs[i % 3])
                if sync:
                    torch.cuda.synchronize()
                cur = bufs[i % 3]
            torch.cuda.synchronize()
            return cur.clone()

        want = chain(True)
        assert all(torch.equal(chain(False), want) for _ in range(5))
        assert bool(torch.isfinite(want.float()).all())


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32")])
@pytest.mark.parametrize("rows", [5, 270])
def test_activations_and_types(act, dtype, out, rows):
    check(problem(rows, 140, 192, dtype, out, act=act, seed=3, std=3.0))


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("gate_rows", [1, 7, 32, 300, 1000])
@pytest.mark.parametrize("residual", ["", "rows", "broadcast"])
def test_gate_groups_and_residuals(rows, gate_rows, residual):
    check(problem(rows, 133, 96, gate_rows=gate_rows, residual=residual, bias=gate_rows != 7, act="silu", seed=gate_rows))


@pytest.mark.parametrize("rows,ld_out", [(5, 131), (70, 200), (300, 133)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_output_rows_of_any_stride_and_in_place_residual(rows, ld_out, out):
    check(problem(rows, 129, 80, out=out, residual="rows", gate_rows=11), ld_out=ld_out)
    check(problem(rows, 129, 80, out=out, residual="rows", gate_rows=11), ld_out=ld_out, in_place=True)


def test_column_ranges_of_wider_operands():
    gen = torch.Generator(device="cuda").manual_seed(8)
    s = problem(50, 96, 64, seed=8)
    wide_x, wide_w = randn(gen, 50, 400).bfloat16(), randn(gen, 96, 256, std=0.1).bfloat16()
    s["x"], s["w"] = wide_x[:, 136:200], wide_w[:, 64:128]
    wide_gate = randn(gen, 5, 3 * 96)
    s["gate"], s["gate_rows"] = wide_gate[:, 96:192], 10
    check(s)


@pytest.mark.parametrize("rows", [4, 300])
def test_infinities_and_nan_stay_in_their_rows_and_columns(rows):
    s = problem(rows, 150, 100, seed=5)
    s["x"][1, 3] = float("inf")
    s["x"][2, 4] = float("nan")
    s["w"][7, 9] = float("nan")
    s["bias"][11] = float("-inf")
    ws = api.attn_workspace()
    out = torch.empty((rows, 150), device="cuda", dtype=torch.bfloat16)
    call(s, out, ws)
    with np.errstate(invalid="ignore"):
        ref = f64(s["x"]) @ f64(s["w"]).T + f64(s["bias"])
    got = f64(out)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
    clean = np.isfinite(ref)
    s2 = problem(rows, 150, 100, seed=5)
    ref2, tol = expected(s2)
    assert np.all(np.abs(got[clean] - ref2[clean]) <= tol[clean])


def test_half_precision_overflow_is_infinite_as_a_cast_is():
    x = torch.full((3, 64), 100.0, device="cuda", dtype=torch.float16)
    w = torch.full((2, 64), 100.0, device="cuda", dtype=torch.float16)
    w[1] = -100.0
    out = torch.empty((3, 2), device="cuda", dtype=torch.float16)
    api.sdvg_linear(x, w, out, api.attn_workspace())
    assert f64(out)[:, 0].tolist() == [math.inf] * 3 and f64(out)[:, 1].tolist() == [-math.inf] * 3


@pytest.mark.parametrize("act", ["silu", "gelu_tanh", "gelu"])
def test_activations_far_out(act):
    v = torch.tensor([-3e4, -200.0, -88.0, -30.0, -10.0, -5.0, -1.0, -1e-3, 0.0, 1e-3, 1.0, 10.0, 100.0, 3e4], device="cuda")
    x = torch.zeros((1, 8), device="cuda", dtype=torch.bfloat16)
    w = torch.zeros((len(v), 8), device="cuda", dtype=torch.bfloat16)
    out = torch.empty((1, len(v)), device="cuda")
    api.sdvg_linear(x, w, out, api.attn_workspace(), bias=v, act=ACTS[act])
    ref = O.activation(f64(v), act)[None]
    assert_close(out, ref, 2.0 ** -14 * np.abs(ref) + 1e-36)


def test_nothing_to_do():
    ws = api.attn_workspace()
    x, w = torch.zeros((4, 16), device="cuda", dtype=torch.bfloat16), torch.zeros((8, 16), device="cuda", dtype=torch.bfloat16)
    api.sdvg_linear(x[:0], w, torch.empty((0, 8), device="cuda"), ws)
    api.sdvg_linear(x, w[:0], torch.empty((4, 0), device="cuda"), ws)


@pytest.mark.parametrize("rows,cols,inner", [(3, 640, 2048), (200, 384, 1024), (700, 512, 512)])
def test_equal_calls_give_equal_bits_on_any_stream_and_from_a_graph(rows, cols, inner):
    s = problem(rows, cols, inner, act="gelu_tanh", gate_rows=64, residual="rows", out="fp32")
    ws = api.attn_workspace()
    first = torch.empty((rows, cols), device="cuda")
    call(s, first, ws)
    torch.cuda.synchronize()
    # two streams at once, one workspace each
    streams, outs, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(first) for _ in range(2)], \
        [api.attn_workspace() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, o, w in zip(streams, outs, spaces):
            call(s, o, w, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    # captured and replayed on new inputs
    again = torch.zeros_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(s, again, ws)
    keep = s["x"].clone()
    s["x"].copy_(torch.flip(keep, (0,)))
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(again, first)
    s["x"].copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, first)
    assert all(api.sdvg_block_attn_status(w) == api.SDVG_OK for w in [ws] + spaces)


def test_offsets_past_32_bits():
    ld = (1 << 30) + 8
    s = problem(5, 40, 48, out="bf16", residual="rows")
    big = torch.empty((5 * ld,), device="cuda", dtype=torch.bfloat16)
    out = big.view(5, ld)[:, :40]
    far = torch.empty((5 * ld,), device="cuda", dtype=torch.bfloat16).view(5, ld)
    far[:, :48] = s["x"]
    ref, tol = expected(s)
    s["x"] = far[:, :48]
    call(s, out, api.attn_workspace())
    assert_close(out, ref, tol)


@pytest.mark.parametrize("rows,cols,inner", [(1560, 1536, 1536), (4680, 512, 768), (2, 15360, 5120)])
def test_model_sized(rows, cols, inner):
    s = problem(rows, cols, inner, act="gelu_tanh", gate_rows=1560, residual="rows", seed=21)
    x, w = s["x"].double(), s["w"].double()
    v = x @ w.t() + s["bias"].double()
    a = v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))
    g = s["gate"].double().repeat_interleave(1560, 0)[:rows]
    ref = a * g + s["residual"].double()
    err = (inner + 2) * 2.0 ** -23 * (x.abs() @ w.abs().t() + s["bias"].double().abs())
    err = g.abs() * (1.13 * err + 2.0 ** -14 * a.abs()) + 2.0 ** -22 * (g.abs() * a.abs() + s["residual"].double().abs())
    tol = err + 2.0 ** -8 * (ref.abs() + err)
    out = torch.full((rows, cols), float("nan"), device="cuda", dtype=torch.bfloat16)
    call(s, out, api.attn_workspace())
    assert bool(((out.double() - ref).abs() <= tol).all())


def test_binding_refuses_mismatched_tensors():
    ws = api.attn_workspace()
    s = problem(4, 24, 16)
    out = torch.empty((4, 24), device="cuda", dtype=torch.bfloat16)
    for change in (dict(w=s["w"].half()), dict(bias=s["bias"][:-1]), dict(bias=s["bias"].half()), dict(residual=out[:3]),
                   dict(residual=out.float()), dict(gate=torch.ones((2, 24), device="cuda"), gate_rows=1),
                   dict(gate=torch.ones((1, 24), device="cuda"), gate_rows=0), dict(x=s["x"].t()), dict(x=s["x"].cpu())):
        with pytest.raises((ValueError, api.SdvgError)):
            call({**s, **change}, out, ws)
    shifted = torch.zeros((4 * 16 + 1,), device="cuda", dtype=torch.bfloat16)[1:].view(4, 16)
    with pytest.raises(api.SdvgError) as e:
        call({**s, "x": shifted}, out, ws)
    assert e.value.status == api.SDVG_ERR_MISALIGNED


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
def test_activations_of_infinities_nan_and_the_largest_values(act, rows, out):
    """In both kernels, whether the infinity comes from the bias or from a sum past the range of fp32."""
    v = torch.tensor([math.inf, -math.inf, math.nan, 3e38, -3e38, 1e20, -1e20, 40.0, -40.0, 0.0, 0.0], device="cuda")
    x = torch.full((rows, 8), 2.0 ** 100, device="cuda", dtype=torch.bfloat16)
    w = torch.zeros((len(v), 8), device="cuda", dtype=torch.bfloat16)
    w[-2], w[-1] = 2.0 ** 100, -(2.0 ** 100)
    got = torch.zeros((rows, len(v)), device="cuda", dtype=DTYPES[out])
    api.sdvg_linear(x, w, got, api.attn_workspace(), bias=v, act=ACTS[act])
    sums = f64(v)
    sums[-2:] = math.inf, -math.inf
    with np.errstate(invalid="ignore"):
        ref = np.broadcast_to(O.activation(sums, act), (rows, len(v)))
    with np.errstate(invalid="ignore"):
        tol = 2.0 ** -14 * np.abs(ref) + 1e-36 + rounding(ref, DTYPES[out])
    assert_close(got, ref, tol)
