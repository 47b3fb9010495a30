"""Host-side checks of the dense operators' C entry points, and pins of their fp64 definitions; no GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import dense_oracle as O
from oracle import sdvg_oracle as SO
from paper_2604_17397_b200 import api, build, synth

X, W, B, G, R, OUT, WS = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


def linear_args(**change):
    a = dict(x=X, ld_x=64, w=W, ld_w=64, bias=B, act=0, gate=None, ld_gate=0, gate_rows=0, residual=None, ld_residual=0,
             out=OUT, ld_out=32, rows=4, cols=32, inner=64, in_type=0, out_type=0, ws=WS, ws_bytes=256, stream=None)
    assert set(change) <= set(a)
    return list({**a, **change}.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "BAD_SHAPE"), (dict(cols=-1), "BAD_SHAPE"), (dict(inner=0), "BAD_SHAPE"),
    (dict(rows=0x7fffffff, ld_x=64), "BAD_SHAPE"), (dict(inner=(1 << 26) + 1, ld_x=1 << 27, ld_w=1 << 27), "BAD_SHAPE"), (dict(ld_x=56), "BAD_SHAPE"), (dict(ld_w=56), "BAD_SHAPE"),
    (dict(ld_out=31), "BAD_SHAPE"), (dict(residual=R, ld_residual=31), "BAD_SHAPE"), (dict(residual=R, ld_residual=-32), "BAD_SHAPE"),
    (dict(gate=G, gate_rows=2, ld_gate=31), "BAD_SHAPE"), (dict(ld_x=1 << 40), "BAD_SHAPE"),
    (dict(in_type=2), "INVALID_ARG"), (dict(in_type=-1), "INVALID_ARG"), (dict(out_type=3), "INVALID_ARG"),
    (dict(act=4), "INVALID_ARG"), (dict(act=-1), "INVALID_ARG"), (dict(gate=G, gate_rows=0, ld_gate=32), "INVALID_ARG"),
    (dict(x=None), "INVALID_ARG"), (dict(w=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"),
    (dict(ws_bytes=255), "INVALID_ARG"),
    (dict(x=X + 8), "MISALIGNED"), (dict(w=W + 2), "MISALIGNED"), (dict(ld_x=68), "MISALIGNED"), (dict(ld_w=65), "MISALIGNED"),
    (dict(out=OUT + 1), "MISALIGNED"), (dict(out=OUT + 2, out_type=2), "MISALIGNED"), (dict(bias=B + 2), "MISALIGNED"),
    (dict(gate=G + 1, gate_rows=4), "MISALIGNED"), (dict(residual=R + 1, ld_residual=0), "MISALIGNED"), (dict(ws=WS + 16), "MISALIGNED"),
])
def test_linear_refuses_on_the_host(lib, change, status):
    assert lib.sdvg_linear(*linear_args(**change)) == getattr(api, "SDVG_ERR_" + status)


def test_linear_with_nothing_to_do(lib):
    assert lib.sdvg_linear(*linear_args(rows=0, x=None, out=None)) == api.SDVG_OK
    assert lib.sdvg_linear(*linear_args(cols=0, w=None)) == api.SDVG_OK


def test_the_binding_refuses_what_is_not_on_a_gpu(lib):
    x, ws = torch.zeros((2, 16), dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError):
        api.sdvg_linear(x, x, x, ws)
    with pytest.raises(ValueError):
        api.sdvg_gated_norm(x, x)
    b = api._binding()
    for call in (lambda: b.linear(x, x, x, ws, None, 0, None, None, 0, 0), lambda: b.linear(None, x, x, ws, None, 0, None, None, 0, 0),
                 lambda: b.gated_norm(x, x, None, None, 0, 0, None, None, 2, None, None, None, None, 0, 1e-6, 0),
                 lambda: b.qk_norm(0, 1, 1, 64, None, x, x, None, None, 0, 1e-6, None, None, 1, 1, 1, 0, x, 1, 0, 1, 0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        b.linear(x)
    with pytest.raises(TypeError):
        b.gated_norm(x)


def norm_args(**change):
    a = dict(x=X, ld_x=32, x_type=0, y=None, ld_y=0, y_type=0, post=0, post_weight=None, gate=None, ld_gate=0, gate_rows=0,
             x_out=None, ld_x_out=0, norm=2, weight=None, bias=None, scale=None, shift=None, ld_mod=0, mod_rows=0, eps=1e-6,
             out=OUT, ld_out=32, out_type=0, rows=4, cols=32, stream=None)
    assert set(change) <= set(a)
    return list({**a, **change}.values())


Y = dict(y=W, ld_y=32)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "BAD_SHAPE"), (dict(cols=0), "BAD_SHAPE"), (dict(ld_x=31), "BAD_SHAPE"), (dict(y=W, ld_y=31), "BAD_SHAPE"),
    (dict(ld_out=31), "BAD_SHAPE"), (dict(x_out=R, ld_x_out=31), "BAD_SHAPE"), (dict(scale=G, mod_rows=2, ld_mod=31), "BAD_SHAPE"),
    (dict(gate=G, gate_rows=2, ld_gate=31, **Y), "BAD_SHAPE"),
    (dict(norm=3), "INVALID_ARG"), (dict(post=-1, **Y), "INVALID_ARG"), (dict(x_type=3), "INVALID_ARG"),
    (dict(out_type=-1), "INVALID_ARG"), (dict(y_type=3, **Y), "INVALID_ARG"), (dict(eps=-1e-6), "INVALID_ARG"),
    (dict(eps=math.nan), "INVALID_ARG"), (dict(eps=math.inf), "INVALID_ARG"), (dict(post=1), "INVALID_ARG"),
    (dict(post_weight=B), "INVALID_ARG"), (dict(gate=G, gate_rows=4), "INVALID_ARG"), (dict(gate=G, gate_rows=0, **Y), "INVALID_ARG"),
    (dict(shift=G, mod_rows=0), "INVALID_ARG"), (dict(x=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(x=X + 1), "MISALIGNED"), (dict(x_type=2, x=X + 2), "MISALIGNED"), (dict(y=W + 1, ld_y=32), "MISALIGNED"),
    (dict(out=OUT + 1), "MISALIGNED"), (dict(weight=B + 2), "MISALIGNED"), (dict(scale=G + 2, mod_rows=4), "MISALIGNED"),
])
def test_gated_norm_refuses_on_the_host(lib, change, status):
    assert lib.sdvg_gated_norm(*norm_args(**change)) == getattr(api, "SDVG_ERR_" + status)


def test_gated_norm_with_nothing_to_do(lib):
    assert lib.sdvg_gated_norm(*norm_args(rows=0, x=None, out=None)) == api.SDVG_OK


def test_qk_norm_refuses_on_the_host(lib):
    import ctypes as C
    h, h8, wide = C.c_void_p(), C.c_void_p(), C.c_void_p()
    assert lib.sdvg_cache_create(C.byref(h), 0x10000, 0x20000, 3, 2, 64, 64) == api.SDVG_OK
    assert lib.sdvg_cache_create_e4m3(C.byref(h8), 0x10000, 0x20000, 3, 2, 64, 128) == api.SDVG_OK
    assert lib.sdvg_cache_create(C.byref(wide), 0x10000, 0x20000, 3, 129, 64, 128) == api.SDVG_OK
    base = dict(cache=h, q=X, ld_q=128, k=W, ld_k=128, v=B, ld_v=384, q_weight=G, k_weight=None, scope=0, eps=1e-6, q_out=OUT,
                k_out=None, frames=1, grid_h=8, grid_w=8, frame_offset=0, tab=0x80000, tab_frames=4, block=0,
                flags=api.SDVG_STAGE, evicted=None, stream=None)
    for change, status in [
            (dict(cache=None), "INVALID_ARG"), (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"),
            (dict(q=None), "INVALID_ARG"), (dict(q_out=None), "INVALID_ARG"), (dict(scope=2), "INVALID_ARG"),
            (dict(eps=-1.0), "INVALID_ARG"), (dict(eps=math.nan), "INVALID_ARG"), (dict(tab=None), "INVALID_ARG"),
            (dict(flags=3), "INVALID_ARG"), (dict(cache=h8), "BAD_SHAPE"), (dict(ld_q=120), "BAD_SHAPE"),
            (dict(ld_k=64), "BAD_SHAPE"), (dict(ld_v=0), "BAD_SHAPE"), (dict(grid_w=7), "BAD_SHAPE"),
            (dict(cache=wide, ld_q=20000, ld_k=20000, ld_v=20000), "BAD_SHAPE"),
            (dict(ld_k=132), "MISALIGNED"), (dict(q=X + 8), "MISALIGNED"), (dict(q_weight=G + 4), "MISALIGNED"),
            (dict(q_out=OUT + 2), "MISALIGNED"), (dict(block=1), "BAD_STATE"), (dict(frame_offset=4), "BAD_STATE")]:
        assert lib.sdvg_qk_norm_rope3d_commit(*{**base, **change}.values()) == getattr(api, "SDVG_ERR_" + status), change
    for c in (h, h8, wide):
        lib.sdvg_cache_destroy(c)


# ---- the definitions against library routines and closed forms -------------------------------------------------

def test_activations_are_torchs():
    v = torch.linspace(-12, 12, 1001, dtype=torch.float64)
    for act, ref in (("silu", torch.nn.functional.silu(v)), ("gelu", torch.nn.functional.gelu(v)),
                     ("gelu_tanh", torch.nn.functional.gelu(v, approximate="tanh"))):
        assert np.allclose(O.activation(v.numpy(), act), ref.numpy(), rtol=1e-10, atol=1e-14)


def test_norms_are_torchs_and_compose():
    gen = torch.Generator().manual_seed(0)
    x, y = (torch.randn((6, 40), generator=gen, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(40, generator=gen, dtype=torch.float64) for _ in range(2))
    g, sc, sh = (torch.randn((n, 40), generator=gen, dtype=torch.float64) for n in (2, 3, 3))
    s, o = O.gated_norm_ref(x.numpy(), y.numpy(), "rms", w.numpy(), g.numpy(), 4, "layer", None, b.numpy(), sc.numpy(),
                            sh.numpy(), 2, 1e-5)
    s_t = x + g.repeat_interleave(4, 0)[:6] * torch.nn.functional.rms_norm(y, (40,), w, 1e-5)
    o_t = (torch.nn.functional.layer_norm(s_t, (40,), eps=1e-5) + b) * (1 + sc.repeat_interleave(2, 0)) + sh.repeat_interleave(2, 0)
    assert np.allclose(s, s_t.numpy(), atol=1e-13) and np.allclose(o, o_t.numpy(), atol=1e-13)


def test_linear_is_torchs():
    gen = torch.Generator().manual_seed(1)
    x, w, b = torch.randn((5, 9), generator=gen), torch.randn((4, 9), generator=gen), torch.randn(4, generator=gen)
    ref = torch.nn.functional.gelu(torch.nn.functional.linear(x.double(), w.double(), b.double()))
    gate, res = torch.randn((2, 4), generator=gen).double(), torch.randn((5, 4), generator=gen).double()
    got = O.linear_ref(x.double().numpy(), w.double().numpy(), b.double().numpy(), "gelu", gate.numpy(), 3, res.numpy())
    assert np.allclose(got, (res + gate[[0, 0, 0, 1, 1]] * ref).numpy(), atol=1e-12)


@pytest.mark.parametrize("scope", ["row", "head"])
def test_qk_norm_without_scaling_is_the_rotary_embedding(scope):
    """Rows of +-1 (unit mean square) and eps = 0: the norm is the identity, what is left is the pinned rotation."""
    gen = np.random.default_rng(2)
    grid, dim, heads = (2, 3, 4), 64, 2
    x = gen.choice([-1.0, 1.0], (24, heads, dim))
    tab = SO.rope_table(dim, 6, 3, 4)
    got = O.qk_norm_rope_ref(x, None, scope, 0.0, grid, 4, tab, 6)
    ref = SO.rope_ref(synth.f32_to_bf16_bits(x.astype(np.float32)), grid, 4)
    assert np.allclose(got, ref, atol=1e-6)


def test_overlapped_kernels_do_not_read_through_the_read_only_path():
    """A kernel that starts under the end of the one before it may read what that one writes; non-coherent loads are allowed only
    for data that nothing writes while the kernel lives."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(build.__file__), "csrc")
    text = {f: re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read()) for f in os.listdir(csrc)}
    overlapped = [f for f, t in text.items() if f.endswith(".cu") and "overlap_wait()" in t]
    assert {"gated_norm.cu", "linear.cu", "qk_norm.cu"} <= set(overlapped)
    for f in overlapped + ["row_team.cuh", "elem_types.cuh"]:
        assert not re.search(r"__ldg\w*\(|ld\.global\S*\.nc|__restrict__", text[f]), f


class OnPaper(torch.Tensor):
    """A tensor that says it is on a GPU and has no memory: the binding takes it, and the library refuses its null address."""

    @staticmethod
    def __new__(cls, *shape, dtype=torch.bfloat16):
        return torch.Tensor._make_wrapper_subclass(cls, shape, dtype=dtype, device="cuda")

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError


def without_address(*shape, dtype):
    """One whose address cannot be asked for, as that of a tensor that is being traced."""
    t = OnPaper(*shape, dtype=dtype)
    torch._C._set_throw_on_mutable_data_ptr(t)
    return t


def linear_on_paper(**change):
    a = dict(x=OnPaper(4, 64), w=OnPaper(8, 64), out=OnPaper(4, 8), ws=OnPaper(256, dtype=torch.uint8), bias=None, act=0, residual=None,
             gate=None, gate_rows=0, stream=0)
    return api._binding().linear(*{**a, **change}.values())


def qk_on_paper(cache, **change):
    block = lambda: OnPaper(64, 2, 64)
    a = dict(handle=cache.value, tokens=64, heads=2, dim=64, q=None, k=block(), v=block(), q_weight=None, k_weight=None, scope=0, eps=1e-6,
             q_out=None, k_out=None, frames=1, grid_h=8, grid_w=8, offset=0,
             table=OnPaper(api.lib().sdvg_rope3d_table_floats(64, 4, 8, 8), dtype=torch.float32), tab_frames=4, block=0,
             flags=api.SDVG_STAGE, stream=0)
    return api._binding().qk_norm(*{**a, **change}.values())


@pytest.fixture
def ring(lib):
    import ctypes as C
    h = C.c_void_p()
    assert lib.sdvg_cache_create(C.byref(h), 0x10000, 0x20000, 3, 2, 64, 64) == api.SDVG_OK
    yield h
    lib.sdvg_cache_destroy(h)


def test_a_tensor_without_an_address_raises(ring):
    """In every place: also the ones read last, just before the interpreter lock is given up."""
    assert linear_on_paper() == api.SDVG_ERR_INVALID_ARG and qk_on_paper(ring) == -1000 - api.SDVG_ERR_INVALID_ARG
    for change in (dict(ws=without_address(256, dtype=torch.uint8)), dict(x=without_address(4, 64, dtype=torch.bfloat16)),
                   dict(bias=without_address(8, dtype=torch.float32))):
        with pytest.raises(RuntimeError):
            linear_on_paper(**change)
    n = api.lib().sdvg_rope3d_table_floats(64, 4, 8, 8)
    for change in (dict(table=without_address(n, dtype=torch.float32)), dict(v=without_address(64, 2, 64, dtype=torch.bfloat16))):
        with pytest.raises(RuntimeError):
            qk_on_paper(ring, **change)
    x = OnPaper(4, 64)
    with pytest.raises(RuntimeError):
        api._binding().gated_norm(x, without_address(4, 64, dtype=torch.bfloat16), None, None, 0, 0, None, None, 2, None, None, None, None, 0,
                                  1e-6, 0)


def test_the_binding_refuses_a_rotary_table_that_is_too_short(ring):
    n = api.lib().sdvg_rope3d_table_floats(64, 4, 8, 8)
    table = lambda floats: OnPaper(floats, dtype=torch.float32)
    reached = -1000 - api.SDVG_ERR_INVALID_ARG                  # the library, which refuses the null addresses
    assert qk_on_paper(ring, table=table(n)) == qk_on_paper(ring, table=table(n + 5)) == reached
    for change in (dict(table=table(n - 1)), dict(tab_frames=5), dict(grid_h=9), dict(grid_w=1 << 20), dict(tab_frames=1 << 30),
                   dict(table=OnPaper(n, dtype=torch.bfloat16))):
        with pytest.raises(ValueError, match="table"):
            qk_on_paper(ring, **change)
    assert qk_on_paper(ring, tab_frames=0) == qk_on_paper(ring, grid_h=0) == reached


@pytest.mark.parametrize("change", [dict(cols=0x7fffffff), dict(cols=0x7fffffff - 1023), dict(rows=0x7fffffff), dict(rows=0x7fffffff - 1023),
                                    dict(cols=0x7fffffff - 100, y=W, ld_y=1 << 31)])
def test_gated_norm_refuses_extents_at_the_end_of_an_int(lib, change):
    """A column counter that steps by the threads of a CTA, or rows rounded up to whole CTAs, would pass the end of its type."""
    wide = dict(ld_x=1 << 31, ld_out=1 << 31) if "cols" in change else {}
    assert lib.sdvg_gated_norm(*norm_args(**{**wide, **change})) == api.SDVG_ERR_BAD_SHAPE


def test_gated_norm_takes_extents_just_below(lib):
    for change in (dict(cols=0x7fffffff - 1024, ld_x=1 << 31, ld_out=1 << 31), dict(rows=0x7fffffff - 1024)):
        # everything is checked before the pointers' alignment
        assert lib.sdvg_gated_norm(*norm_args(**change, out=OUT + 1)) == api.SDVG_ERR_MISALIGNED


def test_rotary_tables_past_32_bits_are_refused(lib, ring):
    """Offsets into the table are ints, in (cos, sin) pairs: 12 per frame position and 10 per row and column with head_dim 64."""
    most = (2 ** 31 - 1 - 8 * 20) // 12

    def commit(tab_frames, offset=0):
        return lib.sdvg_qk_norm_rope3d_commit(ring, X, 128, W, 128, B, 128, None, None, 0, 1e-6, OUT, None, 1, 8, 8, offset, G, tab_frames, 1,
                                              api.SDVG_STAGE, None, None)

    def rope(tab_frames, offset=0):
        return lib.sdvg_rope3d_qk(X, W, OUT, R, 64, 2, 64, 1, 8, 8, offset, G, tab_frames, None)

    for call in (commit, rope):
        for tab_frames in (most + 1, 1 << 30, 2 ** 31 - 1):
            assert call(tab_frames) == call(tab_frames, tab_frames - 1) == api.SDVG_ERR_BAD_SHAPE
        assert call(most, most) == api.SDVG_ERR_BAD_STATE       # past the table's frames: the next check
    assert commit(most) == api.SDVG_ERR_BAD_STATE               # block 1 before block 0
