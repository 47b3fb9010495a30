"""Host-side checks of the 8-bit dense operators' C entry points, and pins of their fp64 definitions; no GPU."""
import numpy as np
import pytest
import torch

from oracle import e4m3_blocks_oracle as B
from oracle import sdvg_oracle as O
from paper_2604_17397_b200 import api, build
from test_dense_cpu import OnPaper, without_address

X, XS, W, WS, B_, G, R, OUT, OS, SPACE = (0x10000 * i for i in range(1, 11))


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


def linear_args(**change):
    a = dict(x=X, ld_x=64, xs=XS, ld_xs=4, w=W, ld_w=64, ws=WS, ld_ws=4, w_rows=128, bias=B_, act=0, gate=None, ld_gate=0, gate_rows=0,
             residual=None, ld_residual=0, out=OUT, ld_out=32, os=None, ld_os=0, rows=4, cols=32, inner=64, out_type=0, space=SPACE,
             space_bytes=256, stream=None)
    assert set(change) <= set(a)
    return list({**a, **change}.values())


OUT8 = dict(out_type=3, os=OS, ld_os=1)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "BAD_SHAPE"), (dict(cols=-1), "BAD_SHAPE"), (dict(inner=0), "BAD_SHAPE"), (dict(rows=0x7fffffff), "BAD_SHAPE"),
    (dict(inner=(1 << 26) + 1, ld_x=1 << 27, ld_w=1 << 27), "BAD_SHAPE"), (dict(ld_x=48), "BAD_SHAPE"), (dict(ld_w=48), "BAD_SHAPE"),
    (dict(ld_out=31), "BAD_SHAPE"), (dict(ld_xs=0), "BAD_SHAPE"), (dict(cols=129, ld_out=129, ld_ws=0), "BAD_SHAPE"),
    (dict(w_rows=1, ld_ws=0), "BAD_SHAPE"), (dict(inner=513, ld_x=528, ld_w=528), "BAD_SHAPE"),
    (dict(residual=R, ld_residual=31), "BAD_SHAPE"), (dict(gate=G, gate_rows=2, ld_gate=31), "BAD_SHAPE"),
    (dict(ld_x=1 << 40), "BAD_SHAPE"), (dict(**{**OUT8, "ld_os": 0}), "BAD_SHAPE"),
    (dict(out_type=4), "INVALID_ARG"), (dict(out_type=-1), "INVALID_ARG"), (dict(act=4), "INVALID_ARG"), (dict(w_rows=64), "INVALID_ARG"),
    (dict(w_rows=0), "INVALID_ARG"), (dict(gate=G, gate_rows=0, ld_gate=32), "INVALID_ARG"), (dict(out_type=3), "INVALID_ARG"),
    (dict(os=OS, ld_os=1), "INVALID_ARG"), (dict(residual=R, ld_residual=32, **OUT8), "INVALID_ARG"),
    (dict(x=None), "INVALID_ARG"), (dict(xs=None), "INVALID_ARG"), (dict(w=None), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"),
    (dict(out=None), "INVALID_ARG"), (dict(space=None), "INVALID_ARG"), (dict(space_bytes=255), "INVALID_ARG"),
    (dict(x=X + 8), "MISALIGNED"), (dict(w=W + 4), "MISALIGNED"), (dict(ld_x=72), "MISALIGNED"), (dict(ld_w=65), "MISALIGNED"),
    (dict(xs=XS + 2), "MISALIGNED"), (dict(ws=WS + 1), "MISALIGNED"), (dict(ld_xs=5), "MISALIGNED"),
    (dict(cols=129, ld_out=129, ld_ws=6), "MISALIGNED"), (dict(out=OUT + 1), "MISALIGNED"), (dict(out=OUT + 2, out_type=2), "MISALIGNED"),
    (dict(bias=B_ + 2), "MISALIGNED"), (dict(gate=G + 1, gate_rows=4), "MISALIGNED"), (dict(space=SPACE + 16), "MISALIGNED"),
])
def test_linear_refuses_on_the_host(lib, change, status):
    assert lib.sdvg_linear_e4m3(*linear_args(**change)) == getattr(api, "SDVG_ERR_" + status)


def test_strides_of_single_rows_are_not_looked_at(lib):
    one = dict(rows=1, cols=1, ld_x=0, ld_xs=0, ld_w=0, ld_ws=0, ld_out=0, space=SPACE + 16)
    assert lib.sdvg_linear_e4m3(*linear_args(**one)) == api.SDVG_ERR_MISALIGNED          # the workspace, checked last
    assert lib.sdvg_linear_e4m3(*linear_args(**{**one, **OUT8, "ld_os": 0, "out": OUT + 1})) == api.SDVG_ERR_MISALIGNED


def test_nothing_to_do(lib):
    assert lib.sdvg_linear_e4m3(*linear_args(rows=0, x=None, out=None)) == api.SDVG_OK
    assert lib.sdvg_linear_e4m3(*linear_args(cols=0, w=None)) == api.SDVG_OK
    assert lib.sdvg_quant_e4m3_blocks(None, 0, 0, None, 0, None, 0, 1, 0, 8, None) == api.SDVG_OK
    assert lib.sdvg_dequant_e4m3_blocks(None, 0, None, 0, 128, None, 0, 2, 8, 0, None) == api.SDVG_OK


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "BAD_SHAPE"), (dict(cols=-1), "BAD_SHAPE"), (dict(rows=0x7fffffff), "BAD_SHAPE"), (dict(ld_x=199), "BAD_SHAPE"),
    (dict(ld_8=199), "BAD_SHAPE"), (dict(ld_s=1), "BAD_SHAPE"), (dict(rows=2 ** 31 - 1025, cols=2 ** 20, ld_x=2 ** 20, ld_8=2 ** 20,
                                                                      ld_s=2 ** 20), "BAD_SHAPE"),
    (dict(type=3), "INVALID_ARG"), (dict(type=-1), "INVALID_ARG"), (dict(block=2), "INVALID_ARG"), (dict(block=0), "INVALID_ARG"),
    (dict(x=None), "INVALID_ARG"), (dict(x8=None), "INVALID_ARG"), (dict(scale=None), "INVALID_ARG"),
    (dict(x=X + 1), "MISALIGNED"), (dict(type=2, x=X + 2), "MISALIGNED"),
])
def test_quantisation_refuses_on_the_host(lib, change, status):
    a = dict(x=X, ld_x=200, type=0, x8=OUT, ld_8=200, scale=OS, ld_s=2, block=1, rows=300, cols=200)
    assert set(change) <= set(a)
    x, ld_x, t, x8, ld_8, s, ld_s, block, rows, cols = {**a, **change}.values()
    want = getattr(api, "SDVG_ERR_" + status)
    assert lib.sdvg_quant_e4m3_blocks(x, ld_x, t, x8, ld_8, s, ld_s, block, rows, cols, None) == want
    assert lib.sdvg_dequant_e4m3_blocks(x8, ld_8, s, ld_s, block, x, ld_x, t, rows, cols, None) == want


def norm_args(**change):
    a = dict(x=X, ld_x=200, x_type=0, y=None, ld_y=0, y_type=0, post=0, post_weight=None, gate=None, ld_gate=0, gate_rows=0, x_out=None,
             ld_x_out=0, norm=2, weight=None, bias=None, scale=None, shift=None, ld_mod=0, mod_rows=0, eps=1e-6, out=OUT, ld_out=200, os=OS,
             ld_os=2, rows=4, cols=200, stream=None)
    assert set(change) <= set(a)
    return list({**a, **change}.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "BAD_SHAPE"), (dict(cols=0), "BAD_SHAPE"), (dict(rows=0x7fffffff), "BAD_SHAPE"), (dict(ld_x=199), "BAD_SHAPE"),
    (dict(ld_out=199), "BAD_SHAPE"), (dict(ld_os=1), "BAD_SHAPE"), (dict(x_out=R, ld_x_out=199), "BAD_SHAPE"),
    (dict(scale=G, mod_rows=2, ld_mod=199), "BAD_SHAPE"), (dict(norm=3), "INVALID_ARG"), (dict(x_type=3), "INVALID_ARG"),
    (dict(y=W, ld_y=200, y_type=3), "INVALID_ARG"), (dict(post=1), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"),
    (dict(shift=G, mod_rows=0), "INVALID_ARG"), (dict(x=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"), (dict(os=None), "INVALID_ARG"),
    (dict(out=None, x_out=R, ld_x_out=200), "INVALID_ARG"), (dict(os=None, x_out=R, ld_x_out=200), "INVALID_ARG"),
    (dict(x=X + 1), "MISALIGNED"), (dict(weight=B_ + 2), "MISALIGNED"), (dict(x_out=R + 1, ld_x_out=200), "MISALIGNED"),
])
def test_gated_norm_refuses_on_the_host(lib, change, status):
    assert lib.sdvg_gated_norm_e4m3(*norm_args(**change)) == getattr(api, "SDVG_ERR_" + status)


def test_gated_norm_with_nothing_to_do_and_codes_of_any_alignment(lib):
    assert lib.sdvg_gated_norm_e4m3(*norm_args(rows=0, x=None, out=None, os=None)) == api.SDVG_OK
    assert lib.sdvg_gated_norm_e4m3(*norm_args(out=OUT + 1, os=OS + 1, weight=B_ + 1)) == api.SDVG_ERR_MISALIGNED
    assert lib.sdvg_gated_norm(X, 200, 0, None, 0, 0, 0, None, None, 0, 0, None, 0, 2, None, None, None, None, 0, 0, 1e-6, OUT, 200, 3, 4, 200,
                               None) == api.SDVG_ERR_INVALID_ARG


def u8(*shape):
    return OnPaper(*shape, dtype=torch.uint8)


def linear_on_paper(**change):
    a = dict(x=u8(4, 300), xs=u8(4, 3), w=u8(200, 300), ws=u8(2, 3), out=OnPaper(4, 200), space=u8(256), bias=None, act=0, residual=None,
             gate=None, gate_rows=0, out_scale=None, stream=0)
    assert set(change) <= set(a)
    return api._binding().linear_e4m3(*{**a, **change}.values())


def test_the_binding_reads_and_refuses(lib):
    reached = api.SDVG_ERR_INVALID_ARG                          # the library, which refuses the null addresses
    assert linear_on_paper() == linear_on_paper(ws=u8(200, 3)) == reached
    assert linear_on_paper(out=u8(4, 200), out_scale=u8(4, 2)) == reached
    for change in (dict(xs=u8(4, 2)), dict(xs=u8(3, 3)), dict(ws=u8(3, 3)), dict(ws=u8(2, 4)), dict(ws=u8(6)), dict(x=OnPaper(4, 300)),
                   dict(w=u8(200, 299)), dict(out=u8(4, 200)), dict(out_scale=u8(4, 2)), dict(out=u8(4, 200), out_scale=u8(4, 3)),
                   dict(out=u8(4, 199), out_scale=u8(4, 2)), dict(xs=OnPaper(4, 3)), dict(out=OnPaper(4, 201)),
                   dict(residual=OnPaper(4, 200, dtype=torch.float32)), dict(gate=OnPaper(2, 200, dtype=torch.float32), gate_rows=1),
                   dict(bias=OnPaper(199, dtype=torch.float32)), dict(x=u8(300))):
        with pytest.raises(ValueError):
            linear_on_paper(**change)
    for change in (dict(ws=without_address(2, 3, dtype=torch.uint8)), dict(space=without_address(256, dtype=torch.uint8))):
        with pytest.raises(RuntimeError):
            linear_on_paper(**change)
    norm = lambda x, out, scale: api._binding().gated_norm_e4m3(x, out, None, None, 0, 0, None, None, 2, None, None, None, None, 0, 1e-6, 0, scale)
    assert norm(OnPaper(4, 200), u8(4, 200), u8(4, 2)) == reached
    for bad in ((OnPaper(4, 200), OnPaper(4, 200), u8(4, 2)), (OnPaper(4, 200), u8(4, 200), u8(4, 3)), (OnPaper(4, 200), u8(4, 201), u8(4, 2)),
                (u8(4, 200), u8(4, 200), u8(4, 2)), (OnPaper(4, 200), None, u8(4, 2)), (OnPaper(4, 200), u8(4, 200), None)):
        with pytest.raises(ValueError):
            norm(*bad)
    blocks = api._binding().e4m3_blocks
    for way in (0, 1):
        assert blocks(OnPaper(200, 300), u8(200, 300), u8(200, 3), way, 0) == reached
        assert blocks(OnPaper(200, 300, dtype=torch.float32), u8(200, 300), u8(2, 3), way, 0) == reached
        for bad in ((u8(200, 300), u8(200, 300), u8(2, 3)), (OnPaper(200, 300), u8(200, 299), u8(2, 3)),
                    (OnPaper(200, 300), u8(200, 300), u8(3, 3)), (OnPaper(200), u8(200), u8(2)),
                    (torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.uint8))):
            with pytest.raises(ValueError):
                blocks(*bad, way, 0)
    with pytest.raises(TypeError):
        blocks()


# ---- the definitions ------------------------------------------------------------------------------------

def test_scales_are_the_smallest_that_hold_their_block():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 300)) * 2.0 ** rng.integers(-30, 30, (200, 1))
    for block_rows in (1, 128):
        codes, s = B.quantise(x, block_rows)
        f = B.of_elements(s, *x.shape, block_rows)
        assert (np.abs(x) <= 448 * f).all()
        top = np.array([[np.abs(x[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]).max() for j in range(3)]
                        for i in range(s.shape[0])])
        assert (top > 224 * 2.0 ** (s.astype(float) - 127)).all()
        assert (np.abs(B.values(codes, s, block_rows) - x) <= B.half_step(np.abs(x), f)).all()


def test_codes_and_scale_bytes_are_torchs_types():
    x = np.random.default_rng(1).standard_normal((5, 256))
    codes, s = B.quantise(x, 1)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double()
    f = torch.from_numpy(s).view(torch.float8_e8m0fnu).double().repeat_interleave(128, 1)
    assert np.array_equal((t * f).numpy(), B.values(codes, s, 1))
    assert torch.equal((torch.from_numpy(x) / f).float().to(torch.float8_e4m3fn).view(torch.uint8), torch.from_numpy(codes))


def test_special_values():
    x = np.zeros((1, 384))
    x[0, 0], x[0, 128], x[0, 129] = np.nan, np.inf, 3.0
    codes, s = B.quantise(x, 1)
    assert s.tolist() == [[1, 247, 1]] and codes[0, 0] == 0x7F and codes[0, 128] == 0x7E and codes[0, 129] == 0
    assert O.e4m3_tile_scale_exponent(0.0) == -126


# ---- ring write and read-back ---------------------------------------------------------------------------

@pytest.fixture
def rings(lib):
    """(static, tiled, bf16, too wide) with 2 heads (129) and 64 tokens."""
    import ctypes as C
    made = []
    for heads, e4m3, tiles in ((2, True, False), (2, True, True), (2, False, False), (129, True, True)):
        h = C.c_void_p()
        create = lib.sdvg_cache_create_e4m3 if e4m3 else lib.sdvg_cache_create
        assert create(C.byref(h), 0x10000, 0x20000, 3, heads, 64, 128) == api.SDVG_OK
        if tiles:
            assert lib.sdvg_cache_set_tile_scales(h, 0x30000, 0x40000) == api.SDVG_OK
        made.append(h)
    yield made
    for h in made:
        lib.sdvg_cache_destroy(h)


def test_qk_norm_refuses_on_the_host(lib, rings):
    static, tiled, bf16, wide = rings
    base = dict(cache=None, q=X, ld_q=256, k=W, ld_k=256, v=B_, ld_v=768, q_weight=G, k_weight=None, scope=0, eps=1e-6, q8=OUT)
    pos = dict(frames=1, grid_h=8, grid_w=8, frame_offset=0, tab=0x80000, tab_frames=4, block=0, flags=api.SDVG_STAGE, evicted=None)
    calls = {"static": ({**base, "cache": static, "qi": XS, "ki": XS, "vi": XS, **pos, "stream": None}, lib.sdvg_qk_norm_rope3d_commit_e4m3),
             "tiled": ({**base, "cache": tiled, "qs": XS, **pos, "ws": 0x90000, "ws_bytes": 256 + 64 * 8, "stream": None},
                       lib.sdvg_qk_norm_rope3d_commit_e4m3_tiled)}
    shared = [
        (dict(cache=None), "INVALID_ARG"), (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"),
        (dict(q8=None), "INVALID_ARG"), (dict(scope=2), "INVALID_ARG"), (dict(eps=-1.0), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"),
        (dict(tab=None), "INVALID_ARG"), (dict(flags=3), "INVALID_ARG"), (dict(cache=bf16), "BAD_SHAPE"), (dict(ld_q=248), "BAD_SHAPE"),
        (dict(ld_k=128), "BAD_SHAPE"), (dict(ld_v=0), "BAD_SHAPE"), (dict(grid_w=7), "BAD_SHAPE"),
        (dict(cache=wide, ld_q=20000, ld_k=20000, ld_v=20000), "BAD_SHAPE"), (dict(ld_k=260), "MISALIGNED"), (dict(q=X + 8), "MISALIGNED"),
        (dict(q_weight=G + 4), "MISALIGNED"), (dict(q8=OUT + 2), "MISALIGNED"), (dict(block=1), "BAD_STATE"), (dict(frame_offset=4), "BAD_STATE"),
        (dict(tab_frames=1 << 30), "BAD_SHAPE")]
    own = {"static": [(dict(ki=None), "INVALID_ARG"), (dict(vi=None), "INVALID_ARG"), (dict(qi=None), "INVALID_ARG"), (dict(ki=XS + 2), "MISALIGNED")],
           "tiled": [(dict(qs=None), "INVALID_ARG"), (dict(qs=XS + 2), "MISALIGNED"), (dict(cache=static), "BAD_STATE"),
                     (dict(ws=None), "INVALID_ARG"), (dict(ws_bytes=256 + 64 * 8 - 1), "INVALID_ARG"), (dict(ws=0x90010), "MISALIGNED")]}
    for kind, (args, call) in calls.items():
        for change, status in shared + own[kind]:
            assert set(change) <= set(args)
            assert call(*{**args, **change}.values()) == getattr(api, "SDVG_ERR_" + status), (kind, change)
    assert lib.sdvg_qk_norm_workspace_bytes(0) == 0 and lib.sdvg_qk_norm_workspace_bytes(4680) == 256 + 8 * 4680


def test_read_back_refuses_on_the_host(lib, rings):
    static, tiled, bf16, _ = rings
    f = lib.sdvg_cache_read_block_e4m3
    for args, status in [((None, 0, XS, XS, OUT, OS), "INVALID_ARG"), ((static, 0, XS, XS, None, None), "INVALID_ARG"),
                         ((static, 3, XS, XS, OUT, OS), "INVALID_ARG"), ((static, -1, XS, XS, OUT, OS), "INVALID_ARG"),
                         ((static, 0, XS, None, OUT, OS), "INVALID_ARG"), ((static, 0, None, XS, OUT, None), "INVALID_ARG"),
                         ((static, 0, None, None, OUT, OS), "BAD_STATE"), ((bf16, 0, XS, XS, OUT, OS), "BAD_SHAPE"),
                         ((tiled, 0, None, None, OUT + 8, OS), "MISALIGNED"), ((static, 0, XS + 1, XS, OUT, OS), "MISALIGNED")]:
        assert f(*args, None) == getattr(api, "SDVG_ERR_" + status), args


def test_the_binding_of_the_ring_writes(lib, rings):
    static, tiled, _, _ = rings
    block = lambda *shape: OnPaper(*(shape or (64, 2, 128)))
    n = lib.sdvg_rope3d_table_floats(128, 4, 8, 8)
    f32 = lambda *shape: OnPaper(*shape, dtype=torch.float32)

    def call(ring, fn, more, **change):
        a = dict(handle=ring.value, tokens=64, heads=2, dim=128, q=block(), k=block(), v=block(), q_weight=None, k_weight=None, scope=0,
                 eps=1e-6, q8=u8(64, 2, 128), k_out=None, frames=1, grid_h=8, grid_w=8, offset=0, table=f32(n), tab_frames=4, block=0,
                 flags=api.SDVG_STAGE, stream=0)
        assert set(change) <= set(a)
        return fn(*{**a, **change}.values(), *more)

    b, reached = api._binding(), -1000 - api.SDVG_ERR_INVALID_ARG
    inv = (f32(2), f32(2), f32(2))
    scales = (f32(2, 1), u8(256 + 64 * 8))
    assert call(static, b.qk_norm_e4m3, inv) == call(tiled, b.qk_norm_e4m3_tiled, scales) == reached
    assert call(static, b.qk_norm_e4m3, inv, q=None, q8=None) == call(tiled, b.qk_norm_e4m3_tiled, (None, None)) == reached
    for ring, fn, more in ((static, b.qk_norm_e4m3, inv), (tiled, b.qk_norm_e4m3_tiled, scales)):
        for change in (dict(q8=block()), dict(q8=u8(64, 2, 64)), dict(k=u8(64, 2, 128)), dict(table=f32(n - 1)), dict(q_weight=f32(255))):
            with pytest.raises(ValueError):
                call(ring, fn, more, **change)
        with pytest.raises(TypeError):
            fn()
    for more in ((f32(3), f32(2), f32(2)), (f32(2), f32(2), block()), (f32(2), f32(2, 1), f32(2))):
        with pytest.raises(ValueError):
            call(static, b.qk_norm_e4m3, more)
    for more in ((f32(2, 2), None), (f32(1, 2), None), (u8(2, 1), None), (f32(2, 1), 5)):
        with pytest.raises(ValueError):
            call(tiled, b.qk_norm_e4m3_tiled, more)


def test_the_binding_of_the_read_back(lib, rings):
    static = rings[0]
    read = lambda k, v, ks=OnPaper(2, dtype=torch.float32), vs=OnPaper(2, dtype=torch.float32), slot=0: api._binding().read_block_e4m3(
        static.value, 64, 2, slot, k, v, ks, vs, 0)
    block = lambda: OnPaper(64, 2, 128)
    assert read(block(), block()) == read(None, None) == read(block(), block(), slot=5) == api.SDVG_ERR_INVALID_ARG
    for bad in ((OnPaper(64, 2, 64), None), (u8(64, 2, 128), None), (OnPaper(63, 2, 128), None), (None, OnPaper(64, 256))):
        with pytest.raises(ValueError):
            read(*bad)
    for scale in (OnPaper(3, dtype=torch.float32), OnPaper(2), OnPaper(2, 1, dtype=torch.float32)):
        with pytest.raises(ValueError):
            read(block(), block(), ks=scale)
    with pytest.raises(TypeError):
        api._binding().read_block_e4m3()
