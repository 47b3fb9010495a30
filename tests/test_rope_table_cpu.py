"""The older entry points' rotary table, whose length the binding holds against the grid and frames; no GPU."""
import pytest
import torch

from paper_2604_17397_b200 import api, build
from test_dense_cpu import OnPaper

GRID, TOKENS, HEADS, FRAMES = (2, 4, 8), 64, 2, 6


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return api.lib()


class FakeRing:
    """A cache handle over addresses that nothing reads."""

    def __init__(self, lib, e4m3, tiled):
        import ctypes as C
        self.lib, self.handle = lib, C.c_void_p()
        self.heads, self.block_tokens, self.head_dim = HEADS, TOKENS, 128
        create = lib.sdvg_cache_create_e4m3 if e4m3 else lib.sdvg_cache_create
        assert create(C.byref(self.handle), 0x10000, 0x20000, 3, HEADS, TOKENS, 128) == api.SDVG_OK
        if tiled:
            assert lib.sdvg_cache_set_tile_scales(self.handle, 0x30000, 0x40000) == api.SDVG_OK


def entry_points(ring, e4m3, tiled, table):
    """Calls of the entry points of this kind of ring, on tensors without memory."""
    t = lambda: OnPaper(TOKENS, HEADS, 128)
    u = lambda: OnPaper(TOKENS, HEADS, 128, dtype=torch.uint8)
    sc = lambda: OnPaper(HEADS, dtype=torch.float32)
    ts = lambda: OnPaper(HEADS, 1, dtype=torch.float32)
    ws = OnPaper(512, dtype=torch.uint8)
    if tiled:
        return [lambda: api.sdvg_rope3d_qk_commit_e4m3_tiled(ring, t(), t(), t(), u(), ts(), GRID, 0, table, FRAMES, 0, 1, stream=0),
                lambda: api.sdvg_block_steps_e4m3_tiled(ring, [t()], [t()], [t()], [u()], [ts()], [t()], GRID, 0, table, FRAMES, 0, 1.0, ws,
                                                        stream=0)]
    if e4m3:
        return [lambda: api.sdvg_rope3d_qk_commit_e4m3(ring, t(), t(), t(), u(), sc(), sc(), sc(), GRID, 0, table, FRAMES, 0, 1, stream=0),
                lambda: api.sdvg_block_steps_e4m3(ring, [t()], [t()], [t()], [u()], [t()], sc(), sc(), sc(), sc(), sc(), GRID, 0, table,
                                                  FRAMES, 0, 1.0, ws, stream=0)]
    return [lambda: api.sdvg_rope3d_qk(t(), t(), t(), t(), GRID, 0, table, FRAMES, stream=0),
            lambda: api.sdvg_rope3d_qk_commit(ring, t(), t(), t(), t(), None, GRID, 0, table, FRAMES, 0, 1, stream=0),
            lambda: api.sdvg_block_steps(ring, [t()], [t()], [t()], [t()], [t()], GRID, 0, table, FRAMES, 0, 1.0, ws, stream=0)]


@pytest.mark.parametrize("e4m3,tiled", [(False, False), (True, False), (True, True)])
def test_a_short_table_is_refused(lib, e4m3, tiled):
    ring = FakeRing(lib, e4m3, tiled)
    n = lib.sdvg_rope3d_table_floats(128, FRAMES, GRID[1], GRID[2])
    for floats in (n, n + 3):                           # reaches the library, which refuses the null addresses
        for call in entry_points(ring, e4m3, tiled, OnPaper(floats, dtype=torch.float32)):
            with pytest.raises(api.SdvgError) as e:
                call()
            assert e.value.status == api.SDVG_ERR_INVALID_ARG
    for table in (OnPaper(n - 1, dtype=torch.float32), OnPaper(2 * n, dtype=torch.bfloat16)):
        for call in entry_points(ring, e4m3, tiled, table):
            with pytest.raises(ValueError, match="table"):
                call()
    lib.sdvg_cache_destroy(ring.handle)
