"""The 8-bit layers do not keep the 16-bit matrices that they were made of; no GPU."""
import weakref

import torch

from paper_2604_17397_b200 import schedule
from test_layer_cpu import lib  # noqa: F401 (the fixture builds the library)
from test_layer_e4m3_cpu import TOKENS, model, record, weights  # noqa: F401

MATRICES = ("w_qkv", "w_out", "w_up", "w_down")


def test_a_layer_keeps_its_8_bit_matrices_alone(record):  # noqa: F811
    w = weights(256, b_up=torch.zeros(1024), q_norm=torch.ones(256))
    seen = [weakref.ref(getattr(w, name)) for name in MATRICES]
    layer = schedule.TransformerLayerE4M3(w, model("m", 2, 128))
    assert all(getattr(w, name) is not None for name in MATRICES)                # the caller's are the caller's
    assert layer.w.b_up is w.b_up and layer.w.q_norm is w.q_norm
    record.clear()
    del w
    assert all(ref() is None for ref in seen)
    x, mod = torch.zeros((TOKENS, 256), dtype=torch.bfloat16), torch.zeros((2, 6 * 256))
    layer.step(x, mod, 0, x)
    layer.commit(x, mod, 0)


def test_a_time_modulation_keeps_its_8_bit_matrices_alone(record):  # noqa: F811
    mat = lambda n, k: torch.zeros((n, k), dtype=torch.bfloat16)
    tm = schedule.TimeModulation(mat(256, 128), mat(256, 256), mat(1536, 256), torch.zeros(256), torch.zeros(256), torch.zeros(1536),
                                 torch.zeros((1, 1536)))
    seen = [weakref.ref(t) for t in (tm.w1, tm.w2, tm.w_mod)]
    eight = schedule.TimeModulationE4M3(tm)
    assert tm.w1 is not None and eight.tm.b1 is tm.b1
    record.clear()
    del tm
    assert all(ref() is None for ref in seen)
    assert eight(torch.zeros((2, 128), dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8)).shape == (2, 1536)
