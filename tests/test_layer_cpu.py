"""Host glue of the transformer layer and of the schedule around it, with the library's calls replaced by a record; no GPU."""
import types

import pytest
import torch

from paper_2604_17397_b200 import api, build, schedule

HEADS, DIM, GRID = 2, 64, (2, 2, 3)
WIDTH, TOKENS = HEADS * DIM, 12


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()                                       # the text of an error comes from the library
    return api.lib()


class Record:
    """Takes the library calls a layer makes; `gives_up(workspace, columns)` says whether this linear layer gives up on a wait."""

    def __init__(self, monkeypatch, accept=()):
        self.calls, self.gives_up, self.accept = [], lambda ws, cols: False, accept
        self.bad = set()                                # workspaces whose status word says so
        for name in ("sdvg_gated_norm", "sdvg_linear", "sdvg_qk_norm_rope3d_commit", "sdvg_block_attn_fwd", "sdvg_route",
                     "sdvg_block_attn_status"):
            monkeypatch.setattr(api, name, getattr(self, name[5:]))

    def gated_norm(self, x, out, **kw):
        self.calls.append(("norm", kw))

    def linear(self, x, w, out, workspace, **kw):
        self.calls.append(("linear", out.shape[1]))
        if self.gives_up(workspace, out.shape[1]):
            self.bad.add(workspace.data_ptr())

    def qk_norm_rope3d_commit(self, cache, q, k, v, *rest):
        block, flags = rest[-2:]
        self.calls.append(("ring", cache.name, block, flags))
        return -1

    def block_attn_fwd(self, *args):
        self.calls.append(("attention",))

    def route(self, scores, offsets, n, frames, first, tau, accept, qmin, *rest):
        accept.fill_(int(first in self.accept))

    def block_attn_status(self, workspace):
        return api.SDVG_ERR_TIMEOUT if workspace.data_ptr() in self.bad else api.SDVG_OK


def model(name):
    cache = types.SimpleNamespace(name=name, heads=HEADS, head_dim=DIM, block_tokens=TOKENS, slots=3)
    return schedule.ModelState(cache, GRID, torch.zeros(8), 16, 1.0, torch.zeros(256, dtype=torch.uint8))


def layer(m):
    mat = lambda n, k: torch.zeros((n, k), dtype=torch.bfloat16)
    return schedule.TransformerLayer(schedule.LayerWeights(mat(3 * WIDTH, WIDTH), mat(WIDTH, WIDTH), mat(4 * WIDTH, WIDTH),
                                                           mat(WIDTH, 4 * WIDTH)), m)


def provider(*_):
    x = torch.zeros((TOKENS, WIDTH), dtype=torch.bfloat16)
    return x, torch.zeros((GRID[0], 6 * WIDTH)), torch.empty_like(x)


def run(blocks, drafter, target):
    return schedule.run_schedule(blocks, 2, torch.zeros((blocks, 2)), 0.0, drafter, target, provider,
                                 drafter_layer=layer(drafter), target_layer=layer(target))


@pytest.mark.parametrize("who", ["drafter", "target"])
@pytest.mark.parametrize("at,accept", [(0, ()), (1, (1,)), (2, (1, 2)), (2, ())])
def test_a_commits_projection_that_gave_up_reaches_no_ring(monkeypatch, who, at, accept):
    """The k and v of a final commit come from a product with bounded waits: the block of one that gave up is not committed, and
    the schedule raises, also where the branch was accepted and in the last block."""
    r, models = Record(monkeypatch, accept), {"drafter": model("drafter"), "target": model("target")}
    seen = []

    def gives_up(ws, cols):
        if cols == 2 * WIDTH and ws is models[who].workspace:      # k and v of a final commit
            seen.append(1)
            return len(seen) == at + 1
        return False

    r.gives_up = gives_up
    with pytest.raises(api.SdvgError) as e:
        run(3, models["drafter"], models["target"])
    assert e.value.status == api.SDVG_ERR_TIMEOUT and len(seen) == at + 1
    final = [c[2] for c in r.calls if c[0] == "ring" and c[1] == who and c[3] == api.SDVG_FINAL]
    assert final == list(range(at))


def test_a_schedule_without_a_give_up_commits_every_block(monkeypatch):
    r = Record(monkeypatch, (1,))
    res = run(3, model("drafter"), model("target"))
    assert res.accept.tolist() == [0, 1, 0] and res.target_source == ["regenerated", "accepted", "regenerated"]
    for who in ("drafter", "target"):
        assert [c[2] for c in r.calls if c[0] == "ring" and c[1] == who and c[3] == api.SDVG_FINAL] == [0, 1, 2]


def test_a_commit_of_its_own_reads_no_status(monkeypatch):
    """So that it can be captured; the caller reads the status when it suits."""
    r, m = Record(monkeypatch), model("drafter")
    r.gives_up = lambda ws, cols: True
    x, mod, _ = provider()
    assert layer(m).commit(x, mod, 0) == -1
    with pytest.raises(api.SdvgError):
        layer(m).commit(x, mod, 0, check=True)
    assert [c[0] for c in r.calls] == ["norm", "linear", "ring", "norm", "linear"]


@pytest.mark.parametrize("groups", [1, 2, 3, 5, 7, 11, 12, 20])
def test_modulation_rows_of_any_number(monkeypatch, groups):
    """Token t uses row t // ceil(tokens / groups); the calls get as many rows as that reaches, which is what they ask for."""
    r, m = Record(monkeypatch), model("drafter")
    x, _, x_out = provider()
    mod = torch.arange(groups, dtype=torch.float32)[:, None].expand(groups, 6 * WIDTH).contiguous()
    layer(m).step(x, mod, 0, x_out)
    rows = -(-TOKENS // groups)
    for kw in [c[1] for c in r.calls if c[0] == "norm"]:
        assert kw["modulate_rows"] == rows
        assert kw["scale"].shape == kw["shift"].shape == (-(-TOKENS // rows), WIDTH)
        assert kw["scale"][:, 0].tolist() == [float(i) for i in range(-(-TOKENS // rows))]


@pytest.mark.parametrize("current", [0, 1])
def test_a_layer_runs_with_its_own_device_current(monkeypatch, current):
    """The attention, the ring writes of 8-bit caches and the status read launch on the current device and its stream, whatever
    their tensors' device; the norms and products go by their tensors.  All of a step has to be in one stream."""
    r, m = Record(monkeypatch), model("drafter")
    one = layer(m)
    at, seen = [current], []

    class Device:
        def __init__(self, dev):
            self.dev = torch.device(dev).index

        def __enter__(self):
            self.before, at[0] = at[0], self.dev

        def __exit__(self, *_):
            at[0] = self.before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for name in ("sdvg_gated_norm", "sdvg_linear", "sdvg_qk_norm_rope3d_commit", "sdvg_block_attn_fwd", "sdvg_block_attn_status"):
        def call(*args, f=getattr(api, name), **kw):
            seen.append(at[0])
            return f(*args, **kw)
        monkeypatch.setattr(api, name, call)
    m.table = types.SimpleNamespace(device=torch.device("cuda", 1))
    x, mod, x_out = provider()
    one.step(x, mod, 0, x_out)
    m.check_status("step")
    one.commit(x, mod, 0, check=True)
    assert seen == [1] * 13 and at == [current]
