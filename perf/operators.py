"""The dense operators around a block's attention, as cases that can be timed and compared.

A denoising step of a transformer whose attention this library computes needs, around that attention,

  linear   out = residual + gate[group] * act(x W^T + bias): the projections before and after the attention, the
           feed-forward pair, the few-row products that turn a time embedding into modulation vectors
  norm     s = x + gate[group] * post(y), out = pre(s) * (1 + scale[group]) + shift[group]: the residual add of one
           sublayer's output and the modulated norm that opens the next, in one pass over the rows
  qk       RMS norm of q and k, 3D rotary embedding, and the provisional write of the block's k and v into its ring
           slot, read straight from the rows of a fused QKV projection

``run`` computes a case in plain torch operations in 32 bits, or (``own``) through the library.  ``exact`` is the same
definition in 64 bits, written apart.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
FRAMES, GRID_H, GRID_W = 3, 30, 52            # latent frames of a block and their grid: 4680 tokens


# ---------------------------------------------------------------- cases

def _linear(name, m, k, n, dtype="bf16", out="", bias=True, act="none", gate=0, residual=""):
    """gate: rows that share a gate vector (0: no gate); residual: "" or "rows" or "broadcast" (one row for all)."""
    return {"name": name, "op": "linear", "m": m, "k": k, "n": n, "dtype": dtype, "out": out or dtype, "bias": bias,
            "act": act, "gate": gate, "residual": residual}


def _norm(name, rows, cols, x="bf16", y="", out="bf16", norm="layer", affine=False, modulate=0, gate=0, post="none"):
    """modulate, gate: rows that share a (scale, shift) pair or a gate (0: none); y "": no sublayer output to add."""
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "x": x, "y": y, "out": out, "norm": norm,
            "affine": affine, "modulate": modulate, "gate": gate, "post": post}


def _qk(name, heads, dim, frames, grid_h, grid_w, slots, block, scope="row", fused=True):
    """fused: q, k and v are column ranges of one QKV matrix; block: the block being generated (earlier ones are committed)."""
    return {"name": name, "op": "qk", "heads": heads, "dim": dim, "frames": frames, "grid_h": grid_h, "grid_w": grid_w,
            "slots": slots, "block": block, "scope": scope, "fused": fused}


def listed():
    tok = FRAMES * GRID_H * GRID_W
    frame = GRID_H * GRID_W
    return [
        # sinusoidal time features of one step to the drafter's width: one row, launch latency
        _linear("linear_time_embed", 1, 256, 1536, act="silu"),
        # one row per latent frame to the six modulation vectors of the target, fp32, plus their learned offsets
        _linear("linear_time_modulation", 3, 5120, 6 * 5120, out="fp32", residual="broadcast"),
        # the text tokens of a prompt to the target's width, once per video
        _linear("linear_text", 512, 4096, 5120, act="gelu_tanh"),
        # the target's fused QKV projection of a block
        _linear("linear_qkv_target", tok, 5120, 3 * 5120),
        # the target's attention output projection with its gate and residual
        _linear("linear_out_target", tok, 5120, 5120, gate=frame, residual="rows"),
        # the target's feed-forward expansion (the largest product of a layer)
        _linear("linear_ffn_up_target", tok, 5120, 4 * 5120, act="gelu_tanh"),
        # the drafter's feed-forward contraction, half precision onto an fp32 residual stream
        _linear("linear_ffn_down_drafter", tok, 4 * 1536, 1536, dtype="fp16", out="fp32", gate=frame, residual="rows"),
        # the modulated norm of one token: launch latency
        _norm("norm_single", 1, 1536, modulate=1),
        # the target's residual add and the modulated norm of the next sublayer, one block
        _norm("norm_block_target", tok, 5120, y="bf16", modulate=frame, gate=frame),
        # norms before and after the sublayer on an fp32 stream of odd width, ragged rows
        _norm("norm_sandwich_odd", 1561, 1537, x="fp32", y="bf16", norm="rms", affine=True, gate=521, post="rms"),
        # the smallest block: 2 heads of 64, two frames of 32 tokens, per-head norms
        _qk("qk_tiny", 2, 64, 2, 4, 8, 3, 1, scope="head", fused=False),
        # the target's block: 40 heads of 128 out of the fused QKV rows, ring of 7
        _qk("qk_target", 40, 128, FRAMES, GRID_H, GRID_W, 7, 2),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "qk"])
    if op == "linear":
        m, k, n = _log(rng, 1, 4680), _log(rng, 64, 6144), _log(rng, 1, 20480)
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        case = _linear("", m, k, n, dtype, rng.choice([dtype, dtype, "fp32"]), rng.random() < 0.8,
                       rng.choice(["none", "silu", "gelu_tanh", "gelu"]), rng.choice([0, _log(rng, 1, m)]),
                       rng.choice(["", "rows", "rows", "broadcast"]))
    elif op == "norm":
        rows, cols = _log(rng, 1, 4680), _log(rng, 16, 5120)
        y = rng.choice(["", "bf16", "fp32"])
        case = _norm("", rows, cols, rng.choice(["bf16", "fp16", "fp32"]), y, rng.choice(["bf16", "fp16", "fp32"]),
                     rng.choice(["layer", "rms"]), rng.random() < 0.4, rng.choice([0, _log(rng, 1, rows)]),
                     rng.choice([0, _log(rng, 1, rows)]) if y else 0, rng.choice(["none", "rms", "layer"]) if y else "none")
    else:
        case = _qk("", _log(rng, 1, 40), rng.choice([64, 128]), rng.randint(1, 3), _log(rng, 1, 30), _log(rng, 1, 52),
                   rng.randint(1, 4), rng.randint(0, 3), rng.choice(["row", "head"]), rng.random() < 0.7)
    del case["name"]
    return case


def work(case):
    """Every input read once and every output written once; the multiply-adds of the products, a few per element elsewhere."""
    if case["op"] == "linear":
        m, k, n, b, o = case["m"], case["k"], case["n"], BYTES[case["dtype"]], BYTES[case["out"]]
        rows = {"": 0, "rows": m, "broadcast": 1}[case["residual"]]
        groups = -(-m // case["gate"]) if case["gate"] else 0
        return {"bytes": (m + n) * k * b + (m + rows) * n * o + 4 * n * (groups + case["bias"]), "flops": 2 * m * k * n}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        vectors = 2 * case["affine"] + (case["post"] != "none")
        vectors += (2 * -(-rows // case["modulate"]) if case["modulate"] else 0)
        vectors += (-(-rows // case["gate"]) if case["gate"] else 0)
        streams = BYTES[case["x"]] + BYTES[case["out"]] + ((BYTES[case["y"]] + BYTES[case["x"]]) if case["y"] else 0)
        return {"bytes": rows * cols * streams + 4 * cols * vectors, "flops": 12 * rows * cols}
    elems = case["frames"] * case["grid_h"] * case["grid_w"] * case["heads"] * case["dim"]
    return {"bytes": 6 * 2 * elems, "flops": 2 * 8 * elems}


# ---------------------------------------------------------------- inputs

def _rows(gen, rows, cols, dtype, std=1.0, spread=0.0, pad=8):
    """[rows, cols] of a buffer whose row stride is a multiple of `pad`; spread: some columns are larger, as activations' are."""
    stride = -(-cols // pad) * pad
    x = torch.randn((rows, stride), generator=gen, device="cuda", dtype=torch.float32) * std
    if spread:
        x *= 1 + spread * torch.rand(stride, generator=gen, device="cuda") ** 8
    return x.to(dtype)[:, :cols]


def _vec(gen, *shape, std=0.5, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std + mean


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case)}
    if case["op"] == "linear":
        m, k, n, t, o = case["m"], case["k"], case["n"], DTYPES[case["dtype"]], DTYPES[case["out"]]
        s["x"] = _rows(gen, m, k, t, spread=4.0)
        s["w"] = _rows(gen, n, k, t, std=1 / math.sqrt(k))
        s["bias"] = _vec(gen, n) if case["bias"] else None
        s["gate"] = _vec(gen, -(-m // case["gate"]), n) if case["gate"] else None
        s["residual"] = None
        if case["residual"]:
            rows = _rows(gen, m if case["residual"] == "rows" else 1, n, o, std=2.0)
            s["residual"] = rows.expand(m, n)
        s["out"] = torch.empty((m, n), device="cuda", dtype=o)
    elif case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        per_col = _vec(gen, cols, std=0.5)
        s["x"] = (_rows(gen, rows, cols, torch.float32, std=2.0, spread=20.0, pad=1) + per_col).to(DTYPES[case["x"]])
        s["y"] = _rows(gen, rows, cols, DTYPES[case["y"]], spread=4.0, pad=1) if case["y"] else None
        s["gate"] = _vec(gen, -(-rows // case["gate"]), cols) if case["gate"] else None
        s["scale"] = _vec(gen, -(-rows // case["modulate"]), cols, std=0.3) if case["modulate"] else None
        s["shift"] = _vec(gen, -(-rows // case["modulate"]), cols, std=0.3) if case["modulate"] else None
        s["weight"] = _vec(gen, cols, std=0.2, mean=1.0) if case["affine"] else None
        s["bias"] = _vec(gen, cols, std=0.2) if case["affine"] and case["norm"] == "layer" else None
        s["post_weight"] = _vec(gen, cols, std=0.2, mean=1.0) if case["post"] != "none" else None
        s["x_out"] = torch.empty_like(s["x"]) if case["y"] else None
        s["out"] = torch.empty((rows, cols), device="cuda", dtype=DTYPES[case["out"]])
    else:
        h, d = case["heads"], case["dim"]
        t, c = case["frames"] * case["grid_h"] * case["grid_w"], case["heads"] * case["dim"]
        if case["fused"]:
            qkv = _rows(gen, t, 3 * c, torch.bfloat16, std=1.5, spread=4.0)
            s["q"], s["k"], s["v"] = (qkv[:, i * c:(i + 1) * c].view(t, h, d) for i in range(3))
        else:
            s["q"], s["k"], s["v"] = (_rows(gen, t, c, torch.bfloat16, std=1.5).view(t, h, d) for _ in range(3))
        width = c if case["scope"] == "row" else d
        s["q_weight"], s["k_weight"] = (_vec(gen, width, std=0.2, mean=1.0) for _ in range(2))
        s["q_out"] = torch.empty((t, h, d), device="cuda", dtype=torch.bfloat16)
        s["tab_frames"] = (case["block"] + 1) * case["frames"]
        s["table"] = _table(d, s["tab_frames"], case["grid_h"], case["grid_w"]).cuda()
    return s


def _pairs(dim):
    return dim // 2 - 2 * (dim // 6), dim // 6, dim // 6


def _table(dim, tab_frames, grid_h, grid_w):
    """(cos, sin) pairs, fp32: frame positions, then rows, then columns; angles in 64 bits."""
    parts = []
    for count, positions in zip(_pairs(dim), (tab_frames, grid_h, grid_w)):
        omega = 10000.0 ** (-torch.arange(count, dtype=torch.float64) / count)
        angle = torch.arange(positions, dtype=torch.float64)[:, None] * omega
        parts.append(torch.stack([angle.cos(), angle.sin()], -1).reshape(-1))
    return torch.cat(parts).float()


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2604_17397_b200 import api
        s["api"] = api
    if case["op"] == "qk":
        shape = (case["heads"], case["slots"], s["q"].shape[0], case["dim"])
        if own:
            cache = s["cache"] = api.Cache(case["slots"], case["heads"], s["q"].shape[0], case["dim"])
            zero = torch.zeros_like(s["q_out"])
            for b in range(case["block"]):
                api.sdvg_kv_commit(cache, zero, zero, b, api.SDVG_FINAL)
            s["ring_k"], s["ring_v"] = (raw[ptr - raw.data_ptr():][:math.prod(shape) * 2].view(torch.bfloat16).view(shape)
                                        for raw, ptr in ((cache._k_raw, cache.k_ptr), (cache._v_raw, cache.v_ptr)))
        else:
            s["ring_k"], s["ring_v"] = (torch.zeros(shape, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    elif own and case["op"] == "linear":
        s["workspace"] = api.attn_workspace()
        s["act"] = {"none": api.SDVG_ACT_NONE, "silu": api.SDVG_ACT_SILU, "gelu_tanh": api.SDVG_ACT_GELU_TANH,
                    "gelu": api.SDVG_ACT_GELU}[case["act"]]
    elif own:
        kinds = {"none": api.SDVG_NORM_NONE, "rms": api.SDVG_NORM_RMS, "layer": api.SDVG_NORM_LAYER}
        s["norm"], s["post_norm"] = kinds[case["norm"]], kinds[case["post"]]
    return s


# ---------------------------------------------------------------- the operators

def run(s):
    return {"linear": _run_linear, "norm": _run_norm, "qk": _run_qk}[s["case"]["op"]](s)


def _act(v, act):
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v


def _of_rows(vectors, rows, per_group):
    """The group's vector for every row."""
    return vectors[torch.arange(rows, device=vectors.device) // per_group]


def _run_linear(s):
    case = s["case"]
    if own:
        s["api"].sdvg_linear(s["x"], s["w"], s["out"], s["workspace"], bias=s["bias"], act=s["act"],
                             residual=s["residual"], gate=s["gate"], gate_rows=case["gate"])
        return s["out"]
    v = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        v = v + s["bias"]
    v = _act(v, case["act"])
    if s["gate"] is not None:
        v = v * _of_rows(s["gate"], case["m"], case["gate"])
    if s["residual"] is not None:
        v = v + s["residual"].float()
    return v.to(DTYPES[case["out"]])


def _norm_plain(v, kind, eps=1e-6):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v if kind == "none" else v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)


def _run_norm(s):
    case = s["case"]
    if own:
        s["api"].sdvg_gated_norm(s["x"], s["out"], y=s["y"], gate=s["gate"], gate_rows=case["gate"],
                                 post_norm=s["post_norm"], post_weight=s["post_weight"], x_out=s["x_out"],
                                 norm=s["norm"], weight=s["weight"], bias=s["bias"], scale=s["scale"],
                                 shift=s["shift"], modulate_rows=case["modulate"], eps=1e-6)
        return (s["x_out"], s["out"]) if s["y"] is not None else s["out"]
    rows, v = case["rows"], s["x"].float()
    if s["y"] is not None:
        y = _norm_plain(s["y"].float(), case["post"])
        if s["post_weight"] is not None:
            y = y * s["post_weight"]
        if s["gate"] is not None:
            y = y * _of_rows(s["gate"], rows, case["gate"])
        v = v + y
    o = _norm_plain(v, case["norm"])
    if s["weight"] is not None:
        o = o * s["weight"]
    if s["bias"] is not None:
        o = o + s["bias"]
    if s["scale"] is not None:
        o = o * (1 + _of_rows(s["scale"], rows, case["modulate"])) + _of_rows(s["shift"], rows, case["modulate"])
    o = o.to(DTYPES[case["out"]])
    return (v.to(s["x"].dtype), o) if s["y"] is not None else o


def _rotary(s):
    """cos and sin of every token's pairs: [tokens, 1, dim / 2] each."""
    case, tab = s["case"], s["table"]
    t = torch.arange(s["q"].shape[0], device="cuda")
    hw = case["grid_h"] * case["grid_w"]
    at = (case["block"] * case["frames"] + t // hw, t % hw // case["grid_w"], t % case["grid_w"])
    begin, cs = 0, []
    for count, positions, where in zip(_pairs(case["dim"]), (s["tab_frames"], case["grid_h"], case["grid_w"]), at):
        cs.append(tab[begin:begin + 2 * count * positions].view(positions, count, 2)[where])
        begin += 2 * count * positions
    cs = torch.cat(cs, 1)[:, None]
    return cs[..., 0], cs[..., 1]


def _run_qk(s):
    case = s["case"]
    slot = case["block"] % case["slots"]
    if own:
        api = s["api"]
        scope = api.SDVG_SCOPE_ROW if case["scope"] == "row" else api.SDVG_SCOPE_HEAD
        api.sdvg_qk_norm_rope3d_commit(s["cache"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], scope, 1e-6,
                                       s["q_out"], None, (case["frames"], case["grid_h"], case["grid_w"]),
                                       case["block"] * case["frames"], s["table"], s["tab_frames"], case["block"],
                                       api.SDVG_STAGE)
        return s["q_out"], s["ring_k"][:, slot], s["ring_v"][:, slot]
    cos, sin = _rotary(s)
    turned = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        v = x.float()
        if case["scope"] == "row":
            v = (_norm_plain(v.flatten(1), "rms") * w).view(v.shape)
        else:
            v = _norm_plain(v, "rms") * w
        re, im = v[..., 0::2], v[..., 1::2]
        turned.append(torch.stack([re * cos - im * sin, re * sin + im * cos], -1).flatten(2).to(torch.bfloat16))
    s["ring_k"][:, slot] = turned[1].transpose(0, 1)
    s["ring_v"][:, slot] = s["v"].transpose(0, 1)
    return turned[0], s["ring_k"][:, slot], s["ring_v"][:, slot]


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    return {"linear": _exact_linear, "norm": _exact_norm, "qk": _exact_qk}[case["op"]](case, d)


def _repeat(vectors, rows, per_group):
    return vectors.repeat_interleave(per_group, 0)[:rows]


def _exact_linear(case, d):
    z = torch.einsum("mk,nk->mn", d["x"], d["w"])
    if "bias" in d:
        z += d["bias"]
    if case["act"] == "silu":
        z *= torch.sigmoid(z)
    elif case["act"] == "gelu_tanh":
        z *= torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))       # (1 + tanh u) / 2 = sigmoid(2 u)
    elif case["act"] == "gelu":
        z *= torch.erfc(-z / math.sqrt(2)) / 2
    if "gate" in d:
        z *= _repeat(d["gate"], case["m"], case["gate"])
    return z + d["residual"] if "residual" in d else z


def _exact_normed(v, kind):
    if kind == "none":
        return v
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    return (v - mean) / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + 1e-6)


def _exact_norm(case, d):
    z = d["x"]
    if case["y"]:
        y = _exact_normed(d["y"], case["post"])
        if case["post"] != "none":
            y = y * d["post_weight"]
        z = z + (y * _repeat(d["gate"], case["rows"], case["gate"]) if case["gate"] else y)
    o = _exact_normed(z, case["norm"])
    if case["affine"]:
        o = o * d["weight"] + (d["bias"] if "bias" in d else 0.0)
    if case["modulate"]:
        o = o * (1 + _repeat(d["scale"], case["rows"], case["modulate"])) + _repeat(d["shift"], case["rows"], case["modulate"])
    return (z, o) if case["y"] else o


def _exact_qk(case, d):
    t, h, dim = d["q"].shape
    f, gh, gw = case["frames"], case["grid_h"], case["grid_w"]
    sizes = [n * p for n, p in zip(_pairs(dim), ((case["block"] + 1) * f, gh, gw))]
    z = torch.view_as_complex(d["table"].view(-1, 2))
    frame, row, col = (part.view(-1, n) for part, n in zip(z.split(sizes), _pairs(dim)))
    frame = frame[case["block"] * f:]
    turn = torch.cat([frame[:, None, None].expand(f, gh, gw, -1), row[None, :, None].expand(f, gh, gw, -1),
                      col[None, None].expand(f, gh, gw, -1)], -1).reshape(t, 1, dim // 2)
    got = []
    for x, w in ((d["q"], d["q_weight"]), (d["k"], d["k_weight"])):
        x = _exact_normed(x.reshape(t, -1) if case["scope"] == "row" else x.reshape(t * h, dim), "rms") * w
        got.append(torch.view_as_real(torch.view_as_complex(x.reshape(t, h, dim // 2, 2)) * turn).reshape(t, h, dim))
    return got[0], got[1].transpose(0, 1), None
