"""The 8-bit side of a transformer layer around the block attention, as cases that can be timed and compared.

The library's rings and its attention take 8-bit floating point (E4M3) with power-of-two scales.  A layer that keeps its
weights and the rows between its operators in that form as well needs

  linear8  out = residual + gate[group] * act(x W^T + bias) with x and W in E4M3, one power-of-two scale per 128 consecutive
           elements of a row of x and per 128 x 128 block of W; the outputs may be E4M3 rows of the same form again
  norm8    s = x + gate[group] * post(y), out = pre(s) * (1 + scale[group]) + shift[group] written as such rows (with no norm
           and nothing to add: the quantisation of rows)
  commit8  RMS norm of q and k, 3D rotary embedding, and the quantising write of the block's k and v into its slot of an
           8-bit ring, straight from the rows of a fused QKV projection; with static scales per head, or with scales that
           are chosen from the data per 128 tokens and head, and then read back
  read8    a slot of an 8-bit ring as bf16 tensors

``run`` computes a case in plain torch operations in 32 bits, or (``own``) through the library.  ``exact`` is the same
definition in 64 bits without the last rounding, written apart.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1 + 1 / 128}
FRAMES, GRID_H, GRID_W = 3, 30, 52            # latent frames of a block and their grid: 4680 tokens


# ---------------------------------------------------------------- cases

def _linear(name, m, k, n, out="bf16", bias=True, act="none", gate=0, residual=""):
    """gate: rows that share a gate vector (0: no gate); residual: "" or "rows" or "broadcast" (one row for all)."""
    return {"name": name, "op": "linear8", "m": m, "k": k, "n": n, "out": out, "bias": bias, "act": act, "gate": gate,
            "residual": residual}


def _norm(name, rows, cols, x="bf16", y="", norm="layer", affine=False, modulate=0, gate=0, post="none"):
    """modulate, gate: rows that share a (scale, shift) pair or a gate (0: none); y "": no sublayer output to add."""
    return {"name": name, "op": "norm8", "rows": rows, "cols": cols, "x": x, "y": y, "norm": norm, "affine": affine,
            "modulate": modulate, "gate": gate, "post": post}


def _commit(name, heads, frames, grid_h, grid_w, slots, block, tiled, scope="row", fused=True):
    """fused: q, k and v are column ranges of one QKV matrix; block: the block being generated."""
    return {"name": name, "op": "commit8", "heads": heads, "frames": frames, "grid_h": grid_h, "grid_w": grid_w,
            "slots": slots, "block": block, "tiled": tiled, "scope": scope, "fused": fused}


def _read(name, heads, tokens, slots, slot, tiled):
    return {"name": name, "op": "read8", "heads": heads, "tokens": tokens, "slots": slots, "slot": slot, "tiled": tiled}


def listed():
    tok = FRAMES * GRID_H * GRID_W
    frame = GRID_H * GRID_W
    return [
        # the second product of a time embedding at the drafter's width, one step: one row, launch latency
        _linear("linear8_time_embed", 1, 1536, 1536, act="silu"),
        # one row per latent frame to the six modulation vectors of the target, fp32, plus their learned offsets
        _linear("linear8_time_modulation", 3, 5120, 6 * 5120, out="fp32", residual="broadcast"),
        # a ragged batch of tokens through a projection of odd sizes, half precision
        _linear("linear8_ragged", 333, 1111, 777, out="fp16", act="gelu", gate=100, residual="rows"),
        # the target's fused QKV projection of a block
        _linear("linear8_qkv_target", tok, 5120, 3 * 5120),
        # the target's attention output projection with its gate, onto an fp32 residual stream
        _linear("linear8_out_target", tok, 5120, 5120, out="fp32", gate=frame, residual="rows"),
        # the target's feed-forward expansion (the largest product of a layer), quantised for the product after it
        _linear("linear8_ffn_up_target", tok, 5120, 4 * 5120, out="e4m3", act="gelu_tanh"),
        # the target's residual add and the modulated norm of the next sublayer, one block
        _norm("norm8_block_target", tok, 5120, y="bf16", modulate=frame, gate=frame),
        # rows of odd length on an fp32 stream, quantised as they are
        _norm("norm8_rows_odd", 1561, 1537, x="fp32", norm="none"),
        # a block of one token in the drafter's ring: launch latency
        _commit("commit8_single", 12, 1, 1, 1, 3, 1, tiled=False, scope="head"),
        # the target's block out of the fused QKV rows, ring of 7, scales chosen from the data, and the slot read back
        _commit("commit8_target_tiled", 40, FRAMES, GRID_H, GRID_W, 7, 2, tiled=True),
        # a small ring with scales chosen from the data
        _read("read8_small", 2, 300, 3, 1, tiled=True),
        # a slot of the target's ring with static scales
        _read("read8_target", 40, tok, 7, 3, tiled=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["linear8", "linear8", "norm8", "commit8", "commit8", "read8"])
    if op == "linear8":
        m, k, n = _log(rng, 1, 4680), _log(rng, 64, 5120), _log(rng, 1, 20480)
        out = rng.choice(["bf16", "fp16", "fp32", "e4m3"])
        case = _linear("", m, k, n, out, rng.random() < 0.8, rng.choice(["none", "silu", "gelu_tanh", "gelu"]),
                       rng.choice([0, _log(rng, 1, m)]), "" if out == "e4m3" else rng.choice(["", "rows", "broadcast"]))
    elif op == "norm8":
        rows, cols = _log(rng, 1, 4680), _log(rng, 16, 5120)
        y = rng.choice(["", "bf16", "fp32"])
        case = _norm("", rows, cols, rng.choice(["bf16", "fp16", "fp32"]), y, rng.choice(["none", "layer", "rms"]),
                     rng.random() < 0.4, rng.choice([0, _log(rng, 1, rows)]), rng.choice([0, _log(rng, 1, rows)]) if y else 0,
                     rng.choice(["none", "rms", "layer"]) if y else "none")
    elif op == "commit8":
        case = _commit("", _log(rng, 1, 40), rng.randint(1, 3), _log(rng, 1, 30), _log(rng, 1, 52), rng.randint(1, 4),
                       rng.randint(0, 3), rng.random() < 0.5, rng.choice(["row", "head"]), rng.random() < 0.7)
    else:
        slots = rng.randint(1, 4)
        case = _read("", _log(rng, 1, 40), _log(rng, 1, 4680), slots, rng.randrange(slots), rng.random() < 0.5)
    del case["name"]
    return case


def work(case):
    """Every input read once and every output written once; the multiply-adds of the products, a few per element elsewhere."""
    if case["op"] == "linear8":
        m, k, n, o = case["m"], case["k"], case["n"], BYTES[case["out"]]
        rows = {"": 0, "rows": m, "broadcast": 1}[case["residual"]]
        groups = -(-m // case["gate"]) if case["gate"] else 0
        blocks = -(-k // 128)
        return {"bytes": (m + n) * k + (m + -(-n // 128)) * blocks + (m + rows) * n * o + 4 * n * (groups + case["bias"]),
                "flops": 2 * m * k * n}
    if case["op"] == "norm8":
        rows, cols = case["rows"], case["cols"]
        vectors = 2 * case["affine"] + (case["post"] != "none")
        vectors += (2 * -(-rows // case["modulate"]) if case["modulate"] else 0)
        vectors += (-(-rows // case["gate"]) if case["gate"] else 0)
        streams = BYTES[case["x"]] + BYTES["e4m3"] + ((BYTES[case["y"]] + BYTES[case["x"]]) if case["y"] else 0)
        return {"bytes": rows * cols * streams + 4 * cols * vectors, "flops": 14 * rows * cols}
    if case["op"] == "commit8":
        elems = case["frames"] * case["grid_h"] * case["grid_w"] * case["heads"] * 128
        # three bf16 tensors in, three of codes out; read back: two of codes in and two bf16 out
        return {"bytes": (9 + (6 if case["tiled"] else 0)) * elems, "flops": 20 * elems}
    elems = case["tokens"] * case["heads"] * 128
    return {"bytes": 6 * elems, "flops": 2 * elems}


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


def _scale_exponent(amax):
    """The smallest e in [-126, 120] with amax <= 448 * 2^e."""
    m, x = torch.frexp(amax)
    e = (x - 9 + (m > 0.875)).clamp(-126, 120)
    return torch.where(amax == 0, -126, torch.where(torch.isinf(amax), 120, e))


def _power(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _blocks(v, block_rows):
    """[row blocks, block_rows, column blocks, 128] of a matrix padded with zeros."""
    r, c = v.shape
    v = torch.nn.functional.pad(v, (0, -c % 128, 0, -r % block_rows))
    return v.view(v.shape[0] // block_rows, block_rows, -1, 128)


def _codes(v):
    return v.clamp(-448, 448).to(torch.float8_e4m3fn)


def _quantised(v, block_rows=1):
    """(codes, scales): E4M3 values of v / scale, one power of two per block_rows x 128 block as an exponent byte."""
    b = _blocks(v, block_rows)
    e = _scale_exponent(b.abs().amax((1, 3)))
    codes = _codes(b * _power(-e)[:, None, :, None]).view(b.shape[0] * block_rows, -1)[:v.shape[0], :v.shape[1]]
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _padded(t, pad):
    """The same matrix in a buffer whose row stride is a multiple of `pad`."""
    buf = torch.zeros((t.shape[0], -(-t.shape[1] // pad) * pad), dtype=torch.uint8, device=t.device)
    buf[:, :t.shape[1]] = t.view(torch.uint8)
    return buf[:, :t.shape[1]]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case)}
    if case["op"] == "linear8":
        m, k, n = case["m"], case["k"], case["n"]
        # quantised matrices as they come: uint8 codes and exponent bytes, row strides multiples of 16
        for what, v, block in (("x", _rows(gen, m, k, torch.float32, spread=4.0), 1),
                               ("w", _rows(gen, n, k, torch.float32, std=1 / math.sqrt(k)), 128)):
            codes, scale = _quantised(v, block)
            s[what], s[what + "_scale"] = _padded(codes, 16), _padded(scale, 16)
        s["bias"] = _vec(gen, n) if case["bias"] else None
        s["gate"] = _vec(gen, -(-m // case["gate"]), n) if case["gate"] else None
        s["residual"] = None
        if case["residual"]:
            rows = _rows(gen, m if case["residual"] == "rows" else 1, n, DTYPES[case["out"]], std=2.0)
            s["residual"] = rows.expand(m, n)
        s["out"] = torch.empty((m, n), device="cuda", dtype=torch.uint8 if case["out"] == "e4m3" else DTYPES[case["out"]])
        s["out_scale"] = torch.empty((m, -(-n // 128)), device="cuda", dtype=torch.uint8) if case["out"] == "e4m3" else None
    elif case["op"] == "norm8":
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
        s["out"] = torch.empty((rows, cols), device="cuda", dtype=torch.uint8)
        s["out_scale"] = torch.empty((rows, -(-cols // 128)), device="cuda", dtype=torch.uint8)
    elif case["op"] == "commit8":
        h, d = case["heads"], 128
        t, c = case["frames"] * case["grid_h"] * case["grid_w"], h * d
        if case["fused"]:
            qkv = _rows(gen, t, 3 * c, torch.bfloat16, std=1.5, spread=4.0)
            s["q"], s["k"], s["v"] = (qkv[:, i * c:(i + 1) * c].unflatten(1, (h, d)) for i in range(3))
        else:
            s["q"], s["k"], s["v"] = (_rows(gen, t, c, torch.bfloat16, std=1.5).view(t, h, d) for _ in range(3))
        width = c if case["scope"] == "row" else d
        s["q_weight"], s["k_weight"] = (_vec(gen, width, std=0.2, mean=1.0) for _ in range(2))
        if not case["tiled"]:
            # sized for values up to 12 to 24 standard deviations, a head with another
            s["inv"] = [448.0 / (12 + 12 * torch.rand(h, generator=gen, device="cuda")) for _ in range(3)]
        s["q8"] = torch.empty((t, h, d), device="cuda", dtype=torch.uint8)
        s["tab_frames"] = (case["block"] + 1) * case["frames"]
        s["table"] = _table(d, s["tab_frames"], case["grid_h"], case["grid_w"]).cuda()
    else:
        h, t, n = case["heads"], case["tokens"], case["slots"]
        for what in ("k", "v"):
            s["ring_" + what] = _codes(torch.randn((h, n, t, 128), generator=gen, device="cuda") * 60)
            shape = (h, n, -(-t // 128)) if case["tiled"] else (h,)
            e = torch.randint(-9, -3, shape, generator=gen, device="cuda")
            s["scale_" + what] = _power(e) if case["tiled"] else 0.02 + 0.02 * torch.rand(shape, generator=gen, device="cuda")
        s["out_k"], s["out_v"] = (torch.empty((t, h, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
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


def _ring_views(cache):
    """The two rings of a cache, [heads, slots, tokens, 128] codes."""
    n = cache.heads * cache.slots * cache.block_tokens * 128
    return [raw[ptr - raw.data_ptr():][:n].view(torch.float8_e4m3fn).view(cache.heads, cache.slots, cache.block_tokens, 128)
            for raw, ptr in ((cache._k_raw, cache.k_ptr), (cache._v_raw, cache.v_ptr))]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2604_17397_b200 import api
        s["api"] = api
    if case["op"] == "commit8":
        t, h = s["q"].shape[:2]
        if own:
            cache = s["cache"] = api.Cache(case["slots"], h, t, 128, e4m3=True, tile_scales=case["tiled"])
            zero = torch.zeros((t, h, 128), dtype=torch.bfloat16, device="cuda")
            one = torch.ones(h, device="cuda")
            for b in range(case["block"]):
                if case["tiled"]:
                    api.sdvg_kv_commit_e4m3_tiled(cache, zero, zero, b, api.SDVG_FINAL)
                else:
                    api.sdvg_kv_commit_e4m3(cache, zero, zero, one, one, b, api.SDVG_FINAL)
            s["ring_k"], s["ring_v"] = _ring_views(cache)
            s["scope"] = api.SDVG_SCOPE_ROW if case["scope"] == "row" else api.SDVG_SCOPE_HEAD
            if case["tiled"]:
                s["q_scale"] = torch.empty((h, cache.tiles), device="cuda")
                s["workspace"] = api.qk_norm_workspace(t)
        else:
            s["ring_k"], s["ring_v"] = (torch.zeros((h, case["slots"], t, 128), device="cuda", dtype=torch.float8_e4m3fn)
                                        for _ in range(2))
        if case["tiled"]:
            s["out_k"], s["out_v"] = (torch.empty((t, h, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    elif own and case["op"] == "read8":
        cache = s["cache"] = api.Cache(case["slots"], case["heads"], case["tokens"], 128, e4m3=True, tile_scales=case["tiled"])
        for ring, what in zip(_ring_views(cache), "kv"):
            ring.copy_(s["ring_" + what])
        if case["tiled"]:
            cache.k_scale.copy_(s["scale_k"])
            cache.v_scale.copy_(s["scale_v"])
            s["scale_k"] = s["scale_v"] = None                   # the ring's own
    elif own and case["op"] == "linear8":
        s["workspace"] = api.attn_workspace()
        s["act"] = {"none": api.SDVG_ACT_NONE, "silu": api.SDVG_ACT_SILU, "gelu_tanh": api.SDVG_ACT_GELU_TANH,
                    "gelu": api.SDVG_ACT_GELU}[case["act"]]
    elif own:
        kinds = {"none": api.SDVG_NORM_NONE, "rms": api.SDVG_NORM_RMS, "layer": api.SDVG_NORM_LAYER}
        s["norm"], s["post_norm"] = kinds[case["norm"]], kinds[case["post"]]
    return s


# ---------------------------------------------------------------- the operators

def run(s):
    return {"linear8": _run_linear, "norm8": _run_norm, "commit8": _run_commit, "read8": _run_read}[s["case"]["op"]](s)


def _values(codes):
    return codes.view(torch.float8_e4m3fn)


def _dequantised(codes, scale, block_rows, dtype=torch.float32):
    r, c = codes.shape
    f = scale.view(torch.float8_e8m0fnu).to(dtype).repeat_interleave(128, 1)[:, :c]
    return _values(codes).to(dtype) * f.repeat_interleave(block_rows, 0)[:r]


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
        s["api"].sdvg_linear_e4m3(s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"], s["workspace"], bias=s["bias"],
                                  act=s["act"], residual=s["residual"], gate=s["gate"], gate_rows=case["gate"],
                                  out_scale=s["out_scale"])
        if case["out"] == "e4m3":
            return _values(s["out"]), s["out_scale"].view(torch.float8_e8m0fnu)
        return s["out"]
    v = _dequantised(s["x"], s["x_scale"], 1) @ _dequantised(s["w"], s["w_scale"], 128).t()
    if s["bias"] is not None:
        v = v + s["bias"]
    v = _act(v, case["act"])
    if s["gate"] is not None:
        v = v * _of_rows(s["gate"], case["m"], case["gate"])
    if s["residual"] is not None:
        v = v + s["residual"].float()
    return _quantised(v) if case["out"] == "e4m3" else v.to(DTYPES[case["out"]])


def _norm_plain(v, kind, eps=1e-6):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v if kind == "none" else v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)


def _run_norm(s):
    case = s["case"]
    if own:
        s["api"].sdvg_gated_norm_e4m3(s["x"], s["out"], s["out_scale"], y=s["y"], gate=s["gate"], gate_rows=case["gate"],
                                      post_norm=s["post_norm"], post_weight=s["post_weight"], x_out=s["x_out"],
                                      norm=s["norm"], weight=s["weight"], bias=s["bias"], scale=s["scale"],
                                      shift=s["shift"], modulate_rows=case["modulate"], eps=1e-6)
        out = (_values(s["out"]), s["out_scale"].view(torch.float8_e8m0fnu))
        return (s["x_out"], *out) if s["y"] is not None else out
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
    o = _quantised(o)
    return (v.to(s["x"].dtype), *o) if s["y"] is not None else o


def _rotary(s):
    """cos and sin of every token's pairs: [tokens, 1, dim / 2] each."""
    case, tab = s["case"], s["table"]
    t = torch.arange(s["q"].shape[0], device="cuda")
    hw = case["grid_h"] * case["grid_w"]
    at = (case["block"] * case["frames"] + t // hw, t % hw // case["grid_w"], t % case["grid_w"])
    begin, cs = 0, []
    for count, positions, where in zip(_pairs(128), (s["tab_frames"], case["grid_h"], case["grid_w"]), at):
        cs.append(tab[begin:begin + 2 * count * positions].view(positions, count, 2)[where])
        begin += 2 * count * positions
    cs = torch.cat(cs, 1)[:, None]
    return cs[..., 0], cs[..., 1]


def _tile_scales(v):
    """[tokens, heads, 128] -> the exponent of every (tile of 128 tokens, head)."""
    t = v.shape[0]
    v = torch.nn.functional.pad(v, (0, 0, 0, 0, 0, -t % 128)).view(-1, 128, v.shape[1], 128)
    return _scale_exponent(v.abs().amax((1, 3)))


def _run_commit(s):
    case = s["case"]
    slot = case["block"] % case["slots"]
    if own:
        api = s["api"]
        grid, offset = (case["frames"], case["grid_h"], case["grid_w"]), case["block"] * case["frames"]
        if case["tiled"]:
            api.sdvg_qk_norm_rope3d_commit_e4m3_tiled(s["cache"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"],
                                                      s["scope"], 1e-6, s["q8"], s["q_scale"], grid, offset, s["table"],
                                                      s["tab_frames"], case["block"], api.SDVG_STAGE, s["workspace"])
            api.sdvg_cache_read_block_e4m3(s["cache"], slot, s["out_k"], s["out_v"])
            return _values(s["q8"]), s["ring_k"][:, slot], s["ring_v"][:, slot], s["out_k"], s["out_v"]
        api.sdvg_qk_norm_rope3d_commit_e4m3(s["cache"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["scope"],
                                            1e-6, s["q8"], *s["inv"], grid, offset, s["table"], s["tab_frames"],
                                            case["block"], api.SDVG_STAGE)
        return _values(s["q8"]), s["ring_k"][:, slot], s["ring_v"][:, slot]
    cos, sin = _rotary(s)
    turned = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        v = x.float()
        if case["scope"] == "row":
            v = (_norm_plain(v.flatten(1), "rms") * w).view(v.shape)
        else:
            v = _norm_plain(v, "rms") * w
        re, im = v[..., 0::2], v[..., 1::2]
        turned.append(torch.stack([re * cos - im * sin, re * sin + im * cos], -1).flatten(2))
    turned.append(s["v"].float())
    if case["tiled"]:
        tokens = torch.arange(turned[0].shape[0], device="cuda")
        e = [_tile_scales(v)[tokens // 128][..., None] for v in turned]
        q, k, v = (_codes(v * _power(-x)) for v, x in zip(turned, e))
    else:
        q, k, v = (_codes(v * inv[:, None]) for v, inv in zip(turned, s["inv"]))
    s["ring_k"][:, slot] = k.transpose(0, 1)
    s["ring_v"][:, slot] = v.transpose(0, 1)
    if not case["tiled"]:
        return q, s["ring_k"][:, slot], s["ring_v"][:, slot]
    # and back, from the ring
    s["out_k"].copy_(s["ring_k"][:, slot].transpose(0, 1).float() * _power(e[1]))
    s["out_v"].copy_(s["ring_v"][:, slot].transpose(0, 1).float() * _power(e[2]))
    return q, s["ring_k"][:, slot], s["ring_v"][:, slot], s["out_k"], s["out_v"]


def _run_read(s):
    case = s["case"]
    if own:
        s["api"].sdvg_cache_read_block_e4m3(s["cache"], case["slot"], s["out_k"], s["out_v"], s["scale_k"], s["scale_v"])
        return s["out_k"], s["out_v"]
    got = []
    for what in "kv":
        v, scale = s["ring_" + what][:, case["slot"]].float(), s["scale_" + what]
        if case["tiled"]:
            scale = scale[:, case["slot"]].repeat_interleave(128, 1)[:, :case["tokens"], None]
        else:
            scale = scale[:, None, None]
        got.append((v * scale).transpose(0, 1).contiguous().to(torch.bfloat16))
    return tuple(got)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"linear8": _exact_linear, "norm8": _exact_norm, "commit8": _exact_commit, "read8": _exact_read}[case["op"]](case, s)


def _double(s):
    return {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.dtype != torch.uint8}


def _exact_scale(largest):
    """2^e with the smallest e in [-126, 120] that brings `largest` to 448 or less."""
    return torch.exp2(torch.ceil(torch.log2(largest / 448)).clamp(-126, 120))


def _exact_rows(z):
    """(values in units of their scales, scales) with one scale per 128 columns; the values without their rounding."""
    n = z.shape[1]
    blocks = torch.nn.functional.pad(z, (0, -n % 128)).unflatten(1, (-1, 128))
    scale = _exact_scale(blocks.abs().amax(2))
    return (blocks / scale[..., None]).flatten(1)[:, :n], scale


def _repeat(vectors, rows, per_group):
    return vectors.repeat_interleave(per_group, 0)[:rows]


def _exact_matrix(codes, scale, block_rows):
    n, k = codes.shape
    z = codes.view(torch.float8_e4m3fn).double()
    power = torch.exp2(scale.double() - 127)
    at = torch.arange(n, device="cuda")[:, None] // block_rows, torch.arange(k, device="cuda")[None] // 128
    return z * power[at]


def _exact_linear(case, s):
    d = _double({k: v for k, v in s.items() if not k.startswith("out")})
    z = torch.einsum("mk,nk->mn", _exact_matrix(s["x"], s["x_scale"], 1), _exact_matrix(s["w"], s["w_scale"], 128))
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
    if "residual" in d:
        z += d["residual"]
    return _exact_rows(z) if case["out"] == "e4m3" else z


def _exact_normed(v, kind):
    if kind == "none":
        return v
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    return (v - mean) / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + 1e-6)


def _exact_norm(case, s):
    d = _double(s)
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
    o = _exact_rows(o)
    return (z, *o) if case["y"] else o


def _exact_commit(case, s):
    d = _double(s)
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
    got.append(d["v"])
    if case["tiled"]:
        for z in got:
            for part in z.split(128):
                part /= _exact_scale(part.abs().amax((0, 2)))[:, None]
        # what is read back is the codes times their scales: rounded to 8 bits, for which 64 bits have no value
        return got[0], got[1].transpose(0, 1), got[2].transpose(0, 1), None, None
    q, k, v = ((z * inv.double()[:, None]).clamp(-448, 448) for z, inv in zip(got, s["inv"]))
    return q, k.transpose(0, 1), v.transpose(0, 1)


def _exact_read(case, s):
    got = []
    for what in ("k", "v"):
        z, scale = s["ring_" + what].double()[:, case["slot"]], s["scale_" + what].double()
        if case["tiled"]:
            z = torch.stack([z[:, i] * scale[:, case["slot"], i // 128, None] for i in range(case["tokens"])])
        else:
            z = torch.einsum("htd,h->thd", z, scale)
        got.append(z)
    return got
