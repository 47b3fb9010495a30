"""Tolerances of the dense operators' tests, derived from the arithmetic (all inputs and results as fp64 arrays).

U = 2^-24 is half a step of fp32.  Sums: adding n terms in any order in fp32 is off by at most n * 2U * sum|terms| even
when every addition truncates.  A value rounded to type t is off by eps(t) / 2 relative (plus half the smallest
subnormal).
"""
import numpy as np
import torch

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}


def rounding(ref, dtype):
    return torch.finfo(dtype).eps / 2 * np.abs(ref) + TINY[dtype]


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def linear_tolerance(x, w, bias, act, gate_of_rows, residual, ref, dtype):
    from oracle import dense_oracle as O
    mag = np.abs(x) @ np.abs(w).T
    v = x @ w.T + (0 if bias is None else bias)
    err = (x.shape[1] + 2) * 2 * U * (mag + (0 if bias is None else np.abs(bias)))
    a = O.activation(v, act)
    if act != "none":
        # slopes of the activations are below 1.13; their own error is relative: the exponential's argument z is off by
        # 4U relative, e^z by |z| 4U + (2 + 1.2 |z|) 2U, |z| <= 88 where the value is not yet zero: 2^-14 in all
        err = 1.13 * err + 2.0 ** -14 * np.abs(a) + 1e-36
    g = 1.0 if gate_of_rows is None else np.abs(gate_of_rows)
    err = g * err + 4 * U * (g * np.abs(a) + (0 if residual is None else np.abs(residual)))
    return err + rounding(np.abs(ref) + err, dtype)


def norm_error(v, e_v, kind, eps):
    """(normed, bound on its error) for values v known up to e_v; a sum of n values runs at most n / 64 + 32 additions deep."""
    from oracle import dense_oracle as O
    n = v.shape[-1]
    o = O.norm_ref(v, kind, eps)
    if kind == "none":
        return o, e_v
    depth = (n / 64 + 32) * U
    mean_abs = np.abs(v).mean(-1, keepdims=True)
    mean = v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    e_mean = depth * mean_abs + e_v.mean(-1, keepdims=True) if kind == "layer" else 0.0
    d = v - mean
    e_d = e_v + e_mean + U * (np.abs(d) + np.abs(v))
    rstd = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    # variance: relative depth of the sum plus what the centred values' errors do to it (first and second order)
    e_var = (2 * np.abs(d) * e_d + e_d * e_d).mean(-1, keepdims=True) + (depth + 4 * U) / rstd ** 2
    rel = np.minimum(e_var * rstd ** 2, 1.0)
    return o, rstd * e_d + np.abs(o) * (rel + 6 * U)


def gated_norm_tolerance(x, y, post, post_weight, gate_of_rows, norm, weight, bias, scale, shift, eps, refs, x_dtype, out_dtype):
    """Bounds for (x_out, out)."""
    e_s = np.zeros_like(x)
    if y is not None:
        o, e = norm_error(y, np.zeros_like(y), post, eps)
        f = (1.0 if post_weight is None else np.abs(post_weight)) * (1.0 if gate_of_rows is None else np.abs(gate_of_rows))
        e_s = f * (e + 4 * U * np.abs(o)) + 2 * U * (np.abs(x) + f * np.abs(o))
    s, ref = refs
    o, e = norm_error(s, e_s, norm, eps)
    terms = np.abs(o)
    for factor, addend in ((weight, bias), (None if scale is None else 1 + np.abs(scale), shift)):
        if factor is not None:
            e, terms = e * np.abs(factor), terms * np.abs(factor)
        if addend is not None:
            terms = terms + np.abs(addend)
    e = e + 6 * U * terms
    return e_s + rounding(np.abs(s) + e_s, x_dtype), e + rounding(np.abs(ref) + e, out_dtype)


def assert_close(got, ref, tol, what=""):
    """Elementwise |got - ref| <= tol; infinities and NaN in the same places."""
    got = f64(got) if torch.is_tensor(got) else got
    assert got.shape == ref.shape, (got.shape, ref.shape)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in other places"
    fine = np.isfinite(ref)
    inf = ~fine & ~np.isnan(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities differ"
    over = np.abs(got[fine] - ref[fine]) - np.broadcast_to(tol, ref.shape)[fine]
    assert not over.size or over.max() <= 0, f"{what}: {int((over > 0).sum())} of {over.size} beyond the bound, worst by {over.max():.3e}"
