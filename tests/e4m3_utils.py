"""What the tests of operators with 8-bit outputs share."""
import numpy as np

from dense_utils import assert_close
from oracle import e4m3_blocks_oracle as B
from oracle import sdvg_oracle as O


def check_quantised(codes, scale, ref, err):
    """Rows of codes of values known up to err: the scale is that of some value within it, the codes are within half a step."""
    e = scale.cpu().numpy().astype(np.int64)
    lo, hi = (B.scale_bytes(np.maximum(np.abs(ref) + d, 0), 1).astype(np.int64) for d in (-err, err))
    assert ((lo <= e) & (e <= hi)).all()
    f = B.of_elements(scale.cpu().numpy(), *ref.shape, 1)
    tol = err + B.half_step(np.abs(ref) + err, f)
    assert_close(B.values(codes.cpu().numpy(), scale.cpu().numpy(), 1), ref, tol, "codes")


def half_step_tiles(codes, scale, ref, err):
    """Codes [tokens, heads, 128] with a scale per tile of 128 tokens and head ([heads, tiles]) of values known up to err."""
    tokens, heads, _ = ref.shape
    for h in range(heads):
        for t in range(-(-tokens // 128)):
            part = slice(128 * t, 128 * t + 128)
            a, d = np.abs(ref[part, h]), err[part, h]
            lo, hi = (O.e4m3_tile_scale_exponent(np.nan_to_num(np.maximum(a + x, 0)).max()) for x in (-d, d))
            assert 2.0 ** lo <= scale[h, t] <= 2.0 ** hi, (h, t)
    f = scale.T[np.arange(tokens) // 128][..., None].astype(np.float64)
    tol = err + B.half_step(np.abs(ref) + err, f)
    assert_close(O.e4m3_decode(codes.cpu().numpy()) * f, ref, tol, "codes")
