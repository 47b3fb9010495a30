"""What the tests of operators with 8-bit outputs share."""
import numpy as np

from dense_utils import assert_close
from oracle import e4m3_blocks_oracle as B


def check_quantised(codes, scale, ref, err):
    """Rows of codes of values known up to err: the scale is that of some value within it, the codes are within half a step."""
    e = scale.cpu().numpy().astype(np.int64)
    lo, hi = (B.scale_bytes(np.maximum(np.abs(ref) + d, 0), 1).astype(np.int64) for d in (-err, err))
    assert ((lo <= e) & (e <= hi)).all()
    f = B.of_elements(scale.cpu().numpy(), *ref.shape, 1)
    tol = err + B.half_step(np.abs(ref) + err, f)
    assert_close(B.values(codes.cpu().numpy(), scale.cpu().numpy(), 1), ref, tol, "codes")
