"""Numbers that serve.h states of the cache's 8-bit rows and of the verification's arithmetic."""
import numpy as np

from tests import serve_ref as S


def test_what_falls_into_the_subnormals():
    """A row's largest is above 224 * 2^e, the least normal number is 2^-6: below 2^-6 / 224 = 2^-13.8 of the largest."""
    top = (np.arange(0x4000, 0x4100, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)   # two binades
    small = top[:, None] * 2.0 ** -np.arange(13.0, 16.0, 1.0 / 16)
    e = S.row_exponent(top[:, None])
    held = small * 2.0 ** -e[:, None].astype(np.float64)
    subnormal = held < 2.0 ** -6
    ratio = small / top[:, None]
    assert (ratio[subnormal] < 2.0 ** -6 / 224).all() and 2.0 ** -13.81 < 2.0 ** -6 / 224 < 2.0 ** -13.8
    assert ratio[subnormal].max() > 2.0 ** -13.9 and (subnormal | (ratio >= 2.0 ** -6 / 448)).all()
    # where the least exponent holds, larger parts of the row do
    assert S.row_exponent(np.array([[2.0 ** -100]]))[0] == S.EXP_LOW
