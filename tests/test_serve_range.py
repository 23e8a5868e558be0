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


def test_accuracy_of_the_exponentials():
    """2^(n / 32) 2^(f / 32) with |f| <= 1/2 by a series to degree 4, its argument rounded once more where it is
    formed from m c32 < 2^20 (half a unit: 2^-34): 3e-12 in all.  A token's share is a quotient of two."""
    f = np.linspace(-0.5, 0.5, 100001)
    x = f * np.log(2.0) / 32
    series = 1 + x * (1 + x / 2 * (1 + x / 3 * (1 + x / 4)))
    off = np.abs(series / np.exp2(f / 32) - 1).max()
    assert 1e-12 < off < 1.3e-12
    assert off + 2.0 ** -34 * np.log(2.0) / 32 + 2.0 ** -38 * np.log(2.0) / 32 * 3 < 3e-12
