"""Numbers that serve.h states of the cache's 8-bit rows and of the verification's arithmetic."""
import numpy as np

from paper_2608_13524_amd import dartree as D
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


def test_a_workspace_belongs_to_its_sizes():
    """Smaller calls can need more than larger ones; never more than 65 MiB for attention."""
    def attention(b, n, ctx, heads=(32, 8)):
        return D.tree_attention_paged_workspace_size(D.AttnParams(b, n, ctx, *heads, 128, 0.1),
                                                     D.CacheParams(b, heads[1], 128, 64, 10, ctx // 64, D.CACHE_E4M3))
    assert attention(4, 512, 2048) == 0 < attention(2, 512, 2048)
    most = max(attention(b, n, ctx, heads) for b in (1, 3, 8, 64) for n in (1, 4, 16, 33, 100, 512, 4096)
               for ctx in (64, 1024, 4096, 65536) for heads in ((32, 8), (8, 8), (8, 1)))
    assert most == 65 << 20
    assert D.verify_tree_workspace_size(8, 64, 16, 151936) < D.verify_tree_workspace_size(4, 64, 16, 151936)
