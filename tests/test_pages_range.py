"""The largest pools that the calls on a page table take, without a GPU."""
import pytest

from paper_2608_13524_amd import dartree as D

TOP = (1 << 31) - 1


@pytest.mark.parametrize("num_pages", [1, 31, 32, 33, TOP - 32, TOP - 31, TOP - 30, TOP - 1, TOP])
def test_workspace_holds_the_bitmaps_and_the_free_list(num_pages):
    """Two bitmaps of a bit a page and a number for each page and request, each rounded up to 256 bytes."""
    up = lambda n: (n + 63) // 64 * 64 * 4
    p = D.CacheParams(5, 1, 128, 16, num_pages, 3, D.CACHE_BF16)
    assert D.pages_workspace_size(p) == 2 * up((num_pages + 31) // 32) + up(5) + up(num_pages)
