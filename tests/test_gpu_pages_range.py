"""Pages of the largest pools on the GPU, against plain loops over the pages that the table names."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests.gpu_util import device, say

pytestmark = pytest.mark.gpu
TOP = (1 << 31) - 1


@pytest.mark.parametrize("num_pages", [TOP - 32, TOP - 30, TOP])
def test_pools_of_the_most_pages(num_pages):
    """2^31 - 1 pages and the numbers around the last full word of a bitmap: free pages from the front, one shared
    page copied, the highest ones moved to the front."""
    dev = device()
    p = D.CacheParams(2, 1, 128, 16, num_pages, 4, D.CACHE_BF16)
    rows = [[0, num_pages - 1, 7, -1], [num_pages - 2, 3, 7, num_pages]]
    table = torch.tensor(rows, dtype=torch.int32) if num_pages <= TOP - 1 else torch.tensor([rows[0], rows[1][:3] + [-5]], dtype=torch.int32)
    table = table.to(dev)
    out = torch.empty_like(table)
    pairs = torch.full((num_pages // 2, 2), -9, dtype=torch.int32, device=dev)
    totals, granted = (torch.full((2,), -9, dtype=torch.int32, device=dev) for _ in range(2))
    ws = torch.empty(D.pages_workspace_size(p), dtype=torch.uint8, device=dev)
    start = torch.tensor([40, 56], dtype=torch.int32, device=dev)
    say(f"pages_reserve pages={num_pages}")
    D.pages_reserve(p, table, out, 8, start, None, pairs, totals, granted, ws)     # columns 2 and 3
    torch.cuda.synchronize()
    assert out.tolist() == [[0, num_pages - 1, 1, -1], [num_pages - 2, 3, 7, 2]]
    assert pairs[:2].tolist() == [[7, 1], [-9, -9]] and totals.tolist() == [1, num_pages - 5 - 2] and granted.tolist() == [1, 1]
    say(f"pages_compact pages={num_pages}")
    moved = torch.empty_like(table)
    D.pages_compact(p, table, moved, pairs, totals, ws)                             # in use: 0, 3, 7 and the last two
    torch.cuda.synchronize()
    assert totals.tolist() == [3, 5] and pairs[:4].tolist() == [[7, 1], [num_pages - 2, 2], [num_pages - 1, 4], [-9, -9]]
    assert moved.tolist() == [[0, 4, 1, -1], [2, 3, 1, -1]]
    del pairs, ws
    torch.cuda.empty_cache()
