"""Few tiles of 128 query rows over a long context: many blocks share a tile, and
their partial results are joined by eight groups of lanes.  Tolerance: test_gpu_paged.py's."""
import pytest

from tests.test_gpu_cache import BF, E8
from tests.test_gpu_paged import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [E8, BF])
@pytest.mark.parametrize("b,n,lens,nodes", [(1, 200, [65459], [200]), (1, 200, [300], [130]), (2, 100, [40001, 17], [100, 5])])
def test_many_parts_of_wide_tiles(kind, b, n, lens, nodes):
    """A ragged end, fewer steps than blocks, a long request beside a short one; pages missing."""
    Case(b, n, 65536, 8, 1, 64, kind, lens=lens, num_nodes=nodes, holes=[(0, 1, -1), (0, 400, 1 << 28)], seed=21).check(heads=[0, 7])
