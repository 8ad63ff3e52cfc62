"""Chunk attention of sequences whose context, or whole window, lies behind the last position that the block table has: a table of one row, whose last entry nothing follows."""
import pytest

from tests.test_gpu_chunk import _check, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("new,heads,kv,dim", [(1, 2, 1, 64), (9, 8, 2, 128), (40, 8, 1, 128), (70, 4, 1, 256)])
def test_one_row(new, heads, kv, dim, tree):
    cache, table, first, _, q, seen, positions = _setup(new, [new], [50], heads, kv, dim, tree=tree)
    cap = table.shape[1] * 16
    for behind in (-1, 0, 1, 40, 1 << 29):
        for window, sinks in ((0, 0), (1, 0), (30, 0), (30, 5)):
            at = None if positions is None else positions - 50 + cap + behind
            _check((cache, table, first, [cap + behind], q, seen, at), window, sinks)
