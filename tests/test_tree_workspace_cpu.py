"""The workspace that kvq_tree_workspace_bytes names is enough for the cache at every length, whichever kernel takes it there."""
import os

import pytest

import paper_2505_18610_amd as kq

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")


def needed(tiles, batch, q, kv, nodes):
    c = kq.KvqCache(kq.KvqConfig(1, batch, q, kv, 32 * tiles, page_tokens=32), [1 << 40], [2], arena_bytes=1 << 32)
    return c.kvq_tree_workspace_bytes(nodes)


# the kernels for 16 and 32 rows, pairs of wavefronts, four and twelve, units that fill the device and a few
SHAPES = [(1, 64, 8, 1), (4, 64, 8, 1), (1, 16, 8, 16), (1, 28, 4, 16), (1, 8, 2, 4), (2, 8, 8, 33), (1, 64, 8, 25), (4, 40, 8, 64), (1, 8, 1, 24), (1, 16, 1, 1024),
          (16, 8, 2, 20)]


@pytest.mark.parametrize("shape", SHAPES)
def test_a_longer_cache_needs_no_less(shape):
    most = 0
    for tiles in [*range(1, 700), *range(700, 6000, 37)]:
        now = needed(tiles, *shape)
        assert now >= most, (tiles, now, most)
        most = now


def test_lengths_that_take_more_than_their_doubles():
    assert needed(2048, 1, 64, 8, 1) >= needed(1015, 1, 64, 8, 1) >= 4325376
    assert needed(64, 4, 64, 8, 1) >= needed(56, 4, 64, 8, 1)
    # no more than what as many ranges as are ever taken hold
    assert needed(1 << 16, 1, 64, 8, 1) <= 65 * 8 * (8 * 64 * 4 + 64) * 4
