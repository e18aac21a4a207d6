"""Refusals of kvq_tree_attention and its workspace sizes; nothing is launched here."""
import os

import pytest

import paper_2505_18610_amd as kq

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")
A = 1 << 20  # an address that is never used


@pytest.fixture(scope="module")
def cache():
    return kq.KvqCache(kq.KvqConfig(2, 2, 8, 2, 4096, page_tokens=64), [1 << 30] * 2, [2] * 2, arena_bytes=1 << 28)


def call(cache, layer=0, q=A, k=A, v=A, n=4, mask=A, out=A, scale=0.0, ws=None, handle=True):
    return kq.load_library().kvq_tree_attention(cache.handle if handle else None, layer, q, k, v, n, mask, 0, out, 0, scale, ws, 0, None)


@pytest.mark.parametrize("bad", [
    dict(handle=False), dict(layer=-1), dict(layer=2), dict(q=None), dict(k=None), dict(v=None), dict(mask=None), dict(out=None), dict(n=0),
    dict(n=-1), dict(n=1025), dict(q=A + 8), dict(k=A + 2), dict(v=A + 4), dict(out=A + 8), dict(mask=A + 2), dict(ws=A + 8),
    dict(scale=float("nan")), dict(scale=float("inf"))])
def test_refusals(cache, bad):
    assert call(cache, **bad) == kq.KVQ_E_INVALID


def test_accounting_only_cache(cache):
    assert call(cache) == kq.KVQ_E_STATE


def test_workspace(cache):
    sizes = [cache.kvq_tree_workspace_bytes(n) for n in (1, 4, 16, 64, 1024)]
    assert all(s > 0 and s % 16 == 0 for s in sizes[:3])
    assert cache.kvq_tree_workspace_bytes(0) == 0 and cache.kvq_tree_workspace_bytes(1025) == 0
    short = kq.KvqCache(kq.KvqConfig(1, 1, 8, 2, 64, page_tokens=64), [1 << 30], [2], arena_bytes=1 << 26)
    assert short.kvq_tree_workspace_bytes(8) == 0  # two tiles are one range
