"""Bookkeeping and refusals of kvq_cache_fork, kvq_cache_truncate and kvq_cache_read on accounting-only caches."""
import os

import pytest

import paper_2505_18610_amd as kq

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")
A = 1 << 20  # an address that is never used


class _Tokens:  # stands for a tensor of n new tokens (an accounting-only cache looks at the count alone)
    def __init__(self, n):
        self.shape = (0, 0, n, 128)


def make(batch=2, layers=1, page=64, policy=kq.KVQ_POLICY_PAPER, window=0, budget=1 << 40, max_tokens=4096, arena=1 << 28, kv=2, group=32, tiers=()):
    c = kq.KvqCache(kq.KvqConfig(layers, batch, 4 * kv, kv, max_tokens, page_tokens=page, policy=policy, window=window, group=group),
                    [budget] * layers, [2] * layers, arena_bytes=arena)
    for n, bits in tiers:
        kq.load_library().kvq_quantize_append(c.handle, 0, None, None, n, bits, None)
    return c


def fork(d, s, layer=0, n=-1, m=None):
    return kq.load_library().kvq_cache_fork(d.handle if d else None, s.handle if s else None, layer, m, n, None)


TIERS = [(128, 2), (64, 8), (100, 16)]


def test_fork_keeps_widths_and_counts_bytes():
    s, d = make(tiers=TIERS), make(batch=5)
    free = d.kvq_cache_arena_free_bytes()
    assert fork(d, s, m=A) == kq.KVQ_OK
    a, b = s.kvq_cache_describe(0), d.kvq_cache_describe(0)
    assert a[0] == b[0] and a[2:] == b[2:] and 5 * a[1] == 2 * b[1]
    held = free - d.kvq_cache_arena_free_bytes()
    assert fork(d, s, m=A) == kq.KVQ_OK and free - d.kvq_cache_arena_free_bytes() == held
    assert fork(d, s, n=150, m=A) == kq.KVQ_OK and d.kvq_cache_describe(0)[2] == 150
    assert fork(d, s, n=0, m=A) == kq.KVQ_OK and d.kvq_cache_arena_free_bytes() == free


def test_fork_in_place():
    s = make(tiers=TIERS)
    before, free = s.kvq_cache_describe(0), s.kvq_cache_arena_free_bytes()
    assert fork(s, s, m=A) == kq.KVQ_OK
    assert s.kvq_cache_describe(0) == before and s.kvq_cache_arena_free_bytes() == free
    assert fork(s, s, n=100, m=A) == kq.KVQ_OK and s.kvq_cache_describe(0)[2] == 100


def test_refusals():
    s = make(tiers=TIERS)
    d = make(tiers=[(10, 4)])
    state = d.kvq_cache_describe(0), d.kvq_cache_arena_free_bytes()
    assert fork(None, s) == kq.KVQ_E_INVALID and fork(d, None) == kq.KVQ_E_INVALID
    for bad in (dict(layer=-1), dict(layer=1), dict(n=-2), dict(m=A + 2)):
        assert fork(d, s, **bad) == kq.KVQ_E_INVALID
    for other in (make(page=32), make(kv=1), make(group=64)):
        assert fork(other, s) == kq.KVQ_E_INVALID
    assert fork(make(batch=3), s) == kq.KVQ_E_INVALID                       # sequences that nothing is said of
    assert fork(make(batch=3), make(batch=1, tiers=TIERS)) == kq.KVQ_OK
    i = make()
    i.kvq_cache_set_option(kq.KVQ_OPT_TIER16, kq.KVQ_TIER16_INT16)
    assert fork(i, s) == kq.KVQ_E_INVALID
    assert fork(d, s, n=293) == kq.KVQ_E_STATE
    assert fork(make(max_tokens=200), s) == kq.KVQ_E_STATE
    small = make(budget=10000, tiers=[(10, 4)])
    before = small.kvq_cache_describe(0)
    assert fork(small, s) == kq.KVQ_E_BUDGET and small.kvq_cache_describe(0) == before
    full = make(tiers=[(10, 4)], arena=5 << 20)
    before = full.kvq_cache_describe(0), full.kvq_cache_arena_free_bytes()
    big = make(tiers=[(2048, 16)])
    assert fork(full, big) == kq.KVQ_E_OOM and (full.kvq_cache_describe(0), full.kvq_cache_arena_free_bytes()) == before
    assert (d.kvq_cache_describe(0), d.kvq_cache_arena_free_bytes()) == state


@pytest.mark.parametrize("kind", [dict(policy=kq.KVQ_POLICY_OLDEST_FIRST), dict(window=64)])
def test_a_cut_inside_a_narrow_page(kind):
    s = make(tiers=TIERS, **kind)
    lib = kq.load_library()
    for n in (100, 129):
        assert lib.kvq_cache_truncate(s.handle, 0, n, None) == kq.KVQ_E_STATE
        assert fork(s, s, n=n) == kq.KVQ_E_STATE and fork(make(**kind), s, n=n) == kq.KVQ_E_STATE
        assert fork(make(), s, n=n) == kq.KVQ_OK  # there appends go on at the block's width
    for n in (250, 192, 128, 64, 0):
        assert lib.kvq_cache_truncate(s.handle, 0, n, None) == kq.KVQ_OK and s.kvq_cache_describe(0)[2] == n


def test_truncate():
    s = make(tiers=TIERS)
    lib, whole = kq.load_library(), make().kvq_cache_arena_free_bytes()
    assert lib.kvq_cache_truncate(None, 0, 0, None) == kq.KVQ_E_INVALID
    for layer, n in ((-1, 0), (1, 0), (0, -1)):
        assert lib.kvq_cache_truncate(s.handle, layer, n, None) == kq.KVQ_E_INVALID
    assert lib.kvq_cache_truncate(s.handle, 0, 293, None) == kq.KVQ_E_STATE
    for n in (292, 200, 192, 191, 130, 100, 5, 0):
        assert lib.kvq_cache_truncate(s.handle, 0, n, None) == kq.KVQ_OK
        ref = make(tiers=[(min(m, max(0, n - t)), b) for t, (m, b) in zip((0, 128, 192), TIERS) if n > t])
        assert s.kvq_cache_describe(0)[:3] == ref.kvq_cache_describe(0)[:3]
        assert s.kvq_cache_arena_free_bytes() == ref.kvq_cache_arena_free_bytes()
    assert s.kvq_cache_arena_free_bytes() == whole


def test_read():
    s = make(tiers=TIERS)
    lib = kq.load_library()
    for layer, t, n, k, v in ((-1, 0, 1, A, A), (1, 0, 1, A, A), (0, -1, 1, A, A), (0, 0, -1, A, A), (0, 0, 1, None, A), (0, 0, 1, A, None),
                              (0, 0, 1, A + 8, A), (0, 0, 1, A, A + 4)):
        assert lib.kvq_cache_read(s.handle, layer, t, n, k, v, 0, None) == kq.KVQ_E_INVALID
    assert lib.kvq_cache_read(None, 0, 0, 1, A, A, 0, None) == kq.KVQ_E_INVALID
    assert lib.kvq_cache_read(s.handle, 0, 0, 1, A, A, 0, None) == kq.KVQ_E_STATE  # nothing is held on a device
