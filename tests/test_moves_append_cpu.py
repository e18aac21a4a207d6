"""Blocks go on behind a fork or a cut: what an append that leaves the width to the policy does there, on accounting-only caches."""
import os

import pytest

import paper_2505_18610_amd as kq
from test_moves_cpu import A, TIERS, fork, make

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")


def append(c, n, bits=0):
    return kq.load_library().kvq_quantize_append(c.handle, 0, None, None, n, bits, None)


def widths(c):
    """Width of every token."""
    return [b for t0, t1, b in c.kvq_cache_describe(0)[0] for _ in range(t0, t1)]


def truncated(n, **kw):
    c = make(tiers=TIERS, **kw)
    assert kq.load_library().kvq_cache_truncate(c.handle, 0, n, None) == kq.KVQ_OK
    return c


def forked(n, **kw):
    c = make(**kw)
    assert fork(c, make(tiers=TIERS), n=n) == kq.KVQ_OK
    return c


def forked_from_a_window(n, **kw):
    c = make(**kw)
    assert fork(c, make(tiers=TIERS, window=128), n=n if n > 192 else -1) == kq.KVQ_OK
    return c


def in_place(n, **kw):
    c = make(tiers=TIERS, **kw)
    assert fork(c, c, n=n, m=A) == kq.KVQ_OK
    return c


@pytest.mark.parametrize("way", [truncated, forked, in_place, forked_from_a_window])
@pytest.mark.parametrize("n", [1, 64, 100, 127, 128, 129, 150, 191, 192, 193, 250, 291, 292])
@pytest.mark.parametrize("more", [1, 5, 200])
def test_the_next_token_of_a_block_without_a_window(way, n, more):
    """A page that is partly filled is filled at its own width, also where the rest of the block is narrower."""
    if way is truncated and n == 292:
        return  # (nothing is cut)
    c = way(n)
    before = widths(c)
    n = len(before)
    assert append(c, more) == kq.KVQ_OK
    assert widths(c) == before + [before[-1] if n % 64 else min(before)] * more
    while len(widths(c)) % 64:  # (one by one, as a decoder appends)
        last = widths(c)[-1]
        assert append(c, 1) == kq.KVQ_OK and widths(c)[-1] == last
    assert append(c, 1) == kq.KVQ_OK and widths(c)[-1] == min(widths(c))


def test_a_sink_of_another_length():
    """The forked page is one of the sink's: the block's width (16, of no pages behind the sink) is not that page's."""
    s = make(tiers=[(40, 2)])
    c = kq.KvqCache(kq.KvqConfig(1, 2, 8, 2, 4096, page_tokens=64, n_sink=64), [1 << 40], [2], arena_bytes=1 << 28)
    assert fork(c, s) == kq.KVQ_OK and append(c, 24) == kq.KVQ_OK and set(widths(c)) == {2}
    assert append(c, 1) == kq.KVQ_OK and widths(c)[-1] == 16


def test_explicit_widths_are_refused_as_before():
    c = truncated(150)
    assert append(c, 1, 2) == kq.KVQ_E_STATE and append(c, 1, 8) == kq.KVQ_OK
    # a block that was appended to at explicit widths is not one that was cut
    c = make(tiers=[(64, 2), (10, 8)])
    assert append(c, 1) == kq.KVQ_E_STATE
    c.kvq_cache_reset(0)
    assert append(c, 10, 8) == kq.KVQ_OK and append(c, 60) == kq.KVQ_OK


def test_emptied_blocks_forget():
    c = truncated(150)
    c.kvq_cache_reset(0)
    for n, bits in ((128, 2), (22, 8)):
        assert append(c, n, bits) == kq.KVQ_OK
    assert append(c, 1) == kq.KVQ_E_STATE  # page 2 is not the one that was cut


@pytest.mark.parametrize("kind", [dict(policy=kq.KVQ_POLICY_OLDEST_FIRST), dict(window=64)])
@pytest.mark.parametrize("n", [100, 128])
def test_a_whole_block_into_a_cache_that_appends_at_16(kind, n):
    """100 tokens end inside a page of 8 bits, in which the source goes on and the other cache could not."""
    s, d = make(tiers=[(n, 16)]), make(tiers=[(10, 16)], **kind)
    s.kvq_progressive_requant(0)
    before = d.kvq_cache_describe(0), d.kvq_cache_arena_free_bytes()
    if n % 64:
        for m in (-1, n, 70):
            assert fork(d, s, n=m) == kq.KVQ_E_STATE
        assert (d.kvq_cache_describe(0), d.kvq_cache_arena_free_bytes()) == before
        assert fork(d, s, n=64) == kq.KVQ_OK and append(d, 1) == kq.KVQ_OK and widths(d) == [8] * 64 + [16]
    else:
        assert fork(d, s) == kq.KVQ_OK and append(d, 1) == kq.KVQ_OK and widths(d) == [8] * n + [16]
    assert append(s, 1) == kq.KVQ_OK
    # a block that no such append follows where it is may be copied whole: what is left of it is to be read
    s = make(tiers=[(100, 8)], **kind)
    assert append(s, 1) == kq.KVQ_E_STATE
    assert fork(make(**kind), s) == kq.KVQ_OK and fork(s, s, m=A) == kq.KVQ_OK
