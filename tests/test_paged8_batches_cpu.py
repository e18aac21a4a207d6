"""Which batches attention on the paged cache of 8-bit floating point takes; nothing is launched here."""
import os
import random

import pytest

import paper_2505_18610_amd as kq
from paged8_lines import sums
from test_paged8_cpu import attend, diff, structs

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")


def need(n_seqs, tokens, max_rows, n_rows, q, maps=0, kv=8, page=64):
    pages = tokens // page
    return kq.load_library().kvq_paged8_workspace_bytes(*structs(dict(n_kv_heads=kv, page_tokens=page), dict(
        n_seqs=n_seqs, table_pages=pages, table_stride=pages, max_rows=max_rows, n_rows=n_rows)), q, maps)


@pytest.mark.parametrize("maps", [0, 1])
@pytest.mark.parametrize("n_seqs,tokens,max_rows,n_rows", [
    (64, 131072, 2048, 2111), (64, 131072, 1024, 1087), (32, 131072, 2048, 2079), (32, 131072, 4096, 4127), (256, 32768, 2048, 2303), (256, 131072, 512, 767),
    (128, 65536, 1024, 1151), (64, 32768, 2048, 2111), (64, 131072, 1024, 65536), (1, 131072, 131072, 131072), (16, 131072, 8192, 131072),
    (512, 131072, 8192, 16384), (256, 131072, 131072, 131072)])
def test_serving_batches_are_taken(n_seqs, tokens, max_rows, n_rows, maps):
    """Chunks beside single tokens, whole prompts, and batches any of whose sequences may have all rows of a call."""
    for q in (32, 40, 64):
        assert need(n_seqs, tokens, max_rows, n_rows, q, maps) > 0


def test_what_one_call_does_not_take():
    """The limits of the header, from both sides."""
    assert need(4096, 131072, 1, 4096, 64) > 0 and need(4096, 131072, 64, 4096, 64) > 0
    assert need(4096, 32 << 15, 1, 4096, 64) > 0 and need(4096, (32 << 15) + 64, 1, 4096, 64) == 0  # 2^12 sequences x 2^3 heads x 2^15 tiles
    assert need(4096, 32 << 14, 64, 4096, 64) > 0 and need(4096, (32 << 14) + 64, 64, 4096, 64) == 0  # two blocks of 32 rows
    assert need(4096, 32 << 13, 64, 4096, 64, 1) > 0 and need(4096, (32 << 13) + 64, 64, 4096, 64, 1) == 0
    rows = 1 << 20
    assert need(1, 131072, rows, rows, 8) > 0 and need(1, 131072, rows, rows, 64) == 0
    for call in (attend, diff):
        assert call(batch=dict(n_seqs=1, table_pages=2048, table_stride=2048, max_rows=1 << 24, n_rows=1 << 24)) == kq.KVQ_E_INVALID


def test_sums_of_batches_that_are_taken():
    """The line of all chunks stays within 2^30 for every batch that is taken, and its shares within the workgroups."""
    g = random.Random(3)
    taken = 0
    for _ in range(400):
        n = g.choice([1, 2, 7, 64, 65, 300, 4096])
        kv, gqa, tokens = g.choice([1, 2, 8]), g.choice([1, 2, 8, 16]), 64 * round(2 ** g.uniform(0, 15))
        n_rows = max(n, round(2 ** g.uniform(0, 18)))
        cuts = sorted(g.randrange(n_rows + 1) for _ in range(n - 1))
        rows = [b - a for a, b in zip([0] + cuts, cuts + [n_rows])]
        lengths = [g.choice([tokens, g.randrange(tokens + 1)]) for _ in rows]
        if not need(n, tokens, max(rows), n_rows, kv * gqa, kv=kv):
            continue
        taken += 1
        total, groups, units = sums(kv, gqa, rows, lengths, max(rows), n_rows, tokens)
        assert total <= 1 << 30 and -(-total // max(16, -(-total // groups))) <= groups
        few = [(-(-r * gqa // 32), m) for r, m in zip(rows, lengths) if r * gqa <= 64]
        assert sum(b * max(1, -(-m // 32)) for b, m in few) * kv <= 1 << 30
    assert taken > 100
