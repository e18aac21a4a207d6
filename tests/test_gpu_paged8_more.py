"""The paged cache of 8-bit floating point where its kernels can go wrong by how a call is cut, and at the ends of its ranges."""
import pytest
import torch

import paper_2505_18610_amd as kq
from paged8_lines import line
from paged8_plain import D, attention, check
from test_gpu_paged8 import Pair, attend, begins, in_blocks, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("diff", [False, True])
def test_units_of_every_number_of_pieces(diff):
    """Blocks cut into 5 to 11 pieces, among them 6 and 11: their last pieces have no neighbour at a level between two at which they have one."""
    lengths = [32 * (95 + 4 * s) + 7 for s in range(33)]
    rows = [16] * 33
    assert in_blocks(1, 16, rows, lengths, diff)
    pieces = line(1, 16, rows, lengths, 16, -(-max(lengths) // 64) * 64)[1]
    assert {5, 6, 7, 8, 9, 10, 11} <= set(pieces)
    c = Pair(1, 64, 33, -(-max(lengths) // 64), seed=41).filled(lengths)
    attend(c, 16, rows, lengths, diff=diff)


@pytest.mark.parametrize("diff", [False, True])
def test_wide_batch(diff):
    """256 sequences with tables for 131,072 tokens, any of which may have 8,192 rows: a few chunks beside single tokens.  The line of chunks is
    measured by the rows that there are; row numbers that have it otherwise leave the chunks alone, and the workspace as it was."""
    n, kv, gqa, n_rows = 256, 2, 16, 8192
    lengths = [40 + 3 * s for s in range(n)]
    lengths[3], lengths[100], lengths[255] = 3000, 700, 1300
    rows = [1] * n
    rows[3], rows[100], rows[255], rows[7], rows[200] = 500, 333, 9, 0, 3
    c = Pair(kv, 64, n, 47, seed=42).filled(lengths)
    table = torch.full((n, 2048), -1, dtype=torch.int32)
    table[:, :47] = c.table
    begin, lens = ints(begins(rows)), ints(lengths)
    batch = kq.KvqPaged8Batch(table.cuda(), lens, begin, max_rows=n_rows)
    g = torch.Generator().manual_seed(7)
    q, lam = torch.randn(n_rows, kv * gqa, D, generator=g).half(), torch.rand(kv * gqa, generator=g)
    q_dev, lam_dev = q.cuda(), lam.cuda()
    out = torch.empty_like(q_dev)
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, kv * gqa, n_rows, diff), dtype=torch.uint8, device="cuda")

    def call():
        out.fill_(777.0)
        if diff:
            c.cache.kvq_paged8_diff_attention(batch, q_dev, lam_dev, out, workspace=ws)
        else:
            c.cache.kvq_paged8_attention(batch, q_dev, out, workspace=ws)

    m = sum(rows)
    want, tol, _, _ = attention(c.plain, c.table, lengths, begins(rows), q[:m], lam=lam if diff else None)
    for turn in range(2):
        call()
        check(out[:m], want, tol)
        assert bool((out[m:] == 777.0).all())
        if turn == 0:  # every other sequence has all rows
            begin.copy_(ints([0, n_rows] * 128 + [0]))
            call()
            assert bool((out == 777.0).all())
            begin.copy_(ints(begins(rows)))
