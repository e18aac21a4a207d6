"""The paged cache of 8-bit floating point where its kernels can go wrong by how a call is cut, and at the ends of its ranges."""
import pytest
import torch

import paper_2505_18610_amd as kq
from paged8_lines import line
from paged8_plain import D, Plain, attention, check
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


def test_append_beyond_the_table():
    """A sequence that outgrows its table leaves what it holds: a step at the first token beyond, rows that begin in front of the table's end and end behind
    it, rows that are all behind it, by as little and as much as there is."""
    for page in (32, 128):
        cap = 3 * page
        have = [cap, cap, cap - 16, cap - 1, cap, 40]
        c = Pair(2, page, 6, 3, seed=43).filled(have)
        before = c.codes.clone(), c.words.clone()
        for rows, lengths in (([1] * 6, [cap + 1, cap + 900, 1 << 30, (1 << 31) - 1, cap + 1, cap + 1]), ([5, 1, 33, 0, 2, 64], [cap + 5, cap + 6, cap + 40, cap + 9, cap + 2, cap + 64])):
            c.append(rows, lengths, *c.new(rows, 50.0, 64))
            c.same()
            assert torch.equal(before[0], c.codes) and torch.equal(before[1], c.words)
        rows, lengths = [30, 1, 30, 2, 3, 1], [cap + 14, cap + 1, cap + 14, cap + 1, cap + 1, 41]
        k, v, cs = c.new(rows, 3.0, 32)
        c.append(rows, lengths, k, v, cs)
        c.same()
        got = kq.KvqPaged8Batch(c.table.cuda(), ints([cap] * 6), ints([16 * s for s in range(7)]), 16)
        keys, values = (torch.zeros(96, 2, D, device="cuda") for _ in range(2))
        c.cache.kvq_paged8_read(got, keys, values)
        # of 30 rows that end 14 tokens beyond, the first 16 are the table's last
        want = v[31:47].float()
        assert bool(((values[32:48].cpu() - want).abs() <= want.abs() * 2.0 ** -4 + want.abs().amax() * 2.0 ** -17).all())


def test_read_beyond_the_table():
    """Rows of tokens that the table does not have stay as they were; the others are their own tokens."""
    cap = 3 * 64
    c = Pair(2, 64, 4, 3, seed=44).filled([cap] * 4)
    rows, lengths = [30, 1, 5, 300], [cap + 14, cap + 1, 1 << 30, cap + 290]
    for dtype in (torch.float16, torch.float32):
        k, v = (torch.full((sum(rows), 2, D), 777.0, dtype=dtype, device="cuda") for _ in range(2))
        c.cache.kvq_paged8_read(c.batch(rows, lengths), k, v)
        whole = [torch.empty(4 * cap, 2, D, dtype=dtype, device="cuda") for _ in range(2)]
        c.cache.kvq_paged8_read(c.batch([cap] * 4, [cap] * 4), *whole)
        for got, all_of in zip((k, v), whole):
            assert torch.equal(got[:16], all_of[cap - 16:cap]) and bool((got[16:36] == 777.0).all())
            first = cap + 290 - 300  # the fourth's rows are tokens cap - 10 and on
            assert torch.equal(got[36:46], all_of[3 * cap + first:4 * cap]) and bool((got[46:] == 777.0).all())


@pytest.mark.parametrize("diff", [False, True])
def test_queries_beyond_the_table(diff):
    """They see all that the table has; the rows in front of them what they saw without those behind."""
    cap = 10 * 32
    c = Pair(4, 32, 5, 10, seed=45).filled([cap, cap, cap, cap, 200])
    attend(c, 16, [1, 3, 8, 2, 1], [cap + 1, cap + 2, 1 << 30, (1 << 31) - 1, 200], diff=diff)
    rows, lengths = [300, 290, 310, 90, 100], [cap + 150, cap + 290, 1 << 30, cap + 1, 200]
    assert in_blocks(4, 4, rows, [cap, cap, cap, cap, 200], diff)
    attend(c, 16, rows, lengths, diff=diff)


@pytest.mark.parametrize("diff", [False, True])
def test_outputs_of_the_largest_values(diff):
    """Values above 63,488 round to a code of 65,536: outputs of 16 bits take the largest there is, of finite values none is infinite; NaN stays."""
    for kv, gqa, rows, lengths in ((1, 4, [1, 2, 6, 1], [40, 2, 6, 300]), (4, 4, [600, 600], [600, 600])):
        assert in_blocks(kv, gqa, rows, lengths, diff) == (kv == 4)
        c = Pair(kv, 32, len(rows), max(lengths) // 32 + 1, seed=46)
        k, v, _ = c.new(lengths)
        v = torch.where(torch.arange(D)[None, None] % 3 == 0, -65504.0, 65504.0).expand_as(v).half().clone()
        v[lengths[0] - 1, 0, 5] = float("nan")
        c.append(lengths, lengths, k, v)
        for out in (torch.float16, torch.float32):
            attend(c, kv * gqa, rows, lengths, out=out, diff=diff, norm=False, out_scale=1.0)
        n = sum(rows)
        q, lam = torch.randn(n, kv * gqa, D, generator=c.g).half().cuda(), torch.full((kv * gqa,), -1.0, device="cuda")
        batch, got = c.batch(rows, lengths), torch.empty(n, kv * gqa, D, device="cuda").half()
        ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, kv * gqa, n, diff), dtype=torch.uint8, device="cuda")
        if diff:  # (twice 65,536)
            c.cache.kvq_paged8_diff_attention(batch, q, lam, got, workspace=ws)
        else:
            c.cache.kvq_paged8_attention(batch, q, got, workspace=ws)
        nan = torch.isnan(got)
        assert bool(nan[rows[0] - 1, :gqa, 5].all()) and int(nan.sum()) == gqa
        assert torch.equal(got.abs()[~nan], torch.full_like(got, 65504.0)[~nan])


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("power", [-24, -21, -14, -4])
def test_small_values(power, diff):
    """Values down to the smallest of fp16 count for what they are: against the same values times a power of two, which takes them to the order of one,
    where the oracle's bounds have no absolute part that matters."""
    for kv, gqa, rows, lengths in ((2, 4, [1, 2, 6, 1], [40, 2, 700, 300]), (4, 4, [600, 600], [600, 600])):
        assert in_blocks(kv, gqa, rows, lengths, diff) == (kv == 4)
        c = Pair(kv, 32, len(rows), max(lengths) // 32 + 1, seed=47)
        k, v, _ = c.new(lengths)
        v = ((1 + v.float().abs()).clamp(max=4) * v.float().sign() * 2.0 ** power).half()
        c.append(lengths, lengths, k, v)
        large = Plain(c.plain.codes, c.plain.words)
        large.words[..., 1] -= power
        n, heads = sum(rows), kv * gqa
        q, lam = torch.randn(n, heads, D, generator=c.g).half(), torch.rand(heads, generator=c.g)
        weight = torch.randn(D, generator=c.g)
        batch = c.batch(rows, lengths)
        ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, heads, n, diff), dtype=torch.uint8, device="cuda")
        got = torch.empty(n, heads, D, device="cuda")
        if diff:
            c.cache.kvq_paged8_diff_attention(batch, q.cuda(), lam.cuda(), got, workspace=ws)
        else:
            c.cache.kvq_paged8_attention(batch, q.cuda(), got, workspace=ws)
        want, tol, _, _ = attention(large, c.table, lengths, begins(rows), q, lam=lam if diff else None, out_eps=2.0 ** -24)
        check(got.double() * 2.0 ** -power, want, tol)
        if diff:  # (a norm without eps does not see the size)
            c.cache.kvq_paged8_diff_attention(batch, q.cuda(), lam.cuda(), got, norm_weight=weight.cuda(), norm_eps=0.0, workspace=ws)
            want, tol, _, _ = attention(large, c.table, lengths, begins(rows), q, lam=lam, weight=weight, eps=0.0, out_eps=2.0 ** -24)
            check(got, want, tol)


def graded(kv, pages, gains, seed, nan=()):
    """Pages of 64 tokens, one sequence's, whose values are positive and of the size `gains` says page by page; keys of four sizes in turn."""
    c = Pair(kv, 64, 1, pages, seed=seed)
    k, v, _ = c.new([64 * pages])
    of = torch.arange(64 * pages) // 64
    k = (k.float() * torch.tensor([0.25, 1.0, 0.5, 2.0])[of % 4, None, None]).half()
    v = (v.float().abs() * torch.tensor(gains)[of, None, None]).half()
    for page, token, head, channel in nan:
        v[64 * page + token, head, channel] = float("nan")
    c.append([64 * pages], [64 * pages], k, v)
    return c


@pytest.mark.parametrize("diff", [False, True])
def test_chunk_pieces_of_many_tiles(diff):
    """A workgroup has more than 128 tiles of one block, so that it comes to a second and a third lot of 64 tables' entries and scale words: pages of many
    scales, among them one behind the first lot that is larger than all before, NaN and a missing page behind it.  Rows here and there."""
    kv, gqa, n, pages = 4, 16, 12000, 188
    rows = 512
    gains = [2.0 ** (p % 7 - 6) * (1.0 if p < 70 else 16.0 if p < 130 else 200.0) for p in range(pages)]
    c = graded(kv, pages, gains, 48, nan=((140, 41, 1, 100), (184, 30, 2, 7)))
    table = c.table.clone()
    table[0, 120] = -1
    share, _, longest = line(kv, gqa, [rows], [n], rows, pages * 64)
    assert longest > 128 and in_blocks(kv, gqa, [rows], [n], diff)
    g = torch.Generator().manual_seed(8)
    q, lam = (0.5 * torch.randn(rows, kv * gqa, D, generator=g)).half(), torch.rand(kv * gqa, generator=g)
    batch = c.batch([rows], [n], table)
    got, lse = torch.empty(rows, kv * gqa, D, device="cuda"), torch.empty(kv * gqa, rows, device="cuda")
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, kv * gqa, rows, diff), dtype=torch.uint8, device="cuda")
    if diff:
        c.cache.kvq_paged8_diff_attention(batch, q.cuda(), lam.cuda(), got, workspace=ws)
    else:
        c.cache.kvq_paged8_attention(batch, q.cuda(), got, lse=lse, workspace=ws)
    some = [0, 17, 255, 306, 511]  # (token 11,806 is NaN, row 318)
    want, tol, wl, tl = attention(c.plain, table.expand(5, -1), [n - rows + i + 1 for i in some], list(range(6)), q[some], lam=lam if diff else None, out_eps=2.0 ** -24)
    check(got[some], want, tol)
    assert bool(torch.isnan(got[:, 16:32, 100]).all())
    assert bool(torch.isnan(got[318:, 32:48, 7]).all()) and not bool(torch.isnan(got[:318, 32:48, 7]).any())
    if not diff:
        check(lse[:, some], wl, tl)


@pytest.mark.parametrize("gqa,rows,diff", [(8, 1, False), (16, 1, False), (16, 2, False), (8, 1, True), (16, 1, True)])
def test_pieces_of_few_rows_of_many_tiles(gqa, rows, diff):
    """A wavefront has more than 64 tiles, for the same reasons: 128 sequences of 65,536 tokens and a little less over 40 pages that they share."""
    kv, n, pages = 2, 128, 40
    gains = [2.0 ** (p % 5 - 4) * (1.0 if p < 20 else 16.0 if p < 30 else 200.0) for p in range(pages)]
    c = graded(kv, pages, gains, 49, nan=((39, 3, 1, 9),))
    g = torch.Generator().manual_seed(9)
    which = torch.randint(0, 20, (n, 1024), generator=g)
    which[:, 300:500] = torch.randint(0, 30, (n, 200), generator=g)
    which[:, 800:] = torch.randint(0, 39, (n, 224), generator=g)
    which[77, 900] = 39
    table = c.table[0][which].contiguous()
    table[5, 950] = -1
    lengths = [65536 - 3 * s for s in range(n)]
    units, tiles = n * kv, sum(-(-x // 32) for x in lengths) * kv
    at_a_time = 512 if gqa * rows * (2 if diff else 1) <= 16 else 256
    assert -(-tiles // at_a_time) > 512 and gqa * rows <= 64 and units <= 256
    q, lam = (0.5 * torch.randn(n * rows, kv * gqa, D, generator=g)).half(), torch.rand(kv * gqa, generator=g)
    batch = c.batch([rows] * n, lengths, table)
    got = torch.empty(n * rows, kv * gqa, D, device="cuda")
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, kv * gqa, n * rows, diff), dtype=torch.uint8, device="cuda")
    if diff:
        c.cache.kvq_paged8_diff_attention(batch, q.cuda(), lam.cuda(), got, workspace=ws)
    else:
        c.cache.kvq_paged8_attention(batch, q.cuda(), got, workspace=ws)
    for s in (5, 77):
        at = slice(s * rows, (s + 1) * rows)
        want, tol, _, _ = attention(c.plain, table[s:s + 1], [lengths[s]], [0, rows], q[at], lam=lam if diff else None, out_eps=2.0 ** -24)
        check(got[at], want, tol)
    nan = torch.isnan(got)
    assert bool(nan[77 * rows:78 * rows, gqa:, 9].all()) and int(nan.sum()) == rows * gqa
