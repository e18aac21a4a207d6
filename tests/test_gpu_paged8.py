"""The paged cache of 8-bit floating point: appends and read-back bit for bit, attention against 64 bits."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq
from paged8_plain import D, Plain, attention, check

pytestmark = pytest.mark.gpu


def begins(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pair:
    """The same pages in the library and in plain form; pages of the sequences dealt out at random, anything in them at first."""

    def __init__(self, kv, page, n_seqs, pages_each, seed=0, spare=3):
        self.g = torch.Generator().manual_seed(seed)
        n = n_seqs * pages_each + spare
        codes = torch.randint(0, 256, (n, kv, page // 32, 2, 4096), generator=self.g, dtype=torch.uint8)
        words = torch.randint(-1 << 31, (1 << 31) - 1, (n, kv, 2), generator=self.g, dtype=torch.int32)
        self.table = torch.randperm(n, generator=self.g)[:n_seqs * pages_each].reshape(n_seqs, pages_each).int()
        self.plain = Plain(codes, words)
        self.codes, self.words = codes.cuda(), words.cuda()
        self.cache = kq.KvqPaged8(self.codes, self.words)
        self.kv, self.page = kv, page

    def batch(self, rows, lengths, table=None, max_rows=None, no_rows=False):
        table = (self.table if table is None else table).cuda()
        return kq.KvqPaged8Batch(table, ints(lengths), None if no_rows else ints(begins(rows)), max_rows or max([1] + list(rows)))

    def new(self, rows, gain=1.0, pair=None):
        n = sum(rows)
        k, v = (gain * torch.randn(n, self.kv, D, generator=self.g) for _ in range(2))
        k[:, :, 5] *= 20
        cs = None if pair is None else torch.randn(n, 2 * pair, generator=self.g)
        return k.half(), v.half(), cs

    def append(self, rows, lengths, k, v, cs=None, table=None):
        self.cache.kvq_paged8_append(self.batch(rows, lengths, table), k.cuda(), v.cuda(), None if cs is None else cs.cuda())
        self.plain.append(self.table if table is None else table, lengths, begins(rows), k, v, cs)

    def same(self):
        got, want = self.codes.cpu(), self.plain.codes
        nan = ((want & 0x7f) == 0x7f) & ((got & 0x7f) == 0x7f)  # (the sign of a NaN says nothing)
        assert torch.equal(torch.where(nan, want, got), want)
        assert torch.equal(self.words.cpu(), self.plain.words)

    def filled(self, lengths, gain=1.0):
        k, v, _ = self.new(lengths, gain)
        self.append(lengths, lengths, k, v)
        return self


@pytest.mark.parametrize("pair", [None, 64, 32])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_append(page, pair):
    """Prompts, then single tokens, then a few, ever larger ones, so that scales rise in the middle of pages and tiles."""
    c = Pair(2, page, 5, 512 // page + 2, seed=page)
    lengths = [0] * 5
    for step, rows in enumerate([[1, 31, 32, 33, 300], [1] * 5, [1] * 5, [0, 70, 3, 1, 64], [1] * 5, [2, 0, 40, 1, 7]]):
        lengths = [n + r for n, r in zip(lengths, rows)]
        c.append(rows, lengths, *c.new(rows, 2.0 ** step, pair))
        c.same()


def test_append_small_and_large_values():
    """Zeros, the smallest and the largest fp16 values, and rotations that take them beyond it."""
    c = Pair(1, 32, 4, 2, seed=3)
    for gain in (0.0, 2.0 ** -24, 2.0 ** -14, 60000.0):
        k, v, cs = c.new([3] * 4, 1.0, 64)
        k, v = (x.float().clamp(-1, 1) * gain for x in (k, v))
        n = {0.0: 3, 2.0 ** -24: 6, 2.0 ** -14: 9, 60000.0: 12}[gain]
        c.append([3] * 4, [n] * 4, k.half(), v.half(), cs)
        c.same()


def test_append_nonfinite():
    c = Pair(2, 64, 2, 2, seed=4)
    k, v, cs = c.new([50, 40], 1.0, 64)
    k[3, 0, 7], k[60, 1, 100], v[5, 1, 3], v[77, 0, 127], v[78, 0, 1] = math.inf, math.nan, -math.inf, math.nan, math.inf
    c.append([50, 40], [50, 40], k, v, cs)
    c.same()
    assert int((c.words.cpu()[c.table[:, 0].long()] >> 8).sum()) == 4
    c.append([1, 1], [51, 41], *c.new([1, 1], 100.0, 64))  # the marks stay while the page is filled
    c.same()


def test_append_what_does_not_exist():
    """More rows than tokens, no tokens, pages that are not there, tokens beyond the table: nothing is written for them."""
    c = Pair(2, 32, 6, 3, seed=5).filled([40, 10, 0, 96, 96, 33])
    table = c.table.clone()
    table[0, 1], table[4, 2] = -1, 1 << 20
    rows, lengths = [50, 20, 5, 30, 96, 0], [60, 12, 0, 110, 96, 33]
    k, v, cs = c.new(rows, 3.0, 32)
    c.append(rows, lengths, k, v, cs, table)
    c.same()
    c.cache.kvq_paged8_append(c.batch([1] * 6, [-5] * 6), *(x[:6].contiguous().cuda() for x in (k, v)))
    c.same()


def test_append_rows_beyond():
    """max_rows and the tensors' rows bound what a sequence has, whatever its row numbers say."""
    c = Pair(1, 32, 2, 4, seed=6)
    k, v, _ = c.new([20])
    batch = kq.KvqPaged8Batch(c.table.cuda(), ints([8, 100]), ints([0, 8, 1 << 30]), 8)
    c.cache.kvq_paged8_append(batch, k.cuda(), v.cuda())
    c.plain.append(c.table, [8, 100], [0, 8, 16], k, v)
    c.same()


def test_append_strides():
    c = Pair(3, 64, 2, 2, seed=7)
    rows = [70, 20]
    k, v, cs = c.new(rows, 1.0, 64)
    both = torch.empty(90, 6, D).half()
    both[:, :3], both[:, 3:] = k, v
    major = v.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    c.cache.kvq_paged8_append(c.batch(rows, rows), both.cuda()[:, :3], major, cs.cuda())
    c.plain.append(c.table, rows, begins(rows), k, v, cs)
    c.same()


@pytest.mark.parametrize("n_seqs", [1, 70, 300])
def test_append_and_read_many_sequences(n_seqs):
    """More sequences than a wavefront has lanes, one of them long, so that workgroups look for their pages."""
    c = Pair(1, 32, n_seqs, 12, seed=8)
    rows = [1 + 7 * s % 5 for s in range(n_seqs)]
    rows[n_seqs // 2] = 370
    lengths = [r + 11 * s % 14 for s, r in enumerate(rows)]
    lengths = [min(n, 12 * 32) for n in lengths]
    c.filled([n - r for n, r in zip(lengths, rows)])
    c.append(rows, lengths, *c.new(rows))
    c.same()
    read(c, rows, lengths, torch.float16)


def read(c, rows, lengths, dtype, table=None):
    n, mark = sum(rows) + 3, 777.0  # three rows of nobody
    k, v = (torch.full((n, c.kv, D), mark, dtype=dtype, device="cuda") for _ in range(2))
    c.cache.kvq_paged8_read(c.batch(rows, lengths, table), k, v)
    want = [torch.full((n, c.kv, D), mark, dtype=torch.float64) for _ in range(2)]
    for s, (r, b) in enumerate(zip(rows, begins(rows))):
        m = max(0, min(lengths[s], c.table.shape[1] * c.page))
        for h in range(c.kv):
            *kv, there = c.plain.values((c.table if table is None else table)[s], m, h)
            for w, x in zip(want, kv):
                for i in range(r):
                    t = m - r + i
                    if t >= 0 and there[t]:
                        w[b + i, h] = x[t]
    for got, w in zip((k, v), want):
        if dtype == torch.float16:
            w = w.clamp(-65504, 65504)
        assert torch.equal(torch.nan_to_num(got.cpu(), 1.5), torch.nan_to_num(w.to(dtype), 1.5))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("page", [32, 256])
def test_read(page, dtype):
    lengths = [1, 40, 257, 300]
    c = Pair(3, page, 4, 320 // page + 1, seed=9).filled(lengths, 100.0)
    read(c, lengths, lengths, dtype)
    read(c, [1, 5, 0, 290], lengths, dtype)
    read(c, [3, 2, 1, 7], [1, 0, 257, -3], dtype)  # rows of tokens that do not exist stay as they were
    table = c.table.clone()
    table[3, 0], table[2, 0] = -1, 1 << 20
    read(c, [1, 40, 257, 300], lengths, dtype, table)


def test_read_largest():
    """A rounded code may stand for more than the largest fp16 value."""
    c = Pair(1, 32, 1, 1, seed=10)
    k, v = torch.full((4, 1, D), 65504.0).half(), torch.full((4, 1, D), -65504.0).half()
    k[1, 0, 0] = math.nan
    c.append([4], [4], k, v)
    read(c, [4], [4], torch.float16)
    read(c, [4], [4], torch.float32)


def attend(c, q_heads, rows, lengths, out=torch.float16, scale=0.0, diff=False, norm=True, lse=True, table=None, no_rows=False, spread=1.0,
           seed=1, out_scale=0.25, eps=1e-5, max_rows=None):
    g = torch.Generator().manual_seed(seed)
    n = sum(rows) + (0 if no_rows else 2)
    q = (spread * torch.randn(n, q_heads, D, generator=g)).half()
    lam, weight = 1.5 * torch.rand(q_heads, generator=g) - 0.3, torch.randn(D, generator=g)
    batch = c.batch(rows, lengths, table, max_rows, no_rows)
    got = torch.full((n, q_heads, D), 777.0, dtype=out, device="cuda")
    logs = torch.full((q_heads, n), 777.0, device="cuda") if lse and not diff else None
    need = kq.kvq_paged8_workspace_bytes(c.cache, batch, q_heads, n, diff)
    assert need > 0
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    each = []
    for _ in range(2):  # the second time over the workspace that the first has left
        if diff:
            c.cache.kvq_paged8_diff_attention(batch, q.cuda(), lam.cuda(), got, norm_weight=weight.cuda() if norm else None, norm_eps=eps,
                                              out_scale=out_scale, softmax_scale=scale, workspace=ws)
        else:
            c.cache.kvq_paged8_attention(batch, q.cuda(), got, softmax_scale=scale, lse=logs, workspace=ws)
        each.append(got.clone())
    assert torch.equal(*(torch.nan_to_num(x, 5.0) for x in each))
    want, tol, wl, tl = attention(c.plain, c.table if table is None else table, lengths, begins(rows), q, scale, lam if diff else None,
                                  weight if norm else None, eps, out_scale, 2.0 ** -11 if out == torch.float16 else 2.0 ** -24)
    m = sum(rows)
    check(got[:m], want[:m], tol[:m])
    assert bool((got[m:] == 777.0).all())
    if logs is not None:
        wl, tl, gl = wl[:, :m], tl[:, :m], logs[:, :m].double().cpu()
        empty = wl == -math.inf
        assert torch.equal(gl == -math.inf, empty)
        check(torch.where(empty, torch.zeros_like(gl), gl), torch.where(empty, torch.zeros_like(wl), wl), tl)
        assert bool((logs[:, m:] == 777.0).all())


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("kv,gqa", [(1, 1), (2, 4), (1, 5), (3, 7), (2, 16), (1, 11)])
@pytest.mark.parametrize("page", [32, 128])
def test_single_tokens(page, kv, gqa, diff):
    lengths = [1, 2, 31, 32, 33, 64, 257, 700]
    c = Pair(kv, page, 8, 704 // page + 1, seed=11).filled(lengths)
    attend(c, kv * gqa, [1] * 8, lengths, diff=diff)
    attend(c, kv * gqa, [1] * 8, lengths, diff=diff, no_rows=True, out=torch.float32)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("rows", [[2, 3, 1, 4], [8, 1, 0, 5], [17, 40, 33, 1], [130, 64, 200, 129]])
@pytest.mark.parametrize("gqa", [1, 4, 7])
def test_rows(rows, gqa, diff):
    lengths = [rows[0], 300, 257, 513]
    c = Pair(2, 64, 4, 9, seed=12).filled(lengths)
    attend(c, 2 * gqa, rows, lengths, diff=diff, norm=gqa != 4)


def in_blocks(kv, gqa, rows, lengths, diff):
    """Whether sequences of more than 64 rows x heads are taken in blocks of 256 (calls of more than 512 units of 32 rows, or of 40,000 tiles of
    units): asked so that the tests below are of that kernel."""
    units = [-(-r * gqa * (2 if diff else 1) // 32) * kv for r in rows]
    return sum(units) > 512 or sum(u * max(1, -(-n // 32)) for u, n in zip(units, lengths)) > 40000


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("page,kv,gqa,rows,lengths", [
    (64, 4, 4, [400, 257, 70, 300], [400, 900, 257, 513]), (32, 3, 7, [300, 1, 257, 12], [301, 64, 270, 1000]), (256, 8, 1, [700, 900, 65, 64], [3000, 900, 65, 640]),
    (128, 2, 16, [180, 160, 33], [180, 1000, 290]), (64, 5, 5, [650], [650])])
def test_chunks(page, kv, gqa, rows, lengths, diff):
    """Blocks of 256 rows beside sequences of few, whole prompts and chunks behind cached tokens; blocks that end inside a token's heads."""
    if not in_blocks(kv, gqa, rows, lengths, diff):
        rows, lengths = rows * 3, lengths * 3
    assert in_blocks(kv, gqa, rows, lengths, diff)
    c = Pair(kv, page, len(rows), max(lengths) // page + 1, seed=30).filled(lengths)
    attend(c, kv * gqa, rows, lengths, diff=diff, norm=gqa != 4, out=torch.float32 if gqa == 7 else torch.float16, scale=-0.1 if gqa == 5 else 0.0)


@pytest.mark.parametrize("kv,gqa,rows,lengths", [
    (2, 4, [1, 1, 1], [33, 700, 1025]), (1, 2, [1, 4], [9001, 4097]), (1, 8, [8], [30000]), (2, 4, [40, 1], [900, 50]),   # pieces of few rows
    (4, 4, [500, 300, 300], [500, 1100, 300]), (1, 16, [80], [36000])])                                                    # blocks of 256
def test_every_tile_counts(kv, gqa, rows, lengths):
    """Equal weights, and values that are zero but for one channel in each tile: a tile that is lost or counted twice is a part of its channel that
    no bound lets pass."""
    c = Pair(kv, 64, len(rows), max(lengths) // 64 + 1, seed=34)
    k, v, _ = c.new(lengths)
    tile = torch.cat([torch.arange(n) // 32 for n in lengths])
    v = torch.where(torch.arange(D)[None, None] == (tile % D)[:, None, None], torch.full_like(v, 96.0), torch.zeros_like(v))
    c.append(lengths, lengths, k, v)
    attend(c, kv * gqa, rows, lengths, spread=0.0)
    attend(c, kv * gqa, rows, lengths, spread=0.0, diff=True, norm=False)


@pytest.mark.parametrize("diff", [False, True])
def test_chunk_in_many_pieces(diff):
    """One block's rows over many tiles, which several workgroups share; and a block of two pieces."""
    for kv, gqa, rows, lengths in ((1, 16, [70], [38500]), (2, 16, [90, 17], [14000, 9000])):
        assert in_blocks(kv, gqa, rows, lengths, diff)
        c = Pair(kv, 128, len(rows), max(lengths) // 128 + 1, seed=31).filled(lengths)
        attend(c, kv * gqa, rows, lengths, diff=diff)


@pytest.mark.parametrize("diff", [False, True])
def test_cut_blocks_of_few_rows(diff):
    """Blocks most of whose wavefronts have no rows, each cut into pieces of several workgroups, which go on to another block after a piece: equal
    bits, whoever joins the pieces."""
    rows, lengths = [17, 20, 24, 19, 30, 17, 22, 17, 18, 40], [3000 + 41 * s for s in range(10)]
    c = Pair(8, 64, 10, 54, seed=38).filled(lengths)
    rows = rows if diff else [2 * r for r in rows]
    assert in_blocks(8, 4, rows, lengths, diff)
    attend(c, 32, rows, lengths, diff=diff)
    batch, n = c.batch(rows, lengths), sum(rows)
    q, lam = torch.randn(n, 32, D, generator=torch.Generator().manual_seed(39)).half().cuda(), torch.ones(32, device="cuda")
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, 32, n, diff), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(20)]
    for out in outs:
        if diff:
            c.cache.kvq_paged8_diff_attention(batch, q, lam, out, workspace=ws)
        else:
            c.cache.kvq_paged8_attention(batch, q, out, workspace=ws)
    assert all(torch.equal(outs[0], out) for out in outs)


@pytest.mark.parametrize("diff", [False, True])
def test_chunks_of_what_does_not_exist(diff):
    """Rows that see nothing, pages that are not there, NaN among keys and values, lengths beyond the table: in blocks of 256 rows."""
    rows, lengths = [300, 280, 310, 90, 290], [150, 280, 0, 1 << 30, 290]
    have = [150, 280, 0, 320, 290]
    c = Pair(4, 32, 5, 10, seed=32)
    k, v, _ = c.new(have)
    k[10, 0, 3], v[149, 1, 77], v[150 + 100, 2, 5], v[150 + 279, 3, 0], k[150 + 200, 1, 1] = math.nan, math.inf, math.nan, math.nan, math.inf
    c.append(have, have, k, v)
    table = c.table.clone()
    table[3, 2], table[3, 9], table[4, 0] = -1, 1 << 20, -7
    assert in_blocks(4, 4, rows, [150, 280, 0, 320, 290], diff)
    attend(c, 16, rows, lengths, diff=diff, table=table)
    attend(c, 16, rows, lengths, diff=diff, table=table, eps=0.0, norm=True, max_rows=310)


def test_chunk_captured():
    """A captured call whose rows and lengths change between replays, from few rows to blocks of 256, over one workspace."""
    c = Pair(4, 64, 4, 12, seed=33).filled([600, 700, 64, 300])
    g = torch.Generator().manual_seed(5)
    n, heads = 1400, 16
    q = torch.randn(n, heads, D, generator=g).half()
    q_dev, out = q.cuda(), torch.empty(n, heads, D, device="cuda").half()
    begin, lengths = ints([0, 1, 2, 3, 4]), ints([1, 1, 1, 1])
    batch = kq.KvqPaged8Batch(c.table.cuda(), lengths, begin, max_rows=700)
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, heads, n), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.kvq_paged8_attention(batch, q_dev, out, workspace=ws, stream=torch.cuda.current_stream())
    for rows, held in (([1, 1, 1, 1], [600, 700, 64, 300]), ([600, 300, 64, 300], [600, 700, 64, 300]), ([0, 500, 20, 100], [5, 500, 64, 299]),
                       ([600, 300, 64, 300], [600, 700, 64, 300]), ([2, 0, 0, 7], [33, 700, 64, 300])):
        begin.copy_(ints(begins(rows)))
        lengths.copy_(ints(held))
        out.fill_(777.0)
        graph.replay()
        want, tol, _, _ = attention(c.plain, c.table, held, begins(rows), q)
        check(out[:sum(rows)], want[:sum(rows)], tol[:sum(rows)])
        assert bool((out[sum(rows):] == 777.0).all())


@pytest.mark.parametrize("diff", [False, True])
def test_rows_that_see_nothing(diff):
    """More rows than tokens, no tokens, lengths below zero: zeros, also behind a norm without eps."""
    c = Pair(2, 32, 5, 4, seed=13).filled([0, 3, 0, 40, 128])
    attend(c, 8, [1, 5, 3, 45, 2], [0, 3, -7, 40, 1 << 30], diff=diff)
    attend(c, 8, [1, 150, 3, 1, 2], [0, 3, -7, 40, 128], diff=diff, eps=0.0)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("rows", [1, 70])
def test_pages_that_are_not_there(rows, diff):
    lengths = [100, 128, 70, 96]
    c = Pair(2, 32, 4, 4, seed=14).filled(lengths)
    table = c.table.clone()
    table[0, 0], table[0, 2], table[1, 3], table[3, :] = -1, 1 << 29, -(1 << 31), -1
    attend(c, 8, [rows] * 4, lengths, diff=diff, table=table)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("rows", [1, 6, 80])
def test_nonfinite(rows, diff):
    """NaN among keys reaches the rows that see them; among values those rows' channels; and nobody else, nor what follows in the page."""
    c = Pair(2, 64, 3, 4, seed=15)
    lengths = [200, 130, 90]
    k, v, _ = c.new(lengths)
    k[195, 0, 3], v[197, 1, 77], v[198, 1, 5], v[200 + 127, 0, 0] = math.nan, math.inf, math.nan, math.nan
    c.append(lengths, lengths, k, v)
    attend(c, 8, [rows] * 3, lengths, diff=diff)
    attend(c, 8, [rows] * 3, [195, 126, 90], diff=diff)  # the tokens behind have been taken back


def test_leading_and_equal_keys():
    """Scores that spread over hundreds, and one row whose keys are all the same."""
    c = Pair(1, 32, 2, 40, seed=16)
    lengths = [1200, 1000]
    k, v, _ = c.new(lengths)
    k[1200:] = k[1200]
    c.append(lengths, lengths, k, v)
    for spread in (0.0, 1.0, 8.0, 300.0):
        attend(c, 8, [1, 1], lengths, spread=spread)
        attend(c, 8, [1, 1], lengths, spread=spread, diff=True)


@pytest.mark.parametrize("scale", [0.3, -0.2, 1e-30, 4.0])
def test_scales(scale):
    c = Pair(2, 32, 2, 10, seed=17).filled([300, 77])
    attend(c, 8, [1, 3], [300, 77], scale=scale)
    attend(c, 8, [1, 3], [300, 77], scale=scale, diff=True)


@pytest.mark.parametrize("gain", [2.0 ** -22, 2.0 ** -10, 30000.0])
def test_sizes_of_values(gain):
    """Values at both ends of fp16, and pages of one size beside pages of another."""
    c = Pair(2, 32, 2, 10, seed=18)
    lengths = [290, 64]
    k, v, _ = c.new(lengths)
    v = (v.float().clamp(-2, 2) * gain).half()
    v[32:64] = (v[32:64].float() / 64).half()
    c.append(lengths, lengths, k, v)
    attend(c, 4, [1, 1], lengths, out=torch.float32)


def test_long_and_short_together():
    """Units over many workgroups beside units that share one, more sequences than lanes."""
    lengths = [3000] + [1 + 13 * s % 90 for s in range(80)]
    c = Pair(2, 32, 81, 94, seed=19).filled(lengths)
    attend(c, 8, [1] * 81, lengths)
    attend(c, 8, [1] * 81, lengths, diff=True)
    attend(c, 8, [9] + [1] * 79 + [2], lengths)


@pytest.mark.parametrize("diff", [False, True])
@pytest.mark.parametrize("n,kv,gqa,rows,most", [(150, 4, 2, 1, 300), (90, 8, 4, 4, 200), (1100, 1, 4, 1, 40), (70, 8, 16, 1, 33)])
def test_many_short_sequences(n, kv, gqa, rows, most, diff):
    """More units than workgroups that the device takes at a time; more sequences than a wavefront has lanes."""
    lengths = [1 + (37 * s) % most for s in range(n)]
    counts = [min(rows, x) if s % 7 else 0 for s, x in enumerate(lengths)]
    c = Pair(kv, 32, n, most // 32 + 1, seed=35).filled(lengths)
    attend(c, kv * gqa, counts, lengths, diff=diff, lse=rows == 1)


def test_chunks_of_many_sequences():
    """Blocks of 256 rows of more sequences than a wavefront has lanes, beside single tokens."""
    rows = [1 if s % 3 else 70 + s for s in range(75)]
    lengths = [r + 5 * s % 50 for s, r in enumerate(rows)]
    assert in_blocks(2, 4, rows, lengths, False)
    c = Pair(2, 64, 75, 4, seed=36).filled(lengths)
    attend(c, 8, rows, lengths)
    attend(c, 8, rows, lengths, diff=True)


def test_queries_that_are_not_finite():
    """NaN in a query is its row's own affair, and so is an infinity."""
    for rows, lengths, kv in (([1, 1], [500, 40], 2), ([600, 600], [700, 600], 4)):
        c = Pair(kv, 64, 2, 12, seed=37).filled(lengths)
        n = sum(rows)
        q = torch.randn(n, 4 * kv, D, generator=torch.Generator().manual_seed(6)).half().cuda()
        batch = c.batch(rows, lengths)
        ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, 4 * kv, n), dtype=torch.uint8, device="cuda")
        want, got = torch.empty_like(q), torch.empty_like(q)
        c.cache.kvq_paged8_attention(batch, q, want, workspace=ws)
        q[1, 2, 7], q[0, 3, 100] = math.nan, math.inf
        c.cache.kvq_paged8_attention(batch, q, got, workspace=ws)
        assert bool(torch.isnan(got[1, 2]).all()) and bool(torch.isnan(got[0, 3]).any())
        want[1, 2], want[0, 3] = got[1, 2], got[0, 3]
        assert torch.equal(torch.nan_to_num(want, 5.0), torch.nan_to_num(got, 5.0))


def test_shared_pages():
    """Two sequences over the same pages, which differ in length; the order of pages is the table's."""
    c = Pair(2, 32, 3, 5, seed=20).filled([160, 100, 20])
    table = c.table.clone()
    table[1, :4], table[2, :4] = table[0, :4], table[0, :4].flip(0)
    attend(c, 8, [1, 4, 1], [160, 100, 128], table=table)


def test_strides_of_queries_and_outputs():
    c = Pair(2, 32, 2, 4, seed=21).filled([100, 50])
    g = torch.Generator().manual_seed(2)
    q = torch.randn(2, 8, D, generator=g).half()
    batch = c.batch([1, 1], [100, 50])
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, 8, 2), dtype=torch.uint8, device="cuda")
    plain = torch.empty(2, 8, D, device="cuda").half()
    c.cache.kvq_paged8_attention(batch, q.cuda(), plain, workspace=ws)
    sliced = torch.full((8, 2, 160), 7.0, device="cuda").half().transpose(0, 1)[:, :, 16:144]
    wide = torch.zeros(2, 24, D, device="cuda").half()
    wide[:, 8:16] = q.cuda()
    c.cache.kvq_paged8_attention(batch, wide[:, 8:16], sliced, workspace=ws)
    assert torch.equal(sliced, plain)


def test_other_stream_and_workspace_of_another_batch():
    """One workspace for calls of different shapes in turn, on a stream of its own."""
    c = Pair(2, 32, 4, 30, seed=22).filled([900, 333, 64, 1])
    big = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(3)
    stream = torch.cuda.Stream()
    want = {}
    for turn in range(3):
        for heads, rows in ((2, 1), (32, 1), (8, 3), (8, 40)):
            g.manual_seed(heads + rows)
            q = torch.randn(4 * rows, heads, D, generator=g).half().cuda()
            out = torch.empty_like(q)
            batch = c.batch([rows] * 4, [900, 333, 64, 1])
            torch.cuda.synchronize()
            c.cache.kvq_paged8_attention(batch, q, out, workspace=big, stream=stream)
            stream.synchronize()
            assert torch.equal(want.setdefault((heads, rows), out.clone()), out)


@pytest.mark.parametrize("diff", [False, True])
def test_captured_steps_while_sequences_grow(diff):
    """One captured step, append and attention, replayed while lengths, tables and a new sequence change on the device; two graphs share a
    workspace."""
    c = Pair(2, 32, 3, 12, seed=23).filled([30, 0, 64])
    plain = c.plain
    g = torch.Generator().manual_seed(4)
    k, v, q = (torch.zeros(3, h, D, device="cuda").half() for h in (2, 2, 8))
    cs, lengths = torch.zeros(3, 128, device="cuda"), ints([0, 0, 0])
    table = torch.full((3, 12), -1, dtype=torch.int32, device="cuda")
    batch = kq.KvqPaged8Batch(table, lengths)
    lam = torch.rand(8, generator=g)
    lam_dev = lam.cuda()
    outs = [torch.zeros(3, 8, D, device="cuda").half() for _ in range(2)]
    ws = torch.zeros(kq.kvq_paged8_workspace_bytes(c.cache, batch, 8, 3, diff), dtype=torch.uint8, device="cuda")

    def step(out, stream):
        c.cache.kvq_paged8_append(batch, k, v, cs, stream=stream)
        if diff:
            c.cache.kvq_paged8_diff_attention(batch, q, lam_dev, out, workspace=ws, stream=stream)
        else:
            c.cache.kvq_paged8_attention(batch, q, out, workspace=ws, stream=stream)

    graphs = []
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(out, torch.cuda.current_stream())
        graphs.append(graph)
    n = [30, 0, 64]
    for turn in range(40):
        n = [n[0] + 1, n[1] + 1 if turn > 3 else 0, n[2] + 5 if turn % 2 else n[2] + 1]
        n[2] = 64 + turn + 1
        at = c.table.clone()
        at[:, 10:] = -1
        kk, vv, _ = c.new([1, 1, 1], 1.0 + turn)
        qq, angles = torch.randn(3, 8, D, generator=g).half(), torch.randn(3, 128, generator=g)
        k.copy_(kk), v.copy_(vv), q.copy_(qq), cs.copy_(angles), lengths.copy_(ints(n)), table.copy_(at)
        graphs[turn % 2].replay()
        plain.append(at, n, [0, 1, 2, 3], kk, vv, angles)
        if turn % 5 < 2:
            want, tol, _, _ = attention(plain, at, n, [0, 1, 2, 3], qq, lam=lam if diff else None)
            check(outs[turn % 2], want, tol)
    c.same()


def test_one_batch_for_calls_of_different_rows():
    """A batch object serves calls with more and fewer rows in their tensors, and with another max_rows, in turn."""
    c = Pair(2, 64, 3, 4, seed=40).filled([100, 200, 70])
    batch = kq.KvqPaged8Batch(c.table.cuda(), ints([100, 200, 70]), ints([0, 1, 3, 4]), 2)
    outs = []
    for n, most in ((4, 2), (3, 2), (4, 1), (4, 2)):
        batch.max_rows = most
        k, v = (torch.full((n, 2, D), 777.0, device="cuda") for _ in range(2))
        c.cache.kvq_paged8_read(batch, k, v)
        outs.append(k)
    full, fewer_rows, fewer_a_sequence, again = outs
    assert torch.equal(full, again) and bool((full != 777.0).all())
    assert torch.equal(fewer_rows, full[:3])
    assert bool((fewer_a_sequence[2] == 777.0).all()) and torch.equal(fewer_a_sequence[[0, 3]], full[[0, 3]])
