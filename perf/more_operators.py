"""Cases by which the paged cache of 8-bit floating point and what works on it are followed.

A case is a dict of plain values; `op` names the operator:

  append   KvqPaged8.kvq_paged8_append: new tokens of every sequence go into its pages, keys rotated on the way; what the pages that
           they touch hold afterwards comes back as values, by kvq_paged8_read
  attend   KvqPaged8.kvq_paged8_attention: the last rows of every sequence attend to its tokens up to their own
  diff     KvqPaged8.kvq_paged8_diff_attention: the same with the difference of two softmax maps over the two halves of the channels
  read     KvqPaged8.kvq_paged8_read: cached tokens back as values

`seqs` is a list "rows:tokens ..." (the rows are the last of the tokens).  A page holds `page` tokens of every KV head; keys and values
are e4m3 codes with one power of two for each page, head and kind.  Codes of 32 tokens form a tile, bytes in this order (lane = 16 j + n):

  keys    [sub 2][gh 2][j 4][nh 4][nl 4][gl 2][i 8]:  token 8 nh + 4 sub + nl, channel 64 gh + 32 gl + 8 j + i
  values  [th 4][j 4][n 16][tl 2][i 8]:               token 8 j + i, channel 32 th + 16 tl + n

A scale word is the exponent plus 64.  Where `own` is false the same is computed with elementary torch operations in 32 bits; `exact`
computes it in 64 bits from the definition.
"""
import math

import torch

own = False

D = 128
TOP = 448.0  # the largest e4m3 value
LOW = -40  # the smallest exponent of a scale
ROPE_BASE = 1.0e6


# ------------------------------------------------------------------------------------------------------------- cases
def _append(name, kv, seqs, page, pair=64, out="fp16"):
    return dict(name=name, op="append", kv=kv, seqs=seqs, page=page, pair=pair, out=out)


def _attend(name, q, kv, seqs, page, lse=False):
    return dict(name=name, op="attend", q=q, kv=kv, seqs=seqs, page=page, lse=lse)


def _diff(name, q, kv, seqs, page, norm=True):
    return dict(name=name, op="diff", q=q, kv=kv, seqs=seqs, page=page, norm=norm)


def _read(name, kv, seqs, page, out="fp16"):
    return dict(name=name, op="read", kv=kv, seqs=seqs, page=page, out=out)


def _ragged(rows, lengths):
    return " ".join("%d:%d" % (rows, n) for n in lengths)


def listed():
    return [
        # the smallest: one user's new token with the KV heads of the library's "tiny" workload
        _append("append_step_tiny", 2, "1:765", 32),
        # one decode step of a serving batch: 64 sequences of unequal length, one token each, two maps of 64 channels
        _append("append_step", 8, _ragged(1, [100 + 139 * i for i in range(64)]), 64, pair=32),
        # four 32B-shaped prompts of 32K tokens
        _append("append_prompts", 8, _ragged(32768, [32768] * 4), 128),
        # one user of the "tiny" workload, 1,001 tokens
        _attend("attend_tiny", 8, 2, "1:1001", 32),
        # one decode step of a serving batch: 48 sequences with 7B-shaped heads, from 41 tokens to 30,000
        _attend("attend_ragged", 28, 4, _ragged(1, [int(41 * 1.1505 ** i) for i in range(48)]), 64, lse=True),
        # the 32B-shaped step that the library is benched on: four sequences of 32K tokens
        _attend("attend_32b", 40, 8, _ragged(1, [32768] * 4), 128),
        # the last chunk of 1,024 of two 32B-shaped prompts of 16,000 tokens
        _attend("attend_chunk", 40, 8, "1024:16000 1024:16000", 64),
        # one user, four drafted tokens in a row
        _diff("diff_tiny", 8, 2, "4:1501", 32),
        # a decode step of eight sequences up to 16K tokens
        _diff("diff_step", 40, 8, _ragged(1, [16384, 15000, 16001, 9001, 12288, 16383, 4097, 13130]), 128),
        # a whole prompt
        _diff("diff_prompt", 28, 4, "8192:8192", 64, norm=False),
        # the cached part of an ordinary chat
        _read("read_chat", 8, "2372:2500", 64),
        # the whole of four 32B-shaped sequences
        _read("read_32b", 8, _ragged(32768, [32768] * 4), 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "diff", "diff", "read"])
    kv, page = rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 128, 256])
    q = kv * rng.choice([1, 2, 4, 5, 7, 8, 16])
    n = rng.choice([1, 1, 2, 4, 9, 16, 33, 80])
    most = max(64, min(120000, 1000000 // (n * kv)))
    tokens = [_log(rng, 1, most) for _ in range(n)]
    if op in ("append", "read"):
        kind = rng.choice(["one", "few", "all"])
        rows = [1 if kind == "one" else min(t, _log(rng, 1, 40)) if kind == "few" else t for t in tokens]
        seqs = " ".join("%d:%d" % x for x in zip(rows, tokens))
        out = rng.choice(["fp16", "fp16", "fp32"])
        c = _append("", kv, seqs, page, rng.choice([64, 64, 32]), out) if op == "append" else _read("", kv, seqs, page, out)
    else:
        # one row each; drafted tokens; chunks of prompts; chunks beside single rows
        kind = rng.choice(["one", "one", "few", "chunk", "mixed"])
        room = 4.0e9 / q  # pairs of rows and tokens that cost no more than the largest listed case
        rows = []
        for t in tokens:
            r = 1 if kind == "one" or (kind == "mixed" and rng.random() < 0.7) else _log(rng, 1, 8) if kind == "few" else _log(rng, 1, 4096)
            r = max(1, min(r, t, int(room / n / t)))
            rows.append(r)
        seqs = " ".join("%d:%d" % x for x in zip(rows, tokens))
        c = _attend("", q, kv, seqs, page, rng.random() < 0.4) if op == "attend" else _diff("", q, kv, seqs, page, rng.random() < 0.6)
    return {k: v for k, v in c.items() if k != "name"}


# ------------------------------------------------------------------------------------------------------------ inputs
def _gen(seed, stream):
    return torch.Generator("cuda").manual_seed(int(seed) * 1009 + stream)


def _seqs(case):
    return [tuple(int(x) for x in s.split(":")) for s in case["seqs"].split()]


def _angles(positions, pair):
    """fp32 [n, 2 pair]: the cosines and sines of channel pairs (i, i + pair) at the positions."""
    i = torch.arange(pair, device="cuda", dtype=torch.float64)
    a = positions.double()[:, None] * (ROPE_BASE ** (-i / pair))[None, :]
    return torch.cat([a.cos(), a.sin()], -1).float()


def _rotated(x, angles):
    """Keys [n, heads, 128] in 32 bits, rotated in pairs (i, i + pair) of every run of 2 pair channels."""
    pair = angles.shape[1] // 2
    c, s = angles[:, None, None, :pair], angles[:, None, None, pair:]
    x = x.float().unflatten(-1, (D // (2 * pair), 2 * pair))
    a, b = x[..., :pair], x[..., pair:]
    return torch.cat([a * c - b * s, a * s + b * c], -1).flatten(-2)


def _exponent(x):
    """The smallest e >= LOW with |x| <= 448 2^e, elementwise on non-negative 32-bit values."""
    m, e = torch.frexp(x)  # x = m 2^e, 1/2 <= m < 1, and 448 = 7/8 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(x == 0, torch.full_like(e, LOW), e.clamp(min=LOW))


def _codes(x, e):
    """e4m3 values of x 2^-e, 32 bits in."""
    return torch.ldexp(x, -e).clamp(-TOP, TOP).to(torch.float8_e4m3fn)


def _to_tiles(k, v):
    """e4m3 keys and values [pages, page, kv, 128] as the bytes of tiles [pages, kv, page / 32, 2, 4096]."""
    pages, page, kv, _ = k.shape
    t = page // 32
    k = k.view(torch.uint8).reshape(pages, t, 4, 2, 4, kv, 2, 2, 4, 8)  # nh sub nl | gh gl j i
    v = v.view(torch.uint8).reshape(pages, t, 4, 8, kv, 4, 2, 16)  # j i | th tl n
    k = k.permute(0, 5, 1, 3, 6, 8, 2, 4, 7, 9).reshape(pages, kv, t, 1, 4096)
    v = v.permute(0, 4, 1, 5, 2, 7, 6, 3).reshape(pages, kv, t, 1, 4096)
    return torch.cat([k, v], 3)


def _from_tiles(tiles, words):
    """Keys and values [pages, page, kv, 128] that tiles [pages, kv, page / 32, 2, 4096] stand for, 32 bits."""
    pages, kv, t = tiles.shape[:3]
    k = tiles[:, :, :, 0].reshape(pages, kv, t, 2, 2, 4, 4, 4, 2, 8).permute(0, 2, 6, 3, 7, 1, 4, 8, 5, 9)
    v = tiles[:, :, :, 1].reshape(pages, kv, t, 4, 4, 16, 2, 8).permute(0, 2, 4, 7, 1, 3, 6, 5)
    k, v = (x.reshape(pages, t * 32, kv, D).view(torch.float8_e4m3fn).float() for x in (k, v))
    e = words - 64
    return torch.ldexp(k, e[:, None, :, 0, None]), torch.ldexp(v, e[:, None, :, 1, None])


def _gains(seed, kv):
    """Key channels: four of every head are 20 times as large."""
    g, gain = _gen(seed, 1), torch.ones(kv, D, device="cuda")
    gain.scatter_(1, torch.rand(kv, D, generator=g, device="cuda").topk(4, 1).indices, 20.0)
    return gain


def _cached(case, seed):
    """Pages in any order: (tiles, scale words, table on the host).  Of an append case the tokens in front of the new ones are cached;
    what no token has been written to holds anything."""
    kv, page, seqs, pair = case["kv"], case["page"], _seqs(case), case.get("pair", 32 if case["op"] == "diff" else 64)
    held = [n - r if case["op"] == "append" else n for r, n in seqs]
    need = [-(-n // page) for _, n in seqs]
    n_pages, g = sum(need) + 3, _gen(seed, 2)
    order = torch.randperm(n_pages, generator=g, device="cuda")
    tiles = torch.randint(0, 256, (n_pages, kv, page // 32, 2, 4096), generator=g, device="cuda", dtype=torch.uint8)
    words = torch.randint(24, 72, (n_pages, kv, 2), generator=g, device="cuda", dtype=torch.int32)
    table = torch.full((len(seqs), max(need)), -1, dtype=torch.int32, device="cuda")
    gain, first = _gains(seed, kv), 0
    for s, n in enumerate(held):
        mine = order[first:first + need[s]]
        table[s, :need[s]] = mine.int()
        first += need[s]
        if n == 0:
            continue
        k = torch.randn(n, kv, D, generator=g, device="cuda") * gain
        k = _rotated(k, _angles(torch.arange(n, device="cuda"), pair))
        v = torch.randn(n, kv, D, generator=g, device="cuda")
        tail = -n % 32  # a tile's slots behind the last token are zero
        got, left = -(-n // page), -(-n // page) * page - n
        k, v = (torch.nn.functional.pad(x.half().float(), (0, 0, 0, 0, 0, left)).unflatten(0, (got, page)) for x in (k, v))
        ek, ev = (_exponent(x.abs().amax((1, 3))) for x in (k, v))
        fresh = _to_tiles(_codes(k, ek[:, None, :, None]), _codes(v, ev[:, None, :, None]))
        whole = (n + tail - (got - 1) * page) // 32  # tiles of the last page that hold a token
        tiles[mine[:got - 1]] = fresh[:got - 1]
        tiles[mine[got - 1], :, :whole] = fresh[got - 1, :, :whole]
        words[mine[:got]] = torch.stack([ek, ev], -1).int() + 64
    return tiles, words, table


def _new(case, seed):
    """New tokens, packed: keys before their rotation and values fp16 [rows, kv, 128], angles fp32 [rows, 2 pair]."""
    g, rows = _gen(seed, 3), sum(r for r, _ in _seqs(case))
    k = torch.randn(rows, case["kv"], D, generator=g, device="cuda") * _gains(seed, case["kv"])
    v = torch.randn(rows, case["kv"], D, generator=g, device="cuda")
    at = torch.cat([torch.arange(n - r, n, device="cuda") for r, n in _seqs(case)])
    return k.half(), v.half(), _angles(at, case["pair"])


def _queries(case, seed):
    """fp16 [rows, heads, 128], unit normals (rotation leaves them so), and for two maps the learned weights of the heads, of the norm."""
    g, rows = _gen(seed, 4), sum(r for r, _ in _seqs(case))
    q = torch.randn(rows, case["q"], D, generator=g, device="cuda").half()
    lam = 0.8 - 0.6 * torch.rand(case["q"], generator=g, device="cuda")
    weight = 1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")
    return q, lam, weight


def _begins(rows):
    begin = [0]
    for r in rows:
        begin.append(begin[-1] + r)
    return begin


def _back(case):
    """Rows of each sequence that come back from an append: from the first slot of the first page that it touches on."""
    return [n - (n - r) // case["page"] * case["page"] for r, n in _seqs(case)]


def _dtype(case):
    return torch.float32 if case["out"] == "fp32" else torch.float16


def prepare(case, seed):
    st = {"case": case}
    st["tiles"], st["words"], st["table"] = _cached(case, seed)
    rows = [r for r, _ in _seqs(case)]
    st["begin"] = torch.tensor(_begins(rows), dtype=torch.int32, device="cuda")
    st["lengths"] = torch.tensor([n for _, n in _seqs(case)], dtype=torch.int32, device="cuda")
    total = sum(rows)
    if case["op"] == "append":
        st["k"], st["v"], st["angles"] = _new(case, seed)
        st["back"] = torch.tensor(_begins(_back(case)), dtype=torch.int32, device="cuda")
        total = sum(_back(case))
    if case["op"] in ("append", "read"):
        st["k_out"], st["v_out"] = (torch.empty(total, case["kv"], D, dtype=_dtype(case), device="cuda") for _ in range(2))
    else:
        st["q"], st["lam"], st["weight"] = _queries(case, seed)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(case["q"], total, device="cuda") if case.get("lse") else None
    if own:  # the handles and the workspace that a serving program keeps
        import paper_2505_18610_amd as kq

        st["cache"] = kq.KvqPaged8(st["tiles"], st["words"])
        st["batch"] = kq.KvqPaged8Batch(st["table"], st["lengths"], st["begin"], max_rows=max(rows))
        if case["op"] == "append":
            st["touched"] = kq.KvqPaged8Batch(st["table"], st["lengths"], st["back"], max_rows=max(_back(case)))
        if case["op"] in ("attend", "diff"):
            need = kq.kvq_paged8_workspace_bytes(st["cache"], st["batch"], case["q"], total, case["op"] == "diff")
            st["workspace"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    return st


# -------------------------------------------------------------------------------------------------------------- pass
def run(st):
    return (_run_own if own else _run_plain)(st, st["case"])


def _run_own(st, case):
    cache = st["cache"]
    if case["op"] == "append":
        cache.kvq_paged8_append(st["batch"], st["k"], st["v"], st["angles"])
        cache.kvq_paged8_read(st["touched"], st["k_out"], st["v_out"])
        return st["k_out"], st["v_out"]
    if case["op"] == "read":
        cache.kvq_paged8_read(st["batch"], st["k_out"], st["v_out"])
        return st["k_out"], st["v_out"]
    if case["op"] == "attend":
        cache.kvq_paged8_attention(st["batch"], st["q"], st["out"], lse=st["lse"], workspace=st["workspace"])
        return (st["out"], st["lse"]) if case["lse"] else st["out"]
    cache.kvq_paged8_diff_attention(st["batch"], st["q"], st["lam"], st["out"], norm_weight=st["weight"] if case["norm"] else None,
                                    norm_eps=1e-5, out_scale=0.2, workspace=st["workspace"])
    return st["out"]


def _softmax_product(s, v):
    """softmax(s) v in 32 bits and the log of the sum of exponentials."""
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m)
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / total, (m + torch.log(total))[..., 0]


def _run_plain(st, case):
    return (_plain_append if case["op"] == "append" else _plain_read if case["op"] == "read" else _plain_attend)(st, case)


def _spread(counts, total):
    """Which of the sequences each of `total` things belongs to that are counted by sequence, and its number in it."""
    of = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts, output_size=total)
    return of, torch.arange(total, device="cuda") - (counts.cumsum(0) - counts)[of]


def _plain_append(st, case):
    page, seqs = case["page"], _seqs(case)
    lengths, rows = st["lengths"].long(), st["begin"].diff().long()
    first = (lengths - rows) // page  # the first page that is touched, and the tokens in it already
    old, got = lengths - rows - first * page, -(-lengths // page) - first
    n_pages = sum(-(-n // page) - (n - r) // page for r, n in seqs)
    of, i = _spread(got, n_pages)
    mine, begins = st["table"][of, first[of] + i].long(), got.cumsum(0) - got
    of, i = _spread(rows, st["k"].shape[0])
    new_at = begins[of] * page + old[of] + i
    of, i = _spread(old + rows, st["k_out"].shape[0])
    back_at = begins[of] * page + i
    mark = torch.arange(page, device="cuda")[None, :] < old[:, None]  # slots of a first page that are held
    was = _from_tiles(st["tiles"][mine[begins]], st["words"][mine[begins]])
    codes, exponents = [], []
    for kind, (x, out) in enumerate(((_rotated(st["k"], st["angles"]), st["k_out"]), (st["v"].float(), st["v_out"]))):
        pages = torch.zeros(n_pages * page, case["kv"], D, device="cuda")
        pages[new_at] = x
        pages = pages.unflatten(0, (n_pages, page))
        e = _exponent(pages.abs().amax((1, 3)))
        # a page that holds tokens already: its scale is kept or raised, and then they are rounded again
        kept = torch.maximum(e[begins], st["words"][mine[begins], :, kind] - 64)
        e[begins] = torch.where(old[:, None] > 0, kept, e[begins])
        pages[begins] = torch.where(mark[:, :, None, None], was[kind], pages[begins])
        c = _codes(pages, e[:, None, :, None])
        out.copy_(torch.ldexp(c.float(), e[:, None, :, None]).flatten(0, 1)[back_at])
        codes.append(c)
        exponents.append(e)
    st["tiles"][mine] = _to_tiles(*codes)
    st["words"][mine] = torch.stack(exponents, -1).int() + 64
    return st["k_out"], st["v_out"]


def _plain_read(st, case):
    page, seqs = case["page"], _seqs(case)
    lengths, rows = st["lengths"].long(), st["begin"].diff().long()
    first = (lengths - rows) // page
    got = -(-lengths // page) - first
    of, i = _spread(got, sum(-(-n // page) - (n - r) // page for r, n in seqs))
    mine = st["table"][of, first[of] + i].long()
    of, i = _spread(rows, st["k_out"].shape[0])
    at = (got.cumsum(0) - got)[of] * page + (lengths - rows - first * page)[of] + i
    for out, x in zip((st["k_out"], st["v_out"]), _from_tiles(st["tiles"][mine], st["words"][mine])):
        out.copy_(x.flatten(0, 1)[at])
    return st["k_out"], st["v_out"]


def _plain_attend(st, case):
    kv, g, page, a = case["kv"], case["q"] // case["kv"], case["page"], 0
    for s, (r, n) in enumerate(_seqs(case)):
        mine = st["table"][s, :-(-n // page)].long()
        k, v = (x.flatten(0, 1)[:n].transpose(0, 1) for x in _from_tiles(st["tiles"][mine], st["words"][mine]))
        k, v = k.transpose(1, 2).contiguous(), v.contiguous()  # [kv, 128, n], [kv, n, 128]
        step = max(1, (1 << 29) // (case["q"] * n))
        for x in range(0, r, step):
            y = min(r, x + step)
            q = st["q"][a + x:a + y].float().transpose(0, 1).reshape(kv, g * (y - x), D)
            hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n - r + x, n - r + y, device="cuda")[:, None]
            hidden = hidden.repeat(g, 1)
            if case["op"] == "attend":
                sc = (torch.matmul(q, k) * D ** -0.5).masked_fill_(hidden, -math.inf)
                o, l = _softmax_product(sc, v)
                if case["lse"]:
                    st["lse"][:, a + x:a + y] = l.reshape(case["q"], y - x)
            else:
                o = []
                for c in (0, 64):
                    sc = (torch.matmul(q[..., c:c + 64].contiguous(), k[:, c:c + 64].contiguous()) * 64 ** -0.5)
                    o.append(_softmax_product(sc.masked_fill_(hidden, -math.inf), v)[0].reshape(kv, g, y - x, D))
                o = o[0] - st["lam"].reshape(kv, g, 1, 1) * o[1]
                if case["norm"]:
                    o = o * torch.rsqrt((o * o).mean(-1, keepdim=True) + 1e-5) * st["weight"]
                o = o * 0.2
            st["out"][a + x:a + y] = o.reshape(case["q"], y - x, D).transpose(0, 1).to(st["out"].dtype)
        a += r
    return (st["out"], st["lse"]) if case.get("lse") else st["out"]


# ------------------------------------------------------------------------------------------------- the same, exactly
def _exact_values(codes, word):
    """uint8 codes and the scale words of their pages, 64 bits: sign, 4 bits of exponent, 3 of mantissa."""
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    size = torch.where(e == 0, m * 2.0 ** -9, (8.0 + m) * torch.exp2(e.double() - 10.0))
    return torch.where(c >= 128, -size, size) * torch.exp2(word.double() - 64.0)


def _exact_sequence(case, tiles, words, table, s, begin, end):
    """Tokens begin .. end - 1 of sequence s, fp64 [kv, tokens, 128] twice: byte by byte from where the layout puts it."""
    page = case["page"]
    t = torch.arange(begin, end, device="cuda")
    c = torch.arange(D, device="cuda")
    at = table[s].long()[t // page]
    tile, slot = (t % page) // 32, (t % 32)[:, None]
    lane_k = 16 * (c % 32 // 8)[None] + 4 * (slot // 8) + slot % 4
    chunk_k = 2 * (slot // 4 % 2) + (c // 64)[None]
    byte_k = (chunk_k * 64 + lane_k) * 16 + (c // 32 % 2 * 8 + c % 8)[None]
    lane_v = 16 * (slot // 8) + (c % 16)[None]
    byte_v = ((c // 32)[None] * 64 + lane_v) * 16 + (c // 16 % 2 * 8)[None] + slot % 8
    both = []
    for kind, byte in enumerate((byte_k, byte_v)):
        heads = []
        for h in range(case["kv"]):
            flat = ((at * case["kv"] + h) * (page // 32) + tile) * 2 + kind
            codes = tiles.reshape(-1)[flat[:, None] * 4096 + byte]
            heads.append(_exact_values(codes, words[at, h, kind][:, None]))
        both.append(torch.stack(heads))
    return both


def _exact_round(x, e):
    """x [.., 128] in 64 bits to e4m3 multiples of 2^e, ties to even, as values."""
    y = x * 2.0 ** -e
    size = y.abs().clamp(max=TOP)
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(y) * torch.clamp(torch.round(size / step) * step, max=TOP) * 2.0 ** e


def _exact_append(case, seed):
    tiles, words, table = _cached(case, seed)
    k, v, angles = _new(case, seed)
    pair, page, outs, a = case["pair"], case["page"], ([], []), 0
    i = torch.arange(D, device="cuda")
    lower = i % (2 * pair) < pair
    other = torch.where(lower, i + pair, i - pair)
    sign = torch.where(lower, -1.0, 1.0).double()
    cos, sin = angles[:, i % pair].double(), angles[:, pair + i % pair].double()
    for s, (r, n) in enumerate(_seqs(case)):
        x = k[a:a + r].double()
        x = x * cos[a:a + r, None] + x[..., other] * sign * sin[a:a + r, None]
        fresh = (x, v[a:a + r].double())
        old = (n - r) % page
        held = _exact_sequence(case, tiles, words, table, s, n - r - old, n - r)
        for kind in (0, 1):
            got = torch.cat([held[kind].transpose(0, 1), fresh[kind]])
            pages = -(-got.shape[0] // page)
            low = torch.full((pages, case["kv"]), LOW, dtype=torch.int64, device="cuda")
            if old:
                low[0] = words[table[s, (n - r) // page].long(), :, kind] - 64
            new = torch.nn.functional.pad(fresh[kind].abs(), (0, 0, 0, 0, old, pages * page - got.shape[0])).unflatten(0, (pages, page))
            big = new.amax((1, 3))
            e = torch.ceil(torch.log2((big / TOP).clamp(min=2.0 ** LOW))).long()
            e = torch.where(torch.exp2(e.double() - 1) * TOP >= big, e - 1, e)  # (the logarithm is rounded)
            e = torch.where(torch.exp2(e.double()) * TOP < big, e + 1, e)
            e = torch.maximum(e, low).double().repeat_interleave(page, 0)[:got.shape[0], :, None]
            outs[kind].append(_exact_round(got, e))
        a += r
    return torch.cat(outs[0]), torch.cat(outs[1])


def exact(case, seed):
    if case["op"] == "append":
        return _exact_append(case, seed)
    tiles, words, table = _cached(case, seed)
    seqs, kv = _seqs(case), case["kv"]
    if case["op"] == "read":
        both = [_exact_sequence(case, tiles, words, table, s, n - r, n) for s, (r, n) in enumerate(seqs)]
        return tuple(torch.cat([x[kind] for x in both], 1).transpose(0, 1).contiguous() for kind in (0, 1))
    q, lam, weight = _queries(case, seed)
    g = case["q"] // kv
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(case["q"], q.shape[0], dtype=torch.float64, device="cuda")
    a = 0
    for s, (r, n) in enumerate(seqs):
        k, v = _exact_sequence(case, tiles, words, table, s, 0, n)
        for h in range(case["q"]):
            for x in range(0, r, 4096):
                y = min(r, x + 4096)
                seen = torch.arange(n - r + x, n - r + y, device="cuda")[:, None] >= torch.arange(n, device="cuda")[None]
                p = []
                for c0, c1 in ((0, D),) if case["op"] == "attend" else ((0, 64), (64, D)):
                    sc = q[a + x:a + y, h, c0:c1].double() @ k[h // g, :, c0:c1].t() / (c1 - c0) ** 0.5
                    sc[~seen] = -math.inf
                    lse[h, a + x:a + y] = torch.logsumexp(sc, -1)
                    p.append(torch.softmax(sc, -1))
                o = p[0] if len(p) == 1 else p[0] - lam[h].double() * p[1]
                o = o @ v[h // g]
                if case["op"] == "diff":
                    if case["norm"]:
                        o = o / torch.sqrt((o ** 2).mean(-1, keepdim=True) + 1e-5) * weight.double()
                    o = 0.2 * o
                out[a + x:a + y, h] = o
        a += r
    return (out, lse) if case.get("lse") else out


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    seqs, kv, wide = _seqs(case), case["kv"], 4 if case.get("out") == "fp32" else 2
    rows, tokens = sum(r for r, _ in seqs), sum(n for _, n in seqs)
    if case["op"] == "append":
        back = sum(_back(case))
        return {"bytes": rows * (kv * D * (4 + 2) + 8 * case["pair"]) + back * kv * 2 * D * (1 + wide), "flops": rows * kv * D * 8}
    if case["op"] == "read":
        return {"bytes": rows * kv * 2 * D * (1 + wide), "flops": rows * kv * 2 * D}
    pairs = sum(r * (n - r) + r * (r + 1) // 2 for r, n in seqs)
    return {"bytes": tokens * kv * 2 * D + rows * case["q"] * (D * 4 + (4 if case.get("lse") else 0)),
            "flops": (4 if case["op"] == "attend" else 6) * D * case["q"] * pairs}
