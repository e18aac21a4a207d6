"""The paged cache of 8-bit floating point in plain form, on the CPU: appends page by page, attention in 64 bits, and how far the library may
be from it."""
import math

import torch

D, TOP, LOW = 128, 448.0, -40


def tile_bytes():
    """[token 32][channel 128] -> byte of a K tile, of a V tile."""
    t, c = torch.arange(32)[:, None], torch.arange(D)[None]
    lane_k, slot_k = 16 * (c % 32 // 8) + 4 * (t // 8) + t % 4, (t // 4 % 2 * 4 + c // 32) * 8 + c % 8
    lane_v, slot_v = 16 * (t // 8) + c % 16, c // 16 * 8 + t % 8
    return [(slot // 16 * 64 + lane) * 16 + slot % 16 for lane, slot in ((lane_k, slot_k), (lane_v, slot_v))]


AT = tile_bytes()


def rotate(k, cos_sin):
    """fp32 keys [n, heads, 128], every product and sum rounded."""
    if cos_sin is None:
        return k.float()
    pair = cos_sin.shape[1] // 2
    c, s = cos_sin[:, None, None, :pair], cos_sin[:, None, None, pair:]
    x = k.float().reshape(k.shape[0], k.shape[1], D // (2 * pair), 2 * pair)
    a, b = x[..., :pair], x[..., pair:]
    return torch.cat([a * c - b * s, a * s + b * c], -1).reshape(k.shape)


def exponent(largest):
    """The smallest e >= LOW with largest <= 448 2^e."""
    if largest == 0:
        return LOW
    e = math.frexp(largest / TOP)[1]
    return max(LOW, e - 1 if largest <= math.ldexp(TOP, e - 1) else e)


def to_codes(x, e):
    """e4m3 bytes of x 2^-e (64 bits in, so that nothing is rounded before)."""
    y = x.double() * 2.0 ** -e
    y = torch.where(torch.isfinite(y), y, torch.full_like(y, math.nan))
    size = y.abs().nan_to_num(0.0)
    step = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    r = (torch.round(size / step) * step).clamp(max=TOP) * torch.where(torch.signbit(y), -1.0, 1.0)
    return torch.where(torch.isnan(y), torch.full_like(r, math.nan), r).float().to(torch.float8_e4m3fn).view(torch.uint8)


def value(codes, e):
    return codes.view(torch.float8_e4m3fn).double() * 2.0 ** e


class Plain:
    """codes [pages, kv, tiles, 2, 4096] and words [pages, kv, 2] as the library keeps them, on the CPU."""

    def __init__(self, codes, words):
        self.codes, self.words = codes.clone(), words.clone()
        self.pages, self.kv, tiles = codes.shape[:3]
        self.page = 32 * tiles

    def tokens(self, page, kv, kind):
        """uint8 [page tokens, 128] of one page and head."""
        return self.codes[page, kv, :, kind][:, AT[kind]].reshape(self.page, D)

    def append(self, table, lengths, begin, k, v, cos_sin=None):
        new = (rotate(k, cos_sin), v.float())
        for s in range(len(lengths)):
            r, n = begin[s + 1] - begin[s], lengths[s]
            n = max(0, n)
            held = min(n, table.shape[1] * self.page)  # tokens beyond the table do not exist
            first = max(0, n - r)
            for at in range(first // self.page, -(-held // self.page)) if r else ():
                page = int(table[s, at])
                if not 0 <= page < self.pages:
                    continue
                t0 = at * self.page
                b, e = max(0, first - t0), min(self.page, held - t0)
                for kv in range(self.kv):
                    for kind in (0, 1):
                        x = new[kind][begin[s] + t0 + b - (n - r):begin[s] + t0 + e - (n - r), kv]
                        self._page(page, kv, kind, b, e, x)

    def _page(self, page, kv, kind, b, e, x):
        good = torch.isfinite(x)
        largest = float(x.abs()[good].max()) if good.any() else 0.0
        ex, nan = exponent(largest), 0 if good.all() else 0x100
        held = self.tokens(page, kv, kind)
        if b:
            old = int(self.words[page, kv, kind])
            old_e = (old & 0xff) - 64
            nan |= old & 0x100
            ex = max(ex, old_e)
            if ex != old_e:
                held[:b] = to_codes(value(held[:b], old_e), ex)
        first = -(-b // 32) * 32  # tiles that held no token are written whole
        held[min(first, e):-(-e // 32) * 32] = 0
        held[b:e] = to_codes(x, ex)
        whole = held.reshape(-1, 32, D)
        for t in range(-(-e // 32)):
            self.codes[page, kv, t, kind][AT[kind].reshape(-1)] = whole[t].reshape(-1)
        self.words[page, kv, kind] = (ex + 64) | nan

    def values(self, table_row, n, kv):
        """Keys and values [n, 128] of one sequence and head, 64 bits, and which of the tokens exist."""
        out, there = [], torch.ones(n, dtype=torch.bool)
        for kind in (0, 1):
            rows = torch.zeros(n, D, dtype=torch.float64)
            for at in range(-(-n // self.page)):
                page, b = int(table_row[at]), at * self.page
                if not 0 <= page < self.pages:
                    there[b:b + self.page] = False
                    continue
                e = (int(self.words[page, kv, kind]) & 0xff) - 64
                rows[b:b + self.page] = value(self.tokens(page, kv, kind), e)[:n - b]
            out.append(rows)
        return out[0], out[1], there


def attention(plain, table, lengths, begin, q, scale=0.0, lam=None, weight=None, eps=1e-5, out_scale=1.0, out_eps=2.0 ** -11):
    """64 bits: (out, bound of its error, lse, bound) for queries [rows, heads, 128]; rows of no sequence are NaN.

    The bound.  Scores: 128 products summed in 32 bits, ds = 130 2^-24 scale |q| . |k| at most, with the exponential's own 2^-22; a
    probability is rounded to fp16 once (2^-11 of it, or 2^-32 of the row's leading one) in the product and in the sum that divides; sums of n
    terms in 32 bits.  With a = sum p |v|: (2 2^-11 + 2 max ds + (n + 64) 2^-23) a + n 2^-30 max |v|, and values below 2^-20 are held to 2^-24.
    Then the output is rounded, out_eps of it."""
    rows, heads, _ = q.shape
    g = heads // plain.kv
    maps = 1 if lam is None else 2
    w = D // maps
    scale = scale or w ** -0.5
    out = torch.full((rows, heads, D), math.nan, dtype=torch.float64)
    tol, lse, ltol = out.clone(), torch.full((heads, rows), math.nan, dtype=torch.float64), torch.full((heads, rows), math.nan, dtype=torch.float64)
    for s in range(len(lengths)):
        r, end = begin[s + 1] - begin[s], max(0, lengths[s])
        n = min(end, table.shape[1] * plain.page)
        if not r:
            continue
        a, b = begin[s], begin[s + 1]
        i = torch.arange(r)
        for kv in range(plain.kv):
            k, v, there = plain.values(table[s], n, kv)
            sees = (torch.arange(n)[None] <= end - r + i[:, None]) & there[None]
            for h in range(kv * g, kv * g + g):
                o, e = torch.zeros(r, D, dtype=torch.float64), torch.zeros(r, D, dtype=torch.float64)
                for m in range(maps):
                    c = slice(m * w, m * w + w)
                    qq, kk = q[a:b, h, c].double(), k[:, c]
                    sc = (qq @ torch.nan_to_num(kk).t()) * scale
                    sc = sc + torch.where(torch.isnan(kk).any(1), math.nan, 0.0)[None]
                    ds = (qq.abs() @ torch.nan_to_num(kk).abs().t()) * abs(scale) * 130 * 2.0 ** -24
                    sc = torch.where(sees, sc, torch.full_like(sc, -math.inf))
                    top = sc.amax(1, keepdim=True) if n else torch.zeros(r, 1, dtype=torch.float64)
                    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                    p = torch.exp(sc - top)
                    total = p.sum(1, keepdim=True)
                    p = p / torch.where(total == 0, torch.ones_like(total), total)
                    bad = torch.isnan(v)
                    o_m = p @ torch.nan_to_num(v)
                    o_m = torch.where((sees.double() @ bad.double()) > 0, torch.full_like(o_m, math.nan), o_m)
                    ds_max = (ds * sees).amax(1, keepdim=True) if n else torch.zeros(r, 1, dtype=torch.float64)
                    size = p @ torch.nan_to_num(v).abs()
                    big = torch.nan_to_num(v).abs().max() if n else 0.0
                    e_m = (2.0 ** -10 + 2 * ds_max + 2.0 ** -21 + (n + 64) * 2.0 ** -23) * size + n * 2.0 ** -30 * big + 2.0 ** -24
                    f = 1.0 if m == 0 else -float(lam[h])
                    o, e = o + f * o_m, e + abs(f) * e_m
                    if maps == 1:
                        lse[h, a:b] = (top + torch.log(total))[:, 0]
                        ltol[h, a:b] = (ds_max[:, 0] + 2.0 ** -21 + (n + 64) * 2.0 ** -24) + 2.0 ** -22 * lse[h, a:b].abs().nan_to_num(0, 0, 0)
                if maps == 2:
                    e = e + 2.0 ** -23 * o.abs()
                    if weight is not None:
                        rho = torch.sqrt((o ** 2).mean(1, keepdim=True) + eps)
                        off = torch.sqrt((e ** 2).mean(1, keepdim=True))
                        # first order, doubled where the error is not small beside the norm
                        ww = weight.double().abs()[None] / torch.where(rho == 0, torch.ones_like(rho), rho)
                        grown = 1 + 2 * off / torch.where(rho == 0, torch.ones_like(rho), rho)
                        e = ww * (e + o.abs() * off / torch.where(rho == 0, torch.ones_like(rho), rho)) * grown + ww * o.abs() * 2.0 ** -20
                        o = torch.where(rho == 0, torch.zeros_like(o), o / rho) * weight.double()[None]
                    o, e = o * out_scale, e * abs(out_scale)
                if out_eps == 2.0 ** -11:  # outputs of 16 bits: magnitudes beyond the largest become it
                    o = o.clamp(-65504, 65504)
                out[a:b, h], tol[a:b, h] = o, e + out_eps * (o.abs() + e) + 2.0 ** -25
    return out, tol, lse, ltol


def check(got, want, tol):
    got = got.double().cpu()
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(got), bad)
    off = (got - want).abs()[~bad]
    assert bool((off <= tol[~bad]).all()), float((off / tol[~bad]).max())
