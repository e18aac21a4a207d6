"""The plain form of the paged cache of 8-bit floating point, where a sequence outgrows its table."""
import torch

from paged8_plain import D, Plain, attention, exponent, to_codes, value


def filled(n, page=32, pages=2):
    p = Plain(torch.zeros(pages, 1, page // 32, 2, 4096, dtype=torch.uint8), torch.zeros(pages, 1, 2, dtype=torch.int32))
    table = torch.arange(pages, dtype=torch.int32)[None]
    x = torch.arange(1, n + 1).half()[:, None, None].expand(n, 1, D) / 8  # token t holds (t + 1) / 8
    p.append(table, [n], [0, n], x, x)
    return p, table


def test_rows_beyond_the_table_are_not_appended():
    p, table = filled(64)
    codes, words = p.codes.clone(), p.words.clone()
    x = torch.full((1, 1, D), 100.0).half()
    for n in (65, 66, 1 << 30):
        p.append(table, [n], [0, 1], x, x)
    assert torch.equal(codes, p.codes) and torch.equal(words, p.words)
    p, table = filled(50)
    x = (torch.arange(30).half() + 20)[:, None, None].expand(30, 1, D)
    p.append(table, [78], [0, 30], x, x)  # tokens 48 .. 77, of which 64 and on are not there
    k, _, _ = p.values(table[0], 64, 0)
    e = exponent(35.0)  # of the rows that are there
    assert torch.equal(k[48:], value(to_codes(x[:16, 0].float(), e), e)) and float(k[47, 0]) == 6.0


def test_queries_beyond_the_table_see_all_of_it():
    p, table = filled(64)
    q = torch.zeros(4, 1, D).half()  # equal weights: the mean of what a row sees
    out, _, _, _ = attention(p, table, [66], [0, 4], q)  # tokens 62 .. 65
    _, v, _ = p.values(table[0], 64, 0)
    means = [float(v[:n, 0].mean()) for n in (63, 64, 64, 64)]
    assert torch.allclose(out[:, 0, 0], torch.tensor(means, dtype=torch.float64), rtol=1e-12)
