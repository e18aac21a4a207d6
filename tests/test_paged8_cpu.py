"""Refusals of the calls on the paged cache of 8-bit floating point, its workspace sizes and its plain form; nothing is launched here."""
import ctypes as C
import os

import pytest
import torch

import paper_2505_18610_amd as kq
from paged8_plain import AT, Plain, exponent, rotate, to_codes, value
from paper_2505_18610_amd.binding import _Paged8, _Paged8Batch, _Paged8Rows

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")
A = 1 << 20  # an address that is never used


def structs(cache=None, batch=None):
    c = dict(codes_dev=A, words_dev=A, n_pages=10, n_kv_heads=2, page_tokens=64)
    b = dict(table_dev=A, lengths_dev=A, row_begin_dev=A, table_stride=8, n_seqs=3, table_pages=8, n_rows=6, max_rows=4)
    c.update(cache or {}), b.update(batch or {})
    return C.byref(_Paged8(**c)), C.byref(_Paged8Batch(**b))


def rows(heads, **kw):
    return C.byref(_Paged8Rows(**{**dict(data_dev=A, row_stride=heads * 128, head_stride=128), **kw}))


def append(cache=None, batch=None, k={}, v={}, cs=A, pair=64):
    return kq.load_library().kvq_paged8_append(*structs(cache, batch), rows(2, **k), rows(2, **v), cs, pair, None)


def read(cache=None, batch=None, k={}, v={}, fp32=0):
    return kq.load_library().kvq_paged8_read(*structs(cache, batch), rows(2, **k), rows(2, **v), fp32, None)


def attend(cache=None, batch=None, q={}, out={}, heads=8, fp32=0, scale=0.0, lse=None, ws=A, ws_bytes=1 << 40):
    return kq.load_library().kvq_paged8_attention(*structs(cache, batch), rows(heads, **q), rows(heads, **out), heads, fp32, scale, lse, ws, ws_bytes, None)


def diff(cache=None, batch=None, q={}, out={}, heads=8, fp32=0, scale=0.0, lam=A, weight=A, eps=1e-5, out_scale=1.0, ws=A, ws_bytes=1 << 40):
    return kq.load_library().kvq_paged8_diff_attention(*structs(cache, batch), rows(heads, **q), lam, rows(heads, **out), heads, fp32, scale, weight,
                                                       eps, out_scale, ws, ws_bytes, None)


SHARED = [dict(cache=x) for x in (
    dict(codes_dev=None), dict(codes_dev=A + 8), dict(words_dev=None), dict(words_dev=A + 4), dict(n_pages=0), dict(n_kv_heads=0), dict(page_tokens=16),
    dict(page_tokens=48), dict(page_tokens=512), dict(n_kv_heads=1 << 17))] + [dict(batch=x) for x in (
        dict(table_dev=None), dict(table_dev=A + 2), dict(lengths_dev=None), dict(lengths_dev=A + 1), dict(row_begin_dev=A + 2), dict(table_stride=7),
        dict(table_stride=-8), dict(n_seqs=-1), dict(n_seqs=4097), dict(table_pages=0), dict(table_pages=1 << 27, table_stride=1 << 27), dict(n_rows=-1),
        dict(n_rows=1 << 30), dict(max_rows=0), dict(row_begin_dev=None, n_rows=2))]


@pytest.mark.parametrize("bad", SHARED)
def test_refusals_of_all(bad):
    for call in (append, read, attend, diff):
        assert call(**bad) == kq.KVQ_E_INVALID


@pytest.mark.parametrize("bad", [dict(k=dict(data_dev=None)), dict(v=dict(data_dev=A + 8)), dict(k=dict(row_stride=-256)), dict(v=dict(head_stride=132)),
                                 dict(cs=A + 4), dict(pair=16), dict(pair=0), dict(k=dict(row_stride=1 << 40))])
def test_refusals_of_append(bad):
    assert append(**bad) == kq.KVQ_E_INVALID


@pytest.mark.parametrize("bad", [dict(k=dict(data_dev=None)), dict(v=dict(data_dev=A + 4)), dict(k=dict(row_stride=0)), dict(v=dict(head_stride=64)),
                                 dict(k=dict(row_stride=128)), dict(k=dict(row_stride=260), fp32=0), dict(v=dict(row_stride=258), fp32=1)])
def test_refusals_of_read(bad):
    assert read(**bad) == kq.KVQ_E_INVALID


ATTENTION = [dict(q=dict(data_dev=None)), dict(q=dict(row_stride=1020)), dict(out=dict(data_dev=A + 2)), dict(out=dict(row_stride=512)),
             dict(out=dict(head_stride=0)), dict(heads=7), dict(heads=34), dict(heads=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=None),
             dict(ws=A + 8), dict(ws_bytes=1000), dict(batch=dict(n_seqs=4096, table_pages=1 << 20, table_stride=1 << 20, max_rows=4))]


@pytest.mark.parametrize("bad", ATTENTION)
def test_refusals_of_attention(bad):
    assert attend(**bad) == kq.KVQ_E_INVALID
    assert diff(**bad) == kq.KVQ_E_INVALID


def test_more_refusals():
    assert attend(lse=A + 2) == kq.KVQ_E_INVALID
    for bad in (dict(lam=None), dict(lam=A + 2), dict(weight=A + 4), dict(eps=-1.0), dict(eps=float("nan")), dict(out_scale=float("inf"))):
        assert diff(**bad) == kq.KVQ_E_INVALID


@pytest.mark.parametrize("batch", [dict(n_seqs=0, table_dev=None, lengths_dev=None, row_begin_dev=None, n_rows=0), dict(n_rows=0)])
def test_nothing_to_do(batch):
    none = dict(data_dev=None)
    assert append(batch=batch, k=none, v=none) == read(batch=batch, k=none, v=none) == kq.KVQ_OK
    assert attend(batch=batch, q=none, out=none, ws=None, ws_bytes=0) == diff(batch=batch, q=none, out=none, ws=None, ws_bytes=0) == kq.KVQ_OK


def test_workspace_bytes():
    def need(heads=8, maps=0, **batch):
        return kq.load_library().kvq_paged8_workspace_bytes(*structs(None, batch), heads, maps)

    few = need()
    assert few > 0 and few % 16 == 0 and need(maps=1) >= few and need(heads=7) == 0 and need(max_rows=0) == 0
    assert need(table_pages=1024, table_stride=1024) > few
    assert attend(ws_bytes=few - 1) == kq.KVQ_E_INVALID


def test_plain_exponent_and_codes():
    """The plain form's own rounding against torch's conversion, and the exponent's definition."""
    g = torch.Generator().manual_seed(0)
    x = torch.cat([torch.randn(4096, generator=g) * 2.0 ** e for e in range(-12, 9)]).clamp(-448, 448)
    ties = (torch.arange(0, 127).to(torch.uint8).view(torch.float8_e4m3fn).double())
    x = torch.cat([x, ((ties[1:] + ties[:-1]) / 2).float(), ties.float(), -ties.float()])
    assert torch.equal(to_codes(x, 0), x.to(torch.float8_e4m3fn).view(torch.uint8))
    for e in (-40, -33, -1, 0, 8, 20):
        top = 448.0 * 2.0 ** e
        assert exponent(top) == e and exponent(top * (1 + 1e-12)) == e + 1 and (e == -40 or exponent(top / 2 * (1 + 1e-12)) == e)
    assert exponent(0.0) == -40 and exponent(1e-30) == -40
    assert float(value(to_codes(torch.tensor([1.0]), -8), -8)) == 1.0


def test_plain_layout_is_that_of_the_header():
    """The plain form's tile bytes from kvq_layout.h's slots against the bytes that include/kvq.h lists."""
    for t in range(32):
        for c in range(128):
            nh, sub, nl, gh, gl, j, i = t // 8, t // 4 % 2, t % 4, c // 64, c // 32 % 2, c // 8 % 4, c % 8
            assert AT[0][t, c] == (((((sub * 2 + gh) * 4 + j) * 4 + nh) * 4 + nl) * 2 + gl) * 8 + i
            j, i, th, tl, n = t // 8, t % 8, c // 32, c // 16 % 2, c % 16
            assert AT[1][t, c] == (((th * 4 + j) * 16 + n) * 2 + tl) * 8 + i


def test_plain_append_raises_scales():
    """Tokens of twice the size, one after the other: the page's exponent follows, held codes stay what they stood for."""
    p = Plain(torch.zeros(1, 1, 1, 2, 4096, dtype=torch.uint8), torch.zeros(1, 1, 2, dtype=torch.int32))
    table = torch.zeros(1, 1, dtype=torch.int32)
    for n in range(1, 9):
        x = torch.full((1, 1, 128), 2.0 ** n).half()
        p.append(table, [n], [0, 1], x, x)
    k, v, _ = p.values(table[0], 8, 0)
    assert torch.equal(k[:, 0], 2.0 ** torch.arange(1, 9).double()) and torch.equal(k, v)
    assert p.words.tolist() == [[[64, 64]]]


def test_plain_rotation_keeps_lengths():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 2, 128, generator=g).half()
    for pair in (64, 32):
        a = torch.rand(5, pair, generator=g) * 6
        y = rotate(x, torch.cat([a.cos(), a.sin()], 1))
        w = 2 * pair
        assert torch.allclose(y.reshape(5, 2, -1, w).norm(dim=-1), x.float().reshape(5, 2, -1, w).norm(dim=-1), rtol=1e-5)
        assert not torch.equal(y, x.float())
