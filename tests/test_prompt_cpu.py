"""Refusals of kvq_prompt_attention and its workspace sizes; nothing is launched here."""
import ctypes as C
import os

import pytest

import paper_2505_18610_amd as kq
from paper_2505_18610_amd.binding import _Prompt, _rows

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")
A = 1 << 20  # an address that is never used


def call(n_q=8, n_kv=2, strides=None, scale=0.0, q=A, k=A, v=A, out=A, lse=None, qb=(0, 10), kb=None, n=None, ws=None, null=False):
    s = dict(q_token=n_q * 128, q_head=128, k_token=n_kv * 128, k_head=128, v_token=n_kv * 128, v_head=128, out_token=n_q * 128, out_head=128)
    s.update(strides or {})
    d = _Prompt(n_q, n_kv, *(s[x + "_" + y] for x in ("q", "k", "v", "out") for y in ("token", "head")), 0, scale)
    return kq.load_library().kvq_prompt_attention(None if null else C.byref(d), q, k, v, out, lse, None if qb is None else _rows(qb),
                                                  None if kb is None else _rows(kb), len(qb) - 1 if n is None else n, ws, 0, None)


@pytest.mark.parametrize("bad", [
    dict(null=True), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=A + 2), dict(k=A + 8), dict(v=A + 4), dict(out=A + 8),
    dict(lse=A + 2), dict(ws=A + 4), dict(n_q=7), dict(n_q=34), dict(n_kv=0), dict(n_q=0), dict(qb=None, n=1), dict(n=0), dict(n=-1),
    dict(qb=(0, 10, 9)), dict(qb=(-1, 10)), dict(kb=(0, -3)), dict(kb=(5, 4)), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(strides={"q_token": 1020}), dict(strides={"k_head": 4}), dict(strides={"q_head": -128}), dict(strides={"k_token": 0}),
    dict(strides={"v_token": 64}), dict(strides={"v_token": 1 << 22}), dict(strides={"out_token": 0}), dict(strides={"out_head": 0})])
def test_refusals(bad):
    assert call(**bad) == kq.KVQ_E_INVALID


def test_nothing_to_do():
    assert call(qb=(4, 4), q=None, out=None) == kq.KVQ_OK


def test_workspace():
    assert kq.kvq_prompt_workspace_bytes(64, 8, [0, 32768]) == 0                    # row blocks enough for every compute unit
    assert kq.kvq_prompt_workspace_bytes(8, 2, [0, 4], [0, 100]) == 0               # too few keys to cut
    few = kq.kvq_prompt_workspace_bytes(8, 2, [0, 4], [0, 30000])                   # 16 rows over many
    assert few > 0 and few % 16 == 0
    assert kq.kvq_prompt_workspace_bytes(7, 2, [0, 4]) == 0 and kq.kvq_prompt_workspace_bytes(8, 2, [4, 0]) == 0
