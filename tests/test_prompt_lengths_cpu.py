"""kvq_prompt_attention and its workspace at the last row numbers of 32 bits; nothing is launched here."""
import os

import pytest

import paper_2505_18610_amd as kq
from test_prompt_cpu import call

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")
LAST = 2 ** 31 - 1


@pytest.mark.parametrize("rows", [(0, LAST), (0, LAST - 4095), (LAST - 10, LAST), (0, 5, LAST)])
def test_rows_that_pass_32_bits_when_they_are_rounded_up(rows):
    few = list(range(len(rows)))
    assert call(qb=rows) == kq.KVQ_E_INVALID and call(qb=few, kb=rows) == kq.KVQ_E_INVALID
    assert kq.kvq_prompt_workspace_bytes(8, 2, rows) == 0 and kq.kvq_prompt_workspace_bytes(8, 2, few, rows) == 0


def test_rows_just_below():
    top = LAST - 4096
    assert kq.kvq_prompt_workspace_bytes(8, 2, [0, 4], [0, top]) > 0
    assert kq.kvq_prompt_workspace_bytes(8, 2, [0, 4], [0, top]) == kq.kvq_prompt_workspace_bytes(8, 2, [top - 4, top], [0, top])


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="an accepted call would be launched")
def test_a_call_that_is_too_large_enqueues_nothing():
    """The first sequence has a launch of its own, in front of the second's, which has more row blocks than a launch takes."""
    qb, kb = (0, 1, LAST - 5000), (0, 200, 300)
    assert call(n_q=64, n_kv=64, qb=qb, kb=kb) == kq.KVQ_E_INVALID
    assert call(n_q=64, n_kv=64, qb=qb[:2], kb=kb[:2]) not in (kq.KVQ_OK, kq.KVQ_E_INVALID)  # (there is no device)
