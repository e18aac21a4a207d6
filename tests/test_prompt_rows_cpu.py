"""kvq_prompt_attention refuses outputs whose rows share memory; nothing is launched here (an accepted call finds no device)."""
import os

import pytest

import paper_2505_18610_amd as kq
from test_prompt_cpu import call

pytestmark = pytest.mark.skipif(not os.path.exists(kq.library_path()), reason="libkvq.so not built")


def overlap(token, head, n, heads):
    """By the definition: the rows sorted by where they begin lie 128 apart."""
    at = sorted(t * token + h * head for t in range(n) for h in range(heads))
    return any(b - a < 128 for a, b in zip(at, at[1:]))


def refused(token, head, n, heads):
    return call(n_q=heads, n_kv=heads, qb=(0, n), strides=dict(out_token=token, out_head=head)) == kq.KVQ_E_INVALID


@pytest.mark.parametrize("token,head,n,heads", [(128, 128, 2, 2), (128, 256, 3, 2), (192, 128, 10, 8), (1024, 1016, 10, 8), (384, 256, 10, 4), (1024, 1024, 2, 8)])
def test_rows_that_share_memory(token, head, n, heads):
    assert overlap(token, head, n, heads) and refused(token, head, n, heads)


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="accepted calls would be launched")
def test_every_layout_by_the_definition():
    for token in range(128, 900, 56):
        for head in range(128, 900, 56):
            for n in (1, 2, 3, 7):
                for heads in (1, 2, 5):
                    assert refused(token, head, n, heads) == overlap(token, head, n, heads), (token, head, n, heads)
