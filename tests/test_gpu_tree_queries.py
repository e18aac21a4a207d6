"""A query whose sums of 32 channels pass the fp16 range leaves the others of its call as exact as they are without it."""
import math

import pytest
import torch

from test_gpu_tree import D, cached, make, nodes, tree_mask
from test_gpu_tree_exact import check, run
from tree_bounds import tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,hq,hkv", [(2, 4, 1), (4, 8, 1), (9, 8, 2), (40, 8, 2), (20, 16, 1)])
@pytest.mark.parametrize("tiers,int16", [([(3000, 4)], False), ([(512, 2), (704, 8), (77, 16)], False), ([(1100, 16)], True)])
def test_a_large_query(n, hq, hkv, tiers, int16):
    """Keys of a thousand and queries of a thousandth, so that scores are ordinary, and one query of thousands."""
    c, lam, g = make(1, hq, hkv, tiers, int16=int16, wide=1000.0, seed=n)
    q, k, v = nodes(c, g, n)
    q, k = (q.float() * 1e-3).half(), (k.float() * 1000).half()
    sees = tree_mask(n, 1, n)
    big = q.clone()
    big[0, 1, n // 2] = 3000.0
    check(c, lam, big, k, v, sees)
    want, tol = tree(*cached(c), q, k, v, sees, lam, 1 / math.sqrt(D), False)
    big[0, 1, n // 2] = math.inf  # and one that is not finite
    bad = (run(c, big, k, v, sees).double() - want).abs() > tol
    bad[0, 1, n // 2] = False
    assert not bad.any(), int(bad.sum())
