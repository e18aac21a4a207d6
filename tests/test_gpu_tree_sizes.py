"""kvq_tree_attention at the sizes from which other kernels take it: blocks of rows that are cut into ranges of a long cache, full and not, in four
and in twelve wavefronts, with one, two and four groups of channels a token."""
import math

import pytest
import torch

from test_gpu_tree import check, make, nodes, tree_mask

pytestmark = pytest.mark.gpu

LONG = [(20480, 2), (12288, 4), (4096, 8), (77, 16)]
# batch, query heads, KV heads, nodes, tiers, page
CASES = {
    "four wavefronts, a last block of 4 rows": (2, 16, 4, 33, [(6144, 2), (2048, 8), (1000, 16)], 64),
    "four wavefronts, a last block of 72 rows": (2, 32, 4, 25, [(6144, 4), (2048, 8), (1000, 16)], 128),
    "four wavefronts, full blocks": (2, 32, 4, 32, [(8192, 2), (31, 16)], 256),
    "twelve, 320 rows": (2, 32, 2, 20, LONG, 64),
    "twelve, 273 rows": (2, 26, 2, 21, LONG, 32),
    "twelve, full": (2, 32, 2, 24, LONG, 256),
    "twelve, two blocks of 20 groups": (1, 32, 2, 40, [(36864, 4), (100, 16)], 128),
    "twelve, two blocks of which the last lacks a group": (1, 28, 2, 42, [(36864, 8), (33, 16)], 128),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_long_caches(name, group):
    batch, hq, hkv, n, tiers, page = CASES[name]
    c, lam, g = make(batch, hq, hkv, tiers, page=page, group=group, seed=n, reparam=group == 64)
    q, k, v = nodes(c, g, n)
    sees = tree_mask(n, batch, n)
    a = check(c, lam, q, k, v, sees)
    assert torch.equal(a, check(c, lam, q, k, v, sees)), "equal calls give equal bits"


@pytest.mark.parametrize("name", ["four wavefronts, a last block of 4 rows", "twelve, 273 rows"])
@pytest.mark.parametrize("workspace", [True, False])
def test_fp32_outputs_and_no_ranges(name, workspace):
    batch, hq, hkv, n, tiers, page = CASES[name]
    c, lam, g = make(batch, hq, hkv, tiers, page=page, seed=3)
    check(c, lam, *nodes(c, g, n), tree_mask(n, batch, 1), out_dtype=torch.float32, workspace=workspace)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("n", [33, 80])
def test_integer_16_bit_tier(n, group):
    c, lam, g = make(2, 16, 4, [(4096, 4), (5000, 16)], group=group, int16=True)
    check(c, lam, *nodes(c, g, n), tree_mask(n, 2, n))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("name", ["four wavefronts, a last block of 72 rows", "twelve, 320 rows", "twelve, two blocks of which the last lacks a group"])
def test_nodes_that_are_not_seen_do_not_reach(name, bad):
    batch, hq, hkv, n, tiers, page = CASES[name]
    c, lam, g = make(batch, hq, hkv, tiers, page=page)
    q, k, v = nodes(c, g, n)
    v[:, 1, n // 2, 3::16] = bad
    check(c, lam, q, k, v, tree_mask(n, batch, 2))
