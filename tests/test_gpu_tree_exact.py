"""kvq_tree_attention within what its roundings allow (tests/tree_bounds.py), over caches so long that a lost tile is little, with many nodes, and
with a mark in every tile."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_tree import D, MIXED, cached, make, nodes, tree_mask, words
from test_gpu_tree_sizes import CASES
from tree_bounds import tree

pytestmark = pytest.mark.gpu


def run(c, q, k, v, sees, dtype=torch.float32, workspace=True):
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    need = c.kvq_tree_workspace_bytes(q.shape[2])
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and workspace else None
    c.kvq_tree_attention(0, q, k, v, words(sees), out, workspace=ws)
    return out


def check(c, lam, q, k, v, sees, dtype=torch.float32, workspace=True):
    out = run(c, q, k, v, sees, dtype, workspace)
    want, tol = tree(*cached(c), q, k, v, sees, lam, 1 / math.sqrt(D), dtype == torch.float16)
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((out.double() - want).abs() / tol).max()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("group", [32, 128])
def test_long_caches(name, group):
    batch, hq, hkv, n, tiers, page = CASES[name]
    c, lam, g = make(batch, hq, hkv, tiers, page=page, group=group, seed=n, reparam=group == 128)
    check(c, lam, *nodes(c, g, n), tree_mask(n, batch, n))


@pytest.mark.parametrize("n,hq,hkv", [(1, 8, 2), (4, 8, 2), (8, 8, 2), (12, 8, 1), (16, 28, 4)])
@pytest.mark.parametrize("tiers", [MIXED, [(8448, 4), (553, 16)], [(20000, 2)]])
@pytest.mark.parametrize("int16", [False, True])
def test_few_rows(n, hq, hkv, tiers, int16):
    c, lam, g = make(1, hq, hkv, tiers, int16=int16, seed=n, wide=3.0)
    q, k, v = nodes(c, g, n)
    check(c, lam, q, k, v, tree_mask(n, 1, n))
    check(c, lam, q, k, v, tree_mask(n, 1, n), torch.float16, workspace=False)


@pytest.mark.parametrize("n", [131, 256, 500, 777, 1023, 1024])
@pytest.mark.parametrize("tiers", [[], [(40, 16)], [(2048, 2), (700, 8)], [(9000, 4)]])
@pytest.mark.parametrize("hq,hkv,int16", [(8, 1, False), (2, 2, True)])
def test_many_nodes(n, tiers, hq, hkv, int16):
    c, lam, g = make(1, hq, hkv, tiers, int16=int16, seed=n)
    check(c, lam, *nodes(c, g, n), tree_mask(n, 1, n))


@pytest.mark.parametrize("n", [33, 200])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_integer_16_bit_tier(n, group):
    c, lam, g = make(2, 16, 2, [(2048, 2), (4096, 4), (2048, 8), (5000, 16)], group=group, int16=True)
    check(c, lam, *nodes(c, g, n), tree_mask(n, 2, n))


MARKED = {**{k: v for k, v in CASES.items()},
          "one node": (1, 4, 1, 1, [(4096, 4), (9000, 16)], 64), "four nodes": (2, 8, 2, 4, [(4096, 2), (4096, 8), (70, 16)], 256),
          "32 rows": (1, 8, 1, 4, [(30016, 2), (31, 16)], 32), "pairs": (1, 28, 4, 16, [(8448, 4), (553, 16)], 128), "short": (3, 8, 2, 20, [(40, 8)], 32)}


@pytest.mark.parametrize("name", MARKED)
@pytest.mark.parametrize("workspace", [True, False])
def test_every_tile_counts_once(name, workspace):
    """Queries of zeros weigh every key alike.  Values are zero but for a one in channel t % 128 of the tokens of tile t, so that a lost tile, or one
    that is taken twice, is a tenth of a channel's sum or more; all that is rounded is code * S + Z."""
    batch, hq, hkv, n, tiers, page = MARKED[name]
    c, lam, g = make(batch, hq, hkv, tiers, page=page)
    T = sum(t for t, _ in tiers)
    c.kvq_cache_truncate(0, 0)
    t = torch.arange(T, device="cuda")
    V = ((t // 32 % 128)[:, None] == torch.arange(D, device="cuda")).half().expand(batch, hkv, T, D)
    K = torch.randn(batch, hkv, T, D, generator=g, device="cuda").half()
    at = 0
    for m, bits in tiers:
        c.kvq_quantize_append(0, K[:, :, at:at + m].contiguous(), V[:, :, at:at + m].contiguous(), bits)
        at += m
    q = torch.zeros(batch, hq, n, D, dtype=torch.float16, device="cuda")
    k = torch.randn(batch, hkv, n, D, generator=g, device="cuda").half()
    v = torch.zeros_like(k)
    sees = torch.eye(n, dtype=torch.bool)
    out = run(c, q, k, v, sees, workspace=workspace).double()
    want = cached(c)[1].sum(2) / (T + 1)  # [batch, hkv, D]
    want = want.repeat_interleave(hq // hkv, 1)[:, :, None].expand_as(out)
    assert float(((out - want).abs() - (2.0 ** -11 + 2.0 ** -20) * want).max()) <= 0
