"""Rows in which one key leads all others by many nats: what the others weigh together is not lost, in prompt and in tree attention.

The leading key's score is `gap` above that of all others, which are equal, so every rounding goes the same way.  A weight is rounded to fp16
2^7 above the leading key's scale at the least: it loses 2^-11 of itself or 2^-32 of the leading weight.  The scale has 32 bits, three roundings, and is
multiplied into exponents of up to 36: 2^-17 of a weight.  Sums of n equal weights have n / 8 additions of 32 bits a lane, and the products with the
values n / 8 as well (a matrix instruction takes its 32 in four steps), n / 4 the log of the sum; the roundings of equal weights all go the
same way."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_prompt import D
from test_gpu_tree import make, words

pytestmark = pytest.mark.gpu
GAPS = [0.0, 5.0, 9.5, 12.0, 14.0, 16.0, 17.0, 17.5, 18.0, 19.0, 20.0]


def gap_of(gap):
    """The gap as fp16 queries and keys give it: q = 1 in channel 0, k = gap * sqrt(128)."""
    return float(torch.tensor(gap * math.sqrt(D)).half()) / math.sqrt(D)


def want_and_tol(gap, n, lead_value):
    """All other values are 1."""
    w = math.exp(-gap) * n
    want = (w + lead_value) / (w + 1)
    # of the others' sum; it is in the numerator and, of rows that add it to a leading weight, in the denominator
    lost = 2.0 ** -11 * w + n * 2.0 ** -32 + 2.0 ** -17 * w
    tol = 0.0 if lead_value == 1 else lost / (w + 1)
    return want, tol + (2.0 ** -20 + 2 * 2.0 ** -24 * n / 8) * want


@pytest.mark.parametrize("n", [200, 4096, 32768, 131072])
@pytest.mark.parametrize("nq,heads", [(1, 4), (5, 4), (9, 16), (70, 8)])
@pytest.mark.parametrize("workspace", [True, False])
def test_prompt(n, nq, heads, workspace):
    for at in (0, n // 2, n - nq):  # where the leading key is
        for lead in (0.0, 1.0):
            for gap in GAPS:
                q = torch.zeros(nq, heads, D, dtype=torch.float16, device="cuda")
                q[:, :, 0] = 1
                k = torch.zeros(n + 1, 1, D, dtype=torch.float16, device="cuda")
                v = torch.ones(n + 1, 1, D, dtype=torch.float16, device="cuda")
                k[at, 0, 0] = gap * math.sqrt(D)
                v[at] = lead
                out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
                lse = torch.empty(heads, nq, device="cuda")
                qb, kb = [0, nq], [0, n + 1]
                need = kq.kvq_prompt_workspace_bytes(heads, 1, qb, kb)
                ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and workspace else None
                kq.kvq_prompt_attention(q, k, v, out, qb, kb, lse=lse, workspace=ws)
                g = gap_of(gap)
                for i in (0, nq - 1):
                    others = n + 1 - nq + i  # keys that row i sees, less the leading one
                    want, tol = want_and_tol(g, others, lead)
                    got = out[i].double()
                    assert float((got - want).abs().max()) <= tol, (at, lead, gap, i, float(got[0, 0]), want, tol)
                    total = g + math.log1p(math.exp(-g) * others)
                    assert float((lse[:, i].double() - total).abs().max()) <= 2.0 ** -19 * (g + 1) + 2.0 ** -24 * n / 4, (at, gap, i)


@pytest.mark.parametrize("n", [200, 4096, 40000])
@pytest.mark.parametrize("nodes,heads", [(1, 4), (3, 8), (9, 8), (40, 8)])
@pytest.mark.parametrize("workspace", [True, False])
def test_tree(n, nodes, heads, workspace):
    """The leading key is a node that all nodes see, or a cached token; the other nodes see themselves."""
    c, lam, g = make(1, heads, 1, [(n, 16)], page=256)
    c.kvq_cache_truncate(0, 0)
    half = n // 2
    k = torch.zeros(1, 1, n, D, dtype=torch.float16, device="cuda")
    v = torch.ones_like(k)
    c.kvq_quantize_append(0, k, v, 16)
    need = c.kvq_tree_workspace_bytes(nodes)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and workspace else None
    for cached in (False, True):
        for gap in GAPS:
            q = torch.zeros(1, heads, nodes, D, dtype=torch.float16, device="cuda")
            q[..., 0] = 1
            kn, vn = torch.zeros(1, 1, nodes, D, dtype=torch.float16, device="cuda"), torch.zeros(1, 1, nodes, D, dtype=torch.float16, device="cuda")
            sees = torch.zeros(nodes, nodes, dtype=torch.bool)
            if cached:
                c.kvq_cache_truncate(0, half)
                k[0, 0, half, 0], v[0, 0, half] = gap * math.sqrt(D), 0
                c.kvq_quantize_append(0, k[:, :, half:].contiguous(), v[:, :, half:].contiguous(), 16)
            else:
                kn[0, 0, 0, 0] = gap * math.sqrt(D)
                sees[:, 0] = True
            out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
            c.kvq_tree_attention(0, q, kn, vn, words(sees), out, workspace=ws)
            want, tol = want_and_tol(gap_of(gap), n - cached, 0.0)
            got = out.double()
            assert float((got - want).abs().max()) <= tol, (cached, gap, float(got[0, 0, 0, 0]), want, tol)
