"""Infinite and NaN values among those that a query of kvq_prompt_attention sees: what they make of a row does not depend on the tile that they
lie in, on how little they weigh, or on the ranges that the keys are cut into."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_prompt import D, begins, check, inputs

pytestmark = pytest.mark.gpu


def lighter(gap, seed, heads, kv, nq, nk, at):
    """Inputs whose key `at` has a score about `gap` nats below the others'."""
    q, k, v = inputs(seed, heads, kv, nq, nk)
    q, k = q * 0.25, k * 0.25
    q[:, :, 0], k[:, :, 0] = 4, 0
    k[at, :, 0] = -gap * math.sqrt(D) / 4
    return q, k, v


def check_with(q, k, v, bad, qb, kb, out_dtype=torch.float16, workspace=True):
    """bad: [(key row, KV head, channels, value)].  With zeros in their place the outputs are those of the 64-bit formula; with the values a row
    that sees one has it added, to the last bit of everything else."""
    clean, dirty = v.clone(), v.clone()
    for row, head, channels, _ in bad:
        clean[row, head, channels] = 0
    for row, head, channels, x in bad:
        dirty[row, head, channels] = x
    want = check(q, k, clean, qb, kb, out_dtype, workspace=workspace)
    g = q.shape[1] // k.shape[1]
    for row, head, channels, x in bad:
        i = max(n for n in range(len(kb) - 1) if kb[n] <= row)
        first = qb[i + 1] - (kb[i + 1] - row)  # the first query row that sees it
        want[max(first, qb[i]):qb[i + 1], head * g:(head + 1) * g, channels] += x
    out = torch.empty_like(want)
    need = kq.kvq_prompt_workspace_bytes(q.shape[1], k.shape[1], qb, kb)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need and workspace else None
    kq.kvq_prompt_attention(q, k, dirty, out, qb, kb, workspace=ws)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.nan_to_num(out, 7.0, 8.0, 9.0), torch.nan_to_num(want, 7.0, 8.0, 9.0))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("gap", [0, 15, 25, 60, 100])
@pytest.mark.parametrize("nq,nk,at", [(200, 200, 10), (200, 200, 150), (300, 300, 299), (40, 700, 3), (1, 100, 99), (129, 1000, 870), (513, 513, 0)])
def test_light_keys_that_are_seen(bad, gap, nq, nk, at):
    q, k, v = lighter(gap, nk, 6, 2, nq, nk, at)
    for out in (torch.float16, torch.float32):
        check_with(q, k, v, [(at, h, slice(5, None, 16), bad) for h in range(2)], [0, nq], [0, nk], out)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("gap", [0, 30, 100, 200])
@pytest.mark.parametrize("nq,nk,at", [(4, 5000, 17), (4, 5000, 4990), (16, 9000, 4000), (33, 3000, 2999), (130, 4000, 1)])
def test_light_keys_in_ranges(bad, gap, nq, nk, at):
    assert kq.kvq_prompt_workspace_bytes(8, 1, [0, nq], [0, nk]) > 0
    q, k, v = lighter(gap, nk, 8, 1, nq, nk, at)
    x = [(at, 0, slice(3, None, 32), bad)]
    check_with(q, k, v, x, [0, nq], [0, nk])
    check_with(q, k, v, x, [0, nq], [0, nk], torch.float32, workspace=False)


def test_one_sequence_of_many():
    lengths = [100, 900, 33, 512, 1]
    b = begins(lengths)
    q, k, v = inputs(1, 4, 2, b[-1], b[-1])
    x = [(b[1] + 20, 0, 7, math.inf), (b[3] + 500, 1, 9, math.nan), (b[1] + 30, 0, 7, -math.inf), (b[1] + 600, 1, 100, -math.inf)]
    check_with(q, k, v, x, b, b)
    check_with(q, k, v, x, b, b, torch.float32)


def test_queries_and_keys_that_are_not_finite():
    """A NaN key makes every row NaN that sees it, a NaN query its own row, and values are looked at as ever."""
    q, k, v = inputs(2, 4, 2, 300, 300)
    q[100, 1] = math.nan
    v[200, :, 5] = math.inf
    out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
    kq.kvq_prompt_attention(q, k, v, out, [0, 300])
    assert torch.isnan(out[100, 1]).all() and torch.isfinite(out[:100]).all() and torch.isfinite(out[101:200]).all()
    assert (out[200:, :, 5] == math.inf).all() and torch.isfinite(out[200:, :, 6]).all()
    k[150] = math.nan
    kq.kvq_prompt_attention(q, k, v, out, [0, 300])
    assert torch.isnan(out[150:]).all() and torch.isfinite(out[:100]).all()
