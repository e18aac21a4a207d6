"""tests/tree_bounds.py holds for the roundings that it allows, and not for a tile that is lost, taken twice or rounded further."""
import math

import pytest
import torch

from tree_bounds import bounded, weights

T, ROWS = 36941, 16


@pytest.fixture(scope="module")
def case():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, 128, generator=g).half().double() for n in (ROWS, T, T))
    s = q @ k.t() / math.sqrt(128)
    reach = (q.abs() @ k.abs().t()).amax(1) / math.sqrt(128)
    want, tol = bounded(weights(s), v, reach, False)
    return q, k, v, s, want, tol


def taken(s, v):
    """Weights rounded to fp16 below 2^15, values as they are, sums of the rounded weights."""
    e = torch.exp2(((s - s.amax(1, keepdim=True)) * math.log2(math.e) + 7)).half().double()
    return (e @ v) / e.sum(1, keepdim=True)


def test_the_roundings_that_are_allowed(case):
    q, k, v, s, want, tol = case
    assert bool(((taken(s, v) - want).abs() <= tol).all())
    rounded = (v * (1 + (torch.rand(v.shape, generator=torch.Generator().manual_seed(2), dtype=torch.float64) * 2 - 1) * 2.0 ** -11))
    assert bool(((taken(s, rounded) - want).abs() <= tol).all())


@pytest.mark.parametrize("first", [0, 32 * 100, 32 * 1153])
def test_a_lost_tile_and_one_that_is_taken_twice(case, first):
    q, k, v, s, want, tol = case
    keep = torch.ones(T, dtype=torch.bool)
    keep[first:first + 32] = False
    for rows, values in ((s[:, keep], v[keep]), (torch.cat([s, s[:, ~keep]], 1), torch.cat([v, v[~keep]]))):
        assert int(((taken(rows, values) - want).abs() > tol).sum()) > 0.3 * want.numel()


def test_keys_rounded_to_fp16(case):
    """As a less exact kernel would have them: code * S + Z of four bits, rounded, where the product is taken with the codes."""
    q, k, v, s, want, tol = case
    wide = k.clone()
    wide[:, :4] *= 20  # (channels as calibration finds them)
    lo, hi = wide.view(T, 4, 32).amin(-1, keepdim=True).half().double(), wide.view(T, 4, 32).amax(-1, keepdim=True)
    S = ((hi - lo) / 15).half().double()
    exact = (((wide.view(T, 4, 32) - lo) / S).round().clamp(0, 15) * S + lo).view(T, 128)
    reach = (q.abs() @ exact.abs().t()).amax(1) / math.sqrt(128)
    want, tol = bounded(weights(q @ exact.t() / math.sqrt(128)), v, reach, False)
    ok, not_ok = (taken(q @ x.t() / math.sqrt(128), v) for x in (exact, exact.half().double()))
    assert bool(((ok - want).abs() <= tol).all())
    assert bool(((not_ok - want).abs() > tol).any())
