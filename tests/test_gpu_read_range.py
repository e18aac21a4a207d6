"""kvq_cache_read at the end of the fp16 range: scales are rounded, so that code * S + Z may pass the largest value where no value did."""
import math

import pytest
import torch

import paper_2505_18610_amd as kq
from test_gpu_tree import D, cached, make

pytestmark = pytest.mark.gpu
MOST = 65504.0


def edges(g, n):
    x = (torch.randn(2, 2, n, D, generator=g, device="cuda") * 100).half()
    x[..., ::7], x[..., 1::7], x[..., 2::7] = MOST, -MOST, 0.0
    return x


@pytest.mark.parametrize("bits,int16", [(2, False), (4, False), (8, False), (16, False), (16, True), (4, True)])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("reparam", [False, True])
def test_the_largest_values(bits, int16, group, reparam):
    c, lam, g = make(2, 4, 2, [], int16=int16, group=group)
    if reparam:  # (of one and more: what is stored is the key divided by it)
        lam = 1 + 3 * torch.rand(2, D, generator=g, device="cuda")
        c.kvq_cache_set_reparam(0, lam)
    k, v = edges(g, 100), edges(g, 100)
    c.kvq_quantize_append(0, k, v, bits)
    want = list(cached(c))
    if bits < 16:  # (of 16 the scale is rounded down)
        assert float(want[1].abs().max()) >= 65520  # (what rounds to infinity)
    if lam is not None:
        want[0] = want[0] * lam.double()[:, None, :]
    for dtype in (torch.float16, torch.float32):
        outs = [torch.empty(2, 2, 100, D, dtype=dtype, device="cuda") for _ in range(2)]
        c.kvq_cache_read(0, 0, *outs)
        for x, y in zip(outs, want):
            if dtype == torch.float16:
                y = y.clamp(-MOST, MOST)
            assert torch.isfinite(x).all()
            step = 2.0 ** -11 if dtype == torch.float16 else 0.0
            # of 32 bits: code * S + Z, and the factor's product
            assert float(((x.double() - y).abs() - (step + 2 * 2.0 ** -24) * y.abs() - 2.0 ** -25).max()) <= 0


def test_infinities_stay():
    c, lam, g = make(1, 4, 2, [])
    k, v = (torch.randn(1, 2, 50, D, generator=g, device="cuda").half() for _ in range(2))
    v[0, 1, 20, 5], v[0, 0, 30, 6], v[0, 0, 31, 7] = math.inf, -math.inf, math.nan
    c.kvq_quantize_append(0, k, v, 16)
    for dtype in (torch.float16, torch.float32):
        outs = [torch.empty(1, 2, 50, D, dtype=dtype, device="cuda") for _ in range(2)]
        c.kvq_cache_read(0, 0, *outs)
        assert torch.equal(outs[0], k.to(dtype)) and torch.equal(torch.nan_to_num(outs[1], 7, 8, 9), torch.nan_to_num(v.to(dtype), 7, 8, 9))
        assert torch.equal(torch.isnan(outs[1]), torch.isnan(v))


def test_a_prefix_that_is_read_back_and_attended_to():
    """A second chunk over what a first one has left, whose values are at the end of the range."""
    c, lam, g = make(1, 4, 1, [])
    k = torch.randn(1, 1, 200, D, generator=g, device="cuda").half()
    v = edges(g, 200)[:1, :1].contiguous()
    c.kvq_quantize_append(0, k, v, 4)
    K, V = (torch.empty(1, 1, 200, D, dtype=torch.float16, device="cuda") for _ in range(2))
    c.kvq_cache_read(0, 0, K, V)
    q = torch.randn(10, 4, D, generator=g, device="cuda").half()
    out = torch.empty(10, 4, D, dtype=torch.float32, device="cuda")
    kq.kvq_prompt_attention(q, K[0].transpose(0, 1), V[0].transpose(0, 1), out, [0, 10], [0, 200])
    assert torch.isfinite(out).all()
